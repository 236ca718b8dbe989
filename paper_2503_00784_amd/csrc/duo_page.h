// Many requests on a paged cache: the plan of a step, the append of its keys and values, the commit of accepted branches.
#pragma once
#include "../../include/duo_verify.h"
#include "duo_common.h"
#include "duo_page_rules.h"

// ---- what a plan leaves in the workspace (page_layout gives the places)
struct PageHeader {  // one, PAGE_HEADER_INTS
    int32_t magic, ok;
    int32_t requests, hq, hkv, head_dim, page_slots, max_pages, max_rows, max_new;  // what the plan was made for
    int32_t stream_items, tile_items, merges;
    int32_t rows, free_in, free_out, released;
};
constexpr int32_t PAGE_MAGIC = 0x70616765;
static_assert(sizeof(PageHeader) <= PAGE_HEADER_INTS * 4, "the header has its place");

struct __align__(16) PageInfo {  // one per request
    int32_t cached, trunk, n, k;
    int32_t row0, rows, held, need;
    int32_t take0, rel0;         // pages taken and released by the requests before it
    int32_t item0, chunks;       // its first item (of its kind) and the key ranges per tile
    int32_t part0, merge0;       // first partial result and first merge, if its tiles are cut
    int32_t tiles, streamed;
};
static_assert(sizeof(PageInfo) == PAGE_INFO_INTS * 4, "the place of a request");

struct __align__(16) PageItem {  // one workgroup per item and kv head
    int32_t request, cached, trunk, k;
    int32_t row0;                // the request's first row in the step's matrices
    int32_t first, count;        // the tile's rows: pairs (token, query head of the group), first of them and how many
    int32_t block0, blocks;      // key range
    int32_t slots;               // cached + new rows
    int32_t part;                // partial result, or -1: the item is its tile's only one and writes the output
    int32_t last_block;          // of the request
    int32_t pad[4];
};
static_assert(sizeof(PageItem) == PAGE_ITEM_INTS * 4, "the place of an item");

struct __align__(16) PageMerge {  // some rows of a tile whose keys were cut
    int32_t row0, first, count;  // the request's first row; pairs first .. first + count - 1
    int32_t part0, parts;        // its tile's partial results
    int32_t in_tile, streamed, pad;
};
static_assert(sizeof(PageMerge) == PAGE_MERGE_INTS * 4, "the place of a merge");

struct PagePlanArgs {
    const int32_t *cached, *trunk, *n, *k;
    const int32_t *table_in, *held_in, *free_in, *count_in;
    int32_t *table_out, *held_out, *free_out, *count_out;
    int32_t *row_start, *position, *slot, *status;
    int32_t requests, max_rows, max_new, n_pages, page_shift, max_pages;
    int32_t hq, hkv, head_dim;
    char* ws;
    PageLayout lay;
};

// Exclusive sums of N quantities over the threads of a workgroup of up to 1024, and their totals: within the waves, then over the waves' totals, which
// the first lanes of the workgroup sum up, sixteen to a quantity.
template <int N>
struct PageScan {
    int wave[16][N], total[N];
};
template <int N>
__device__ __forceinline__ void block_scan(int (&v)[N], int (&total)[N], PageScan<N>& lds) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = (blockDim.x + 63) >> 6;
    int own[N];
#pragma unroll
    for (int i = 0; i < N; ++i) own[i] = v[i];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        int up[N];
#pragma unroll
        for (int i = 0; i < N; ++i) up[i] = __shfl_up(v[i], o, 64);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += lane >= o ? up[i] : 0;
    }
    if (lane == 63) {
#pragma unroll
        for (int i = 0; i < N; ++i) lds.wave[wave][i] = v[i];
    }
    __syncthreads();
    if (wave == 0) {
        for (int j = lane; j < 16 * N; j += 64) {  // 16 lanes a quantity: no quantity is divided between two turns
            const int w = j & 15, i = j >> 4;
            int x = w < waves ? lds.wave[w][i] : 0;
            const int mine = x;
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) {
                const int up = __shfl_up(x, o, 16);
                x += w >= o ? up : 0;
            }
            if (w == 15) lds.total[i] = x;
            lds.wave[w][i] = x - mine;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] += lds.wave[wave][i] - own[i];
        total[i] = lds.total[i];
    }
}

// Part one of a plan, one workgroup: checks, sums over the requests, how the attention is cut.  A thread takes PER consecutive requests.
// What bounds it is the latency of a chain of a dozen dependent steps (loads, two scans, stores).
constexpr int PAGE_PLAN_THREADS = 1024;
struct PageSumLds {
    PageScan<6> sums;
    PageScan<5> cuts;
    int bad;
};

// What part two asks of part one: info, header and, in a row of their own, the rel0 of all requests.
struct PagePlanned {
    PageHeader* hdr;
    PageInfo* info;
    int* released;
};
__device__ __forceinline__ PagePlanned page_planned(const PagePlanArgs& a) {
    return {reinterpret_cast<PageHeader*>(a.ws), reinterpret_cast<PageInfo*>(a.ws + a.lay.info), reinterpret_cast<int*>(a.ws + a.lay.released)};
}

template <int PER>
__device__ __forceinline__ void page_sum(const PagePlanArgs& a, PageSumLds& lds) {
    const PagePlanned out = page_planned(a);
    const int group = a.hq / a.hkv, page = 1 << a.page_shift, max_slots = a.max_pages << a.page_shift;
    const int per = (a.requests + (int)blockDim.x - 1) / (int)blockDim.x;
    const int F = *a.count_in;
    if (threadIdx.x == 0) lds.bad = 0;
    __syncthreads();

    PageInfo p[PER];
    int wrong = 0;
    // the attention's work (tiles * blocks) in two halves, whose sums stay inside 32 bits
    enum { ROWS, REL, TAKE, WORK_S, WORK_T, WORK_T_HIGH, SUMS };
    int sum[SUMS] = {};
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int r = threadIdx.x * per + i;
        p[i] = PageInfo{};
        if (i >= per || r >= a.requests) continue;
        PageInfo& q = p[i];
        q.cached = a.cached[r], q.trunk = a.trunk[r], q.n = a.n[r], q.k = a.k[r], q.held = a.held_in[r];
        const long long rows = (long long)q.trunk + (long long)q.n * q.k;
        const bool fits = q.cached >= 0 && q.trunk >= 0 && q.n >= 0 && q.k >= 0 && rows <= a.max_new && q.cached + rows <= max_slots &&
                          q.held >= 0 && q.held <= a.max_pages;
        wrong |= !fits;
        if (!fits) q.cached = q.trunk = q.n = q.k = 0, q.held = q.held < 0 ? 0 : q.held > a.max_pages ? a.max_pages : q.held;
        q.rows = fits ? (int)rows : 0;
        q.need = (q.cached + q.rows + page - 1) >> a.page_shift;
        const PageWork w = page_work(q.cached, q.rows, group);
        q.tiles = w.tiles, q.streamed = w.streamed;
        const long long work = (long long)w.tiles * w.blocks;
        sum[ROWS] += q.rows;
        sum[REL] += q.held > q.need ? q.held - q.need : 0;
        sum[TAKE] += q.need > q.held ? q.need - q.held : 0;
        sum[WORK_S] += w.streamed ? (int)work : 0;
        sum[WORK_T] += w.streamed ? 0 : (int)(work & 0xffff);
        sum[WORK_T_HIGH] += w.streamed ? 0 : (int)(work >> 16);
    }
    if (wrong) lds.bad = 1;
    int total[SUMS];
    block_scan(sum, total, lds.sums);  // its barriers stand between the flag's writes and its read
    int status = lds.bad ? DUO_PAGE_BAD_REQUEST : 0;
    if (F < 0 || F > a.n_pages || total[ROWS] > a.max_rows || total[REL] > a.n_pages - F) status |= DUO_PAGE_BAD_REQUEST;
    else if (total[TAKE] > F + total[REL]) status |= DUO_PAGE_NO_PAGES;
    const bool ok = status == 0;

    // the cuts
    const int range_s = page_stream_range(total[WORK_S], a.hkv, page_stream_cut(a.max_new, group), max_slots >> 5);
    const int range_t = page_range(((long long)total[WORK_T_HIGH] << 16) + total[WORK_T], a.hkv, PAGE_TILE_TARGET, PAGE_TILE_MIN_BLOCKS);
    enum { ITEM_S, ITEM_T, PART_S, PART_T, MERGE, CUTS };
    int cut[CUTS] = {};
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        PageInfo& q = p[i];
        if (q.tiles == 0 || !ok) continue;
        const int blocks = (q.cached + q.rows + 31) / 32;
        q.chunks = page_chunks(blocks, q.streamed ? range_s : range_t);
        const int items = q.tiles * q.chunks;
        cut[ITEM_S] += q.streamed ? items : 0;
        cut[ITEM_T] += q.streamed ? 0 : items;
        if (q.chunks == 1) continue;
        cut[PART_S] += q.streamed ? items : 0;
        cut[PART_T] += q.streamed ? 0 : items;
        cut[MERGE] += page_merge_entries(q.rows * group, q.chunks);
    }
    int cuts[CUTS];
    block_scan(cut, cuts, lds.cuts);

    if (threadIdx.x == 0) {
        *out.hdr = PageHeader{PAGE_MAGIC, ok, a.requests, a.hq, a.hkv, a.head_dim, page, a.max_pages, a.max_rows, a.max_new,
                              cuts[ITEM_S], cuts[ITEM_T], cuts[MERGE], ok ? total[ROWS] : 0, ok ? F : 0, ok ? F + total[REL] - total[TAKE] : 0,
                              ok ? total[REL] : 0};
        *a.status = status;
        if (ok) *a.count_out = F + total[REL] - total[TAKE];
        else if (a.count_out != a.count_in) *a.count_out = F;
        a.row_start[a.requests] = ok ? total[ROWS] : 0;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int r = threadIdx.x * per + i;
        if (i >= per || r >= a.requests) continue;
        PageInfo& q = p[i];
        if (!ok) {  // nothing changes: no rows, the pages of before (a copy of the tables where `to` is not `from`)
            if (a.held_out != a.held_in) a.held_out[r] = a.held_in[r];
            a.row_start[r] = 0;
            q = PageInfo{};
            out.info[r] = q, out.released[r] = 0;
            continue;
        }
        q.row0 = sum[ROWS], q.rel0 = sum[REL], q.take0 = sum[TAKE];
        sum[ROWS] += q.rows;
        sum[REL] += q.held > q.need ? q.held - q.need : 0;
        sum[TAKE] += q.need > q.held ? q.need - q.held : 0;
        const int items = q.tiles * q.chunks;
        q.item0 = q.streamed ? cut[ITEM_S] : cut[ITEM_T];
        cut[ITEM_S] += q.streamed ? items : 0;
        cut[ITEM_T] += q.streamed ? 0 : items;
        q.part0 = -1;
        if (q.chunks > 1) {
            q.part0 = q.streamed ? cut[PART_S] : cut[PART_T], q.merge0 = cut[MERGE];
            cut[PART_S] += q.streamed ? items : 0;
            cut[PART_T] += q.streamed ? 0 : items;
            cut[MERGE] += page_merge_entries(q.rows * group, q.chunks);
        }
        out.info[r] = q, out.released[r] = q.rel0;
        a.held_out[r] = q.need;
        a.row_start[r] = q.row0;
    }
}

// Part two: everything that is as long as rows, pages or items.
// In place this is safe: columns that are written ([held, need) of requests that grow) are read by nobody, columns that are read ([need, held)
// of requests that shrink) are written by nobody, and the stack is read below its old count only and written from there on only.
template <class Released>
__device__ __forceinline__ int released_page(const PagePlanArgs& a, const PageInfo* info, const Released& released, int rank) {
    int lo = 0, hi = a.requests - 1;  // the last request whose released pages start at or before rank and that has any there
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (released(mid) <= rank) lo = mid;
        else hi = mid - 1;
    }
    return a.table_in[(size_t)lo * a.max_pages + info[lo].need + (rank - released(lo))];
}

// The rows behind the last, and the free stack where the tables are not planned in place.
__device__ __forceinline__ void page_fill_rest(const PagePlanArgs& a, const PageHeader& hdr, int t0, int step) {
    for (int i = hdr.rows + t0; i < a.max_rows; i += step) a.position[i] = a.slot[i] = -1;
    if (a.table_out != a.table_in) {
        const int kept = hdr.ok ? min(hdr.free_in, hdr.free_out) : min(max(*a.count_in, 0), a.n_pages);
        for (int i = t0; i < kept; i += step) a.free_out[i] = a.free_in[i];
    }
}

// One request: its pages, its rows, its part of the attention's schedule.  released(i): rel0 of request i.
template <class Released>
__device__ __forceinline__ void page_fill_request(const PagePlanArgs& a, const PageHeader& hdr, const PageInfo* info, const Released& released, int r, int t0,
                                                  int step) {
    const int group = a.hq / a.hkv;
    const bool copies = a.table_out != a.table_in;
    const int32_t* const line_in = a.table_in + (size_t)r * a.max_pages;
    int32_t* const line = a.table_out + (size_t)r * a.max_pages;
    if (!hdr.ok) {
        if (copies) {
            const int held = min(max(a.held_in[r], 0), a.max_pages);
            for (int c = t0; c < held; c += step) line[c] = line_in[c];
        }
        return;
    }
    const PageInfo p = info[r];
    const int top = hdr.free_in + hdr.released;
    // the page of column c: kept, or popped from the free pages with the released ones behind them
    auto page_of = [&](int c) {
        if (c < p.held) return line_in[c];
        const int x = top - 1 - (p.take0 + c - p.held);
        return x < hdr.free_in ? a.free_in[x] : released_page(a, info, released, x - hdr.free_in);
    };
    for (int c = (copies ? 0 : p.held) + t0; c < p.need; c += step) line[c] = page_of(c);
    for (int c = p.need + t0; c < p.held; c += step) {
        const int x = hdr.free_in + p.rel0 + c - p.need;
        if (x < hdr.free_out) a.free_out[x] = line_in[c];
    }
    for (int t = t0; t < p.rows; t += step) {
        const int logical = p.cached + t;
        a.position[p.row0 + t] = t < p.trunk ? logical : p.cached + p.trunk + (t - p.trunk) % p.k;
        const int page = page_of(logical >> a.page_shift);
        const bool known = (unsigned)page < (unsigned)a.n_pages;
        a.slot[p.row0 + t] = known ? (page << a.page_shift) + (logical & ((1 << a.page_shift) - 1)) : -1;
        if (!known) atomicOr(a.status, DUO_PAGE_BAD_PAGE);
    }
    // the items of the attention; late tiles see the most keys and go first
    const int items = p.tiles * p.chunks;
    PageItem* const out = reinterpret_cast<PageItem*>(a.ws + (p.streamed ? a.lay.stream : a.lay.tile)) + p.item0;
    const int pairs = p.rows * group;
    for (int i = t0; i < items; i += step) {
        const int tile = p.tiles - 1 - i / p.chunks, chunk = i % p.chunks;
        const int first = tile * PAGE_TILE_ROWS, count = p.streamed ? pairs : min(PAGE_TILE_ROWS, pairs - first);
        const int blocks = page_tile_blocks(p.cached, first, count, group), length = page_chunk_blocks(blocks, p.chunks);
        PageItem it;
        it.request = r, it.cached = p.cached, it.trunk = p.trunk, it.k = p.k, it.row0 = p.row0, it.first = first, it.count = count;
        it.block0 = chunk * length;
        it.blocks = max(0, min(length, blocks - it.block0));
        it.slots = p.cached + p.rows;
        it.part = p.chunks > 1 ? p.part0 + tile * p.chunks + chunk : -1;
        it.last_block = (it.slots - 1) >> 5;
        it.pad[0] = it.pad[1] = it.pad[2] = it.pad[3] = 0;
        out[i] = it;
    }
    if (p.chunks > 1) {
        const int rows = page_merge_rows(p.chunks), entries = page_merge_entries(pairs, p.chunks);
        PageMerge* const merge = reinterpret_cast<PageMerge*>(a.ws + a.lay.merge) + p.merge0;
        for (int i = t0; i < entries; i += step) {
            const int first = i * rows, tile = p.streamed ? 0 : first / PAGE_TILE_ROWS, tile_first = tile * PAGE_TILE_ROWS;
            const int count = p.streamed ? pairs : min(PAGE_TILE_ROWS, pairs - tile_first);
            const int blocks = page_tile_blocks(p.cached, tile_first, count, group), length = page_chunk_blocks(blocks, p.chunks);
            PageMerge m;
            m.row0 = p.row0, m.first = first, m.count = min(rows, pairs - first);
            m.part0 = p.part0 + tile * p.chunks, m.parts = (blocks + length - 1) / length;
            m.in_tile = first - tile_first, m.streamed = p.streamed, m.pad = 0;
            merge[i] = m;
        }
    }
}

template <int PER>
__global__ __launch_bounds__(PAGE_PLAN_THREADS) void page_sum_kernel(PagePlanArgs a) {
    __shared__ PageSumLds lds;
    page_sum<PER>(a, lds);
}

// blockIdx.x < requests: request blockIdx.x, its threads spread over gridDim.y workgroups; the workgroups beyond see to the rest.  Where a request takes
// pages that others release, the search for whose they are goes through LDS (414
// requests: 13.0 us for both launches, 12.0 so).
__global__ __launch_bounds__(256) void page_fill_kernel(PagePlanArgs a) {
    __shared__ int released[PAGE_MAX_REQUESTS];
    const PagePlanned in = page_planned(a);
    const PageHeader hdr = *in.hdr;
    const int t0 = blockIdx.y * blockDim.x + threadIdx.x, step = gridDim.y * blockDim.x;
    if ((int)blockIdx.x >= a.requests) {
        page_fill_rest(a, hdr, ((int)blockIdx.x - a.requests) * step + t0, ((int)gridDim.x - a.requests) * step);
        return;
    }
    const PageInfo p = in.info[blockIdx.x];
    if (p.need > p.held && hdr.released > 0) {
        for (int i = threadIdx.x; i < a.requests; i += blockDim.x) released[i] = in.released[i];
        __syncthreads();
    }
    page_fill_request(a, hdr, in.info, [&](int i) { return released[i]; }, blockIdx.x, t0, step);
}

// Both parts in one workgroup, a wave per request: for steps of up to PAGE_SMALL_REQUESTS requests, PAGE_SMALL_ROWS rows and PAGE_SMALL_PAGES pages,
// where a second launch is what a plan costs (4 requests: 7.2 us in two launches, 6.1 so; 16 requests:
// 7.4 in two, 9.0).
constexpr int PAGE_SMALL_REQUESTS = 8, PAGE_SMALL_ROWS = 4096, PAGE_SMALL_PAGES = 16384;
__global__ __launch_bounds__(PAGE_PLAN_THREADS) void page_plan_kernel(PagePlanArgs a) {
    __shared__ PageSumLds lds;
    page_sum<1>(a, lds);
    __syncthreads();  // what the workgroup has written to memory is there for all of it
    const PagePlanned in = page_planned(a);
    const PageHeader hdr = *in.hdr;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (wave < a.requests) page_fill_request(a, hdr, in.info, [&](int i) { return in.info[i].rel0; }, wave, lane, 64);
    page_fill_rest(a, hdr, threadIdx.x, blockDim.x);
}

// ---- append
struct PageAppendArgs {
    const u16 *q, *k, *v;
    u16* q_out;
    size_t q_stride, k_stride, v_stride, q_out_stride;
    u16 *kc, *vc;  // this layer's pages
    const int32_t *position, *slot;
    int32_t* status;
    int32_t rows, hq, hkv, page_shift, n_pages;
    int32_t heads_each, rope_groups;
    double turns[64];  // theta^(-2d/D) / 2 pi: turns per position
};

// A workgroup takes 32 rows: blockIdx.y < rope_groups: `heads_each` query and key heads, otherwise one head's values.  What bounds it at many rows is
// the bytes.
//
// Rotation: a thread takes eight channels and their eight partners of a row, forms their angles once and goes through the heads: two 16-byte
// loads and stores each; K's eight channels of a slot are one 16-byte piece of a tile.  The angle is reduced in double precision (position
// times turns is within 2^-29 turns at 2^23 positions), sine and cosine of the remainder are fp32.
//
// Values: a tile holds eight consecutive slots of a channel together.  Eight rows in a row that fill such a piece (all but the ends of a
// request's rows) are turned around through LDS and written 16 bytes a channel; other rows two bytes a channel.  A workgroup sees to the pieces
// that start in its rows, so it reads up to seven rows more.
//
// 8410 rows of 32 query and 8 key heads of 128: 50 us from cold caches (4.1 TB/s of what is read and written once; a copy of 2 GiB reaches 4.9), 35
// where the last-level cache still holds the rows, as behind the projection that wrote them; 80 there with a sine and cosine for every head and two
// bytes a channel throughout.
constexpr int PAGE_APPEND_ROWS = 32;

template <int D>
__device__ __forceinline__ void page_rope(const PageAppendArgs& a) {
    constexpr int TPH = D / 16, HPP = 256 / (PAGE_APPEND_ROWS * TPH);  // threads per row and head, heads at a time
    const int part = threadIdx.x % TPH, row = blockIdx.x * PAGE_APPEND_ROWS + threadIdx.x / TPH % PAGE_APPEND_ROWS;
    if (row >= a.rows) return;
    const int slot = a.slot[row];
    if (slot < 0) return;
    const int page = slot >> a.page_shift, in_page = slot & ((1 << a.page_shift) - 1);
    const bool known = page < a.n_pages;
    const double pos = (double)a.position[row];
    float sn[8], cs[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double t = pos * a.turns[part * 8 + e];
        sincospif(2.0f * (float)(t - floor(t)), &sn[e], &cs[e]);
    }
    const int last = min((int)(blockIdx.y + 1) * a.heads_each, a.hq + a.hkv);
    for (int head = blockIdx.y * a.heads_each + threadIdx.x / (TPH * PAGE_APPEND_ROWS); head < last; head += HPP) {
        const u16* src = head < a.hq ? a.q + (size_t)row * a.q_stride + head * D : a.k + (size_t)row * a.k_stride + (head - a.hq) * D;
        src += part * 8;
        Frag8 x, y, xo, yo;
        x.q = *reinterpret_cast<const u32x4*>(src);
        y.q = *reinterpret_cast<const u32x4*>(src + D / 2);
        float xf[8], yf[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float u = elem_to_f32(x.h[e]), v = elem_to_f32(y.h[e]);
            xf[e] = u * cs[e] - v * sn[e];
            yf[e] = v * cs[e] + u * sn[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) xo.q[e] = pack_elem2(xf[2 * e], xf[2 * e + 1]), yo.q[e] = pack_elem2(yf[2 * e], yf[2 * e + 1]);
        if (head < a.hq) {
            u16* dst = a.q_out + (size_t)row * a.q_out_stride + head * D + part * 8;
            *reinterpret_cast<u32x4*>(dst) = xo.q;
            *reinterpret_cast<u32x4*>(dst + D / 2) = yo.q;
        } else if (known) {
            u16* plane = a.kc + (((size_t)page * a.hkv + (head - a.hq)) << a.page_shift) * D;
            *reinterpret_cast<u32x4*>(plane + k_cache_offset(D, in_page, part * 8)) = xo.q;
            *reinterpret_cast<u32x4*>(plane + k_cache_offset(D, in_page, part * 8 + D / 2)) = yo.q;
        } else if (part == 0) {
            atomicOr(a.status, DUO_PAGE_BAD_PAGE);
        }
    }
}

template <int D>
__device__ __forceinline__ void page_values(const PageAppendArgs& a) {
    constexpr int R = PAGE_APPEND_ROWS, SEEN = R + 7, CHUNKS = D / 8, PAD = D + 2;
    __shared__ u16 v[SEEN * PAD];
    __shared__ int slots[7 + SEEN], pieces[R], singles[R], counts[2];
    const int head = blockIdx.y - a.rope_groups, row0 = blockIdx.x * R;
    if (threadIdx.x < 2) counts[threadIdx.x] = 0;
    for (int i = threadIdx.x; i < 7 + SEEN; i += blockDim.x) {  // rows row0 - 7 .. row0 + R + 6
        const int row = row0 - 7 + i;
        int s = row >= 0 && row < a.rows ? a.slot[row] : -1;
        slots[i] = s >= 0 && s >> a.page_shift < a.n_pages ? s : -1;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < SEEN * CHUNKS; i += blockDim.x) {
        const int r = i / CHUNKS, d = i % CHUNKS * 8;
        if (slots[7 + r] < 0) continue;
        const u32x4 x = *reinterpret_cast<const u32x4*>(a.v + (size_t)(row0 + r) * a.v_stride + head * D + d);
#pragma unroll
        for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t*>(&v[r * PAD + d + 2 * e]) = x[e];
    }
    if (threadIdx.x < R && slots[7 + threadIdx.x] >= 0) {
        const int s = slots[7 + threadIdx.x], first = 7 + threadIdx.x - (s & 7);  // where the row's piece would start
        bool whole = true;
#pragma unroll
        for (int e = 0; e < 8; ++e) whole &= slots[first + e] == (s & ~7) + e;
        if (!whole) singles[atomicAdd(&counts[1], 1)] = threadIdx.x;  // the order of the lists does not matter
        else if ((s & 7) == 0) pieces[atomicAdd(&counts[0], 1)] = threadIdx.x;
    }
    __syncthreads();
    auto plane = [&](int s) { return a.vc + (((size_t)(s >> a.page_shift) * a.hkv + head) << a.page_shift) * D; };
    const int mask = (1 << a.page_shift) - 1;
    for (int i = threadIdx.x; i < counts[0] * D; i += blockDim.x) {
        const int r = pieces[i / D], d = i % D, s = slots[7 + r];
        Frag8 f;
#pragma unroll
        for (int e = 0; e < 8; ++e) f.h[e] = v[(r + e) * PAD + d];
        *reinterpret_cast<u32x4*>(plane(s) + v_cache_offset(D, s & mask, d)) = f.q;
    }
    for (int i = threadIdx.x; i < counts[1] * D; i += blockDim.x) {
        const int r = singles[i / D], d = i % D, s = slots[7 + r];
        plane(s)[v_cache_offset(D, s & mask, d)] = v[r * PAD + d];
    }
}

template <int D>
__global__ __launch_bounds__(256) void page_append_kernel(PageAppendArgs a) {
    if ((int)blockIdx.y < a.rope_groups) page_rope<D>(a);
    else page_values<D>(a);
}

// ---- commit
struct PageCommitArgs {
    u16 *kc, *vc;
    const int32_t *cached, *table, *records;
    int32_t *cached_out, *status;
    int32_t requests, layers, hkv, page_shift, n_pages, max_pages, max_new, hq, head_dim, max_rows;
    const char* ws;
    size_t info;
};

__device__ __forceinline__ bool page_plan_is(const PageHeader& h, int requests, int hq, int hkv, int D, int page_shift, int max_pages, int max_rows, int max_new) {
    return h.magic == PAGE_MAGIC && h.requests == requests && h.hq == hq && h.hkv == hkv && h.head_dim == D && h.page_slots == 1 << page_shift &&
           h.max_pages == max_pages && h.max_rows == max_rows && h.max_new == max_new;
}

// One workgroup per (request, layer, kv head).  K: a slot's eight channels are a 16-byte piece; V: eight slots of a channel are, read as such and
// written two bytes each, since source and target lie differently in theirs.  Source and target share no slot (branch 0 lies where it belongs,
// branch i >= 1 starts i * k >= a slots further on).  What bounds it is three dependent round trips: plan and record, page ids, data.
// 48 requests, 16 layers of 8 heads: 18 us with a load and two page lookups for every value, 15 so.
template <int D>
__global__ __launch_bounds__(128) void page_commit_kernel(PageCommitArgs a) {
    const int r = blockIdx.x, layer = blockIdx.y, head = blockIdx.z;
    const PageHeader hdr = *reinterpret_cast<const PageHeader*>(a.ws);
    const PageInfo p = reinterpret_cast<const PageInfo*>(a.ws + a.info)[r];  // of no meaning without a plan
    const int branch = a.records[4 * r], accepted = a.records[4 * r + 1], token = a.records[4 * r + 2];
    const bool first = layer == 0 && head == 0 && threadIdx.x == 0;
    const bool known = page_plan_is(hdr, a.requests, a.hq, a.hkv, D, a.page_shift, a.max_pages, a.max_rows, a.max_new);
    if (!known || !hdr.ok) {
        if (first) {
            if (!known) atomicOr(a.status, DUO_PAGE_NO_PLAN);
            a.cached_out[r] = a.cached[r];
        }
        return;
    }
    int moved = 0, after = p.cached + p.trunk;
    if (p.n > 0 && p.k > 0) {
        if (branch < -1 || branch >= p.n || (branch >= 0 && (accepted < 0 || accepted > p.k))) {
            after = p.cached;
            if (first) atomicOr(a.status, DUO_PAGE_BAD_RECORD);
        } else if (branch < 0) {
            if (token < 0) after = p.cached;
        } else {
            after += accepted;
            moved = branch > 0 ? accepted : 0;
        }
    }
    if (first) a.cached_out[r] = after;
    if (moved == 0) return;
    const int to0 = p.cached + p.trunk, from0 = to0 + branch * p.k;
    const int32_t* line = a.table + (size_t)r * a.max_pages;
    const size_t layer_pages = (size_t)layer * a.n_pages;
    const int mask = (1 << a.page_shift) - 1;
    auto page_at = [&](int logical) {
        const int page = line[logical >> a.page_shift];
        const bool fine = (unsigned)page < (unsigned)a.n_pages;
        if (!fine) atomicOr(a.status, DUO_PAGE_BAD_PAGE);
        return fine ? page : -1;
    };
    auto plane = [&](u16* base, int page) { return base + (((layer_pages + page) * a.hkv + head) << a.page_shift) * D; };
    // the targets lie in one page or two as a rule: looked up once, like the source's first and last
    const int to_page0 = page_at(to0), to_page1 = page_at(to0 + moved - 1), from_page0 = page_at(from0), from_page1 = page_at(from0 + moved - 1);
    auto page_of = [&](int logical, int first, int last, int page0, int page1) {
        const int at = logical >> a.page_shift;
        return at == first >> a.page_shift ? page0 : at == last >> a.page_shift ? page1 : page_at(logical);
    };
    auto to_page = [&](int logical) { return page_of(logical, to0, to0 + moved - 1, to_page0, to_page1); };
    auto from_page = [&](int logical) { return page_of(logical, from0, from0 + moved - 1, from_page0, from_page1); };
    constexpr int KP = D / 8;
    for (int i = threadIdx.x; i < moved * KP; i += blockDim.x) {
        const int j = i / KP, d = i % KP * 8, from = from_page(from0 + j), to = to_page(to0 + j);
        if (from >= 0 && to >= 0)
            *reinterpret_cast<u32x4*>(plane(a.kc, to) + k_cache_offset(D, (to0 + j) & mask, d)) =
                *reinterpret_cast<const u32x4*>(plane(a.kc, from) + k_cache_offset(D, (from0 + j) & mask, d));
    }
    const int group0 = from0 >> 3, groups = ((from0 + moved - 1) >> 3) - group0 + 1;
    for (int i = threadIdx.x; i < groups * D; i += blockDim.x) {
        const int d = i % D, slot0 = (group0 + i / D) * 8, from = from_page(slot0);  // a group lies in one page
        if (from < 0) continue;
        Frag8 f;
        f.q = *reinterpret_cast<const u32x4*>(plane(a.vc, from) + v_cache_offset(D, slot0 & mask, d));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int j = slot0 + e - from0;
            if (j < 0 || j >= moved) continue;
            const int to = to_page(to0 + j);
            if (to >= 0) plane(a.vc, to)[v_cache_offset(D, (to0 + j) & mask, d)] = f.h[e];
        }
    }
}
