// Attention of a planned step over the paged cache (see duo_page.h for the plan, duo_page_rules.h for how it is cut).
//
// Both kernels form S^T = K Q^T and O^T += V^T P^T with the matrix units on the cache's operand tiles.  A block's key order is such that the
// accumulators of S^T are the operand of P^T in the same lane, so nothing crosses lanes between the two products.  The softmax runs online: a
// row's reference m lags its maximum by up to 2^8, so that weights are at most 2^8, and moves (with the output rescaled) only when a score
// goes beyond; sums are fp32.
#pragma once
#include "duo_attn.h"
#include "duo_page.h"

typedef float f32x16 __attribute__((ext_vector_type(16)));

struct PageAttnArgs {
    const u16* q;
    u16* out;
    size_t q_stride, out_stride;
    const u16 *kc, *vc;  // this layer's pages
    const int32_t* table;
    int32_t* status;
    const char* ws;
    size_t info, items, merge;
    float *part_stream, *part_tile;
    int32_t stream_rows;
    int32_t requests, hq, hkv, page_shift, n_pages, max_pages, max_rows, max_new;
    float scale_log2;
};

constexpr float PAGE_LAG = 8.f, PAGE_MOST = 256.f;  // the largest softmax weight and its log2: so far the reference may stay behind

// What a row sees: slots below `before`, and slots from `lo` to `hi`.
struct PageSight {
    int before, lo, hi;
    __device__ __forceinline__ bool operator()(int slot) const { return (slot < before) | ((slot >= lo) & (slot <= hi)); }
};
__device__ __forceinline__ PageSight page_sight(const PageItem& it, int token, bool valid) {
    PageSight s;
    if (!valid) {
        s.before = 0, s.lo = 1, s.hi = 0;
    } else if (token < it.trunk) {
        s.before = it.cached + token + 1, s.lo = 1, s.hi = 0;
    } else {
        s.before = it.cached + it.trunk;
        s.lo = s.before + (token - it.trunk) / it.k * it.k;
        s.hi = it.cached + token;
    }
    return s;
}

__device__ __forceinline__ PageItem page_item(const PageItem* p) {  // the same for a whole workgroup: in scalar registers
    union {
        PageItem it;
        int v[PAGE_ITEM_INTS];
    } u;
    u.it = *p;
#pragma unroll
    for (int i = 0; i < PAGE_ITEM_INTS; ++i) u.v[i] = __builtin_amdgcn_readfirstlane(u.v[i]);
    return u.it;
}
// 16 bytes per lane from global memory to LDS, lane after lane from `lds` on.  In assembly because of the waits: a wave that both requests
// and reads LDS would otherwise wait for all of its requests in front of every read.  The wave waits for them itself (page_stage_landed).
__device__ __forceinline__ void page_load_lds(const u16* src, uint32_t lane_bytes, uint32_t lds) {  // src and lds the same in all lanes
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(lane_bytes), "s"(src), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p);
}
// All but the newest N of this wave's vector memory requests and all of its LDS reads have come back; then the workgroup's barrier.  Nothing
// moves across.
template <int N>
__device__ __forceinline__ void page_stage_landed() {
    static_assert(N >= 0 && N <= 63, "the memory counter has six bits");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Keeps a value's elements whose keys are below `valid` (of eight consecutive keys), the others become zero.
__device__ __forceinline__ elem8 keep_keys(elem8 v, int valid) {
    Frag8 f;
    f.v = v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t mask = valid > 2 * e + 1 ? 0xffffffffu : valid > 2 * e ? 0xffffu : 0u;
        f.q[e] &= mask;
    }
    return f.v;
}
// Bits 15 and 31 of the result are set where an element of such a pair is infinite or not a number (an exponent of all ones: one more
// carries into the sign's place); the other bits mean nothing.
__device__ __forceinline__ uint32_t not_finite(uint32_t pair) {
#ifdef DUO_FP16
    return (pair & 0x7fff7fffu) + 0x04000400u;
#else
    return (pair & 0x7fff7fffu) + 0x00800080u;
#endif
}
__device__ __forceinline__ uint32_t not_finite(elem8 v) {
    Frag8 f;
    f.v = v;
    return not_finite(f.q[0]) | not_finite(f.q[1]) | not_finite(f.q[2]) | not_finite(f.q[3]);
}
constexpr uint32_t NOT_FINITE = 0x80008000u;
// The same with infinities and NaN replaced by zero.
__device__ __forceinline__ elem8 finite_part(elem8 v) {
    Frag8 f;
    f.v = v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t bad = not_finite(f.q[e]) & NOT_FINITE;
        f.q[e] &= ~((bad >> 15) * 0xffffu);
    }
    return f.v;
}
// The V operand with key `key` of the block alone, where this lane holds keys from 8 * (lane's key group) on.
__device__ __forceinline__ elem8 one_key(elem8 v, int key, bool mine) {
    Frag8 f;
    f.v = v;
#pragma unroll
    for (int e = 0; e < 4; ++e) f.q[e] &= !mine ? 0u : (key & 7) == 2 * e ? 0xffffu : (key & 7) == 2 * e + 1 ? 0xffff0000u : 0u;
    return f.v;
}

// ---- few rows: the cache's bytes bound the time
//
// Four waves, wave w takes blocks w, w + 4, ... of the item and holds all RT tiles of 16 rows.  Keys and values come straight into
// registers, 1 KiB per load and each byte once: the next block's keys are requested when this block's scores are done, its values when
// its products are, so a wave always has 8 to 16 KiB in flight.  The waves' states are joined through LDS.
template <int D, int RT>
__global__ __launch_bounds__(256) void page_stream_kernel(PageAttnArgs a) {
    constexpr int KS = D / 32, DT = D / 16, NW = 4;
    __shared__ f32x4 lds_o[NW][DT * 64];
    __shared__ float lds_ml[NW][RT][2][16];
    const int index = blockIdx.x / a.hkv, hk = blockIdx.x - index * a.hkv;
    const PageHeader* hdr = reinterpret_cast<const PageHeader*>(a.ws);
    if (!page_plan_is(*hdr, a.requests, a.hq, a.hkv, D, a.page_shift, a.max_pages, a.max_rows, a.max_new)) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.status, DUO_PAGE_NO_PLAN);
        return;
    }
    if (index >= hdr->stream_items) return;
    const PageItem it = page_item(reinterpret_cast<const PageItem*>(a.ws + a.items) + index);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int c = lane & 15, g = lane >> 4;
    const int group = a.hq / a.hkv;
    const int tiles = (it.count + 15) >> 4;  // at most RT: max_new bounds it

    elem8 qf[RT][KS];
    PageSight sight[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = rt * 16 + c;
        const bool valid = r < it.count;
        const int token = valid ? r / group : 0, gq = valid ? r - token * group : 0;
        sight[rt] = page_sight(it, token, valid);
        const u16* qp = a.q + (size_t)(it.row0 + token) * a.q_stride + (hk * group + gq) * D + g * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            Frag8 f;
            f.q = valid ? *reinterpret_cast<const u32x4*>(qp + ks * 32) : u32x4{0u, 0u, 0u, 0u};
            qf[rt][ks] = f.v;
        }
    }
    const int sees_all = it.cached + (it.trunk > 0 ? 1 : 0);  // slots below are seen by every row
    const int nb = it.blocks > wave ? (it.blocks - wave + NW - 1) / NW : 0;
    const int32_t* line = a.table + (size_t)it.request * a.max_pages;
    const int shift = a.page_shift - 5;  // blocks per page

    // Page ids of the wave's next 64 blocks, one per lane: a scalar load per block would stand in front of its addresses.
    int ids = 0;
    auto fetch_ids = [&](int i) {  // blocks i .. i + 63 of the wave
        const int b = min(it.block0 + wave + NW * (i + lane), it.last_block);
        const int id = line[b >> shift];
        const bool fine = (unsigned)id < (unsigned)a.n_pages;
        if (!fine) atomicOr(a.status, DUO_PAGE_BAD_PAGE);
        ids = fine ? id : 0;
    };
    auto block_at = [&](int i) {  // element offset of block i of the wave in the layer's pages
        const int b = min(it.block0 + wave + NW * i, it.last_block);
        const int id = __builtin_amdgcn_readlane(ids, i & 63);
        return ((((size_t)id * a.hkv + hk) << a.page_shift) + ((b & ((1 << shift) - 1)) << 5)) * D + lane * 8;
    };
    elem8 kf[2][KS], vf[DT];
    auto load_k = [&](size_t at) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) kf[t][ks] = load_frag_stream(a.kc + at + (t * KS + ks) * 512);
    };
    auto load_v = [&](size_t at) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vf[dt] = load_frag_stream(a.vc + at + dt * 512);
    };

    f32x4 o[RT][DT];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = -INFINITY, l[rt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[rt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (nb > 0) {
        fetch_ids(0);
        size_t at = block_at(0);
        load_k(at);
        load_v(at);
        for (int i = 0; i < nb; ++i) {
            const int kb = (it.block0 + wave + NW * i) * 32;
            const bool masked = kb + 32 > sees_all;
            f32x4 s[RT][2];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                if (rt > 0 && rt >= tiles) continue;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) acc = mfma16(kf[t][ks], qf[rt][ks], acc);
                    s[rt][t] = acc;
                }
            }
            if (((i + 1) & 63) == 0) fetch_ids(i + 1);
            at = block_at(i + 1 < nb ? i + 1 : i);
            if (i + 1 < nb) load_k(at);
            Frag8 ph[RT], pl[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                if (rt > 0 && rt >= tiles) continue;
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = s[rt][j >> 2][j & 3];
                if (masked) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = sight[rt](kb + g * 8 + j) ? x[j] : -INFINITY;
                }
                float top = x[0];
#pragma unroll
                for (int j = 1; j < 8; ++j) top = fmaxf(top, x[j]);
                top *= a.scale_log2;
                if (__ballot(top > m[rt] + PAGE_LAG)) {
                    const float m_new = fmaxf(m[rt], lane_groups_max(top));
                    const float alpha = exp2f(m[rt] - (m_new == -INFINITY ? 0.f : m_new));
                    m[rt] = m_new;
                    l[rt] *= alpha;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) o[rt][dt] = o[rt][dt] * alpha;
                }
                const float ref = m[rt] == -INFINITY ? 0.f : m[rt];
                float w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    w[j] = exp2f(fmaf(x[j], a.scale_log2, -ref));
                    l[rt] += w[j];
                }
                split_elem8(w, ph[rt].q, pl[rt].q);
            }
            uint32_t odd = 0;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                if (masked) vf[dt] = keep_keys(vf[dt], it.slots - kb - g * 8);  // slots behind the last may hold anything
                odd |= not_finite(vf[dt]);
            }
            if (!__any((odd & NOT_FINITE) != 0)) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    if (rt > 0 && rt >= tiles) continue;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        o[rt][dt] = mfma16(vf[dt], pl[rt].v, o[rt][dt]);
                        o[rt][dt] = mfma16(vf[dt], ph[rt].v, o[rt][dt]);
                    }
                }
            } else {  // infinities or NaN among the values: key by key, added only where it is seen (0 * inf is not 0), lo halves with what is finite (lo * inf has any sign)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
#pragma unroll 1
                    for (int key = 0; key < 32; ++key) {
                        const elem8 v = one_key(vf[dt], key, g == key >> 3), fin = finite_part(v);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) {
                            if (rt > 0 && rt >= tiles) continue;
                            f32x4 add = mfma16(fin, pl[rt].v, f32x4{0.f, 0.f, 0.f, 0.f});
                            add = mfma16(v, ph[rt].v, add);
                            const bool seen = sight[rt](kb + key);
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[rt][dt][e] += seen ? add[e] : 0.f;
                        }
                    }
                }
            }
            if (i + 1 < nb) load_v(at);
        }
    }

    // Join the waves: a tile at a time, wave w adds its quarter of the channels in wave order.
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        l[rt] += __shfl_xor(l[rt], 16, 64);
        l[rt] += __shfl_xor(l[rt], 32, 64);
        if (g == 0) lds_ml[wave][rt][0][c] = m[rt], lds_ml[wave][rt][1][c] = l[rt];
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        if (rt > 0 && rt >= tiles) continue;  // the same for the whole workgroup
        __syncthreads();
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) lds_o[wave][dt * 64 + lane] = o[rt][dt];
        __syncthreads();
        float top = lds_ml[0][rt][0][c];
#pragma unroll
        for (int w = 1; w < NW; ++w) top = fmaxf(top, lds_ml[w][rt][0][c]);
        float f[NW], sum = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float mw = lds_ml[w][rt][0][c], lw = lds_ml[w][rt][1][c];
            f[w] = exp2f(mw - (top == -INFINITY ? 0.f : top));
            sum += lw * f[w];
        }
        const int r = rt * 16 + c;
        if (r >= it.count) continue;
        const int token = r / group, gq = r - token * group;
        const float inv = 1.0f / sum;
#pragma unroll
        for (int i = 0; i < DT / NW; ++i) {
            const int dt = wave * (DT / NW) + i;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NW; ++w) acc += lds_o[w][dt * 64 + lane] * f[w];
            if (it.part < 0) {
                u32x2 v;
                v[0] = pack_elem2(acc[0] * inv, acc[1] * inv);
                v[1] = pack_elem2(acc[2] * inv, acc[3] * inv);
                u16* dst = a.out + (size_t)(it.row0 + token) * a.out_stride + (hk * group + gq) * D + dt * 16 + g * 4;
                *reinterpret_cast<u32x2*>(dst) = v;
            } else {
                float* dst = a.part_stream + (((size_t)it.part * a.hkv + hk) * a.stream_rows + r) * (D + 4);
                *reinterpret_cast<f32x4*>(dst + dt * 16 + g * 4) = acc;
                if (dt == 0 && g == 0) dst[D] = top, dst[D + 1] = sum;
            }
        }
    }
}

// ---- many rows: the matrix units bound the time
//
// Four waves of 32 rows; keys and values of two blocks (a stage) at a time are put in LDS for all of them by 16-byte loads from global memory to
// LDS.  32 x 32 x 16 products: the tiles' lanes are picked from LDS so that a lane's scores are eight consecutive keys twice over,
// which is the operand of the second product.  The scores of a stage are formed while the weights of the one before are, so K runs a stage
// ahead of V; one barrier a stage.
__device__ __forceinline__ f32x16 mfma32(elem8 a, elem8 b, f32x16 c) {
    // D[32x32] += A[32x16] * B[16x32]; lane l supplies A[l%32][8*(l/32) .. +8] and B[8*(l/32) .. +8][l%32]; register i of lane l is
    // D[8*(i/4) + 4*(l/32) + i%4][l%32].
#ifdef DUO_FP16
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
#else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
#endif
}
__device__ __forceinline__ float lane_halves_max(float x) {
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

template <int D>
__global__ __launch_bounds__(256, 2) void page_tile_kernel(PageAttnArgs a) {
    constexpr int KS = D / 32, DT = D / 16, C32 = D / 32, NW = 4;
    constexpr int KT = 2 * KS, BPS = 2;            // 1 KiB tiles of a block's keys (and DT of its values), blocks a stage
    constexpr int KPW = BPS * KT / NW, VPW = BPS * DT / NW;  // tiles that a wave moves, of one block: waves 0 and 1 the first, 2 and 3 the second
    static_assert(NW * 32 == PAGE_TILE_ROWS && KT == DT && NW == 2 * BPS, "a workgroup takes a tile, two waves move a block");
    __shared__ u32x4 lds_k[2][BPS * KT * 64], lds_v[2][BPS * DT * 64];
    const int index = blockIdx.x / a.hkv, hk = blockIdx.x - index * a.hkv;
    const PageItem it = page_item(reinterpret_cast<const PageItem*>(a.ws + a.items) + index);  // of no meaning behind the last
    const PageHeader* hdr = reinterpret_cast<const PageHeader*>(a.ws);
    if (!page_plan_is(*hdr, a.requests, a.hq, a.hkv, D, a.page_shift, a.max_pages, a.max_rows, a.max_new)) return;  // reported by the other kernel
    if (index >= hdr->tile_items) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int col = lane & 31, half = lane >> 5;
    const int group = a.hq / a.hkv;

    // The wave moves half a block of keys and half a block of values a stage.  Stage st holds the values of blocks 2 st and 2 st + 1 of the range and the
    // keys of 2 st + 1 and 2 st + 2; stage -1 the keys of block 0.  Blocks behind the range repeat its last one and are not used.
    const int32_t* line = a.table + (size_t)it.request * a.max_pages;
    const int shift = a.page_shift - 5;
    const int nst = (it.blocks + BPS - 1) / BPS;
    const int my_block = wave >> 1, my_tile = (wave & 1) * KPW;
    const uint32_t lds_k_mine = lds_address(lds_k) + (my_block * KT + my_tile) * 1024, lds_v_mine = lds_address(lds_v) + (my_block * DT + my_tile) * 1024;
    auto fetch_id = [&](int b) {  // page of block b of the range, b differs from lane to lane
        const int id = line[min(it.block0 + min(b, it.blocks - 1), it.last_block) >> shift];
        const bool fine = (unsigned)id < (unsigned)a.n_pages;
        if (!fine) atomicOr(a.status, DUO_PAGE_BAD_PAGE);
        return fine ? id : 0;
    };
    auto place = [&](int id, int b) {  // of this wave's tiles of block b
        const int in_page = (it.block0 + min(b, it.blocks - 1)) & ((1 << shift) - 1);
        return ((((size_t)id * a.hkv + hk) << a.page_shift) + (in_page << 5)) * D + my_tile * 512;
    };
    int ids_k = 0, ids_v = 0;  // pages of the wave's blocks in stages st .. st + 63
    auto request = [&](int st) {
        if ((st & 63) == 0) {
            ids_k = fetch_id((st + lane) * BPS + my_block + 1);
            ids_v = fetch_id((st + lane) * BPS + my_block);
        }
        const u16* k = a.kc + place(__builtin_amdgcn_readlane(ids_k, st & 63), st * BPS + my_block + 1);
        const u16* v = a.vc + place(__builtin_amdgcn_readlane(ids_v, st & 63), st * BPS + my_block);
#pragma unroll
        for (int i = 0; i < VPW; ++i) page_load_lds(v + i * 512, lane * 16, lds_v_mine + (st & 1) * (BPS * DT * 1024) + i * 1024);
#pragma unroll
        for (int i = 0; i < KPW; ++i) page_load_lds(k + i * 512, lane * 16, lds_k_mine + (st & 1) * (BPS * KT * 1024) + i * 1024);
    };
    if (nst > 0) {
        {
            const u16* k = a.kc + place(__builtin_amdgcn_readfirstlane(fetch_id(0)), 0);
            const int half_mine = (my_block * (KPW / 2)) ;  // block 0 is shared out among all four waves
#pragma unroll
            for (int i = 0; i < KPW / 2; ++i)
                page_load_lds(k + (half_mine + i) * 512, lane * 16, lds_address(lds_k) + ((BPS + 1) * KT + my_tile + half_mine + i) * 1024);
        }
        request(0);
    }

    const int r = wave * 32 + col;  // of the tile
    const bool valid = r < it.count;
    const int pair = it.first + (valid ? r : 0);  // rows behind the tile's last take the first's queries and see nothing
    const int token = pair / group, gq = pair - token * group;
    const PageSight sight = page_sight(it, token, valid);
    elem8 qf[KT];
    {
        const u16* qp = a.q + (size_t)(it.row0 + token) * a.q_stride + (hk * group + gq) * D + half * 8;
#pragma unroll
        for (int s = 0; s < KT; ++s) {
            Frag8 f;
            f.q = *reinterpret_cast<const u32x4*>(qp + s * 16);
            qf[s] = f.v;
        }
    }
    // the last slot that any of the wave's rows sees
    const int rows_here = min(32, it.count - wave * 32);
    const int sees_last = rows_here > 0 ? it.cached + (it.first + wave * 32 + rows_here - 1) / group : -1;

    f32x16 o[C32];
    float m = -INFINITY, l = 0.f;
    auto zero = [] {
        f32x16 z;
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = 0.f;
        return z;
    };
#pragma unroll
    for (int d = 0; d < C32; ++d) o[d] = zero();
    const int frag_k = (col >> 4) * KS * 64 + half * 16 + (col & 15), frag_v = (col >> 4) * 64 + half * 16 + (col & 15);
    auto value_frag = [&](int st, int z, int d, int jj) {
        Frag8 f;
        f.q = lds_v[st & 1][z * DT * 64 + frag_v + 2 * d * 64 + 2 * jj * 16];
        return f.v;
    };
    auto take_keys = [&](elem8 (&f)[KT], int st, int z) {
#pragma unroll
        for (int j = 0; j < KT; ++j) {
            Frag8 x;
            x.q = lds_k[st & 1][z * KT * 64 + frag_k + (j >> 1) * 64 + (j & 1) * 32];
            f[j] = x.v;
        }
    };
    auto take_values = [&](elem8 (&f)[C32][2], int st, int z) {
#pragma unroll
        for (int d = 0; d < C32; ++d)
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) f[d][jj] = value_frag(st, z, d, jj);
    };
    auto scores = [&](const elem8 (&f)[KT]) {
        f32x16 s = zero();
#pragma unroll
        for (int j = 0; j < KT; ++j) s = mfma32(f[j], qf[j], s);
        return s;
    };
    auto add_values = [&](const elem8 (&f)[C32][2], const Frag8 (&p)[2]) {
#pragma unroll
        for (int d = 0; d < C32; ++d)
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) o[d] = mfma32(f[d][jj], p[jj].v, o[d]);
    };
    // The softmax weights of a block, as operands; l takes their sum.  The row's reference stays where it is while a lane's weights sum to no more
    // than 2^8, so none of them is larger: no maximum is looked for.  It moves, to the maximum, when they sum to more, and at the first
    // block (m = -inf makes infinities or NaN of them).
    auto weigh = [&](const f32x16& s, Frag8 (&p)[2], auto order) {
        auto with = [&](float ref) {
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int jj = 0; jj < 2; ++jj)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 4 * jj + 8 * (e >> 1) + 2 * (e & 1);
                    const float w0 = exp2_raw(fmaf(s[i], a.scale_log2, -ref)), w1 = exp2_raw(fmaf(s[i + 1], a.scale_log2, -ref));
                    sum[0] += w0;
                    sum[1] += w1;
                    p[jj].q[e] = pack_elem2(w0, w1);
                }
            return sum[0] + sum[1];
        };
        float sum = with(m);
        order();
        if (__builtin_expect(__ballot(!(sum <= PAGE_MOST)) != 0, 0)) {
            asm volatile("");  // a branch, rather than both sides of it every time
            float top = s[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
            const float m_new = fmaxf(m, lane_halves_max(top * a.scale_log2)), ref = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = exp2_raw(m - ref);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < C32; ++d) o[d] = o[d] * alpha;
            sum = with(ref);
        }
        l += sum;
    };
    // The values of a block that some rows do not see whole.
    auto add_masked = [&](int st, int z, int kb, const Frag8 (&p)[2]) {
        auto kept = [&](int d, int jj) { return keep_keys(value_frag(st, z, d, jj), it.slots - kb - 8 * (2 * jj + half)); };  // slots behind the last may hold anything
        uint32_t odd = 0;
#pragma unroll
        for (int d = 0; d < C32; ++d) odd |= not_finite(kept(d, 0)) | not_finite(kept(d, 1));
        if (__builtin_expect(!__any((odd & NOT_FINITE) != 0), 1)) {
#pragma unroll
            for (int d = 0; d < C32; ++d)
#pragma unroll
                for (int jj = 0; jj < 2; ++jj) o[d] = mfma32(kept(d, jj), p[jj].v, o[d]);
            return;
        }
        const int keys = min(32, it.slots - kb);  // key by key, each added only where it is seen: 0 * inf is not 0
#pragma unroll
        for (int d = 0; d < C32; ++d) {
#pragma unroll 1
            for (int key = 0; key < keys; ++key) {
                const int jj = key >> 4;
                Frag8 w;
                w.q = jj ? p[1].q : p[0].q;
                const f32x16 add = mfma32(one_key(value_frag(st, z, d, jj), key, half == ((key >> 3) & 1)), w.v, zero());
                const bool seen = sight(kb + key);
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] += seen ? add[i] : 0.f;
            }
        }
    };

    if (nst > 0) {
        // Stages that every row of the workgroup sees whole come first.
        const int all_see = it.cached + min(it.first / group + 1, it.trunk) - it.block0 * 32;
        const int whole = min(max(all_see, 0) / (32 * BPS), it.blocks / BPS);
        page_stage_landed<KPW + VPW>();  // the keys of block 0
        elem8 kf[KT], vf[C32][2];
        Frag8 p[2];
        take_keys(kf, -1, 1);
        f32x16 s0 = scores(kf), s1;
        int st = 0;
#pragma unroll 1
        for (; st < whole; ++st) {
            page_stage_landed<0>();  // stage st is there, stage st - 1 drained
            request(st + 1);
            take_keys(kf, st, 0);
            take_values(vf, st, 0);
            s1 = scores(kf);
            weigh(s0, p, [] {});
            take_keys(kf, st, 1);
            add_values(vf, p);
            take_values(vf, st, 1);
            s0 = scores(kf);
            weigh(s1, p, [] {});
            add_values(vf, p);
        }
        auto masked = [&](f32x16& s, int b) {  // block b of the range, its scores s
            const int kb = (it.block0 + b) * 32;
            if (b >= it.blocks || kb > sees_last) return;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = sight(kb + 8 * (half + 2 * ((i >> 2) & 1)) + 4 * (i >> 3) + (i & 3)) ? s[i] : -INFINITY;
            weigh(s, p, [] {});
            add_masked(st, b & 1, kb, p);
        };
#pragma unroll 1
        for (; st < nst; ++st) {
            page_stage_landed<0>();
            request(st + 1);
            masked(s0, st * BPS);
            take_keys(kf, st, 0);
            s1 = scores(kf);
            masked(s1, st * BPS + 1);
            take_keys(kf, st, 1);
            s0 = scores(kf);
        }
        page_stage_landed<0>();  // nothing is in flight to LDS when the workgroup ends
    }

    l += __shfl_xor(l, 32, 64);
    if (!valid) return;
    if (it.part < 0) {
        const float inv = 1.0f / l;
        u16* dst = a.out + (size_t)(it.row0 + token) * a.out_stride + (hk * group + gq) * D + half * 4;
#pragma unroll
        for (int d = 0; d < C32; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                u32x2 v;
                v[0] = pack_elem2(o[d][4 * j] * inv, o[d][4 * j + 1] * inv);
                v[1] = pack_elem2(o[d][4 * j + 2] * inv, o[d][4 * j + 3] * inv);
                *reinterpret_cast<u32x2*>(dst + d * 32 + j * 8) = v;
            }
    } else {
        float* dst = a.part_tile + (((size_t)it.part * a.hkv + hk) * PAGE_TILE_ROWS + r) * (D + 4);
#pragma unroll
        for (int d = 0; d < C32; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<f32x4*>(dst + d * 32 + j * 8 + half * 4) = f32x4{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]};
        if (half == 0) dst[D] = m, dst[D + 1] = l;
    }
}

// ---- tiles whose keys were cut: one wave per row joins the ranges' partial results in their order
template <int D>
__global__ __launch_bounds__(256) void page_merge_kernel(PageAttnArgs a) {
    const PageHeader* hdr = reinterpret_cast<const PageHeader*>(a.ws);
    if (!page_plan_is(*hdr, a.requests, a.hq, a.hkv, D, a.page_shift, a.max_pages, a.max_rows, a.max_new)) return;
    const int index = blockIdx.x / a.hkv, hk = blockIdx.x - index * a.hkv;
    if (index >= hdr->merges) return;
    const PageMerge mg = reinterpret_cast<const PageMerge*>(a.ws + a.merge)[index];
    const int lane = threadIdx.x & 63, group = a.hq / a.hkv;
    const int rows = mg.streamed ? a.stream_rows : PAGE_TILE_ROWS;
    const float* part = mg.streamed ? a.part_stream : a.part_tile;
    constexpr int E = D / 64;
    for (int r = blockIdx.y * 4 + (threadIdx.x >> 6); r < mg.count; r += gridDim.y * 4) {
        const float* src = part + (((size_t)mg.part0 * a.hkv + hk) * rows + r) * (D + 4);
        const size_t step = (size_t)a.hkv * rows * (D + 4);
        float top = -INFINITY, sum = 0.f, acc[E] = {};
        for (int i0 = 0; i0 < mg.parts; i0 += 4) {
            float mi[4], li[4], v[4][E];
#pragma unroll
            for (int i = 0; i < 4; ++i) {  // ranges behind the last repeat it with no weight
                const float* p = src + step * min(i0 + i, mg.parts - 1);
                mi[i] = i0 + i < mg.parts ? p[D] : -INFINITY;
                li[i] = i0 + i < mg.parts ? p[D + 1] : 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) v[i][e] = p[lane + e * 64];
            }
            float t = top;
#pragma unroll
            for (int i = 0; i < 4; ++i) t = fmaxf(t, mi[i]);
            const float ref = t == -INFINITY ? 0.f : t;
            const float w0 = exp2f(top - ref);
            sum *= w0;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] *= w0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i0 + i >= mg.parts) continue;
                const float w = exp2f(mi[i] - ref);
                sum += li[i] * w;
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] += v[i][e] * w;
            }
            top = t;
        }
        const int pair = mg.first + r, token = pair / group, gq = pair - token * group;
        u16* dst = a.out + (size_t)(mg.row0 + token) * a.out_stride + (hk * group + gq) * D;
#pragma unroll
        for (int e = 0; e < E; ++e) dst[lane + e * 64] = (u16)pack_elem2(acc[e] / sum, 0.f);
    }
}
