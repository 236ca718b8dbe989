// Attention of a planned step over the paged cache (see duo_page.h for the plan, duo_page_rules.h for how it is cut).
//
// All kernels form S^T = K Q^T and O^T += V^T P^T with the matrix units on the cache's operand tiles.  A block's key order is such that the
// accumulators of S^T are the operand of P^T in the same lane, so nothing crosses lanes between the two products.  The softmax runs online: a
// row's reference m lags its maximum by up to 2^8, so that weights are at most that (raised by 2^7 in fp16, see PAGE_RAISE), and moves (with the
// output rescaled) only when a score goes beyond; sums are fp32.
#pragma once
#include <type_traits>

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
    size_t stream, tile, merge;
    float *part_stream, *part_tile;
    int32_t stream_rows, tile_items;  // rows kept per streamed partial result; room for tiled items
    int32_t requests, hq, hkv, page_shift, n_pages, max_pages, max_rows, max_new;
    float scale_log2;
};

// How far the reference may stay behind a score, as a log2, and how far the weights are raised on top, so that the 16-bit type holds as small ones as
// it can: fp16 ends at 2^16 and rounds to zero below 2^-25, which then is 2^-32 of the reference's weight.  Sums and outputs are raised alike, so
// the factor falls out of their quotient.  (Without it a key in front of a flat tail 2^-25 below lost the tail: 131000 keys, 0.4 % of the sum.)
#ifdef DUO_FP16
constexpr float PAGE_LAG = 8.f, PAGE_RAISE = 7.f, PAGE_MOST = 32768.f;  // PAGE_MOST: the largest weight, 2^(lag + raise)
__device__ __forceinline__ float page_exponent_offset(float ref) { return PAGE_RAISE - ref; }
#else
constexpr float PAGE_LAG = 8.f, PAGE_MOST = 256.f;
__device__ __forceinline__ float page_exponent_offset(float ref) { return -ref; }
#endif

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
// ONCE: with the non-temporal hint, for what one workgroup alone reads.
template <bool ONCE>
__device__ __forceinline__ void page_load_lds(const u16* src, uint32_t lane_bytes, uint32_t lds) {  // src and lds the same in all lanes
    if (ONCE) asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(lane_bytes), "s"(src), "s"(lds) : "memory", "m0");
    else asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(lane_bytes), "s"(src), "s"(lds) : "memory", "m0");
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

// The queries have come: waited for here, in front of a loop.  A wait for them inside it would be a wait for the newest request at every turn.
template <int N>
__device__ __forceinline__ void page_queries_landed(elem8 (&q)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(q[i]));
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
// Values that are not finite, where some rows do not see their key: 0 * inf is not 0, so they stay out of the product of weights and values, and a
// second product says which rows see which of them: codes of the values (1 for inf, 64 for -inf, 4096 for NaN, of at most 32 keys) times
// ones where a row sees a key.
__device__ __forceinline__ elem8 finite_part(elem8 v) {
    Frag8 f;
    f.v = v;
#pragma unroll
    for (int e = 0; e < 4; ++e) f.q[e] &= ~(((not_finite(f.q[e]) & NOT_FINITE) >> 15) * 0xffffu);
    return f.v;
}
__device__ __forceinline__ elem8 code_part(elem8 v) {
#ifdef DUO_FP16
    constexpr u16 INF = 0x7c00, C_INF = 0x3c00, C_MINUS = 0x5400, C_NAN = 0x6c00;
#else
    constexpr u16 INF = 0x7f80, C_INF = 0x3f80, C_MINUS = 0x4280, C_NAN = 0x4580;
#endif
    Frag8 f;
    f.v = v;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const u16 x = f.h[e], size = x & 0x7fff;
        f.h[e] = size < INF ? 0 : size > INF ? C_NAN : x == INF ? C_INF : C_MINUS;
    }
    return f.v;
}
__device__ __forceinline__ elem8 seen_part(const PageSight& sight, int first) {  // ones for the keys first .. first + 7 that the row sees
    Frag8 f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f.h[e] = sight(first + e) ? f32_to_elem(1.f) : (u16)0;
    return f.v;
}
__device__ __forceinline__ float decoded(float sum) {  // what the values of a sum of codes add up to
    const float minus = floorf(sum * (1.f / 64)), plus = sum - 64.f * minus;
    const float x = (plus > 0.f ? INFINITY : 0.f) + (minus > 0.f ? -INFINITY : 0.f);  // both: NaN
    return sum >= 4096.f ? NAN : x;
}

// ---- up to 16 rows: the cache's bytes bound the time
//
// NW waves, wave w takes blocks w, w + NW, ... of the item.  Keys and values come straight into registers, 1 KiB per load and each byte once: the
// next block's keys are requested when this block's scores are done, its values when its products are, so a wave always has 8 to 16 KiB
// in flight and eight waves fit a compute unit.  The waves' states are joined through LDS.  64 decoding requests, 640 MB: 104 us, 6.1 TB/s; 115
// with keys and values a whole block ahead, where four waves fit.
template <int D, int NW>
struct PageStreamLds {
    f32x4 o[NW][D / 16 * 64];
    float ml[NW][2][16];
};
template <int D, int NW>
__device__ __forceinline__ void page_stream(const PageAttnArgs& a, int place, PageStreamLds<D, NW>& lds) {
    constexpr int KS = D / 32, DT = D / 16;
    auto& lds_o = lds.o;
    auto& lds_ml = lds.ml;
    const int index = place / a.hkv, hk = place - index * a.hkv;
    const PageItem it = page_item(reinterpret_cast<const PageItem*>(a.ws + a.stream) + index);  // of no meaning behind the last
    const PageHeader* hdr = reinterpret_cast<const PageHeader*>(a.ws);
    if (!page_plan_is(*hdr, a.requests, a.hq, a.hkv, D, a.page_shift, a.max_pages, a.max_rows, a.max_new)) {
        if (place == 0 && threadIdx.x == 0) atomicOr(a.status, DUO_PAGE_NO_PLAN);
        return;
    }
    if (index >= hdr->stream_items) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int c = lane & 15, g = lane >> 4;
    const int group = a.hq / a.hkv;
    const bool valid = c < it.count;  // the item's row c
    const int token = valid ? c / group : 0, gq = valid ? c - token * group : 0;
    const PageSight sight = page_sight(it, token, valid);

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

    f32x4 o[DT];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (nb > 0) {
        fetch_ids(0);
        size_t at = block_at(0);
        load_k(at);
        load_v(at);
        elem8 qf[KS];
        {
            const u16* qp = a.q + (size_t)(it.row0 + token) * a.q_stride + (hk * group + gq) * D + g * 8;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) qf[ks] = load_frag(qp + ks * 32);  // a column without a row takes the first row's and sees nothing
        }
        page_queries_landed(qf);
        for (int i = 0; i < nb; ++i) {
            const int kb = (it.block0 + wave + NW * i) * 32;
            const bool masked = kb + 32 > sees_all;
            float s[8];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) acc = mfma16(kf[t][ks], qf[ks], acc);
#pragma unroll
                for (int e = 0; e < 4; ++e) s[4 * t + e] = acc[e];
            }
            if (((i + 1) & 63) == 0) fetch_ids(i + 1);
            at = block_at(i + 1 < nb ? i + 1 : i);
            if (i + 1 < nb) load_k(at);
            if (masked) {
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] = sight(kb + g * 8 + j) ? s[j] : -INFINITY;
            }
            float top = s[0];
#pragma unroll
            for (int j = 1; j < 8; ++j) top = fmaxf(top, s[j]);
            top *= a.scale_log2;
            if (__ballot(top > m + PAGE_LAG)) {
                const float m_new = fmaxf(m, lane_groups_max(top));
                const float alpha = exp2f(m - (m_new == -INFINITY ? 0.f : m_new));
                m = m_new;
                l *= alpha;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] = o[dt] * alpha;
            }
            const float offset = page_exponent_offset(m == -INFINITY ? 0.f : m);
            float w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                w[j] = exp2f(fmaf(s[j], a.scale_log2, offset));
                l += w[j];
            }
            Frag8 ph, pl;
            split_elem8(w, ph.q, pl.q);
            uint32_t odd = 0;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                if (masked) vf[dt] = keep_keys(vf[dt], it.slots - kb - g * 8);  // slots behind the last may hold anything
                odd |= not_finite(vf[dt]);
            }
            if (__builtin_expect(!__any((odd & NOT_FINITE) != 0), 1)) {
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    o[dt] = mfma16(vf[dt], pl.v, o[dt]);
                    o[dt] = mfma16(vf[dt], ph.v, o[dt]);
                }
            } else {
                const elem8 seen = seen_part(sight, kb + g * 8);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const elem8 v = finite_part(vf[dt]);
                    o[dt] = mfma16(v, pl.v, o[dt]);
                    o[dt] = mfma16(v, ph.v, o[dt]);
                    const f32x4 code = mfma16(code_part(vf[dt]), seen, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[dt][e] += decoded(code[e]);
                }
            }
            if (i + 1 < nb) load_v(at);
        }
    }

    // Join the waves: each adds its part of the channels in wave order.
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (g == 0) lds_ml[wave][0][c] = m, lds_ml[wave][1][c] = l;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) lds_o[wave][dt * 64 + lane] = o[dt];
    __syncthreads();
    if (!valid) return;
    float top = lds_ml[0][0][c];
#pragma unroll
    for (int w = 1; w < NW; ++w) top = fmaxf(top, lds_ml[w][0][c]);
    float f[NW], sum = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        f[w] = exp2f(lds_ml[w][0][c] - (top == -INFINITY ? 0.f : top));
        sum += lds_ml[w][1][c] * f[w];
    }
    const float inv = 1.0f / sum;
#pragma unroll
    for (int i = 0; i < (DT + NW - 1) / NW; ++i) {
        const int dt = wave * ((DT + NW - 1) / NW) + i;
        if (dt >= DT) break;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) acc += lds_o[w][dt * 64 + lane] * f[w];
        if (it.part < 0) {
            u32x2 v;
            v[0] = pack_elem2(acc[0] * inv, acc[1] * inv);
            v[1] = pack_elem2(acc[2] * inv, acc[3] * inv);
            *reinterpret_cast<u32x2*>(a.out + (size_t)(it.row0 + token) * a.out_stride + (hk * group + gq) * D + dt * 16 + g * 4) = v;
        } else {
            float* dst = a.part_stream + (((size_t)it.part * a.hkv + hk) * a.stream_rows + c) * (D + 4);
            *reinterpret_cast<f32x4*>(dst + dt * 16 + g * 4) = acc;
            if (dt == 0 && g == 0) dst[D] = top, dst[D + 1] = sum;
        }
    }
}
template <int D, int NW>
__global__ __launch_bounds__(64 * NW) void page_stream_kernel(PageAttnArgs a) {
    __shared__ PageStreamLds<D, NW> lds;
    page_stream<D, NW>(a, blockIdx.x, lds);
}

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

// 32 rows of a wave in 32 x 32 x 16 products.  A lane (col, half) picks its 16 bytes of K and V^T tiles from LDS so that it holds, of row `col`,
// the scores of eight consecutive keys twice over, which is the operand of the second product.
template <int D>
struct PageRows {
    static constexpr int KS = D / 32, KT = 2 * KS, DT = D / 16, C32 = D / 32;
    f32x16 o[C32];
    float m = -INFINITY, l = 0.f;  // the exponents' reference; this lane's part of the weights' sum
    elem8 qf[KT];
    PageSight sight;
    int token, gq;    // of row `col`
    int whole, last;  // slots below are seen by all of the 32 rows; the last that any of them sees, -1 without a row
    bool valid;

    static __device__ __forceinline__ f32x16 zero() {
        f32x16 z;
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = 0.f;
        return z;
    }
    static __device__ __forceinline__ int key_of(int i, int half) { return 8 * (half + 2 * ((i >> 2) & 1)) + 4 * (i >> 3) + (i & 3); }  // of register i of the scores
    static __device__ __forceinline__ elem8 key_frag(const u32x4* block, int j, int lane) {
        Frag8 f;
        f.q = block[((lane >> 4) & 1) * KS * 64 + (lane >> 5) * 16 + (lane & 15) + (j >> 1) * 64 + (j & 1) * 32];
        return f.v;
    }
    static __device__ __forceinline__ elem8 value_frag(const u32x4* block, int d, int jj, int lane) {
        Frag8 f;
        f.q = block[((lane >> 4) & 1) * 64 + (lane >> 5) * 16 + (lane & 15) + 2 * d * 64 + 2 * jj * 16];
        return f.v;
    }
    __device__ __forceinline__ void load(const PageAttnArgs& a, const PageItem& it, int hk, int first, int lane) {  // rows first .. first + 31 of the tile
        const int group = a.hq / a.hkv, r = first + (lane & 31);
        valid = r < it.count;
        const int pair = it.first + (valid ? r : 0);  // rows behind the tile's last take the first's queries and see nothing
        token = pair / group, gq = pair - token * group;
        sight = page_sight(it, token, valid);
        const int here = min(32, it.count - first);
        whole = it.cached + min((it.first + first) / group + 1, it.trunk);
        last = here > 0 ? it.cached + (it.first + first + here - 1) / group : -1;
        const u16* qp = a.q + (size_t)(it.row0 + token) * a.q_stride + (hk * group + gq) * D + (lane >> 5) * 8;
#pragma unroll
        for (int s = 0; s < KT; ++s) qf[s] = load_frag(qp + s * 16);
#pragma unroll
        for (int d = 0; d < C32; ++d) o[d] = zero();
    }
    __device__ __forceinline__ f32x16 scores(const elem8 (&f)[KT]) const {
        f32x16 s = zero();
#pragma unroll
        for (int j = 0; j < KT; ++j) s = mfma32(f[j], qf[j], s);
        return s;
    }
    // The softmax weights of a block, as operands; l takes their sum.  The row's reference stays where it is while a lane's weights sum to no more
    // than PAGE_MOST, so none of them is larger: no maximum is looked for.  It moves, to the maximum, when they sum to more, and at the first
    // block (m = -inf makes infinities or NaN of them).  PAIR: hi and lo parts of the weights, otherwise rounded once: in tiles, which the matrix units
    // bound.  There it makes the root-mean-square error against 64 bits 1.3 times that of the output's own rounding (relative: bf16 0.0021 next to
    // 0.0016, fp16 2.6e-4 next to 2.1e-4); pairs leave the latter alone and cost half as many products again: packed prompts 239 us instead of 184, chunks 40
    // instead of 35.
    // Not STEADY: the reference follows the maximum at every block, without a branch around the outputs (which cost page_tile<128> copies of them in
    // memory).
    template <bool PAIR, bool STEADY>
    __device__ __forceinline__ void weigh(const f32x16& s, float scale, Frag8 (&p)[2], Frag8 (&lo)[2]) {
        auto with = [&](float ref) {
            const float offset = page_exponent_offset(ref);
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) {
                float w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    w[e] = exp2_raw(fmaf(s[4 * jj + 8 * (e >> 2) + (e & 3)], scale, offset));
                    sum[e & 1] += w[e];
                }
                if (PAIR) {
                    split_elem8(w, p[jj].q, lo[jj].q);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[jj].q[e] = pack_elem2(w[2 * e], w[2 * e + 1]);
                }
            }
            return sum[0] + sum[1];
        };
        auto move = [&] {
            float top = s[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
            const float m_new = fmaxf(m, lane_halves_max(top * scale)), ref = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = exp2_raw(m - ref);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < C32; ++d) o[d] = o[d] * alpha;
            return with(ref);
        };
        if (!STEADY) {
            l += move();
            return;
        }
        float sum = with(m);
        if (__builtin_expect(__ballot(!(sum <= PAGE_MOST)) != 0, 0)) {
            asm volatile("");  // a branch, rather than both sides of it every time
            sum = move();
        }
        l += sum;
    }
    __device__ __forceinline__ void mask(f32x16& s, int kb, int half) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = sight(kb + key_of(i, half)) ? s[i] : -INFINITY;
    }
    static __device__ __forceinline__ void take_keys(elem8 (&f)[KT], const u32x4* block, int lane) {
#pragma unroll
        for (int j = 0; j < KT; ++j) f[j] = key_frag(block, j, lane);
    }
    static __device__ __forceinline__ void take_values(elem8 (&f)[C32][2], const u32x4* block, int lane) {
#pragma unroll
        for (int d = 0; d < C32; ++d)
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) f[d][jj] = value_frag(block, d, jj, lane);
    }
    template <bool PAIR>
    __device__ __forceinline__ void add(const elem8 (&f)[C32][2], const Frag8 (&p)[2], const Frag8 (&lo)[2]) {  // O += V P
#pragma unroll
        for (int d = 0; d < C32; ++d)
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) {
                if (PAIR) o[d] = mfma32(f[d][jj], lo[jj].v, o[d]);
                o[d] = mfma32(f[d][jj], p[jj].v, o[d]);
            }
    }
    // Before the values of a block that some rows may not see whole, or with pairs of weights (lo * inf has any sign), enter the product: what is
    // behind the last of its `keys` slots in use and what is not finite becomes zero.  Returns whether there is any of the latter, which
    // add_codes then makes good.
    static __device__ __forceinline__ bool clean(elem8 (&f)[C32][2], int keys, int half) {
        if (keys < 32) {  // slots behind the last may hold anything
#pragma unroll
            for (int d = 0; d < C32; ++d)
#pragma unroll
                for (int jj = 0; jj < 2; ++jj) f[d][jj] = keep_keys(f[d][jj], keys - 8 * (2 * jj + half));
        }
        uint32_t odd = 0;
#pragma unroll
        for (int d = 0; d < C32; ++d) odd |= not_finite(f[d][0]) | not_finite(f[d][1]);
        const bool any = __any((odd & NOT_FINITE) != 0);
        if (__builtin_expect(any, 0)) {
            asm volatile("");
#pragma unroll
            for (int d = 0; d < C32; ++d) f[d][0] = finite_part(f[d][0]), f[d][1] = finite_part(f[d][1]);
        }
        return any;
    }
    // Whether an output of any lane's is infinite or not a number: times zero it is not zero.
    __device__ __forceinline__ bool not_finite_output() const {
        float sum = 0.f;
#pragma unroll
        for (int d = 0; d < C32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) sum = fmaf(o[d][i], 0.f, sum);
        return __any(sum != 0.f);
    }
    // What the values of a block (its tiles in global memory) that are not finite add to channels 32 d .. 32 d + 31 of the rows that see them.
    __device__ __forceinline__ void add_codes(f32x16& x, int d, const u16* tiles, int kb, int keys, int lane) const {
        const int half = lane >> 5;
        f32x16 code = zero();
#pragma unroll
        for (int jj = 0; jj < 2; ++jj) {
            const elem8 f = load_frag(tiles + ((2 * d + ((lane >> 4) & 1)) * 64 + (2 * jj + half) * 16 + (lane & 15)) * 8);
            code = mfma32(code_part(keep_keys(f, keys - 8 * (2 * jj + half))), seen_part(sight, kb + 16 * jj + 8 * half), code);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] += decoded(code[i]);
    }
};

// Four channels of a row, from channel `at` of its head on: to the output, or unnormalised to the partial result.
__device__ __forceinline__ void page_store4(u16* dst, const f32x4& v) {
    u32x2 w;
    w[0] = pack_elem2(v[0], v[1]);
    w[1] = pack_elem2(v[2], v[3]);
    *reinterpret_cast<u32x2*>(dst) = w;
}

// The pages of blocks `first + lane * step` of an item's range, and where a block lies.  Blocks behind the range repeat its last one.
struct PageBlocks {
    const int32_t* line;
    int block0, blocks, last, shift, n_pages, page_shift, hkv, hk;
    int32_t* status;
    __device__ __forceinline__ PageBlocks(const PageAttnArgs& a, const PageItem& it, int head)
        : line(a.table + (size_t)it.request * a.max_pages), block0(it.block0), blocks(it.blocks), last(it.last_block), shift(a.page_shift - 5), n_pages(a.n_pages),
          page_shift(a.page_shift), hkv(a.hkv), hk(head), status(a.status) {}
    __device__ __forceinline__ int id(int b) const {  // differs from lane to lane
        const int page = line[min(block0 + min(b, blocks - 1), last) >> shift];
        const bool fine = (unsigned)page < (unsigned)n_pages;
        if (!fine) atomicOr(status, DUO_PAGE_BAD_PAGE);
        return fine ? page : 0;
    }
    template <int D>
    __device__ __forceinline__ size_t place(int page, int b) const {
        const int in_page = (block0 + min(b, blocks - 1)) & ((1 << shift) - 1);
        return ((((size_t)page * hkv + hk) << page_shift) + (in_page << 5)) * D;
    }
};

// ---- 17 to 64 rows: still the cache's bytes
//
// TEAMS teams of UNITS waves, a wave for every 32 rows of the item.  Team z takes blocks z, z + TEAMS, ...: a stage is a block for each team, put in
// LDS by 16-byte loads from global memory to LDS one stage ahead of its use.  Several workgroups fit a compute unit, so that 64 KiB are in
// flight and one's start and end go under the other's loads.  The teams' states are joined through LDS.  One team at heads of 128 (32 KiB of LDS
// a workgroup): 16 x 33 rows of 32 heads 85 us with two, 80 with one (the two launches; 4.7 TB/s); two at heads of 64.
template <int D, int UNITS, int TEAMS>
struct PageTeamLds {
    u32x4 kv[2][TEAMS * 2 * PageRows<D>::KT * 64];
    float ml[TEAMS][UNITS][2][32];
};
template <int D, int UNITS, int TEAMS>
__device__ __forceinline__ void page_team(const PageAttnArgs& a, size_t items, int place, PageTeamLds<D, UNITS, TEAMS>& lds) {
    using Rows = PageRows<D>;
    constexpr int KT = Rows::KT, DT = Rows::DT, C32 = Rows::C32, TILES = KT + DT, PER_WAVE = TILES / UNITS;
    static_assert(TILES % UNITS == 0, "a team's waves move equal parts of its block");
    static_assert(sizeof(lds.kv) >= sizeof(f32x4) * TEAMS * UNITS * C32 * 4 * 64, "the teams' outputs fit");
    auto& lds_kv = lds.kv;
    auto& lds_ml = lds.ml;
    const int index = place / a.hkv, hk = place - index * a.hkv;
    const PageItem it = page_item(reinterpret_cast<const PageItem*>(a.ws + items) + index);  // of no meaning behind the last
    const PageHeader* hdr = reinterpret_cast<const PageHeader*>(a.ws);
    if (!page_plan_is(*hdr, a.requests, a.hq, a.hkv, D, a.page_shift, a.max_pages, a.max_rows, a.max_new)) {
        if (place == 0 && threadIdx.x == 0) atomicOr(a.status, DUO_PAGE_NO_PLAN);
        return;
    }
    if (index >= hdr->stream_items) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int col = lane & 31, half = lane >> 5;
    const int unit = wave % UNITS, team = wave / UNITS;

    const PageBlocks where(a, it, hk);
    const int nst = (it.blocks + TEAMS - 1) / TEAMS;
    const uint32_t lds_mine = lds_address(lds_kv) + (team * TILES + unit * PER_WAVE) * 1024;
    int ids = 0;  // pages of the team's blocks in stages st .. st + 63
    auto request = [&](int st) {
        if ((st & 63) == 0) ids = where.id((st + lane) * TEAMS + team);
        const size_t at = where.place<D>(__builtin_amdgcn_readlane(ids, st & 63), st * TEAMS + team);
#pragma unroll
        for (int i = 0; i < PER_WAVE; ++i) {
            const int j = unit * PER_WAVE + i;
            const u16* src = j < KT ? a.kc + at + j * 512 : a.vc + at + (j - KT) * 512;
            page_load_lds<true>(src, lane * 16, lds_mine + (st & 1) * (TEAMS * TILES * 1024) + i * 1024);
        }
    };
    if (nst > 0) request(0);
    Rows rows;
    rows.load(a, it, hk, unit * 32, lane);
    bool odd = false;
    page_queries_landed(rows.qf);
    for (int st = 0; st < nst; ++st) {
        page_stage_landed<0>();  // stage st is there, stage st - 1 drained
        if (st + 1 < nst) request(st + 1);
        const int b = st * TEAMS + team, kb = (it.block0 + b) * 32;
        if (b >= it.blocks || kb > rows.last) continue;
        const u32x4* block = lds_kv[st & 1] + team * TILES * 64;
        elem8 kf[KT], vf[C32][2];
        Rows::take_keys(kf, block, lane);
        Rows::take_values(vf, block + KT * 64, lane);
        f32x16 s = rows.scores(kf);
        if (kb + 32 > rows.whole) rows.mask(s, kb, half);
        Frag8 p[2], lo[2];
        rows.template weigh<true, true>(s, a.scale_log2, p, lo);
        odd |= Rows::clean(vf, it.slots - kb, half);
        rows.template add<true>(vf, p, lo);
    }
    auto output = [&](int d) {
        f32x16 x = rows.o[d];
        if (__builtin_expect(odd, 0)) {
            for (int b = team; b < it.blocks; b += TEAMS) {
                const int kb = (it.block0 + b) * 32, id = __builtin_amdgcn_readfirstlane(where.id(b));
                if (kb <= rows.last) rows.add_codes(x, d, a.vc + where.place<D>(id, b), kb, it.slots - kb, lane);
            }
        }
        return x;
    };

    // Join the teams: a wave adds its half of its unit's channels in team order.
    rows.l += __shfl_xor(rows.l, 32, 64);
    page_stage_landed<0>();
    f32x4* const lds_o = reinterpret_cast<f32x4*>(lds_kv);
    if (half == 0) lds_ml[team][unit][0][col] = rows.m, lds_ml[team][unit][1][col] = rows.l;
#pragma unroll
    for (int d = 0; d < C32; ++d) {
        const f32x16 x = output(d);
#pragma unroll
        for (int q = 0; q < 4; ++q) lds_o[((team * UNITS + unit) * C32 * 4 + d * 4 + q) * 64 + lane] = f32x4{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
    }
    __syncthreads();
    if (!rows.valid) return;
    float top = lds_ml[0][unit][0][col];
#pragma unroll
    for (int z = 1; z < TEAMS; ++z) top = fmaxf(top, lds_ml[z][unit][0][col]);
    float f[TEAMS], sum = 0.f;
#pragma unroll
    for (int z = 0; z < TEAMS; ++z) {
        f[z] = exp2f(lds_ml[z][unit][0][col] - (top == -INFINITY ? 0.f : top));
        sum += lds_ml[z][unit][1][col] * f[z];
    }
    const float inv = 1.0f / sum;
    u16* const out = a.out + (size_t)(it.row0 + rows.token) * a.out_stride + (hk * (a.hq / a.hkv) + rows.gq) * D + half * 4;
    float* const part = a.part_stream + (((size_t)(it.part < 0 ? 0 : it.part) * a.hkv + hk) * a.stream_rows + unit * 32 + col) * (D + 4);
#pragma unroll
    for (int i = 0; i < 4 * C32 / TEAMS; ++i) {
        const int x = team * (4 * C32 / TEAMS) + i;  // channels 8 x + 4 half .. + 3
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int z = 0; z < TEAMS; ++z) acc += lds_o[((z * UNITS + unit) * C32 * 4 + x) * 64 + lane] * f[z];
        if (it.part < 0) page_store4(out + x * 8, acc * inv);
        else *reinterpret_cast<f32x4*>(part + x * 8 + half * 4) = acc;
    }
    if (it.part >= 0 && team == 0 && half == 0) part[D] = top, part[D + 1] = sum;
}
template <int D, int UNITS, int TEAMS>
__global__ __launch_bounds__(64 * TEAMS * UNITS, 2) void page_team_kernel(PageAttnArgs a) {
    __shared__ PageTeamLds<D, UNITS, TEAMS> lds;
    page_team<D, UNITS, TEAMS>(a, a.stream, blockIdx.x, lds);
}

// ---- many rows: the matrix units bound the time
//
// Four waves of 32 rows share the keys and values of two blocks (a stage) at a time, put in LDS by 16-byte loads from global memory to LDS.  The
// scores of a block are formed while the weights of the one before are, so keys run a block ahead of the values: stage st holds the values of
// blocks 2 st and 2 st + 1 of the range and the keys of 2 st + 1 and 2 st + 2, stage -1 the keys of block 0.  One barrier a stage; two
// workgroups fit a compute unit, and one's start and end go under the other's products.  Five packed prompts of 900 to 4000 tokens, 32 heads over 8: 179 us on the better card,
// 895 TFLOP/s of the causal half; 1135 in the loop over whole stages (a library product of 8192^3 reaches 1257).  There both
// waves of a SIMD take 1500 cycles a block, of which the matrix unit is busy for 1024 and the vector unit for about 840 (exponentials have a quarter of
// the rate).
template <int D>
struct PageTileLds {
    static constexpr int BPS = 2;  // blocks a stage
    u32x4 k[2][BPS * PageRows<D>::KT * 64], v[2][BPS * PageRows<D>::DT * 64];
};
template <int D>
__device__ __forceinline__ void page_tile(const PageAttnArgs& a, size_t items, int place, PageTileLds<D>& lds) {
    using Rows = PageRows<D>;
    constexpr int KT = Rows::KT, DT = Rows::DT, C32 = Rows::C32, NW = 4, BPS = PageTileLds<D>::BPS;  // tiles of a block's keys, of its values
    constexpr int KPW = BPS * KT / NW, VPW = BPS * DT / NW;
    static_assert(NW * 32 == PAGE_TILE_ROWS && KT == DT && NW == 2 * BPS, "a workgroup takes a tile, two waves move a block");
    auto& lds_k = lds.k;
    auto& lds_v = lds.v;
    const int index = place / a.hkv, hk = place - index * a.hkv;
    const PageItem it = page_item(reinterpret_cast<const PageItem*>(a.ws + items) + index);  // of no meaning behind the last
    const PageHeader* hdr = reinterpret_cast<const PageHeader*>(a.ws);
    if (!page_plan_is(*hdr, a.requests, a.hq, a.hkv, D, a.page_shift, a.max_pages, a.max_rows, a.max_new)) return;  // reported by page_team
    if (index >= hdr->tile_items) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int col = lane & 31, half = lane >> 5;

    const PageBlocks where(a, it, hk);
    const int nst = (it.blocks + BPS - 1) / BPS;
    const int my_block = wave >> 1, my_tile = (wave & 1) * KPW;  // of a stage
    const uint32_t lds_k_mine = lds_address(lds_k) + (my_block * KT + my_tile) * 1024, lds_v_mine = lds_address(lds_v) + (my_block * DT + my_tile) * 1024;
    int ids_k = 0, ids_v = 0;  // pages of the wave's blocks in stages st .. st + 63
    // A stage's loads go out in four parts, spread over the stage before: a wave that issues all at once stands still for 600 of a stage's 2500 cycles
    // (16 requests of 132 rows: 55 us so, 52 in parts; the packed prompts 185 and 179).
    const u16 *next_k = nullptr, *next_v = nullptr;
    uint32_t next_at = 0;
    auto request_part = [&](int part) {  // of the stage begun
#pragma unroll
        for (int i = 0; i < VPW + KPW; ++i) {
            if (i * 4 / (VPW + KPW) != part) continue;
            if (i < VPW) page_load_lds<false>(next_v + i * 512, lane * 16, lds_v_mine + next_at * (BPS * DT * 1024) + i * 1024);
            else page_load_lds<false>(next_k + (i - VPW) * 512, lane * 16, lds_k_mine + next_at * (BPS * KT * 1024) + (i - VPW) * 1024);
        }
    };
    auto begin = [&](int st) {
        if ((st & 63) == 0) {
            ids_k = where.id((st + lane) * BPS + my_block + 1);
            ids_v = where.id((st + lane) * BPS + my_block);
        }
        next_k = a.kc + where.place<D>(__builtin_amdgcn_readlane(ids_k, st & 63), st * BPS + my_block + 1) + my_tile * 512;
        next_v = a.vc + where.place<D>(__builtin_amdgcn_readlane(ids_v, st & 63), st * BPS + my_block) + my_tile * 512;
        next_at = st & 1;
    };
    auto request = [&](int st) {
        begin(st);
#pragma unroll
        for (int part = 0; part < 4; ++part) request_part(part);
    };
    if (nst > 0) {
        const int mine = wave * (KT / NW);  // block 0's keys are shared out among all four waves
        const u16* k = a.kc + where.place<D>(__builtin_amdgcn_readfirstlane(where.id(0)), 0) + mine * 512;
#pragma unroll
        for (int i = 0; i < KT / NW; ++i) page_load_lds<false>(k + i * 512, lane * 16, lds_address(lds_k) + ((2 * BPS - 1) * KT + mine + i) * 1024);
        request(0);
    }
    if (wave * 32 >= it.count) {  // a wave without rows only moves its part of the blocks
        if (nst > 0) {
            page_stage_landed<KPW + VPW>();
            for (int st = 0; st < nst; ++st) {
                page_stage_landed<0>();
                request(st + 1);
            }
            page_stage_landed<0>();
        }
        return;
    }
    Rows rows;
    rows.load(a, it, hk, wave * 32, lane);
    auto take_keys = [&](elem8 (&f)[KT], int st, int z) { Rows::take_keys(f, lds_k[st & 1] + z * KT * 64, lane); };
    auto take_values = [&](elem8 (&f)[C32][2], int st, int z) { Rows::take_values(f, lds_v[st & 1] + z * DT * 64, lane); };

    // Stages that every row of the workgroup sees whole come first.
    const int all_see = it.cached + min(it.first / (a.hq / a.hkv) + 1, it.trunk) - it.block0 * 32;
    const int whole = min(max(all_see, 0) / (32 * BPS), it.blocks / BPS);
    bool odd = false;
    if (nst > 0) {
        page_stage_landed<KPW + VPW>();  // the keys of block 0
        auto scores_of = [&](int st, int z) {
            elem8 kf[KT];
            take_keys(kf, st, z);
            return rows.scores(kf);
        };
        f32x16 s0 = scores_of(-1, 1);
        int st = 0;
#pragma unroll 1
        for (; st < whole; ++st) {
            page_stage_landed<0>();  // stage st is there, stage st - 1 drained
            begin(st + 1);
            elem8 kf[KT], vf[C32][2];
            Frag8 p[2];
            take_keys(kf, st, 0);
            take_values(vf, st, 0);
            request_part(0);
            const f32x16 s1 = rows.scores(kf);
            request_part(1);
            rows.template weigh<false, true>(s0, a.scale_log2, p, p);
            request_part(2);
            take_keys(kf, st, 1);
            rows.template add<false>(vf, p, p);
            take_values(vf, st, 1);
            request_part(3);
            s0 = rows.scores(kf);
            rows.template weigh<false, true>(s1, a.scale_log2, p, p);
            rows.template add<false>(vf, p, p);
        }
        // Then what some row does not see: for this wave, blocks that all of its rows see, blocks that some see in part, and the rest, of which it only
        // moves its share.  Three loops, since a branch around the products would have the outputs copied (to memory, at heads of 128).
        const int seen_whole = min(max(rows.whole / 32 - it.block0, whole * BPS), it.blocks), seen = min(max(rows.last / 32 + 1 - it.block0, seen_whole), it.blocks);
        int b = whole * BPS;
        auto enter = [&] {
            if (b % BPS == 0) {
                page_stage_landed<0>();
                request(b / BPS + 1);
            }
        };
#pragma unroll 1
        for (; b < seen_whole; ++b) {
            enter();
            Frag8 p[2];
            rows.template weigh<false, false>(s0, a.scale_log2, p, p);
            elem8 vf[C32][2];
            take_values(vf, b / BPS, b % BPS);
            rows.template add<false>(vf, p, p);
            s0 = scores_of(b / BPS, b % BPS);
        }
#pragma unroll 1
        for (; b < seen; ++b) {
            enter();
            int own = half;
            asm volatile("" : "+v"(own));  // keeps what follows from it inside the loop: kept in registers across it, it would push others to memory
            const int kb = (it.block0 + b) * 32;
            Frag8 p[2];
            rows.mask(s0, kb, own);
            rows.template weigh<false, false>(s0, a.scale_log2, p, p);
            elem8 vf[C32][2];
            take_values(vf, b / BPS, b % BPS);
            odd |= Rows::clean(vf, it.slots - kb, own);
            rows.template add<false>(vf, p, p);
            s0 = scores_of(b / BPS, b % BPS);
        }
        for (; b < nst * BPS; ++b) enter();
        page_stage_landed<0>();  // nothing is in flight to LDS when the workgroup ends
    }
    // Values that are not finite enter the products of blocks that all rows see as they are, and a weight that rounding made zero makes NaN of an
    // infinite one.  They leave outputs that are not finite: what the values seen come to replaces those.
    odd |= rows.not_finite_output();
    auto output = [&](int d) {
        f32x16 x = rows.o[d];
        if (__builtin_expect(odd, 0)) {
            f32x16 y = Rows::zero();
            for (int b = 0; b < it.blocks; ++b) {
                const int kb = (it.block0 + b) * 32, id = __builtin_amdgcn_readfirstlane(where.id(b));
                if (kb <= rows.last) rows.add_codes(y, d, a.vc + where.place<D>(id, b), kb, it.slots - kb, lane);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = y[i] == 0.f ? x[i] : y[i];
        }
        return x;
    };

    rows.l += __shfl_xor(rows.l, 32, 64);
    const float inv = 1.0f / rows.l;
    u16* const out = a.out + (size_t)(it.row0 + rows.token) * a.out_stride + (hk * (a.hq / a.hkv) + rows.gq) * D + half * 4;
    float* const part = a.part_tile + (((size_t)(it.part < 0 ? 0 : it.part) * a.hkv + hk) * PAGE_TILE_ROWS + wave * 32 + col) * (D + 4);
#pragma unroll
    for (int d = 0; d < C32; ++d) {
        const f32x16 x = output(d);  // its products need all lanes
        if (!rows.valid) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4 v = {x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
            if (it.part < 0) page_store4(out + d * 32 + q * 8, v * inv);
            else *reinterpret_cast<f32x4*>(part + d * 32 + q * 8 + half * 4) = v;
        }
    }
    if (!rows.valid) return;
    if (it.part >= 0 && half == 0) part[D] = rows.m, part[D + 1] = rows.l;
}

// A step that may hold requests of every kind: the tiles first, which take longest.  Requests of up to 16 rows go through the registers here too (64
// decoding requests beside a chunk of 512 rows: 138 us, 150 with teams for them); beside requests of 17 to 64 rows alone they do not, where both kinds
// wait for the cache's bytes (8 requests of 33 rows and 8 of 1 to 4: 85 us with teams for all, 93).
template <int D>
__global__ __launch_bounds__(256, 2) void page_mixed_kernel(PageAttnArgs a) {
    __shared__ union Lds {
        PageTileLds<D> tile;
        PageTeamLds<D, 2, 2> team;
        PageStreamLds<D, 4> stream;
        __device__ Lds() {}
    } lds;
    const int place = (int)blockIdx.x - a.tile_items * a.hkv;
    if (place < 0) {
        page_tile<D>(a, a.tile, blockIdx.x, lds.tile);
        return;
    }
    const int rows = __builtin_amdgcn_readfirstlane(reinterpret_cast<const PageItem*>(a.ws + a.stream)[place / a.hkv].count);  // of no meaning behind the last
    if (rows <= 16) page_stream<D, 4>(a, place, lds.stream);
    else page_team<D, 2, 2>(a, a.stream, place, lds.team);
}

// ---- tiles whose keys were cut: the ranges' partial results of a row are joined in their order
//
// Up to PAGE_MERGE_RANGES ranges: a wave takes whole rows, several at once, since what it waits for is its loads.  More: the workgroup's four
// waves take a quarter of the ranges each and the quarters are joined through LDS (a single row behind 131000 keys has 128 ranges: one wave would go
// through 16 dependent rounds of loads).  What bounds it is a launch and the latency of the header, an entry and the loads: 4 us with nothing to join,
// 5 us for 64 single rows in a few ranges each, 5.7 for 16 x 33 rows of 32 heads.
template <int E>
struct PageJoin {  // a running maximum, sum and output
    float top = -INFINITY, sum = 0.f, acc[E] = {};
    template <int N>
    __device__ __forceinline__ void add(const float (&mi)[N], const float (&li)[N], const float (&v)[N][E]) {  // li = 0 and mi = -inf: nothing
        float t = top;
#pragma unroll
        for (int i = 0; i < N; ++i) t = fmaxf(t, mi[i]);
        const float ref = t == -INFINITY ? 0.f : t;
        const float w0 = exp2f(top - ref);
        sum *= w0;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] *= w0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float w = exp2f(mi[i] - ref);
            sum += li[i] * w;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] += v[i][e] * w;
        }
        top = t;
    }
};

template <int D>
__global__ __launch_bounds__(256) void page_merge_kernel(PageAttnArgs a) {
    constexpr int E = D / 64, N = PAGE_MERGE_RANGES;
    __shared__ float lds_v[4][D], lds_ml[4][2];
    const PageMerge* const merges = reinterpret_cast<const PageMerge*>(a.ws + a.merge);
    PageMerge mg = merges[blockIdx.x / a.hkv];  // requested with the header; of no meaning behind the last
    const PageHeader hdr = *reinterpret_cast<const PageHeader*>(a.ws);
    if (!page_plan_is(hdr, a.requests, a.hq, a.hkv, D, a.page_shift, a.max_pages, a.max_rows, a.max_new)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, group = a.hq / a.hkv;
    const int units = hdr.merges * a.hkv;  // an entry (some rows of a tile), a head
    for (int unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const int index = unit / a.hkv, hk = unit - index * a.hkv;
        if (unit != (int)blockIdx.x) mg = merges[index];
        const int rows = mg.streamed ? a.stream_rows : PAGE_TILE_ROWS;
        const float* part = (mg.streamed ? a.part_stream : a.part_tile) + ((size_t)mg.part0 * a.hkv + hk) * rows * (D + 4);
        const size_t step = (size_t)a.hkv * rows * (D + 4);
        // ranges i0 .. i0 + M - 1 of a row, as far as they come before `last`: what lies behind is the last again, of no weight
        auto fetch = [&](auto& mi, auto& li, auto& v, int r, int i0, int last) {
            constexpr int M = sizeof(mi) / sizeof(float);
            const float* src = part + (size_t)(mg.in_tile + r) * (D + 4);
#pragma unroll
            for (int i = 0; i < M; ++i) {
                const float* p = src + step * min(i0 + i, last - 1);
                mi[i] = p[D], li[i] = p[D + 1];
#pragma unroll
                for (int e = 0; e < E; ++e) v[i][e] = p[lane + e * 64];
            }
#pragma unroll
            for (int i = 0; i < M; ++i) {
                const bool has = i0 + i < last;
                mi[i] = has ? mi[i] : -INFINITY, li[i] = has ? li[i] : 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) v[i][e] = has ? v[i][e] : 0.f;
            }
        };
        auto store = [&](const PageJoin<E>& x, int r) {
            const int pair = mg.first + r, token = pair / group, gq = pair - token * group;
            u16* dst = a.out + (size_t)(mg.row0 + token) * a.out_stride + (hk * group + gq) * D;
#pragma unroll
            for (int e = 0; e < E; ++e) dst[lane + e * 64] = (u16)pack_elem2(x.acc[e] / x.sum, 0.f);
        };
        // rows wave, wave + 4, ...: R of them at once, all their loads in flight together
        auto rows_at_once = [&](auto ranges, auto at_once) {
            constexpr int M = ranges, R = at_once;
#pragma unroll 1
            for (int r0 = wave; r0 < mg.count; r0 += 4 * R) {
                float mi[R][M], li[R][M], v[R][M][E];
#pragma unroll
                for (int i = 0; i < R; ++i) fetch(mi[i], li[i], v[i], min(r0 + 4 * i, mg.count - 1), 0, mg.parts);
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    PageJoin<E> x;
                    x.add(mi[i], li[i], v[i]);
                    if (r0 + 4 * i < mg.count) store(x, r0 + 4 * i);
                }
            }
        };
        if (mg.parts <= 2) {  // loads of ranges that are not there cost a chunk of 512 rows of 32 heads 1 us
            rows_at_once(std::integral_constant<int, 2>{}, std::integral_constant<int, 4>{});
            continue;
        }
        if (mg.parts <= N / 2) {
            rows_at_once(std::integral_constant<int, N / 2>{}, std::integral_constant<int, 4>{});
            continue;
        }
        if (mg.parts <= N) {
            rows_at_once(std::integral_constant<int, N>{}, std::integral_constant<int, 2>{});
            continue;
        }
        const int quarter = (mg.parts + 3) / 4;
        for (int r = 0; r < mg.count; ++r) {
            PageJoin<E> x;
            const int last = min((wave + 1) * quarter, mg.parts);
            for (int i0 = wave * quarter; i0 < last; i0 += N) {
                float mi[N], li[N], v[N][E];
                fetch(mi, li, v, r, i0, last);
                x.add(mi, li, v);
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; ++e) lds_v[wave][lane + e * 64] = x.acc[e];
            if (lane == 0) lds_ml[wave][0] = x.top, lds_ml[wave][1] = x.sum;
            __syncthreads();
            if (wave == (r & 3)) {
                PageJoin<E> all;
                float mi[4], li[4], v[4][E];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    mi[w] = lds_ml[w][0], li[w] = lds_ml[w][1];
#pragma unroll
                    for (int e = 0; e < E; ++e) v[w][e] = lds_v[w][lane + e * 64];
                }
                all.add(mi, li, v);
                store(all, r);
            }
        }
    }
}
