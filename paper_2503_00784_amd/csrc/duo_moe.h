// A layer of experts for the few rows of a verify step:
//   l = x R^T,  S = the top_k experts of a row by l,  g = softmax(l) on S,  y = sum over e in S of g_e * (silu(x G_e^T) * (x U_e^T)) D_e^T.
//
// With few rows the layer is the stream of the chosen experts' matrices, so every kernel is laid out around that stream: it is read once, in
// tiles, straight into the registers of the matrix units, and everything else (rows, lists, hidden values) comes out of the caches.
#pragma once
#include "duo_e4m3.h"

constexpr int MOE_MAX_EXPERTS = 512, MOE_MAX_TOP = 16, MOE_MAX_ROWS = 80;
constexpr int MOE_MASK_WORDS = 3;  // bits of 80 rows

struct MoeArgs {
    const u16* x;       // [rows][d]
    u16* y;             // [rows][d]
    const u16* router;  // [experts][d]
    const uint8_t* experts;  // gate, up and down matrix of every expert
    const int32_t* position; // [rows] or null: rows with a negative one are left out
    int32_t* chosen;    // [rows][top]
    float* share;       // [rows][top]
    double* logits;     // [rows][experts]
    int32_t* lists;     // see MoeLists
    u16* hidden;        // [rows * top][2][ff_pad]: bf16 pairs
    int64_t x_stride, y_stride;
    size_t expert_bytes, up_at, down_at;  // bytes of an expert, of what lies in front of its up and down matrices
    int rows, d, ff, ff_pad, n_experts, top, renormalise;
};

// The schedule in the workspace, as int32: active experts, their numbers, how many rows each has, which hidden row (row * top + place) a row has at
// an active expert (-1: none), and the rows of every active expert in ascending order.
struct MoeLists {
    int32_t* base;
    int most;  // active experts at most: the smaller of n_experts and rows * top
    __device__ __forceinline__ int& active() const { return base[0]; }
    __device__ __forceinline__ int& expert(int a) const { return base[4 + a]; }
    __device__ __forceinline__ int& count(int a) const { return base[4 + most + a]; }
    __device__ __forceinline__ int& hidden_of(int a, int row) const { return base[4 + 2 * most + a * MOE_MAX_ROWS + row]; }
    __device__ __forceinline__ int& entry(int a, int i) const { return base[4 + (2 + MOE_MAX_ROWS) * most + a * MOE_MAX_ROWS + i]; }
    static __host__ __device__ size_t words(int most) { return 4 + (size_t)most * (2 + 2 * MOE_MAX_ROWS); }
};
__host__ __device__ inline int moe_most(int experts, int rows, int top) { return experts < rows * top ? experts : rows * top; }

// ---- router: a wave per (expert, row), sums in 64 bits: which of two experts with nearly equal logits a row takes decides its whole output, and
// must not hang on the order of a sum.
__global__ __launch_bounds__(256) void moe_logits_kernel(MoeArgs a) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int e = blockIdx.x * 4 + wave, t = blockIdx.y;
    if (e >= a.n_experts || (a.position && a.position[t] < 0)) return;
    const u16* x = a.x + (int64_t)t * a.x_stride;
    const u16* r = a.router + (size_t)e * a.d;
    double sum = 0.0;
    for (int k = lane * 8; k < a.d; k += 512) {
        Frag8 u, v;
        u.q = *reinterpret_cast<const u32x4*>(x + k);
        v.q = *reinterpret_cast<const u32x4*>(r + k);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += (double)(elem_to_f32(u.h[i]) * elem_to_f32(v.h[i]));  // the fp32 product of two 16-bit values is exact
    }
    sum = wave_sum(sum);
    if (lane == 0) a.logits[(size_t)t * a.n_experts + e] = sum;
}

// One workgroup: every wave chooses for the rows wave, wave + 16, ...; then the lists.  NaN counts as the least of values; equal ones are taken in
// ascending order of the experts.
__global__ __launch_bounds__(1024) void moe_select_kernel(MoeArgs a) {
    __shared__ uint32_t rows_of[MOE_MAX_EXPERTS][MOE_MASK_WORDS];
    __shared__ uint32_t used[MOE_MAX_EXPERTS / 32];
    __shared__ int16_t chosen[MOE_MAX_ROWS * MOE_MAX_TOP];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    constexpr int PER = MOE_MAX_EXPERTS / 64;
    const double lowest = -__builtin_huge_val();
    for (int i = threadIdx.x; i < MOE_MAX_EXPERTS * MOE_MASK_WORDS; i += 1024) (&rows_of[0][0])[i] = 0u;
    if (threadIdx.x < MOE_MAX_EXPERTS / 32) used[threadIdx.x] = 0u;
    for (int i = threadIdx.x; i < a.rows * a.top; i += 1024) chosen[i] = -1;
    __syncthreads();
    for (int t = wave; t < a.rows; t += 16) {
        if (a.position && a.position[t] < 0) continue;
        const double* l = a.logits + (size_t)t * a.n_experts;
        double raw[PER], v[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = i * 64 + lane;
            raw[i] = e < a.n_experts ? l[e] : lowest;
            v[i] = raw[i] == raw[i] ? raw[i] : lowest;
        }
        uint32_t taken = 0u;
        double top_value = 0.0, mine = 0.0;  // mine: the logit of the expert that lane i < top holds
        for (int j = 0; j < a.top; ++j) {
            double best = lowest;
            int at = 0x7fffffff;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int e = i * 64 + lane;
                if (e < a.n_experts && !(taken >> i & 1u) && (v[i] > best || at == 0x7fffffff)) best = v[i], at = e;
            }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) {
                const double other = __shfl_xor(best, o, 64);
                const int oat = __shfl_xor(at, o, 64);
                if (oat != 0x7fffffff && (at == 0x7fffffff || other > best || (other == best && oat < at))) best = other, at = oat;
            }
            double value = 0.0;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (at == i * 64 + lane) taken |= 1u << i, value = raw[i];
            value = __shfl(value, at & 63, 64);
            if (j == 0) top_value = value;
            if (lane == j) mine = value;
            if (lane == 0) {
                chosen[t * a.top + j] = (int16_t)at;
                a.chosen[t * a.top + j] = at;
                atomicOr(&rows_of[at][t >> 5], 1u << (t & 31));
                atomicOr(&used[at >> 5], 1u << (at & 31));
            }
        }
        const double p = lane < a.top ? exp(mine - top_value) : 0.0;
        double sum = p;
        if (!a.renormalise) {
            sum = 0.0;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (i * 64 + lane < a.n_experts) sum += exp(raw[i] - top_value);
        }
        sum = wave_sum(sum);
        if (lane < a.top) a.share[t * a.top + lane] = (float)(p / sum);
    }
    __syncthreads();
    const MoeLists lists{a.lists, moe_most(a.n_experts, a.rows, a.top)};
    auto place_of = [&](int e) {  // among the active experts
        int n = __popc(used[e >> 5] & ((1u << (e & 31)) - 1u));
        for (int w = 0; w < e >> 5; ++w) n += __popc(used[w]);
        return n;
    };
    if (threadIdx.x < a.n_experts) {
        const int e = threadIdx.x;
        if (used[e >> 5] >> (e & 31) & 1u) {
            const int at = place_of(e);
            lists.expert(at) = e;
            lists.count(at) = __popc(rows_of[e][0]) + __popc(rows_of[e][1]) + __popc(rows_of[e][2]);
        }
    }
    if (threadIdx.x == 0) {
        int n = 0;
        for (int w = 0; w < MOE_MAX_EXPERTS / 32; ++w) n += __popc(used[w]);
        lists.active() = n;
    }
    for (int i = threadIdx.x; i < a.n_experts * MOE_MAX_ROWS; i += 1024) {  // rows without the expert
        const int e = i / MOE_MAX_ROWS, t = i % MOE_MAX_ROWS;
        if ((used[e >> 5] >> (e & 31) & 1u) && !(rows_of[e][t >> 5] >> (t & 31) & 1u)) lists.hidden_of(place_of(e), t) = -1;
    }
    for (int i = threadIdx.x; i < a.rows * a.top; i += 1024) {
        const int e = chosen[i], t = i / a.top;
        if (e < 0) continue;
        const int at = place_of(e);
        int n = __popc(rows_of[e][t >> 5] & ((1u << (t & 31)) - 1u));
        for (int w = 0; w < t >> 5; ++w) n += __popc(rows_of[e][w]);
        lists.hidden_of(at, t) = i;
        lists.entry(at, n) = i;
    }
}

// A band's tiles of 128 columns as operands, from a matrix in 16 bits (tiles of 16 x 32, the library's streaming layout) or in e4m3 with block
// scales.  column(i, g): the first of the eight columns of the block that a lane of group g holds in operand i.
struct Wide {  // 16 bits
    static constexpr bool SCALED = false;
    u32x4 v[4];
    static __host__ __device__ size_t bytes(int N, int K) { return (size_t)((N + 31) / 32) * 32 * K * 2; }
    static __device__ __forceinline__ int column(int i, int g) { return 32 * i + 8 * g; }
    __device__ __forceinline__ void load(const uint8_t* m, int, int K, int band, int j, int lane) {
        const u32x4* p = reinterpret_cast<const u32x4*>(m) + ((size_t)band * (K >> 5) + 4 * j) * 64 + lane;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = 4 * j + i < K >> 5 ? __builtin_nontemporal_load(p + i * 64) : u32x4{0u, 0u, 0u, 0u};
    }
    __device__ __forceinline__ elem8 operand(int i) const { return __builtin_bit_cast(elem8, v[i]); }
    __device__ __forceinline__ float scale() const { return 1.f; }
};
struct Narrow {  // e4m3; the block's scale is applied to the sums of its products
    static constexpr bool SCALED = true;
    u32x4 v[2];
    int byte;
    static __host__ __device__ size_t bytes(int N, int K) { return scaled_bytes(N, K); }
    static __device__ __forceinline__ int column(int i, int g) { return 64 * (i >> 1) + 16 * g + 8 * (i & 1); }
    __device__ __forceinline__ void load(const uint8_t* m, int N, int K, int band, int j, int lane) {
        const int KB = scaled_blocks(K);
        const u32x4* p = reinterpret_cast<const u32x4*>(m + ((size_t)band * KB + j) * SCALED_TILE) + lane;
        v[0] = __builtin_nontemporal_load(p);
        v[1] = __builtin_nontemporal_load(p + 64);
        byte = m[scaled_tile_bytes(N, K) + (size_t)(band >> 3) * KB + j];
    }
    __device__ __forceinline__ uint32_t word(int i, int n) const { return v[i >> 1][2 * (i & 1) + n]; }
    __device__ __forceinline__ elem8 operand(int i) const {  // e4m3 values without their scale: exact in either 16-bit type
#ifdef DUO_FP16
        union {
            f16x2 p[4];
            elem8 v;
        } f;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            f.p[2 * n] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word(i, n), 1.0f, false);
            f.p[2 * n + 1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word(i, n), 1.0f, true);
        }
        return f.v;
#else
        return e4m3_to_bf16(word(i, 0), word(i, 1), 1.0f);
#endif
    }
    __device__ __forceinline__ float scale() const { return scale_of(byte); }
};

// ---- gate and up.  A workgroup owns 16 hidden channels of one active expert: a band of its gate and one of its up matrix, which its waves read in
// turns of 128 columns; the sums of the waves are added through LDS in wave order.  Hidden values are left as bf16 pairs hi + lo (16 bits of
// mantissa, fp32's range in either build), with the row's share of the expert in them.
template <class W, int MT, int NW>
__global__ __launch_bounds__(64 * NW) void moe_gate_up_kernel(MoeArgs a) {
    __shared__ f32x4 part[NW][2 * MT][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const MoeLists lists{a.lists, moe_most(a.n_experts, a.rows, a.top)};
    const int at = blockIdx.y, band = blockIdx.x;
    if (at >= lists.active()) return;
    const uint8_t* gate = a.experts + (size_t)lists.expert(at) * a.expert_bytes;
    const uint8_t* up = gate + a.up_at;
    const int count = lists.count(at), KB = scaled_blocks(a.d);
    for (int first = 0; first < count; first += 16 * MT) {
        const u16* row[MT];
        int entry[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int i = first + m * 16 + c;
            entry[m] = i < count ? lists.entry(at, i) : -1;
            row[m] = i < count ? a.x + (int64_t)(entry[m] / a.top) * a.x_stride : nullptr;
        }
        f32x4 acc[2][MT];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[b][m] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int j = wave; j < KB; j += NW) {
            W w[2];
            w[0].load(gate, a.ff, a.d, band, j, lane);
            w[1].load(up, a.ff, a.d, band, j, lane);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                f32x4 sum[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int k = j * 128 + W::column(i, g);
                    Frag8 x;
                    x.q = row[m] && k < a.d ? *reinterpret_cast<const u32x4*>(row[m] + k) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
                    for (int b = 0; b < 2; ++b) sum[b] = mfma16(w[b].operand(i), x.v, sum[b]);
                }
#pragma unroll
                for (int b = 0; b < 2; ++b) acc[b][m] += sum[b] * w[b].scale();
            }
        }
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int m = 0; m < MT; ++m) part[wave][b * MT + m][lane] = acc[b][m];
        __syncthreads();
        for (int m = wave; m < MT; m += NW) {
            f32x4 s = part[0][m][lane], u = part[0][MT + m][lane];
            for (int w = 1; w < NW; ++w) s += part[w][m][lane], u += part[w][MT + m][lane];
            const int i = first + m * 16 + c;
            if (i < count) {
                const int p = lists.entry(at, i);
                const float share = a.share[p];
                u16 hi[4], lo[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float h = s[q] / (1.0f + expf(-s[q])) * u[q] * share;
                    const __bf16 b = (__bf16)h;
                    hi[q] = __builtin_bit_cast(u16, b);
                    lo[q] = __builtin_bit_cast(u16, (__bf16)(h - (float)b));
                }
                u16* dst = a.hidden + (size_t)p * 2 * a.ff_pad + band * 16 + 4 * g;
                *reinterpret_cast<uint2*>(dst) = make_uint2(hi[0] | (uint32_t)hi[1] << 16, hi[2] | (uint32_t)hi[3] << 16);
                *reinterpret_cast<uint2*>(dst + a.ff_pad) = make_uint2(lo[0] | (uint32_t)lo[1] << 16, lo[2] | (uint32_t)lo[3] << 16);
            }
        }
        __syncthreads();
    }
}

// operand i of a down matrix as bf16: as it is, or, where the 16-bit type is fp16, as the sum of two (8 + 3 bits of mantissa)
template <class W>
struct DownOperand {
    static constexpr int PARTS =
#ifdef DUO_FP16
        W::SCALED ? 1 : 2;
#else
        1;
#endif
    bf16x8 v[PARTS];
    __device__ __forceinline__ explicit DownOperand(const W& w, int i) {
        if constexpr (W::SCALED) v[0] = e4m3_to_bf16(w.word(i, 0), w.word(i, 1), 1.0f);
        else if constexpr (PARTS == 1) v[0] = __builtin_bit_cast(bf16x8, w.v[i]);
        else {
            Frag8 f;
            f.q = w.v[i];
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                const float x = elem_to_f32(f.h[n]);
                v[0][n] = (__bf16)x;
                v[PARTS - 1][n] = (__bf16)(x - (float)v[0][n]);
            }
        }
    }
};

// ---- down.  A workgroup owns 16 output channels of all rows; its waves take (active expert, 128 hidden channels) in turn.  The columns of the
// product are the step's rows, with zeros where a row did not choose the expert, so that all experts add into the same sums and every output is
// formed in one place.
template <class W, int MT, int NW>
__global__ __launch_bounds__(64 * NW) void moe_down_kernel(MoeArgs a) {
    __shared__ f32x4 part[NW][MT][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const MoeLists lists{a.lists, moe_most(a.n_experts, a.rows, a.top)};
    const int band = blockIdx.x, KB = scaled_blocks(a.ff), items = lists.active() * KB;
    f32x4 acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int item = wave; item < items; item += NW) {
        const int at = item / KB, j = item - at * KB;
        W w;
        w.load(a.experts + (size_t)lists.expert(at) * a.expert_bytes + a.down_at, a.d, a.ff, band, j, lane);
        const float scale = w.scale();
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int t = m * 16 + c, p = t < a.rows ? lists.hidden_of(at, t) : -1;
            if (!__any(p >= 0)) continue;  // no row of this tile: the same for every lane
            const u16* h = a.hidden + (size_t)(p < 0 ? 0 : p) * 2 * a.ff_pad;
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = j * 128 + W::column(i, g);
                const bool in = p >= 0 && k < a.ff;
                Bf16Frag hi, lo;
                hi.q = in ? *reinterpret_cast<const u32x4*>(h + k) : u32x4{0u, 0u, 0u, 0u};
                lo.q = in ? *reinterpret_cast<const u32x4*>(h + a.ff_pad + k) : u32x4{0u, 0u, 0u, 0u};
                const DownOperand<W> o(w, i);
                sum = mfma_bf16(o.v[0], hi.v, sum);
                sum = mfma_bf16(o.v[0], lo.v, sum);
                if constexpr (o.PARTS == 2) sum = mfma_bf16(o.v[o.PARTS - 1], hi.v, sum);
            }
            acc[m] += sum * scale;
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) part[wave][m][lane] = acc[m];
    __syncthreads();
    for (int m = wave; m < MT; m += NW) {
        f32x4 v = part[0][m][lane];
        for (int w = 1; w < NW; ++w) v += part[w][m][lane];
        const int t = m * 16 + c;
        if (t < a.rows && !(a.position && a.position[t] < 0)) {
            u16* y = a.y + (int64_t)t * a.y_stride + band * 16 + 4 * g;
            *reinterpret_cast<uint2*>(y) = make_uint2(pack_elem2(v[0], v[1]), pack_elem2(v[2], v[3]));
        }
    }
}
