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
    const uint8_t* experts;   // gate, up and down matrix of every expert
    const int32_t* position;  // [rows] or null: rows with a negative one are left out
    int32_t* chosen_out;      // [rows][top], or null
    float* share_out;
    // workspace
    int32_t* chosen;    // [rows][top], -1 where a row is left out
    float* share;       // [rows][top]
    double* logits;     // [rows][experts], where a kernel of its own forms them
    u16* packed;        // [rows][d_pad]: x, zeros behind d
    u16* hidden;        // [rows * top][2][ff_pad]: bf16 pairs, zeros behind ff
    float* partial;     // [rows * top][d]: outputs in front of the sum over a row's experts
    int64_t x_stride, y_stride;
    size_t expert_bytes, up_at, down_at;  // bytes of an expert, of what lies in front of its up and down matrices
    int rows, d, d_pad, ff, ff_pad, n_experts, top, renormalise;
};

// ---- router.  Logits in 64 bits: which of two experts with nearly equal logits a row takes decides its whole output, and must not hang on the order
// of a sum.  A wave forms those of four experts for one row: 64 lanes x 8 columns at a time, then a butterfly over the lanes.
__device__ __forceinline__ void router_logits(const MoeArgs& a, const u16* x, int e0, int lane, double (&sum)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = 0.0;
    const u16* r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = a.router + (size_t)min(e0 + i, a.n_experts - 1) * a.d;
    for (int k = lane * 8; k < a.d; k += 512) {
        Frag8 u, v[4];
        u.q = *reinterpret_cast<const u32x4*>(x + k);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i].q = *reinterpret_cast<const u32x4*>(r[i] + k);
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const double f = (double)elem_to_f32(u.h[n]);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = fma(f, (double)elem_to_f32(v[i].h[n]), sum[i]);
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor(sum[i], o, 64);
}

__global__ __launch_bounds__(256) void moe_logits_kernel(MoeArgs a) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int e0 = (blockIdx.x * 4 + wave) * 4, t = blockIdx.y;
    if (e0 >= a.n_experts || (a.position && a.position[t] < 0)) return;
    double sum[4];
    router_logits(a, a.x + (int64_t)t * a.x_stride, e0, lane, sum);
    if (lane == 0)
        for (int i = 0; i < 4 && e0 + i < a.n_experts; ++i) a.logits[(size_t)t * a.n_experts + e0 + i] = sum[i];
}

// One workgroup a row: logits (INSIDE: formed here), the rank of every expert, which is the number of experts in front of it (so that all are found
// at once: no search of top_k rounds), shares, and the row's copy for the products.  NaN counts as the least of values; equal ones rank by their number.
template <bool INSIDE>
__global__ __launch_bounds__(1024) void moe_router_kernel(MoeArgs a) {
    __shared__ double raw[MOE_MAX_EXPERTS], key[MOE_MAX_EXPERTS];
    __shared__ int rank[MOE_MAX_EXPERTS], order[MOE_MAX_TOP];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, t = blockIdx.x, n = a.n_experts;
    if (a.position && a.position[t] < 0) {
        if (tid < a.top) a.chosen[t * a.top + tid] = -1;
        return;
    }
    const u16* x = a.x + (int64_t)t * a.x_stride;
    for (int k = tid * 8; k < a.d_pad; k += 8192)
        *reinterpret_cast<u32x4*>(a.packed + (size_t)t * a.d_pad + k) = k < a.d ? *reinterpret_cast<const u32x4*>(x + k) : u32x4{0u, 0u, 0u, 0u};
    const double lowest = -__builtin_huge_val();
    if constexpr (INSIDE) {
        for (int e0 = 4 * wave; e0 < n; e0 += 64) {
            double sum[4];
            router_logits(a, x, e0, lane, sum);
            if (lane == 0)
                for (int i = 0; i < 4 && e0 + i < n; ++i) raw[e0 + i] = sum[i], key[e0 + i] = sum[i] == sum[i] ? sum[i] : lowest;
        }
    } else if (tid < n) {
        const double l = a.logits[(size_t)t * n + tid];
        raw[tid] = l, key[tid] = l == l ? l : lowest;
    }
    if (tid < MOE_MAX_EXPERTS) rank[tid] = 0;
    __syncthreads();
    // thread (e, part): the experts of a part of the list that stand in front of e
    int width = 32;
    while (width < n) width *= 2;
    const int e = tid & (width - 1), parts = 1024 / width, each = (n + parts - 1) / parts, first = tid / width * each, last = min(first + each, n);
    if (e < n) {
        const double mine = key[e];
        int ahead = 0;
        for (int j = first; j < last; ++j) ahead += key[j] > mine || (key[j] == mine && j < e);
        if (ahead) atomicAdd(&rank[e], ahead);
    }
    __syncthreads();
    if (tid < n && rank[tid] < a.top) order[rank[tid]] = tid;
    __syncthreads();
    if (wave != 0) return;
    const double most = raw[order[0]];
    const int mine = lane < a.top ? order[lane] : 0;
    const double p = lane < a.top ? exp(raw[mine] - most) : 0.0;
    double sum = p;
    if (!a.renormalise) {
        sum = 0.0;
        for (int i = lane; i < n; i += 64) sum += exp(raw[i] - most);
    }
    sum = wave_sum(sum);
    if (lane < a.top) {
        const int at = t * a.top + lane;
        const float share = (float)(p / sum);
        a.chosen[at] = mine, a.share[at] = share;
        if (a.chosen_out) a.chosen_out[at] = mine;
        if (a.share_out) a.share_out[at] = share;
    }
}

// The rows of the workgroup's expert: number `at` among those that a row has chosen, in ascending order; -1 if there are fewer.  Every workgroup finds
// them for itself from the list of choices, at most 1280 words out of the caches: cheaper than a launch between the router and the products.
struct ExpertRows {
    uint32_t used[MOE_MAX_EXPERTS / 32], mask[MOE_MASK_WORDS];
    int16_t entry[MOE_MAX_ROWS];  // row * top + place, in ascending order
};
template <int THREADS>
__device__ __forceinline__ int find_expert(const MoeArgs& a, ExpertRows& r, int at, int& count) {
    constexpr int EACH = (MOE_MAX_ROWS * MOE_MAX_TOP + THREADS - 1) / THREADS;
    const int tid = threadIdx.x, entries = a.rows * a.top;
    int chosen[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) chosen[i] = i * THREADS + tid < entries ? a.chosen[i * THREADS + tid] : -1;
    for (int i = tid; i < MOE_MAX_EXPERTS / 32 + MOE_MASK_WORDS; i += THREADS) (i < MOE_MAX_EXPERTS / 32 ? r.used[i] : r.mask[i - MOE_MAX_EXPERTS / 32]) = 0u;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (chosen[i] >= 0) atomicOr(&r.used[chosen[i] >> 5], 1u << (chosen[i] & 31));
    __syncthreads();
    int e = -1, left = at;
    for (int w = 0; w < MOE_MAX_EXPERTS / 32; ++w) {
        uint32_t bits = r.used[w];
        const int here = __popc(bits);
        if (left < here && e < 0) {
            for (int i = 0; i < left; ++i) bits &= bits - 1u;
            e = 32 * w + __ffs(bits) - 1;
        }
        left -= here;
    }
    e = __builtin_amdgcn_readfirstlane(e);
    if (e < 0) return -1;
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (chosen[i] == e) {
            const int t = (i * THREADS + tid) / a.top;
            atomicOr(&r.mask[t >> 5], 1u << (t & 31));
        }
    __syncthreads();
    count = __builtin_amdgcn_readfirstlane(__popc(r.mask[0]) + __popc(r.mask[1]) + __popc(r.mask[2]));
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (chosen[i] == e) {
            const int t = (i * THREADS + tid) / a.top;
            int n = __popc(r.mask[t >> 5] & ((1u << (t & 31)) - 1u));
            for (int w = 0; w < t >> 5; ++w) n += __popc(r.mask[w]);
            r.entry[n] = (int16_t)(i * THREADS + tid);
        }
    __syncthreads();
    return e;
}

// Rows are read through buffer descriptors: lanes without a row ask for an offset behind the end and get zeros without a memory access, and the
// loop has no branch around its loads, so that the compiler can count them.  Offsets stay below 2^31 (80 rows x 16 experts x 65536 channels x 4
// bytes are 2^28.4).
constexpr uint32_t NO_ROW = 0x80000000u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_buffer(const void* p, size_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (uint32_t)bytes, 0x00027000);
}
__device__ __forceinline__ u32x4 row_load(__amdgpu_buffer_rsrc_t r, uint32_t offset) { return __builtin_amdgcn_raw_buffer_load_b128(r, (int)offset, 0, 0); }

// A band's tiles of 128 columns as operands, from a matrix in 16 bits (tiles of 16 x 32, the library's streaming layout) or in e4m3 with block
// scales.  column(i, g): the first of the eight columns of the block that a lane of group g holds in operand i.
struct Wide {  // 16 bits
    static constexpr bool SCALED = false;
    u32x4 v[4];
    static __host__ __device__ size_t bytes(int N, int K) { return (size_t)((N + 31) / 32) * 32 * K * 2; }
    static __device__ __forceinline__ int column(int i, int g) { return 32 * i + 8 * g; }
    __device__ __forceinline__ void load(const uint8_t* m, int, int K, int band, int j, int lane) {
        const u32x4* p = reinterpret_cast<const u32x4*>(m) + (size_t)band * (K >> 5) * 64 + lane;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_nontemporal_load(p + min(4 * j + i, (K >> 5) - 1) * 64);
    }
    // zeros in the columns from K on, which `load` does not read
    __device__ __forceinline__ void cut(int K, int j) {
#pragma unroll
        for (int i = 1; i < 4; ++i)
            if (4 * j + i >= K >> 5) v[i] = u32x4{0u, 0u, 0u, 0u};
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
    __device__ __forceinline__ void cut(int, int) {}
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

// sum += (or, with block scales, sum += scale *) what the four operands of a block give
template <class W>
__device__ __forceinline__ void add_block(f32x4& sum, const f32x4& block, const W& w) {
    if constexpr (W::SCALED) {
        const float s = w.scale();
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = fmaf(block[i], s, sum[i]);
    } else sum = block;
}

// ---- gate and up.  A workgroup owns 16 hidden channels of one expert: a band of its gate and one of its up matrix, which its waves read in turns of
// 128 columns, PF of them on their way at any time; the sums of the waves are added through LDS in wave order.  The columns of the product are the
// rows that chose the expert, 16 MT at a time.  Hidden values are left as bf16 pairs hi + lo (16 bits of mantissa, fp32's range in either build),
// with the row's share of the expert in them.
template <class W, int MT, int NW, int PF>
__global__ __launch_bounds__(64 * NW) void moe_gate_up_kernel(MoeArgs a) {
    __shared__ f32x4 part[NW][2 * MT][64];
    __shared__ ExpertRows rows;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int band = blockIdx.x, KB = a.d_pad >> 7, n = (KB - wave + NW - 1) / NW;
    int count = 0;
    const int e = find_expert<64 * NW>(a, rows, blockIdx.y, count);
    if (e < 0) return;
    const uint8_t* gate = a.experts + (size_t)e * a.expert_bytes;
    const uint8_t* up = gate + a.up_at;
    const __amdgpu_buffer_rsrc_t xs = row_buffer(a.packed, (size_t)a.rows * a.d_pad * 2);
    for (int first = 0; first < count; first += 16 * MT) {
        uint32_t row[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int i = first + m * 16 + c;
            row[m] = i < count ? (uint32_t)(rows.entry[i] / a.top) * a.d_pad * 2 : NO_ROW;
        }
        f32x4 acc[2][MT];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[b][m] = f32x4{0.f, 0.f, 0.f, 0.f};
        W w[PF][2];
        u32x4 x[PF][MT][4];
        auto load = [&](int s, int i) {
            const int j = max(min(wave + NW * min(i, n - 1), KB - 1), 0);
            w[s][0].load(gate, a.ff, a.d, band, j, lane);
            w[s][1].load(up, a.ff, a.d, band, j, lane);
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) x[s][m][q] = row_load(xs, row[m] + (uint32_t)(j * 128 + W::column(q, g)) * 2);
        };
        auto products = [&](int s, int i) {
            const int j = wave + NW * i;
            if ((j + 1) * 128 > a.d) w[s][0].cut(a.d, j), w[s][1].cut(a.d, j);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                elem8 o[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) o[q] = w[s][b].operand(q);
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    if (first + m * 16 < count) {  // the same for every lane
                        f32x4 sum = W::SCALED ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[b][m];
#pragma unroll
                        for (int q = 0; q < 4; ++q) sum = mfma16(o[q], __builtin_bit_cast(elem8, x[s][m][q]), sum);
                        add_block(acc[b][m], sum, w[s][b]);
                    }
            }
        };
#pragma unroll
        for (int s = 0; s < PF; ++s) load(s, s);
        int i = 0;
        for (; i + PF < n; i += PF) {
#pragma unroll
            for (int s = 0; s < PF; ++s) {
                products(s, i + s);
                load(s, i + s + PF);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int s = 0; s < PF; ++s)
            if (i + s < n) products(s, i + s);
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int m = 0; m < MT; ++m) part[wave][b * MT + m][lane] = acc[b][m];
        __syncthreads();
        for (int m = wave; m < MT; m += NW) {
            f32x4 s = part[0][m][lane], u = part[0][MT + m][lane];
            for (int v = 1; v < NW; ++v) s += part[v][m][lane], u += part[v][MT + m][lane];
            const int at = first + m * 16 + c;
            if (at < count) {
                const int p = rows.entry[at];
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
                if (band == gridDim.x - 1)  // zeros up to the end of the last block
                    for (int k = a.ff + 4 * g; k < a.ff_pad; k += 16)
                        *reinterpret_cast<uint2*>(a.hidden + (size_t)p * 2 * a.ff_pad + k) = *reinterpret_cast<uint2*>(a.hidden + ((size_t)p * 2 + 1) * a.ff_pad + k) = make_uint2(0u, 0u);
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

// sum += a block of a down matrix times hidden pairs (hi in x[0 .. 3], lo in x[4 .. 7])
template <class W>
__device__ __forceinline__ void down_block(f32x4& acc, const W& w, const DownOperand<W> (&o)[4], const u32x4 (&x)[8]) {
    f32x4 sum = W::SCALED ? f32x4{0.f, 0.f, 0.f, 0.f} : acc;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const bf16x8 hi = __builtin_bit_cast(bf16x8, x[q]), lo = __builtin_bit_cast(bf16x8, x[4 + q]);
        sum = mfma_bf16(o[q].v[0], hi, sum);
        sum = mfma_bf16(o[q].v[0], lo, sum);
        if constexpr (DownOperand<W>::PARTS == 2) sum = mfma_bf16(o[q].v[DownOperand<W>::PARTS - 1], hi, sum);
    }
    add_block(acc, sum, w);
}

// ---- down, up to 16 rows.  A workgroup owns 16 output channels of all rows; its waves share out (expert, 128 hidden channels) in runs.  The columns
// of the product are the step's rows, with zeros where a row did not choose the expert, so that all experts add into the same sums and an output is
// formed in one place.
constexpr int MOE_FEW_ROWS = 16;
template <class W, int NW, int PF>
__global__ __launch_bounds__(64 * NW) void moe_down_few_kernel(MoeArgs a) {
    __shared__ f32x4 part[NW][64];
    __shared__ uint32_t used[MOE_MAX_EXPERTS / 32];
    __shared__ int16_t expert[MOE_FEW_ROWS * MOE_MAX_TOP], entry[MOE_FEW_ROWS * MOE_MAX_TOP][MOE_FEW_ROWS];  // of the active experts; -1: not chosen
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4, tid = threadIdx.x;
    const int band = blockIdx.x, KB = a.ff_pad >> 7, entries = a.rows * a.top;  // at most 256 entries
    static_assert(64 * NW >= MOE_FEW_ROWS * MOE_MAX_TOP, "a thread per entry");
    const int mine = tid < entries ? a.chosen[tid] : -1;
    if (tid < MOE_MAX_EXPERTS / 32) used[tid] = 0u;
    for (int i = tid; i < entries * MOE_FEW_ROWS; i += 64 * NW) (&entry[0][0])[i] = -1;
    __syncthreads();
    if (mine >= 0) atomicOr(&used[mine >> 5], 1u << (mine & 31));
    __syncthreads();
    int active = 0, at = 0;
    for (int w = 0; w < MOE_MAX_EXPERTS / 32; ++w) {
        if (w == mine >> 5) at = active + __popc(used[w] & ((1u << (mine & 31)) - 1u));
        active += __popc(used[w]);
    }
    if (mine >= 0) expert[at] = (int16_t)mine, entry[at][tid / a.top] = (int16_t)tid;
    __syncthreads();
    active = __builtin_amdgcn_readfirstlane(active);
    const int items = active * KB, begin = wave * items / NW, end = (wave + 1) * items / NW;  // at most 256 * 512 items
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (begin < end) {
        const __amdgpu_buffer_rsrc_t hs = row_buffer(a.hidden, (size_t)entries * a.ff_pad * 4);
        int to_load = begin, la = begin / KB, lj = begin - la * KB, ci = begin - la * KB;  // ci: the block of columns of the next item to compute
        W w[PF];
        u32x4 x[PF][8];
        auto load = [&](int s) {
            const int e = __builtin_amdgcn_readfirstlane(expert[la]), p = entry[la][c];
            const uint32_t row = p < 0 ? NO_ROW : (uint32_t)p * a.ff_pad * 4;
            w[s].load(a.experts + (size_t)e * a.expert_bytes + a.down_at, a.d, a.ff, band, lj, lane);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t k = (uint32_t)(lj * 128 + W::column(q, g)) * 2;
                x[s][q] = row_load(hs, row + k);
                x[s][4 + q] = row_load(hs, row + (uint32_t)a.ff_pad * 2 + k);
            }
            if (to_load + 1 < end) {  // the last one again where there is none
                ++to_load;
                if (++lj == KB) lj = 0, ++la;
            }
        };
        auto products = [&](int s) {
            if ((ci + 1) * 128 > a.ff) w[s].cut(a.ff, ci);
            if (++ci == KB) ci = 0;
            const DownOperand<W> o[4] = {DownOperand<W>(w[s], 0), DownOperand<W>(w[s], 1), DownOperand<W>(w[s], 2), DownOperand<W>(w[s], 3)};
            down_block(acc, w[s], o, x[s]);
        };
#pragma unroll
        for (int s = 0; s < PF; ++s) load(s);
        int i = begin;
        for (; i + PF < end; i += PF) {
#pragma unroll
            for (int s = 0; s < PF; ++s) {
                products(s);
                load(s);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int s = 0; s < PF; ++s)
            if (i + s < end) products(s);
    }
    part[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
        f32x4 v = part[0][lane];
        for (int w = 1; w < NW; ++w) v += part[w][lane];
        if (c < a.rows && !(a.position && a.position[c] < 0)) {
            u16* y = a.y + (int64_t)c * a.y_stride + band * 16 + 4 * g;
            *reinterpret_cast<uint2*>(y) = make_uint2(pack_elem2(v[0], v[1]), pack_elem2(v[2], v[3]));
        }
    }
}

// ---- down, more rows.  As gate and up: a workgroup owns NB bands of one expert, the columns are the rows that chose it; what a row gets from each of
// its experts is left apart in fp32 and added up by moe_combine_kernel in the order of its choices.
template <class W, int MT, int NB, int NW, int PF>
__global__ __launch_bounds__(64 * NW) void moe_down_kernel(MoeArgs a) {
    __shared__ f32x4 part[NW][NB * MT][64];
    __shared__ ExpertRows rows;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int band0 = blockIdx.x * NB, KB = a.ff_pad >> 7, n = (KB - wave + NW - 1) / NW;  // d is a multiple of 64: NB divides its bands
    int count = 0;
    const int e = find_expert<64 * NW>(a, rows, blockIdx.y, count);
    if (e < 0) return;
    const uint8_t* down = a.experts + (size_t)e * a.expert_bytes + a.down_at;
    const __amdgpu_buffer_rsrc_t hs = row_buffer(a.hidden, (size_t)a.rows * a.top * a.ff_pad * 4);
    for (int first = 0; first < count; first += 16 * MT) {
        uint32_t row[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int i = first + m * 16 + c;
            row[m] = i < count ? (uint32_t)rows.entry[i] * a.ff_pad * 4 : NO_ROW;
        }
        f32x4 acc[NB][MT];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[b][m] = f32x4{0.f, 0.f, 0.f, 0.f};
        W w[PF][NB];
        u32x4 x[PF][MT][8];
        auto load = [&](int s, int i) {
            const int j = max(min(wave + NW * min(i, n - 1), KB - 1), 0);
#pragma unroll
            for (int b = 0; b < NB; ++b) w[s][b].load(down, a.d, a.ff, band0 + b, j, lane);
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t k = (uint32_t)(j * 128 + W::column(q, g)) * 2;
                    x[s][m][q] = row_load(hs, row[m] + k);
                    x[s][m][4 + q] = row_load(hs, row[m] + (uint32_t)a.ff_pad * 2 + k);
                }
        };
        auto products = [&](int s, int i) {
            const int j = wave + NW * i;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if ((j + 1) * 128 > a.ff) w[s][b].cut(a.ff, j);
                const DownOperand<W> o[4] = {DownOperand<W>(w[s][b], 0), DownOperand<W>(w[s][b], 1), DownOperand<W>(w[s][b], 2), DownOperand<W>(w[s][b], 3)};
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    if (first + m * 16 < count) down_block(acc[b][m], w[s][b], o, x[s][m]);  // the same for every lane
            }
        };
#pragma unroll
        for (int s = 0; s < PF; ++s) load(s, s);
        int i = 0;
        for (; i + PF < n; i += PF) {
#pragma unroll
            for (int s = 0; s < PF; ++s) {
                products(s, i + s);
                load(s, i + s + PF);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int s = 0; s < PF; ++s)
            if (i + s < n) products(s, i + s);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int m = 0; m < MT; ++m) part[wave][b * MT + m][lane] = acc[b][m];
        __syncthreads();
        for (int t = wave; t < NB * MT; t += NW) {
            f32x4 v = part[0][t][lane];
            for (int u = 1; u < NW; ++u) v += part[u][t][lane];
            const int at = first + (t % MT) * 16 + c;
            if (at < count) *reinterpret_cast<f32x4*>(a.partial + (size_t)rows.entry[at] * a.d + (band0 + t / MT) * 16 + 4 * g) = v;
        }
        __syncthreads();
    }
}

// a thread: four outputs of a row
__global__ __launch_bounds__(256) void moe_combine_kernel(MoeArgs a) {
    const int t = blockIdx.y, k = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (k >= a.d || (a.position && a.position[t] < 0)) return;
    const float* p = a.partial + (size_t)t * a.top * a.d + k;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < a.top; ++j) v += *reinterpret_cast<const f32x4*>(p + (size_t)j * a.d);
    *reinterpret_cast<uint2*>(a.y + (int64_t)t * a.y_stride + k) = make_uint2(pack_elem2(v[0], v[1]), pack_elem2(v[2], v[3]));
}
