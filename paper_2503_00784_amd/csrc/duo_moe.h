// A layer of experts for the few rows of a verify step:
//   l = x R^T,  S = the top_k experts of a row by l,  g = softmax(l) on S,  y = sum over e in S of g_e * (silu(x G_e^T) * (x U_e^T)) D_e^T.
//
// With few rows the layer is the stream of the chosen experts' matrices, so every kernel is laid out around that stream: it is read once, in
// tiles, straight into the registers of the matrix units, and everything else (rows, lists, hidden values) comes out of the caches.
#pragma once
#include "duo_e4m3.h"

constexpr int MOE_MAX_EXPERTS = 512, MOE_MAX_TOP = 16, MOE_MAX_ROWS = 80;

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
    double* logits;     // [logit_parts][rows][experts]
    u16* hidden;        // [rows * top][2][ff_pad]: bf16 pairs, zeros behind ff
    float* partial;     // [rows * top][d]: outputs in front of the sum over a row's experts
    int64_t x_stride, y_stride;
    size_t expert_bytes, up_at, down_at;  // bytes of an expert, of what lies in front of its up and down matrices
    int rows, d, ff, ff_pad, n_experts, top, renormalise;
};

// ---- router.  Logits in 64 bits: which of two experts with nearly equal logits a row takes decides its whole output, and must not hang on the order
// of a sum.  16 experts x 16 rows a workgroup, by the 64-bit matrix instruction (16 x 16 x 4): it leaves one conversion to 64 bits a lane and operand
// for 1024 products, where a loop over the columns has one for every product or four, and no sums over lanes.  A lane's eight consecutive columns of
// a 16-byte load go into eight instructions, which wait for each other; so the columns are spread over up to 64 waves in 16 workgroups (one workgroup
// of 16 waves: 7.4 us for one row of 2048 columns and 64 experts), whose sums moe_choice_kernel adds.  How they are spread follows from the number of
// columns alone: a row's logits are the same bits whoever its neighbours are.
typedef double f64x4 __attribute__((ext_vector_type(4)));
constexpr int LOGIT_WAVES = 4;
__host__ __device__ inline int logit_parts(int d) { return d >= 2048 ? 16 : (d + 127) / 128; }
__global__ __launch_bounds__(64 * LOGIT_WAVES) void moe_logits_kernel(MoeArgs a) {
    __shared__ double part[LOGIT_WAVES][4][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int e0 = blockIdx.y * 16, t0 = blockIdx.z * 16;
    // experts and rows behind the last: the last one again, for nothing; rows that are left out are not read
    const u16* r = a.router + (size_t)min(e0 + c, a.n_experts - 1) * a.d + 8 * g;
    const int t = min(t0 + c, a.rows - 1);
    const bool live = !(a.position && a.position[t] < 0);
    const u16* x = a.x + (int64_t)t * a.x_stride + 8 * g;
    f64x4 sum = {0.0, 0.0, 0.0, 0.0};
    for (int k = 32 * (blockIdx.x * LOGIT_WAVES + wave); k < a.d; k += 32 * LOGIT_WAVES * gridDim.x) {
        Frag8 u, v;
        u.q = *reinterpret_cast<const u32x4*>(r + k);
        v.q = live ? *reinterpret_cast<const u32x4*>(x + k) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int n = 0; n < 8; ++n) sum = __builtin_amdgcn_mfma_f64_16x16x4f64((double)elem_to_f32(u.h[n]), (double)elem_to_f32(v.h[n]), sum, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) part[wave][i][lane] = sum[i];
    __syncthreads();
    // wave i, register i of its lanes: expert 4 i + g, row c
    const double s = part[0][wave][lane] + part[1][wave][lane] + part[2][wave][lane] + part[3][wave][lane];
    const int e = e0 + 4 * wave + g;
    if (e < a.n_experts && t0 + c < a.rows) a.logits[((size_t)blockIdx.x * a.rows + t0 + c) * a.n_experts + e] = s;
}

// One workgroup a row: its logits' parts added up, the rank of every expert, which is the number of experts in front of it (all at once: no search of top_k
// rounds), and the shares.  NaN counts as minus infinity; equal ones rank by their number.
constexpr int CHOICE_THREADS = 512;
__global__ __launch_bounds__(CHOICE_THREADS) void moe_choice_kernel(MoeArgs a) {
    __shared__ double raw[MOE_MAX_EXPERTS], key[MOE_MAX_EXPERTS];
    __shared__ int rank[MOE_MAX_EXPERTS], order[MOE_MAX_TOP];
    static_assert(CHOICE_THREADS >= MOE_MAX_EXPERTS, "a thread for every expert");
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, t = blockIdx.x, n = a.n_experts;
    if (a.position && a.position[t] < 0) {
        if (tid < a.top) a.chosen[t * a.top + tid] = -1;
        return;
    }
    if (tid < n) {
        double parts[16], l = 0.0;
        const int n_parts = logit_parts(a.d);
#pragma unroll
        for (int i = 0; i < 16; ++i) parts[i] = a.logits[((size_t)min(i, n_parts - 1) * a.rows + t) * n + tid];
#pragma unroll
        for (int i = 0; i < 16; ++i) l += i < n_parts ? parts[i] : 0.0;
        raw[tid] = l, key[tid] = l == l ? l : -__builtin_huge_val();
        rank[tid] = 0;
    }
    __syncthreads();
    // thread (e, part): the experts of a part of the list that stand in front of e
    int shift = 5;
    while (1 << shift < n) ++shift;
    const int parts = CHOICE_THREADS >> shift, e = tid & ((1 << shift) - 1), each = (n + parts - 1) / parts, first = (tid >> shift) * each, last = min(first + each, n);
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

// Both in one launch for small routers: a workgroup for 16 rows, whose 16 waves share out (16 experts, part of the columns).  One compute unit has to form
// all products of 16 rows, a 64-bit instruction every 64 clocks on each of its four matrix units: 4 experts of 768 columns 4.6 us (3.0 + 3.0 in two
// launches), but 32 experts of 2048 columns 16 us (4.8 + 4.6).
constexpr int ROUTER_WAVES = 16, ROUTER_EXPERTS = 32;
__host__ inline bool router_in_one(int experts, int d) { return experts <= ROUTER_EXPERTS && (experts > 16 ? 2 : 1) * d <= 1024; }
__global__ __launch_bounds__(64 * ROUTER_WAVES) void moe_router_kernel(MoeArgs a) {
    __shared__ double part[ROUTER_WAVES][4][64], raw[16][ROUTER_EXPERTS];
    __shared__ int order[16][MOE_MAX_TOP];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4, n = a.n_experts;
    const int tiles = n > 16 ? 2 : 1, tile = wave & (tiles - 1), parts = ROUTER_WAVES / tiles, t0 = blockIdx.x * 16;
    {
        const u16* r = a.router + (size_t)min(16 * tile + c, n - 1) * a.d + 8 * g;
        const int t = min(t0 + c, a.rows - 1);
        const bool live = !(a.position && a.position[t] < 0);
        const u16* x = a.x + (int64_t)t * a.x_stride + 8 * g;
        f64x4 sum = {0.0, 0.0, 0.0, 0.0};
        for (int k = 32 * (wave / tiles); k < a.d; k += 32 * parts) {
            Frag8 u, v;
            u.q = *reinterpret_cast<const u32x4*>(r + k);
            v.q = live ? *reinterpret_cast<const u32x4*>(x + k) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = __builtin_amdgcn_mfma_f64_16x16x4f64((double)elem_to_f32(u.h[i]), (double)elem_to_f32(v.h[i]), sum, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) part[wave][i][lane] = sum[i];
    }
    __syncthreads();
    if (threadIdx.x < 16 * ROUTER_EXPERTS) {  // register i of lane (c, g): expert 4 i + g of the tile, row c
        const int row = threadIdx.x & 15, e = threadIdx.x >> 4, w = e >> 4;
        if (w < tiles) {
            double s = 0.0;
            for (int p = 0; p < parts; ++p) s += part[p * tiles + w][(e & 15) >> 2][(e & 3) * 16 + row];
            raw[row][e] = s;
        }
    }
    __syncthreads();
    const int t = t0 + wave;  // a wave a row from here on
    if (t >= a.rows) return;
    if (a.position && a.position[t] < 0) {
        if (lane < a.top) a.chosen[t * a.top + lane] = -1;
        return;
    }
    const double lowest = -__builtin_huge_val();
    const int e = lane & 31;  // the lanes of one half compare with even experts, those of the other with odd ones
    const double l = raw[wave][min(e, n - 1)], mine = l == l ? l : lowest;
    int ahead = 0;
    for (int j = lane >> 5; j < n; j += 2) {
        const double o = raw[wave][j], other = o == o ? o : lowest;
        ahead += other > mine || (other == mine && j < e);
    }
    ahead += __shfl_xor(ahead, 32, 64);
    if (lane < n && ahead < a.top) order[wave][ahead] = e;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
    const int at = lane < a.top ? order[wave][lane] : 0;
    const double most = raw[wave][order[wave][0]];
    const double p = lane < a.top ? exp(raw[wave][at] - most) : 0.0;
    const double sum = wave_sum(a.renormalise ? p : lane < n ? exp(l - most) : 0.0);
    if (lane < a.top) {
        const float share = (float)(p / sum);
        a.chosen[t * a.top + lane] = at, a.share[t * a.top + lane] = share;
        if (a.chosen_out) a.chosen_out[t * a.top + lane] = at;
        if (a.share_out) a.share_out[t * a.top + lane] = share;
    }
}

// What the waves of a workgroup have written to LDS, and nothing else, is there for all of them; loads from memory stay on their way.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The expert of the workgroups at place `at` of the grid: the expert of that number or, where the rows make fewer choices than there are experts, that of
// choice number `at` (-1 if its row is left out).  The same for every lane.
__device__ __forceinline__ int expert_at(const MoeArgs& a, int at) { return a.rows * a.top < a.n_experts ? __builtin_amdgcn_readfirstlane(a.chosen[at]) : at; }

// The rows that chose it.  Every workgroup finds them for itself from the list of choices, at most 1280 words out of the caches, which costs less than
// a launch that makes lists.  Their order is left to the atomics: each is a column of its own in the products, and comes out the same wherever it stands.
struct ExpertRows {
    int count, first;             // first: the first choice of the expert
    int16_t entry[MOE_MAX_ROWS];  // row * top + place
};
// false: nothing to do here, no row chose the expert or the workgroups of an earlier choice have it
template <int THREADS>
__device__ __forceinline__ bool find_rows(const MoeArgs& a, ExpertRows& r, int at, int e) {
    constexpr int EACH = (MOE_MAX_ROWS * MOE_MAX_TOP + THREADS - 1) / THREADS;
    const int tid = threadIdx.x, entries = a.rows * a.top;
    if (a.rows == 1 && entries < a.n_experts) {  // choice `at` is the only one of its expert
        if (tid == 0) r.count = 1, r.entry[0] = (int16_t)at;
        lds_barrier();
        return true;
    }
    int chosen[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) chosen[i] = i * THREADS + tid < entries ? a.chosen[i * THREADS + tid] : -1;
    if (tid == 0) r.count = 0, r.first = 0x7fffffff;
    lds_barrier();
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (chosen[i] == e) {
            r.entry[atomicAdd(&r.count, 1)] = (int16_t)(i * THREADS + tid);
            atomicMin(&r.first, i * THREADS + tid);
        }
    lds_barrier();
    return r.count > 0 && (entries >= a.n_experts || r.first == at);
}

// Rows are read through buffer descriptors: lanes without a row ask for an offset behind the end and get zeros without a memory access, and the
// loop has no branch around its loads, so that the compiler can count them.  Offsets stay below 2^31: 80 rows x 16 experts x 65536 channels x 4
// bytes are 2^28.4, 80 rows at the largest distance of 2^23 elements 2^30.4.
constexpr uint32_t NO_ROW = 0x80000000u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_buffer(const void* p, size_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (uint32_t)bytes, 0x00027000);
}
__device__ __forceinline__ u32x4 row_load(__amdgpu_buffer_rsrc_t r, uint32_t offset) { return __builtin_amdgcn_raw_buffer_load_b128(r, (int)offset, 0, 0); }

// A band's tiles of 128 columns as operands, from a matrix in 16 bits (tiles of 16 x 32, the library's streaming layout) or in e4m3 with block
// scales.  column(i, g): the first of the eight columns of the block that a lane of group g holds in operand i.
struct Wide {  // 16 bits
    static constexpr bool SCALED = false, SCALED_SUMS = false;
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
};
// e4m3.  bf16 operands are values times scale, exact.  (A scale on the sums of a block's products with the bare values, up to 448 whatever they stand for,
// comes too late for rows and hidden values from 2^119 on.)  fp16 has no room for every scale, and its rows, below 2^16, cannot make such sums too large:
// there it goes on the sums.
struct Narrow {
#ifdef DUO_FP16
    static constexpr bool SCALED = true, SCALED_SUMS = true;
#else
    static constexpr bool SCALED = true, SCALED_SUMS = false;
#endif
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
    __device__ __forceinline__ bf16x8 operand_bf16(int i) const { return e4m3_to_bf16(word(i, 0), word(i, 1), scale()); }
    __device__ __forceinline__ elem8 operand(int i) const {
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
        return operand_bf16(i);
#endif
    }
    __device__ __forceinline__ float scale() const { return scale_of(byte); }
};

// what the four operands of a block have added to the sum takes its place; where the scale is still to come, sum += scale * that
template <class W>
__device__ __forceinline__ void add_block(f32x4& sum, const f32x4& block, const W& w) {
    if constexpr (W::SCALED_SUMS) {
        const float s = w.scale();
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = fmaf(block[i], s, sum[i]);
    } else sum = block;
}

// h as bf16 pairs hi + lo.  Magnitudes that would round to 2^128 are cut instead, and lo is zero where hi is an infinity, which so stays one.  (In fp16
// there is neither: sums over finite rows and matrices stay below 2^45, hidden values below 2^90.)
__device__ __forceinline__ void hidden_pairs(const float (&h)[4], u16 (&hi)[4], u16 (&lo)[4]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const __bf16 b = (__bf16)h[q];
        hi[q] = __builtin_bit_cast(u16, b);
        lo[q] = __builtin_bit_cast(u16, (__bf16)(h[q] - (float)b));
    }
#ifndef DUO_FP16
    constexpr float LARGEST = 0x1.fep127f;  // of bf16
    if (fmaxf(fmaxf(fabsf(h[0]), fabsf(h[1])), fmaxf(fabsf(h[2]), fabsf(h[3]))) > LARGEST)  // (fmaxf passes over NaN, whose pair is NaN already)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (fabsf(h[q]) > LARGEST) {
                hi[q] = (u16)(__float_as_uint(h[q]) >> 16);
                lo[q] = fabsf(h[q]) == __builtin_huge_valf() ? (u16)0 : __builtin_bit_cast(u16, (__bf16)(h[q] - __uint_as_float((uint32_t)hi[q] << 16)));
            }
#endif
}

// ---- gate and up.  A workgroup owns 16 hidden channels of one expert: a band of its gate and one of its up matrix, which its waves read in turns of
// 128 columns, PF of them at a time: while a wave forms the products of one, PF - 1 are on their way.  With PF = 1, as for two and three tiles of rows,
// none is: it waits a whole latency for each, and the other waves of its SIMD have to fill the gap.  The sums of the waves
// are added through LDS in wave order.  The columns of the product are the rows that chose the expert, 16 MT at a time.  Hidden values are left as bf16 pairs hi + lo (16 bits of mantissa, fp32's range in either build),
// with the row's share of the expert in them.
template <class W, int MT, int NW, int PF>
__global__ __launch_bounds__(64 * NW) void moe_gate_up_kernel(MoeArgs a) {
    __shared__ f32x4 part[NW][2 * MT][64];
    __shared__ ExpertRows rows;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int band = blockIdx.x, KB = (a.d + 127) >> 7, n = (KB - wave + NW - 1) / NW;
    const int e = expert_at(a, blockIdx.y);
    if (e < 0) return;
    const uint8_t* gate = a.experts + (size_t)e * a.expert_bytes;
    const uint8_t* up = gate + a.up_at;
    W w[PF][2];
    auto block = [&](int i) { return max(min(wave + NW * min(i, n - 1), KB - 1), 0); };
    auto load_weights = [&](int s, int i) {
        w[s][0].load(gate, a.ff, a.d, band, block(i), lane);
        w[s][1].load(up, a.ff, a.d, band, block(i), lane);
    };
    if (!find_rows<64 * NW>(a, rows, blockIdx.y, e)) return;
    const int count = __builtin_amdgcn_readfirstlane(rows.count);
    const __amdgpu_buffer_rsrc_t xs = row_buffer(a.x, ((size_t)(a.rows - 1) * a.x_stride + a.d) * 2);
    for (int first = 0; first < count; first += 16 * MT) {
        uint32_t row[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int i = first + m * 16 + c;
            row[m] = i < count ? (uint32_t)(rows.entry[i] / a.top) * (uint32_t)a.x_stride * 2 : NO_ROW;
        }
        f32x4 acc[2][MT];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[b][m] = f32x4{0.f, 0.f, 0.f, 0.f};
        u32x4 x[PF][MT][4];
        auto load_rows = [&](int s, int i) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) x[s][m][q] = row_load(xs, row[m] + (uint32_t)(block(i) * 128 + W::column(q, g)) * 2);
        };
        auto products = [&](int s, int i) {
            const int j = wave + NW * i;
            if ((j + 1) * 128 > a.d) {  // columns from d on: zeros, whatever lies behind the rows
                w[s][0].cut(a.d, j), w[s][1].cut(a.d, j);
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (j * 128 + W::column(q, g) >= a.d) x[s][m][q] = u32x4{0u, 0u, 0u, 0u};
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                elem8 o[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) o[q] = w[s][b].operand(q);
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    if (first + m * 16 < count) {  // the same for every lane
                        f32x4 sum = W::SCALED_SUMS ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[b][m];
#pragma unroll
                        for (int q = 0; q < 4; ++q) sum = mfma16(o[q], __builtin_bit_cast(elem8, x[s][m][q]), sum);
                        add_block(acc[b][m], sum, w[s][b]);
                    }
            }
        };
#pragma unroll
        for (int s = 0; s < PF; ++s) load_weights(s, s), load_rows(s, s);
        int i = 0;
        for (; i + PF < n; i += PF) {
#pragma unroll
            for (int s = 0; s < PF; ++s) {
                products(s, i + s);
                load_weights(s, i + s + PF);
                load_rows(s, i + s + PF);
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
                float h[4];
                u16 hi[4], lo[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) h[q] = s[q] / (1.0f + expf(-s[q])) * u[q] * share;
                hidden_pairs(h, hi, lo);
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
        if constexpr (W::SCALED) v[0] = w.operand_bf16(i);
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
__device__ __forceinline__ void down_block(f32x4& sum, const DownOperand<W> (&o)[4], const u32x4 (&x)[8]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const bf16x8 hi = __builtin_bit_cast(bf16x8, x[q]), lo = __builtin_bit_cast(bf16x8, x[4 + q]);
        sum = mfma_bf16(o[q].v[0], hi, sum);
        sum = mfma_bf16(o[q].v[0], lo, sum);
        if constexpr (DownOperand<W>::PARTS == 2) sum = mfma_bf16(o[q].v[DownOperand<W>::PARTS - 1], hi, sum);
    }
}

// ---- down.  As gate and up: a workgroup owns NB bands of one expert, the columns are the rows that chose it; what a row gets from each of its experts
// is left apart in fp32 and added up by moe_combine_kernel in the order of its choices.  (One workgroup for 16 outputs of all rows and all experts
// needs neither, but then a few hundred workgroups read everything, 16 columns at a time: 16 rows on 50 active experts of 2048 x 1408 in 8 bits 62 us,
// 27 + 4 like this; one row on 6 in 16 bits 12.5, 8.5 + 3.)
// ONE choice a row: there is nothing to add, and the outputs go where they belong.
template <class W, int MT, int NB, int NW, int PF, bool ONE>
__global__ __launch_bounds__(64 * NW) void moe_down_kernel(MoeArgs a) {
    __shared__ f32x4 part[NW][NB * MT][64];
    __shared__ ExpertRows rows;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int band0 = blockIdx.x * NB, KB = a.ff_pad >> 7, n = (KB - wave + NW - 1) / NW;  // d is a multiple of 64: NB divides its bands
    const int e = expert_at(a, blockIdx.y);
    if (e < 0) return;
    const uint8_t* down = a.experts + (size_t)e * a.expert_bytes + a.down_at;
    W w[PF][NB];
    auto block = [&](int i) { return max(min(wave + NW * min(i, n - 1), KB - 1), 0); };
    auto load_weights = [&](int s, int i) {
#pragma unroll
        for (int b = 0; b < NB; ++b) w[s][b].load(down, a.d, a.ff, band0 + b, block(i), lane);
    };
    if (!find_rows<64 * NW>(a, rows, blockIdx.y, e)) return;
    const int count = __builtin_amdgcn_readfirstlane(rows.count);
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
        u32x4 x[PF][MT][8];
        auto load_rows = [&](int s, int i) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t k = (uint32_t)(block(i) * 128 + W::column(q, g)) * 2;
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
                    if (first + m * 16 < count) down_block<W>(acc[b][m], o, x[s][m]);  // the same for every lane
            }
        };
#pragma unroll
        for (int s = 0; s < PF; ++s) load_weights(s, s), load_rows(s, s);
        int i = 0;
        for (; i + PF < n; i += PF) {
#pragma unroll
            for (int s = 0; s < PF; ++s) {
                products(s, i + s);
                load_weights(s, i + s + PF);
                load_rows(s, i + s + PF);
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
            if (at < count) {
                const int p = rows.entry[at], k = (band0 + t / MT) * 16 + 4 * g;
                if constexpr (ONE) *reinterpret_cast<uint2*>(a.y + (int64_t)p * a.y_stride + k) = make_uint2(pack_elem2(v[0], v[1]), pack_elem2(v[2], v[3]));
                else *reinterpret_cast<f32x4*>(a.partial + (size_t)p * a.d + k) = v;
            }
        }
        __syncthreads();
    }
}

// a thread: four outputs of a row
__global__ __launch_bounds__(256) void moe_combine_kernel(MoeArgs a) {
    const int t = blockIdx.y, k = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (k >= a.d || (a.position && a.position[t] < 0)) return;
    const float* p = a.partial + (size_t)t * a.top * a.d + k;
    f32x4 v = *reinterpret_cast<const f32x4*>(p);
    for (int j = 1; j < a.top; j += 4) {  // four loads at a time
        f32x4 u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = *reinterpret_cast<const f32x4*>(p + (size_t)min(j + i, a.top - 1) * a.d);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (j + i < a.top) v += u[i];
    }
    *reinterpret_cast<uint2*>(a.y + (int64_t)t * a.y_stride + k) = make_uint2(pack_elem2(v[0], v[1]), pack_elem2(v[2], v[3]));
}
