// Products on matrices in e4m3 with block scales: packing, a kernel that streams the matrix past a few rows, and one for many rows.
#pragma once
#include "duo_e4m3.h"

// 32 values of a row as a lane of an operand holds them: columns 64 h + 16 g + 8 i .. +8 of a block in v[2 h + i], g = lane / 16.
struct RowPiece {
    u32x4 v[4];
    // row: the row's first element, or null for a row of zeros; k: first column of the block; columns from K on are zeros (K % 32 == 0)
    __device__ __forceinline__ void load(const u16* row, int k, int K, int g) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = k + 64 * h + 16 * g;
            const bool in = row != nullptr && c < K;
            const u32x4* p = reinterpret_cast<const u32x4*>(row + c);
            v[2 * h] = in ? p[0] : u32x4{0u, 0u, 0u, 0u};
            v[2 * h + 1] = in ? p[1] : u32x4{0u, 0u, 0u, 0u};
        }
    }
    // e + 127 of the block this row has here: the largest magnitude of the four lanes that share the row.  Infinities and NaN count too: their row
    // is NaN whatever becomes of its other values.
    __device__ __forceinline__ int scale() const {
        uint32_t m = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) m = max_patterns(m, v[i][j] & 0x7fff7fffu);
        m = max(m & 0xffffu, m >> 16);
        const auto a = __builtin_amdgcn_permlane16_swap(m, m, false, false);
        m = max(a[0], a[1]);
        const auto b = __builtin_amdgcn_permlane32_swap(m, m, false, false);
        m = max(b[0], b[1]);
        return scale_byte(m);
    }
    __device__ __forceinline__ void quantise(float s, u32x4 (&q)[2]) const {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                q[h][2 * i] = to_e4m3(v[2 * h + i][0], v[2 * h + i][1], s);
                q[h][2 * i + 1] = to_e4m3(v[2 * h + i][2], v[2 * h + i][3], s);
            }
    }
};

// ---- matrices, once: one workgroup per block of 128 x 128.  Only finite values count for the scale, so that a row with an infinity leaves the
// other rows of its block as they are.
__global__ __launch_bounds__(256) void scaled_pack_kernel(const u16* __restrict__ src, int N, int K, uint8_t* __restrict__ dst) {
    __shared__ uint32_t most[4];
    const int KB = scaled_blocks(K), j = blockIdx.x, rb = blockIdx.y;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    RowPiece x[2];  // wave w: bands 2 w and 2 w + 1 of the block
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int row = rb * SCALE_BLOCK + (2 * wave + i) * 16 + r;
        x[i].load(row < N ? src + (size_t)row * K : nullptr, j * SCALE_BLOCK, K, g);
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t p = (x[i].v[a][b] >> (16 * half)) & 0x7fffu;
                    m = (__float_as_uint(elem_to_f32((u16)p)) & 0x7f800000u) != 0x7f800000u ? max(m, p) : m;
                }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
    if (lane == 0) most[wave] = m;
    __syncthreads();
    const int byte = scale_byte(max(max(most[0], most[1]), max(most[2], most[3])));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        u32x4 q[2];
        x[i].quantise(scale_of(byte), q);
        u32x4* tile = reinterpret_cast<u32x4*>(dst + ((size_t)(rb * 8 + 2 * wave + i) * KB + j) * SCALED_TILE);
        tile[lane] = q[0];
        tile[64 + lane] = q[1];
    }
    if (threadIdx.x == 0) dst[scaled_tile_bytes(N, K) + (size_t)rb * KB + j] = (uint8_t)byte;
}

struct ScaledArgs {
    const u16* x;          // [rows][K], x_stride elements from row to row
    const uint8_t* w;      // tiles, then the scales
    void* y;               // 16-bit or fp32 [rows][N]
    uint8_t* xq;           // many rows: tiles of the activations, then their scales [K / 128][row tiles * 16]
    size_t w_scales, x_scales;  // bytes in front of the scales
    int64_t x_stride, y_stride;
    int rows, N, K, KB, row_tiles;
};

// four consecutive outputs (features n .. n + 3) of one row; n and the strides are multiples of 4, so the store is as wide as it looks
template <bool FP32>
__device__ __forceinline__ void store_outputs(const ScaledArgs& a, int row, int n, f32x4 v) {
    if (row >= a.rows || n >= a.N) return;
    if constexpr (FP32) {
        float* y = static_cast<float*>(a.y) + (size_t)row * a.y_stride + n;
        if (n + 4 <= a.N) *reinterpret_cast<f32x4*>(y) = v;
        else
            for (int i = 0; i < a.N - n; ++i) y[i] = v[i];
    } else {
        u16* y = static_cast<u16*>(a.y) + (size_t)row * a.y_stride + n;
        const uint32_t lo = pack_elem2(v[0], v[1]), hi = pack_elem2(v[2], v[3]);
        if (n + 4 <= a.N) *reinterpret_cast<uint2*>(y) = make_uint2(lo, hi);
        else
            for (int i = 0; i < a.N - n; ++i) y[i] = (u16)((i < 2 ? lo : hi) >> (16 * (i & 1)));
    }
}

// ---- few rows: a workgroup owns NB bands, its NW waves take the blocks of columns in turn and add up what they have through LDS, in wave order.
template <int MT, int NB, int NW, bool FP32>
__global__ __launch_bounds__(64 * NW) void scaled_stream_kernel(ScaledArgs a) {
    __shared__ f32x4 part[NW][NB * MT][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int band0 = blockIdx.x * NB, last = scaled_blocks(a.N) * 8 - 1;
    const u16* row[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) row[m] = m * 16 + c < a.rows ? a.x + (int64_t)(m * 16 + c) * a.x_stride : nullptr;
    f32x4 acc[NB][MT];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[b][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int j = wave; j < a.KB; j += NW) {
        bf16x8 w[NB][4];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int band = min(band0 + b, last);
            const u32x4* tile = reinterpret_cast<const u32x4*>(a.w + ((size_t)band * a.KB + j) * SCALED_TILE) + lane;
            const u32x4 q0 = __builtin_nontemporal_load(tile), q1 = __builtin_nontemporal_load(tile + 64);
            const float s = scale_of(a.w[a.w_scales + (size_t)(band >> 3) * a.KB + j]);
            w[b][0] = e4m3_to_bf16(q0[0], q0[1], s);
            w[b][1] = e4m3_to_bf16(q0[2], q0[3], s);
            w[b][2] = e4m3_to_bf16(q1[0], q1[1], s);
            w[b][3] = e4m3_to_bf16(q1[2], q1[3], s);
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            RowPiece x;
            u32x4 q[2];
            x.load(row[m], j * SCALE_BLOCK, a.K, g);
            const float s = scale_of(x.scale());
            x.quantise(s, q);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bf16x8 v = e4m3_to_bf16(q[i >> 1][2 * (i & 1)], q[i >> 1][2 * (i & 1) + 1], s);
#pragma unroll
                for (int b = 0; b < NB; ++b) acc[b][m] = mfma_bf16(w[b][i], v, acc[b][m]);
            }
        }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int m = 0; m < MT; ++m) part[wave][b * MT + m][lane] = acc[b][m];
    __syncthreads();
    for (int t = wave; t < NB * MT; t += NW) {
        f32x4 v = part[0][t][lane];
        for (int w = 1; w < NW; ++w) v += part[w][t][lane];
        store_outputs<FP32>(a, (t % MT) * 16 + c, (band0 + t / MT) * 16 + 4 * g, v);
    }
}

// ---- many rows, first the activations: one wave per tile of 16 rows x 128 columns
__global__ __launch_bounds__(256) void scaled_rows_kernel(ScaledArgs a) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int tile = blockIdx.y * 4 + wave, j = blockIdx.x;
    if (tile >= a.row_tiles) return;
    const int r = tile * 16 + c;
    RowPiece x;
    u32x4 q[2];
    x.load(r < a.rows ? a.x + (int64_t)r * a.x_stride : nullptr, j * SCALE_BLOCK, a.K, g);
    const int byte = x.scale();
    x.quantise(scale_of(byte), q);
    u32x4* dst = reinterpret_cast<u32x4*>(a.xq + ((size_t)tile * a.KB + j) * SCALED_TILE);
    dst[lane] = q[0];
    dst[64 + lane] = q[1];
    if (g == 0) a.xq[a.x_scales + ((size_t)j * a.row_tiles + tile) * 16 + c] = (uint8_t)byte;
}

// then the product: four waves, each 4 bands x 4 row tiles.
template <bool FP32>
__global__ __launch_bounds__(256) void scaled_block_kernel(ScaledArgs a) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int band0 = blockIdx.x * 8 + (wave & 1) * 4, tile0 = blockIdx.y * 8 + (wave >> 1) * 4;
    f32x4 acc[4][4];
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int m = 0; m < 4; ++m) acc[b][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < a.KB; ++j) {
        u32x4 w[4][2], x[4][2];
        int sx[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u32x4* wt = reinterpret_cast<const u32x4*>(a.w + ((size_t)(band0 + i) * a.KB + j) * SCALED_TILE) + lane;
            w[i][0] = wt[0], w[i][1] = wt[64];
            const int tile = min(tile0 + i, a.row_tiles - 1);
            const u32x4* xt = reinterpret_cast<const u32x4*>(a.xq + ((size_t)tile * a.KB + j) * SCALED_TILE) + lane;
            x[i][0] = xt[0], x[i][1] = xt[64];
            sx[i] = a.xq[a.x_scales + ((size_t)j * a.row_tiles + tile) * 16 + c];
        }
        const int sw = a.w[a.w_scales + (size_t)(band0 >> 3) * a.KB + j];
        if constexpr (FP32) {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                bf16x8 v[4], u[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = e4m3_to_bf16(w[i][s >> 1][2 * (s & 1)], w[i][s >> 1][2 * (s & 1) + 1], scale_of(sw));
                    u[i] = e4m3_to_bf16(x[i][s >> 1][2 * (s & 1)], x[i][s >> 1][2 * (s & 1) + 1], scale_of(sx[i]));
                }
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int m = 0; m < 4; ++m) acc[b][m] = mfma_bf16(v[b], u[m], acc[b][m]);
            }
        } else {
            auto both = [](const u32x4 (&q)[2]) {
                return i32x8{(int)q[0][0], (int)q[0][1], (int)q[0][2], (int)q[0][3], (int)q[1][0], (int)q[1][1], (int)q[1][2], (int)q[1][3]};
            };
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int m = 0; m < 4; ++m)
                    acc[b][m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(both(w[b]), both(x[m]), acc[b][m], 0, 0, 0, sw, 0, sx[m]);
        }
    }
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int m = 0; m < 4; ++m) store_outputs<FP32>(a, (tile0 + m) * 16 + c, (band0 + b) * 16 + 4 * g, acc[b][m]);
}
