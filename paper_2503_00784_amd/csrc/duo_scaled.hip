// C ABI of the products on 8-bit matrices: host-side validation and launches (kernels in duo_scaled.h).
#include "../../include/duo_verify.h"

#include "duo_internal.h"
#include "duo_scaled.h"

namespace {

bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

int check_matrix(int N, int K) { return N < 1 || N > DUO_SCALED_MAX_N || K < 32 || K % 32 || K > DUO_SCALED_MAX_K ? DUO_ERR_SHAPE : DUO_OK; }

// Whether a launch of its own brings the rows to e4m3 before the product; if not, every workgroup does it for itself, which for more than 16 rows
// costs more than the launch unless there are few columns: 26 rows of 96 x 14784 25 us, 16 with the launch; 17 of 22016 x 4096 22.2, 20.0; 17 of 8192 x
// 1024 4.6, 6.8.
bool rows_first(int rows, int K) { return rows > DUO_SCALED_DIRECT_ROWS && !(rows <= 32 && K <= 2048); }
size_t rows_bytes(int rows, int K) {  // of the workspace: tiles and scales of the rows
    const int tiles = (rows + 15) / 16, blocks = scaled_blocks(K);
    return rows_first(rows, K) ? (size_t)tiles * blocks * SCALED_TILE + row_scale_bytes(tiles, blocks) : 0;
}

template <int MT, int NB, int NW, int PF, bool READY, bool FP32>
void launch_bands(const ScaledArgs& a, hipStream_t s) {
    const int bands = (a.N + 15) / 16;
    duo_internal_prof(DUO_PROF_SCALED);
    DUO_LAUNCH((scaled_stream_kernel<MT, NB, NW, PF, READY, FP32>), dim3((bands + NB - 1) / NB), dim3(64 * NW), s, a);
}
// Bands a workgroup, waves, blocks of columns a wave has on their way.  Few bands: one or two a workgroup, so that there is one workgroup for every
// compute unit; up to 1024 bands four, all workgroups at once in one round; beyond, what leaves the rounds even.  us for 9 rows, 4096 columns:
// 256 bands 5.9 (one band, eight waves; two bands 7.1), 768 bands 10.5 (four; two 11.4), 1376 bands 17.0 (two; four 18.5), 8016 bands 80 (two or four).
template <int MT, bool FP32>
void launch_direct(const ScaledArgs& a, hipStream_t s) {
    const int bands = (a.N + 15) / 16;
    if (bands <= 256) launch_bands<MT, 1, 8, (MT == 1 ? 2 : 1), false, FP32>(a, s);
    else if (bands <= 512) launch_bands<MT, 2, 8, (MT == 1 ? 2 : 1), false, FP32>(a, s);
    else if (bands <= 1024) launch_bands<MT, 4, (MT == 1 ? 8 : 4), (MT == 1 ? 1 : 2), false, FP32>(a, s);
    else if constexpr (MT == 1) launch_bands<MT, 2, 8, 2, false, FP32>(a, s);
    else launch_bands<MT, 4, 4, 1, false, FP32>(a, s);
}
// The same where the rows are ready.  us for 33 rows, 4096 columns, with the 3 us of the launch in front: 256 bands 9.7 (one band, eight waves), 768 15.7
// (four bands; two 17.3), 1376 23.9 (two; four 24.9), 8016 91 (four bands and one wave; two bands 110); two tiles of rows 8.2, 13.9, 20.2 and 84 (four bands and four waves).
template <int MT, bool FP32>
void launch_ready(const ScaledArgs& a, hipStream_t s) {
    const int bands = (a.N + 15) / 16;
    if (bands <= 256) launch_bands<MT, 1, 8, 2, true, FP32>(a, s);
    else if (bands <= 512) launch_bands<MT, 2, 8, 2, true, FP32>(a, s);
    else if (bands <= 1024) launch_bands<MT, 4, 4, 2, true, FP32>(a, s);
    else if (bands <= 1536 || (MT == 2 && bands <= 4096)) launch_bands<MT, 2, 4, 2, true, FP32>(a, s);
    else if constexpr (MT == 2) launch_bands<MT, 4, 4, 2, true, FP32>(a, s);
    else if (bands <= 4096) launch_bands<MT, 4, 2, 2, true, FP32>(a, s);
    else launch_bands<MT, 4, 1, 2, true, FP32>(a, s);
}

// ---- more than DUO_MAX_ROWS rows: which block, and over how many workgroups the columns are split.
struct BlockPlan {
    int block, splits;
};
size_t part_stride(int N) { return ((size_t)N + 3) / 4 * 4; }

// What is through first: rounds of the chip times what a step of 128 columns takes with as many workgroups on every compute unit as fit, or with one
// where there are not more; and, where the columns are split, the launch that adds up the parts.  The steps were measured on 4096 columns of
// 4111 rows x 28672, 999 x 12288, 700 x 5120, 300 and 100 x 4096.
// us, 16-bit outputs: 999 rows, 12288 x 4096: 192 x 256 48, 256 x 256 54, 128 x 256 67; 5120 x 13824: 160 x 128 76, 192 x 128 88, 128 x 256 102;
// 700 rows, 5120 x 4096: 128 x 128 of eight waves 22, of four 32; 300 rows, 4096 x 4096: 64 x 128 17, 128 x 128 20; 100 rows: 64 x 64 14, 64 x 128 17.
BlockPlan plan_blocks(int rows, int N, int K, bool fp32) {
    struct Block {
        int bands, tiles, a_unit;
        double narrow, wide, narrow_alone, wide_alone;  // us a step; wide: fp32 outputs (256 x 256 has no LDS for them, 128 x 256 and 64 x 128 are never the first)
        bool can_split;
    };
    static constexpr Block blocks[] = {{16, 16, 1, 1.70, 1e9, 1.70, 1e9, false},   {12, 16, 1, 1.48, 2.55, 1.48, 2.55, false}, {8, 16, 1, 1.08, 1e9, 1.08, 1e9, false},
                                       {8, 8, 2, 1.09, 1.72, 1.00, 1.19, false},   {12, 8, 1, 0.94, 1.60, 0.94, 1.60, false},  {8, 12, 1, 0.92, 1.60, 0.92, 1.60, false},
                                       {10, 8, 1, 0.77, 1.30, 0.77, 1.30, false},  {8, 8, 1, 0.66, 1.08, 0.66, 1.08, true},    {4, 8, 2, 0.69, 1e9, 0.52, 1e9, true},
                                       {4, 4, 2, 0.55, 0.65, 0.44, 0.67, true}};
    const int bands = scaled_blocks(N) * 8, tiles = (rows + 15) / 16, KB = scaled_blocks(K);
    BlockPlan best{0, 1};
    double least = 1e18;
    for (int i = 0; i < 10; ++i) {
        const Block& k = blocks[i];
        const int n = (bands + k.bands - 1) / k.bands * ((tiles + k.tiles - 1) / k.tiles), at_once = 256 * k.a_unit;
        for (int splits = 1; splits <= (k.can_split && n <= 256 ? 8 : 1) && (splits == 1 || KB >= 4 * splits); splits *= 2) {
            const int m = n * splits;
            const double step = m <= 256 ? (fp32 ? k.wide_alone : k.narrow_alone) : ((m + at_once - 1) / at_once) * (fp32 ? k.wide : k.narrow);
            const double t = step * ((KB + splits - 1) / splits) + (splits > 1 ? 4.0 + 8e-6 / 4.0 * splits * rows * (double)N : 0.0);  // parts at 4 TB/s, written and read
            if (t < least) least = t, best = BlockPlan{i, splits};
        }
    }
    const int each = (KB + best.splits - 1) / best.splits;
    best.splits = (KB + each - 1) / each;  // none is empty
    return best;
}
size_t part_bytes(int rows, int N, int K, bool fp32) {
    if (rows <= DUO_MAX_ROWS) return 0;
    const BlockPlan p = plan_blocks(rows, N, K, fp32);
    return p.splits > 1 ? (size_t)p.splits * rows * part_stride(N) * 4 : 0;
}
size_t workspace_of(int rows, int N, int K) {  // for either type of outputs
    const size_t narrow = part_bytes(rows, N, K, false), wide = part_bytes(rows, N, K, true);
    return ((rows_bytes(rows, K) + 15) & ~(size_t)15) + (narrow > wide ? narrow : wide);
}

template <int WB, int WM, int GB, int GM, int STAGES, bool EXACT, bool FP32>
void launch_block(const ScaledArgs& a, int splits, hipStream_t s) {
    const int blocks = (scaled_blocks(a.N) * 8 + WB * GB - 1) / (WB * GB) * ((a.row_tiles + WM * GM - 1) / (WM * GM));
    duo_internal_prof(DUO_PROF_SCALED);
    DUO_LAUNCH((scaled_block_kernel<WB, WM, GB, GM, STAGES, EXACT, FP32>), dim3((blocks + 7) / 8 * 8, splits), dim3(64 * GB * GM), s, a);
}
template <bool FP32>
void launch_blocks(ScaledArgs a, hipStream_t s) {
    const BlockPlan p = plan_blocks(a.rows, a.N, a.K, FP32);
    a.split_blocks = (a.KB + p.splits - 1) / p.splits, a.y_split = 0;
    if (p.splits > 1) {
        ScaledArgs b = a;
        float* const part = reinterpret_cast<float*>(a.xq + ((rows_bytes(a.rows, a.K) + 15) & ~(size_t)15));
        b.y = part, b.y_stride = (int64_t)part_stride(a.N), b.y_split = b.y_stride * a.rows;
        if (p.block == 7) launch_block<2, 4, 4, 2, 4, FP32, true>(b, p.splits, s);
        else if (p.block == 9) launch_block<2, 4, 2, 1, 4, FP32, true>(b, p.splits, s);
        else if constexpr (!FP32) launch_block<2, 4, 2, 2, 3, FP32, true>(b, p.splits, s);
        const int64_t quads = (int64_t)a.rows * (b.y_stride / 4);
        duo_internal_prof(DUO_PROF_SCALED);
        DUO_LAUNCH((scaled_join_kernel<FP32>), dim3((unsigned)((quads + 255) / 256)), dim3(256), s, a, part, p.splits, (int)b.y_stride);
        return;
    }
    if constexpr (!FP32) {
        if (p.block == 0) return launch_block<8, 4, 2, 4, 2, FP32, FP32>(a, 1, s);
        if (p.block == 2) return launch_block<4, 4, 2, 4, 3, FP32, FP32>(a, 1, s);
        if (p.block == 8) return launch_block<2, 4, 2, 2, 3, FP32, FP32>(a, 1, s);
    }
    switch (p.block) {
        case 1: return launch_block<4, 4, 3, 4, 2, FP32, FP32>(a, 1, s);
        case 3: return launch_block<4, 4, 2, 2, 2, FP32, FP32>(a, 1, s);
        case 4: return launch_block<4, 4, 3, 2, 3, FP32, FP32>(a, 1, s);
        case 5: return launch_block<4, 4, 2, 3, 3, FP32, FP32>(a, 1, s);
        case 6: return launch_block<2, 4, 5, 2, 3, FP32, FP32>(a, 1, s);
        case 7: return launch_block<2, 4, 4, 2, 4, FP32, FP32>(a, 1, s);
        default: return launch_block<2, 4, 2, 1, 4, FP32, FP32>(a, 1, s);
    }
}

template <bool FP32>
void launch_product(const ScaledArgs& a, hipStream_t s) {
    if (!rows_first(a.rows, a.K)) return a.row_tiles == 1 ? launch_direct<1, FP32>(a, s) : launch_direct<2, FP32>(a, s);
    duo_internal_prof(DUO_PROF_SCALED);
    DUO_LAUNCH(scaled_rows_kernel, dim3(a.KB, (a.row_tiles + 3) / 4), dim3(256), s, a);
    if (a.rows <= DUO_MAX_ROWS) switch (a.row_tiles) {
            case 2: return launch_ready<2, FP32>(a, s);
            case 3: return launch_ready<3, FP32>(a, s);
            case 4: return launch_ready<4, FP32>(a, s);
            default: return launch_ready<5, FP32>(a, s);
        }
    launch_blocks<FP32>(a, s);
}

}  // namespace

extern "C" size_t duo_scaled_bytes(int N, int K) { return check_matrix(N, K) ? 0 : scaled_bytes(N, K); }

extern "C" int duo_scaled_pack(const uint16_t* src, int N, int K, void* dst, void* hip_stream) {
    if (!src || !dst) return DUO_ERR_NULL;
    if (const int rc = check_matrix(N, K)) return rc;
    if (off16(src) || off16(dst)) return DUO_ERR_ALIGN;
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();  // not of an earlier call
    DUO_LAUNCH(scaled_pack_kernel, dim3(scaled_blocks(K), scaled_blocks(N)), dim3(256), s, src, N, K, static_cast<uint8_t*>(dst));
    return duo_internal_hip_ok(hipGetLastError(), "duo_scaled_pack");
}

extern "C" int duo_scaled_workspace_bytes(int rows, int N, int K, size_t* bytes) {
    if (!bytes) return DUO_ERR_NULL;
    if (const int rc = check_matrix(N, K)) return rc;
    if (rows < 1 || rows > DUO_SCALED_MAX_ROWS) return DUO_ERR_SHAPE;
    *bytes = workspace_of(rows, N, K);
    return DUO_OK;
}

extern "C" int duo_scaled_gemm(const uint16_t* x, int64_t x_stride, const void* w, void* y, int64_t y_stride, int y_fp32, int rows, int N, int K,
                               void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (!x || !w || !y) return DUO_ERR_NULL;
    if (const int rc = check_matrix(N, K)) return rc;
    if (rows < 1 || rows > DUO_SCALED_MAX_ROWS) return DUO_ERR_SHAPE;
    if (y_fp32 != 0 && y_fp32 != 1) return DUO_ERR_ARG;
    if (off16(x) || off16(w) || off16(y) || x_stride % 8 || y_stride % (y_fp32 ? 4 : 8)) return DUO_ERR_ALIGN;
    if (rows > 1 && (x_stride < K || y_stride < N || x_stride > DUO_SCALED_MAX_STRIDE || y_stride > DUO_SCALED_MAX_STRIDE)) return DUO_ERR_SHAPE;
    // what is written meets nothing that other workgroups still read
    const char *x0 = reinterpret_cast<const char*>(x), *y0 = static_cast<const char*>(y), *w0 = static_cast<const char*>(w);
    const int64_t last = rows - 1;
    const char *x1 = x0 + 2 * (last * x_stride + K), *y1 = y0 + (y_fp32 ? 4 : 2) * (last * y_stride + N), *w1 = w0 + scaled_bytes(N, K);
    if ((y0 < x1 && x0 < y1) || (y0 < w1 && w0 < y1)) return DUO_ERR_ARG;
    const size_t need = workspace_of(rows, N, K);
    if (need) {
        if (!workspace) return DUO_ERR_NULL;
        if (off16(workspace)) return DUO_ERR_ALIGN;
        if (workspace_bytes < need) return DUO_ERR_WORKSPACE;
    }
    ScaledArgs a{};
    a.x = x, a.w = static_cast<const uint8_t*>(w), a.y = y, a.xq = static_cast<uint8_t*>(workspace);
    a.x_stride = x_stride, a.y_stride = y_stride;
    a.rows = rows, a.N = N, a.K = K, a.KB = scaled_blocks(K), a.row_tiles = (rows + 15) / 16;
    a.w_scales = scaled_tile_bytes(N, K), a.x_scales = (size_t)a.row_tiles * a.KB * SCALED_TILE;
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();  // not of an earlier call
    if (y_fp32) launch_product<true>(a, s);
    else launch_product<false>(a, s);
    return duo_internal_hip_ok(hipGetLastError(), "duo_scaled_gemm");
}
