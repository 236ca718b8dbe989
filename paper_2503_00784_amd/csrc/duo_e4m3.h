// Matrices and rows held in 8-bit floating point (e4m3: 4 exponent bits, 3 mantissa bits, largest magnitude 448, no infinities), with one
// power of two for every block of 128.
//
// A block with the largest finite magnitude a gets s = 2^e, e the smallest integer with a <= 448 s, kept within [-110, 120]; its values are
// q = e4m3(v / s), rounded to nearest even.  Matrices have a scale for every 128 rows x 128 columns, activations one for every 128 values of a
// row.  v / s is exact because s is a power of two, so a value has one rounding, which depends on nothing but the block; a scale that is up to
// twice larger than it had to be costs a floating type no mantissa bit.  e4m3 times a scale is a bf16 value (4 bits of mantissa, |e| small
// enough for normal numbers), which is what the kernels that need exact products rely on.  Infinities and NaN become e4m3's NaN.
//
// Layout: as the 16-bit matrices, bands of 16 rows and tiles in the order in which a wave's registers take them.  A tile is 16 rows x 128
// columns, 2 KiB; lane l holds row l % 16, and of half h of the columns the 16 bytes of columns 64 h + 16 (l / 16) .. +16, at byte
// 1024 h + 16 l.  Tile (band, block of columns j) is number band * ceil(K / 128) + j.  Rows are padded to a multiple of 128 and columns to a
// multiple of 128 with zeros.  Behind the tiles one byte for every block, e + 127, [N / 128][K / 128].
#pragma once
#include "duo_common.h"

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef u16 u16x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int SCALE_BLOCK = 128;
constexpr int SCALED_TILE = 2048;  // bytes of a tile
constexpr int SCALE_EXP_MIN = -110, SCALE_EXP_MAX = 120;

__host__ __device__ inline int scaled_blocks(int n) { return (n + SCALE_BLOCK - 1) / SCALE_BLOCK; }
__host__ __device__ inline size_t scaled_tile_bytes(int N, int K) { return (size_t)scaled_blocks(N) * 8 * scaled_blocks(K) * SCALED_TILE; }
__host__ __device__ inline size_t scaled_bytes(int N, int K) {
    return scaled_tile_bytes(N, K) + (((size_t)scaled_blocks(N) * scaled_blocks(K) + 15) & ~(size_t)15);
}

// e + 127 of a block whose largest magnitude has the 16-bit pattern p (sign cleared).  448 is 1.75 * 2^8.
__device__ __forceinline__ int scale_byte(uint32_t p) {
    const uint32_t b = __float_as_uint(elem_to_f32((u16)p));
    int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = e < SCALE_EXP_MIN ? SCALE_EXP_MIN : e > SCALE_EXP_MAX ? SCALE_EXP_MAX : e;
    return e + 127;
}
__device__ __forceinline__ float scale_of(int byte) { return __uint_as_float((uint32_t)byte << 23); }

// the larger of each half of two registers of two sign-cleared 16-bit patterns (which are ordered as their values are)
__device__ __forceinline__ uint32_t max_patterns(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// two registers of two 16-bit values each -> four e4m3 of value / scale: the hardware conversion divides by a power of two and rounds once
__device__ __forceinline__ uint32_t to_e4m3(uint32_t lo, uint32_t hi, float scale) {
    s16x2 q = {0, 0};
#ifdef DUO_FP16
    q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(q, __builtin_bit_cast(f16x2, lo), scale, false);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(q, __builtin_bit_cast(f16x2, hi), scale, true);
#else
    q = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(q, __builtin_bit_cast(bf16x2, lo), scale, false);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(q, __builtin_bit_cast(bf16x2, hi), scale, true);
#endif
    return __builtin_bit_cast(uint32_t, q);
}

union Bf16Frag {
    bf16x8 v;
    bf16x2 p[4];
    u32x4 q;
};
// eight e4m3 -> bf16 operand of value * scale, exact
__device__ __forceinline__ bf16x8 e4m3_to_bf16(uint32_t lo, uint32_t hi, float scale) {
    Bf16Frag f;
    f.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    f.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    f.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    f.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return f.v;
}
__device__ __forceinline__ f32x4 mfma_bf16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
