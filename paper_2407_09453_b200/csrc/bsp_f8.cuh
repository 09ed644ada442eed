// Pieces shared by the kernels on 8-bit floating-point matrices (bsp_f8 of bsp.h): the place of a scale, the choice of a block's
// exponent, and the conversions of the two formats.  Values are e4m3 or e5m2, scales are bytes b that stand for 2^(b - 127).
#pragma once
#include <cuda_fp16.h>
#include "bsp_internal.cuh"

namespace bsp {

constexpr int kF8Block = 128;                       // entries of a row that share a scale
constexpr int kF8Atom = 512;                        // scales of 128 rows x 4 blocks

inline int64_t f8_pitch(int64_t cols) { return (cols + 15) / 16 * 16; }
__host__ __device__ inline int64_t f8_blocks(int64_t cols) { return (cols + kF8Block - 1) / kF8Block; }
__host__ __device__ inline int64_t f8_atoms(int64_t cols) { return (f8_blocks(cols) + 3) / 4; }
inline int64_t f8_scale_bytes(int64_t rows, int64_t cols) { return f8_blocks(rows) * f8_atoms(cols) * kF8Atom; }

inline int f8_log2(int block) { return block == 4 ? 2 : block == 8 ? 3 : 4; }      // sides of Gamma's blocks

// Place of the scale of row r and block b among the scales of a matrix with `atoms` atoms per 128 rows: the order in which
// tcgen05.cp takes 128 rows to 32 lanes of tensor memory (row r to lane r % 32, column r / 32, four blocks to a column's bytes).
__host__ __device__ inline int64_t f8_scale_at(int64_t r, int64_t b, int64_t atoms)
{
    return ((r >> 7) * atoms + (b >> 2)) * kF8Atom + (r & 31) * 16 + ((r >> 5) & 3) * 4 + (b & 3);
}

// The smallest e with amax <= MAX 2^e as the byte e + 127, from the bits of a finite float32 amax >= 0.  MAX is 1.75 2^8 (e4m3) or
// 1.75 2^15 (e5m2): a fraction above 0.75 needs one exponent more, which the addition carries over.  A block of zeros has scale 1.
template <bool kE5>
__device__ __forceinline__ uint32_t f8_scale_byte(uint32_t amax)
{
    const int e = (int)((amax + 0x1FFFFFu) >> 23) - (kE5 ? 15 : 8);
    return amax == 0u ? 127u : (uint32_t)(e < 0 ? 0 : e);
}
// 2^(127 - b): what entries are multiplied with on their way to 8 bits, exactly (b is at most 247, so this is a normal value).
__device__ __forceinline__ float f8_inverse(uint32_t b) { return __uint_as_float((254u - b) << 23); }
// 2^(b - 127); a subnormal for b = 0, NaN for b = 255.
__device__ __forceinline__ float f8_scale(uint32_t b) { return __uint_as_float(b == 0u ? 0x00400000u : b == 255u ? 0x7FFFFFFFu : b << 23); }

// Two values to 8 bits, the first in the low byte: nearest, ties to even; NaN stays NaN; beyond the largest value (no entry is, after
// the division by its block's scale) they would saturate.
template <bool kE5>
__device__ __forceinline__ uint32_t f8_pack(float lo, float hi)
{
    uint16_t q;
    if constexpr (kE5) asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;\n" : "=h"(q) : "f"(hi), "f"(lo));
    else asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(q) : "f"(hi), "f"(lo));
    return q;
}
// Two 8-bit values (low byte first) to float32, exactly.
template <bool kE5>
__device__ __forceinline__ float2 f8_unpack(uint32_t q)
{
    uint32_t h;
    if constexpr (kE5) asm("cvt.rn.f16x2.e5m2x2 %0, %1;\n" : "=r"(h) : "h"((uint16_t)q));
    else asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(h) : "h"((uint16_t)q));
    return __half22float2(*(const __half2 *)&h);
}

bsp_status launch_quantize_f8(const void *X, bsp_dtype xtype, int64_t P, int64_t I, int64_t ldx, const bsp_wdesc *wd, const uint8_t *gamma,
                              const bsp_f8 *rows, const bsp_f8 *cols, float *colsum, void *ws, cudaStream_t st);
bsp_status launch_dequantize_f8(const bsp_f8 &m, void *X, bsp_dtype xtype, int64_t ldx, bool transpose, cudaStream_t st);
bsp_status launch_gemm_f8(const bsp_f8 &x, const bsp_f8 &w, const float *bias, const bsp_wdesc *wd, const uint8_t *gamma, void *Y, bsp_dtype ytype,
                          void *ws, cudaStream_t st);
bsp_status launch_linear_f8(const bsp_f8 &w, const void *X, bsp_dtype xtype, int64_t P, int64_t ldx, const bsp_f8 &x, const float *bias, void *Y,
                            bsp_dtype ytype, void *ws, cudaStream_t st);

}  // namespace bsp
