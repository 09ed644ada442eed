// To 8-bit floating point and back: activations and gradients with one power-of-two scale for 128 entries along the axis that a
// product sums over, weights Gamma (.) W with one scale per block of 128 x 128, each in both orientations from one pass over the
// input; column sums (the gradient of a bias) beside them.  Section "Compiler and its Code generation" (8-bit tensors with
// power-of-two scales) and Section "Training and Quantization" of the paper.
//
// A block's scale is 2^e with the smallest e for which its largest entry fits the format, so x 2^-e is exact and an entry is rounded
// once, to the format.  A tile of 128 x 128 entries is one block of scales in either orientation: a CTA reads it once into
// registers (thread (tx, ty) holds rows 8 ty .. 8 ty + 7 of columns 8 tx .. 8 tx + 7), finds the largest entry of every row by shuffles
// and of every column through shared memory, and writes both forms, the transposed one through shared memory so that its rows
// leave in pieces of 128 bytes.  Bound by HBM: e + 2 bytes an entry.
#include "bsp_f8.cuh"

namespace bsp {
namespace {

constexpr int kQThreads = 256;

struct QParams {
    const void *X;
    int64_t P, I, ldx;
    int vec;                      // rows of X can be read 16 bytes at a time
    uint8_t *rows, *rows_scale, *cols, *cols_scale;
    int64_t rows_pitch, cols_pitch, rows_atoms, cols_atoms;
    float *partial;               // column sums of every tile of 128 positions, [P / 128][I]
    const uint8_t *gamma;         // weights: Gamma, or NULL for all ones
    int bo, bi;                   // logarithms of the sizes of Gamma's blocks
    int64_t NBi;
    int64_t tiles_i;
};

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t bf16_max2(uint32_t a, uint32_t b)      // (passes by NaN)
{
    const __nv_bfloat162 m = __hmax2(*(const __nv_bfloat162 *)&a, *(const __nv_bfloat162 *)&b);
    return *(const uint32_t *)&m;
}

// Two float32 operations in one instruction (the quantisers are bound by the instructions they issue: 76 % of the cycles).
__device__ __forceinline__ void mul2(float &a, float &b, float f)
{
    asm("{\n .reg .b64 x, y;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %2};\n mul.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}\n" : "+f"(a), "+f"(b) : "f"(f));
}
__device__ __forceinline__ void add2(float &a, float &b, float c, float d)
{
    asm("{\n .reg .b64 x, y;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %3};\n add.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}\n" : "+f"(a), "+f"(b) : "f"(c), "f"(d));
}
template <bool kE5>
__device__ __forceinline__ uint32_t q_pack2(float a, float b, float f)
{
    mul2(a, b, f);
    return f8_pack<kE5>(a, b);
}

// 8 x 8 entries in registers, bfloat16 as they come (two to a word), so that four CTAs fit an SM (three: 28.2 us for 8192 x 4096 in both orientations, four 26.7).
template <typename T>
struct QEntries {
    static constexpr int kWords = sizeof(T) == 2 ? 4 : 8;          // words of eight entries
    uint32_t w[8][kWords];

    __device__ __forceinline__ float at(int j, int i) const
    {
        if constexpr (sizeof(T) == 2) return i & 1 ? bf16_hi(w[j][i >> 1]) : bf16_lo(w[j][i >> 1]);
        else return __uint_as_float(w[j][i]);
    }
    __device__ __forceinline__ void load(int j, const T *p)
    {
        const uint4 a = load_free((const uint4 *)p);
        w[j][0] = a.x; w[j][1] = a.y; w[j][2] = a.z; w[j][3] = a.w;
        if constexpr (sizeof(T) == 4) {
            const uint4 b = load_free((const uint4 *)p + 1);
            w[j][4] = b.x; w[j][5] = b.y; w[j][6] = b.z; w[j][7] = b.w;
        }
    }
    __device__ __forceinline__ void load_some(int j, const T *p, int64_t n)      // n entries, which may be none, from anywhere
    {
        if constexpr (sizeof(T) == 2) {
            // whole words, each of which holds an entry of the eight
            if (n >= 8) {
                const uint32_t odd = ((uint32_t)(uintptr_t)p & 2u) << 3, *q = (const uint32_t *)((uintptr_t)p & ~(uintptr_t)3);
                uint32_t a[5];
#pragma unroll
                for (int k = 0; k < 5; ++k) a[k] = k < 4 || odd ? load_free(q + k) : 0u;
#pragma unroll
                for (int k = 0; k < 4; ++k) w[j][k] = __funnelshift_r(a[k], a[k + 1], odd);
                return;
            }
        }
#pragma unroll
        for (int k = 0; k < kWords; ++k) {
            if constexpr (sizeof(T) == 2) {
                const uint32_t lo = 2 * k < n ? (uint32_t)*((const uint16_t *)p + 2 * k) : 0u, hi = 2 * k + 1 < n ? (uint32_t)*((const uint16_t *)p + 2 * k + 1) : 0u;
                w[j][k] = lo | hi << 16;
            } else w[j][k] = k < n ? *((const uint32_t *)p + k) : 0u;
        }
    }
    __device__ __forceinline__ void drop(int jh, int ih)                          // 4 x 4 entries become zeros
    {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < kWords / 2; ++k) w[jh + j][ih * kWords / 8 + k] = 0u;
    }
    // Infinities become NaN, so that they neither enter a scale nor come out as the format's largest value.
    __device__ __forceinline__ void no_infinity()
    {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int k = 0; k < kWords; ++k) {
                if constexpr (sizeof(T) == 2) {
                    if ((w[j][k] & 0x7FFFu) == 0x7F80u) w[j][k] |= 0x7Fu;
                    if ((w[j][k] & 0x7FFF0000u) == 0x7F800000u) w[j][k] |= 0x7F0000u;
                } else if ((w[j][k] & 0x7FFFFFFFu) == 0x7F800000u) w[j][k] |= 0x7FFFFFu;
            }
    }
    // Largest magnitudes of the rows over the 16 lanes that share them (NaN is passed by).
    __device__ __forceinline__ void row_max(float (&m)[8]) const
    {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                uint32_t a[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t x = bf16_max2(w[j + h][0] & 0x7FFF7FFFu, w[j + h][1] & 0x7FFF7FFFu);
                    x = bf16_max2(x, bf16_max2(w[j + h][2] & 0x7FFF7FFFu, w[j + h][3] & 0x7FFF7FFFu));
                    a[h] = x;
                }
                // (the first row's two halves against the second row's: one word with a row in each half)
                uint32_t r = bf16_max2(__byte_perm(a[0], a[1], 0x5410), __byte_perm(a[0], a[1], 0x7632));
#pragma unroll
                for (int d = 8; d > 0; d >>= 1) r = bf16_max2(r, __shfl_xor_sync(0xFFFFFFFFu, r, d));
                r = bf16_max2(r, 0u);                              // (rows of nothing but NaN)
                m[j] = bf16_lo(r); m[j + 1] = bf16_hi(r);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float x = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) x = fmaxf(x, fabsf(at(j, i)));
#pragma unroll
                for (int d = 8; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, d));
                m[j] = x;
            }
        }
    }
    // Largest magnitudes of the columns over the rows of a warp.
    __device__ __forceinline__ void col_max(float (&m)[8]) const
    {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t x = 0u;
#pragma unroll
                for (int j = 0; j < 8; ++j) x = bf16_max2(x, w[j][k] & 0x7FFF7FFFu);
                x = bf16_max2(x, __shfl_xor_sync(0xFFFFFFFFu, x, 16));
                m[2 * k] = bf16_lo(x); m[2 * k + 1] = bf16_hi(x);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float x = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) x = fmaxf(x, fabsf(at(j, i)));
                m[i] = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 16));
            }
        }
    }
};

template <typename T, bool kE5, bool kWeights>
__global__ void __launch_bounds__(kQThreads, sizeof(T) == 2 ? 4 : 2) quantize_f8_kernel(const QParams p)
{
    __shared__ __align__(16) uint8_t s_cols[kF8Block * kF8Block];
    __shared__ __align__(16) float s_max[8][kF8Block], s_sum[8][kF8Block];
    __shared__ __align__(16) float s_inv[kF8Block];
    __shared__ uint8_t s_row[kF8Block];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, tx = tid & 15, ty = tid >> 4;
    const int64_t ti = (int64_t)blockIdx.x % p.tiles_i, tp = (int64_t)blockIdx.x / p.tiles_i;
    const int64_t c0 = ti * kF8Block + tx * 8, r0 = tp * kF8Block + ty * 8;
    wait_for_previous();
    const T *X = from_here((const T *)p.X) + r0 * p.ldx + c0;

    QEntries<T> v;
    if (p.vec && (tp + 1) * kF8Block <= p.P && (ti + 1) * kF8Block <= p.I) {         // (all loads ahead of their first use)
#pragma unroll
        for (int j = 0; j < 8; ++j) v.load(j, X + j * p.ldx);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t n = r0 + j < p.P ? p.I - c0 : 0;
            if (p.vec && n >= 8) v.load(j, X + j * p.ldx);
            else v.load_some(j, X + j * p.ldx, n);
        }
    }
    if constexpr (kWeights) {
        // a block of Gamma covers whole groups of four rows and of four columns, whatever its shape; dropped weights are zeros, whatever
        // they hold
        if (p.gamma != nullptr) {
            const uint8_t *gamma = from_here(p.gamma);
#pragma unroll
            for (int jh = 0; jh < 8; jh += 4)
#pragma unroll
                for (int ih = 0; ih < 8; ih += 4)
                    if (r0 + jh < p.P && c0 + ih < p.I && load_free(gamma + ((r0 + jh) >> p.bo) * p.NBi + ((c0 + ih) >> p.bi)) == 0u) v.drop(jh, ih);
        }
    }
    if (p.partial != nullptr) {
        float s[8];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            s[i] = s[i + 1] = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) add2(s[i], s[i + 1], v.at(j, i), v.at(j, i + 1));
            s[i] += __shfl_xor_sync(0xFFFFFFFFu, s[i], 16);
            s[i + 1] += __shfl_xor_sync(0xFFFFFFFFu, s[i + 1], 16);
        }
        if (lane < 16) {
            *(float4 *)&s_sum[warp][tx * 8] = make_float4(s[0], s[1], s[2], s[3]);
            *(float4 *)&s_sum[warp][tx * 8 + 4] = make_float4(s[4], s[5], s[6], s[7]);
        }
    }
    float rmax[8];
    v.row_max(rmax);
    bool inf = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) inf |= rmax[j] == __uint_as_float(0x7F800000u);
    if (__any_sync(0xFFFFFFFFu, inf)) {
        v.no_infinity();
        v.row_max(rmax);
    }
    if constexpr (kWeights) {
        // one scale for the tile
        float m = rmax[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) m = fmaxf(m, rmax[j]);
        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
        if (lane == 0) s_max[0][warp] = m;
        __syncthreads();
        m = s_max[0][0];
#pragma unroll
        for (int w = 1; w < 8; ++w) m = fmaxf(m, s_max[0][w]);
#pragma unroll
        for (int j = 0; j < 8; ++j) rmax[j] = m;
    } else if (p.cols != nullptr) {
        float m[8];
        v.col_max(m);
        if (lane < 16) {
            *(float4 *)&s_max[warp][tx * 8] = make_float4(m[0], m[1], m[2], m[3]);
            *(float4 *)&s_max[warp][tx * 8 + 4] = make_float4(m[4], m[5], m[6], m[7]);
        }
    }

    // rows form: eight bytes a thread and row, 128 bytes a row of the tile
    if (p.rows != nullptr) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t b = f8_scale_byte<kE5>(__float_as_uint(rmax[j]));
            const float f = f8_inverse(b);
            uint2 w;
            w.x = q_pack2<kE5>(v.at(j, 0), v.at(j, 1), f) | q_pack2<kE5>(v.at(j, 2), v.at(j, 3), f) << 16;
            w.y = q_pack2<kE5>(v.at(j, 4), v.at(j, 5), f) | q_pack2<kE5>(v.at(j, 6), v.at(j, 7), f) << 16;
            if (r0 + j < p.P && c0 < p.rows_pitch) *(uint2 *)(p.rows + (r0 + j) * p.rows_pitch + c0) = w;
            if (tx == 0) s_row[ty * 8 + j] = (uint8_t)b;
        }
    }
    __syncthreads();
    if (tid < kF8Block) {
        const int64_t c = ti * kF8Block + tid;
        // (the scales reach whole groups of 128 rows, in either orientation; four instructions for a tile's instead of 64: 26.7 -> 24.6 us)
        if (p.rows != nullptr) p.rows_scale[f8_scale_at(tp * kF8Block + tid, ti, p.rows_atoms)] = s_row[tid];
        if (p.cols != nullptr) {
            float m = rmax[0];
            if constexpr (!kWeights) {
                m = s_max[0][tid];
#pragma unroll
                for (int w = 1; w < 8; ++w) m = fmaxf(m, s_max[w][tid]);
            }
            const uint32_t b = f8_scale_byte<kE5>(__float_as_uint(m));
            s_inv[tid] = f8_inverse(b);
            p.cols_scale[f8_scale_at(c, tp, p.cols_atoms)] = (uint8_t)b;
        }
        if (p.partial != nullptr && c < p.I) {
            float s = s_sum[0][tid];
#pragma unroll
            for (int w = 1; w < 8; ++w) s += s_sum[w][tid];
            p.partial[tp * p.I + c] = s;
        }
    }
    if (p.cols == nullptr) return;
    __syncthreads();
    // transposed form: the eight bytes of a column's rows to shared memory, 8-byte piece ty of column c at place ty ^ (c / 8) so that the
    // lanes of a half warp, eight columns apart, meet different banks
    float inv[8];
    *(float4 *)&inv[0] = *(const float4 *)&s_inv[tx * 8];
    *(float4 *)&inv[4] = *(const float4 *)&s_inv[tx * 8 + 4];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float f = inv[i];
        uint2 w;
        w.x = q_pack2<kE5>(v.at(0, i), v.at(1, i), f) | q_pack2<kE5>(v.at(2, i), v.at(3, i), f) << 16;
        w.y = q_pack2<kE5>(v.at(4, i), v.at(5, i), f) | q_pack2<kE5>(v.at(6, i), v.at(7, i), f) << 16;
        *(uint2 *)(s_cols + (tx * 8 + i) * kF8Block + ((ty ^ tx) << 3)) = w;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int piece = u * kQThreads + tid, col = piece >> 3, at = piece & 7, x = col >> 3;
        const int64_t c = ti * kF8Block + col, r = tp * kF8Block + at * 16;
        uint4 w = *(const uint4 *)(s_cols + col * kF8Block + ((at ^ (x >> 1)) << 4));
        if (x & 1) w = make_uint4(w.z, w.w, w.x, w.y);
        if (c < p.I && r < p.cols_pitch) *(uint4 *)(p.cols + c * p.cols_pitch + r) = w;
    }
}

// Sums of the tiles' column sums, in the order of the tiles.
__global__ void __launch_bounds__(256) colsum_kernel(const float *partial, int64_t tiles, int64_t I, float *out)
{
    __shared__ float s[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    wait_for_previous();
    partial = from_here(partial);
    float sum = 0.f;
    if (c < I)
        for (int64_t t = warp; t < tiles; t += 8) sum += __uint_as_float(load_free((const uint32_t *)(partial + t * I + c)));
    s[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && c < I) {
#pragma unroll
        for (int w = 1; w < 8; ++w) sum += s[w][lane];
        out[c] = sum;
    }
}

// ---- back ----

struct DParams {
    const uint8_t *data, *scale;
    int64_t rows, cols, pitch, atoms, ldx, tiles;
    void *X;
    int vec;
};

// 16 bytes of a row of X (eight bfloat16 entries, four float32); `n` entries exist.
__device__ __forceinline__ void d_store(__nv_bfloat16 *x, const float (&v)[8], int n, int vec)
{
    if (vec && n >= 8) {
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            o[i] = *(const uint32_t *)&h;
        }
        *(uint4 *)x = make_uint4(o[0], o[1], o[2], o[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) x[i] = __float2bfloat16_rn(v[i]);
    }
}
__device__ __forceinline__ void d_store(float *x, const float (&v)[4], int n, int vec)
{
    if (vec && n >= 4) *(float4 *)x = make_float4(v[0], v[1], v[2], v[3]);
    else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) x[i] = v[i];
    }
}
// kBytes 8-bit values of a row; the pitch of the rows is a multiple of 16, so all of them lie in it.
template <int kBytes>
__device__ __forceinline__ void d_load(const uint8_t *p, uint32_t (&w)[kBytes / 4])
{
    if constexpr (kBytes == 4) w[0] = load_free((const uint32_t *)p);
    else if constexpr (kBytes == 8) { const uint2 a = load_free((const uint2 *)p); w[0] = a.x; w[1] = a.y; }
    else { const uint4 a = load_free((const uint4 *)p); w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; }
}

// A tile of 128 x 128 per CTA, 64 entries a thread, in stores of 16 bytes that lie side by side.  As it lies: a thread takes 16 bytes of X
// of eight rows (16 of float32), whose lanes cover 128 columns.  Transposed: of as many columns, and a warp covers 64 rows x 32 columns,
// so that it reads whole sectors of 32 bytes and writes 128 bytes of a row of X or more at once.
// kWide (bfloat16, transposed; 128 threads): 128 entries a thread, so that a warp covers 128 rows and writes 256 bytes side by side: 11.7 -> 10.1 us
// for 4096 x 4096, but 2.2 -> 2.6 for 64 x 2048, whose few CTAs have fewer threads then (kWideTiles).
template <typename T, bool kE5, bool kTranspose, bool kWide>
__global__ void __launch_bounds__(256) dequantize_f8_kernel(const DParams p)
{
    constexpr int kV = 16 / sizeof(T), kN = kWide ? 16 : 64 / kV;
    constexpr int kRows = kTranspose ? kV : kN, kCols = kTranspose ? kN : kV;      // of the matrix, to a thread
    constexpr int kAcross = (kTranspose ? 32 : 128) / kCols;                        // lanes side by side
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = (kTranspose ? (warp & 3) * 32 : 0) + lane % kAcross * kCols;
    const int row = (kTranspose ? (warp >> 2) * (32 / kAcross * kRows) : warp * 16) + lane / kAcross * kRows;
    const int64_t tk = (int64_t)blockIdx.x % p.tiles, tr = (int64_t)blockIdx.x / p.tiles;
    const int64_t k0 = tk * kF8Block + col, r0 = tr * kF8Block + row;
    wait_for_previous();
    if (k0 >= p.cols || r0 >= p.rows) return;
    const int nk = p.cols - k0 < kCols ? (int)(p.cols - k0) : kCols, nr = p.rows - r0 < kRows ? (int)(p.rows - r0) : kRows;
    const uint8_t *data = from_here(p.data) + r0 * p.pitch + k0, *scale = from_here(p.scale) + f8_scale_at(r0, tk, p.atoms);
    uint32_t w[kRows][kCols / 4], b[kRows];
#pragma unroll
    for (int j = 0; j < kRows; ++j) {                   // (the scales of a thread's rows, which lie in one group of 32, are 16 bytes apart)
        if (j < nr) d_load<kCols>(data + j * p.pitch, w[j]);
        else
#pragma unroll
            for (int i = 0; i < kCols / 4; ++i) w[j][i] = 0u;
        b[j] = load_free(scale + j * 16);
    }
    T *X = (T *)p.X;
    if constexpr (!kTranspose) {
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
            if (j >= nr) break;
            const float f = f8_scale(b[j]);
            float v[kV];
#pragma unroll
            for (int i = 0; i < kV; i += 2) {
                const float2 a = f8_unpack<kE5>(w[j][i / 4] >> (8 * (i & 2)) & 0xFFFFu);
                v[i] = a.x * f; v[i + 1] = a.y * f;
            }
            d_store(X + (r0 + j) * p.ldx + k0, v, nk, p.vec);
        }
    } else {
        float f[kRows];
#pragma unroll
        for (int j = 0; j < kRows; ++j) f[j] = f8_scale(b[j]);
#pragma unroll
        for (int i = 0; i < kCols; i += 2) {
            float lo[kV], hi[kV];
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const float2 t = f8_unpack<kE5>(w[j][i / 4] >> (8 * (i & 2)) & 0xFFFFu);
                lo[j] = t.x * f[j]; hi[j] = t.y * f[j];
            }
            if (i < nk) d_store(X + (k0 + i) * p.ldx + r0, lo, nr, p.vec);
            if (i + 1 < nk) d_store(X + (k0 + i + 1) * p.ldx + r0, hi, nr, p.vec);
        }
    }
}

// The same for rows of X that cannot be written 16 bytes at a time: a lane takes an aligned word of a row of X, so that a warp writes 128 bytes
// side by side wherever the row begins.  As it lies: two bfloat16 columns (or one float32) of a row; transposed: two rows (one) of the
// matrix for 16 columns, where a word may hold the second entry of the lane before.
template <typename T, bool kE5, bool kTranspose>
__global__ void __launch_bounds__(256) dequantize_f8_any_kernel(const DParams p)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t tk = (int64_t)blockIdx.x % p.tiles, tr = (int64_t)blockIdx.x / p.tiles, k0 = tk * kF8Block, r0 = tr * kF8Block;
    wait_for_previous();
    const uint8_t *data = from_here(p.data), *scale = from_here(p.scale);
    const int nk = p.cols - k0 < kF8Block ? (int)(p.cols - k0) : kF8Block, nr = p.rows - r0 < kF8Block ? (int)(p.rows - r0) : kF8Block;
    constexpr int kPer = 4 / sizeof(T);                 // entries of a word
    if constexpr (!kTranspose) {
        // (a lane holds four columns of a row and hands them to the lanes that write them)
#pragma unroll 4
        for (int j = warp; j < nr; j += 8) {
            T *x = (T *)p.X + (r0 + j) * p.ldx + k0;
            const uint32_t mine = lane * 4 < nk ? load_free((const uint32_t *)(data + (r0 + j) * p.pitch + k0) + lane) : 0u;
            const float f = f8_scale(load_free(scale + f8_scale_at(r0 + j, tk, p.atoms)));
            const int odd = sizeof(T) == 2 ? (int)((uintptr_t)x >> 1 & 1) : 0;
#pragma unroll
            for (int i = 0; i < 128 / (32 * kPer) + (kPer == 2 ? 1 : 0); ++i) {
                const int c = (i * 32 + lane) * kPer - odd;
                if (i * 32 * kPer - odd >= nk) break;
                float v[kPer];
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    v[e] = f8_unpack<kE5>(__shfl_sync(0xFFFFFFFFu, mine, (c + e) >> 2 & 31) >> (8 * ((c + e) & 3)) & 0xFFu).x * f;
                if constexpr (kPer == 1) { if (c < nk) x[c] = v[0]; }
                else if (c >= 0 && c + 1 < nk) {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(v[0], v[1]);
                    *(uint32_t *)(x + c) = *(const uint32_t *)&h;
                } else {
                    if (c >= 0 && c < nk) x[c] = __float2bfloat16_rn(v[0]);
                    if (c + 1 >= 0 && c + 1 < nk) x[c + 1] = __float2bfloat16_rn(v[1]);
                }
            }
        }
    } else {
        // a warp: 16 columns of 32 kPer rows, then of the next 32 kPer
        const int c0 = warp * 16;
        if (c0 >= nk) return;
        for (int i = 0; i < 128 / (32 * kPer); ++i) {
            const int r = (i * 32 + lane) * kPer;
            uint4 w[kPer];
            float f[kPer];
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                w[e] = r + e < nr ? load_free((const uint4 *)(data + (r0 + r + e) * p.pitch + k0 + c0)) : make_uint4(0u, 0u, 0u, 0u);
                f[e] = r + e < nr ? f8_scale(load_free(scale + f8_scale_at(r0 + r + e, tk, p.atoms))) : 0.f;
            }
#pragma unroll
            for (int c = 0; c < 16; ++c) {
                if (c0 + c >= nk) break;
                T *x = (T *)p.X + (k0 + c0 + c) * p.ldx + r0 + r;
                float v[kPer];
#pragma unroll
                for (int e = 0; e < kPer; ++e) v[e] = f8_unpack<kE5>((c < 4 ? w[e].x : c < 8 ? w[e].y : c < 12 ? w[e].z : w[e].w) >> (8 * (c & 3)) & 0xFFu).x * f[e];
                if constexpr (kPer == 1) { if (r < nr) *x = v[0]; }
                else {
                    const __nv_bfloat16 own = __float2bfloat16_rn(v[0]), second = __float2bfloat16_rn(v[1]);
                    const uint32_t lo = __bfloat16_as_ushort(own), hi = __bfloat16_as_ushort(second), before = __shfl_up_sync(0xFFFFFFFFu, hi, 1);
                    if (((uintptr_t)x & 2u) == 0u) {
                        if (r + 1 < nr) *(uint32_t *)x = lo | hi << 16;
                        else if (r < nr) *x = own;
                    } else {
                        if (r < nr) {
                            if (lane > 0) *(uint32_t *)(x - 1) = before | lo << 16;
                            else *x = own;
                        } else if (lane > 0 && r - 1 < nr) *(x - 1) = __ushort_as_bfloat16((unsigned short)before);
                        if (lane == 31 && r + 1 < nr) x[1] = second;
                    }
                }
            }
        }
    }
}

// Tiles above which the wide form of the transposed bfloat16 restore is taken: two for each of 148 SMs, as many CTAs as fit beside the waiting ones of the
// kernel that follows.  Measured on 16 to 2048 tiles, us narrow and wide, in a row and (in brackets) with another kernel between: 128 tiles 3.4 and 3.8
// (5.6 and 6.0), 256 tiles 4.66 and 4.71 (6.8 and 6.9), 288 4.8 and 4.9 (7.0 and 7.0), 320 6.5 and 5.5 (7.8 and 7.7), 512 7.0 and 7.6 (9.2 and 8.8), 784 9.8
// and 8.5 (12.0 and 10.6), 1024 11.7 and 10.1 (13.9 and 12.6).
constexpr int64_t kWideTiles = 296;

bool rows_of_16(const void *X, int64_t ldx, int esz) { return ((uintptr_t)X & 15u) == 0 && ldx * esz % 16 == 0; }

}  // namespace

bsp_status launch_quantize_f8(const void *X, bsp_dtype xtype, int64_t P, int64_t I, int64_t ldx, const bsp_wdesc *wd, const uint8_t *gamma,
                              const bsp_f8 *rows, const bsp_f8 *cols, float *colsum, void *ws, cudaStream_t st)
{
    QParams p = {};
    p.X = X; p.P = P; p.I = I; p.ldx = ldx;
    p.vec = rows_of_16(X, ldx, elem_bytes(xtype));
    if (rows) { p.rows = (uint8_t *)rows->data; p.rows_scale = (uint8_t *)rows->scale; p.rows_pitch = f8_pitch(I); p.rows_atoms = f8_atoms(I); }
    if (cols) { p.cols = (uint8_t *)cols->data; p.cols_scale = (uint8_t *)cols->scale; p.cols_pitch = f8_pitch(P); p.cols_atoms = f8_atoms(P); }
    if (colsum) p.partial = (float *)((char *)ws + kWsHeader);
    if (wd) { p.gamma = gamma; p.bo = f8_log2(wd->bo); p.bi = f8_log2(wd->bi); p.NBi = wd->I / wd->bi; }
    p.tiles_i = f8_blocks(I);
    const int64_t tiles_p = f8_blocks(P), tiles = p.tiles_i * tiles_p;
    if (tiles > 0x7FFFFFFF) return BSP_ERR_SHAPE;
    const bool e5 = (rows ? rows->type : cols ? cols->type : BSP_E4M3) == BSP_E5M2, half = xtype == BSP_BF16;
    typedef void (*Kernel)(const QParams);
    static const Kernel kernels[2][2][2] = {
        {{quantize_f8_kernel<float, false, false>, quantize_f8_kernel<float, false, true>}, {quantize_f8_kernel<float, true, false>, quantize_f8_kernel<float, true, true>}},
        {{quantize_f8_kernel<__nv_bfloat16, false, false>, quantize_f8_kernel<__nv_bfloat16, false, true>},
         {quantize_f8_kernel<__nv_bfloat16, true, false>, quantize_f8_kernel<__nv_bfloat16, true, true>}}};
    BSP_CUDA_OK(launch_after(kernels[half][e5][wd != nullptr], dim3((unsigned)tiles), dim3(kQThreads), 0, st, p));
    if (colsum) BSP_CUDA_OK(launch_after(colsum_kernel, dim3((unsigned)((I + 31) / 32)), dim3(256), 0, st, (const float *)p.partial, tiles_p, I, colsum));
    return BSP_OK;
}

bsp_status launch_dequantize_f8(const bsp_f8 &m, void *X, bsp_dtype xtype, int64_t ldx, bool transpose, cudaStream_t st)
{
    DParams p = {};
    p.data = (const uint8_t *)m.data; p.scale = (const uint8_t *)m.scale;
    p.rows = m.rows; p.cols = m.cols; p.pitch = f8_pitch(m.cols); p.atoms = f8_atoms(m.cols); p.ldx = ldx; p.X = X;
    p.vec = rows_of_16(X, ldx, elem_bytes(xtype));
    p.tiles = f8_blocks(m.cols);
    const int64_t tiles = p.tiles * f8_blocks(m.rows);
    if (tiles > 0x7FFFFFFF) return BSP_ERR_SHAPE;
    typedef void (*Kernel)(const DParams);
    static const Kernel kernels[2][2][2] = {
        {{dequantize_f8_kernel<float, false, false, false>, dequantize_f8_kernel<float, false, true, false>},
         {dequantize_f8_kernel<float, true, false, false>, dequantize_f8_kernel<float, true, true, false>}},
        {{dequantize_f8_kernel<__nv_bfloat16, false, false, false>, dequantize_f8_kernel<__nv_bfloat16, false, true, false>},
         {dequantize_f8_kernel<__nv_bfloat16, true, false, false>, dequantize_f8_kernel<__nv_bfloat16, true, true, false>}}};
    if (p.vec && transpose && xtype == BSP_BF16 && tiles > kWideTiles) {
        BSP_CUDA_OK(launch_after(m.type == BSP_E5M2 ? dequantize_f8_kernel<__nv_bfloat16, true, true, true> : dequantize_f8_kernel<__nv_bfloat16, false, true, true>,
                                 dim3((unsigned)tiles), dim3(128), 0, st, p));
        return BSP_OK;
    }
    static const Kernel any[2][2][2] = {
        {{dequantize_f8_any_kernel<float, false, false>, dequantize_f8_any_kernel<float, false, true>}, {dequantize_f8_any_kernel<float, true, false>, dequantize_f8_any_kernel<float, true, true>}},
        {{dequantize_f8_any_kernel<__nv_bfloat16, false, false>, dequantize_f8_any_kernel<__nv_bfloat16, false, true>},
         {dequantize_f8_any_kernel<__nv_bfloat16, true, false>, dequantize_f8_any_kernel<__nv_bfloat16, true, true>}}};
    BSP_CUDA_OK(launch_after((p.vec ? kernels : any)[xtype == BSP_BF16][m.type == BSP_E5M2][transpose], dim3((unsigned)tiles), dim3(256), 0, st, p));
    return BSP_OK;
}

}  // namespace bsp
