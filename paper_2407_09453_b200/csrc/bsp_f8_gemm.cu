// Products of 8-bit floating-point matrices with a power-of-two scale for 128 entries of the summed axis, on 5th-generation tensor cores:
// Y[m][n] = bias[n] + sum_k x[m][k] w[n][k] (the forward pass and the gradient of the input of a linear layer, whose operands differ only in
// which orientation they were quantised in) and dW[o][i] = Gamma * sum_p dy[o][p] x[i][p] (the gradient of the kept weights from
// the 8-bit checkpoints).  Introduction (Y = W*X + b), Section "Training and Quantization" and Section "Compiler and its Code
// generation" (8-bit tensors with power-of-two scales) of the paper.
//
// tcgen05.mma kind::mxf8f6f4 multiplies 128 x BN x 32 entries and applies one scale byte per row and 32 entries of either operand itself, with
// sums in float32: a block of 128 entries is four MMAs with the same scale byte (the instruction names one of the four bytes in
// a tensor-memory column).  So the scales cost one tcgen05.cp of 512 bytes per 128 rows and 512 entries, and no arithmetic on
// the accumulators.
#include "bsp_f8.cuh"
#include "bsp_tc.cuh"

namespace bsp {
namespace {

constexpr int kFsThreads = 256;                     // producer warp, MMA warp, two idle warps until the store, four epilogue warps
constexpr int kFsScaleBytes = 3 * kF8Atom;          // scales of a stage: 128 rows of A, up to 256 rows of B
constexpr int kFsMaxStages = 8;
constexpr int kFsSets = 4;                          // scale sets in tensor memory, 16 columns each (A 4, B up to 8)
constexpr int kFsSmem = 227 * 1024;
static_assert(kFsMaxStages <= 4 * (kFsSets - 1) + 1, "a set is written again only when the MMAs that read it are done: the ring's barriers see to that");

struct FsParams {
    CUtensorMap tma, tmb;         // values as bytes, (K, rows), box 128 x 128 and 128 x BN, 128-byte swizzle; zeros past the ends
    const uint8_t *sa, *sb;       // scales
    int64_t atoms;                // atoms per 128 rows
    int M, N, BN, n_kb, tiles_n, split, stages, stage_bytes;
    uint32_t idesc;
    int a_e5, b_e5;
    uint8_t *Y;
    int bf16, transposed, vec;    // element (m, n) at Y[m N + n], or at Y[n M + m]
    const float *bias;
    const uint8_t *gamma;
    int bo, bi, NBi;
    int *status;
};

struct FsTail {
    uint64_t full[kFsMaxStages], empty[kFsMaxStages], acc;
    uint32_t tmem, fail;
};

// Four partial sums of this CTA's tile or of the same tile in another CTA of the cluster.
__device__ __forceinline__ float4 fs_peer4(uint32_t addr, uint32_t rank)
{
    float4 v;
    asm volatile("{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %4, %5;\n ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n}\n"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr), "r"(rank) : "memory");
    return v;
}

// One tile of 128 x BN per cluster; CTA r of the cluster sums its share of the blocks, and the shares are added up in the order of the
// ranks through distributed shared memory.
__global__ void __launch_bounds__(kFsThreads, 1) gemm_f8_kernel(const __grid_constant__ FsParams p)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    FsTail &tail = *(FsTail *)(smem + (size_t)p.stages * (p.stage_bytes + kFsScaleBytes));
    volatile uint32_t &s_fail = tail.fail;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
    const int S = p.stages, split = p.split, tile = (int)blockIdx.x / split, rank = (int)blockIdx.x - tile * split;
    const int tm = tile / p.tiles_n, tn = tile - tm * p.tiles_n, m0 = tm * 128, n0 = tn * p.BN, BN = p.BN;
    const int kb0 = (int)((long long)p.n_kb * rank / split), kb1 = (int)((long long)p.n_kb * (rank + 1) / split);
    const uint32_t ring = sm32(smem), scales = ring + (uint32_t)(S * p.stage_bytes);
    const uint32_t cols = BN + 64 <= 128 ? 128u : BN + 64 <= 256 ? 256u : 512u;

    if (tid == 0) {
        for (int s = 0; s < S; ++s) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(sm32(&tail.full[s])), "r"(1) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(sm32(&tail.empty[s])), "r"(1) : "memory");
        }
        asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(sm32(&tail.acc)), "r"(1) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        s_fail = (ring & 1023u) == 0u ? 0u : 2u;
        asm volatile("prefetch.tensormap [%0];\n" ::"l"(&p.tma) : "memory");
        asm volatile("prefetch.tensormap [%0];\n" ::"l"(&p.tmb) : "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(sm32(&tail.tmem)), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    wait_for_previous<false>();
    if (warp == 0) let_next_start();
    if (tid == 0 && s_fail) atomicMax(p.status, (int)BSP_ERR_CUDA);
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, tail.tmem, 0), sf = tmem + cols - 64u;
    const bool run = __shfl_sync(0xFFFFFFFFu, s_fail, 0) == 0u;
    const uint32_t full0 = sm32(&tail.full[0]), empty0 = sm32(&tail.empty[0]);
    // atoms of B's scales: those of the tile's rows, of which the second may not exist
    const int at_b = n0 >> 7, two = BN > 128 && n0 + 128 < p.N ? 1 : 0;

    if (warp == 0) {
        // ================= producer =================
        if (run) {
            const uint8_t *sa = p.sa + (int64_t)tm * p.atoms * kF8Atom, *sb = p.sb + (int64_t)at_b * p.atoms * kF8Atom, *sb2 = sb + p.atoms * kF8Atom;
            uint32_t slot = 0, par = 1, issued = 0;
            bool ok = true;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!__all_sync(0xFFFFFFFFu, gt_poll(empty0 + slot * 8u, par)) || s_fail) { ok = false; break; }
                const uint32_t with_scales = kb == kb0 || (kb & 3) == 0 ? 1u : 0u, dst = ring + slot * (uint32_t)p.stage_bytes, sdst = scales + slot * kFsScaleBytes;
                const uint32_t bytes = (uint32_t)p.stage_bytes + with_scales * (uint32_t)((2 + two) * kF8Atom);
                const int64_t at = (int64_t)(kb >> 2) * kF8Atom;
                asm volatile("{\n .reg .pred e, s, t;\n elect.sync _|e, 0xFFFFFFFF;\n setp.ne.b32 s, %9, 0;\n and.pred s, s, e;\n setp.ne.b32 t, %10, 0;\n and.pred t, t, s;\n"
                             " @e mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n"
                             " @e cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%2], [%3, {%4, %5}], [%0];\n"
                             " @e cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%6], [%7, {%4, %8}], [%0];\n"
                             " @s cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%11], [%12], 512, [%0];\n"
                             " @s cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%13], [%14], 512, [%0];\n"
                             " @t cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%15], [%16], 512, [%0];\n}\n"
                             ::"r"(full0 + slot * 8u), "r"(bytes), "r"(dst), "l"(&p.tma), "r"(kb * 128), "r"(m0), "r"(dst + 16384u), "l"(&p.tmb), "r"(n0),
                               "r"(with_scales), "r"(two), "r"(sdst), "l"(sa + at), "r"(sdst + 512u), "l"(sb + at), "r"(sdst + 1024u), "l"(sb2 + at) : "memory");
                ++issued;
                if (++slot == (uint32_t)S) { slot = 0; par ^= 1u; }
            }
            if (!ok && lane == 0) {
                // a wait ran out: the loads in flight still write into this CTA's memory
                atomicExch(&tail.fail, 1u);
                for (uint32_t back = 0; back < (uint32_t)S && back < issued; ++back) {
                    const uint32_t it = issued - 1u - back;
                    gt_poll(full0 + (it % (uint32_t)S) * 8u, (it / (uint32_t)S) & 1u);
                }
            }
        }
    } else if (warp == 1) {
        // ================= MMA issuer =================
        if (run) {
            uint32_t slot = 0, par = 0, set = 0, acc = 0;
            bool ok = true;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!gt_poll_stage(full0 + slot * 8u, par)) { ok = false; break; }
                const uint32_t with_scales = kb == kb0 || (kb & 3) == 0 ? 1u : 0u;
                if (with_scales && kb != kb0) set = set + 1u == kFsSets ? 0u : set + 1u;
                const uint32_t a16 = (ring + slot * (uint32_t)p.stage_bytes) >> 4, s16 = (scales + slot * kFsScaleBytes) >> 4;
                const uint64_t da = kGtDesc | (uint64_t)(a16 & 0x3FFFu), db = kGtDesc | (uint64_t)((a16 + 1024u) & 0x3FFFu);
                // scales: 32 rows of 16 bytes without swizzle, groups of eight rows 128 bytes apart
                const uint64_t ds = (1ull << 16) | (8ull << 32) | (1ull << 46) | (uint64_t)(s16 & 0x3FFFu);
                const uint32_t fa = sf + set * 16u, fb = fa + 8u, id = (uint32_t)kb & 3u;
                const uint32_t idesc = p.idesc | (id << 4) | (id << 29);
                asm volatile("{\n .reg .pred e, s, t, p, q;\n .reg .b64 a1, a2, a3, b1, b2, b3, s1, s2;\n .reg .b32 f2;\n"
                             " elect.sync _|e, 0xFFFFFFFF;\n setp.ne.b32 s, %8, 0;\n and.pred s, s, e;\n setp.ne.b32 t, %9, 0;\n and.pred t, t, s;\n"
                             " setp.ne.b32 p, %10, 0;\n setp.eq.b32 q, %10, %10;\n"
                             " add.u64 s1, %4, 32;\n add.u64 s2, %4, 64;\n add.u32 f2, %6, 4;\n"
                             " @s tcgen05.cp.cta_group::1.32x128b.warpx4 [%5], %4;\n"
                             " @s tcgen05.cp.cta_group::1.32x128b.warpx4 [%6], s1;\n"
                             " @t tcgen05.cp.cta_group::1.32x128b.warpx4 [f2], s2;\n"
                             " add.u64 a1, %1, 2;\n add.u64 a2, %1, 4;\n add.u64 a3, %1, 6;\n"
                             " add.u64 b1, %2, 2;\n add.u64 b2, %2, 4;\n add.u64 b3, %2, 6;\n"
                             " @e tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%5], [%6], p;\n"
                             " @e tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a1, b1, %3, [%5], [%6], q;\n"
                             " @e tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a2, b2, %3, [%5], [%6], q;\n"
                             " @e tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a3, b3, %3, [%5], [%6], q;\n"
                             " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%7];\n}\n"
                             ::"r"(tmem), "l"(da), "l"(db), "r"(idesc), "l"(ds), "r"(fa), "r"(fb), "r"(empty0 + slot * 8u), "r"(with_scales), "r"(two), "r"(acc)
                             : "memory");
                acc = 1u;
                if (++slot == (uint32_t)S) { slot = 0; par ^= 1u; }
            }
            if (ok) gt_commit_elected<false>(sm32(&tail.acc));
            else if (lane == 0) atomicExch(&tail.fail, 1u);
        }
    } else if (warp >= 4) {
        // ================= accumulators to shared memory =================
        // (All MMAs are done, so the ring is free.)  Rows of n for an output whose rows are n, pitch BN + 4 words; rows of m otherwise.
        if (run) {
            if (!__all_sync(0xFFFFFFFFu, gt_wait(sm32(&tail.acc), 0u))) { if (lane == 0) atomicExch(&tail.fail, 1u); }
            else {
                asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                const int q = warp & 3, m = q * 32 + lane;
                float *part = (float *)smem;
                for (int c = 0; c < BN; c += 16) {
                    uint32_t v[16];
                    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
                                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
                                   "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                                 : "r"(tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)c) : "memory");
                    asm volatile("tcgen05.wait::ld.sync.aligned;\n"
                                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
                                   "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]) :: "memory");
                    if (p.transposed) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) part[(c + e) * 128 + m] = __uint_as_float(v[e]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 16; e += 4) *(uint4 *)(part + m * (BN + 4) + c + e) = make_uint4(v[e], v[e + 1], v[e + 2], v[e + 3]);
                    }
                }
            }
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    if (split > 1) gt_sync_all<true>(); else __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(cols) : "memory");

    // ================= the shares added up, bias, Gamma, output =================
    // CTA r stores the r-th part of the tile's pieces of four.
    if (run && s_fail == 0u) {
        const int rows = p.transposed ? (p.N - n0 < BN ? p.N - n0 : BN) : (p.M - m0 < 128 ? p.M - m0 : 128);
        const int per_row = p.transposed ? 32 : BN / 4, pitch = p.transposed ? 128 : BN + 4;
        const int lead0 = p.transposed ? n0 : m0, in0 = p.transposed ? m0 : n0, in_end = p.transposed ? p.M : p.N;
        const int units = rows * per_row, u0 = (int)((long long)units * rank / split), u1 = (int)((long long)units * (rank + 1) / split);
        const float *bias = from_here(p.bias);
        const uint8_t *gamma = from_here(p.gamma);
        for (int u = u0 + tid; u < u1; u += kFsThreads) {
            const int r = u / per_row, c = (u - r * per_row) * 4, in = in0 + c;
            if (in >= in_end) continue;
            const uint32_t at = ring + (uint32_t)(r * pitch + c) * 4u;
            float4 v;
            if (split == 1) v = *(const float4 *)(smem + (at - ring));
            else {
                v = fs_peer4(at, 0u);
                for (int s = 1; s < split; ++s) {
                    const float4 w = fs_peer4(at, (uint32_t)s);
                    v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
                }
            }
            const int left = in_end - in;
            if (bias != nullptr) {
                float b[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) b[e] = e < left ? __uint_as_float(load_free((const uint32_t *)bias + in + e)) : 0.f;
                v.x += b[0]; v.y += b[1]; v.z += b[2]; v.w += b[3];
            }
            if (gamma != nullptr && load_free(gamma + (int64_t)((lead0 + r) / p.bo) * p.NBi + in / p.bi) == 0u) v = make_float4(0.f, 0.f, 0.f, 0.f);
            const int64_t out = (int64_t)(lead0 + r) * in_end + in;
            const float x[4] = {v.x, v.y, v.z, v.w};
            if (p.bf16) {
                __nv_bfloat16 *y = (__nv_bfloat16 *)p.Y + out;
                if (p.vec) {
                    const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
                    *(uint2 *)y = make_uint2(*(const uint32_t *)&a, *(const uint32_t *)&b);
                } else
#pragma unroll
                    for (int e = 0; e < 4; ++e) if (e < left) y[e] = __float2bfloat16_rn(x[e]);
            } else {
                float *y = (float *)p.Y + out;
                if (p.vec) *(float4 *)y = v;
                else
#pragma unroll
                    for (int e = 0; e < 4; ++e) if (e < left) y[e] = x[e];
            }
        }
    }
    if (split > 1) gt_sync_all<true>();           // (no CTA leaves while another reads its memory)
    if (s_fail == 1u && tid == 0) atomicMax(p.status, (int)BSP_ERR_TIMEOUT);
}

bsp_status fs_map(CUtensorMap *map, const bsp_f8 &m, int box_rows)
{
    GtEncodeFn enc = gt_encode();
    if (!enc) return BSP_ERR_CUDA;
    const cuuint64_t gdim[2] = {(cuuint64_t)m.cols, (cuuint64_t)m.rows}, gstr[1] = {(cuuint64_t)f8_pitch(m.cols)};
    const cuuint32_t box[2] = {128u, (cuuint32_t)box_rows}, estr[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, m.data, gdim, gstr, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? BSP_OK : BSP_ERR_CUDA;
}

}  // namespace

bsp_status launch_gemm_f8(const bsp_f8 &x, const bsp_f8 &w, const float *bias, const bsp_wdesc *wd, const uint8_t *gamma, void *Y, bsp_dtype ytype,
                          void *ws, cudaStream_t st)
{
    static int n_sm[kGtMaxDevices] = {};
    static bool opted[kGtMaxDevices] = {};
    int dev = 0;
    BSP_CUDA_OK(cudaGetDevice(&dev));
    if (dev < 0 || dev >= kGtMaxDevices) return BSP_ERR_CUDA;
    if (!opted[dev]) {
        BSP_CUDA_OK(cudaFuncSetAttribute(gemm_f8_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFsSmem));
        opted[dev] = true;
    }
    if (n_sm[dev] == 0) BSP_CUDA_OK(cudaDeviceGetAttribute(&n_sm[dev], cudaDevAttrMultiProcessorCount, dev));
    FsParams p = {};
    // few rows of x become the columns of the MMA, whose rows are then the channels
    p.transposed = wd == nullptr && x.rows <= 64;
    const bsp_f8 &a = p.transposed ? w : x, &b = p.transposed ? x : w;
    p.M = (int)a.rows; p.N = (int)b.rows;
    p.n_kb = (int)f8_blocks(x.cols);
    p.atoms = f8_atoms(x.cols);
    p.sa = (const uint8_t *)a.scale; p.sb = (const uint8_t *)b.scale;
    const long long tiles_m = f8_blocks(p.M);
    p.BN = p.N <= 16 ? 16 : p.N <= 32 ? 32 : p.N <= 64 ? 64 : 128;
    if (tiles_m * ((p.N + 255) / 256) >= n_sm[dev]) p.BN = 256;
    p.tiles_n = (p.N + p.BN - 1) / p.BN;
    const long long tiles = tiles_m * p.tiles_n;
    p.split = 1;
    while (p.split < 8 && tiles * p.split * 2 <= n_sm[dev] && p.n_kb >= p.split * 2 * 2) p.split *= 2;
    if (tiles * p.split > 0x7FFFFFFF) return BSP_ERR_SHAPE;
    p.stage_bytes = 16384 + p.BN * 128;
    // the ring; the accumulators of a tile lie in it afterwards
    const int tail = (int)sizeof(FsTail), per_stage = p.stage_bytes + kFsScaleBytes;
    p.stages = (kFsSmem - tail) / per_stage;
    if (p.stages > kFsMaxStages) p.stages = kFsMaxStages;
    const int part = p.transposed ? p.BN * 512 : 128 * (p.BN + 4) * 4;
    const int want = (p.n_kb + p.split - 1) / p.split;
    if (p.stages > want) p.stages = want;
    while (p.stages * p.stage_bytes < part) ++p.stages;
    const size_t smem = (size_t)p.stages * per_stage + tail;
    const uint32_t fa = a.type == BSP_E5M2 ? 1u : 0u, fb = b.type == BSP_E5M2 ? 1u : 0u;
    // formats of A and B, N / 8, scales of 8 exponent bits, M / 128; both operands K-major
    p.idesc = (fa << 7) | (fb << 10) | ((uint32_t)(p.BN >> 3) << 17) | (1u << 23) | (1u << 27);
    p.Y = (uint8_t *)Y; p.bf16 = ytype == BSP_BF16;
    p.vec = (p.transposed ? p.M : p.N) % 4 == 0;
    p.bias = bias;
    if (wd) { p.gamma = gamma; p.bo = wd->bo; p.bi = wd->bi; p.NBi = wd->I / wd->bi; }
    p.status = (int *)ws;
    bsp_status rc = fs_map(&p.tma, a, 128);
    if (rc == BSP_OK) rc = fs_map(&p.tmb, b, p.BN);
    if (rc != BSP_OK) return rc;
    BSP_CUDA_OK(launch_after_clusters(gemm_f8_kernel, dim3((unsigned)(tiles * p.split)), dim3(kFsThreads), smem, st, p.split, 1, p));
    return BSP_OK;
}

}  // namespace bsp
