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
#include <type_traits>
#include "bsp_f8.cuh"
#include "bsp_tc.cuh"

namespace bsp {
namespace {

constexpr int kFsThreads = 256;                     // producer warp, MMA warp, two idle warps until the store, four epilogue warps
constexpr int kFsScaleBytes = 3 * kF8Atom;          // scales of a stage: 128 rows of A, up to 256 rows of B
constexpr int kFsMaxStages = 8;
constexpr int kFsSets = 4;                          // scale sets in tensor memory, 16 columns each (A 4, B up to 8)
constexpr int kFsSmem = 227 * 1024;
// Shared-memory descriptor of an atom of scales: 32 rows of 16 bytes without swizzle, groups of eight rows 128 bytes apart.
constexpr uint64_t kFsScaleDesc = (1ull << 16) | (8ull << 32) | (1ull << 46);
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

// 16 consecutive accumulator columns of this thread's tensor-memory lane.
__device__ __forceinline__ void fs_load16(uint32_t taddr, uint32_t (&v)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
                   "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;\n"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
                   "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]) :: "memory");
}

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
                const uint64_t ds = kFsScaleDesc | (uint64_t)(s16 & 0x3FFFu);
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
                    fs_load16(tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)c, v);
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

// ---- large products: persistent pairs of CTAs ----

constexpr int kFpThreads = 384;                     // producer warp, MMA warp, two that idle, two groups of four epilogue warps
// Registers of a thread: the float32 form of the epilogue holds 128 sums.  (40 + 2 x 232 is 3 x 168, what the CTA is launched with.)
constexpr int kFpFew = 40, kFpMany = 232;
constexpr int kFpStage = 32768;                     // 128 rows of A and 128 rows (half of the tile's) of B
constexpr int kFpStages = 5;
constexpr int kFpStaging = 16384;                   // of a group: 128 rows of 128 bytes
constexpr int kFpSecond = 192;                      // first column of the second accumulator: the last 64 of the first lie under it
constexpr int kFpChunk = 16;                        // blocks of 128 entries that are summed in the tensor core before float32 registers take over

struct FpParams {
    CUtensorMap tma, tmb;         // values as bytes, (K, rows), box 128 x 128, 128-byte swizzle
    CUtensorMap tsa, tsb;         // scales as words, (128, atoms, rows / 128), boxes of one and of two atoms
    CUtensorMap tmy;              // Y as bytes, (N ey, M), box 128 bytes x 128 rows, 128-byte swizzle
    int M, N, n_kb, tiles_n, n_tiles;
    uint32_t idesc, m_tn;
    const float *bias;
    const uint8_t *gamma;
    int bo, bi, NBi;              // Gamma's blocks: logarithms of their sizes, blocks in a row
    int *status;
};

struct FpTail {
    uint64_t full[kFpStages], empty[kFpStages], acc_full[2], acc_free;
    uint32_t tmem, fail;
    __align__(16) float bias[2][128];
};
constexpr int kFpSmem = kFpStages * (kFpStage + kFsScaleBytes) + 2 * kFpStaging + (int)sizeof(FpTail);
static_assert(kFpSmem <= kFsSmem, "shared memory of a CTA");

// A pair of CTAs owns tiles of 256 x 256: CTA r of the pair the rows 128 r .. of the tile, and loads these and its half of the tile's rows
// of B; the leader issues MMAs of 256 x 256 x 32 for both.  Two accumulators of 256 columns that overlap by 64, whose columns the
// epilogue reads first, leave 64 columns for the scales: the next tile's MMAs start when these 64 have been read.
// kF32: sums of kFpChunk blocks in the tensor core, of these in registers (256 instructions in a row, 8192 entries, were off by 1.9e-6 of
// the result, 64 by ...).
template <bool kF32>
__global__ void __launch_bounds__(kFpThreads, 1) gemm_f8_pair_kernel(const __grid_constant__ FpParams p)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    FpTail &tail = *(FpTail *)(smem + kFpStages * (kFpStage + kFsScaleBytes) + 2 * kFpStaging);
    volatile uint32_t &s_fail = tail.fail;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
    const uint32_t ring = sm32(smem), staging = ring + kFpStages * kFpStage, scales = staging + 2 * kFpStaging;
    uint32_t rank;
    asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(rank));
    const uint32_t full0 = sm32(&tail.full[0]), empty0 = sm32(&tail.empty[0]);
    uint32_t lead_full0, lead_free;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;\n" : "=r"(lead_full0) : "r"(full0));
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;\n" : "=r"(lead_free) : "r"(sm32(&tail.acc_free)));
    const int t_first = (int)(blockIdx.x >> 1), t_step = (int)(gridDim.x >> 1), n_kb = p.n_kb;

    if (tid == 0) {
        for (int s = 0; s < kFpStages; ++s) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(sm32(&tail.full[s])), "r"(1) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(sm32(&tail.empty[s])), "r"(1) : "memory");
        }
        for (int b = 0; b < 2; ++b) asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(sm32(&tail.acc_full[b])), "r"(1) : "memory");
        asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(sm32(&tail.acc_free)), "r"(16) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        s_fail = (ring & 1023u) == 0u ? 0u : 2u;
        const CUtensorMap *maps[5] = {&p.tma, &p.tmb, &p.tsa, &p.tsb, &p.tmy};
        for (const CUtensorMap *m : maps) asm volatile("prefetch.tensormap [%0];\n" ::"l"(m) : "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(sm32(&tail.tmem)), "r"(kGtTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
    }
    wait_for_previous<false>();
    if (warp == 0) let_next_start();
    if (tid == 0 && s_fail) atomicMax(p.status, (int)BSP_ERR_CUDA);
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    gt_sync_all<true>();
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, tail.tmem, 0);
    const bool run = __shfl_sync(0xFFFFFFFFu, s_fail, 0) == 0u;   // (both CTAs of a launch lie alike)

    // (each in its own branch: where the branches meet, the smaller number holds for the compiler)
    if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kFpFew));
    if (warp == 0) {
        // ================= producer: this CTA's rows of A, its half of B, the scales of its rows and of all of B's =================
        if (run) {
            uint32_t slot = 0, par = 1, issued = 0;
            bool ok = true;
            for (int tile = t_first; tile < p.n_tiles && ok; tile += t_step) {
                int mp, tn;
                gt_divmod(tile, p.tiles_n, p.m_tn, mp, tn);
                const int ma = 2 * mp + (int)rank, m0 = ma * 128, n0 = tn * 256 + (int)rank * 128;
                if (s_fail) { ok = false; break; }
                for (int kb = 0; kb < n_kb; ++kb) {
                    if (!__all_sync(0xFFFFFFFFu, gt_poll(empty0 + slot * 8u, par))) { ok = false; break; }
                    const uint32_t with = (kb & 3) == 0 ? 1u : 0u, dst = ring + slot * kFpStage, sdst = scales + slot * kFsScaleBytes;
                    const uint32_t bytes = 2u * (kFpStage + with * kFsScaleBytes), bar = lead_full0 + slot * 8u;
                    asm volatile("{\n .reg .pred e, l, s;\n elect.sync _|e, 0xFFFFFFFF;\n setp.eq.u32 l, %2, 0;\n and.pred l, l, e;\n setp.ne.b32 s, %3, 0;\n and.pred s, s, e;\n"
                                 " @l mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n"
                                 " @s cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%11], [%12, {%15, %13, %14}], [%4];\n"
                                 " @s cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%16], [%17, {%15, %13, %18}], [%4];\n"
                                 " @e cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%5], [%6, {%7, %8}], [%4];\n"
                                 " @e cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%9], [%10, {%7, %19}], [%4];\n}\n"
                                 ::"r"(full0 + slot * 8u), "r"(bytes), "r"(rank), "r"(with), "r"(bar), "r"(dst), "l"(&p.tma), "r"(kb * 128), "r"(m0), "r"(dst + 16384u), "l"(&p.tmb),
                                   "r"(sdst), "l"(&p.tsa), "r"(kb >> 2), "r"(ma), "r"(0), "r"(sdst + 512u), "l"(&p.tsb), "r"(2 * tn), "r"(n0) : "memory");
                    ++issued;
                    if (++slot == kFpStages) { slot = 0; par ^= 1u; }
                }
            }
            if (!ok && lane == 0) {
                atomicExch(&tail.fail, 1u);
                // (the follower's loads announce themselves to the leader; both CTAs meet before either leaves)
                for (uint32_t back = 0; back < (uint32_t)kFpStages && back < issued && rank == 0; ++back) {
                    const uint32_t it = issued - 1u - back;
                    gt_poll(full0 + (it % (uint32_t)kFpStages) * 8u, (it / (uint32_t)kFpStages) & 1u);
                }
            }
        }
    } else if (warp == 1) {
        // ================= MMA issuer (the leader's, for both) =================
        if (run && rank == 0) {
            uint32_t slot = 0, par = 0, set = 0, unit = 0;
            bool ok = true, full_now = false;
            for (int tile = t_first; tile < p.n_tiles && ok; tile += t_step) {
                for (int kb = 0; kb < n_kb; ++kb) {
                    const bool fresh = kF32 ? kb % kFpChunk == 0 : kb == 0;
                    if (fresh) {
                        // the accumulator before this one has been read where they overlap, and the one before that altogether
                        if (unit > 0 && !gt_poll(sm32(&tail.acc_free), (unit - 1u) & 1u)) ok = false;
                        if (s_fail) ok = false;
                        ok = __all_sync(0xFFFFFFFFu, ok);
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                    }
                    const uint32_t d = tmem + (unit & 1u) * kFpSecond;
                    if (!full_now && !gt_poll_stage(full0 + slot * 8u, par)) { ok = false; break; }
                    const uint32_t with = (kb & 3) == 0 ? 1u : 0u;
                    if (with) set = (set + 1u) & (kFsSets - 1u);
                    const uint32_t a16 = (ring + slot * kFpStage) >> 4, s16 = (scales + slot * kFsScaleBytes) >> 4;
                    const uint64_t da = kGtDesc | (uint64_t)(a16 & 0x3FFFu), db = kGtDesc | (uint64_t)((a16 + 1024u) & 0x3FFFu);
                    const uint64_t ds = kFsScaleDesc | (uint64_t)(s16 & 0x3FFFu);
                    const uint32_t fa = tmem + 448u + set * 16u, fb = fa + 8u, id = (uint32_t)kb & 3u, idesc = p.idesc | (id << 4) | (id << 29);
                    const bool wrap = slot + 1u == (uint32_t)kFpStages;
                    uint32_t next;
                    asm volatile("{\n .reg .pred e, s, p, q, f, v;\n .reg .b64 a1, a2, a3, b1, b2, b3, s1, s2;\n .reg .b32 f2;\n"
                                 " elect.sync _|e, 0xFFFFFFFF;\n setp.ne.b32 s, %9, 0;\n and.pred s, s, e;\n setp.ne.b32 p, %10, 0;\n setp.eq.b32 q, %10, %10;\n"
                                 " add.u64 s1, %5, 32;\n add.u64 s2, %5, 64;\n add.u32 f2, %7, 4;\n"
                                 " @s tcgen05.cp.cta_group::2.32x128b.warpx4 [%6], %5;\n"
                                 " @s tcgen05.cp.cta_group::2.32x128b.warpx4 [%7], s1;\n"
                                 " @s tcgen05.cp.cta_group::2.32x128b.warpx4 [f2], s2;\n"
                                 " add.u64 a1, %2, 2;\n add.u64 a2, %2, 4;\n add.u64 a3, %2, 6;\n"
                                 " add.u64 b1, %3, 2;\n add.u64 b2, %3, 4;\n add.u64 b3, %3, 6;\n"
                                 " @e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%1], %2, %3, %4, [%6], [%7], p;\n"
                                 " @e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%1], a1, b1, %4, [%6], [%7], q;\n"
                                 " mbarrier.test_wait.parity.shared::cta.b64 f, [%12], %13;\n"
                                 " @e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%1], a2, b2, %4, [%6], [%7], q;\n"
                                 " @e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%1], a3, b3, %4, [%6], [%7], q;\n"
                                 " @e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%8], %11;\n"
                                 " vote.sync.all.pred v, f, 0xFFFFFFFF;\n tcgen05.fence::after_thread_sync;\n selp.b32 %0, 1, 0, v;\n}\n"
                                 : "=r"(next) : "r"(d), "l"(da), "l"(db), "r"(idesc), "l"(ds), "r"(fa), "r"(fb), "r"(empty0 + slot * 8u), "r"(with), "r"(fresh ? 0u : 1u),
                                   "h"((unsigned short)3), "r"(full0 + (wrap ? 0u : slot + 1u) * 8u), "r"(wrap ? par ^ 1u : par) : "memory");
                    full_now = next != 0u;
                    if (wrap) { slot = 0; par ^= 1u; } else ++slot;
                    if (kb + 1 == n_kb || (kF32 && (kb + 1) % kFpChunk == 0)) {
                        gt_commit_elected<true>(sm32(&tail.acc_full[unit & 1u]));
                        ++unit;
                    }
                }
            }
            if (!ok && lane == 0) atomicExch(&tail.fail, 1u);
        }
    }
    } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(kFpMany));
    if (run) {
        // ================= epilogue =================
        // Group g takes the columns 64 g + (0 .. 63) and 128 + 64 g + (0 .. 63) of every tile; the ones that lie under the other accumulator
        // first: the upper half of the first accumulator, the lower half of the second.
        const int q = warp & 3, grp = (warp - 4) >> 2, row = q * 32 + lane;
        const uint32_t sg = staging + (uint32_t)(grp * kFpStaging), lanes = (uint32_t)(q * 32) << 16;
        const bool issuer = q == 0 && lane == 0;
        const float *bias_of = from_here(p.bias);
        const uint8_t *gamma = from_here(p.gamma);
        const int chunks = kF32 ? (n_kb + kFpChunk - 1) / kFpChunk : 1;
        uint32_t unit = 0;
        bool ok = true;
        auto hand_back = [&]() {
            asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
            __syncwarp();
            if (lane == 0) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];\n" ::"r"(lead_free) : "memory");
        };
        for (int tile = t_first; tile < p.n_tiles; tile += t_step) {
            int mp, tn;
            gt_divmod(tile, p.tiles_n, p.m_tn, mp, tn);
            const int m0 = (2 * mp + (int)rank) * 128, n0 = tn * 256, m = m0 + row;
            {   // the bias of the group's 128 columns (everybody is past the barriers of the last tile's rounds)
                const int n = n0 + (row >> 6) * 128 + grp * 64 + (row & 63);
                const float b = bias_of != nullptr && n < p.N ? __uint_as_float(load_free((const uint32_t *)bias_of + n)) : 0.f;
                tail.bias[grp][row] = b;
            }
            // stores 128 bytes of every row: columns c0 .. of the tile
            auto store = [&](const uint32_t (&out)[32], int c0) {
                if (issuer) asm volatile("cp.async.bulk.wait_group.read 0;\n" ::: "memory");
                gt_group_sync(1 + grp);
                gt_store_round(sg + (uint32_t)row * 128u, (uint32_t)row & 7u, true, out);
                asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                gt_group_sync(1 + grp);
                if (issuer && n0 + c0 < p.N && m0 < p.M && ok) {
                    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];\n"
                                 ::"l"(&p.tmy), "r"(sg), "r"((n0 + c0) * (kF32 ? 4 : 2)), "r"(m0) : "memory");
                    asm volatile("cp.async.bulk.commit_group;\n" ::: "memory");
                }
            };
            if constexpr (kF32) {
                float acc[4][32];
                for (int c = 0; c < chunks; ++c, ++unit) {
                    const uint32_t second = unit & 1u, t = tmem + lanes + second * kFpSecond + (uint32_t)grp * 64u;
                    if (s_fail) ok = false;
                    if (ok && !gt_wait(sm32(&tail.acc_full[second]), (unit >> 1) & 1u)) ok = false;
                    __syncwarp();
                    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                    if (second == (uint32_t)grp) hand_back();            // (this group has no column under the other accumulator)
                    auto take = [&](auto half_c) {
                        constexpr int half = decltype(half_c)::value;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            uint32_t v[16];
                            fs_load16(t + half * 128u + k * 16u, v);
                            float *sum = acc[half * 2 + (k >> 1)] + (k & 1) * 16;
#pragma unroll
                            for (int e = 0; e < 16; ++e) sum[e] = c == 0 ? __uint_as_float(v[e]) : sum[e] + __uint_as_float(v[e]);
                        }
                    };
                    if (second) {
                        take(std::integral_constant<int, 0>());
                        if (grp == 0) hand_back();
                        take(std::integral_constant<int, 1>());
                    } else {
                        take(std::integral_constant<int, 1>());
                        if (grp == 1) hand_back();
                        take(std::integral_constant<int, 0>());
                    }
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int c0 = (r >> 1) * 128 + grp * 64 + (r & 1) * 32;
                    uint32_t out[32];
                    const float *b = tail.bias[grp] + r * 32;
                    if (r == 0) gt_group_sync(1 + grp);                  // (the bias is there)
#pragma unroll
                    for (int e = 0; e < 32; ++e) out[e] = __float_as_uint(acc[r][e] + b[e]);
                    if (gamma != nullptr && m < p.M) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const int n = n0 + c0 + e;
                            if (n < p.N && load_free(gamma + (int64_t)(m >> p.bo) * p.NBi + (n >> p.bi)) == 0u) out[e] = out[e + 1] = out[e + 2] = out[e + 3] = 0u;
                        }
                    }
                    store(out, c0);
                }
            } else {
                const uint32_t second = unit & 1u, t = tmem + lanes + second * kFpSecond + (uint32_t)grp * 64u;
                if (s_fail) ok = false;
                if (ok && !gt_wait(sm32(&tail.acc_full[second]), (unit >> 1) & 1u)) ok = false;
                __syncwarp();
                asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                if (second == (uint32_t)grp) hand_back();
                gt_group_sync(1 + grp);                                  // (the bias is there)
#pragma unroll 1
                for (int r = 0; r < 2; ++r) {
                    const uint32_t half = second ? (uint32_t)r : 1u - (uint32_t)r;
                    uint32_t out[32];
                    gt_epilogue_round<false, 2, false>(t + half * 128u, (const uint32_t *)tail.bias[grp] + half * 64u, 64, 0, out);
                    if (r == 0 && second != (uint32_t)grp) hand_back();
                    store(out, (int)half * 128 + grp * 64);
                }
                ++unit;
            }
        }
        if (issuer) asm volatile("cp.async.bulk.wait_group.read 0;\n" ::: "memory");
        if (!ok && lane == 0) atomicExch(&tail.fail, 1u);
    }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    gt_sync_all<true>();
    if (s_fail == 1u && tid == 0) atomicMax(p.status, (int)BSP_ERR_TIMEOUT);
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(kGtTmemCols) : "memory");
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

// Scales as a tensor of words: 128 words an atom, `atoms` atoms per 128 rows.
bsp_status fp_scale_map(CUtensorMap *map, const bsp_f8 &m, int box_blocks)
{
    GtEncodeFn enc = gt_encode();
    if (!enc) return BSP_ERR_CUDA;
    const cuuint64_t atoms = (cuuint64_t)f8_atoms(m.cols), gdim[3] = {128, atoms, (cuuint64_t)f8_blocks(m.rows)}, gstr[2] = {kF8Atom, kF8Atom * atoms};
    const cuuint32_t box[3] = {128u, 1u, (cuuint32_t)box_blocks}, estr[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, m.scale, gdim, gstr, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? BSP_OK : BSP_ERR_CUDA;
}

bsp_status launch_pairs(const bsp_f8 &x, const bsp_f8 &w, const float *bias, const bsp_wdesc *wd, const uint8_t *gamma, void *Y, bsp_dtype ytype, void *ws,
                        int sms, cudaStream_t st)
{
    FpParams p = {};
    const int ey = ytype == BSP_BF16 ? 2 : 4;
    p.M = (int)x.rows; p.N = (int)w.rows; p.n_kb = (int)f8_blocks(x.cols);
    p.tiles_n = (p.N + 255) / 256;
    const long long tiles = (long long)((p.M + 255) / 256) * p.tiles_n;
    if (tiles > 0x7FFFFFFF - 4096) return BSP_ERR_SHAPE;
    p.n_tiles = (int)tiles;
    p.m_tn = gt_magic(p.tiles_n);
    // formats, N / 8, scales of 8 exponent bits, M / 128
    p.idesc = ((x.type == BSP_E5M2 ? 1u : 0u) << 7) | ((w.type == BSP_E5M2 ? 1u : 0u) << 10) | (32u << 17) | (1u << 23) | (2u << 27);
    p.bias = bias;
    if (wd) { p.gamma = gamma; p.bo = f8_log2(wd->bo); p.bi = f8_log2(wd->bi); p.NBi = wd->I / wd->bi; }
    p.status = (int *)ws;
    bsp_status rc = fs_map(&p.tma, x, 128);
    if (rc == BSP_OK) rc = fs_map(&p.tmb, w, 128);
    if (rc == BSP_OK) rc = fp_scale_map(&p.tsa, x, 1);
    if (rc == BSP_OK) rc = fp_scale_map(&p.tsb, w, 2);
    if (rc != BSP_OK) return rc;
    const cuuint64_t gdim[2] = {(cuuint64_t)p.N * ey, (cuuint64_t)p.M}, gstr[1] = {(cuuint64_t)p.N * ey};
    const cuuint32_t box[2] = {128u, 128u}, estr[2] = {1, 1};
    if (gt_encode()(&p.tmy, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, Y, gdim, gstr, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                    CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return BSP_ERR_CUDA;
    const int pairs = p.n_tiles < sms / 2 ? p.n_tiles : sms / 2;
    BSP_CUDA_OK(launch_after_clusters(ey == 4 ? gemm_f8_pair_kernel<true> : gemm_f8_pair_kernel<false>, dim3((unsigned)(2 * pairs)), dim3(kFpThreads), kFpSmem, st, 2, 1, p));
    return BSP_OK;
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
        BSP_CUDA_OK(cudaFuncSetAttribute(gemm_f8_pair_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kFpSmem));
        BSP_CUDA_OK(cudaFuncSetAttribute(gemm_f8_pair_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kFpSmem));
        opted[dev] = true;
    }
    if (n_sm[dev] == 0) BSP_CUDA_OK(cudaDeviceGetAttribute(&n_sm[dev], cudaDevAttrMultiProcessorCount, dev));
    // large products, whose rows of Y a tensor map can describe
    const long long pair_tiles = ((x.rows + 255) / 256) * ((w.rows + 255) / 256);
    if (pair_tiles * 2 >= n_sm[dev] && w.rows * (ytype == BSP_BF16 ? 2 : 4) % 16 == 0 && n_sm[dev] >= 2)
        return launch_pairs(x, w, bias, wd, gamma, Y, ytype, ws, n_sm[dev], st);
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
