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
#include <atomic>
#include <type_traits>
#include "bsp_f8.cuh"
#include "bsp_f8_tiles.cuh"
#include "bsp_tc.cuh"

namespace bsp {
namespace {

constexpr int kFsThreads = 320;                     // producer warp, MMA warp, two groups of four epilogue warps
constexpr int kFsMaxStages = 8;
constexpr int kFsSets = 4;                          // scale sets in tensor memory, 16 columns each (A 4, B up to 8)
constexpr int kFsSmem = 227 * 1024;
constexpr int kFsChunk = 16;                        // blocks of 128 entries that are summed in the tensor core before float32 registers take over
constexpr int kFsScales = 2 * kF8Atom;              // scales of a stage: 128 rows of A and of B
// Shared-memory descriptor of an atom of scales: 32 rows of 16 bytes without swizzle, groups of eight rows 128 bytes apart.
constexpr uint64_t kFsScaleDesc = (1ull << 16) | (8ull << 32) | (1ull << 46);
static_assert(kFsMaxStages <= 4 * (kFsSets - 1) + 1, "a set is written again only when the MMAs that read it are done: the ring's barriers see to that");

// ---- small and middle products: a tile of 128 x BN for a CTA, or for a cluster that shares the summed axis ----

struct FsParams {
    CUtensorMap tma, tmb;         // values as bytes, (K, rows), box 128 x 128 and 128 x BN, 128-byte swizzle; zeros past the ends
    CUtensorMap tmy;              // where `staged`: Y as bytes, (N ey, M), box 128 bytes x 128 rows, 128-byte swizzle
    const uint8_t *sa, *sb;       // scales
    int64_t atoms;                // atoms per 128 rows
    int M, N, BN, n_kb, tiles_n, split, stages, stage_bytes;
    int off_x, off_recv, off_scales, off_tail;      // offsets in shared memory
    uint32_t idesc;
    uint8_t *Y;
    int bf16, transposed, vec;    // element (m, n) at Y[m N + n], or at Y[n M + m]; rows that can be written four entries at a time
    int staged;                   // the output leaves by TMA stores
    const float *bias;
    const uint8_t *gamma;
    int bo, bi, NBi;              // Gamma's blocks: logarithms of their sizes, blocks in a row
    const void *X;                // kX: the rows of B before they are quantised, ldx entries apart
    int64_t ldx, K;
    int xvec;                     // rows of X can be read 16 bytes at a time
    int *status;
};

struct FsTail {
    uint64_t full[kFsMaxStages], empty[kFsMaxStages], acc_full[2], acc_free[2], x_ready, shares;
    uint32_t tmem, fail;
    __align__(16) float bias[128];
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

// 16 bytes of X, or zeros: a predicate instead of a branch, so that the loads of a thread's rows go out together.
__device__ __forceinline__ uint4 fs_load_if(const void *p, bool there)
{
    uint4 v;
    asm("{\n .reg .pred q;\n setp.ne.b32 q, %5, 0;\n mov.b32 %0, 0;\n mov.b32 %1, 0;\n mov.b32 %2, 0;\n mov.b32 %3, 0;\n @q ld.global.v4.b32 {%0, %1, %2, %3}, [%4];\n}\n"
        : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w) : "l"(p), "r"((uint32_t)there));
    return v;
}

// What an element becomes, two neighbours of a row at a time.
__device__ __forceinline__ uint32_t fs_pack(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *(const uint32_t *)&h;
}

// One tile of 128 x BN per cluster.  CTA r of the cluster sums its share of the blocks and sends the rows of the output that CTA s stores to s
// (one bulk copy between their shared memories); s adds the shares up in the order of the ranks.
// (A cluster of eight finds room for 15 of its kind on the 148 SMs, of four for 33, of two for 74.)
// Chunks of kFsChunk blocks go to two accumulators in turn and are added up in registers (256 instructions in a row into one
// accumulator, 8192 entries, were off by 1.9e-6 of the result, chunks by 5.5e-7; plain float32 sums by 4.2e-7).
// T: type of X where its rows are quantised here (rows of B, e4m3), void where B comes as an 8-bit matrix.
template <typename T>
__global__ void __launch_bounds__(kFsThreads, std::is_same_v<T, void> ? 1 : 2) gemm_f8_tile_kernel(const __grid_constant__ FsParams p)
{
    constexpr bool kX = !std::is_same_v<T, void>;
    constexpr int kPieces = kX ? 2 : 4;               // 16-column pieces of a warp's sums: tiles with X have at most 64 columns
    extern __shared__ __align__(1024) uint8_t smem[];
    FsTail &tail = *(FsTail *)(smem + p.off_tail);
    volatile uint32_t &s_fail = tail.fail;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
    const int S = p.stages, split = p.split, tile = (int)blockIdx.x / split, rank = (int)blockIdx.x - tile * split;
    const int tm = tile / p.tiles_n, tn = tile - tm * p.tiles_n, m0 = tm * 128, n0 = tn * p.BN, BN = p.BN;
    const int kb0 = (int)((long long)p.n_kb * rank / split), kb1 = (int)((long long)p.n_kb * (rank + 1) / split);
    const uint32_t ring = sm32(smem), scales = ring + (uint32_t)p.off_scales, xs = ring + (uint32_t)p.off_x;
    const uint32_t xs_scales = xs + (uint32_t)((kb1 - kb0) * BN * 128);      // (kX)
    const uint32_t cols = BN <= 32 ? 128u : BN <= 64 ? 256u : 512u;          // two accumulators and 64 columns of scales

    // the bytes that the other CTAs of the cluster will send (lines: rows of the output in this tile; `per` of them to a CTA)
    const int valid_n = p.N - n0 < BN ? p.N - n0 : BN, valid_m = p.M - m0 < 128 ? p.M - m0 : 128;
    const int lines = p.transposed ? valid_n : valid_m, per = (p.transposed ? BN : 128) / split, line_bytes = p.transposed ? 512 : BN * 4;

    if (tid == 0) {
        for (int s = 0; s < S; ++s) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(sm32(&tail.full[s])), "r"(1) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(sm32(&tail.empty[s])), "r"(1) : "memory");
        }
        for (int b = 0; b < 2; ++b) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(sm32(&tail.acc_full[b])), "r"(1) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(sm32(&tail.acc_free[b])), "r"(8) : "memory");
        }
        asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(sm32(&tail.x_ready)), "r"(8) : "memory");
        asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(sm32(&tail.shares)), "r"(1) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        if (split > 1) {
            const int n = lines - rank * per < per ? lines - rank * per : per;
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(sm32(&tail.shares)), "r"(n > 0 ? (uint32_t)((split - 1) * n * line_bytes) : 0u) : "memory");
        }
        s_fail = (ring & 1023u) == 0u ? 0u : 2u;
        asm volatile("prefetch.tensormap [%0];\n" ::"l"(&p.tma) : "memory");
        if constexpr (!kX) asm volatile("prefetch.tensormap [%0];\n" ::"l"(&p.tmb) : "memory");
    }
    __syncwarp();
    // The CTAs of a cluster run, with their barriers set up, once this barrier is complete: what they send each other waits for it.  It comes
    // ahead of the allocation, and tensor memory is given back before a CTA waits for the others' shares: no CTA holds it while it
    // waits for one that may still wait for columns, so clusters of several streams on the same SMs cannot stop one another.
    if (split > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;\n" ::: "memory");
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(sm32(&tail.tmem)), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    if constexpr (kX) {
        // The weights of this CTA on their way to L2 while the kernel before this one ends, where shared memory has room for both: a cache
        // that is coherent, so it does not matter whether that kernel wrote them.
        if (warp == 0)
            for (int kb = kb0; kb < kb1; ++kb)
                asm volatile("{\n .reg .pred e;\n elect.sync _|e, 0xFFFFFFFF;\n @e cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];\n}\n"
                             ::"l"(&p.tma), "r"(kb * 128), "r"(m0) : "memory");
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

    float acc[kPieces][16];                           // (epilogue warps)
    if (warp == 0) {
        // ================= producer =================
        if (run) {
            const uint8_t *sa = p.sa + (int64_t)tm * p.atoms * kF8Atom, *sb = p.sb + (int64_t)(n0 >> 7) * p.atoms * kF8Atom;
            uint32_t slot = 0, par = 1, issued = 0;
            bool ok = true;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!__all_sync(0xFFFFFFFFu, gt_poll(empty0 + slot * 8u, par)) || s_fail) { ok = false; break; }
                const uint32_t with = kb == kb0 || (kb & 3) == 0 ? 1u : 0u, dst = ring + slot * (uint32_t)p.stage_bytes, sdst = scales + slot * kFsScales;
                const uint32_t bytes = (uint32_t)p.stage_bytes + with * (kX ? kF8Atom : 2 * kF8Atom);
                const int64_t at = (int64_t)(kb >> 2) * kF8Atom;
                if constexpr (kX)
                    asm volatile("{\n .reg .pred e, s;\n elect.sync _|e, 0xFFFFFFFF;\n setp.ne.b32 s, %6, 0;\n and.pred s, s, e;\n"
                                 " @e mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n"
                                 " @s cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%7], [%8], 512, [%0];\n"
                                 " @e cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%2], [%3, {%4, %5}], [%0];\n}\n"
                                 ::"r"(full0 + slot * 8u), "r"(bytes), "r"(dst), "l"(&p.tma), "r"(kb * 128), "r"(m0), "r"(with), "r"(sdst), "l"(sa + at) : "memory");
                else
                    asm volatile("{\n .reg .pred e, s;\n elect.sync _|e, 0xFFFFFFFF;\n setp.ne.b32 s, %9, 0;\n and.pred s, s, e;\n"
                                 " @e mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n"
                                 " @s cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%10], [%11], 512, [%0];\n"
                                 " @s cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%12], [%13], 512, [%0];\n"
                                 " @e cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%2], [%3, {%4, %5}], [%0];\n"
                                 " @e cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%6], [%7, {%4, %8}], [%0];\n}\n"
                                 ::"r"(full0 + slot * 8u), "r"(bytes), "r"(dst), "l"(&p.tma), "r"(kb * 128), "r"(m0), "r"(dst + 16384u), "l"(&p.tmb), "r"(n0),
                                   "r"(with), "r"(sdst), "l"(sa + at), "r"(sdst + kF8Atom), "l"(sb + at) : "memory");
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
            uint32_t slot = 0, par = 0, set = 0, chunk = 0;
            bool ok = true;
            if constexpr (kX) ok = gt_poll_stage(sm32(&tail.x_ready), 0u);
            for (int kb = kb0; kb < kb1 && ok; ++kb) {
                const bool fresh = (kb - kb0) % kFsChunk == 0;
                if (fresh && chunk >= 2u && !gt_poll_stage(sm32(&tail.acc_free[chunk & 1u]), ((chunk >> 1) & 1u) ^ 1u)) { ok = false; break; }
                if (!gt_poll_stage(full0 + slot * 8u, par)) { ok = false; break; }
                const uint32_t with = kb == kb0 || (kb & 3) == 0 ? 1u : 0u;
                if (with && kb != kb0) set = (set + 1u) & (kFsSets - 1u);
                const uint32_t a16 = (ring + slot * (uint32_t)p.stage_bytes) >> 4, s16 = (scales + slot * kFsScales) >> 4;
                const uint32_t b16 = kX ? (xs + (uint32_t)((kb - kb0) * BN * 128)) >> 4 : a16 + 1024u;
                const uint32_t t16 = kX ? (xs_scales + (uint32_t)((kb >> 2) - (kb0 >> 2)) * kF8Atom) >> 4 : s16 + (kF8Atom >> 4);
                const uint64_t da = kGtDesc | (uint64_t)(a16 & 0x3FFFu), db = kGtDesc | (uint64_t)(b16 & 0x3FFFu);
                const uint64_t ds = kFsScaleDesc | (uint64_t)(s16 & 0x3FFFu), dt = kFsScaleDesc | (uint64_t)(t16 & 0x3FFFu);
                // A tile of 32 or 64 rows of B that starts inside an atom: its columns of scales move to the front, as an MMA takes scales from a
                // multiple of four columns on (any other address is a misaligned one).
                const uint32_t skip = (uint32_t)(n0 & 127) >> 5;
                if (with && skip) {
                    const uint32_t at = (t16 << 4) + (uint32_t)lane * 16u;
                    uint32_t w[4];
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
                    const uint32_t lo = skip == 1u ? w[1] : skip == 2u ? w[2] : w[3], hi = skip == 1u ? w[2] : w[3];
                    asm volatile("st.shared.v2.b32 [%0], {%1, %2};\n fence.proxy.async.shared::cta;\n" ::"r"(at), "r"(lo), "r"(hi) : "memory");
                    __syncwarp();
                }
                const uint32_t fa = sf + set * 16u, fb = fa + 8u, id = (uint32_t)kb & 3u, idesc = p.idesc | (id << 4) | (id << 29);
                asm volatile("{\n .reg .pred e, s, p, q;\n .reg .b64 a1, a2, a3, b1, b2, b3;\n"
                             " elect.sync _|e, 0xFFFFFFFF;\n setp.ne.b32 s, %9, 0;\n and.pred s, s, e;\n setp.ne.b32 p, %10, 0;\n setp.eq.b32 q, %10, %10;\n"
                             " @s tcgen05.cp.cta_group::1.32x128b.warpx4 [%6], %4;\n"
                             " @s tcgen05.cp.cta_group::1.32x128b.warpx4 [%7], %5;\n"
                             " add.u64 a1, %1, 2;\n add.u64 a2, %1, 4;\n add.u64 a3, %1, 6;\n"
                             " add.u64 b1, %2, 2;\n add.u64 b2, %2, 4;\n add.u64 b3, %2, 6;\n"
                             " @e tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%6], [%7], p;\n"
                             " @e tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a1, b1, %3, [%6], [%7], q;\n"
                             " @e tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a2, b2, %3, [%6], [%7], q;\n"
                             " @e tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a3, b3, %3, [%6], [%7], q;\n"
                             " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%8];\n}\n"
                             ::"r"(tmem + (chunk & 1u) * (uint32_t)BN), "l"(da), "l"(db), "r"(idesc), "l"(ds), "l"(dt), "r"(fa), "r"(fb), "r"(empty0 + slot * 8u), "r"(with),
                               "r"(fresh ? 0u : 1u) : "memory");
                if (++slot == (uint32_t)S) { slot = 0; par ^= 1u; }
                if (kb + 1 == kb1 || (kb + 1 - kb0) % kFsChunk == 0) {
                    gt_commit_elected<false>(sm32(&tail.acc_full[chunk & 1u]));
                    ++chunk;
                }
            }
            if (!ok && lane == 0) atomicExch(&tail.fail, 1u);
        }
    } else if (run) {
        const int w = warp - 2, q = warp & 3, grp = w >> 2;
        if constexpr (kX) {
            // ================= rows of X to 8 bits: half a warp takes 128 entries of a row, eight to a lane =================
            const T *X = from_here((const T *)p.X);
            const int rows = p.N < BN ? p.N : BN, items = (kb1 - kb0) * rows, l = lane & 15;
            const uint32_t recip = 65536u / (uint32_t)rows + 1u;          // (items are at most 768: the quotient is exact)
            auto pass = [&](auto batch_c) {
            constexpr int kBatch = decltype(batch_c)::value;            // (items in flight; what lies past the last is worked on too)
            for (int i0 = w * 2 + (lane >> 4); i0 - (lane >> 4) < items; i0 += 16 * kBatch) {
                constexpr int kRaw = sizeof(T) / 2;                     // words of 16 bytes in eight entries
                uint4 raw[kBatch][kRaw];
                float v[kBatch][8], m[kBatch];
                bool odd = false;                                       // entries that do not come 16 bytes at a time
#pragma unroll
                for (int u = 0; u < kBatch; ++u) {
                    const int i = i0 + 16 * u, b = (int)((uint32_t)i * recip >> 16), r = i - b * rows;
                    const int64_t c = (int64_t)(kb0 + b) * kF8Block + l * 8;
                    const bool whole = p.xvec && i < items && c + 8 <= p.K;
                    odd |= !whole && i < items && c < p.K;
#pragma unroll
                    for (int k = 0; k < kRaw; ++k) raw[u][k] = fs_load_if(X + r * p.ldx + c + k * 4, whole);
                }
#pragma unroll
                for (int u = 0; u < kBatch; ++u) {
                    if constexpr (sizeof(T) == 4) {
                        const uint4 a = raw[u][0], c = raw[u][kRaw - 1];
                        v[u][0] = __uint_as_float(a.x); v[u][1] = __uint_as_float(a.y); v[u][2] = __uint_as_float(a.z); v[u][3] = __uint_as_float(a.w);
                        v[u][4] = __uint_as_float(c.x); v[u][5] = __uint_as_float(c.y); v[u][6] = __uint_as_float(c.z); v[u][7] = __uint_as_float(c.w);
                    } else {
                        const uint32_t a[4] = {raw[u][0].x, raw[u][0].y, raw[u][0].z, raw[u][0].w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) { v[u][2 * k] = __uint_as_float(a[k] << 16); v[u][2 * k + 1] = __uint_as_float(a[k] & 0xFFFF0000u); }
                    }
                }
                if (__any_sync(0xFFFFFFFFu, odd)) {
#pragma unroll
                    for (int u = 0; u < kBatch; ++u) {
                        const int i = i0 + 16 * u, b = (int)((uint32_t)i * recip >> 16), r = i - b * rows;
                        const int64_t c = (int64_t)(kb0 + b) * kF8Block + l * 8;
                        if (i < items && (!p.xvec || c + 8 > p.K))
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[u][e] = c + e < p.K ? (float)X[r * p.ldx + c + e] : 0.f;
                    }
                }
                auto largest = [&]() {
#pragma unroll
                    for (int u = 0; u < kBatch; ++u) {
                        m[u] = fmaxf(0.f, fabsf(v[u][0]));
#pragma unroll
                        for (int e = 1; e < 8; ++e) m[u] = fmaxf(m[u], fabsf(v[u][e]));
                    }
#pragma unroll
                    for (int d = 8; d > 0; d >>= 1)
#pragma unroll
                        for (int u = 0; u < kBatch; ++u) m[u] = fmaxf(m[u], __shfl_xor_sync(0xFFFFFFFFu, m[u], d));
                };
                largest();
                float top = m[0];
#pragma unroll
                for (int u = 1; u < kBatch; ++u) top = fmaxf(top, m[u]);
                if (__any_sync(0xFFFFFFFFu, top == __uint_as_float(0x7F800000u))) {        // (infinities become NaN and enter no scale)
#pragma unroll
                    for (int u = 0; u < kBatch; ++u)
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (fabsf(v[u][e]) == __uint_as_float(0x7F800000u)) v[u][e] = __uint_as_float(0x7FFFFFFFu);
                    largest();
                }
#pragma unroll
                for (int u = 0; u < kBatch; ++u) {
                    const int i = i0 + 16 * u, b = (int)((uint32_t)i * recip >> 16), r = i - b * rows;
                    const uint32_t byte = f8_scale_byte<false>(__float_as_uint(m[u]));
                    const float f = f8_inverse(byte);
                    if (i < items) {
                        const uint32_t lo = f8_pack<false>(v[u][0] * f, v[u][1] * f) | f8_pack<false>(v[u][2] * f, v[u][3] * f) << 16;
                        const uint32_t hi = f8_pack<false>(v[u][4] * f, v[u][5] * f) | f8_pack<false>(v[u][6] * f, v[u][7] * f) << 16;
                        const uint32_t row = xs + (uint32_t)(b * BN * 128 + r * 128);
                        asm volatile("st.shared.v2.b32 [%0], {%1, %2};\n" ::"r"(row + ((((uint32_t)l >> 1) ^ ((uint32_t)r & 7u)) << 4) + ((uint32_t)l & 1u) * 8u), "r"(lo), "r"(hi) : "memory");
                        if (l == 0)
                            asm volatile("st.shared.u8 [%0], %1;\n" ::"r"(xs_scales + (uint32_t)(((kb0 + b) >> 2) - (kb0 >> 2)) * kF8Atom +
                                                                         (uint32_t)((r & 31) * 16 + (r >> 5) * 4 + ((kb0 + b) & 3))), "r"(byte) : "memory");
                    }
                }
            }
            };
            if (items <= 32) pass(std::integral_constant<int, 2>());
            else pass(std::integral_constant<int, 4>());               // (64 items 1.2 us; eight at a time did not fit the registers of half an SM)
            asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
            __syncwarp();
            if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(sm32(&tail.x_ready)) : "memory");
        }
        // ================= sums: group g takes the columns BN / 2 g .. (all 16 where there are no more) =================
        const float *bias = from_here(p.bias);
        if (tid - 64 < 128) {
            const int at = tid - 64, i = p.transposed ? m0 + at : n0 + at;
            tail.bias[at] = bias != nullptr && i < (p.transposed ? p.M : p.N) && (p.transposed || at < BN) ? __uint_as_float(load_free((const uint32_t *)bias + i)) : 0.f;
        }
        const int pieces = BN >= 32 ? BN / 32 : 1 - grp;
        const int chunks = (kb1 - kb0 + kFsChunk - 1) / kFsChunk;
        for (int c = 0; c < chunks; ++c) {
            const uint32_t buf = (uint32_t)c & 1u;
            if (!__all_sync(0xFFFFFFFFu, gt_wait(sm32(&tail.acc_full[buf]), ((uint32_t)c >> 1) & 1u) && s_fail == 0u)) { if (lane == 0) atomicExch(&tail.fail, 1u); break; }
            asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
            const uint32_t t = tmem + ((uint32_t)(q * 32) << 16) + buf * (uint32_t)BN + (uint32_t)(grp * (BN / 2));
#pragma unroll
            for (int k = 0; k < kPieces; ++k)
                if (k < pieces) {
                    uint32_t v[16];
                    fs_load16(t + (uint32_t)k * 16u, v);
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[k][e] = c == 0 ? __uint_as_float(v[e]) : acc[k][e] + __uint_as_float(v[e]);
                }
            asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
            __syncwarp();
            if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(sm32(&tail.acc_free[buf])) : "memory");
        }
    }
    // ================= tensor memory has been read =================
    __syncwarp();
    if (warp == 0) {
        asm volatile("bar.sync 2, 288;\n tcgen05.fence::after_thread_sync;\n" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(cols) : "memory");
    } else if (warp >= 2) asm volatile("tcgen05.fence::before_thread_sync;\n bar.arrive 2, 288;\n" ::: "memory");
    // ================= the shares to the CTAs that store them =================
    const int row = (warp & 3) * 32 + lane, grp = (warp - 2) >> 2;
    const int first = grp * (BN / 2), pieces = BN >= 32 ? BN / 32 : 1 - grp;
    const bool epilogue = warp >= 2;
    if (split > 1) {
        asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
        if (epilogue) {
            // the tile by lines to the ring, which is free; the lines that another CTA stores go to it in one copy, to the place of this rank
            // (lines of BN entries: 16-byte piece j of line r at place j ^ (r % 8), so that the lanes, a line each, meet different banks)
#pragma unroll
            for (int k = 0; k < kPieces; ++k)
                if (k < pieces) {
                    if (p.transposed) {
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            asm volatile("st.shared.f32 [%0], %1;\n" ::"r"(ring + (uint32_t)((first + k * 16 + e) * 128 + row) * 4u), "f"(acc[k][e]) : "memory");
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};\n" ::"r"(ring + (uint32_t)(row * line_bytes) + ((((uint32_t)(first + k * 16) >> 2) + e) ^ ((uint32_t)row & 7u)) * 16u),
                                         "f"(acc[k][4 * e]), "f"(acc[k][4 * e + 1]), "f"(acc[k][4 * e + 2]), "f"(acc[k][4 * e + 3]) : "memory");
                    }
                }
            asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
            asm volatile("bar.sync 1, 256;\n" ::: "memory");
            const int to = tid - 64, n = lines - to * per < per ? lines - to * per : per;
            if (run && to < split && to != rank && n > 0)
                asm volatile("{\n .reg .b32 a, b;\n mapa.shared::cluster.u32 a, %0, %1;\n mapa.shared::cluster.u32 b, %2, %1;\n"
                             " cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [a], [%3], %4, [b];\n}\n"
                             ::"r"(ring + (uint32_t)p.off_recv + (uint32_t)(rank * per * line_bytes)), "r"(to), "r"(sm32(&tail.shares)), "r"(ring + (uint32_t)(to * per * line_bytes)),
                               "r"((uint32_t)(n * line_bytes)) : "memory");
            if (run && !gt_wait(sm32(&tail.shares), 0u)) atomicExch(&tail.fail, 1u);
            __syncwarp();
        }
        // (complete once all shares have arrived everywhere: no CTA leaves while its memory is still read; nothing else passes by it)
        asm volatile("barrier.cluster.arrive.relaxed.aligned;\n" ::: "memory");
    } else __syncthreads();
    // (without a cluster whoever gave up did so before the barrier, and all warps see the same; with one no barrier of the CTA alone follows)
    const bool fine = run && s_fail == 0u;
    const uint8_t *gamma = from_here(p.gamma);
    const int ey = p.bf16 ? 2 : 4;
    if (!epilogue || !fine) {
    } else if (split > 1) {
        // four entries of a line to a thread, the shares in the order of the ranks
        const int l0 = rank * per, n = lines - l0 < per ? lines - l0 : per, shift = p.transposed ? 5 : 31 - __clz(BN >> 2);
        const int in0 = p.transposed ? m0 : n0, in_end = p.transposed ? p.M : p.N, lead0 = p.transposed ? n0 : m0;
        const uint32_t own = ring + (uint32_t)(l0 * line_bytes), recv = ring + (uint32_t)p.off_recv, share = (uint32_t)(per * line_bytes);
        auto join = [&](auto split_c) {
            constexpr int kSplit = decltype(split_c)::value;            // (with branches on the number 600 cycles a turn)
        for (int u = tid - 64; u < n << shift; u += 256) {
            const int l = u >> shift, j = u - (l << shift), in = in0 + j * 4;
            if (in >= in_end) continue;
            const uint32_t at = (uint32_t)(l * line_bytes) + (uint32_t)(p.transposed ? j : j ^ ((l0 + l) & 7)) * 16u;
            float4 w[kSplit];
#pragma unroll
            for (int s = 0; s < kSplit; ++s)
                asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];\n" : "=f"(w[s].x), "=f"(w[s].y), "=f"(w[s].z), "=f"(w[s].w) : "r"((s == rank ? own : recv + (uint32_t)s * share) + at));
            float v[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
            for (int s = 1; s < kSplit; ++s) { v[0] += w[s].x; v[1] += w[s].y; v[2] += w[s].z; v[3] += w[s].w; }
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += tail.bias[j * 4 + e];
            if (gamma != nullptr && load_free(gamma + (int64_t)((lead0 + l0 + l) >> p.bo) * p.NBi + (in >> p.bi)) == 0u) v[0] = v[1] = v[2] = v[3] = 0.f;
            const int64_t out = (int64_t)(lead0 + l0 + l) * in_end + in;
            if (p.vec) {
                if (p.bf16) *(uint2 *)((__nv_bfloat16 *)p.Y + out) = make_uint2(fs_pack(v[0], v[1]), fs_pack(v[2], v[3]));
                else *(float4 *)((float *)p.Y + out) = make_float4(v[0], v[1], v[2], v[3]);
            } else
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (in + e < in_end) {
                        if (p.bf16) ((__nv_bfloat16 *)p.Y)[out + e] = __float2bfloat16_rn(v[e]);
                        else ((float *)p.Y)[out + e] = v[e];
                    }
        }
        };
        if (split == 2) join(std::integral_constant<int, 2>());
        else if (split == 4) join(std::integral_constant<int, 4>());
        else join(std::integral_constant<int, 8>());
    } else {
        const int m = m0 + row;
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
            if (k < pieces) {
                const int c0 = first + k * 16;
                if (p.transposed) {
                    if (m < p.M)
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (c0 + e < valid_n) {
                                const float v = acc[k][e] + tail.bias[row];
                                const int64_t at = (int64_t)(n0 + c0 + e) * p.M + m;
                                if (p.bf16) ((__nv_bfloat16 *)p.Y)[at] = __float2bfloat16_rn(v);
                                else ((float *)p.Y)[at] = v;
                            }
                    continue;
                }
                float v[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = acc[k][e] + tail.bias[c0 + e];
                if (gamma != nullptr && m < p.M) {
#pragma unroll
                    for (int e = 0; e < 16; e += 4)
                        if (c0 + e < valid_n && load_free(gamma + (int64_t)(m >> p.bo) * p.NBi + ((n0 + c0 + e) >> p.bi)) == 0u) v[e] = v[e + 1] = v[e + 2] = v[e + 3] = 0.f;
                }
                if (p.staged) {
                    // to the ring, which is free: slabs of 128 bytes of every row under the swizzle of the stores
                    const uint32_t byte = (uint32_t)(c0 * ey), slab = ring + (byte >> 7) * 16384u + (uint32_t)row * 128u, piece = (byte & 127u) >> 4, sw = (uint32_t)row & 7u;
                    if (p.bf16) {
#pragma unroll
                        for (uint32_t j = 0; j < 2u; ++j)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(slab + (((piece + j) ^ sw) << 4)), "r"(fs_pack(v[8 * j], v[8 * j + 1])),
                                         "r"(fs_pack(v[8 * j + 2], v[8 * j + 3])), "r"(fs_pack(v[8 * j + 4], v[8 * j + 5])), "r"(fs_pack(v[8 * j + 6], v[8 * j + 7])) : "memory");
                    } else {
#pragma unroll
                        for (uint32_t j = 0; j < 4u; ++j)
                            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};\n" ::"r"(slab + (((piece + j) ^ sw) << 4)), "f"(v[4 * j]), "f"(v[4 * j + 1]), "f"(v[4 * j + 2]),
                                         "f"(v[4 * j + 3]) : "memory");
                    }
                } else if (m < p.M) {
                    const int64_t at = (int64_t)m * p.N + n0 + c0;
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        if (p.vec && c0 + e + 4 <= valid_n) {
                            if (p.bf16) *(uint2 *)((__nv_bfloat16 *)p.Y + at + e) = make_uint2(fs_pack(v[e], v[e + 1]), fs_pack(v[e + 2], v[e + 3]));
                            else *(float4 *)((float *)p.Y + at + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
                        } else
#pragma unroll
                            for (int f = 0; f < 4; ++f)
                                if (c0 + e + f < valid_n) {
                                    if (p.bf16) ((__nv_bfloat16 *)p.Y)[at + e + f] = __float2bfloat16_rn(v[e + f]);
                                    else ((float *)p.Y)[at + e + f] = v[e + f];
                                }
                    }
                }
            }
        if (p.staged) {
            asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
            asm volatile("bar.sync 1, 256;\n" ::: "memory");
            if (tid == 64) {
                for (int b = 0; b * 128 < BN * ey; ++b)
                    if (n0 + b * 128 / ey < p.N)
                        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];\n"
                                     ::"l"(&p.tmy), "r"(ring + (uint32_t)b * 16384u), "r"(n0 * ey + b * 128), "r"(m0) : "memory");
                asm volatile("cp.async.bulk.commit_group;\n cp.async.bulk.wait_group.read 0;\n" ::: "memory");
            }
        }
    }
    __syncwarp();
    if (split > 1) asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
    else __syncthreads();
    if (s_fail == 1u && tid == 0) atomicMax(p.status, (int)BSP_ERR_TIMEOUT);
}

// ---- large products: persistent pairs of CTAs ----

constexpr int kFpThreads = 384;                     // producer warp, MMA warp, two that idle, two groups of four epilogue warps
// Registers of a thread: the float32 form of the epilogue holds 128 sums.  (40 + 2 x 232 is 3 x 168, what the CTA is launched with.)
constexpr int kFpFew = 40, kFpMany = 232;
constexpr int kFpStage = 32768;                     // 128 rows of A and 128 rows (half of the tile's) of B
constexpr int kFpStages = 5;
constexpr int kFpScales = 3 * kF8Atom;          // scales of a stage: 128 rows of A, 256 rows of B
constexpr int kFpStaging = 16384;                   // of a group: 128 rows of 128 bytes
constexpr int kFpChunk = 16;                        // most blocks of a chunk (64 instructions: sums of 8192 entries off by 5.5e-7; 22 blocks 9.7e-7)
// ... for a bfloat16 output, whose own rounding is 2^-9: 256 instructions, off by 1.1e-5 of a sum of products of one sign (2048 entries 1.8e-6).  Without
// an end the error grew with the sum: 6.5e-5 at 32768 entries, 8.3e-4 at 262144.  Joining costs 2 % of the time of 8192 x 16384 x 4096.
constexpr int kFpChunkHalf = 64;
constexpr int kFpSecond = 192;                      // first column of the second accumulator: the last 64 of the first lie under it

struct FpParams {
    CUtensorMap tma, tmb, tmb64;  // values as bytes, (K, rows), box 128 x 128 (64 rows of B in tiles of 128 columns), 128-byte swizzle
    CUtensorMap tsa, tsb;         // scales as words, (128, atoms, rows / 128), boxes of one and of two atoms
    CUtensorMap tmy;              // Y as bytes, (N ey, M), box 128 bytes x 128 rows, 128-byte swizzle
    int M, N, n_kb, tiles_n, n_tiles;
    int n_wide;                   // tiles of 256 columns; the rest are halves of such
    int chunk;                    // blocks of 128 entries that are summed in the tensor core before float32 registers take over
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
constexpr int kFpSmem = kFpStages * (kFpStage + kFpScales) + 2 * kFpStaging + (int)sizeof(FpTail);
static_assert(kFpSmem <= kFsSmem, "shared memory of a CTA");

// Tile `tile` of a pair: its rows 256 mp .., its columns n0 .., whether it has 128 columns instead of 256.
__device__ __forceinline__ void fp_tile(const FpParams &p, int tile, int &mp, int &n0, bool &narrow)
{
    int tn, half = 0, t = tile;
    narrow = tile >= p.n_wide;
    if (narrow) { half = (tile - p.n_wide) & 1; t = p.n_wide + ((tile - p.n_wide) >> 1); }
    gt_divmod(t, p.tiles_n, p.m_tn, mp, tn);
    n0 = tn * 256 + half * 128;
}

// A pair of CTAs owns tiles of 256 x 256: CTA r of the pair the rows 128 r .. of the tile, and loads these and its half of the tile's rows
// of B; the leader issues MMAs of 256 x 256 x 32 for both.  Two accumulators of 256 columns that overlap by 64, whose columns the
// epilogue reads first, leave 64 columns for the scales: the next tile's MMAs start when these 64 have been read.
// Where the tiles of the last wave leave half of the pairs idle they are halved (4096 x 4096 sums of 8192 entries, 34 tiles in the last wave of 74
// pairs: 131 -> 125 us when this was added).
// kSums: chunks of up to kFpChunk blocks (kFpChunkHalf for a bfloat16 output) are summed in the tensor core, these in registers (as above).  A
// change of accumulators costs the end of the last MMAs, a read of the columns that overlap and the start of the next MMAs: as few chunks as the
// error allows, and where one is enough for a bfloat16 output it goes from tensor memory to the store without the registers in between.
template <bool kF32, bool kSums>
__global__ void __launch_bounds__(kFpThreads, 1) gemm_f8_pair_kernel(const __grid_constant__ FpParams p)
{
    static_assert(kSums || !kF32, "a float32 output is joined in registers");
    extern __shared__ __align__(1024) uint8_t smem[];
    FpTail &tail = *(FpTail *)(smem + kFpStages * (kFpStage + kFpScales) + 2 * kFpStaging);
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
        const CUtensorMap *maps[6] = {&p.tma, &p.tmb, &p.tmb64, &p.tsa, &p.tsb, &p.tmy};
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
                int mp, nt;
                bool narrow;
                fp_tile(p, tile, mp, nt, narrow);
                const int ma = 2 * mp + (int)rank, m0 = ma * 128, n0 = nt + (int)rank * (narrow ? 64 : 128);
                const CUtensorMap *tmb = narrow ? &p.tmb64 : &p.tmb;
                const uint32_t values = narrow ? 16384u + 8192u : (uint32_t)kFpStage;
                if (s_fail) { ok = false; break; }
                for (int kb = 0; kb < n_kb; ++kb) {
                    if (!__all_sync(0xFFFFFFFFu, gt_poll(empty0 + slot * 8u, par))) { ok = false; break; }
                    const uint32_t with = (kb & 3) == 0 ? 1u : 0u, dst = ring + slot * kFpStage, sdst = scales + slot * kFpScales;
                    const uint32_t bytes = 2u * (values + with * kFpScales), bar = lead_full0 + slot * 8u;
                    asm volatile("{\n .reg .pred e, l, s;\n elect.sync _|e, 0xFFFFFFFF;\n setp.eq.u32 l, %2, 0;\n and.pred l, l, e;\n setp.ne.b32 s, %3, 0;\n and.pred s, s, e;\n"
                                 " @l mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n"
                                 " @s cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%11], [%12, {%15, %13, %14}], [%4];\n"
                                 " @s cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%16], [%17, {%15, %13, %18}], [%4];\n"
                                 " @e cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%5], [%6, {%7, %8}], [%4];\n"
                                 " @e cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%9], [%10, {%7, %19}], [%4];\n}\n"
                                 ::"r"(full0 + slot * 8u), "r"(bytes), "r"(rank), "r"(with), "r"(bar), "r"(dst), "l"(&p.tma), "r"(kb * 128), "r"(m0), "r"(dst + 16384u), "l"(tmb),
                                   "r"(sdst), "l"(&p.tsa), "r"(kb >> 2), "r"(ma), "r"(0), "r"(sdst + 512u), "l"(&p.tsb), "r"(nt >> 7), "r"(n0) : "memory");
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
            int left = 0;                 // blocks of this chunk to come
            bool ok = true, full_now = false;
            for (int tile = t_first; tile < p.n_tiles && ok; tile += t_step) {
                const uint32_t tile_idesc = p.idesc | ((tile >= p.n_wide ? 16u : 32u) << 17);
                for (int kb = 0; kb < n_kb; ++kb) {
                    const bool fresh = left == 0;
                    if (fresh) left = p.chunk;
                    --left;
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
                    const uint32_t a16 = (ring + slot * kFpStage) >> 4, s16 = (scales + slot * kFpScales) >> 4;
                    const uint64_t da = kGtDesc | (uint64_t)(a16 & 0x3FFFu), db = kGtDesc | (uint64_t)((a16 + 1024u) & 0x3FFFu);
                    const uint64_t ds = kFsScaleDesc | (uint64_t)(s16 & 0x3FFFu);
                    const uint32_t fa = tmem + 448u + set * 16u, fb = fa + 8u, id = (uint32_t)kb & 3u, idesc = tile_idesc | (id << 4) | (id << 29);
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
                    if (kb + 1 == n_kb || left == 0) {
                        left = 0;
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
        // The groups take 64 columns (128 bytes of bfloat16; 32 of float32) in turn, first the ones that lie under the other accumulator: the
        // upper end of the first accumulator, the lower end of the second.
        const int q = warp & 3, grp = (warp - 4) >> 2, row = q * 32 + lane;
        const uint32_t sg = staging + (uint32_t)(grp * kFpStaging), lanes = (uint32_t)(q * 32) << 16;
        const bool issuer = q == 0 && lane == 0;
        const float *bias_of = from_here(p.bias);
        const uint8_t *gamma = from_here(p.gamma);
        const int chunks = kSums ? (n_kb + p.chunk - 1) / p.chunk : 1;
        uint32_t unit = 0;
        bool ok = true;
        // (Only tensor memory passes by this barrier, and the tcgen05 fences order that; a release at cluster scope also waited for the
        // thread's other memory operations, 1700 cycles at every change of accumulators: 118 -> 105 us for 4096 x 8192 x 4096.)
        auto hand_back = [&]() {
            asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
            __syncwarp();
            if (lane == 0) asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];\n" ::"r"(lead_free) : "memory");
        };
        for (int tile = t_first; tile < p.n_tiles; tile += t_step) {
            int mp, n0;
            bool narrow;
            fp_tile(p, tile, mp, n0, narrow);
            const int m0 = (2 * mp + (int)rank) * 128, m = m0 + row;
            {   // the bias of the group's 128 columns (everybody is past the barriers of the last tile's rounds)
                const int n = n0 + (kF32 ? (row >> 5) * 64 + grp * 32 + (row & 31) : (row >> 6) * 128 + grp * 64 + (row & 63));
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
            if constexpr (kSums) {
                // 32 columns of the tile at a time: a round of the stores in float32, half of one in bfloat16
                const int own = grp * (kF32 ? 32 : 64);
                auto at = [](int r) { return kF32 ? r * 64 : (r >> 1) * 128 + (r & 1) * 32; };
                float acc[4][32];
                for (int c = 0; c < chunks; ++c, ++unit) {
                    const uint32_t second = unit & 1u, t = tmem + lanes + second * kFpSecond + (uint32_t)own;
                    if (s_fail) ok = false;
                    if (ok && !gt_wait(sm32(&tail.acc_full[second]), (unit >> 1) & 1u)) ok = false;
                    __syncwarp();
                    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                    auto take = [&](auto r_c) {
                        constexpr int r = decltype(r_c)::value;
                        if (r >= 2 && narrow) return;
                        uint32_t v[32];
                        gt_load32(t + (uint32_t)at(r), v);
#pragma unroll
                        for (int e = 0; e < 32; ++e) acc[r][e] = c == 0 ? __uint_as_float(v[e]) : acc[r][e] + __uint_as_float(v[e]);
                    };
                    if constexpr (!kF32) {
                        // all 64 columns that overlap are one group's
                        if (second == (uint32_t)grp) hand_back();
                        if (second) {
                            take(std::integral_constant<int, 0>());
                            take(std::integral_constant<int, 1>());
                            if (second != (uint32_t)grp) hand_back();
                            take(std::integral_constant<int, 2>());
                            take(std::integral_constant<int, 3>());
                        } else {
                            take(std::integral_constant<int, 2>());
                            take(std::integral_constant<int, 3>());
                            if (second != (uint32_t)grp) hand_back();
                            take(std::integral_constant<int, 0>());
                            take(std::integral_constant<int, 1>());
                        }
                    } else if (second) {
                        take(std::integral_constant<int, 0>());
                        hand_back();
                        take(std::integral_constant<int, 1>());
                        take(std::integral_constant<int, 2>());
                        take(std::integral_constant<int, 3>());
                    } else {
                        take(std::integral_constant<int, 3>());
                        hand_back();
                        take(std::integral_constant<int, 0>());
                        take(std::integral_constant<int, 1>());
                        take(std::integral_constant<int, 2>());
                    }
                }
                gt_group_sync(1 + grp);                                  // (the bias is there)
                if constexpr (!kF32) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (h == 1 && narrow) break;
                        uint32_t out[32];
                        const float *b = tail.bias[grp] + h * 64;
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const int i = 2 * e & 31, r = 2 * h + (e >> 4);
                            out[e] = fs_pack(acc[r][i] + b[2 * e], acc[r][i + 1] + b[2 * e + 1]);
                        }
                        store(out, h * 128 + own);
                    }
                } else
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int c0 = at(r) + own;
                    if (r >= 2 && narrow) break;
                    uint32_t out[32];
                    const float *b = tail.bias[grp] + r * 32;
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
                    if (half == 1u && narrow) {
                        if (r == 0 && second != (uint32_t)grp) hand_back();
                        continue;
                    }
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

// Y as bytes in rows of `row` bytes, in boxes of 128 bytes x 128 rows.
bsp_status fs_y_map(CUtensorMap *map, void *Y, int64_t rows, int64_t row)
{
    GtEncodeFn enc = gt_encode();
    if (!enc) return BSP_ERR_CUDA;
    const cuuint64_t gdim[2] = {(cuuint64_t)row, (cuuint64_t)rows}, gstr[1] = {(cuuint64_t)row};
    const cuuint32_t box[2] = {128u, 128u}, estr[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, Y, gdim, gstr, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? BSP_OK : BSP_ERR_CUDA;
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
    const int pairs_there = sms / 2;
    F8PairTiles t;
    if (!f8_pair_tiles(p.M, p.N, pairs_there, t)) return BSP_ERR_SHAPE;
    p.tiles_n = t.across; p.n_wide = t.whole; p.n_tiles = t.all;
    p.m_tn = gt_magic(p.tiles_n);
    const int most = ey == 2 ? kFpChunkHalf : kFpChunk, chunks = (p.n_kb + most - 1) / most;
    p.chunk = (p.n_kb + chunks - 1) / chunks;
    // formats, scales of 8 exponent bits, M / 128 (N / 8 by tile)
    p.idesc = ((x.type == BSP_E5M2 ? 1u : 0u) << 7) | ((w.type == BSP_E5M2 ? 1u : 0u) << 10) | (1u << 23) | (2u << 27);
    p.bias = bias;
    if (wd) { p.gamma = gamma; p.bo = f8_log2(wd->bo); p.bi = f8_log2(wd->bi); p.NBi = wd->I / wd->bi; }
    p.status = (int *)ws;
    bsp_status rc = fs_map(&p.tma, x, 128);
    if (rc == BSP_OK) rc = fs_map(&p.tmb, w, 128);
    if (rc == BSP_OK) rc = fs_map(&p.tmb64, w, 64);
    if (rc == BSP_OK) rc = fp_scale_map(&p.tsa, x, 1);
    if (rc == BSP_OK) rc = fp_scale_map(&p.tsb, w, 2);
    if (rc == BSP_OK) rc = fs_y_map(&p.tmy, Y, p.M, (int64_t)p.N * ey);
    if (rc != BSP_OK) return rc;
    const int pairs = p.n_tiles < pairs_there ? p.n_tiles : pairs_there;
    const auto kernel = ey == 4 ? gemm_f8_pair_kernel<true, true> : chunks > 1 ? gemm_f8_pair_kernel<false, true> : gemm_f8_pair_kernel<false, false>;
    BSP_CUDA_OK(launch_after_clusters(kernel, dim3((unsigned)(2 * pairs)), dim3(kFpThreads), kFpSmem, st, 2, 1, p));
    return BSP_OK;
}

}  // namespace

namespace {

// What a device has room for: SMs, and clusters of 1, 2, 4 and 8 CTAs of the tile kernel at a time (those with X take half of an SM).
struct FsDevice { int sms, clusters[4], clusters_x[4]; };
bsp_status fs_device(FsDevice &d)
{
    static std::atomic<int> state[kGtMaxDevices];          // 0 unknown, 1 being written, 2 known
    static FsDevice known[kGtMaxDevices];
    int dev = 0;
    BSP_CUDA_OK(cudaGetDevice(&dev));
    if (dev < 0 || dev >= kGtMaxDevices) return BSP_ERR_CUDA;
    if (state[dev].load(std::memory_order_acquire) == 2) {
        d = known[dev];
        return BSP_OK;
    }
    d = {};
    BSP_CUDA_OK(cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev));
    void (*const tiles[3])(const FsParams) = {gemm_f8_tile_kernel<void>, gemm_f8_tile_kernel<float>, gemm_f8_tile_kernel<__nv_bfloat16>};
    for (auto k : tiles) BSP_CUDA_OK(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kFsSmem));
    void (*const pairs[3])(const FpParams) = {gemm_f8_pair_kernel<true, true>, gemm_f8_pair_kernel<false, true>, gemm_f8_pair_kernel<false, false>};
    for (auto k : pairs) BSP_CUDA_OK(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kFpSmem));
    for (int i = 0; i < 4; ++i) {
        cudaLaunchAttribute at = {};
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim.x = 1u << i; at.val.clusterDim.y = at.val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(1024); cfg.blockDim = dim3(kFsThreads); cfg.dynamicSmemBytes = kFsSmem; cfg.attrs = &at; cfg.numAttrs = 1;
        BSP_CUDA_OK(cudaOccupancyMaxActiveClusters(&d.clusters[i], gemm_f8_tile_kernel<void>, &cfg));
        cfg.dynamicSmemBytes = kFsSmem / 2 - 1024;
        BSP_CUDA_OK(cudaOccupancyMaxActiveClusters(&d.clusters_x[i], gemm_f8_tile_kernel<float>, &cfg));
    }
    if (d.sms < 1 || d.clusters[0] < 1 || d.clusters_x[0] < 1) return BSP_ERR_CUDA;
    int none = 0;
    if (state[dev].compare_exchange_strong(none, 1)) {
        known[dev] = d;
        state[dev].store(2, std::memory_order_release);
    }
    return BSP_OK;
}

// What FsParams and a choice of kernel follow from: x [M][K] times w [N][K], or, where `X` is given, its rows instead of x's.
struct FsJob {
    const bsp_f8 *x, *w;
    const void *X;
    bsp_dtype xtype;
    int64_t P, ldx;
    const float *bias;
    const bsp_wdesc *wd;
    const uint8_t *gamma;
    void *Y;
    bsp_dtype ytype;
    void *ws;
};

// Columns of a tile and CTAs that share the summed axis: the pair with the lowest estimate in cycles.  A block of 128 entries costs its MMAs or
// its loads, at about 50 bytes a clock and SM; what comes before and after was measured by phases (1023 x 2048 x 1000 and 1024 x 12544 x 256: 4600
// cycles for 64 columns without a cluster; 7100 for 64 over four CTAs and 10700 for 128 over two, whose shares take 0.6 cycles an entry).
struct FsChoice { int BN, split; double cycles; };
constexpr int64_t kFsRow = 0x7FFFFF00;               // bytes of a row of Y that a tensor map's coordinates, which count bytes, reach
constexpr int kFsPlaceRows = 768;                   // rows of 128 bytes of X that a CTA may hold where it quantises X itself
FsChoice fs_choose(const FsDevice &d, int64_t M, int64_t N, int n_kb, bool transposed, bool in_place)
{
    FsChoice best = {0, 0, -1.0};
    const int widths[4] = {16, 32, 64, 128};
    for (int i = 0; i < 4; ++i) {
        const int bn = widths[i];
        if (transposed ? (bn < N || (i > 0 && widths[i - 1] >= N)) : (bn > 32 && widths[i - 1] >= N) || bn < 32) continue;
        for (int j = 0; j < 4; ++j) {
            const int split = 1 << j, there = in_place ? d.clusters_x[j] : d.clusters[j];
            if (there < 1 || (split > 1 && n_kb < 2 * split)) continue;
            const double tiles = (double)f8_blocks(M) * (double)((N + bn - 1) / bn);
            const double waves = tiles <= there ? 1.0 : (double)(int64_t)((tiles + there - 1) / there);
            const double mma = 4.0 * (32 + bn / 4 > bn / 2 ? 32 + bn / 4 : bn / 2), feed = 128.0 * (128 + (in_place ? 0 : bn)) / 50.0;
            const int kb = (n_kb + split - 1) / split;
            if (in_place && kb * bn > kFsPlaceRows) continue;
            const int items = kb * (int)(in_place ? N : 0);                 // rows of 128 entries of X
            const double rows_x = items == 0 ? 0.0 : items <= 32 ? 1200.0 : 2400.0 * ((items + 63) / 64);
            const double block = mma > feed ? mma : feed, entries = transposed ? (double)N * 128 : (double)(M < 128 ? M : 128) * bn;
            const double alone = 3600.0 + 16.0 * bn, joined = (transposed ? 3400.0 + 60.0 * split : split == 8 ? 8000.0 : 5000.0 + 250.0 * split) + 0.47 * entries / split;
            const double cycles = waves * (rows_x + kb * (transposed || block > 480.0 ? block : 480.0) + (split > 1 ? joined : alone));
            if (best.cycles < 0 || cycles < best.cycles) best = {bn, split, cycles};
        }
    }
    return best;
}

bsp_status launch_tiles(const FsDevice &d, const FsJob &j, const FsChoice &c, bool transposed, cudaStream_t st)
{
    FsParams p = {};
    const int64_t K = j.w->cols, P = j.X ? j.P : j.x->rows;
    p.transposed = transposed;
    const bsp_f8 *a = transposed ? j.w : j.x, *b = transposed ? j.x : j.w;       // (b is NULL where X is quantised in place)
    p.M = (int)(transposed ? j.w->rows : P); p.N = (int)(transposed ? P : j.w->rows);
    p.BN = c.BN; p.split = c.split;
    p.n_kb = (int)f8_blocks(K);
    p.atoms = f8_atoms(K);
    p.sa = (const uint8_t *)a->scale; p.sb = b ? (const uint8_t *)b->scale : nullptr;
    int64_t ctas;
    if (!f8_tile_grid(p.M, p.N, p.BN, p.split, p.tiles_n, ctas)) return BSP_ERR_SHAPE;
    const int ey = j.ytype == BSP_BF16 ? 2 : 4, kb = (p.n_kb + p.split - 1) / p.split;
    p.staged = !transposed && p.split == 1 && p.BN >= 64 && (int64_t)p.N * ey % 16 == 0 && (int64_t)p.N * ey < kFsRow;
    // ring | X in 8 bits and its scales | shares of the cluster's CTAs | scales of the stages | barriers
    p.stage_bytes = 16384 + (j.X ? 0 : p.BN * 128);
    const int x_bytes = j.X ? kb * p.BN * 128 + (kb / 4 + 2) * kF8Atom : 0, recv = p.split > 1 ? p.BN * 512 : 0;
    const int tail = (int)sizeof(FsTail);
    p.stages = (kFsSmem - tail - x_bytes - recv) / (p.stage_bytes + kFsScales);
    if (p.stages > kFsMaxStages) p.stages = kFsMaxStages;
    if (p.stages > kb) p.stages = kb;
    // (with X: half of an SM, so that the next layer's CTAs find room while this one's run)
    const int half = (kFsSmem / 2 - 1024 - tail - x_bytes - recv) / (p.stage_bytes + kFsScales);
    if (j.X && half >= 2 && p.stages > half) p.stages = half;
    int ring = p.stages * p.stage_bytes;
    if (p.staged && ring < p.BN * ey * 128) ring = p.BN * ey * 128;
    if (p.split > 1 && ring < p.BN * 512) ring = p.BN * 512;
    p.off_x = ring; p.off_recv = ring + (x_bytes + 1023) / 1024 * 1024; p.off_scales = p.off_recv + recv; p.off_tail = p.off_scales + p.stages * kFsScales;
    const int smem = p.off_tail + tail;
    if (p.stages < 1 || smem > kFsSmem) return BSP_ERR_SHAPE;
    // formats of A and B, N / 8, scales of 8 exponent bits, M / 128; both operands K-major
    const uint32_t fa = a->type == BSP_E5M2 ? 1u : 0u, fb = b && b->type == BSP_E5M2 ? 1u : 0u;
    p.idesc = (fa << 7) | (fb << 10) | ((uint32_t)(p.BN >> 3) << 17) | (1u << 23) | (1u << 27);
    p.Y = (uint8_t *)j.Y; p.bf16 = j.ytype == BSP_BF16;
    p.vec = (transposed ? p.M : p.N) % 4 == 0;
    p.bias = j.bias;
    if (j.wd) { p.gamma = j.gamma; p.bo = f8_log2(j.wd->bo); p.bi = f8_log2(j.wd->bi); p.NBi = j.wd->I / j.wd->bi; }
    p.X = j.X; p.ldx = j.ldx; p.K = K;
    if (j.X) p.xvec = (uintptr_t)j.X % 16 == 0 && j.ldx * elem_bytes(j.xtype) % 16 == 0;
    p.status = (int *)j.ws;
    bsp_status rc = fs_map(&p.tma, *a, 128);
    if (rc == BSP_OK && b) rc = fs_map(&p.tmb, *b, p.BN);
    if (rc == BSP_OK && p.staged) rc = fs_y_map(&p.tmy, j.Y, p.M, (int64_t)p.N * ey);
    if (rc != BSP_OK) return rc;
    const auto kernel = !j.X ? gemm_f8_tile_kernel<void> : j.xtype == BSP_F32 ? gemm_f8_tile_kernel<float> : gemm_f8_tile_kernel<__nv_bfloat16>;
    BSP_CUDA_OK(launch_after_clusters(kernel, dim3((unsigned)ctas), dim3(kFsThreads), (size_t)smem, st, p.split, 1, p));
    return BSP_OK;
}

}  // namespace

bsp_status launch_gemm_f8(const bsp_f8 &x, const bsp_f8 &w, const float *bias, const bsp_wdesc *wd, const uint8_t *gamma, void *Y, bsp_dtype ytype,
                          void *ws, cudaStream_t st)
{
    FsDevice d;
    const bsp_status rc = fs_device(d);
    if (rc != BSP_OK) return rc;
    // few rows of x become the columns of the MMA, whose rows are then the channels
    const bool transposed = wd == nullptr && x.rows <= 64;
    const int n_kb = (int)f8_blocks(x.cols);
    const FsChoice c = fs_choose(d, transposed ? w.rows : x.rows, transposed ? x.rows : w.rows, n_kb, transposed, false);
    // pairs of CTAs, where a tensor map can describe the rows of Y
    const double tiles = (double)((x.rows + 255) / 256) * (double)((w.rows + 255) / 256), pairs = d.sms / 2;
    const int64_t row = w.rows * (ytype == BSP_BF16 ? 2 : 4);
    if (!transposed && d.sms >= 2 && row % 16 == 0 && row < kFsRow) {
        const double waves = (double)(int64_t)(tiles / pairs), rest = tiles - waves * pairs;
        const double cycles = (waves + (rest == 0.0 ? 0.0 : 2.0 * rest <= pairs ? 0.74 : 1.0)) * (n_kb * 690.0 + 1500.0) + 4500.0;
        if (cycles < c.cycles) return launch_pairs(x, w, bias, wd, gamma, Y, ytype, ws, d.sms, st);
    }
    return launch_tiles(d, FsJob{&x, &w, nullptr, BSP_F32, 0, 0, bias, wd, gamma, Y, ytype, ws}, c, transposed, st);
}

// Few rows of X are quantised by the CTAs that multiply them (each its share of the channels, again for every 128 channels of the output),
// others go through `x`, which lies in the workspace.
bsp_status launch_linear_f8(const bsp_f8 &w, const void *X, bsp_dtype xtype, int64_t P, int64_t ldx, const bsp_f8 &x, const float *bias, void *Y,
                            bsp_dtype ytype, void *ws, cudaStream_t st)
{
    FsDevice d;
    bsp_status rc = fs_device(d);
    if (rc != BSP_OK) return rc;
    if (P <= 64) {
        const int n_kb = (int)f8_blocks(w.cols);
        const FsChoice c = fs_choose(d, w.rows, P, n_kb, true, true);
        // (another launch costs about 3500 cycles: 16 positions on 2048 x 1000 weights 4.5 us in place, 6.3 in two launches; 64 on 4096 x 4096 20 and 9.5)
        if (c.cycles >= 0 && c.cycles <= fs_choose(d, w.rows, P, n_kb, true, false).cycles + 3500.0) return launch_tiles(d, FsJob{nullptr, &w, X, xtype, P, ldx, bias, nullptr, nullptr, Y, ytype, ws}, c, true, st);
    }
    rc = launch_quantize_f8(X, xtype, P, w.cols, ldx, nullptr, nullptr, &x, nullptr, nullptr, ws, st);
    return rc != BSP_OK ? rc : launch_gemm_f8(x, w, bias, nullptr, nullptr, Y, ytype, ws, st);
}

}  // namespace bsp
