// The contraction of the linear cross entropy on the tensor cores, with the softmax statistics, the probabilities or
// the gradient's scaling in its epilogue.
//
// CTA pairs (tcgen05 cta_group::2) on tiles of 256 rows x bn columns: each CTA stages its 128 rows of A and half of
// the columns' B by TMA (64 of K per stage, 128-byte swizzle), the leader issues M = 256 MMAs, and two
// accumulators in tensor memory let the epilogue of a tile run under the MMAs of the next.  K-major tiles are one box
// of [rows][64]; MN-major tiles (a matrix read transposed) are boxes of [64 of K][64 of MN], one behind the other.
//
// Epilogues, two warps per TMEM lane quarter, each on one half of the tile's columns, a thread per row:
//   LSE    running maximum m and sum s of 2^(z log2 e - m), over the half tile: one (m, s) per row and half tile goes to
//          memory instead of bn logits
//   PROB   p = 2^(z log2 e - lse2), minus one at the target, as the 16-bit operand of the two gradient products
//   ROW    both in one, where a tile holds all classes: the two warps of a quarter exchange their halves' (m, s)
//   STORE  scaled and rounded once, or added to an fp32 slab
// Outputs go through shared memory in blocks of 32 rows x 32 columns and from there by TMA (or, for rows that start anywhere,
// turned, by the lanes): a thread holds a row, and 16 bytes of 32 different rows per store instruction cost the
// epilogue more than its arithmetic (PROB, 919 x 50021 from 1000 features: 134 us stored by the threads, 87 without stores).
#include <cuda.h>
#include <atomic>

#include "ops_common.cuh"
#include "gemm_tc.cuh"
#include "tc_ptx.cuh"
#include "xent_gemm.cuh"

namespace cert {

namespace {

constexpr int BM = 128;
constexpr int BK = 64;
constexpr int kEpiWarps = 8;
constexpr int kThreads = 64 + kEpiWarps * 32;
constexpr int kATile = BM * BK * 2;
constexpr int kMaxStages = 12;
// The tensor cores truncate as they add to an accumulator: a bias that grows with the number of additions (losses of 4096
// features 2.9e-6 off, relative, in one accumulator).  Where fp32 accuracy is wanted (SUMS) an accumulator takes only this
// many K blocks, 512 terms of float32 operands (six products each) or 1024 of 16-bit ones, and the epilogue's threads add
// the results in registers, rounded to nearest.  16-bit operands, 256 rows, 8192 classes, 1024 to 8192 features, relative
// error of the losses: 1024 terms 1.5e-7 to 3.5e-7, 512 terms 0.8e-7 to 2.2e-7, a float32 product 0.5e-7 to 1.8e-7 for
// values around zero and 5e-7 to 4e-6 for positive ones.  64 rows, 65536 classes, 4096 features, loss alone: 114.7 us
// against 124.0 with 512 terms; 4096 rows, 32768 classes, 2048 features, with gradients: 1.62 ms against 1.69.
constexpr int kSumBlocks32 = 8, kSumBlocks16 = 16;
// Gradient products of 16-bit operands are rounded to that type, which hides the bias of a short accumulator and not of a long one:
// for terms of one sign it is some 1.2e-7 to 2.3e-7 per 16 of them.  So K beyond 4096 terms (float16; its rounding's root mean
// square is 2.1e-4) or 32768 (bfloat16, 1.7e-3) goes into accumulators of 4096 terms: the bias stays at 6e-5.
// float16, 262144 rows behind a ReLU, 512 features, 8192 classes: dW 9.7e-4 off, relative, in one accumulator, 2.9e-4 so, its
// rounding alone 2.1e-4; 1531 x 1000 x 50021 with 40 % ignored: 454 us against 448.
constexpr int kSumBlocksStore = 64;
constexpr int kStoreTermsHalf = 4096, kStoreTermsBf16 = 32768;
// Probabilities take their logits' error times the logit; with more features than this their logits are added up as the losses'
// are, to the same bits.  (Always: 1531 x 1000 x 50021 483 us against 455.)
constexpr int kProbTermsHalf = 1024, kProbTermsBf16 = 4096;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct __align__(16) Bars {
    uint64_t full[kMaxStages];
    uint64_t empty[kMaxStages];
    uint64_t acc_full[2];
    uint64_t acc_empty[2];
    uint64_t row_meet[4];                // ROW: the two warps of a quarter
    uint32_t tmem_base;
    uint32_t abort_flag;
};

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// The element of an unrolled array whose number is `at`: as a comparison per element the compiler turns it into an index,
// and the array goes to local memory.
__device__ __forceinline__ void select_if(float &to, float from, int at, int e) {
    asm("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %2, %3;\n\tselp.f32 %0, %1, %0, p;\n\t}" : "+f"(to) : "f"(from), "r"(at), "r"(e));
}
__device__ __forceinline__ void minus_if(float &x, float y, int at, int e) {
    asm("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %2, %3;\n\t@p sub.f32 %0, %0, %1;\n\t}" : "+f"(x) : "f"(y), "r"(at), "r"(e));
}

// Half of what tmem_ld32 reads: beside 128 sums a thread has no room for 32 more values (1531 x 1000 x 50021, float16: 443 us
// against 463 with 32, 64 x 65536: 122 against 124, 1024 x 1024 x 8192 float32: 368 against 375).
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr)
        : "memory");
}

template <int PENDING>
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PENDING) : "memory"); }
// A lane's 32 16-bit numbers as its row of a 32 x 32 block, the 16-byte pieces exchanged as TMA's 64-byte swizzle has them.
__device__ __forceinline__ void block16(uint8_t *block, int lane, const uint32_t (&w)[16]) {
#pragma unroll
    for (int g = 0; g < 4; ++g)
        *reinterpret_cast<uint4 *>(block + lane * 64 + ((g ^ ((lane >> 1) & 3)) << 4)) = make_uint4(w[g * 4], w[g * 4 + 1], w[g * 4 + 2], w[g * 4 + 3]);
}
// The warp's block on its way; add: to what is there, in fp32 (one launch adds to a place once, so no order matters).
__device__ __forceinline__ void send_block(const CUtensorMap *map, const uint8_t *block, int x, int y, int lane, bool add) {
    fence_async_smem();
    __syncwarp();
    if (lane == 0) {
        if (add)
            asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.bulk_group [%0, {%2, %3}], [%1];"
                         ::"l"(map), "r"(smem_u32(block)), "r"(x), "r"(y) : "memory");
        else tma_store_2d(map, smem_u32(block), x, y);
        tma_store_commit();
    }
}

// Descriptor of an MN-major tile: 64 elements of MN per 128-byte row, a row per k; 8-row groups 1024 bytes apart, the
// next 64 elements of MN one box (64 rows = 8192 bytes) further.
__device__ __forceinline__ uint64_t make_desc_mn(uint32_t smem_addr) {
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr >> 4) & 0x3FFF);
    d |= (uint64_t)(8192 >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// The bounded wait of the pipelines, by a whole warp with one answer for all its lanes.  A barrier that is ready costs one
// instruction and a vote; the flag that another warp gave up is looked at only where there is something to wait for (a
// stage's MMAs are 512 cycles, every load on this path counts).
__device__ __forceinline__ bool pipe_wait(uint32_t bar, uint32_t parity, volatile uint32_t *abort_flag) {
    if (__all_sync(0xffffffffu, try_wait(bar, parity))) return true;
    const long long t0 = clock64();
    while (true) {
        const bool ready = __all_sync(0xffffffffu, try_wait(bar, parity));
        const bool out = *abort_flag || (unsigned long long)(clock64() - t0) > kWaitCycles;
        if (__any_sync(0xffffffffu, out)) return false;
        if (ready) return true;
    }
}

// Two warps meet: both have written, or read, what they share before either goes on.  A warp that gave up elsewhere never comes,
// so this wait has its limit too (a hardware barrier has none).
__device__ __forceinline__ bool pair_meet(uint64_t *bar, uint32_t &phase, int lane, volatile uint32_t *abort_flag) {
    __syncwarp();
    if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
    const bool met = pipe_wait(smem_u32(bar), phase, abort_flag);
    phase ^= 1;
    return met;
}

// One lane of a converged warp.  The producer and the MMA issuer run as whole warps and elect a lane for the instruction
// itself: what they count up is then known to be the same in all lanes and sits in uniform registers, where the descriptors,
// coordinates and barriers of TMA and MMA instructions have to be (as one thread's values they are moved there each time:
// 340 ns per 64 of K instead of 512 cycles).
__device__ __forceinline__ bool elect_one() {
    uint32_t is;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
    return is != 0;
}

struct Tile { int m, n, split; };

// Tiles in the order they are handed out: `raster` row panels together, all their column tiles, panels fastest.  The
// pairs that run at the same time then share both operands' tiles in L2.
__device__ __forceinline__ Tile tile_of(int t, int tiles_m, int tiles_n, int raster) {
    Tile r;
    const int per = tiles_m * tiles_n;
    r.split = t / per;
    t -= r.split * per;
    const int group = t / (raster * tiles_n);
    const int first = group * raster;
    const int height = min(raster, tiles_m - first);
    t -= first * tiles_n;
    r.n = t / height;
    r.m = first + t - r.n * height;
    return r;
}

// What a launch has to do for one product.
struct Shape { int M, tiles_m, tiles_n, num_kb, kb_per, sum_blocks, total; };

template <int EPI, bool SUMS>
__device__ __forceinline__ Shape shape_of(const XentGemmArgs &a) {
    Shape s;
    s.M = a.m_count ? min(a.M, *a.m_count) : a.M;
    const int K = a.k_count ? min(a.K, *a.k_count) : a.K;
    s.tiles_m = (s.M + 2 * BM - 1) / (2 * BM);
    s.tiles_n = (a.N + a.bn - 1) / a.bn;
    s.num_kb = (K + BK - 1) / BK;
    const int splits = a.most_splits > 1 ? xent_splits(s.tiles_m * s.tiles_n, a.split_kb ? a.split_kb : s.num_kb, a.segs, a.pairs, a.most_splits) : 1;
    s.kb_per = (s.num_kb + splits - 1) / splits;
    s.total = s.tiles_m * s.tiles_n * splits;
    // K blocks per accumulator
    s.sum_blocks = !SUMS ? max(1, s.kb_per) : a.segs > 1 ? kSumBlocks32 : EPI == XENT_EPI_STORE ? kSumBlocksStore : kSumBlocks16;
    return s;
}

// STORE may carry two products (dx and dW: neither waits for the other): tiles of the second follow those of the first.
template <int EPI, bool SUMS>
__global__ void __launch_bounds__(kThreads, 1)
xent_gemm_kernel(const __grid_constant__ CUtensorMap map_a0, const __grid_constant__ CUtensorMap map_b0,
                 const __grid_constant__ CUtensorMap map_a1, const __grid_constant__ CUtensorMap map_b1,
                 const __grid_constant__ CUtensorMap map_o0, const __grid_constant__ CUtensorMap map_o1,
                 const __grid_constant__ XentGemmArgs g0, const __grid_constant__ XentGemmArgs g1, const int stages,
                 const uint32_t stage_bytes, const uint32_t slab_bytes) {
    constexpr bool kStore = EPI == XENT_EPI_STORE, B_MN = kStore;
    pdl_trigger();
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *slabs = smem + (size_t)stages * stage_bytes;      // [epilogue warps][slab_bytes]
    Bars *bars = reinterpret_cast<Bars *>(slabs + kEpiWarps * slab_bytes);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int group = (int)cluster_id_x(), n_groups = (int)num_clusters_x();
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) {
            mbar_init(&bars->full[s], 1);
            mbar_init(&bars->empty[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars->acc_full[i], 1);
            mbar_init(&bars->acc_empty[i], kEpiWarps * 2);
        }
        if (EPI == XENT_EPI_ROW)
            for (int i = 0; i < 4; ++i) mbar_init(&bars->row_meet[i], 2);
        bars->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 0 && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a0) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b0) : "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                         smem_u32(&bars->tmem_base)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync_all();
    tcgen05_fence_after();
    pdl_wait();
    const uint32_t tmem_base = bars->tmem_base;
    volatile uint32_t *abort_flag = &bars->abort_flag;

    const Shape s0 = shape_of<EPI, SUMS>(g0), s1 = kStore ? shape_of<EPI, SUMS>(g1) : Shape{};
    const int total = s0.total + (kStore ? s1.total : 0);

    const uint32_t smem0 = smem_u32(smem), full0 = smem_u32(&bars->full[0]), empty0 = smem_u32(&bars->empty[0]);
    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer
        {
            const uint32_t lead_full0 = map_to_cta(full0, 0);     // the leader counts both CTAs' bytes
            int s = 0, armed = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int t = group; t < total && ok; t += n_groups) {
                const bool second = kStore && t >= s0.total;
                const XentGemmArgs &a = second ? g1 : g0;
                const Shape &sh = second ? s1 : s0;
                const CUtensorMap *map_a = second ? &map_a1 : &map_a0, *map_b = second ? &map_b1 : &map_b0;
                const bool A_MN = kStore && a.a_mn;
                const int BN = a.bn, BNL = BN / 2;
                const uint32_t tx = (kATile + (uint32_t)BNL * BK * 2) * 2;
                const Tile tl = tile_of(second ? t - s0.total : t, sh.tiles_m, sh.tiles_n, a.raster);
                const int arow = tl.m * (2 * BM) + (int)rank * BM + a.a_mn0;
                const int brow = tl.n * BN + (int)rank * BNL + a.b_mn0;
                const int kb0 = tl.split * sh.kb_per, kb1 = min(sh.num_kb, kb0 + sh.kb_per);
                const int segs = a.segs;
                for (int kc = kb0; kc < kb1 && ok; kc += sh.sum_blocks)
                for (int sg = 0; sg < segs && ok; ++sg) {
                    const int kend = min(kb1, kc + sh.sum_blocks);
                    // coordinates along the contiguous axis and across it, of this K block
                    int ax = a.a_part[sg] * a.a_pitch + (A_MN ? arow : kc * BK + a.a_k0), ay = A_MN ? kc * BK + a.a_k0 : arow;
                    int bx = a.b_part[sg] * a.b_pitch + (B_MN ? brow : kc * BK + a.b_k0), by = B_MN ? kc * BK + a.b_k0 : brow;
                    for (int kb = kc; kb < kend; ++kb) {
                        if (!pipe_wait(empty0 + 8u * s, phase ^ 1, abort_flag)) { ok = false; break; }
                        const uint32_t sa = smem0 + (uint32_t)s * stage_bytes, sb = sa + kATile, bar = lead_full0 + 8u * s;
                        const bool one = elect_one();
                        if (one && rank == 0)
                            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(full0 + 8u * s), "r"(tx) : "memory");
                        if (one) {
                            tma_load_2d<2>(sa, map_a, bar, ax, ay);
                            if (A_MN) tma_load_2d<2>(sa + 8192u, map_a, bar, ax + 64, ay);
                            tma_load_2d<2>(sb, map_b, bar, bx, by);
                            if (B_MN && BNL > 64) tma_load_2d<2>(sb + 8192u, map_b, bar, bx + 64, by);
                        }
                        __syncwarp();
                        if (A_MN) ay += BK;
                        else ax += BK;
                        if (B_MN) by += BK;
                        else bx += BK;
                        ++armed;
                        if (++s == stages) { s = 0; phase ^= 1; }
                    }
                }
            }
            if (!ok && lane == 0) {
                *abort_flag = 1;
                atomicOr(g0.status, 1);
                if (rank == 0) {
                    // copies in flight land before the CTA gives its shared memory back
                    int back = armed < stages ? armed : stages, ss = s;
                    uint32_t ph = phase;
                    for (int i = 0; i < back; ++i) {
                        if (--ss < 0) { ss = stages - 1; ph ^= 1; }
                        mbar_wait(&bars->full[ss], ph);
                    }
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer (the leader CTA)
        if (rank == 0) {
            // (the address field of a descriptor counts 16 bytes; all of shared memory fits it, so stages just add to it)
            const uint32_t acc_empty_l = smem_u32(&bars->acc_empty[0]);
            int s = 0, lt = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int t = group; t < total && ok; t += n_groups) {
                const bool second = kStore && t >= s0.total;
                const XentGemmArgs &a = second ? g1 : g0;
                const Shape &sh = second ? s1 : s0;
                const bool A_MN = kStore && a.a_mn;
                const uint32_t fmt = a.bf16 ? 1u : 0u;
                const uint32_t idesc = (1u << 4) | (fmt << 7) | (fmt << 10) | ((A_MN ? 1u : 0u) << 15) | ((B_MN ? 1u : 0u) << 16) |
                                       ((uint32_t)(a.bn >> 3) << 17) | ((uint32_t)((2 * BM) >> 4) << 24);
                const uint64_t desc_a0 = A_MN ? make_desc_mn(smem0) : make_desc(smem0);
                const uint64_t desc_b0 = B_MN ? make_desc_mn(smem0 + kATile) : make_desc(smem0 + kATile);
                const uint64_t a_step = A_MN ? 2048 >> 4 : 2;     // 16 of K: 16 rows of 128 bytes, or 32 bytes along a row
                const int segs = a.segs;
                const Tile tl = tile_of(second ? t - s0.total : t, sh.tiles_m, sh.tiles_n, a.raster);
                const int kb0 = tl.split * sh.kb_per, kb1 = min(sh.num_kb, kb0 + sh.kb_per);
                // (nothing to sum, kb1 <= kb0: the epilogue writes zeros)
                for (int kc = kb0; kc < kb1 && ok; kc += sh.sum_blocks) {
                    const int acc = lt & 1;
                    const uint32_t acc_phase = (lt >> 1) & 1;
                    ++lt;
                    if (!pipe_wait(acc_empty_l + 8u * acc, acc_phase ^ 1, abort_flag)) { ok = false; break; }
                    tcgen05_fence_after();
                    const uint32_t d = tmem_base + (uint32_t)(acc * 256);
                    const int steps = segs * (min(kb1, kc + sh.sum_blocks) - kc);
                    for (int i = 0; i < steps; ++i) {
                        if (!pipe_wait(full0 + 8u * s, phase, abort_flag)) { ok = false; break; }
                        tcgen05_fence_after();
                        const uint64_t at = (uint64_t)((uint32_t)s * (stage_bytes >> 4));
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < BK / 16; ++k)
                                mma_f16<2>(d, desc_a0 + at + (uint64_t)k * a_step,
                                           desc_b0 + at + (uint64_t)(B_MN ? k * (2048 >> 4) : k * 2), idesc, (i | k) ? 1u : 0u);
                            tcgen05_commit<2>(&bars->empty[s]);
                            if (i == steps - 1) tcgen05_commit<2>(&bars->acc_full[acc]);
                        }
                        __syncwarp();
                        if (++s == stages) { s = 0; phase ^= 1; }
                    }
                }
            }
            if (!ok && lane == 0) {
                *abort_flag = 1;
                atomicOr(g0.status, 1);
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const uint32_t acc_full0 = smem_u32(&bars->acc_full[0]);
        const uint32_t acc_empty0 = map_to_cta(smem_u32(&bars->acc_empty[0]), 0);
        uint8_t *slab = slabs + (warp - 2) * slab_bytes;
        int turn = 0;                                          // which half of the slab the next 16-bit block takes
        uint32_t met = 0;                                      // phase of the meetings with the quarter's other warp
        bool ok = true;
        int lt = 0;
        for (int t = group; t < total && ok; t += n_groups) {
            const bool second = kStore && t >= s0.total;
            const XentGemmArgs &a = second ? g1 : g0;
            const Shape &sh = second ? s1 : s0;
            const CUtensorMap *map_o = second ? &map_o1 : &map_o0;
            const int BN = a.bn, M = sh.M, sum_blocks = sh.sum_blocks;
            const int chunks = BN / 32;
            const int c_begin = half ? (chunks + 1) / 2 : 0, c_end = half ? chunks : (chunks + 1) / 2;
            float scale = a.out_scale;
            if (kStore && a.count) scale /= (float)max(1, *a.count);
            const Tile tl = tile_of(second ? t - s0.total : t, sh.tiles_m, sh.tiles_n, a.raster);
            const int kb0 = tl.split * sh.kb_per, kb1 = min(sh.num_kb, kb0 + sh.kb_per);
            const bool empty = kb1 <= kb0;
            int acc = lt & 1;
            const int row0 = tl.m * (2 * BM) + (int)rank * BM + quarter * 32;
            const int row = row0 + lane;
            const bool row_ok = row < M;
            float sum[SUMS ? 4 : 1][32];
            if (SUMS) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 32; ++e) sum[SUMS ? i : 0][e] = 0.0f;
                for (int kc = kb0; kc < kb1; kc += sum_blocks) {
                    acc = lt & 1;
                    if (!pipe_wait(acc_full0 + 8u * acc, (lt >> 1) & 1, abort_flag)) { ok = false; break; }
                    ++lt;
                    tcgen05_fence_after();
                    const uint32_t t_addr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(acc * 256 + c_begin * 32);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (c_begin + i < c_end) {
#pragma unroll
                            for (int h = 0; h < 32; h += 16) {
                                uint32_t v[16];
                                __syncwarp();
                                tmem_ld16(t_addr + (uint32_t)(i * 32 + h), v);
                                tmem_ld_wait();
#pragma unroll
                                for (int e = 0; e < 16; ++e) sum[SUMS ? i : 0][h + e] += __uint_as_float(v[e]);
                            }
                        }
                    }
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(acc_empty0 + (uint32_t)(acc * sizeof(uint64_t)));
                }
                if (!ok) break;
            } else if (!empty) {
                if (!pipe_wait(acc_full0 + 8u * acc, (lt >> 1) & 1, abort_flag)) { ok = false; break; }
                ++lt;
                tcgen05_fence_after();
            }
            const uint32_t t_addr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(acc * 256);

            float run_m = -INFINITY, run_s = 0.0f;           // LSE
            const int tgt = (EPI != XENT_EPI_STORE && row_ok) ? a.target[row] - a.class0 : -1;
            float2 stat = (EPI == XENT_EPI_PROB && row_ok) ? a.stat[row] : make_float2(0.0f, INFINITY);
            long long out_row = row;
            if (EPI == XENT_EPI_STORE && a.row_map && row_ok) out_row = a.row_map[row];

            if (kStore && lane == 0) bulk_wait_read<0>();    // (the tile before may have used the slab in another way)
            if (EPI == XENT_EPI_ROW) {
                // logits in place of the sums, and this half's maximum, sum and target
                float top = -INFINITY, zt = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (c_begin + i >= c_end) break;
                    const int col0 = tl.n * BN + (c_begin + i) * 32;
                    float(&z)[32] = sum[SUMS ? i : 0];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        if (a.bias) z[e] += __ldg(a.bias + col0 + e);
                        if (col0 + e >= a.N) z[e] = -INFINITY;
                        top = fmaxf(top, z[e]);
                        select_if(zt, z[e], tgt - col0, e);
                    }
                }
                const float m_half = top * kLog2e, sub_half = top == -INFINITY ? 0.0f : m_half;
                float s_half = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (c_begin + i >= c_end) break;
#pragma unroll
                    for (int e = 0; e < 32; ++e) s_half += ex2(fmaf(sum[SUMS ? i : 0][e], kLog2e, -sub_half));
                }
                float4 *half_row = reinterpret_cast<float4 *>(bars + 1) + quarter * 32 + lane;    // [half][row]: maximum, sum, target
                half_row[half * BM] = make_float4(m_half, s_half, zt, 0.0f);
                if (!pair_meet(&bars->row_meet[quarter], met, lane, abort_flag)) { ok = false; break; }
                const float4 h0 = half_row[0], h1 = half_row[BM];
                if (!pair_meet(&bars->row_meet[quarter], met, lane, abort_flag)) { ok = false; break; }      // read before the next tile's
                const float m = fmaxf(h0.x, h1.x), sub = m == -INFINITY ? 0.0f : m;
                const float s = h0.y * ex2(h0.x - sub) + h1.y * ex2(h1.x - sub), l2s = log2f(s);
                double nll = 0.0;
                if (row_ok) {
                    // no class left in the row: every probability is zero
                    if (s != 0.0f) stat = make_float2(sub, l2s);
                    if (half == 0) {
                        const float t_logit = h0.z + h1.z;
                        const float l = t_logit == -INFINITY ? INFINITY : kLn2 * (fmaf(-t_logit, kLog2e, sub) + l2s);
                        if (a.row_losses) CERT_ST(a.row_losses[a.row_of[row]], l);
                        nll = (double)l;
                    }
                }
                if (half == 0) {
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) nll += __shfl_xor_sync(0xffffffffu, nll, o);
                    if (lane == 0 && row0 < M) CERT_ST(a.loss_sum[row0 >> 5], nll);
                }
            }
#pragma unroll(SUMS ? 4 : 1)
            for (int i = 0; i < 4; ++i) {
                const int c = c_begin + i;
                if (c >= c_end || (EPI == XENT_EPI_ROW && !a.prob)) break;      // (the loss alone)
                const int col0 = tl.n * BN + c * 32;
                // (uniform over the warp; probabilities are written to the tile's end or the pitch, zeros behind the last class)
                if (col0 >= ((EPI == XENT_EPI_PROB || EPI == XENT_EPI_ROW) ? a.prob_pitch : a.N)) break;
                uint32_t v[32];
                if (SUMS) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(sum[SUMS ? i : 0][e]);
                } else if (empty) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = 0u;
                } else {
                    __syncwarp();
                    tmem_ld32(t_addr + (uint32_t)(c * 32), v);
                    tmem_ld_wait();
                }
                if (EPI == XENT_EPI_LSE || EPI == XENT_EPI_PROB) {
                    if (a.bias && xent_reads_bias(col0, a.N)) {
#pragma unroll
                        for (int g = 0; g < 8; ++g) {
                            const float4 b4 = __ldg(reinterpret_cast<const float4 *>(a.bias + col0) + g);
                            v[g * 4] = __float_as_uint(__uint_as_float(v[g * 4]) + b4.x);
                            v[g * 4 + 1] = __float_as_uint(__uint_as_float(v[g * 4 + 1]) + b4.y);
                            v[g * 4 + 2] = __float_as_uint(__uint_as_float(v[g * 4 + 2]) + b4.z);
                            v[g * 4 + 3] = __float_as_uint(__uint_as_float(v[g * 4 + 3]) + b4.w);
                        }
                    }
                    if (col0 + 32 > a.N) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (col0 + e >= a.N) v[e] = 0xff800000u;     // -infinity: no such class
                    }
                }
                if (EPI == XENT_EPI_LSE) {
                    float top = __uint_as_float(v[0]);
#pragma unroll
                    for (int e = 1; e < 32; ++e) top = fmaxf(top, __uint_as_float(v[e]));
                    const float m_new = fmaxf(run_m, top * kLog2e);
                    // with nothing but -infinity so far the differences below would be NaN
                    const float sub = m_new == -INFINITY ? 0.0f : m_new;
                    float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f, s3 = 0.0f;
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        s0 += ex2(fmaf(__uint_as_float(v[e]), kLog2e, -sub));
                        s1 += ex2(fmaf(__uint_as_float(v[e + 1]), kLog2e, -sub));
                        s2 += ex2(fmaf(__uint_as_float(v[e + 2]), kLog2e, -sub));
                        s3 += ex2(fmaf(__uint_as_float(v[e + 3]), kLog2e, -sub));
                    }
                    run_s = fmaf(run_s, ex2(run_m - sub), (s0 + s1) + (s2 + s3));
                    run_m = m_new;
                    if (tgt >= col0 && tgt < col0 + 32) {
                        float zt = 0.0f;
#pragma unroll
                        for (int e = 0; e < 32; ++e) select_if(zt, __uint_as_float(v[e]), tgt - col0, e);
                        CERT_ST(a.target_logit[row], zt);
                    }
                } else if (EPI == XENT_EPI_PROB || EPI == XENT_EPI_ROW) {
                    // the same maximum as in the sum, so its rounding cancels; infinity for a row that does not count
                    const float log2_sum = stat.y - a.prob_log2_scale;
                    const float one = ex2(a.prob_log2_scale);
                    float p[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        p[e] = ex2(fmaf(__uint_as_float(v[e]), kLog2e, -stat.x) - log2_sum);
                    }
                    if (__any_sync(0xffffffffu, tgt >= col0 && tgt < col0 + 32)) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) minus_if(p[e], one, tgt - col0, e);
                    }
                    if (row0 + 32 > M) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) p[e] = row_ok ? p[e] : 0.0f;     // also where stale operands gave NaN
                    }
                    if (a.prob_parts == 1) {
                        // two blocks in turn: the one before may still be read
                        if (lane == 0) bulk_wait_read<1>();
                        __syncwarp();
                        uint8_t *block = slab + turn * 2048;
                        turn ^= 1;
                        uint32_t w[16];
#pragma unroll
                        for (int q = 0; q < 16; ++q) w[q] = pack2(p[2 * q], p[2 * q + 1], a.bf16);
                        block16(block, lane, w);
                        send_block(map_o, block, col0, row0, lane, false);
                    } else {
                        if (lane == 0) bulk_wait_read<0>();
                        __syncwarp();
                        float r[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) r[e] = p[e];
#pragma unroll
                        for (int part = 0; part < 3; ++part) {
                            uint32_t w[16];
#pragma unroll
                            for (int q = 0; q < 16; ++q) {
                                w[q] = pack2(r[2 * q], r[2 * q + 1], true);
                                r[2 * q] -= __uint_as_float(w[q] << 16);
                                r[2 * q + 1] -= __uint_as_float(w[q] & 0xffff0000u);
                            }
                            block16(slab + part * 2048, lane, w);
                        }
                        fence_async_smem();
                        __syncwarp();
                        if (lane == 0) {
#pragma unroll
                            for (int part = 0; part < 3; ++part)
                                tma_store_2d(map_o, smem_u32(slab + part * 2048), part * a.prob_pitch + col0, row0);
                            tma_store_commit();
                        }
                    }
                    if (a.colsum && row0 < a.rows_pad) {
                        // sums over the warp's 32 rows by recursive halving: lane L ends with column L, in a fixed order
#pragma unroll
                        for (int dd = 16; dd >= 1; dd >>= 1) {
                            const bool up = (lane & dd) != 0;
#pragma unroll
                            for (int j = 0; j < dd; ++j) {
                                const float send = up ? p[j] : p[j + dd];
                                const float keep = up ? p[j + dd] : p[j];
                                p[j] = keep + __shfl_xor_sync(0xffffffffu, send, dd);
                            }
                        }
                        CERT_ST(a.colsum[(size_t)(row0 >> 5) * a.colsum_ld + col0 + lane], p[0]);
                    }
                } else if (a.tma_out && row0 + 32 <= M) {
                    if (a.out_type == CERT_TYPE_F32) {
                        if (lane == 0) bulk_wait_read<0>();
                        __syncwarp();
                        float f[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) f[e] = __uint_as_float(v[e]) * scale;
                        // 128 bytes per row, the 16-byte pieces exchanged as TMA's 128-byte swizzle has them
#pragma unroll
                        for (int g = 0; g < 8; ++g)
                            *reinterpret_cast<float4 *>(slab + lane * 128 + ((g ^ (lane & 7)) << 4)) = make_float4(f[g * 4], f[g * 4 + 1], f[g * 4 + 2], f[g * 4 + 3]);
                        send_block(map_o, slab, col0, tl.split * a.split_rows + row0, lane, a.add != 0);
                    } else {
                        if (lane == 0) bulk_wait_read<1>();
                        __syncwarp();
                        uint8_t *block = slab + turn * 2048;
                        turn ^= 1;
                        uint32_t w[16];
#pragma unroll
                        for (int q = 0; q < 16; ++q)
                            w[q] = pack2(__uint_as_float(v[q * 2]) * scale, __uint_as_float(v[q * 2 + 1]) * scale, a.out_type == CERT_TYPE_BF16);
                        block16(block, lane, w);
                        send_block(map_o, block, col0, row0, lane, false);
                    }
                } else if (row0 < M) {
                    // rows that start anywhere or go to places of their own, and the last rows: the warp's block is turned in
                    // shared memory, so that a store is 32 neighbouring elements of a row instead of one of each row
                    float *block = reinterpret_cast<float *>(slab);
                    if (lane == 0) bulk_wait_read<0>();
                    __syncwarp();
#pragma unroll
                    for (int e = 0; e < 32; ++e) block[lane * 32 + (e ^ lane)] = __uint_as_float(v[e]) * scale;
                    __syncwarp();
                    const int last = min(32, M - row0);
                    const bool col_ok = col0 + lane < a.N;
                    if (a.rows_16 && !a.add && col0 + 32 <= a.N) {
                        // 16 bytes per lane: four lanes a row (16 bits), or eight
                        const bool f32 = a.out_type == CERT_TYPE_F32;
                        const int per = f32 ? 8 : 4, c = lane & (per - 1);
                        for (int r0 = 0; r0 < last; r0 += 32 / per) {
                            const int r = r0 + lane / per;
                            const long long to = __shfl_sync(0xffffffffu, out_row, r);
                            float f[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (!f32 || e < 4) f[e] = block[r * 32 + ((c * (32 / per) + e) ^ r)];
                            if (r >= last) continue;
                            char *o = reinterpret_cast<char *>(a.out) +
                                      ((f32 ? (size_t)tl.split * a.out_split_stride : 0) + (size_t)to * a.out_ld + col0 + c * (32 / per)) * (f32 ? 4 : 2);
                            const bool bf = a.out_type == CERT_TYPE_BF16;
                            if (f32) CERT_ST(*reinterpret_cast<float4 *>(o), make_float4(f[0], f[1], f[2], f[3]));
                            else CERT_ST(*reinterpret_cast<uint4 *>(o), make_uint4(pack2(f[0], f[1], bf), pack2(f[2], f[3], bf), pack2(f[4], f[5], bf), pack2(f[6], f[7], bf)));
                        }
                        __syncwarp();
                        continue;
                    }
                    for (int r = 0; r < last; ++r) {
                        const long long to = __shfl_sync(0xffffffffu, out_row, r);
                        const float f = block[r * 32 + (lane ^ r)];
                        if (!col_ok) continue;
                        if (a.out_type == CERT_TYPE_F32) {
                            float *o = reinterpret_cast<float *>(a.out) + (size_t)tl.split * a.out_split_stride + (size_t)to * a.out_ld + col0 + lane;
                            CERT_ST(*o, a.add ? f + *o : f);
                        } else {
                            store_from_float(a.out, to * a.out_ld + col0 + lane, a.out_type, f);
                        }
                    }
                    __syncwarp();
                }
            }
            if (EPI == XENT_EPI_LSE && row_ok)
                CERT_ST(a.partial[(size_t)(a.slot0 + tl.n * 2 + half) * a.rows_pad + row], make_float2(run_m, run_s));
            if (!SUMS && !empty) {
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(acc_empty0 + (uint32_t)(acc * sizeof(uint64_t)));
            }
        }
        if (EPI != XENT_EPI_LSE && lane == 0) tma_store_wait_all();
        if (!ok) {
            *abort_flag = 1;
            if (lane == 0) atomicOr(g0.status, 1);
        }
    }
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync_all();
    if (warp == 1) {
        tcgen05_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    }
}

typedef CUresult (*EncodeTiledXent)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                    const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                    CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
std::atomic<EncodeTiledXent> g_encode{nullptr};

template <int EPI, bool SUMS>
void launch_one(int pairs, const XentMap &a0, const XentMap &b0, const XentMap &o0, const XentGemmArgs &g0, const XentMap &a1,
                const XentMap &b1, const XentMap &o1, const XentGemmArgs &g1, cudaStream_t st) {
    constexpr bool kStore = EPI == XENT_EPI_STORE;
    const int bn = kStore && g1.N && g1.bn > g0.bn ? g1.bn : g0.bn;
    const int stage_bytes = kATile + bn / 2 * BK * 2;
    const int slab = EPI == XENT_EPI_LSE ? 0 : !kStore && g0.prob_parts > 1 ? 3 * 2048 : 4096;
    const int extra = (int)sizeof(Bars) + (EPI == XENT_EPI_ROW ? 2 * BM * (int)sizeof(float4) : 0) + kEpiWarps * slab + 1024;
    int stages = (kTcSmemMax - extra) / stage_bytes;
    if (stages > kMaxStages) stages = kMaxStages;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(pairs * 2), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = (size_t)stages * stage_bytes + extra;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled() ? 2 : 1;
    auto tensor_map = [](const XentMap &m) -> const CUtensorMap & { return reinterpret_cast<const CUtensorMap &>(m); };
    cudaLaunchKernelEx(&cfg, xent_gemm_kernel<EPI, SUMS>, tensor_map(a0), tensor_map(b0), tensor_map(a1), tensor_map(b1),
                       tensor_map(o0), tensor_map(o1), g0, g1, stages, (uint32_t)stage_bytes, (uint32_t)slab);
}

template <int EPI, bool SUMS>
bool allow_smem() {
    return cudaFuncSetAttribute(xent_gemm_kernel<EPI, SUMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kTcSmemMax) == cudaSuccess;
}

}  // namespace

bool xent_gemm_prepare() {
    if (!g_encode.load()) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres) != cudaSuccess ||
            qres != cudaDriverEntryPointSuccess || !fn) {
            cudaGetLastError();
            return false;
        }
        g_encode = reinterpret_cast<EncodeTiledXent>(fn);
    }
    if (!allow_smem<XENT_EPI_LSE, true>() || !allow_smem<XENT_EPI_ROW, true>() || !allow_smem<XENT_EPI_PROB, false>() ||
        !allow_smem<XENT_EPI_PROB, true>() || !allow_smem<XENT_EPI_STORE, false>() || !allow_smem<XENT_EPI_STORE, true>()) {
        cudaGetLastError();
        return false;
    }
    return true;
}

bool xent_make_map(XentMap *m, const void *base, bool bf16, long long inner, long long outer, long long pitch_elems,
                   int box_inner, int box_outer) {
    const EncodeTiledXent encode = g_encode.load();
    if (!encode) return false;
    cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer};
    cuuint64_t strides[1] = {(cuuint64_t)pitch_elems * 2};
    cuuint32_t box[2] = {(cuuint32_t)box_inner, (cuuint32_t)box_outer};
    cuuint32_t estr[2] = {1u, 1u};
    return encode(reinterpret_cast<CUtensorMap *>(m), bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                    2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool xent_make_out_map(XentMap *m, const void *base, int type, long long inner, long long outer, long long pitch_elems) {
    const int es = type_size(type);
    const EncodeTiledXent encode = g_encode.load();
    if (!encode || !aligned(base, 16) || (pitch_elems * es) % 16 != 0 || pitch_elems * es >= (1LL << 40)) return false;
    cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer};
    cuuint64_t strides[1] = {(cuuint64_t)(pitch_elems * es)};
    cuuint32_t box[2] = {32, 32};
    cuuint32_t estr[2] = {1u, 1u};
    const CUtensorMapDataType t = type == CERT_TYPE_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                : type == CERT_TYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    return encode(reinterpret_cast<CUtensorMap *>(m), t, 2, const_cast<void *>(base), dims, strides, box, estr,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, type == CERT_TYPE_F32 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                    CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

void launch_xent_gemm(int epi, int pairs, const XentMap &a, const XentMap &b, const XentMap &out, const XentGemmArgs &args, cudaStream_t st) {
    // sums in registers for the loss, for everything in float32, and for long sums
    if (epi == XENT_EPI_LSE) launch_one<XENT_EPI_LSE, true>(pairs, a, b, a, args, a, b, a, args, st);
    else if (epi == XENT_EPI_ROW) launch_one<XENT_EPI_ROW, true>(pairs, a, b, out, args, a, b, out, args, st);
    else if (args.segs > 1 || args.K > (args.bf16 ? kProbTermsBf16 : kProbTermsHalf)) launch_one<XENT_EPI_PROB, true>(pairs, a, b, out, args, a, b, out, args, st);
    else launch_one<XENT_EPI_PROB, false>(pairs, a, b, out, args, a, b, out, args, st);
}

void launch_xent_store(int pairs, const XentProduct &p, const XentProduct &q, cudaStream_t st) {
    const int K = q.args.N && q.args.K > p.args.K ? q.args.K : p.args.K;       // (the device may cut it into ranges, or not)
    if (p.args.segs > 1 || K > (p.args.bf16 ? kStoreTermsBf16 : kStoreTermsHalf)) launch_one<XENT_EPI_STORE, true>(pairs, p.a, p.b, p.out, p.args, q.a, q.b, q.out, q.args, st);
    else launch_one<XENT_EPI_STORE, false>(pairs, p.a, p.b, p.out, p.args, q.a, q.b, q.out, q.args, st);
}

}  // namespace cert
