// Layers with 4-bit weights: y = x W^T + b for a few rows of x, W[n][k] = scale[n][g] (code[n][k] - zero[n][g]).
//
// Bound by reading the codes (half a byte per weight) and, close behind, by the integer units that unpack them, so everything
// else is kept off both.  The weights lie in records of 16 rows x 256 of K, scales and codes together, in the order in which
// a warp's lanes need them, 16 bytes of codes per lane for every 64 of K.  One block per multiprocessor holds x (or a panel of
// K of it) in shared memory and streams its rows' records, 8 to a stage, one for each of half its 16 warps; a 17th warp
// copies whole stages with cp.async.bulk as far ahead as shared memory goes, and three more add up the warps' sums, so that
// the 16 never wait for one another.  The products run on mma.sync in float16, weights as the 16-row operand, x as its
// 8 columns.  A code becomes a float16 with one AND-OR, 1024 + code, or 1024 + 16 code four bits higher (bfloat16's mantissa
// has no room for the second form), and one multiply-add that takes the constant and the zero point off; 1024 plus an integer in
// the last bits is the published way to do this (Kim, Henry, Fahim and Awadalla 2022, Who Says Elephants Can't Run).
// x goes in as float16 times a power of two per row, which puts the row's largest value below 2^15: a bfloat16's eight bits stay
// exact down to 2^-29 of the largest and are off by at most 2^-40 of it below; a float32 takes two columns, hi and lo, 22 bits.
// A group's sum is multiplied by its scale in fp32; the warps' sums are added in a fixed order.
// Measured: 28672 x 8192 in groups of 128, bfloat16, one row of x: 28.5 to 29.7 us over three cards, 121 MB of records at 4.1-4.2 TB/s;
// the copies alone, without the products, 21 us.  11009 x 4096 in groups of 64 with zero points, float16, 13 rows: 14.2 us (floor of the bytes 3.8),
// the reads of x from shared memory, 16 columns for each record, and the five rounds of items being what is left.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <new>
#include <type_traits>

#include "ops_common.cuh"
#include "tc_ptx.cuh"

struct cert_int4 {
    cert::OpBuffers mem;
    int device = 0, sms = 1;
    int N = 0, K = 0, group = 0, type = 0;
    int row_tiles = 0, k_tiles = 0, groups = 0, chunks = 0;
    bool zeros = false;
    int record = 0;                      // bytes of a record: 16 rows x 256 of K
    unsigned char *records = nullptr;    // [row_tiles][chunks]: scales, zero points, codes
    int *status = nullptr;
};

namespace cert {
namespace {

constexpr int kWarps = 16;
constexpr int kChunk = 256;              // of K, per record
constexpr int kPerStage = 8;               // records per copy and stage
constexpr int kMaxStages = 16;
constexpr int kSmemBlock = 224 * 1024;

// Where lane (r, t) of a tile finds weight q (0 .. 31) of its 16 bytes: word s = q / 8 of step s; the nibble pair (i, i + 4)
// is register i of the 16-row operand: rows r and r + 8 in turn, two of K each.
__device__ __forceinline__ void place(int lane, int q, int &row, int &k) {
    const int s = q >> 3, nib = q & 7, i = nib & 3, second = nib >> 2;
    const int t = lane & 3;
    row = (lane >> 2) + ((i & 1) ? 8 : 0);
    k = 32 * (s >> 1) + 8 * t + 4 * (s & 1) + ((i & 2) ? 2 : 0) + second;
}

// A record holds what a warp needs for 16 rows x 256 of K, in the order of one copy: the groups' scales, rows r and r + 8
// next to each other ([group][8][2]), their zero points likewise, then the codes of four pieces of 64.  Scales behind the
// last group are zero.
struct RecordShape {
    int K, N, k_tiles, groups, chunks, group, type, has_zeros, record;
    __host__ __device__ int per_chunk() const { return kChunk / group; }
    __host__ __device__ int zero_at() const { return per_chunk() * 16 * (type == CERT_TYPE_F32 ? 4 : 2); }
    __host__ __device__ int code_at() const { return zero_at() + (has_zeros ? per_chunk() * 16 : 0); }
};

__global__ void int4_repack_kernel(const unsigned char *__restrict__ codes, const RecordShape g, unsigned char *out, long long total) {
    const int row_bytes = (g.K + 1) / 2;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (long long)gridDim.x * blockDim.x) {
        const int lane = (int)(i & 31), p = (int)(i >> 5) & 3;
        const long long rec = i >> 7;
        const int k0 = (int)(rec % g.chunks) * kChunk + p * 64;
        const long long n0 = rec / g.chunks * 16;
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int q = 0; q < 32; ++q) {
            int row, k;
            place(lane, q, row, k);
            const long long n = n0 + row;
            k += k0;
            uint32_t c = 8;
            if (n < g.N && k < g.K) {
                const unsigned char b = codes[n * row_bytes + (k >> 1)];
                c = (k & 1) ? b >> 4 : b & 15;
            }
            w[q >> 3] |= c << (4 * (q & 7));
        }
        CERT_ST(*reinterpret_cast<uint4 *>(out + rec * g.record + g.code_at() + p * 512 + lane * 16), make_uint4(w[0], w[1], w[2], w[3]));
    }
}

template <typename S>
__global__ void int4_repack_groups_kernel(const S *__restrict__ scales, const unsigned char *__restrict__ zeros, const RecordShape g,
                                          unsigned char *out, long long total) {
    const int per = g.per_chunk() * 16;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (long long)gridDim.x * blockDim.x) {
        const long long rec = i / per;
        const int at = (int)(i - rec * per), j = at & 15;
        const int gr = (int)(rec % g.chunks) * g.per_chunk() + (at >> 4);
        const long long n = rec / g.chunks * 16 + (j >> 1) + (j & 1) * 8;
        const bool in = n < g.N && gr < g.groups;
        S v;
        memset(&v, 0, sizeof(S));
        if (in) v = scales[n * g.groups + gr];
        CERT_ST(reinterpret_cast<S *>(out + rec * g.record)[at], v);
        if (zeros) CERT_ST(out[rec * g.record + g.zero_at() + at], (unsigned char)(in ? zeros[n * g.groups + gr] & 15 : 8));
    }
}

__global__ void int4_dequantize_kernel(const unsigned char *__restrict__ records, const RecordShape g, float *out, long long total) {
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (long long)gridDim.x * blockDim.x) {
        const int lane = (int)(i & 31), p = (int)(i >> 5) & 3;
        const long long rec = i >> 7;
        const unsigned char *r = records + rec * g.record;
        const uint4 u = *reinterpret_cast<const uint4 *>(r + g.code_at() + p * 512 + lane * 16);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int q = 0; q < 32; ++q) {
            int row, k;
            place(lane, q, row, k);
            const long long n = rec / g.chunks * 16 + row;
            const int in_chunk = p * 64 + k;
            k = (int)(rec % g.chunks) * kChunk + in_chunk;
            if (n >= g.N || k >= g.K) continue;
            const int at = in_chunk / g.group * 16 + (row & 7) * 2 + (row >> 3);
            const float z = g.has_zeros ? (float)r[g.zero_at() + at] : 8.0f;
            const float c = (float)((w[q >> 3] >> (4 * (q & 7))) & 15);
            CERT_ST(out[n * g.K + k], (c - z) * load_as_float(r, at, g.type));
        }
    }
}

// One warp per group of a row.
template <typename T>
__global__ void __launch_bounds__(256)
int4_quantize_kernel(const T *__restrict__ w, long long ldw, int N, int K, int group, int groups, unsigned char *codes, T *scales,
                     unsigned char *zeros) {
    const int lane = threadIdx.x & 31;
    const long long id = ((long long)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
    if (id >= (long long)N * groups) return;
    const long long n = id / groups;
    const int g = (int)(id - n * groups);
    const int k0 = g * group, k1 = min(K, k0 + group);
    float hi = 0.0f, lo = 0.0f;
    bool finite = true;
    for (int k = k0 + lane; k < k1; k += 32) {
        const float v = to_float(w[n * ldw + k]);
        hi = fmaxf(hi, v);
        lo = fminf(lo, v);
        finite = finite && fabsf(v) < INFINITY;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    }
    // no code stands for a NaN or an infinity: the scale does, so that the group's weights do not come back as ordinary numbers
    finite = __all_sync(0xffffffffu, finite);
    const T st = from_float<T>(!finite ? NAN : zeros ? (hi - lo) / 15.0f : fmaxf(hi, -lo) / 7.0f);
    const float s = to_float(st);
    const bool usable = s > 0.0f;
    const float z = zeros ? (usable ? fminf(fmaxf(rintf(-lo / s), 0.0f), 15.0f) : 0.0f) : 8.0f;
    const int row_bytes = (K + 1) / 2;
    for (int k = k0 + 2 * lane; k < k1; k += 64) {
        unsigned byte = 0;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float c = z;
            if (usable && k + e < k1) c = fminf(fmaxf(rintf(to_float(w[n * ldw + k + e]) / s) + z, 0.0f), 15.0f);
            byte |= (unsigned)c << (4 * e);
        }
        CERT_ST(codes[n * row_bytes + (k >> 1)], (unsigned char)byte);
    }
    if (lane == 0) {
        CERT_ST(scales[id], st);
        if (zeros) CERT_ST(zeros[id], (unsigned char)z);
    }
}

// ---------------------------------------------------------------- the product

// d = a b, or d += a b: the first product of a group takes a zero that needs no register.
template <bool FIRST>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    const float c0 = FIRST ? 0.0f : d[0], c1 = FIRST ? 0.0f : d[1], c2 = FIRST ? 0.0f : d[2], c3 = FIRST ? 0.0f : d[3];
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}

// (a & b) | c in one instruction (with two constants among them the compiler takes two)
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
// A constant the compiler keeps in a register.
__device__ __forceinline__ uint32_t in_register(uint32_t v) {
    uint32_t r;
    asm volatile("mov.b32 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

__device__ __forceinline__ uint32_t fma2_half(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}

__device__ __forceinline__ void mbar_arrive(uint64_t *bar, uint32_t count) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}
// Buffers for the warps' sums, 10 KB or 20 KB each.
__host__ __device__ constexpr int sums_bufs(int nt) { return nt == 1 ? 4 : 2; }

__device__ __forceinline__ void bulk_copy(void *dst, const void *src, uint32_t bytes, uint64_t *bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}

// A block takes consecutive row tiles (items) and numbers their records one after the other, f = item * chunks + chunk; stage s
// holds records 8 s .. 8 s + 7, and record f belongs to warp f mod 16.  That spreads any number of chunks evenly, and
// a stage is one or two contiguous copies.  A warp keeps its sums over the records of an item and leaves them in one of a
// few buffers in shared memory with the last; the adding warps take an item when all of its warps have.
struct Int4Args {
    const unsigned char *records;
    const void *x, *bias;
    void *y;
    long long ldx, ldy;
    int rows, rows_pass, relu, vec;                  // rows of x, and how many of them a block takes
    int N, K, row_tiles, chunks;
    int panel_chunks, panels;                        // chunks of K whose x is in shared memory at a time
    int x_pitch;                                     // bytes from one column of x to the next
    int stages;
    int red_off, x_off, out_off;                     // in shared memory
    int *status;
};

// The power of two for a row whose largest value has these bits: it ends up in [2^14, 2^15); and its inverse.
__device__ __forceinline__ float scale_of(uint32_t top) { return __uint_as_float(min(268u - (top >> 23), 253u) << 23); }
__device__ __forceinline__ float unscale_of(uint32_t top) { return __uint_as_float((254u - min(268u - (top >> 23), 253u)) << 23); }

// Eight elements of a row from column k on, zero behind K.
__device__ __forceinline__ void load8(const uint16_t *p, int k, int K, int vec, uint32_t (&w)[4]) {
    if (vec && k + 8 <= K) {
        const uint4 u = __ldg(reinterpret_cast<const uint4 *>(p + k));
        w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] = (k + 2 * e < K ? (uint32_t)p[k + 2 * e] : 0u) | (k + 2 * e + 1 < K ? (uint32_t)p[k + 2 * e + 1] << 16 : 0u);
    }
}
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, int k, int K, int vec, float (&v)[8]) {
    uint32_t w[4];
    load8(reinterpret_cast<const uint16_t *>(p), k, K, vec, w);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(w[e] << 16);
        v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const float *p, int k, int K, int vec, float (&v)[8]) {
    if (vec && k + 8 <= K) {
        const float4 a = __ldg(reinterpret_cast<const float4 *>(p + k)), b = __ldg(reinterpret_cast<const float4 *>(p + k) + 1);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = k + e < K ? p[k + e] : 0.0f;
    }
}

constexpr int kAddWarps = 3;
constexpr int kThreads = (kWarps + 1 + kAddWarps) * 32;

// The adding warps' counts of finished items.  The buffer of an item is free once all of them are done with the item kBufs
// before it.  Counts and not a barrier's phases: with K shorter than the warps' 16 chunks a warp skips items, by more than a
// phase's parity can tell apart.
__device__ __forceinline__ void count_release(uint32_t *count, uint32_t v) {
    asm volatile("st.release.cta.shared::cta.u32 [%0], %1;" ::"r"(smem_u32(count)), "r"(v) : "memory");
}
__device__ __forceinline__ bool counts_reach(const uint32_t *counts, int least, int lane) {
    const uint32_t at = smem_u32(counts + (lane < kAddWarps ? lane : 0));
    const long long t0 = clock64();
    for (;;) {
        uint32_t v;
        asm volatile("ld.acquire.cta.shared::cta.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
        if (__all_sync(0xffffffffu, (int)v >= least)) break;
        if (__any_sync(0xffffffffu, (unsigned long long)(clock64() - t0) > kWaitCycles)) return false;
    }
    __syncwarp();
    return true;
}

__device__ __forceinline__ void consumers_meet() { asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory"); }

// NT: column tiles (8 columns each) of the x operand; SHIFT: log2 of the group.
// The codes are made exact, code - zero, before the product.  Left in it with their constant, which a group's sum of x can take
// off afterwards, they fill the accumulator with up to 1024 times x, and for x of one sign (behind a ReLU) its truncation errors
// add up: float16, K = 4096, outputs off by 2.5e-4 (groups of 64) to 8.0e-4 (256) of their root mean square, where rounding them
// alone is 2.1e-4, and so it is now.  28672 x 8192, one row: 29.1 us against 27.8; 11009 x 4096, 13 rows, which needs no
// sums of x any more: 14.8 against 16.1.
template <typename T, int NT, bool ZEROS, int SHIFT>
__global__ void __launch_bounds__(kThreads, 1)
int4_matvec_kernel(const __grid_constant__ Int4Args a) {
    constexpr bool kF32 = std::is_same<T, float>::value;
    constexpr bool kScaled = !std::is_same<T, __half>::value;         // x takes a power of two per row
    constexpr uint32_t kMagic = 0x64006400u;                          // 1024, whose last ten bits are ones
    constexpr int GC = kChunk >> SHIFT;                               // groups of a chunk
    constexpr int kZeroAt = GC * 16 * (kF32 ? 4 : 2), kCodeAt = kZeroAt + (ZEROS ? GC * 16 : 0), kRecord = kCodeAt + 2048;
    constexpr int GSTEPS = (1 << SHIFT) / 16;                         // products per group
    constexpr int COLS = 8 * NT;
    constexpr int kCol = 20, kRed = kCol * COLS;                      // sums of a warp: [column][16 rows], 20 apart for the banks
    constexpr int kBufs = sums_bufs(NT);
    using S2 = typename std::conditional<kF32, float2, uint32_t>::type;
    pdl_trigger();
    extern __shared__ __align__(128) unsigned char smem[];            // the ring: [stages][16] records; then the rest
    __shared__ __align__(8) uint64_t full[kMaxStages], empty[kMaxStages], sums_full[kBufs];
    __shared__ uint32_t added[kAddWarps];                             // items that each adding warp is done with
    __shared__ uint32_t row_top[16];                                  // largest |x| of each row, as its bits
    // the same in all lanes, and known to be: what follows from it stays off the lanes' integer units
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31, r = lane >> 2, t = lane & 3;
    // this block's row tiles
    const int each = a.row_tiles / (int)gridDim.x, more = a.row_tiles - each * (int)gridDim.x;
    const int items = each + ((int)blockIdx.x < more ? 1 : 0);
    const int rt0 = (int)blockIdx.x * each + min((int)blockIdx.x, more);
    const int m0 = blockIdx.y * a.rows_pass;
    const int rows = min(a.rows - m0, a.rows_pass);
    const int cols = kF32 ? 2 * rows : rows;

    if (threadIdx.x < 16) row_top[threadIdx.x] = 0u;
    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], kPerStage);
        }
        for (int i = 0; i < kBufs; ++i) mbar_init(&sums_full[i], kWarps);
        for (int i = 0; i < kAddWarps; ++i) added[i] = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();

    if (warp == kWarps) {
        // ------------------------------------------------------------ copies (weights only: x may come from the kernel before)
        if (lane == 0) {
            int stage = 0, issued = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int panel = 0; panel < a.panels && ok; ++panel) {
                const int c0 = panel * a.panel_chunks, nc = min(a.panel_chunks, a.chunks - c0);
                int left = items * nc, c = 0;
                const unsigned char *src = a.records + ((long long)rt0 * a.chunks + c0) * kRecord;   // of the item's first chunk
                while (left > 0) {
                    if (!mbar_wait(&empty[stage], phase ^ 1)) { ok = false; break; }
                    const int n = min(left, kPerStage);
                    mbar_arrive_expect_tx(&full[stage], (uint32_t)(n * kRecord));
                    for (int done = 0; done < n;) {
                        const int len = min(n - done, nc - c);        // to the item's end at most
                        bulk_copy(smem + (stage * kPerStage + done) * kRecord, src + (long long)c * kRecord, (uint32_t)(len * kRecord), &full[stage]);
                        done += len;
                        c += len;
                        if (c == nc) {
                            c = 0;
                            src += (long long)a.chunks * kRecord;
                        }
                    }
                    ++issued;
                    left -= n;
                    if (++stage == a.stages) { stage = 0; phase ^= 1; }
                }
            }
            if (!ok) atomicOr(a.status, 1);
            // the last copies land before the block gives its shared memory back, even where a consumer gave up waiting
            for (int i = min(issued, a.stages); i > 0; --i) {
                if (--stage < 0) { stage = a.stages - 1; phase ^= 1; }
                mbar_wait(&full[stage], phase);
            }
        }
        return;
    }

    float *red = reinterpret_cast<float *>(smem + a.red_off);         // [kBufs][kWarps][kRed]
    pdl_wait();

    if (warp > kWarps) {
        // ------------------------------------------------------------ the sums of an item's warps, in the order of the warps
        float *outs = reinterpret_cast<float *>(smem + a.out_off);    // [items][rows][16]: sums of the panels so far
        const int id = threadIdx.x - (kWarps + 1) * 32;
        bool ok = true;
        int turn = 0;                                                 // items so far, over the panels
        for (int panel = 0; panel < a.panels; ++panel) {
            const int nc = min(a.panel_chunks, a.chunks - panel * a.panel_chunks);
            for (int item = 0; item < items; ++item, ++turn) {
                const int buf = turn & (kBufs - 1);
                if (ok && !mbar_wait(&sums_full[buf], (turn / kBufs) & 1)) {
                    ok = false;
                    if (lane == 0) atomicOr(a.status, 1);
                }
                const int end = (item + 1) * nc;
                for (int i = id; i < 16 * rows; i += kAddWarps * 32) {
                    const int row = i & 15, m = i >> 4, n = (rt0 + item) * 16 + row;
                    const float *o = red + buf * kWarps * kRed + (kF32 ? 2 * m : m) * kCol + row;
                    float v = 0.0f;
#pragma unroll
                    for (int w = 0; w < kWarps; ++w, o += kRed) {
                        // fewer chunks than warps: warp w has one of them, or none
                        if (nc < kWarps && ((end - 1 - w) & (kWarps - 1)) >= nc) continue;
                        v += kF32 ? o[kCol] + o[0] : o[0];
                    }
                    if (kScaled) v *= unscale_of(row_top[m]);
                    if (n >= a.N) continue;
                    float *sum = outs + (item * rows + m) * 16 + row;
                    if (panel) v += *sum;
                    if (panel < a.panels - 1) {
                        *sum = v;
                        continue;
                    }
                    if (a.bias) v += to_float(reinterpret_cast<const T *>(a.bias)[n]);
                    if (a.relu && v < 0.0f) v = 0.0f;
                    CERT_ST(reinterpret_cast<T *>(a.y)[(long long)(m0 + m) * a.ldy + n], from_float<T>(v));
                }
                __syncwarp();
                if (lane == 0) count_release(&added[warp - kWarps - 1], (uint32_t)turn + 1);
            }
        }
        return;
    }

    const uint32_t low = in_register(0x000f000fu), high = in_register(0x00f000f0u), magic = in_register(kMagic);
    bool ok = true;
    int before = 0, turn = 0;                                         // stages and items of the panels before
    // x is staged by `share` warps per row, this one taking every share-th 256 of K from x_begin on
    const int share = kWarps / rows, x_row = warp / share, x_begin = x_row < rows ? warp - x_row * share : a.chunks;
    const T *x = reinterpret_cast<const T *>(a.x) + (long long)(m0 + min(x_row, rows - 1)) * a.ldx;
    if constexpr (kScaled) {
        uint32_t top = 0;                                             // the row's largest value
#pragma unroll 4
        for (int j = x_begin; j < a.chunks; j += share) {
            float v[8];
            load8(x, j * kChunk + lane * 8, a.K, a.vec, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
        }
        top = __reduce_max_sync(0xffffffffu, top);
        if (lane == 0 && x_row < rows) atomicMax(&row_top[x_row], top);
        consumers_meet();
    }
    for (int panel = 0; panel < a.panels; ++panel) {
        const int nc = min(a.panel_chunks, a.chunks - panel * a.panel_chunks), k_first = panel * a.panel_chunks * kChunk;
        if (panel) consumers_meet();                                  // the last panel's x has been read
        // x of the panel as float16, zero behind K: column c at c * x_pitch
        const int m = x_row;
        const float scale = kScaled ? scale_of(row_top[min(m, rows - 1)]) : 1.0f;
#pragma unroll 4
        for (int j = x_begin; j < nc; j += share) {
            const int kk = j * kChunk + lane * 8;
            unsigned char *dst = smem + a.x_off + kk * 2;
            if constexpr (!kScaled) {
                uint32_t w[4];
                load8(reinterpret_cast<const uint16_t *>(x), k_first + kk, a.K, a.vec, w);
                *reinterpret_cast<uint4 *>(dst + m * a.x_pitch) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
                float v[8];
                load8(x, k_first + kk, a.K, a.vec, v);
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float f = v[2 * e] * scale, g = v[2 * e + 1] * scale;
                    hi[e] = pack2(f, g, false);
                    const float2 h = __half22float2(*reinterpret_cast<const __half2 *>(&hi[e]));
                    // an infinity stays in hi
                    lo[e] = pack2(fabsf(h.x) < INFINITY ? f - h.x : 0.0f, fabsf(h.y) < INFINITY ? g - h.y : 0.0f, false);
                }
                *reinterpret_cast<uint4 *>(dst + (kF32 ? 2 * m : m) * a.x_pitch) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                if (kF32) *reinterpret_cast<uint4 *>(dst + (2 * m + 1) * a.x_pitch) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
        }
        consumers_meet();
        // this lane's column of each tile; a column that is not there reads another's, and its sums are not looked at
        const unsigned char *xl[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) xl[j] = smem + a.x_off + min(j * 8 + r, cols - 1) * a.x_pitch + t * 16;
        float acc[NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[j][e] = 0.0f;
        const int records = items * nc;
        int c = warp, item = 0;                                       // of this warp's next record
        while (c >= nc && item < items) { c -= nc; ++item; }
        // its stage: one of every kWarps / kPerStage
        int stage = before + warp / kPerStage;
        uint32_t phase = (uint32_t)(stage / a.stages) & 1u;
        stage %= a.stages;
        const int staged = (records + kPerStage - 1) / kPerStage * kPerStage;   // every warp of a stage lets it go, record or not
        for (int f0 = 0; f0 + warp < staged; f0 += kWarps) {
            if (ok && !mbar_wait(&full[stage], phase)) {
                ok = false;
                if (lane == 0) atomicOr(a.status, 1);
            }
            if (f0 + warp < records) {
                const unsigned char *rec = smem + (stage * kPerStage + warp % kPerStage) * kRecord;
                const int xo = c * kChunk * 2;
                float part[NT][4];
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    uint32_t b[NT][2][4];
#pragma unroll
                    for (int j = 0; j < NT; ++j)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint4 u = *reinterpret_cast<const uint4 *>(xl[j] + xo + (p * 64 + h * 32) * 2);
                            b[j][h][0] = u.x; b[j][h][1] = u.y; b[j][h][2] = u.z; b[j][h][3] = u.w;
                        }
                    const uint4 w = *reinterpret_cast<const uint4 *>(rec + kCodeAt + p * 512 + lane * 16);
                    const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        const int step = p * 4 + s, g = step / GSTEPS;
                        // rows r: 1024 + code; rows r + 8, four bits higher: 1024 + 16 code
                        const uint32_t up = word[s] >> 8;
                        uint32_t q[4] = {and_or(word[s], low, magic), and_or(word[s], high, magic), and_or(up, low, magic), and_or(up, high, magic)};
                        // code - zero and (1024 + 16 code) / 16 - (64 + zero), both exact
                        uint32_t z0 = 0xe408e408u, z1 = 0xd480d480u;                // -1032, -72
                        if (ZEROS) {
                            const uint32_t zz = *reinterpret_cast<const unsigned short *>(rec + kZeroAt + (g * 8 + r) * 2);
                            z0 = 0xe400e400u | ((zz & 15u) * 0x00010001u);
                            z1 = 0xd400d400u | (((zz >> 8) & 15u) * 0x00100010u);
                        }
                        q[0] = fma2_half(q[0], 0x3c003c00u, z0);
                        q[1] = fma2_half(q[1], 0x2c002c00u, z1);
                        q[2] = fma2_half(q[2], 0x3c003c00u, z0);
                        q[3] = fma2_half(q[3], 0x2c002c00u, z1);
#pragma unroll
                        for (int j = 0; j < NT; ++j) {
                            if (step % GSTEPS == 0) mma16816<true>(part[j], q, b[j][s >> 1][(s & 1) * 2], b[j][s >> 1][(s & 1) * 2 + 1]);
                            else mma16816<false>(part[j], q, b[j][s >> 1][(s & 1) * 2], b[j][s >> 1][(s & 1) * 2 + 1]);
                        }
                        if (step % GSTEPS == GSTEPS - 1) {
                            const S2 v = *reinterpret_cast<const S2 *>(rec + (g * 8 + r) * sizeof(S2));
                            float s0, s1;
                            if constexpr (kF32) { s0 = v.x; s1 = v.y; }
                            else if constexpr (kScaled) { s0 = __uint_as_float(v << 16); s1 = __uint_as_float(v & 0xffff0000u); }
                            else {
                                s0 = __half2float(__ushort_as_half((unsigned short)(v & 0xffffu)));
                                s1 = __half2float(__ushort_as_half((unsigned short)(v >> 16)));
                            }
#pragma unroll
                            for (int j = 0; j < NT; ++j) {
                                acc[j][0] = fmaf(part[j][0], s0, acc[j][0]);
                                acc[j][1] = fmaf(part[j][1], s0, acc[j][1]);
                                acc[j][2] = fmaf(part[j][2], s1, acc[j][2]);
                                acc[j][3] = fmaf(part[j][3], s1, acc[j][3]);
                            }
                        }
                    }
                }
                c += kWarps;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[stage], 1);
            stage += kWarps / kPerStage;
            if (stage >= a.stages) { stage -= a.stages; phase ^= 1; }
            if (f0 + warp < records && c >= nc) {
                // the item's last record of this warp: lane (r, t) holds rows r, r + 8 and columns 2t, 2t + 1 of each tile
                const int n = turn + item, buf = n & (kBufs - 1);
                if (ok && !counts_reach(added, n - kBufs + 1, lane)) {
                    ok = false;
                    if (lane == 0) atomicOr(a.status, 1);
                }
                float *o = red + (buf * kWarps + warp) * kRed + 2 * t * kCol + r;
#pragma unroll
                for (int j = 0; j < NT; ++j, o += 8 * kCol) {
                    o[0] = acc[j][0];
                    o[kCol] = acc[j][1];
                    o[8] = acc[j][2];
                    o[kCol + 8] = acc[j][3];
                    acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
                }
                __syncwarp();
                // (with fewer chunks than warps the last chunk's warp arrives for those that have none)
                if (lane == 0) mbar_arrive(&sums_full[buf], nc < kWarps && c - kWarps == nc - 1 ? 1 + kWarps - nc : 1);
                while (c >= nc) { c -= nc; ++item; }
            }
        }
        turn += items;
        before += (records + kPerStage - 1) / kPerStage;
    }
}

template <typename T, int NT, bool ZEROS, int SHIFT>
cert_status_t launch_matvec3(const cert_int4 *op, Int4Args a, cudaStream_t st) {
    constexpr bool kF32 = std::is_same<T, float>::value;
    const int stage_bytes = kPerStage * op->record;
    const int rows = a.rows_pass, cols = kF32 ? 2 * rows : rows;
    const int red = sums_bufs(NT) * kWarps * 20 * 8 * NT * 4;
    const int blocks = std::min(op->row_tiles, op->sms), items = (op->row_tiles + blocks - 1) / blocks;
    // the panel of x: all of K where it leaves two stages and half the memory, else equal parts
    const int x_chunk = cols * kChunk * 2;
    const long long outs = (long long)items * 16 * rows * 4;
    const int room = std::min(kSmemBlock - red - 4 * stage_bytes - 64 * cols - 128, kSmemBlock / 2);
    int most = room / x_chunk;
    a.panels = 1;
    if (most < a.chunks) {
        most = room > outs ? (int)((room - outs) / x_chunk) : 0;
        if (most < 1) return CERT_ERR_UNSUPPORTED;
        a.panels = (a.chunks + most - 1) / most;
    }
    a.panel_chunks = (a.chunks + a.panels - 1) / a.panels;
    a.panels = (a.chunks + a.panel_chunks - 1) / a.panel_chunks;
    a.x_pitch = a.panel_chunks * kChunk * 2 + 64;                     // eight lanes' 16 bytes: two columns, all banks
    const int x_bytes = cols * a.x_pitch, out_bytes = a.panels > 1 ? (int)outs : 0;
    // an even number: a stage's place then belongs to one half of the warps, which have seen what was there before land
    a.stages = std::min(kMaxStages, (kSmemBlock - 128 - red - x_bytes - out_bytes) / stage_bytes) & ~1;
    a.red_off = (a.stages * stage_bytes + 127) / 128 * 128;
    a.x_off = a.red_off + red;
    a.out_off = a.x_off + x_bytes;
    const int smem = a.out_off + out_bytes;
    auto kernel = int4_matvec_kernel<T, NT, ZEROS, SHIFT>;
    static std::atomic<bool> allowed[64] = {};
    if (!allowed[op->device & 63]) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBlock) != cudaSuccess) {
            cudaGetLastError();
            return CERT_ERR_CUDA;
        }
        allowed[op->device & 63] = true;
    }
    const dim3 grid((unsigned)blocks, (unsigned)((a.rows + a.rows_pass - 1) / a.rows_pass));
    launch_chained(kernel, grid, dim3(kThreads), (size_t)smem, st, a);
    return CERT_OK;
}

template <typename T, int NT, bool ZEROS>
cert_status_t launch_matvec2(const cert_int4 *op, const Int4Args &a, cudaStream_t st) {
    switch (op->group) {
    case 32: return launch_matvec3<T, NT, ZEROS, 5>(op, a, st);
    case 64: return launch_matvec3<T, NT, ZEROS, 6>(op, a, st);
    case 128: return launch_matvec3<T, NT, ZEROS, 7>(op, a, st);
    default: return launch_matvec3<T, NT, ZEROS, 8>(op, a, st);
    }
}

template <typename T, int NT>
cert_status_t launch_matvec(const cert_int4 *op, const Int4Args &a, cudaStream_t st) {
    return op->zeros ? launch_matvec2<T, NT, true>(op, a, st) : launch_matvec2<T, NT, false>(op, a, st);
}

// Rows of x per pass: as many as there are, up to 16 (8 in float32); fewer where the sums of many items over several panels
// of a long K would not fit beside the rest.
template <typename T>
cert_status_t launch_rows(const cert_int4 *op, Int4Args a, cudaStream_t st) {
    constexpr bool kF32 = std::is_same<T, float>::value;
    cert_status_t s = CERT_ERR_UNSUPPORTED;
    for (a.rows_pass = std::min(a.rows, kF32 ? 8 : 16); s == CERT_ERR_UNSUPPORTED && a.rows_pass > 0; a.rows_pass /= 2) {
        s = a.rows_pass <= (kF32 ? 4 : 8) ? launch_matvec<T, 1>(op, a, st) : launch_matvec<T, 2>(op, a, st);
    }
    return s;
}

RecordShape shape_of(const cert_int4 *op) {
    RecordShape g = {op->K, op->N, op->k_tiles, op->groups, op->chunks, op->group, op->type, op->zeros, 0};
    g.record = g.code_at() + 2048;
    return g;
}

inline unsigned blocks_for(long long items, int sms) { return (unsigned)std::max<long long>(1, std::min<long long>((items + 255) / 256, (long long)sms * 32)); }

}  // namespace
}  // namespace cert

extern "C" {

cert_status_t cert_int4_create(const unsigned char *codes, const void *scales, const unsigned char *zeros, int out_features,
                               int in_features, int group, int type, void *stream, cert_int4_t **out) {
    using namespace cert;
    if (!codes || !scales || !out || out_features < 1 || in_features < 1 || !type_ok(type)) return CERT_ERR_INVALID_ARG;
    if (group != 32 && group != 64 && group != 128 && group != 256) return CERT_ERR_UNSUPPORTED;
    if (out_features > (1 << 26) || in_features > (1 << 26) || !aligned(scales, type_size(type))) return CERT_ERR_INVALID_ARG;
    cert_int4 *op = new (std::nothrow) cert_int4;
    if (!op) return CERT_ERR_OOM;
    op->N = out_features; op->K = in_features; op->group = group; op->type = type;
    op->row_tiles = (out_features + 15) / 16;
    op->k_tiles = (in_features + 63) / 64;
    op->groups = (in_features + group - 1) / group;
    op->chunks = (op->k_tiles + 3) / 4;
    op->zeros = zeros != nullptr;
    const RecordShape shape = shape_of(op);
    op->record = shape.record;
    if (cudaGetDevice(&op->device) != cudaSuccess ||
        cudaDeviceGetAttribute(&op->sms, cudaDevAttrMultiProcessorCount, op->device) != cudaSuccess) {
        cudaGetLastError();
        delete op;
        return CERT_ERR_CUDA;
    }
    const long long records = (long long)op->row_tiles * op->chunks;
    const long long words = records * 128, gs = records * shape.per_chunk() * 16;
    if (!op->mem.alloc(&op->records, (size_t)records * op->record) || !op->mem.alloc(&op->status, 1, true)) {
        op->mem.release();
        delete op;
        return CERT_ERR_OOM;
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
#ifdef CERT_BOUNDS
    op->mem.permit({}, op->status);
#endif
    int4_repack_kernel<<<blocks_for(words, op->sms), 256, 0, st>>>(codes, shape, op->records, words);
    if (type == CERT_TYPE_F32)
        int4_repack_groups_kernel<<<blocks_for(gs, op->sms), 256, 0, st>>>(reinterpret_cast<const float *>(scales), zeros, shape, op->records, gs);
    else
        int4_repack_groups_kernel<<<blocks_for(gs, op->sms), 256, 0, st>>>(reinterpret_cast<const uint16_t *>(scales), zeros, shape, op->records, gs);
    cert_status_t s = launch_status();
    // The product's copying warp reads the records before it waits for the kernel in front of it, and only what the host has
    // seen to be complete is sure to be visible to it then.
    if (cudaDeviceSynchronize() != cudaSuccess) {
        cudaGetLastError();
        if (s == CERT_OK) s = CERT_ERR_CUDA;
    }
    if (s != CERT_OK) {
        op->mem.release();
        delete op;
        return s;
    }
    *out = op;
    return CERT_OK;
}

cert_status_t cert_int4_matvec(cert_int4_t *op, const void *x, long long ldx, int rows, const void *bias, int relu, void *y,
                               long long ldy, void *stream) {
    using namespace cert;
    if (!op || rows < 0 || !on_device(op->device)) return CERT_ERR_INVALID_ARG;
    if (rows == 0) return CERT_OK;
    const size_t es = (size_t)type_size(op->type);
    if (!x || !y || ldx < op->K || ldy < op->N || !aligned(x, es) || !aligned(y, es) || !aligned(bias, es)) return CERT_ERR_INVALID_ARG;
    if (rows > 65535) return CERT_ERR_BATCH_TOO_LARGE;
#ifdef CERT_BOUNDS
    op->mem.permit({{y, ((size_t)(rows - 1) * ldy + op->N) * es}}, op->status);
#endif
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    Int4Args a = {};
    a.records = op->records;
    a.x = x; a.bias = bias; a.y = y;
    a.ldx = ldx; a.ldy = ldy;
    a.rows = rows; a.relu = relu;
    a.vec = aligned(x, 16) && (ldx * (long long)es) % 16 == 0;
    a.N = op->N; a.K = op->K; a.row_tiles = op->row_tiles; 
    a.chunks = op->chunks;
    a.status = op->status;
    const cert_status_t s = op->type == CERT_TYPE_F32 ? launch_rows<float>(op, a, st)
                          : op->type == CERT_TYPE_BF16 ? launch_rows<__nv_bfloat16>(op, a, st) : launch_rows<__half>(op, a, st);
    if (s != CERT_OK) return s;
    return launch_status();
}

cert_status_t cert_int4_dequantize(cert_int4_t *op, float *weight, void *stream) {
    using namespace cert;
    if (!op || !weight || !aligned(weight, 4) || !on_device(op->device)) return CERT_ERR_INVALID_ARG;
#ifdef CERT_BOUNDS
    op->mem.permit({{weight, (size_t)op->N * op->K * 4}}, op->status);
#endif
    const long long words = (long long)op->row_tiles * op->chunks * 128;
    int4_dequantize_kernel<<<blocks_for(words, op->sms), 256, 0, static_cast<cudaStream_t>(stream)>>>(
        op->records, shape_of(op), weight, words);
    return launch_status();
}

cert_status_t cert_int4_quantize(const void *weight, long long ldw, int out_features, int in_features, int group, int type,
                                 unsigned char *codes, void *scales, unsigned char *zeros, void *stream) {
    using namespace cert;
    if (!weight || !codes || !scales || out_features < 1 || in_features < 1 || ldw < in_features || !type_ok(type)) return CERT_ERR_INVALID_ARG;
    if (group != 32 && group != 64 && group != 128 && group != 256) return CERT_ERR_UNSUPPORTED;
    if (!aligned(weight, type_size(type)) || !aligned(scales, type_size(type))) return CERT_ERR_INVALID_ARG;
    const int groups = (in_features + group - 1) / group;
    const long long blocks = ((long long)out_features * groups + 7) / 8;
    if (blocks > 0x7fffffffLL) return CERT_ERR_UNSUPPORTED;
#ifdef CERT_BOUNDS
    {
        const size_t n = (size_t)out_features;
        OpBuffers none;
        none.permit({{codes, n * ((in_features + 1) / 2)}, {scales, n * groups * type_size(type)}, {zeros, zeros ? n * groups : 0}}, nullptr);
    }
#endif
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (type == CERT_TYPE_F32)
        int4_quantize_kernel<float><<<(unsigned)blocks, 256, 0, st>>>(reinterpret_cast<const float *>(weight), ldw, out_features, in_features, group, groups, codes, reinterpret_cast<float *>(scales), zeros);
    else if (type == CERT_TYPE_BF16)
        int4_quantize_kernel<__nv_bfloat16><<<(unsigned)blocks, 256, 0, st>>>(reinterpret_cast<const __nv_bfloat16 *>(weight), ldw, out_features, in_features, group, groups, codes, reinterpret_cast<__nv_bfloat16 *>(scales), zeros);
    else
        int4_quantize_kernel<__half><<<(unsigned)blocks, 256, 0, st>>>(reinterpret_cast<const __half *>(weight), ldw, out_features, in_features, group, groups, codes, reinterpret_cast<__half *>(scales), zeros);
    return launch_status();
}

cert_status_t cert_int4_last_status(cert_int4_t *op, void *stream) {
    if (!op || !cert::on_device(op->device)) return CERT_ERR_INVALID_ARG;
    return cert::read_status(op->status, static_cast<cudaStream_t>(stream));
}

int cert_int4_check_guards(cert_int4_t *op, void *stream) {
    return op && cert::on_device(op->device) ? op->mem.check(static_cast<cudaStream_t>(stream)) : -1;
}

cert_status_t cert_int4_destroy(cert_int4_t *op) {
    if (!op || !cert::on_device(op->device)) return CERT_ERR_INVALID_ARG;
    const bool ok = cudaDeviceSynchronize() == cudaSuccess;
    if (!ok) cudaGetLastError();
    const bool freed = op->mem.release();
    delete op;
    return ok && freed ? CERT_OK : CERT_ERR_CUDA;
}

}  // extern "C"
