// Softmax cross entropy of a linear layer over many classes, and its gradient, without the logits in memory.
//
//   z = x W^T + b,  loss_t = lse_t - z_t,y(t),  dz = s (softmax(z) - onehot),  dx = dz W,  dW = dz^T x,  db = sum dz
//
// Steps of a call:
//   1 rows     the rows that count are numbered (order kept) and gathered into a padded copy of x
//   2 LSE      z tile by tile on the tensor cores; per row and half tile the pair (max, sum of exponentials)
//   3 combine  pairs -> row statistics -> losses
//   4 for each piece of the classes: PROB recomputes the piece's z and stores p - onehot in 16 bits;
//     dx += p W, dW = p^T x
// With up to 256 classes a tile holds whole rows, and one product (ROW) takes the place of LSE, combine and PROB.
// With up to 16 classes and not too many rows all of it is two launches of another kind (xent_few.cu).
// 2TVD operations for the loss, 8TVD with gradients; the probabilities of a piece stay below kProbBytes.
// Sizes and cuts are worked out in xent_plan.cuh.  16-bit probabilities are a choice: both gradient products take them as
// operands, and a second part would make 12TVD of the 8.  bfloat16 gradients are 1.9e-3 off, relative, where their own rounding is
// 1.7e-3 (4096 x 2048 x 32768), float16 ones 2.3e-4 against 2.1e-4; float32 keeps three parts.
#include <algorithm>
#include <cmath>
#include <new>

#include "ops_common.cuh"
#include "xent_few.cuh"
#include "xent_gemm.cuh"

struct cert_xent {
    int max_rows = 0, type = 0, device = 0, pairs = 1, sms = 1;
    bool with_grad = false;
    cert::XentSizes size = {};
    cert::OpBuffers mem;
    std::mutex calls;
    int *status = nullptr;
    int *pos = nullptr, *idx = nullptr, *tgt = nullptr;   // row -> number among the kept ones (-1: ignored); back; class
    int *counts = nullptr;                                // [0] kept rows, [1] rows with a bad target, [2] ticket
    void *xc = nullptr;                                   // [rows_pad][parts * Dp] kept rows
    float2 *partial = nullptr;                            // [slots][rows_pad]
    float *target_logit = nullptr;
    float2 *stat = nullptr;
    double *block_sum = nullptr;
    float *bias32 = nullptr;                              // [V rounded up to 256]
    void *wbuf = nullptr;                                 // [piece][parts * Dp] copy of a piece of the weights
    void *prob = nullptr;                                 // [rows_pad][parts * piece]
    float *dx32 = nullptr;                                // [splits][rows_pad][Dp]
    float *dw32 = nullptr;                                // [splits][classes][Dp], where the classes are few
    float *colsum = nullptr;                              // [rows_pad / 32][piece]
    // Maps of the workspace for the last call's sizes (encoding one costs the host about as much as a launch's arguments).
    cert::XentMap map_x, map_x_mn, map_p, map_p_mn, map_po, map_dx32, map_dw32;
    int map_rows = -1, map_piece = -1, map_dx_most = 0, map_dw_most = 0;
    int few_rows = 0;                                     // calls of up to so many rows run on the fp32 units
    double *few_loss = nullptr;                           // [blocks]
    float *few_dw = nullptr, *few_db = nullptr;           // [blocks][16][D4], [blocks][16]
};

namespace cert {
namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kHalfShift = 14;                        // float16 probabilities are stored times 2^14

// x0 + x1 + x2 = x to 24 bits, each a bfloat16; what is not finite (or rounds to infinity) stays in the first.
__device__ __forceinline__ void split3(float x, float &h, float &m, float &l) {
    h = __bfloat162float(__float2bfloat16_rn(x));
    if (!(fabsf(h) < INFINITY)) {
        h = (fabsf(x) < INFINITY) ? copysignf(__uint_as_float(0x7f7f0000u), x) : x;
        m = l = 0.0f;
        if (!(fabsf(x) < INFINITY)) return;
    }
    const float r = x - h;
    m = __bfloat162float(__float2bfloat16_rn(r));
    l = r - m;
}

// Eight elements (from column d on) of a row into `parts` 16-bit numbers each, columns from D on zero; src == nullptr: zeros.
template <typename T>
__device__ __forceinline__ void pack8(const T *src, int d, int D, int Dp, int vec_ok, uint16_t *dst) {
    if constexpr (sizeof(T) == 2) {
        uint4 raw = make_uint4(0, 0, 0, 0);
        if (src && vec_ok && d + 8 <= D) raw = __ldg(reinterpret_cast<const uint4 *>(src + d));
        else if (src) {
            const uint16_t *s16 = reinterpret_cast<const uint16_t *>(src) + d;
            uint32_t w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                w[q] = (d + 2 * q < D ? (uint32_t)s16[2 * q] : 0u) | (d + 2 * q + 1 < D ? (uint32_t)s16[2 * q + 1] << 16 : 0u);
            raw = make_uint4(w[0], w[1], w[2], w[3]);
        }
        CERT_ST(*reinterpret_cast<uint4 *>(dst + d), raw);
    } else {
        float v[8];
        if (src && vec_ok && d + 8 <= D) {
            const float4 a = __ldg(reinterpret_cast<const float4 *>(src + d)), b = __ldg(reinterpret_cast<const float4 *>(src + d) + 1);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (src && d + e < D) ? src[d + e] : 0.0f;
        }
        uint32_t w[3][4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float h0, m0, l0, h1, m1, l1;
            split3(v[2 * q], h0, m0, l0);
            split3(v[2 * q + 1], h1, m1, l1);
            w[0][q] = pack2(h0, h1, true);
            w[1][q] = pack2(m0, m1, true);
            w[2][q] = pack2(l0, l1, true);
        }
#pragma unroll
        for (int part = 0; part < 3; ++part)
            CERT_ST(*reinterpret_cast<uint4 *>(dst + (long long)part * Dp + d), make_uint4(w[part][0], w[part][1], w[part][2], w[part][3]));
    }
}

// A piece of the weights into padded rows.
template <typename T>
__global__ void __launch_bounds__(256)
xent_pack_kernel(const T *__restrict__ src, long long ld, int rows, int D, int Dp, int parts, uint16_t *dst, int vec_ok) {
    pdl_trigger();
    pdl_wait();
    const int per = Dp / 8;
    const long long total = (long long)rows * per;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (long long)gridDim.x * blockDim.x) {
        const int p = (int)(i / per), d = (int)(i - (long long)p * per) * 8;
        pack8(src + (long long)p * ld, d, D, Dp, vec_ok, dst + (long long)p * parts * Dp);
    }
}

// Sum of v over the block's 256 threads, in every thread.
__device__ __forceinline__ int block_count(int v, int *scratch) {
    v = __reduce_add_sync(0xffffffffu, v);
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) v += scratch[w];
    __syncthreads();
    return v;
}

struct BeginArgs {
    const void *target;
    int is64, rows, classes;
    long long ignore;
    int *pos, *idx, *tgt, *counts, *status;
    float *row_losses;
    long long ldx;
    int D, Dp, parts, vec_ok;
    uint16_t *xc;
    const void *bias;
    int bias_type, Vp;
    float *bias32;
    void *dx_zero;                   // rows that do not count are zeroed here, or null
    long long lddx;
};

// Eight columns of a row of dx that does not count.
__device__ __forceinline__ void zero8(const BeginArgs &a, int row, int d) {
    if (!a.dx_zero) return;
    for (int e = d; e < min(d + 8, a.D); ++e) store_from_float(a.dx_zero, (long long)row * a.lddx + e, a.bias_type, 0.0f);
}

// A bias as the kernels use it: a type's lowest value as a mask would leave the fp32 range times log2 e, and a row with nothing else
// would have no finite maximum.
__device__ __forceinline__ float usable_bias(float b) {
    constexpr float kMost = 1.7014118346046923e38f;        // 2^127
    if (b < -kMost && b > -INFINITY) return -kMost;
    return b > kMost && b < INFINITY ? kMost : b;
}

// Start of a call.  A block takes consecutive rows (and, in grids of two dimensions, a share of their columns): it counts the rows before them that count, numbers its own in order and
// copies them to their places in the padded x.  The last block knows the total; it clears the rows up to the next multiple
// of 64, so that a block of K that reaches over the end adds nothing.  The bias becomes float32 on the way.
template <typename T>
__global__ void __launch_bounds__(256)
xent_begin_kernel(const T *__restrict__ x, const BeginArgs a) {
    pdl_trigger();
    __shared__ int scratch[8], place[256];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_wait();
    auto target_of = [&](int r) {
        return a.is64 ? reinterpret_cast<const long long *>(a.target)[r] : (long long)reinterpret_cast<const int *>(a.target)[r];
    };
    const int each = (a.rows + gridDim.x - 1) / gridDim.x;
    const int first = min(a.rows, (int)blockIdx.x * each), end = min(a.rows, first + each);
    int kept = 0, wrong = 0;
#pragma unroll 4
    for (int r = tid; r < first; r += 256) {
        const long long y = target_of(r);
        const bool in = y >= 0 && y < a.classes && y != a.ignore;
        kept += in;
        wrong += !in && y != a.ignore;
    }
    int base = block_count(kept, scratch);
    wrong = block_count(wrong, scratch);
    if (a.bias && blockIdx.y == 0)
        for (int i = blockIdx.x * 256 + tid; i < a.Vp; i += gridDim.x * 256)
            CERT_ST(a.bias32[i], i < a.classes ? usable_bias(load_as_float(a.bias, i, a.bias_type)) : 0.0f);
    const int per = a.Dp / 8;
    for (int r0 = first; r0 < end; r0 += 256) {
        const int r = r0 + tid;
        const long long y = r < end ? target_of(r) : a.ignore;
        const bool keep = y >= 0 && y < a.classes && y != a.ignore, bad = !keep && y != a.ignore;
        const unsigned mask = __ballot_sync(0xffffffffu, keep);
        if (lane == 0) scratch[warp] = __popc(mask);
        __syncthreads();
        int at = base, total = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            if (w < warp) at += scratch[w];
            total += scratch[w];
        }
        at += __popc(mask & ((1u << lane) - 1));
        place[tid] = keep ? at : -1;
        if (r < end && blockIdx.y == 0) {
            CERT_ST(a.pos[r], keep ? at : -1);
            if (a.row_losses && !keep) CERT_ST(a.row_losses[r], bad ? NAN : 0.0f);
        }
        if (keep && blockIdx.y == 0) {
            CERT_ST(a.idx[at], r);
            CERT_ST(a.tgt[at], (int)y);
        }
        wrong += __syncthreads_count(bad);
        const int n = min(256, end - r0);
        // (this block's share of the columns: d0 .. d1, eight at a time)
        const int d0 = (int)((long long)per * blockIdx.y / gridDim.y), width = (int)((long long)per * (blockIdx.y + 1) / gridDim.y) - d0;
        for (int i0 = tid; i0 < n * width; i0 += 4 * 256) {
            if (sizeof(T) == 2 && a.vec_ok) {
                // whole 16 bytes, four loads before the first store
                uint4 u[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int i = i0 + q * 256, k = min(i / width, n - 1), d = (d0 + i - i / width * width) * 8;
                    u[q] = make_uint4(0, 0, 0, 0);
                    if (i < n * width && place[k] >= 0 && d + 8 <= a.D) u[q] = __ldg(reinterpret_cast<const uint4 *>(x + (long long)(r0 + k) * a.ldx + d));
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int i = i0 + q * 256, k = i / width, d = (d0 + i - k * width) * 8;
                    if (i >= n * width) break;
                    const int p = place[k];
                    if (p < 0) zero8(a, r0 + k, d);
                    else if (d + 8 <= a.D || d >= a.D) CERT_ST(*reinterpret_cast<uint4 *>(a.xc + (long long)p * a.Dp + d), u[q]);
                    else pack8(x + (long long)(r0 + k) * a.ldx, d, a.D, a.Dp, 0, a.xc + (long long)p * a.Dp);
                }
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int i = i0 + q * 256, k = i / width, d = (d0 + i - k * width) * 8;
                    if (i >= n * width) break;
                    const int p = place[k];
                    if (p < 0) zero8(a, r0 + k, d);
                    else pack8(x + (long long)(r0 + k) * a.ldx, d, a.D, a.Dp, a.vec_ok, a.xc + (long long)p * a.parts * a.Dp);
                }
            }
        }
        base += total;
        __syncthreads();
    }
    if (blockIdx.x == gridDim.x - 1 && blockIdx.y == 0) {
        for (int i = tid; i < ((base + 63) / 64 * 64 - base) * per; i += 256) {
            const int k = i / per;
            pack8((const T *)nullptr, (i - k * per) * 8, a.D, a.Dp, 0, a.xc + (long long)(base + k) * a.parts * a.Dp);
        }
        if (tid == 0) {
            CERT_ST(a.counts[0], base);
            CERT_ST(a.counts[1], wrong);
            CERT_ST(a.counts[2], 0);
            if (wrong) atomicOr(a.status, 8);
        }
    }
}

// (max, sum) of every slot -> row statistics and losses; the last block adds the blocks' sums in order.
// 32 rows per block, 32 threads per row.
__global__ void __launch_bounds__(1024)
xent_combine_kernel(const float2 *__restrict__ partial, int rows_pad, int slots, int *counts, const int *__restrict__ idx,
                    const float *__restrict__ target_logit, float2 *stat, float *row_losses, double *block_sum,
                    int mean, float *loss) {
    pdl_trigger();
    pdl_wait();
    __shared__ float2 part[32][33];
    __shared__ int last;
    const int n = counts[0];
    const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5;
    const int row = blockIdx.x * 32 + lane;
    float m = -INFINITY, s = 0.0f;
    if (row < n) {
        for (int i = grp; i < slots; i += 32 * 8) {        // eight pairs in flight
            float2 p[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                p[u] = i + 32 * u < slots ? partial[(size_t)(i + 32 * u) * rows_pad + row] : make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float t = fmaxf(m, p[u].x);
                const float sub = t == -INFINITY ? 0.0f : t;
                s = s * exp2f(m - sub) + p[u].y * exp2f(p[u].x - sub);
                m = t;
            }
        }
    }
    part[grp][lane] = make_float2(m, s);
    __syncthreads();
    if (grp == 0) {
        double l = 0.0;
        if (row < n) {
            float top = -INFINITY;
#pragma unroll
            for (int g = 0; g < 32; ++g) top = fmaxf(top, part[g][lane].x);
            const float sub = top == -INFINITY ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (int g = 0; g < 32; ++g) sum += part[g][lane].y * exp2f(part[g][lane].x - sub);
            const float l2s = log2f(sum), zt = target_logit[row];
            // no class left in the row: every probability is zero
            CERT_ST(stat[row], sum == 0.0f ? make_float2(0.0f, INFINITY) : make_float2(sub, l2s));
            const float nll = zt == -INFINITY ? INFINITY : kLn2 * (fmaf(-zt, kLog2e, sub) + l2s);
            if (row_losses) CERT_ST(row_losses[idx[row]], nll);
            l = (double)nll;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        if (lane == 0) {
            CERT_ST(block_sum[blockIdx.x], l);
            __threadfence();
            last = atomicAdd(&counts[2], 1) == (int)gridDim.x - 1;
        }
    }
    __syncthreads();
    if (last && grp == 0) {
        __threadfence();
        double t = 0.0;
        for (int b = lane; b < (int)gridDim.x; b += 32) t += *(volatile double *)&block_sum[b];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        if (lane == 0) {
            if (mean) t /= (double)max(1, n);
            CERT_ST(*loss, counts[1] ? NAN : (float)t);
        }
    }
}

// The end of a call: what is still to be added up, scaled and rounded.  Blocks [0, dx_blocks) take dx, the next dw_blocks dW,
// the rest db.
struct FinishArgs {
    const int *counts;
    int mean, type, D, Dp, segs, pairs;
    float scale;
    int dx_blocks, dw_blocks;
    // dx: the slabs of each row that counts, zero for the others
    const float *dx32;
    const int *pos;
    int rows, dx_most, dx_kb, dx_bn;
    long long dx_slab;
    void *dx;
    long long lddx;
    // dW: the slabs of classes [0, width)
    const float *dw32;
    int width, dw_most, dw_bn;
    long long dw_slab;
    void *dw;
    long long lddw;
    // db: column sums of groups of 32 rows
    const float *colsum;
    int colsum_ld, class0;
    void *db;
    // the loss, where ROW has left sums over groups of 32 rows: the last block's
    const double *loss_sum;
    float *loss;
};

__device__ __forceinline__ void add_slabs(const float *src, int splits, long long slab, int d, int D, float scale, void *dst, long long at,
                                          int type) {
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int s = 0; s < splits; ++s) {
        const float4 f = *reinterpret_cast<const float4 *>(src + (size_t)s * slab);
        v.x += f.x; v.y += f.y; v.z += f.z; v.w += f.w;
    }
    const float w[4] = {v.x * scale, v.y * scale, v.z * scale, v.w * scale};
    char *o = reinterpret_cast<char *>(dst) + at * (type == CERT_TYPE_F32 ? 4 : 2);
    if (d + 4 <= D && (reinterpret_cast<uintptr_t>(o) & (type == CERT_TYPE_F32 ? 15 : 7)) == 0) {
        if (type == CERT_TYPE_F32) CERT_ST(*reinterpret_cast<float4 *>(o), make_float4(w[0], w[1], w[2], w[3]));
        else CERT_ST(*reinterpret_cast<uint2 *>(o), make_uint2(pack2(w[0], w[1], type == CERT_TYPE_BF16), pack2(w[2], w[3], type == CERT_TYPE_BF16)));
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (d + e < D) store_from_float(dst, at + e, type, w[e]);
}

__global__ void __launch_bounds__(256)
xent_finish_kernel(const __grid_constant__ FinishArgs a) {
    pdl_trigger();
    pdl_wait();
    const int n = a.counts[0];
    const float scale = a.mean ? a.scale / (float)max(1, n) : a.scale;
    const int per = (a.D + 3) / 4;
    int b = blockIdx.x;
    if (a.loss && b == (int)gridDim.x - 1) {
        __shared__ double sums[8];
        double t = 0.0;
        for (int g = threadIdx.x; g < (n + 31) / 32; g += 256) t += a.loss_sum[g];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = t;
        __syncthreads();
        if (threadIdx.x == 0) {
            t = 0.0;
#pragma unroll
            for (int w = 0; w < 8; ++w) t += sums[w];
            if (a.mean) t /= (double)max(1, n);
            CERT_ST(*a.loss, a.counts[1] ? NAN : (float)t);
        }
        return;
    }
    if (b < a.dx_blocks) {
        const int tiles = (n + kXentPairRows - 1) / kXentPairRows * ((a.D + a.dx_bn - 1) / a.dx_bn);
        const int splits = a.dx_most > 1 ? xent_splits(tiles, a.dx_kb, a.segs, a.pairs, a.dx_most) : 1;
        for (long long i = (long long)b * 256 + threadIdx.x; i < (long long)a.rows * per; i += (long long)a.dx_blocks * 256) {
            const int t = (int)(i / per), d = (int)(i - (long long)t * per) * 4, p = a.pos[t];
            add_slabs(a.dx32 + (size_t)max(p, 0) * a.Dp + d, p < 0 ? 0 : splits, a.dx_slab, d, a.D, scale, a.dx, (long long)t * a.lddx + d, a.type);
        }
        return;
    }
    b -= a.dx_blocks;
    if (b < a.dw_blocks) {
        const int tiles = (a.width + kXentPairRows - 1) / kXentPairRows * ((a.D + a.dw_bn - 1) / a.dw_bn);
        const int splits = xent_splits(tiles, (n + 63) / 64, a.segs, a.pairs, a.dw_most);
        for (long long i = (long long)b * 256 + threadIdx.x; i < (long long)a.width * per; i += (long long)a.dw_blocks * 256) {
            const int v = (int)(i / per), d = (int)(i - (long long)v * per) * 4;
            add_slabs(a.dw32 + (size_t)v * a.Dp + d, splits, a.dw_slab, d, a.D, scale, a.dw, (long long)v * a.lddw + d, a.type);
        }
        return;
    }
    b -= a.dw_blocks;
    __shared__ float part[8][32];
    const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5;
    const int c = b * 32 + lane, groups = (n + 31) / 32;
    float s = 0.0f;
    if (c < a.width)
        for (int g = grp; g < groups; g += 8) s += a.colsum[(size_t)g * a.colsum_ld + c];
    part[grp][lane] = s;
    __syncthreads();
    if (grp == 0 && c < a.width) {
        float t = 0.0f;
#pragma unroll
        for (int g = 0; g < 8; ++g) t += part[g][lane];
        store_from_float(a.db, (long long)a.class0 + c, a.type, t * scale);
    }
}

// Calls of up to so many rows run in xent_few.cu, the others on the tensor cores.  There a call's time grows with rows x
// features (about 10 ns per 1000 elements of x, with gradients), here it is launches and, for 16-bit types, far less per element.
// Ten classes, with gradients, there against here: bfloat16, 256 x 1024 18 us against 30, 2048 x 1024 31 against 36, 8192 x 256
// 38 against 41, 16384 x 128 54 against 44, 8192 x 512 49 against 43, 256 x 4096 59 against 36, 4096 x 4096 187 against 89, 65536 x 784 683 against 254.  float32, 256 x 1024 17 us
// against 48, 4096 x 4096 191 against 242, 65536 x 784 649 against 567: always there, since the few large calls that would gain
// up to a quarter would need a copy of x in three parts, and a sure row, whose loss is a small difference of logits, is more exact there (fp64 sums).
int few_rows(int type, int max_rows, int features, int classes) {
    if (!xent_few_fits(features, classes)) return 0;
    if (type == CERT_TYPE_F32) return max_rows;
    return features <= 2048 ? std::min(max_rows, std::min(8192, (1 << 21) / features)) : 0;
}

void set_segments(XentGemmArgs &g, int parts) {
    if (parts == 1) {
        g.segs = 1;
        g.a_part[0] = g.b_part[0] = 0;
        return;
    }
    // all products of parts down to 2^-16 of the first, the small ones first
    static const signed char pa[6] = {2, 0, 1, 1, 0, 0}, pb[6] = {0, 2, 1, 0, 1, 0};
    g.segs = 6;
    for (int i = 0; i < 6; ++i) { g.a_part[i] = pa[i]; g.b_part[i] = pb[i]; }
}

void pack_weights(cert_xent *op, const void *src, long long ld, int rows, cudaStream_t st) {
    const int vec = aligned(src, 16) && (ld * type_size(op->type)) % 16 == 0;
    const XentSizes &size = op->size;
    const long long items = (long long)rows * (size.Dp / 8);
    const dim3 blocks((unsigned)std::min<long long>(ceil_div_ll(items, 256), (long long)op->sms * 16));
    uint16_t *dst = reinterpret_cast<uint16_t *>(op->wbuf);
    if (op->type == CERT_TYPE_F32)
        launch_chained(xent_pack_kernel<float>, blocks, dim3(256), 0, st, reinterpret_cast<const float *>(src), ld, rows, size.D, size.Dp, size.parts, dst, vec);
    else
        launch_chained(xent_pack_kernel<uint16_t>, blocks, dim3(256), 0, st, reinterpret_cast<const uint16_t *>(src), ld, rows, size.D, size.Dp, size.parts, dst, vec);
}

cert_status_t run(cert_xent *op, const cert_xent_args_t &q, cudaStream_t st) {
    const XentSizes &size = op->size;
    const int T = q.rows, D = size.D, V = size.V, Dp = size.Dp, parts = size.parts, es = type_size(op->type);
    const bool bf16 = op->type != CERT_TYPE_F16;
    const bool want_grad = q.dx || q.dweight || q.dbias;
    const int mean = q.reduction == CERT_REDUCE_MEAN;
    const int *count = op->counts;

    if (op->few_rows > 0 && T <= op->few_rows) {
        FewArgs f = {};
        f.rows = T; f.D = D; f.V = V; f.type = op->type;
        f.x = q.x; f.weight = q.weight; f.bias = q.bias; f.target = q.target;
        f.ldx = q.ldx; f.ldw = q.ldw; f.ignore = q.ignore_index;
        f.is64 = q.target_is_64; f.mean = mean; f.grad_scale = q.grad_scale;
        f.loss = q.loss; f.row_losses = q.row_losses;
        f.dx = q.dx; f.dweight = q.dweight; f.dbias = q.dbias; f.lddx = q.lddx; f.lddw = q.lddw;
        f.status = op->status; f.counts = op->counts;
        f.dw_part = op->few_dw; f.db_part = op->few_db; f.loss_part = op->few_loss;
        launch_xent_few(f, op->sms, st);
        return launch_status();
    }

    const bool direct = parts == 1 && aligned(q.weight, 16) && (q.ldw * es) % 16 == 0;
    const XentPlan plan = xent_plan(size, T, direct, want_grad, op->pairs);
    const int rows_pad = plan.rows_pad, tiles_m = plan.tiles_m, copy_piece = plan.copy_piece, piece = plan.piece, pieces = plan.pieces;

    XentMap map_w = {}, map_w_mn = {};
    XentGemmArgs base = {};
    base.bf16 = bf16;
    base.status = op->status;
    base.target = op->tgt;
    base.rows_pad = rows_pad;
    base.most_splits = 1;
    base.pairs = op->pairs;
    base.raster = 8;
    set_segments(base, parts);

    // ---- the gradient's pieces and splits
    const float unscale = q.grad_scale * (bf16 ? 1.0f : 1.0f / (1 << kHalfShift));
    const size_t slab = plan.slab, dw_slab = plan.dw_slab;
    const int dx_kb = plan.dx_kb, bn_dx = plan.bn_dx, dx_most = plan.dx_most, bn_dw = plan.bn_dw, dw_most = plan.dw_most;
    const bool dx_direct = pieces == 1 && dx_most == 1, dw_direct = dw_most == 1;
    if (op->map_rows != T || op->map_piece != (want_grad ? piece : 0) || op->map_dx_most != dx_most || op->map_dw_most != dw_most) {
        op->map_rows = -1;
        // (rows behind the last come in as zeros without being fetched)
        const int x_rows = std::max(T, 1), type16 = bf16 ? CERT_TYPE_BF16 : CERT_TYPE_F16;
        const long long x_row = (long long)parts * Dp, p_row = (long long)parts * piece;
        if (!xent_make_map(&op->map_x, op->xc, bf16, x_row, x_rows, x_row, 64, 128)) return CERT_ERR_CUDA;
        if (want_grad && (!xent_make_out_map(&op->map_po, op->prob, type16, p_row, rows_pad, p_row) ||
                          !xent_make_map(&op->map_p, op->prob, bf16, p_row, rows_pad, p_row, 64, 128) ||
                          !xent_make_map(&op->map_p_mn, op->prob, bf16, p_row, rows_pad, p_row, 64, 64) ||
                          !xent_make_map(&op->map_x_mn, op->xc, bf16, x_row, x_rows, x_row, 64, 64) ||
                          !xent_make_out_map(&op->map_dx32, op->dx32, CERT_TYPE_F32, Dp, (long long)dx_most * rows_pad, Dp) ||
                          (!dw_direct && !xent_make_out_map(&op->map_dw32, op->dw32, CERT_TYPE_F32, Dp, (long long)dw_most * std::min(piece, V), Dp))))
            return CERT_ERR_CUDA;
        op->map_rows = T; op->map_piece = want_grad ? piece : 0; op->map_dx_most = dx_most; op->map_dw_most = dw_most;
    }

    {
        BeginArgs g = {};
        g.target = q.target; g.is64 = q.target_is_64; g.rows = T; g.classes = V; g.ignore = q.ignore_index;
        g.pos = op->pos; g.idx = op->idx; g.tgt = op->tgt; g.counts = op->counts; g.status = op->status;
        g.row_losses = q.row_losses;
        g.ldx = q.ldx; g.D = D; g.Dp = Dp; g.parts = parts;
        g.vec_ok = aligned(q.x, 16) && (q.ldx * es) % 16 == 0;
        g.xc = reinterpret_cast<uint16_t *>(op->xc);
        g.bias = q.bias; g.bias_type = op->type; g.Vp = size.Vp; g.bias32 = op->bias32;
        g.dx_zero = dx_direct ? q.dx : nullptr;
        g.lddx = q.lddx;
        const int by_rows = std::max(1, std::min(op->sms * 4, T));
        const dim3 blocks((unsigned)by_rows, (unsigned)std::max(1, std::min(op->sms * 4 / by_rows, Dp / 8 / 256)));
        if (op->type == CERT_TYPE_F32) launch_chained(xent_begin_kernel<float>, blocks, dim3(256), 0, st, reinterpret_cast<const float *>(q.x), g);
        else launch_chained(xent_begin_kernel<uint16_t>, blocks, dim3(256), 0, st, reinterpret_cast<const uint16_t *>(q.x), g);
    }

    const bool by_row = plan.by_row;

    // ---- softmax statistics
    if (!by_row) {
        const int bn = plan.bn_lse;
        int slots = 0;
        for (int c0 = 0; c0 < V; c0 += copy_piece) {
            const int width = std::min(copy_piece, V - c0);
            XentGemmArgs g = base;
            g.M = rows_pad; g.m_count = count;
            g.N = width; g.K = D;
            g.bn = bn;
            g.raster = 16;
            g.a_pitch = g.b_pitch = Dp;
            if (direct) {
                if (!xent_make_map(&map_w, q.weight, bf16, D, V, q.ldw, 64, bn / 2)) return CERT_ERR_CUDA;
                g.b_mn0 = c0;
            } else {
                pack_weights(op, reinterpret_cast<const char *>(q.weight) + (long long)c0 * q.ldw * es, q.ldw, width, st);
                if (!xent_make_map(&map_w, op->wbuf, bf16, (long long)parts * Dp, width, (long long)parts * Dp, 64, bn / 2))
                    return CERT_ERR_CUDA;
            }
            g.bias = q.bias ? op->bias32 + c0 : nullptr;
            g.class0 = c0;
            g.partial = op->partial;
            g.slot0 = slots;
            g.target_logit = op->target_logit;
            const long long tiles = (long long)tiles_m * ceil_div_ll(width, bn);
            launch_xent_gemm(XENT_EPI_LSE, (int)std::min<long long>(tiles, op->pairs), op->map_x, map_w, op->map_x, g, st);
            slots += 2 * (int)ceil_div_ll(width, bn);
        }
        launch_chained(xent_combine_kernel, dim3((unsigned)ceil_div_ll(std::max(T, 1), 32)), dim3(1024), 0, st,
                       (const float2 *)op->partial, rows_pad, slots, op->counts, (const int *)op->idx,
                       (const float *)op->target_logit, op->stat, q.row_losses, op->block_sum, mean, q.loss);
    }
    if (!want_grad && !by_row) return launch_status();

    // ---- gradient, one piece of the classes after the other
    for (int c0 = 0; c0 < V; c0 += piece) {
        const int width = std::min(piece, V - c0);
        const int bn_p = xent_prob_bn(size, plan, T, width, op->pairs);
        if (direct) {
            if (!xent_make_map(&map_w, q.weight, bf16, D, V, q.ldw, 64, bn_p / 2) ||
                !xent_make_map(&map_w_mn, q.weight, bf16, D, V, q.ldw, 64, 64))
                return CERT_ERR_CUDA;
        } else {
            if (by_row || pieces > 1 || copy_piece < V)     // else it still holds all of them
                pack_weights(op, reinterpret_cast<const char *>(q.weight) + (long long)c0 * q.ldw * es, q.ldw, width, st);
            if (!xent_make_map(&map_w, op->wbuf, bf16, (long long)parts * Dp, width, (long long)parts * Dp, 64, bn_p / 2) ||
                !xent_make_map(&map_w_mn, op->wbuf, bf16, (long long)parts * Dp, width, (long long)parts * Dp, 64, 64))
                return CERT_ERR_CUDA;
        }
        XentGemmArgs g = base;                    // p - onehot of the piece
        g.M = rows_pad; g.m_count = count;
        g.N = width; g.K = D;
        g.bn = bn_p;
        g.raster = 16;
        g.a_pitch = g.b_pitch = Dp;
        g.b_mn0 = direct ? c0 : 0;
        g.bias = q.bias ? op->bias32 + c0 : nullptr;
        g.class0 = c0;
        g.stat = op->stat;
        g.prob = want_grad ? op->prob : nullptr;
        g.prob_ld = (long long)parts * piece;
        g.prob_parts = parts;
        g.prob_pitch = piece;
        g.prob_log2_scale = bf16 ? 0.0f : (float)kHalfShift;
        g.colsum = q.dbias ? op->colsum : nullptr;
        g.colsum_ld = piece;
        g.row_losses = q.row_losses;
        g.row_of = op->idx;
        g.loss_sum = op->block_sum;
        launch_xent_gemm(by_row ? XENT_EPI_ROW : XENT_EPI_PROB, (int)std::min<long long>((long long)tiles_m * ceil_div_ll(width, bn_p), op->pairs),
                         op->map_x, map_w, op->map_po, g, st);
        // dx and dW in one launch, the one with more to sum per tile first
        XentProduct px = {}, pw = {};
        XentGemmArgs &x = px.args, &w = pw.args;
        x = w = base;
        x.N = w.N = 0;
        x.bn = bn_dx; w.bn = bn_dw;
        long long tiles_x = 0, tiles_w = 0;
        if (q.dx) {
            px.a = op->map_p; px.b = map_w_mn;
            x.M = rows_pad; x.m_count = count;
            x.N = D;
            x.most_splits = dx_most;
            x.split_kb = dx_kb;
            x.a_pitch = piece; x.b_pitch = Dp;
            if (dx_direct) {
                x.out = q.dx; x.out_type = op->type; x.out_ld = q.lddx;
                x.out_scale = unscale;
                x.count = mean ? count : nullptr;
                x.row_map = op->idx;
                x.rows_16 = aligned(q.dx, 16) && (q.lddx * es) % 16 == 0;
            } else {
                x.out = op->dx32; x.out_type = CERT_TYPE_F32; x.out_ld = Dp;
                x.out_split_stride = (long long)slab;
                x.out_scale = 1.0f;
                x.split_rows = rows_pad;
                x.tma_out = 1;
                px.out = op->map_dx32;
            }
            x.b_k0 = direct ? c0 : 0;
            x.K = width;
            x.add = !dx_direct && c0 > 0;
            tiles_x = (long long)tiles_m * ceil_div_ll(D, bn_dx) * dx_most;
        }
        if (q.dweight) {
            pw.a = op->map_p_mn; pw.b = op->map_x_mn;
            w.a_mn = 1;
            w.M = width;
            w.N = D; w.k_count = count;
            const int tiles_v = (int)ceil_div_ll(width, kXentPairRows);
            w.a_pitch = piece; w.b_pitch = Dp;
            w.K = rows_pad;
            if (dw_direct) {
                char *out = reinterpret_cast<char *>(q.dweight) + (long long)c0 * q.lddw * es;
                w.out = out;
                w.out_type = op->type; w.out_ld = q.lddw;
                w.tma_out = xent_make_out_map(&pw.out, out, op->type, D, width, q.lddw);
                w.out_scale = unscale;
                w.count = mean ? count : nullptr;
            } else {
                w.most_splits = dw_most;
                w.out = op->dw32; w.out_type = CERT_TYPE_F32; w.out_ld = Dp;
                w.out_split_stride = (long long)dw_slab;
                w.out_scale = 1.0f;
                w.split_rows = std::min(piece, V);
                w.tma_out = 1;
                pw.out = op->map_dw32;
            }
            tiles_w = (long long)tiles_v * ceil_div_ll(D, w.bn) * dw_most;
        }
        if (tiles_x + tiles_w) {
            const int pairs = (int)std::min<long long>(tiles_x + tiles_w, op->pairs);
            if (!tiles_w || (tiles_x && (long long)x.K / dx_most >= (long long)rows_pad / dw_most)) launch_xent_store(pairs, px, pw, st);
            else launch_xent_store(pairs, pw, px, st);
        }
        const bool last = c0 + piece >= V, fin_dx = last && q.dx && !dx_direct, fin_dw = q.dweight && !dw_direct;
        if (fin_dx || fin_dw || q.dbias || by_row) {
            FinishArgs f = {};
            f.counts = op->counts; f.mean = mean; f.type = op->type; f.D = D; f.Dp = Dp; f.segs = base.segs; f.pairs = op->pairs;
            f.scale = unscale;
            const long long per = (D + 3) / 4;
            if (fin_dx) {
                f.dx_blocks = (int)std::min<long long>(std::max<long long>(1, ceil_div_ll(T * per, 256)), (long long)op->sms * 16);
                f.dx32 = op->dx32; f.pos = op->pos; f.rows = T; f.dx_most = dx_most; f.dx_kb = dx_kb; f.dx_bn = bn_dx;
                f.dx_slab = (long long)slab; f.dx = q.dx; f.lddx = q.lddx;
            }
            f.width = width;
            if (fin_dw) {
                f.dw_blocks = (int)std::min<long long>(ceil_div_ll(width * per, 256), (long long)op->sms * 16);
                f.dw32 = op->dw32; f.dw_most = dw_most; f.dw_bn = bn_dw; f.dw_slab = (long long)dw_slab;
                f.dw = q.dweight; f.lddw = q.lddw;
            }
            int db_blocks = 0;
            if (q.dbias) {
                db_blocks = (int)ceil_div_ll(width, 32);
                f.colsum = op->colsum; f.colsum_ld = piece; f.class0 = c0; f.db = q.dbias;
            }
            if (by_row) {
                f.loss_sum = op->block_sum;
                f.loss = q.loss;
            }
            launch_chained(xent_finish_kernel, dim3((unsigned)(f.dx_blocks + f.dw_blocks + db_blocks + (by_row ? 1 : 0))), dim3(256), 0, st, f);
        }
    }
    return launch_status();
}

}  // namespace
}  // namespace cert

extern "C" {

cert_status_t cert_xent_create(int max_rows, int features, int classes, int type, int with_grad, cert_xent_t **out) {
    using namespace cert;
    if (!out || max_rows < 1 || features < 1 || classes < 1 || !type_ok(type)) return CERT_ERR_INVALID_ARG;
    if (max_rows > (1 << 24) || features > (1 << 20) || classes > (1 << 28)) return CERT_ERR_UNSUPPORTED;
    cert_xent *op = new (std::nothrow) cert_xent;
    if (!op) return CERT_ERR_OOM;
    op->max_rows = max_rows; op->type = type;
    op->with_grad = with_grad != 0;
    op->size = xent_sizes(max_rows, features, classes, type, op->with_grad);
    const XentSizes &size = op->size;
    int sms = 0;
    cert_status_t fail = CERT_OK;
    if (cudaGetDevice(&op->device) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, op->device) != cudaSuccess || !xent_gemm_prepare() ||
        !xent_few_prepare()) {
        cudaGetLastError();
        delete op;
        return CERT_ERR_CUDA;
    }
    op->sms = sms;
    op->pairs = std::max(1, sms / 2);
    op->few_rows = few_rows(type, max_rows, features, classes);
    bool ok = op->mem.alloc(&op->status, 1, true) && op->mem.alloc(&op->counts, 4, true);
    if (ok && op->few_rows > 0) {
        const size_t blocks = (size_t)std::max(xent_few_blocks(op->few_rows, sms), xent_few_blocks(std::min(op->few_rows, 8 * sms), sms));
        ok = op->mem.alloc(&op->few_loss, blocks) && op->mem.alloc(&op->few_db, blocks * kFewClasses) &&
             op->mem.alloc(&op->few_dw, op->with_grad ? blocks * kFewClasses * (size_t)xent_up(features, 4) : 1);
    }
    if (op->few_rows < max_rows) {
        const size_t rows_pad = size.rows_pad;
        ok = ok && op->mem.alloc(&op->pos, rows_pad) && op->mem.alloc(&op->idx, rows_pad) && op->mem.alloc(&op->tgt, rows_pad) &&
             op->mem.alloc(reinterpret_cast<unsigned char **>(&op->xc), rows_pad * (size_t)size.row_bytes, true) &&
             op->mem.alloc(&op->partial, size.partial_cap) && op->mem.alloc(&op->target_logit, rows_pad) &&
             op->mem.alloc(&op->stat, rows_pad) && op->mem.alloc(&op->block_sum, rows_pad / 32) &&
             op->mem.alloc(&op->bias32, (size_t)size.Vp) &&
             op->mem.alloc(reinterpret_cast<unsigned char **>(&op->wbuf), size.wbuf_bytes);
        if (ok && op->with_grad)
            ok = op->mem.alloc(reinterpret_cast<unsigned char **>(&op->prob), size.prob_bytes, true) &&
                 op->mem.alloc(&op->dx32, size.dx32_floats) && op->mem.alloc(&op->dw32, size.dw32_floats) && op->mem.alloc(&op->colsum, size.colsum_floats);
    }
    if (!ok) fail = CERT_ERR_OOM;
    if (fail == CERT_OK && cudaDeviceSynchronize() != cudaSuccess) { cudaGetLastError(); fail = CERT_ERR_CUDA; }
    if (fail != CERT_OK) {
        op->mem.release();
        delete op;
        return fail;
    }
    *out = op;
    return CERT_OK;
}

cert_status_t cert_xent_run(cert_xent_t *op, const cert_xent_args_t *q, void *stream) {
    using namespace cert;
    if (!op || !q || !q->loss || q->rows < 0 || !on_device(op->device)) return CERT_ERR_INVALID_ARG;
    if (q->rows > op->max_rows) return CERT_ERR_BATCH_TOO_LARGE;
    if (q->reduction != CERT_REDUCE_MEAN && q->reduction != CERT_REDUCE_SUM) return CERT_ERR_INVALID_ARG;
    if (!q->weight || q->ldw < op->size.D || (q->rows > 0 && (!q->x || !q->target || q->ldx < op->size.D))) return CERT_ERR_INVALID_ARG;
    if (!std::isfinite(q->grad_scale)) return CERT_ERR_INVALID_ARG;
    const size_t es = (size_t)type_size(op->type);
    if ((q->x && !aligned(q->x, es)) || !aligned(q->weight, es) || (q->bias && !aligned(q->bias, es)) ||
        (q->dx && !aligned(q->dx, es)) || (q->dweight && !aligned(q->dweight, es)) || (q->dbias && !aligned(q->dbias, es)) ||
        !aligned(q->target, q->target_is_64 ? 8 : 4) || !aligned(q->loss, 4) || !aligned(q->row_losses, 4))
        return CERT_ERR_INVALID_ARG;
    if ((q->dx && q->lddx < op->size.D) || (q->dweight && q->lddw < op->size.D)) return CERT_ERR_INVALID_ARG;
    if ((q->dx || q->dweight || q->dbias) && !op->with_grad) return CERT_ERR_UNSUPPORTED;
    const OpLock lock(op->calls);
    if (!lock.held()) return CERT_ERR_CUDA;
#ifdef CERT_BOUNDS
    {
        const size_t n = (size_t)q->rows, d = (size_t)op->size.D;
        op->mem.permit({{q->loss, 4}, {q->row_losses, n * 4}, {q->dx, n ? ((n - 1) * q->lddx + d) * es : 0},
                        {q->dweight, ((size_t)(op->size.V - 1) * q->lddw + d) * es}, {q->dbias, (size_t)op->size.V * es}}, op->status);
    }
#endif
    return run(op, *q, static_cast<cudaStream_t>(stream));
}

cert_status_t cert_xent_last_status(cert_xent_t *op, void *stream) {
    if (!op || !cert::on_device(op->device)) return CERT_ERR_INVALID_ARG;
    return cert::read_status(op->status, static_cast<cudaStream_t>(stream));
}

int cert_xent_check_guards(cert_xent_t *op, void *stream) {
    return op && cert::on_device(op->device) ? op->mem.check(static_cast<cudaStream_t>(stream)) : -1;
}

cert_status_t cert_xent_destroy(cert_xent_t *op) {
    if (!op || !cert::on_device(op->device)) return CERT_ERR_INVALID_ARG;
    const bool ok = cudaDeviceSynchronize() == cudaSuccess;
    if (!ok) cudaGetLastError();
    const bool freed = op->mem.release();
    delete op;
    return ok && freed ? CERT_OK : CERT_ERR_CUDA;
}

}  // extern "C"
