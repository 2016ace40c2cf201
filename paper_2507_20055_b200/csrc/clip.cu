// The 2-norm over many tensors and the tensors scaled to at most max_norm.
//
// The list is cut into pieces of about 32 KB once, at create; both kernels walk the pieces with every block of the
// grid.  Bound by memory: the tensors are read for the norm and read again for the scaling, 3 bytes moved for each of the
// list's where it does not stay in L2; the second pass walks backwards, so that it begins with what L2 still holds.
// 2 GB of bfloat16: 941 us, 6 GB at 6.4 TB/s; 24 MB of float32, which stay in L2: 15.5 us; 60 tensors of 1.6 MB in all: 5.2 us.
#include <algorithm>
#include <cmath>
#include <new>
#include <type_traits>

#include "ops_common.cuh"

namespace cert {
namespace {

constexpr int kPiece = 32768;            // bytes of a piece of a long list
constexpr int kThreads = 512;            // 4 x 16 bytes per thread and piece
constexpr int kBlocksPerSm = 4;

struct Piece {
    const char *in;
    char *out;
    int elements;
    short type;
    short vec;                           // in and out start on 16-byte boundaries
};

}  // namespace
}  // namespace cert

struct cert_clip {
    cert::OpBuffers mem;
    std::mutex calls;
    int device = 0, sms = 1;
    int n_pieces = 0;
    cert::Piece *pieces = nullptr;
    double *partial = nullptr;
    int *status = nullptr;
    std::vector<cert_tensor_t> outs;     // for the checking build: what the scaling may write
};

namespace cert {
namespace {

// The squares of the values of 16 bytes added to s.
template <typename T>
__device__ __forceinline__ float squares16(const uint4 &u, float s) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) s = fmaf(__uint_as_float(w[i]), __uint_as_float(w[i]), s);
        else {
            float a, b;
            if constexpr (std::is_same<T, __nv_bfloat16>::value) { a = __uint_as_float(w[i] << 16); b = __uint_as_float(w[i] & 0xffff0000u); }
            else { const float2 h = __half22float2(*reinterpret_cast<const __half2 *>(&w[i])); a = h.x; b = h.y; }
            s = fmaf(b, b, fmaf(a, a, s));
        }
    }
    return s;
}

// Sum of squares of a thread's share of a piece, in fp32 where it is safe, else in fp64.
template <typename T>
__device__ __forceinline__ double share_squares(const T *p, int n, bool vec) {
    constexpr int V = 16 / sizeof(T);
    float s = 0.0f;
    unsigned any = 0;                    // the values' bits: zero if there are only zeros
    const int nv = vec ? n / V : 0;
    const uint4 *src = reinterpret_cast<const uint4 *>(p) + threadIdx.x;
    int left = nv - (int)threadIdx.x;
    for (; left > 3 * kThreads; left -= 4 * kThreads, src += 4 * kThreads) {      // four loads in flight
        uint4 u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = src[i * kThreads];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            any |= u[i].x | u[i].y | u[i].z | u[i].w;
            s = squares16<T>(u[i], s);
        }
    }
    for (; left > 0; left -= kThreads, src += kThreads) {
        const uint4 u = *src;
        any |= u.x | u.y | u.z | u.w;
        s = squares16<T>(u, s);
    }
    for (int i = nv * V + threadIdx.x; i < n; i += kThreads) {
        const float f = to_float(p[i]);
        any |= __float_as_uint(f);
        s = fmaf(f, f, s);
    }
    // s may have overflowed, or lost squares below 1e-38: then once more in fp64 (this share alone)
    if (s < 1e30f && (s > 1e-28f || (any & 0x7fffffffu) == 0)) return (double)s;
    double d = 0.0;
    for (int i = threadIdx.x; i < nv; i += kThreads) {
#pragma unroll
        for (int j = 0; j < V; ++j) { const double f = (double)to_float(p[i * V + j]); d = fma(f, f, d); }
    }
    for (int i = nv * V + threadIdx.x; i < n; i += kThreads) { const double f = (double)to_float(p[i]); d = fma(f, f, d); }
    return d;
}

__device__ double block_sum(double v, double *scratch) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = threadIdx.x < kThreads / 32 ? scratch[threadIdx.x] : 0.0;
    if (threadIdx.x < 32) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    }
    return v;
}

__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
clip_norm_kernel(const Piece *__restrict__ pieces, int n_pieces, double *partial) {
    pdl_trigger();
    pdl_wait();
    __shared__ double scratch[kThreads / 32];
    double d = 0.0;
    for (int i = blockIdx.x; i < n_pieces; i += gridDim.x) {
        const Piece p = pieces[i];
        if (p.type == CERT_TYPE_F32) d += share_squares(reinterpret_cast<const float *>(p.in), p.elements, p.vec);
        else if (p.type == CERT_TYPE_BF16) d += share_squares(reinterpret_cast<const __nv_bfloat16 *>(p.in), p.elements, p.vec);
        else d += share_squares(reinterpret_cast<const __half *>(p.in), p.elements, p.vec);
    }
    d = block_sum(d, scratch);
    if (threadIdx.x == 0) CERT_ST(partial[blockIdx.x], d);
}

// The values of 16 bytes times f.
template <typename T>
__device__ __forceinline__ void scale16(uint4 &u, float f) {
    uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(__uint_as_float(w[i]) * f);
        else if constexpr (std::is_same<T, __nv_bfloat16>::value)
            w[i] = pack2(__uint_as_float(w[i] << 16) * f, __uint_as_float(w[i] & 0xffff0000u) * f, true);
        else {
            const float2 h = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
            w[i] = pack2(h.x * f, h.y * f, false);
        }
    }
    u = make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T>
__device__ __forceinline__ void scale_piece(const T *in, T *out, int n, bool vec, float f) {
    constexpr int V = 16 / sizeof(T);
    const int nv = vec ? n / V : 0;
    const uint4 *src = reinterpret_cast<const uint4 *>(in) + threadIdx.x;
    uint4 *dst = reinterpret_cast<uint4 *>(out) + threadIdx.x;
    int left = nv - (int)threadIdx.x;
    for (; left > 3 * kThreads; left -= 4 * kThreads, src += 4 * kThreads, dst += 4 * kThreads) {   // four loads in flight
        uint4 u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = src[i * kThreads];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            scale16<T>(u[i], f);
            CERT_ST(dst[i * kThreads], u[i]);
        }
    }
    for (; left > 0; left -= kThreads, src += kThreads, dst += kThreads) {
        uint4 u = *src;
        scale16<T>(u, f);
        CERT_ST(*dst, u);
    }
    for (int i = nv * V + threadIdx.x; i < n; i += kThreads) CERT_ST(out[i], from_float<T>(to_float(in[i]) * f));
}

// Every block adds the first kernel's sums for itself, in an order that is always the same (quicker than a last block that
// adds them at the end of the first kernel and others that wait for its one number).
template <int BLOCKS>
__global__ void __launch_bounds__(kThreads, BLOCKS)
clip_scale_kernel(const Piece *__restrict__ pieces, int n_pieces, const double *__restrict__ partial, int n_partial, float max_norm,
                  float *norm_out) {
    pdl_trigger();
    __shared__ double scratch[kThreads / 32];
    __shared__ float factor;
    pdl_wait();
    double d = 0.0;
    for (int i = threadIdx.x; i < n_partial; i += kThreads) d += partial[i];
    d = block_sum(d, scratch);
    if (threadIdx.x == 0) {
        const float norm = (float)sqrt(d), f = max_norm / (norm + 1e-6f);
        factor = f > 1.0f ? 1.0f : f;                          // and NaN stays NaN
        if (blockIdx.x == 0) CERT_ST(*norm_out, norm);
    }
    __syncthreads();
    const float f = factor;
    for (int i = n_pieces - 1 - (int)blockIdx.x; i >= 0; i -= gridDim.x) {
        const Piece p = pieces[i];
        if (f == 1.0f && p.in == p.out) continue;
        if (p.type == CERT_TYPE_F32) scale_piece(reinterpret_cast<const float *>(p.in), reinterpret_cast<float *>(p.out), p.elements, p.vec, f);
        else if (p.type == CERT_TYPE_BF16) scale_piece(reinterpret_cast<const __nv_bfloat16 *>(p.in), reinterpret_cast<__nv_bfloat16 *>(p.out), p.elements, p.vec, f);
        else scale_piece(reinterpret_cast<const __half *>(p.in), reinterpret_cast<__half *>(p.out), p.elements, p.vec, f);
    }
}

// Cuts the list into pieces of at most `bytes`, each within one tensor; up to the first 16-byte boundary, where both sides come
// to one together, a piece of its own.
void cut(const cert_tensor_t *tensors, int n, void *const *out, int bytes, std::vector<Piece> &list) {
    list.clear();
    for (int i = 0; i < n; ++i) {
        const cert_tensor_t &t = tensors[i];
        if (t.elements == 0) continue;
        const int es = type_size(t.type), per = bytes / es;
        const char *in = reinterpret_cast<const char *>(t.data);
        char *o = reinterpret_cast<char *>(out ? out[i] : t.data);
        long long at = 0;
        const size_t off = reinterpret_cast<uintptr_t>(in) & 15;
        if (off && off == (reinterpret_cast<uintptr_t>(o) & 15)) {
            at = std::min<long long>(t.elements, (long long)(16 - off) / es);
            list.push_back({in, o, (int)at, (short)t.type, 0});
        }
        for (; at < t.elements; at += per) {
            const char *a = in + at * es;
            char *b = o + at * es;
            list.push_back({a, b, (int)std::min<long long>(per, t.elements - at), (short)t.type,
                            (short)(aligned(a, 16) && aligned(b, 16))});
        }
    }
}

}  // namespace
}  // namespace cert

extern "C" {

cert_status_t cert_clip_create(const cert_tensor_t *tensors, int n, void *const *out, cert_clip_t **handle) {
    using namespace cert;
    if (!handle || n < 0 || (n > 0 && !tensors)) return CERT_ERR_INVALID_ARG;
    long long count = 0;
    for (int i = 0; i < n; ++i) {
        const cert_tensor_t &t = tensors[i];
        if (t.elements < 0 || !type_ok(t.type)) return CERT_ERR_INVALID_ARG;
        const void *o = out ? out[i] : t.data;
        if (t.elements > 0 && (!t.data || !o || !aligned(t.data, type_size(t.type)) || !aligned(o, type_size(t.type))))
            return CERT_ERR_INVALID_ARG;
        count += t.elements / (kPiece / type_size(t.type)) + 2;
    }
    if (count > 0x7fffffff) return CERT_ERR_UNSUPPORTED;
    cert_clip *op = new (std::nothrow) cert_clip;
    if (!op) return CERT_ERR_OOM;
    if (cudaGetDevice(&op->device) != cudaSuccess ||
        cudaDeviceGetAttribute(&op->sms, cudaDevAttrMultiProcessorCount, op->device) != cudaSuccess) {
        cudaGetLastError();
        delete op;
        return CERT_ERR_CUDA;
    }
    std::vector<Piece> list;
    try {
        op->outs.reserve(n);
        long long bytes = 0;
        for (int i = 0; i < n; ++i) {
            if (tensors[i].elements == 0) continue;
            op->outs.push_back({out ? out[i] : tensors[i].data, tensors[i].elements, tensors[i].type});
            bytes += tensors[i].elements * type_size(tensors[i].type);
        }
        // Pieces of 32 KB, four 16-byte loads of each thread, where there are many per block; fewer are made of a size that gives
        // every block the same number (24 MB: 741 pieces for 592 blocks would be two rounds, the second almost empty).
        const long long blocks = (long long)op->sms * kBlocksPerSm;
        int piece = kPiece;
        if (bytes < 8 * blocks * kPiece) {
            const long long rounds = std::max<long long>(1, (bytes + blocks * kPiece - 1) / (blocks * kPiece));
            piece = (int)std::max<long long>(2048, (bytes / (rounds * blocks) + 15) / 16 * 16);
            cut(tensors, n, out, piece, list);
            // the tensors' ends are pieces too: a little larger until the rounds suffice
            for (int i = 0; i < 16 && (long long)list.size() > rounds * blocks && piece < 2 * kPiece; ++i) {
                piece += (piece / 16 + 15) / 16 * 16;
                cut(tensors, n, out, piece, list);
            }
        } else {
            cut(tensors, n, out, piece, list);
        }
    } catch (const std::bad_alloc &) {
        delete op;
        return CERT_ERR_OOM;
    }
    op->n_pieces = (int)list.size();
    cert_status_t fail = CERT_OK;
    if (!op->mem.alloc(&op->pieces, std::max<size_t>(1, list.size())) ||
               !op->mem.alloc(&op->partial, (size_t)op->sms * kBlocksPerSm) || !op->mem.alloc(&op->status, 1, true)) {
        fail = CERT_ERR_OOM;
    } else if ((!list.empty() && cudaMemcpy(op->pieces, list.data(), list.size() * sizeof(Piece), cudaMemcpyHostToDevice) != cudaSuccess) ||
               cudaDeviceSynchronize() != cudaSuccess) {
        cudaGetLastError();
        fail = CERT_ERR_CUDA;
    }
    if (fail != CERT_OK) {
        op->mem.release();
        delete op;
        return fail;
    }
    *handle = op;
    return CERT_OK;
}

cert_status_t cert_clip_run(cert_clip_t *op, float max_norm, float *norm_out, void *stream) {
    using namespace cert;
    if (!op || !norm_out || !aligned(norm_out, 4) || !(max_norm >= 0.0f) || !on_device(op->device)) return CERT_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const OpLock lock(op->calls);
    if (!lock.held()) return CERT_ERR_CUDA;
#ifdef CERT_BOUNDS
    {
        std::vector<OpBuffers::Out> outs = {{norm_out, 4}};
        for (const cert_tensor_t &t : op->outs) outs.push_back({t.data, (size_t)t.elements * type_size(t.type)});
        op->mem.permit(outs, op->status);
    }
#endif
    const int blocks = std::max(1, std::min(op->n_pieces, op->sms * kBlocksPerSm));
    launch_chained(clip_norm_kernel, dim3(blocks), dim3(kThreads), 0, st, (const Piece *)op->pieces, op->n_pieces, op->partial);
    // Reading and writing at once, two blocks per multiprocessor move more than four where there is enough to do (2 GB of
    // bfloat16: 941 us both kernels, against 960); a short list wants all its blocks at once (24 MB: 15.5 us against 16.2).
    if (op->n_pieces > 8 * op->sms * kBlocksPerSm)
        launch_chained(clip_scale_kernel<2>, dim3(op->sms * 2), dim3(kThreads), 0, st, (const Piece *)op->pieces, op->n_pieces,
                       (const double *)op->partial, blocks, max_norm, norm_out);
    else
        launch_chained(clip_scale_kernel<kBlocksPerSm>, dim3(blocks), dim3(kThreads), 0, st, (const Piece *)op->pieces, op->n_pieces,
                       (const double *)op->partial, blocks, max_norm, norm_out);
    return launch_status();
}

cert_status_t cert_clip_last_status(cert_clip_t *op, void *stream) {
    if (!op || !cert::on_device(op->device)) return CERT_ERR_INVALID_ARG;
    return cert::read_status(op->status, static_cast<cudaStream_t>(stream));
}

int cert_clip_check_guards(cert_clip_t *op, void *stream) {
    return op && cert::on_device(op->device) ? op->mem.check(static_cast<cudaStream_t>(stream)) : -1;
}

cert_status_t cert_clip_destroy(cert_clip_t *op) {
    if (!op || !cert::on_device(op->device)) return CERT_ERR_INVALID_ARG;
    const bool ok = cudaDeviceSynchronize() == cudaSuccess;
    if (!ok) cudaGetLastError();
    const bool freed = op->mem.release();
    delete op;
    return ok && freed ? CERT_OK : CERT_ERR_CUDA;
}

}  // extern "C"
