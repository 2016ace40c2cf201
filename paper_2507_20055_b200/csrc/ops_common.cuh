// What the operators beside the certifiers share (linear_xent.cu, clip.cu, int4.cu): element types, device
// buffers with guard words, and the table of writable buffers of the checking build.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <cstring>
#include <mutex>
#include <vector>

#include "common.cuh"

namespace cert {

inline int type_size(int type) { return type == CERT_TYPE_F32 ? 4 : 2; }
inline bool type_ok(int type) { return type == CERT_TYPE_F32 || type == CERT_TYPE_BF16 || type == CERT_TYPE_F16; }
inline bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Device memory owned by an operator's handle.  Every buffer is kGuard bytes longer at either end, filled with a fixed
// pattern that check() reads back (as cert_net_check_guards does for a net).
class OpBuffers {
public:
    static constexpr size_t kGuard = 256;
    static constexpr int kByte = 0xA5;

    template <typename T>
    bool alloc(T **p, size_t count, bool zero = false) {
        const size_t bytes = (count * sizeof(T) + 255) & ~size_t(255);
        unsigned char *base = nullptr;
        if (cudaMalloc(reinterpret_cast<void **>(&base), bytes + 2 * kGuard) != cudaSuccess) {
            cudaGetLastError();
            return false;
        }
        try {
            all_.push_back({base, bytes});
        } catch (...) {                      // no exception may reach the C ABI
            cudaFree(base);
            return false;
        }
        if (cudaMemset(base, kByte, kGuard) != cudaSuccess ||
            cudaMemset(base + kGuard + bytes, kByte, kGuard) != cudaSuccess ||
            (zero && cudaMemset(base + kGuard, 0, bytes) != cudaSuccess)) {
            cudaGetLastError();
            return false;
        }
        *p = reinterpret_cast<T *>(base + kGuard);
        return true;
    }
    int check(cudaStream_t st) const {
        if (cudaStreamSynchronize(st) != cudaSuccess) { cudaGetLastError(); return -1; }
        unsigned char host[2 * kGuard];
        for (size_t i = 0; i < all_.size(); ++i) {
            if (cudaMemcpy(host, all_[i].base, kGuard, cudaMemcpyDeviceToHost) != cudaSuccess ||
                cudaMemcpy(host + kGuard, all_[i].base + kGuard + all_[i].bytes, kGuard, cudaMemcpyDeviceToHost) !=
                    cudaSuccess) {
                cudaGetLastError();
                return -1;
            }
            for (unsigned char c : host)
                if (c != kByte) return (int)i + 1;
        }
        return 0;
    }
    bool release() {
        bool ok = true;
        for (const Piece &p : all_) ok = (cudaFree(p.base) == cudaSuccess) && ok;
        all_.clear();
        if (!ok) cudaGetLastError();
        return ok;
    }
#ifdef CERT_BOUNDS
    // Checking build: the next kernels may write this handle's buffers and the given ones.
    struct Out { const void *p; size_t bytes; };
    void permit(const std::vector<Out> &outs, int *status) const {
        static BoundsTable t;
        t.n = 0;
        t.status = status;
        for (const Piece &p : all_) add(t, p.base + kGuard, p.bytes);
        for (const Out &o : outs)
            if (o.p) add(t, o.p, o.bytes);
        bounds_upload_all(&t);
    }
#endif

private:
    struct Piece { unsigned char *base; size_t bytes; };
    std::vector<Piece> all_;
#ifdef CERT_BOUNDS
    static void add(BoundsTable &t, const void *p, size_t bytes) {
        if (t.n >= kBoundsMax) return;
        t.lo[t.n] = (unsigned long long)p;
        t.hi[t.n] = t.lo[t.n] + bytes;
        ++t.n;
    }
#endif
};

// Whether the device that a handle was made on is current: with another one, the default stream is that device's, and a launch
// would get pointers of this one.  A host thread whose first call of CUDA this is has a current device but no context yet; a
// launch would make one, encoding a tensor map needs it before that.
inline bool on_device(int device) {
    static thread_local int ready = -1;
    int current = -1;
    if (cudaGetDevice(&current) != cudaSuccess || current != device || (ready != device && cudaSetDevice(device) != cudaSuccess)) {
        cudaGetLastError();
        return false;
    }
    ready = device;
    return true;
}

// One host thread at a time in a call on a handle: its launches stay together on the stream, and what the handle remembers of the
// last call is one call's.
class OpLock {
public:
    explicit OpLock(std::mutex &m) noexcept : m_(m) {
        try {
            m_.lock();
            held_ = true;
        } catch (...) {                      // no exception may reach the C ABI
        }
    }
    ~OpLock() { if (held_) m_.unlock(); }
    OpLock(const OpLock &) = delete;
    OpLock &operator=(const OpLock &) = delete;
    bool held() const { return held_; }

private:
    std::mutex &m_;
    bool held_ = false;
};

// The status word of a handle as a return code; clears it.
inline cert_status_t read_status(int *status_dev, cudaStream_t st) {
    int s = 0;
    if (cudaMemcpyAsync(&s, status_dev, sizeof(int), cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess) {
        cudaGetLastError();
        return CERT_ERR_CUDA;
    }
    if (s && (cudaMemsetAsync(status_dev, 0, sizeof(int), st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)) {
        cudaGetLastError();
        return CERT_ERR_CUDA;
    }
    return (s & 1) ? CERT_ERR_TIMEOUT : (s & 4) ? CERT_ERR_BOUNDS : (s & 8) ? CERT_ERR_INVALID_ARG : CERT_OK;
}

inline cert_status_t launch_status() {
    if (cudaPeekAtLastError() != cudaSuccess) {
        cudaGetLastError();
        return CERT_ERR_CUDA;
    }
    return CERT_OK;
}

#ifdef __CUDACC__
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
// Element i of an array of a type known at run time only.
__device__ __forceinline__ float load_as_float(const void *p, long long i, int type) {
    return type == CERT_TYPE_F32 ? reinterpret_cast<const float *>(p)[i]
         : type == CERT_TYPE_BF16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(p)[i])
                                  : __half2float(reinterpret_cast<const __half *>(p)[i]);
}
__device__ __forceinline__ void store_from_float(void *p, long long i, int type, float v) {
    if (type == CERT_TYPE_F32) CERT_ST(reinterpret_cast<float *>(p)[i], v);
    else if (type == CERT_TYPE_BF16) CERT_ST(reinterpret_cast<__nv_bfloat16 *>(p)[i], __float2bfloat16_rn(v));
    else CERT_ST(reinterpret_cast<__half *>(p)[i], __float2half_rn(v));
}
// Two values as a pair of 16-bit numbers, the first in the low half.
__device__ __forceinline__ uint32_t pack2(float a, float b, bool bf16) {
    uint32_t r;
    if (bf16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
#endif

}  // namespace cert
