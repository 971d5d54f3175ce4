// Shared by the operators around the step (skew_clip.cu, skew_embed.cu, skew_gate.cu): the reason of a
// failed call, device queries, launches, and 8-element vector accesses. Not part of the public ABI.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "skewadam.h"

namespace skew {

// Sets skew_ops_last_error of this thread and returns `code` (skew_ops.cpp).
int ops_fail(int code, const char *fmt, ...);

// SMs of the current device (0 after a failed query).
int ops_sm_count();

inline int ops_cuda(cudaError_t e, const char *what) {
    return e == cudaSuccess ? SKEW_OK : ops_fail(SKEW_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

#ifdef __CUDACC__

// Lets `k` have up to `bytes` of dynamic shared memory on the current device: asked once for a kernel and device
// (0.5 us a call otherwise).
template <auto k>
cudaError_t ops_allow_smem(int bytes) {
    static std::atomic<uint64_t> allowed{0};  // by device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
    if (allowed.load(std::memory_order_acquire) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) allowed.fetch_or(bit, std::memory_order_release);
    return e;
}

// `after`: a programmatic dependent of the launch before it (it starts up while that one ends; the kernel
// orders itself by wait_launch_before).
template <typename... P, typename... Q>
cudaError_t ops_launch(bool after, void (*k)(P...), uint32_t grid, uint32_t threads, size_t smem, cudaStream_t s, Q... args) {
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = &at;
    cfg.numAttrs = after ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, k, static_cast<P>(args)...);
}

namespace {

constexpr uint32_t kFullMask = 0xFFFFFFFFu;

__device__ __forceinline__ void wait_launch_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void release_launch_after() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ uint4 ld_stream(const void *p) {  // read once
    uint4 u;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
    return u;
}

__device__ __forceinline__ void st_stream(void *p, uint4 u) {  // not read again soon
    asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(u.x), "r"(u.y), "r"(u.z), "r"(u.w) : "memory");
}

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

__device__ __forceinline__ uint32_t pack_bf16(float low, float high) {  // to nearest even
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(high), "f"(low));
    return w;
}

// One element, and eight consecutive ones on a 16-byte boundary, of an fp32 or bf16 array.
template <bool F32>
__device__ __forceinline__ float load1(const void *p, int64_t i) {
    if constexpr (F32)
        return static_cast<const float *>(p)[i];
    else
        return __uint_as_float(uint32_t(static_cast<const uint16_t *>(p)[i]) << 16);
}

template <bool F32>
__device__ __forceinline__ void store1(void *p, int64_t i, float x) {
    if constexpr (F32)
        static_cast<float *>(p)[i] = x;
    else
        static_cast<uint16_t *>(p)[i] = uint16_t(pack_bf16(x, 0.f));
}

template <bool F32>
struct Vec8 {  // raw: converted after all loads of a batch are under way
    uint4 u[F32 ? 2 : 1];
    __device__ __forceinline__ float at(int k) const {
        if constexpr (F32) {
            const uint4 v = u[k >> 2];
            return __uint_as_float((k & 3) == 0 ? v.x : (k & 3) == 1 ? v.y : (k & 3) == 2 ? v.z : v.w);
        } else {
            const uint32_t w = (k >> 1) == 0 ? u[0].x : (k >> 1) == 1 ? u[0].y : (k >> 1) == 2 ? u[0].z : u[0].w;
            return (k & 1) ? bf16_high(w) : bf16_low(w);
        }
    }
};

template <bool F32>
__device__ __forceinline__ const char *elem_ptr(const void *p, int64_t i) {
    return static_cast<const char *>(p) + i * (F32 ? 4 : 2);
}

template <bool F32>
__device__ __forceinline__ Vec8<F32> load8_cached(const void *p, int64_t i) {  // likely read again
    const uint4 *q = reinterpret_cast<const uint4 *>(elem_ptr<F32>(p, i));
    Vec8<F32> v;
    v.u[0] = q[0];
    if constexpr (F32) v.u[1] = q[1];
    return v;
}

template <bool F32>
__device__ __forceinline__ void store8(void *p, int64_t i, const float (&x)[8]) {
    char *q = const_cast<char *>(elem_ptr<F32>(p, i));
    if constexpr (F32) {
        st_stream(q, make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])));
        st_stream(q + 16, make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])));
    } else {
        st_stream(q, make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])));
    }
}

}  // namespace

#endif  // __CUDACC__

}  // namespace skew
