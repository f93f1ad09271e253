// What the training operators share: element types, vector loads and stores, reductions, host-side checks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dropcompute_train.h"

namespace dct {

constexpr int64_t kMaxDim = int64_t(1) << 30;

// Bounds the launches of this library on one device; the multiprocessor count is read once per device.
inline int sm_count()
{
    static int cached[64] = {};                 // 0 = not read yet; a racing second read stores the same value
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return 0;
    if (dev < 64) {
        const int have = __atomic_load_n(&cached[dev], __ATOMIC_RELAXED);
        if (have) return have;
    }
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (dev < 64) __atomic_store_n(&cached[dev], n, __ATOMIC_RELAXED);
    return n;
}

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int elem_bytes(int32_t dtype) { return dtype == DC_F32 ? 4 : 2; }
inline bool on(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
// rows of a matrix whose starts all fall on `a`-byte boundaries
inline bool rows_on(const void *p, int64_t stride, int eb, size_t a) { return on(p, a) && (size_t)(stride * eb) % a == 0; }

// Kernels follow each other, those of one call and of calls in a row, with programmatic dependent launch: the next one may start,
// and set itself up, while this one runs, and waits in follow() until this one is done and its writes are visible.  Every kernel
// calls it before it touches global memory, so all that went before in the stream is done too.  The next one is let in only after
// the wait, so that two kernels at most are on the device: let in before it, whole chains were, and under a kernel trace the device
// did not get to their end.  Without all this a step of seven kernels (251 x 5003 x 129) takes 58.8 us instead of 42.7.
template <class... P, class... A> int launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, const A &...args)
{
    cudaLaunchConfig_t c = {};
    c.gridDim = grid;
    c.blockDim = dim3((unsigned)threads);
    c.dynamicSmemBytes = smem;
    c.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    c.attrs = at;
    c.numAttrs = 1;
    if (cudaLaunchKernelEx(&c, kernel, static_cast<P>(args)...) == cudaSuccess) return DC_OK;
    cudaGetLastError();                      // the status says it; the caller's next check of its own does not find it again
    return DC_ERR_CUDA;
}
__device__ __forceinline__ void follow()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// A pack of adjacent elements of a row: 16 bytes where rows start on 16-byte boundaries, one element otherwise.
template <class T, int N> struct alignas(sizeof(T) * N) Pack { T v[N]; };

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ float from_f<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_f<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

}  // namespace dct
