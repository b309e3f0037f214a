// Element types of the layer operators (omc_type): loads, stores and conversions.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "omc_internal.h"

namespace omc {
int note_cuda(cudaError_t e);

namespace el {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// A 32-bit word of T as FP32 values (one or two), and back.
template <typename T> struct Word;
template <> struct Word<float> {
    static constexpr int N = 1;
    static __device__ __forceinline__ void unpack(uint32_t w, float *v) { v[0] = __uint_as_float(w); }
    static __device__ __forceinline__ uint32_t pack(const float *v) { return __float_as_uint(v[0]); }
};
template <> struct Word<__half> {
    static constexpr int N = 2;
    static __device__ __forceinline__ void unpack(uint32_t w, float *v)
    {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
        v[0] = f.x;
        v[1] = f.y;
    }
    static __device__ __forceinline__ uint32_t pack(const float *v)
    {
        const __half2 h = __floats2half2_rn(v[0], v[1]);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
};
template <> struct Word<__nv_bfloat16> {
    static constexpr int N = 2;
    static __device__ __forceinline__ void unpack(uint32_t w, float *v)
    {
        v[0] = __uint_as_float(w << 16);
        v[1] = __uint_as_float(w & 0xFFFF0000u);
    }
    static __device__ __forceinline__ uint32_t pack(const float *v)
    {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[0], v[1]);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
};

// Two FP32 values in one instruction each.
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)));
    return *reinterpret_cast<float2 *>(&r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)));
    return *reinterpret_cast<float2 *>(&r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(r) : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)), "l"(*reinterpret_cast<uint64_t *>(&c)));
    return *reinterpret_cast<float2 *>(&r);
}
__device__ __forceinline__ float2 twice(float v) { return make_float2(v, v); }

// 32 bytes, to a 32-byte boundary.
__device__ __forceinline__ void store32(void *p, const uint32_t *w)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}

// Every kernel of the layer operators lets its successor start early and waits for the kernel before it here,
// in every CTA and before any global access: a CTA that left without waiting could let the successor's wait end
// while that earlier kernel still runs.  What it writes may be what this kernel reads, within this kernel's own
// lifetime: inputs are read by ordinary loads, never by those for memory that nobody writes meanwhile (so no __restrict__ on them).
__device__ __forceinline__ void enter_stream_order()
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

inline size_t size_of(int type) { return type == OMC_TYPE_F32 ? 4 : 2; }
inline bool type_ok(int type) { return type == OMC_TYPE_F32 || type == OMC_TYPE_F16 || type == OMC_TYPE_BF16; }
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

constexpr int MAX_DEVICES = 64;

// SMs of the current device, asked for once per device.
inline uint32_t sm_count()
{
    static std::atomic<int> known[MAX_DEVICES];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return DEFAULT_SMS;
    if (dev < MAX_DEVICES && (n = known[dev].load(std::memory_order_relaxed)) > 0) return (uint32_t)n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return DEFAULT_SMS;
    if (dev < MAX_DEVICES) known[dev].store(n, std::memory_order_relaxed);
    return (uint32_t)n;
}

// More dynamic shared memory than a kernel has by default: the runtime is told once per kernel and device, always the same.
constexpr uint32_t MOST_SMEM = 220 * 1024;
template <auto KERNEL>
int allow_smem(uint32_t bytes)
{
    static std::atomic<bool> told[MAX_DEVICES];
    if (bytes <= 40 * 1024) return OMC_OK;
    int dev = 0;
    if (const int rc = note_cuda(cudaGetDevice(&dev))) return rc;
    if (dev < MAX_DEVICES && told[dev].load(std::memory_order_acquire)) return OMC_OK;
    if (const int rc = note_cuda(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)MOST_SMEM))) return rc;
    if (dev < MAX_DEVICES) told[dev].store(true, std::memory_order_release);
    return OMC_OK;
}

// Launch as the programmatic dependent of the kernel before it on the stream.
template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, uint32_t threads, uint32_t smem, uint32_t cluster, void *stream, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

}  // namespace el
}  // namespace omc
