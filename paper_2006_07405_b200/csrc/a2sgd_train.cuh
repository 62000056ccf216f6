// What the training operators (a2sgd_adamw.cu, a2sgd_layer_norm.cu, a2sgd_gated_ffn.cu) share:
// element types, conversions, vector accesses and the host's launch helper.
#pragma once

#include "../../include/a2sgd.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace a2sgd_train {

// ------------------------------------------------------------------ element types
template <typename T>
__device__ __forceinline__ float to_f32(T x);
template <>
__device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <>
__device__ __forceinline__ float to_f32<__half>(__half x) { return __half2float(x); }

// One rounding to the nearest value of the type, ties to even (the identity for fp32).
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

__device__ __forceinline__ float lo_f32(uint32_t w, __nv_bfloat16) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f32(uint32_t w, __nv_bfloat16) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ float lo_f32(uint32_t w, __half) { return __half2float(__ushort_as_half((unsigned short)w)); }
__device__ __forceinline__ float hi_f32(uint32_t w, __half)
{
    return __half2float(__ushort_as_half((unsigned short)(w >> 16)));
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __nv_bfloat16)
{
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&p);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __half)
{
    const __half2 p = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&p);
}

// ------------------------------------------------------------------ eight elements at a time
// Streaming reads (no L1 allocation): each byte is used once.  16-byte alignment for the 16-bit
// types; 16 for fp32 too (two 128-bit accesses).
__device__ __forceinline__ uint4 ld_stream(const void *p)
{
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
                 : "l"(p));
    return r;
}
__device__ __forceinline__ void st_stream(void *p, uint4 v)
{
    asm volatile("st.global.L1::no_allocate.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
                 : "memory");
}

// Eight elements as loaded, still packed.
template <typename T>
struct Raw8 {
    uint4 q;
    __device__ __forceinline__ void load(const T *p) { q = ld_stream(p); }
    __device__ __forceinline__ void zero() { q = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void unpack(float (&f)[8]) const
    {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = lo_f32(w[i], T());
            f[2 * i + 1] = hi_f32(w[i], T());
        }
    }
};
template <>
struct Raw8<float> {
    uint4 a, b;
    __device__ __forceinline__ void load(const float *p)
    {
        a = ld_stream(p);
        b = ld_stream(p + 4);
    }
    __device__ __forceinline__ void zero() { a = b = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void unpack(float (&f)[8]) const
    {
        f[0] = __uint_as_float(a.x), f[1] = __uint_as_float(a.y), f[2] = __uint_as_float(a.z), f[3] = __uint_as_float(a.w);
        f[4] = __uint_as_float(b.x), f[5] = __uint_as_float(b.y), f[6] = __uint_as_float(b.z), f[7] = __uint_as_float(b.w);
    }
};

template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&f)[8])
{
    st_stream(p, make_uint4(pack2(f[0], f[1], T()), pack2(f[2], f[3], T()), pack2(f[4], f[5], T()), pack2(f[6], f[7], T())));
}
template <>
__device__ __forceinline__ void store8<float>(float *p, const float (&f)[8])
{
    st_stream(p, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
    st_stream(p + 4, make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])));
}

// ------------------------------------------------------------------ two fp32 operations in one instruction
// sm_100's packed fp32 arithmetic: each half is the single operation, rounded to nearest.  It halves what
// the element-wise kernels have to issue.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float lo, float hi)
{
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ f32x2 pair(float both) { return pair(both, both); }
__device__ __forceinline__ void unpair(f32x2 p, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p)); }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 add2_down(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("add.rm.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// A sum of products that each have to be rounded for themselves: the compiler fuses a packed product and a packed sum
// into a fused multiply-add even where both name their rounding (a x + (-0) in the product's place as well), so the
// sum is made of two single ones.
__device__ __forceinline__ f32x2 add2_of_products(f32x2 a, f32x2 b)
{
    float a0, a1, b0, b1;
    unpair(a, a0, a1);
    unpair(b, b0, b1);
    return pair(__fadd_rn(a0, b0), __fadd_rn(a1, b1));
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float sum2(f32x2 p)
{
    float lo, hi;
    unpair(p, lo, hi);
    return lo + hi;
}

// 256-bit accesses of fp32 data (32-byte alignment), marked evict-first in L2 as in the gradient
// path's kernels: a training step touches these bytes once, with gigabytes in between.
__device__ __forceinline__ void ld256(const float *p, float (&f)[8])
{
    asm volatile("ld.global.L1::no_allocate.L2::evict_first.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]), "=f"(f[4]), "=f"(f[5]), "=f"(f[6]), "=f"(f[7])
                 : "l"(p));
}
__device__ __forceinline__ void st256(float *p, const float (&f)[8])
{
    asm volatile("st.global.L1::no_allocate.L2::evict_first.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(f[0]),
                 "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7])
                 : "memory");
}

// ------------------------------------------------------------------ programmatic dependent launch
// Every kernel here is launched with programmatic stream serialisation: it may become resident
// while its predecessor drains, waits for the predecessor's end before its first global access,
// and lets its successor be scheduled in the same way.
__device__ __forceinline__ void wait_prior_grid() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void release_next_grid() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ------------------------------------------------------------------ host
inline cudaError_t launch(const void *fn, dim3 grid, unsigned threads, size_t smem, void **params, cudaStream_t s,
                          unsigned cluster = 1)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelExC(&cfg, fn, params);
}

struct DeviceGuard {
    int prev = -1, target = -1;
    bool ok = true;
    explicit DeviceGuard(int dev) : target(dev)
    {
        if (cudaGetDevice(&prev) != cudaSuccess || (prev != dev && cudaSetDevice(dev) != cudaSuccess)) {
            (void)cudaGetLastError();
            ok = false;
        }
    }
    ~DeviceGuard()
    {
        if (ok && prev != target) cudaSetDevice(prev);
    }
};

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline size_t size_of(int dtype) { return dtype == A2SGD_F32 ? 4 : 2; }
inline bool known(int dtype) { return dtype == A2SGD_F32 || dtype == A2SGD_BF16 || dtype == A2SGD_F16; }

// SMs of a device; asked once a device.
int sm_count(int device);
// CTAs of a kernel that an SM of `device`, the current one, holds at once, at least 1; asked once a kernel, device and shape.
int resident_ctas(const void *fn, unsigned threads, size_t smem, int device);

// Lets a kernel use that much dynamic shared memory on the current device; once a kernel, device and amount.
cudaError_t allow_smem(const void *fn, size_t bytes);

// Whether a device's count has moved since this was last asked with the same stream (before the first time: since 0).
// Each stream is told for itself, and each thread for its own per-thread default stream.
bool count_moved(int device, cudaStream_t stream, unsigned int count);

} // namespace a2sgd_train

#define A2_TRAIN_CUDA(call)              \
    do {                                 \
        if ((call) != cudaSuccess) {     \
            (void)cudaGetLastError();    \
            return A2SGD_ERR_CUDA;       \
        }                                \
    } while (0)
