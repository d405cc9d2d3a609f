// Inputs and outputs of the few-bit operators in fp32, fp16 or bf16: eight elements at a time, as one
// access of 32 or 16 bytes (two of 16) where the rows are aligned, else one by one.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "mpq_internal.cuh"

namespace mpq {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v)
{
    return __float2bfloat16_rn(v);
}

// Two consecutive elements of one 4-byte word, the lower address first.
__device__ __forceinline__ float2 unpack2(uint32_t w, __half)
{
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}
__device__ __forceinline__ float2 unpack2(uint32_t w, __nv_bfloat16)
{
    return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w));
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __half)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __nv_bfloat16)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// Two floats at once, each rounded as one alone.
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<const uint64_t *>(&a)),
        "l"(*reinterpret_cast<const uint64_t *>(&b)));
    return *reinterpret_cast<const float2 *>(&r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(*reinterpret_cast<const uint64_t *>(&a)),
        "l"(*reinterpret_cast<const uint64_t *>(&b)), "l"(*reinterpret_cast<const uint64_t *>(&c)));
    return *reinterpret_cast<const float2 *>(&r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<const uint64_t *>(&a)),
        "l"(*reinterpret_cast<const uint64_t *>(&b)));
    return *reinterpret_cast<const float2 *>(&r);
}

// Eight elements from p (16-byte aligned).  Ordinary loads: in a kernel that begins with griddep_wait
// what they read may have been written by the kernel before.
__device__ __forceinline__ void load8(const float *p, float (&v)[8])
{
    if (((uintptr_t)p & 31) == 0) {      // one 32-byte access
        asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]),
                       "=f"(v[6]), "=f"(v[7])
                     : "l"(__cvta_generic_to_global(p)) : "memory");
        return;
    }
    const float4 a = reinterpret_cast<const float4 *>(p)[0];
    const float4 b = reinterpret_cast<const float4 *>(p)[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
    v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&v)[8])
{
    const uint4 a = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2(w[i], T());
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

// max(|a|, |b|, |c|); NaN if any is.
__device__ __forceinline__ float max_abs(float a, float b, float c)
{
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// max |x| of N elements (even) as fp32 bits: the order of non-negative floats, infinities and NaN above
// every finite value.
template <int N>
__device__ __forceinline__ uint32_t top_bits(const float (&v)[N])
{
    float m = max_abs(v[0], v[1], v[1]);
#pragma unroll
    for (int i = 2; i < N; i += 2) m = max_abs(m, v[i], v[i + 1]);
    return __float_as_uint(m);
}

__device__ __forceinline__ void store8(float *p, const float (&v)[8])
{
    if (((uintptr_t)p & 31) == 0) {
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     :: "l"(__cvta_generic_to_global(p)), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
                        "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                     : "memory");
        return;
    }
    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&v)[8])
{
    *reinterpret_cast<uint4 *>(p) =
        make_uint4(pack2(v[0], v[1], T()), pack2(v[2], v[3], T()), pack2(v[4], v[5], T()),
                   pack2(v[6], v[7], T()));
}

// Eight words from p on (16-byte aligned).
__device__ __forceinline__ void load_words(const uint32_t *p, uint32_t (&w)[8])
{
    if (((uintptr_t)p & 31) == 0) {
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]),
                       "=r"(w[6]), "=r"(w[7])
                     : "l"(__cvta_generic_to_global(p)) : "memory");
    } else {
        const uint4 a = reinterpret_cast<const uint4 *>(p)[0];
        const uint4 b = reinterpret_cast<const uint4 *>(p)[1];
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
        w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
    }
}

// Sixteen elements from p on, to p on (16-byte aligned): 32-byte accesses where p is 32-byte aligned.
template <typename T>
__device__ __forceinline__ void load16(const T *p, float (&v)[16])
{
    if constexpr (sizeof(T) == 4) {
        float a[8], b[8];
        load8(p, a);
        load8(p + 8, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = a[i], v[8 + i] = b[i];
    } else {
        uint32_t w[8];
        load_words(reinterpret_cast<const uint32_t *>(p), w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 f = unpack2(w[i], T());
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    }
}

// Eight words to p on (16-byte aligned).
__device__ __forceinline__ void store_words(uint32_t *p, const uint32_t (&w)[8])
{
    if (((uintptr_t)p & 31) == 0) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     :: "l"(__cvta_generic_to_global(p)), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                        "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
    } else {
        reinterpret_cast<uint4 *>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4 *>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

template <typename T>
__device__ __forceinline__ void store16(T *p, const float (&v)[16])
{
    if constexpr (sizeof(T) == 4) {
        float a[8], b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = v[i], b[i] = v[8 + i];
        store8(p, a);
        store8(p + 8, b);
    } else {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = pack2(v[2 * i], v[2 * i + 1], T());
        store_words(reinterpret_cast<uint32_t *>(p), w);
    }
}

// 32 consecutive elements, as load16's.
template <typename T>
__device__ __forceinline__ void load32(const T *p, float (&v)[32])
{
    float a[16], b[16];
    load16(p, a);
    load16(p + 16, b);
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = a[i], v[16 + i] = b[i];
}

// Host: bytes of an element type, 0 for a number that names none.
inline int type_size(int type)
{
    return type == MPQ_F32 ? 4 : type == MPQ_F16 || type == MPQ_BF16 ? 2 : 0;
}

// Host: rows of `ld` elements from `p` on, each 16-byte aligned.
inline bool rows_aligned(const void *p, int type, long long ld)
{
    return ((uintptr_t)p & 15) == 0 && (ld * type_size(type)) % 16 == 0;
}

// Host: fn(T()) for the element type `type` names (one that type_size knows).
template <typename F>
mpq_status by_type(int type, F &&fn)
{
    if (type == MPQ_F32) return fn(float());
    if (type == MPQ_F16) return fn(__half());
    return fn(__nv_bfloat16());
}

// Host: launch of a kernel that begins with griddep_wait (its blocks are resident before the kernel
// ahead of it on the stream ends).
template <typename... P, typename... A>
mpq_status launch_waiting(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem,
                          cudaStream_t stream, const char *what, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
    return cuda_status(e != cudaSuccess ? e : cudaGetLastError(), what);
}

}  // namespace mpq
