// Row vectors of the elementwise and row-sum kernels: V neighbouring elements of fp32 or bf16 as fp32 values, in one access where the whole
// vector is inside the row.
#pragma once

#include <type_traits>

#include "vec.cuh"

namespace gnnfd {

// V elements as they lie in memory
template <typename T, int V>
struct Raw {
    static constexpr int kBytes = V * (int)sizeof(T);
    uint32_t w[kBytes < 4 ? 1 : kBytes / 4];
    __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (kBytes == 16) {
            const uint4 v = load16(p);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else if constexpr (kBytes == 8) {
            asm("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
        } else if constexpr (kBytes == 4) {
            asm("ld.global.b32 %0, [%1];" : "=r"(w[0]) : "l"(p));
        } else {
            unsigned short h;
            asm("ld.global.b16 %0, [%1];" : "=h"(h) : "l"(p));
            w[0] = h;
        }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < (kBytes < 4 ? 1 : kBytes / 4); ++i) w[i] = 0u;
    }
    __device__ __forceinline__ void get(float (&x)[V]) const
    {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if constexpr (sizeof(T) == 4) x[i] = __uint_as_float(w[i]);
            else x[i] = __uint_as_float((i & 1) ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
        }
    }
};

// the same at once as fp32 values
template <typename T, int V>
__device__ __forceinline__ void load_packed(const T* p, float (&x)[V])
{
    Raw<T, V> raw;
    raw.load(p);
    raw.get(x);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

template <typename T, int V>
__device__ __forceinline__ void store_packed(T* p, const float (&x)[V])
{
    if constexpr (sizeof(T) == 4) {
        if constexpr (V % 4 == 0) {
#pragma unroll
            for (int i = 0; i < V; i += 4) __stcs(reinterpret_cast<float4*>(p + i), make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]));
        } else if constexpr (V == 2) {
            __stcs(reinterpret_cast<float2*>(p), make_float2(x[0], x[1]));
        } else {
            __stcs(p, x[0]);
        }
    } else {
        if constexpr (V == 8) {
            __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]),
                                                           pack_bf16(x[6], x[7])));
        } else if constexpr (V == 4) {
            __stcs(reinterpret_cast<uint2*>(p), make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])));
        } else if constexpr (V == 2) {
            __stcs(reinterpret_cast<unsigned int*>(p), pack_bf16(x[0], x[1]));
        } else {
            *p = __float2bfloat16_rn(x[0]);
        }
    }
}

// Two neighbouring elements in one instruction (the same roundings as one by one): x * m + c.
__device__ __forceinline__ void scale_shift_pair(float& x, float& y, float m, float n, float c, float d)
{
    asm("{\n\t.reg .b64 p, q, r;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\tmov.b64 r, {%0, %1};\n\t"
        "fma.rn.f32x2 r, r, p, q;\n\tmov.b64 {%0, %1}, r;\n\t}" : "+f"(x), "+f"(y) : "f"(m), "f"(n), "f"(c), "f"(d));
}
// (x, y) += (a, b) * (c, d)
__device__ __forceinline__ void fma_pairs(float& x, float& y, float a, float b, float c, float d)
{
    asm("{\n\t.reg .b64 p, q, r;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\tmov.b64 r, {%0, %1};\n\t"
        "fma.rn.f32x2 r, p, q, r;\n\tmov.b64 {%0, %1}, r;\n\t}" : "+f"(x), "+f"(y) : "f"(a), "f"(b), "f"(c), "f"(d));
}
// x[i] += c[i], x[i] = x[i] * m[i] + c[i], x[i] *= m[i] and s[i] += x[i] * y[i]; CS: one c for all
template <int V, int CS>
__device__ __forceinline__ void add_minus(float (&x)[V], const float (&c)[CS])
{
    if constexpr (V == 1) x[0] -= c[0];
    else
#pragma unroll
        for (int i = 0; i < V; i += 2) add_pair(x[i], x[i + 1], -c[CS == 1 ? 0 : i], -c[CS == 1 ? 0 : i + 1]);
}
template <int V>
__device__ __forceinline__ void add_all(float (&s)[V], const float (&x)[V])
{
    if constexpr (V == 1) s[0] += x[0];
    else
#pragma unroll
        for (int i = 0; i < V; i += 2) add_pair(s[i], s[i + 1], x[i], x[i + 1]);
}
template <int V>
__device__ __forceinline__ void scale_shift(float (&x)[V], const float (&m)[V], const float (&c)[V])
{
    if constexpr (V == 1) x[0] = fmaf(x[0], m[0], c[0]);
    else
#pragma unroll
        for (int i = 0; i < V; i += 2) scale_shift_pair(x[i], x[i + 1], m[i], m[i + 1], c[i], c[i + 1]);
}
template <int V>
__device__ __forceinline__ void multiply(float (&x)[V], const float (&m)[V])
{
    if constexpr (V == 1) x[0] *= m[0];
    else
#pragma unroll
        for (int i = 0; i < V; i += 2) mul_pair(x[i], x[i + 1], m[i], m[i + 1]);
}
template <int V>
__device__ __forceinline__ void add_products(float (&s)[V], const float (&x)[V], const float (&y)[V])
{
    if constexpr (V == 1) s[0] = fmaf(x[0], y[0], s[0]);
    else
#pragma unroll
        for (int i = 0; i < V; i += 2) fma_pairs(s[i], s[i + 1], x[i], x[i + 1], y[i], y[i + 1]);
}

// x[i] = m * x[i], x[i] = m * x[i] + c for constants
template <int V>
__device__ __forceinline__ void scale(float (&x)[V], float m)
{
    if constexpr (V == 1) x[0] *= m;
    else
#pragma unroll
        for (int i = 0; i < V; i += 2) mul_pair(x[i], x[i + 1], m, m);
}
template <int V>
__device__ __forceinline__ void scale_shift(float (&x)[V], float m, float c)
{
    if constexpr (V == 1) x[0] = fmaf(x[0], m, c);
    else
#pragma unroll
        for (int i = 0; i < V; i += 2) scale_shift_pair(x[i], x[i + 1], m, m, c, c);
}

// a vector into fp32 or bf16, as the flag says
template <int V>
__device__ __forceinline__ void store_row(void* out, int bf16, int64_t at, const float (&x)[V])
{
    if (bf16) store_packed<__nv_bfloat16, V>(static_cast<__nv_bfloat16*>(out) + at, x);
    else store_packed<float, V>(static_cast<float*>(out) + at, x);
}

// the same where the row may end inside the vector (`left` columns from its first element on); columns past the end read as 0
template <typename T, int V>
__device__ __forceinline__ void load_row(const T* p, int left, float (&x)[V])
{
    if (left >= V) {
        load_packed<T, V>(p, x);
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float one[1] = {0.f};
        if (i < left) load_packed<T, 1>(p + i, one);
        x[i] = one[0];
    }
}

// ---- host side

// whether rows of elements of `size` bytes, `ld` apart, can be read and written in vectors of v elements (accesses have 16 bytes at most)
inline bool rows_fit(const void* p, int64_t ld, int size, int v)
{
    const int bytes = v * size < 16 ? v * size : 16;
    return (uintptr_t)p % bytes == 0 && ld * size % bytes == 0;
}

// f(elements per vector) for the widths there are; TI: float or __nv_bfloat16
template <typename TI, typename F>
inline int with_vector(int v, F f)
{
    switch (v) {
        case 8: if constexpr (sizeof(TI) == 2) return f(std::integral_constant<int, 8>());
        case 4: return f(std::integral_constant<int, 4>());
        case 2: return f(std::integral_constant<int, 2>());
        default: return f(std::integral_constant<int, 1>());
    }
}

}  // namespace gnnfd
