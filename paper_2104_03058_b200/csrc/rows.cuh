// Row vectors of the elementwise and row-sum kernels: V neighbouring elements of fp32 or bf16 as fp32 values, in one access where the whole
// vector is inside the row.
#pragma once

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
}  // namespace gnnfd
