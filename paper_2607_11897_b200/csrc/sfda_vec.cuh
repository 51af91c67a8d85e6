// Loads and stores of V consecutive elements as fp32 values, with the widest access that V and the type make.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "sfda_tc_ptx.cuh"

namespace sfda {

template <int V>
__device__ __forceinline__ void ld_vec(const float *p, float (&x)[V])
{
    if constexpr (V % 4 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 v = *reinterpret_cast<const float4 *>(p + i);
            x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
        }
    } else if constexpr (V == 2) {
        const float2 v = *reinterpret_cast<const float2 *>(p);
        x[0] = v.x; x[1] = v.y;
    } else {
        static_assert(V == 1, "1, 2 or a multiple of 4 elements");
        x[0] = p[0];
    }
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
template <int V>
__device__ __forceinline__ void ld_vec(const __nv_bfloat16 *p, float (&x)[V])
{
    if constexpr (V == 8) {
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
    } else if constexpr (V == 4) {
        const uint2 v = *reinterpret_cast<const uint2 *>(p);
        x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
    } else if constexpr (V == 2) {
        const uint32_t v = *reinterpret_cast<const uint32_t *>(p);
        x[0] = bf16_lo(v); x[1] = bf16_hi(v);
    } else {
        static_assert(V == 1, "1, 2, 4 or 8 elements");
        x[0] = __bfloat162float(p[0]);
    }
}
template <int V>
__device__ __forceinline__ void st_vec(float *p, const float (&x)[V])
{
    if constexpr (V % 4 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 4) *reinterpret_cast<float4 *>(p + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    } else if constexpr (V == 2) {
        *reinterpret_cast<float2 *>(p) = make_float2(x[0], x[1]);
    } else {
        p[0] = x[0];
    }
}
template <int V>
__device__ __forceinline__ void st_vec(__nv_bfloat16 *p, const float (&x)[V])
{
    if constexpr (V == 8) {
        uint4 v;
        v.x = tc::pack_bf16(x[0], x[1]); v.y = tc::pack_bf16(x[2], x[3]);
        v.z = tc::pack_bf16(x[4], x[5]); v.w = tc::pack_bf16(x[6], x[7]);
        *reinterpret_cast<uint4 *>(p) = v;
    } else if constexpr (V == 4) {
        uint2 v;
        v.x = tc::pack_bf16(x[0], x[1]); v.y = tc::pack_bf16(x[2], x[3]);
        *reinterpret_cast<uint2 *>(p) = v;
    } else if constexpr (V == 2) {
        *reinterpret_cast<uint32_t *>(p) = tc::pack_bf16(x[0], x[1]);
    } else {
        p[0] = __float2bfloat16_rn(x[0]);
    }
}

// V elements as they lie in memory, to be in flight while something else is computed.
template <typename T, int V>
struct Raw {
    static constexpr int kWords = V * (int)sizeof(T) / 4;
    uint32_t w[kWords > 0 ? kWords : 1];
    __device__ __forceinline__ void load(const T *p)
    {
        if constexpr (kWords >= 4) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const uint4 v = *reinterpret_cast<const uint4 *>(reinterpret_cast<const uint32_t *>(p) + i);
                w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
            }
        } else if constexpr (kWords == 2) {
            const uint2 v = *reinterpret_cast<const uint2 *>(p);
            w[0] = v.x; w[1] = v.y;
        } else if constexpr (kWords == 1) {
            w[0] = *reinterpret_cast<const uint32_t *>(p);
        } else {
            w[0] = *reinterpret_cast<const uint16_t *>(p);
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < (kWords > 0 ? kWords : 1); ++i) w[i] = 0;
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
    }
};

}  // namespace sfda
