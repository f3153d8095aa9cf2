// What the row operators (distill.hip, verify.hip, top_topics.hip, norm.hip, log_probs.hip, product.hip) share: element
// types, reductions over a wave and over a workgroup.
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include <cmath>

#include "common.hpp"

namespace lda {

inline size_t type_bytes(int32_t type) { return type == LDA_F32 ? 4 : 2; }
inline bool known_type(int32_t type) { return type == LDA_F32 || type == LDA_F16 || type == LDA_BF16; }
inline size_t index_bytes(int32_t type) { return type == LDA_I32 ? 4 : 8; }
inline bool known_index(int32_t type) { return type == LDA_I32 || type == LDA_I64; }
inline bool aligned_to(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// The elements that a 16-byte chunk holds, as floats.  bf16 is the upper half of a float.
template <class T>
struct Row;

template <>
struct Row<float> {
    static constexpr int kChunk = 4;
    static __device__ __forceinline__ float one(const float* p) { return *p; }
    static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[4])
    {
        x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y);
        x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[4])
    {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    static __device__ __forceinline__ float from(float x) { return x; }
};

template <>
struct Row<__half> {
    static constexpr int kChunk = 8;
    static __device__ __forceinline__ float one(const __half* p) { return __half2float(*p); }
    static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[8])
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __half2float(__ushort_as_half((unsigned short)(w[i] & 0xFFFFu)));
            x[2 * i + 1] = __half2float(__ushort_as_half((unsigned short)(w[i] >> 16)));
        }
    }
    static __device__ __forceinline__ uint32_t two(float lo, float hi)  // rounded to nearest even
    {
        return (uint32_t)__half_as_ushort(__float2half_rn(lo)) | ((uint32_t)__half_as_ushort(__float2half_rn(hi)) << 16);
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[8])
    {
        return make_uint4(two(x[0], x[1]), two(x[2], x[3]), two(x[4], x[5]), two(x[6], x[7]));
    }
    static __device__ __forceinline__ __half from(float x) { return __float2half_rn(x); }
};

template <>
struct Row<__hip_bfloat16> {
    static constexpr int kChunk = 8;
    typedef __bf16 two_t __attribute__((ext_vector_type(2)));
    typedef float two_f __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ float one(const __hip_bfloat16* p)
    {
        return __uint_as_float((uint32_t) * reinterpret_cast<const uint16_t*>(p) << 16);
    }
    static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[8])
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ uint32_t two(float lo, float hi)  // rounded to nearest even
    {
        const two_f f = {lo, hi};
        const two_t b = __builtin_convertvector(f, two_t);
        return __builtin_bit_cast(uint32_t, b);
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[8])
    {
        return make_uint4(two(x[0], x[1]), two(x[2], x[3]), two(x[4], x[5]), two(x[6], x[7]));
    }
    static __device__ __forceinline__ __hip_bfloat16 from(float x)
    {
        return __builtin_bit_cast(__hip_bfloat16, (uint16_t)two(x, 0.0f));
    }
};

__device__ __forceinline__ int64_t index_at(const void* p, int32_t type, int64_t i)
{
    return type == LDA_I32 ? (int64_t) static_cast<const int32_t*>(p)[i] : static_cast<const int64_t*>(p)[i];
}

__device__ __forceinline__ float element_at(const void* p, int32_t type, int64_t i)
{
    if (type == LDA_F32) return static_cast<const float*>(p)[i];
    if (type == LDA_F16) return Row<__half>::one(static_cast<const __half*>(p) + i);
    return Row<__hip_bfloat16>::one(static_cast<const __hip_bfloat16*>(p) + i);
}

// Sums and scans over a whole wave by lane shifts inside the vector ALU (row_shr 1, 2, 4, 8 inside rows of
// 16 lanes, then the rows' last lanes broadcast): some 25 cycles a step, an LDS permute takes 130.
// Every lane has to be active.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t shifted_in(uint32_t fill, uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)fill, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float shifted_in(float fill, float v)
{
    return __uint_as_float(shifted_in<CTRL, ROWS>(__float_as_uint(fill), __float_as_uint(v)));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int32_t shifted_in(int32_t fill, int32_t v)
{
    return (int32_t)shifted_in<CTRL, ROWS>((uint32_t)fill, (uint32_t)v);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double shifted_in(double fill, double v)
{
    const uint64_t f = __builtin_bit_cast(uint64_t, fill), b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = shifted_in<CTRL, ROWS>((uint32_t)f, (uint32_t)b);
    const uint32_t hi = shifted_in<CTRL, ROWS>((uint32_t)(f >> 32), (uint32_t)(b >> 32));
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
template <class V, class F>
__device__ __forceinline__ V wave_scan(V v, V none, F f)  // inclusive
{
    v = f(v, shifted_in<0x111, 0xf>(none, v));
    v = f(v, shifted_in<0x112, 0xf>(none, v));
    v = f(v, shifted_in<0x114, 0xf>(none, v));
    v = f(v, shifted_in<0x118, 0xf>(none, v));
    v = f(v, shifted_in<0x142, 0xa>(none, v));
    v = f(v, shifted_in<0x143, 0xc>(none, v));
    return v;
}
__device__ __forceinline__ float lane_value(float v, int lane)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane));
}
__device__ __forceinline__ int32_t lane_value(int32_t v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ double lane_value(double v, int lane)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
template <class V>
__device__ __forceinline__ V wave_prefix(V v)  // inclusive
{
    return wave_scan(v, V(0), [](V a, V b) { return a + b; });
}
template <class V>
__device__ __forceinline__ V wave_sum(V v)
{
    return lane_value(wave_prefix(v), kWave - 1);
}
__device__ __forceinline__ float wave_max(float v)
{
    return lane_value(wave_scan(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); }), kWave - 1);
}

// Sum over the workgroup, the same in every thread; `part` holds one value a wave.
template <int BLOCK, class V>
__device__ __forceinline__ V block_sum(V v, V* part)
{
    v = wave_sum(v);
    if (BLOCK == kWave) return v;
    __syncthreads();
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    V s = part[0];
#pragma unroll 4
    for (int w = 1; w < BLOCK / kWave; ++w) s += part[w];
    return s;
}

}  // namespace lda
