// What operators on rows of logits (distill.hip, log_probs.hip) share: the softmax's running base and sum, and
// rows that start anywhere.
#pragma once

#include "rows.hpp"

namespace lda {

__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }
// exp((x - base) / T), exp2 in hardware.  The difference comes first: masks of the type's lowest value
// times c would overflow, and a row of nothing else has to come out even.
__device__ __forceinline__ float exp_above(float x, float base, float c)
{
    return __builtin_amdgcn_exp2f((x - base) * c);
}

__device__ __forceinline__ void join(float& m, float& s, float m2, float s2, float c)
{
    const float top = fmaxf(m, m2), base = base_of(top);
    s = s * exp_above(m, base, c) + s2 * exp_above(m2, base, c);
    m = top;
}
__device__ __forceinline__ void wave_join(float& m, float& s, float c)
{
    const float top = wave_max(m);
    s = wave_sum(s * exp_above(m, base_of(top), c));
    m = top;
}
template <int BLOCK>
__device__ __forceinline__ void block_join(float& m, float& s, float c, float2* part)
{
    wave_join(m, s, c);
    if (BLOCK == kWave) return;
    __syncthreads();
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = make_float2(m, s);
    __syncthreads();
    m = part[0].x;
    s = part[0].y;
#pragma unroll 1
    for (int w = 1; w < BLOCK / kWave; ++w) join(m, s, part[w].x, part[w].y, c);
}

// A row as the whole 16-byte chunks of memory inside it, and the elements before and behind
// those (fewer than two chunks), which a thread each takes.
template <class T>
struct SplitRow {
    static constexpr int E = Row<T>::kChunk;
    const T* p;
    int32_t head, whole, extras;  // elements, chunks, elements

    __device__ __forceinline__ SplitRow(const T* row, int32_t V) : p(row)
    {
        const int32_t lead = (int32_t)(((uintptr_t)row & 15u) / sizeof(T));
        head = min((E - lead) % E, V);
        whole = (V - head) / E;
        extras = V - whole * E;
    }
    __device__ __forceinline__ int32_t chunk(int32_t i) const { return head + i * E; }
    __device__ __forceinline__ int32_t extra(int32_t i) const { return i < head ? i : i + whole * E; }
    __device__ __forceinline__ uint4 load(int32_t i) const { return *reinterpret_cast<const uint4*>(p + chunk(i)); }
};

template <class T>
__device__ __forceinline__ void store_chunk(T* g, const float (&x)[Row<T>::kChunk])
{
    const uint4 r = Row<T>::pack(x);
    __builtin_memcpy(g, &r, 16);  // from any element on: the hardware takes unaligned addresses
}

}  // namespace lda
