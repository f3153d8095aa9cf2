// Root-mean-square norm of rows with the residual's addition, to the rows' type or to 8 bits with a scale a
// row, and its gradient (the formulas stand at lda_norm_rows in lda_mi355x.h).
//
// A row is a workgroup's, in registers from its load to its store: a thread holds CHUNKS times 8 elements, 8
// adjacent ones a chunk, and reads nothing twice.  Rows too wide for that are read again from the cache
// (CHUNKS = 0).
#include <type_traits>

#include "rows.hpp"

namespace lda {

constexpr int kNormChunk = 8;
constexpr int kNormStats = 2;

struct NormArgs {
    int64_t rows, row0;
    int32_t H;
    const void* x;
    int64_t x_stride;
    const void* residual;
    int64_t residual_stride;
    const void* weight;
    int32_t weight_type;
    float eps;
    void* out;  // y, or 8-bit numbers
    int64_t out_stride;
    void* sum;
    int64_t sum_stride;
    float* scale;
    float* stats;  // [rows][kNormStats]
};

struct NormGradArgs {
    int64_t rows;
    int32_t H;
    const void* h;  // the sum, or x where there is no residual
    int64_t h_stride;
    const void* weight;
    int32_t weight_type;
    const float* stats;
    const void* y_grad;
    int64_t y_grad_stride;
    const void* sum_grad;
    int64_t sum_grad_stride;
    void* x_grad;
    int64_t x_grad_stride;
    void* residual_grad;
    int64_t residual_grad_stride;
    float* partial;  // [groups][H], or NULL: no gradient of the weight
    void* weight_grad;
    int32_t groups, column0;  // column0: of a launch of norm_weight_grad_kernel
};

// The 8 elements from p on; p is aligned to its type, which is all that the hardware's loads ask for.
__device__ __forceinline__ void load8(const float* p, float (&v)[8])
{
    __builtin_memcpy(v, p, 32);
}
template <class T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8])
{
    uint4 r;
    __builtin_memcpy(&r, p, 16);
    Row<T>::unpack(r, v);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) { __builtin_memcpy(p, v, 32); }
template <class T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8])
{
    const uint4 r = Row<T>::pack(v);
    __builtin_memcpy(p, &r, 16);
}
// A row's elements from i on: 8, or what is left of the row with 0 behind it
template <class T>
__device__ __forceinline__ void load_some(const T* row, int32_t i, int32_t H, float (&v)[8])
{
    if (i + 8 <= H) {
        load8(row + i, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = i + e < H ? Row<T>::one(row + i + e) : 0.0f;
    }
}
template <class T>
__device__ __forceinline__ void store_some(T* row, int32_t i, int32_t H, const float (&v)[8])
{
    if (i + 8 <= H) {
        store8(row + i, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i + e < H) row[i + e] = Row<T>::from(v[e]);
    }
}
template <class T>
__device__ __forceinline__ void load_weight(const void* w, int32_t type, int32_t i, int32_t H, float (&v)[8])
{
    if (!w) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 1.0f;
    } else if (type == LDA_F32) {
        load_some(static_cast<const float*>(w), i, H, v);
    } else {
        load_some(static_cast<const T*>(w), i, H, v);
    }
}

template <int BLOCK>
__device__ __forceinline__ uint32_t block_top(uint32_t v, uint32_t* part)  // largest, the same in every thread
{
    v = (uint32_t)lane_value((int32_t)wave_scan(v, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; }), kWave - 1);
    if (BLOCK == kWave) return v;
    __syncthreads();
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < BLOCK / kWave; ++w) v = max(v, part[w]);
    return v;
}

// What a thread's sum over a row is held in.  A thread has 16 numbers of a row in registers, and any number of a wider one:
// 32 bits would be rounded the same way at each addition where the numbers are alike (1.1 in 2^26 places: 6e-4 of
// the squares).  Each chunk is summed in 32.
template <bool WIDE>
using RowSum = std::conditional_t<WIDE, double, float>;

// n = (h * first) * second.  first is 1 but where squares leave 32 bits.
struct NormFactor {
    float first, second;
    __device__ __forceinline__ float of(float h) const { return (h * first) * second; }
};
// Sums of squares within these are good: none overflowed, and what underflowed is nothing beside them.
constexpr float kLeastSquares = 0x1p-80f, kMostSquares = 0x1p120f;

__device__ __forceinline__ NormFactor factor_of(float squares, float first, int32_t H, float eps)
{
    const float mean = squares / (float)H + eps * first * first;
    return {first, mean == 0.0f ? 0.0f : 1.0f / sqrtf(mean)};
}
// The power of two that brings a magnitude near 1
__device__ __forceinline__ float power_for(uint32_t top)
{
    const int e = (int)(top >> 23);
    if (e == 255 || top == 0) return 1.0f;
    return __uint_as_float((uint32_t)max(254 - e, 1) << 23);
}

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// 8 bits: a number's place among the levels, y / scale rounded to nearest even
constexpr uint32_t kLeastTop = (127 - 100) << 23;  // 2^-100: rows of less count as zeros
struct Levels {
    float k, scale;
    bool none;
    __device__ __forceinline__ Levels(uint32_t top, float most)
    {
        const bool odd = top >= 0x7F800000u;
        none = odd || top < kLeastTop;
        scale = odd ? NAN : none ? 0.0f : __uint_as_float(top) / most;
        k = none ? 0.0f : 1.0f / scale;
    }
};
// Where a level in 32 bits lies so near the middle of two numbers of Q that its roundings (some 4 of 2^-24) could
// take it to the wrong side: that middle.  false elsewhere.
template <class Q>
__device__ __forceinline__ bool near_middle(float level, float& middle);
template <>
__device__ __forceinline__ bool near_middle<int8_t>(float level, float& middle)
{
    middle = floorf(level) + 0.5f;
    return fabsf(level - middle) <= 0x1p-20f * fabsf(middle);
}
struct E4m3 {
    uint8_t bits;
};
template <>
__device__ __forceinline__ bool near_middle<E4m3>(float level, float& middle)  // 3 bits behind the leading one, 2^-9 at least
{
    if (fabsf(level) < 0x1p-6f) {
        middle = (floorf(level * 0x1p9f) + 0.5f) * 0x1p-9f;
        return fabsf(level - middle) <= 0x1p-20f * fabsf(middle);
    }
    const uint32_t bits = __float_as_uint(level);
    middle = __uint_as_float((bits & 0xFFF00000u) | 0x80000u);
    return (bits & 0xFFFFFu) - (0x80000u - 16u) <= 32u;
}
// Whether any of them may be, by fewer instructions
template <class Q>
__device__ __forceinline__ bool any_near_middle(const float (&v)[8])
{
    bool some = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (std::is_same<Q, int8_t>::value) some = some || fabsf(fabsf(v[e] - rintf(v[e])) - 0.5f) <= 0x1p-12f;
        else some = some || (__float_as_uint(v[e]) << 12) + (0x80000000u + (16u << 12)) <= 32u << 12;
    }
    if (std::is_same<Q, int8_t>::value) return some;
    float least = fabsf(v[0]);
#pragma unroll
    for (int e = 1; e < 8; ++e) least = fminf(least, fabsf(v[e]));
    return some || least < 0x1p-6f;
}
template <class Q>
__device__ __forceinline__ uint2 pack_levels(const float (&v)[8]);
template <>
__device__ __forceinline__ uint2 pack_levels<int8_t>(const float (&v)[8])
{
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int32_t q = (int32_t)rintf(fminf(fmaxf(v[e], -127.0f), 127.0f));
        w[e / 4] |= ((uint32_t)q & 0xFFu) << (e % 4 * 8);
    }
    return make_uint2(w[0], w[1]);
}
template <>
__device__ __forceinline__ uint2 pack_levels<E4m3>(const float (&v)[8])
{
    int w[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
        float c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = fminf(fmaxf(v[e + i], -448.0f), 448.0f);
        w[e / 4] = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], w[e / 4], false);
        w[e / 4] = __builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], w[e / 4], true);
    }
    return make_uint2((uint32_t)w[0], (uint32_t)w[1]);
}
template <class Q>
constexpr float most_of() { return std::is_same<Q, E4m3>::value ? 448.0f : 127.0f; }

template <class Q>
__device__ __forceinline__ void store_levels(Q* row, int32_t i, int32_t H, uint2 w)
{
    if (i + 8 <= H) {
        __builtin_memcpy(row + i, &w, 8);
    } else {
        const uint32_t b[2] = {w.x, w.y};
        uint8_t* const p = reinterpret_cast<uint8_t*>(row);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i + e < H) p[i + e] = (uint8_t)(b[e / 4] >> (e % 4 * 8));
    }
}

// T: of x and y; S: of the residual and the sum; Q: T, or 8 bits.  Bound by memory: 16384 x 8192 bf16 with a bf16
// residual to e4m3 take 183 us, one call after the other (194 under the profiler), to int8 179 to 188, 5.1 TB/s of read and
// written bytes (a copy of 1 GiB: 5.15), 165 with levels rounded from 32 bits alone; 8192 x 4096 bf16 with a float32 residual
// 83 us.  One row of 4096: 2.5 us, the latency of its loads and of a
// reduction.  A row's elements and weights stay in registers, 16 of each at most, between the reductions.
template <class T, class S, class Q, int BLOCK, int CHUNKS>
__global__ __launch_bounds__(BLOCK) void norm_kernel(NormArgs a)
{
    constexpr bool k8 = !std::is_same<Q, T>::value, kWide = CHUNKS == 0;
    constexpr int kHeld = kWide ? 1 : CHUNKS, kStep = BLOCK * kNormChunk;
    __shared__ RowSum<kWide> part[BLOCK / kWave];
    __shared__ uint32_t part_top[BLOCK / kWave];
    const int32_t tid = (int32_t)threadIdx.x, H = a.H;
    const int64_t row = a.row0 + blockIdx.x;
    const T* const x = static_cast<const T*>(a.x) + row * a.x_stride;
    const S* const r = a.residual ? static_cast<const S*>(a.residual) + row * a.residual_stride : nullptr;
    S* const sum = static_cast<S*>(a.sum) + row * a.sum_stride;
    Q* const out = static_cast<Q*>(a.out) + row * a.out_stride;
    float h[kHeld][8];
    // the sum as it is written: what is normed, and what the gradient reads
    const auto load = [&](int32_t i, float (&v)[8]) {
        load_some(x, i, H, v);
        if (!r) return;
        float b[8];
        load_some(r, i, H, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const S s = Row<S>::from(v[e] + b[e]);
            v[e] = Row<S>::one(&s);
        }
    };
    const auto each = [&](auto f) {
        if (kWide) {
            for (int32_t i = tid * kNormChunk; i < H; i += kStep) {
                load(i, h[0]);
                f(i, 0);
            }
        } else {
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j) {
                const int32_t i = j * kStep + tid * kNormChunk;
                if (i < H) f(i, j);
            }
        }
    };
    if (!kWide) {
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            const int32_t i = j * kStep + tid * kNormChunk;
            if (i < H) load(i, h[j]);
        }
    }
    const auto sum_of_squares = [&](float first, auto also) {
        RowSum<kWide> s = 0;
        each([&](int32_t i, int j) {
            also(i, j);
            float t = kWide ? 0.0f : (float)s;
#pragma unroll
            for (int e = 0; e < 8; ++e) t = __builtin_fmaf(h[j][e] * first, h[j][e] * first, t);
            s = kWide ? s + t : t;
        });
        return (float)block_sum<BLOCK>(s, part);
    };
    float squares = sum_of_squares(1.0f, [&](int32_t i, int j) {
        if (r) store_some(sum, i, H, h[j]);
    });
    float first = 1.0f;
    // rare: squares left 32 bits and eps does not hide it, or the row is 0
    if (!(squares + (float)H * a.eps >= kLeastSquares && squares <= kMostSquares)) {
        uint32_t top = 0;
        each([&](int32_t, int j) {
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, magnitude(h[j][e]));
        });
        first = power_for(max(block_top<BLOCK>(top, part_top), __float_as_uint(sqrtf(a.eps))));
        squares = sum_of_squares(first, [](int32_t, int) {});
    }
    const NormFactor f = factor_of(squares, first, H, a.eps);
    if (a.stats && tid == 0) *reinterpret_cast<float2*>(a.stats + row * kNormStats) = make_float2(f.first, f.second);
    float w[kHeld][8];
    const auto weigh = [&](int32_t i, int j) { load_weight<T>(a.weight, a.weight_type, i, H, w[j]); };
    const auto normed = [&](int j, int e) { return f.of(h[j][e]) * w[j][e]; };
    if constexpr (!k8) {
        each([&](int32_t i, int j) {
            weigh(i, j);
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = normed(j, e);
            store_some(out, i, H, y);
        });
    } else {
        // A level is h w over the largest |h w| of the row, times Q's largest: the root cancels.  It is taken in 32 bits,
        // and again in 64, from h and w themselves, where it lies so near the middle of two numbers that roundings
        // would decide: of rows in 16 bits many lie right there.
        __shared__ unsigned long long largest;  // the bits of the largest |h w|, in 64
        uint32_t top = 0;
        const auto top_of = [&](int32_t i, int j) {
            uint32_t t = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) t = max(t, i + e < H ? magnitude(normed(j, e)) : 0u);
            return t;
        };
        uint32_t tops[kHeld];
        each([&](int32_t i, int j) {
            weigh(i, j);
            tops[j] = top_of(i, j);
            top = max(top, tops[j]);
        });
        if (tid == 0) largest = 0;
        top = block_top<BLOCK>(top, part_top);
        const Levels l(top, most_of<Q>());
        if (tid == 0) a.scale[row] = l.scale;
        if (BLOCK == kWave) wave_lds_order();
        const auto exact = [&](int j, int e) { return (double)h[j][e] * (double)w[j][e]; };
        each([&](int32_t i, int j) {
            if (kWide) {
                weigh(i, j);
                tops[j] = top_of(i, j);
            }
            if (l.none || tops[j] + 4 < top) return;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (i + e < H && magnitude(normed(j, e)) + 4 >= top)
                    atomicMax(&largest, __builtin_bit_cast(unsigned long long, fabs(exact(j, e))));
        });
        if (BLOCK == kWave) wave_lds_order();
        else __syncthreads();
        const double most = __builtin_bit_cast(double, largest);
        each([&](int32_t i, int j) {
            if (kWide) weigh(i, j);
            float level[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) level[e] = normed(j, e) * l.k;
            if (!l.none && any_near_middle<Q>(level)) {
                double inverse = __builtin_amdgcn_rcp(most);  // a quotient in 64 bits takes three times as long
                inverse = __builtin_fma(__builtin_fma(-most, inverse, 1.0), inverse, inverse);
                inverse = __builtin_fma(__builtin_fma(-most, inverse, 1.0), inverse, inverse);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float middle;
                    if (!near_middle<Q>(level[e], middle) || i + e >= H) continue;
                    const double to = exact(j, e) * (inverse * (double)most_of<Q>()), off = to - (double)middle;
                    // the neighbour of the middle on the level's side, which rounds as the level does
                    level[e] = fabs(off) <= 0x1p-48 * fabs(to) ? middle : middle + (off > 0.0 ? 1.0f : -1.0f) * 0x1p-20f * fabsf(middle);
                }
            }
            store_levels(out, i, H, l.none ? make_uint2(0, 0) : pack_levels<Q>(level));
        });
    }
}

// The gradient of rows blockIdx.x, + gridDim.x, ...; what they give the weight is summed in registers and
// written as one row of `partial`.  Bound by memory: 8192 x 4096 bf16 with a float32 sum 99 us, 5.4 TB/s, and 5 for the
// partial rows.  Atomics in place of these would be in another order each time.
template <class T, class S, int BLOCK, int CHUNKS>
__global__ __launch_bounds__(BLOCK) void norm_grad_kernel(NormGradArgs a)
{
    constexpr bool kWide = CHUNKS == 0;
    constexpr int kHeld = kWide ? 1 : CHUNKS, kStep = BLOCK * kNormChunk;
    __shared__ RowSum<kWide> part[BLOCK / kWave];
    const int32_t tid = (int32_t)threadIdx.x, H = a.H;
    float n[kHeld][8], g[kHeld][8], w[kHeld][8], sums[kHeld][8];
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[j][e] = 0.0f;
        if (!kWide) load_weight<T>(a.weight, a.weight_type, j * kStep + tid * kNormChunk, H, w[j]);
    }
    float* const partial = a.partial ? a.partial + (int64_t)blockIdx.x * H : nullptr;
    bool fresh = true;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const S* const h = static_cast<const S*>(a.h) + row * a.h_stride;
        const T* const gy = static_cast<const T*>(a.y_grad) + row * a.y_grad_stride;
        const S* const gh = a.sum_grad ? static_cast<const S*>(a.sum_grad) + row * a.sum_grad_stride : nullptr;
        T* const gx = a.x_grad ? static_cast<T*>(a.x_grad) + row * a.x_grad_stride : nullptr;
        S* const gr = a.residual_grad ? static_cast<S*>(a.residual_grad) + row * a.residual_grad_stride : nullptr;
        const float2 st = *reinterpret_cast<const float2*>(a.stats + row * kNormStats);
        const NormFactor f{st.x, st.y};
        const auto each = [&](auto go) {
            if (kWide) {
                for (int32_t i = tid * kNormChunk; i < H; i += kStep) go(i, 0);
            } else {
#pragma unroll
                for (int j = 0; j < CHUNKS; ++j) {
                    const int32_t i = j * kStep + tid * kNormChunk;
                    if (i < H) go(i, j);
                }
            }
        };
        const auto load = [&](int32_t i, int j) {
            load_some(h, i, H, n[j]);
            load_some(gy, i, H, g[j]);
#pragma unroll
            for (int e = 0; e < 8; ++e) n[j][e] = f.of(n[j][e]);
            if (kWide) load_weight<T>(a.weight, a.weight_type, i, H, w[j]);
        };
        if (!kWide) each(load);
        RowSum<kWide> sum = 0;
        each([&](int32_t i, int j) {
            if (kWide) load(i, j);
            float t = kWide ? 0.0f : (float)sum;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float gn = g[j][e] * n[j][e];
                if (kWide) sums[0][e] = gn;
                else if (i + e < H) sums[j][e] += gn;
                t = __builtin_fmaf(gn, i + e < H ? w[j][e] : 0.0f, t);
            }
            sum = kWide ? sum + t : t;
            if (kWide && partial) {
                float before[8];
                if (!fresh) load_some(partial, i, H, before);
#pragma unroll
                for (int e = 0; e < 8; ++e) before[e] = fresh ? sums[0][e] : before[e] + sums[0][e];
                store_some(partial, i, H, before);
            }
        });
        fresh = false;
        if (!gx && !gr) continue;
        const float along = (float)block_sum<BLOCK>(sum, part) / (float)H;
        each([&](int32_t i, int j) {
            if (kWide) load(i, j);
            float b[8];
            if (gh) load_some(gh, i, H, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = ((g[j][e] * w[j][e] - n[j][e] * along) * f.second) * f.first;
                b[e] = gh ? b[e] + d : d;
            }
            if (gx) store_some(gx, i, H, b);
            if (gr) store_some(gr, i, H, b);
        });
    }
    if (!kWide && partial) {
#pragma unroll
        for (int j = 0; j < kHeld; ++j) {
            const int32_t i = j * kStep + tid * kNormChunk;
            if (i < H) store_some(partial, i, H, sums[j]);
        }
    }
}

// The weight's gradient: a column's partial sums, by kWeightLanes threads in order.
constexpr int kWeightBlock = 64, kWeightLanes = 16;
template <class W>
__global__ __launch_bounds__(kWeightBlock * kWeightLanes) void norm_weight_grad_kernel(NormGradArgs a)
{
    __shared__ float part[kWeightLanes][kWeightBlock];
    const int32_t column = a.column0 + (int32_t)(blockIdx.x * kWeightBlock + threadIdx.x % kWeightBlock), q = threadIdx.x / kWeightBlock;
    float s = 0.0f;
    if (column < a.H) {
#pragma unroll 8
        for (int32_t i = q; i < a.groups; i += kWeightLanes) s += a.partial[(int64_t)i * a.H + column];
    }
    part[q][threadIdx.x % kWeightBlock] = s;
    __syncthreads();
    if (q != 0 || column >= a.H) return;
#pragma unroll
    for (int i = 1; i < kWeightLanes; ++i) s += part[i][threadIdx.x];
    static_cast<W*>(a.weight_grad)[column] = Row<W>::from(s);
}

static int check_norm(const lda_norm_rows* d, const char* call)
{
    if (!d) return fail(nullptr, LDA_ERR_ARG, "%s: NULL rows", call);
    for (int32_t r : d->reserved)
        if (r != 0) return fail(nullptr, LDA_ERR_ARG, "%s: reserved fields must be zero", call);
    if (d->reserved_word != 0) return fail(nullptr, LDA_ERR_ARG, "%s: reserved fields must be zero", call);
    if (d->rows < 0 || d->width < 1) return fail(nullptr, LDA_ERR_ARG, "%s: rows >= 0 and width >= 1 needed", call);
    if (d->width > 1 << 30) return fail(nullptr, LDA_ERR_UNSUPPORTED, "%s: at most 2^30 numbers a row", call);
    if (!known_type(d->x_type) || !known_type(d->sum_type) || !known_type(d->weight_type))
        return fail(nullptr, LDA_ERR_ARG, "%s: unknown type", call);
    if (d->sum_type != d->x_type && d->sum_type != LDA_F32)
        return fail(nullptr, LDA_ERR_ARG, "%s: the sum has x's type or 32 bits", call);
    if (d->weight_type != d->x_type && d->weight_type != LDA_F32)
        return fail(nullptr, LDA_ERR_ARG, "%s: the weight has x's type or 32 bits", call);
    if (!(d->eps >= 0.0f) || !(d->eps <= 3.0e38f))
        return fail(nullptr, LDA_ERR_ARG, "%s: eps must be finite and not negative", call);
    if (!aligned_to(d->weight, type_bytes(d->weight_type)))
        return fail(nullptr, LDA_ERR_ARG, "%s: a pointer is not aligned to its type", call);
    return LDA_OK;
}

// Threads and chunks of a thread that hold a row, 0 chunks: a row too wide for registers; and how many workgroups share
// the rows of a gradient (each has its partial sum of the weight's).  8192 x 1024 bf16: 10.6 us by 64 threads of two
// chunks, 13.6 by 256 of one; x 4096: 38.8 by 512, 40.4 by 256 of two, 46 by 1024.  Gradients, of a bf16 residual too, of 65536 x 512: 60 us by 2048
// workgroups, 174 by 512 (without a residual 43 by 2048); of 8192 x 8192: 104 by 512, 110 by 1024; of 8192 x 4096 with a float32 sum and the partial sums' own
// pass: 105 by 512, 111 by 1024.
struct NormShape {
    int block, chunks, groups;
};
static NormShape norm_shape(int32_t H)
{
    static constexpr NormShape kShapes[] = {{64, 1, 2048}, {64, 2, 2048}, {256, 1, 1024}, {512, 1, 512}, {512, 2, 512}, {1024, 2, 512}};
    for (const NormShape& s : kShapes)
        if (H <= s.block * s.chunks * kNormChunk) return s;
    return {1024, 0, 512};
}

template <class F>
static void with_shape(NormShape s, F f)
{
    using std::integral_constant;
    const auto one = integral_constant<int, 1>{};
    const auto two = integral_constant<int, 2>{};
    if (s.block == 64 && s.chunks == 1) f(integral_constant<int, 64>{}, one);
    else if (s.block == 64) f(integral_constant<int, 64>{}, two);
    else if (s.block == 256) f(integral_constant<int, 256>{}, one);
    else if (s.block == 512 && s.chunks == 1) f(integral_constant<int, 512>{}, one);
    else if (s.block == 512) f(integral_constant<int, 512>{}, two);
    else if (s.chunks == 2) f(integral_constant<int, 1024>{}, two);
    else f(integral_constant<int, 1024>{}, integral_constant<int, 0>{});
}
template <class F>
static void with_types(int32_t x, int32_t sum, F f)
{
    if (x == LDA_F32) f(float{}, float{});
    else if (x == LDA_F16 && sum == LDA_F32) f(__half{}, float{});
    else if (x == LDA_F16) f(__half{}, __half{});
    else if (sum == LDA_F32) f(__hip_bfloat16{}, float{});
    else f(__hip_bfloat16{}, __hip_bfloat16{});
}

// levels: -1 for y in x's type, else LDA_INT8 or LDA_E4M3
static int launch_norm(const lda_norm_rows* d, const char* call, int32_t levels, void* out, int64_t out_stride, float* scale,
                       void* sum, int64_t sum_stride, float* stats)
{
    if (d->rows == 0) return LDA_OK;
    if (!d->x || !out || (d->residual && !sum)) return fail(nullptr, LDA_ERR_ARG, "%s: NULL pointer", call);
    const size_t xb = type_bytes(d->x_type), sb = type_bytes(d->sum_type);
    if (!aligned_to(d->x, xb) || !aligned_to(d->residual, sb) || !aligned_to(sum, sb) || !aligned_to(scale, 4) ||
        !aligned_to(stats, 8) || !aligned_to(out, levels < 0 ? xb : 1))
        return fail(nullptr, LDA_ERR_ARG, "%s: a pointer is not aligned to its type", call);
    if (d->rows > 1 && (out_stride < d->width || (d->residual && sum_stride < d->width)))
        return fail(nullptr, LDA_ERR_ARG, "%s: rows of an output overlap", call);
    NormArgs a{};
    a.rows = d->rows;
    a.H = d->width;
    a.x = d->x;
    a.x_stride = d->x_stride;
    a.residual = d->residual;
    a.residual_stride = d->residual_stride;
    a.weight = d->weight;
    a.weight_type = d->weight_type;
    a.eps = d->eps;
    a.out = out;
    a.out_stride = out_stride;
    a.sum = sum;
    a.sum_stride = sum_stride;
    a.scale = scale;
    a.stats = stats;
    const hipStream_t stream = static_cast<hipStream_t>(d->hip_stream);
    with_types(d->x_type, d->sum_type, [&](auto t, auto s) {
        with_shape(norm_shape(a.H), [&](auto block, auto chunks) {
            using T = decltype(t);
            using S = decltype(s);
            for (a.row0 = 0; a.row0 < a.rows; a.row0 += 1 << 20) {
                const unsigned n = (unsigned)(a.rows - a.row0 < (1 << 20) ? a.rows - a.row0 : 1 << 20);
                if (levels < 0) norm_kernel<T, S, T, block(), chunks()><<<n, block(), 0, stream>>>(a);
                else if (levels == LDA_INT8) norm_kernel<T, S, int8_t, block(), chunks()><<<n, block(), 0, stream>>>(a);
                else norm_kernel<T, S, E4m3, block(), chunks()><<<n, block(), 0, stream>>>(a);
            }
        });
    });
    LDA_HIP(static_cast<lda_ctx*>(nullptr), hipGetLastError());
    return LDA_OK;
}

static int32_t grad_groups(const lda_norm_rows* d)
{
    const int32_t most = norm_shape(d->width).groups;
    return (int32_t)(d->rows < most ? d->rows : most);
}

}  // namespace lda

using namespace lda;

extern "C" {

int lda_norm(const lda_norm_rows* d, void* y, int64_t y_stride, void* sum, int64_t sum_stride, float* stats)
try {
    const int rc = check_norm(d, "lda_norm");
    if (rc != LDA_OK) return rc;
    return launch_norm(d, "lda_norm", -1, y, y_stride, nullptr, sum, sum_stride, stats);
} catch (...) {
    return LDA_ERR_OOM;
}

int lda_norm_bytes(const lda_norm_rows* d, int32_t levels, void* out, int64_t out_stride, float* scale, void* sum,
                   int64_t sum_stride)
try {
    const int rc = check_norm(d, "lda_norm_bytes");
    if (rc != LDA_OK) return rc;
    if (levels != LDA_INT8 && levels != LDA_E4M3) return fail(nullptr, LDA_ERR_ARG, "lda_norm_bytes: unknown type");
    if (d->rows > 0 && !scale) return fail(nullptr, LDA_ERR_ARG, "lda_norm_bytes: NULL scale");
    return launch_norm(d, "lda_norm_bytes", levels, out, out_stride, scale, sum, sum_stride, nullptr);
} catch (...) {
    return LDA_ERR_OOM;
}

int64_t lda_norm_grad_workspace(const lda_norm_rows* d)
try {
    const int rc = check_norm(d, "lda_norm_grad_workspace");
    if (rc != LDA_OK) return rc;
    return (int64_t)grad_groups(d) * d->width * (int64_t)sizeof(float);
} catch (...) {
    return LDA_ERR_OOM;
}

int lda_norm_grad(const lda_norm_rows* d, const lda_norm_gradients* g)
try {
    const int rc = check_norm(d, "lda_norm_grad");
    if (rc != LDA_OK) return rc;
    if (!g) return fail(nullptr, LDA_ERR_ARG, "lda_norm_grad: NULL gradients");
    for (int32_t r : g->reserved)
        if (r != 0) return fail(nullptr, LDA_ERR_ARG, "lda_norm_grad: reserved fields must be zero");
    const size_t xb = type_bytes(d->x_type), sb = type_bytes(d->sum_type);
    const bool with_weight = g->weight_grad != nullptr;
    if (!aligned_to(g->weight_grad, type_bytes(d->weight_type)))
        return fail(nullptr, LDA_ERR_ARG, "lda_norm_grad: a pointer is not aligned to its type");
    if (d->rows == 0 && !with_weight) return LDA_OK;
    const void* h = d->residual ? g->sum : d->x;
    if (d->rows > 0) {
        if (!h || !g->stats || !g->y_grad) return fail(nullptr, LDA_ERR_ARG, "lda_norm_grad: NULL pointer");
        if (!aligned_to(h, d->residual ? sb : xb) || !aligned_to(g->y_grad, xb) || !aligned_to(g->sum_grad, sb) ||
            !aligned_to(g->stats, 8) || !aligned_to(g->x_grad, xb) || !aligned_to(g->residual_grad, sb))
            return fail(nullptr, LDA_ERR_ARG, "lda_norm_grad: a pointer is not aligned to its type");
        if (d->rows > 1 && ((g->x_grad && g->x_grad_stride < d->width) || (g->residual_grad && g->residual_grad_stride < d->width)))
            return fail(nullptr, LDA_ERR_ARG, "lda_norm_grad: rows of an output overlap");
    }
    NormGradArgs a{};
    a.rows = d->rows;
    a.H = d->width;
    a.h = h;
    a.h_stride = d->residual ? g->sum_stride : d->x_stride;
    a.weight = d->weight;
    a.weight_type = d->weight_type;
    a.stats = g->stats;
    a.y_grad = g->y_grad;
    a.y_grad_stride = g->y_grad_stride;
    a.sum_grad = g->sum_grad;
    a.sum_grad_stride = g->sum_grad_stride;
    a.x_grad = g->x_grad;
    a.x_grad_stride = g->x_grad_stride;
    a.residual_grad = g->residual_grad;
    a.residual_grad_stride = g->residual_grad_stride;
    a.weight_grad = g->weight_grad;
    a.groups = grad_groups(d);
    if (with_weight && d->rows > 0) {
        const int64_t need = (int64_t)a.groups * a.H * (int64_t)sizeof(float);
        if (!g->workspace || g->workspace_bytes < need || !aligned_to(g->workspace, 16))
            return fail(nullptr, LDA_ERR_ARG, "lda_norm_grad: needs a workspace of %lld bytes, aligned to 16", (long long)need);
        a.partial = static_cast<float*>(g->workspace);
    }
    const hipStream_t stream = static_cast<hipStream_t>(d->hip_stream);
    // without a residual the sum is x
    with_types(d->x_type, d->residual ? d->sum_type : d->x_type, [&](auto t, auto s) {
        using T = decltype(t);
        using S = decltype(s);
        if (a.rows > 0 && (a.x_grad || a.residual_grad || a.partial))
            with_shape(norm_shape(a.H), [&](auto block, auto chunks) {
                // without sums of the weight's a workgroup a row would do as well
                norm_grad_kernel<T, S, block(), chunks()><<<a.groups, block(), 0, stream>>>(a);
            });
        if (!with_weight) return;
        constexpr int32_t kMost = 1 << 20;  // a launch has less than 2^32 threads
        for (; a.column0 < a.H; a.column0 += kMost * kWeightBlock) {
            const int32_t left = (a.H - a.column0 + kWeightBlock - 1) / kWeightBlock;
            const unsigned n = (unsigned)(left < kMost ? left : kMost);
            if (d->weight_type == LDA_F32) norm_weight_grad_kernel<float><<<n, kWeightBlock * kWeightLanes, 0, stream>>>(a);
            else norm_weight_grad_kernel<T><<<n, kWeightBlock * kWeightLanes, 0, stream>>>(a);
        }
    });
    LDA_HIP(static_cast<lda_ctx*>(nullptr), hipGetLastError());
    return LDA_OK;
} catch (...) {
    return LDA_ERR_OOM;
}

}  // extern "C"
