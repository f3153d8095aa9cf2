// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and the gradient of the
// first two (the formulas stand at lda_log_prob_rows in lda_mi355x.h).
//
// One pass: a thread keeps a base m, s = sum e^y and u = sum y e^y with y = (S - m) / T of what it has seen, the
// entropy is log s - u / s.  The largest go along: what exceeds a bound under which the k-th largest cannot lie is
// put on a list in LDS, and the bound rises when the list is cut to its k largest.  Elements are compared as one
// number each, the logit's place in the order of numbers above the class's complement, so that no two are equal and
// ties need no care.  Rows are cut into slices where there are few; the slices' sums and lists join.
#include <type_traits>

#include "softmax_rows.hpp"

namespace lda {

constexpr int32_t kMostTop = 256;
constexpr int kScanBlock = 256;
constexpr int kScanLoads = 4;  // 16-byte loads of a thread in flight
constexpr int32_t kBatch = kScanBlock * kScanLoads;
constexpr int32_t kJoinList = 4096, kJoinEach = 4;
constexpr int32_t kGradLoads = 8;
constexpr int32_t kGradSlice = kScanBlock * kGradLoads;
constexpr int32_t kLogProbStats = 4;
// The base is left where it is until a logit exceeds it by this, in powers of 2: the entropy is a difference
// of numbers that grow with it
constexpr float kRise = 2.0f;
constexpr float kFloorY = -1.0e4f;  // powers of 2: none is left of e^y, and y e^y is 0 and not a NaN

typedef unsigned long long u64;

// Where k are wanted so many do as well: a bound among them is found by the first bits that differ, nearly always
__host__ __device__ constexpr int32_t enough(int32_t k) { return k + (k / 4 > 8 ? k / 4 : 8); }

struct LogProbArgs {
    int64_t rows, row0;
    int32_t V, k;
    const void* logits;
    int64_t logits_stride;
    const void* tokens;
    int64_t tokens_stride;
    int32_t tokens_type;
    float T, c;  // c = log2(e) / T
    int32_t slices, slice_chunks, room;  // room: of a list in LDS
    struct LogProbPart* parts;  // [rows][slices]
    u64* lists;                 // [rows][slices][enough(k)]
    float* log_prob;
    float* entropy;
    int32_t* ids;
    float* top;
    float* stats;
};

struct LogProbPart {
    float m, s, u;  // u in powers of 2
    int32_t n;      // of the list
};

struct LogProbGradArgs {
    int64_t rows, row0;
    int32_t V;
    const void* logits;
    int64_t logits_stride;
    const void* tokens;
    int64_t tokens_stride;
    int32_t tokens_type;
    float T, c;
    const float* stats;
    const float* log_prob_grad;
    int64_t log_prob_grad_stride;
    const float* entropy_grad;
    int64_t entropy_grad_stride;
    void* grad;
    int64_t grad_stride;
    int32_t slices;  // of kGradSlice chunks each
};

// A row's sums, of a thread's share or joined
struct Sums {
    float m, s, u;

    static __device__ __forceinline__ Sums none() { return Sums{-INFINITY, 0.0f, 0.0f}; }
    template <int N>
    __device__ __forceinline__ float add(const float (&x)[N], float c)  // returns the largest
    {
        float top = x[0];
#pragma unroll
        for (int e = 1; e < N; ++e) top = fmaxf(top, x[e]);
        if ((top - m) * c > kRise) move(top, c);
        const float base = base_of(m);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float y = (x[e] - base) * c, p = __builtin_amdgcn_exp2f(y);
            s += p;
            u = __builtin_fmaf(fmaxf(y, kFloorY), p, u);
        }
        return top;
    }
    __device__ __forceinline__ void move(float to, float c)
    {
        const float d = fmaxf((m - base_of(to)) * c, kFloorY), f = __builtin_amdgcn_exp2f(d);
        u = f * __builtin_fmaf(d, s, u);
        s *= f;
        m = to;
    }
    __device__ __forceinline__ void wave_join(float c)
    {
        move(wave_max(m), c);
        s = wave_sum(s);
        u = wave_sum(u);
    }
    __device__ __forceinline__ void join(Sums o, float c)
    {
        const float to = fmaxf(m, o.m);
        move(to, c);
        o.move(to, c);
        s += o.s;
        u += o.u;
    }
    template <int BLOCK>
    __device__ __forceinline__ void block_join(float c, Sums* part)
    {
        wave_join(c);
        __syncthreads();
        if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = *this;
        __syncthreads();
        *this = part[0];
#pragma unroll
        for (int w = 1; w < BLOCK / kWave; ++w) join(part[w], c);
    }
};

// Logits in the order of numbers, -0 as 0, the lower class first; 0 is none
__device__ __forceinline__ u64 place_of(float x, int32_t id)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    const uint32_t order = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return (u64)order << 32 | (uint32_t)~id;
}
__device__ __forceinline__ int32_t id_of(u64 place) { return (int32_t)~(uint32_t)place; }
__device__ __forceinline__ float logit_of(u64 place)
{
    const uint32_t order = (uint32_t)(place >> 32);
    return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order);
}

struct ListLds {
    int32_t histogram[256];
    int32_t count, chosen;
    uint32_t high[16], low[16];
    int32_t number[16];
    u64 best[enough(kMostTop)];
};

__device__ __forceinline__ uint32_t wave_most(uint32_t v)
{
    return (uint32_t)lane_value((int32_t)wave_scan(v, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; }), kWave - 1);
}

// A bound that at least k and at most enough(k) of the workgroup's numbers reach, which each(f) gives to f; 1 where there
// are fewer.  By 8 bits at a time from the first on that is not the same in all.  (Bits that are the same in all would
// put every number into one bin, one after the other.)
template <int BLOCK, class Each>
__device__ __forceinline__ u64 bound_of(Each each, int32_t k, ListLds& l)
{
    constexpr int kWaves = BLOCK / kWave;
    const int32_t tid = (int32_t)threadIdx.x, lane = tid % kWave;
    uint32_t high = 0, low = 0;  // of the upper halves; the least as its complement
    int32_t number = 0;
    each([&](u64 key) {
        if (key == 0) return;
        high = max(high, (uint32_t)(key >> 32));
        low = max(low, ~(uint32_t)(key >> 32));
        ++number;
    });
    high = wave_most(high);
    low = wave_most(low);
    number = wave_sum(number);
    if (lane == 0) {
        l.high[tid / kWave] = high;
        l.low[tid / kWave] = low;
        l.number[tid / kWave] = number;
    }
    for (int32_t i = tid; i < 256; i += BLOCK) l.histogram[i] = 0;
    __syncthreads();
    high = l.high[0];
    low = l.low[0];
    number = l.number[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        high = max(high, l.high[w]);
        low = max(low, l.low[w]);
        number += l.number[w];
    }
    const int32_t most = enough(k);
    if (number <= most) {
        __syncthreads();
        return 1;
    }
    int32_t taken = 0;  // above the prefix
    const uint32_t differ = high ^ ~low;
    int32_t bits = differ == 0 ? 32 : 64 - __builtin_clz(differ);  // the lowest ones, that differ
    u64 prefix = bits == 64 ? 0 : ((u64)high << 32) >> bits;
    for (;;) {
        const int32_t shift = max(bits - 8, 0);
        each([&](u64 key) {
            if (key != 0 && (bits == 64 || key >> bits == prefix))
                atomicAdd(&l.histogram[(uint32_t)(key >> shift) & ((1u << (bits - shift)) - 1u)], 1);
        });
        __syncthreads();
        // every wave for itself: a lane has four bins, the highest first
        int32_t n[4], mine = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) mine += n[q] = l.histogram[255 - (4 * lane + q)];
        const int32_t upto = wave_prefix(mine);
        int32_t digit = 0, above = taken + upto - mine;
        bool found = false;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (!found) {
                digit = 255 - (4 * lane + q);
                above += n[q];
                found = above >= k;
                if (found) mine = n[q];
            }
        }
        const int32_t at = __builtin_ctzll(__ballot(found));
        digit = lane_value(digit, at);
        above = lane_value(above, at);
        taken = above - lane_value(mine, at);
        prefix = prefix << (bits - shift) | (uint32_t)digit;
        bits = shift;
        __syncthreads();
        if (above <= most || bits == 0) return prefix << bits;
        for (int32_t i = tid; i < 256; i += BLOCK) l.histogram[i] = 0;
        __syncthreads();
    }
}

// The list's entries of at least `bound`, at most enough(k), to l.best; their number in every thread
template <int BLOCK>
__device__ __forceinline__ int32_t choose(const u64* list, int32_t n, u64 bound, ListLds& l)
{
    if (threadIdx.x == 0) l.chosen = 0;
    __syncthreads();
    for (int32_t i = (int32_t)threadIdx.x; i < n; i += BLOCK) {
        const u64 key = list[i];
        if (key >= bound) l.best[atomicAdd(&l.chosen, 1)] = key;
    }
    __syncthreads();
    return l.chosen;
}

// Cuts the list to enough(k) of its largest, which then are in l.best too; returns bound_of()'s
template <int BLOCK>
__device__ __forceinline__ u64 cut(u64* list, int32_t n, int32_t k, ListLds& l)
{
    const u64 bound = bound_of<BLOCK>([&](auto f) {
        for (int32_t i = (int32_t)threadIdx.x; i < n; i += BLOCK) f(list[i]);
    }, k, l);
    const int32_t some = choose<BLOCK>(list, n, bound, l);
    for (int32_t i = (int32_t)threadIdx.x; i < some; i += BLOCK) list[i] = l.best[i];
    if (threadIdx.x == 0) l.count = some;
    __syncthreads();
    return bound;
}

// What the next numbers have to exceed where `least` ones of at least that are there
__device__ __forceinline__ u64 raised(u64 bound, u64 least) { return least > bound + 1 ? least - 1 : bound; }

// What a row's sums say; the largest are in l.best
template <int BLOCK, bool TOP>
__device__ __forceinline__ void finish_row(const LogProbArgs& a, int64_t row, const Sums& sum, int32_t n, ListLds& l, float x,
                                           bool given)
{
    const double inv_t = 1.0 / (double)a.T, m = (double)base_of(sum.m), log_s = log((double)sum.s);
    const bool none = !(sum.s == sum.s);
    if (threadIdx.x == 0) {
        float h = sum.s == 0.0f ? 0.0f : (float)(log_s - (double)sum.u * 0.693147180559945309417 / (double)sum.s);
        float lp = 0.0f;
        if (given) lp = none ? NAN : sum.s == 0.0f ? -INFINITY : (float)(((double)x - m) * inv_t - log_s);
        a.log_prob[row] = lp;
        if (h < 0.0f) h = 0.0f;
        if (a.entropy) a.entropy[row] = h;
        if (a.stats) *reinterpret_cast<float4*>(a.stats + row * kLogProbStats) = make_float4(sum.m, sum.s, h, 0.0f);
    }
    if (!TOP) return;
    for (int32_t i = (int32_t)threadIdx.x; i < max(a.k, n); i += BLOCK) {
        int32_t at = i, id = -1;
        float top = none ? NAN : -INFINITY;
        if (i < n) {
            const u64 key = l.best[i];
            at = 0;
#pragma unroll 8
            for (int32_t j = 0; j < n; ++j) at += l.best[j] > key;
            if (at >= a.k) continue;
            if (!none) {
                id = id_of(key);
                top = (float)(((double)logit_of(key) - m) * inv_t - log_s);
            }
        }
        a.ids[row * a.k + at] = id;
        a.top[row * a.k + at] = top;
    }
}

template <class T>
__device__ __forceinline__ bool given_token(const LogProbArgs& a, int64_t row, float& x)
{
    x = 0.0f;
    if (threadIdx.x != 0) return false;
    const int64_t t = index_at(a.tokens, a.tokens_type, row * a.tokens_stride);
    if (t < 0 || t >= a.V) return false;
    x = Row<T>::one(static_cast<const T*>(a.logits) + row * a.logits_stride + t);
    return true;
}

// A slice of a row a workgroup.  The first batch gives a bound from its chunks' largest; the others are read without
// a barrier, each thread puts down what exceeds the bound, which rises each time as much again has been read: of a row in
// no order some k more come each time.  Where more came than there is room for (a row that rises) they are gone through
// again, the bound raised from batch to batch.  Without alternatives bound by memory, 48 x 10^6 float32 30 us, or as much by
// its 10 vector instructions an element, 2048 x 141043 bf16 152 us (3.8 TB/s); 2048 x 101636 fp16 with the top 64
// 110 us (82 without), 64 x 141043 bf16 with the top 20 in 18 slices each 13.7.
template <class T, bool TOP>
__global__ __launch_bounds__(kScanBlock) void log_probs_kernel(LogProbArgs a)
{
    constexpr int E = Row<T>::kChunk;
    extern __shared__ __align__(16) u64 list[];
    __shared__ Sums part[kScanBlock / kWave];
    __shared__ ListLds l;
    const int32_t tid = (int32_t)threadIdx.x, slice = (int32_t)blockIdx.y;
    const int64_t row = a.row0 + blockIdx.x;
    const SplitRow<T> r(static_cast<const T*>(a.logits) + row * a.logits_stride, a.V);
    const int32_t first = slice * a.slice_chunks, last = min(r.whole, first + a.slice_chunks);
    const bool has_extra = slice == 0 && tid < r.extras;
    const float extra[1] = {has_extra ? Row<T>::one(r.p + r.extra(tid)) : -INFINITY};
    float token_x = 0.0f;
    const bool given = a.slices == 1 && given_token<T>(a, row, token_x);
    Sums sum = Sums::none();
    if (has_extra) sum.add(extra, a.c);
    u64 bound = place_of(-INFINITY, 0);
    float bound_x = logit_of(bound + 1);  // what exceeds the bound is at least this, and above -infinity
    float tops[kScanLoads];               // the largest of a batch's chunks
    const auto put_one = [&](float x, int32_t id, u64 least, float least_x) {
        if (!(x >= least_x)) return;
        const u64 key = place_of(x, id);
        if (key < least) return;
        const int32_t n = atomicAdd(&l.count, 1);
        if (n < a.room) list[n] = key;
    };
    // Takes a batch: into the sums, if `sums`, and onto the list, if `puts`, each element that exceeds the bound
    const auto take = [&](int32_t at, auto sums, auto puts) {
        uint4 raw[kScanLoads];
#pragma unroll
        for (int j = 0; j < kScanLoads; ++j) {
            const int32_t i = at + j * kScanBlock + tid;
            if (i < last) raw[j] = r.load(i);
        }
#pragma unroll
        for (int j = 0; j < kScanLoads; ++j) {
            const int32_t i = at + j * kScanBlock + tid;
            tops[j] = -INFINITY;
            if (i >= last) continue;
            float x[E];
            Row<T>::unpack(raw[j], x);
            if (sums()) {
                tops[j] = sum.add(x, a.c);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) tops[j] = fmaxf(tops[j], x[e]);
            }
            if (puts() && tops[j] >= bound_x) {
#pragma unroll
                for (int e = 0; e < E; ++e) put_one(x[e], r.chunk(i) + e, bound + 1, bound_x);
            }
        }
    };
    // Puts down what a batch that has been taken has of at least `least`, read again: rare, and the chunks' registers
    // are worth more to others
    const auto put = [&](int32_t at, u64 least) {
        const float least_x = logit_of(least);
        uint32_t some = 0;
#pragma unroll
        for (int j = 0; j < kScanLoads; ++j) some |= tops[j] >= least_x ? 1u << j : 0u;
        while (some != 0) {
            const int32_t i = at + __builtin_ctz(some) * kScanBlock + tid;
            some &= some - 1;
            float x[E];
            Row<T>::unpack(r.load(i), x);
#pragma unroll
            for (int e = 0; e < E; ++e) put_one(x[e], r.chunk(i) + e, least, least_x);
        }
    };
    // What a batch's elements have to be at least, from the batch alone: a bound of its chunks' largest, of those that
    // exceed the bound.  A chunk's largest counts as the last element of its chunk, which it is at least.  At least k elements
    // reach it, or all do that exceed the bound; and the chunks that have some are enough(k) at most, and two that end beyond
    // the bound or the new one and have equal ones before.
    const auto least_of = [&](int32_t at) {
        u64 keys[kScanLoads];
#pragma unroll
        for (int j = 0; j < kScanLoads; ++j) {
            keys[j] = 0;
            if (!(tops[j] >= bound_x)) continue;
            const u64 key = place_of(tops[j], r.chunk(at + j * kScanBlock + tid) + E - 1);
            if (key > bound) keys[j] = key;
        }
        const u64 least = bound_of<kScanBlock>([&](auto f) {
#pragma unroll
            for (int j = 0; j < kScanLoads; ++j) f(keys[j]);
        }, a.k, l);
        return least > bound ? least : bound + 1;
    };
    int32_t n = 0;
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    if constexpr (!TOP) {
        for (int32_t at = first; at < last; at += kBatch) take(at, yes, no);
    } else {
        if (tid == 0) l.count = 0;
        take(first, yes, no);
        if ((int64_t)(last - first + 2) * E > a.room) {  // (with the elements beside the chunks)
            bound = raised(bound, least_of(first));
            bound_x = logit_of(bound + 1);
        } else {
            __syncthreads();
        }
        put(first, bound + 1);
        if (has_extra) put_one(extra[0], r.extra(tid), bound + 1, bound_x);
        if (last - first > kBatch) {
            __syncthreads();
            int32_t kept = l.count, safe = first + kBatch, at = safe;  // the list at `safe`
            __syncthreads();
            for (int32_t until = kBatch;; until *= 2) {  // as many again as there were
                const int32_t end = until < last - at ? at + until : last;
                for (; at < end; at += kBatch) take(at, yes, yes);
                __syncthreads();
                n = l.count;
                __syncthreads();
                if (at >= last || n > a.room) break;
                if (n >= 2 * enough(a.k)) {
                    bound = raised(bound, cut<kScanBlock>(list, n, a.k, l));
                    bound_x = logit_of(bound + 1);
                    n = l.count;
                    __syncthreads();  // every wave has read it before a fast one puts the next on the list
                }
                kept = n;
                safe = at;
            }
            if (n > a.room) {
                if (tid == 0) l.count = kept;
                for (int32_t b = safe; b < last; b += kBatch) {
                    __syncthreads();
                    n = l.count;
                    if (n > a.room - E * (enough(a.k) + 2)) {
                        __syncthreads();
                        bound = raised(bound, cut<kScanBlock>(list, n, a.k, l));
                        bound_x = logit_of(bound + 1);
                    }
                    if (b >= at) take(b, yes, no);
                    else take(b, no, no);  // the sums have these
                    put(b, least_of(b));
                }
            }
        }
        __syncthreads();
        n = l.count;
        __syncthreads();
        if (n > enough(a.k)) {
            cut<kScanBlock>(list, n, a.k, l);
            n = l.count;
        } else {
            choose<kScanBlock>(list, n, 0, l);
        }
    }
    sum.block_join<kScanBlock>(a.c, part);
    if (a.slices == 1) {
        finish_row<kScanBlock, TOP>(a, row, sum, n, l, token_x, given);
        return;
    }
    const int64_t at = row * a.slices + slice;
    if (tid == 0) a.parts[at] = LogProbPart{sum.m, sum.s, sum.u, n};
    if (TOP)
        for (int32_t i = tid; i < n; i += kScanBlock) a.lists[at * enough(a.k) + i] = l.best[i];
}

// A row's slices joined, a workgroup a row: 4 to 6 us of latency
template <class T, bool TOP>
__global__ __launch_bounds__(kScanBlock) void log_probs_join_kernel(LogProbArgs a)
{
    __shared__ u64 list[TOP ? kJoinList : 1];
    __shared__ Sums part[kScanBlock / kWave];
    __shared__ ListLds l;
    const int32_t tid = (int32_t)threadIdx.x;
    const int64_t row = a.row0 + blockIdx.x;
    const LogProbPart* const parts = a.parts + row * a.slices;
    float token_x;
    const bool given = given_token<T>(a, row, token_x);
    Sums sum = Sums::none();
    for (int32_t i = tid; i < a.slices; i += kScanBlock) {
        sum.join(Sums{parts[i].m, parts[i].s, parts[i].u}, a.c);
    }
    int32_t n = 0;
    if constexpr (TOP) {
        if (tid == 0) l.count = 0;
        __syncthreads();
        u64 bound = 0;
        const int32_t each = enough(a.k), total = a.slices * each;
        const u64* const lists = a.lists + row * total;
        for (int32_t at = 0; at < total; at += kScanBlock * kJoinEach) {
            u64 key[kJoinEach];
#pragma unroll
            for (int j = 0; j < kJoinEach; ++j) {
                const int32_t i = at + j * kScanBlock + tid;
                key[j] = 0;
                if (i < total && i % each < parts[i / each].n) key[j] = lists[i];
            }
#pragma unroll
            for (int j = 0; j < kJoinEach; ++j)
                if (key[j] > bound) list[atomicAdd(&l.count, 1)] = key[j];
            __syncthreads();
            n = l.count;
            __syncthreads();
            if (n > kJoinList - kScanBlock * kJoinEach) {
                bound = raised(bound, cut<kScanBlock>(list, n, a.k, l));
                n = l.count;
                __syncthreads();
            }
        }
        if (n > enough(a.k)) {
            cut<kScanBlock>(list, n, a.k, l);
            n = l.count;
        } else {
            choose<kScanBlock>(list, n, 0, l);
        }
    }
    sum.block_join<kScanBlock>(a.c, part);
    finish_row<kScanBlock, TOP>(a, row, sum, n, l, token_x, given);
}

// A slice of a row's gradient a workgroup.  With e = 2^y it is e (A + B y), and 1 / T times the token's own weight
// more at the token.  Bound by memory: 2048 x 141043 bf16 214 us, 5.4 TB/s of read and written bytes.
template <class T>
__global__ __launch_bounds__(kScanBlock) void log_probs_grad_kernel(LogProbGradArgs a)
{
    constexpr int E = Row<T>::kChunk;
    const int32_t tid = (int32_t)threadIdx.x;
    const int64_t row = a.row0 + blockIdx.x;
    const SplitRow<T> r(static_cast<const T*>(a.logits) + row * a.logits_stride, a.V);
    T* const g = static_cast<T*>(a.grad) + row * a.grad_stride;
    const int64_t token = index_at(a.tokens, a.tokens_type, row * a.tokens_stride);
    const bool given = token >= 0 && token < a.V;
    const float lg = given && a.log_prob_grad ? a.log_prob_grad[row * a.log_prob_grad_stride] : 0.0f;
    const float hg = a.entropy_grad ? a.entropy_grad[row * a.entropy_grad_stride] : 0.0f;
    const float4 st = *reinterpret_cast<const float4*>(a.stats + row * kLogProbStats);
    const bool out = (lg == 0.0f && hg == 0.0f) || st.y == 0.0f;
    const float base = base_of(st.x), share = -1.0f / (st.y * a.T);
    const float A = share * (lg + hg * (st.z - logf(st.y))), B = share * (hg * 0.69314718056f);
    const auto dense = [&](float x) {
        const float y = (x - base) * a.c, e = __builtin_amdgcn_exp2f(y);
        return e * __builtin_fmaf(B, fmaxf(y, kFloorY), A);
    };
    for (int32_t slice = (int32_t)blockIdx.y; slice < a.slices; slice += (int32_t)gridDim.y) {
        const int32_t i0 = slice * kGradSlice + tid;
        uint4 raw[kGradLoads];
        if (!out) {
#pragma unroll
            for (int j = 0; j < kGradLoads; ++j)
                if (i0 + j * kScanBlock < r.whole) raw[j] = r.load(i0 + j * kScanBlock);
        }
        if (slice == 0 && tid < r.extras) {
            const int32_t v = r.extra(tid);
            g[v] = Row<T>::from(out ? 0.0f : dense(Row<T>::one(r.p + v)));
        }
#pragma unroll
        for (int j = 0; j < kGradLoads; ++j) {
            const int32_t i = i0 + j * kScanBlock;
            if (i >= r.whole) continue;
            float x[E];
            Row<T>::unpack(raw[j], x);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = out ? 0.0f : dense(x[e]);
            store_chunk(g + r.chunk(i), x);
        }
        if (out || lg == 0.0f) continue;
        const int32_t v0 = r.chunk(min(r.whole, slice * kGradSlice)), v1 = r.chunk(min(r.whole, (slice + 1) * kGradSlice));
        if (!((token >= v0 && token < v1) || (slice == 0 && (token < r.head || token >= r.chunk(r.whole))))) continue;
        __syncthreads();  // the token's place is written again, by another thread
        if (tid == 0) g[token] = Row<T>::from(dense(Row<T>::one(r.p + token)) + lg / a.T);
    }
}

static int check_log_probs(const lda_log_prob_rows* d, const char* call)
{
    if (!d) return fail(nullptr, LDA_ERR_ARG, "%s: NULL rows", call);
    for (int32_t r : d->reserved)
        if (r != 0) return fail(nullptr, LDA_ERR_ARG, "%s: reserved fields must be zero", call);
    if (d->reserved_word != 0) return fail(nullptr, LDA_ERR_ARG, "%s: reserved fields must be zero", call);
    if (d->rows < 0 || d->classes < 1 || d->top < 0)
        return fail(nullptr, LDA_ERR_ARG, "%s: rows >= 0, classes >= 1, top >= 0 needed", call);
    if (!known_type(d->logits_type) || !known_index(d->tokens_type))
        return fail(nullptr, LDA_ERR_ARG, "%s: unknown type", call);
    if (!(d->temperature >= 1.0f / 1024.0f) || !(d->temperature <= 1024.0f))
        return fail(nullptr, LDA_ERR_ARG, "%s: temperature must lie in [1/1024, 1024]", call);
    if (d->top > kMostTop) return fail(nullptr, LDA_ERR_UNSUPPORTED, "%s: at most %d alternatives", call, kMostTop);
    if (d->rows == 0) return LDA_OK;
    if (!d->logits || !d->tokens) return fail(nullptr, LDA_ERR_ARG, "%s: NULL pointer", call);
    if (!aligned_to(d->logits, type_bytes(d->logits_type)) || !aligned_to(d->tokens, index_bytes(d->tokens_type)))
        return fail(nullptr, LDA_ERR_ARG, "%s: a pointer is not aligned to its type", call);
    return LDA_OK;
}

// Slices of a row: enough workgroups to fill the GPU (1024; 2048 rows of 101636 take 103 us whole, 128 in two slices), each a
// chunk of every thread at least, or whole batches (64 rows of 141043 with the top 20: 21 us by slices of two batches, 19
// of one)
struct Slices {
    int32_t count, chunks;
};
static Slices slices_of(const lda_log_prob_rows* d)
{
    const int64_t whole = (int64_t)d->classes / (16 / (int64_t)type_bytes(d->logits_type)) + 1;
    const int64_t wanted = d->rows >= 1024 ? 1 : 1024 / (d->rows < 1 ? 1 : d->rows);
    const int64_t most = (whole + kScanBlock - 1) / kScanBlock;
    int64_t count = wanted < most ? wanted : most;
    if (count == 1) return {1, (int32_t)whole};
    int64_t chunks = (whole + count - 1) / count;
    chunks = chunks > kBatch ? (chunks + kBatch / 2) / kBatch * kBatch : (chunks + kScanBlock - 1) / kScanBlock * kScanBlock;
    count = (whole + chunks - 1) / chunks;
    return {(int32_t)count, (int32_t)chunks};
}

static int64_t log_prob_bytes(const lda_log_prob_rows* d)
{
    const int64_t count = slices_of(d).count;
    if (d->rows == 0 || count == 1) return 0;
    return d->rows * count * ((int64_t)sizeof(LogProbPart) + (d->top > 0 ? enough(d->top) : 0) * (int64_t)sizeof(u64));
}

}  // namespace lda

using namespace lda;

extern "C" {

int64_t lda_log_probs_workspace(const lda_log_prob_rows* d)
try {
    const int rc = check_log_probs(d, "lda_log_probs_workspace");
    if (rc != LDA_OK) return rc;
    return log_prob_bytes(d);
} catch (...) {
    return LDA_ERR_OOM;
}

int lda_log_probs(const lda_log_prob_rows* d, float* log_prob, float* entropy, int32_t* ids, float* top, float* stats)
try {
    const int rc = check_log_probs(d, "lda_log_probs");
    if (rc != LDA_OK) return rc;
    if (d->rows == 0) return LDA_OK;
    if (!log_prob || (d->top > 0 && (!ids || !top))) return fail(nullptr, LDA_ERR_ARG, "lda_log_probs: NULL pointer");
    if (!aligned_to(log_prob, 4) || !aligned_to(entropy, 4) || !aligned_to(ids, 4) || !aligned_to(top, 4) || !aligned_to(stats, 16))
        return fail(nullptr, LDA_ERR_ARG, "lda_log_probs: an output is not aligned to its type, or stats to 16 bytes");
    const int64_t need = log_prob_bytes(d);
    if (need > 0 && (!d->workspace || d->workspace_bytes < need || !aligned_to(d->workspace, 16)))
        return fail(nullptr, LDA_ERR_ARG, "lda_log_probs: needs a workspace of %lld bytes, aligned to 16", (long long)need);
    const Slices slices = slices_of(d);
    LogProbArgs a{};
    a.rows = d->rows;
    a.V = d->classes;
    a.k = d->top;
    a.logits = d->logits;
    a.logits_stride = d->logits_stride;
    a.tokens = d->tokens;
    a.tokens_stride = d->tokens_stride;
    a.tokens_type = d->tokens_type;
    a.T = d->temperature;
    a.c = (float)(1.44269504088896340736 / (double)d->temperature);
    a.slices = slices.count;
    a.slice_chunks = slices.chunks;
    a.log_prob = log_prob;
    a.entropy = entropy;
    a.ids = ids;
    a.top = top;
    a.stats = stats;
    if (need > 0) {
        a.parts = static_cast<LogProbPart*>(d->workspace);
        a.lists = reinterpret_cast<u64*>(a.parts + d->rows * slices.count);
    }
    const hipStream_t stream = static_cast<hipStream_t>(d->hip_stream);
    const auto typed = [&](auto t) {
        using T = decltype(t);
        // what a cut leaves, what a batch may bring behind it, and some hundreds between two cuts
        a.room = enough(a.k) + Row<T>::kChunk * (enough(a.k) + 2) + 768;
        const size_t lds = a.k > 0 ? (size_t)a.room * sizeof(u64) : 0;
        for (a.row0 = 0; a.row0 < a.rows; a.row0 += 1 << 20) {
            const unsigned n = (unsigned)(a.rows - a.row0 < (1 << 20) ? a.rows - a.row0 : 1 << 20);
            const dim3 grid(n, (unsigned)a.slices);
            if (a.k > 0) log_probs_kernel<T, true><<<grid, kScanBlock, lds, stream>>>(a);
            else log_probs_kernel<T, false><<<grid, kScanBlock, 0, stream>>>(a);
            if (a.slices == 1) continue;
            if (a.k > 0) log_probs_join_kernel<T, true><<<n, kScanBlock, 0, stream>>>(a);
            else log_probs_join_kernel<T, false><<<n, kScanBlock, 0, stream>>>(a);
        }
    };
    if (d->logits_type == LDA_F32) typed(float{});
    else if (d->logits_type == LDA_F16) typed(__half{});
    else typed(__hip_bfloat16{});
    LDA_HIP(static_cast<lda_ctx*>(nullptr), hipGetLastError());
    return LDA_OK;
} catch (...) {
    return LDA_ERR_OOM;
}

int lda_log_probs_grad(const lda_log_prob_rows* d, const float* stats, const float* log_prob_grad, int64_t log_prob_grad_stride,
                       const float* entropy_grad, int64_t entropy_grad_stride, void* grad, int64_t grad_stride)
try {
    const int rc = check_log_probs(d, "lda_log_probs_grad");
    if (rc != LDA_OK) return rc;
    if (d->rows == 0) return LDA_OK;
    if (!stats || !grad) return fail(nullptr, LDA_ERR_ARG, "lda_log_probs_grad: NULL pointer");
    if (!aligned_to(stats, 16) || !aligned_to(log_prob_grad, 4) || !aligned_to(entropy_grad, 4) ||
        !aligned_to(grad, type_bytes(d->logits_type)))
        return fail(nullptr, LDA_ERR_ARG, "lda_log_probs_grad: a pointer is not aligned to its type, or stats to 16 bytes");
    if (d->rows > 1 && grad_stride < d->classes)
        return fail(nullptr, LDA_ERR_ARG, "lda_log_probs_grad: rows of the gradient overlap");
    LogProbGradArgs a{};
    a.rows = d->rows;
    a.V = d->classes;
    a.logits = d->logits;
    a.logits_stride = d->logits_stride;
    a.tokens = d->tokens;
    a.tokens_stride = d->tokens_stride;
    a.tokens_type = d->tokens_type;
    a.T = d->temperature;
    a.c = (float)(1.44269504088896340736 / (double)d->temperature);
    a.stats = stats;
    a.log_prob_grad = log_prob_grad;
    a.log_prob_grad_stride = log_prob_grad_stride;
    a.entropy_grad = entropy_grad;
    a.entropy_grad_stride = entropy_grad_stride;
    a.grad = grad;
    a.grad_stride = grad_stride;
    const hipStream_t stream = static_cast<hipStream_t>(d->hip_stream);
    const auto typed = [&](auto t) {
        using T = decltype(t);
        const int64_t whole = (int64_t)a.V / Row<T>::kChunk + 1;
        a.slices = (int32_t)((whole + kGradSlice - 1) / kGradSlice);
        const unsigned slices = (unsigned)(a.slices < 32768 ? a.slices : 32768);
        for (a.row0 = 0; a.row0 < a.rows; a.row0 += 1 << 20) {
            const unsigned n = (unsigned)(a.rows - a.row0 < (1 << 20) ? a.rows - a.row0 : 1 << 20);
            log_probs_grad_kernel<T><<<dim3(n, slices), kScanBlock, 0, stream>>>(a);
        }
    };
    if (d->logits_type == LDA_F32) typed(float{});
    else if (d->logits_type == LDA_F16) typed(__half{});
    else typed(__hip_bfloat16{});
    LDA_HIP(static_cast<lda_ctx*>(nullptr), hipGetLastError());
    return LDA_OK;
} catch (...) {
    return LDA_ERR_OOM;
}

}  // extern "C"
