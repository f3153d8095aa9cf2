// Top topics of documents: teacher rows out of an assignment (lda_topic_rows in lda_mi355x.h).
//
// A topic with its count is one key, the count above the inverted topic: all keys of a document
// differ, larger keys come first in the output, and "the k largest" is one set.  What is done a document
// depends on its length and its number of topics alone, which the host does not know:
//   a wave, with a table of counts in LDS, takes documents of up to kWaveTokens tokens and kWaveTopics
//     topics (all that have at most so many tokens, and most of the others);
//   a workgroup of 1024 takes the rest, with a counter a topic in LDS, a range of topics at a time, and
//     the best k chosen by histograms of the counts; or with a table, which holds up to kTableTopics topics
//     whatever K is.
//   Of the longest documents every range is a workgroup's, and their best are put together afterwards, where
//     the caller has given a workspace for that.
// The first kernel leaves marks in the rows that the others have to take.
#include <algorithm>

#include "rows.hpp"

namespace lda {

constexpr int32_t kMostTopSlots = 1024;
constexpr uint32_t kInverted = (1u << kMixTopicBits) - 1u;  // a key's topic is kInverted - (key & kInverted)
constexpr int32_t kUnfinished = -2;      // in a row's first id, between the kernels
constexpr int32_t kSplit = -3;           // the same; kSplit - i: place i of the workspace has its ranges

constexpr int kWaveBlock = 256;          // four documents at a time
constexpr int32_t kWaveTopics = 512;     // the table has twice as many slots
constexpr int32_t kWaveTokens = 4095;    // the count of a 32-bit key has 12 bits
constexpr int kLongBlock = 1024;
constexpr int32_t kTableSlots = 12288, kTableTopics = 8192;
constexpr int32_t kLongWords = 31;       // words of counters in LDS, a thread at most
// Where a document's topics take several ranges, a table is the faster one up to so many tokens a range:
// it takes some 15 us and 2.8 us per 1000 tokens whatever K is (8000 topics among 40 000 tokens), a
// range of counters some 30 us and 0.2 us per 1000 tokens.
constexpr int32_t kTableTokens = 4096;
constexpr int32_t kNarrowRange = 2 * kLongWords * kLongBlock;  // topics with 16-bit counters
constexpr int32_t kWideRange = kLongWords * kLongBlock;
constexpr int32_t kWideTokens = 65536;   // from here on 32-bit counters
constexpr int32_t kSplitTokens = 16384;  // shorter documents are not split
constexpr int64_t kSplitBytes = 64 << 20;  // of workspace at most
constexpr int32_t kDigit = 10;           // bits of a key that a histogram takes at a time

struct TopicArgs {
    int64_t rows;
    const int32_t* docs;
    int64_t documents;
    const void* offsets;
    int32_t offsets_type;
    int32_t K;
    const int32_t* z;
    const int32_t* const* z_now;  // NULL, or where z is instead, if anywhere: work that a graph replays
    int64_t tokens;
    int32_t k;
    double alpha;
    int32_t* ids;
    float* logits;
    float* log_norm;
    // documents that are split: how many, their rows; per document and range (topics, tokens) and the keys
    int32_t wide_places, places, ranges;
    int32_t* n_split;        // [2] of kWideTokens or more, which take the first wide_places: they begin first; of less
    int64_t* split_rows;     // [places]
    int2* split_n;           // [places][ranges]
    uint64_t* split_keys;    // [places][ranges][k]
};

__host__ __device__ __forceinline__ int32_t ranges_of(int32_t K, int64_t L)
{
    const int32_t range = L < kWideTokens ? kNarrowRange : kWideRange;
    return (K + range - 1) / range;
}
__device__ __forceinline__ const int32_t* assignment(const TopicArgs& a)
{
    const int32_t* const z = a.z_now ? *a.z_now : nullptr;
    return z ? z : a.z;
}

// Split where a workgroup would take long: where 32-bit counters are needed, or a few ranges (where there
// are more, a table is the better one).
__device__ __forceinline__ bool split_document(const TopicArgs& a, int64_t L)
{
    if (a.places == 0 || L < kSplitTokens) return false;
    return L >= kWideTokens ? a.ranges > 1 : (ranges_of(a.K, L) > 1 && ranges_of(a.K, L) <= 4);
}

__device__ __forceinline__ void document_of(const TopicArgs& a, int64_t row, int64_t& g0, int64_t& g1)
{
    const int64_t d = a.docs ? (int64_t)a.docs[row] : row;
    g0 = g1 = 0;
    if (d < 0 || d >= a.documents) return;
    g0 = min(max(index_at(a.offsets, a.offsets_type, d), (int64_t)0), a.tokens);
    g1 = min(max(index_at(a.offsets, a.offsets_type, d + 1), g0), a.tokens);
    g1 = min(g1, g0 + INT32_MAX);
}

constexpr int kAhead = 4;  // rounds of 64 tokens that are read ahead
__device__ __forceinline__ void first_tokens(const int32_t* z, int32_t L, int32_t (&next)[kAhead])
{
    const int32_t lane = (int32_t)threadIdx.x % kWave;
#pragma unroll
    for (int e = 0; e < kAhead; ++e) next[e] = e * kWave + lane < L ? z[e * kWave + lane] : -1;
}

// One document's counts in a table of 2 kWaveTopics keys (0: empty), and its best k topics, by one wave.
// `used` has room for kWaveTopics slots; the table is empty before and after.  A key has the topic, inverted
// within the bits that K takes, below the count.  `next` holds the document's first tokens; all_read()
// is called when they are read, for the next document's to be on their way while this one's topics are chosen.
// Returns the number of tokens counted, -1 if there are too many topics.
template <class Read, class LogCount>
__device__ __forceinline__ int32_t topics_by_wave(const TopicArgs& a, int64_t row, const int32_t* z, int32_t L, int32_t (&next)[kAhead],
                                                  uint32_t* table, uint16_t* used, Read all_read, LogCount log_count)
{
    const uint32_t bits = 32u - (uint32_t)__builtin_clz((uint32_t)a.K);
    const uint32_t inverted = (1u << bits) - 1u, one = 1u << bits;
    constexpr int32_t kSlots = 2 * kWaveTopics, kEach = kWaveTopics / kWave;
    const int32_t lane = (int32_t)threadIdx.x % kWave;
    int32_t n = 0, counted = 0;
    bool many = false;
    for (int32_t i0 = 0; i0 < L && !many; i0 += kAhead * kWave) {
        int32_t topic[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const int32_t i = i0 + (kAhead + e) * kWave + lane;
            topic[e] = next[e];
            next[e] = i < L ? z[i] : -1;
        }
        // the rounds' look-ups side by side: one after the other they would wait for LDS each
        int32_t mine[kAhead];
        if (a.K <= kSlots) {  // a slot a topic: no search
            uint32_t was[kAhead];
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
                const bool open = (uint32_t)topic[e] < (uint32_t)a.K;
                counted += (int32_t)__popcll(__ballot(open));
                was[e] = open ? atomicAdd(&table[topic[e]], one) : 1u;
            }
#pragma unroll
            for (int e = 0; e < kAhead; ++e) mine[e] = was[e] == 0 ? topic[e] : -1;
        } else {
            int32_t h[kAhead];  // -1: found
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
                const bool open = (uint32_t)topic[e] < (uint32_t)a.K;
                counted += (int32_t)__popcll(__ballot(open));
                h[e] = open ? (int32_t)(((uint32_t)topic[e] * 0x9E3779B1u) >> (32 - __builtin_ctz(kSlots))) : -1;
                mine[e] = -1;
            }
            // half the slots stay empty: every search ends
            while (__ballot(max(max(h[0], h[1]), max(h[2], h[3])) >= 0)) {
                uint32_t v[kAhead];
#pragma unroll
                for (int e = 0; e < kAhead; ++e) v[e] = table[max(h[e], 0)];
#pragma unroll
                for (int e = 0; e < kAhead; ++e)
                    if (h[e] >= 0 && v[e] == 0) {
                        v[e] = atomicCAS(&table[h[e]], 0u, one | (inverted - (uint32_t)topic[e]));
                        if (v[e] == 0) {
                            mine[e] = h[e];
                            h[e] = -1;
                        }
                    }
#pragma unroll
                for (int e = 0; e < kAhead; ++e)
                    if (h[e] >= 0) {
                        if ((v[e] & inverted) == inverted - (uint32_t)topic[e]) {
                            atomicAdd(&table[h[e]], one);
                            h[e] = -1;
                        } else {
                            h[e] = (h[e] + 1) & (kSlots - 1);
                        }
                    }
            }
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const uint64_t fresh = __ballot(mine[e] >= 0);
            if (mine[e] >= 0)
                used[n + (int32_t)__builtin_amdgcn_mbcnt_hi((uint32_t)(fresh >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)fresh, 0u))] =
                    (uint16_t)mine[e];
            n += (int32_t)__popcll(fresh);
        }
        many = n + min(kAhead * kWave, L - i0 - kAhead * kWave) > kWaveTopics;
    }
    all_read();
    wave_lds_order();
    // the keys, into registers; the table is cleared behind them
    uint32_t key[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int32_t i = e * kWave + lane;
        key[e] = 0;
        if (e * kWave < n && i < n) {
            const uint32_t h = used[i];
            key[e] = table[h];
            if (a.K <= kSlots) key[e] |= inverted - h;
            table[h] = 0;
        }
    }
    if (many) {
        wave_lds_order();
        return -1;
    }
    int32_t n_best = n;
    uint32_t least = 1;
    if (n > kWave && n > a.k) {
        // too many to rank them all: a border below which lie all but k, bit by bit
        least = 0;
        uint32_t step = one << (31 - __builtin_clz((uint32_t)L));
        if (n <= 2 * kWave) {  // most documents
            for (; step != 0; step >>= 1) {
                const uint32_t at = least | step;
                const int32_t above = (int32_t)__popcll(__ballot(key[0] >= at)) + (int32_t)__popcll(__ballot(key[1] >= at));
                least = above >= a.k ? at : least;
            }
        } else {
            for (; step != 0; step >>= 1) {
                const uint32_t at = least | step;
                int32_t above = 0;
#pragma unroll
                for (int e = 0; e < kEach; ++e) above += (int32_t)__popcll(__ballot(key[e] >= at));
                least = above >= a.k ? at : least;
            }
        }
        n_best = a.k;
    }
    // those side by side, in the table's room
    wave_lds_order();
    uint32_t* keys = table;
    int32_t at = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        if (e * kWave >= n) continue;
        const bool in = key[e] >= least;
        const uint64_t some = __ballot(in);
        if (in) keys[at + (int32_t)__builtin_amdgcn_mbcnt_hi((uint32_t)(some >> 32),
                                                             __builtin_amdgcn_mbcnt_lo((uint32_t)some, 0u))] = key[e];
        at += (int32_t)__popcll(some);
    }
    wave_lds_order();
    // (what lies behind them, up to a whole vector, is 0: no key is smaller)
    const uint4* four = reinterpret_cast<const uint4*>(keys);
    int32_t* const ids = a.ids + row * a.k;
    float* const logits = a.logits + row * a.k;
    for (int32_t i = lane; i < n_best; i += kWave) {
        const uint32_t own = keys[i];
        int32_t place = 0;
        for (int32_t j = 0; j < (n_best + 3) / 4; ++j) {
            const uint4 v = four[j];
            place += (v.x > own) + (v.y > own) + (v.z > own) + (v.w > own);
        }
        if (place < a.k) {
            ids[place] = (int32_t)(inverted - (own & inverted));
            logits[place] = log_count((int32_t)(own >> bits));
        }
    }
    for (int32_t i = n_best + lane; i < a.k; i += kWave) {
        ids[i] = -1;
        logits[i] = -INFINITY;
    }
    wave_lds_order();
    for (int32_t i = lane; i < n_best; i += kWave) keys[i] = 0;
    wave_lds_order();
    return counted;
}

// Bound by the number of instructions: 300 000 documents of 330 tokens in 1000 topics, 32 slots, take 370 us (1.3 TB/s of
// z and outputs), some 320 vector and 500 scalar instructions a document, more than one in every issue
// slot of the SIMDs.  (Ranking all keys instead of finding a border first, 530 vector and 440 scalar, was 3 % slower.)
// 100 000 documents of 100 tokens in 10 000 topics: 98 us.
__global__ __launch_bounds__(kWaveBlock, 6) void wave_topics_kernel(TopicArgs a)
{
    constexpr int kWaves = kWaveBlock / kWave;
    a.z = assignment(a);
    __shared__ __align__(16) uint32_t table[kWaves][2 * kWaveTopics];
    __shared__ uint16_t used[kWaves][kWaveTopics];
    __shared__ float log_of[kWaveTopics + 1], norm_of[kWaveTopics + 1];  // of count + alpha, of tokens + K alpha
    const int32_t tid = (int32_t)threadIdx.x, lane = tid % kWave;
    const int32_t wave = __builtin_amdgcn_readfirstlane(tid / kWave);  // what is a wave's is scalar
    for (int32_t i = tid; i < kWaves * 2 * kWaveTopics; i += kWaveBlock) (&table[0][0])[i] = 0;
    const double k_alpha = (double)a.K * a.alpha;
    // the logarithms are tabled only where a wave has more than two documents, where both meet. Documents of 90
    // tokens, with the tables and without: 6 000 16.1 and 13.8 us, 12 000 20.0 and 19.8, 16 000 21.4 and 22.4,
    // 300 000 205 and 276; of 330 tokens, 300 000: 367 and 426
    const bool logs = a.rows > 2 * (int64_t)gridDim.x * kWaves;
    for (int32_t i = tid; logs && i <= kWaveTopics; i += kWaveBlock) {
        log_of[i] = (float)log((double)i + a.alpha);
        norm_of[i] = (float)log((double)i + k_alpha);
    }
    __syncthreads();
    const int64_t step = (int64_t)gridDim.x * kWaves;
    int64_t row = (int64_t)blockIdx.x * kWaves + wave, g0 = 0, g1 = 0;
    int32_t next[kAhead];
    const auto tokens = [&]() { return g1 - g0 > kWaveTokens ? 0 : (int32_t)(g1 - g0); };
    if (row < a.rows) document_of(a, row, g0, g1);
    first_tokens(a.z + g0, tokens(), next);
    for (; row < a.rows; row += step) {
        const int32_t L = tokens();
        const int64_t length = g1 - g0;
        const bool longer = length > kWaveTokens;
        const int32_t* const z = a.z + g0;
        g0 = g1 = 0;
        if (row + step < a.rows) document_of(a, row + step, g0, g1);
        const auto read_next = [&]() { first_tokens(a.z + g0, tokens(), next); };
        if (longer) {
            if (lane == 0) {
                int32_t mark = kUnfinished;
                if (split_document(a, length)) {
                    const bool wide = length >= kWideTokens;
                    const int32_t place = (wide ? 0 : a.wide_places) + atomicAdd(&a.n_split[wide ? 0 : 1], 1);
                    if (place < (wide ? a.wide_places : a.places)) {
                        a.split_rows[place] = row;
                        mark = kSplit - place;
                    }
                }
                a.ids[row * a.k] = mark;
            }
            read_next();
            continue;
        }
        const int32_t counted = topics_by_wave(a, row, z, L, next, table[wave], used[wave], read_next, [&](int32_t n) {
            return logs && n <= kWaveTopics ? log_of[n] : (float)log((double)n + a.alpha);
        });
        if (lane != 0) continue;
        if (counted < 0) a.ids[row * a.k] = kUnfinished;
        else if (a.log_norm) a.log_norm[row] = logs && counted <= kWaveTopics ? norm_of[counted] : (float)log((double)counted + k_alpha);
    }
}

// The rows of this workgroup that the waves left: every gridDim.x-th row is this workgroup's, BLOCK of
// them are looked at together.  f(row, g0, L) is called for one after the other.
template <int BLOCK, class F>
__device__ __forceinline__ void for_rows_left(const TopicArgs& a, int32_t* mine, int32_t* n_mine, F f)
{
    for (int64_t r0 = blockIdx.x; r0 < a.rows; r0 += (int64_t)gridDim.x * BLOCK) {
        __syncthreads();
        if (threadIdx.x == 0) *n_mine = 0;
        __syncthreads();
        const int64_t row = r0 + (int64_t)threadIdx.x * gridDim.x;
        if (row < a.rows) {
            int64_t g0, g1;
            document_of(a, row, g0, g1);
            if (g1 - g0 > kWaveTokens || (g1 - g0 > kWaveTopics && a.ids[row * a.k] == kUnfinished)) mine[atomicAdd(n_mine, 1)] = (int32_t)threadIdx.x;
        }
        __syncthreads();
        const int32_t n = *n_mine;
        for (int32_t i = 0; i < n; ++i) {
            const int64_t at = r0 + (int64_t)mine[i] * gridDim.x;
            int64_t g0, g1;
            document_of(a, at, g0, g1);
            f(at, g0, (int32_t)(g1 - g0));
        }
    }
}

__device__ __forceinline__ uint64_t long_key(uint32_t count, int32_t topic)
{
    return ((uint64_t)count << kMixTopicBits) | (uint64_t)(kInverted - (uint32_t)topic);
}

// Exclusive prefix sum over the workgroup; total: of all threads
template <int BLOCK>
__device__ __forceinline__ int32_t block_prefix(int32_t v, int32_t* part, int32_t& total)
{
    const int32_t lane = (int32_t)threadIdx.x % kWave, wave = (int32_t)threadIdx.x / kWave;
    const int32_t sum = wave_prefix(v);
    __syncthreads();
    if (lane == kWave - 1) part[wave] = sum;
    __syncthreads();
    int32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < BLOCK / kWave; ++w) {
        before += w < wave ? part[w] : 0;
        total += part[w];
    }
    return before + sum - v;
}

struct TableLds {
    uint32_t topic[kTableSlots];  // kInverted: empty
    uint32_t count[kTableSlots];
    uint16_t used[kTableTopics];
};
struct LongLds {
    union {
        TableLds table;
        uint32_t count[kLongWords * kLongBlock];
    };
    uint64_t keys[2 * kMostTopSlots];  // the best so far, and the range's behind them
    uint64_t best[kMostTopSlots];
    uint32_t histogram[1 << kDigit];
    int32_t mine[kLongBlock];
    int32_t part[kLongBlock / kWave];
    int32_t n_mine, n_keys, n_used, digit, over;
};
static_assert(sizeof(LongLds) <= 160 * 1024, "LDS of a CU");

// After a histogram: the digit where the `need`-th largest value lies, `need` less the values of larger
// digits; all: the values there are (fewer than need: digit -1).
__device__ __forceinline__ int32_t find_digit(LongLds& lds, int32_t& need, int32_t& all)
{
    const int32_t tid = (int32_t)threadIdx.x;
    if (tid == 0) lds.digit = -1;
    __syncthreads();
    const int32_t d = (1 << kDigit) - 1 - tid;
    const int32_t here = (int32_t)lds.histogram[d];
    const int32_t above = block_prefix<kLongBlock>(here, lds.part, all);
    if (above < need && above + here >= need) {
        lds.digit = d;
        lds.over = above;
    }
    __syncthreads();
    const int32_t digit = lds.digit;
    if (digit >= 0) need -= lds.over;
    return digit;
}
static_assert(1 << kDigit == kLongBlock, "a thread a digit");

__device__ __forceinline__ void clear_histogram(LongLds& lds)
{
    __syncthreads();
    lds.histogram[threadIdx.x] = 0;
    __syncthreads();
}

// The `need`-th largest of the workgroup's values (all below 2^most_bits, need of them or more), and
// how many values equal to it are among the `need` largest.  each(f) calls f(value) for the thread's own.
template <class Each>
__device__ __forceinline__ uint32_t nth_largest(LongLds& lds, int32_t most_bits, int32_t& need, Each each)
{
    int32_t shift = max(0, most_bits - kDigit), bits = most_bits - shift, all;
    uint32_t prefix = 0;
    bool first = true;
    for (;;) {
        clear_histogram(lds);
        each([&](uint32_t v) {
            if (first || (v >> (shift + bits)) == prefix) atomicAdd(&lds.histogram[(v >> shift) & ((1u << bits) - 1u)], 1u);
        });
        prefix = (prefix << bits) | (uint32_t)find_digit(lds, need, all);
        if (shift == 0) return prefix;
        first = false;
        bits = min(shift, kDigit);
        shift -= bits;
    }
}

// The n keys in order of size, the best k of them to `best`.  A key's place is the number of larger ones,
// which some threads of a wave count together where there are few keys.
__device__ __forceinline__ void order_keys(const uint64_t* keys, int32_t n, int32_t k, uint64_t* best)
{
    int32_t together = 1;
    while (together < kWave && 2 * together * n <= kLongBlock) together *= 2;
    const int32_t q = (int32_t)threadIdx.x % together;
    for (int32_t i = (int32_t)threadIdx.x / together; i < n; i += kLongBlock / together) {
        const uint64_t key = keys[i];
        int32_t place = 0;
#pragma unroll 4
        for (int32_t j = q; j < n; j += together) place += keys[j] > key;
        for (int32_t d = together / 2; d > 0; d /= 2) place += __shfl_xor(place, d, kWave);
        if (q == 0 && place < k) best[place] = key;
    }
    __syncthreads();
}

__device__ __forceinline__ void write_keys(const TopicArgs& a, int64_t row, const uint64_t* best, int32_t n, int32_t counted)
{
    for (int32_t i = (int32_t)threadIdx.x; i < a.k; i += kLongBlock) {
        const uint64_t key = i < n ? best[i] : 0;
        a.ids[row * a.k + i] = i < n ? (int32_t)(kInverted - (uint32_t)(key & kInverted)) : -1;
        a.logits[row * a.k + i] = i < n ? (float)log((double)(key >> kMixTopicBits) + a.alpha) : -INFINITY;
    }
    if (threadIdx.x == 0 && a.log_norm) a.log_norm[row] = (float)log((double)counted + (double)a.K * a.alpha);
}

// A document's few frequent topics would have their lanes wait for each other at one counter in every
// round.  A wave counts those that stand out among its first tokens in scalar registers.
struct HotTopics {
    static constexpr int kHot = 2;
    int32_t topic[kHot], tokens[kHot];
    __device__ __forceinline__ HotTopics(int32_t t, bool open)
    {
        uint64_t left = __ballot(open);
#pragma unroll
        for (int q = 0; q < kHot; ++q) {
            topic[q] = -1;
            tokens[q] = 0;
            for (int tries = 0; tries < 4 && left; ++tries) {
                const int32_t own = __builtin_amdgcn_readlane(t, (int)__builtin_ctzll(left));
                const uint64_t same = __ballot(t == own);
                left &= ~same;
                if (__popcll(same) < 4) continue;
                topic[q] = own;
                break;
            }
        }
    }
    // what is left to count of a round's tokens
    __device__ __forceinline__ bool left(int32_t t, bool open)
    {
#pragma unroll
        for (int q = 0; q < kHot; ++q) {
            const uint64_t same = __ballot(open && t == topic[q]);
            tokens[q] += (int32_t)__popcll(same);
            open = open && t != topic[q];
        }
        return open;
    }
};

// Counts in buckets that keep their order: one each below 64, then 32 for every power of two
__device__ __forceinline__ uint32_t bucket_of(uint32_t c)
{
    if (c < 64) return c;
    const uint32_t e = 31 - (uint32_t)__builtin_clz(c);
    return 64 + ((e - 6) << 5) + ((c >> (e - 5)) & 31u);
}

// The k-th largest count (0: there are no more than k), into `ties` how many of the topics that have it
// are among the best k, into `equal` how many of them this thread has.  each(f) calls f(count) for the
// thread's share; first(few, f) the same for counts above 3 only, and counts those of 1, 2 and 3.
template <class First, class Each>
__device__ __forceinline__ uint32_t least_count(LongLds& lds, int32_t k, int32_t& ties, int32_t& equal, First first, Each each)
{
    // most topics have a few tokens: their buckets would be everybody's
    int32_t few[3] = {0, 0, 0};
    clear_histogram(lds);
    first(few, [&](uint32_t c) { atomicAdd(&lds.histogram[bucket_of(c)], 1u); });
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        const int32_t n = wave_sum(few[q]);
        if (threadIdx.x % kWave == 0 && n > 0) atomicAdd(&lds.histogram[q + 1], (uint32_t)n);
    }
    int32_t all;
    ties = k;
    const int32_t bucket = find_digit(lds, ties, all);
    equal = 0;
    if (all <= k) return 0;
    uint32_t least = (uint32_t)bucket;
    if (bucket >= 64) {
        const int32_t bits = ((bucket - 64) >> 5) + 1;  // of a count that its bucket leaves open
        const uint32_t low = (32u + ((uint32_t)bucket & 31u)) << bits;
        least = low + nth_largest(lds, bits, ties, [&](auto f) {
                    each([&](uint32_t c) {
                        if (c - low < 1u << bits) f(c - low);
                    });
                });
    }
    if (least <= 3) equal = least == 1 ? few[0] : least == 2 ? few[1] : few[2];
    else each([&](uint32_t c) { equal += c == least; });
    return least;
}

// The document's counts in a table; false, and nothing written, if it has too many topics for one
__device__ __forceinline__ bool topics_by_table(const TopicArgs& a, int64_t row, int64_t g0, int32_t L, LongLds& lds)
{
    constexpr int kLoads = 8;
    const int32_t tid = (int32_t)threadIdx.x, lane = tid % kWave;
    const uint64_t below = (1ull << lane) - 1;
    TableLds& table = lds.table;
    __syncthreads();
    for (int32_t i = tid; i < kTableSlots; i += kLongBlock) {
        table.topic[i] = kInverted;
        table.count[i] = 0;
    }
    if (tid == 0) lds.n_used = 0;
    __syncthreads();
    int32_t counted = 0;
    int32_t next[kLoads];
#pragma unroll
    for (int e = 0; e < kLoads; ++e) next[e] = e * kLongBlock + tid < L ? a.z[g0 + e * kLongBlock + tid] : -1;
    HotTopics hot(next[0], next[0] >= 0 && next[0] < a.K);
    // n tokens of topic t, where open
    const auto insert = [&](int32_t t, uint32_t tokens, bool open) {
        uint32_t h = __umulhi((uint32_t)t * 0x9E3779B1u, (uint32_t)kTableSlots);
        bool full = false;
        while (__ballot(open)) {
            bool mine = false;
            if (open) {
                uint32_t v = table.topic[h];
                if (v == kInverted) {
                    v = atomicCAS(&table.topic[h], kInverted, (uint32_t)t);
                    mine = v == kInverted;
                }
                if (mine || v == (uint32_t)t) {
                    atomicAdd(&table.count[h], tokens);
                    open = false;
                } else {
                    h = h + 1 == (uint32_t)kTableSlots ? 0 : h + 1;
                }
            }
            const uint64_t fresh = __ballot(mine);
            if (fresh) {
                int32_t at = 0;
                if (lane == 0) at = atomicAdd(&lds.n_used, (int32_t)__popcll(fresh));
                at = __builtin_amdgcn_readfirstlane(at);
                const int32_t own = at + (int32_t)__popcll(fresh & below);
                if (mine && own < kTableTopics) table.used[own] = (uint16_t)h;
                // given up: a wave takes 64 slots at most after that
                full = at + (int32_t)__popcll(fresh) > kTableTopics;
                if (full) break;
            }
        }
        return full;
    };
    bool full = false;
    for (int64_t i0 = 0; i0 < L && !full; i0 += kLoads * kLongBlock) {
        int32_t topic[kLoads];
#pragma unroll
        for (int e = 0; e < kLoads; ++e) {
            const int64_t i = i0 + (e + kLoads) * kLongBlock + tid;
            topic[e] = next[e];
            next[e] = i < L ? a.z[g0 + i] : -1;
        }
#pragma unroll
        for (int e = 0; e < kLoads; ++e) {
            const int32_t t = topic[e];
            if (i0 + e * kLongBlock >= L || full) break;
            const bool open = t >= 0 && t < a.K;
            counted += open;
            full = insert(t, 1u, hot.left(t, open));
        }
    }
#pragma unroll
    for (int q = 0; q < HotTopics::kHot; ++q)
        if (hot.tokens[q] > 0) full = insert(hot.topic[q], (uint32_t)hot.tokens[q], lane == 0) || full;
    counted = block_sum<kLongBlock>(counted, lds.part);
    const int32_t n = lds.n_used;
    if (n > kTableTopics) return false;
    const auto each = [&](auto f) {
        for (int32_t i = tid; i < n; i += kLongBlock) {
            const uint32_t h = table.used[i];
            f(table.count[h], table.topic[h]);
        }
    };
    int32_t ties, equal;
    const uint32_t least = least_count(
        lds, a.k, ties, equal,
        [&](int32_t(&few)[3], auto f) {
            each([&](uint32_t c, uint32_t) {
                few[0] += c == 1;
                few[1] += c == 2;
                few[2] += c == 3;
                if (c > 3) f(c);
            });
        },
        [&](auto f) { each([&](uint32_t c, uint32_t) { f(c); }); });
    uint32_t after = 0;  // of the topics with the least count, those whose inverse is at least this
    if (least > 0) {
        after = nth_largest(lds, (int32_t)kMixTopicBits, ties, [&](auto f) {
            each([&](uint32_t c, uint32_t t) {
                if (c == least) f(kInverted - t);
            });
        });
    }
    __syncthreads();
    if (tid == 0) lds.n_keys = 0;
    __syncthreads();
    each([&](uint32_t c, uint32_t t) {
        if (c > least || (c == least && kInverted - t >= after)) lds.keys[atomicAdd(&lds.n_keys, 1)] = long_key(c, (int32_t)t);
    });
    __syncthreads();
    const int32_t n_best = min(n, a.k);
    order_keys(lds.keys, n_best, a.k, lds.best);
    write_keys(a, row, lds.best, n_best, counted);
    return true;
}

// The best k topics of one range, of topics from t0 on, to lds.keys, n_first on; returns the thread's
// share of the tokens counted.  Counters are 16-bit for documents of less than 2^16 tokens (twice the
// topics a range), else 32-bit.
template <bool WIDE>
__device__ __forceinline__ int32_t best_of_range(const TopicArgs& a, const int32_t* z, int32_t L, int32_t t0, int32_t n_first,
                                                 LongLds& lds)
{
    constexpr int32_t kPer = WIDE ? 1 : 2, kRange = WIDE ? kWideRange : kNarrowRange;
    constexpr int kLoads = 2;
    const int32_t tid = (int32_t)threadIdx.x;
    int32_t counted = 0;
    const int32_t nt = min(kRange, a.K - t0);
    // words of a thread, an odd number for their banks; topics [tid * each * kPer, ..) of the range
    const int32_t each_words = ((nt + kPer - 1) / kPer + kLongBlock - 1) / kLongBlock | 1;
    uint32_t* const own = lds.count + tid * each_words;
    // f(count, topic of the range) for the thread's own topics in ascending order
    const auto each = [&](auto f) {
        uint32_t next_word = own[0];
#pragma unroll 1
        for (int32_t j = 0; j < each_words; ++j) {
            const uint32_t w = next_word;
            next_word = own[min(j + 1, each_words - 1)];
            if (w == 0) continue;
            const int32_t t = (tid * each_words + j) * kPer;
            if (WIDE) {
                f(w, t);
            } else {
                if (w & 0xFFFFu) f(w & 0xFFFFu, t);
                if (w >> 16) f(w >> 16, t + 1);
            }
        }
    };
    // four neighbours a load
    int4 next[kLoads];
    const auto load = [&](int32_t i0, int32_t e) {
        const int64_t i = (int64_t)i0 + (e * kLongBlock + tid) * 4;
        int4 v;
        if (i + 4 <= L) {
            __builtin_memcpy(&v, z + i, 16);
        } else {
            v.x = i < L ? z[i] : -1;
            v.y = i + 1 < L ? z[i + 1] : -1;
            v.z = i + 2 < L ? z[i + 2] : -1;
            v.w = -1;
        }
        return v;
    };
#pragma unroll
    for (int e = 0; e < kLoads; ++e) next[e] = load(0, e);
    __syncthreads();
    for (int32_t i = tid; i < each_words * kLongBlock; i += kLongBlock) lds.count[i] = 0;
    __syncthreads();
    const auto count = [&](uint32_t at, uint32_t tokens) {
        if (WIDE) atomicAdd(&lds.count[at], tokens);
        else atomicAdd(&lds.count[at / 2], tokens << (16 * (at & 1)));
    };
    HotTopics hot((int32_t)((uint32_t)next[0].x - (uint32_t)t0), (uint32_t)next[0].x - (uint32_t)t0 < (uint32_t)nt);
    for (int64_t i0 = 0; i0 < L; i0 += kLoads * kLongBlock * 4) {
        int4 topic[kLoads];
#pragma unroll
        for (int e = 0; e < kLoads; ++e) {
            topic[e] = next[e];
            if (i0 + kLoads * kLongBlock * 4 < L) next[e] = load((int32_t)(i0 + kLoads * kLongBlock * 4), e);
        }
#pragma unroll
        for (int e = 0; e < kLoads; ++e) {
            const int32_t four[4] = {topic[e].x, topic[e].y, topic[e].z, topic[e].w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t at = (uint32_t)four[q] - (uint32_t)t0;  // (-1 and topics of other ranges lie beyond)
                const bool open = at < (uint32_t)nt;
                counted += open;
                if (hot.left((int32_t)at, open)) count(at, 1u);
            }
        }
    }
#pragma unroll
    for (int q = 0; q < HotTopics::kHot; ++q)
        if (hot.tokens[q] > 0 && tid % kWave == 0) count((uint32_t)hot.topic[q], (uint32_t)hot.tokens[q]);
    __syncthreads();
    const auto parts = [&](uint32_t w, uint32_t& low, uint32_t& high) {
        low = WIDE ? w : w & 0xFFFFu;
        high = WIDE ? 0u : w >> 16;
    };
    // topics come in ascending order: ties go to the first
    int32_t ties, equal, total;
    const uint32_t least = least_count(
        lds, a.k, ties, equal,
        [&](int32_t(&few)[3], auto f) {
#pragma unroll 2
            for (int32_t j = 0; j < each_words; ++j) {  // without a branch for the many words of nothing or little
                uint32_t low, high;
                parts(own[j], low, high);
#pragma unroll
                for (uint32_t q = 0; q < 3; ++q) few[q] += (int32_t)(low == q + 1) + (int32_t)(high == q + 1);
                if (max(low, high) > 3) {
                    if (low > 3) f(low);
                    if (high > 3) f(high);
                }
            }
        },
        [&](auto f) { each([&](uint32_t c, int32_t) { f(c); }); });
    const int32_t before = least > 0 ? block_prefix<kLongBlock>(equal, lds.part, total) : 0;
    int32_t take = min(max(ties - before, 0), equal);  // of the thread's topics with the least count
    __syncthreads();
    if (tid == 0) lds.n_keys = n_first;
    __syncthreads();
    const uint32_t from = least > 0 && take > 0 ? least : least + 1;
#pragma unroll 2
    for (int32_t j = 0; j < each_words; ++j) {
        uint32_t c[2];
        parts(own[j], c[0], c[1]);
        if (max(c[0], c[1]) < from) continue;
        for (int32_t q = 0; q < kPer; ++q) {
            if (c[q] > least || (c[q] == least && least > 0 && take-- > 0))
                lds.keys[atomicAdd(&lds.n_keys, 1)] = long_key(c[q], t0 + (tid * each_words + j) * kPer + q);
        }
    }
    __syncthreads();
    return counted;
}

template <bool WIDE>
__device__ __forceinline__ void topics_by_counters(const TopicArgs& a, int64_t row, int64_t g0, int32_t L, LongLds& lds)
{
    int32_t n_best = 0, counted = 0;
    for (int32_t t0 = 0; t0 < a.K; t0 += WIDE ? kWideRange : kNarrowRange) {
        counted += best_of_range<WIDE>(a, a.z + g0, L, t0, n_best, lds);
        const int32_t n = lds.n_keys;
        order_keys(lds.keys, n, a.k, lds.best);
        n_best = min(n, a.k);
        for (int32_t i = (int32_t)threadIdx.x; i < n_best; i += kLongBlock) lds.keys[i] = lds.best[i];
    }
    counted = block_sum<kLongBlock>(counted, lds.part);
    write_keys(a, row, lds.best, n_best, counted);
}

// The ranges of the documents that are split, a workgroup each.  A document of 440 000 tokens in 100 000 topics: 100 us
// for all that it takes (340 with its four ranges one after the other); counting takes 75 us of them, some
// 25 instructions a round of 64 tokens on the four SIMDs of one CU.  (A range of 63 488 topics is looked through twice, 31
// words a thread: 4 us each.)
__global__ __launch_bounds__(kLongBlock) void range_topics_kernel(TopicArgs a)
{
    extern __shared__ __align__(16) unsigned char raw[];
    LongLds& lds = *reinterpret_cast<LongLds*>(raw);
    const int32_t tid = (int32_t)threadIdx.x;
    const int32_t wide = min(a.n_split[0], a.wide_places), others = min(a.n_split[1], a.places - a.wide_places);
    const int64_t n = ((int64_t)wide + others) * a.ranges;
    for (int64_t q = blockIdx.x; q < n; q += gridDim.x) {
        const int32_t at = (int32_t)(q / a.ranges), range = (int32_t)(q % a.ranges);
        const int32_t place = at < wide ? at : a.wide_places + at - wide;
        const int64_t i = (int64_t)place * a.ranges + range;
        int64_t g0, g1;
        document_of(a, a.split_rows[place], g0, g1);
        const int32_t L = (int32_t)(g1 - g0);
        if (range >= ranges_of(a.K, L)) continue;
        int32_t counted;
        if (L < kWideTokens) counted = best_of_range<false>(a, a.z + g0, L, range * kNarrowRange, 0, lds);
        else counted = best_of_range<true>(a, a.z + g0, L, range * kWideRange, 0, lds);
        counted = block_sum<kLongBlock>(counted, lds.part);
        const int32_t n_keys = lds.n_keys;
        if (tid == 0) a.split_n[i] = make_int2(n_keys, counted);
        for (int32_t j = tid; j < n_keys; j += kLongBlock) a.split_keys[i * a.k + j] = lds.keys[j];
        __syncthreads();
    }
}

// and put together: as many ranges at a time as are ordered quickly
__device__ __forceinline__ void join_ranges(const TopicArgs& a, int64_t row, int32_t L, int32_t place, LongLds& lds)
{
    const int32_t tid = (int32_t)threadIdx.x, ranges = ranges_of(a.K, L), most = max(2 * a.k, 512);
    int32_t n_best = 0, counted = 0;
    for (int32_t r = 0; r < ranges;) {
        int32_t n = n_best;
        __syncthreads();
        for (; r < ranges; ++r) {
            const int64_t i = (int64_t)place * a.ranges + r;
            const int2 part = a.split_n[i];
            if (n + part.x > most) break;
            for (int32_t j = tid; j < part.x; j += kLongBlock) lds.keys[n + j] = a.split_keys[i * a.k + j];
            n += part.x;
            counted += part.y;
        }
        __syncthreads();
        order_keys(lds.keys, n, a.k, lds.best);
        n_best = min(n, a.k);
        for (int32_t i = tid; i < n_best; i += kLongBlock) lds.keys[i] = lds.best[i];
    }
    write_keys(a, row, lds.best, n_best, counted);
}

__global__ __launch_bounds__(kLongBlock) void long_topics_kernel(TopicArgs a)
{
    extern __shared__ __align__(16) unsigned char raw[];
    LongLds& lds = *reinterpret_cast<LongLds*>(raw);
    a.z = assignment(a);
    for_rows_left<kLongBlock>(a, lds.mine, &lds.n_mine, [&](int64_t row, int64_t g0, int32_t L) {
        const int32_t mark = a.ids[row * a.k], ranges = ranges_of(a.K, L);
        if (mark <= kSplit) {
            join_ranges(a, row, L, kSplit - mark, lds);
            return;
        }
        if (ranges > 1 && L / kTableTokens < ranges && topics_by_table(a, row, g0, L, lds)) return;
        if (L < kWideTokens) {
            topics_by_counters<false>(a, row, g0, L, lds);
        } else {
            topics_by_counters<true>(a, row, g0, L, lds);
        }
    });
}

__global__ void no_splits_kernel(int32_t* n_split) { n_split[0] = n_split[1] = 0; }

// Places for documents that are split: those of kWideTokens, the others; at most `room` in all
struct SplitPlaces {
    int64_t wide, others;
};
static SplitPlaces split_places(const lda_topic_rows* d, int64_t room)
{
    if (d->K <= kWideRange) return {0, 0};
    const auto most = [&](int64_t tokens) {
        if (d->tokens < tokens) return (int64_t)0;
        return d->docs || d->rows < d->tokens / tokens ? d->rows : d->tokens / tokens;
    };
    SplitPlaces p{most(kWideTokens), most(kSplitTokens)};
    if (p.wide > room / 2 && p.wide + p.others > room) p.wide = room / 2;
    if (p.others > room - p.wide) p.others = room - p.wide;
    return p;
}
static int64_t place_bytes(const lda_topic_rows* d) { return 8 + (int64_t)ranges_of(d->K, kWideTokens) * (8 + 8 * d->slots); }
static int64_t topics_bytes(const lda_topic_rows* d)
{
    const SplitPlaces p = split_places(d, kSplitBytes / place_bytes(d));
    return p.wide + p.others == 0 ? 0 : 16 + (p.wide + p.others) * place_bytes(d);
}

static int launch_top_topics(lda_ctx* c, const TopicArgs& a, hipStream_t stream)
{
    if (a.rows == 0) return LDA_OK;
    const auto grid = [&](int64_t rows_each, int64_t most) {
        const int64_t n = (a.rows + rows_each - 1) / rows_each;
        return (unsigned)(n < most ? n : most);
    };
    if (a.places > 0) no_splits_kernel<<<1, 1, 0, stream>>>(a.n_split);
    // documents cannot be longer than all of z
    wave_topics_kernel<<<grid(kWaveBlock / kWave, 256 * 6), kWaveBlock, 0, stream>>>(a);
    if (a.tokens > kWaveTopics) {
        if (a.places > 0) {
            LDA_HIP(c, hipFuncSetAttribute(reinterpret_cast<const void*>(range_topics_kernel),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(LongLds)));
            range_topics_kernel<<<(unsigned)std::min<int64_t>((int64_t)a.places * a.ranges, 1024), kLongBlock, sizeof(LongLds), stream>>>(a);
        }
        LDA_HIP(c, hipFuncSetAttribute(reinterpret_cast<const void*>(long_topics_kernel),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(LongLds)));
        long_topics_kernel<<<a.rows <= 1024 ? (unsigned)a.rows : 256u, kLongBlock, sizeof(LongLds), stream>>>(a);
    }
    LDA_HIP(c, hipGetLastError());
    return LDA_OK;
}

static int check_outputs(lda_ctx* c, const char* call, int64_t rows, int32_t slots, const int32_t* ids,
                         const float* logits, const float* log_norm)
{
    if (rows < 0 || slots < 1) return fail(c, LDA_ERR_ARG, "%s: rows >= 0, slots >= 1 needed", call);
    if (slots > kMostTopSlots) return fail(c, LDA_ERR_UNSUPPORTED, "%s: at most %d slots", call, kMostTopSlots);
    if (rows > 0 && (!ids || !logits)) return fail(c, LDA_ERR_ARG, "%s: NULL output", call);
    if (!aligned_to(ids, 4) || !aligned_to(logits, 4) || !aligned_to(log_norm, 4))
        return fail(c, LDA_ERR_ARG, "%s: a pointer is not aligned to its type", call);
    return LDA_OK;
}

static int check_topics(const lda_topic_rows* d, const char* call)
{
    if (!d) return fail(nullptr, LDA_ERR_ARG, "%s: NULL rows", call);
    for (int32_t r : d->reserved)
        if (r != 0) return fail(nullptr, LDA_ERR_ARG, "%s: reserved fields must be zero", call);
    if (d->reserved_word != 0) return fail(nullptr, LDA_ERR_ARG, "%s: reserved fields must be zero", call);
    if (d->rows < 0 || d->slots < 1) return fail(nullptr, LDA_ERR_ARG, "%s: rows >= 0, slots >= 1 needed", call);
    if (d->slots > kMostTopSlots) return fail(nullptr, LDA_ERR_UNSUPPORTED, "%s: at most %d slots", call, kMostTopSlots);
    if (d->documents < 0 || d->tokens < 0 || d->K < 1 || (!d->docs && d->documents < d->rows))
        return fail(nullptr, LDA_ERR_ARG, "%s: documents >= 0 (>= rows without docs), tokens >= 0, K >= 1 needed", call);
    if (d->K > (1 << 20) - 2) return fail(nullptr, LDA_ERR_UNSUPPORTED, "%s: K must be at most 2^20 - 2", call);
    if (!(d->alpha > 0.0) || !(d->alpha < 1e300))
        return fail(nullptr, LDA_ERR_ARG, "%s: alpha must be positive and finite", call);
    if (!known_index(d->offsets_type)) return fail(nullptr, LDA_ERR_ARG, "%s: unknown type", call);
    if (d->workspace_bytes < 0 || !aligned_to(d->workspace, 16))
        return fail(nullptr, LDA_ERR_ARG, "%s: a workspace aligned to 16 bytes needed, or none", call);
    if (d->rows == 0) return LDA_OK;
    if ((d->documents > 0 && !d->offsets) || (d->tokens > 0 && !d->z))
        return fail(nullptr, LDA_ERR_ARG, "%s: NULL pointer", call);
    if (!aligned_to(d->docs, 4) || !aligned_to(d->offsets, index_bytes(d->offsets_type)) || !aligned_to(d->z, 4))
        return fail(nullptr, LDA_ERR_ARG, "%s: a pointer is not aligned to its type", call);
    return LDA_OK;
}

}  // namespace lda

using namespace lda;

extern "C" {

int64_t lda_topics_workspace(const lda_topic_rows* d)
try {
    const int rc = check_topics(d, "lda_topics_workspace");
    return rc != LDA_OK ? rc : topics_bytes(d);
} catch (...) {
    return LDA_ERR_OOM;
}

int lda_top_topics(const lda_topic_rows* d, int32_t* ids, float* logits, float* log_norm)
try {
    const char* call = "lda_top_topics";
    int rc = check_topics(d, call);
    if (rc == LDA_OK) rc = check_outputs(nullptr, call, d->rows, d->slots, ids, logits, log_norm);
    if (rc != LDA_OK || d->rows == 0) return rc;
    TopicArgs a{};
    a.rows = d->rows;
    a.docs = d->docs;
    a.documents = d->documents;
    a.offsets = d->offsets;
    a.offsets_type = d->offsets_type;
    a.K = d->K;
    a.z = d->z;
    a.tokens = d->tokens;
    a.k = d->slots;
    a.alpha = d->alpha;
    a.ids = ids;
    a.logits = logits;
    a.log_norm = log_norm;
    if (d->workspace) {
        // as many documents as there is room for
        const int64_t room = d->workspace_bytes < 16 ? 0 : (d->workspace_bytes - 16) / place_bytes(d);
        const SplitPlaces p = split_places(d, room < (1 << 24) ? room : 1 << 24);
        a.wide_places = (int32_t)p.wide;
        a.places = (int32_t)(p.wide + p.others);
        a.ranges = ranges_of(d->K, kWideTokens);
        a.n_split = static_cast<int32_t*>(d->workspace);
        a.split_rows = reinterpret_cast<int64_t*>(a.n_split + 4);
        a.split_n = reinterpret_cast<int2*>(a.split_rows + a.places);
        a.split_keys = reinterpret_cast<uint64_t*>(a.split_n + (int64_t)a.places * a.ranges);
    }
    return launch_top_topics(nullptr, a, static_cast<hipStream_t>(d->hip_stream));
} catch (...) {
    return LDA_ERR_OOM;
}

int lda_doc_topics(lda_ctx* c, int64_t rows, const int32_t* docs, int32_t slots, int32_t* ids, float* logits,
                   float* log_norm)
try {
    if (!c) return LDA_ERR_ARG;
    const char* call = "lda_doc_topics";
    if (c->streamed)
        return fail(c, LDA_ERR_UNSUPPORTED, "%s: not with streamed data blocks", call);
    const int rc = check_outputs(c, call, rows, slots, ids, logits, log_norm);
    if (rc != LDA_OK) return rc;
    if (!docs && rows > c->D) return fail(c, LDA_ERR_ARG, "%s: more rows than documents", call);
    if (!aligned_to(docs, 4)) return fail(c, LDA_ERR_ARG, "%s: a pointer is not aligned to its type", call);
    int device = -1;
    LDA_HIP(c, hipGetDevice(&device));
    if (device != c->device)
        return fail(c, LDA_ERR_ARG, "%s: device %d has to be the current one, not %d", call, c->device, device);
    TopicArgs a{};
    a.rows = rows;
    a.docs = docs;
    a.documents = c->D;
    a.offsets = c->d_doff;
    a.offsets_type = LDA_I32;
    a.K = c->K;
    a.z = c->d_z;
    if (stream_is_captured(c)) {  // replays come after sweeps that the host calls then
        c->z_in_graph = true;
        a.z_now = c->z_now();
    }
    a.tokens = c->N;
    a.k = slots;
    a.alpha = c->alpha;
    a.ids = ids;
    a.logits = logits;
    a.log_norm = log_norm;
    return launch_top_topics(c, a, c->stream);
} catch (...) {
    return LDA_ERR_OOM;
}

}  // extern "C"
