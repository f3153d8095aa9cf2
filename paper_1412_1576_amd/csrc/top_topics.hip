// Top topics of documents: teacher rows out of an assignment (lda_topic_rows in lda_mi355x.h).
//
// A topic with its count is one key, the count above the inverted topic: all keys of a document
// differ, larger keys come first in the output, and "the k largest" is one set.  What is done a document
// depends on its length alone (the host does not know it):
//   up to kWaveTokens   a wave; counts in an open-addressing table in LDS, the keys ranked against each other
//   up to kTableTokens  a workgroup of 1024, the same
//   longer              a workgroup of 1024; a counter a topic in LDS, a range of topics at a time
// One kernel takes the first, one the others; each looks through all rows and leaves the others' alone.
#include "rows.hpp"

namespace lda {

constexpr int32_t kMostTopSlots = 1024;
constexpr uint32_t kInverted = (1u << kMixTopicBits) - 1u;  // a key's topic is kInverted - (key & kInverted)

constexpr int kWaveBlock = 256;          // four documents at a time
constexpr int32_t kWaveTokens = 512;     // table: twice as many slots
constexpr int32_t kTableTokens = 4095;   // the count of a 32-bit key has 12 bits
constexpr int kLongBlock = 1024;
constexpr int32_t kLongWords = 31;       // counters in LDS, a thread: an odd number, for its banks
constexpr int32_t kDigit = 10;           // bits of a count that a histogram takes at a time

struct TopicArgs {
    int64_t rows;
    const int32_t* docs;
    int64_t documents;
    const void* offsets;
    int32_t offsets_type;
    int32_t K;
    const int32_t* z;
    int64_t tokens;
    int32_t k;
    double alpha;
    int32_t* ids;
    float* logits;
    float* log_norm;
};

__device__ __forceinline__ void document_of(const TopicArgs& a, int64_t row, int64_t& g0, int64_t& g1)
{
    const int64_t d = a.docs ? (int64_t)a.docs[row] : row;
    g0 = g1 = 0;
    if (d < 0 || d >= a.documents) return;
    g0 = min(max(index_at(a.offsets, a.offsets_type, d), (int64_t)0), a.tokens);
    g1 = min(max(index_at(a.offsets, a.offsets_type, d + 1), g0), a.tokens);
    g1 = min(g1, g0 + INT32_MAX);
}

// Which threads work on a document together
template <int TEAM>
struct Team {
    static __device__ __forceinline__ int32_t rank() { return (int32_t)threadIdx.x % TEAM; }
    // LDS written by some threads of the team is read by others after this
    static __device__ __forceinline__ void order()
    {
        if (TEAM == kWave) wave_lds_order();
        else __syncthreads();
    }
    // sum of a wave's count (the same in its lanes) over the team
    static __device__ __forceinline__ int32_t sum(int32_t wave_count, int32_t* part)
    {
        if (TEAM == kWave) return wave_count;
        __syncthreads();
        if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = wave_count;
        __syncthreads();
        int32_t s = 0;
#pragma unroll
        for (int w = 0; w < TEAM / kWave; ++w) s += part[w];
        return s;
    }
};

// One document's counts in a table of SLOTS keys (0: empty), and its best k topics.  `keys` holds
// the document's keys and `best` (SLOTS / 2 each); the table is empty before and after.
template <int TEAM, int SLOTS, class LogCount>
__device__ __forceinline__ int32_t topics_by_table(const TopicArgs& a, int64_t row, int64_t g0, int32_t L,
                                                   uint32_t* table, uint32_t* keys, uint16_t* used, int32_t* n_used,
                                                   int32_t* part, LogCount log_count)
{
    constexpr int kEach = SLOTS / 2 / TEAM;  // keys a thread may hold
    const int32_t me = Team<TEAM>::rank(), lane = (int32_t)threadIdx.x % kWave;
    const uint64_t below = (1ull << lane) - 1;
    int32_t n = 0, counted = 0;
    if (TEAM > kWave) {
        if (me == 0) *n_used = 0;
        __syncthreads();  // and the table is empty
    }
    for (int32_t i0 = 0; i0 < L; i0 += TEAM) {
        const int32_t i = i0 + me;
        const int32_t t = i < L ? a.z[g0 + i] : -1;
        bool open = t >= 0 && t < a.K;
        counted += (int32_t)__popcll(__ballot(open));
        const uint32_t inv = kInverted - (uint32_t)t;
        uint32_t h = ((uint32_t)t * 0x9E3779B1u) >> (32 - __builtin_ctz(SLOTS));
        int32_t mine = -1;
        while (__ballot(open)) {  // at most half the slots are in use: every search ends
            if (open) {
                uint32_t v = table[h];
                if (v == 0) v = atomicCAS(&table[h], 0u, (1u << kMixTopicBits) | inv);
                if (v == 0) {
                    mine = (int32_t)h;
                    open = false;
                } else if ((v & kInverted) == inv) {
                    atomicAdd(&table[h], 1u << kMixTopicBits);
                    open = false;
                } else {
                    h = (h + 1) & (SLOTS - 1);
                }
            }
        }
        const uint64_t fresh = __ballot(mine >= 0);
        int32_t at = n;
        if (TEAM > kWave) {
            if (lane == 0) at = atomicAdd(n_used, (int32_t)__popcll(fresh));
            at = __shfl(at, 0, kWave);
        }
        if (mine >= 0) used[at + (int32_t)__popcll(fresh & below)] = (uint16_t)mine;
        n += (int32_t)__popcll(fresh);
    }
    counted = Team<TEAM>::sum(counted, part);
    Team<TEAM>::order();
    if (TEAM > kWave) {
        n = *n_used;
        __syncthreads();
    }
    // the keys, into registers and side by side in LDS; the table is cleared behind them
    uint32_t key[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int32_t i = e * TEAM + me;
        key[e] = 0;
        if (e * TEAM < n && i < n) {
            const uint32_t h = used[i];
            key[e] = table[h];
            table[h] = 0;
        }
    }
    int32_t n_best = n;
    uint32_t least = 1;
    if (n > (TEAM == kWave ? 2 * kWave : 8 * kWave) && n > a.k) {
        // too many to rank them all: the smallest of the best k first, bit by bit
        least = 0;
        for (int bit = 31 - __builtin_clz((uint32_t)L) + (int)kMixTopicBits; bit >= 0; --bit) {
            const uint32_t at = least | (1u << bit);
            int32_t above = 0;
#pragma unroll
            for (int e = 0; e < kEach; ++e)
                if (e * TEAM < n) above += (int32_t)__popcll(__ballot(key[e] >= at));
            if (Team<TEAM>::sum(above, part) >= a.k) least = at;
        }
        n_best = a.k;
    }
    if (TEAM > kWave) {
        if (me == 0) *n_used = 0;
        __syncthreads();
    }
    int32_t at = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        if (e * TEAM >= n) continue;
        const bool in = key[e] >= least;
        const uint64_t some = __ballot(in);
        if (TEAM > kWave) {
            if (lane == 0) at = atomicAdd(n_used, (int32_t)__popcll(some));
            at = __shfl(at, 0, kWave);
        }
        if (in) keys[at + (int32_t)__popcll(some & below)] = key[e];
        at += (int32_t)__popcll(some);
    }
    // up to a whole number of vectors
    if (me < 4) keys[n_best + me] = 0;
    Team<TEAM>::order();
    const uint4* four = reinterpret_cast<const uint4*>(keys);
    for (int32_t i = me; i < n_best; i += TEAM) {
        const uint32_t own = keys[i];
        int32_t place = 0;
        for (int32_t j = 0; j < (n_best + 3) / 4; ++j) {
            const uint4 v = four[j];
            place += (v.x > own) + (v.y > own) + (v.z > own) + (v.w > own);
        }
        if (place < a.k) {
            a.ids[row * a.k + place] = (int32_t)(kInverted - (own & kInverted));
            a.logits[row * a.k + place] = log_count((int32_t)(own >> kMixTopicBits));
        }
    }
    for (int32_t i = n_best + me; i < a.k; i += TEAM) {
        a.ids[row * a.k + i] = -1;
        a.logits[row * a.k + i] = -INFINITY;
    }
    Team<TEAM>::order();
    return counted;
}

__global__ __launch_bounds__(kWaveBlock) void wave_topics_kernel(TopicArgs a)
{
    constexpr int kWaves = kWaveBlock / kWave, kSlots = 2 * kWaveTokens;
    __shared__ __align__(16) uint32_t table[kWaves][kSlots];
    __shared__ __align__(16) uint32_t keys[kWaves][kWaveTokens + 4];
    __shared__ uint16_t used[kWaves][kWaveTokens];
    __shared__ float log_of[kWaveTokens + 1];  // of count + alpha
    const int32_t tid = (int32_t)threadIdx.x, wave = tid / kWave, lane = tid % kWave;
    for (int32_t i = tid; i < kWaves * kSlots; i += kWaveBlock) (&table[0][0])[i] = 0;
    for (int32_t i = tid; i <= kWaveTokens; i += kWaveBlock) log_of[i] = (float)log((double)i + a.alpha);
    __syncthreads();
    const double k_alpha = (double)a.K * a.alpha;
    for (int64_t row = (int64_t)blockIdx.x * kWaves + wave; row < a.rows; row += (int64_t)gridDim.x * kWaves) {
        int64_t g0, g1;
        document_of(a, row, g0, g1);
        if (g1 - g0 > kWaveTokens) continue;
        const int32_t counted = topics_by_table<kWave, kSlots>(a, row, g0, (int32_t)(g1 - g0), table[wave], keys[wave],
                                                               used[wave], nullptr, nullptr,
                                                               [&](int32_t n) { return log_of[n]; });
        if (lane == 0 && a.log_norm) a.log_norm[row] = (float)log((double)counted + k_alpha);
    }
}

// The rows of this workgroup whose documents have lo .. hi tokens: every gridDim.x-th row is this
// workgroup's, BLOCK of them are looked at together.  f(row, g0, L) is called for one after the other.
template <int BLOCK, class F>
__device__ __forceinline__ void for_rows_of_length(const TopicArgs& a, int32_t lo, int32_t hi, int32_t* mine, int32_t* n_mine,
                                                   F f)
{
    for (int64_t r0 = blockIdx.x; r0 < a.rows; r0 += (int64_t)gridDim.x * BLOCK) {
        __syncthreads();
        if (threadIdx.x == 0) *n_mine = 0;
        __syncthreads();
        const int64_t row = r0 + (int64_t)threadIdx.x * gridDim.x;
        if (row < a.rows) {
            int64_t g0, g1;
            document_of(a, row, g0, g1);
            if (g1 - g0 >= lo && g1 - g0 <= hi) mine[atomicAdd(n_mine, 1)] = (int32_t)threadIdx.x;
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
    int32_t sum = v;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int32_t o = __shfl_up(sum, d, kWave);
        if (lane >= d) sum += o;
    }
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
    uint32_t table[2 * (kTableTokens + 1)];
    uint32_t keys[kTableTokens + 5];
    uint16_t used[kTableTokens + 1];
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
    int32_t n_mine, n_keys, digit, over;
};
static_assert(sizeof(LongLds) <= 160 * 1024, "LDS of a CU");

// Counters are 16-bit for documents of less than 2^16 tokens (twice the topics a range), else 32-bit.
template <bool WIDE>
__device__ __forceinline__ void topics_by_counters(const TopicArgs& a, int64_t row, int64_t g0, int32_t L, LongLds& lds)
{
    constexpr int32_t kRange = (WIDE ? 1 : 2) * kLongWords * kLongBlock, kPer = WIDE ? 1 : 2;
    const int32_t tid = (int32_t)threadIdx.x;
    uint32_t* own = lds.count + tid * kLongWords;  // topics [tid * kLongWords * kPer, ..) of the range
    // f(count, topic of the range) for the thread's own topics in ascending order
    auto each = [&](auto f) {
#pragma unroll 1
        for (int32_t j = 0; j < kLongWords; ++j) {
            const uint32_t w = own[j];
            if (w == 0) continue;
            const int32_t t = (tid * kLongWords + j) * kPer;
            if (WIDE) {
                f(w, t);
            } else {
                if (w & 0xFFFFu) f(w & 0xFFFFu, t);
                if (w >> 16) f(w >> 16, t + 1);
            }
        }
    };
    int32_t n_best = 0, counted = 0;
    for (int32_t t0 = 0; t0 < a.K; t0 += kRange) {
        const int32_t nt = min(kRange, a.K - t0);
        __syncthreads();
        for (int32_t i = tid; i < kLongWords * kLongBlock; i += kLongBlock) lds.count[i] = 0;
        __syncthreads();
        constexpr int kLoads = 16;  // in flight together
        for (int64_t i0 = 0; i0 < L; i0 += kLoads * kLongBlock) {
            int32_t t[kLoads];
#pragma unroll
            for (int e = 0; e < kLoads; ++e) {
                const int64_t i = i0 + e * kLongBlock + tid;
                t[e] = i < L ? a.z[g0 + i] : -1;
            }
#pragma unroll
            for (int e = 0; e < kLoads; ++e) {
                const uint32_t at = (uint32_t)t[e] - (uint32_t)t0;
                if (t[e] < 0 || at >= (uint32_t)nt) continue;
                if (WIDE) atomicAdd(&lds.count[at], 1u);
                else atomicAdd(&lds.count[at / 2], 1u << (16 * (at & 1)));
            }
        }
        __syncthreads();
        int32_t some = 0, most = 0, tokens = 0;
        each([&](uint32_t c, int32_t) {
            ++some;
            tokens += (int32_t)c;
            most = max(most, (int32_t)c);
        });
        some = block_sum<kLongBlock>(some, lds.part);
        counted += block_sum<kLongBlock>(tokens, lds.part);
        most = wave_reduce(most, [](int32_t x, int32_t y) { return max(x, y); });
        __syncthreads();
        if (tid % kWave == 0) lds.part[tid / kWave] = most;
        __syncthreads();
        for (int w = 0; w < kLongBlock / kWave; ++w) most = max(most, lds.part[w]);
        // the smallest count among the best k of the range, digit by digit from the top, and how many of
        // the topics that have just that count are among them
        int32_t least = 1, ties = some;
        if (some > a.k) {
            int32_t need = a.k;   // of the topics whose count has the prefix found so far
            int32_t shift = max(0, 32 - (int32_t)__builtin_clz((uint32_t)most) - kDigit), bits = 32 - shift;
            uint32_t prefix = 0;
            for (;;) {
                __syncthreads();
                for (int32_t i = tid; i < 1 << kDigit; i += kLongBlock) lds.histogram[i] = 0;
                __syncthreads();
                const uint32_t mask = (1u << min(bits, kDigit)) - 1u;
                each([&](uint32_t c, int32_t) {
                    const bool in = bits > kDigit ? true : ((uint64_t)c >> (shift + bits)) == prefix;
                    if (in) atomicAdd(&lds.histogram[(c >> shift) & mask], 1u);
                });
                __syncthreads();
                // digit d is the one when fewer than `need` lie above it and no fewer with its own
                const int32_t d = (1 << kDigit) - 1 - tid;
                const int32_t here = (int32_t)lds.histogram[d];
                int32_t all;
                const int32_t above = block_prefix<kLongBlock>(here, lds.part, all);
                if (above < need && above + here >= need) {
                    lds.digit = d;
                    lds.over = above;
                }
                __syncthreads();
                prefix = (prefix << min(bits, kDigit)) | (uint32_t)lds.digit;
                need -= lds.over;
                if (shift == 0) break;
                bits = min(shift, kDigit);
                shift -= bits;
            }
            least = (int32_t)prefix;
            ties = need;
        }
        // the range's best behind those of the ranges before: ties by their order
        __syncthreads();
        if (tid == 0) lds.n_keys = n_best;
        int32_t equal = 0, all;
        each([&](uint32_t c, int32_t) { equal += (int32_t)c == least; });
        int32_t at = block_prefix<kLongBlock>(equal, lds.part, all);
        each([&](uint32_t c, int32_t t) {
            bool in = (int32_t)c > least;
            if ((int32_t)c == least) in = at++ < ties;
            if (in) lds.keys[atomicAdd(&lds.n_keys, 1)] = long_key(c, t0 + t);
        });
        __syncthreads();
        // their places, and the best k of them in order
        const int32_t n = lds.n_keys;
        for (int32_t i = tid; i < n; i += kLongBlock) {
            const uint64_t key = lds.keys[i];
            int32_t place = 0;
            for (int32_t j = 0; j < n; ++j) place += lds.keys[j] > key;
            if (place < a.k) lds.best[place] = key;
        }
        __syncthreads();
        n_best = min(n, a.k);
        for (int32_t i = tid; i < n_best; i += kLongBlock) lds.keys[i] = lds.best[i];
    }
    for (int32_t i = tid; i < a.k; i += kLongBlock) {
        const uint64_t key = i < n_best ? lds.best[i] : 0;
        a.ids[row * a.k + i] = i < n_best ? (int32_t)(kInverted - (uint32_t)(key & kInverted)) : -1;
        a.logits[row * a.k + i] = i < n_best ? (float)log((double)(key >> kMixTopicBits) + a.alpha) : -INFINITY;
    }
    if (tid == 0 && a.log_norm) a.log_norm[row] = (float)log((double)counted + (double)a.K * a.alpha);
}

__global__ __launch_bounds__(kLongBlock) void long_topics_kernel(TopicArgs a)
{
    extern __shared__ __align__(16) unsigned char raw[];
    LongLds& lds = *reinterpret_cast<LongLds*>(raw);
    for_rows_of_length<kLongBlock>(a, kWaveTokens + 1, INT32_MAX, lds.mine, &lds.n_mine,
                                   [&](int64_t row, int64_t g0, int32_t L) {
        if (L <= kTableTokens) {
            constexpr int kSlots = 2 * (kTableTokens + 1);
            TableLds& t = lds.table;
            __syncthreads();
            for (int32_t i = (int32_t)threadIdx.x; i < kSlots; i += kLongBlock) t.table[i] = 0;
            const int32_t counted = topics_by_table<kLongBlock, kSlots>(
                a, row, g0, L, t.table, t.keys, t.used, &lds.n_keys, lds.part,
                [&](int32_t n) { return (float)log((double)n + a.alpha); });
            if (threadIdx.x == 0 && a.log_norm) a.log_norm[row] = (float)log((double)counted + (double)a.K * a.alpha);
        } else if (L < 65536) {
            topics_by_counters<false>(a, row, g0, L, lds);
        } else {
            topics_by_counters<true>(a, row, g0, L, lds);
        }
    });
}

static int launch_top_topics(lda_ctx* c, const TopicArgs& a, hipStream_t stream)
{
    if (a.rows == 0) return LDA_OK;
    const auto grid = [&](int64_t rows_each, int64_t most) {
        const int64_t n = (a.rows + rows_each - 1) / rows_each;
        return (unsigned)(n < most ? n : most);
    };
    // documents cannot be longer than all of z
    wave_topics_kernel<<<grid(kWaveBlock / kWave, 256 * 5), kWaveBlock, 0, stream>>>(a);
    if (a.tokens > kWaveTokens) {
        LDA_HIP(c, hipFuncSetAttribute(reinterpret_cast<const void*>(long_topics_kernel),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(LongLds)));
        long_topics_kernel<<<grid(1, 256), kLongBlock, sizeof(LongLds), stream>>>(a);
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

}  // namespace lda

using namespace lda;

extern "C" {

int lda_top_topics(const lda_topic_rows* d, int32_t* ids, float* logits, float* log_norm)
try {
    const char* call = "lda_top_topics";
    if (!d) return fail(nullptr, LDA_ERR_ARG, "%s: NULL rows", call);
    for (int32_t r : d->reserved)
        if (r != 0) return fail(nullptr, LDA_ERR_ARG, "%s: reserved fields must be zero", call);
    if (d->reserved_word != 0) return fail(nullptr, LDA_ERR_ARG, "%s: reserved fields must be zero", call);
    const int rc = check_outputs(nullptr, call, d->rows, d->slots, ids, logits, log_norm);
    if (rc != LDA_OK) return rc;
    if (d->documents < 0 || d->tokens < 0 || d->K < 1 || (!d->docs && d->documents < d->rows))
        return fail(nullptr, LDA_ERR_ARG, "%s: documents >= 0 (>= rows without docs), tokens >= 0, K >= 1 needed", call);
    if (d->K > (1 << 20) - 2) return fail(nullptr, LDA_ERR_UNSUPPORTED, "%s: K must be at most 2^20 - 2", call);
    if (!(d->alpha > 0.0) || !(d->alpha < 1e300))
        return fail(nullptr, LDA_ERR_ARG, "%s: alpha must be positive and finite", call);
    if (!known_index(d->offsets_type)) return fail(nullptr, LDA_ERR_ARG, "%s: unknown type", call);
    if (d->rows == 0) return LDA_OK;
    if ((d->documents > 0 && !d->offsets) || (d->tokens > 0 && !d->z))
        return fail(nullptr, LDA_ERR_ARG, "%s: NULL pointer", call);
    if (!aligned_to(d->docs, 4) || !aligned_to(d->offsets, index_bytes(d->offsets_type)) || !aligned_to(d->z, 4))
        return fail(nullptr, LDA_ERR_ARG, "%s: a pointer is not aligned to its type", call);
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
    TopicArgs a{};
    a.rows = rows;
    a.docs = docs;
    a.documents = c->D;
    a.offsets = c->d_doff;
    a.offsets_type = LDA_I32;
    a.K = c->K;
    a.z = c->d_z;
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
