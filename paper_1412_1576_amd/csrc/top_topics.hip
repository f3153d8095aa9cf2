// Top topics of documents: teacher rows out of an assignment (lda_topic_rows in lda_mi355x.h).
//
// A document's counts are formed in LDS, one counter a topic, for a range of topics at a time;
// the best of a range and of the ranges before it are kept.  A topic with its count is one 64-bit key,
// (count, then the lower topic), so that all keys differ and "the k largest" is one set.
#include "rows.hpp"

namespace lda {

constexpr int32_t kMostTopSlots = 1024;
constexpr int kTopBlock = 256;
constexpr int32_t kRangeTopics = 12288;

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

__device__ __forceinline__ uint64_t topic_key(uint32_t count, int32_t topic)
{
    return ((uint64_t)count << kMixTopicBits) | (uint64_t)((1u << kMixTopicBits) - 1u - (uint32_t)topic);
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

__global__ __launch_bounds__(kTopBlock) void top_topics_kernel(TopicArgs a)
{
    __shared__ uint32_t count[kRangeTopics];
    __shared__ uint64_t best[2 * kMostTopSlots];  // of the ranges before, and the new ones
    __shared__ int32_t parti[kTopBlock / kWave];
    __shared__ int32_t n_new;
    const int32_t tid = (int32_t)threadIdx.x;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        int64_t g0, g1;
        document_of(a, row, g0, g1);
        uint64_t* old = best;
        uint64_t* fresh = best + kMostTopSlots;
        int32_t n_old = 0;
        int64_t counted = 0;
        for (int32_t t0 = 0; t0 < a.K; t0 += kRangeTopics) {
            const int32_t nt = min(kRangeTopics, a.K - t0);
            for (int32_t i = tid; i < nt; i += kTopBlock) count[i] = 0;
            __syncthreads();
            for (int64_t g = g0 + tid; g < g1; g += kTopBlock) {
                const uint32_t t = (uint32_t)(a.z[g] - t0);
                if (a.z[g] >= t0 && t < (uint32_t)nt) atomicAdd(&count[t], 1u);
            }
            __syncthreads();
            int32_t some = 0, in_range = 0;
            for (int32_t i = tid; i < nt; i += kTopBlock) {
                some += count[i] > 0;
                in_range += (int32_t)count[i];
            }
            some = block_sum<kTopBlock>(some, parti);
            counted += block_sum<kTopBlock>(in_range, parti);
            // the smallest key that is still among the best k, found bit by bit
            uint64_t least = 0;
            if (some + n_old > a.k) {
                for (int bit = 31 + (int)kMixTopicBits; bit >= 0; --bit) {
                    const uint64_t at = least | (1ull << bit);
                    int32_t above = 0;
                    for (int32_t i = tid; i < nt; i += kTopBlock)
                        above += count[i] > 0 && topic_key(count[i], t0 + i) >= at;
                    for (int32_t i = tid; i < n_old; i += kTopBlock) above += old[i] >= at;
                    if (block_sum<kTopBlock>(above, parti) >= a.k) least = at;
                }
            }
            __syncthreads();
            if (tid == 0) n_new = 0;
            __syncthreads();
            for (int32_t i = tid; i < nt; i += kTopBlock)
                if (count[i] > 0) {
                    const uint64_t key = topic_key(count[i], t0 + i);
                    if (key >= least) fresh[atomicAdd(&n_new, 1)] = key;
                }
            for (int32_t i = tid; i < n_old; i += kTopBlock)
                if (old[i] >= least) fresh[atomicAdd(&n_new, 1)] = old[i];
            __syncthreads();
            n_old = n_new;
            uint64_t* other = old;
            old = fresh;
            fresh = other;
            __syncthreads();
        }
        // places by counting the larger keys
        for (int32_t i = tid; i < a.k; i += kTopBlock) {
            if (i < n_old) {
                const uint64_t key = old[i];
                int32_t place = 0;
                for (int32_t j = 0; j < n_old; ++j) place += old[j] > key;
                const int64_t at = row * a.k + place;
                a.ids[at] = (int32_t)((1u << kMixTopicBits) - 1u - (uint32_t)(key & ((1u << kMixTopicBits) - 1u)));
                a.logits[at] = (float)log((double)(key >> kMixTopicBits) + a.alpha);
            } else {
                a.ids[row * a.k + i] = -1;
                a.logits[row * a.k + i] = -INFINITY;
            }
        }
        if (tid == 0 && a.log_norm) a.log_norm[row] = (float)log((double)counted + (double)a.K * a.alpha);
        __syncthreads();
    }
}

static int launch_top_topics(lda_ctx* c, const TopicArgs& a, hipStream_t stream)
{
    if (a.rows == 0) return LDA_OK;
    const unsigned grid = (unsigned)(a.rows < (1 << 20) ? a.rows : (1 << 20));
    top_topics_kernel<<<grid, kTopBlock, 0, stream>>>(a);
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
