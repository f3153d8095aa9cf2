// Verification of drafted tokens (the rule stands at lda_draft_rows in lda_mi355x.h): how many
// drafts are accepted, and a draw from what the target has left at the first that is not.
//
// The accept tests touch two numbers a draft; the draw reads one row of the target, and the draft's
// row beside it after a rejection.  A row is summed in slices by as many workgroups as it has
// slices; a second kernel walks the slices' sums to the one that holds the draw's place and looks
// only through that.  Masses and sums are 64-bit: p - q of two floats is then all but exact, and a
// draw's place differs from another order of summation by some 2^-50 of the row's mass.
#include "rows.hpp"

namespace lda {

constexpr int32_t kMostSteps = 4096;
constexpr int kVerifyBlock = 256;
constexpr int32_t kSliceElements = 4096;

struct SliceMass {
    double left, target;  // of max(0, p - q), of p
};

struct VerifyArgs {
    int64_t sequences;
    int32_t steps, V;
    const void* target;
    int64_t target_sequence_stride, target_row_stride;
    const void* draft;
    int64_t draft_sequence_stride, draft_row_stride;
    const void* tokens;
    int64_t tokens_stride;
    const int32_t* lengths;
    const float* accept_u;
    int64_t accept_u_stride;
    const float* draw_u;
    int32_t tokens_type;
    int32_t slices;
    SliceMass* sums;  // [sequences][slices]
    int32_t* accepted;
    void* out;
    int64_t out_stride;
};

// Accepted drafts of sequence b: every wave finds them for itself, 64 tests at a time.
template <class T>
__device__ __forceinline__ int32_t count_accepted(const VerifyArgs& a, int64_t b, int32_t& n)
{
    const int lane = threadIdx.x % kWave;
    n = a.lengths ? min(max(a.lengths[b], 0), a.steps) : a.steps;
    const T* p = static_cast<const T*>(a.target) + b * a.target_sequence_stride;
    const T* q = static_cast<const T*>(a.draft) + b * a.draft_sequence_stride;
    for (int32_t i0 = 0; i0 < n; i0 += kWave) {
        const int32_t i = i0 + lane;
        bool ok = false;
        if (i < n) {
            const int64_t x = index_at(a.tokens, a.tokens_type, b * a.tokens_stride + i);
            if (x >= 0 && x < a.V) {
                const double u = (double)a.accept_u[b * a.accept_u_stride + i];
                ok = u * (double)Row<T>::one(q + i * a.draft_row_stride + x) <
                     (double)Row<T>::one(p + i * a.target_row_stride + x);
            }
        }
        const uint64_t stopped = ~__ballot(ok);
        if (stopped) return min(n, i0 + (int32_t)__builtin_ctzll(stopped));
    }
    return n;
}

// p, and max(0, p - q) with q where a draft was rejected; a NaN has no mass
__device__ __forceinline__ double mass_of(double x) { return x > 0.0 ? x : 0.0; }

// sums[b][slice] of the masses of elements [slice * kSliceElements, ..)
template <class T>
__global__ __launch_bounds__(kVerifyBlock) void verify_sums_kernel(VerifyArgs a)
{
    __shared__ double part[kVerifyBlock / kWave];
    for (int64_t b = blockIdx.x; b < a.sequences; b += gridDim.x) {
        int32_t n;
        const int32_t k = count_accepted<T>(a, b, n);
        const T* p = static_cast<const T*>(a.target) + b * a.target_sequence_stride + k * a.target_row_stride;
        const T* q = k < n ? static_cast<const T*>(a.draft) + b * a.draft_sequence_stride + k * a.draft_row_stride : nullptr;
        for (int32_t slice = (int32_t)blockIdx.y; slice < a.slices; slice += (int32_t)gridDim.y) {
            const int64_t v0 = (int64_t)slice * kSliceElements;
            const int64_t v1 = min(v0 + kSliceElements, (int64_t)a.V);
            double left = 0.0, target = 0.0;
            for (int64_t v = v0 + threadIdx.x; v < v1; v += kVerifyBlock) {
                const double pv = (double)Row<T>::one(p + v);
                target += mass_of(pv);
                if (q) left += mass_of(pv - (double)Row<T>::one(q + v));
            }
            target = block_sum<kVerifyBlock>(target, part);
            left = q ? block_sum<kVerifyBlock>(left, part) : target;
            if (threadIdx.x == 0) a.sums[b * a.slices + slice] = SliceMass{left, target};
        }
    }
}

// One workgroup a sequence: the slice of the draw's place, the element in it, the outputs.
template <class T>
__global__ __launch_bounds__(kVerifyBlock) void verify_draw_kernel(VerifyArgs a)
{
    __shared__ double scan[kVerifyBlock / kWave];
    __shared__ int64_t found[2];
    const int32_t tid = (int32_t)threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    for (int64_t b = blockIdx.x; b < a.sequences; b += gridDim.x) {
        int32_t n;
        const int32_t k = count_accepted<T>(a, b, n);
        const T* p = static_cast<const T*>(a.target) + b * a.target_sequence_stride + k * a.target_row_stride;
        const T* q = k < n ? static_cast<const T*>(a.draft) + b * a.draft_sequence_stride + k * a.draft_row_stride : nullptr;
        const SliceMass* sums = a.sums + b * a.slices;
        // every wave walks the sums in the same order, 64 slices at a time
        double left = 0.0, target = 0.0;
        for (int32_t s = lane; s < a.slices; s += kWave) {
            left += sums[s].left;
            target += sums[s].target;
        }
        left = wave_sum(left);
        target = wave_sum(target);
        if (!(left > 0.0)) q = nullptr;
        const bool whole = q == nullptr;
        const double total = whole ? target : left;
        const double place = (double)a.draw_u[b] * total;
        double before = 0.0;
        int32_t slice = -1, last = -1;
        for (int32_t s0 = 0; s0 < a.slices && slice < 0; s0 += kWave) {
            const int32_t s = s0 + lane;
            const double own = s < a.slices ? (whole ? sums[s].target : sums[s].left) : 0.0;
            double sum = own;
#pragma unroll
            for (int d = 1; d < kWave; d <<= 1) {
                const double o = __shfl_up(sum, d, kWave);
                if (lane >= d) sum += o;
            }
            const uint64_t some = __ballot(own > 0.0);
            const uint64_t past = __ballot(own > 0.0 && before + sum > place);
            if (some) last = s0 + 63 - (int32_t)__builtin_clzll(some);
            if (past) {
                const int at = __builtin_ctzll(past);
                slice = s0 + at;
                before += __shfl(sum, at, kWave) - __shfl(own, at, kWave);
            } else {
                before += __shfl(sum, kWave - 1, kWave);
            }
        }
        const bool inside = slice >= 0;
        if (!inside) slice = last;  // the last element of any mass
        int64_t token = -1;
        if (slice >= 0) {
            const int64_t v0 = (int64_t)slice * kSliceElements;
            const int64_t v1 = min(v0 + kSliceElements, (int64_t)a.V);
            constexpr int kEach = kSliceElements / kVerifyBlock;
            // a thread holds kEach neighbours
            double mass[kEach], sum = 0.0;
            const int64_t v = v0 + (int64_t)tid * kEach;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                mass[e] = 0.0;
                if (v + e < v1) {
                    const double pv = (double)Row<T>::one(p + v + e);
                    mass[e] = mass_of(whole ? pv : pv - (double)Row<T>::one(q + v + e));
                }
                sum += mass[e];
            }
            double upto = sum;
#pragma unroll
            for (int d = 1; d < kWave; d <<= 1) {
                const double o = __shfl_up(upto, d, kWave);
                if (lane >= d) upto += o;
            }
            __syncthreads();
            if (lane == kWave - 1) scan[wave] = upto;
            if (tid < 2) found[tid] = tid == 0 ? INT64_MAX : -1;
            __syncthreads();
            double run = before + (upto - sum);
            for (int w = 0; w < wave; ++w) run += scan[w];
            int64_t hit = INT64_MAX, most = -1;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                run += mass[e];
                if (mass[e] > 0.0) {
                    most = v + e;
                    if (inside && run > place && hit == INT64_MAX) hit = v + e;
                }
            }
            if (hit != INT64_MAX) atomicMin((long long*)&found[0], (long long)hit);
            if (most >= 0) atomicMax((long long*)&found[1], (long long)most);
            __syncthreads();
            token = found[0] != INT64_MAX ? found[0] : found[1];
        }
        if (tid == 0) a.accepted[b] = k;
        for (int32_t i = tid; i <= a.steps; i += kVerifyBlock) {
            int64_t x = i == k ? token : -1;
            if (i < k) x = index_at(a.tokens, a.tokens_type, b * a.tokens_stride + i);
            if (a.tokens_type == LDA_I32) static_cast<int32_t*>(a.out)[b * a.out_stride + i] = (int32_t)x;
            else static_cast<int64_t*>(a.out)[b * a.out_stride + i] = x;
        }
    }
}

static int64_t verify_slices(const lda_draft_rows* d)
{
    return ((int64_t)d->classes + kSliceElements - 1) / kSliceElements;
}

static int check_verify(const lda_draft_rows* d, const char* call)
{
    if (!d) return fail(nullptr, LDA_ERR_ARG, "%s: NULL rows", call);
    for (int32_t r : d->reserved)
        if (r != 0) return fail(nullptr, LDA_ERR_ARG, "%s: reserved fields must be zero", call);
    if (d->sequences < 0 || d->steps < 0 || d->classes < 1)
        return fail(nullptr, LDA_ERR_ARG, "%s: sequences >= 0, steps >= 0, classes >= 1 needed", call);
    if (d->steps > kMostSteps) return fail(nullptr, LDA_ERR_UNSUPPORTED, "%s: at most %d steps", call, kMostSteps);
    if (d->sequences > (int64_t)1 << 31) return fail(nullptr, LDA_ERR_UNSUPPORTED, "%s: too many sequences", call);
    if (!known_type(d->probs_type) || !known_index(d->tokens_type))
        return fail(nullptr, LDA_ERR_ARG, "%s: unknown type", call);
    if (d->sequences == 0) return LDA_OK;
    if (!d->target || !d->draw_u || (d->steps > 0 && (!d->draft || !d->tokens || !d->accept_u)))
        return fail(nullptr, LDA_ERR_ARG, "%s: NULL pointer", call);
    const size_t size = type_bytes(d->probs_type);
    if (!aligned_to(d->target, size) || !aligned_to(d->draft, size) || !aligned_to(d->tokens, index_bytes(d->tokens_type)) ||
        !aligned_to(d->lengths, 4) || !aligned_to(d->accept_u, 4) || !aligned_to(d->draw_u, 4))
        return fail(nullptr, LDA_ERR_ARG, "%s: a pointer is not aligned to its type", call);
    return LDA_OK;
}

template <class T>
static void launch_verify_typed(const VerifyArgs& a, hipStream_t stream)
{
    const unsigned gx = (unsigned)(a.sequences < (1 << 20) ? a.sequences : (1 << 20));
    const unsigned gy = (unsigned)(a.slices < 4096 ? a.slices : 4096);
    verify_sums_kernel<T><<<dim3(gx, gy), kVerifyBlock, 0, stream>>>(a);
    verify_draw_kernel<T><<<gx, kVerifyBlock, 0, stream>>>(a);
}

}  // namespace lda

using namespace lda;

extern "C" {

int64_t lda_verify_workspace(const lda_draft_rows* d)
try {
    const int rc = check_verify(d, "lda_verify_workspace");
    if (rc != LDA_OK) return rc;
    return d->sequences * verify_slices(d) * (int64_t)sizeof(SliceMass);
} catch (...) {
    return LDA_ERR_OOM;
}

int lda_verify_drafts(const lda_draft_rows* d, int32_t* accepted, void* out, int64_t out_stride)
try {
    const char* call = "lda_verify_drafts";
    const int rc = check_verify(d, call);
    if (rc != LDA_OK) return rc;
    if (d->sequences == 0) return LDA_OK;
    if (!accepted || !out) return fail(nullptr, LDA_ERR_ARG, "%s: NULL output", call);
    if (!aligned_to(accepted, 4) || !aligned_to(out, index_bytes(d->tokens_type)))
        return fail(nullptr, LDA_ERR_ARG, "%s: a pointer is not aligned to its type", call);
    if (d->sequences > 1 && out_stride < (int64_t)d->steps + 1)
        return fail(nullptr, LDA_ERR_ARG, "%s: rows of out overlap", call);
    VerifyArgs a{};
    a.sequences = d->sequences;
    a.steps = d->steps;
    a.V = d->classes;
    a.target = d->target;
    a.target_sequence_stride = d->target_sequence_stride;
    a.target_row_stride = d->target_row_stride;
    a.draft = d->draft;
    a.draft_sequence_stride = d->draft_sequence_stride;
    a.draft_row_stride = d->draft_row_stride;
    a.tokens = d->tokens;
    a.tokens_stride = d->tokens_stride;
    a.lengths = d->steps > 0 ? d->lengths : nullptr;
    a.accept_u = d->accept_u;
    a.accept_u_stride = d->accept_u_stride;
    a.draw_u = d->draw_u;
    a.tokens_type = d->tokens_type;
    a.slices = (int32_t)verify_slices(d);
    const int64_t need = a.sequences * a.slices * (int64_t)sizeof(SliceMass);
    if (!d->workspace || d->workspace_bytes < need || !aligned_to(d->workspace, 16))
        return fail(nullptr, LDA_ERR_ARG, "%s: needs a workspace of %lld bytes, aligned to 16", call, (long long)need);
    a.sums = static_cast<SliceMass*>(d->workspace);
    a.accepted = accepted;
    a.out = out;
    a.out_stride = out_stride;
    const hipStream_t stream = static_cast<hipStream_t>(d->hip_stream);
    if (d->probs_type == LDA_F32) launch_verify_typed<float>(a, stream);
    else if (d->probs_type == LDA_F16) launch_verify_typed<__half>(a, stream);
    else launch_verify_typed<__hip_bfloat16>(a, stream);
    LDA_HIP(static_cast<lda_ctx*>(nullptr), hipGetLastError());
    return LDA_OK;
} catch (...) {
    return LDA_ERR_OOM;
}

}  // extern "C"
