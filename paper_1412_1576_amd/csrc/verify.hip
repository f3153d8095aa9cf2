// Verification of drafted tokens (the rule stands at lda_draft_rows in lda_mi355x.h): how many
// drafts are accepted, and a draw from what the target has left at the first that is not.
//
// The accept tests touch two numbers a draft; the draw reads one row of the target, and the draft's
// row beside it after a rejection.  Rows of up to kDirectClasses classes are one workgroup's, which
// holds the masses in registers.  Longer ones are summed in segments of kSegment classes, and a wave walks
// the sums to the segment that holds the draw's place and looks only through that: inside a workgroup, or for long rows
// and many sequences the sums by as many waves as fill the GPU and the draws in a second kernel.  Masses and sums are 64-bit: p - q of two floats is
// then all but exact, and a draw's place differs from another order of summation by 2^-53 of the row's mass an
// addition, of which 30 + V / 65536 lie on a way through the sums.
#include "rows.hpp"

namespace lda {

constexpr int32_t kMostSteps = 4096;
constexpr int kVerifyBlock = 256;
constexpr int32_t kSegment = 1024;
constexpr int kEach = kSegment / kWave;                       // neighbours a lane holds in a draw
constexpr int32_t kDirectClasses = kVerifyBlock * kEach;
constexpr int kRowBlock = 1024;
constexpr int64_t kRowBytes = 81920;
constexpr int32_t kRowSegments = (int32_t)(kRowBytes / 2 / kSegment);

struct Mass {
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
    int32_t segments, each;  // of a row; of them, a wave's
    Mass* sums;              // [sequences][segments]; NULL: a row is one workgroup's
    int2* found;             // [sequences] accepted drafts, drafts there are
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

__device__ __forceinline__ double mass_of(double x) { return x > 0.0 ? x : 0.0; }  // a NaN has none

// The target's row of the draw, and the draft's row where one was rejected (else NULL)
template <class T>
struct DrawRows {
    const T *p, *q;
    __device__ __forceinline__ DrawRows(const VerifyArgs& a, int64_t b, int32_t k, int32_t n)
    {
        p = static_cast<const T*>(a.target) + b * a.target_sequence_stride + k * a.target_row_stride;
        q = k < n ? static_cast<const T*>(a.draft) + b * a.draft_sequence_stride + k * a.draft_row_stride : nullptr;
    }
};

// 16 bytes from anywhere (the hardware takes unaligned addresses), as floats
template <class T>
__device__ __forceinline__ void load_anywhere(const T* p, float (&x)[Row<T>::kChunk])
{
    uint4 r;
    __builtin_memcpy(&r, p, 16);
    Row<T>::unpack(r, x);
}

// elements v .. v + N - 1, 0 from V on
template <class T, int N>
__device__ __forceinline__ void load_run(const T* p, int64_t v, int32_t V, float (&x)[N])
{
    constexpr int E = Row<T>::kChunk;
    if (v + N <= V) {
#pragma unroll
        for (int i = 0; i < N; i += E) {
            float y[E];
            load_anywhere(p + v + i, y);
#pragma unroll
            for (int e = 0; e < E; ++e) x[i + e] = y[e];
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = v + i < V ? Row<T>::one(p + v + i) : 0.0f;
    }
}

// The draw among a thread's neighbours: the first of mass past the place, and the last of mass
__device__ __forceinline__ void look_through(const double (&mass)[kEach], double run, double place, int32_t& hit, int32_t& last)
{
    hit = last = -1;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        run += mass[e];
        if (mass[e] > 0.0) {
            last = e;
            if (hit < 0 && run > place) hit = e;
        }
    }
}

__device__ __forceinline__ void write_result(const VerifyArgs& a, int64_t b, int32_t k, int64_t token, int32_t tid, int32_t step)
{
    if (tid == 0) a.accepted[b] = k;
    for (int32_t i = tid; i <= a.steps; i += step) {
        int64_t x = i == k ? token : -1;
        if (i < k) x = index_at(a.tokens, a.tokens_type, b * a.tokens_stride + i);
        if (a.tokens_type == LDA_I32) static_cast<int32_t*>(a.out)[b * a.out_stride + i] = (int32_t)x;
        else static_cast<int64_t*>(a.out)[b * a.out_stride + i] = x;
    }
}

// A workgroup a sequence, kEach neighbours of the row a thread: 64 draws among 1000 classes 4.6 us, latency
template <class T>
__global__ __launch_bounds__(kVerifyBlock) void verify_direct_kernel(VerifyArgs a)
{
    constexpr int kWaves = kVerifyBlock / kWave;
    __shared__ Mass part[kWaves];
    __shared__ int32_t place_of[2][kWaves];
    const int32_t tid = (int32_t)threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    for (int64_t b = blockIdx.x; b < a.sequences; b += gridDim.x) {
        const double u = (double)a.draw_u[b];
        int32_t n;
        const int32_t k = count_accepted<T>(a, b, n);
        const DrawRows<T> rows(a, b, k, n);
        const int64_t v = (int64_t)tid * kEach;
        float p[kEach], q[kEach] = {};
        load_run<T, kEach>(rows.p, v, a.V, p);
        if (rows.q) load_run<T, kEach>(rows.q, v, a.V, q);
        double mass[kEach], target = 0.0, left = 0.0;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            target += mass_of((double)p[e]);
            mass[e] = mass_of((double)p[e] - (double)q[e]);
            left += mass[e];
        }
        double upto = wave_prefix(left);
        const double all_target = wave_sum(target);
        __syncthreads();
        if (lane == kWave - 1) part[wave] = Mass{upto, all_target};
        __syncthreads();
        double before = 0.0, total = 0.0;
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) before += part[w].left;
            total += part[w].left;
        }
        if (!(total > 0.0)) {  // nothing left: from the target
#pragma unroll
            for (int e = 0; e < kEach; ++e) mass[e] = mass_of((double)p[e]);
            left = target;
            upto = wave_prefix(target);
            before = total = 0.0;
            for (int w = 0; w < kWaves; ++w) {
                if (w < wave) before += part[w].target;
                total += part[w].target;
            }
        }
        int32_t hit, last;
        look_through(mass, before + (upto - left), u * total, hit, last);
        const uint64_t hits = __ballot(hit >= 0), lasts = __ballot(last >= 0);
        const int32_t at_hit = hits ? (int32_t)__builtin_ctzll(hits) : 0;
        const int32_t at_last = lasts ? 63 - (int32_t)__builtin_clzll(lasts) : 0;
        hit = __shfl(hit, at_hit, kWave);
        last = __shfl(last, at_last, kWave);
        if (lane == 0) {
            place_of[0][wave] = hits ? (wave * kWave + at_hit) * kEach + hit : -1;
            place_of[1][wave] = lasts ? (wave * kWave + at_last) * kEach + last : -1;
        }
        __syncthreads();
        int64_t token = -1;
        for (int w = kWaves - 1; w >= 0; --w)
            if (place_of[0][w] >= 0) token = place_of[0][w];
        for (int w = kWaves - 1; w >= 0 && token < 0; --w) token = place_of[1][w];
        write_result(a, b, k, token, tid, kVerifyBlock);
    }
}

// A wave's sums of segment s, in every lane
template <class T>
__device__ __forceinline__ Mass sum_segment(const VerifyArgs& a, const DrawRows<T>& rows, int32_t s)
{
    constexpr int E = Row<T>::kChunk, kLoads = kSegment / kWave / E;
    const int32_t lane = (int32_t)threadIdx.x % kWave;
    double left = 0.0, target = 0.0;
    float p[kLoads][E], q[kLoads][E] = {};
#pragma unroll
    for (int j = 0; j < kLoads; ++j) load_run<T, E>(rows.p, (int64_t)s * kSegment + (j * kWave + lane) * E, a.V, p[j]);
    if (rows.q) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) load_run<T, E>(rows.q, (int64_t)s * kSegment + (j * kWave + lane) * E, a.V, q[j]);
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            target += mass_of((double)p[j][e]);
            left += mass_of((double)p[j][e] - (double)q[j][e]);
        }
    return Mass{wave_sum(left), wave_sum(target)};
}

// A wave's draw: the segment of its place, then the element in it
template <class T>
__device__ __forceinline__ int64_t draw(const VerifyArgs& a, DrawRows<T> rows, const Mass* sums, double u)
{
    const int32_t lane = (int32_t)threadIdx.x % kWave;
    double left = 0.0, target = 0.0;
    for (int32_t s = lane; s < a.segments; s += kWave) {
        left += sums[s].left;
        target += sums[s].target;
    }
    left = wave_sum(left);
    target = wave_sum(target);
    const bool whole = !(left > 0.0);
    if (whole) rows.q = nullptr;
    const double place = u * (whole ? target : left);
    // 64 sums at a time, in order
    double before = 0.0;
    int32_t segment = -1, last = -1;
    for (int32_t s0 = 0; s0 < a.segments && segment < 0; s0 += kWave) {
        const int32_t s = s0 + lane;
        const double own = s < a.segments ? (whole ? sums[s].target : sums[s].left) : 0.0;
        const double sum = wave_prefix(own);
        const uint64_t some = __ballot(own > 0.0);
        const uint64_t past = __ballot(own > 0.0 && before + sum > place);
        if (some) last = s0 + 63 - (int32_t)__builtin_clzll(some);
        if (past) {
            const int at = __builtin_ctzll(past);
            segment = s0 + at;
            before += lane_value(sum - own, at);
        } else {
            before += lane_value(sum, kWave - 1);
        }
    }
    const bool inside = segment >= 0;
    if (!inside) segment = last;  // the last element of any mass
    if (segment < 0) return -1;
    const int64_t v = (int64_t)segment * kSegment + lane * kEach;
    float p[kEach], q[kEach] = {};
    load_run<T, kEach>(rows.p, v, a.V, p);
    if (rows.q) load_run<T, kEach>(rows.q, v, a.V, q);
    double mass[kEach], sum = 0.0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        mass[e] = mass_of((double)p[e] - (double)q[e]);
        sum += mass[e];
    }
    const double upto = wave_prefix(sum);
    int32_t hit, most;
    look_through(mass, before + (upto - sum), place, hit, most);
    const uint64_t hits = __ballot(inside && hit >= 0), some = __ballot(most >= 0);
    if (!hits && !some) return -1;
    const int at = hits ? __builtin_ctzll(hits) : 63 - (int)__builtin_clzll(some);
    return (int64_t)segment * kSegment + at * kEach + lane_value(hits ? hit : most, at);
}

// A workgroup a sequence, a row longer than its registers: the segments' sums in LDS
template <class T>
__global__ __launch_bounds__(kRowBlock) void verify_row_kernel(VerifyArgs a)
{
    constexpr int kWaves = kRowBlock / kWave;
    __shared__ Mass sums[kRowSegments];
    const int32_t wave = __builtin_amdgcn_readfirstlane((int32_t)threadIdx.x / kWave), lane = (int32_t)threadIdx.x % kWave;
    for (int64_t b = blockIdx.x; b < a.sequences; b += gridDim.x) {
        const double u = (double)a.draw_u[b];
        int32_t n;
        const int32_t k = count_accepted<T>(a, b, n);
        const DrawRows<T> rows(a, b, k, n);
        __syncthreads();  // the last sequence's sums are read
        for (int32_t s = wave; s < a.segments; s += kWaves) {
            const Mass m = sum_segment(a, rows, s);
            if (lane == 0) sums[s] = m;
        }
        __syncthreads();
        if (wave == 0) write_result(a, b, k, draw(a, rows, sums, u), lane, kWave);
    }
}

// sums[b][segment] of the masses; blockIdx.y walks the segments, each wave of it `each` of them.  Bound
// by memory where there are many sequences: 256 x 4 drafts x 141043 f32 take 51 us (some 246 MB, 4.8 TB/s); by the
// accept tests' two dependent loads and the launch where there are few (1 x 4 x 141043: 4.8 us).
template <class T>
__global__ __launch_bounds__(kVerifyBlock) void verify_sums_kernel(VerifyArgs a)
{
    const int32_t lane = (int32_t)threadIdx.x % kWave;
    const int32_t s0 = (int32_t)(blockIdx.y * (kVerifyBlock / kWave) + threadIdx.x / kWave) * a.each;
    const int32_t s1 = min(a.segments, s0 + a.each);
    for (int64_t b = blockIdx.x; b < a.sequences; b += gridDim.x) {
        if (s0 >= s1) break;
        int32_t n;
        const int32_t k = count_accepted<T>(a, b, n);
        if (s0 == 0 && lane == 0) a.found[b] = make_int2(k, n);
        const DrawRows<T> rows(a, b, k, n);
        for (int32_t s = s0; s < s1; ++s) {
            const Mass m = sum_segment(a, rows, s);
            if (lane == 0) a.sums[b * a.segments + s] = m;
        }
    }
}

// A wave a sequence: 4 to 5 us, the latency of its loads one after the other
template <class T>
__global__ __launch_bounds__(kWave) void verify_draw_kernel(VerifyArgs a)
{
    for (int64_t b = blockIdx.x; b < a.sequences; b += gridDim.x) {
        const int2 found = a.found[b];
        const DrawRows<T> rows(a, b, found.x, found.y);
        const int64_t token = draw(a, rows, a.sums + b * a.segments, (double)a.draw_u[b]);
        write_result(a, b, found.x, token, (int32_t)threadIdx.x, kWave);
    }
}

static int64_t verify_segments(const lda_draft_rows* d)
{
    return d->classes <= kDirectClasses ? 0 : ((int64_t)d->classes + kSegment - 1) / kSegment;
}
// One launch costs the host some 4 us less than two, and rows of up to 80 KB take a workgroup hardly longer
// than the two kernels (20000 f32, 2 steps: 1 sequence 8.1 us, in two 7.3; 64: 10.7 and 9.4; 256: 12.9 and 13.2; but
// 512: 23 and 20; 60000 f32, 64 sequences: 18 and 11).
static bool row_in_one(const lda_draft_rows* d)
{
    return (int64_t)d->classes * (int64_t)type_bytes(d->probs_type) <= kRowBytes && d->sequences <= 256;
}
static int64_t verify_bytes(const lda_draft_rows* d)
{
    const int64_t segments = verify_segments(d);
    return segments == 0 || row_in_one(d) ? 0 : d->sequences * (segments * (int64_t)sizeof(Mass) + (int64_t)sizeof(int2));
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
static void launch_verify_typed(VerifyArgs& a, hipStream_t stream)
{
    const unsigned gx = (unsigned)(a.sequences < (1 << 20) ? a.sequences : (1 << 20));
    if (a.segments == 0) {
        verify_direct_kernel<T><<<gx, kVerifyBlock, 0, stream>>>(a);
        return;
    }
    if (a.sums == nullptr) {
        verify_row_kernel<T><<<gx, kRowBlock, 0, stream>>>(a);
        return;
    }
    // some 8 workgroups a CU, as every wave begins with the accept tests
    constexpr int64_t kWaves = kVerifyBlock / kWave, kMost = 256 * 8;
    int64_t each = a.sequences * a.segments / (kMost * kWaves);
    const int64_t least = (a.segments + 65535 * kWaves - 1) / (65535 * kWaves);
    if (each < least) each = least;
    if (each < 1) each = 1;
    a.each = (int32_t)(each < a.segments ? each : a.segments);
    const unsigned gy = (unsigned)((a.segments + kWaves * a.each - 1) / (kWaves * a.each));
    verify_sums_kernel<T><<<dim3(gx, gy), kVerifyBlock, 0, stream>>>(a);
    verify_draw_kernel<T><<<gx, kWave, 0, stream>>>(a);
}

}  // namespace lda

using namespace lda;

extern "C" {

int64_t lda_verify_workspace(const lda_draft_rows* d)
try {
    const int rc = check_verify(d, "lda_verify_workspace");
    if (rc != LDA_OK) return rc;
    return verify_bytes(d);
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
    a.segments = (int32_t)verify_segments(d);
    const int64_t need = verify_bytes(d);
    if (need > 0 && (!d->workspace || d->workspace_bytes < need || !aligned_to(d->workspace, 16)))
        return fail(nullptr, LDA_ERR_ARG, "%s: needs a workspace of %lld bytes, aligned to 16", call, (long long)need);
    if (need > 0) {
        a.sums = static_cast<Mass*>(d->workspace);
        a.found = reinterpret_cast<int2*>(a.sums + a.sequences * a.segments);
    }
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
