// Distillation from a teacher's top logits: the loss of every row and its gradient (the formulas
// stand at lda_distill_rows in lda_mi355x.h).
//
// A row's softmax needs its largest logit m and s = sum exp((S - m) / T), both found in one pass with
// the running form: a thread keeps (m, s) of what it has seen and scales s when m grows, the pairs
// of threads, waves and slices join the same way.  The teacher's masses touch only k of the V
// classes, so they are evaluated apart: the loss gathers k logits, the gradient is
// written as if the teacher had its floor r everywhere and the k places are overwritten.
#include "rows.hpp"

namespace lda {

constexpr int32_t kMostSlots = 1024;

// What a slice of a row tells about its softmax.  ssum and ninf (finite logits summed, logits of
// -infinity counted) are only there where the teacher has a floor.
struct RowPart {
    float m, s;
    double ssum;
    int32_t ninf, pad;
};

struct DistillArgs {
    int64_t rows;
    int32_t V, k;
    const void* logits;
    int64_t logits_stride;
    const void* ids;
    int64_t ids_stride;
    const void* teacher;
    int64_t teacher_stride;
    const float* log_norm;
    const float* weight;
    int64_t weight_stride;
    int32_t ids_type, teacher_type;
    float T, c;             // c = log2(e) / T
    int32_t slices;         // of a row, slice_chunks chunks of 16 bytes each
    int32_t slice_chunks;
    RowPart* parts;         // [rows][slices]; NULL: a row is one slice
    const float* stats_in;  // [rows][2]: the softmax is known
    float* loss;
    float* stats;
    void* grad;
    int64_t grad_stride;
};

// exp((x - m) / T) with exp2 in hardware; m finite or the row's own infinity or NaN
__device__ __forceinline__ float exp_above(float x, float m, float c)
{
    return __builtin_amdgcn_exp2f((x - m) * c);
}
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }

__device__ __forceinline__ void join(float& m, float& s, float m2, float s2, float c)
{
    const float top = fmaxf(m, m2), base = base_of(top);
    s = s * exp_above(m, base, c) + s2 * exp_above(m2, base, c);
    m = top;
}

template <int BLOCK>
__device__ __forceinline__ void block_join(float& m, float& s, float c, float2* part)
{
#pragma unroll
    for (int d = kWave / 2; d > 0; d >>= 1) {
        const float m2 = __shfl_xor(m, d, kWave), s2 = __shfl_xor(s, d, kWave);
        join(m, s, m2, s2, c);
    }
    if (BLOCK == kWave) return;
    __syncthreads();
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = make_float2(m, s);
    __syncthreads();
    m = part[0].x;
    s = part[0].y;
#pragma unroll
    for (int w = 1; w < BLOCK / kWave; ++w) join(m, s, part[w].x, part[w].y, c);
}

// The teacher's slots in LDS.  A slot without a mass has id -1.
struct TeacherSlots {
    int32_t* id;   // [k]
    float* p;      // [k] mass of the slot
    float* all;    // [k] mass of the slot's class (all its slots)
    float* logit;  // [k] the student's logit there
    double* head;  // sum of p, sum of p log p
    __device__ __forceinline__ TeacherSlots(unsigned char* lds, int32_t k)
    {
        head = reinterpret_cast<double*>(lds);
        id = reinterpret_cast<int32_t*>(lds + 16);
        p = reinterpret_cast<float*>(id + k);
        all = p + k;
        logit = all + k;
    }
};
inline size_t slots_lds(int32_t k) { return 16 + 16 * (size_t)k; }

// One wave's work: ids, masses, their sum and their entropy.
__device__ void read_teacher(const DistillArgs& a, int64_t row, const TeacherSlots& ts)
{
    const int lane = threadIdx.x % kWave;
    const int64_t ids0 = row * a.ids_stride, t0 = row * a.teacher_stride;
    const double inv_t = 1.0 / (double)a.T;
    float top = -INFINITY;
    for (int32_t j = lane; j < a.k; j += kWave) {
        const int64_t id = index_at(a.ids, a.ids_type, ids0 + j);
        const bool full = id >= 0 && id < a.V;
        const float t = full ? element_at(a.teacher, a.teacher_type, t0 + j) : -INFINITY;
        ts.id[j] = full ? (int32_t)id : -1;
        ts.p[j] = t;
        top = fmaxf(top, t);
    }
    top = wave_reduce(top, [](float x, float y) { return fmaxf(x, y); });
    double shift, log_sum = 0.0;
    if (a.log_norm) {
        shift = (double)a.log_norm[row];
    } else {
        shift = (double)base_of(top) * inv_t;
        double sum = 0.0;
        for (int32_t j = lane; j < a.k; j += kWave) sum += exp((double)ts.p[j] * inv_t - shift);
        sum = wave_sum(sum);
        log_sum = sum == 0.0 ? 0.0 : log(sum);
    }
    double mass = 0.0, entropy = 0.0;
    for (int32_t j = lane; j < a.k; j += kWave) {
        const double log_p = (double)ts.p[j] * inv_t - shift - log_sum;
        const double p = exp(log_p);
        ts.p[j] = (float)p;
        mass += p;
        if (p != 0.0) entropy += p * log_p;
    }
    mass = wave_sum(mass);
    entropy = wave_sum(entropy);
    if (lane == 0) {
        ts.head[0] = mass;
        ts.head[1] = entropy;
    }
}

// (m, s) and the floor's sums of chunks [c0, c1) of a row
template <class T, bool REST, int BLOCK>
__device__ __forceinline__ void scan_chunks(const ChunkedRow<T>& r, int32_t c0, int32_t c1, float c, float& m,
                                            float& s, double& ssum, int32_t& ninf)
{
    constexpr int E = Row<T>::kChunk;
    m = -INFINITY;
    s = 0.0f;
    ssum = 0.0;
    ninf = 0;
    for (int32_t i = c0 + (int32_t)threadIdx.x; i < c1; i += BLOCK) {
        float x[E];
        r.load(i, x, -INFINITY);
        float top = x[0];
#pragma unroll
        for (int e = 1; e < E; ++e) top = fmaxf(top, x[e]);
        if (top > m) {
            s *= exp_above(m, top, c);
            m = top;
        }
        const float base = base_of(m);
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) sum += exp_above(x[e], base, c);
        s += sum;
        if (REST) {
            const int64_t v = r.first(i);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool none = x[e] == -INFINITY;
                ssum += none ? 0.0 : (double)x[e];
                ninf += none && v + e >= 0 && v + e < r.V;
            }
        }
    }
}

// One workgroup a row or a slice of it.  FORM: kPart writes the slice's RowPart; kWhole has the
// row's softmax itself, kJoin takes it from the parts or from stats_in; both then do what of
// loss, stats and gradient is asked for.
enum DistillForm { kPart, kWhole, kJoin };

template <class T, bool REST, int BLOCK, int FORM>
__global__ __launch_bounds__(BLOCK) void distill_kernel(DistillArgs a)
{
    constexpr int E = Row<T>::kChunk;
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ float2 part2[BLOCK / kWave];
    __shared__ double partd[BLOCK / kWave];
    __shared__ int32_t parti[BLOCK / kWave];
    const TeacherSlots ts(lds, a.k);
    const int32_t tid = (int32_t)threadIdx.x, slice = (int32_t)blockIdx.y;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const ChunkedRow<T> r(static_cast<const T*>(a.logits) + row * a.logits_stride, a.V);
        const float w = a.weight ? a.weight[row * a.weight_stride] : 1.0f;
        const int32_t c0 = slice * a.slice_chunks;
        const int32_t c1 = (int32_t)min((int64_t)r.chunks(), (int64_t)c0 + a.slice_chunks);
        bool out = a.grad && w == 0.0f;  // left out
        float m = -INFINITY, s = 0.0f;
        double ssum = 0.0;
        int32_t ninf = 0;
        if (FORM != kPart) {
            if (tid < kWave) read_teacher(a, row, ts);
        }
        if (FORM != kJoin && !out) {
            scan_chunks<T, REST, BLOCK>(r, c0, c1, a.c, m, s, ssum, ninf);
            block_join<BLOCK>(m, s, a.c, part2);
            if (REST) {
                ssum = block_sum<BLOCK>(ssum, partd);
                ninf = block_sum<BLOCK>(ninf, parti);
            }
        }
        if (FORM == kPart) {
            if (tid == 0 && !out) a.parts[row * a.slices + slice] = RowPart{m, s, ssum, ninf, 0};
            continue;
        }
        if (FORM == kJoin && !out) {
            if (a.stats_in) {
                m = a.stats_in[2 * row];
                s = a.stats_in[2 * row + 1];
            } else {
                m = -INFINITY;
                s = 0.0f;
                for (int32_t q = 0; q < a.slices; ++q) {  // every thread the same: few, and in cache
                    const RowPart part = a.parts[row * a.slices + q];
                    join(m, s, part.m, part.s, a.c);
                    ssum += part.ssum;
                    ninf += part.ninf;
                }
            }
        }
        __syncthreads();
        const double mass = ts.head[0], entropy = ts.head[1];
        // the slots: the class's whole mass, the student's logit, and the loss's sums
        const bool first_slice = slice == 0;
        const bool want_loss = a.loss && first_slice;
        const double inv_t = 1.0 / (double)a.T;
        const double base = (double)base_of(m), log_s = log((double)s);
        double cross = 0.0, named_sum = 0.0;
        int32_t named = 0, named_inf = 0;
        bool infinite = false;
        if (!out) {
            for (int32_t j = tid; j < a.k; j += BLOCK) {
                const int32_t id = ts.id[j];
                if (id < 0) continue;
                const float x = Row<T>::one(r.p + id);
                ts.logit[j] = x;
                if (REST || a.grad) {
                    float all = 0.0f;
                    bool first = true;
                    for (int32_t i = 0; i < a.k; ++i) {
                        if (ts.id[i] != id) continue;
                        all += ts.p[i];
                        first = first && i >= j;
                    }
                    ts.all[j] = all;
                    if (REST && first) {
                        ++named;
                        if (x == -INFINITY) ++named_inf;
                        else named_sum += (double)x;
                    }
                }
                const double p = (double)ts.p[j];
                if (p != 0.0) {
                    if (x == -INFINITY) infinite = true;
                    else cross += p * (((double)x - base) * inv_t - log_s);
                }
            }
        }
        double floor_mass = 0.0;
        int32_t others = 0;
        if (REST) {
            named = block_sum<BLOCK>(named, parti);
            others = a.V - named;
            const double left = 1.0 - mass;
            floor_mass = others > 0 && left > 0.0 ? left / (double)others : 0.0;
        }
        const double all_mass = mass + floor_mass * (double)others;
        if (want_loss) {
            cross = block_sum<BLOCK>(cross, partd);
            infinite = block_sum<BLOCK>((int32_t)infinite, parti) != 0;
            double rest = 0.0;
            if (REST) {
                named_sum = block_sum<BLOCK>(named_sum, partd);
                named_inf = block_sum<BLOCK>(named_inf, parti);
                if (floor_mass > 0.0) {
                    rest = floor_mass * ((double)others * (log(floor_mass) + log_s) -
                                         (ssum - named_sum - (double)others * base) * inv_t);
                    infinite = infinite || ninf > named_inf;
                }
            }
            if (tid == 0) {
                double loss = infinite ? (double)INFINITY : (double)a.T * (double)a.T * (entropy - cross + rest);
                if (!(s == s) || !(mass == mass)) loss = (double)NAN;
                if (out || all_mass == 0.0) loss = 0.0;
                a.loss[row] = (float)loss;
                if (a.stats) {
                    a.stats[2 * row] = m;
                    a.stats[2 * row + 1] = s;
                }
            }
        }
        if (a.grad) {
            out = out || all_mass == 0.0;
            T* g = static_cast<T*>(a.grad) + row * a.grad_stride;
            const bool together = (((uintptr_t)g ^ (uintptr_t)r.p) & 15u) == 0;
            const float wt = w * a.T, b = base_of(m);
            const float scale = s == 0.0f ? 0.0f : (float)all_mass * wt / s, low = (float)floor_mass * wt;
            for (int32_t i = c0 + tid; i < c1; i += BLOCK) {
                float x[E];
                if (!out) {
                    r.load(i, x, -INFINITY);
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] = exp_above(x[e], b, a.c) * scale - low;
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] = 0.0f;
                }
                const int64_t v = r.first(i);
                if (together && r.whole(v)) {
                    *reinterpret_cast<uint4*>(g + v) = Row<T>::pack(x);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (v + e >= 0 && v + e < a.V) g[v + e] = Row<T>::from(x[e]);
                }
            }
            __syncthreads();  // the places of the slots are written again, by other threads
            if (!out) {
                const int64_t v0 = r.first(c0), v1 = r.first(c1);
                for (int32_t j = tid; j < a.k; j += BLOCK) {
                    const int32_t id = ts.id[j];
                    if (id < 0 || id < v0 || id >= v1) continue;
                    g[id] = Row<T>::from(exp_above(ts.logit[j], b, a.c) * scale - ts.all[j] * wt);
                }
            }
        }
        __syncthreads();  // the LDS is the next row's
    }
}

constexpr int kBlock = 256;
constexpr int32_t kSliceBytes = 32768;

static int32_t distill_slices(const lda_distill_rows* d)
{
    const int64_t bytes = (int64_t)d->classes * (int64_t)type_bytes(d->logits_type) + 16;
    if (d->rows >= 1024) return 1;
    const int64_t most = (bytes + kSliceBytes - 1) / kSliceBytes;
    return (int32_t)(most < 1 ? 1 : most > 1024 ? 1024 : most);
}

static int check_distill(const lda_distill_rows* d, const char* call)
{
    if (!d) return fail(nullptr, LDA_ERR_ARG, "%s: NULL rows", call);
    for (int32_t r : d->reserved)
        if (r != 0) return fail(nullptr, LDA_ERR_ARG, "%s: reserved fields must be zero", call);
    if (d->rows < 0 || d->classes < 1 || d->slots < 0)
        return fail(nullptr, LDA_ERR_ARG, "%s: rows >= 0, classes >= 1, slots >= 0 needed", call);
    if (!known_type(d->logits_type) || !known_type(d->teacher_type) || !known_index(d->ids_type))
        return fail(nullptr, LDA_ERR_ARG, "%s: unknown type", call);
    if (!(d->temperature >= 1.0f / 1024.0f) || !(d->temperature <= 1024.0f))
        return fail(nullptr, LDA_ERR_ARG, "%s: temperature must lie in [1/1024, 1024]", call);
    if (d->slots > kMostSlots)
        return fail(nullptr, LDA_ERR_UNSUPPORTED, "%s: at most %d slots", call, kMostSlots);
    if (d->rows == 0) return LDA_OK;
    if (!d->logits || (d->slots > 0 && (!d->ids || !d->teacher)))
        return fail(nullptr, LDA_ERR_ARG, "%s: NULL pointer", call);
    if (!aligned_to(d->logits, type_bytes(d->logits_type)) || !aligned_to(d->teacher, type_bytes(d->teacher_type)) ||
        !aligned_to(d->ids, index_bytes(d->ids_type)) || !aligned_to(d->log_norm, 4) || !aligned_to(d->weight, 4))
        return fail(nullptr, LDA_ERR_ARG, "%s: a pointer is not aligned to its type", call);
    return LDA_OK;
}

template <class T, bool REST>
static void launch_distill_typed(const DistillArgs& a, hipStream_t stream)
{
    const unsigned gx = (unsigned)(a.rows < (1 << 20) ? a.rows : (1 << 20));
    const dim3 one(gx, 1), all(gx, (unsigned)a.slices);
    const size_t lds = slots_lds(a.k);
    if (a.stats_in) {
        distill_kernel<T, REST, kBlock, kJoin><<<all, kBlock, lds, stream>>>(a);
    } else if (a.slices == 1) {
        distill_kernel<T, REST, kBlock, kWhole><<<one, kBlock, lds, stream>>>(a);
    } else {
        distill_kernel<T, REST, kBlock, kPart><<<all, kBlock, lds, stream>>>(a);
        distill_kernel<T, REST, kBlock, kJoin><<<a.grad ? all : one, kBlock, lds, stream>>>(a);
    }
}

static int launch_distill(const lda_distill_rows* d, const char* call, float* loss, float* stats,
                          const float* stats_in, void* grad, int64_t grad_stride)
{
    if (d->rows == 0) return LDA_OK;
    if (!aligned_to(loss, 4) || !aligned_to(stats, 4) || !aligned_to(stats_in, 4) ||
        !aligned_to(grad, type_bytes(d->logits_type)))
        return fail(nullptr, LDA_ERR_ARG, "%s: a pointer is not aligned to its type", call);
    DistillArgs a{};
    a.rows = d->rows;
    a.V = d->classes;
    a.k = d->slots;
    a.logits = d->logits;
    a.logits_stride = d->logits_stride;
    a.ids = d->ids;
    a.ids_stride = d->ids_stride;
    a.teacher = d->teacher;
    a.teacher_stride = d->teacher_stride;
    a.log_norm = d->log_norm;
    a.weight = grad ? d->weight : nullptr;
    a.weight_stride = d->weight_stride;
    a.ids_type = d->ids_type;
    a.teacher_type = d->teacher_type;
    a.T = d->temperature;
    a.c = (float)(1.44269504088896340736 / (double)d->temperature);
    a.loss = loss;
    a.stats = stats;
    a.stats_in = stats_in;
    a.grad = grad;
    a.grad_stride = grad_stride;
    a.slices = distill_slices(d);
    const int64_t chunk = 16 / (int64_t)type_bytes(d->logits_type);
    const int64_t chunks = (d->classes + chunk - 1) / chunk + 1;  // wherever the row starts
    a.slice_chunks = (int32_t)((chunks + a.slices - 1) / a.slices);
    if (a.slices > 1 && !stats_in) {
        const int64_t need = a.rows * a.slices * (int64_t)sizeof(RowPart);
        if (!d->workspace || d->workspace_bytes < need || !aligned_to(d->workspace, 16))
            return fail(nullptr, LDA_ERR_ARG, "%s: needs a workspace of %lld bytes, aligned to 16", call, (long long)need);
        a.parts = static_cast<RowPart*>(d->workspace);
    }
    const hipStream_t stream = static_cast<hipStream_t>(d->hip_stream);
    const bool rest = d->log_norm != nullptr;
    switch (d->logits_type) {
    case LDA_F32:
        rest ? launch_distill_typed<float, true>(a, stream) : launch_distill_typed<float, false>(a, stream);
        break;
    case LDA_F16:
        rest ? launch_distill_typed<__half, true>(a, stream) : launch_distill_typed<__half, false>(a, stream);
        break;
    default:
        rest ? launch_distill_typed<__hip_bfloat16, true>(a, stream) : launch_distill_typed<__hip_bfloat16, false>(a, stream);
    }
    LDA_HIP(static_cast<lda_ctx*>(nullptr), hipGetLastError());
    return LDA_OK;
}

}  // namespace lda

using namespace lda;

extern "C" {

int64_t lda_distill_workspace(const lda_distill_rows* d)
try {
    const int rc = check_distill(d, "lda_distill_workspace");
    if (rc != LDA_OK) return rc;
    const int32_t slices = distill_slices(d);
    return slices == 1 ? 0 : d->rows * slices * (int64_t)sizeof(RowPart);
} catch (...) {
    return LDA_ERR_OOM;
}

int lda_distill_loss(const lda_distill_rows* d, float* loss, float* stats)
try {
    const int rc = check_distill(d, "lda_distill_loss");
    if (rc != LDA_OK) return rc;
    if (d->rows > 0 && !loss) return fail(nullptr, LDA_ERR_ARG, "lda_distill_loss: NULL loss");
    return launch_distill(d, "lda_distill_loss", loss, stats, nullptr, nullptr, 0);
} catch (...) {
    return LDA_ERR_OOM;
}

int lda_distill_grad(const lda_distill_rows* d, const float* stats, void* grad, int64_t grad_stride)
try {
    const int rc = check_distill(d, "lda_distill_grad");
    if (rc != LDA_OK) return rc;
    if (d->rows > 0 && (!stats || !grad)) return fail(nullptr, LDA_ERR_ARG, "lda_distill_grad: NULL pointer");
    if (d->rows > 1 && grad_stride < d->classes)
        return fail(nullptr, LDA_ERR_ARG, "lda_distill_grad: rows of the gradient overlap");
    return launch_distill(d, "lda_distill_grad", nullptr, nullptr, stats, grad, grad_stride);
} catch (...) {
    return LDA_ERR_OOM;
}

int lda_distill_step(const lda_distill_rows* d, float* loss, void* grad, int64_t grad_stride)
try {
    const int rc = check_distill(d, "lda_distill_step");
    if (rc != LDA_OK) return rc;
    if (d->rows > 0 && (!loss || !grad)) return fail(nullptr, LDA_ERR_ARG, "lda_distill_step: NULL pointer");
    if (d->rows > 1 && grad_stride < d->classes)
        return fail(nullptr, LDA_ERR_ARG, "lda_distill_step: rows of the gradient overlap");
    return launch_distill(d, "lda_distill_step", loss, nullptr, nullptr, grad, grad_stride);
} catch (...) {
    return LDA_ERR_OOM;
}

}  // extern "C"
