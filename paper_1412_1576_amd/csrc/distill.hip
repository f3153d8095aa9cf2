// Distillation from a teacher's top logits: the loss of every row and its gradient (the formulas
// stand at lda_distill_rows in lda_mi355x.h).
//
// A row's softmax needs a base m near its largest logit and s = sum exp((S - m) / T), both found in
// one pass: a thread keeps (m, s) of what it has seen and scales s only when a logit lies far above m; the
// pairs of threads, waves and slices join.  The teacher touches k of the V classes: the loss
// gathers k logits, the gradient is written as if the teacher had its floor everywhere and
// the k places are written again.
//
// Rows that fit a workgroup's registers are read from memory once, loss and gradient both
// (distill_rows_kernel).  Longer rows, and long ones where there are too few to fill the GPU, are cut
// into slices: distill_part_kernel, then distill_join_kernel, which reads them a second time for the gradient.
#include "softmax_rows.hpp"

namespace lda {

constexpr int32_t kMostSlots = 1024;
constexpr int kPartBlock = 256;
constexpr int kSliceLoads = 8;                                // 16-byte loads of a thread in flight
constexpr int32_t kSliceChunks = kPartBlock * kSliceLoads;    // 32 KB
constexpr int32_t kStatFloats = 8;
constexpr float kFar = 16.0f;  // a base is left where it is until a logit exceeds it by this, in powers of 2
constexpr float kLeastSum = -0x1p100f;  // sums of 8 differences from the base above this have none near the end of 32 bits

// What a slice of a row tells about its softmax.  scaled_sum (of c (S - m) over the logits above -infinity but for
// deep ones that have a slot) and n (their number) are only there where the teacher has a floor.
struct RowPart {
    float m, s;
    double scaled_sum;
    int32_t n, pad;
};

// What the slots say: masses are exp(t / T - z), their sum; the floor of the other classes and their
// number.
struct TeacherPart {
    double mass, z, floor;
    int32_t others, pad;
};

// A row's softmax and teacher, all that its gradient needs
struct RowStats {
    float m, s, mass, floor;
    double z;
};
static_assert(sizeof(RowStats) <= kStatFloats * sizeof(float), "stats");

struct DistillArgs {
    int64_t rows, row0;     // a launch's rows begin with row0
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
    int32_t slices;         // of kSliceChunks chunks each
    RowPart* parts;         // [rows][slices]
    TeacherPart* teachers;  // [rows]
    const float* stats_in;  // [rows][kStatFloats]
    float* loss;
    float* stats;
    void* grad;
    int64_t grad_stride;
};

// What a sum of c (S - from) over n logits is with another base.  Sums of the logits themselves would lose
// everything in a row of the type's lowest value, whose differences are 0.
__device__ __forceinline__ double rebased(double scaled_sum, int32_t n, float from, float to, float c)
{
    return n > 0 ? scaled_sum + (double)n * (((double)from - (double)to) * (double)c) : scaled_sum;
}

// Whether any thread of the workgroup has something, in two steps with the barriers of a block_join between
// them (__syncthreads_or takes 1 us)
template <int BLOCK>
__device__ __forceinline__ void put_any(int has, uint32_t* part)
{
    const uint64_t some = __ballot(has);
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = some != 0;
    if (BLOCK == kWave) wave_lds_order();
}
template <int BLOCK>
__device__ __forceinline__ bool get_any(const uint32_t* part)
{
    return __ballot(part[threadIdx.x % (BLOCK / kWave)] != 0) != 0;
}

// c (S - base) over classes without a slot whose logit lies above -infinity, and their number: what the floor's part
// of the loss needs.  Every class is added while the row is read, and those that have a slot are taken out when
// the slots are there.  A mask's large number, added and taken out, would leave nothing of the others: logits
// below `deep` are passed over and looked at again, with the bits of the classes that have a slot, in rows that have any
// (2048 x 10000 f32: 40 us without, 44 with a fifth of a row masked, 46 with each second class; masks of -infinity 41).
struct BesideSums {
    double sum;
    int32_t n;

    __device__ __forceinline__ void add(float x, float base, float c)
    {
        if (x == -INFINITY) return;
        sum += ((double)x - (double)base) * (double)c;
        ++n;
    }
    __device__ __forceinline__ void take_out(float x, float deep, float base, float c)
    {
        if (!(x >= deep)) return;
        sum -= ((double)x - (double)base) * (double)c;
        --n;
    }
    template <int N>
    __device__ __forceinline__ void add_deep(const float (&x)[N], float deep, float base, float c, uint32_t named)
    {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (x[e] < deep && !(named >> e & 1u)) add(x[e], base, c);
    }
};
// What is taken out leaves roundings of its chunk's sum in 32 bits behind, some 2^-24 of 8 times this, times the
// floor.  In rows of a few thousand classes most may have a slot, in longer ones one of ten.
constexpr float kDeepOfShort = -64.0f, kDeepOfLong = -1024.0f;

// Which classes of COUNT chunks, from chunk c0 on, and of the extras have a slot: a byte a chunk, a bit an
// element
template <int COUNT>
struct NamedBits {
    static constexpr int kWords = (COUNT + 3) / 4 + 1;  // the extras' behind the chunks'
    uint32_t word[kWords];

    __device__ __forceinline__ void clear(int32_t thread, int32_t threads)
    {
        for (int32_t i = thread; i < kWords; i += threads) word[i] = 0;
    }
    template <class T>
    __device__ __forceinline__ void mark(const SplitRow<T>& r, int32_t c0, int32_t id)
    {
        constexpr int E = SplitRow<T>::E;
        const int32_t at = id - r.head, chunk = at / E - c0;
        if (at < 0 || at >= r.whole * E) {
            atomicOr(&word[kWords - 1], 1u << (at < 0 ? id : id - r.whole * E));
        } else if (chunk >= 0 && chunk < COUNT) {
            atomicOr(&word[chunk / 4], 1u << (chunk % 4 * 8 + at % E));
        }
    }
    __device__ __forceinline__ uint32_t of_chunk(int32_t i) const { return reinterpret_cast<const uint8_t*>(word)[i]; }
    __device__ __forceinline__ uint32_t of_extra(int32_t i) const { return word[kWords - 1] >> i & 1u; }
};

// The running form of one thread's share; REST: with the sums beside the slots, of the same base
template <bool REST>
struct Running {
    float m = -INFINITY, s = 0.0f;
    BesideSums beside{};
    int any_deep = 0;

    template <int N>
    __device__ __forceinline__ void add(const float (&x)[N], float c, float deep)
    {
        float top = x[0];
#pragma unroll
        for (int e = 1; e < N; ++e) top = fmaxf(top, x[e]);
        if ((top - m) * c > kFar) {
            s *= exp_above(m, top, c);
            if (REST) beside.sum = rebased(beside.sum, beside.n, m, top, c);
            m = top;
        }
        const float base = base_of(m);
        float y[N], sum = 0.0f;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            y[e] = (x[e] - base) * c;
            sum += __builtin_amdgcn_exp2f(y[e]);
        }
        s += sum;
        if (REST) {
            float least = x[0], some = y[0];
#pragma unroll
            for (int e = 1; e < N; ++e) {
                least = fminf(least, x[e]);
                some += y[e];
            }
            if (least >= deep && some > kLeastSum) {
                beside.sum += (double)some;
                beside.n += N;
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (x[e] >= deep) beside.add(x[e], base, c);
                    else any_deep |= x[e] != -INFINITY;
                }
            }
        }
    }
};

// A row's slots in LDS
struct Slots {
    TeacherPart* head;
    int32_t* id;  // -1: empty
    float* p;     // mass of the slot
    float* t;     // the teacher's logit
    float* x;     // the student's
    int32_t* table;  // [2^log2 >= 2 k] for find_twice, with k > kPairs
    int32_t* twice;
    __device__ __forceinline__ Slots(unsigned char* lds, int32_t k)
    {
        const int32_t n = (k + 3) / 4 * 4;
        head = reinterpret_cast<TeacherPart*>(lds);
        id = reinterpret_cast<int32_t*>(lds + sizeof(TeacherPart));
        p = reinterpret_cast<float*>(id + n);
        t = p + n;
        x = t + n;
        twice = reinterpret_cast<int32_t*>(x + n);
        table = twice + 1;
    }
};
static_assert(sizeof(TeacherPart) % 16 == 0, "vectors behind it");
// Up to so many slots, slots of one class are found by comparing all with all.
constexpr int32_t kPairs = 64;
__host__ __device__ __forceinline__ int32_t table_bits(int32_t k) { return 33 - __builtin_clz((uint32_t)k - 1u); }  // k >= 2
inline size_t slots_lds(int32_t k)
{
    return sizeof(TeacherPart) + 16 * ((size_t)(k + 3) / 4 * 4) + (k > kPairs ? 4 + ((size_t)4 << table_bits(k)) : 0);
}

// exp(t / T - z): none for t = -infinity, which empty slots have, also where the norm is -infinity
__device__ __forceinline__ double slot_mass(float t, double inv_t, double z)
{
    return t == -INFINITY ? 0.0 : exp((double)t * inv_t - z);
}

// One wave's work: ids, logits of both sides and masses of a row's slots.
template <class T>
__device__ __forceinline__ void read_teacher(const DistillArgs& a, int64_t row, const T* logits, const Slots& slots)
{
    const int lane = threadIdx.x % kWave;
    const double inv_t = 1.0 / (double)a.T;
    float top = -INFINITY;
    double z = a.log_norm ? (double)a.log_norm[row] : 0.0;
    for (int32_t j = lane; j < (a.k + 3) / 4 * 4; j += kWave) {
        int32_t id = -1;
        float t = -INFINITY;
        if (j < a.k) {
            const int64_t at = index_at(a.ids, a.ids_type, row * a.ids_stride + j);
            t = element_at(a.teacher, a.teacher_type, row * a.teacher_stride + j);
            if (at >= 0 && at < a.V) id = (int32_t)at;
            else t = -INFINITY;
        }
        slots.id[j] = id;
        slots.t[j] = t;
        slots.x[j] = id >= 0 ? Row<T>::one(logits + id) : 0.0f;
        top = fmaxf(top, t);
    }
    double mass;
    if (a.log_norm) {
        mass = 0.0;
        for (int32_t j = lane; j < (a.k + 3) / 4 * 4; j += kWave) {
            const double p = slot_mass(slots.t[j], inv_t, z);
            slots.p[j] = (float)p;
            mass += p;
        }
        mass = wave_sum(mass);
    } else {
        top = base_of(wave_max(top));
        double sum = 0.0;
        for (int32_t j = lane; j < a.k; j += kWave) sum += exp(((double)slots.t[j] - (double)top) * inv_t);
        sum = wave_sum(sum);
        z = (double)top * inv_t + (sum == 0.0 ? 0.0 : log(sum));
        for (int32_t j = lane; j < (a.k + 3) / 4 * 4; j += kWave) slots.p[j] = (float)slot_mass(slots.t[j], inv_t, z);
        mass = sum == 0.0 ? 0.0 : sum / sum;  // 1, or what is not a number
    }
    if (mass == (double)INFINITY) mass = (double)NAN;  // so that all of loss and gradient is
    if (lane == 0) {
        slots.head->mass = mass;
        slots.head->z = z;
    }
}

// Does any class have two slots?  The whole workgroup; the answer is the same in every thread.  Nearly
// always none has, and then no slot needs to look at the others: 256 slots of 4000 rows of 700 classes take 19 us, 41 when
// they do (8 slots: 14); 64 slots 15.0, by the table 15.6.
template <int BLOCK>
__device__ __forceinline__ bool find_twice(const Slots& slots, int32_t k)
{
    if (k <= kPairs) return true;  // they may
    const int32_t tid = (int32_t)threadIdx.x, bits = table_bits(k), size = 1 << bits;
    for (int32_t i = tid; i < size; i += BLOCK) slots.table[i] = -1;
    if (tid == 0) *slots.twice = 0;
    __syncthreads();
    for (int32_t j = tid; j < k; j += BLOCK) {
        const int32_t id = slots.id[j];
        if (id < 0) continue;
        int32_t h = (int32_t)(((uint32_t)id * 0x9E3779B1u) >> (32 - bits));
        for (;;) {  // half the table stays empty
            const int32_t other = atomicCAS(&slots.table[h], -1, id);
            if (other == -1) break;
            if (other == id) {
                atomicOr(slots.twice, 1);
                break;
            }
            h = (h + 1) & (size - 1);
        }
    }
    __syncthreads();
    return *slots.twice != 0;
}

// Is slot j the first of its class, and what is the mass of all of them?  Read from LDS by
// the whole workgroup in step, four at a time.
__device__ __forceinline__ bool first_of_class(const Slots& slots, bool twice, int32_t k, int32_t j, int32_t id, float& all)
{
    if (!twice) {
        all = slots.p[j];
        return true;
    }
    all = 0.0f;
    bool first = true;
    for (int32_t i = 0; i < k; i += 4) {
        const int4 other = *reinterpret_cast<const int4*>(slots.id + i);
        const float4 p = *reinterpret_cast<const float4*>(slots.p + i);
        const int32_t o[4] = {other.x, other.y, other.z, other.w};
        const float q[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool same = o[e] == id;
            all += same ? q[e] : 0.0f;
            first = first && !(same && i + e < j);
        }
    }
    return first;
}

__device__ __forceinline__ double floor_of(double mass, int32_t others)
{
    const double left = 1.0 - mass;
    return others > 0 && left > 0.0 ? left / (double)others : 0.0;
}

// The factors of a row's gradient: w T (M q - floor), and in the slots' places w T (M q - P)
struct Gradient {
    float base, c, scale, low, wt;
    __device__ __forceinline__ Gradient(float m, float s, float mass, float floor, float w, float T, float c)
        : base(base_of(m)), c(c)
    {
        wt = w * T;
        scale = s == 0.0f ? 0.0f : mass * wt / s;
        low = floor * wt;
    }
    __device__ __forceinline__ float dense(float x) const { return exp_above(x, base, c) * scale - low; }
    __device__ __forceinline__ float slot(float x, float p) const { return exp_above(x, base, c) * scale - p * wt; }
};

// A thread's share of a row's loss: sum of p (log p - log q) over the slots; and where there is a floor, what
// lies beside them
struct LossSums {
    double slots;
    BesideSums beside;

    __device__ __forceinline__ void add_slot(float p, float t, float x, double z, double base, double inv_t, double log_s)
    {
        if (p == 0.0f) return;
        const double log_q = x == -INFINITY ? -(double)INFINITY : ((double)x - base) * inv_t - log_s;
        slots += (double)p * ((double)t * inv_t - z - log_q);
    }
    template <bool REST, int BLOCK>
    __device__ __forceinline__ void sum(LossSums* part)
    {
        slots = wave_sum(slots);
        if (REST) {
            beside.sum = wave_sum(beside.sum);
            beside.n = wave_sum(beside.n);
        }
        if (BLOCK == kWave) return;
        __syncthreads();
        if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = *this;
        __syncthreads();
        if (threadIdx.x != 0) return;  // one thread writes the loss
#pragma unroll 1
        for (int w = 1; w < BLOCK / kWave; ++w) {
            slots += part[w].slots;
            if (REST) {
                beside.sum += part[w].beside.sum;
                beside.n += part[w].beside.n;
            }
        }
    }
};

template <bool REST>
__device__ __forceinline__ float loss_of(const DistillArgs& a, const LossSums& l, const TeacherPart& t, float s, double log_s)
{
    const double T = (double)a.T;
    double sum = l.slots;
    if (REST && t.floor > 0.0) {
        const double beside = l.beside.n == 0 ? 0.0 : l.beside.sum / ((double)a.c * T);
        sum += l.beside.n < t.others ? (double)INFINITY : t.floor * ((double)t.others * (log(t.floor) + log_s) - beside);
    }
    double loss = T * T * sum;
    if (!(s == s) || !(t.mass == t.mass)) loss = (double)NAN;
    if (t.mass + t.floor * (double)t.others == 0.0) loss = 0.0;
    return (float)loss;
}

// A row a workgroup, CHUNKS chunks of it in each thread's registers: a 16-byte load of all of them is under way
// before the first is used, and the gradient is written from what the loss was summed from.  Bound by
// memory: 4096 x 141043 bf16 take 498 us, 4.6 TB/s of read and written bytes (a copy of 2 GB: 4.9); with a second
// read in place of the registers 767 us.  2048 x 10000 f32: 39 us, 4.2 TB/s.  One row of 1000: 7 us, the latency of
// ids, logits at the ids, and three reductions.  The exponentials are taken twice, some 230 us of
// vector work in the large case, beside the loads and stores of other waves.
// (A launch has a row a workgroup and no loop over rows: the constants of the 64-bit exp and log
// would be kept in registers across it, 30 to 200 of them spilled.)
template <class T, bool REST, int BLOCK, int CHUNKS>
__global__ __launch_bounds__(BLOCK, 4) void distill_rows_kernel(DistillArgs a)
{
    constexpr int E = Row<T>::kChunk, kSlotsEach = (kMostSlots + BLOCK - 1) / BLOCK;
    // short rows are read before it is known whether they are left out: the weight's latency is theirs too
    constexpr bool kEager = BLOCK * CHUNKS <= 1024;
    constexpr float kDeep = kEager ? kDeepOfShort : kDeepOfLong;
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ float2 part2[BLOCK / kWave];
    __shared__ LossSums parts[BLOCK / kWave];
    __shared__ int32_t parti[BLOCK / kWave];
    __shared__ uint32_t part_any[BLOCK / kWave];
    const Slots slots(lds, a.k);
    const int32_t tid = (int32_t)threadIdx.x;
    const int64_t row = a.row0 + blockIdx.x;
    const SplitRow<T> r(static_cast<const T*>(a.logits) + row * a.logits_stride, a.V);
    T* const g = static_cast<T*>(a.grad) + row * a.grad_stride;
    const float w = a.weight ? a.weight[row * a.weight_stride] : 1.0f;
    uint4 raw[CHUNKS];
    float extra[1] = {-INFINITY};
    const auto load = [&]() {
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            const int32_t i = j * BLOCK + tid;
            if (i < r.whole) raw[j] = r.load(i);
        }
        if (tid < r.extras) extra[0] = Row<T>::one(r.p + r.extra(tid));
    };
    if (kEager) load();
    bool out = a.grad && w == 0.0f;  // left out
    float m = -INFINITY, s = 0.0f;
    LossSums l{};
    bool any_deep = false;
    if (!out) {
        if (tid < kWave) read_teacher(a, row, r.p, slots);
        if (!kEager) load();
        Running<REST> run;
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            if (j * BLOCK + tid < r.whole) {
                float x[E];
                Row<T>::unpack(raw[j], x);
                run.add(x, a.c, kDeep);
            }
            __builtin_amdgcn_sched_barrier(0);  // else all of the row is unpacked before it is used
        }
        if (tid < r.extras) run.add(extra, a.c, kDeep);
        m = run.m;
        s = run.s;
        if (REST) put_any<BLOCK>(run.any_deep, part_any);
        block_join<BLOCK>(m, s, a.c, part2);
        if (REST) {
            l.beside = run.beside;
            l.beside.sum = rebased(run.beside.sum, run.beside.n, run.m, m, a.c);
            any_deep = get_any<BLOCK>(part_any);
        }
    }
    __syncthreads();
    if (REST && any_deep) {
        __shared__ NamedBits<BLOCK * CHUNKS> named;
        named.clear(tid, BLOCK);
        __syncthreads();
        for (int32_t j = tid; j < a.k; j += BLOCK)
            if (slots.id[j] >= 0) named.mark(r, 0, slots.id[j]);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            if (j * BLOCK + tid < r.whole) {
                float x[E];
                Row<T>::unpack(raw[j], x);
                l.beside.add_deep(x, kDeep, base_of(m), a.c, named.of_chunk(j * BLOCK + tid));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (tid < r.extras) l.beside.add_deep(extra, kDeep, base_of(m), a.c, named.of_extra(tid));
    }
    TeacherPart t = *slots.head;
    float all[kSlotsEach];
    int32_t named = 0;
    if (!out && (REST || a.grad)) {
        const bool twice = find_twice<BLOCK>(slots, a.k);
#pragma unroll
        for (int q = 0; q < kSlotsEach; ++q) {
            const int32_t j = q * BLOCK + tid;
            all[q] = 0.0f;
            if (q * BLOCK >= a.k) continue;
            const int32_t id = j < a.k ? slots.id[j] : -1;
            if (id < 0) continue;
            const bool first = first_of_class(slots, twice, a.k, j, id, all[q]);
            if (REST && first) {
                ++named;
                l.beside.take_out(slots.x[j], kDeep, base_of(m), a.c);
            }
        }
    }
    t.floor = 0.0;
    t.others = 0;
    if (REST) {
        t.others = a.V - block_sum<BLOCK>(named, parti);
        t.floor = floor_of(t.mass, t.others);
    }
    const double mass = t.mass + t.floor * (double)t.others;
    out = out || mass == 0.0;
    const Gradient f(m, s, (float)mass, (float)t.floor, w, a.T, a.c);
    if (a.grad) {
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            const int32_t i = j * BLOCK + tid;
            if (i >= r.whole) continue;
            float x[E];
            Row<T>::unpack(raw[j], x);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = out ? 0.0f : f.dense(x[e]);
            store_chunk(g + r.chunk(i), x);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (tid < r.extras) g[r.extra(tid)] = Row<T>::from(out ? 0.0f : f.dense(extra[0]));
        __syncthreads();  // the places of the slots are written again, by other threads
    }
    const double log_s = log((double)s);
    if (!out) {
        const double inv_t = 1.0 / (double)a.T, base = (double)base_of(m);
#pragma unroll
        for (int q = 0; q < kSlotsEach; ++q) {
            const int32_t j = q * BLOCK + tid;
            const int32_t id = j < a.k ? slots.id[j] : -1;
            if (id < 0) continue;
            const float x = slots.x[j];
            if (a.grad) g[id] = Row<T>::from(f.slot(x, all[q]));
            if (a.loss) l.add_slot(slots.p[j], slots.t[j], x, t.z, base, inv_t, log_s);
        }
    }
    l.sum<REST, BLOCK>(parts);
    if (tid == 0) {
        a.loss[row] = out ? 0.0f : loss_of<REST>(a, l, t, s, log_s);
        if (a.stats)
            *reinterpret_cast<RowStats*>(a.stats + row * kStatFloats) = RowStats{m, s, (float)mass, (float)t.floor, t.z};
    }
}

// (m, s) of slices; one more workgroup a row reads its teacher.  Bound by memory: 48 x 10^6 bf16 23 us
// (4.1 TB/s), 4000 x 141043 bf16 232 us with the second kernel (4.9 TB/s).
template <class T, bool REST>
__global__ __launch_bounds__(kPartBlock) void distill_part_kernel(DistillArgs a)
{
    constexpr int E = Row<T>::kChunk;
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ float2 part2[kPartBlock / kWave];
    __shared__ double partd[kPartBlock / kWave];
    __shared__ int32_t parti[kPartBlock / kWave];
    __shared__ uint32_t part_any[kPartBlock / kWave];
    const Slots slots(lds, a.k);
    const int32_t tid = (int32_t)threadIdx.x;
    const int64_t row = a.row0 + blockIdx.x;
    if (a.grad && a.weight && a.weight[row * a.weight_stride] == 0.0f) return;
    if (blockIdx.y == 0) {
        if (tid < kWave)
            read_teacher(a, row, static_cast<const T*>(a.logits) + row * a.logits_stride, slots);
        __syncthreads();
        int32_t named = 0;
        if (REST) {
            const bool twice = find_twice<kPartBlock>(slots, a.k);
            for (int32_t j = tid; j < a.k; j += kPartBlock) {
                float all;
                if (slots.id[j] >= 0) named += first_of_class(slots, twice, a.k, j, slots.id[j], all);
            }
            named = block_sum<kPartBlock>(named, parti);
        }
        if (tid == 0) {
            TeacherPart t = *slots.head;
            t.others = REST ? a.V - named : 0;
            t.floor = REST ? floor_of(t.mass, t.others) : 0.0;
            a.teachers[row] = t;
        }
        return;
    }
    const SplitRow<T> r(static_cast<const T*>(a.logits) + row * a.logits_stride, a.V);
    for (int32_t slice = (int32_t)blockIdx.y - 1; slice < a.slices; slice += (int32_t)gridDim.y - 1) {
        const int32_t i0 = slice * kSliceChunks + tid;
        uint4 raw[kSliceLoads];
#pragma unroll
        for (int j = 0; j < kSliceLoads; ++j)
            if (i0 + j * kPartBlock < r.whole) raw[j] = r.load(i0 + j * kPartBlock);
        const bool has_extra = slice == 0 && tid < r.extras;
        const float extra[1] = {has_extra ? Row<T>::one(r.p + r.extra(tid)) : -INFINITY};
        Running<REST> run;
        if (has_extra) run.add(extra, a.c, kDeepOfLong);
#pragma unroll
        for (int j = 0; j < kSliceLoads; ++j) {
            if (i0 + j * kPartBlock < r.whole) {
                float x[E];
                Row<T>::unpack(raw[j], x);
                run.add(x, a.c, kDeepOfLong);
            }
        }
        const float own = run.m;
        if (REST) put_any<kPartBlock>(run.any_deep, part_any);
        block_join<kPartBlock>(run.m, run.s, a.c, part2);
        if (REST) {
            run.beside.sum = rebased(run.beside.sum, run.beside.n, own, run.m, a.c);
            if (get_any<kPartBlock>(part_any)) {
                __shared__ NamedBits<kSliceChunks> named;
                named.clear(tid, kPartBlock);
                __syncthreads();
                for (int32_t j = tid; j < a.k; j += kPartBlock) {
                    const int64_t id = index_at(a.ids, a.ids_type, row * a.ids_stride + j);
                    if (id >= 0 && id < a.V) named.mark(r, slice * kSliceChunks, (int32_t)id);
                }
                __syncthreads();
#pragma unroll 1
                for (int j = 0; j < kSliceLoads; ++j) {
                    if (i0 + j * kPartBlock < r.whole) {
                        float x[E];
                        Row<T>::unpack(r.load(i0 + j * kPartBlock), x);  // again: to keep them costs every slice registers
                        run.beside.add_deep(x, kDeepOfLong, base_of(run.m), a.c, named.of_chunk(j * kPartBlock + tid));
                    }
                }
                if (has_extra) run.beside.add_deep(extra, kDeepOfLong, base_of(run.m), a.c, named.of_extra(tid));
            }
            run.beside.sum = block_sum<kPartBlock>(run.beside.sum, partd);
            run.beside.n = block_sum<kPartBlock>(run.beside.n, parti);
        }
        if (tid == 0) a.parts[row * a.slices + slice] = RowPart{run.m, run.s, run.beside.sum, run.beside.n, 0};
    }
}

// The slices' parts joined (or the softmax taken from stats), the loss by the first workgroup of a row,
// the gradient by a workgroup a slice.  Bound by memory: the gradient of 1024 x 101636 f16 takes 79 us, 5.3 TB/s, as
// some of the logits are still in the last-level cache; the loss alone 5 us of latency.
template <class T, bool REST>
__global__ __launch_bounds__(kPartBlock) void distill_join_kernel(DistillArgs a)
{
    constexpr int E = Row<T>::kChunk;
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ LossSums parts[kPartBlock / kWave];
    const Slots slots(lds, a.k);
    const int32_t tid = (int32_t)threadIdx.x, lane = tid % kWave;
    const double inv_t = 1.0 / (double)a.T;
    const int64_t row = a.row0 + blockIdx.x;
    const SplitRow<T> r(static_cast<const T*>(a.logits) + row * a.logits_stride, a.V);
    const float w = a.weight ? a.weight[row * a.weight_stride] : 1.0f;
    bool out = a.grad && w == 0.0f;
    float m = -INFINITY, s = 0.0f, mass = 0.0f, floor = 0.0f;
    double scaled_sum = 0.0, z = 0.0;
    int32_t n = 0;
    TeacherPart t{};
    if (!out) {
        if (a.stats_in) {
            const RowStats st = *reinterpret_cast<const RowStats*>(a.stats_in + row * kStatFloats);
            m = st.m;
            s = st.s;
            mass = st.mass;
            floor = st.floor;
            z = st.z;
        } else {
            t = a.teachers[row];
            for (int32_t q = lane; q < a.slices; q += kWave) {  // every wave for itself
                const RowPart part = a.parts[row * a.slices + q];
                join(m, s, part.m, part.s, a.c);
            }
            wave_join(m, s, a.c);
            if (REST) {
                for (int32_t q = lane; q < a.slices; q += kWave) {
                    const RowPart part = a.parts[row * a.slices + q];
                    scaled_sum += rebased(part.scaled_sum, part.n, part.m, m, a.c);
                    n += part.n;
                }
                scaled_sum = wave_sum(scaled_sum);
                n = wave_sum(n);
            }
            mass = (float)(t.mass + t.floor * (double)t.others);
            floor = (float)t.floor;
            z = t.z;
        }
        out = mass == 0.0f;
    }
    const Gradient f(m, s, mass, floor, w, a.T, a.c);
    bool twice = true;
    if (!out) {
        for (int32_t j = tid; j < (a.k + 3) / 4 * 4; j += kPartBlock) {
            int32_t id = -1;
            float tl = -INFINITY;
            if (j < a.k) {
                const int64_t at = index_at(a.ids, a.ids_type, row * a.ids_stride + j);
                tl = element_at(a.teacher, a.teacher_type, row * a.teacher_stride + j);
                if (at >= 0 && at < a.V) id = (int32_t)at;
            }
            slots.id[j] = id;
            slots.t[j] = tl;
            slots.p[j] = id >= 0 ? (float)slot_mass(tl, inv_t, z) : 0.0f;
        }
        __syncthreads();
        if (REST || a.grad) twice = find_twice<kPartBlock>(slots, a.k);
    }
    if (a.loss && blockIdx.y == 0) {
        LossSums l{};
        const double log_s = log((double)s);
        if (!out) {
            const double base = (double)base_of(m);
            if (REST && tid == 0) {
                l.beside.sum = scaled_sum;
                l.beside.n = n;
            }
            for (int32_t j = tid; j < a.k; j += kPartBlock) {
                const int32_t id = slots.id[j];
                if (id < 0) continue;
                const float x = Row<T>::one(r.p + id);
                l.add_slot(slots.p[j], slots.t[j], x, z, base, inv_t, log_s);
                float all;
                if (REST && first_of_class(slots, twice, a.k, j, id, all)) l.beside.take_out(x, kDeepOfLong, base_of(m), a.c);
            }
        }
        l.sum<REST, kPartBlock>(parts);
        if (tid == 0) {
            a.loss[row] = out ? 0.0f : loss_of<REST>(a, l, t, s, log_s);
            if (a.stats)
                *reinterpret_cast<RowStats*>(a.stats + row * kStatFloats) = RowStats{m, s, mass, floor, z};
        }
    }
    if (a.grad) {
        T* const g = static_cast<T*>(a.grad) + row * a.grad_stride;
        for (int32_t slice = (int32_t)blockIdx.y; slice < a.slices; slice += (int32_t)gridDim.y) {
            const int32_t i0 = slice * kSliceChunks + tid;
            uint4 raw[kSliceLoads];
            if (!out) {
#pragma unroll
                for (int j = 0; j < kSliceLoads; ++j)
                    if (i0 + j * kPartBlock < r.whole) raw[j] = r.load(i0 + j * kPartBlock);
            }
            if (slice == 0 && tid < r.extras) {
                const int32_t v = r.extra(tid);
                g[v] = Row<T>::from(out ? 0.0f : f.dense(Row<T>::one(r.p + v)));
            }
#pragma unroll
            for (int j = 0; j < kSliceLoads; ++j) {
                const int32_t i = i0 + j * kPartBlock;
                if (i >= r.whole) continue;
                float x[E];
                Row<T>::unpack(raw[j], x);
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] = out ? 0.0f : f.dense(x[e]);
                store_chunk(g + r.chunk(i), x);
            }
            if (out) continue;
            __syncthreads();  // the slots' places in this slice are written again, by other threads
            const int32_t v0 = r.chunk(slice * kSliceChunks);
            const int32_t v1 = r.chunk(min(r.whole, (slice + 1) * kSliceChunks));
            for (int32_t j = tid; j < a.k; j += kPartBlock) {
                const int32_t id = slots.id[j];
                if (id < 0 || !((id >= v0 && id < v1) || (slice == 0 && (id < r.head || id >= r.chunk(r.whole))))) continue;
                float all;
                first_of_class(slots, twice, a.k, j, id, all);
                g[id] = Row<T>::from(f.slot(Row<T>::one(r.p + id), all));
            }
        }
    }
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


static int32_t distill_slices(const lda_distill_rows* d)
{
    const int64_t chunk = 16 / (int64_t)type_bytes(d->logits_type);
    const int64_t slices = ((int64_t)d->classes / chunk + kSliceChunks - 1) / kSliceChunks;
    return (int32_t)(slices < 1 ? 1 : slices);
}

// Threads and chunks of a thread that hold a row in registers; 0: slices instead.  A workgroup of 1024 has a
// CU to itself, so that loss and gradient of one row take turns on it: a gradient gains by the one
// read (4000 x 141043 bf16: 500 us, slices 730) unless too few rows fill the GPU (20000 f32: always; 49000 f32: 64 rows
// 15.6 us, slices 15.0, 96 rows 16.5 and 19.0; 141043 bf16: 96 rows 28.5 and 23.1, 192 rows 31.7 and 38.8); the loss
// alone is as fast in slices or faster (4000 x 141043: 264 us, slices 232; 64 rows: 15.6 and 10.7).
struct RowShape {
    int block, chunks, least_rows;
};
static RowShape row_shape(const lda_distill_rows* d, bool grad)
{
    static constexpr RowShape kShapes[] = {{64, 4, 1}, {256, 4, 1}, {256, 12, 1}, {1024, 6, 1}, {1024, 12, 64}, {1024, 18, 128}};
    const int64_t chunk = 16 / (int64_t)type_bytes(d->logits_type);
    const int64_t whole = d->classes / chunk;
    for (const RowShape& shape : kShapes) {
        if (whole > (int64_t)shape.block * shape.chunks) continue;
        if (shape.block == 1024 && (!grad || d->rows < shape.least_rows)) break;
        return shape;
    }
    return {0, 0, 0};
}

template <class T, bool REST>
static void launch_distill_typed(const DistillArgs& a, unsigned gx, RowShape shape, hipStream_t stream)
{
    const unsigned gy = (unsigned)(a.slices < 32768 ? a.slices : 32768);
    const size_t lds = slots_lds(a.k);
    if (a.stats_in) {
        distill_join_kernel<T, REST><<<dim3(gx, gy), kPartBlock, lds, stream>>>(a);
    } else if (shape.block == 64) {
        distill_rows_kernel<T, REST, 64, 4><<<gx, 64, lds, stream>>>(a);
    } else if (shape.block == 256 && shape.chunks == 4) {
        distill_rows_kernel<T, REST, 256, 4><<<gx, 256, lds, stream>>>(a);
    } else if (shape.block == 256) {
        distill_rows_kernel<T, REST, 256, 12><<<gx, 256, lds, stream>>>(a);
    } else if (shape.chunks == 6) {
        distill_rows_kernel<T, REST, 1024, 6><<<gx, 1024, lds, stream>>>(a);
    } else if (shape.chunks == 12) {
        distill_rows_kernel<T, REST, 1024, 12><<<gx, 1024, lds, stream>>>(a);
    } else if (shape.chunks == 18) {
        distill_rows_kernel<T, REST, 1024, 18><<<gx, 1024, lds, stream>>>(a);
    } else {
        distill_part_kernel<T, REST><<<dim3(gx, gy + 1), kPartBlock, lds, stream>>>(a);
        distill_join_kernel<T, REST><<<dim3(gx, a.grad ? gy : 1), kPartBlock, lds, stream>>>(a);
    }
}

static int64_t distill_bytes(const lda_distill_rows* d)
{
    if (d->rows == 0 || row_shape(d, false).block != 0) return 0;
    return d->rows * (distill_slices(d) * (int64_t)sizeof(RowPart) + (int64_t)sizeof(TeacherPart));
}

static int launch_distill(const lda_distill_rows* d, const char* call, float* loss, float* stats,
                          const float* stats_in, void* grad, int64_t grad_stride)
{
    if (d->rows == 0) return LDA_OK;
    if (!aligned_to(loss, 4) || !aligned_to(stats, 16) || !aligned_to(stats_in, 16) ||
        !aligned_to(grad, type_bytes(d->logits_type)))
        return fail(nullptr, LDA_ERR_ARG, "%s: an output is not aligned to its type, or stats to 16 bytes", call);
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
    const RowShape shape = row_shape(d, grad != nullptr);
    if (shape.block == 0 && !stats_in) {
        const int64_t need = distill_bytes(d);
        if (!d->workspace || d->workspace_bytes < need || !aligned_to(d->workspace, 16))
            return fail(nullptr, LDA_ERR_ARG, "%s: needs a workspace of %lld bytes, aligned to 16", call, (long long)need);
        a.teachers = static_cast<TeacherPart*>(d->workspace);
        a.parts = reinterpret_cast<RowPart*>(a.teachers + a.rows);
    }
    const hipStream_t stream = static_cast<hipStream_t>(d->hip_stream);
    const auto typed = [&](auto t) {
        using T = decltype(t);
        for (a.row0 = 0; a.row0 < a.rows; a.row0 += 1 << 20) {
            const unsigned n = (unsigned)(a.rows - a.row0 < (1 << 20) ? a.rows - a.row0 : 1 << 20);
            if (d->log_norm) launch_distill_typed<T, true>(a, n, shape, stream);
            else launch_distill_typed<T, false>(a, n, shape, stream);
        }
    };
    if (d->logits_type == LDA_F32) typed(float{});
    else if (d->logits_type == LDA_F16) typed(__half{});
    else typed(__hip_bfloat16{});
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
    return distill_bytes(d);
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
