// Product of 8-bit integers with a scale for each row of both sides: rows of numbers times the classes' weights
// (the formula stands at lda_product_rows in lda_mi355x.h).  Sums are 32-bit integers and exact, so that neither the
// order of a sum nor the way it is split shows in the result.
//
// Few rows (product_few_kernel): the weights are read once from memory straight into the matrix instructions'
// registers, and that is what bounds it.  Many rows (product_tile_kernel): tiles of both sides go through LDS, two
// buffers, the fragments of a step read while the one before multiplies.  With too few tiles for the GPU the long axis
// is split over workgroups and a second kernel adds up.
#include <type_traits>

#include "rows.hpp"

namespace lda {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));

constexpr int32_t kMostWidth = 131071;  // times 128^2 below 2^31
constexpr int kStep = 64;               // bytes of a row that a step of the few-rows kernel takes
constexpr int kTileK = 128;             // bytes of a row in a tile

struct ProductArgs {
    int64_t M;
    int32_t N, K;
    const int8_t* a;
    int64_t a_stride;
    const float* a_scale;
    const int8_t* b;
    int64_t b_stride;
    const float* b_scale;
    void* out;
    int64_t out_stride;
    int32_t splits, split_k;  // bytes of a row in each, a multiple of kTileK
    int32_t* partial;         // [splits][M][N]
    int32_t tiles_m, tiles_n;
};

// 16 bytes of a row from k on, 0 behind `end`
template <bool ALIGNED>
__device__ __forceinline__ i32x4 load16(const int8_t* row, int32_t k, int32_t end)
{
    i32x4 v = {0, 0, 0, 0};
    if (ALIGNED) {
        if (k < end) v = *reinterpret_cast<const i32x4*>(row + k);  // end is a multiple of 16
    } else if (k + 16 <= end) {
        __builtin_memcpy(&v, row + k, 16);
    } else if (k < end) {
        const int32_t n = end - k;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (i < n) v[i / 4] |= (int32_t)((uint32_t)(uint8_t)row[k + i] << (i % 4 * 8));
    }
    return v;
}

__device__ __forceinline__ float scaled(int32_t sum, float sa, float sb)
{
    float v = ((float)sum * sa) * sb;
    asm("" : "+v"(v));  // else the last product and a rounding to fp16 become one instruction, with one rounding less
    return v;
}

template <class T>
__device__ __forceinline__ void store_few(T* p, const float (&v)[4])  // 4 adjacent elements, aligned to one
{
    if constexpr (std::is_same<T, float>::value) {
        __builtin_memcpy(p, v, 16);
    } else {
        const uint2 w = make_uint2(Row<T>::two(v[0], v[1]), Row<T>::two(v[2], v[3]));
        __builtin_memcpy(p, &w, 8);
    }
}

// Up to 16 MT rows times 16 CT classes a workgroup; its waves take the row's steps in turn and join in LDS.
template <class T, int MT, int CT, bool ALIGNED>
__global__ __launch_bounds__(256) void product_few_kernel(ProductArgs p)
{
    constexpr int kWaves = 4, kClasses = 16 * CT, kRows = 16 * MT;
    __shared__ int32_t part[kWaves][kRows][kClasses + 4];
    const int32_t tid = (int32_t)threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int32_t n0 = (int32_t)blockIdx.x * kClasses, split = (int32_t)blockIdx.y;
    const int32_t from = split * p.split_k, end = min(p.K, from + p.split_k);
    const int32_t r = lane % 16, g = lane / 16 * 16;
    const int8_t *a[MT], *b[CT];
#pragma unroll
    for (int i = 0; i < MT; ++i) a[i] = p.a + min((int64_t)(16 * i + r), p.M - 1) * p.a_stride;
#pragma unroll
    for (int i = 0; i < CT; ++i) b[i] = p.b + (int64_t)min(n0 + 16 * i + r, p.N - 1) * p.b_stride;
    i32x4 sum[CT][MT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int m = 0; m < MT; ++m) sum[c][m] = i32x4{0, 0, 0, 0};
    constexpr int kUnroll = MT * CT >= 8 ? 2 : 4;
    for (int32_t k = from + wave * kStep + g; k - g < end; k += kUnroll * kWaves * kStep) {
        i32x4 x[kUnroll][MT], w[kUnroll][CT];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int32_t at = k + u * kWaves * kStep;
#pragma unroll
            for (int c = 0; c < CT; ++c) w[u][c] = load16<ALIGNED>(b[c], at, end);
#pragma unroll
            for (int m = 0; m < MT; ++m) x[u][m] = load16<ALIGNED>(a[m], at, end);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    sum[c][m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u][c], x[u][m], sum[c][m], 0, 0, 0);
    }
    // lane: 4 adjacent classes of a row
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int m = 0; m < MT; ++m)
            *reinterpret_cast<i32x4*>(&part[wave][16 * m + lane % 16][16 * c + lane / 16 * 4]) = sum[c][m];
    __syncthreads();
    T* const out = static_cast<T*>(p.out);
    for (int32_t i = tid; i < kRows * kClasses; i += 256) {
        const int32_t m = i / kClasses, c = i % kClasses, n = n0 + c;
        if (m >= p.M || n >= p.N) continue;
        const int32_t s = part[0][m][c] + part[1][m][c] + part[2][m][c] + part[3][m][c];
        if (p.splits > 1) p.partial[((int64_t)split * p.M + m) * p.N + n] = s;
        else out[m * p.out_stride + n] = Row<T>::from(scaled(s, p.a_scale[m], p.b_scale[n]));
    }
}

// A tile of TM rows times TN classes a workgroup of WM x WN waves.  LDS has rows of kTileK bytes, their 16-byte pieces
// in an order that changes from row to row, so that reads down a column of pieces meet all banks.
template <class T, int TM, int TN, int WM, int WN, bool ALIGNED>
__global__ __launch_bounds__(WM * WN * 64, 1) void product_tile_kernel(ProductArgs p)
{
    constexpr int kThreads = WM * WN * 64, kMi = TM / WM / 32, kNi = TN / WN / 32, kSteps = kTileK / 32;
    constexpr int kRowsAtOnce = kThreads / 8, kLoadsA = TM / kRowsAtOnce, kLoadsB = TN / kRowsAtOnce;
    extern __shared__ __align__(16) int8_t lds[];  // [2][TM + TN][kTileK]
    constexpr int kBuffer = (TM + TN) * kTileK;
    const int32_t tid = (int32_t)threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int32_t tile = (int32_t)blockIdx.x;
    const int32_t tm = tile % p.tiles_m, tn = tile / p.tiles_m % p.tiles_n, split = tile / p.tiles_m / p.tiles_n;
    const int64_t m0 = (int64_t)tm * TM;
    const int32_t n0 = tn * TN;
    const int32_t from = split * p.split_k, end = min(p.K, from + p.split_k);
    // what a thread loads: piece tid % 8 of rows tid / 8, + kRowsAtOnce, ...
    const int32_t piece = tid % 8 * 16, row0 = tid / 8;
    const int8_t *a[kLoadsA], *b[kLoadsB];
#pragma unroll
    for (int i = 0; i < kLoadsA; ++i) a[i] = p.a + min(m0 + row0 + i * kRowsAtOnce, p.M - 1) * p.a_stride;
#pragma unroll
    for (int i = 0; i < kLoadsB; ++i) b[i] = p.b + (int64_t)min(n0 + row0 + i * kRowsAtOnce, p.N - 1) * p.b_stride;
    i32x4 held[kLoadsA + kLoadsB];
    const auto load = [&](int32_t k) {
#pragma unroll
        for (int i = 0; i < kLoadsA; ++i) held[i] = load16<ALIGNED>(a[i], k + piece, end);
#pragma unroll
        for (int i = 0; i < kLoadsB; ++i) held[kLoadsA + i] = load16<ALIGNED>(b[i], k + piece, end);
    };
    const int32_t put_at = row0 * kTileK + (piece ^ (row0 % 8 * 16));  // kRowsAtOnce is a multiple of 8
    const auto put = [&](int buffer) {
        int8_t* const to = lds + buffer * kBuffer + put_at;
#pragma unroll
        for (int i = 0; i < kLoadsA + kLoadsB; ++i) *reinterpret_cast<i32x4*>(to + i * kRowsAtOnce * kTileK) = held[i];
    };
    const int32_t wm = wave % WM * (TM / WM), wn = wave / WM * (TN / WN);
    const int32_t r = lane % 32, half = lane / 32 * 16, turn = r % 8 * 16;
    const int8_t* const read_a = lds + (wm + r) * kTileK;
    const int8_t* const read_b = lds + (TM + wn + r) * kTileK;
    i32x4 fa[2][kMi], fb[2][kNi];
    const auto read = [&](int buffer, int step, int set) {
        const int32_t at = buffer * kBuffer + ((step * 32 + half) ^ turn);
#pragma unroll
        for (int i = 0; i < kNi; ++i) fb[set][i] = *reinterpret_cast<const i32x4*>(read_b + at + i * 32 * kTileK);
#pragma unroll
        for (int i = 0; i < kMi; ++i) fa[set][i] = *reinterpret_cast<const i32x4*>(read_a + at + i * 32 * kTileK);
    };
    i32x16 sum[kNi][kMi];
#pragma unroll
    for (int n = 0; n < kNi; ++n)
#pragma unroll
        for (int m = 0; m < kMi; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[n][m][i] = 0;
    load(from);
    put(0);
    load(from + kTileK);
    __syncthreads();
    read(0, 0, 0);
    int buffer = 0;
    for (int32_t k = from; k < end; k += kTileK) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            if (s < kSteps - 1) {
                read(buffer, s + 1, (s + 1) % 2);
            } else {
                __syncthreads();  // the next tile is there, and nobody reads this one any more
                read(buffer ^ 1, 0, 0);
            }
#pragma unroll
            for (int n = 0; n < kNi; ++n)
#pragma unroll
                for (int m = 0; m < kMi; ++m)
                    sum[n][m] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[s % 2][n], fa[s % 2][m], sum[n][m], 0, 0, 0);
            if (s == 1) {
                put(buffer ^ 1);
                load(k + 2 * kTileK);
            }
        }
        buffer ^= 1;
    }
    // lane: a row, 4 adjacent classes at a time
    T* const out = static_cast<T*>(p.out);
#pragma unroll
    for (int m = 0; m < kMi; ++m) {
        const int64_t row = m0 + wm + 32 * m + lane % 32;
        if (row >= p.M) continue;
        const float sa = p.a_scale[row];
#pragma unroll
        for (int n = 0; n < kNi; ++n) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int32_t c = n0 + wn + 32 * n + 8 * q + lane / 32 * 4;
                if (p.splits > 1) {
                    int32_t* const to = p.partial + ((int64_t)split * p.M + row) * p.N;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (c + i < p.N) to[c + i] = sum[n][m][4 * q + i];
                    continue;
                }
                T* const to = out + row * p.out_stride;
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = c + i < p.N ? scaled(sum[n][m][4 * q + i], sa, p.b_scale[c + i]) : 0.0f;
                if (c + 4 <= p.N) {
                    store_few(to + c, v);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (c + i < p.N) to[c + i] = Row<T>::from(v[i]);
                }
            }
        }
    }
}

// The splits' sums added up; none of a width of 0
template <class T>
__global__ __launch_bounds__(256) void product_join_kernel(ProductArgs p)
{
    const int64_t cells = p.M * p.N;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < cells; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / p.N;
        const int32_t n = (int32_t)(i % p.N);
        int32_t s = 0;
        for (int32_t q = 0; q < p.splits; ++q) s += p.partial[(int64_t)q * cells + i];
        static_cast<T*>(p.out)[m * p.out_stride + n] = Row<T>::from(scaled(s, p.a_scale[m], p.b_scale[n]));
    }
}

static int check_product(const lda_product_rows* d, const char* call)
{
    if (!d) return fail(nullptr, LDA_ERR_ARG, "%s: NULL rows", call);
    for (int32_t r : d->reserved)
        if (r != 0) return fail(nullptr, LDA_ERR_ARG, "%s: reserved fields must be zero", call);
    if (d->reserved_word != 0) return fail(nullptr, LDA_ERR_ARG, "%s: reserved fields must be zero", call);
    if (d->rows < 0 || d->classes < 1 || d->width < 0)
        return fail(nullptr, LDA_ERR_ARG, "%s: rows >= 0, classes >= 1, width >= 0 needed", call);
    if (!known_type(d->out_type)) return fail(nullptr, LDA_ERR_ARG, "%s: unknown type", call);
    if (d->width > kMostWidth)
        return fail(nullptr, LDA_ERR_UNSUPPORTED, "%s: at most %d numbers a row (sums are 32-bit)", call, kMostWidth);
    if (d->rows > (int64_t)1 << 31) return fail(nullptr, LDA_ERR_UNSUPPORTED, "%s: at most 2^31 rows", call);
    if (d->rows == 0) return LDA_OK;
    if (!d->a_scale || !d->b_scale || (d->width > 0 && (!d->a || !d->b)))
        return fail(nullptr, LDA_ERR_ARG, "%s: NULL pointer", call);
    if (!aligned_to(d->a_scale, 4) || !aligned_to(d->b_scale, 4))
        return fail(nullptr, LDA_ERR_ARG, "%s: a pointer is not aligned to its type", call);
    return LDA_OK;
}

enum class ProductKind { kFew, kTile128, kTile256 };
struct ProductPlan {
    ProductKind kind;
    int classes, splits;  // of the few-rows kernel: 16-class tiles of a wave
    int32_t split_k;
};
static ProductPlan plan_product(const lda_product_rows* d)
{
    ProductPlan p{};
    int64_t groups;
    if (d->rows <= 64) {
        p.kind = ProductKind::kFew;
        p.classes = d->classes >= 32768 && d->rows <= 48 ? 4 : d->classes >= 16384 ? 2 : 1;
        groups = ((int64_t)d->classes + 16 * p.classes - 1) / (16 * p.classes);
    } else {
        const auto tiles = [&](int64_t m, int64_t n) { return ((d->rows + m - 1) / m) * ((d->classes + n - 1) / n); };
        p.kind = tiles(256, 256) >= 768 ? ProductKind::kTile256 : ProductKind::kTile128;
        groups = p.kind == ProductKind::kTile256 ? tiles(256, 256) : tiles(128, 128);
    }
    // a split has 1024 bytes of a row at least
    int64_t splits = groups >= 192 ? 1 : 256 / (groups < 1 ? 1 : groups);
    const int64_t most = d->width / 1024;
    if (splits > most) splits = most;
    if (splits < 1) splits = 1;
    const int64_t pieces = ((int64_t)d->width + kTileK - 1) / kTileK;
    const int64_t each = (pieces + splits - 1) / splits;
    p.split_k = (int32_t)((each < 1 ? 1 : each) * kTileK);
    p.splits = (int)((pieces + (each < 1 ? 1 : each) - 1) / (each < 1 ? 1 : each));
    if (p.splits < 1) p.splits = 1;
    return p;
}

static int64_t product_bytes(const lda_product_rows* d)
{
    if (d->rows == 0 || d->width == 0) return 0;
    const ProductPlan p = plan_product(d);
    return p.splits == 1 ? 0 : (int64_t)p.splits * d->rows * d->classes * (int64_t)sizeof(int32_t);
}

template <class T>
static void launch_join(const ProductArgs& a, hipStream_t stream)
{
    const int64_t n = (a.M * a.N + 255) / 256;
    product_join_kernel<T><<<(unsigned)(n < 8192 ? n : 8192), 256, 0, stream>>>(a);
}

template <class T, bool ALIGNED>
static hipError_t launch_product(ProductArgs a, const ProductPlan& plan, hipStream_t stream)
{
    a.splits = plan.splits;
    a.split_k = plan.split_k;
    const auto few = [&](auto mt, auto ct) {
        const dim3 grid((unsigned)((a.N + 16 * ct() - 1) / (16 * ct())), (unsigned)a.splits);
        product_few_kernel<T, mt(), ct(), ALIGNED><<<grid, 256, 0, stream>>>(a);
    };
    const auto tile = [&](auto tm, auto tn, auto wm, auto wn) {
        a.tiles_m = (int32_t)((a.M + tm() - 1) / tm());
        a.tiles_n = (a.N + tn() - 1) / tn();
        constexpr size_t lds = 2 * (tm() + tn()) * kTileK;
        const auto kernel = product_tile_kernel<T, tm(), tn(), wm(), wn(), ALIGNED>;
        if (lds > 65536) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (e != hipSuccess) return e;
        }
        const unsigned n = (unsigned)((int64_t)a.tiles_m * a.tiles_n * a.splits);
        kernel<<<n, wm() * wn() * 64, lds, stream>>>(a);
        return hipSuccess;
    };
    using std::integral_constant;
    if (plan.kind == ProductKind::kFew) {
        const int mt = (int)((a.M + 15) / 16);
        const auto with = [&](auto ct) {
            if (mt == 1) few(integral_constant<int, 1>{}, ct);
            else if (mt == 2) few(integral_constant<int, 2>{}, ct);
            else if (mt == 3) few(integral_constant<int, 3>{}, ct);
            else few(integral_constant<int, 4>{}, ct);
        };
        if (plan.classes == 4) {
            const auto ct = integral_constant<int, 4>{};
            if (mt == 1) few(integral_constant<int, 1>{}, ct);
            else if (mt == 2) few(integral_constant<int, 2>{}, ct);
            else few(integral_constant<int, 3>{}, ct);
        } else if (plan.classes == 2) {
            with(integral_constant<int, 2>{});
        } else {
            with(integral_constant<int, 1>{});
        }
    } else {
        const auto c256 = integral_constant<int, 256>{};
        const auto c128 = integral_constant<int, 128>{};
        const auto c2 = integral_constant<int, 2>{};
        const hipError_t e = plan.kind == ProductKind::kTile256 ? tile(c256, c256, c2, c2) : tile(c128, c128, c2, c2);
        if (e != hipSuccess) return e;
    }
    if (a.splits > 1) launch_join<T>(a, stream);
    return hipGetLastError();
}

}  // namespace lda

using namespace lda;

extern "C" {

int64_t lda_product_workspace(const lda_product_rows* d)
try {
    const int rc = check_product(d, "lda_product_workspace");
    if (rc != LDA_OK) return rc;
    return product_bytes(d);
} catch (...) {
    return LDA_ERR_OOM;
}

int lda_product(const lda_product_rows* d, void* out, int64_t out_stride)
try {
    const int rc = check_product(d, "lda_product");
    if (rc != LDA_OK) return rc;
    if (d->rows == 0) return LDA_OK;
    if (!out) return fail(nullptr, LDA_ERR_ARG, "lda_product: NULL out");
    if (!aligned_to(out, type_bytes(d->out_type))) return fail(nullptr, LDA_ERR_ARG, "lda_product: out is not aligned to its type");
    if (d->rows > 1 && out_stride < d->classes) return fail(nullptr, LDA_ERR_ARG, "lda_product: rows of out overlap");
    const int64_t need = product_bytes(d);
    if (need > 0 && (!d->workspace || d->workspace_bytes < need || !aligned_to(d->workspace, 16)))
        return fail(nullptr, LDA_ERR_ARG, "lda_product: needs a workspace of %lld bytes, aligned to 16", (long long)need);
    ProductArgs a{};
    a.M = d->rows;
    a.N = d->classes;
    a.K = d->width;
    a.a = static_cast<const int8_t*>(d->a);
    a.a_stride = d->a_stride;
    a.a_scale = d->a_scale;
    a.b = static_cast<const int8_t*>(d->b);
    a.b_stride = d->b_stride;
    a.b_scale = d->b_scale;
    a.out = out;
    a.out_stride = out_stride;
    a.partial = static_cast<int32_t*>(d->workspace);
    const hipStream_t stream = static_cast<hipStream_t>(d->hip_stream);
    const bool aligned = a.K % 16 == 0 && aligned_to(a.a, 16) && aligned_to(a.b, 16) && a.a_stride % 16 == 0 && a.b_stride % 16 == 0;
    const auto typed = [&](auto t) -> hipError_t {
        using T = decltype(t);
        if (a.K == 0) {
            launch_join<T>(a, stream);
            return hipGetLastError();
        }
        const ProductPlan plan = plan_product(d);
        return aligned ? launch_product<T, true>(a, plan, stream) : launch_product<T, false>(a, plan, stream);
    };
    const hipError_t e = d->out_type == LDA_F32 ? typed(float{}) : d->out_type == LDA_F16 ? typed(__half{}) : typed(__hip_bfloat16{});
    LDA_HIP(static_cast<lda_ctx*>(nullptr), e);
    return LDA_OK;
} catch (...) {
    return LDA_ERR_OOM;
}

}  // extern "C"
