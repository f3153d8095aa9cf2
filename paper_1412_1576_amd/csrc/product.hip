// Product of 8-bit integers with a scale for each row of both sides: rows of numbers times the classes' weights
// (the formula stands at lda_product_rows in lda_mi355x.h).  Sums are 32-bit integers and exact, so that neither the
// order of a sum nor the way it is split shows in the result.
//
// Few rows (product_few_kernel): the weights are read once from memory straight into the matrix instructions'
// registers, and that is what bounds it.  Many rows (product_tile_kernel): tiles of both sides go through LDS, two
// buffers, the fragments of a step read while the one before multiplies.  With too few tiles for the GPU the long axis
// is split over workgroups and a second kernel adds up.
#include <atomic>
#include <type_traits>

#include "rows.hpp"
#include "xcd.hpp"

namespace lda {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));

constexpr int32_t kMostWidth = 131071;  // times 128^2 below 2^31
constexpr int kStep = 64;               // bytes of a row that a step of the few-rows kernel takes
constexpr int kTileK = 128;             // bytes of a row in a tile
constexpr int kCus = 256, kLdsOfCu = 160 * 1024;
constexpr int kRawBuffer = 0x00020000;  // a buffer resource's last word: no swizzle, 32-bit data

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
    int32_t block0;           // of the few-rows kernel, whose blocks are launched in stretches
};

__device__ __forceinline__ i32x4 load16(const int8_t* from)
{
    i32x4 v;
    __builtin_memcpy(&v, from, 16);
    return v;
}
// 16 bytes of a row from k on, 0 behind `end`
__device__ __forceinline__ i32x4 load16(const int8_t* row, int32_t k, int32_t end)
{
    i32x4 v = {0, 0, 0, 0};
    if (k + 16 <= end) {
        v = load16(row + k);
    } else if (k < end) {
        const int32_t n = end - k;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (i < n) v[i / 4] |= (int32_t)((uint32_t)(uint8_t)row[k + i] << (i % 4 * 8));
    }
    return v;
}

__device__ __forceinline__ float scaled(float v, float scale)
{
    v *= scale;
    asm("" : "+v"(v));  // else this and a rounding to fp16 become one instruction, with one rounding less
    return v;
}
__device__ __forceinline__ float scaled(int32_t sum, float sa, float sb) { return scaled((float)sum * sa, sb); }

// Up to 16 rows times 16 CT classes a workgroup; its waves take the row's steps in turn and join in LDS.  Rows lie
// anywhere: the hardware's loads take any address.  1 x 4096 x 141043: 108 us, 5.3 TB/s of weights; 1 x 1000 x 1024 is
// the host's call.
template <class T, int CT>
__global__ __launch_bounds__(256) void product_few_kernel(ProductArgs p)
{
    constexpr int kWaves = 4, kClasses = 16 * CT, kUnroll = 4;
    __shared__ int32_t part[kWaves][16][kClasses + 4];
    const int32_t tid = (int32_t)threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int32_t n0 = (p.block0 + (int32_t)blockIdx.x) * kClasses, left = p.N - n0, split = (int32_t)blockIdx.y;
    const int32_t from = split * p.split_k, end = min(p.K, from + p.split_k);
    const int32_t r = lane % 16, g = lane / 16 * 16;
    const int8_t* const a = p.a + min((int64_t)r, p.M - 1) * p.a_stride;
    const int8_t* b[CT];
#pragma unroll
    for (int i = 0; i < CT; ++i) b[i] = p.b + (int64_t)(n0 + min(16 * i + r, left - 1)) * p.b_stride;
    i32x4 sum[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) sum[c] = i32x4{0, 0, 0, 0};
    const auto take = [&](auto steps, auto whole, int32_t k) {
        i32x4 x[steps()], w[steps()][CT];
#pragma unroll
        for (int u = 0; u < steps(); ++u) {
            const int32_t at = k + u * kWaves * kStep;
#pragma unroll
            for (int c = 0; c < CT; ++c)
                w[u][c] = whole() ? load16(b[c] + at) : load16(b[c], at, end);
            x[u] = whole() ? load16(a + at) : load16(a, at, end);
        }
#pragma unroll
        for (int u = 0; u < steps(); ++u)
#pragma unroll
            for (int c = 0; c < CT; ++c) sum[c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u][c], x[u], sum[c], 0, 0, 0);
    };
    int32_t k = from + wave * kStep + g;
    for (; k - g + (kUnroll - 1) * kWaves * kStep + kStep <= end; k += kUnroll * kWaves * kStep)
        take(std::integral_constant<int, kUnroll>{}, std::true_type{}, k);
    for (; k - g < end; k += kWaves * kStep) take(std::integral_constant<int, 1>{}, std::false_type{}, k);
    // lane: 4 adjacent classes of a row
#pragma unroll
    for (int c = 0; c < CT; ++c) *reinterpret_cast<i32x4*>(&part[wave][r][16 * c + g / 4]) = sum[c];
    __syncthreads();
    T* const out = static_cast<T*>(p.out);
    for (int32_t i = tid; i < 16 * kClasses; i += 256) {
        const int32_t m = i / kClasses, c = i % kClasses;
        if (m >= p.M || c >= left) continue;
        const int32_t n = n0 + c;
        const int32_t s = part[0][m][c] + part[1][m][c] + part[2][m][c] + part[3][m][c];
        if (p.splits > 1) p.partial[((int64_t)split * p.M + m) * p.N + n] = s;
        else out[m * p.out_stride + n] = Row<T>::from(scaled(s, p.a_scale[m], p.b_scale[n]));
    }
}

// The order of a step of product_tile_kernel: reads from LDS behind the first products, then writes and loads, a pair
// behind each product.  Left alone the compiler puts reads where they are used, and waits.
template <int PRODUCTS, int READS, int PAIRS>
__device__ __forceinline__ void interleave(bool pairs)
{
    if (PRODUCTS < 4) return;  // few products: memory is what is waited for
    constexpr int kReadsEach = READS * 2 > PRODUCTS ? 2 : 1, kFirst = (READS + kReadsEach - 1) / kReadsEach;
    constexpr int kRest = PRODUCTS > kFirst ? PRODUCTS - kFirst : 1, kPairsEach = (PAIRS + kRest - 1) / kRest;
#pragma unroll
    for (int i = 0; i < PRODUCTS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // matrix
        if (i < kFirst) {
            __builtin_amdgcn_sched_group_barrier(0x100, kReadsEach, 0);  // LDS read
        } else if (pairs) {
            __builtin_amdgcn_sched_group_barrier(0x200, kPairsEach, 0);  // LDS write
            __builtin_amdgcn_sched_group_barrier(0x020, kPairsEach, 0);  // memory read
        }
    }
}

// A tile of the result and of the long axis: where both sides' rows begin and how many there are
struct ProductTile {
    int64_t m0;
    int32_t n0, split, rows_a, rows_b, from, end;
    const int8_t *a, *b;
};
// Workgroups go to the 8 XCDs in turn: each XCD has a stretch of the tiles, in groups of kTileGroup rows of tiles, so that
// those under way on it at once share what its L2 holds of both sides.  Number `turn` of workgroup `block`; false
// where it has no more.
constexpr int32_t kTileGroup = 8;
template <int TM, int TN>
__device__ __forceinline__ bool find_tile(const ProductArgs& p, int32_t block, int32_t turn, ProductTile& t)
{
    const int32_t tiles = p.tiles_m * p.tiles_n * p.splits;
    const int32_t xcd = block % kXcds, each = tiles / kXcds, more = tiles % kXcds;
    const int32_t at = block / kXcds + turn * ((int32_t)gridDim.x / kXcds);
    if (at >= each + (xcd < more)) return false;
    int32_t tile = xcd * each + min(xcd, more) + at;
    t.split = tile / (p.tiles_m * p.tiles_n);
    tile %= p.tiles_m * p.tiles_n;
    const int32_t group = tile / (kTileGroup * p.tiles_n), rest = tile % (kTileGroup * p.tiles_n);
    const int32_t high = min(kTileGroup, p.tiles_m - group * kTileGroup);
    t.m0 = (int64_t)(group * kTileGroup + rest % high) * TM;
    t.n0 = rest / high * TN;
    t.rows_a = (int32_t)min((int64_t)TM, p.M - t.m0);
    t.rows_b = min(TN, p.N - t.n0);
    t.from = t.split * p.split_k;
    t.end = min(p.K, t.from + p.split_k);
    t.a = p.a + t.m0 * p.a_stride;
    t.b = p.b + (int64_t)t.n0 * p.b_stride;
    return true;
}

// Where a wave's 32 rows pass through LDS on their way out: as many classes of a row as the wave has, since memory's lines
// that are written in parts cost time (rows of 141 043 16-bit numbers begin anywhere; 4096 x 1024 of them took 948 us by 64
// classes at a time).  The waves that find no room in the piece that nobody reads any more have some behind it.
template <int TM, int TN, int WM, int WN>
struct ProductStage {
    static constexpr int kBlocks = TM >= 128 ? TN / WN / 32 : 1;  // of 32 classes
    static constexpr int kRow = kBlocks * 32 + 4, kBytes = 32 * kRow * 4;
    static constexpr int kFit = (TM + TN) * kTileK / kBytes, kInside = kFit < WM * WN ? kFit : WM * WN;
    static constexpr size_t kLds = (TM + TN) * (2 * kTileK + sizeof(float)) + (WM * WN - kInside) * kBytes;
};

// Tiles of TM rows times TN classes, one after the other, by a workgroup of WM x WN waves.  The pieces of both sides
// are one stream over all of a workgroup's tiles: two pieces of the long axis are under way while one is multiplied, also
// from one tile to the next, so that a tile's beginning waits for nothing and its stores drain behind the next one's
// products.  LDS has rows of kTileK bytes, their 16-byte pieces in an order that changes every two rows, so that 16 rows'
// reads of a column of pieces meet all banks (with an order that changed every row a third of LDS's cycles were
// conflicts).  4096 x 4096 x 141043 by 256 x 256: 2.15 ms, 2.2 Pop/s, the matrix units busy 63 % of the cycles at the 1.47 GHz
// that the card's power leaves; 48 x 5120 x 101636 by 64 x 128: 113 us, 4.7 TB/s of weights.
template <class T, int TM, int TN, int WM, int WN, bool ALIGNED>
__global__ __launch_bounds__(WM * WN * 64, 1) void product_tile_kernel(ProductArgs p)
{
    constexpr int kThreads = WM * WN * 64, kMi = TM / WM / 32, kNi = TN / WN / 32, kSteps = kTileK / 32;
    constexpr int kRowsAtOnce = kThreads / 8, kLoadsA = TM / kRowsAtOnce, kLoadsB = TN / kRowsAtOnce, kLoads = kLoadsA + kLoadsB;
    static_assert(kRowsAtOnce % 16 == 0 && TM % kRowsAtOnce == 0 && TN % kRowsAtOnce == 0 && TM <= kThreads && TN <= kThreads, "shape");
    using Stage = ProductStage<TM, TN, WM, WN>;
    extern __shared__ __align__(16) int8_t lds[];  // [2][TM + TN][kTileK], [TM + TN] scales, stages
    constexpr int kBuffer = (TM + TN) * kTileK;
    float* const scale_a = reinterpret_cast<float*>(lds + 2 * kBuffer);
    float* const scale_b = scale_a + TM;
    const int32_t tid = (int32_t)threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    // What a thread loads: 16 bytes at `piece` of rows tid / 8, + kRowsAtOnce, ...
    const int32_t piece = tid % 8 * 16, row0 = tid / 8;
    const uint32_t at_a = (uint32_t)row0 * (uint32_t)p.a_stride + (uint32_t)piece, step_a = kRowsAtOnce * (uint32_t)p.a_stride;
    const uint32_t at_b = (uint32_t)row0 * (uint32_t)p.b_stride + (uint32_t)piece, step_b = kRowsAtOnce * (uint32_t)p.b_stride;
    // The stream.  ALIGNED: through buffers that end where a tile's last row ends; what lies beyond reads as 0.
    ProductTile next{};
    int32_t turn = 0, k_next = 0;
    __amdgpu_buffer_rsrc_t buffer_a, buffer_b;
    const auto open = [&]() {
        const bool some = find_tile<TM, TN>(p, (int32_t)blockIdx.x, turn, next);
        k_next = next.from;
        if (!some) {  // nothing is read any more
            next.rows_a = next.rows_b = 0;
            next.end = 1 << 30;
            k_next = 0;
        }
        ++turn;
        if (ALIGNED) {
            buffer_a = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(next.a), 0, some ? (next.rows_a - 1) * (int32_t)p.a_stride + p.K : 0, kRawBuffer);
            buffer_b = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(next.b), 0, some ? (next.rows_b - 1) * (int32_t)p.b_stride + p.K : 0, kRawBuffer);
        }
        return some;
    };
    const auto advance = [&]() {
        k_next += kTileK;
        if (k_next >= next.end) open();
    };
    i32x4 held[kLoads];
    const auto load = [&](int i) {  // those of a first
        const bool of_a = i < kLoadsA;
        const int j = of_a ? i : i - kLoadsA;
        if (ALIGNED) {
            // behind the row's end: a place beyond the buffer, for one side
            const uint32_t beyond = k_next + piece < next.end ? 0u : 1u << 31;
            held[i] = __builtin_bit_cast(i32x4, of_a ? __builtin_amdgcn_raw_buffer_load_b128(buffer_a, (at_a + ((uint32_t)k_next + j * step_a)) | beyond, 0, 0)
                                                     : __builtin_amdgcn_raw_buffer_load_b128(buffer_b, at_b + ((uint32_t)k_next + j * step_b), 0, 0));
        } else {
            const int8_t* const row = of_a ? next.a + min(row0 + j * kRowsAtOnce, next.rows_a - 1) * p.a_stride
                                           : next.b + min(row0 + j * kRowsAtOnce, next.rows_b - 1) * p.b_stride;
            if (next.rows_a == 0) held[i] = i32x4{0, 0, 0, 0};
            else if (k_next + kTileK <= next.end) held[i] = load16(row + k_next + piece);
            else held[i] = load16(row, k_next + piece, next.end);
        }
    };
    const int32_t put_at = row0 * kTileK + (piece ^ (row0 / 2 % 8 * 16));
    const auto put = [&](int i, int buffer) {
        *reinterpret_cast<i32x4*>(lds + buffer * kBuffer + put_at + i * kRowsAtOnce * kTileK) = held[i];
    };
    const int32_t wm = wave % WM * (TM / WM), wn = wave / WM * (TN / WN);
    const int32_t r = lane % 32, half = lane / 32 * 16, order = r / 2 % 8 * 16;
    const int8_t* const read_a = lds + (wm + r) * kTileK;
    const int8_t* const read_b = lds + (TM + wn + r) * kTileK;
    i32x4 fa[2][kMi], fb[2][kNi];
    const auto read = [&](int buffer, int step, int set) {
        const int32_t at = buffer * kBuffer + ((step * 32 + half) ^ order);
#pragma unroll
        for (int i = 0; i < kNi; ++i) fb[set][i] = *reinterpret_cast<const i32x4*>(read_b + at + i * 32 * kTileK);
#pragma unroll
        for (int i = 0; i < kMi; ++i) fa[set][i] = *reinterpret_cast<const i32x4*>(read_a + at + i * 32 * kTileK);
    };
    if (!open()) return;
    ProductTile tile = next;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load(i);
    advance();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        put(i, 0);
        load(i);
    }
    // (where a tile is one piece long the stream is a tile ahead already)
    __syncthreads();
    read(0, 0, 0);
    int buffer = 0;
    for (int32_t mine = 1;; ++mine) {
        // held until they are wanted, behind the products
        const float own_a = tid < tile.rows_a ? p.a_scale[tile.m0 + tid] : 0.0f;
        const float own_b = tid < tile.rows_b ? p.b_scale[tile.n0 + tid] : 0.0f;
        i32x16 sum[kNi][kMi];
#pragma unroll
        for (int n = 0; n < kNi; ++n)
#pragma unroll
            for (int m = 0; m < kMi; ++m)
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[n][m][i] = 0;
        int32_t k = tile.from;
        do {
            advance();
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                if (s == kSteps - 1) __syncthreads();  // the next piece is there, and nobody reads this one any more
                if (s < kSteps - 1) read(buffer, s + 1, (s + 1) % 2);
                else read(buffer ^ 1, 0, 0);
                // the next piece into LDS, half of it at a time, and the one after it into the registers that this frees
                if (s == 1 || s == 2) {
#pragma unroll
                    for (int i = (s - 1) * kLoads / 2; i < s * kLoads / 2; ++i) {
                        put(i, buffer ^ 1);
                        load(i);
                    }
                }
#pragma unroll
                for (int n = 0; n < kNi; ++n)
#pragma unroll
                    for (int m = 0; m < kMi; ++m)
                        sum[n][m] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[s % 2][n], fa[s % 2][m], sum[n][m], 0, 0, 0);
                interleave<kMi * kNi, kMi + kNi, (kLoads + 1) / 2>(s == 1 || s == 2);
                __builtin_amdgcn_sched_barrier(0);
            }
            buffer ^= 1;
            k += kTileK;
        } while (k < tile.end);
        // (the sums stay in their registers until they are written: the compiler fetched them in every turn of the loop, or all at
        // once behind it.  With all 512 registers of a lane taken, tiles of 256 x 256 still put 132 to 192 bytes into memory, before the
        // loops, that are read between a tile's products and its way out, none in the loop of products)
#pragma unroll
        for (int n = 0; n < kNi; ++n)
#pragma unroll
            for (int m = 0; m < kMi; ++m) asm volatile("" : "+a"(sum[n][m]));
        // A lane has 4 adjacent classes of a row at a time.  A wave's 32 rows pass through LDS, by the piece that nobody reads
        // any more, as 32-bit words, so that what goes to memory are rows' 16-byte pieces side by side and a lane needs
        // the same classes' scales all along: stores straight from the registers took longer than the products of 4096
        // numbers, scales fetched beside each 4 sums a third of that.
        if (tid < TM) scale_a[tid] = own_a;
        if (tid < TN) scale_b[tid] = own_b;
        __syncthreads();
        const auto write = [&](auto* out, int64_t stride, auto before, auto behind) {
            using O = std::remove_pointer_t<decltype(out)>;
            constexpr int kEach = 16 / (int)sizeof(O), kBlocks = Stage::kBlocks, kRow = Stage::kRow;
            constexpr int kPieces = kBlocks * 32 / kEach, kRowsEach = kWave / kPieces;
            uint32_t* const stage = reinterpret_cast<uint32_t*>(
                wave < Stage::kInside ? lds + (buffer ^ 1) * kBuffer + wave * Stage::kBytes
                                      : reinterpret_cast<int8_t*>(scale_b + TN) + (wave - Stage::kInside) * Stage::kBytes);
            const int32_t c = lane % kPieces * kEach, row1 = lane / kPieces;
            float sa[kMi];
#pragma unroll
            for (int m = 0; m < kMi; ++m) sa[m] = scale_a[wm + 32 * m + r];
#pragma unroll
            for (int n0 = 0; n0 < kNi; n0 += kBlocks) {
                float sb[kEach];
#pragma unroll
                for (int i = 0; i < kEach; ++i) sb[i] = scale_b[wn + 32 * n0 + c + i];
                const int32_t left = tile.rows_b - wn - 32 * n0 - c;
#pragma unroll
                for (int m = 0; m < kMi; ++m) {
#pragma unroll
                    for (int n = 0; n < kBlocks; ++n) {
                        i32x16 block = sum[n0 + n][m];
                        asm volatile("" : "+a"(block));
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            uint4 w;
                            w.x = before(block[4 * q], sa[m]);
                            w.y = before(block[4 * q + 1], sa[m]);
                            w.z = before(block[4 * q + 2], sa[m]);
                            w.w = before(block[4 * q + 3], sa[m]);
                            *reinterpret_cast<uint4*>(stage + r * kRow + 32 * n + 8 * q + lane / 32 * 4) = w;
                        }
                    }
                    wave_lds_order();
                    O* to = out + (tile.m0 + wm + 32 * m + row1) * stride + tile.n0 + wn + 32 * n0 + c;
#pragma unroll
                    for (int j = 0; j < 32 / kRowsEach; ++j, to += kRowsEach * stride) {
                        const int32_t row = row1 + j * kRowsEach;
                        uint32_t w[kEach];
#pragma unroll
                        for (int i = 0; i < kEach; i += 4)
                            *reinterpret_cast<uint4*>(w + i) = *reinterpret_cast<const uint4*>(stage + row * kRow + c + i);
                        const uint4 v = behind(w, sb);
                        if (wm + 32 * m + row >= tile.rows_a || left <= 0) continue;
                        if (left >= kEach) {
                            __builtin_memcpy(to, &v, 16);  // the hardware takes unaligned addresses
                        } else {
                            O each[kEach];
                            __builtin_memcpy(each, &v, 16);
#pragma unroll
                            for (int i = 0; i < kEach; ++i)
                                if (i < left) to[i] = each[i];
                        }
                    }
                    wave_lds_order();
                }
            }
        };
        if (p.splits > 1) {
            write(p.partial + (int64_t)tile.split * p.M * p.N, (int64_t)p.N, [](int32_t s, float) { return (uint32_t)s; },
                  [](const uint32_t (&w)[4], const float (&)[4]) { return make_uint4(w[0], w[1], w[2], w[3]); });
        } else {
            write(static_cast<T*>(p.out), p.out_stride, [](int32_t s, float sa) { return __float_as_uint((float)s * sa); },
                  [](const uint32_t (&w)[Row<T>::kChunk], const float (&sb)[Row<T>::kChunk]) {
                      float v[Row<T>::kChunk];
#pragma unroll
                      for (int i = 0; i < Row<T>::kChunk; ++i) v[i] = scaled(__uint_as_float(w[i]), sb[i]);
                      return Row<T>::pack(v);
                  });
        }
        if (!find_tile<TM, TN>(p, (int32_t)blockIdx.x, mine, tile)) return;
        __syncthreads();  // the stream goes on into what this has passed through
    }
}

// Rows that lie anywhere, side by side in pieces of 16 bytes, with zeros behind a row's end; a wave a row.  Both
// sides in one launch.
struct PackArgs {
    const int8_t* from[2];
    int64_t stride[2], rows[2];
    i32x4* to[2];
    int32_t width;
};
__global__ __launch_bounds__(256) void product_pack_kernel(PackArgs p)
{
    const int side = (int)blockIdx.y;
    const int8_t* const from = side ? p.from[1] : p.from[0];
    const int64_t stride = side ? p.stride[1] : p.stride[0], rows = side ? p.rows[1] : p.rows[0];
    i32x4* const to = side ? p.to[1] : p.to[0];
    const int32_t pieces = (p.width + 15) / 16;
    for (int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave; row < rows; row += (int64_t)gridDim.x * 4)
        for (int32_t i = threadIdx.x % kWave; i < pieces; i += kWave) to[row * pieces + i] = load16(from + row * stride, i * 16, p.width);
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
    if (d->rows > (int64_t)1 << 31 || d->rows * d->classes > (int64_t)1 << 40)
        return fail(nullptr, LDA_ERR_UNSUPPORTED, "%s: at most 2^31 rows and 2^40 results", call);
    if (d->rows == 0) return LDA_OK;
    if (!d->a_scale || !d->b_scale || (d->width > 0 && (!d->a || !d->b)))
        return fail(nullptr, LDA_ERR_ARG, "%s: NULL pointer", call);
    if (!aligned_to(d->a_scale, 4) || !aligned_to(d->b_scale, 4))
        return fail(nullptr, LDA_ERR_ARG, "%s: a pointer is not aligned to its type", call);
    return LDA_OK;
}

enum class ProductKind { kFew, kTile64, kTile128, kTile256 };
struct ProductPlan {
    ProductKind kind;
    int classes, splits;    // of the few-rows kernel: 16-class tiles of a wave
    int32_t split_k;
    bool aligned;           // for the tiles' buffers; otherwise rows are read where they lie
    int64_t a_bytes, b_bytes;  // of rows that are packed first
};
// Loads of 16 bytes at multiples of 16, places inside a tile in 32 bits
static bool in_pieces(const void* p, int64_t stride)
{
    return aligned_to(p, 16) && stride % 16 == 0 && stride >= 0 && stride < 1 << 22;
}
static ProductPlan plan_product(const lda_product_rows* d)
{
    ProductPlan p{};
    int64_t groups;
    const auto tiles = [&](int64_t m, int64_t n) { return ((d->rows + m - 1) / m) * ((d->classes + n - 1) / n); };
    const bool whole = d->width % 16 == 0, a_fine = whole && in_pieces(d->a, d->a_stride), b_fine = whole && in_pieces(d->b, d->b_stride);
    p.aligned = a_fine && b_fine;
    // 16 x 5120 x 101636: 137 us by the few-rows kernel, 106 by tiles; 16 x 4096 x 10000: 15.5 and 16 (in 3 splits, two
    // launches); 8 x 4096 x 141043: 119 and 127
    if (d->rows <= 8 || (d->rows <= 16 && d->classes < 65536)) {
        p.kind = ProductKind::kFew;
        p.classes = d->classes >= 32768 ? 4 : d->classes >= 16384 ? 2 : 1;
        groups = tiles(16, 16 * p.classes);
    } else if (d->rows <= 64) {
        p.kind = ProductKind::kTile64;
        groups = tiles(64, 128);
    } else {
        // 4096 x 4096 x 32768 (2048 tiles of 256 x 256): 544 us by these, 810 by 128 x 128; 2048 x 4096 x 10000 (320): 113 and 99.
        // Between the two what counts is how full the last round of 256 CUs is (4096 x 4096 x 8192, two whole rounds: 137 and 166),
        // which this rule does not ask.
        // Up to 128 rows half of a larger tile would be empty (100 x 4096 x 200003: 194 us by 128 x 128, 259), and nothing is
        // packed, while the larger tile has buffers alone.
        p.kind = d->rows > 128 && tiles(256, 256) >= 768 ? ProductKind::kTile256 : ProductKind::kTile128;
        groups = p.kind == ProductKind::kTile256 ? tiles(256, 256) : tiles(128, 128);
        const int64_t packed = ((int64_t)d->width + 15) / 16 * 16;
        // 516 x 7937 x 21153: 277 us as they lie, 245 packed first (227 on another card, 56 of it the packing); 87 x 10049 x 14837:
        // 76 and 105
        if (d->rows > 128 && !a_fine) p.a_bytes = d->rows * packed;
        if (d->rows > 128 && !b_fine) p.b_bytes = d->classes * packed;
        if (d->rows > 128) p.aligned = true;
    }
    // A split's second kernel takes 4 to 5 us and a launch, so that a split has some bytes of a row at least.  1 x 16384 x
    // 1000: 11 us whole, 12 to 15 in 2 splits; 1 x 131008 x 1000: 81 whole, 29 in 4 (as many as 63 workgroups make), 27 in 16; 300 x
    // 2048 x 2000: 12 whole, 16 in 2; 300 x 8192 x 1000: 33 and 20 in 4
    int64_t splits = groups >= 192 ? 1 : 256 / (groups < 1 ? 1 : groups);
    const int64_t most = d->width / (p.kind == ProductKind::kFew ? 16384 : 2048);
    if (splits > most) splits = most;
    if (splits < 1) splits = 1;
    const int64_t pieces = ((int64_t)d->width + kTileK - 1) / kTileK;
    const int64_t each = pieces < 1 ? 1 : (pieces + splits - 1) / splits;
    p.split_k = (int32_t)(each * kTileK);
    p.splits = pieces < 1 ? 1 : (int)((pieces + each - 1) / each);
    return p;
}

static int64_t product_bytes(const lda_product_rows* d)
{
    if (d->rows == 0 || d->width == 0) return 0;
    const ProductPlan p = plan_product(d);
    return p.a_bytes + p.b_bytes + (p.splits == 1 ? 0 : (int64_t)p.splits * d->rows * d->classes * (int64_t)sizeof(int32_t));
}

template <class T>
static void launch_join(const ProductArgs& a, hipStream_t stream)
{
    const int64_t n = (a.M * a.N + 255) / 256;
    product_join_kernel<T><<<(unsigned)(n < 8192 ? n : 8192), 256, 0, stream>>>(a);
}

// Packs the sides that the plan wants packed to the workspace's beginning; returns what lies behind
static int8_t* pack(ProductArgs& a, const ProductPlan& plan, int8_t* room, hipStream_t stream)
{
    if (plan.a_bytes == 0 && plan.b_bytes == 0) return room;
    PackArgs p{};
    const int64_t packed = ((int64_t)a.K + 15) / 16 * 16;
    p.width = a.K;
    if (plan.a_bytes > 0) {
        p.from[0] = a.a;
        p.stride[0] = a.a_stride;
        p.rows[0] = a.M;
        p.to[0] = reinterpret_cast<i32x4*>(room);
        a.a = room;
        a.a_stride = packed;
        room += plan.a_bytes;
    }
    if (plan.b_bytes > 0) {
        p.from[1] = a.b;
        p.stride[1] = a.b_stride;
        p.rows[1] = a.N;
        p.to[1] = reinterpret_cast<i32x4*>(room);
        a.b = room;
        a.b_stride = packed;
        room += plan.b_bytes;
    }
    a.K = (int32_t)packed;  // with the zeros
    const int64_t blocks = ((p.rows[0] > p.rows[1] ? p.rows[0] : p.rows[1]) + 3) / 4;
    product_pack_kernel<<<dim3((unsigned)(blocks < 16384 ? blocks : 16384), 2), 256, 0, stream>>>(p);
    return room;
}

template <class T>
static hipError_t launch_product(ProductArgs a, const ProductPlan& plan, hipStream_t stream)
{
    a.splits = plan.splits;
    a.split_k = plan.split_k;
    const auto few = [&](auto ct) {
        // a launch has less than 2^32 threads
        constexpr int32_t kMost = 1 << 22;
        const int32_t blocks = (int32_t)(((int64_t)a.N + 16 * ct() - 1) / (16 * ct()));
        for (a.block0 = 0; a.block0 < blocks; a.block0 += kMost) {
            const dim3 grid((unsigned)(blocks - a.block0 < kMost ? blocks - a.block0 : kMost), (unsigned)a.splits);
            product_few_kernel<T, ct()><<<grid, 256, 0, stream>>>(a);
        }
    };
    const auto tile = [&](auto tm, auto tn, auto wm, auto wn, auto aligned) {
        a.tiles_m = (int32_t)((a.M + tm() - 1) / tm());
        a.tiles_n = (int32_t)(((int64_t)a.N + tn() - 1) / tn());
        constexpr size_t lds = ProductStage<tm(), tn(), wm(), wn()>::kLds;
        const auto kernel = product_tile_kernel<T, tm(), tn(), wm(), wn(), aligned()>;
        if (lds > 65536) {
            static std::atomic<uint64_t> allowed{0};  // a bit a device: once is enough
            int device = 0;
            hipError_t e = hipGetDevice(&device);
            if (e != hipSuccess) return e;
            if (device > 63 || !(allowed.load(std::memory_order_relaxed) >> device & 1)) {
                e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
                if (e != hipSuccess) return e;
                if (device <= 63) allowed.fetch_or((uint64_t)1 << device, std::memory_order_relaxed);
            }
        }
        // as many workgroups as there is room for at once, a multiple of the XCDs
        const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n * a.splits, room = kCus * (int64_t)(kLdsOfCu / lds);
        const unsigned n = (unsigned)(((tiles < room ? tiles : room) + kXcds - 1) / kXcds * kXcds);
        kernel<<<n, wm() * wn() * 64, lds, stream>>>(a);
        return hipSuccess;
    };
    using std::integral_constant;
    if (plan.kind == ProductKind::kFew) {
        if (plan.classes == 4) few(integral_constant<int, 4>{});
        else if (plan.classes == 2) few(integral_constant<int, 2>{});
        else few(integral_constant<int, 1>{});
    } else {
        const auto c256 = integral_constant<int, 256>{};
        const auto c128 = integral_constant<int, 128>{};
        const auto c64 = integral_constant<int, 64>{};
        const auto c2 = integral_constant<int, 2>{};
        constexpr std::true_type yes{};
        if (plan.kind == ProductKind::kTile256 && !plan.aligned) return hipErrorInvalidValue;  // no plan has this
        const hipError_t e = plan.kind == ProductKind::kTile256   ? tile(c256, c256, c2, c2, yes)
                             : plan.kind == ProductKind::kTile128 ? (plan.aligned ? tile(c128, c128, c2, c2, yes) : tile(c128, c128, c2, c2, std::false_type{}))
                             : plan.aligned                       ? tile(c64, c128, c2, c2, yes)
                                                                  : tile(c64, c128, c2, c2, std::false_type{});
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
    const hipStream_t stream = static_cast<hipStream_t>(d->hip_stream);
    const ProductPlan plan = plan_product(d);
    a.partial = reinterpret_cast<int32_t*>(a.K > 0 ? pack(a, plan, static_cast<int8_t*>(d->workspace), stream) : nullptr);
    const auto typed = [&](auto t) -> hipError_t {
        using T = decltype(t);
        if (a.K == 0) {
            launch_join<T>(a, stream);
            return hipGetLastError();
        }
        return launch_product<T>(a, plan, stream);
    };
    const hipError_t e = d->out_type == LDA_F32 ? typed(float{}) : d->out_type == LDA_F16 ? typed(__half{}) : typed(__hip_bfloat16{});
    LDA_HIP(static_cast<lda_ctx*>(nullptr), e);
    return LDA_OK;
} catch (...) {
    return LDA_ERR_OOM;
}

}  // extern "C"
