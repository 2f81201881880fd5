// Linear maps per group of consecutive rows:  y[r] = x[r] w[g];  dx[r] = dy[r] w[g]^T;  dw[g] = x_g^T dy_g  (r in group g).
// Groups have any sizes, so the work is cut into output tiles and a workgroup finds its tile from the offsets: tiles of rows are
// counted per group (a launch has room for the tiles of any division of the rows, those left over end at once).
// The products run on the matrix cores (grouped_tile.h).
// Measured, bf16 (a large product of the library reaches 1110 TFLOP/s here, under the power limit): 262 144 rows in 16 groups, 1024 -> 4096,
// forward 2.14 ms (1030 TFLOP/s), gradient of the rows 2.02 (1090), of the weights 2.2 to 2.4 (920 to 1000); 139 264 rows in 8 groups, 256 -> 768:
// 85, 65 and 79 us, where 56 are the bytes of each.  One row in each of 16 groups, 4096 -> 4096: 76 us = 7.0 TB/s of weights.  fp32: 30 000
// rows, 2048 -> 2048, 1.8 ms (140 TFLOP/s of 154).  The matrix units are busy for 58 % of the cycles of a long product, at 1.65 GHz; other
// orders of the loads and reads of a step, priorities and tiles of four waves moved nothing by more than the clock does.
#include <cmath>

#include "grouped_tile.h"
#include "layers.h"

namespace kunlun {

namespace {

// Tile t of the tiles of `height` rows of all groups: its group, first row and number of rows (0: there is no such tile).  The rows
// behind the last group count as group G.  slot: how many tiles of groups of several tiles come before it (-1: its group has no other).
// Called by whole waves.
struct RowTile {
    int group, rows, slot;
    int64_t row0;
};
__device__ __forceinline__ int tiles_of(const int32_t* offsets, int G, int64_t total, int height, int g, int64_t& lo, int& len) {
    lo = offsets[g < G ? g : G];
    int64_t hi = g < G ? offsets[g + 1] : total;
    if (hi > total) hi = total;
    if (lo < 0) lo = 0;
    len = g <= G && hi > lo ? (int)(hi - lo) : 0;
    return (int)(((int64_t)len + height - 1) / height);
}
__device__ __forceinline__ int wave_prefix(int x) {  // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const int v = __shfl_up(x, o);
        if (lane >= o) x += v;
    }
    return x;
}
template <bool SLOTS>
__device__ __forceinline__ RowTile find_row_tile(const int32_t* offsets, int G, int64_t total, int height, int64_t t) {
    const int lane = threadIdx.x & 63;
    RowTile r = {0, 0, -1, 0};
    int slots = 0;
    for (int g0 = 0; g0 <= G; g0 += 64) {
        int64_t lo;
        int len;
        const int tiles = tiles_of(offsets, G, total, height, g0 + lane, lo, len);
        const int upto = wave_prefix(tiles);
        const int shared = SLOTS ? wave_prefix(tiles > 1 ? tiles : 0) : 0;
        const uint64_t beyond = __builtin_amdgcn_ballot_w64(upto > t);
        if (beyond) {
            const int at = __ffsll((unsigned long long)beyond) - 1;
            const int n = __builtin_amdgcn_readlane(tiles, at), k = (int)(t - (__builtin_amdgcn_readlane(upto, at) - n));
            r.group = g0 + at;
            r.row0 = __builtin_amdgcn_readlane((int)lo, at) + (int64_t)k * height;
            const int64_t left = __builtin_amdgcn_readlane(len, at) - (int64_t)k * height;
            r.rows = left < height ? (int)left : height;
            if (SLOTS && n > 1) r.slot = slots + __builtin_amdgcn_readlane(shared, at) - n + k;
            break;
        }
        t -= __builtin_amdgcn_readlane(upto, 63);
        if (SLOTS) slots += __builtin_amdgcn_readlane(shared, 63);
    }
    return r;
}
// All tiles, with those behind the last group or without.
__device__ __forceinline__ int64_t count_row_tiles(const int32_t* offsets, int G, int64_t total, int height, bool rest) {
    int64_t n = 0;
    for (int g0 = 0; g0 <= G; g0 += 64) {
        const int g = g0 + (int)(threadIdx.x & 63);
        int64_t lo;
        int len;
        const int tiles = tiles_of(offsets, G, total, height, g, lo, len);
        n += __builtin_amdgcn_readlane(wave_prefix(g < G || rest ? tiles : 0), 63);
    }
    return n;
}
// Row tiles that a launch has room for: every group, and the rows behind them, may end inside a tile.
int64_t row_tiles(int G, int64_t total, int height) { return (total + height - 1) / height + G + 1; }

// Which output tile a workgroup takes, of m_tiles x n_tiles that there are (m_tiles is known on the device only).  Workgroup i runs on XCD
// i % 8, and each XCD has its own L2: it takes `unit` tiles in a row (what it computes at a time), the XCDs in turn, and what is left of
// the last turn is split evenly.  Tiles are numbered in bands of `band` row tiles, column after column, so that those at work on an XCD
// share rows of one operand and columns of the other.
__device__ __forceinline__ bool tile_of(int64_t m_tiles, int n_tiles, int band, int unit, int64_t& mt, int& nt) {
    const int64_t id = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, xcd = id & 7, j = id >> 3;
    const int64_t all = m_tiles * n_tiles, turns = all / (8 * unit), rest = all - turns * 8 * unit, per = (rest + 7) / 8;
    int64_t at = j / unit < turns ? (j / unit * 8 + xcd) * unit + j % unit : turns * 8 * unit + xcd * per + (j - turns * unit);
    if (j / unit >= turns && (j - turns * unit >= per || at >= all)) return false;
    const int64_t b = at / ((int64_t)band * n_tiles), first = b * band;
    const int in = (int)(at - first * n_tiles), height = m_tiles - first < band ? (int)(m_tiles - first) : band;
    mt = first + in % height;
    nt = in / height;
    return true;
}
// Room for `all` tiles (two dimensions: one holds at most 2^32 threads)
dim3 tile_grid(int64_t all, int threads) {
    all = (all + 7) / 8 * 8;
    const int64_t most = largest_grid(threads) / 8 * 8;
    return all <= most ? dim3((unsigned)all) : dim3((unsigned)most, (unsigned)((all + most - 1) / most));
}

// out[r, :] = in[r, :] W  (B_COLUMNS: W = w[g] [K, N];  else W = w[g]^T of w[g] [N, K])
template <typename S, typename T, bool B_COLUMNS>
__global__ __launch_bounds__(S::THREADS, 2) void grouped_rows_kernel(const T* __restrict__ in, const T* __restrict__ w, T* __restrict__ out,
                                                                  const int32_t* __restrict__ offsets, int G, int64_t total, int K, int N,
                                                                  bool fill_rest, int n_tiles, int band) {
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int64_t mt;
    int nt;
    if (!tile_of(count_row_tiles(offsets, G, total, S::BM, fill_rest), n_tiles, band, 32 * S::PER_CU, mt, nt)) return;
    constexpr uint32_t E = sizeof(T);
    const RowTile t = find_row_tile<false>(offsets, G, total, S::BM, mt);
    const int n0 = nt * S::BN;
    f32x16 acc[S::NB][S::MB] = {};
    if (t.group < G) {
        const T* wg = w + (int64_t)t.group * K * N;
        const GroupedOperand a = {(const char*)(in + t.row0 * K), (uint32_t)K * E, t.rows};
        const GroupedOperand b = {(const char*)(B_COLUMNS ? wg + n0 : wg + (int64_t)n0 * K), (uint32_t)(B_COLUMNS ? N : K) * E, N - n0};
        grouped_product<S, T, false, B_COLUMNS>(acc, lds, a, b, K, lane, wave);
    }
    grouped_store<S, T>(acc, lds, out + t.row0 * N + n0, N, t.rows, N - n0, lane, wave);
}

// The same for few rows and long contractions: 32 x 32 outputs per workgroup, whose eight waves take an eighth of the contraction each, through
// rings of their own (no barriers), and add up in order.  Five rows of 3416 values, 464 columns, fp32: 18 us (70 by Small tiles); bound by the latency of a wave's steps.
constexpr int DEEP = 32, DEEP_WAVES = 8;
template <typename T, bool B_COLUMNS>
__global__ __launch_bounds__(64 * DEEP_WAVES, 2) void grouped_rows_deep_kernel(const T* __restrict__ in, const T* __restrict__ w, T* __restrict__ out,
                                                                               const int32_t* __restrict__ offsets, int G, int64_t total, int K,
                                                                               int N, bool fill_rest, int n_tiles, int band) {
    using S = GroupedShape<DEEP, DEEP, 1, 1, 2>;  // of one wave
    __shared__ __attribute__((aligned(1024))) char lds[DEEP_WAVES * 2 * S::STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int64_t mt;
    int nt;
    if (!tile_of(count_row_tiles(offsets, G, total, DEEP, fill_rest), n_tiles, band, 32, mt, nt)) return;
    constexpr uint32_t E = sizeof(T);
    const RowTile t = find_row_tile<false>(offsets, G, total, DEEP, mt);
    const int n0 = nt * DEEP;
    f32x16 acc[1][1] = {};
    char* const mine = lds + wave * (2 * S::STAGE);
    if (t.group < G) {
        const T* wg = w + (int64_t)t.group * K * N;
        GroupedDma<T, DEEP, 1, false> dma_a;
        GroupedDma<T, DEEP, 1, B_COLUMNS> dma_b;
        dma_a.init({(const char*)(in + t.row0 * K), (uint32_t)K * E, t.rows}, lane, 0);
        dma_b.init({(const char*)(B_COLUMNS ? wg + n0 : wg + (int64_t)n0 * K), (uint32_t)(B_COLUMNS ? N : K) * E, N - n0}, lane, 0);
        GroupedFrag<T, DEEP, false> frag_a;
        GroupedFrag<T, DEEP, B_COLUMNS> frag_b;
        frag_a.init(lane, 0);
        frag_b.init(lane, 0);
        constexpr int STEP = decltype(dma_a)::STEP, LOADS = decltype(dma_a)::LOADS + decltype(dma_b)::LOADS;
        const int steps = (K + STEP - 1) / STEP, per = (steps + DEEP_WAVES - 1) / DEEP_WAVES;
        const int k0 = wave * per, k1 = k0 + per < steps ? k0 + per : steps;
        const uint32_t lds0 = lds_address(mine);
        auto issue = [&](int k) {
            const uint32_t stage = lds0 + (k & 1) * S::STAGE;
            dma_a.issue(k, K - k * STEP, stage);
            dma_b.issue(k, K - k * STEP, stage + S::A_BYTES);
        };
        if (k0 < k1) issue(k0);
        for (int k = k0; k < k1; ++k) {
            wait_lds();  // the reads of the step before: its stage is loaded next
            if (k + 1 < k1) {
                issue(k + 1);
                wait_vmcnt<LOADS>();
            } else {
                wait_vmcnt<0>();
            }
            asm volatile("" ::: "memory");  // (the step is read behind the wait)
            const char* ta = mine + (k & 1) * S::STAGE;
            grouped_step<S, T>(acc, ta, ta + S::A_BYTES, frag_a, frag_b);
        }
        wait_lds();
    }
    // a wave's sums as rows of 33 floats in its own ring; then two outputs per thread
    float* const sums = (float*)mine;
#pragma unroll
    for (int v = 0; v < 16; ++v) sums[(lane & 31) * 33 + c_row(v, lane >> 5)] = acc[0][0][v];
    __syncthreads();
    const int m = threadIdx.x / 16, n = threadIdx.x % 16 * 2;
    float total_0 = 0.f, total_1 = 0.f;
#pragma unroll
    for (int q = 0; q < DEEP_WAVES; ++q) {
        const float* const p = (const float*)(lds + q * (2 * S::STAGE)) + m * 33 + n;
        total_0 += p[0];
        total_1 += p[1];
    }
    if (m < t.rows && n0 + n < N) {
        T* const o = out + (t.row0 + m) * N + n0 + n;
        o[0] = from_float<T>(total_0);
        o[1] = from_float<T>(total_1);
    }
}

// dw[g] = x^T dy over a range of `height` rows of group g, to dw where the group has no other range, else to the range's slot of `partial`.
template <typename S, typename T>
__global__ __launch_bounds__(S::THREADS) void grouped_weights_kernel(const T* __restrict__ x, const T* __restrict__ dy, T* __restrict__ dw,
                                                                     float* __restrict__ partial, const int32_t* __restrict__ offsets, int G,
                                                                     int64_t total, int K, int N, int height, int64_t slots, int n_tiles, int band) {
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int64_t mt;
    int nt;
    const int k_tiles = (K + S::BM - 1) / S::BM;
    if (!tile_of(count_row_tiles(offsets, G, total, height, false) * k_tiles, n_tiles, band, 32 * S::PER_CU, mt, nt)) return;
    const RowTile t = find_row_tile<true>(offsets, G, total, height, mt / k_tiles);
    if (t.slot >= slots) return;  // (offsets that are none)
    const int k0 = (int)(mt % k_tiles) * S::BM, n0 = nt * S::BN;
    const GroupedOperand a = {(const char*)(x + t.row0 * K + k0), (uint32_t)(K * sizeof(T)), K - k0};
    const GroupedOperand b = {(const char*)(dy + t.row0 * N + n0), (uint32_t)(N * sizeof(T)), N - n0};
    f32x16 acc[S::NB][S::MB] = {};
    grouped_product<S, T, true, true>(acc, lds, a, b, t.rows, lane, wave);
    if (t.slot < 0)
        grouped_store<S, T>(acc, lds, dw + ((int64_t)t.group * K + k0) * N + n0, N, K - k0, N - n0, lane, wave);
    else
        grouped_store<S, float>(acc, lds, partial + ((int64_t)t.slot * K + k0) * N + n0, N, K - k0, N - n0, lane, wave);
}

// dw[g] where group g has not exactly one range: the sum of its slots in order, zeros without any.  Four values per thread.
constexpr int SLOT_FETCH = 8;  // loads in flight
template <typename T>
__global__ __launch_bounds__(256) void grouped_join_kernel(const float* __restrict__ partial, T* __restrict__ dw,
                                                           const int32_t* __restrict__ offsets, int G, int64_t total, int64_t per_group, int height,
                                                           int64_t slots) {
    const int g = blockIdx.y;
    int64_t lo;
    int len, slot = 0;
    for (int g0 = 0; g0 < g; g0 += 64) {
        int n = tiles_of(offsets, G, total, height, g0 + (threadIdx.x & 63), lo, len);
        if (n <= 1 || g0 + (int)(threadIdx.x & 63) >= g) n = 0;
        slot += __builtin_amdgcn_readlane(wave_prefix(n), 63);
    }
    const int ranges = tiles_of(offsets, G, total, height, g, lo, len);
    if (ranges == 1 || (ranges > 1 && slot + ranges > slots)) return;  // (the second: offsets that are none)
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < per_group; i += (int64_t)gridDim.x * 1024) {
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        const float* p = partial + (int64_t)slot * per_group + i;
        for (int k = 0; k < ranges; k += SLOT_FETCH) {
            f32x4 x[SLOT_FETCH];
#pragma unroll
            for (int u = 0; u < SLOT_FETCH; ++u) x[u] = __builtin_nontemporal_load((const f32x4*)(p + (int64_t)(k + u < ranges ? k + u : k) * per_group));
#pragma unroll
            for (int u = 0; u < SLOT_FETCH; ++u)
                if (k + u < ranges) sum += x[u];
        }
        typedef __attribute__((ext_vector_type(4))) T T4;
        T4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (T)sum[e];
        *(T4*)(dw + g * per_group + i) = o;
    }
}

constexpr int BAND = 4;  // row tiles of a band (tile_of)

using Large = GroupedShape<256, 256, 2, 4, 2>;   // one workgroup of eight waves per compute unit
using Lower = GroupedShape<192, 256, 2, 4, 2>;   // likewise
using Middle = GroupedShape<128, 128, 2, 2, 2>;  // two of four waves
using Small = GroupedShape<64, 64, 2, 2, 3>;     // three of four waves, two steps in flight

template <typename S, typename T, bool B_COLUMNS>
void rows_of(const void* in, const void* w, void* out, const int32_t* offsets, int G, int64_t total, int K, int N, bool fill_rest,
             hipStream_t stream) {
    const int n_tiles = (N + S::BN - 1) / S::BN;
    hipLaunchKernelGGL((grouped_rows_kernel<S, T, B_COLUMNS>), tile_grid(row_tiles(G, total, S::BM) * n_tiles, S::THREADS), dim3(S::THREADS), 0, stream, (const T*)in, (const T*)w,
                       (T*)out, offsets, G, total, K, N, fill_rest, n_tiles, BAND);
}
template <typename T, bool B_COLUMNS>
void rows_deep(const void* in, const void* w, void* out, const int32_t* offsets, int G, int64_t total, int K, int N, bool fill_rest,
               hipStream_t stream) {
    const int n_tiles = (N + DEEP - 1) / DEEP;
    hipLaunchKernelGGL((grouped_rows_deep_kernel<T, B_COLUMNS>), tile_grid(row_tiles(G, total, DEEP) * n_tiles, 64 * DEEP_WAVES),
                       dim3(64 * DEEP_WAVES), 0, stream, (const T*)in, (const T*)w, (T*)out, offsets, G, total, K, N, fill_rest, n_tiles, BAND);
}

// Tiles of a launch that have rows, about: one per group where groups are smaller than a tile, else every group ends half a tile early.
int64_t tiles_with_rows(int G, int64_t total, int columns, int height, int width) {
    const int64_t groups = G < total ? G : total;
    return (total < groups * height ? groups : total / height + groups / 2) * ((columns + width - 1) / width);
}
// Whether 32 x 32 tiles of eight waves over the contraction are faster than Small ones of four over the outputs: us of their rounds (a round
// holds one Deep or three Small workgroups per compute unit) as measured; Small waits for each of its steps, Deep for an eighth of them.
// bf16: 5 rows, 3416 -> 464: 7.6 / 18.8 us, 64 rows, 4096 -> 4096: 13.5 / 22.0, 61 rows in 3 groups, 1264 -> 3728: 12.0 / 10.2; fp32: 18 / 70,
// 24 / 86, 20 / 30.
bool deep_pays(int G, int64_t total, int K, int N, int elt) {
    const int64_t steps = ((int64_t)K * elt + 127) / 128, cu = compute_units();
    const double deep = (double)((tiles_with_rows(G, total, N, DEEP, DEEP) + cu - 1) / cu) * (4 + 0.14 * steps);
    const double small = (double)((tiles_with_rows(G, total, N, 64, 64) + 3 * cu - 1) / (3 * cu)) * (3 + (elt == 4 ? 0.66 : 0.33) * steps);
    return deep < small;
}

// The largest tile of which there are enough to fill the device.  A Large tile moves least through LDS (262 144 rows, 1024 -> 4096: 1000
// TFLOP/s against 800 Middle and 520 Small) and pays from about 150 tiles on (20 000 rows, 512 -> 512, 170 tiles: 20 / 22 / 29 us; 16 groups
// of 128 rows, 4096 -> 1024, 64 tiles: 91 / 48 / 47 us); two Middle ones fit a compute unit, and the transposing reads of a Small one
// cost more (bf16, 16 groups of one row, 4096 -> 4096: 78 / 90 us; of w^T, 98 / 90 us).  fp32 is bound by the matrix instructions, so that
// idle compute units cost most (9973 rows, 200 -> 328, 240 Middle tiles: 34 / 23 us).
template <typename T, bool B_COLUMNS>
void rows(const void* in, const void* w, void* out, const int32_t* offsets, int G, int64_t total, int K, int N, bool fill_rest,
          hipStream_t stream) {
    const int cu = compute_units();
    if constexpr (sizeof(T) == 2)
        if (const int64_t large = tiles_with_rows(G, total, N, 256, 256); large >= cu * 6 / 10 && total >= 96 * (int64_t)(G < total ? G : total)) {
            // rounds of one tile per compute unit, a Lower one at 3/4 of the work and 1.1 times the time for it
            const int64_t lower = tiles_with_rows(G, total, N, 192, 256);
            if (total >= 512 * (int64_t)G && (lower + cu - 1) / cu * 192 * 11 < (large + cu - 1) / cu * 256 * 10)
                return rows_of<Lower, T, B_COLUMNS>(in, w, out, offsets, G, total, K, N, fill_rest, stream);
            return rows_of<Large, T, B_COLUMNS>(in, w, out, offsets, G, total, K, N, fill_rest, stream);
        }
    if (tiles_with_rows(G, total, N, 128, 128) >= (sizeof(T) == 2 && B_COLUMNS ? cu : 2 * cu))
        rows_of<Middle, T, B_COLUMNS>(in, w, out, offsets, G, total, K, N, fill_rest, stream);
    else if (deep_pays(G, total, K, N, sizeof(T)))
        rows_deep<T, B_COLUMNS>(in, w, out, offsets, G, total, K, N, fill_rest, stream);
    else
        rows_of<Small, T, B_COLUMNS>(in, w, out, offsets, G, total, K, N, fill_rest, stream);
}

// How the weights' gradient is cut: the tile, and the rows per range.
struct WeightsPlan {
    int tile, height;
    int64_t slots;
};
// Few ranges leave compute units idle or wait for the longest, many leave partial sums (8 bytes of traffic per weight and range) and
// short pipelines.  The fastest by a model of that: us per 64 rows of a tile when the device is full, and per tile beyond that, as measured (a
// Large tile at 1000 TFLOP/s, a Middle one at 850, a Small one at 500; fp32 at 135 and 120), traffic at 5 TB/s.  139 264 rows in 8 groups,
// 256 -> 768: 85 ranges of 1700 rows in one round of Large tiles, against 175 of 832 in three.
WeightsPlan plan_weights(int G, int64_t total, int K, int N, int dtype) {
    struct Tile {
        int size, per_cu;
        double step;
    };
    static constexpr Tile BF16[] = {{256, 1, 2.05}, {128, 2, 1.27}, {64, 2, 0.52}}, FP32[] = {{128, 2, 8.0}, {64, 2, 2.2}};
    constexpr double FIXED = 4.0;
    const double cu = compute_units(), groups = G < total ? G : total, more = groups / 2 + std::sqrt(groups / 3);  // last ranges of groups, hardly ever more
    WeightsPlan best = {64, 1 << 20, 0};
    double best_time = -1;
    for (int i = 0; i < (dtype == KUNLUN_FP32 ? 2 : 3); ++i) {
        const Tile t = dtype == KUNLUN_FP32 ? FP32[i] : BF16[i];
        const double tiles = (double)((K + t.size - 1) / t.size) * ((N + t.size - 1) / t.size), resident = cu * t.per_cu;
        const auto consider = [&](double rows) {
            const int64_t height = (int64_t)(rows / 64 + 1) * 64;
            if (height < 256 || height > (1 << 30)) return;
            const double length = height < total ? height : total, ranges = total / (double)height + more;
            const double rounds = ranges * tiles / resident, whole = length / 64 * t.step + FIXED;
            double time = rounds <= 1 ? whole : rounds * (total / ranges / 64 * t.step + FIXED) + whole;
            if (height < total) time += (total / (double)height + (height * groups < total ? groups / 2 : 0)) * K * N * 8 / 5e6;
            if (best_time < 0 || time < best_time) {
                best_time = time;
                best = {t.size, (int)height, 0};
            }
        };
        for (double rows = 512; rows < 2.0 * total + 512; rows *= 1.25) consider(rows);
        for (int r = 1; r <= 4; ++r)  // whole rounds
            if (const double ranges = r * resident / tiles - more; ranges >= 1) consider(total / ranges);
    }
    best.slots = best.height < total ? 2 * total / best.height : 0;  // (a group with a slot has more than one range, so more rows than one)
    return best;
}
template <typename S, typename T>
void weights_of(const WeightsPlan& p, const void* x, const void* dy, void* dw, float* partial, const int32_t* offsets, int G, int64_t total, int K,
                int N, hipStream_t stream) {
    const int n_tiles = (N + S::BN - 1) / S::BN, k_tiles = (K + S::BM - 1) / S::BM;
    hipLaunchKernelGGL((grouped_weights_kernel<S, T>), tile_grid(row_tiles(G, total, p.height) * k_tiles * n_tiles, S::THREADS), dim3(S::THREADS), 0, stream, (const T*)x, (const T*)dy, (T*)dw,
                       partial, offsets, G, total, K, N, p.height, p.slots, n_tiles,
                       k_tiles < BAND ? k_tiles : BAND);
}
template <typename T>
void weights(const void* x, const void* dy, void* dw, const int32_t* offsets, int G, int64_t total, int K, int N, int dtype, void* workspace,
             hipStream_t stream) {
    const WeightsPlan p = plan_weights(G, total, K, N, dtype);
    float* partial = (float*)workspace;
    if (total > 0) {
        if constexpr (sizeof(T) == 2)
            if (p.tile == 256) weights_of<Large, T>(p, x, dy, dw, partial, offsets, G, total, K, N, stream);
        if (p.tile == 128) weights_of<Middle, T>(p, x, dy, dw, partial, offsets, G, total, K, N, stream);
        if (p.tile == 64) weights_of<Small, T>(p, x, dy, dw, partial, offsets, G, total, K, N, stream);
    }
    const int64_t per_group = (int64_t)K * N, blocks = (per_group + 1023) / 1024;
    hipLaunchKernelGGL(grouped_join_kernel<T>, dim3((unsigned)(blocks < 1024 ? blocks : 1024), (unsigned)G), dim3(256), 0, stream, partial, (T*)dw,
                       offsets, G, total, per_group, p.height, p.slots);
}

}  // namespace

hipError_t launch_grouped_linear_fwd(const void* x, const void* w, void* y, const int32_t* offsets, int G, int64_t total, int K, int N,
                                     bool fill_rest, int dtype, hipStream_t stream) {
    if (dtype == KUNLUN_FP32) rows<float, true>(x, w, y, offsets, G, total, K, N, fill_rest, stream);
    else rows<bf16_t, true>(x, w, y, offsets, G, total, K, N, fill_rest, stream);
    return hipGetLastError();
}

size_t grouped_linear_bwd_workspace(int G, int64_t total, int K, int N, int dtype) {
    return align_up(256 + (size_t)plan_weights(G, total, K, N, dtype).slots * K * N * sizeof(float), 256);
}

hipError_t launch_grouped_linear_bwd(const void* x, const void* w, const void* dy, void* dx, void* dw, const int32_t* offsets, int G,
                                     int64_t total, int K, int N, bool fill_rest, int dtype, void* workspace, hipStream_t stream) {
    if (dtype == KUNLUN_FP32) {
        if (dx && total > 0) rows<float, false>(dy, w, dx, offsets, G, total, N, K, fill_rest, stream);
        if (dw) weights<float>(x, dy, dw, offsets, G, total, K, N, dtype, workspace, stream);
    } else {
        if (dx && total > 0) rows<bf16_t, false>(dy, w, dx, offsets, G, total, N, K, fill_rest, stream);
        if (dw) weights<bf16_t>(x, dy, dw, offsets, G, total, K, N, dtype, workspace, stream);
    }
    return hipGetLastError();
}

}  // namespace kunlun
