// Linear maps per group of consecutive rows:  y[r] = x[r] w[g];  dx[r] = dy[r] w[g]^T;  dw[g] = x_g^T dy_g  (r in group g).
// Groups have any sizes, so the work is cut into output tiles and a workgroup finds its tile from the offsets: tiles of rows are
// counted per group (a launch has room for the tiles of any division of the rows, those left over end at once).
// bf16: matrix cores (grouped_tile.h); fp32: plain fp32 arithmetic.
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
            const int n = __shfl(tiles, at), k = (int)(t - (__shfl(upto, at) - n));
            r.group = g0 + at;
            r.row0 = __shfl((int)lo, at) + (int64_t)k * height;
            const int left = (int)(__shfl(len, at) - (int64_t)k * height);
            r.rows = left < height ? left : height;
            if (SLOTS && n > 1) r.slot = slots + __shfl(shared, at) - n + k;
            break;
        }
        t -= __shfl(upto, 63);
        if (SLOTS) slots += __shfl(shared, 63);
    }
    r.group = __builtin_amdgcn_readfirstlane(r.group);
    r.rows = __builtin_amdgcn_readfirstlane(r.rows);
    r.slot = __builtin_amdgcn_readfirstlane(r.slot);
    r.row0 = __builtin_amdgcn_readfirstlane((int)r.row0);
    return r;
}
// Row tiles that a launch has room for: every group, and the rows behind them, may end inside a tile.
int64_t row_tiles(int G, int64_t total, int height) { return (total + height - 1) / height + G + 1; }

constexpr int TILE = 64, STEP = 16;

// C [m, n] = sum over k of A(m, k) B(k, n): 64 x 64 outputs, 4 x 4 per thread, fp32 sums.
template <typename A, typename B>
__device__ __forceinline__ void tile_product(float (&acc)[4][4], A a, B b, int K) {
    __shared__ float sa[STEP][TILE + 4], sb[STEP][TILE + 4];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int k0 = 0; k0 < K; k0 += STEP) {
        __syncthreads();
        for (int i = threadIdx.x; i < STEP * TILE; i += 256) {
            sa[i / TILE][i % TILE] = k0 + i / TILE < K ? a(i % TILE, k0 + i / TILE) : 0.f;
            sb[i / TILE][i % TILE] = k0 + i / TILE < K ? b(k0 + i / TILE, i % TILE) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < STEP; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[k][4 * ty + i], sb[k][4 * tx + j], acc[i][j]);
    }
}

// out[r, n] = sum over k of in[r, k] w[g][k, n], or (TRANSPOSED) of in[r, k] w[g][n, k]
template <typename T, bool TRANSPOSED>
__global__ __launch_bounds__(256) void grouped_rows_kernel(const T* __restrict__ in, const T* __restrict__ w, T* __restrict__ out,
                                                           const int32_t* __restrict__ offsets, int G, int64_t total, int K, int N, bool fill_rest) {
    const int n_tiles = (N + TILE - 1) / TILE;
    const RowTile t = find_row_tile<false>(offsets, G, total, TILE, blockIdx.x / n_tiles);
    if (t.rows == 0 || (t.group == G && !fill_rest)) return;
    const int n0 = (int)(blockIdx.x % n_tiles) * TILE;
    const T* wg = w + (int64_t)t.group * K * N;
    float acc[4][4] = {};
    if (t.group < G) tile_product(acc, [&](int m, int k) { return m < t.rows ? to_float(in[(t.row0 + m) * K + k]) : 0.f; },
                 [&](int k, int n) { return n0 + n < N ? to_float(TRANSPOSED ? wg[(int64_t)(n0 + n) * K + k] : wg[(int64_t)k * N + n0 + n]) : 0.f; }, K);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j)
            if (4 * ty + i < t.rows && n0 + 4 * tx + j < N) out[(t.row0 + 4 * ty + i) * N + n0 + 4 * tx + j] = from_float<T>(acc[i][j]);
}

// dw[g][k, n] = sum over the rows r of group g of x[r, k] dy[r, n]
template <typename T>
__global__ __launch_bounds__(256) void grouped_weights_kernel(const T* __restrict__ x, const T* __restrict__ dy, T* __restrict__ dw,
                                                              const int32_t* __restrict__ offsets, int64_t total, int K, int N) {
    const int n_tiles = (N + TILE - 1) / TILE, k_tiles = (K + TILE - 1) / TILE;
    const int g = blockIdx.x / (n_tiles * k_tiles), in_group = blockIdx.x % (n_tiles * k_tiles);
    const int k0 = in_group / n_tiles * TILE, n0 = in_group % n_tiles * TILE;
    int64_t lo = offsets[g], hi = offsets[g + 1];
    if (hi > total) hi = total;
    if (lo < 0) lo = 0;
    float acc[4][4] = {};
    tile_product(acc, [&](int m, int r) { return k0 + m < K ? to_float(x[(lo + r) * K + k0 + m]) : 0.f; },
                 [&](int r, int n) { return n0 + n < N ? to_float(dy[(lo + r) * N + n0 + n]) : 0.f; }, hi > lo ? (int)(hi - lo) : 0);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j)
            if (k0 + 4 * ty + i < K && n0 + 4 * tx + j < N) dw[((int64_t)g * K + k0 + 4 * ty + i) * N + n0 + 4 * tx + j] = from_float<T>(acc[i][j]);
}

// ---- matrix cores ----

// Output tiles in blocks of up to SUPER_M x SUPER_N, a block on one XCD (workgroup i runs on XCD i % 8) at a time: its workgroups share rows of
// one operand and columns of the other in that XCD's L2.  Blocks go round the XCDs, so that tiles left over at the end cost all the same.
struct TileOrder {
    int64_t m_tiles;
    int n_tiles, super_m, super_n;
};
__host__ __device__ inline int64_t super_blocks(const TileOrder& o) {
    return (o.m_tiles + o.super_m - 1) / o.super_m * ((o.n_tiles + o.super_n - 1) / o.super_n);
}
__device__ __forceinline__ bool tile_of(const TileOrder& o, int64_t& mt, int& nt) {
    const int64_t id = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, j = id >> 3;
    const int size = o.super_m * o.super_n, in = (int)(j % size), across = (o.n_tiles + o.super_n - 1) / o.super_n;
    const int64_t block = j / size * 8 + (id & 7);
    mt = block / across * o.super_m + in % o.super_m;
    nt = (int)(block % across) * o.super_n + in / o.super_m;
    return mt < o.m_tiles && nt < o.n_tiles;
}
// (two dimensions: one holds at most 2^32 threads)
dim3 tile_grid(const TileOrder& o, int threads) {
    const int64_t all = (super_blocks(o) + 7) / 8 * 8 * o.super_m * o.super_n, most = largest_grid(threads) / 8 * 8;
    return all <= most ? dim3((unsigned)all) : dim3((unsigned)most, (unsigned)((all + most - 1) / most));
}

// out[r, :] = in[r, :] W  (B_COLUMNS: W = w[g] [K, N];  else W = w[g]^T of w[g] [N, K])
template <typename S, bool B_COLUMNS>
__global__ __launch_bounds__(S::THREADS) void grouped_rows_mfma_kernel(const bf16_t* __restrict__ in, const bf16_t* __restrict__ w,
                                                                       bf16_t* __restrict__ out, const int32_t* __restrict__ offsets, int G,
                                                                       int64_t total, int K, int N, bool fill_rest, TileOrder order) {
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int64_t mt;
    int nt;
    if (!tile_of(order, mt, nt)) return;
    const RowTile t = find_row_tile<false>(offsets, G, total, S::BM, mt);
    if (t.rows == 0 || (t.group == G && !fill_rest)) return;
    const int n0 = nt * S::BN;
    f32x16 acc[S::NB][S::MB] = {};
    if (t.group < G) {
        const bf16_t* wg = w + (int64_t)t.group * K * N;
        const GroupedOperand a = {(const char*)(in + t.row0 * K), (uint32_t)K * 2, t.rows};
        const GroupedOperand b = {(const char*)(B_COLUMNS ? wg + n0 : wg + (int64_t)n0 * K), (uint32_t)(B_COLUMNS ? N : K) * 2, N - n0};
        grouped_product<S, false, B_COLUMNS>(acc, lds, a, b, K, lane, wave);
    }
    grouped_store<S, bf16_t>(acc, lds, out + t.row0 * N + n0, N, t.rows, N - n0, lane, wave);
}

// dw[g] = x^T dy over a range of `height` rows of group g, to dw where the group has no other range, else to the range's slot of `partial`.
template <typename S>
__global__ __launch_bounds__(S::THREADS) void grouped_weights_mfma_kernel(const bf16_t* __restrict__ x, const bf16_t* __restrict__ dy,
                                                                          bf16_t* __restrict__ dw, float* __restrict__ partial,
                                                                          const int32_t* __restrict__ offsets, int G, int64_t total, int K, int N,
                                                                          int height, TileOrder order) {
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int64_t mt;
    int nt;
    if (!tile_of(order, mt, nt)) return;
    const int k_tiles = (K + S::BM - 1) / S::BM;
    const RowTile t = find_row_tile<true>(offsets, G, total, height, mt / k_tiles);
    if (t.rows == 0 || t.group == G) return;
    const int k0 = (int)(mt % k_tiles) * S::BM, n0 = nt * S::BN;
    const GroupedOperand a = {(const char*)(x + t.row0 * K + k0), (uint32_t)K * 2, K - k0};
    const GroupedOperand b = {(const char*)(dy + t.row0 * N + n0), (uint32_t)N * 2, N - n0};
    f32x16 acc[S::NB][S::MB] = {};
    grouped_product<S, true, true>(acc, lds, a, b, t.rows, lane, wave);
    if (t.slot < 0)
        grouped_store<S, bf16_t>(acc, lds, dw + ((int64_t)t.group * K + k0) * N + n0, N, K - k0, N - n0, lane, wave);
    else
        grouped_store<S, float>(acc, lds, partial + ((int64_t)t.slot * K + k0) * N + n0, N, K - k0, N - n0, lane, wave);
}

// dw[g] where group g has not exactly one range: the sum of its slots in order, zeros without any.  Four values per thread.
__global__ __launch_bounds__(256) void grouped_join_kernel(const float* __restrict__ partial, bf16_t* __restrict__ dw,
                                                           const int32_t* __restrict__ offsets, int G, int64_t total, int64_t per_group, int height) {
    const int g = blockIdx.y;
    int64_t lo;
    int len, slot = 0;
    for (int g0 = 0; g0 < g; g0 += 64) {
        int n = tiles_of(offsets, G, total, height, g0 + (threadIdx.x & 63), lo, len);
        if (n <= 1 || g0 + (int)(threadIdx.x & 63) >= g) n = 0;
        slot += __shfl(wave_prefix(n), 63);
    }
    const int ranges = tiles_of(offsets, G, total, height, g, lo, len);
    if (ranges == 1) return;
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < per_group; i += (int64_t)gridDim.x * 1024) {
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        const float* p = partial + (int64_t)slot * per_group + i;
        for (int k = 0; k < ranges; ++k) sum += *(const f32x4*)(p + (int64_t)k * per_group);
        bf16x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (bf16_t)sum[e];
        *(bf16x4*)(dw + g * per_group + i) = o;
    }
}

using Large = GroupedShape<256, 256, 2, 4, 2>;   // one workgroup of eight waves per compute unit
using Middle = GroupedShape<128, 128, 2, 2, 2>;  // two of four waves
using Small = GroupedShape<64, 64, 2, 2, 4>;     // two of four waves, three steps in flight

template <typename S, bool B_COLUMNS>
void rows_mfma(const void* in, const void* w, void* out, const int32_t* offsets, int G, int64_t total, int K, int N, bool fill_rest,
               hipStream_t stream) {
    const int n_tiles = (N + S::BN - 1) / S::BN;
    const TileOrder order = {row_tiles(G, total, S::BM), n_tiles, 4, n_tiles < 8 ? n_tiles : 8};
    hipLaunchKernelGGL((grouped_rows_mfma_kernel<S, B_COLUMNS>), tile_grid(order, S::THREADS), dim3(S::THREADS), 0, stream, (const bf16_t*)in,
                       (const bf16_t*)w, (bf16_t*)out, offsets, G, total, K, N, fill_rest, order);
}
template <bool B_COLUMNS>
void rows_bf16(const void* in, const void* w, void* out, const int32_t* offsets, int G, int64_t total, int K, int N, bool fill_rest,
               hipStream_t stream) {
    if (total >= (int64_t)G * 256 && N > 128 && total / 256 * ((N + 255) / 256) >= compute_units())
        rows_mfma<Large, B_COLUMNS>(in, w, out, offsets, G, total, K, N, fill_rest, stream);
    else if (total >= (int64_t)G * 96)
        rows_mfma<Middle, B_COLUMNS>(in, w, out, offsets, G, total, K, N, fill_rest, stream);
    else
        rows_mfma<Small, B_COLUMNS>(in, w, out, offsets, G, total, K, N, fill_rest, stream);
}

// How the weights' gradient is cut: the tile shape, and the rows per range so that the device is filled about twice.
struct WeightsPlan {
    bool large;
    int height;
    int64_t slots;
};
WeightsPlan plan_weights(int64_t total, int K, int N) {
    WeightsPlan p;
    p.large = K > 128 && N > 128 && (int64_t)((K + 255) / 256) * ((N + 255) / 256) * (total / 512) >= compute_units();
    const int tile = p.large ? 256 : 128;
    const int64_t tiles = (int64_t)((K + tile - 1) / tile) * ((N + tile - 1) / tile), resident = (int64_t)compute_units() * (p.large ? 1 : 2);
    int64_t height = total * tiles / (2 * resident);
    height = (height + GL_STEP - 1) / GL_STEP * GL_STEP;
    p.height = (int)(height < 512 ? 512 : height > (1 << 30) ? 1 << 30 : height);
    p.slots = 2 * total / p.height;  // (a group with a slot has more than one range, so more rows than one)
    return p;
}
template <typename S>
void weights_mfma(const WeightsPlan& p, const void* x, const void* dy, void* dw, float* partial, const int32_t* offsets, int G, int64_t total, int K,
                  int N, hipStream_t stream) {
    const int n_tiles = (N + S::BN - 1) / S::BN, k_tiles = (K + S::BM - 1) / S::BM;
    const TileOrder order = {((total + p.height - 1) / p.height + G) * k_tiles, n_tiles, k_tiles < 4 ? k_tiles : 4, n_tiles < 8 ? n_tiles : 8};
    hipLaunchKernelGGL(grouped_weights_mfma_kernel<S>, tile_grid(order, S::THREADS), dim3(S::THREADS), 0, stream, (const bf16_t*)x, (const bf16_t*)dy,
                       (bf16_t*)dw, partial, offsets, G, total, K, N, p.height, order);
}
void weights_bf16(const void* x, const void* dy, void* dw, const int32_t* offsets, int G, int64_t total, int K, int N, void* workspace,
                  hipStream_t stream) {
    const WeightsPlan p = plan_weights(total, K, N);
    float* partial = (float*)workspace;
    if (total > 0) {
        if (p.large) weights_mfma<Large>(p, x, dy, dw, partial, offsets, G, total, K, N, stream);
        else weights_mfma<Middle>(p, x, dy, dw, partial, offsets, G, total, K, N, stream);
    }
    const int64_t per_group = (int64_t)K * N, blocks = (per_group + 1023) / 1024;
    hipLaunchKernelGGL(grouped_join_kernel, dim3((unsigned)(blocks < 1024 ? blocks : 1024), (unsigned)G), dim3(256), 0, stream, partial, (bf16_t*)dw,
                       offsets, G, total, per_group, p.height);
}

template <typename T, bool TRANSPOSED>
void launch_rows(const void* in, const void* w, void* out, const int32_t* offsets, int G, int64_t total, int K, int N, bool fill_rest, hipStream_t stream) {
    const int64_t blocks = row_tiles(G, total, TILE) * ((N + TILE - 1) / TILE);
    hipLaunchKernelGGL((grouped_rows_kernel<T, TRANSPOSED>), dim3((unsigned)blocks), dim3(256), 0, stream, (const T*)in, (const T*)w, (T*)out, offsets,
                       G, total, K, N, fill_rest);
}
template <typename T>
void launch_weights(const void* x, const void* dy, void* dw, const int32_t* offsets, int G, int64_t total, int K, int N, hipStream_t stream) {
    const int64_t blocks = (int64_t)G * ((N + TILE - 1) / TILE) * ((K + TILE - 1) / TILE);
    hipLaunchKernelGGL(grouped_weights_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, stream, (const T*)x, (const T*)dy, (T*)dw, offsets, total, K,
                       N);
}

}  // namespace

hipError_t launch_grouped_linear_fwd(const void* x, const void* w, void* y, const int32_t* offsets, int G, int64_t total, int K, int N,
                                     bool fill_rest, int dtype, hipStream_t stream) {
    if (dtype == KUNLUN_FP32) launch_rows<float, false>(x, w, y, offsets, G, total, K, N, fill_rest, stream);
    else rows_bf16<true>(x, w, y, offsets, G, total, K, N, fill_rest, stream);
    return hipGetLastError();
}

size_t grouped_linear_bwd_workspace(int G, int64_t total, int K, int N, int dtype) {
    const WeightsPlan p = plan_weights(total, K, N);
    return align_up(256 + (dtype == KUNLUN_FP32 ? 0 : (size_t)p.slots * K * N * sizeof(float)), 256);
}

hipError_t launch_grouped_linear_bwd(const void* x, const void* w, const void* dy, void* dx, void* dw, const int32_t* offsets, int G,
                                     int64_t total, int K, int N, bool fill_rest, int dtype, void* workspace, hipStream_t stream) {
    if (dtype == KUNLUN_FP32) {
        if (dx && total > 0) launch_rows<float, true>(dy, w, dx, offsets, G, total, N, K, fill_rest, stream);
        if (dw) launch_weights<float>(x, dy, dw, offsets, G, total, K, N, stream);
    } else {
        if (dx && total > 0) rows_bf16<false>(dy, w, dx, offsets, G, total, N, K, fill_rest, stream);
        if (dw) weights_bf16(x, dy, dw, offsets, G, total, K, N, workspace, stream);
    }
    return hipGetLastError();
}

}  // namespace kunlun
