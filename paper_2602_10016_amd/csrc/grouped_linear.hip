// Linear maps per group of consecutive rows:  y[r] = x[r] w[g];  dx[r] = dy[r] w[g]^T;  dw[g] = x_g^T dy_g  (r in group g).
// Groups have any sizes, so the work is cut into output tiles and a workgroup finds its tile from the offsets: tiles of rows are
// counted per group (a launch has room for the tiles of any division of the rows, those left over end at once).
#include "layers.h"

namespace kunlun {

namespace {

// Tile t of the tiles of `height` rows of all groups: its group, first row and number of rows (0: there is no such tile).  The rows
// behind the last group count as group G.  Called by whole waves.
struct RowTile {
    int group, rows;
    int64_t row0;
};
__device__ __forceinline__ RowTile find_row_tile(const int32_t* offsets, int G, int64_t total, int height, int64_t t) {
    const int lane = threadIdx.x & 63;
    RowTile r = {0, 0, 0};
    for (int g0 = 0; g0 <= G; g0 += 64) {
        const int g = g0 + lane < G ? g0 + lane : G;
        int64_t lo = offsets[g], hi = g < G ? offsets[g + 1] : total;
        if (hi > total) hi = total;
        if (lo < 0) lo = 0;
        const int len = g0 + lane <= G && hi > lo ? (int)(hi - lo) : 0;
        const int tiles = (len + height - 1) / height;
        int upto = tiles;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int v = __shfl_up(upto, o);
            if (lane >= o) upto += v;
        }
        const uint64_t beyond = __builtin_amdgcn_ballot_w64(upto > t);
        if (beyond) {
            const int at = __ffsll((unsigned long long)beyond) - 1;
            const int k = (int)(t - (__shfl(upto, at) - __shfl(tiles, at)));
            r.group = g0 + at;
            r.row0 = __shfl((int)lo, at) + (int64_t)k * height;
            const int left = __shfl(len, at) - k * height;
            r.rows = left < height ? left : height;
            return r;
        }
        t -= __shfl(upto, 63);
    }
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
    const RowTile t = find_row_tile(offsets, G, total, TILE, blockIdx.x / n_tiles);
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
    else launch_rows<bf16_t, false>(x, w, y, offsets, G, total, K, N, fill_rest, stream);
    return hipGetLastError();
}

size_t grouped_linear_bwd_workspace(int G, int64_t total, int K, int N, int dtype) { return 256; }

hipError_t launch_grouped_linear_bwd(const void* x, const void* w, const void* dy, void* dx, void* dw, const int32_t* offsets, int G,
                                     int64_t total, int K, int N, bool fill_rest, int dtype, void* workspace, hipStream_t stream) {
    if (dtype == KUNLUN_FP32) {
        if (dx && total > 0) launch_rows<float, true>(dy, w, dx, offsets, G, total, N, K, fill_rest, stream);
        if (dw) launch_weights<float>(x, dy, dw, offsets, G, total, K, N, stream);
    } else {
        if (dx && total > 0) launch_rows<bf16_t, true>(dy, w, dx, offsets, G, total, N, K, fill_rest, stream);
        if (dw) launch_weights<bf16_t>(x, dy, dw, offsets, G, total, K, N, stream);
    }
    return hipGetLastError();
}

}  // namespace kunlun
