// Embedding lookup and the gradient of its table.
//     out[r] = scale * table[ids[r]],     d_table[v] = scale * sum of d_out[r] over the r with ids[r] = v
// Both move rows and compute next to nothing: bound by memory.  A row is held by the lanes of a group (a power of two of them,
// one 16-byte piece each), so that narrow rows share a wave and every access is as wide as the row allows.
//
// The gradient sorts (id, position) pairs with a stable radix sort, then lane groups walk fixed ranges of the sorted pairs and
// add the rows of equal ids in registers: no float atomics, so equal calls give equal bits, and a row of d_out is read once
// wherever it lies.  A run of equal ids inside one range is written to its table row at once; a run that crosses ranges leaves
// one fp32 partial sum per range, which a second kernel adds in order (an id may be in a large part of the rows).  Table rows
// that no id names are found by searching the sorted ids and set to zero in the same launch, so every table row is
// written exactly once.
#include "layers.h"

namespace kunlun {

namespace {

constexpr int THREADS = 256;
constexpr int FETCH = 4;  // rows in flight per lane group of the lookup
constexpr int64_t GRID_MOST = 1 << 14;  // workgroups; each loops beyond that

template <typename ID>
__device__ __forceinline__ bool in_table(ID id, int64_t rows) {
    return (uint64_t)(int64_t)id < (uint64_t)rows;
}

template <typename T, int W, typename ID>
__global__ __launch_bounds__(THREADS) void embedding_fwd_kernel(const T* __restrict__ table, const ID* __restrict__ ids, T* __restrict__ out,
                                                                int64_t n, int64_t rows, int D, float scale, int lanes) {
    const int pieces = (D + W - 1) / W, lane = threadIdx.x % lanes;
    const int64_t groups = (int64_t)gridDim.x * (THREADS / lanes);
    for (int64_t r0 = ((int64_t)blockIdx.x * (THREADS / lanes) + threadIdx.x / lanes) * FETCH; r0 < n; r0 += groups * FETCH) {
        bool ok[FETCH];
        const T* src[FETCH];
#pragma unroll
        for (int u = 0; u < FETCH; ++u) {
            const ID id = ids[r0 + u < n ? r0 + u : n - 1];
            ok[u] = in_table(id, rows);
            src[u] = table + (ok[u] ? (int64_t)id : 0) * D;
        }
        for (int c = lane; c < pieces; c += lanes) {
            const int at = piece_start(c, D, W);
            Piece<T, W> x[FETCH];
#pragma unroll
            for (int u = 0; u < FETCH; ++u)
                if (rows > 0) x[u] = load_piece_kept<T, W>(src[u] + at);
#pragma unroll
            for (int u = 0; u < FETCH; ++u) {
                if (r0 + u >= n) break;
                Piece<T, W> y;
#pragma unroll
                for (int j = 0; j < W; ++j) y.v[j] = from_float<T>(ok[u] ? to_float(x[u].v[j]) * scale : 0.f);
                store_piece<T, W>(out + (r0 + u) * D + at, y);
            }
        }
    }
}

// ---- sorting ----

constexpr int SORT_THREADS = 512, SORT_WAVES = SORT_THREADS / 64;
constexpr int DIGIT_MOST = 10;  // bits of a digit: two passes up to a million table rows
constexpr int BINS_MOST = 1 << DIGIT_MOST;
constexpr int SORT_BLOCKS = 128;  // most ranges of one pass: every range reads the counts of all

// Where a pass reads: the ids themselves (first pass) or the pairs of the pass before.  An id outside the table sorts as
// `rows`, behind every id of the table.
template <typename ID>
__device__ __forceinline__ uint32_t key_at(const ID* ids, const uint32_t* keys, int64_t i, uint32_t rows) {
    if (keys) return keys[i];
    const ID id = ids[i];
    return in_table(id, rows) ? (uint32_t)id : rows;
}

template <typename ID>
__global__ __launch_bounds__(SORT_THREADS) void digit_count_kernel(const ID* __restrict__ ids, const uint32_t* __restrict__ keys,
                                                                   uint32_t* __restrict__ counts, int64_t n, int64_t per_block, uint32_t rows,
                                                                   int shift, int bits) {
    __shared__ uint32_t count[BINS_MOST];
    const int bins = 1 << bits;
    for (int d = threadIdx.x; d < bins; d += SORT_THREADS) count[d] = 0;
    __syncthreads();
    const int64_t begin = blockIdx.x * per_block, end = begin + per_block < n ? begin + per_block : n;
    for (int64_t i = begin + threadIdx.x; i < end; i += SORT_THREADS) atomicAdd(&count[(key_at(ids, keys, i, rows) >> shift) & (bins - 1)], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < bins; d += SORT_THREADS) counts[(int64_t)blockIdx.x * bins + d] = count[d];
}

// Stable: ranges in order, waves in order inside a range, 64 pairs at a time inside a wave, lanes in order.
template <typename ID>
__global__ __launch_bounds__(SORT_THREADS) void digit_scatter_kernel(const ID* __restrict__ ids, const uint32_t* __restrict__ keys,
                                                                     const uint32_t* __restrict__ positions, const uint32_t* __restrict__ counts,
                                                                     uint32_t* __restrict__ keys_out, uint32_t* __restrict__ positions_out, int64_t n,
                                                                     int64_t per_block, uint32_t rows, int shift, int bits) {
    __shared__ uint32_t next[SORT_WAVES][BINS_MOST];  // where a wave's next pair of a digit goes
    __shared__ uint32_t wave_sums[SORT_WAVES];
    const int bins = 1 << bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t begin = blockIdx.x * per_block, end = begin + per_block < n ? begin + per_block : n;
    const int64_t per_wave = per_block / SORT_WAVES;  // (a multiple of 64)
    const int64_t w0 = begin + wave * per_wave, w1 = w0 + per_wave < end ? w0 + per_wave : end;
    for (int d = lane; d < bins; d += 64) next[wave][d] = 0;
    __syncthreads();
    for (int64_t i = w0 + lane; i < w1; i += 64) atomicAdd(&next[wave][(key_at(ids, keys, i, rows) >> shift) & (bins - 1)], 1u);
    // pairs of smaller digits in all ranges, and of this digit in the ranges before
    uint32_t carry = 0;
    for (int d0 = 0; d0 < bins; d0 += SORT_THREADS) {
        const int d = d0 + threadIdx.x;
        uint32_t all = 0, before = 0;
        if (d < bins)
            for (int b = 0; b < (int)gridDim.x; ++b) {
                const uint32_t c = counts[(int64_t)b * bins + d];
                all += c;
                before += b < (int)blockIdx.x ? c : 0;
            }
        uint32_t upto = all;  // inclusive sum over the lanes, then over the waves
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const uint32_t v = __shfl_up(upto, o);
            if (lane >= o) upto += v;
        }
        __syncthreads();  // the sums of the chunk before are read; the waves' counts are complete
        if (lane == 63) wave_sums[wave] = upto;
        __syncthreads();
        uint32_t base = carry + upto - all + before, total = 0;
        for (int w = 0; w < SORT_WAVES; ++w) {
            if (w < wave) base += wave_sums[w];
            total += wave_sums[w];
        }
        carry += total;
        if (d < bins)
            for (int w = 0; w < SORT_WAVES; ++w) {
                const uint32_t c = next[w][d];
                next[w][d] = base;
                base += c;
            }
    }
    __syncthreads();
    for (int64_t i0 = w0; i0 < w1; i0 += 64) {
        const int64_t i = i0 + lane;
        const bool ok = i < w1;
        const uint32_t key = ok ? key_at(ids, keys, i, rows) : 0;
        const uint32_t d = (key >> shift) & (bins - 1);
        uint64_t same = __builtin_amdgcn_ballot_w64(ok);  // lanes of this digit
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __builtin_amdgcn_ballot_w64((d >> b) & 1);
            same &= (d >> b) & 1 ? set : ~set;
        }
        const int first = ok ? __ffsll((unsigned long long)same) - 1 : lane;
        uint32_t to = 0;
        if (ok && lane == first) to = atomicAdd(&next[wave][d], (uint32_t)__popcll(same));
        to = __shfl(to, first) + __popcll(same & (((uint64_t)1 << lane) - 1));
        if (ok) {
            keys_out[to] = key;
            positions_out[to] = positions ? positions[i] : (uint32_t)i;
        }
    }
}

// ---- sums of the rows of equal ids ----

constexpr int ADD_FETCH = 8;  // rows in flight per lane group
constexpr int ZERO_ROWS = 64; // table rows that a workgroup searches for

__device__ __forceinline__ int64_t first_at_least(const uint32_t* keys, int64_t lo, int64_t hi, uint32_t key) {
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (keys[mid] < key) lo = mid + 1; else hi = mid;
    }
    return lo;
}

// Lane group g of the first `add_blocks` workgroups walks the sorted pairs g * chunk .. + chunk; the workgroups behind them set the
// table rows without an id to zero.  blockIdx.y: the tile of up to 64 pieces of a row.
template <typename T, int W>
__global__ __launch_bounds__(THREADS) void embedding_add_kernel(const T* __restrict__ d_out, const uint32_t* __restrict__ keys,
                                                                const uint32_t* __restrict__ positions, T* __restrict__ d_table,
                                                                float* __restrict__ partial, int64_t n, uint32_t rows, int D, float scale, int lanes,
                                                                int64_t chunk, int64_t add_blocks) {
    const int pieces = (D + W - 1) / W;
    const int c = blockIdx.y * 64 + threadIdx.x % lanes;
    const bool has = c < pieces;
    const int at = piece_start(has ? c : pieces - 1, D, W);
    const int group = threadIdx.x / lanes, groups = THREADS / lanes;
    if (blockIdx.x >= add_blocks) {
        __shared__ int absent[ZERO_ROWS];
        Piece<T, W> zero;
#pragma unroll
        for (int j = 0; j < W; ++j) zero.v[j] = from_float<T>(0.f);
        for (int64_t v0 = (blockIdx.x - add_blocks) * ZERO_ROWS; v0 < rows; v0 += (gridDim.x - add_blocks) * ZERO_ROWS) {
            if (threadIdx.x < ZERO_ROWS) {
                const int64_t v = v0 + threadIdx.x;
                bool none = v < rows;
                if (none) {
                    const int64_t i = first_at_least(keys, 0, n, (uint32_t)v);
                    none = i == n || keys[i] != (uint32_t)v;
                }
                absent[threadIdx.x] = none;
            }
            __syncthreads();
            for (int k = group; k < ZERO_ROWS; k += groups)
                if (absent[k] && has) store_piece<T, W>(d_table + (v0 + k) * D + at, zero);
            __syncthreads();
        }
        return;
    }
    const int64_t walker = blockIdx.x * groups + group;
    const int64_t i0 = walker * chunk, i1 = i0 + chunk < n ? i0 + chunk : n;
    if (i0 >= n || !has) return;
    float acc[W];
#pragma unroll
    for (int j = 0; j < W; ++j) acc[j] = 0.f;
    uint32_t key = keys[i0];
    bool from_before = i0 > 0 && keys[i0 - 1] == key;
    auto finish = [&](bool goes_on) {
        if (key >= rows) return;
        if (!from_before && !goes_on) {
            Piece<T, W> y;
#pragma unroll
            for (int j = 0; j < W; ++j) y.v[j] = from_float<T>(acc[j] * scale);
            store_piece<T, W>(d_table + (int64_t)key * D + at, y);
        } else {  // slot 0: the run came from the range before; slot 1: it begins here
            float* p = partial + ((walker * 2 + (from_before ? 0 : 1)) * pieces + c) * W;
#pragma unroll
            for (int j = 0; j < W; ++j) p[j] = acc[j];
        }
    };
    for (int64_t i = i0; i < i1; i += ADD_FETCH) {
        uint32_t k[ADD_FETCH];
        Piece<T, W> x[ADD_FETCH];
#pragma unroll
        for (int u = 0; u < ADD_FETCH; ++u) {
            const int64_t e = i + u < i1 ? i + u : i1 - 1;
            k[u] = keys[e];
            x[u] = load_piece<T, W>(d_out + (int64_t)positions[e] * D + at);
        }
#pragma unroll
        for (int u = 0; u < ADD_FETCH; ++u) {
            if (i + u >= i1) break;
            if (k[u] != key) {
                finish(false);
                key = k[u];
                from_before = false;
#pragma unroll
                for (int j = 0; j < W; ++j) acc[j] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < W; ++j) acc[j] += to_float(x[u].v[j]);
        }
    }
    finish(i1 < n && keys[i1] == key);
}

// Runs that cross ranges: the lane group of the range where one begins adds its partial sums in order.
template <typename T, int W>
__global__ __launch_bounds__(THREADS) void embedding_join_kernel(const uint32_t* __restrict__ keys, const float* __restrict__ partial,
                                                                 T* __restrict__ d_table, int64_t n, uint32_t rows, int D, float scale, int lanes,
                                                                 int64_t chunk) {
    const int pieces = (D + W - 1) / W;
    const int c = blockIdx.y * 64 + threadIdx.x % lanes;
    const int64_t walker = (int64_t)blockIdx.x * (THREADS / lanes) + threadIdx.x / lanes;
    const int64_t i0 = walker * chunk, i1 = i0 + chunk;
    if (i1 >= n || c >= pieces) return;
    const uint32_t key = keys[i1 - 1];
    if (key >= rows || keys[i1] != key || (i0 > 0 && keys[i0 - 1] == key)) return;
    const int64_t last = (first_at_least(keys, i1, n, key + 1) - 1) / chunk;  // the range that holds the run's last pair
    float acc[W];
    const float* p = partial + ((walker * 2 + 1) * pieces + c) * W;
#pragma unroll
    for (int j = 0; j < W; ++j) acc[j] = p[j];
    for (int64_t r = walker + 1; r <= last; ++r) {
        p = partial + ((r * 2) * pieces + c) * W;
#pragma unroll
        for (int j = 0; j < W; ++j) acc[j] += p[j];
    }
    Piece<T, W> y;
#pragma unroll
    for (int j = 0; j < W; ++j) y.v[j] = from_float<T>(acc[j] * scale);
    store_piece<T, W>(d_table + (int64_t)key * D + piece_start(c, D, W), y);
}

template <typename T>
int piece_width(int D) { return D * sizeof(T) >= 16 ? 16 / (int)sizeof(T) : 1; }

template <typename T, int W, typename ID>
void embedding_fwd(const void* table, const void* ids, void* out, int64_t n, int64_t rows, int D, float scale, hipStream_t stream) {
    const int lanes = lanes_per_row(pieces_per_row(D, W));
    const int64_t per_block = (int64_t)(THREADS / lanes) * FETCH;
    const int64_t blocks = (n + per_block - 1) / per_block;
    hipLaunchKernelGGL((embedding_fwd_kernel<T, W, ID>), dim3((unsigned)(blocks < GRID_MOST ? blocks : GRID_MOST)), dim3(THREADS), 0, stream,
                       (const T*)table, (const ID*)ids, (T*)out, n, rows, D, scale, lanes);
}
template <typename T, int W>
void embedding_fwd(const void* table, const void* ids, void* out, int64_t n, int64_t rows, int D, float scale, int id_bytes, hipStream_t stream) {
    if (id_bytes == 8) embedding_fwd<T, W, int64_t>(table, ids, out, n, rows, D, scale, stream);
    else embedding_fwd<T, W, int32_t>(table, ids, out, n, rows, D, scale, stream);
}

// Pairs per lane group: ranges enough to fill the device (about 16 waves per compute unit of them), long ones otherwise, so that
// few runs cross a range and leave partial sums.
constexpr int64_t CHUNK_LEAST = 8, RANGES_MOST = 16384;
int64_t add_chunk(int64_t n) {
    int64_t chunk = CHUNK_LEAST;
    while ((n + chunk - 1) / chunk > RANGES_MOST) chunk *= 2;
    return chunk;
}
int64_t ranges_at_most(int64_t n) {
    const int64_t r = (n + CHUNK_LEAST - 1) / CHUNK_LEAST;
    return r < RANGES_MOST ? r : RANGES_MOST;
}

struct SortSpace {
    uint32_t *keys[2], *positions[2], *counts;
    float* partial;
    size_t bytes;
    SortSpace(char* base, int64_t n, int D, int dtype) {
        const size_t pairs = align_up((size_t)n * 4, 256);
        size_t at = 0;
        auto take = [&](size_t b) { char* p = base + at; at += b; return p; };
        for (int i = 0; i < 2; ++i) {
            keys[i] = (uint32_t*)take(pairs);
            positions[i] = (uint32_t*)take(pairs);
        }
        counts = (uint32_t*)take((size_t)SORT_BLOCKS * BINS_MOST * 4);
        const int W = dtype == KUNLUN_FP32 ? piece_width<float>(D) : piece_width<bf16_t>(D);
        partial = (float*)take(align_up((size_t)ranges_at_most(n) * 2 * pieces_per_row(D, W) * W * 4, 256));
        bytes = at;
    }
};

template <typename ID>
int sort_ids(const void* ids, const SortSpace& s, int64_t n, int64_t rows, hipStream_t stream) {
    int bits = 1;
    while (rows >> bits) ++bits;  // keys are 0 .. rows
    const int passes = (bits + DIGIT_MOST - 1) / DIGIT_MOST, digit = (bits + passes - 1) / passes;
    constexpr int64_t STEP = SORT_WAVES * 64;
    int64_t per_block = (n + SORT_BLOCKS - 1) / SORT_BLOCKS;
    per_block = (per_block + STEP - 1) / STEP * STEP;
    const unsigned blocks = (unsigned)((n + per_block - 1) / per_block);
    for (int p = 0; p < passes; ++p) {
        const uint32_t* keys = p ? s.keys[(p + 1) & 1] : nullptr;
        const uint32_t* positions = p ? s.positions[(p + 1) & 1] : nullptr;
        hipLaunchKernelGGL(digit_count_kernel<ID>, dim3(blocks), dim3(SORT_THREADS), 0, stream, (const ID*)ids, keys, s.counts, n, per_block,
                           (uint32_t)rows, p * digit, digit);
        hipLaunchKernelGGL(digit_scatter_kernel<ID>, dim3(blocks), dim3(SORT_THREADS), 0, stream, (const ID*)ids, keys, positions, s.counts,
                           s.keys[p & 1], s.positions[p & 1], n, per_block, (uint32_t)rows, p * digit, digit);
    }
    return (passes - 1) & 1;
}

template <typename T, int W>
void embedding_bwd(const void* d_out, const SortSpace& s, int sorted, void* d_table, int64_t n, int64_t rows, int D, float scale, hipStream_t stream) {
    const int pieces = pieces_per_row(D, W), lanes = lanes_per_row(pieces), groups = THREADS / lanes;
    const int64_t chunk = add_chunk(n), ranges = (n + chunk - 1) / chunk;
    const int64_t add_blocks = (ranges + groups - 1) / groups, zero_all = (rows + ZERO_ROWS - 1) / ZERO_ROWS;
    const int64_t zero_blocks = zero_all < GRID_MOST ? zero_all : GRID_MOST;
    const unsigned tiles = (unsigned)((pieces + 63) / 64);
    hipLaunchKernelGGL((embedding_add_kernel<T, W>), dim3((unsigned)(add_blocks + zero_blocks), tiles), dim3(THREADS), 0, stream, (const T*)d_out,
                       s.keys[sorted], s.positions[sorted], (T*)d_table, s.partial, n, (uint32_t)rows, D, scale, lanes, chunk, add_blocks);
    if (ranges > 1)
        hipLaunchKernelGGL((embedding_join_kernel<T, W>), dim3((unsigned)add_blocks, tiles), dim3(THREADS), 0, stream, s.keys[sorted], s.partial,
                           (T*)d_table, n, (uint32_t)rows, D, scale, lanes, chunk);
}

}  // namespace

hipError_t launch_embedding_fwd(const void* table, const void* ids, void* out, int64_t n, int64_t rows, int D, float scale, int id_bytes,
                                int dtype, hipStream_t stream) {
    if (dtype == KUNLUN_FP32) {
        if (piece_width<float>(D) == 4) embedding_fwd<float, 4>(table, ids, out, n, rows, D, scale, id_bytes, stream);
        else embedding_fwd<float, 1>(table, ids, out, n, rows, D, scale, id_bytes, stream);
    } else {
        if (piece_width<bf16_t>(D) == 8) embedding_fwd<bf16_t, 8>(table, ids, out, n, rows, D, scale, id_bytes, stream);
        else embedding_fwd<bf16_t, 1>(table, ids, out, n, rows, D, scale, id_bytes, stream);
    }
    return hipGetLastError();
}

size_t embedding_bwd_workspace(int64_t n, int D, int dtype) { return SortSpace(nullptr, n, D, dtype).bytes; }

hipError_t launch_embedding_bwd(const void* d_out, const void* ids, void* d_table, int64_t n, int64_t rows, int D, float scale,
                                int id_bytes, int dtype, void* workspace, hipStream_t stream) {
    const SortSpace s((char*)workspace, n, D, dtype);
    int sorted = 0;
    if (n > 0) sorted = id_bytes == 8 ? sort_ids<int64_t>(ids, s, n, rows, stream) : sort_ids<int32_t>(ids, s, n, rows, stream);
    if (dtype == KUNLUN_FP32) {
        if (piece_width<float>(D) == 4) embedding_bwd<float, 4>(d_out, s, sorted, d_table, n, rows, D, scale, stream);
        else embedding_bwd<float, 1>(d_out, s, sorted, d_table, n, rows, D, scale, stream);
    } else {
        if (piece_width<bf16_t>(D) == 8) embedding_bwd<bf16_t, 8>(d_out, s, sorted, d_table, n, rows, D, scale, stream);
        else embedding_bwd<bf16_t, 1>(d_out, s, sorted, d_table, n, rows, D, scale, stream);
    }
    return hipGetLastError();
}

}  // namespace kunlun
