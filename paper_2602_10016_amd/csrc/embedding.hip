// Embedding lookup and the gradient of its table.
//     out[r] = scale * table[ids[r]],     d_table[v] = scale * sum of d_out[r] over the r with ids[r] = v
// Both move rows and compute next to nothing: bound by memory.  A row is held by the lanes of a group (a power of two of them,
// one 16-byte piece each), so that narrow rows share a wave and every access is as wide as the row allows.
//
// The gradient sorts (id, position) pairs with a stable radix sort, then lane groups walk fixed ranges of the sorted pairs and
// add the rows of equal ids in registers: no float atomics, so equal calls give equal bits, and a row of d_out is read once
// wherever it lies.  A run of equal ids inside one range is written to its table row at once; a run that crosses ranges leaves
// one fp32 partial sum per range (or one for all ranges of a workgroup that are inside it), which a second kernel adds in order: an id may
// be in a large part of the rows.  Small tables are set
// to zero beside the sort; in larger ones the rows that no id names are found among the sorted ids, so that they are written once.
// Measured (bf16; a copy reaches 5.07 TB/s here): lookup of 139 264 rows of 256 21 us (5.6 TB/s, repeated rows come from the caches);
// gradient of 1 144 603 rows of 1024 into a million 934 us (4.7 TB/s), of which the sums are 870, sorting 60 in six launches and joining 22;
// of 139 264 rows of 256 into 200 000 75 us: sorting 42 in four launches that leave most compute units idle, sums 23, joining 9.
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
//
// A stable radix sort of (key, position) pairs, 8 bytes each.  A pass counts the digits of every range of pairs, scans the counts over the
// ranges, and moves the pairs: a workgroup takes SORT_TILE pairs at a time, ranks them (lanes of a wave by ballots over the digit's bits, waves in
// order), puts them in order in LDS and writes runs of equal digits, which a scattered store per pair would turn into a memory transaction
// each.  Up to SORT_TILE pairs one workgroup makes all passes in LDS in one launch.

constexpr int SORT_THREADS = 512, SORT_WAVES = SORT_THREADS / 64, SORT_KEYS = 8;  // pairs per lane and tile
constexpr int SORT_TILE = SORT_THREADS * SORT_KEYS;
constexpr int DIGIT_MOST = 10;  // bits of a digit: two passes up to a million table rows
constexpr int BINS_MOST = 1 << DIGIT_MOST;
constexpr int64_t SORT_RANGES = 512;  // most ranges of a pass
constexpr int64_t FILL_BLOCKS = 192;
constexpr unsigned SCAN_RANGES = 64;  // from more on a launch of its own scans the counts

// The workgroups of a sorting launch behind its first `ranges` ones set a part of the table's gradient to zero meanwhile.
struct Fill {
    char* base;
    int64_t begin, end;  // bytes, multiples of 16 but for the end of the last part
};
__device__ __forceinline__ void fill_zero(const Fill& f, int block, int blocks) {
    const u32x4_any zero = {0, 0, 0, 0};
    for (int64_t i = f.begin + ((int64_t)block * SORT_THREADS + threadIdx.x) * 16; i < f.end; i += (int64_t)blocks * SORT_THREADS * 16) {
        if (i + 16 <= f.end) __builtin_nontemporal_store(zero, (u32x4_any*)(f.base + i));
        else
            for (int64_t k = i; k < f.end; k += 2) *(uint16_t*)(f.base + k) = 0;
    }
}

// Where a pass reads: the ids themselves (first pass) or the pairs of the pass before.  An id outside the table sorts as
// `rows`, behind every id of the table.
template <typename ID>
__device__ __forceinline__ uint2 pair_at(const ID* ids, const uint2* pairs, int64_t i, uint32_t rows) {
    if (pairs) return pairs[i];
    const ID id = ids[i];
    return make_uint2(in_table(id, rows) ? (uint32_t)id : rows, (uint32_t)i);
}

template <typename ID>
__global__ __launch_bounds__(SORT_THREADS) void digit_count_kernel(const ID* __restrict__ ids, const uint2* __restrict__ pairs,
                                                                   uint32_t* __restrict__ counts, int64_t n, int64_t per_range, int ranges,
                                                                   uint32_t rows, int shift, int bits, Fill fill) {
    if ((int)blockIdx.x >= ranges) return fill_zero(fill, blockIdx.x - ranges, gridDim.x - ranges);
    __shared__ uint32_t count[BINS_MOST];
    const int bins = 1 << bits;
    for (int d = threadIdx.x; d < bins; d += SORT_THREADS) count[d] = 0;
    __syncthreads();
    const int64_t begin = blockIdx.x * per_range, end = begin + per_range < n ? begin + per_range : n;
    for (int64_t i0 = begin + threadIdx.x; i0 < end; i0 += SORT_TILE) {
        uint32_t k[SORT_KEYS];
#pragma unroll
        for (int u = 0; u < SORT_KEYS; ++u) k[u] = pair_at(ids, pairs, i0 + u * SORT_THREADS < end ? i0 + u * SORT_THREADS : i0, rows).x;
#pragma unroll
        for (int u = 0; u < SORT_KEYS; ++u)
            if (i0 + u * SORT_THREADS < end) atomicAdd(&count[(k[u] >> shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < bins; d += SORT_THREADS) counts[(int64_t)blockIdx.x * bins + d] = count[d];
}

// counts[range][digit] -> the sum over the ranges before; totals[digit].  32 digits x 32 parts of the ranges per workgroup.
constexpr int SCAN_PARTS = 32, SCAN_FETCH = 16;  // loads in flight
__global__ __launch_bounds__(32 * SCAN_PARTS) void digit_scan_kernel(uint32_t* __restrict__ counts, uint32_t* __restrict__ totals, int ranges,
                                                                     int bins) {
    __shared__ uint32_t sums[SCAN_PARTS][32];
    const int col = threadIdx.x & 31, part = threadIdx.x >> 5, mine = blockIdx.x * 32 + col, d = mine < bins ? mine : 0;
    const bool has = mine < bins;
    const int per = (ranges + SCAN_PARTS - 1) / SCAN_PARTS, r0 = part * per, r1 = r0 + per < ranges ? r0 + per : ranges;
    uint32_t sum = 0;
    for (int r = r0; r < r1; r += SCAN_FETCH) {
        uint32_t c[SCAN_FETCH];
#pragma unroll
        for (int u = 0; u < SCAN_FETCH; ++u) c[u] = counts[(int64_t)(r + u < r1 ? r + u : r) * bins + d];
#pragma unroll
        for (int u = 0; u < SCAN_FETCH; ++u) sum += r + u < r1 ? c[u] : 0;
    }
    sums[part][col] = sum;
    __syncthreads();
    uint32_t before = 0;
    for (int q = 0; q < part; ++q) before += sums[q][col];
    if (part == SCAN_PARTS - 1 && has) totals[d] = before + sum;
    for (int r = r0; r < r1; r += SCAN_FETCH) {
        uint32_t c[SCAN_FETCH];
#pragma unroll
        for (int u = 0; u < SCAN_FETCH; ++u) c[u] = counts[(int64_t)(r + u < r1 ? r + u : r) * bins + d];
#pragma unroll
        for (int u = 0; u < SCAN_FETCH; ++u)
            if (r + u < r1 && has) {
                counts[(int64_t)(r + u) * bins + d] = before;
                before += c[u];
            }
    }
}

// Sums over the digits before, of a number per digit: x[v] of digit BINS_MOST / SORT_THREADS * threadIdx.x + v.
constexpr int DIGITS = BINS_MOST / SORT_THREADS;  // per thread
__device__ __forceinline__ void scan_digits(uint32_t (&x)[DIGITS], uint32_t* wave_sums) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t mine = 0;
#pragma unroll
    for (int v = 0; v < DIGITS; ++v) mine += x[v];
    uint32_t upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const uint32_t y = __shfl_up(upto, o);
        if (lane >= o) upto += y;
    }
    if (lane == 63) wave_sums[wave] = upto;
    __syncthreads();
    uint32_t at = upto - mine;
    for (int w = 0; w < wave; ++w) at += wave_sums[w];
#pragma unroll
    for (int v = 0; v < DIGITS; ++v) {
        const uint32_t c = x[v];
        x[v] = at;
        at += c;
    }
}

// Puts the first `count` pairs of a tile (pair u of a lane is number (wave * SORT_KEYS + u) * 64 + lane) into `sorted` in the order of
// their digits.  next: scratch; afterwards begin[d] is where digit d begins.
struct SortSpaceLds {
    uint32_t next[SORT_WAVES][BINS_MOST];  // where a wave's next pair of a digit goes
    uint32_t begin[BINS_MOST];
    uint32_t wave_sums[SORT_WAVES];
    uint2 sorted[SORT_TILE];
};
__device__ __forceinline__ void sort_tile(SortSpaceLds& s, const uint2 (&pair)[SORT_KEYS], int count, int shift, int bits) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, mask = (1 << bits) - 1;
    for (int d = lane; d < BINS_MOST; d += 64) s.next[wave][d] = 0;
    uint32_t rank[SORT_KEYS];  // among the wave's pairs of the digit
#pragma unroll
    for (int u = 0; u < SORT_KEYS; ++u) {
        const bool ok = (wave * SORT_KEYS + u) * 64 + lane < count;
        const uint32_t d = (pair[u].x >> shift) & mask;
        uint64_t same = __builtin_amdgcn_ballot_w64(ok);  // lanes of this digit
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __builtin_amdgcn_ballot_w64((d >> b) & 1);
            same &= (d >> b) & 1 ? set : ~set;
        }
        const int first = ok ? __ffsll((unsigned long long)same) - 1 : lane;
        uint32_t r = 0;
        if (ok && lane == first) r = atomicAdd(&s.next[wave][d], (uint32_t)__popcll(same));
        rank[u] = __shfl(r, first) + __popcll(same & (((uint64_t)1 << lane) - 1));
    }
    __syncthreads();
    uint32_t at[DIGITS];
#pragma unroll
    for (int v = 0; v < DIGITS; ++v) {
        const int d = DIGITS * threadIdx.x + v;
        uint32_t sum = 0;
#pragma unroll
        for (int w = 0; w < SORT_WAVES; ++w) {
            const uint32_t c = s.next[w][d];
            s.next[w][d] = sum;
            sum += c;
        }
        at[v] = sum;
    }
    scan_digits(at, s.wave_sums);
#pragma unroll
    for (int v = 0; v < DIGITS; ++v) s.begin[DIGITS * threadIdx.x + v] = at[v];
    __syncthreads();
#pragma unroll
    for (int u = 0; u < SORT_KEYS; ++u)
        if ((wave * SORT_KEYS + u) * 64 + lane < count) {
            const uint32_t d = (pair[u].x >> shift) & mask;
            s.sorted[s.begin[d] + s.next[wave][d] + rank[u]] = pair[u];
        }
    __syncthreads();
}

template <typename ID>
__device__ __forceinline__ void load_tile(uint2 (&pair)[SORT_KEYS], const ID* ids, const uint2* pairs, int64_t i0, int count, uint32_t rows) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int u = 0; u < SORT_KEYS; ++u) {
        const int i = (wave * SORT_KEYS + u) * 64 + lane;
        pair[u] = pair_at(ids, pairs, i0 + (i < count ? i : count - 1), rows);
    }
}

template <typename ID>
__global__ __launch_bounds__(SORT_THREADS) void digit_move_kernel(const ID* __restrict__ ids, const uint2* __restrict__ pairs,
                                                                  const uint32_t* __restrict__ counts, const uint32_t* __restrict__ totals,
                                                                  uint2* __restrict__ out, uint32_t* __restrict__ keys_out,
                                                                  uint32_t* __restrict__ positions_out, int64_t n, int64_t per_range, int ranges,
                                                                  uint32_t rows, int shift, int bits, Fill fill) {
    if ((int)blockIdx.x >= ranges) return fill_zero(fill, blockIdx.x - ranges, gridDim.x - ranges);
    __shared__ SortSpaceLds s;
    __shared__ uint32_t to[BINS_MOST];  // where the range's next pair of a digit goes
    const int bins = 1 << bits;
    uint32_t at[DIGITS] = {}, before[DIGITS] = {};
    const int d0 = DIGITS * threadIdx.x;
    static_assert(DIGITS == 2, "a thread's counts are one load");
    if (d0 < bins) {
        if (totals) {
            const uint2 all = *(const uint2*)(totals + d0), mine = *(const uint2*)(counts + (int64_t)blockIdx.x * bins + d0);
            at[0] = all.x; at[1] = all.y; before[0] = mine.x; before[1] = mine.y;
        } else {
            for (int r0 = 0; r0 < ranges; r0 += SCAN_FETCH) {
                uint2 c[SCAN_FETCH];
#pragma unroll
                for (int u = 0; u < SCAN_FETCH; ++u) c[u] = *(const uint2*)(counts + (int64_t)(r0 + u < ranges ? r0 + u : r0) * bins + d0);
#pragma unroll
                for (int u = 0; u < SCAN_FETCH; ++u) {
                    if (r0 + u < ranges) { at[0] += c[u].x; at[1] += c[u].y; }
                    if (r0 + u < (int)blockIdx.x) { before[0] += c[u].x; before[1] += c[u].y; }
                }
            }
        }
    }
    scan_digits(at, s.wave_sums);
#pragma unroll
    for (int v = 0; v < DIGITS; ++v) to[d0 + v] = at[v] + before[v];
    const int64_t begin = blockIdx.x * per_range, end = begin + per_range < n ? begin + per_range : n;
    for (int64_t i0 = begin; i0 < end; i0 += SORT_TILE) {
        const int count = end - i0 < SORT_TILE ? (int)(end - i0) : SORT_TILE;
        uint2 pair[SORT_KEYS];
        load_tile(pair, ids, pairs, i0, count, rows);
        __syncthreads();  // the tile before is written out
        sort_tile(s, pair, count, shift, bits);
        for (int i = threadIdx.x; i < count; i += SORT_THREADS) {
            const uint2 p = s.sorted[i];
            const uint32_t d = (p.x >> shift) & (bins - 1);
            const uint32_t at = to[d] + i - s.begin[d];
            if (out) out[at] = p;
            else {
                keys_out[at] = p.x;
                positions_out[at] = p.y;
            }
        }
        if (i0 + SORT_TILE >= end) break;
        __syncthreads();
#pragma unroll
        for (int v = 0; v < DIGITS; ++v) {
            const int d = d0 + v;
            if (d < bins) to[d] += (d + 1 < bins ? s.begin[d + 1] : count) - s.begin[d];
        }
    }
}

template <typename ID>
__global__ __launch_bounds__(SORT_THREADS) void sort_small_kernel(const ID* __restrict__ ids, uint32_t* __restrict__ keys_out,
                                                                  uint32_t* __restrict__ positions_out, int n, uint32_t rows, int passes, int bits,
                                                                  Fill fill) {
    if (blockIdx.x > 0) return fill_zero(fill, blockIdx.x - 1, gridDim.x - 1);
    __shared__ SortSpaceLds s;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint2 pair[SORT_KEYS];
    load_tile(pair, ids, (const uint2*)nullptr, 0, n, rows);
    for (int p = 0; p < passes; ++p) {
        sort_tile(s, pair, n, p * bits, bits);
        if (p + 1 < passes) {
#pragma unroll
            for (int u = 0; u < SORT_KEYS; ++u) {
                const int i = (wave * SORT_KEYS + u) * 64 + lane;
                pair[u] = s.sorted[i < n ? i : n - 1];
            }
            __syncthreads();
        }
    }
    for (int i = threadIdx.x; i < n; i += SORT_THREADS) {
        keys_out[i] = s.sorted[i].x;
        positions_out[i] = s.sorted[i].y;
    }
}

// ---- sums of the rows of equal ids ----

constexpr int ADD_FETCH = 8;  // rows in flight per lane group
constexpr int JOIN_FETCH = 8, JOIN_ALONE = 16;  // partial sums in flight; ranges of a run that one lane group adds
constexpr int JOIN_STARTS = 16;                 // ranges per workgroup: few runs that begin in them are long
constexpr int JOIN_SUMS = 16;                   // most parts of a longer one that are added one after another
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
                                                                float* __restrict__ partial, float* __restrict__ whole, int64_t n, uint32_t rows,
                                                                int D, float scale, int lanes, int64_t chunk, int64_t add_blocks) {
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
    float acc[W];
#pragma unroll
    for (int j = 0; j < W; ++j) acc[j] = 0.f;
    // all ranges of the workgroup inside one run: one partial sum for them
    const int64_t b0 = (int64_t)blockIdx.x * groups * chunk, b1 = b0 + groups * chunk;
    if (b0 > 0 && b1 < n && keys[b0 - 1] == keys[b1]) {
        if (keys[b1] >= rows) return;
        __shared__ float parts[THREADS * W];
        for (int64_t i = i0; i < i1; i += ADD_FETCH) {
            Piece<T, W> x[ADD_FETCH];
#pragma unroll
            for (int u = 0; u < ADD_FETCH; ++u) x[u] = load_piece<T, W>(d_out + (int64_t)positions[i + u] * D + at);
#pragma unroll
            for (int u = 0; u < ADD_FETCH; ++u)
#pragma unroll
                for (int j = 0; j < W; ++j) acc[j] += to_float(x[u].v[j]);
        }
#pragma unroll
        for (int j = 0; j < W; ++j) parts[threadIdx.x * W + j] = acc[j];
        __syncthreads();
        if (group > 0 || !has) return;
        for (int g = 1; g < groups; ++g)
#pragma unroll
            for (int j = 0; j < W; ++j) acc[j] += parts[(g * lanes + threadIdx.x) * W + j];
        float* const p = whole + ((int64_t)blockIdx.x * pieces + c) * W;
#pragma unroll
        for (int j = 0; j < W; ++j) p[j] = acc[j];
        return;
    }
    if (i0 >= n || !has) return;
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

// The partial sums of a run behind the range where it begins, in order: of ranges (slot 0) up to the first workgroup of the kernel above
// whose ranges are all inside the run, of those workgroups, of the ranges behind them.
struct RunSums {
    const float *partial, *whole;
    int64_t first, lead, blocks, block0, tail0, count;  // the first range; how many ranges and workgroups; the first workgroup; the range behind
    __device__ __forceinline__ RunSums(const float* partial_, const float* whole_, int64_t walker, int64_t last, int per_block)
        : partial(partial_), whole(whole_), first(walker + 1) {
        block0 = (walker + per_block) / per_block;
        blocks = last / per_block - block0;
        if (blocks <= 0) {
            blocks = 0;
            lead = last - walker;
            tail0 = last + 1;
        } else {
            lead = block0 * per_block - first;
            tail0 = (block0 + blocks) * per_block;
        }
        count = lead + blocks + (last + 1 - tail0);
    }
    __device__ __forceinline__ const float* at(int64_t i, int pieces, int c, int W) const {
        if (i < lead) return partial + ((first + i) * 2 * pieces + c) * W;
        i -= lead;
        if (i < blocks) return whole + ((block0 + i) * pieces + c) * W;
        return partial + ((tail0 + i - blocks) * 2 * pieces + c) * W;
    }
};
// acc += sums begin .. end - 1
template <int W>
__device__ __forceinline__ void add_sums(float (&acc)[W], const RunSums& sums, int64_t begin, int64_t end, int pieces, int c) {
    for (int64_t r = begin; r < end; r += JOIN_FETCH) {
        float x[JOIN_FETCH][W];
#pragma unroll
        for (int u = 0; u < JOIN_FETCH; ++u)
            __builtin_memcpy(x[u], __builtin_assume_aligned(sums.at(r + u < end ? r + u : begin, pieces, c, W), W % 4 ? 4 : 16), sizeof(x[u]));
#pragma unroll
        for (int u = 0; u < JOIN_FETCH; ++u)
#pragma unroll
            for (int j = 0; j < W; ++j) acc[j] += r + u < end ? x[u][j] : 0.f;
    }
}

// Runs that cross ranges.  The lane group of the range where one begins adds its partial sums in order; a run of more than JOIN_ALONE
// sums is shared by the lane groups of the workgroup, each of which adds a part, and the parts are added in order.
template <typename T, int W>
__global__ __launch_bounds__(THREADS) void embedding_join_kernel(const uint32_t* __restrict__ keys, const float* __restrict__ partial,
                                                                 const float* __restrict__ whole,
                                                                 T* __restrict__ d_table, int64_t n, uint32_t rows, int D, float scale, int lanes,
                                                                 int64_t chunk) {
    __shared__ int64_t last_of[JOIN_STARTS];  // of the run that begins in a lane group's range: the last range it is in (0: none to add)
    __shared__ uint32_t key_of[JOIN_STARTS];
    __shared__ float parts[THREADS * W];     // [groups][lanes][W]
    const int pieces = (D + W - 1) / W;
    const int lane = threadIdx.x % lanes, c = blockIdx.y * 64 + lane, group = threadIdx.x / lanes, groups = THREADS / lanes;
    const bool has = c < pieces;
    const int starts = groups < JOIN_STARTS ? groups : JOIN_STARTS;  // ranges that the workgroup looks at
    const int64_t walker0 = (int64_t)blockIdx.x * starts, walker = walker0 + group, i0 = walker * chunk, i1 = i0 + chunk;
    int64_t last = 0;
    uint32_t key = 0;
    if (group < starts && i1 < n) {
        key = keys[i1 - 1];
        const uint32_t behind = keys[i1], before = keys[i0 > 0 ? i0 - 1 : 0], further = keys[i1 + chunk < n ? i1 + chunk : n - 1];
        if (key < rows && behind == key && !(i0 > 0 && before == key)) {
            // the range that holds the run's last pair: most end in the next one, the others are searched for in growing steps
            last = walker + 1;
            if (i1 + chunk < n && further == key) {
                int64_t at = i1 + chunk, step = 2 * chunk;
                for (; at + step < n && keys[at + step] == key; step *= 2) at += step;
                last = (first_at_least(keys, at + 1, at + step < n ? at + step : n, key + 1) - 1) / chunk;
            }
        }
    }
    auto finish = [&](const float (&acc)[W], uint32_t k) {
        Piece<T, W> y;
#pragma unroll
        for (int j = 0; j < W; ++j) y.v[j] = from_float<T>(acc[j] * scale);
        if (has) store_piece<T, W>(d_table + (int64_t)k * D + piece_start(c, D, W), y);
    };
    const int cc = has ? c : pieces - 1;
    const RunSums mine_sums(partial, whole, walker, last ? last : walker, groups);
    const bool together = mine_sums.count > JOIN_ALONE;
    if (last && !together) {
        float acc[W];
        const float* p = partial + ((walker * 2 + 1) * pieces + cc) * W;
#pragma unroll
        for (int j = 0; j < W; ++j) acc[j] = p[j];
        add_sums<W>(acc, mine_sums, 0, mine_sums.count, pieces, cc);
        finish(acc, key);
    }
    if (lane == 0 && group < starts) {
        last_of[group] = together ? last : 0;
        key_of[group] = key;
    }
    __syncthreads();
    for (int w = 0; w < starts; ++w) {
        if (last_of[w] == 0) continue;
        const RunSums sums(partial, whole, walker0 + w, last_of[w], groups);
        const int64_t per = (sums.count + groups - 1) / groups, mine = group * per;
        float acc[W];
#pragma unroll
        for (int j = 0; j < W; ++j) acc[j] = 0.f;
        if (group == 0) {
            const float* p = partial + (((walker0 + w) * 2 + 1) * pieces + cc) * W;
#pragma unroll
            for (int j = 0; j < W; ++j) acc[j] = p[j];
        }
        add_sums<W>(acc, sums, mine, mine + per < sums.count ? mine + per : sums.count, pieces, cc);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < W; ++j) parts[threadIdx.x * W + j] = acc[j];
        __syncthreads();
        const auto add_parts = [&](int g0, int g1) {
            for (int g = g0; g < g1; ++g)
#pragma unroll
                for (int j = 0; j < W; ++j) acc[j] += parts[(g * lanes + lane) * W + j];
        };
        const int joined = groups < JOIN_SUMS ? groups : JOIN_SUMS, span = groups / joined;
        if (span > 1) {  // (many narrow lane groups: their parts in two steps)
            const int g0 = group * span;
            if (group < joined) {
#pragma unroll
                for (int j = 0; j < W; ++j) acc[j] = 0.f;
                add_parts(g0, g0 + span);
            }
            __syncthreads();
            if (group < joined)
#pragma unroll
                for (int j = 0; j < W; ++j) parts[threadIdx.x * W + j] = acc[j];
            __syncthreads();
        }
        if (group == 0) {
            add_parts(1, joined);
            finish(acc, key_of[w]);
        }
    }
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

// Pairs per lane group: ranges enough to fill the device (16 waves per compute unit of them), long ones otherwise, so that few runs
// cross a range and leave partial sums (1.1 million rows of 64, eight lanes each: 119 us with 8942 ranges, 109 us with 35 769).
constexpr int64_t CHUNK_LEAST = 8;
int64_t ranges_most(int lanes) { return lanes < 8 ? 1 << 16 : lanes < 32 ? (1 << 19) / lanes : 1 << 14; }
int64_t add_chunk(int64_t n, int lanes) {
    int64_t chunk = CHUNK_LEAST;
    while ((n + chunk - 1) / chunk > ranges_most(lanes)) chunk *= 2;
    return chunk;
}
int64_t ranges_at_most(int64_t n, int lanes) {
    const int64_t r = (n + CHUNK_LEAST - 1) / CHUNK_LEAST;
    return r < ranges_most(lanes) ? r : ranges_most(lanes);
}

struct SortSpace {
    uint2* pairs[2];
    uint32_t *keys, *positions;  // in the end
    uint32_t *counts, *totals;
    float *partial, *whole;  // per range, per workgroup of ranges
    size_t bytes;
    SortSpace(char* base, int64_t n, int D, int dtype) {
        size_t at = 0;
        auto take = [&](size_t b) { char* p = base + at; at += align_up(b, 256); return p; };
        for (int i = 0; i < 2; ++i) pairs[i] = (uint2*)take((size_t)n * 8);
        keys = (uint32_t*)take((size_t)n * 4);
        positions = (uint32_t*)take((size_t)n * 4);
        const int64_t tiles = (n + SORT_TILE - 1) / SORT_TILE;
        counts = (uint32_t*)take((size_t)(tiles < SORT_RANGES ? tiles : SORT_RANGES) * BINS_MOST * 4);
        totals = (uint32_t*)take(BINS_MOST * 4);
        const int W = dtype == KUNLUN_FP32 ? piece_width<float>(D) : piece_width<bf16_t>(D);
        const int pieces = pieces_per_row(D, W);
        const int lanes = lanes_per_row(pieces);
        const int64_t ranges = ranges_at_most(n, lanes);
        partial = (float*)take((size_t)ranges * 2 * pieces * W * 4);
        whole = (float*)take((size_t)(ranges / (THREADS / lanes) + 1) * pieces * W * 4);
        bytes = at;
    }
};

// fill_bytes > 0: the launches set that much of d_table to zero as well, each an equal part.
template <typename ID>
void sort_ids(const void* ids, const SortSpace& s, int64_t n, int64_t rows, void* d_table, int64_t fill_bytes, hipStream_t stream) {
    int bits = 1;
    while (rows >> bits) ++bits;  // keys are 0 .. rows
    const int passes = (bits + DIGIT_MOST - 1) / DIGIT_MOST, digit = (bits + passes - 1) / passes;
    const int launches = n <= SORT_TILE ? 1 : 2 * passes;
    const int64_t part = (fill_bytes + launches * 16 - 1) / (launches * 16) * 16;
    const unsigned fill_blocks = (unsigned)(part / (SORT_THREADS * 64) < FILL_BLOCKS ? (part + SORT_THREADS * 64 - 1) / (SORT_THREADS * 64) : FILL_BLOCKS);
    int launched = 0;
    const auto fill = [&] {
        const int64_t begin = launched++ * part, end = begin + part;
        return Fill{(char*)d_table, begin < fill_bytes ? begin : fill_bytes, end < fill_bytes ? end : fill_bytes};
    };
    if (n <= SORT_TILE) {
        hipLaunchKernelGGL(sort_small_kernel<ID>, dim3(1 + fill_blocks), dim3(SORT_THREADS), 0, stream, (const ID*)ids, s.keys, s.positions, (int)n, (uint32_t)rows, passes,
                           digit, fill());
        return;
    }
    const int64_t tiles = (n + SORT_TILE - 1) / SORT_TILE, per_range = (tiles + SORT_RANGES - 1) / SORT_RANGES * SORT_TILE;
    const unsigned ranges = (unsigned)((n + per_range - 1) / per_range);
    const int bins = 1 << digit;
    // few ranges: every range sums the counts itself (34 ranges: 8 us for two passes less than with the launch between)
    uint32_t* const totals = ranges > SCAN_RANGES ? s.totals : nullptr;
    for (int p = 0; p < passes; ++p) {
        const uint2* from = p ? s.pairs[(p + 1) & 1] : nullptr;
        hipLaunchKernelGGL(digit_count_kernel<ID>, dim3(ranges + fill_blocks), dim3(SORT_THREADS), 0, stream, (const ID*)ids, from, s.counts, n,
                           per_range, (int)ranges, (uint32_t)rows, p * digit, digit, fill());
        if (totals)
            hipLaunchKernelGGL(digit_scan_kernel, dim3((unsigned)((bins + 31) / 32)), dim3(32 * SCAN_PARTS), 0, stream, s.counts, totals, (int)ranges,
                               bins);
        hipLaunchKernelGGL(digit_move_kernel<ID>, dim3(ranges + fill_blocks), dim3(SORT_THREADS), 0, stream, (const ID*)ids, from, s.counts, totals,
                           p + 1 < passes ? s.pairs[p & 1] : nullptr, s.keys, s.positions, n, per_range, (int)ranges, (uint32_t)rows,
                           p * digit, digit, fill());
    }
}

template <typename T, int W>
void embedding_bwd(const void* d_out, const SortSpace& s, void* d_table, int64_t n, int64_t rows, int D, float scale, bool filled,
                   hipStream_t stream) {
    const int pieces = pieces_per_row(D, W), lanes = lanes_per_row(pieces), groups = THREADS / lanes;
    const int64_t chunk = add_chunk(n, lanes), ranges = (n + chunk - 1) / chunk;
    const int64_t add_blocks = (ranges + groups - 1) / groups, zero_all = (rows + ZERO_ROWS - 1) / ZERO_ROWS;
    const int64_t zero_blocks = filled ? 0 : zero_all < GRID_MOST ? zero_all : GRID_MOST;
    const unsigned tiles = (unsigned)((pieces + 63) / 64);
    hipLaunchKernelGGL((embedding_add_kernel<T, W>), dim3((unsigned)(add_blocks + zero_blocks), tiles), dim3(THREADS), 0, stream, (const T*)d_out,
                       s.keys, s.positions, (T*)d_table, s.partial, s.whole, n, (uint32_t)rows, D, scale, lanes, chunk,
                       add_blocks);
    const int starts = groups < JOIN_STARTS ? groups : JOIN_STARTS;
    if (ranges > 1)
        hipLaunchKernelGGL((embedding_join_kernel<T, W>), dim3((unsigned)((ranges + starts - 1) / starts), tiles), dim3(THREADS), 0, stream, s.keys, s.partial, s.whole,
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

// A gradient up to here is set to zero by the sorting launches, which leave most of the device idle, and rows with ids are written over
// (139 264 rows of 256 into 200 000: 83 -> 78 us, into 500 000: 107 -> 95; 640 into 500 000: 66 -> 54); beyond, the rows without ids are
// found among the sorted ones.
constexpr int64_t FILL_MOST = (int64_t)256 << 20;

hipError_t launch_embedding_bwd(const void* d_out, const void* ids, void* d_table, int64_t n, int64_t rows, int D, float scale,
                                int id_bytes, int dtype, void* workspace, hipStream_t stream) {
    const SortSpace s((char*)workspace, n, D, dtype);
    const int64_t bytes = rows * D * (dtype == KUNLUN_FP32 ? 4 : 2);
    const bool filled = n > 0 && bytes <= FILL_MOST;
    if (n > 0) {
        if (id_bytes == 8) sort_ids<int64_t>(ids, s, n, rows, d_table, filled ? bytes : 0, stream);
        else sort_ids<int32_t>(ids, s, n, rows, d_table, filled ? bytes : 0, stream);
    }
    if (dtype == KUNLUN_FP32) {
        if (piece_width<float>(D) == 4) embedding_bwd<float, 4>(d_out, s, d_table, n, rows, D, scale, filled, stream);
        else embedding_bwd<float, 1>(d_out, s, d_table, n, rows, D, scale, filled, stream);
    } else {
        if (piece_width<bf16_t>(D) == 8) embedding_bwd<bf16_t, 8>(d_out, s, d_table, n, rows, D, scale, filled, stream);
        else embedding_bwd<bf16_t, 1>(d_out, s, d_table, n, rows, D, scale, filled, stream);
    }
    return hipGetLastError();
}

}  // namespace kunlun
