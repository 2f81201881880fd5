// Layer normalisation of rows and its gradients.
//     y = (x - m) r w + b,  m = mean(x), r = 1 / sqrt(mean((x - m)^2) + eps)
//     with h = (x - m) r and g = dy w:  dx = r (g - mean(g) - h mean(g h)),  dw = sum dy h,  db = sum dy  over the rows
// Bound by memory: a row is read once into registers, held by the lanes of a group of up to 64 (narrow rows share a wave) or, beyond
// 32 values per lane, by a whole workgroup; mean and variance are reduced across them (two passes over the registers, so that the
// variance loses nothing to a large mean) and the row is written once.
// The weight's gradients are sums over the rows: every workgroup of the backward launch takes the rows blockIdx + k * grid,
// keeps its columns' sums in registers, joins its lane groups through LDS in order and leaves one fp32 row per workgroup; a
// second kernel adds those in order.  No atomics: equal calls give equal bits.
// Measured (a copy reaches 5.07 TB/s here): forward of 139 264 bf16 rows of 256 29 us (4.9 TB/s); backward of 1 144 603 rows of 1024
// 1.27 ms (5.5 TB/s, two reads to a write); of 9973 fp32 rows of 203 13.0 us, 8.6 of them the rows', 4 the column sums'.  A vector
// operation per step instead of an LDS exchange, and the next row under way, took the latter from 16.7.
#include "layers.h"

namespace kunlun {

namespace {

constexpr int THREADS = 256;
constexpr int VALUES_PER_LANE = 32;  // most values of a row that a lane holds where a wave holds rows

// x + the value of x in the lane that CTRL names, by a vector operation (a shuffle would take an LDS round trip).
template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) {
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
// Sum over the lanes of a group (a power of two up to 64; all lanes of the wave take part), the same in all of them.
__device__ __forceinline__ float lanes_sum(float x, int lanes) {
    if (lanes > 1) x = add_dpp<0xb1>(x);   // lane ^ 1
    if (lanes > 2) x = add_dpp<0x4e>(x);   // lane ^ 2
    if (lanes > 4) x = add_dpp<0x141>(x);  // mirrored in 8 lanes, whose fours are equal by now
    if (lanes > 8) x = add_dpp<0x140>(x);  // mirrored in 16
    if (lanes > 16) {
        const unsigned u = __builtin_bit_cast(unsigned, x);
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        x = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
    }
    if (lanes > 32) {
        const unsigned u = __builtin_bit_cast(unsigned, x);
        const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        x = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
    }
    return x;
}
// Sums of N values over a group, or over the whole workgroup (WIDE).
template <bool WIDE, int N>
__device__ __forceinline__ void group_sums(float (&x)[N], int lanes, float (*scratch)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = lanes_sum(x[i], WIDE ? 64 : lanes);
    if constexpr (WIDE) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) scratch[threadIdx.x >> 6][i] = x[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = scratch[0][i];
#pragma unroll
            for (int w = 1; w < THREADS / 64; ++w) x[i] += scratch[w][i];
        }
    }
}

// Where a lane's pieces lie: piece c of the row starts at at(c); the first dup(c) values of it belong to the piece before (all W: no piece)
template <int W, int VPL>
struct Pieces {
    int at[VPL], dup[VPL];
    __device__ __forceinline__ Pieces(int lane, int lanes, int D) {
        const int n = (D + W - 1) / W;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const int c = lane + i * lanes, held = c < n ? c : n - 1;
            at[i] = piece_start(held, D, W);
            dup[i] = c < n ? piece_dup(c, D, W) : W;
        }
    }
    __device__ __forceinline__ bool has(int i) const { return dup[i] < W; }
};

template <typename T, int W, int VPL, bool WIDE>
__global__ __launch_bounds__(THREADS) void norm_fwd_kernel(const T* __restrict__ x, const T* __restrict__ weight, const T* __restrict__ bias,
                                                           T* __restrict__ y, float* __restrict__ mean, float* __restrict__ rstd, int64_t rows,
                                                           int D, float eps, int lanes) {
    __shared__ float scratch[THREADS / 64][1];
    const int per_row = WIDE ? THREADS : lanes, lane = threadIdx.x % per_row, groups = THREADS / per_row;
    const Pieces<W, VPL> at(lane, per_row, D);
    Piece<T, W> w[VPL], b[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        if (weight) w[i] = load_piece_kept<T, W>(weight + at.at[i]);
        if (bias) b[i] = load_piece_kept<T, W>(bias + at.at[i]);
    }
    const float n = (float)D;  // (divided by, not multiplied by its rounded reciprocal: the mean of equal values is that value)
    const int64_t step = (int64_t)gridDim.x * groups;
    // (every lane of a wave stays in the loop: the sums across lanes need them)
    for (int64_t r0 = (int64_t)blockIdx.x * groups; r0 < rows; r0 += step) {
        const int64_t mine = r0 + threadIdx.x / per_row, r = mine < rows ? mine : rows - 1;
        Piece<T, W> v[VPL];
#pragma unroll
        for (int i = 0; i < VPL; ++i) v[i] = load_piece<T, W>(x + r * D + at.at[i]);
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < VPL; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j) s[0] += j >= at.dup[i] ? to_float(v[i].v[j]) : 0.f;
        group_sums<WIDE>(s, lanes, scratch);
        const float m = s[0] / n;
        s[0] = 0.f;
#pragma unroll
        for (int i = 0; i < VPL; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const float d = to_float(v[i].v[j]) - m;
                s[0] += j >= at.dup[i] ? d * d : 0.f;
            }
        group_sums<WIDE>(s, lanes, scratch);
        const float rs = 1.f / sqrtf(s[0] / n + eps);
        if (mine >= rows) continue;
        if (lane == 0) {
            if (mean) mean[r] = m;
            if (rstd) rstd[r] = rs;
        }
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            if (!at.has(i)) continue;
            Piece<T, W> o;
#pragma unroll
            for (int j = 0; j < W; ++j) {
                float t = (to_float(v[i].v[j]) - m) * rs;
                if (weight) t *= to_float(w[i].v[j]);
                if (bias) t += to_float(b[i].v[j]);
                o.v[j] = from_float<T>(t);
            }
            store_piece<T, W>(y + r * D + at.at[i], o);
        }
    }
}

// partial: [gridDim.x][2][D] sums of dy h and of dy (null: neither is wanted)
template <typename T, int W, int VPL, bool WIDE>
__global__ __launch_bounds__(THREADS) void norm_bwd_kernel(const T* __restrict__ x, const T* __restrict__ weight, const T* __restrict__ dy,
                                                           const float* __restrict__ mean, const float* __restrict__ rstd, T* __restrict__ dx,
                                                           float* __restrict__ partial, int64_t rows, int D, int lanes) {
    extern __shared__ float columns[];  // [groups][D], one of the two sums at a time
    __shared__ float scratch[THREADS / 64][2];
    const int per_row = WIDE ? THREADS : lanes, lane = threadIdx.x % per_row, groups = THREADS / per_row, group = threadIdx.x / per_row;
    const Pieces<W, VPL> at(lane, per_row, D);
    Piece<T, W> w[VPL];
    float dw[VPL][W], db[VPL][W];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        if (weight) w[i] = load_piece_kept<T, W>(weight + at.at[i]);
#pragma unroll
        for (int j = 0; j < W; ++j) dw[i][j] = db[i][j] = 0.f;
    }
    const float n = (float)D;
    const int64_t step = (int64_t)gridDim.x * groups;
    constexpr bool AHEAD = VPL * W <= 16;  // registers to spare: the next row is under way while one is computed
    struct Row {
        Piece<T, W> v[VPL], d[VPL];
        float m, rs;
    };
    auto load = [&](Row& row, int64_t r0) {
        const int64_t r = r0 + group < rows ? r0 + group : rows - 1;
        row.m = mean[r];
        row.rs = rstd[r];
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            row.v[i] = load_piece<T, W>(x + r * D + at.at[i]);
            row.d[i] = load_piece<T, W>(dy + r * D + at.at[i]);
        }
    };
    Row now;
    if (AHEAD) load(now, (int64_t)blockIdx.x * groups);
    for (int64_t r0 = (int64_t)blockIdx.x * groups; r0 < rows; r0 += step) {
        const int64_t r = r0 + group;
        const bool ok = r < rows;
        Row next;
        if (AHEAD) load(next, r0 + step);
        else load(now, r0);
        const float m = now.m, rs = now.rs;
        float sums[2] = {0.f, 0.f};  // of g, of g h
#pragma unroll
        for (int i = 0; i < VPL; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const float h = (to_float(now.v[i].v[j]) - m) * rs, t = to_float(now.d[i].v[j]), g = weight ? t * to_float(w[i].v[j]) : t;
                const bool counts = j >= at.dup[i];
                sums[0] += counts ? g : 0.f;
                sums[1] += counts ? g * h : 0.f;
                dw[i][j] += ok ? t * h : 0.f;
                db[i][j] += ok ? t : 0.f;
            }
        if (dx) {
            group_sums<WIDE>(sums, lanes, scratch);
            const float sg = sums[0] / n, sgh = sums[1] / n;
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                if (!ok || !at.has(i)) continue;
                Piece<T, W> o;
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const float h = (to_float(now.v[i].v[j]) - m) * rs, t = to_float(now.d[i].v[j]), g = weight ? t * to_float(w[i].v[j]) : t;
                    o.v[j] = from_float<T>((g - sg - h * sgh) * rs);
                }
                store_piece<T, W>(dx + r * D + at.at[i], o);
            }
        }
        if (AHEAD) now = next;
    }
    if (!partial) return;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float* out = partial + ((int64_t)blockIdx.x * 2 + k) * D;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            if (at.has(i))
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    if (j < at.dup[i]) continue;
                    if (groups == 1) out[at.at[i] + j] = k ? db[i][j] : dw[i][j];
                    else columns[group * D + at.at[i] + j] = k ? db[i][j] : dw[i][j];
                }
        if (groups == 1) continue;
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += THREADS) {
            float t = columns[c];
            for (int q = 1; q < groups; ++q) t += columns[q * D + c];
            out[c] = t;
        }
    }
}

// out[c] = sum of partial[p][c] over the p: 32 columns x 32 ranges of p per workgroup, ranges joined in order.  Columns 0 .. D - 1 go to
// dw, the rest to db.
constexpr int RANGES = 32, COLUMN_FETCH = 8;
template <typename T>
__global__ __launch_bounds__(32 * RANGES) void norm_columns_kernel(const float* __restrict__ partial, T* __restrict__ dw, T* __restrict__ db,
                                                                   int parts, int D) {
    __shared__ float sums[RANGES][32];
    const int col = threadIdx.x & 31, range = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + col, held = c < 2 * D ? c : 0;
    const int per = (parts + RANGES - 1) / RANGES, p0 = range * per, p1 = p0 + per < parts ? p0 + per : parts;
    float t = 0.f;
    for (int p = p0; p < p1; p += COLUMN_FETCH) {
        float x[COLUMN_FETCH];
#pragma unroll
        for (int u = 0; u < COLUMN_FETCH; ++u) x[u] = partial[(int64_t)(p + u < p1 ? p + u : p0) * 2 * D + held];
#pragma unroll
        for (int u = 0; u < COLUMN_FETCH; ++u) t += p + u < p1 ? x[u] : 0.f;
    }
    sums[range][col] = t;
    __syncthreads();
    if (range != 0 || c >= 2 * D) return;
#pragma unroll
    for (int i = 1; i < RANGES; ++i) t += sums[i][col];
    T* out = c < D ? dw : db;
    if (out) out[c < D ? c : c - D] = from_float<T>(t);
}

// How a row is held: W values per piece, `lanes` lanes (64 for every wave of a workgroup that holds one row: wide), `pieces` per lane
struct RowPlan {
    int W, lanes, vpl;
    bool wide;
};
RowPlan plan_row(int D, int elt) {
    RowPlan p;
    p.W = D * elt >= 16 ? 16 / elt : 1;
    const int pieces = pieces_per_row(D, p.W);
    p.lanes = lanes_per_row(pieces);
    p.wide = pieces > 64 * (VALUES_PER_LANE / p.W);
    const int over = p.wide ? THREADS : p.lanes;
    p.vpl = 1;
    while (p.vpl * over < pieces) p.vpl *= 2;
    return p;
}

// Workgroups of the backward launch, each with a row of partial sums: two per compute unit, four where rows are narrow and what a
// workgroup waits for counts more than the partial sums do
int64_t bwd_blocks(int D) { return D <= 512 ? 1024 : 512; }
int64_t blocks_of(const RowPlan& p, int64_t rows, int64_t most) {
    const int groups = p.wide ? 1 : THREADS / p.lanes;
    const int64_t all = (rows + groups - 1) / groups;
    return all < most ? all : most;
}

template <typename T, int W, int VPL, bool WIDE>
void norm_fwd(const RowPlan& p, const void* x, const void* weight, const void* bias, void* y, float* mean, float* rstd, int64_t rows, int D,
              float eps, hipStream_t stream) {
    hipLaunchKernelGGL((norm_fwd_kernel<T, W, VPL, WIDE>), dim3((unsigned)blocks_of(p, rows, 8192)), dim3(THREADS), 0, stream, (const T*)x,
                       (const T*)weight, (const T*)bias, (T*)y, mean, rstd, rows, D, eps, p.lanes);
}
template <typename T, int W, int VPL, bool WIDE>
void norm_bwd(const RowPlan& p, const void* x, const void* weight, const void* dy, const float* mean, const float* rstd, void* dx, float* partial,
              int64_t rows, int D, hipStream_t stream) {
    const size_t lds = p.wide || !partial ? 0 : (size_t)(THREADS / p.lanes) * D * sizeof(float);
    hipLaunchKernelGGL((norm_bwd_kernel<T, W, VPL, WIDE>), dim3((unsigned)blocks_of(p, rows, bwd_blocks(D))), dim3(THREADS), lds, stream, (const T*)x,
                       (const T*)weight, (const T*)dy, mean, rstd, (T*)dx, partial, rows, D, p.lanes);
}

// Calls F<T, W, VPL, WIDE> for the plan of a row
#define KUNLUN_NORM_CASE(F, TYPE, WIDTH, VPL, WHOLE, ...) \
    if (p.W == WIDTH && p.vpl == VPL && p.wide == WHOLE) return F<TYPE, WIDTH, VPL, WHOLE>(p, __VA_ARGS__), hipGetLastError()
#define KUNLUN_NORM(F, ...)                                  \
    if (dtype == KUNLUN_FP32) {                              \
        KUNLUN_NORM_CASE(F, float, 1, 1, false, __VA_ARGS__);    \
        KUNLUN_NORM_CASE(F, float, 4, 1, false, __VA_ARGS__);    \
        KUNLUN_NORM_CASE(F, float, 4, 2, false, __VA_ARGS__);    \
        KUNLUN_NORM_CASE(F, float, 4, 4, false, __VA_ARGS__);    \
        KUNLUN_NORM_CASE(F, float, 4, 8, false, __VA_ARGS__);    \
        KUNLUN_NORM_CASE(F, float, 4, 4, true, __VA_ARGS__);     \
        KUNLUN_NORM_CASE(F, float, 4, 8, true, __VA_ARGS__);     \
        KUNLUN_NORM_CASE(F, float, 4, 16, true, __VA_ARGS__);    \
    } else {                                                 \
        KUNLUN_NORM_CASE(F, bf16_t, 1, 1, false, __VA_ARGS__);   \
        KUNLUN_NORM_CASE(F, bf16_t, 8, 1, false, __VA_ARGS__);   \
        KUNLUN_NORM_CASE(F, bf16_t, 8, 2, false, __VA_ARGS__);   \
        KUNLUN_NORM_CASE(F, bf16_t, 8, 4, false, __VA_ARGS__);   \
        KUNLUN_NORM_CASE(F, bf16_t, 8, 2, true, __VA_ARGS__);    \
        KUNLUN_NORM_CASE(F, bf16_t, 8, 4, true, __VA_ARGS__);    \
        KUNLUN_NORM_CASE(F, bf16_t, 8, 8, true, __VA_ARGS__);    \
    }                                                        \
    return hipErrorInvalidValue;  /* (a plan without a kernel) */

hipError_t dispatch_fwd(const RowPlan& p, int dtype, const void* x, const void* weight, const void* bias, void* y, float* mean, float* rstd, int64_t rows,
                  int D, float eps, hipStream_t stream) {
    KUNLUN_NORM(norm_fwd, x, weight, bias, y, mean, rstd, rows, D, eps, stream)
}
hipError_t dispatch_bwd(const RowPlan& p, int dtype, const void* x, const void* weight, const void* dy, const float* mean, const float* rstd, void* dx,
                  float* partial, int64_t rows, int D, hipStream_t stream) {
    KUNLUN_NORM(norm_bwd, x, weight, dy, mean, rstd, dx, partial, rows, D, stream)
}

}  // namespace

hipError_t launch_layer_norm_fwd(const void* x, const void* weight, const void* bias, void* y, float* mean, float* rstd, int64_t rows,
                                 int D, float eps, int dtype, hipStream_t stream) {
    return dispatch_fwd(plan_row(D, dtype == KUNLUN_FP32 ? 4 : 2), dtype, x, weight, bias, y, mean, rstd, rows, D, eps, stream);
}

size_t layer_norm_bwd_workspace(int64_t rows, int D, int dtype) {
    const int64_t parts = blocks_of(plan_row(D, dtype == KUNLUN_FP32 ? 4 : 2), rows, bwd_blocks(D));
    return align_up((size_t)(parts > 0 ? parts : 1) * 2 * D * sizeof(float), 256);
}

hipError_t launch_layer_norm_bwd(const void* x, const void* weight, const void* dy, const float* mean, const float* rstd, void* dx,
                                 void* dw, void* db, int64_t rows, int D, int dtype, void* workspace, hipStream_t stream) {
    const RowPlan p = plan_row(D, dtype == KUNLUN_FP32 ? 4 : 2);
    float* partial = dw || db ? (float*)workspace : nullptr;
    const int parts = (int)blocks_of(p, rows, bwd_blocks(D));
    if (rows > 0) {
        const hipError_t e = dispatch_bwd(p, dtype, x, weight, dy, mean, rstd, dx, partial, rows, D, stream);
        if (e != hipSuccess) return e;
    }
    if (partial) {
        const dim3 grid((unsigned)((2 * D + 31) / 32));
        if (dtype == KUNLUN_FP32)
            hipLaunchKernelGGL(norm_columns_kernel<float>, grid, dim3(32 * RANGES), 0, stream, partial, (float*)dw, (float*)db, parts, D);
        else
            hipLaunchKernelGGL(norm_columns_kernel<bf16_t>, grid, dim3(32 * RANGES), 0, stream, partial, (bf16_t*)dw, (bf16_t*)db, parts, D);
    }
    return hipGetLastError();
}

}  // namespace kunlun
