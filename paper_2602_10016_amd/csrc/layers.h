// Shared declarations of the operators in front of attention (include/kunlun_layers.h): launchers, and the access to rows of
// any width and alignment that embedding and layer norm share.
#pragma once
#include "../../include/kunlun_layers.h"
#include "common.h"

namespace kunlun {

// ---- launchers (each enqueues on `stream`, returns the hipError_t of the launch) ----
hipError_t launch_embedding_fwd(const void* table, const void* ids, void* out, int64_t n, int64_t rows, int D, float scale, int id_bytes,
                                int dtype, hipStream_t stream);
size_t embedding_bwd_workspace(int64_t n, int D, int dtype);
hipError_t launch_embedding_bwd(const void* d_out, const void* ids, void* d_table, int64_t n, int64_t rows, int D, float scale,
                                int id_bytes, int dtype, void* workspace, hipStream_t stream);
hipError_t launch_layer_norm_fwd(const void* x, const void* weight, const void* bias, void* y, float* mean, float* rstd, int64_t rows,
                                 int D, float eps, int dtype, hipStream_t stream);
size_t layer_norm_bwd_workspace(int64_t rows, int D, int dtype);
hipError_t launch_layer_norm_bwd(const void* x, const void* weight, const void* dy, const float* mean, const float* rstd, void* dx,
                                 void* dw, void* db, int64_t rows, int D, int dtype, void* workspace, hipStream_t stream);
hipError_t launch_grouped_linear_fwd(const void* x, const void* w, void* y, const int32_t* offsets, int G, int64_t total, int K, int N,
                                     bool fill_rest, int dtype, hipStream_t stream);
size_t grouped_linear_bwd_workspace(int G, int64_t total, int K, int N, int dtype);
hipError_t launch_grouped_linear_bwd(const void* x, const void* w, const void* dy, void* dx, void* dw, const int32_t* offsets, int G,
                                     int64_t total, int K, int N, bool fill_rest, int dtype, void* workspace, hipStream_t stream);

#ifdef __HIPCC__
// A row of D values as pieces of W (16 bytes, or single values where D < 16 bytes).  Where W does not divide D the last piece
// is moved back to end with the row: it holds `dup` values of the piece before it, which sums leave out and stores write twice
// with the same value.  So every access is one wide instruction that stays inside the row; rows of odd widths start at any
// multiple of the value's size, which vector memory instructions of this target take.
typedef __attribute__((ext_vector_type(4), aligned(2))) unsigned int u32x4_any;

template <typename T, int W>
struct Piece {
    T v[W];
};
template <typename T, int W>
__device__ __forceinline__ Piece<T, W> load_piece(const T* p) {
    Piece<T, W> r;
    if constexpr (W == 1) r.v[0] = *p;
    else {
        static_assert(W * sizeof(T) == 16, "a piece is 16 bytes");
        r = __builtin_bit_cast(Piece<T, W>, __builtin_nontemporal_load((const u32x4_any*)p));
    }
    return r;
}
// (without the hint: what many rows read again, weights and table rows)
template <typename T, int W>
__device__ __forceinline__ Piece<T, W> load_piece_kept(const T* p) {
    Piece<T, W> r;
    if constexpr (W == 1) r.v[0] = *p;
    else r = __builtin_bit_cast(Piece<T, W>, *(const u32x4_any*)p);
    return r;
}
template <typename T, int W>
__device__ __forceinline__ void store_piece(T* p, const Piece<T, W>& x) {
    if constexpr (W == 1) *p = x.v[0];
    else __builtin_nontemporal_store(__builtin_bit_cast(u32x4_any, x), (u32x4_any*)p);
}
// First value of piece c, and how many of its values the piece before it holds
__device__ __forceinline__ int piece_start(int c, int D, int W) { return (c + 1) * W <= D ? c * W : D - W; }
__device__ __forceinline__ int piece_dup(int c, int D, int W) { return (c + 1) * W <= D ? 0 : (c + 1) * W - D; }
#endif

// Pieces per row, and the lanes (a power of two up to 64) that hold a row between them
inline int pieces_per_row(int D, int W) { return (D + W - 1) / W; }
inline int lanes_per_row(int pieces) {
    int n = 1;
    while (n < pieces && n < 64) n *= 2;
    return n;
}

}  // namespace kunlun
