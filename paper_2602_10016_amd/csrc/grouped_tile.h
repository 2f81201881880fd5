// The matrix-core product of the grouped linear maps: one BM x BN tile of C = A B per workgroup, bf16 or fp32 operands, fp32 sums.
//
// An operand lies in memory with the contraction along its rows ("row form": [rows, contraction]) or across them ("column form":
// [contraction, columns]).  y = x w has A in row form and B in column form, dx = dy w^T both in row form, dw = x^T dy both in column
// form; nothing is transposed in memory.  Steps of 128 bytes of contraction values (64 bf16, 32 fp32) travel straight from memory into a
// ring of LDS stages (buffer loads to LDS); fragments of a row-form tile are 16-byte reads, of a column-form tile transposing reads
// (bf16, mfma_tile.h) or four reads of a value (fp32).
//   LDS, row form:     128 bytes per row, 16-byte chunk ^= (row / 2) % 8: 16 consecutive rows of one chunk hit 16 different places
//   LDS, column form:  W values per contraction row; bf16: 64-byte group ^= row % 4 (W = 64: (row / 2) % 2, W = 32: nothing), so that four
//                      rows of one group do, too
// fp32 takes v_mfma_f32_32x32x2_f32, whose two contraction values come from the two lane halves: with 16-byte fragments, value t of the chunks
// 2c and 2c + 1.  The order of the contraction is the same for both operands, so it need not be the memory's.
// What lies outside is handled where it is loaded: rows and columns of C outside the tile re-read the last valid one (never stored);
// contraction values outside are zeros in both operands (a buffer load outside its descriptor's range gives zero), so that an infinity next
// to them does no harm.
// The matrix instructions compute C^T = B^T A^T, so that a lane holds consecutive columns of one row of C, which go out through LDS as
// whole rows, with streaming stores: 139 264 rows, 256 -> 768, 95 -> 85 us, 768 -> 256, 84 -> 76.
#pragma once
#include "lds_ring.h"

namespace kunlun {

// s_waitcnt that waits for LDS operations only.
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4)); }

constexpr int GL_STEP_BYTES = 128;            // of contraction values per step
constexpr uint32_t GL_OUTSIDE = 0x80000000u;  // an offset outside every descriptor

// What a workgroup reads: `base` is the tile's first row (row form) or its first column in the first contraction row (column form).
struct GroupedOperand {
    const char* base;
    uint32_t ld;     // bytes from row to row
    int valid;       // rows (row form) or columns (column form) that exist, from the tile's first one on
};

// DMA of one operand tile: EXTENT rows or columns of C, one step of contraction values.
template <typename T, int EXTENT, int WAVES, bool COLUMNS>
struct GroupedDma {
    static constexpr int E = sizeof(T), STEP = GL_STEP_BYTES / E, BYTES = EXTENT * GL_STEP_BYTES;
    static constexpr int LOADS = BYTES / 1024 / WAVES;  // load instructions per wave and step
    static_assert(LOADS >= 1 && LOADS * 1024 * WAVES == BYTES, "a tile splits evenly over the waves");
    static constexpr int ROW_BYTES = COLUMNS ? EXTENT * E : GL_STEP_BYTES, CHUNKS = ROW_BYTES / 16, ROWS = 1024 / ROW_BYTES;
    static_assert(ROW_BYTES <= 1024, "a load instruction fills whole rows");
    uint32_t voff[LOADS];
    const char* base;
    uint32_t ld, span;
    int lane_, wave_;

    __device__ static __forceinline__ int swizzle(int row) {
        if (!COLUMNS) return (row >> 1) & 7;
        return E == 4 || ROW_BYTES == 64 ? 0 : ROW_BYTES >= 256 ? (row & 3) << 2 : ((row >> 1) & 1) << 2;
    }
    __device__ __forceinline__ int row_of(int i) const { return (wave_ * LOADS + i) * ROWS + lane_ / CHUNKS; }
    __device__ __forceinline__ int chunk_of(int i) const { return (lane_ % CHUNKS) ^ swizzle(row_of(i)); }

    __device__ __forceinline__ void init(const GroupedOperand& o, int lane, int wave) {
        lane_ = lane;
        wave_ = wave;
        base = o.base;
        ld = o.ld;
        span = COLUMNS ? 0 : (uint32_t)(o.valid < EXTENT ? o.valid : EXTENT) * ld;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            int row = row_of(i), chunk = chunk_of(i);
            if (COLUMNS) chunk = chunk * (16 / E) < o.valid ? chunk : o.valid / (16 / E) - 1;
            else row = row < o.valid ? row : o.valid - 1;
            voff[i] = (uint32_t)row * ld + chunk * 16;
        }
    }
    // Step k: contraction values STEP k .. of which `left` exist.
    __device__ __forceinline__ void issue(int64_t k, int left, uint32_t lds) const {
        const uint32_t dst = __builtin_amdgcn_readfirstlane(lds + wave_ * (LOADS * 1024));
        const char* const from = base + (COLUMNS ? k * STEP * ld : k * GL_STEP_BYTES);
        const uint32_t bytes = COLUMNS ? (uint32_t)(left < STEP ? left : STEP) * ld : span;
        u32x4 rsrc = make_rsrc_words(from, bytes);
#pragma unroll
        for (int i = 0; i < 4; ++i) rsrc[i] = __builtin_amdgcn_readfirstlane(rsrc[i]);
        if (COLUMNS || left >= STEP) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) load_to_lds_b128(rsrc, voff[i], 0, dst + i * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) load_to_lds_b128(rsrc, chunk_of(i) * (16 / E) < left ? voff[i] : GL_OUTSIDE, 0, dst + i * 1024);
        }
    }
};

// Fragments of an operand tile for a wave whose rows (columns) of C start at `first` (a multiple of 32): 16 bytes of contraction values per
// lane.
template <typename T> struct GroupedFragOf { typedef bf16x8 type; };
template <> struct GroupedFragOf<float> { typedef f32x4 type; };
template <typename T, int EXTENT, bool COLUMNS>
struct GroupedFrag {
    typedef typename GroupedFragOf<T>::type Frag;
    static constexpr int E = sizeof(T), ROW_BYTES = COLUMNS ? EXTENT * E : GL_STEP_BYTES;
    int at[2];
    __device__ __forceinline__ void init(int lane, int first) {
        const int g = lane >> 5;
        at[1] = 0;
        if constexpr (COLUMNS && E == 2) {
            const int s16 = lane & 15, hi16 = (lane >> 4) & 1;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int row = 8 * g + 4 * half + (s16 >> 2), x = ROW_BYTES >= 256 ? row & 3 : ROW_BYTES == 128 ? (row >> 1) & 1 : 0;
                at[half] = row * ROW_BYTES + (((first / 32) ^ x) << 6) + (16 * hi16 + 4 * (s16 & 3)) * 2;
            }
        } else if constexpr (COLUMNS) {
            at[0] = 4 * g * ROW_BYTES + (first + (lane & 31)) * 4;
        } else {
            const int row = first + (lane & 31);
            at[0] = row * ROW_BYTES + ((g ^ ((row >> 1) & 7)) << 4);
        }
    }
    // Chunk 2 c + g of the step's contraction values, of the lane's row (column) in block b of 32
    __device__ __forceinline__ Frag read(const char* tile, int b, int c) const {
        if constexpr (COLUMNS && E == 2) {
            const char* const rows = tile + c * 16 * ROW_BYTES;
            return tr_pair(rows + (at[0] ^ (b << 6)), rows + (at[1] ^ (b << 6)));
        } else if constexpr (COLUMNS) {
            const char* const rows = tile + c * 8 * ROW_BYTES + at[0] + b * 128;
            Frag f;
#pragma unroll
            for (int t = 0; t < 4; ++t) f[t] = *(const float*)(rows + t * ROW_BYTES);
            return f;
        } else {
            return *(const Frag*)(tile + b * 32 * ROW_BYTES + (at[0] ^ (c << 5)));
        }
    }
};
__device__ __forceinline__ f32x16 grouped_mfma(bf16x8 a, bf16x8 b, f32x16 c) { return mfma32(a, b, c); }
__device__ __forceinline__ f32x16 grouped_mfma(f32x4 a, f32x4 b, f32x16 c) {
#pragma unroll
    for (int t = 0; t < 4; ++t) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[t], b[t], c, 0, 0, 0);
    return c;
}

template <int BM_, int BN_, int WM_, int WN_, int STAGES_>
struct GroupedShape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_;
    static constexpr int WAVES = WM * WN, THREADS = WAVES * 64, PER_CU = 8 / WAVES;  // two waves per SIMD
    static constexpr int MB = BM / WM / 32, NB = BN / WN / 32;  // 32 x 32 blocks of a wave
    static constexpr int A_BYTES = BM * GL_STEP_BYTES, STAGE = A_BYTES + BN * GL_STEP_BYTES;
    static constexpr int OUT_ROW = NB * 32 * 4 + 16, OUT = WAVES * 32 * OUT_ROW;  // 32 rows of a wave at a time, padded, room for fp32
    static constexpr int LDS = STAGES * STAGE > OUT ? STAGES * STAGE : OUT;
};

// acc[nb][mb] += the product of one step
template <typename S, typename T, typename FragA, typename FragB>
__device__ __forceinline__ void grouped_step(f32x16 (&acc)[S::NB][S::MB], const char* ta, const char* tb, const FragA& frag_a, const FragB& frag_b) {
#pragma unroll
    for (int c = 0; c < GL_STEP_BYTES / 32; ++c) {
        typename GroupedFragOf<T>::type fa[S::MB], fb[S::NB];
#pragma unroll
        for (int mb = 0; mb < S::MB; ++mb) fa[mb] = frag_a.read(ta, mb, c);
#pragma unroll
        for (int nb = 0; nb < S::NB; ++nb) fb[nb] = frag_b.read(tb, nb, c);
#pragma unroll
        for (int nb = 0; nb < S::NB; ++nb)
#pragma unroll
            for (int mb = 0; mb < S::MB; ++mb) acc[nb][mb] = grouped_mfma(fb[nb], fa[mb], acc[nb][mb]);
    }
}

// acc[nb][mb] += the tile's product over `length` contraction values.
template <typename S, typename T, bool A_COLUMNS, bool B_COLUMNS>
__device__ __forceinline__ void grouped_product(f32x16 (&acc)[S::NB][S::MB], char* lds, const GroupedOperand& a, const GroupedOperand& b, int length,
                                                int lane, int wave) {
    GroupedDma<T, S::BM, S::WAVES, A_COLUMNS> dma_a;
    GroupedDma<T, S::BN, S::WAVES, B_COLUMNS> dma_b;
    dma_a.init(a, lane, wave);
    dma_b.init(b, lane, wave);
    GroupedFrag<T, S::BM, A_COLUMNS> frag_a;
    GroupedFrag<T, S::BN, B_COLUMNS> frag_b;
    const int row0 = wave / S::WN * (S::BM / S::WM), col0 = wave % S::WN * (S::BN / S::WN);
    frag_a.init(lane, row0);
    frag_b.init(lane, col0);
    // Whether any of the wave's rows and columns exist (asked for Small tiles only: 9973 rows, 328 -> 200, fp32: 27 -> 23 us; the branch costs
    // the larger ones up to 7 % and leaves little out)
    const bool live = S::BM > 64 || (row0 < a.valid && col0 < b.valid);
    constexpr int LOADS = decltype(dma_a)::LOADS + decltype(dma_b)::LOADS;
    constexpr int STEP = decltype(dma_a)::STEP;
    const int steps = (length + STEP - 1) / STEP;
    const uint32_t lds0 = lds_address(lds);
    auto issue = [&](int k, int stage) {
        const int left = length - k * STEP;
        dma_a.issue(k, left, lds0 + stage * S::STAGE);
        dma_b.issue(k, left, lds0 + stage * S::STAGE + S::A_BYTES);
    };
#pragma unroll
    for (int k = 0; k < S::STAGES - 1; ++k)
        if (k < steps) issue(k, k);
    int stage = 0;
    for (int k = 0; k < steps; ++k) {
        if (k + S::STAGES - 2 < steps) wait_vmcnt<(S::STAGES - 2) * LOADS>();
        else wait_vmcnt<0>();
        __syncthreads();  // step k has arrived; every wave is done with the stage of step k - 1
        if (k + S::STAGES - 1 < steps) issue(k + S::STAGES - 1, stage == 0 ? S::STAGES - 1 : stage - 1);
        const char* ta = lds + stage * S::STAGE;
        stage = stage == S::STAGES - 1 ? 0 : stage + 1;
        if (live) grouped_step<S, T>(acc, ta, ta + S::A_BYTES, frag_a, frag_b);
    }
    __syncthreads();  // every wave is done with the ring: it stages the output next
}

// The tile as rows of T (bf16 or fp32): rows < `rows`, columns < `columns`, from `out` on with `ld` values per row.  32 rows of a wave at a
// time through its own part of LDS, so that whole pieces of rows go out.
template <typename S, typename T>
__device__ __forceinline__ void grouped_store(const f32x16 (&acc)[S::NB][S::MB], char* lds, T* out, int64_t ld, int rows, int columns, int lane,
                                              int wave) {
    constexpr int E = sizeof(T), PIECES = S::NB * 32 * E / 16, PER_PASS = 64 / PIECES;
    const int r = lane & 31, g = lane >> 5;
    const int row0 = wave / S::WN * (S::BM / S::WM), col0 = wave % S::WN * (S::BN / S::WN);
    char* const mine = lds + wave * (32 * S::OUT_ROW);
#pragma unroll
    for (int mb = 0; mb < S::MB; ++mb) {
#pragma unroll
        for (int nb = 0; nb < S::NB; ++nb)
#pragma unroll
            for (int vg = 0; vg < 4; ++vg) {
                typedef __attribute__((ext_vector_type(4))) T T4;
                T4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = (T)acc[nb][mb][4 * vg + e];
                *(T4*)(mine + r * S::OUT_ROW + (32 * nb + 8 * vg + 4 * g) * E) = o;
            }
#pragma unroll
        for (int i = 0; i < 32 / PER_PASS; ++i) {
            const int row = i * PER_PASS + lane / PIECES, piece = lane % PIECES;
            const u32x4 v = *(const u32x4*)(mine + row * S::OUT_ROW + piece * 16);
            const int m = row0 + 32 * mb + row, n = col0 + piece * (16 / E);
            if (m < rows && n < columns) __builtin_nontemporal_store(v, (u32x4*)(out + (int64_t)m * ld + n));
        }
    }
}

// The same for bf16 tiles of waves of 64 columns, through 4 KB of LDS per wave that are no part of the ring: rows of 128 bytes whose
// 16-byte chunk ^= (row / 2) % 8 instead of padding.
template <typename S>
__device__ __forceinline__ void grouped_store_beside(const f32x16 (&acc)[S::NB][S::MB], char* mine, bf16_t* out, int64_t ld, int rows, int columns,
                                                     int lane, int wave) {
    static_assert(S::NB == 2, "a wave's rows are 128 bytes");
    const int r = lane & 31, g = lane >> 5;
    const int row0 = wave / S::WN * (S::BM / S::WM), col0 = wave % S::WN * (S::BN / S::WN);
#pragma unroll
    for (int mb = 0; mb < S::MB; ++mb) {
#pragma unroll
        for (int nb = 0; nb < S::NB; ++nb)
#pragma unroll
            for (int vg = 0; vg < 4; ++vg) {
                bf16x4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = (bf16_t)acc[nb][mb][4 * vg + e];
                *(bf16x4*)(mine + r * 128 + (((4 * nb + vg) ^ ((r >> 1) & 7)) << 4) + g * 8) = o;
            }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = i * 8 + lane / 8, piece = lane % 8;
            const u32x4 v = *(const u32x4*)(mine + row * 128 + ((piece ^ ((row >> 1) & 7)) << 4));
            const int m = row0 + 32 * mb + row, n = col0 + piece * 8;
            if (m < rows && n < columns) *(u32x4*)(out + (int64_t)m * ld + n) = v;
        }
    }
}

}  // namespace kunlun
