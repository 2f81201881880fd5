// C ABI of the operators in front of attention (include/kunlun_layers.h): argument validation on the host, then the launchers.
#include <cmath>

#include "layers.h"

using namespace kunlun;

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t value_bytes(int dtype) { return dtype == KUNLUN_FP32 ? 4 : 2; }
constexpr int64_t ROWS_END = (int64_t)1 << 31;  // positions and offsets are 32-bit

int check_rows(int64_t rows, int D, int dtype) {
    if (rows < 0 || rows >= ROWS_END || D < 1) return KUNLUN_ERR_SHAPE;
    if (D > KUNLUN_MAX_CHANNELS || (dtype != KUNLUN_BF16 && dtype != KUNLUN_FP32)) return KUNLUN_ERR_UNSUPPORTED;
    return KUNLUN_OK;
}

int check_embedding(int64_t n, int64_t rows, int D, float scale, int id_bytes, int dtype) {
    const int rc = check_rows(rows, D, dtype);
    if (rc != KUNLUN_OK) return rc;
    if (n < 0 || n >= ROWS_END) return KUNLUN_ERR_SHAPE;
    if ((id_bytes != 4 && id_bytes != 8) || !std::isfinite(scale)) return KUNLUN_ERR_UNSUPPORTED;
    return KUNLUN_OK;
}

int check_grouped(int G, int64_t total, int K, int N, int dtype) {
    if (G < 1 || total < 0 || total >= ROWS_END || K < 1 || N < 1) return KUNLUN_ERR_SHAPE;
    if (dtype != KUNLUN_BF16 && dtype != KUNLUN_FP32) return KUNLUN_ERR_UNSUPPORTED;
    const int piece = dtype == KUNLUN_FP32 ? 4 : 8;
    if (G > KUNLUN_MAX_GROUPS || K > KUNLUN_MAX_CHANNELS || N > KUNLUN_MAX_CHANNELS || K % piece != 0 || N % piece != 0)
        return KUNLUN_ERR_UNSUPPORTED;
    return KUNLUN_OK;
}

int check_workspace(const void* workspace, size_t given, size_t need) {
    if (!workspace || given < need) return KUNLUN_ERR_WORKSPACE;
    return aligned(workspace, 256) ? KUNLUN_OK : KUNLUN_ERR_ALIGN;
}

int status(hipError_t e) { return e == hipSuccess ? KUNLUN_OK : KUNLUN_ERR_LAUNCH; }

}  // namespace

extern "C" {

int kunlun_embedding_fwd(const void* table, const void* ids, void* out, int64_t n, int64_t rows, int D, float scale, int id_bytes,
                         int dtype, void* stream) {
    const int rc = check_embedding(n, rows, D, scale, id_bytes, dtype);
    if (rc != KUNLUN_OK) return rc;
    if (n == 0) return KUNLUN_OK;
    if (!ids || !out || (rows > 0 && !table)) return KUNLUN_ERR_NULL;
    const size_t e = value_bytes(dtype);
    if (!aligned(table, e) || !aligned(out, e) || !aligned(ids, id_bytes)) return KUNLUN_ERR_ALIGN;
    return status(launch_embedding_fwd(table, ids, out, n, rows, D, scale, id_bytes, dtype, (hipStream_t)stream));
}

size_t kunlun_embedding_bwd_workspace_bytes(int64_t n, int64_t rows, int D, int dtype) {
    if (check_embedding(n, rows, D, 1.f, 4, dtype) != KUNLUN_OK) return 0;
    return embedding_bwd_workspace(n, D, dtype);
}

int kunlun_embedding_bwd(const void* d_out, const void* ids, void* d_table, int64_t n, int64_t rows, int D, float scale, int id_bytes,
                         int dtype, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_embedding(n, rows, D, scale, id_bytes, dtype);
    if (rc != KUNLUN_OK) return rc;
    if (rows == 0) return KUNLUN_OK;
    if (!d_table || (n > 0 && (!d_out || !ids))) return KUNLUN_ERR_NULL;
    const size_t e = value_bytes(dtype);
    if (!aligned(d_out, e) || !aligned(d_table, e) || !aligned(ids, id_bytes)) return KUNLUN_ERR_ALIGN;
    rc = check_workspace(workspace, workspace_bytes, embedding_bwd_workspace(n, D, dtype));
    if (rc != KUNLUN_OK) return rc;
    return status(launch_embedding_bwd(d_out, ids, d_table, n, rows, D, scale, id_bytes, dtype, workspace, (hipStream_t)stream));
}

int kunlun_layer_norm_fwd(const void* x, const void* weight, const void* bias, void* y, float* mean, float* rstd, int64_t rows, int D,
                          float eps, int dtype, void* stream) {
    const int rc = check_rows(rows, D, dtype);
    if (rc != KUNLUN_OK) return rc;
    if (!std::isfinite(eps) || eps < 0.f) return KUNLUN_ERR_UNSUPPORTED;
    if (rows == 0) return KUNLUN_OK;
    if (!x || !y) return KUNLUN_ERR_NULL;
    const size_t e = value_bytes(dtype);
    if (!aligned(x, e) || !aligned(y, e) || !aligned(weight, e) || !aligned(bias, e) || !aligned(mean, 4) || !aligned(rstd, 4))
        return KUNLUN_ERR_ALIGN;
    return status(launch_layer_norm_fwd(x, weight, bias, y, mean, rstd, rows, D, eps, dtype, (hipStream_t)stream));
}

size_t kunlun_layer_norm_bwd_workspace_bytes(int64_t rows, int D, int dtype) {
    return check_rows(rows, D, dtype) == KUNLUN_OK ? layer_norm_bwd_workspace(rows, D, dtype) : 0;
}

int kunlun_layer_norm_bwd(const void* x, const void* weight, const void* dy, const float* mean, const float* rstd, void* dx, void* dw,
                          void* db, int64_t rows, int D, int dtype, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_rows(rows, D, dtype);
    if (rc != KUNLUN_OK) return rc;
    if (!dx && !dw && !db) return KUNLUN_OK;
    if (rows == 0 && !dw && !db) return KUNLUN_OK;
    if (rows > 0 && (!x || !dy || !mean || !rstd)) return KUNLUN_ERR_NULL;
    const size_t e = value_bytes(dtype);
    if (!aligned(x, e) || !aligned(weight, e) || !aligned(dy, e) || !aligned(dx, e) || !aligned(dw, e) || !aligned(db, e) ||
        !aligned(mean, 4) || !aligned(rstd, 4))
        return KUNLUN_ERR_ALIGN;
    if (dw || db) {
        rc = check_workspace(workspace, workspace_bytes, layer_norm_bwd_workspace(rows, D, dtype));
        if (rc != KUNLUN_OK) return rc;
    }
    return status(launch_layer_norm_bwd(x, weight, dy, mean, rstd, dx, dw, db, rows, D, dtype, workspace, (hipStream_t)stream));
}

int kunlun_grouped_linear_fwd(const void* x, const void* w, void* y, const int32_t* offsets, int G, int64_t total, int K, int N,
                              int fill_rest, int dtype, void* stream) {
    const int rc = check_grouped(G, total, K, N, dtype);
    if (rc != KUNLUN_OK) return rc;
    if (total == 0) return KUNLUN_OK;
    if (!x || !w || !y || !offsets) return KUNLUN_ERR_NULL;
    if (!aligned(x, 16) || !aligned(w, 16) || !aligned(y, 16) || !aligned(offsets, 4)) return KUNLUN_ERR_ALIGN;
    return status(launch_grouped_linear_fwd(x, w, y, offsets, G, total, K, N, fill_rest != 0, dtype, (hipStream_t)stream));
}

size_t kunlun_grouped_linear_bwd_workspace_bytes(int G, int64_t total, int K, int N, int dtype) {
    return check_grouped(G, total, K, N, dtype) == KUNLUN_OK ? grouped_linear_bwd_workspace(G, total, K, N, dtype) : 0;
}

int kunlun_grouped_linear_bwd(const void* x, const void* w, const void* dy, void* dx, void* dw, const int32_t* offsets, int G,
                              int64_t total, int K, int N, int fill_rest, int dtype, void* workspace, size_t workspace_bytes,
                              void* stream) {
    int rc = check_grouped(G, total, K, N, dtype);
    if (rc != KUNLUN_OK) return rc;
    if (!dx && !dw) return KUNLUN_OK;
    if (total == 0 && !dw) return KUNLUN_OK;
    if (!offsets) return KUNLUN_ERR_NULL;
    if (total > 0 && (!dy || (dx && !w) || (dw && !x))) return KUNLUN_ERR_NULL;
    if (!aligned(x, 16) || !aligned(w, 16) || !aligned(dy, 16) || !aligned(dx, 16) || !aligned(dw, 16) || !aligned(offsets, 4))
        return KUNLUN_ERR_ALIGN;
    if (dw) {
        rc = check_workspace(workspace, workspace_bytes, grouped_linear_bwd_workspace(G, total, K, N, dtype));
        if (rc != KUNLUN_OK) return rc;
    }
    return status(launch_grouped_linear_bwd(x, w, dy, dx, dw, offsets, G, total, K, N, fill_rest != 0, dtype, workspace, (hipStream_t)stream));
}

}  // extern "C"
