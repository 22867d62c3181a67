// C-ABI entry points of the operators around the layer: argument checks and launches.
#include <cmath>
#include <initializer_list>

#include "bigmac.h"
#include "internal.h"
#include "mx4.h"
#include "residual_norm.h"

using namespace bigmac;

static __device__ int g_operator_status;

namespace {

inline bool is_aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
inline bool dtype_ok(int32_t dtype) { return dtype == BIGMAC_F32 || dtype == BIGMAC_BF16; }
inline int64_t esize_of(int32_t dtype) { return dtype == BIGMAC_BF16 ? 2 : 4; }

// Device address of the status word, resolved once per device.
int* status_word() {
    static int* cached[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
    if (!cached[dev]) {
        void* p = nullptr;
        if (cudaGetSymbolAddress(&p, g_operator_status) != cudaSuccess) { cudaGetLastError(); return nullptr; }
        cached[dev] = (int*)p;
    }
    return cached[dev];
}

int check_mx4(const bigmac_mx4_t* q, bool stacked_allowed) {
    if (!q || q->rows < 0 || q->K <= 0 || q->E < 0 || q->E > kMaxExperts || (q->offsets && q->E == 0)) return BIGMAC_ERR_INVALID_ARG;
    if (q->K % 32 != 0 || q->K > (1 << 20)) return BIGMAC_ERR_UNSUPPORTED;
    if (q->E > 0 && !q->offsets && !stacked_allowed) return BIGMAC_ERR_INVALID_ARG;
    if (!is_aligned(q->codes, 16) || !is_aligned(q->scales, 16) || !is_aligned(q->offsets, 4)) return BIGMAC_ERR_INVALID_ARG;
    const int64_t rows = q->offsets ? mx4_padded_rows(q->rows, q->E) : (int64_t)q->rows * (q->E > 0 ? q->E : 1);
    if (rows > (int64_t)0x7fffff00) return BIGMAC_ERR_UNSUPPORTED;       // row numbers are 32-bit
    if (rows > 0 && (!q->codes || !q->scales)) return BIGMAC_ERR_INVALID_ARG;
    return BIGMAC_OK;
}
Mx4View view_of(const bigmac_mx4_t* q) {
    const int64_t capacity = q->offsets ? mx4_padded_rows(q->rows, q->E) : q->rows;
    return Mx4View{(uint8_t*)q->codes, (uint8_t*)q->scales, q->rows, q->K, q->E, q->offsets, capacity};
}

// No two sums in one place (the gradients of a vector that both norms share need two).
bool apart(std::initializer_list<const void*> sums) {
    for (auto a = sums.begin(); a != sums.end(); ++a)
        for (auto b = a + 1; b != sums.end(); ++b)
            if (*a && *a == *b) return false;
    return true;
}
// A matrix of the joint: aligned to its elements, rows that do not overlap.  *vec: rows on 16-byte boundaries, too.
bool rows_ok(const bigmac_rows_t& m, int64_t d, int64_t es, bool* vec) {
    if (!m.p) return true;
    if (!is_aligned(m.p, es) || m.ld < d || m.ld > 0x7fffffff) return false;
    if (!is_aligned(m.p, 16) || (m.ld * es) % 16) *vec = false;
    return true;
}
bool vector_ok(const void* p, bool* vec) {
    if (!is_aligned(p, 4)) return false;
    if (!is_aligned(p, 16)) *vec = false;
    return true;
}

int check_residual_norm(const bigmac_residual_norm_t* q, int32_t T, bool backward, ResNorm* a) {
    if (!q || T < 0 || q->d <= 0 || !dtype_ok(q->dtype) || q->post_kind < 0 || q->post_kind > BIGMAC_NORM_LAYER || q->pre_kind < 0 ||
        q->pre_kind > BIGMAC_NORM_LAYER || q->gate_kind < 0 || q->gate_kind > BIGMAC_GATE_FULL)
        return BIGMAC_ERR_INVALID_ARG;
    if (!(q->post_eps >= 0) || !(q->pre_eps >= 0) || !std::isfinite(q->post_eps) || !std::isfinite(q->pre_eps) || !std::isfinite(q->residual_scale))
        return BIGMAC_ERR_INVALID_ARG;
    if (q->d > kResNormMaxWidth || T > kResNormMaxRows) return BIGMAC_ERR_UNSUPPORTED;
    const int64_t es = esize_of(q->dtype);
    *a = ResNorm{q, T, q->d % 8 == 0};
    bool ok = rows_ok(q->x, q->d, es, &a->vec) && rows_ok(q->y, q->d, es, &a->vec) && vector_ok(q->w_post, &a->vec) && vector_ok(q->b_post, &a->vec) &&
              vector_ok(q->w_pre, &a->vec) && vector_ok(q->b_pre, &a->vec) && is_aligned(q->stats, 16);
    ok = ok && (q->gate_kind == BIGMAC_GATE_FULL ? rows_ok(q->gate, q->d, es, &a->vec) : vector_ok(q->gate.p, &a->vec));
    if (!ok) return BIGMAC_ERR_INVALID_ARG;
    if (q->pre_kind == BIGMAC_NORM_NONE && (q->w_pre || q->b_pre)) return BIGMAC_ERR_INVALID_ARG;
    if (q->gate_kind == BIGMAC_GATE_NONE && (q->gate.p || q->dgate.p)) return BIGMAC_ERR_INVALID_ARG;
    if (T == 0) return BIGMAC_OK;                                      // matrices without rows have no address
    if (q->gate_kind != BIGMAC_GATE_NONE && !q->gate.p) return BIGMAC_ERR_INVALID_ARG;
    // the norm, the gate and the parameters of an output that is not there, parameters of a norm that is not
    if (!q->y.p && (q->post_kind != BIGMAC_NORM_NONE || q->gate.p || q->w_post || q->b_post)) return BIGMAC_ERR_INVALID_ARG;
    if (!q->x.p) return BIGMAC_ERR_INVALID_ARG;
    if (!backward) {
        if (!rows_ok(q->r, q->d, es, &a->vec) || !rows_ok(q->n, q->d, es, &a->vec)) return BIGMAC_ERR_INVALID_ARG;
        return (q->pre_kind == BIGMAC_NORM_NONE) == (q->n.p == nullptr) ? BIGMAC_OK : BIGMAC_ERR_INVALID_ARG;
    }
    ok = rows_ok(q->dr, q->d, es, &a->vec) && rows_ok(q->dn, q->d, es, &a->vec) && rows_ok(q->dx, q->d, es, &a->vec) && rows_ok(q->dy, q->d, es, &a->vec);
    ok = ok && (q->gate_kind == BIGMAC_GATE_FULL ? rows_ok(q->dgate, q->d, es, &a->vec) : is_aligned(q->dgate.p, 4));
    ok = ok && is_aligned(q->dw_post, 4) && is_aligned(q->db_post, 4) && is_aligned(q->dw_pre, 4) && is_aligned(q->db_pre, 4);
    if (!ok || (!q->y.p && q->dy.p) || (q->pre_kind == BIGMAC_NORM_NONE && q->dn.p))
        return BIGMAC_ERR_INVALID_ARG;
    if (!q->stats || (!q->dr.p && !q->dn.p)) return BIGMAC_ERR_INVALID_ARG;
    if (!apart({q->dw_post, q->db_post, q->dw_pre, q->db_pre, q->dgate.p})) return BIGMAC_ERR_INVALID_ARG;
    return BIGMAC_OK;
}
size_t residual_norm_scratch(const bigmac_residual_norm_t* q, int32_t T) {
    const bool any = q->dw_post || q->db_post || q->dw_pre || q->db_pre || (q->gate_kind == BIGMAC_GATE_CHANNEL && q->dgate.p);
    return any && T > 0 ? (size_t)residual_norm_parts(T, q->d) * 4 * q->d * sizeof(float) : 0;
}

}  // namespace

extern "C" {

int bigmac_residual_norm_forward(const bigmac_residual_norm_t* q, int32_t T, void* stream) {
    ResNorm a;
    const int s = check_residual_norm(q, T, false, &a);
    if (s != BIGMAC_OK) return s;
    return launch_residual_norm_forward(a, (cudaStream_t)stream) == cudaSuccess ? BIGMAC_OK : BIGMAC_ERR_CUDA;
}

int bigmac_residual_norm_scratch_bytes(const bigmac_residual_norm_t* q, int32_t T, size_t* scratch_bytes) {
    if (!q || !scratch_bytes || T < 0 || q->d <= 0) return BIGMAC_ERR_INVALID_ARG;
    if (q->d > kResNormMaxWidth) return BIGMAC_ERR_UNSUPPORTED;
    *scratch_bytes = residual_norm_scratch(q, T);
    return BIGMAC_OK;
}

int bigmac_residual_norm_backward(const bigmac_residual_norm_t* q, int32_t T, int accumulate, void* scratch, size_t scratch_bytes, void* stream) {
    ResNorm a;
    const int s = check_residual_norm(q, T, true, &a);
    if (s != BIGMAC_OK) return s;
    const size_t need = residual_norm_scratch(q, T);
    if (need && (!scratch || !is_aligned(scratch, 16))) return BIGMAC_ERR_INVALID_ARG;
    if (scratch_bytes < need) return BIGMAC_ERR_WORKSPACE;
    return launch_residual_norm_backward(a, (float*)scratch, accumulate, (cudaStream_t)stream) == cudaSuccess ? BIGMAC_OK : BIGMAC_ERR_CUDA;
}

int bigmac_operator_status(void* stream) {
    int* at = status_word();
    if (!at) return BIGMAC_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)stream;
    int word = 0;
    if (cudaMemcpyAsync(&word, at, sizeof(int), cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaMemsetAsync(at, 0, sizeof(int), st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)
        return BIGMAC_ERR_CUDA;
    return word == 0 ? BIGMAC_OK : BIGMAC_ERR_TIMEOUT;
}

int bigmac_mx4_bytes(int32_t rows, int32_t K, int32_t E, int grouped, size_t* code_bytes, size_t* scale_bytes) {
    if (rows < 0 || K <= 0 || E < 0 || E > kMaxExperts || (grouped && E == 0) || !code_bytes || !scale_bytes) return BIGMAC_ERR_INVALID_ARG;
    if (K % 32 != 0 || K > (1 << 20)) return BIGMAC_ERR_UNSUPPORTED;
    const int64_t one = grouped ? mx4_padded_rows(rows, E) : rows, many = grouped || E == 0 ? 1 : E;
    *code_bytes = (size_t)(one * many) * (K / 2);
    *scale_bytes = (size_t)((one + kMx4Tile - 1) / kMx4Tile * many) * mx4_ktiles(K) * 512;
    return BIGMAC_OK;
}

int bigmac_mx4_quantize(const void* x, int32_t dtype, int32_t x_rows, int64_t ld, const int32_t* slot_of_row, int32_t k, const bigmac_mx4_t* out,
                        void* stream) {
    const int s = check_mx4(out, false);
    if (s != BIGMAC_OK) return s;
    if (!dtype_ok(dtype) || x_rows < 0 || ld < out->K || (ld * esize_of(dtype)) % 16 || !is_aligned(x, 16) || !is_aligned(slot_of_row, 4) ||
        (slot_of_row ? k < 1 : x_rows != out->rows) || (x_rows > 0 && !x))
        return BIGMAC_ERR_INVALID_ARG;
    if (ld > 0x7fffffff) return BIGMAC_ERR_UNSUPPORTED;
    return launch_mx4_quantize(x, dtype, ld, slot_of_row, k, x_rows, view_of(out), (cudaStream_t)stream) == cudaSuccess ? BIGMAC_OK : BIGMAC_ERR_CUDA;
}

int bigmac_mx4_dequantize(const bigmac_mx4_t* q, void* y, int32_t dtype, int64_t ld, void* stream) {
    const int s = check_mx4(q, false);
    if (s != BIGMAC_OK) return s;
    if (!dtype_ok(dtype) || ld < q->K || (ld * esize_of(dtype)) % 16 || !is_aligned(y, 16) || (q->rows > 0 && !y)) return BIGMAC_ERR_INVALID_ARG;
    if (ld > 0x7fffffff) return BIGMAC_ERR_UNSUPPORTED;
    return launch_mx4_dequantize(view_of(q), y, dtype, ld, (cudaStream_t)stream) == cudaSuccess ? BIGMAC_OK : BIGMAC_ERR_CUDA;
}

int bigmac_mx4_matmul(const bigmac_mx4_t* a, const bigmac_mx4_t* w, int32_t act, int32_t dtype, void* c, int64_t ldc, void* stream) {
    int s = check_mx4(a, false);
    if (s == BIGMAC_OK) s = check_mx4(w, true);
    if (s != BIGMAC_OK) return s;
    if (!dtype_ok(dtype) || act < 0 || act > BIGMAC_ACT_IDENTITY || w->offsets || a->K != w->K || a->E != w->E || ldc < w->rows || !is_aligned(c, 16))
        return BIGMAC_ERR_INVALID_ARG;
    if (a->rows == 0 || w->rows == 0) return BIGMAC_OK;
    if (!c) return BIGMAC_ERR_INVALID_ARG;
    int* status = status_word();
    if (!status) return BIGMAC_ERR_CUDA;
    return launch_mx4_matmul(view_of(a), view_of(w), act, dtype, c, ldc, nullptr, status, (cudaStream_t)stream) == cudaSuccess ? BIGMAC_OK : BIGMAC_ERR_CUDA;
}

int bigmac_mx4_matmul_mx4(const bigmac_mx4_t* a, const bigmac_mx4_t* w, int32_t act, const bigmac_mx4_t* out, void* stream) {
    int s = check_mx4(a, false);
    if (s == BIGMAC_OK) s = check_mx4(w, true);
    if (s == BIGMAC_OK) s = check_mx4(out, false);
    if (s != BIGMAC_OK) return s;
    if (act < 0 || act > BIGMAC_ACT_IDENTITY || w->offsets || a->K != w->K || a->E != w->E || out->rows != a->rows || out->K != w->rows ||
        out->E != a->E || out->offsets != a->offsets)
        return BIGMAC_ERR_INVALID_ARG;
    if (a->rows == 0) return BIGMAC_OK;
    if (out->codes == a->codes || out->scales == a->scales) return BIGMAC_ERR_INVALID_ARG;
    int* status = status_word();
    if (!status) return BIGMAC_ERR_CUDA;
    const Mx4View to = view_of(out);
    return launch_mx4_matmul(view_of(a), view_of(w), act, 0, nullptr, 0, &to, status, (cudaStream_t)stream) == cudaSuccess ? BIGMAC_OK : BIGMAC_ERR_CUDA;
}

}  // extern "C"
