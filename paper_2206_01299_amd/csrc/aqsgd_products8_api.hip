// C entries of the 8-bit operators: argument checks (the contract is in include/aqsgd.h).
#include "aqsgd_products8.h"

namespace aqsgd {
namespace {

constexpr int64_t kMaxSide = int64_t{1} << 30;      // rows and columns: their numbers are 32-bit in the kernels

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool known_dtype(int dtype) { return dtype == AQSGD_F32 || dtype == AQSGD_F16 || dtype == AQSGD_BF16; }
uintptr_t elem_bytes(int dtype) { return dtype == AQSGD_F32 ? 4 : 2; }
bool side(int64_t n) { return n >= 0 && n <= kMaxSide; }

// Workgroups of the smallest tile, and bytes of the widest matrix, stay countable.
bool countable(int64_t m, int64_t n) { return ((m + 63) / 64) * ((n + 63) / 64) < (int64_t{1} << 31) - 1; }

int check_quant8(const aqsgd_quant8_desc* d) {
    if (!d) return AQSGD_ERR_NULL;
    if (!known_dtype(d->dtype)) return AQSGD_ERR_DTYPE;
    if (d->rounding != AQSGD_ROUND_NEAREST && d->rounding != AQSGD_ROUND_STOCHASTIC) return AQSGD_ERR_DTYPE;
    if (!side(d->rows) || !side(d->cols) || d->ld < d->cols || d->ld > (int64_t{1} << 40) || !countable(d->rows, d->cols) ||
        (d->rows > 0 && d->ld > (int64_t{1} << 60) / d->rows))
        return AQSGD_ERR_SHAPE;
    return AQSGD_OK;
}

int check_matmul8(const aqsgd_matmul8_desc* d) {
    if (!d) return AQSGD_ERR_NULL;
    if (!known_dtype(d->dtype)) return AQSGD_ERR_DTYPE;
    if (d->message != 0 && d->message != 1) return AQSGD_ERR_DTYPE;
    if (!side(d->m) || !side(d->n) || d->k < 0 || d->k > kMaxSumLength || !countable(d->m, d->n)) return AQSGD_ERR_SHAPE;
    if (d->message && d->k % 16 != 0) return AQSGD_ERR_GROUP;
    return AQSGD_OK;
}

int check_ffn8(const aqsgd_ffn8_desc* d) {
    if (!d) return AQSGD_ERR_NULL;
    if (!known_dtype(d->dtype) || d->act < AQSGD_ACT_SILU || d->act > AQSGD_ACT_GELU_TANH) return AQSGD_ERR_DTYPE;
    if ((d->gated != 0 && d->gated != 1) || d->reserved != 0) return AQSGD_ERR_DTYPE;
    if (!side(d->m) || !side(d->f)) return AQSGD_ERR_SHAPE;
    const int64_t w = d->f * (d->gated ? 2 : 1);
    if (!side(w) || d->k < 0 || d->k > kMaxSumLength || !countable(d->m, w)) return AQSGD_ERR_SHAPE;
    return AQSGD_OK;
}

int status(hipError_t err) { return err == hipSuccess ? AQSGD_OK : AQSGD_ERR_LAUNCH; }

}  // namespace
}  // namespace aqsgd

using namespace aqsgd;

extern "C" {

size_t aqsgd_quant8_stride(int64_t length) { return side(length) ? static_cast<size_t>(code_stride(length)) : 0; }

size_t aqsgd_quant8_workspace_bytes(const aqsgd_quant8_desc* d) {
    return check_quant8(d) == AQSGD_OK ? static_cast<size_t>(quant8_workspace_bytes(d->rows, d->cols)) : 0;
}

int aqsgd_quant8(const aqsgd_quant8_desc* d, const void* x, int8_t* row_codes, float* row_scales, int8_t* col_codes,
                 float* col_scales, float* col_sums, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_quant8(d);
    if (rc != AQSGD_OK) return rc;
    if (d->rows == 0 || d->cols == 0) {              // the other side's vectors are empty
        float* scales = d->rows ? row_scales : col_scales;
        float* sums = d->rows ? nullptr : col_sums;
        if (!aligned(scales, 4) || !aligned(sums, 4)) return AQSGD_ERR_ALIGN;
        if (d->rows + d->cols == 0 || (!scales && !sums)) return AQSGD_OK;
        return status(launch_quant8_empty(scales, sums, d->rows + d->cols, static_cast<hipStream_t>(stream)));
    }
    if (!x || !row_codes != !row_scales || !col_codes != !col_scales) return AQSGD_ERR_NULL;
    if (!aligned(x, elem_bytes(d->dtype)) || !aligned(row_codes, 16) || !aligned(row_scales, 4) || !aligned(col_codes, 16) ||
        !aligned(col_scales, 4) || !aligned(col_sums, 4))
        return AQSGD_ERR_ALIGN;
    if (!row_codes && !col_codes && !col_sums) return AQSGD_OK;
    if (col_codes || col_sums) {
        if (!workspace || workspace_bytes < aqsgd_quant8_workspace_bytes(d)) return AQSGD_ERR_WORKSPACE;
        if (!aligned(workspace, 16)) return AQSGD_ERR_ALIGN;
    }
    Quant8Args a;
    a.x = x;
    a.row_codes = row_codes; a.row_scales = row_scales;
    a.col_codes = col_codes; a.col_scales = col_scales; a.col_sums = col_sums;
    a.workspace = workspace;
    a.ld = d->ld; a.row_stride = code_stride(d->cols); a.col_stride = code_stride(d->rows);
    a.rows = d->rows; a.cols = d->cols;
    a.seed = d->rng_seed;
    return status(launch_quant8(d->dtype, d->rounding, a, static_cast<hipStream_t>(stream)));
}

size_t aqsgd_matmul8_workspace_bytes(const aqsgd_matmul8_desc* d) {
    if (check_matmul8(d) != AQSGD_OK) return 0;
    const ProductShape p{static_cast<int32_t>(d->m), static_cast<int32_t>(d->n), static_cast<int32_t>(d->k)};
    return static_cast<size_t>(product_workspace_bytes(d->message ? kMessage : kPlain, p));
}

int aqsgd_matmul8(const aqsgd_matmul8_desc* d, const void* a_codes, const float* a_scales, const int8_t* b_codes,
                  const float* b_scales, const void* bias, const void* add, void* out, void* workspace,
                  size_t workspace_bytes, void* stream) {
    const int rc = check_matmul8(d);
    if (rc != AQSGD_OK) return rc;
    if (d->m == 0 || d->n == 0) return AQSGD_OK;
    if ((d->k > 0 && (!a_codes || !b_codes)) || !a_scales || !b_scales || !out) return AQSGD_ERR_NULL;
    const uintptr_t e = elem_bytes(d->dtype);
    if (!aligned(a_codes, 16) || !aligned(b_codes, 16) || !aligned(a_scales, 4) || !aligned(b_scales, 4) || !aligned(bias, e) ||
        !aligned(add, e) || !aligned(out, e))
        return AQSGD_ERR_ALIGN;
    const size_t need = aqsgd_matmul8_workspace_bytes(d);
    if (need && (!workspace || workspace_bytes < need)) return AQSGD_ERR_WORKSPACE;
    if (need && !aligned(workspace, 16)) return AQSGD_ERR_ALIGN;
    ProductArgs p = {};
    p.a = static_cast<const uint8_t*>(a_codes); p.a_scales = a_scales;
    p.b = b_codes; p.b_scales = b_scales;
    p.bias = bias; p.add = add; p.out = out;
    p.lda = d->message ? d->k : code_stride(d->k);
    p.ldb = code_stride(d->k);
    p.m = static_cast<int32_t>(d->m); p.n = static_cast<int32_t>(d->n); p.k = static_cast<int32_t>(d->k);
    p.dtype = d->dtype;
    return status(launch_product(d->message ? kMessage : kPlain, p, workspace, static_cast<hipStream_t>(stream)));
}

int aqsgd_ffn8(const aqsgd_ffn8_desc* d, const int8_t* a_codes, const float* a_scales, const int8_t* w_codes,
               const float* w_scales, const void* bias, void* h, void* pre, void* stream) {
    const int rc = check_ffn8(d);
    if (rc != AQSGD_OK) return rc;
    if (d->m == 0 || d->f == 0) return AQSGD_OK;
    if ((d->k > 0 && (!a_codes || !w_codes)) || !a_scales || !w_scales || !h) return AQSGD_ERR_NULL;
    const uintptr_t e = elem_bytes(d->dtype);
    if (!aligned(a_codes, 16) || !aligned(w_codes, 16) || !aligned(a_scales, 4) || !aligned(w_scales, 4) || !aligned(bias, e) ||
        !aligned(h, e) || !aligned(pre, e))
        return AQSGD_ERR_ALIGN;
    ProductArgs p = {};
    p.a = reinterpret_cast<const uint8_t*>(a_codes); p.a_scales = a_scales;
    p.b = w_codes; p.b_scales = w_scales;
    p.bias = bias; p.out = h; p.pre = pre;
    p.lda = p.ldb = code_stride(d->k);
    p.m = static_cast<int32_t>(d->m); p.n = static_cast<int32_t>(d->f * (d->gated ? 2 : 1)); p.k = static_cast<int32_t>(d->k);
    p.dtype = d->dtype; p.act = d->act;
    return status(launch_product(d->gated ? kGated : kActivation, p, nullptr, static_cast<hipStream_t>(stream)));
}

int aqsgd_ffn8_grad(const aqsgd_ffn8_desc* d, const void* dh, const void* pre, void* dpre, void* stream) {
    const int rc = check_ffn8(d);
    if (rc != AQSGD_OK) return rc;
    if (d->m == 0 || d->f == 0) return AQSGD_OK;
    if (!dh || !pre || !dpre) return AQSGD_ERR_NULL;
    const uintptr_t e = elem_bytes(d->dtype);
    if (!aligned(dh, e) || !aligned(pre, e) || !aligned(dpre, e)) return AQSGD_ERR_ALIGN;
    Ffn8GradArgs a;
    a.dh = dh; a.pre = pre; a.dpre = dpre;
    a.m = d->m; a.f = d->f;
    a.dtype = d->dtype; a.act = d->act; a.gated = d->gated;
    return status(launch_ffn8_grad(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
