// C entries of the layer norm and of the weights' update: argument checks (the contract is in include/aqsgd.h) and the
// tables of the launches over many tensors.
#include <optional>

#include "aqsgd_adamw.h"
#include "aqsgd_products8.h"

namespace aqsgd {
namespace {

constexpr int64_t kMaxRows = int64_t{1} << 30, kMaxCols = int64_t{1} << 24;
constexpr int64_t kMaxElements = int64_t{1} << 34;        // of a tensor: its workgroups fit a launch
constexpr int64_t kMaxBlocks = (int64_t{1} << 24) - 1;    // workgroups of 256 lanes: a grid takes fewer than 2^32

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool known_dtype(int dtype) { return dtype == AQSGD_F32 || dtype == AQSGD_F16 || dtype == AQSGD_BF16; }
uintptr_t elem_bytes(int dtype) { return dtype == AQSGD_F32 ? 4 : 2; }
int status(hipError_t err) { return err == hipSuccess ? AQSGD_OK : AQSGD_ERR_LAUNCH; }
bool finite(double x) { return x - x == 0.0; }
bool least0(double x) { return finite(x) && x >= 0.0; }

int check_layernorm(const aqsgd_layernorm_desc* d) {
    if (!d) return AQSGD_ERR_NULL;
    if (!known_dtype(d->dtype)) return AQSGD_ERR_DTYPE;
    if (d->rows < 0 || d->rows > kMaxRows || d->cols < 1 || d->cols > kMaxCols || d->ld < d->cols || d->ld > (int64_t{1} << 40) ||
        (d->rows > 0 && d->ld > (int64_t{1} << 60) / d->rows) || (d->accumulate != 0 && d->accumulate != 1) || !least0(d->eps))
        return AQSGD_ERR_SHAPE;
    return AQSGD_OK;
}

int check_adamw(const aqsgd_adamw_desc* d) {
    if (!d) return AQSGD_ERR_NULL;
    if (!known_dtype(d->dtype) || (d->grad_dtype != d->dtype && d->grad_dtype != AQSGD_F32)) return AQSGD_ERR_DTYPE;
    if (d->rounding != AQSGD_ROUND_NEAREST && d->rounding != AQSGD_ROUND_STOCHASTIC) return AQSGD_ERR_DTYPE;
    if (d->state_bits != 8 && d->state_bits != 32) return AQSGD_ERR_BITS;
    if (d->step < 1 || !least0(d->lr) || !least0(d->eps) || !(d->beta1 >= 0.0 && d->beta1 < 1.0) || !(d->beta2 >= 0.0 && d->beta2 < 1.0))
        return AQSGD_ERR_SHAPE;
    return AQSGD_OK;
}

int check_list(const aqsgd_adamw_tensor* tensors, int32_t n_tensors) {
    if (n_tensors < 0) return AQSGD_ERR_SHAPE;
    if (n_tensors > 0 && !tensors) return AQSGD_ERR_NULL;
    for (int32_t i = 0; i < n_tensors; ++i)
        if (tensors[i].n < 0 || tensors[i].n > kMaxElements) return AQSGD_ERR_SHAPE;
    return AQSGD_OK;
}

int check_tensors(const aqsgd_adamw_desc* d, const aqsgd_adamw_tensor* tensors, int32_t n_tensors) {
    const int rc = check_list(tensors, n_tensors);
    if (rc != AQSGD_OK) return rc;
    const aqsgd_adamw_tensor* before = nullptr;
    for (const aqsgd_adamw_tensor* t = tensors; t != tensors + n_tensors; ++t) {
        if (t->n == 0) continue;
        if (!t->param || !t->grad || !t->state) return AQSGD_ERR_NULL;
        if (t->master ? d->dtype == AQSGD_F32 : before && before->master) return AQSGD_ERR_NULL;
        if (before && !before->master != !t->master) return AQSGD_ERR_NULL;
        if (!aligned(t->param, elem_bytes(d->dtype)) || !aligned(t->grad, elem_bytes(d->grad_dtype)) || !aligned(t->state, 16) || !aligned(t->master, 4))
            return AQSGD_ERR_ALIGN;
        if (!least0(t->weight_decay)) return AQSGD_ERR_SHAPE;
        before = t;
    }
    return AQSGD_OK;
}

// Elements of each workgroup of the norm's first pass: at least 4096, and so many that about 2048 workgroups, what the
// chip holds at once, take all of them.
int64_t norm_span(const aqsgd_adamw_tensor* tensors, int32_t n_tensors) {
    int64_t total = 0;
    for (int32_t i = 0; i < n_tensors; ++i) total += tensors[i].n;
    const int64_t span = (total / 2048 + 1023) / 1024 * 1024;
    return span < 4096 ? 4096 : span;
}
int64_t parts_of(int64_t n, int64_t span) { return (n + span - 1) / span; }
int64_t norm_parts(const aqsgd_adamw_tensor* tensors, int32_t n_tensors) {
    const int64_t span = norm_span(tensors, n_tensors);
    int64_t parts = 0;
    for (int32_t i = 0; i < n_tensors; ++i) parts += parts_of(tensors[i].n, span);
    return parts;
}

}  // namespace
}  // namespace aqsgd

using namespace aqsgd;

extern "C" {

int aqsgd_layernorm(const aqsgd_layernorm_desc* d, const void* x, const void* residual, const void* weight, const void* bias,
                    void* sum, void* y, float* mean, float* rstd, int8_t* row_codes, float* row_scales, void* stream) {
    const int rc = check_layernorm(d);
    if (rc != AQSGD_OK) return rc;
    if (d->rows == 0) return AQSGD_OK;
    if (!x || (sum && !residual) || !mean != !rstd || !row_codes != !row_scales) return AQSGD_ERR_NULL;
    const uintptr_t e = elem_bytes(d->dtype);
    if (!aligned(x, e) || !aligned(residual, e) || !aligned(weight, e) || !aligned(bias, e) || !aligned(sum, e) || !aligned(y, e) ||
        !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(row_codes, 16) || !aligned(row_scales, 4))
        return AQSGD_ERR_ALIGN;
    if ((sum && sum == y) || (d->ld != d->cols && ((sum && sum == x) || (y && y == x)))) return AQSGD_ERR_SHAPE;
    if (!sum && !y && !mean && !row_codes) return AQSGD_OK;
    LayernormArgs a;
    a.x = x; a.residual = residual; a.weight = weight; a.bias = bias;
    a.sum = sum; a.y = y; a.mean = mean; a.rstd = rstd; a.codes = row_codes; a.scales = row_scales;
    a.rows = d->rows; a.ld = d->ld; a.code_stride = code_stride(d->cols);
    a.eps = d->eps;
    a.each = 1.0 / static_cast<double>(d->cols);
    a.cols = static_cast<int32_t>(d->cols);
    return status(launch_layernorm(d->dtype, a, static_cast<hipStream_t>(stream)));
}

size_t aqsgd_layernorm_grad_workspace_bytes(const aqsgd_layernorm_desc* d) {
    return check_layernorm(d) == AQSGD_OK ? static_cast<size_t>(layernorm_grad_workspace_bytes(d->dtype, d->rows, d->cols)) : 0;
}

int aqsgd_layernorm_grad(const aqsgd_layernorm_desc* d, const void* dy, const void* x, const float* mean, const float* rstd,
                         const void* weight, const void* add, void* dx, float* dweight, float* dbias, void* workspace,
                         size_t workspace_bytes, void* stream) {
    const int rc = check_layernorm(d);
    if (rc != AQSGD_OK) return rc;
    const bool sums = dweight || dbias;
    if (!aligned(dweight, 4) || !aligned(dbias, 4)) return AQSGD_ERR_ALIGN;
    if (d->rows == 0 && !sums) return AQSGD_OK;
    if (d->rows > 0) {
        if (!dy || !x || !mean || !rstd || !dx) return AQSGD_ERR_NULL;
        const uintptr_t e = elem_bytes(d->dtype);
        if (!aligned(dy, e) || !aligned(x, e) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(weight, e) || !aligned(add, e) || !aligned(dx, e))
            return AQSGD_ERR_ALIGN;
        const size_t need = sums ? aqsgd_layernorm_grad_workspace_bytes(d) : 0;
        if (need && (!workspace || workspace_bytes < need)) return AQSGD_ERR_WORKSPACE;
        if (need && !aligned(workspace, 16)) return AQSGD_ERR_ALIGN;
        if (dx == x) return AQSGD_ERR_SHAPE;                // other workgroups read x for the columns' sums
    }
    LayernormGradArgs a;
    a.dy = dy; a.x = x; a.mean = mean; a.rstd = rstd; a.weight = weight; a.add = add; a.dx = dx;
    a.dweight = dweight; a.dbias = dbias;
    a.workspace = static_cast<float*>(workspace);
    a.rows = d->rows; a.ld = d->ld;
    a.cols = static_cast<int32_t>(d->cols);
    a.accumulate = d->accumulate;
    return status(launch_layernorm_grad(d->dtype, a, static_cast<hipStream_t>(stream)));
}

size_t aqsgd_adamw_state_bytes(const aqsgd_adamw_desc* d, int64_t n) {
    return check_adamw(d) == AQSGD_OK && n >= 0 && n <= kMaxElements ? static_cast<size_t>(state_bytes(n, d->state_bits)) : 0;
}

int aqsgd_adamw(const aqsgd_adamw_desc* d, const aqsgd_adamw_tensor* tensors, int32_t n_tensors, const float* lr, const int64_t* step,
                const float* scale, void* stream) {
    int rc = check_adamw(d);
    if (rc != AQSGD_OK) return rc;
    rc = check_tensors(d, tensors, n_tensors);
    if (rc != AQSGD_OK) return rc;
    if (!aligned(lr, 4) || !aligned(step, 8) || !aligned(scale, 4)) return AQSGD_ERR_ALIGN;
    AdamwArgs a;
    a.lr = d->lr; a.beta1 = d->beta1; a.beta2 = d->beta2;
    a.step = d->step;
    a.lr_at = lr; a.step_at = step; a.scale = scale;
    a.beta1f = static_cast<float>(d->beta1); a.rest1 = static_cast<float>(1.0 - d->beta1);
    a.beta2f = static_cast<float>(d->beta2); a.rest2 = static_cast<float>(1.0 - d->beta2);
    a.eps = static_cast<float>(d->eps);
    a.length = length_factor(d->lr, d->beta1, d->step);
    a.correct = correct_factor(d->beta2, d->step);
    a.seed = d->rng_seed;
    a.key = d->rng_seed + static_cast<uint64_t>(d->step);
    int held = 0;
    int64_t blocks = 0, groups = 0;
    const auto fits = [&](int64_t more) { return held < kTableTensors && blocks + more <= kMaxBlocks; };
    bool several = false;                                   // more tensors than a table's, or more workgroups than a grid's
    for (int32_t i = 0; i < n_tensors && !several; ++i) {
        const int64_t more = adamw_workgroups(tensors[i].n);
        if (more == 0) continue;
        several = !fits(more);
        ++held;
        blocks += more;
    }
    held = 0;
    blocks = 0;
    std::optional<ProfileSpan> profile;
    if (several) profile.emplace();
    const AdamwKind kind = {d->dtype, d->grad_dtype, d->state_bits, d->rounding};
    UpdateTable table;                                      // entries behind the last tensor's are never looked at
    const auto send = [&] {
        for (int i = held; i < kTableTensors; ++i) table.first[i] = 0xffffffffu;
        const hipError_t err = launch_adamw(kind, table, static_cast<uint32_t>(blocks), a, static_cast<hipStream_t>(stream));
        held = 0;
        blocks = 0;
        return err;
    };
    for (int32_t i = 0; i < n_tensors; ++i) {
        const aqsgd_adamw_tensor& t = tensors[i];
        if (t.n == 0) continue;
        const int64_t more = adamw_workgroups(t.n);
        if (!fits(more))
            if (const hipError_t err = send(); err != hipSuccess) return status(err);
        table.first[held] = static_cast<uint32_t>(blocks);
        table.tensor[held] = {t.param, t.grad, static_cast<char*>(t.state), t.master, t.n, groups, t.weight_decay, decay_factor(d->lr, t.weight_decay)};
        ++held;
        blocks += more;
        groups += state_groups(t.n);
    }
    if (profile) profile->last();
    return held ? status(send()) : AQSGD_OK;
}

size_t aqsgd_grad_norm_workspace_bytes(const aqsgd_adamw_tensor* tensors, int32_t n_tensors) {
    return check_list(tensors, n_tensors) == AQSGD_OK ? static_cast<size_t>(8 * norm_parts(tensors, n_tensors)) : 0;
}

int aqsgd_grad_norm(int32_t grad_dtype, const aqsgd_adamw_tensor* tensors, int32_t n_tensors, double max_norm, const float* loss_scale,
                    float* result, void* workspace, size_t workspace_bytes, void* stream) {
    if (!known_dtype(grad_dtype)) return AQSGD_ERR_DTYPE;
    const int rc = check_list(tensors, n_tensors);
    if (rc != AQSGD_OK) return rc;
    if (!(max_norm >= 0.0)) return AQSGD_ERR_SHAPE;
    if (!result) return AQSGD_ERR_NULL;
    int64_t chunks = 0;
    int32_t full = 0;
    for (int32_t i = 0; i < n_tensors; ++i) {
        if (tensors[i].n == 0) continue;
        if (!tensors[i].grad) return AQSGD_ERR_NULL;
        if (!aligned(tensors[i].grad, elem_bytes(grad_dtype))) return AQSGD_ERR_ALIGN;
        chunks += parts_of(tensors[i].n, norm_chunk(grad_dtype));
        ++full;
    }
    if (!aligned(loss_scale, 4) || !aligned(result, 4)) return AQSGD_ERR_ALIGN;
    const int64_t parts = norm_parts(tensors, n_tensors), span = norm_span(tensors, n_tensors);
    if (parts) {
        if (!workspace || workspace_bytes < static_cast<size_t>(8 * parts)) return AQSGD_ERR_WORKSPACE;
        if (!aligned(workspace, 16)) return AQSGD_ERR_ALIGN;
    }
    NormTable table;
    int held = 0;
    if (full > 0 && full <= kTableTensors && chunks <= kFewChunks) {
        uint32_t at = 0;
        for (int i = held; i < kTableTensors; ++i) table.first[i] = 0xffffffffu;
        for (const aqsgd_adamw_tensor* t = tensors; t != tensors + n_tensors; ++t) {
            if (t->n == 0) continue;
            table.first[held] = at;
            table.grad[held] = t->grad;
            table.n[held] = t->n;
            ++held;
            at += static_cast<uint32_t>(parts_of(t->n, norm_chunk(grad_dtype)));
        }
        return status(launch_grad_norm_few(grad_dtype, table, at, max_norm, loss_scale, result, static_cast<hipStream_t>(stream)));
    }
    double* const partial = static_cast<double*>(workspace);
    std::optional<ProfileSpan> profile;
    if (parts) profile.emplace();
    int64_t blocks = 0, sent = 0;
    const auto send = [&] {
        for (int i = held; i < kTableTensors; ++i) table.first[i] = 0xffffffffu;
        const hipError_t err = launch_grad_squares(grad_dtype, table, static_cast<uint32_t>(blocks), span, partial + sent, static_cast<hipStream_t>(stream));
        sent += blocks;
        held = 0;
        blocks = 0;
        return err;
    };
    for (int32_t i = 0; i < n_tensors; ++i) {
        if (tensors[i].n == 0) continue;
        if (held == kTableTensors)
            if (const hipError_t err = send(); err != hipSuccess) return status(err);
        table.first[held] = static_cast<uint32_t>(blocks);
        table.grad[held] = tensors[i].grad;
        table.n[held] = tensors[i].n;
        ++held;
        blocks += parts_of(tensors[i].n, span);
    }
    if (held)
        if (const hipError_t err = send(); err != hipSuccess) return status(err);
    if (profile) profile->last();
    return status(launch_grad_norm(partial, parts, max_norm, loss_scale, result, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
