// C entry points of the operators around a worker's loss: checks of the arguments, then the
// launch.  Nothing here allocates, synchronises or throws.
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/cdadam.h"
#include "kernels.h"
#include "operators.h"

namespace {

int refuse(const char *fn, const char *fmt, ...)
{
    char msg[256];
    int n = snprintf(msg, sizeof msg, "%s: ", fn);
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg + n, sizeof msg - n, fmt, ap);
    va_end(ap);
    cdadam::set_last_error(msg);
    return CDADAM_ERR_ARG;
}

int launched(const char *fn)
{
    const cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) return CDADAM_OK;
    char msg[256];
    snprintf(msg, sizeof msg, "%s: %s", fn, cudaGetErrorString(e));
    cdadam::set_last_error(msg);
    return CDADAM_ERR_CUDA;
}

bool known(int type) { return type == CDADAM_F32 || type == CDADAM_BF16 || type == CDADAM_F16; }
int size_of(int type) { return type == CDADAM_F32 ? 4 : 2; }
bool misaligned(const void *p, int size) { return p && ((uintptr_t)p & (uintptr_t)(size - 1)) != 0; }

constexpr int64_t kMaxRows = 0x7fffffff;
constexpr int64_t kMaxStride = (int64_t)1 << 31;    // rows * stride * element size stays below 2^64

// A matrix argument: `output` rows must not overlap.
int check_matrix(const char *fn, const char *what, const void *p, int64_t stride, int64_t rows, int64_t cols, int type,
                 bool output)
{
    if (rows > 0 && !p) return refuse(fn, "%s is NULL", what);
    if (misaligned(p, size_of(type))) return refuse(fn, "%s is not aligned to its elements", what);
    if (rows > 1 && (stride < (output ? cols : 0) || stride > kMaxStride))
        return refuse(fn, "%s: row stride %lld is outside [%lld, 2^31]", what, (long long)stride,
                      (long long)(output ? cols : 0));
    return CDADAM_OK;
}

int check_same(const char *fn, const char *what, const void *out, int64_t out_stride, const void *in, int64_t in_stride,
               int64_t rows)
{
    if (rows > 1 && out == in && out_stride != in_stride)
        return refuse(fn, "%s overwrites an input with another row stride", what);
    return CDADAM_OK;
}

int check_rows(const char *fn, int64_t rows)
{
    if (rows < 0 || rows > kMaxRows) return refuse(fn, "rows = %lld is outside [0, 2^31)", (long long)rows);
    return CDADAM_OK;
}

int check_logits(const char *fn, const void *logits, int64_t stride, int64_t rows, int64_t vocab, int type, int index_type,
                 float temperature)
{
    if (!known(type)) return refuse(fn, "unknown element type %d", type);
    if (index_type != CDADAM_I32 && index_type != CDADAM_I64) return refuse(fn, "unknown index type %d", index_type);
    if (int rc = check_rows(fn, rows)) return rc;
    if (vocab < 1 || vocab > CDADAM_MAX_VOCAB)
        return refuse(fn, "vocab = %lld is outside [1, %d]", (long long)vocab, (int)CDADAM_MAX_VOCAB);
    if (!(temperature >= 1e-4f && temperature <= 1e4f)) return refuse(fn, "temperature = %g is outside [1e-4, 1e4]", temperature);
    return check_matrix(fn, "logits", logits, stride, rows, vocab, type, false);
}

// A matrix of bytes.
int check_bytes(const char *fn, const char *what, const void *p, int64_t stride, int64_t rows, int64_t cols, bool output)
{
    if (rows > 0 && !p) return refuse(fn, "%s is NULL", what);
    if (rows > 1 && (stride < (output ? cols : 0) || stride > kMaxStride))
        return refuse(fn, "%s: row stride %lld is outside [%lld, 2^31]", what, (long long)stride, (long long)(output ? cols : 0));
    return CDADAM_OK;
}

// A checkpoint: rows x cols bytes and their exponents.
int check_kept(const char *fn, const void *kept, int64_t kept_stride, const void *exponents, int64_t exponents_stride, int64_t rows,
               int64_t cols, bool output)
{
    if (int rc = check_bytes(fn, "kept", kept, kept_stride, rows, cols, output)) return rc;
    return check_bytes(fn, "exponents", exponents, exponents_stride, rows,
                       (cols + CDADAM_CHECKPOINT_BLOCK - 1) / CDADAM_CHECKPOINT_BLOCK, output);
}

int check_shape(const char *fn, int64_t rows, int64_t cols, int type)
{
    if (!known(type)) return refuse(fn, "unknown element type %d", type);
    if (int rc = check_rows(fn, rows)) return rc;
    if (cols < 1 || cols > CDADAM_MAX_NORM_COLS)
        return refuse(fn, "cols = %lld is outside [1, %d]", (long long)cols, (int)CDADAM_MAX_NORM_COLS);
    return CDADAM_OK;
}

// The stride of a single row says nothing and was not checked: kernels get 0.
cdadam::Matrix matrix(const void *p, int64_t stride, int64_t rows) { return {const_cast<void *>(p), rows > 1 ? stride : 0}; }
cdadam::Rows8 rows8(const int8_t *p, int64_t stride, const float *scale) { return {const_cast<int8_t *>(p), stride, const_cast<float *>(scale)}; }
cdadam::Kept8 kept8(const int8_t *p, int64_t stride, const uint8_t *exponents, int64_t exponents_stride)
{
    return {const_cast<int8_t *>(p), stride, const_cast<uint8_t *>(exponents), exponents_stride};
}

thread_local int wait_limit = -1;

double scale2(float temperature) { return 1.4426950408889634074 / (double)temperature; }
int index_size(int index_type) { return index_type == CDADAM_I64 ? 8 : 4; }

}  // namespace

extern "C" {

int cdadam_set_operator_wait_limit(int polls)
{
    wait_limit = polls < 0 ? -1 : polls;
    return CDADAM_OK;
}

int cdadam_layer_norm(const void *x, int64_t x_stride, const void *weight, const void *bias, int64_t rows, int64_t cols,
                      float eps, int type, int weight_type, void *y, int64_t y_stride, float *mean, float *rstd, void *stream)
{
    static const char fn[] = "cdadam_layer_norm";
    if (!known(type) || !known(weight_type)) return refuse(fn, "unknown element type %d, %d", type, weight_type);
    if (int rc = check_rows(fn, rows)) return rc;
    if (cols < 1 || cols > CDADAM_MAX_NORM_COLS)
        return refuse(fn, "cols = %lld is outside [1, %d]", (long long)cols, (int)CDADAM_MAX_NORM_COLS);
    if (!(eps >= 0.0f) || std::isinf(eps)) return refuse(fn, "eps = %g is not a finite number >= 0", eps);
    if (int rc = check_matrix(fn, "x", x, x_stride, rows, cols, type, false)) return rc;
    if (int rc = check_matrix(fn, "y", y, y_stride, rows, cols, type, true)) return rc;
    if (int rc = check_same(fn, "y", y, y_stride, x, x_stride, rows)) return rc;
    if (misaligned(weight, size_of(weight_type)) || misaligned(bias, size_of(weight_type)) || misaligned(mean, 4) ||
        misaligned(rstd, 4))
        return refuse(fn, "weight, bias, mean or rstd is not aligned to its elements");
    cdadam::NormForward a = {x, x_stride, {weight, weight_type}, {bias, weight_type}, rows, cols, eps, y, y_stride, mean, rstd,
                             wait_limit};
    if (rows == 0) return CDADAM_OK;
    cdadam::launch_layer_norm(a, type, (cudaStream_t)stream);
    return launched(fn);
}

int64_t cdadam_layer_norm_workspace(int64_t rows, int64_t cols, int64_t groups)
{
    if (rows < 0 || rows > kMaxRows || cols < 1 || cols > CDADAM_MAX_NORM_COLS || groups < 1 || groups > 65535) return 0;
    return cdadam::layer_norm_workspace(rows, cols, groups);
}

int cdadam_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, const void *weight,
                               const float *mean, const float *rstd, int64_t rows, int64_t cols, int64_t groups, int type,
                               int weight_type, int grad_type, void *dx, int64_t dx_stride, void *dweight,
                               int64_t dweight_stride, void *dbias, int64_t dbias_stride, int accumulate, void *workspace,
                               int64_t workspace_bytes, void *stream)
{
    static const char fn[] = "cdadam_layer_norm_backward";
    if (!known(type) || !known(weight_type) || !known(grad_type))
        return refuse(fn, "unknown element type %d, %d, %d", type, weight_type, grad_type);
    if (int rc = check_rows(fn, rows)) return rc;
    if (cols < 1 || cols > CDADAM_MAX_NORM_COLS)
        return refuse(fn, "cols = %lld is outside [1, %d]", (long long)cols, (int)CDADAM_MAX_NORM_COLS);
    if (groups < 1 || groups > 65535 || rows % groups != 0)
        return refuse(fn, "%lld rows do not form %lld equal groups (1 .. 65535)", (long long)rows, (long long)groups);
    if (rows > 0 && !dx && !dweight && !dbias) return refuse(fn, "dx, dweight and dbias are all NULL");
    if (int rc = check_matrix(fn, "dy", dy, dy_stride, rows, cols, type, false)) return rc;
    if (int rc = check_matrix(fn, "x", x, x_stride, rows, cols, type, false)) return rc;
    if (rows > 0 && (!mean || !rstd)) return refuse(fn, "mean or rstd is NULL");
    if (dx) {
        if (int rc = check_matrix(fn, "dx", dx, dx_stride, rows, cols, type, true)) return rc;
        if (int rc = check_same(fn, "dx", dx, dx_stride, x, x_stride, rows)) return rc;
        if (int rc = check_same(fn, "dx", dx, dx_stride, dy, dy_stride, rows)) return rc;
    }
    if (dweight) if (int rc = check_matrix(fn, "dweight", dweight, dweight_stride, groups, cols, grad_type, true)) return rc;
    if (dbias) if (int rc = check_matrix(fn, "dbias", dbias, dbias_stride, groups, cols, grad_type, true)) return rc;
    if (misaligned(weight, size_of(weight_type)) || misaligned(mean, 4) || misaligned(rstd, 4))
        return refuse(fn, "weight, mean or rstd is not aligned to its elements");
    const int64_t need = dweight || dbias ? cdadam::layer_norm_workspace(rows, cols, groups) : 0;
    if (need > 0 && (!workspace || workspace_bytes < need || misaligned(workspace, 16)))
        return refuse(fn, "workspace: %lld bytes, 16-byte aligned, are needed, %lld given", (long long)need,
                      (long long)(workspace ? workspace_bytes : 0));
    cdadam::NormBackward a = {dy, dy_stride, x, x_stride, {weight, weight_type}, mean, rstd, rows, cols, groups, dx, dx_stride,
                              dweight, dweight_stride, dbias, dbias_stride, grad_type, accumulate != 0, (float *)workspace,
                              wait_limit};
    cdadam::launch_layer_norm_backward(a, type, (cudaStream_t)stream);
    return launched(fn);
}

int cdadam_token_logprobs(const void *logits, int64_t logits_stride, const void *tokens, int64_t rows, int64_t vocab, int type,
                          int index_type, float temperature, int k, float *logprob, float *entropy, float *lse, void *top_ids,
                          float *top_logprobs, void *stream)
{
    static const char fn[] = "cdadam_token_logprobs";
    if (int rc = check_logits(fn, logits, logits_stride, rows, vocab, type, index_type, temperature)) return rc;
    if (k < 0 || k > CDADAM_MAX_LIST || k > vocab)
        return refuse(fn, "k = %d is outside [0, min(vocab, %d)]", k, (int)CDADAM_MAX_LIST);
    if (logprob && !tokens && rows > 0) return refuse(fn, "logprob without tokens");
    if (!top_ids != !top_logprobs) return refuse(fn, "top_ids and top_logprobs: both or neither");
    const int is = index_size(index_type);
    if (misaligned(tokens, is) || misaligned(top_ids, is) || misaligned(top_logprobs, 4) || misaligned(logprob, 4) ||
        misaligned(entropy, 4) || misaligned(lse, 4))
        return refuse(fn, "a vector is not aligned to its elements");
    if (k == 0) top_ids = nullptr, top_logprobs = nullptr;
    cdadam::Logprobs a = {logits, logits_stride, tokens, rows, vocab, index_type == CDADAM_I64, scale2(temperature),
                          top_ids ? k : 0, logprob, entropy, lse, top_ids, top_logprobs};
    if (rows == 0 || (!logprob && !entropy && !lse && !top_ids)) return CDADAM_OK;
    cdadam::launch_token_logprobs(a, type, (cudaStream_t)stream);
    return launched(fn);
}

int cdadam_token_logprobs_backward(const void *logits, int64_t logits_stride, const void *tokens, int64_t rows, int64_t vocab,
                                   int type, int index_type, float temperature, const float *lse, const float *entropy,
                                   const float *dlogprob, const float *dentropy, void *dlogits, int64_t dlogits_stride,
                                   void *stream)
{
    static const char fn[] = "cdadam_token_logprobs_backward";
    if (int rc = check_logits(fn, logits, logits_stride, rows, vocab, type, index_type, temperature)) return rc;
    if (int rc = check_matrix(fn, "dlogits", dlogits, dlogits_stride, rows, vocab, type, true)) return rc;
    if (int rc = check_same(fn, "dlogits", dlogits, dlogits_stride, logits, logits_stride, rows)) return rc;
    if (rows > 0) {
        if (!lse) return refuse(fn, "lse is NULL");
        if (dentropy && !entropy) return refuse(fn, "dentropy without entropy");
        if (dlogprob && !tokens) return refuse(fn, "dlogprob without tokens");
    }
    if (misaligned(tokens, index_size(index_type)) || misaligned(lse, 4) || misaligned(entropy, 4) || misaligned(dlogprob, 4) ||
        misaligned(dentropy, 4))
        return refuse(fn, "a vector is not aligned to its elements");
    if (rows == 0) return CDADAM_OK;
    const double s = scale2(temperature);
    cdadam::LogprobsBackward a = {logits, logits_stride, tokens, rows, vocab, index_type == CDADAM_I64, s,
                                  (double)(float)s * (double)temperature, (float)(1.0 / (double)temperature), lse, entropy,
                                  dlogprob, dentropy, dlogits, dlogits_stride};
    cdadam::launch_token_logprobs_backward(a, type, (cudaStream_t)stream);
    return launched(fn);
}

int cdadam_distill(const void *logits, int64_t logits_stride, const void *teacher_ids, const float *teacher_logprobs,
                   int64_t rows, int64_t vocab, int k, int type, int index_type, float temperature, int rest,
                   const float *dloss, float *loss, void *dlogits, int64_t dlogits_stride, void *stream)
{
    static const char fn[] = "cdadam_distill";
    if (int rc = check_logits(fn, logits, logits_stride, rows, vocab, type, index_type, temperature)) return rc;
    if (k < 1 || k > CDADAM_MAX_LIST) return refuse(fn, "k = %d is outside [1, %d]", k, (int)CDADAM_MAX_LIST);
    if (rows > 0 && !loss && !dlogits) return refuse(fn, "loss and dlogits are both NULL");
    if (rows > 0 && (!teacher_ids || !teacher_logprobs)) return refuse(fn, "teacher_ids or teacher_logprobs is NULL");
    if (dlogits) {
        if (rows > 0 && !dloss) return refuse(fn, "dlogits without dloss");
        if (int rc = check_matrix(fn, "dlogits", dlogits, dlogits_stride, rows, vocab, type, true)) return rc;
        if (int rc = check_same(fn, "dlogits", dlogits, dlogits_stride, logits, logits_stride, rows)) return rc;
    }
    if (misaligned(teacher_ids, index_size(index_type)) || misaligned(teacher_logprobs, 4) || misaligned(dloss, 4) ||
        misaligned(loss, 4))
        return refuse(fn, "a vector is not aligned to its elements");
    if (rows == 0) return CDADAM_OK;
    cdadam::Distill a = {logits, logits_stride, teacher_ids, teacher_logprobs, rows, vocab, k, index_type == CDADAM_I64,
                         scale2(temperature), (float)(1.0 / (double)temperature), rest != 0, dloss, loss, dlogits,
                         dlogits_stride, wait_limit};
    cdadam::launch_distill(a, type, (cudaStream_t)stream);
    return launched(fn);
}

int cdadam_rms_norm(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, const void *weight, int64_t rows,
                    int64_t cols, float eps, int type, int weight_type, void *total, int64_t total_stride, void *y, int64_t y_stride,
                    int8_t *q, int64_t q_stride, float *scale, int8_t *kept, int64_t kept_stride, uint8_t *exponents,
                    int64_t exponents_stride, float *rstd, void *stream)
{
    static const char fn[] = "cdadam_rms_norm";
    if (int rc = check_shape(fn, rows, cols, type)) return rc;
    if (!known(weight_type)) return refuse(fn, "unknown element type %d", weight_type);
    if (!(eps >= 0.0f) || std::isinf(eps)) return refuse(fn, "eps = %g is not a finite number >= 0", eps);
    if (!q != !scale || !kept != !exponents) return refuse(fn, "q and scale, kept and exponents: both or neither");
    if (rows > 0 && !total && !y && !q && !kept && !rstd) return refuse(fn, "no output is given");
    if (rows > 0 && total && total == y) return refuse(fn, "total and y are the same matrix");
    if (int rc = check_matrix(fn, "x", x, x_stride, rows, cols, type, false)) return rc;
    if (residual) if (int rc = check_matrix(fn, "residual", residual, residual_stride, rows, cols, type, false)) return rc;
    for (int i = 0; i < 2; ++i) {
        const char *const what = i ? "y" : "total";
        void *const p = i ? y : total;
        const int64_t stride = i ? y_stride : total_stride;
        if (!p) continue;
        if (int rc = check_matrix(fn, what, p, stride, rows, cols, type, true)) return rc;
        if (int rc = check_same(fn, what, p, stride, x, x_stride, rows)) return rc;
        if (int rc = check_same(fn, what, p, stride, residual, residual_stride, rows)) return rc;
    }
    if (q) if (int rc = check_bytes(fn, "q", q, q_stride, rows, cols, true)) return rc;
    if (kept) if (int rc = check_kept(fn, kept, kept_stride, exponents, exponents_stride, rows, cols, true)) return rc;
    if (misaligned(weight, size_of(weight_type)) || misaligned(scale, 4) || misaligned(rstd, 4))
        return refuse(fn, "weight, scale or rstd is not aligned to its elements");
    if (rows == 0) return CDADAM_OK;
    cdadam::RmsNorm a = {matrix(x, x_stride, rows), matrix(residual, residual_stride, rows), {weight, weight_type}, rows, cols, eps, 1,
                         matrix(total, total_stride, rows), matrix(y, y_stride, rows), rows8(q, q_stride, scale),
                         kept8(kept, kept_stride, exponents, exponents_stride), rstd};
    cdadam::launch_rms_norm(a, type, (cudaStream_t)stream);
    return launched(fn);
}

int64_t cdadam_rms_norm_workspace(int64_t rows, int64_t cols, int64_t groups)
{
    if (rows < 0 || rows > kMaxRows || cols < 1 || cols > CDADAM_MAX_NORM_COLS || groups < 1 || groups > 65535) return 0;
    return cdadam::rms_norm_workspace(rows, cols, groups);
}

int cdadam_rms_norm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, const uint8_t *exponents,
                             int64_t exponents_stride, const void *weight, const float *rstd, const void *dtotal,
                             int64_t dtotal_stride, int64_t rows, int64_t cols, int64_t groups, int type, int weight_type, int grad_type,
                             void *dx, int64_t dx_stride, void *dweight, int64_t dweight_stride, int accumulate, void *workspace,
                             int64_t workspace_bytes, void *stream)
{
    static const char fn[] = "cdadam_rms_norm_backward";
    if (int rc = check_shape(fn, rows, cols, type)) return rc;
    if (!known(weight_type) || !known(grad_type)) return refuse(fn, "unknown element type %d, %d", weight_type, grad_type);
    if (groups < 1 || groups > 65535 || rows % groups != 0)
        return refuse(fn, "%lld rows do not form %lld equal groups (1 .. 65535)", (long long)rows, (long long)groups);
    if (rows > 0 && !dx && !dweight) return refuse(fn, "dx and dweight are both NULL");
    if (int rc = check_matrix(fn, "dy", dy, dy_stride, rows, cols, type, false)) return rc;
    if (exponents) {
        if (int rc = check_kept(fn, x, x_stride, exponents, exponents_stride, rows, cols, false)) return rc;
    } else if (int rc = check_matrix(fn, "x", x, x_stride, rows, cols, type, false)) return rc;
    if (dtotal) if (int rc = check_matrix(fn, "dtotal", dtotal, dtotal_stride, rows, cols, type, false)) return rc;
    if (rows > 0 && !rstd) return refuse(fn, "rstd is NULL");
    if (dx) {
        if (int rc = check_matrix(fn, "dx", dx, dx_stride, rows, cols, type, true)) return rc;
        if (int rc = check_same(fn, "dx", dx, dx_stride, dy, dy_stride, rows)) return rc;
        if (int rc = check_same(fn, "dx", dx, dx_stride, dtotal, dtotal_stride, rows)) return rc;
        if (rows > 0 && exponents && dx == x) return refuse(fn, "dx overwrites the checkpoint");
        if (!exponents) if (int rc = check_same(fn, "dx", dx, dx_stride, x, x_stride, rows)) return rc;
    }
    if (dweight) if (int rc = check_matrix(fn, "dweight", dweight, dweight_stride, groups, cols, grad_type, true)) return rc;
    if (misaligned(weight, size_of(weight_type)) || misaligned(rstd, 4)) return refuse(fn, "weight or rstd is not aligned to its elements");
    const int64_t need = dweight ? cdadam::rms_norm_workspace(rows, cols, groups) : 0;
    if (need > 0 && (!workspace || workspace_bytes < need || misaligned(workspace, 16)))
        return refuse(fn, "workspace: %lld bytes, 16-byte aligned, are needed, %lld given", (long long)need,
                      (long long)(workspace ? workspace_bytes : 0));
    cdadam::RmsNormBackward a = {matrix(dy, dy_stride, rows), matrix(exponents ? nullptr : x, x_stride, rows),
                                 kept8(exponents ? (const int8_t *)x : nullptr, x_stride, exponents, exponents_stride), {weight, weight_type}, rstd,
                                 matrix(dtotal, dtotal_stride, rows), rows, cols, groups, matrix(dx, dx_stride, rows), dweight, dweight_stride,
                                 grad_type, accumulate != 0, (float *)workspace};
    if (rows == 0 && !dweight) return CDADAM_OK;
    cdadam::launch_rms_norm_backward(a, type, (cudaStream_t)stream);
    return launched(fn);
}

int cdadam_quantize_rows(const void *x, int64_t x_stride, int64_t rows, int64_t cols, int type, int8_t *q, int64_t q_stride, float *scale,
                         void *stream)
{
    static const char fn[] = "cdadam_quantize_rows";
    if (int rc = check_shape(fn, rows, cols, type)) return rc;
    if (int rc = check_matrix(fn, "x", x, x_stride, rows, cols, type, false)) return rc;
    if (int rc = check_bytes(fn, "q", q, q_stride, rows, cols, true)) return rc;
    if (rows > 0 && !scale) return refuse(fn, "scale is NULL");
    if (misaligned(scale, 4)) return refuse(fn, "scale is not aligned to its elements");
    if (rows == 0) return CDADAM_OK;
    cdadam::RmsNorm a = {};
    a.x = matrix(x, x_stride, rows);
    a.rows = rows;
    a.cols = cols;
    a.q = rows8(q, q_stride, scale);
    cdadam::launch_rms_norm(a, type, (cudaStream_t)stream);
    return launched(fn);
}

int cdadam_dequantize_rows(const int8_t *q, int64_t q_stride, const float *scale, int64_t rows, int64_t cols, int type, void *y,
                           int64_t y_stride, void *stream)
{
    static const char fn[] = "cdadam_dequantize_rows";
    if (int rc = check_shape(fn, rows, cols, type)) return rc;
    if (int rc = check_bytes(fn, "q", q, q_stride, rows, cols, false)) return rc;
    if (int rc = check_matrix(fn, "y", y, y_stride, rows, cols, type, true)) return rc;
    if (rows > 0 && !scale) return refuse(fn, "scale is NULL");
    if (misaligned(scale, 4)) return refuse(fn, "scale is not aligned to its elements");
    if (rows == 0) return CDADAM_OK;
    cdadam::launch_restore8(rows8(q, q_stride, scale), kept8(nullptr, 0, nullptr, 0), matrix(y, y_stride, rows), rows, cols, type,
                            (cudaStream_t)stream);
    return launched(fn);
}

int cdadam_checkpoint8(const void *x, int64_t x_stride, int64_t rows, int64_t cols, int type, int8_t *kept, int64_t kept_stride,
                       uint8_t *exponents, int64_t exponents_stride, void *stream)
{
    static const char fn[] = "cdadam_checkpoint8";
    if (int rc = check_shape(fn, rows, cols, type)) return rc;
    if (int rc = check_matrix(fn, "x", x, x_stride, rows, cols, type, false)) return rc;
    if (int rc = check_kept(fn, kept, kept_stride, exponents, exponents_stride, rows, cols, true)) return rc;
    if (rows == 0) return CDADAM_OK;
    cdadam::launch_checkpoint8(matrix(x, x_stride, rows), kept8(kept, kept_stride, exponents, exponents_stride), rows, cols, type,
                               (cudaStream_t)stream);
    return launched(fn);
}

int cdadam_checkpoint8_restore(const int8_t *kept, int64_t kept_stride, const uint8_t *exponents, int64_t exponents_stride, int64_t rows,
                               int64_t cols, int type, void *x, int64_t x_stride, void *stream)
{
    static const char fn[] = "cdadam_checkpoint8_restore";
    if (int rc = check_shape(fn, rows, cols, type)) return rc;
    if (int rc = check_kept(fn, kept, kept_stride, exponents, exponents_stride, rows, cols, false)) return rc;
    if (int rc = check_matrix(fn, "x", x, x_stride, rows, cols, type, true)) return rc;
    if (rows == 0) return CDADAM_OK;
    cdadam::launch_restore8(rows8(nullptr, 0, nullptr), kept8(kept, kept_stride, exponents, exponents_stride), matrix(x, x_stride, rows), rows,
                            cols, type, (cudaStream_t)stream);
    return launched(fn);
}

int cdadam_matmul8(const int8_t *x, int64_t x_stride, const float *x_scale, const int8_t *w, int64_t w_stride, const float *w_scale,
                   const void *bias, int64_t tokens, int64_t channels, int64_t inner, int type, int bias_type, void *y, int64_t y_stride,
                   void *stream)
{
    static const char fn[] = "cdadam_matmul8";
    if (!known(type) || !known(bias_type)) return refuse(fn, "unknown element type %d, %d", type, bias_type);
    constexpr int64_t most = (int64_t)1 << 30;
    if (tokens < 0 || tokens > most || channels < 0 || channels > most)
        return refuse(fn, "tokens = %lld or channels = %lld is outside [0, 2^30]", (long long)tokens, (long long)channels);
    if (inner < 1 || inner > CDADAM_MAX_INNER)
        return refuse(fn, "inner = %lld is outside [1, %d]", (long long)inner, (int)CDADAM_MAX_INNER);
    if ((tokens / 128 + 1) * (channels / 128 + 1) >= (int64_t)1 << 27)
        return refuse(fn, "%lld tokens times %lld channels are too many", (long long)tokens, (long long)channels);
    const int64_t none = tokens && channels ? 0 : 1;
    for (int i = 0; i < 2 && !none; ++i) {
        const char *const what = i ? "w" : "x";
        const int8_t *const p = i ? w : x;
        const int64_t stride = i ? w_stride : x_stride, rows = i ? channels : tokens;
        if (int rc = check_bytes(fn, what, p, stride, rows, inner, true)) return rc;
        if (misaligned(p, 16) || (rows > 1 && stride % 16 != 0)) return refuse(fn, "%s: rows have to start on 16 bytes", what);
        if (!(i ? w_scale : x_scale)) return refuse(fn, "%s_scale is NULL", what);
    }
    if (!none) if (int rc = check_matrix(fn, "y", y, y_stride, tokens, channels, type, true)) return rc;
    if (misaligned(x_scale, 4) || misaligned(w_scale, 4) || misaligned(bias, size_of(bias_type)))
        return refuse(fn, "x_scale, w_scale or bias is not aligned to its elements");
    if (none) return CDADAM_OK;
    cdadam::Matmul8 a = {rows8(x, x_stride, x_scale), rows8(w, w_stride, w_scale), {bias, bias_type}, tokens, channels, inner, y, y_stride,
                         wait_limit};
    if (!cdadam::launch_matmul8(a, type, (cudaStream_t)stream)) {
        const cudaError_t e = cudaGetLastError();       // taken here: it is not the next call's
        char msg[256];
        snprintf(msg, sizeof msg, "%s: the driver did not describe the matrices to the copy engine%s%s", fn, e == cudaSuccess ? "" : ": ",
                 e == cudaSuccess ? "" : cudaGetErrorString(e));
        cdadam::set_last_error(msg);
        return CDADAM_ERR_CUDA;
    }
    return launched(fn);
}

}  // extern "C"
