// C entry points of the sensitivity map's operators (include/fedhe.h): argument checks and the choice of the work space.
#include <string.h>

#include "fedhe_internal.cuh"
#include "fedhe_map.h"

using namespace fedhe;

namespace {

inline bool good(const he_ctx *c) { return c && c->magic == CTX_MAGIC; }
// a context's GPU is the current one
bool here(const he_ctx *c) {
    int device = -1;
    return good(c) && cudaGetDevice(&device) == cudaSuccess && device == c->device;
}
inline size_t type_bytes(int dtype) { return dtype == HE_F32 ? 4 : dtype == HE_BF16 || dtype == HE_F16 ? 2 : 0; }
inline bool natural(const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline int done(cudaError_t e) { return e == cudaSuccess ? HE_OK : HE_ERR_CUDA; }
inline cudaStream_t as_stream(void *s) { return reinterpret_cast<cudaStream_t>(s); }

// sizes that the kernels' indexes and grids hold: rows below 2^28, columns below 2^31
constexpr size_t MOST_ROWS = (size_t)1 << 28, MOST_COLS = (size_t)1 << 31;
inline bool fits(size_t rows, size_t cols) { return rows < MOST_ROWS && cols < MOST_COLS; }

}  // namespace

extern "C" {

int he_token_log_probs(he_ctx *ctx, const void *logits_dev, int dtype, size_t rows, size_t vocab, size_t row_stride,
                       const int64_t *targets_dev, uint32_t top, float *logp_dev, float *lse_dev, float *entropy_dev, float *top_logp_dev,
                       int64_t *top_ids_dev, void *stream) {
    const size_t w = type_bytes(dtype);
    if (!here(ctx) || !w || !vocab || top > HE_MAX_TOP || top > vocab) return HE_ERR_INVALID_ARG;
    if (!fits(rows, vocab)) return HE_ERR_SIZE;
    if (!rows) return HE_OK;
    if (!logits_dev || !targets_dev || !logp_dev || !lse_dev || !entropy_dev || (top && (!top_logp_dev || !top_ids_dev))) return HE_ERR_INVALID_ARG;
    if (!natural(logits_dev, w) || !natural(targets_dev, 8) || !natural(logp_dev, 4) || !natural(lse_dev, 4) || !natural(entropy_dev, 4) ||
        !natural(top_logp_dev, 4) || !natural(top_ids_dev, 8))
        return HE_ERR_INVALID_ARG;
    const LogProbsArgs a{{logits_dev, row_stride}, rows, vocab, targets_dev, top, logp_dev, lse_dev, entropy_dev, top_logp_dev, top_ids_dev};
    return done(launch_log_probs(a, dtype, ctx->sm_count, ctx->dev.status, as_stream(stream)));
}

int he_token_log_probs_backward(he_ctx *ctx, const void *logits_dev, int dtype, size_t rows, size_t vocab, size_t row_stride,
                                const int64_t *targets_dev, const float *lse_dev, const float *dlogp_dev, const float *entropy_dev,
                                const float *dentropy_dev, uint32_t top, const int64_t *top_ids_dev, const float *dtop_dev, void *dlogits_dev,
                                size_t dlogits_stride, void *stream) {
    const size_t w = type_bytes(dtype);
    if (!here(ctx) || !w || !vocab || top > HE_MAX_TOP || top > vocab) return HE_ERR_INVALID_ARG;
    if (!fits(rows, vocab)) return HE_ERR_SIZE;
    if (rows > 1 && dlogits_stride < vocab) return HE_ERR_INVALID_ARG;
    if (!rows) return HE_OK;
    if (!logits_dev || !targets_dev || !lse_dev || !dlogp_dev || !dlogits_dev || (dentropy_dev && !entropy_dev) || (top && (!top_ids_dev || !dtop_dev)))
        return HE_ERR_INVALID_ARG;
    if (!natural(logits_dev, w) || !natural(dlogits_dev, w) || !natural(targets_dev, 8) || !natural(lse_dev, 4) || !natural(dlogp_dev, 4) ||
        !natural(entropy_dev, 4) || !natural(dentropy_dev, 4) || !natural(top_ids_dev, 8) || !natural(dtop_dev, 4))
        return HE_ERR_INVALID_ARG;
    if (logits_dev == dlogits_dev && rows > 1 && row_stride != dlogits_stride) return HE_ERR_INVALID_ARG;
    const LogProbsGradArgs a{{logits_dev, row_stride}, rows, vocab, targets_dev, lse_dev, entropy_dev, dlogp_dev, dentropy_dev, top, top_ids_dev, dtop_dev,
                             {dlogits_dev, dlogits_stride}};
    return done(launch_log_probs_grad(a, dtype, ctx->sm_count, ctx->dev.status, as_stream(stream)));
}

int he_layer_norm(he_ctx *ctx, const void *x_dev, int dtype, size_t rows, size_t width, size_t x_stride, const void *weight_dev,
                  const void *bias_dev, int weight_dtype, float eps, void *y_dev, size_t y_stride, float *mean_dev, float *rstd_dev,
                  void *stream) {
    const size_t w = type_bytes(dtype), ww = type_bytes(weight_dtype);
    if (!here(ctx) || !w || !ww || !width || !(eps >= 0.0f)) return HE_ERR_INVALID_ARG;
    if (!fits(rows, width)) return HE_ERR_SIZE;
    if (rows > 1 && y_stride < width) return HE_ERR_INVALID_ARG;
    if (!rows) return HE_OK;
    if (!x_dev || !y_dev || !mean_dev || !rstd_dev) return HE_ERR_INVALID_ARG;
    if (!natural(x_dev, w) || !natural(y_dev, w) || !natural(weight_dev, ww) || !natural(bias_dev, ww) || !natural(mean_dev, 4) || !natural(rstd_dev, 4))
        return HE_ERR_INVALID_ARG;
    if (x_dev == y_dev && rows > 1 && x_stride != y_stride) return HE_ERR_INVALID_ARG;
    const NormArgs a{{x_dev, x_stride}, rows, width, weight_dev, bias_dev, weight_dtype, eps, {y_dev, y_stride}, mean_dev, rstd_dev};
    return done(launch_norm(a, dtype, ctx->sm_count, ctx->dev.status, as_stream(stream)));
}

size_t he_layer_norm_backward_work_bytes(const he_ctx *ctx, size_t rows, size_t width) {
    return good(ctx) && width && fits(rows, width) ? norm_grad_work_bytes(rows, width, ctx->sm_count) : 0;
}

int he_layer_norm_backward(he_ctx *ctx, const void *dy_dev, size_t dy_stride, const void *x_dev, size_t x_stride, int dtype, size_t rows,
                           size_t width, const float *mean_dev, const float *rstd_dev, const void *weight_dev, int weight_dtype,
                           const int32_t *samples_dev, size_t num_samples, void *dx_dev, size_t dx_stride, float *dweight_dev,
                           float *dbias_dev, void *work_dev, size_t work_bytes, void *stream) {
    const size_t w = type_bytes(dtype), ww = type_bytes(weight_dtype);
    if (!here(ctx) || !w || !ww || !width || !dweight_dev || !dbias_dev || !work_dev) return HE_ERR_INVALID_ARG;
    if (!fits(rows, width) || num_samples >= MOST_ROWS) return HE_ERR_SIZE;
    if (rows > 1 && dx_stride < width) return HE_ERR_INVALID_ARG;
    if (work_bytes < norm_grad_work_bytes(rows, width, ctx->sm_count)) return HE_ERR_INVALID_ARG;
    if (rows && (!dy_dev || !x_dev || !mean_dev || !rstd_dev || !dx_dev)) return HE_ERR_INVALID_ARG;
    if (!natural(dy_dev, w) || !natural(x_dev, w) || !natural(dx_dev, w) || !natural(weight_dev, ww) || !natural(mean_dev, 4) || !natural(rstd_dev, 4) ||
        !natural(samples_dev, 4) || !natural(dweight_dev, 4) || !natural(dbias_dev, 4) || !natural(work_dev, 16))
        return HE_ERR_INVALID_ARG;
    if (rows && (dx_dev == x_dev || dx_dev == dy_dev)) return HE_ERR_INVALID_ARG;
    const NormGradArgs a{{dy_dev, dy_stride}, {x_dev, x_stride}, rows, width, mean_dev, rstd_dev, weight_dev, weight_dtype,
                         samples_dev ? SumOver::SAMPLES : SumOver::ALL, samples_dev, (uint32_t)num_samples, {dx_dev, dx_stride}, dweight_dev, dbias_dev, work_dev};
    return done(launch_norm_grad(a, dtype, ctx->sm_count, ctx->dev.status, as_stream(stream)));
}

size_t he_linear_sensitivity_work_bytes(const he_ctx *ctx, int dtype, size_t rows, size_t inputs, size_t outputs, int samples, int aligned) {
    if (!good(ctx) || !type_bytes(dtype) || !inputs || !outputs || !fits(rows, inputs) || !fits(rows, outputs)) return 0;
    return linear_map_work_bytes(rows, inputs, outputs, dtype, samples != 0, aligned != 0 && dtype != HE_F32, true, ctx->sm_count);
}

int he_linear_sensitivity(he_ctx *ctx, const void *x_dev, size_t x_stride, const void *dy_dev, size_t dy_stride, int dtype, size_t rows,
                          size_t inputs, size_t outputs, const int32_t *samples_dev, size_t num_samples, int accumulate, float *weight_dev,
                          float *bias_dev, void *work_dev, size_t work_bytes, void *stream) {
    const size_t w = type_bytes(dtype);
    if (!here(ctx) || !w || !inputs || !outputs || !weight_dev) return HE_ERR_INVALID_ARG;
    if (!fits(rows, inputs) || !fits(rows, outputs) || num_samples >= MOST_ROWS) return HE_ERR_SIZE;
    if (rows && (!x_dev || !dy_dev)) return HE_ERR_INVALID_ARG;
    if (!natural(x_dev, w) || !natural(dy_dev, w) || !natural(samples_dev, 4) || !natural(weight_dev, 4) || !natural(bias_dev, 4) || !natural(work_dev, 16))
        return HE_ERR_INVALID_ARG;
    const bool aligned = linear_map_aligned({x_dev, x_stride}, inputs, dtype) && linear_map_aligned({dy_dev, dy_stride}, outputs, dtype);
    const size_t need = linear_map_work_bytes(rows, inputs, outputs, dtype, samples_dev != nullptr, aligned, bias_dev != nullptr, ctx->sm_count);
    if (work_bytes < need || (need && !work_dev)) return HE_ERR_INVALID_ARG;
    const LinearMapArgs a{{x_dev, x_stride}, {dy_dev, dy_stride}, rows, inputs, outputs, samples_dev ? SumOver::SAMPLES : SumOver::ROWS, samples_dev,
                          (uint32_t)num_samples, accumulate != 0, weight_dev, bias_dev, work_dev};
    return done(launch_linear_map(a, dtype, ctx->sm_count, ctx->dev.status, as_stream(stream)));
}

}  // extern "C"
