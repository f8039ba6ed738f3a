// Launch wrappers of the sensitivity map's kernels, called by fedhe_map_api.cu after it has checked the arguments.  All of them
// enqueue work on `s` and return the launch status; none synchronises or allocates.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/fedhe.h"

namespace fedhe {

// A row-major matrix; `stride` is the distance of its rows in elements.
struct MatArg {
    const void *p;
    size_t stride;
};
struct MatOut {
    void *p;
    size_t stride;
};

struct LogProbsArgs {
    MatArg logits;
    size_t rows, vocab;
    const int64_t *targets;
    uint32_t top;
    float *logp, *lse, *entropy, *top_logp;
    int64_t *top_ids;
};
// status (here and below): the context's, raised where something inside a kernel does not arrive
cudaError_t launch_log_probs(const LogProbsArgs &a, int dtype, int n_sm, int *status, cudaStream_t s);

struct LogProbsGradArgs {
    MatArg logits;
    size_t rows, vocab;
    const int64_t *targets;
    const float *lse, *entropy, *dlogp, *dentropy;
    uint32_t top;
    const int64_t *top_ids;
    const float *dtop;
    MatOut dlogits;
};
cudaError_t launch_log_probs_grad(const LogProbsGradArgs &a, int dtype, int n_sm, int *status, cudaStream_t s);

struct NormArgs {
    MatArg x;
    size_t rows, width;
    const void *weight, *bias;
    int weight_type;
    float eps;
    MatOut y;
    float *mean, *rstd;
};
cudaError_t launch_norm(const NormArgs &a, int dtype, int n_sm, int *status, cudaStream_t s);

// How rows are summed: all of them, or within a sample with the magnitudes added over the samples, or every row a sample of its own (linear
// layers).
enum class SumOver { ALL, SAMPLES, ROWS };

struct NormGradArgs {
    MatArg dy, x;
    size_t rows, width;
    const float *mean, *rstd;
    const void *weight;
    int weight_type;
    SumOver over;
    const int32_t *offsets;
    uint32_t samples;
    MatOut dx;
    float *dweight, *dbias;
    void *work;
};
size_t norm_grad_work_bytes(size_t rows, size_t width, int n_sm);
cudaError_t launch_norm_grad(const NormGradArgs &a, int dtype, int n_sm, int *status, cudaStream_t s);

// Sums of the columns of a matrix, over all rows or over samples, dst (+)= the sums; work of column_sums_work_bytes()
struct ColumnSumArgs {
    MatArg m;
    size_t rows, width;
    SumOver over;
    const int32_t *offsets;
    uint32_t samples;
    bool accumulate;
    float *dst;
    void *work;
};
size_t column_sums_work_bytes(size_t rows, size_t width, int n_sm);
// early: beside the call's kernel before it, whose results are not used
cudaError_t launch_column_sums(const ColumnSumArgs &a, int dtype, int n_sm, bool early, cudaStream_t s);
// dst (+)= the sum of `runs` partial sums of columns, the first `width` of 3 * width words of each; beside the call's kernel before it, which began when
// they were there
cudaError_t launch_join_sums(const float *heads, uint32_t runs, size_t width, bool accumulate, float *dst, cudaStream_t s);

struct LinearMapArgs {
    MatArg x, dy;
    size_t rows, inputs, outputs;
    SumOver over;                  // SAMPLES or ROWS
    const int32_t *offsets;
    uint32_t samples;
    bool accumulate;
    float *weight, *bias;          // bias may be null
    void *work;
};
// whether the kernels can read a matrix where it lies
bool linear_map_aligned(const MatArg &m, size_t width, int dtype);
size_t linear_map_work_bytes(size_t rows, size_t inputs, size_t outputs, int dtype, bool samples, bool aligned, bool bias, int n_sm);
cudaError_t launch_linear_map(const LinearMapArgs &a, int dtype, int n_sm, int *status, cudaStream_t s);

}  // namespace fedhe
