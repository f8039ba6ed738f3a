// Layer norm and its backward pass, with the sums over rows that make the weights' gradients or, where rows belong to samples, the
// weights' entries of the sensitivity map.
//
//   y = n gamma + beta,  n = (x - mean) rstd,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   dx = rstd (a - mean(a) - n mean(a n)),  a = dy gamma
//   dgamma = sum_t dy n,  dbeta = sum_t dy;   with samples  sum_k |sum_{t in k} dy n|,  sum_k |sum_{t in k} dy|
//
// All sums are in fp32.  Everything is bounded by reading the inputs and writing the results once.
#include "fedhe_map.cuh"

namespace fedhe {

namespace {

// Sum over a block of up to 32 warps; the same value in every thread.  `at`: 32 words.
__device__ __forceinline__ float block_sum(float v, float *at) {
    v = warp_sum(v);
    if ((threadIdx.x & 31u) == 0) at[threadIdx.x / 32] = v;
    __syncthreads();
    v = (threadIdx.x & 31u) < blockDim.x / 32 ? at[threadIdx.x & 31u] : 0.0f;
    v = warp_sum(v);
    __syncthreads();
    return v;
}

template <class T, int V>
__global__ void __launch_bounds__(256) norm_kernel(const NormArgs a) {
    __shared__ float at[32];
    const size_t r = blockIdx.x;
    const T *x = static_cast<const T *>(a.x.p) + r * a.x.stride;
    T *y = static_cast<T *>(a.y.p) + r * a.y.stride;
    const size_t step = (size_t)blockDim.x * V, first = (size_t)threadIdx.x * V;
    float sum = 0.0f;
    for (size_t i = first; i < a.width; i += step) {
        const Pack<T, V> p = load_pack<T, V>(x + i);
#pragma unroll
        for (int e = 0; e < V; e++) sum += to_f32(p.v[e]);
    }
    const float mean = block_sum(sum, at) / (float)a.width;
    sum = 0.0f;
    for (size_t i = first; i < a.width; i += step) {
        const Pack<T, V> p = load_pack<T, V>(x + i);
#pragma unroll
        for (int e = 0; e < V; e++) {
            const float d = to_f32(p.v[e]) - mean;
            sum = fmaf(d, d, sum);
        }
    }
    const float rstd = 1.0f / sqrtf(block_sum(sum, at) / (float)a.width + a.eps);
    for (size_t i = first; i < a.width; i += step) {
        const Pack<T, V> p = load_pack<T, V>(x + i);
        Pack<T, V> o;
#pragma unroll
        for (int e = 0; e < V; e++) {
            const float n = (to_f32(p.v[e]) - mean) * rstd;
            const float g = a.weight ? load_weight(a.weight, a.weight_type, i + e) : 1.0f;
            o.v[e] = from_f32<T>(fmaf(n, g, a.bias ? load_weight(a.bias, a.weight_type, i + e) : 0.0f));
        }
        store_pack<T, V>(y + i, o);
    }
    if (threadIdx.x == 0) {
        a.mean[r] = mean;
        a.rstd[r] = rstd;
    }
}

template <class T, int V>
__global__ void __launch_bounds__(256) norm_grad_kernel(const NormGradArgs a) {
    __shared__ float at[32];
    const size_t r = blockIdx.x;
    const T *x = static_cast<const T *>(a.x.p) + r * a.x.stride, *dy = static_cast<const T *>(a.dy.p) + r * a.dy.stride;
    T *dx = static_cast<T *>(a.dx.p) + r * a.dx.stride;
    const float mean = a.mean[r], rstd = a.rstd[r];
    const size_t step = (size_t)blockDim.x * V, first = (size_t)threadIdx.x * V;
    float sa = 0.0f, san = 0.0f;
    for (size_t i = first; i < a.width; i += step) {
        const Pack<T, V> p = load_pack<T, V>(x + i), g = load_pack<T, V>(dy + i);
#pragma unroll
        for (int e = 0; e < V; e++) {
            const float n = (to_f32(p.v[e]) - mean) * rstd, w = a.weight ? load_weight(a.weight, a.weight_type, i + e) : 1.0f;
            const float b = to_f32(g.v[e]) * w;
            sa += b;
            san = fmaf(b, n, san);
        }
    }
    sa = block_sum(sa, at) / (float)a.width;
    san = block_sum(san, at) / (float)a.width;
    for (size_t i = first; i < a.width; i += step) {
        const Pack<T, V> p = load_pack<T, V>(x + i), g = load_pack<T, V>(dy + i);
        Pack<T, V> o;
#pragma unroll
        for (int e = 0; e < V; e++) {
            const float n = (to_f32(p.v[e]) - mean) * rstd, w = a.weight ? load_weight(a.weight, a.weight_type, i + e) : 1.0f;
            o.v[e] = from_f32<T>(rstd * (fmaf(to_f32(g.v[e]), w, -sa) - n * san));
        }
        store_pack<T, V>(dx + i, o);
    }
}

// ---- sums over rows, within samples ----
//
// A run of consecutive rows is summed to three numbers of a column: `head`, the sum of what belongs to the sample that the run
// begins in; `tail`, of the sample that it ends in; `inner`, the magnitudes of the samples between, which the run holds whole.  A run
// inside one sample has only a head (cut = 0).  Two runs that follow one another join to such a run again, in any grouping, so that rows
// can be shared out evenly however long the samples are; the order of all additions is fixed by the shapes.
struct Run {
    float head, inner, tail;
    int cut;
    __device__ __forceinline__ void join(const Run &o) {
        if (!cut) {
            head += o.head;
            if (o.cut) {
                inner = o.inner;
                tail = o.tail;
                cut = 1;
            }
        } else if (!o.cut) {
            tail += o.head;
        } else {
            inner += fabsf(tail + o.head) + o.inner;
            tail = o.tail;
        }
    }
};

// The runs that a grid of `runs` thread blocks works on, and what they leave: [runs][head, inner, tail][planes][width], then a word for each
// run's cut.
struct RunsOut {
    float *p;
    uint32_t runs;
    size_t width;
    int planes;
    __device__ __forceinline__ float *of(uint32_t run, int what, int plane) const { return p + (((size_t)run * 3 + what) * planes + plane) * width; }
    __device__ __forceinline__ int *cut(uint32_t run) const { return reinterpret_cast<int *>(p + (size_t)runs * 3 * planes * width) + run; }
};

constexpr int SUM_COLS = 32, SUM_WARPS = 8;

// Columns of one matrix (X = false: the sums of m) or of a product (X = true: dy n, and dy).  A block takes SUM_COLS packs of
// columns and a run of rows; its warps take parts of the run in order, which join in shared memory.
template <class T, int V, bool X>
__global__ void __launch_bounds__(SUM_COLS * SUM_WARPS) sums_kernel(const MatArg m, const MatArg xm, const float *mean, const float *rstd, const size_t rows,
                                                                    const size_t width, const SumOver over, const int32_t *offsets,
                                                                    const uint32_t samples, const RunsOut out) {
    constexpr int P = X ? 2 : 1;
    __shared__ Run runs[SUM_WARPS][SUM_COLS];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x / 32, run = blockIdx.y;
    const size_t col = ((size_t)blockIdx.x * SUM_COLS + lane) * V;
    const size_t lo = rows * run / out.runs, hi = rows * (run + 1) / out.runs;
    const size_t begin = lo + (hi - lo) * warp / SUM_WARPS, end = lo + (hi - lo) * (warp + 1) / SUM_WARPS;
    float sum[P][V], head[P][V], inner[P][V];
#pragma unroll
    for (int p = 0; p < P; p++)
#pragma unroll
        for (int e = 0; e < V; e++) sum[p][e] = head[p][e] = inner[p][e] = 0.0f;
    int cut = over == SumOver::ROWS;         // magnitudes of rows: all of them are inner
    SampleWalk walk;
    if (over == SumOver::SAMPLES) {
        walk.seek(offsets, samples, (int64_t)begin);
        cut = walk.begin == (int64_t)begin;  // the run before this one ends with another sample
    }
    if (over != SumOver::SAMPLES) walk.end = INT64_MAX;
    for (size_t r = begin; r < end; r++) {
        if ((int64_t)r >= walk.end) {
#pragma unroll
            for (int p = 0; p < P; p++)
#pragma unroll
                for (int e = 0; e < V; e++) {
                    if (cut) inner[p][e] += fabsf(sum[p][e]);
                    else head[p][e] = sum[p][e];
                    sum[p][e] = 0.0f;
                }
            cut = 1;
            walk.next((int64_t)r);
        }
        if (over == SumOver::SAMPLES && (int64_t)r < walk.begin) continue;      // no sample's row
        if (col < width) {
            const Pack<T, V> g = load_pack<T, V>(static_cast<const T *>(m.p) + r * m.stride + col);
            if (X) {
                const Pack<T, V> x = load_pack<T, V>(static_cast<const T *>(xm.p) + r * xm.stride + col);
                const float mu = mean[r], rs = rstd[r];
#pragma unroll
                for (int e = 0; e < V; e++) sum[0][e] = fmaf(to_f32(g.v[e]), (to_f32(x.v[e]) - mu) * rs, sum[0][e]);
            }
#pragma unroll
            for (int e = 0; e < V; e++) sum[P - 1][e] += to_f32(g.v[e]);
        }
        if (over == SumOver::ROWS)
#pragma unroll
            for (int p = 0; p < P; p++)
#pragma unroll
                for (int e = 0; e < V; e++) {
                    inner[p][e] += fabsf(sum[p][e]);
                    sum[p][e] = 0.0f;
                }
    }
#pragma unroll
    for (int p = 0; p < P; p++)
#pragma unroll
        for (int e = 0; e < V; e++) {
            runs[warp][lane] = cut ? Run{head[p][e], inner[p][e], sum[p][e], 1} : Run{sum[p][e], 0.0f, 0.0f, 0};
            __syncthreads();
            if (warp == 0) {
                Run all = runs[0][lane];
                for (int w = 1; w < SUM_WARPS; w++) all.join(runs[w][lane]);
                if (col + e < width) {
                    out.of(run, 0, p)[col + e] = all.head;
                    out.of(run, 1, p)[col + e] = all.inner;
                    out.of(run, 2, p)[col + e] = all.tail;
                }
                if (blockIdx.x == 0 && lane == 0 && p == 0 && e == 0) *out.cut(run) = all.cut;
            }
            __syncthreads();
        }
}

// Joins all runs of a column: each warp a part of them in order, then the warps' results.
__global__ void __launch_bounds__(1024) sums_join_kernel(const RunsOut in, const bool magnitudes, const bool accumulate, float *dst0, float *dst1) {
    __shared__ Run runs[32][33];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x / 32;
    const int plane = blockIdx.y;
    const size_t col = (size_t)blockIdx.x * 32 + lane;
    float *dst = plane ? dst1 : dst0;
    Run all{0.0f, 0.0f, 0.0f, 0};
    const uint32_t begin = in.runs * warp / 32, end = in.runs * (warp + 1) / 32;
    if (col < in.width)
        for (uint32_t r = begin; r < end; r++)
            all.join(Run{in.of(r, 0, plane)[col], in.of(r, 1, plane)[col], in.of(r, 2, plane)[col], *in.cut(r)});
    runs[warp][lane] = all;
    __syncthreads();
    if (warp || col >= in.width || !dst) return;
    for (int w = 1; w < 32; w++) all.join(runs[w][lane]);
    const float v = magnitudes ? fabsf(all.head) + all.inner + fabsf(all.tail) : all.head;
    dst[col] = accumulate ? dst[col] + v : v;
}

template <class T>
bool wide_rows(const void *p, size_t stride, size_t width) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % WIDE<T> == 0 && width % WIDE<T> == 0;
}

inline uint32_t sum_runs(size_t rows, int n_sm) {
    const size_t most = (size_t)2 * n_sm, r = (rows + SUM_WARPS - 1) / SUM_WARPS;
    return (uint32_t)(r < 1 ? 1 : r < most ? r : most);
}
inline size_t runs_bytes(size_t rows, size_t width, int planes, int n_sm) {
    const size_t runs = sum_runs(rows, n_sm);
    return runs * 3 * planes * width * sizeof(float) + runs * sizeof(int);
}

template <class T, bool X>
cudaError_t sums(const MatArg &m, const MatArg &x, const float *mean, const float *rstd, size_t rows, size_t width, SumOver over,
                 const int32_t *offsets, uint32_t samples, bool accumulate, float *dst0, float *dst1, void *work, int n_sm, cudaStream_t s) {
    const bool wide = wide_rows<T>(m.p, m.stride, width) && (!X || wide_rows<T>(x.p, x.stride, width));
    const RunsOut out{static_cast<float *>(work), sum_runs(rows, n_sm), width, X ? 2 : 1};
    const unsigned cols = SUM_COLS * (wide ? WIDE<T> : 1);
    const dim3 grid(blocks_for(width, cols), out.runs);
    if (wide) sums_kernel<T, WIDE<T>, X><<<grid, SUM_COLS * SUM_WARPS, 0, s>>>(m, x, mean, rstd, rows, width, over, offsets, samples, out);
    else sums_kernel<T, 1, X><<<grid, SUM_COLS * SUM_WARPS, 0, s>>>(m, x, mean, rstd, rows, width, over, offsets, samples, out);
    cudaError_t rc = FEDHE_LAUNCHED();
    if (rc != cudaSuccess) return rc;
    sums_join_kernel<<<dim3(blocks_for(width, 32), X ? 2 : 1), 1024, 0, s>>>(out, over != SumOver::ALL, accumulate, dst0, dst1);
    return FEDHE_LAUNCHED();
}

inline uint32_t row_threads(size_t packs) { return packs >= 256 ? 256 : (uint32_t)(packs + 31) / 32 * 32; }

template <class T>
cudaError_t norm_of(const NormArgs &a, cudaStream_t s) {
    if (a.rows == 0) return cudaSuccess;
    const bool wide = wide_rows<T>(a.x.p, a.x.stride, a.width) && wide_rows<T>(a.y.p, a.y.stride, a.width);
    if (wide) norm_kernel<T, WIDE<T>><<<(unsigned)a.rows, row_threads(a.width / WIDE<T>), 0, s>>>(a);
    else norm_kernel<T, 1><<<(unsigned)a.rows, row_threads(a.width), 0, s>>>(a);
    return FEDHE_LAUNCHED();
}

template <class T>
cudaError_t norm_grad_of(const NormGradArgs &a, int n_sm, cudaStream_t s) {
    if (a.rows) {
        const bool wide = wide_rows<T>(a.x.p, a.x.stride, a.width) && wide_rows<T>(a.dy.p, a.dy.stride, a.width) &&
                          wide_rows<T>(a.dx.p, a.dx.stride, a.width);
        if (wide) norm_grad_kernel<T, WIDE<T>><<<(unsigned)a.rows, row_threads(a.width / WIDE<T>), 0, s>>>(a);
        else norm_grad_kernel<T, 1><<<(unsigned)a.rows, row_threads(a.width), 0, s>>>(a);
        const cudaError_t rc = FEDHE_LAUNCHED();
        if (rc != cudaSuccess) return rc;
    }
    return sums<T, true>(a.dy, a.x, a.mean, a.rstd, a.rows, a.width, a.over, a.offsets, a.samples, false, a.dweight, a.dbias, a.work, n_sm, s);
}

}  // namespace

cudaError_t launch_norm(const NormArgs &a, int dtype, int n_sm, cudaStream_t s) {
    (void)n_sm;
    return dtype == HE_F32 ? norm_of<float>(a, s) : dtype == HE_BF16 ? norm_of<__nv_bfloat16>(a, s) : norm_of<__half>(a, s);
}

size_t norm_grad_work_bytes(size_t rows, size_t width, int n_sm) { return runs_bytes(rows, width, 2, n_sm); }

cudaError_t launch_norm_grad(const NormGradArgs &a, int dtype, int n_sm, cudaStream_t s) {
    return dtype == HE_F32    ? norm_grad_of<float>(a, n_sm, s)
           : dtype == HE_BF16 ? norm_grad_of<__nv_bfloat16>(a, n_sm, s)
                              : norm_grad_of<__half>(a, n_sm, s);
}

size_t column_sums_work_bytes(size_t rows, size_t width, int n_sm) { return runs_bytes(rows, width, 1, n_sm); }

cudaError_t launch_column_sums(const ColumnSumArgs &a, int dtype, int n_sm, cudaStream_t s) {
    const MatArg none{nullptr, 0};
    const auto go = [&](auto t) {
        return sums<decltype(t), false>(a.m, none, nullptr, nullptr, a.rows, a.width, a.over, a.offsets, a.samples, a.accumulate, a.dst, nullptr,
                                        a.work, n_sm, s);
    };
    return dtype == HE_F32 ? go(0.0f) : dtype == HE_BF16 ? go(__nv_bfloat16()) : go(__half());
}

}  // namespace fedhe
