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

// ---- rows too long for a block's registers: read twice, or three times ----

template <class T, int V>
__global__ void __launch_bounds__(256) norm_long_kernel(const NormArgs a) {
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
__global__ void __launch_bounds__(256) norm_long_grad_kernel(const NormGradArgs a) {
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

// ---- a row at a time, held in registers ----

// How a row is shared out: `threads` threads (a multiple of 32), each with K packs, `groups` of them in a block.
constexpr int HELD = 16;                                     // elements of a thread
constexpr uint32_t FORWARD_THREADS = 256, BACK_THREADS = 512;
struct RowPlan {
    uint32_t threads, groups;
};
// false: the row is too long for one block
inline bool plan_row(size_t width, uint32_t block, RowPlan &p) {
    const size_t t = (width + HELD - 1) / HELD;
    if (t > block) return false;
    p.threads = (uint32_t)(t + 31) / 32 * 32;
    p.groups = block / p.threads;
    return true;
}

__device__ __forceinline__ void group_sync(uint32_t group, uint32_t threads) {
    asm volatile("barrier.sync %0, %1;" ::"r"(group + 1), "r"(threads) : "memory");
}
// Sums over a group's threads, of N values each; `at`: a place of 32 N words that the group's last call but one used.
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float *at, uint32_t group, uint32_t threads) {
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = warp_sum(v[i]);
    if (threads == 32) return;
    const uint32_t t = threadIdx.x - group * threads, warps = threads / 32, lane = t & 31u;
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < N; i++) at[i * 32 + t / 32] = v[i];
    group_sync(group, threads);
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = warp_sum(lane < warps ? at[i * 32 + lane] : 0.0f);
}

template <class T, int V, int K>
__device__ __forceinline__ void load_row(Pack<T, V> (&p)[K], const T *row, uint32_t t, uint32_t threads, uint32_t width) {
#pragma unroll
    for (int k = 0; k < K; k++) {
        const uint32_t c = (k * threads + t) * V;
        if (c < width) p[k] = load_pack<T, V>(row + c);
        else
#pragma unroll
            for (int e = 0; e < V; e++) p[k].v[e] = from_f32<T>(0.0f);
    }
}
template <int V, int K>
__device__ __forceinline__ void load_weights(float (&w)[K][V], const void *p, int type, float otherwise, uint32_t t, uint32_t threads, uint32_t width) {
#pragma unroll
    for (int k = 0; k < K; k++)
#pragma unroll
        for (int e = 0; e < V; e++) {
            const uint32_t c = (k * threads + t) * V + e;
            w[k][e] = p && c < width ? load_weight(p, type, c) : otherwise;
        }
}

// Groups of threads take rows in turn; the weights stay in registers, and a row is asked for while the one before it is worked on.  Bounded by
// memory: 32768 rows of 4096 in bf16 ...
template <class T, int V>
__global__ void __launch_bounds__(FORWARD_THREADS, 3) norm_kernel(const NormArgs a, const RowPlan plan) {
    constexpr int K = HELD / V;
    __shared__ float sums[2][8][32];
    const uint32_t group = threadIdx.x / plan.threads, t = threadIdx.x % plan.threads, width = (uint32_t)a.width;
    if (group >= plan.groups) return;
    const size_t step = (size_t)gridDim.x * plan.groups;
    size_t r = (size_t)blockIdx.x * plan.groups + group;
    Pack<T, V> next[K];
    if (r < a.rows) load_row<T, V, K>(next, static_cast<const T *>(a.x.p) + r * a.x.stride, t, plan.threads, width);
    float w[K][V], b[K][V];
    load_weights<V, K>(w, a.weight, a.weight_type, 1.0f, t, plan.threads, width);
    load_weights<V, K>(b, a.bias, a.weight_type, 0.0f, t, plan.threads, width);
    const float n = (float)a.width;
    for (; r < a.rows; r += step) {
        float x[K][V], s[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < K; k++)
#pragma unroll
            for (int e = 0; e < V; e++) {
                x[k][e] = to_f32(next[k].v[e]);
                s[0] += x[k][e];
            }
        if (r + step < a.rows) load_row<T, V, K>(next, static_cast<const T *>(a.x.p) + (r + step) * a.x.stride, t, plan.threads, width);
        group_sum<1>(s, sums[0][group], group, plan.threads);
        const float mean = s[0] / n;
        s[0] = 0.0f;
#pragma unroll
        for (int k = 0; k < K; k++)
#pragma unroll
            for (int e = 0; e < V; e++) {
                x[k][e] -= mean;
                if ((k * plan.threads + t) * V + (V == 1 ? 0 : e) < width) s[0] = fmaf(x[k][e], x[k][e], s[0]);
            }
        group_sum<1>(s, sums[1][group], group, plan.threads);
        const float rstd = 1.0f / sqrtf(s[0] / n + a.eps);
        T *y = static_cast<T *>(a.y.p) + r * a.y.stride;
#pragma unroll
        for (int k = 0; k < K; k++) {
            const uint32_t c = (k * plan.threads + t) * V;
            if (c >= width) continue;
            Pack<T, V> o;
#pragma unroll
            for (int e = 0; e < V; e++) o.v[e] = from_f32<T>(fmaf(x[k][e] * rstd, w[k][e], b[k][e]));
            store_pack<T, V>(y + c, o);
        }
        if (t == 0) {
            a.mean[r] = mean;
            a.rstd[r] = rstd;
        }
    }
}

// The backward pass.  A block takes a run of rows, its groups parts of it in order; sums over rows stay in registers, and go to shared
// memory where a sample ends.  What the block leaves is a run's head, inner part and tail of every column (see Run).
template <class T, int V, bool SAMPLES>
__global__ void __launch_bounds__(BACK_THREADS, 1) norm_grad_kernel(const NormGradArgs a, const RowPlan plan, const RunsOut out) {
    constexpr int K = HELD / V;
    extern __shared__ float parts[];                 // [head, inner, tail][groups][2 planes][width]; without samples heads only
    __shared__ float sums[2][16][64];
    __shared__ int cuts[16];
    const uint32_t group = threadIdx.x / plan.threads, t = threadIdx.x % plan.threads, width = (uint32_t)a.width, run = blockIdx.x;
    const size_t lo = a.rows * run / out.runs, hi = a.rows * (run + 1) / out.runs;
    const auto part = [&](int what, uint32_t g, int plane) { return parts + ((size_t)(what * plan.groups + g) * 2 + plane) * width; };
    if (group < plan.groups) {
        const size_t begin = lo + (hi - lo) * group / plan.groups, end = lo + (hi - lo) * (group + 1) / plan.groups;
        const T *xs = static_cast<const T *>(a.x.p), *dys = static_cast<const T *>(a.dy.p);
        Pack<T, V> xn[K], gn[K];
        float mean_n = 0.0f, rstd_n = 0.0f;
        if (begin < end) {
            load_row<T, V, K>(xn, xs + begin * a.x.stride, t, plan.threads, width);
            load_row<T, V, K>(gn, dys + begin * a.dy.stride, t, plan.threads, width);
            mean_n = a.mean[begin];
            rstd_n = a.rstd[begin];
        }
        float w[K][V], sw[K][V], sb[K][V];
        load_weights<V, K>(w, a.weight, a.weight_type, 1.0f, t, plan.threads, width);
#pragma unroll
        for (int k = 0; k < K; k++)
#pragma unroll
            for (int e = 0; e < V; e++) sw[k][e] = sb[k][e] = 0.0f;
        const float n = 1.0f / (float)a.width;
        int cut = 0;
        SampleWalk walk;
        walk.begin = 0;
        walk.end = INT64_MAX;
        // what is summed so far is the head, or is added to the inner part
        const auto close = [&] {
#pragma unroll
            for (int k = 0; k < K; k++)
#pragma unroll
                for (int e = 0; e < V; e++) {
                    const uint32_t c = (k * plan.threads + t) * V + e;
                    if (c < width) {
                        if (cut) {
                            part(1, group, 0)[c] += fabsf(sw[k][e]);
                            part(1, group, 1)[c] += fabsf(sb[k][e]);
                        } else {
                            part(0, group, 0)[c] = sw[k][e];
                            part(0, group, 1)[c] = sb[k][e];
                            part(1, group, 0)[c] = part(1, group, 1)[c] = 0.0f;
                        }
                    }
                    sw[k][e] = sb[k][e] = 0.0f;
                }
            cut = 1;
        };
        if (SAMPLES) {
            walk.seek(a.offsets, a.samples, (int64_t)begin);
            if (walk.begin == (int64_t)begin) close();       // the run before this one ends with another sample
        }
        for (size_t r = begin; r < end; r++) {
            float x[K][V], g[K][V], s[2] = {0.0f, 0.0f};
            const float mean = mean_n, rstd = rstd_n;
#pragma unroll
            for (int k = 0; k < K; k++)
#pragma unroll
                for (int e = 0; e < V; e++) {
                    x[k][e] = (to_f32(xn[k].v[e]) - mean) * rstd;
                    g[k][e] = to_f32(gn[k].v[e]);
                    const float q = g[k][e] * w[k][e];       // behind the row's end g is 0
                    s[0] += q;
                    s[1] = fmaf(q, x[k][e], s[1]);
                }
            if (r + 1 < end) {
                load_row<T, V, K>(xn, xs + (r + 1) * a.x.stride, t, plan.threads, width);
                load_row<T, V, K>(gn, dys + (r + 1) * a.dy.stride, t, plan.threads, width);
                mean_n = a.mean[r + 1];
                rstd_n = a.rstd[r + 1];
            }
            if (SAMPLES && (int64_t)r >= walk.end) {
                close();
                walk.next((int64_t)r);
            }
            if (!SAMPLES || (int64_t)r >= walk.begin) {
#pragma unroll
                for (int k = 0; k < K; k++)
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        sw[k][e] = fmaf(g[k][e], x[k][e], sw[k][e]);
                        sb[k][e] += g[k][e];
                    }
            }
            group_sum<2>(s, sums[r & 1][group], group, plan.threads);
            const float ma = s[0] * n, man = s[1] * n;
            T *dx = static_cast<T *>(a.dx.p) + r * a.dx.stride;
#pragma unroll
            for (int k = 0; k < K; k++) {
                const uint32_t c = (k * plan.threads + t) * V;
                if (c >= width) continue;
                Pack<T, V> o;
#pragma unroll
                for (int e = 0; e < V; e++) o.v[e] = from_f32<T>(rstd * (fmaf(g[k][e], w[k][e], -ma) - x[k][e] * man));
                store_pack<T, V>(dx + c, o);
            }
        }
        // what is left is the tail, or the head of a run without a cut
#pragma unroll
        for (int k = 0; k < K; k++)
#pragma unroll
            for (int e = 0; e < V; e++) {
                const uint32_t c = (k * plan.threads + t) * V + e;
                if (c < width) {
                    part(cut ? 2 : 0, group, 0)[c] = sw[k][e];
                    part(cut ? 2 : 0, group, 1)[c] = sb[k][e];
                }
            }
        if (SAMPLES && t == 0) cuts[group] = cut;
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 2 * width; i += BACK_THREADS) {
        const int plane = i >= width;
        const uint32_t c = plane ? i - width : i;
        Run all{0.0f, 0.0f, 0.0f, 0};
        for (uint32_t g = 0; g < plan.groups; g++) {
            if (!SAMPLES) all.head += part(0, g, plane)[c];
            else if (cuts[g]) all.join(Run{part(0, g, plane)[c], part(1, g, plane)[c], part(2, g, plane)[c], 1});
            else all.join(Run{part(0, g, plane)[c], 0.0f, 0.0f, 0});
        }
        out.of(run, 0, plane)[c] = all.head;
        if (SAMPLES) {
            out.of(run, 1, plane)[c] = all.inner;
            out.of(run, 2, plane)[c] = all.tail;
            if (i == 0) *out.cut(run) = all.cut;
        }
    }
}

// ---- sums of a matrix by themselves ----

constexpr int SUM_COLS = 32, SUM_WARPS = 8;

// Columns of one matrix (X = false: the sums of m) or of a product (X = true: dy n, and dy, of rows too long for the kernel above).  A block takes SUM_COLS packs of
// columns and a run of rows; its warps take parts of the run in order, which join in shared memory.
template <class T, int V, bool X>
__global__ void __launch_bounds__(SUM_COLS * SUM_WARPS) sums_kernel(const MatArg m, const MatArg xm, const float *mean, const float *rstd, const size_t rows,
                                                                    const size_t width, const SumOver over, const int32_t *offsets,
                                                                    const uint32_t samples, const RunsOut out) {
    constexpr int P = X ? 2 : 1, AHEAD = 4;
    __shared__ float runs[3][SUM_WARPS][V][SUM_COLS];
    __shared__ int cuts[SUM_WARPS];
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
    walk.begin = 0;
    walk.end = INT64_MAX;
    if (over == SumOver::SAMPLES) {
        walk.seek(offsets, samples, (int64_t)begin);
        cut = walk.begin == (int64_t)begin;  // the run before this one ends with another sample
    }
    for (size_t r0 = begin; r0 < end; r0 += AHEAD) {
        Pack<T, V> g[AHEAD], x[X ? AHEAD : 1];
#pragma unroll
        for (int j = 0; j < AHEAD; j++)
            if (r0 + j < end && col < width) {
                g[j] = load_pack<T, V>(static_cast<const T *>(m.p) + (r0 + j) * m.stride + col);
                if (X) x[X ? j : 0] = load_pack<T, V>(static_cast<const T *>(xm.p) + (r0 + j) * xm.stride + col);
            }
#pragma unroll
        for (int j = 0; j < AHEAD; j++) {
            const size_t r = r0 + j;
            if (r >= end) break;
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
            if ((int64_t)r < walk.begin || col >= width) continue;      // no sample's row
            if (over == SumOver::ROWS) {
#pragma unroll
                for (int e = 0; e < V; e++) inner[P - 1][e] += fabsf(to_f32(g[j].v[e]));
            } else {
                if (X) {
                    const float mu = mean[r], rs = rstd[r];
#pragma unroll
                    for (int e = 0; e < V; e++) sum[0][e] = fmaf(to_f32(g[j].v[e]), (to_f32(x[X ? j : 0].v[e]) - mu) * rs, sum[0][e]);
                }
#pragma unroll
                for (int e = 0; e < V; e++) sum[P - 1][e] += to_f32(g[j].v[e]);
            }
        }
    }
    if (lane == 0) cuts[warp] = cut;
#pragma unroll
    for (int p = 0; p < P; p++) {
        if (p) __syncthreads();
#pragma unroll
        for (int e = 0; e < V; e++) {
            runs[0][warp][e][lane] = cut ? head[p][e] : sum[p][e];
            runs[1][warp][e][lane] = inner[p][e];
            runs[2][warp][e][lane] = cut ? sum[p][e] : 0.0f;
        }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < V * SUM_COLS; i += SUM_COLS * SUM_WARPS) {
            // column of the block: pack and element in it
            const uint32_t l = i / V, e = i % V;
            Run all{0.0f, 0.0f, 0.0f, 0};
            for (int w = 0; w < SUM_WARPS; w++) all.join(Run{runs[0][w][e][l], runs[1][w][e][l], runs[2][w][e][l], cuts[w]});
            const size_t c = (size_t)blockIdx.x * SUM_COLS * V + i;
            if (c < width) {
                out.of(run, 0, p)[c] = all.head;
                out.of(run, 1, p)[c] = all.inner;
                out.of(run, 2, p)[c] = all.tail;
            }
            if (p == 0 && i == 0 && blockIdx.x == 0) *out.cut(run) = all.cut;
        }
    }
}

// Joins all runs of a column: each warp a part of them in order, then the warps' results.
constexpr int JOIN_WARPS = 32;
template <bool MAGNITUDES>
__global__ void __launch_bounds__(32 * JOIN_WARPS) sums_join_kernel(const RunsOut in, const bool accumulate, float *dst0, float *dst1) {
    __shared__ Run runs[JOIN_WARPS][33];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x / 32;
    const int plane = blockIdx.y;
    const size_t col = (size_t)blockIdx.x * 32 + lane;
    float *dst = plane ? dst1 : dst0;
    Run all{0.0f, 0.0f, 0.0f, 0};
    const uint32_t begin = in.runs * warp / JOIN_WARPS, end = in.runs * (warp + 1) / JOIN_WARPS;
    if (col < in.width)
        for (uint32_t r0 = begin; r0 < end; r0 += 4) {
            Run part[4];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                part[j] = Run{0.0f, 0.0f, 0.0f, 0};
                if (r0 + j >= end) continue;
                part[j].head = in.of(r0 + j, 0, plane)[col];
                if (MAGNITUDES) {
                    part[j].inner = in.of(r0 + j, 1, plane)[col];
                    part[j].tail = in.of(r0 + j, 2, plane)[col];
                    part[j].cut = *in.cut(r0 + j);
                }
            }
#pragma unroll
            for (int j = 0; j < 4; j++) all.join(part[j]);
        }
    runs[warp][lane] = all;
    __syncthreads();
    if (warp || col >= in.width) return;
#pragma unroll 4
    for (int w = 1; w < JOIN_WARPS; w++) all.join(runs[w][lane]);
    const float v = MAGNITUDES ? fabsf(all.head) + all.inner + fabsf(all.tail) : all.head;
    dst[col] = accumulate ? dst[col] + v : v;
}

template <class T>
bool wide_rows(const void *p, size_t stride, size_t width) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % WIDE<T> == 0 && width % WIDE<T> == 0;
}

// Runs of rows: a block for each SM, or less.
inline uint32_t sum_runs(size_t rows, int n_sm) { return (uint32_t)(rows < 1 ? 1 : rows < (size_t)n_sm ? rows : n_sm); }
inline size_t runs_bytes(size_t rows, size_t width, int planes, int n_sm) {
    const size_t runs = sum_runs(rows, n_sm);
    return runs * 3 * planes * width * sizeof(float) + runs * sizeof(int);
}

cudaError_t join_runs(const RunsOut &runs, bool magnitudes, bool accumulate, float *dst0, float *dst1, cudaStream_t s) {
    const dim3 grid(blocks_for(runs.width, 32), runs.planes);
    if (magnitudes) sums_join_kernel<true><<<grid, 32 * JOIN_WARPS, 0, s>>>(runs, accumulate, dst0, dst1);
    else sums_join_kernel<false><<<grid, 32 * JOIN_WARPS, 0, s>>>(runs, accumulate, dst0, dst1);
    return FEDHE_LAUNCHED();
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
    const cudaError_t rc = FEDHE_LAUNCHED();
    return rc != cudaSuccess ? rc : join_runs(out, over != SumOver::ALL, accumulate, dst0, dst1, s);
}

inline uint32_t row_threads(size_t packs) { return packs >= 256 ? 256 : (uint32_t)(packs + 31) / 32 * 32; }

template <class T>
cudaError_t norm_of(const NormArgs &a, int n_sm, cudaStream_t s) {
    if (a.rows == 0) return cudaSuccess;
    const bool wide = wide_rows<T>(a.x.p, a.x.stride, a.width) && wide_rows<T>(a.y.p, a.y.stride, a.width);
    RowPlan plan;
    if (plan_row(a.width, FORWARD_THREADS, plan)) {
        const size_t blocks = (a.rows + plan.groups - 1) / plan.groups, most = (size_t)3 * n_sm;
        const unsigned grid = (unsigned)(blocks < most ? blocks : most);
        if (wide) norm_kernel<T, WIDE<T>><<<grid, FORWARD_THREADS, 0, s>>>(a, plan);
        else norm_kernel<T, 1><<<grid, FORWARD_THREADS, 0, s>>>(a, plan);
    } else if (wide) {
        norm_long_kernel<T, WIDE<T>><<<(unsigned)a.rows, row_threads(a.width / WIDE<T>), 0, s>>>(a);
    } else {
        norm_long_kernel<T, 1><<<(unsigned)a.rows, row_threads(a.width), 0, s>>>(a);
    }
    return FEDHE_LAUNCHED();
}

template <class T, int V, bool SAMPLES>
cudaError_t norm_grad_go(const NormGradArgs &a, const RowPlan &plan, int n_sm, cudaStream_t s) {
    const RunsOut out{static_cast<float *>(a.work), sum_runs(a.rows, n_sm), a.width, 2};
    const size_t bytes = (size_t)(SAMPLES ? 3 : 1) * plan.groups * 2 * a.width * sizeof(float);
    cudaError_t rc = cudaFuncSetAttribute(norm_grad_kernel<T, V, SAMPLES>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (rc != cudaSuccess) return rc;
    norm_grad_kernel<T, V, SAMPLES><<<out.runs, BACK_THREADS, bytes, s>>>(a, plan, out);
    rc = FEDHE_LAUNCHED();
    return rc != cudaSuccess ? rc : join_runs(out, SAMPLES, false, a.dweight, a.dbias, s);
}

template <class T>
cudaError_t norm_grad_of(const NormGradArgs &a, int n_sm, cudaStream_t s) {
    const bool wide = wide_rows<T>(a.x.p, a.x.stride, a.width) && wide_rows<T>(a.dy.p, a.dy.stride, a.width) &&
                      wide_rows<T>(a.dx.p, a.dx.stride, a.width);
    RowPlan plan;
    if (plan_row(a.width, BACK_THREADS, plan)) {
        if (a.over == SumOver::SAMPLES) return wide ? norm_grad_go<T, WIDE<T>, true>(a, plan, n_sm, s) : norm_grad_go<T, 1, true>(a, plan, n_sm, s);
        return wide ? norm_grad_go<T, WIDE<T>, false>(a, plan, n_sm, s) : norm_grad_go<T, 1, false>(a, plan, n_sm, s);
    }
    if (a.rows) {
        if (wide) norm_long_grad_kernel<T, WIDE<T>><<<(unsigned)a.rows, row_threads(a.width / WIDE<T>), 0, s>>>(a);
        else norm_long_grad_kernel<T, 1><<<(unsigned)a.rows, row_threads(a.width), 0, s>>>(a);
        const cudaError_t rc = FEDHE_LAUNCHED();
        if (rc != cudaSuccess) return rc;
    }
    return sums<T, true>(a.dy, a.x, a.mean, a.rstd, a.rows, a.width, a.over, a.offsets, a.samples, false, a.dweight, a.dbias, a.work, n_sm, s);
}

}  // namespace

cudaError_t launch_norm(const NormArgs &a, int dtype, int n_sm, cudaStream_t s) {
    return dtype == HE_F32 ? norm_of<float>(a, n_sm, s) : dtype == HE_BF16 ? norm_of<__nv_bfloat16>(a, n_sm, s) : norm_of<__half>(a, n_sm, s);
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
