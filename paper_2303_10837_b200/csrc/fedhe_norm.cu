// Layer norm and its backward pass, with the sums over rows that make the weights' gradients or, where rows belong to samples, the
// weights' entries of the sensitivity map.
//
//   y = n gamma + beta,  n = (x - mean) rstd,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   dx = rstd (a - mean(a) - n mean(a n)),  a = dy gamma
//   dgamma = sum_t dy n,  dbeta = sum_t dy;   with samples  sum_k |sum_{t in k} dy n|,  sum_k |sum_{t in k} dy|
//
// All sums are in fp32.  Everything would be bounded by reading the inputs and writing the results once: 32768 rows of 4096 in bf16 take 94 us, 5.7
// TB/s (98 by themselves), the backward pass of 16384 rows 88; what is left is the sums over a row, for which its threads wait, and with few rows the
// beginning and the end.
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

// How a row is shared out: `threads` threads (a multiple of 32), each with `held` elements, `groups` of them in a block.  A group's rows come to
// shared memory by bulk copies, `depth` rows ahead: that many loads in registers would leave room for few warps (32768 rows of 4096 in
// bf16: one ahead in registers 176 us, by copies 119).
struct RowPlan {
    uint32_t threads, groups, depth;
    uint32_t room;                                           // bytes of a row in shared memory
};
constexpr uint32_t MOST_DEPTH = 4;
// false: the row is too long for one block
inline bool plan_row(size_t width, size_t element, uint32_t block, uint32_t held, uint32_t rows_at_once, size_t ring, RowPlan &p) {
    const size_t t = (width + held - 1) / held;
    if (t > block) return false;
    p.threads = (uint32_t)(t + 31) / 32 * 32;
    p.groups = block / p.threads;
    p.room = (uint32_t)((width * element + 15) / 16 * 16 + 16);
    const size_t depth = ring / ((size_t)p.groups * rows_at_once * p.room);
    p.depth = (uint32_t)(depth < MOST_DEPTH ? depth : MOST_DEPTH);
    return p.depth > 0;
}

__device__ __forceinline__ void group_sync(uint32_t group, uint32_t threads) {
    if (threads == 32) __syncwarp();
    else asm volatile("barrier.sync %0, %1;" ::"r"(group + 1), "r"(threads) : "memory");
}

// The rows of a matrix as copies see them: whole 16 bytes, none outside the memory that the matrix spans.  EVEN: every row begins and ends on 16
// bytes, and nothing is left over.
template <class T, bool EVEN>
struct Rows {
    const uint8_t *p;
    size_t pitch;                                            // bytes from row to row
    uintptr_t low, high;                                     // whole 16 bytes of the matrix
    uint32_t bytes;                                          // of a row
    __device__ __forceinline__ Rows(const MatArg &m, size_t rows, uint32_t width)
        : p(static_cast<const uint8_t *>(m.p)), pitch(m.stride * sizeof(T)), bytes(width * (uint32_t)sizeof(T)) {
        low = (reinterpret_cast<uintptr_t>(p) + 15) & ~(uintptr_t)15;
        high = (reinterpret_cast<uintptr_t>(p + (rows - 1) * pitch) + bytes) & ~(uintptr_t)15;
    }
    __device__ __forceinline__ uintptr_t at(size_t r) const { return reinterpret_cast<uintptr_t>(p) + r * pitch; }
    // what is copied of the row at an address
    __device__ __forceinline__ uintptr_t from(uintptr_t row) const {
        const uintptr_t a = row & ~(uintptr_t)15;
        return EVEN ? row : a < low ? low : a;
    }
    __device__ __forceinline__ uint32_t size(uintptr_t row) const {
        if (EVEN) return bytes;
        uintptr_t e = (row + bytes + 15) & ~(uintptr_t)15;
        if (e > high) e = high;
        return e > from(row) ? (uint32_t)(e - from(row)) : 0;
    }
    __device__ __forceinline__ void copy(uintptr_t row, uint32_t room, uint32_t bar) const {
        const uint32_t n = size(row);
        if (!EVEN && !n) return;
        const uint32_t to = EVEN ? room : room + (uint32_t)(from(row) - (row & ~(uintptr_t)15));
        bulk_copy(to, from(row), n, bar);
    }
    // A thread's packs of a row that has been copied; zeros behind its end.  A matrix's first and last bytes that no copy brings come from where they are.
    template <int V, int K>
    __device__ __forceinline__ void get(Pack<T, V> (&v)[K], uintptr_t row, const uint8_t *room, uint32_t t, uint32_t threads, uint32_t width) const {
        const T *in = reinterpret_cast<const T *>(EVEN ? room : room + (row & 15)) + t * V;
#pragma unroll
        for (int k = 0; k < K; k++) {
            if ((k * threads + t) * V < width) v[k] = load_pack<T, V>(in + k * threads * V);
            else
#pragma unroll
                for (int e = 0; e < V; e++) v[k].v[e] = from_f32<T>(0.0f);
        }
        if (!EVEN && (row < low || row + bytes > high)) {
#pragma unroll
            for (int i = 0; i < K * V; i++) {
                const uint32_t c = (i / V * threads + t) * V + i % V;
                const uintptr_t x = row + c * sizeof(T);
                if (c < width && (x < from(row) || x >= from(row) + size(row))) v[i / V].v[i % V] = *reinterpret_cast<const T *>(x);
            }
        }
    }
};

// The sum over the first `lanes` lanes (a power of two; the others hold the same again); the same bits in every lane.
__device__ __forceinline__ float few_sum(float v, uint32_t lanes) {
    for (uint32_t o = lanes / 2; o; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ uint32_t power_above(uint32_t n) { return n <= 1 ? 1 : 2u << (31 - __clz((int)(n - 1))); }
// sum / n, given 1 / n rounded: the product and what is left over.  Exact where the quotient is.
__device__ __forceinline__ float quotient(float sum, float n, float part) {
    const float q = sum * part;
    return fmaf(fmaf(-q, n, sum), part, q);
}
// 1 / sqrt(v): rsqrtf and a step of Newton's iteration
__device__ __forceinline__ float inverse_root(float v) {
    const float r = rsqrtf(v);
    return v > 0.0f && r > 0.0f ? r * fmaf(-0.5f * v * r, r, 1.5f) : r;
}

// A thread's elements, two and two: element e of pack k is the (k V + e) % 2 one of pair (k V + e) / 2.
template <int V, int K>
__device__ __forceinline__ void load_weights(F2 (&w)[K * V / 2], const void *p, int type, float otherwise, uint32_t t, uint32_t threads, uint32_t width) {
    float v[K * V];
#pragma unroll
    for (int i = 0; i < K * V; i++) {
        const uint32_t c = (i / V * threads + t) * V + i % V;
        v[i] = p && c < width ? load_weight(p, type, c) : otherwise;
    }
#pragma unroll
    for (int i = 0; i < K * V; i += 2) w[i / 2] = F2(v[i], v[i + 1]);
}
template <class T, int V, int K>
__device__ __forceinline__ void pairs_of(F2 (&x)[K * V / 2], const Pack<T, V> (&p)[K]) {
#pragma unroll
    for (int i = 0; i < K * V; i += 2) {
        if constexpr (V > 1) x[i / 2] = two_of(p[i / V], i % V / 2);
        else x[i / 2] = F2(to_f32(p[i].v[0]), to_f32(p[i + 1].v[0]));
    }
}
template <class T, int V, int K>
__device__ __forceinline__ void store_row(T *row, const F2 (&x)[K * V / 2], uint32_t t, uint32_t threads, uint32_t width) {
    Pack<T, V> o[K];
#pragma unroll
    for (int i = 0; i < K * V; i += 2) {
        if constexpr (V > 1) {
            set_two(o[i / V], i % V / 2, x[i / 2]);
        } else {
            const float2 v = x[i / 2].both();
            o[i].v[0] = from_f32<T>(v.x);
            o[i + 1].v[0] = from_f32<T>(v.y);
        }
    }
#pragma unroll
    for (int k = 0; k < K; k++) {
        const uint32_t c = (k * threads + t) * V;
        if (c < width) store_pack<T, V>(row + c, o[k]);
    }
}

// Groups of threads take rows in turn; the weights stay in registers.  One row of 4096 takes 4 us, which is a launch's.
template <class T, int V, int HELD, int THREADS, int BLOCKS>
__global__ void __launch_bounds__(THREADS, BLOCKS) norm_kernel(const NormArgs a, const RowPlan plan, int *status) {
    constexpr int K = HELD / V;
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ uint64_t bars[THREADS / 32][MOST_DEPTH];
    __shared__ float2 met[2][THREADS / 32];
    __shared__ float counts[THREADS / 32];
    const uint32_t group = threadIdx.x / plan.threads, t = threadIdx.x % plan.threads, width = (uint32_t)a.width, lane = t & 31u;
    if (group >= plan.groups) return;
    const uint32_t step = gridDim.x * plan.groups, first = blockIdx.x * plan.groups + group, count = (uint32_t)a.rows;
    const Rows<T, (V > 1)> rows(a.x, a.rows, width);
    uint8_t *mine = ring + (size_t)group * plan.depth * plan.room;
    const uint32_t mine_at = shared_at(mine), bar = shared_at(&bars[group][0]);
    uint32_t asked = first;                                  // by the group's first thread: the next row to copy, and where it is
    uintptr_t asked_at = rows.at(first);
    const uintptr_t stride = (uintptr_t)step * rows.pitch;
    const auto ask = [&](uint32_t d) {
        if (asked >= count) return;
        copies_begin(bar + d * 8, rows.size(asked_at));
        rows.copy(asked_at, mine_at + d * plan.room, bar + d * 8);
        asked += step;
        asked_at += stride;
    };
    if (t == 0) {
        for (uint32_t d = 0; d < plan.depth; d++) barrier_init(bar + d * 8, 1);
        barriers_ready();
        for (uint32_t d = 0; d < plan.depth; d++) ask(d);
    }
    F2 w[HELD / 2], b[HELD / 2];
    load_weights<V, K>(w, a.weight, a.weight_type, 1.0f, t, plan.threads, width);
    load_weights<V, K>(b, a.bias, a.weight_type, 0.0f, t, plan.threads, width);
    uint32_t held = 0;                                       // elements of this thread
#pragma unroll
    for (int k = 0; k < K; k++) held += (k * plan.threads + t) * V < width ? V : 0;
    const uint32_t warps = plan.threads / 32, w0 = group * warps, lanes = power_above(warps), other = lane % lanes;
    const float held_warp = (float)__reduce_add_sync(0xffffffffu, held), part = held_warp > 0.0f ? 1.0f / held_warp : 0.0f;
    if (lane == 0) counts[threadIdx.x / 32] = held_warp;
    group_sync(group, plan.threads);
    const float count_other = other < warps ? counts[w0 + other] : 0.0f, part_other = count_other > 0.0f ? 1.0f / count_other : 0.0f;
    const float all = (float)width, part_all = 1.0f / all;
    uint32_t d = 0, turn = 0, odd = 0;
    uintptr_t row = rows.at(first);
    T *y = static_cast<T *>(a.y.p) + (size_t)first * a.y.stride;
    bool lost = false;                                       // a copy did not come: none is waited for any more
    for (uint32_t r = first; r < count; r += step) {
        if (!lost && !copies_done(bar + d * 8, turn)) lost = true;
        F2 x[HELD / 2];
        {
            Pack<T, V> p[K];
            rows.template get<V, K>(p, row, mine + d * plan.room, t, plan.threads, width);
            pairs_of<T, V, K>(x, p);
        }
        // The warp's sum, and squares about what is its mean but for a rounding; the warps' join to the row's squares: sum of squares + count *
        // (difference of means)^2.  So threads meet once, and nothing is lost where the mean is large.
        F2 s = x[0];
#pragma unroll
        for (int i = 1; i < HELD / 2; i++) s = s + x[i];
        const float sum = warp_sum(s.sum()), about = sum * part;
        F2 q(0.0f);
#pragma unroll
        for (int i = 0; i < HELD / 2; i++) {
            const F2 z = x[i] + F2(-about);
            if (V > 1) {
                if ((i * 2 / V * plan.threads + t) * V < width) q = fma2(z, z, q);
            } else {
                const float2 y2 = z.both();
                const F2 of((i * 2 * plan.threads + t) < width ? y2.x : 0.0f, ((i * 2 + 1) * plan.threads + t) < width ? y2.y : 0.0f);
                q = fma2(of, of, q);
            }
        }
        float squares = warp_sum(q.sum()), mean;
        if (warps == 1) {
            mean = quotient(sum, all, part_all);
            __syncwarp();
        } else {
            if (lane == 0) met[odd][threadIdx.x / 32] = make_float2(sum, squares);
            group_sync(group, plan.threads);                 // and the row is in registers: its place takes another
            const float2 m = other < warps ? met[odd][w0 + other] : make_float2(0.0f, 0.0f);
            mean = quotient(few_sum(m.x, lanes), all, part_all);
            const float off = m.x * part_other - mean;
            squares = few_sum(fmaf(count_other * off, off, m.y), lanes);
        }
        const float rstd = inverse_root(fmaf(squares, part_all, a.eps));
        if (t == 0) {
            ask(d);
            a.mean[r] = mean;
            a.rstd[r] = rstd;
        }
#pragma unroll
        for (int i = 0; i < HELD / 2; i++) x[i] = fma2((x[i] + F2(-mean)) * F2(rstd), w[i], b[i]);
        store_row<T, V, K>(y, x, t, plan.threads, width);
        y += step * a.y.stride;
        row += stride;
        odd ^= 1u;
        if (++d == plan.depth) d = 0, turn ^= 1u;
    }
    if (lost) copies_lost(status);
}

// A warp for each row, where there are rows enough: what threads do once for a row (sums over the warp, the row's numbers, the copies) is done by 32 of
// them and not by the 256 of a group above, of which it was two thirds of all instructions.  32768 rows of 4096 in bf16: 98 us where groups take 119.  The
// weights are in shared memory, in packs of four, [weight, bias][fours of a pack][packs].
template <class T, int HELD, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, 1) norm_warp_kernel(const NormArgs a, const RowPlan plan, int *status) {
    constexpr int V = WIDE<T>, K = HELD / V, FOURS = V / 4;
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ uint64_t bars[WARPS][MOST_DEPTH];
    const uint32_t warp = threadIdx.x / 32, t = threadIdx.x & 31u, width = (uint32_t)a.width, packs = width / V;
    const uint32_t step = gridDim.x * plan.groups, first = blockIdx.x * plan.groups + warp, count = (uint32_t)a.rows;
    const Rows<T, true> rows(a.x, a.rows, width);
    float4 *weights = reinterpret_cast<float4 *>(ring);
    uint8_t *mine = ring + (size_t)width * 2 * sizeof(float) + (size_t)warp * plan.depth * plan.room;
    const uint32_t mine_at = shared_at(mine), bar = shared_at(&bars[warp][0]);
    uint32_t asked = warp < plan.groups ? first : count;
    uintptr_t asked_at = rows.at(first);
    const uintptr_t stride = (uintptr_t)step * rows.pitch;
    const auto ask = [&](uint32_t d) {
        if (asked >= count) return;
        copies_begin(bar + d * 8, rows.bytes);
        rows.copy(asked_at, mine_at + d * plan.room, bar + d * 8);
        asked += step;
        asked_at += stride;
    };
    if (t == 0) {
        for (uint32_t d = 0; d < plan.depth; d++) barrier_init(bar + d * 8, 1);
        barriers_ready();
        for (uint32_t d = 0; d < plan.depth; d++) ask(d);
    }
    for (uint32_t c = threadIdx.x; c < width; c += 32 * WARPS) {
        const uint32_t at = (c % V / 4 * packs + c / V) * 4 + c % 4;
        float *w = reinterpret_cast<float *>(weights);
        w[at] = a.weight ? load_weight(a.weight, a.weight_type, c) : 1.0f;
        w[width + at] = a.bias ? load_weight(a.bias, a.weight_type, c) : 0.0f;
    }
    __syncthreads();
    if (warp >= plan.groups) return;
    const float all = (float)width, part = 1.0f / all;
    uint32_t d = 0, turn = 0;
    T *y = static_cast<T *>(a.y.p) + (size_t)first * a.y.stride;
    bool lost = false;                                       // a copy did not come: none is waited for any more
    for (uint32_t r = first; r < count; r += step) {
        if (!lost && !copies_done(bar + d * 8, turn)) lost = true;
        F2 x[HELD / 2], s[4] = {F2(0.0f), F2(0.0f), F2(0.0f), F2(0.0f)}, q[4] = {F2(0.0f), F2(0.0f), F2(0.0f), F2(0.0f)};
        const T *in = reinterpret_cast<const T *>(mine + d * plan.room) + t * V;
#pragma unroll
        for (int k = 0; k < K; k++) {
            if (k * 32 + t < packs) {
                const Pack<T, V> p = load_pack<T, V>(in + k * 32 * V);
#pragma unroll
                for (int i = 0; i < V / 2; i++) {
                    x[k * (V / 2) + i] = two_of(p, i);
                    s[i % 4] = s[i % 4] + x[k * (V / 2) + i];
                }
            }
        }
        // squares about what is the mean but for a rounding
        const float sum = warp_sum(((s[0] + s[1]) + (s[2] + s[3])).sum()), about = sum * part;
        if (t == 0) ask(d);                                  // the row is in registers: its place takes another
#pragma unroll
        for (int k = 0; k < K; k++)
            if (k * 32 + t < packs) {
#pragma unroll
                for (int i = 0; i < V / 2; i++) {
                    const F2 z = x[k * (V / 2) + i] + F2(-about);
                    q[i % 4] = fma2(z, z, q[i % 4]);
                }
            }
        const float squares = warp_sum(((q[0] + q[1]) + (q[2] + q[3])).sum()), mean = quotient(sum, all, part), rstd = inverse_root(fmaf(squares, part, a.eps));
        if (t == 0) {
            a.mean[r] = mean;
            a.rstd[r] = rstd;
        }
#pragma unroll
        for (int k = 0; k < K; k++)
            if (k * 32 + t < packs) {
                Pack<T, V> o;
#pragma unroll
                for (int f = 0; f < FOURS; f++) {
                    const float4 w = weights[f * packs + k * 32 + t], b = weights[width / 4 + f * packs + k * 32 + t];
                    const int i = k * (V / 2) + f * 2;
                    set_two(o, f * 2, fma2((x[i] + F2(-mean)) * F2(rstd), F2(w.x, w.y), F2(b.x, b.y)));
                    set_two(o, f * 2 + 1, fma2((x[i + 1] + F2(-mean)) * F2(rstd), F2(w.z, w.w), F2(b.z, b.w)));
                }
                store_pack<T, V>(y + (k * 32 + t) * V, o);
            }
        y += step * a.y.stride;
        if (++d == plan.depth) d = 0, turn ^= 1u;
    }
    if (lost) copies_lost(status);
}

// The backward pass.  A block takes a run of rows, its groups parts of it in order; sums over rows stay in registers, and go to shared
// memory where a sample ends.  What the block leaves is a run's head, inner part and tail of every column (see Run).
constexpr uint32_t BACK_THREADS = 256;
template <class T, int V, int HELD, bool SAMPLES>
__global__ void __launch_bounds__(BACK_THREADS, 1) norm_grad_kernel(const NormGradArgs a, const RowPlan plan, const RunsOut out, int *status) {
    constexpr int K = HELD / V;
    next_may_begin();
    // heads and inner parts, [groups][2 planes][width] each; then the ring, where the tails go when it is done with.  Without samples the ring, then heads.
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ uint64_t bars[BACK_THREADS / 32][MOST_DEPTH];
    __shared__ float2 met[2][BACK_THREADS / 32];
    __shared__ int cuts[BACK_THREADS / 32];
    const uint32_t group = threadIdx.x / plan.threads, t = threadIdx.x % plan.threads, width = (uint32_t)a.width, run = blockIdx.x, lane = t & 31u;
    const size_t lo = a.rows * run / out.runs, hi = a.rows * (run + 1) / out.runs;
    const size_t plane_words = (size_t)plan.groups * 2 * width;
    float *heads = reinterpret_cast<float *>(ring), *inners = heads + plane_words, *tails = SAMPLES ? inners + plane_words : heads;
    uint8_t *copies = SAMPLES ? ring + (2 * plane_words * sizeof(float) + 15) / 16 * 16 : ring;
    const auto place = [&](float *of, uint32_t g, int plane) { return of + ((size_t)g * 2 + plane) * width; };
    int cut = 0;
    F2 sw[HELD / 2], sb[HELD / 2];
#pragma unroll
    for (int i = 0; i < HELD / 2; i++) sw[i] = sb[i] = F2(0.0f);
    // element i of this thread's, and its column
    const auto element = [](const F2 (&v)[HELD / 2], int i) { return i % 2 ? v[i / 2].both().y : v[i / 2].both().x; };
    const auto column = [&](int i) { return (i / V * plan.threads + t) * V + i % V; };
    if (group < plan.groups) {
        const uint32_t begin = (uint32_t)(lo + (hi - lo) * group / plan.groups), end = (uint32_t)(lo + (hi - lo) * (group + 1) / plan.groups);
        const Rows<T, (V > 1)> xs(a.x, a.rows, width), dys(a.dy, a.rows, width);
        uint8_t *mine = copies + (size_t)group * plan.depth * 2 * plan.room;
        const uint32_t mine_at = shared_at(mine), bar = shared_at(&bars[group][0]);
        uint32_t asked = begin;                              // by the group's first thread: the next rows to copy, and where they are
        uintptr_t x_asked = xs.at(begin), dy_asked = dys.at(begin);
        const auto ask = [&](uint32_t d) {
            if (asked >= end) return;
            copies_begin(bar + d * 8, xs.size(x_asked) + dys.size(dy_asked));
            xs.copy(x_asked, mine_at + d * 2 * plan.room, bar + d * 8);
            dys.copy(dy_asked, mine_at + (d * 2 + 1) * plan.room, bar + d * 8);
            asked++;
            x_asked += xs.pitch;
            dy_asked += dys.pitch;
        };
        if (t == 0) {
            for (uint32_t d = 0; d < plan.depth; d++) barrier_init(bar + d * 8, 1);
            barriers_ready();
            for (uint32_t d = 0; d < plan.depth; d++) ask(d);
        }
        F2 w[HELD / 2];
        load_weights<V, K>(w, a.weight, a.weight_type, 1.0f, t, plan.threads, width);
        SampleWalk walk;
        walk.begin = 0;
        walk.end = INT64_MAX;
        // what is summed so far is the head, or is added to the inner part
        const auto close = [&] {
#pragma unroll
            for (int i = 0; i < HELD; i++) {
                const uint32_t c = column(i);
                if (c < width) {
                    if (cut) {
                        place(inners, group, 0)[c] += fabsf(element(sw, i));
                        place(inners, group, 1)[c] += fabsf(element(sb, i));
                    } else {
                        place(heads, group, 0)[c] = element(sw, i);
                        place(heads, group, 1)[c] = element(sb, i);
                        place(inners, group, 0)[c] = place(inners, group, 1)[c] = 0.0f;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < HELD / 2; i++) sw[i] = sb[i] = F2(0.0f);
            cut = 1;
        };
        if (SAMPLES) {
            walk.seek(a.offsets, a.samples, (int64_t)begin);
            if (walk.begin == (int64_t)begin) close();       // the run before this one ends with another sample
        }
        const uint32_t warps = plan.threads / 32, w0 = group * warps, lanes = power_above(warps), other = lane % lanes;
        const float n = 1.0f / (float)width;
        float mean_next = begin < end ? a.mean[begin] : 0.0f, rstd_next = begin < end ? a.rstd[begin] : 0.0f;
        group_sync(group, plan.threads);
        uint32_t d = 0, turn = 0;
        uintptr_t x_row = xs.at(begin), dy_row = dys.at(begin);
        T *dx = static_cast<T *>(a.dx.p) + (size_t)begin * a.dx.stride;
        bool lost = false;
        for (uint32_t r = begin; r < end; r++) {
            const float mean = mean_next, rstd = rstd_next;
            if (r + 1 < end) {
                mean_next = a.mean[r + 1];
                rstd_next = a.rstd[r + 1];
            }
            if (!lost && !copies_done(bar + d * 8, turn)) lost = true;
            F2 x[HELD / 2], g[HELD / 2], q[HELD / 2], s0(0.0f), s1(0.0f);
            {
                Pack<T, V> px[K], pg[K];
                xs.template get<V, K>(px, x_row, mine + d * 2 * plan.room, t, plan.threads, width);
                dys.template get<V, K>(pg, dy_row, mine + (d * 2 + 1) * plan.room, t, plan.threads, width);
                pairs_of<T, V, K>(x, px);
                pairs_of<T, V, K>(g, pg);
            }
#pragma unroll
            for (int i = 0; i < HELD / 2; i++) {
                x[i] = (x[i] + F2(-mean)) * F2(rstd);
                q[i] = g[i] * w[i];                          // behind the row's end g is 0
                s0 = s0 + q[i];
                s1 = fma2(q[i], x[i], s1);
            }
            float ma = warp_sum(s0.sum()), man = warp_sum(s1.sum());
            if (warps > 1 && lane == 0) met[r & 1][threadIdx.x / 32] = make_float2(ma, man);
            if (SAMPLES && (int64_t)r >= walk.end) {
                close();
                walk.next((int64_t)r);
            }
            if (!SAMPLES || (int64_t)r >= walk.begin) {
#pragma unroll
                for (int i = 0; i < HELD / 2; i++) {
                    sw[i] = fma2(g[i], x[i], sw[i]);
                    sb[i] = sb[i] + g[i];
                }
            }
            group_sync(group, plan.threads);                 // and the rows are in registers: their places take others
            if (t == 0) ask(d);
            if (warps > 1) {
                const float2 m = other < warps ? met[r & 1][w0 + other] : make_float2(0.0f, 0.0f);
                ma = few_sum(m.x, lanes);
                man = few_sum(m.y, lanes);
            }
            ma *= n;
            man *= n;
#pragma unroll
            for (int i = 0; i < HELD / 2; i++) x[i] = F2(rstd) * fma2(x[i], F2(-man), q[i] + F2(-ma));
            store_row<T, V, K>(dx, x, t, plan.threads, width);
            dx += a.dx.stride;
            x_row += xs.pitch;
            dy_row += dys.pitch;
            if (++d == plan.depth) d = 0, turn ^= 1u;
        }
        if (lost) copies_lost(status);
    }
    __syncthreads();                                         // the ring is done with
    if (group < plan.groups) {
        // what is left is the tail, or the head of a run without a cut
        float *to = SAMPLES && cut ? tails : heads;
#pragma unroll
        for (int i = 0; i < HELD; i++) {
            const uint32_t c = column(i);
            if (c < width) {
                place(to, group, 0)[c] = element(sw, i);
                place(to, group, 1)[c] = element(sb, i);
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
            if (!SAMPLES) all.head += place(heads, g, plane)[c];
            else if (cuts[g]) all.join(Run{place(heads, g, plane)[c], place(inners, g, plane)[c], place(tails, g, plane)[c], 1});
            else all.join(Run{place(heads, g, plane)[c], 0.0f, 0.0f, 0});
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
    constexpr int P = X ? 2 : 1, AHEAD = X ? 4 : 8;
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
    int cut = 0;
    next_may_begin();
    SampleWalk walk;
    walk.begin = 0;
    walk.end = INT64_MAX;
    Pack<T, V> g[AHEAD], x[X ? AHEAD : 1];
    const auto load = [&](size_t r0) {
#pragma unroll
        for (int j = 0; j < AHEAD; j++)
            if (r0 + j < end && col < width) {
                g[j] = load_pack<T, V>(static_cast<const T *>(m.p) + (r0 + j) * m.stride + col);
                if (X) x[X ? j : 0] = load_pack<T, V>(static_cast<const T *>(xm.p) + (r0 + j) * xm.stride + col);
            }
    };
    load(begin);
    if (over == SumOver::SAMPLES) {
        walk.seek(offsets, samples, (int64_t)begin);
        cut = walk.begin == (int64_t)begin;  // the run before this one ends with another sample
    }
    for (size_t r0 = begin; r0 < end;) {
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
            if (X) {
                const float mu = mean[r], rs = rstd[r];
#pragma unroll
                for (int e = 0; e < V; e++) sum[0][e] = fmaf(to_f32(g[j].v[e]), (to_f32(x[X ? j : 0].v[e]) - mu) * rs, sum[0][e]);
            }
#pragma unroll
            for (int e = 0; e < V; e++) sum[P - 1][e] += to_f32(g[j].v[e]);
        }
        r0 += AHEAD;
        if (r0 < end) load(r0);
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
    if (blockIdx.x == 0 && blockIdx.y == 0) before_is_done();
}

// Joins all runs of a column: each warp a part of them in order, then the warps' results.  READY: the runs are from a kernel that is known to be done, and not from
// the one before.
constexpr int JOIN_WARPS = 32;
template <bool MAGNITUDES, bool READY>
__global__ void __launch_bounds__(32 * JOIN_WARPS) sums_join_kernel(const RunsOut in, const bool accumulate, float *dst0, float *dst1) {
    __shared__ Run runs[JOIN_WARPS][33];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x / 32;
    const int plane = blockIdx.y;
    const size_t col = (size_t)blockIdx.x * 32 + lane;
    float *dst = plane ? dst1 : dst0;
    Run all{0.0f, 0.0f, 0.0f, 0};
    if (!READY) before_is_done();
    const uint32_t begin = in.runs * warp / JOIN_WARPS, end = in.runs * (warp + 1) / JOIN_WARPS;
    constexpr int AHEAD = 5;                 // of 148 runs a warp has five at most
    if (col < in.width)
        for (uint32_t r0 = begin; r0 < end; r0 += AHEAD) {
            Run part[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; j++) {
                part[j] = Run{0.0f, 0.0f, 0.0f, 0};
                if (r0 + j >= end) continue;
                part[j].head = __ldcg(in.of(r0 + j, 0, plane) + col);
                if (MAGNITUDES) {
                    part[j].inner = __ldcg(in.of(r0 + j, 1, plane) + col);
                    part[j].tail = __ldcg(in.of(r0 + j, 2, plane) + col);
                    part[j].cut = __ldcg(in.cut(r0 + j));
                }
            }
#pragma unroll
            for (int j = 0; j < AHEAD; j++) all.join(part[j]);
        }
    runs[warp][lane] = all;
    for (uint32_t step = 1; step < JOIN_WARPS; step *= 2) {
        __syncthreads();
        if (warp % (2 * step) == 0) {
            all.join(runs[warp + step][lane]);
            runs[warp][lane] = all;
        }
    }
    if (warp == 0 && col < in.width) {
        const float v = MAGNITUDES ? fabsf(all.head) + all.inner + fabsf(all.tail) : all.head;
        dst[col] = accumulate ? dst[col] + v : v;
    }
    if (READY && blockIdx.x == 0) before_is_done();
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
    const auto kernel = magnitudes ? sums_join_kernel<true, false> : sums_join_kernel<false, false>;
    return launch_early(true, kernel, dim3(blocks_for(runs.width, 32), runs.planes), 32 * JOIN_WARPS, 0, s, runs, accumulate, dst0, dst1);
}

template <class T, bool X>
cudaError_t sums(const MatArg &m, const MatArg &x, const float *mean, const float *rstd, size_t rows, size_t width, SumOver over,
                 const int32_t *offsets, uint32_t samples, bool accumulate, float *dst0, float *dst1, void *work, int n_sm, bool early, cudaStream_t s) {
    const bool wide = wide_rows<T>(m.p, m.stride, width) && (!X || wide_rows<T>(x.p, x.stride, width));
    // two blocks on an SM
    const unsigned cols = blocks_for(width, SUM_COLS * (wide ? WIDE<T> : 1)), most = (2 * n_sm + cols - 1) / cols, runs = sum_runs(rows, n_sm);
    const RunsOut out{static_cast<float *>(work), runs < most ? runs : most, width, X ? 2 : 1};
    const dim3 grid(cols, out.runs);
    const auto kernel = wide ? sums_kernel<T, WIDE<T>, X> : sums_kernel<T, 1, X>;
    const cudaError_t rc = launch_early(early, kernel, grid, SUM_COLS * SUM_WARPS, 0, s, m, x, mean, rstd, rows, width, over, offsets, samples, out);
    return rc != cudaSuccess ? rc : join_runs(out, over != SumOver::ALL, accumulate, dst0, dst1, s);
}

inline uint32_t row_threads(size_t packs) { return packs >= 256 ? 256 : (uint32_t)(packs + 31) / 32 * 32; }

template <class T, int V, int HELD, int THREADS, int BLOCKS>
bool norm_go(const NormArgs &a, int n_sm, int *status, cudaStream_t s, cudaError_t &rc) {
    RowPlan plan;
    if (!plan_row(a.width, sizeof(T), THREADS, HELD, 1, MOST_SHARED / BLOCKS - 1024, plan)) return false;
    const auto kernel = norm_kernel<T, V, HELD, THREADS, BLOCKS>;
    const size_t bytes = (size_t)plan.groups * plan.depth * plan.room, blocks = (a.rows + plan.groups - 1) / plan.groups, most = (size_t)BLOCKS * n_sm;
    rc = allow_shared(reinterpret_cast<const void *>(kernel), bytes);
    if (rc != cudaSuccess) return true;
    kernel<<<(unsigned)(blocks < most ? blocks : most), THREADS, bytes, s>>>(a, plan, status);
    rc = FEDHE_LAUNCHED();
    return true;
}

// With fewer than eight rows for each warp the groups below, which are more threads to a row, are as fast or faster (calls by themselves: 8192 rows of 4096
// in fp32 53 and 51 us, 32768: 182 and 188; in bf16 35 and 37, 98 and 119; 32768 rows of 768 in bf16 27 and 35).
template <class T, int HELD, int WARPS>
bool norm_warp_go(const NormArgs &a, int n_sm, int *status, cudaStream_t s, cudaError_t &rc) {
    if (a.width > 32 * HELD || a.rows < (size_t)8 * WARPS * n_sm) return false;
    RowPlan plan;
    plan.threads = 32;
    plan.room = (uint32_t)(a.width * sizeof(T));
    const size_t kept = a.width * 2 * sizeof(float), places = (MOST_SHARED - kept) / plan.room;
    plan.groups = (uint32_t)(places < WARPS ? places : WARPS);
    plan.depth = (uint32_t)(places / plan.groups < MOST_DEPTH ? places / plan.groups : MOST_DEPTH);
    const auto kernel = norm_warp_kernel<T, HELD, WARPS>;
    const size_t bytes = kept + (size_t)plan.groups * plan.depth * plan.room;
    rc = allow_shared(reinterpret_cast<const void *>(kernel), bytes);
    if (rc != cudaSuccess) return true;
    kernel<<<n_sm, 32 * WARPS, bytes, s>>>(a, plan, status);
    rc = FEDHE_LAUNCHED();
    return true;
}

template <class T>
cudaError_t norm_of(const NormArgs &a, int n_sm, int *status, cudaStream_t s) {
    if (a.rows == 0) return cudaSuccess;
    const bool wide = wide_rows<T>(a.x.p, a.x.stride, a.width) && wide_rows<T>(a.y.p, a.y.stride, a.width);
    cudaError_t rc;
    // Up to 512 columns a group below is a warp as well.
    if (wide && a.width > 512 &&
        (norm_warp_go<T, 32, 24>(a, n_sm, status, s, rc) || norm_warp_go<T, 64, 16>(a, n_sm, status, s, rc) || norm_warp_go<T, 128, 12>(a, n_sm, status, s, rc)))
        return rc;
    if (wide ? norm_go<T, WIDE<T>, 16, 256, 3>(a, n_sm, status, s, rc) : norm_go<T, 1, 16, 256, 3>(a, n_sm, status, s, rc)) return rc;
    if (wide ? norm_go<T, WIDE<T>, 16, 1024, 1>(a, n_sm, status, s, rc) : norm_go<T, 1, 16, 1024, 1>(a, n_sm, status, s, rc)) return rc;
    if (wide) norm_long_kernel<T, WIDE<T>><<<(unsigned)a.rows, row_threads(a.width / WIDE<T>), 0, s>>>(a);
    else norm_long_kernel<T, 1><<<(unsigned)a.rows, row_threads(a.width), 0, s>>>(a);
    return FEDHE_LAUNCHED();
}

template <class T, int V, int HELD, bool SAMPLES>
bool norm_grad_go(const NormGradArgs &a, int n_sm, int *status, cudaStream_t s, cudaError_t &rc) {
    RowPlan plan;
    const size_t t = ((a.width + HELD - 1) / HELD + 31) / 32 * 32;
    if (t > BACK_THREADS) return false;
    const size_t plane = (BACK_THREADS / t) * 2 * a.width * sizeof(float), kept = SAMPLES ? (2 * plane + 15) / 16 * 16 : 0;
    if (kept > MOST_SHARED || !plan_row(a.width, sizeof(T), BACK_THREADS, HELD, 2, MOST_SHARED - kept, plan)) return false;
    const auto kernel = norm_grad_kernel<T, V, HELD, SAMPLES>;
    const size_t copies = (size_t)plan.groups * plan.depth * 2 * plan.room, bytes = kept + (copies > plane ? copies : plane);
    const RunsOut out{static_cast<float *>(a.work), sum_runs(a.rows, n_sm), a.width, 2};
    rc = allow_shared(reinterpret_cast<const void *>(kernel), bytes);
    if (rc != cudaSuccess) return true;
    kernel<<<out.runs, BACK_THREADS, bytes, s>>>(a, plan, out, status);
    rc = FEDHE_LAUNCHED();
    if (rc == cudaSuccess) rc = join_runs(out, SAMPLES, false, a.dweight, a.dbias, s);
    return true;
}

// Elements of a thread: 32 for long rows and, of 16-bit types, for much work, of which each row's own instructions then are a smaller part; 16 where what comes
// before and behind the rows counts more, or memory (16384 rows of 4096 in bf16: 108 us with samples and 88 without, with 16 elements 139 and
// 109; 4096 rows of 1024: 31 and 22, 27 and 19; 16384 rows of 4096 in fp32: 164 and 151, 160 and 149).
template <class T, int V>
bool norm_grad_held(const NormGradArgs &a, int n_sm, int *status, cudaStream_t s, cudaError_t &rc) {
    const bool many = V > 1 && sizeof(T) == 2 && a.width > 512 && a.rows * a.width >= (size_t)1 << 23;
    if (a.over == SumOver::SAMPLES) return (!many && norm_grad_go<T, V, 16, true>(a, n_sm, status, s, rc)) || norm_grad_go<T, V, 32, true>(a, n_sm, status, s, rc);
    return (!many && norm_grad_go<T, V, 16, false>(a, n_sm, status, s, rc)) || norm_grad_go<T, V, 32, false>(a, n_sm, status, s, rc);
}

template <class T>
cudaError_t norm_grad_of(const NormGradArgs &a, int n_sm, int *status, cudaStream_t s) {
    const bool wide = wide_rows<T>(a.x.p, a.x.stride, a.width) && wide_rows<T>(a.dy.p, a.dy.stride, a.width) &&
                      wide_rows<T>(a.dx.p, a.dx.stride, a.width);
    cudaError_t rc;
    if (a.rows && (wide ? norm_grad_held<T, WIDE<T>>(a, n_sm, status, s, rc) : norm_grad_held<T, 1>(a, n_sm, status, s, rc))) return rc;
    if (a.rows) {
        if (wide) norm_long_grad_kernel<T, WIDE<T>><<<(unsigned)a.rows, row_threads(a.width / WIDE<T>), 0, s>>>(a);
        else norm_long_grad_kernel<T, 1><<<(unsigned)a.rows, row_threads(a.width), 0, s>>>(a);
        rc = FEDHE_LAUNCHED();
        if (rc != cudaSuccess) return rc;
    }
    return sums<T, true>(a.dy, a.x, a.mean, a.rstd, a.rows, a.width, a.over, a.offsets, a.samples, false, a.dweight, a.dbias, a.work, n_sm, false, s);
}

}  // namespace

cudaError_t launch_norm(const NormArgs &a, int dtype, int n_sm, int *status, cudaStream_t s) {
    return dtype == HE_F32    ? norm_of<float>(a, n_sm, status, s)
           : dtype == HE_BF16 ? norm_of<__nv_bfloat16>(a, n_sm, status, s)
                              : norm_of<__half>(a, n_sm, status, s);
}

cudaError_t launch_join_sums(const float *heads, uint32_t runs, size_t width, bool accumulate, float *dst, cudaStream_t s) {
    return launch_early(true, sums_join_kernel<false, true>, dim3(blocks_for(width, 32)), 32 * JOIN_WARPS, 0, s, RunsOut{const_cast<float *>(heads), runs, width, 1}, accumulate,
                        dst, (float *)nullptr);
}

size_t norm_grad_work_bytes(size_t rows, size_t width, int n_sm) { return runs_bytes(rows, width, 2, n_sm); }

cudaError_t launch_norm_grad(const NormGradArgs &a, int dtype, int n_sm, int *status, cudaStream_t s) {
    return dtype == HE_F32    ? norm_grad_of<float>(a, n_sm, status, s)
           : dtype == HE_BF16 ? norm_grad_of<__nv_bfloat16>(a, n_sm, status, s)
                              : norm_grad_of<__half>(a, n_sm, status, s);
}

size_t column_sums_work_bytes(size_t rows, size_t width, int n_sm) { return runs_bytes(rows, width, 1, n_sm); }

cudaError_t launch_column_sums(const ColumnSumArgs &a, int dtype, int n_sm, bool early, cudaStream_t s) {
    const MatArg none{nullptr, 0};
    const auto go = [&](auto t) {
        return sums<decltype(t), false>(a.m, none, nullptr, nullptr, a.rows, a.width, a.over, a.offsets, a.samples, a.accumulate, a.dst, nullptr,
                                        a.work, n_sm, early, s);
    };
    return dtype == HE_F32 ? go(0.0f) : dtype == HE_BF16 ? go(__nv_bfloat16()) : go(__half());
}

}  // namespace fedhe
