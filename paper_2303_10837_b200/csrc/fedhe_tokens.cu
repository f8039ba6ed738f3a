// Log probabilities of given tokens, with the entropy and the top alternatives of every row of logits, and their gradient.
//
//   lse = m + ln s,  m = max z,  s = sum e^(z - m);   log p_y = (z_y - m) - ln s;   H = ln s - (sum e^(z - m) (z - m)) / s
//   dz_j = sum_i g_i (d_{j,t_i} - p_j) - g_H p_j (log p_j + H)        t_i: the target and the alternatives, g_i their gradients
//
// Both directions are bounded by reading (and writing) the logits once.
#include <cooperative_groups.h>

#include "fedhe_map.cuh"

namespace cg = cooperative_groups;

namespace fedhe {

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float FAR = -1e30f;             // exponents stop here: 2^FAR is 0, and FAR times 0 is 0, not NaN
constexpr int ROW_ELEMENTS = 32;          // of a thread, at a time
constexpr uint32_t FOUND = 1024;          // candidates that a block can hold

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Maximum, sum of 2^t and sum of t 2^t over t = (z - maximum) log2 e.  All in fp32: sums of up to 2^31 terms that are at most 1, as
// partial sums of the threads.
struct Soft {
    float m, s, w;
    __device__ __forceinline__ float base() const { return m == -INFINITY ? 0.0f : m; }
    __device__ __forceinline__ void rise(float to) {         // to a larger maximum
        const float b = to == -INFINITY ? 0.0f : to, d = max_nan((m - b) * LOG2E, FAR), f = ex2(d);
        w = f * (w + s * d);
        s *= f;
        m = to;
    }
    __device__ __forceinline__ void add(float z, float b) {
        const float t = max_nan((z - b) * LOG2E, FAR), e = ex2(t);
        s += e;
        w = fmaf(e, t, w);
    }
    __device__ __forceinline__ void join(Soft o) {
        const float to = fmaxf(m, o.m);
        rise(to);
        o.rise(to);
        s += o.s;
        w += o.w;
    }
};

// Order of the alternatives: the value, NaN as low as -inf, then the lowest index.
__device__ __forceinline__ uint32_t order_of(float z) {
    z = z == z ? z + 0.0f : -INFINITY;                        // -0 becomes 0
    const uint32_t b = __float_as_uint(z);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ uint64_t key_of(float z, uint32_t index) { return (uint64_t)order_of(z) << 32 | (0xffffffffu - index); }

// A row as aligned vectors: vector v holds the elements v * V - shift, .... The first and the last may reach outside; those elements
// are not read.
template <class T>
struct Row {
    static constexpr int V = WIDE<T>;
    const T *p;
    uint32_t n, shift, vectors;
    __device__ __forceinline__ Row(const T *row, uint32_t count) : p(row), n(count) {
        shift = (uint32_t)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
        vectors = (n + shift + V - 1) / V;
    }
    __device__ __forceinline__ int64_t first(uint32_t v) const { return (int64_t)v * V - shift; }
    __device__ __forceinline__ bool whole(uint32_t v) const { return first(v) >= 0 && first(v) + V <= n; }
    __device__ __forceinline__ Pack<T, V> load(uint32_t v) const {
        if (v < vectors && whole(v)) return load_pack<T, V>(p + first(v));
        Pack<T, V> a;
#pragma unroll
        for (int e = 0; e < V; e++) {
            const int64_t i = first(v) + e;
            a.v[e] = i >= 0 && i < (int64_t)n ? p[i] : from_f32<T>(-INFINITY);
        }
        return a;
    }
};

struct Found {
    uint64_t key[FOUND];
    uint64_t best[HE_MAX_TOP];
    uint32_t count, bound[8];
    uint64_t most[8];
};

// The `top` highest of key[0 .. n) in order, to its front; returns how many there are.  By the whole block.
__device__ __forceinline__ uint32_t keep_best(Found &f, uint32_t n, uint32_t top) {
    for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) {
        const uint64_t mine = f.key[i];
        uint32_t above = 0;
        for (uint32_t j = 0; j < n; j++) above += f.key[j] > mine;
        if (above < top) f.best[above] = mine;
    }
    __syncthreads();
    const uint32_t kept = n < top ? n : top;
    for (uint32_t i = threadIdx.x; i < kept; i += blockDim.x) f.key[i] = f.best[i];
    if (threadIdx.x == 0) f.count = kept;
    __syncthreads();
    return kept;
}

// A lower bound of the order of the top-th value of what the block's threads hold, given each thread's maximum: in each warp the
// (top / warps)-th highest maximum of a thread, and the lowest of these over the warps.
__device__ __forceinline__ uint32_t bound_of_top(Found &f, uint32_t mine, uint32_t top) {
    const uint32_t warps = blockDim.x / 32, lane = threadIdx.x & 31u;
    uint32_t got = 0;
    for (uint32_t j = 0; j < (top + warps - 1) / warps; j++) {
        got = __reduce_max_sync(0xffffffffu, mine);
        const uint32_t who = __ballot_sync(0xffffffffu, mine == got);
        if (lane == __ffs(who) - 1) mine = 0;
    }
    if (lane == 0) f.bound[threadIdx.x / 32] = got;
    __syncthreads();
    uint32_t low = f.bound[0];
    for (uint32_t i = 1; i < warps; i++) low = min(low, f.bound[i]);
    return low;
}

// One row by a cluster of C blocks (C = 1: by a block), which take the row's pieces in turn.  A piece stays in registers while its
// maximum, its sums and its candidates for the alternatives are found.  The candidates: values that are not below a bound on the top-th value,
// in shared memory, of which the best are kept now and then and raise the bound.  Rows of many equal values can overflow
// the candidates' room; a piece that does is searched once for each alternative instead.
template <class T, bool TOP>
__global__ void __launch_bounds__(256) log_probs_kernel(const LogProbsArgs a, const uint32_t C) {
    constexpr int V = WIDE<T>, NV = ROW_ELEMENTS / V;
    __shared__ Soft soft[8];
    __shared__ Soft mine;
    __shared__ Found f;
    const uint32_t tid = threadIdx.x, NT = blockDim.x, rank = blockIdx.x % C;
    const size_t r = blockIdx.x / C;
    const Row<T> row(static_cast<const T *>(a.logits.p) + r * a.logits.stride, (uint32_t)a.vocab);
    const uint32_t pieces = (row.vectors + NT * NV - 1) / (NT * NV);
    Soft q{-INFINITY, 0.0f, 0.0f};
    uint32_t held = 0, bound = 0;
    bool full = false;                       // `held` has top candidates, and the bound is the lowest of them
    if (TOP && tid == 0) f.count = 0;
    if (TOP) __syncthreads();
    for (uint32_t c = rank; c < pieces; c += C) {
        Pack<T, V> z[NV];
        const uint32_t v0 = c * NT * NV + tid;
#pragma unroll
        for (int i = 0; i < NV; i++) z[i] = row.load(v0 + i * NT);
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int e = 0; e < V; e++) m = fmaxf(m, to_f32(z[i].v[e]));
        if (m > q.m) q.rise(m);
        const float b = q.base();
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int e = 0; e < V; e++) q.add(to_f32(z[i].v[e]), b);
        if (TOP) {
            const uint32_t high = order_of(m);
            if (c == rank) bound = bound_of_top(f, high, a.top);
            // later pieces have higher indices: with enough candidates a value equal to the bound is too late
            const uint32_t from = full ? bound + 1 : bound;
            if (high >= from) {
#pragma unroll
                for (int i = 0; i < NV; i++)
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        const float x = to_f32(z[i].v[e]);
                        const int64_t j = row.first(v0 + i * NT) + e;
                        if (order_of(x) >= from && j >= 0 && j < (int64_t)row.n) {
                            const uint32_t at = atomicAdd(&f.count, 1u);
                            if (at < FOUND) f.key[at] = key_of(x, (uint32_t)j);
                        }
                    }
            }
            __syncthreads();
            uint32_t n = f.count;
            if (n > FOUND) {
                uint64_t below = ~0ull;
                n = held;
                for (uint32_t t = 0; t < a.top; t++) {
                    uint64_t best = 0;
#pragma unroll
                    for (int i = 0; i < NV; i++)
#pragma unroll
                        for (int e = 0; e < V; e++) {
                            const int64_t j = row.first(v0 + i * NT) + e;
                            if (j < 0 || j >= (int64_t)row.n) continue;
                            const uint64_t k = key_of(to_f32(z[i].v[e]), (uint32_t)j);
                            if (k < below && k > best) best = k;
                        }
#pragma unroll
                    for (int o = 16; o; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
                    if ((tid & 31u) == 0) f.most[tid / 32] = best;
                    __syncthreads();
                    for (uint32_t w = 0; w < NT / 32; w++) best = max(best, f.most[w]);
                    __syncthreads();
                    if (best == 0) break;            // a key of an element is not 0: its index is below 2^32 - 1
                    if (tid == 0) f.key[n] = best;
                    n++;
                    below = best;
                }
                __syncthreads();
                n = keep_best(f, n, a.top);
            } else if (!full || n > FOUND / 2) {
                n = keep_best(f, n, a.top);
            }
            if (n >= a.top) {
                if (!full || n == a.top) bound = max(bound, (uint32_t)(f.key[a.top - 1] >> 32));
                full = true;
            }
            held = n;
            __syncthreads();
            if (tid == 0) f.count = held;
            __syncthreads();
        }
    }
    // the threads' sums, then the warps'
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const Soft p{__shfl_xor_sync(0xffffffffu, q.m, o), __shfl_xor_sync(0xffffffffu, q.s, o), __shfl_xor_sync(0xffffffffu, q.w, o)};
        q.join(p);
    }
    if ((tid & 31u) == 0) soft[tid / 32] = q;
    __syncthreads();
    if (tid == 0) {
        for (uint32_t w = 1; w < NT / 32; w++) q.join(soft[w]);
        mine = q;
    }
    if (TOP) held = keep_best(f, held, a.top);
    else __syncthreads();
    if (C > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        if (rank == 0) {
            if (tid == 0)
                for (uint32_t o = 1; o < C; o++) q.join(*cluster.map_shared_rank(&mine, o));
            if (TOP) {
                uint32_t n = held;
                for (uint32_t o = 1; o < C; o++) {
                    const Found &far = *cluster.map_shared_rank(&f, o);
                    const uint32_t more = far.count;
                    for (uint32_t i = tid; i < more; i += NT) f.key[n + i] = far.key[i];
                    n += more;
                }
                __syncthreads();
                keep_best(f, n, a.top);
            }
        }
        cluster.sync();                      // nobody leaves while its memory is read
        if (rank) return;
        if (tid == 0) mine = q;
        __syncthreads();
    }
    q = mine;
    const bool none = q.s == 0.0f;           // every value is -inf
    const float ln = logf(q.s), b = q.base();
    if (tid == 0) {
        a.lse[r] = none ? -INFINITY : b + ln;
        a.entropy[r] = none ? 0.0f : ln - q.w / q.s * LN2;
        const int64_t y = a.targets[r];
        float lp = 0.0f;
        if (y >= (int64_t)row.n) lp = NAN;
        else if (y >= 0) lp = none ? -INFINITY : (to_f32(row.p[y]) - b) - ln;
        a.logp[r] = lp;
    }
    if (TOP)
        for (uint32_t i = tid; i < a.top; i += NT) {
            const uint64_t k = f.key[i];
            a.top_ids[r * a.top + i] = (int64_t)(0xffffffffu - (uint32_t)k);
            a.top_logp[r * a.top + i] = none ? -INFINITY : (value_of((uint32_t)(k >> 32)) - b) - ln;
        }
}

// Threads of a block: as few as hold a row of up to 256 * 32 elements at once.
inline uint32_t row_threads(size_t vocab) {
    const size_t t = (vocab + ROW_ELEMENTS - 1) / ROW_ELEMENTS;
    return t >= 256 ? 256 : (uint32_t)(t + 31) / 32 * 32;
}

template <class T>
cudaError_t log_probs_of(const LogProbsArgs &a, int n_sm, cudaStream_t s) {
    const uint32_t nt = row_threads(a.vocab);
    const size_t pieces = (a.vocab + WIDE<T> + (size_t)nt * ROW_ELEMENTS - 1) / ((size_t)nt * ROW_ELEMENTS);
    // few rows: a cluster of up to eight blocks shares one, as long as each has a piece
    uint32_t C = 1;
    while (C < 8 && 2 * C <= pieces && a.rows * 2 * C <= (size_t)4 * n_sm) C *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(nt);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {C, 1, 1};
    cfg.attrs = at;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3((unsigned)(a.rows * C));
    const cudaError_t rc = a.top ? cudaLaunchKernelEx(&cfg, log_probs_kernel<T, true>, a, C) : cudaLaunchKernelEx(&cfg, log_probs_kernel<T, false>, a, C);
    if (rc != cudaSuccess) return rc;
    return FEDHE_LAUNCHED();
}

// ---------------------------------------------------------------------------

// One row's part [v0, v1) of vectors by a block.  The elements that a gradient falls on by itself (the target, the alternatives) are computed
// first, from logits that the result may replace, and written last.
template <class T>
__global__ void __launch_bounds__(256) log_probs_grad_kernel(const LogProbsGradArgs a, const uint32_t parts) {
    constexpr int V = WIDE<T>, NV = 4;
    const uint32_t tid = threadIdx.x, NT = blockDim.x, part = blockIdx.x % parts;
    const size_t r = blockIdx.x / parts;
    const Row<T> row(static_cast<const T *>(a.logits.p) + r * a.logits.stride, (uint32_t)a.vocab);
    T *out = static_cast<T *>(a.dlogits.p) + r * a.dlogits.stride;
    const uint32_t v0 = (uint32_t)((uint64_t)row.vectors * part / parts), v1 = (uint32_t)((uint64_t)row.vectors * (part + 1) / parts);
    const int64_t y = a.targets[r];
    const float lse = a.lse[r], gh = a.dentropy ? a.dentropy[r] : 0.0f, H = a.dentropy ? a.entropy[r] : 0.0f;
    const float gy = y < 0 ? 0.0f : y < (int64_t)row.n ? a.dlogp[r] : NAN;
    float G = gy;
    for (uint32_t i = 0; i < a.top; i++) G += a.dtop[r * a.top + i];
    // nothing flows into the row, or every logit of it is -inf: what it holds does not count
    const bool still = lse == -INFINITY || (y < 0 && !a.dentropy && !a.top);
    const auto grad = [&](float z) {
        const float lp = max_nan(z - lse, FAR), p = ex2(lp * LOG2E);
        return -p * fmaf(gh, lp + H, G);
    };
    float own = 0.0f;
    int64_t at = -1;
    if (!still && tid <= a.top) {
        at = tid == a.top ? y : a.top_ids[r * a.top + tid];
        if (at < 0 || at >= (int64_t)row.n || at < row.first(v0) || at >= row.first(v1)) at = -1;
        if (at >= 0) {
            float g = at == y ? gy : 0.0f;
            for (uint32_t i = 0; i < a.top; i++)
                if (a.top_ids[r * a.top + i] == at) g += a.dtop[r * a.top + i];
            own = g + grad(to_f32(row.p[at]));
        }
    }
    __syncthreads();
    const bool alike = ((reinterpret_cast<uintptr_t>(row.p) ^ reinterpret_cast<uintptr_t>(out)) & 15u) == 0;
    for (uint32_t c = v0 + tid; c < v1; c += NT * NV) {
        Pack<T, V> z[NV];
#pragma unroll
        for (int i = 0; i < NV; i++)
            if (!still && c + i * NT < v1) z[i] = row.load(c + i * NT);
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const uint32_t v = c + i * NT;
            if (v >= v1) break;
            Pack<T, V> d;
#pragma unroll
            for (int e = 0; e < V; e++) d.v[e] = from_f32<T>(still ? 0.0f : grad(to_f32(z[i].v[e])));
            if (alike && row.whole(v)) {
                store_pack<T, V>(out + row.first(v), d);
            } else {
#pragma unroll
                for (int e = 0; e < V; e++) {
                    const int64_t j = row.first(v) + e;
                    if (j >= 0 && j < (int64_t)row.n) out[j] = d.v[e];
                }
            }
        }
    }
    __syncthreads();
    if (at >= 0) out[at] = from_f32<T>(own);
}

template <class T>
cudaError_t log_probs_grad_of(const LogProbsGradArgs &a, int n_sm, cudaStream_t s) {
    const size_t vectors = a.vocab / WIDE<T> + 2;
    const uint32_t nt = 256;
    size_t parts = (vectors + nt * 4 - 1) / (nt * 4);
    const size_t wanted = ((size_t)8 * n_sm + a.rows - 1) / a.rows;
    if (parts > wanted) parts = wanted;
    log_probs_grad_kernel<T><<<(unsigned)(a.rows * parts), nt, 0, s>>>(a, (uint32_t)parts);
    return FEDHE_LAUNCHED();
}

}  // namespace

cudaError_t launch_log_probs(const LogProbsArgs &a, int dtype, int n_sm, cudaStream_t s) {
    return dtype == HE_F32    ? log_probs_of<float>(a, n_sm, s)
           : dtype == HE_BF16 ? log_probs_of<__nv_bfloat16>(a, n_sm, s)
                              : log_probs_of<__half>(a, n_sm, s);
}

cudaError_t launch_log_probs_grad(const LogProbsGradArgs &a, int dtype, int n_sm, cudaStream_t s) {
    return dtype == HE_F32    ? log_probs_grad_of<float>(a, n_sm, s)
           : dtype == HE_BF16 ? log_probs_grad_of<__nv_bfloat16>(a, n_sm, s)
                              : log_probs_grad_of<__half>(a, n_sm, s);
}

}  // namespace fedhe
