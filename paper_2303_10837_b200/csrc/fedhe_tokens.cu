// Log probabilities of given tokens, with the entropy and the top alternatives of every row of logits, and their gradient.
//
//   lse = m + ln s,  m = max z,  s = sum e^(z - m);   log p_y = (z_y - m) - ln s;   H = ln s - (sum e^(z - m) (z - m)) / s
//   dz_j = sum_i g_i (d_{j,t_i} - p_j) - g_H p_j (log p_j + H)        t_i: the target and the alternatives, g_i their gradients
//
// Both directions would be bounded by reading (and writing) the logits once.  The gradient is: 8192 x 32768 in bf16 take 170 us, 6.3 TB/s.  Log
// probabilities of 2048 x 131072 in bf16 take 135 us with eight alternatives, 4.0 TB/s, and 111 without.  888 blocks have a row each at a time: calls
// by themselves without alternatives take 57 us for 888 rows, 70 for 900, 102 for 1776, 107 for 1790, 113 for 2048, 144 for 2664.  So the first rows cost
// a call some 20 us more than their bytes, each new round of rows 4 to 12, and what comes in between runs at 6 to 7 TB/s; issue slots are 71 % used with
// alternatives and without.
#include <cooperative_groups.h>

#include "fedhe_map.cuh"

namespace cg = cooperative_groups;

namespace fedhe {

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float FAR = -1e20f;             // exponents stop here: 2^FAR is 0, and FAR times what a row sums up to is no infinity
// In the gradient ln p stops here, where p is 0 already: times an entropy's gradient of up to 2^120 it is no infinity, which 0 would make NaN (p times
// the gradients first holds for all of them, and takes 193 us for 8192 x 32768 in bf16 with the entropy's where this takes 186).
constexpr float LEAST_LN = -104.0f;
constexpr int PACKS = 4;                  // of 16 bytes, that a thread has of a piece
constexpr uint32_t PLACES = 256;          // for candidates of a warp
constexpr uint32_t DEPTH = 3;             // pieces that a warp asks for ahead
constexpr uint32_t PIECE_BYTES = 32 * PACKS * 16;      // of a warp

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Maximum, sum of 2^t and sum of t 2^t over t = (z - maximum) log2 e, two sums side by side.  All in fp32: sums of up to 2^31 terms that are
// at most 1, as partial sums of the threads.
struct Soft {
    float m;
    F2 s, w;
    __device__ __forceinline__ float base() const { return m == -INFINITY ? 0.0f : m; }
    __device__ __forceinline__ void rise(float to) {         // to a larger maximum
        const float b = to == -INFINITY ? 0.0f : to, d = max_nan((m - b) * LOG2E, FAR), f = ex2(d);
        w = F2(f) * fma2(s, F2(d), w);
        s = s * F2(f);
        m = to;
    }
    __device__ __forceinline__ void add(F2 z, float b) {
        const float2 t = ((z + F2(-b)) * F2(LOG2E)).both();
        const float x = max_nan(t.x, FAR), y = max_nan(t.y, FAR);
        const F2 e(ex2(x), ex2(y));
        s = s + e;
        w = fma2(e, F2(x, y), w);
    }
    // the lanes' to one, in every lane
    __device__ __forceinline__ void join_warp() {
        float to = m;
#pragma unroll
        for (int o = 16; o; o >>= 1) to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, o));
        rise(to);
        s = F2(warp_sum(s.sum()), 0.0f);
        w = F2(warp_sum(w.sum()), 0.0f);
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

// A row's first or last vector, by its elements.
template <class T>
__device__ __noinline__ uint4 load_end(const T *p, int64_t first, uint32_t n) {
    Pack<T, WIDE<T>> a;
#pragma unroll
    for (int e = 0; e < WIDE<T>; e++) {
        const int64_t i = first + e;
        a.v[e] = i >= 0 && i < (int64_t)n ? p[i] : from_f32<T>(-INFINITY);
    }
    uint4 w;
    memcpy(&w, &a, 16);
    return w;
}
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
        const uint4 w = load_end<T>(p, first(v), n);
        Pack<T, V> a;
        memcpy(&a, &w, 16);
        return a;
    }
};

template <class T>
__device__ __forceinline__ float top_of(const Pack<T, WIDE<T>> &p) {          // NaN does not count
    float m = to_f32(p.v[0]);
#pragma unroll
    for (int e = 1; e < WIDE<T>; e++) m = fmaxf(m, to_f32(p.v[e]));
    return m;
}
template <>
__device__ __forceinline__ float top_of<__nv_bfloat16>(const Pack<__nv_bfloat16, 8> &p) {
    const __nv_bfloat162 *w = reinterpret_cast<const __nv_bfloat162 *>(&p);
    const __nv_bfloat162 m = __hmax2(__hmax2(w[0], w[1]), __hmax2(w[2], w[3]));
    return fmaxf(__low2float(m), __high2float(m));
}
template <>
__device__ __forceinline__ float top_of<__half>(const Pack<__half, 8> &p) {
    const __half2 *w = reinterpret_cast<const __half2 *>(&p);
    const __half2 m = __hmax2(__hmax2(w[0], w[1]), __hmax2(w[2], w[3]));
    return fmaxf(__low2float(m), __high2float(m));
}

struct Found {
    uint64_t best[2][HE_MAX_TOP];            // the highest so far, in order: one is written from the other and from the candidates
    uint32_t count[8], bound[8], same[8];    // each warp's candidates; bound, and packs whose maximum is that
    uint64_t most[8];
    uint32_t edge;                           // an order that the first piece has `top` values from on
    uint32_t now, held;                      // which of `best`, and how many are there: for the cluster's first block
};

// The `top` highest of what `best` holds and of the warps' candidates, to the other `best`; returns how many there are.  By the whole block, after a
// barrier; `lost` where a warp had more candidates than places.
__device__ __forceinline__ uint32_t keep_best(Found &f, const uint64_t *key, uint32_t now, uint32_t held, uint32_t top, bool &lost) {
    const uint32_t warps = blockDim.x / 32;
    uint32_t n = held;
    for (uint32_t w = 0; w < warps; w++) {
        lost |= f.count[w] > PLACES;
        n += min(f.count[w], PLACES);
    }
    for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) {
        uint64_t mine = 0;
        if (i < held) {
            mine = f.best[now][i];
        } else {
            uint32_t at = i - held;
            for (uint32_t w = 0; w < warps; w++) {
                const uint32_t c = min(f.count[w], PLACES);
                if (at < c) {
                    mine = key[w * PLACES + at];
                    break;
                }
                at -= c;
            }
        }
        uint32_t above = 0;
#pragma unroll 4
        for (uint32_t j = 0; j < held; j++) above += f.best[now][j] > mine;
        for (uint32_t w = 0; w < warps; w++) {
            const uint32_t c = min(f.count[w], PLACES);
#pragma unroll 4
            for (uint32_t j = 0; j < c; j++) above += key[w * PLACES + j] > mine;
        }
        if (above < top) f.best[now ^ 1u][above] = mine;
    }
    __syncthreads();
    return n < top ? n : top;
}

// The k-th highest of the lanes' orders.
__device__ __forceinline__ uint32_t highest_of_warp(uint32_t mine, uint32_t k) {
    uint32_t got = 0;
    for (uint32_t j = 0; j < k; j++) {
        got = __reduce_max_sync(0xffffffffu, mine);
        const uint32_t who = __ballot_sync(0xffffffffu, mine == got);
        if ((threadIdx.x & 31u) == __ffs(who) - 1) mine = 0;
    }
    return got;
}
// The order of the top-th value of what the block's threads hold, or a little less, given each thread's maximum: in each warp the (top / warps)-th highest
// maximum of a thread, and the lowest of these over the warps.  top is at most the number of threads: a warp has 32 maxima.
__device__ __forceinline__ uint32_t bound_of_top(Found &f, uint32_t mine, uint32_t top) {
    const uint32_t warps = blockDim.x / 32, lane = threadIdx.x & 31u;
    const uint32_t got = highest_of_warp(mine, (top + warps - 1) / warps);
    if (lane == 0) f.bound[threadIdx.x / 32] = got;
    __syncthreads();
    uint32_t low = f.bound[0];
    for (uint32_t i = 1; i < warps; i++) low = min(low, f.bound[i]);
    if (threadIdx.x == 0) f.edge = low;
    return low;
}
// The same of a piece that the row does not fill, where some threads have little or nothing, or that has fewer threads than `top` (a row of 2 KB
// that one warp holds whole, with more than 32 alternatives): in each warp the top-th highest maximum of a pack or a little less,
// found by halving, and the highest of these; where packs are few, the top-th value itself (20000 rows of 300 in bf16 with 64 alternatives: 370 us, and 2330 from
// the packs; 6297 of 860 in fp16 with eight: 55 and 66 from the values).  Returns what a candidate has at least: that, or the next above it where many
// are equal to it.
template <class T>
__device__ __noinline__ float bound_of_part(Found &f, const T *p, uint32_t count, uint32_t v0, uint32_t packs, uint32_t k) {
    constexpr int V = WIDE<T>;
    const Row<T> row(p, count);
    const uint32_t warps = blockDim.x / 32, lane = threadIdx.x & 31u;
    const bool by_value = 4 * k > 3 * packs;
    Pack<T, V> z[PACKS];
    uint32_t o[PACKS], low = 0xffffffffu, high = 0;
#pragma unroll
    for (int i = 0; i < PACKS; i++) {
        const uint32_t v = v0 + i * 32;
        if (v < row.vectors) z[i] = row.load(v);
        else
#pragma unroll
            for (int e = 0; e < V; e++) z[i].v[e] = from_f32<T>(-INFINITY);
        o[i] = order_of(top_of<T>(z[i]));
        low = min(low, o[i]);
        high = max(high, o[i]);
    }
    const bool few = k <= 4;                 // of the threads' maxima, one after the other
    uint32_t got = few ? highest_of_warp(high, k) : __reduce_min_sync(0xffffffffu, low);
    high = few ? got + 1 : __reduce_max_sync(0xffffffffu, high) + 1;
    while (high - got > 1) {                 // k at least are not below `got`, fewer not below `high`
        const uint32_t mid = got + (high - got) / 2;
        uint32_t c = 0;
        if (by_value) {
            const float least = value_of(mid);
#pragma unroll
            for (int i = 0; i < PACKS; i++)
#pragma unroll
                for (int e = 0; e < V; e++) c += to_f32(z[i].v[e]) >= least;
        } else {
#pragma unroll
            for (int i = 0; i < PACKS; i++) c += o[i] >= mid;
        }
        c = __reduce_add_sync(0xffffffffu, c);
        if (c < k) {
            high = mid;
        } else {
            got = mid;
            if (c <= k + k / 4) break;
        }
    }
    uint32_t same = 0;
#pragma unroll
    for (int i = 0; i < PACKS; i++) same += __popc(__ballot_sync(0xffffffffu, o[i] == got));
    if (lane == 0) {
        f.bound[threadIdx.x / 32] = got;
        f.same[threadIdx.x / 32] = same;
    }
    __syncthreads();
    uint32_t bound = 0;
    for (uint32_t i = 0; i < warps; i++) bound = max(bound, f.bound[i]);
    bool above = bound <= order_of(-INFINITY);
    for (uint32_t i = 0; i < warps; i++) above |= f.bound[i] == bound && f.same[i] > 4;
    if (threadIdx.x == 0) f.edge = bound;
    return value_of(bound + above);
}

// Fewer than `top` values were above the order f.edge (of many equal values, or -inf), which the first piece alone has so many values from on:
// the rest are of that order, and those with
// the lowest indices lie in that piece.  By a warp; returns how many there are then.
template <class T>
__device__ __noinline__ uint32_t fill(Found &f, uint32_t now, uint32_t held, const T *p, uint32_t count, uint32_t first, uint32_t top) {
    constexpr int V = WIDE<T>;
    const Row<T> row(p, count);
    const uint32_t lane = threadIdx.x & 31u, piece = blockDim.x * PACKS, edge = f.edge;
    for (uint32_t at = first * piece; at < (first + 1) * piece && at < row.vectors && held < top; at += 32) {
        const uint32_t v = at + lane;
        uint32_t like = 0;
        if (v < row.vectors) {
            const Pack<T, V> z = row.load(v);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const int64_t j = row.first(v) + e;
                like |= (uint32_t)(j >= 0 && j < (int64_t)row.n && order_of(to_f32(z.v[e])) == edge) << e;
            }
        }
        uint32_t upto = __popc(like);
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const uint32_t before = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= (uint32_t)o) upto += before;
        }
        for (uint32_t to = held + upto - __popc(like); like && to < top; like &= like - 1, to++)
            f.best[now][to] = (uint64_t)edge << 32 | (0xffffffffu - (uint32_t)(row.first(v) + __ffs(like) - 1));
        held += __shfl_sync(0xffffffffu, upto, 31);
    }
    return held < top ? held : top;
}

// The alternatives of the pieces first, first + step, ... of a row by one search for each of them: where so many values are above the bound that the
// candidates have no room, as in a row that ascends.
template <class T>
__device__ __noinline__ uint32_t search(Found &f, uint32_t now, const T *p, uint32_t count, uint32_t first, uint32_t step, uint32_t pieces, uint32_t top) {
    constexpr int V = WIDE<T>;
    const Row<T> row(p, count);
    const uint32_t NT = blockDim.x;
    uint64_t below = ~0ull;
    uint32_t n = 0;
    __syncthreads();
    for (; n < top; n++) {
        uint64_t best = 0;
        for (uint32_t c = first; c < pieces; c += step)
            for (uint32_t i = 0; i < PACKS; i++) {
                const uint32_t v = (c * PACKS + i) * NT + threadIdx.x;
                if (v >= row.vectors) break;
                const Pack<T, V> z = row.load(v);
#pragma unroll
                for (int e = 0; e < V; e++) {
                    const int64_t j = row.first(v) + e;
                    const uint64_t k = key_of(to_f32(z.v[e]), (uint32_t)j);
                    if (j >= 0 && j < (int64_t)row.n && k < below && k > best) best = k;
                }
            }
#pragma unroll
        for (int o = 16; o; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
        if ((threadIdx.x & 31u) == 0) f.most[threadIdx.x / 32] = best;
        __syncthreads();
        for (uint32_t w = 0; w < NT / 32; w++) best = max(best, f.most[w]);
        __syncthreads();
        if (best == 0) break;                // a key of an element is not 0: its index is below 2^32 - 1
        if (threadIdx.x == 0) f.best[now][n] = best;
        below = best;
    }
    __syncthreads();
    return n;
}

// Rows by clusters of C blocks (C = 1: by blocks), which take a row's pieces in turn; each warp has its part of a piece, PIECE_BYTES in a row, and
// asks for its parts by bulk copies, DEPTH ahead and on into the next row (asked for in registers, one ahead: 307 us for 2048 x
// 131072 in bf16 with eight alternatives; so 193 then).  Candidates for the alternatives are values above a bound of the top-th value,
// at first from the first piece's, raised after 2, 8, 32, ... pieces, between which some three times as many candidates come as are wanted (after 1, 4, 16: with
// eight alternatives up to 2 us more, with 64 up to 7 % less; after 2, 16, 128: with 64 a third more).
template <class T, bool TOP>
__global__ void __launch_bounds__(256, 3) log_probs_kernel(const LogProbsArgs a, const uint32_t C, int *status) {
    constexpr int V = WIDE<T>;
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ uint64_t bars[8][DEPTH];
    __shared__ float soft[3][8];
    __shared__ float mine[3];
    __shared__ Found f;
    const uint32_t tid = threadIdx.x, NT = blockDim.x, warp = tid / 32, lane = tid & 31u, rank = blockIdx.x % C, clusters = gridDim.x / C;
    const uint32_t rows = (uint32_t)a.rows, first_row = blockIdx.x / C, n = (uint32_t)a.vocab;
    const size_t pitch = a.logits.stride * sizeof(T);
    const uintptr_t base = reinterpret_cast<uintptr_t>(a.logits.p);
    // whole 16 bytes of the matrix: no copy reaches outside
    const uintptr_t low = (base + 15) & ~(uintptr_t)15, high = (base + (rows - 1) * pitch + (size_t)n * sizeof(T)) & ~(uintptr_t)15;
    uint8_t *room = ring + warp * DEPTH * PIECE_BYTES;
    uint64_t *key = reinterpret_cast<uint64_t *>(ring + NT / 32 * DEPTH * PIECE_BYTES), *my_key = key + warp * PLACES;
    const uint32_t room_at = shared_at(room), bar = shared_at(&bars[warp][0]);
    // by a warp's first lane: the piece to ask for next, where it and its row's end are, and the row's pieces
    uint32_t asked_row = first_row, asked = rank, asked_pieces = 0;
    uintptr_t asked_at = 0, asked_end = 0;
    const auto enter = [&] {
        const uintptr_t row = base + asked_row * pitch, start = row & ~(uintptr_t)15, end = (row + (size_t)n * sizeof(T) + 15) & ~(uintptr_t)15;
        asked_pieces = ((uint32_t)((end - start) / 16) + NT * PACKS - 1) / (NT * PACKS);
        asked_at = start + (size_t)(rank * NT + warp * 32) * (PACKS * 16);
        asked_end = end < high ? end : high;
        asked = rank;
    };
    const auto ask = [&](uint32_t d) {
        if (asked_row >= rows) return;
        const uintptr_t at = asked_at < low ? low : asked_at, to = asked_at + PIECE_BYTES < asked_end ? asked_at + PIECE_BYTES : asked_end;
        const uint32_t bytes = to > at ? (uint32_t)(to - at) : 0;
        copies_begin(bar + d * 8, bytes);
        if (bytes) bulk_copy(room_at + d * PIECE_BYTES + (uint32_t)(at - asked_at), at, bytes, bar + d * 8);
        asked += C;
        asked_at += (size_t)C * NT * (PACKS * 16);
        if (asked >= asked_pieces) {
            asked_row += clusters;
            enter();
        }
    };
    if (lane == 0) {
        for (uint32_t d = 0; d < DEPTH; d++) barrier_init(bar + d * 8, 1);
        barriers_ready();
        enter();
        for (uint32_t d = 0; d < DEPTH; d++) ask(d);
    }
    __syncwarp();
    uint32_t d = 0, turn = 0;
    bool gone = false;                       // a copy did not come: none is waited for any more
    for (uint32_t r = first_row; r < rows; r += clusters) {
        const Row<T> row(reinterpret_cast<const T *>(base + r * pitch), n);
        const uint32_t pieces = (row.vectors + NT * PACKS - 1) / (NT * PACKS);
        Soft q{-INFINITY, F2(0.0f), F2(0.0f)};
        uint32_t held = 0, now = 0, round = 0, fresh = 0;      // fresh: this warp's candidates
        // vectors that lie in the row as a whole
        const uint32_t whole_from = row.shift ? 1 : 0, whole_to = (row.n + row.shift) / V;
        float from = -INFINITY;              // what a candidate has at least: that or the next above it, later the next above the top-th value so far
        uint32_t raise = 1;                  // the piece after which the bound is raised next
        bool lost = false;
        const bool filled = (rank + 1) * NT * PACKS <= row.vectors && a.top <= NT;
        if (TOP && !filled && rank < pieces) from = bound_of_part<T>(f, row.p, n, (rank * NT + warp * 32) * PACKS + lane, row.vectors - rank * NT * PACKS, a.top);
        for (uint32_t c = rank; c < pieces; c += C, round++) {
            if (!gone && !copies_done(bar + d * 8, turn)) gone = true;
            Pack<T, V> z[PACKS];
            const uint32_t v0 = (c * NT + warp * 32) * PACKS + lane;
            const uint8_t *in = room + d * PIECE_BYTES + lane * 16;
            const bool inside = v0 - lane >= whole_from && v0 - lane + 32 * PACKS <= whole_to;
            if (inside) {
#pragma unroll
                for (int i = 0; i < PACKS; i++) z[i] = load_pack<T, V>(reinterpret_cast<const T *>(in + i * 512));
            } else {
#pragma unroll
                for (int i = 0; i < PACKS; i++) {
                    const uint32_t v = v0 + i * 32;
                    if (v >= row.vectors) {
#pragma unroll
                        for (int e = 0; e < V; e++) z[i].v[e] = from_f32<T>(-INFINITY);
                    } else if (v >= whole_from && v < whole_to) {
                        z[i] = load_pack<T, V>(reinterpret_cast<const T *>(in + i * 512));
                    } else {
                        z[i] = row.load(v);
                    }
                }
            }
            float m = top_of<T>(z[0]);
#pragma unroll
            for (int i = 1; i < PACKS; i++) m = fmaxf(m, top_of<T>(z[i]));
            if (m != m) m = -INFINITY;
            q.rise(fmaxf(m, q.m));           // without a branch: behind one the warp's two parts would go through all of the piece by themselves
            const float b = q.base();
#pragma unroll
            for (int i = 0; i < PACKS; i++)
#pragma unroll
                for (int e = 0; e < V / 2; e++) q.add(two_of(z[i], e), b);
            if (TOP) {
                if (round == 0 && filled) from = value_of(bound_of_top(f, order_of(m), a.top) + 1);
                // threads that have a candidate, few: the warp looks through the values of one after the other, a lane at each value
                for (uint32_t who = __ballot_sync(0xffffffffu, m >= from); who; who &= who - 1) {
                    const uint32_t l = __ffs(who) - 1, i = lane / V, e = lane % V, j = (v0 - lane + i * 32 + l) * V + e - row.shift;      // outside the row: above n
                    bool hit = i < PACKS && j < n;
                    const float x = !hit ? 0.0f : to_f32(inside ? reinterpret_cast<const T *>(in - lane * 16 + (i * 32 + l) * 16)[e] : row.p[j]);
                    hit = hit && x >= from;
                    const uint32_t hits = __ballot_sync(0xffffffffu, hit), at = fresh + __popc(hits & ((1u << lane) - 1));
                    if (hit && at < PLACES) my_key[at] = key_of(x, j);
                    fresh += __popc(hits);
                }
                if (round == raise || c + C >= pieces) {
                    raise = raise * 4 + 3;
                    if (lane == 0) f.count[warp] = fresh;
                    __syncthreads();
                    held = keep_best(f, key, now, held, a.top, lost);
                    now ^= 1u;
                    fresh = 0;
                    // later pieces have higher indices: with enough candidates a value equal to the lowest of them is too late
                    if (held == a.top) from = fmaxf(from, value_of((uint32_t)(f.best[now][a.top - 1] >> 32) + 1));
                }
            }
            __syncwarp();
            if (lane == 0) ask(d);
            if (++d == DEPTH) d = 0, turn ^= 1u;
        }
        if (TOP) {
            if (held < a.top && rank < pieces) {
                if (warp == 0) {
                    const uint32_t with = fill<T>(f, now, held, row.p, n, rank, a.top);
                    if (lane == 0) f.held = with;
                }
                __syncthreads();
                held = f.held;
            }
            if (lost) held = search<T>(f, now, row.p, n, rank, C, pieces, a.top);
        }
        // the threads' sums, then the warps'
        q.join_warp();
        if (lane == 0) {
            soft[0][warp] = q.m;
            soft[1][warp] = q.s.sum();
            soft[2][warp] = q.w.sum();
        }
        __syncthreads();
        if (tid < 32) {
            // NT / 32 is at most 8: the lanes behind hold nothing
            const bool some = tid < NT / 32;
            q = Soft{some ? soft[0][tid] : -INFINITY, F2(some ? soft[1][tid] : 0.0f, 0.0f), F2(some ? soft[2][tid] : 0.0f, 0.0f)};
            q.join_warp();
            if (tid == 0) {
                mine[0] = q.m;
                mine[1] = q.s.sum();
                mine[2] = q.w.sum();
            }
        }
        if (C > 1) {
            cg::cluster_group cluster = cg::this_cluster();
            if (TOP && tid == 0) {
                f.now = now;
                f.held = held;
            }
            cluster.sync();
            if (rank == 0) {
                if (tid < 32) {
                    const bool some = tid < C;
                    const float *there = cluster.map_shared_rank(mine, some ? tid : 0);
                    q = Soft{some ? there[0] : -INFINITY, F2(some ? there[1] : 0.0f, 0.0f), F2(some ? there[2] : 0.0f, 0.0f)};
                    q.join_warp();
                }
                if (TOP) {
                    // the blocks' alternatives beside one another, as the first warps' candidates
                    for (uint32_t i = tid; i < C * a.top; i += NT) {
                        const Found &there = *cluster.map_shared_rank(&f, i / a.top);
                        key[i] = i % a.top < there.held ? there.best[there.now][i % a.top] : 0;
                    }
                    if (lane == 0) f.count[warp] = warp * PLACES < C * a.top ? min(C * a.top - warp * PLACES, PLACES) : 0;
                    __syncthreads();
                    keep_best(f, key, now, 0, a.top, lost);
                    now ^= 1u;
                }
            }
            cluster.sync();                  // nobody goes on while its memory is read
            if (rank) continue;
            if (tid == 0) {
                mine[0] = q.m;
                mine[1] = q.s.sum();
                mine[2] = q.w.sum();
            }
        }
        __syncthreads();
        const float m = mine[0], sum = mine[1];
        const bool none = sum == 0.0f;       // every value is -inf
        const float ln = logf(sum), b = m == -INFINITY ? 0.0f : m;
        if (tid == 0) {
            a.lse[r] = none ? -INFINITY : b + ln;
            a.entropy[r] = none ? 0.0f : ln - mine[2] / sum * LN2;
            const int64_t y = a.targets[r];
            float lp = 0.0f;
            if (y >= (int64_t)row.n) lp = NAN;
            else if (y >= 0) lp = none ? -INFINITY : (to_f32(row.p[y]) - b) - ln;
            a.logp[r] = lp;
        }
        if (TOP) {
            for (uint32_t i = tid; i < a.top; i += NT) {
                const uint64_t k = f.best[now][i];
                a.top_ids[(size_t)r * a.top + i] = (int64_t)(0xffffffffu - (uint32_t)k);
                a.top_logp[(size_t)r * a.top + i] = none ? -INFINITY : (value_of((uint32_t)(k >> 32)) - b) - ln;
            }
        }
        __syncthreads();                     // `mine` and the candidates are the next row's
    }
    if (gone) copies_lost(status);
}

// Threads of a block: as few as hold a row at once, up to 128, of which an SM has six blocks, so that one's barriers and searches are hidden by the
// others (2048 x 131072 with eight alternatives: 256 threads 189 us, 128 151, 64 190); up to 256 where there are fewer rows than SMs (one row: 14.4
// and 23.2 us).
inline uint32_t row_threads(size_t bytes, size_t rows, int n_sm) {
    const size_t t = (bytes + 15 + PACKS * 16 - 1) / (PACKS * 16), most = rows < (size_t)n_sm ? 256 : 128;
    return t >= most ? (uint32_t)most : (uint32_t)(t + 31) / 32 * 32;
}

template <class T>
cudaError_t log_probs_of(const LogProbsArgs &a, int n_sm, int *status, cudaStream_t s) {
    const uint32_t nt = row_threads(a.vocab * sizeof(T), a.rows, n_sm);
    const size_t pieces = (a.vocab * sizeof(T) + 15 + (size_t)nt * PACKS * 16 - 1) / ((size_t)nt * PACKS * 16);
    const uint32_t bytes = nt / 32 * (DEPTH * PIECE_BYTES + (a.top ? PLACES * 8 : 0));
    // blocks that an SM holds: 768 threads by the registers, and shared memory
    uint32_t held = 768 / nt;
    const uint32_t by_memory = (uint32_t)((222u << 10) / (bytes + (a.top ? sizeof(Found) : 0) + 1536));
    if (held > by_memory) held = by_memory;
    if (held > 24) held = 24;
    const size_t most = (size_t)held * n_sm;
    // few rows: a cluster of up to eight blocks shares one, as long as each has a piece
    uint32_t C = 1;
    while (C < 8 && 2 * C <= pieces && a.rows * 2 * C <= most + n_sm) C *= 2;
    const size_t clusters = most / C ? most / C : 1;
    const auto kernel = a.top ? log_probs_kernel<T, true> : log_probs_kernel<T, false>;
    cudaError_t rc = allow_shared(reinterpret_cast<const void *>(kernel), bytes);
    if (rc != cudaSuccess) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(nt);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {C, 1, 1};
    cfg.attrs = at;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3((unsigned)((C > 1 || a.rows < clusters ? a.rows : clusters) * C));
    rc = cudaLaunchKernelEx(&cfg, kernel, a, C, status);
    if (rc != cudaSuccess) return rc;
    return FEDHE_LAUNCHED();
}

// ---------------------------------------------------------------------------

// What flows into a row.
struct Flow {
    int64_t y;
    float lse, gy, G, gh, H;                 // gradients of the target's log probability, of all log probabilities, of the entropy; the entropy
    bool still;                              // nothing flows, or every logit is -inf: whatever the row holds, zeros come out
};

// Warps take parts of rows in turn, `run` pieces of PIECE_BYTES each, and ask for the pieces by bulk copies, GRAD_DEPTH ahead; a part needs nothing but
// its row's numbers, so no warp waits for another.  The elements that a gradient falls on by itself (the target, the alternatives) get it before the one rounding.
constexpr uint32_t GRAD_THREADS = 128, GRAD_DEPTH = 4, GRAD_BLOCKS = 4;
template <class T, bool ENTROPY, bool TOP>
__global__ void __launch_bounds__(GRAD_THREADS, GRAD_BLOCKS) log_probs_grad_kernel(const LogProbsGradArgs a, const uint32_t pieces, const uint32_t run, const bool stream, int *status) {
    constexpr int V = WIDE<T>;
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ uint64_t bars[GRAD_THREADS / 32][GRAD_DEPTH];
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31u, rows = (uint32_t)a.rows, n = (uint32_t)a.vocab;
    const uint32_t warps = gridDim.x * (GRAD_THREADS / 32), me = blockIdx.x * (GRAD_THREADS / 32) + warp;
    const uint32_t parts = (pieces + run - 1) / run, rows_on = warps / parts, parts_on = warps % parts;       // from a warp's part to its next one
    const size_t pitch = a.logits.stride * sizeof(T);
    const uintptr_t base = reinterpret_cast<uintptr_t>(a.logits.p);
    const uintptr_t low = (base + 15) & ~(uintptr_t)15, high = (base + (rows - 1) * pitch + (size_t)n * sizeof(T)) & ~(uintptr_t)15;
    uint8_t *room = ring + warp * GRAD_DEPTH * PIECE_BYTES;
    const uint32_t room_at = shared_at(room), bar = shared_at(&bars[warp][0]);
    const auto on = [&](uint32_t &row, uint32_t &part) {
        row += rows_on;
        part += parts_on;
        if (part >= parts) part -= parts, row++;
    };
    uint32_t asked_row = me / parts, asked = me % parts, asked_left = 0;       // by the first lane: the part whose pieces are asked for
    uintptr_t asked_at = 0, asked_end = 0;
    const auto enter = [&] {
        const uintptr_t row = base + asked_row * pitch;
        asked_at = (row & ~(uintptr_t)15) + (size_t)asked * run * PIECE_BYTES;
        asked_end = (row + (size_t)n * sizeof(T) + 15) & ~(uintptr_t)15;
        if (asked_end > high) asked_end = high;
        asked_left = min(run, pieces - asked * run);
    };
    const auto ask = [&](uint32_t d) {
        if (asked_row >= rows) return;
        const uintptr_t at = asked_at < low ? low : asked_at, to = asked_at + PIECE_BYTES < asked_end ? asked_at + PIECE_BYTES : asked_end;
        const uint32_t bytes = to > at ? (uint32_t)(to - at) : 0;
        copies_begin(bar + d * 8, bytes);
        if (bytes) bulk_copy(room_at + d * PIECE_BYTES + (uint32_t)(at - asked_at), at, bytes, bar + d * 8);
        asked_at += PIECE_BYTES;
        if (--asked_left == 0) {
            on(asked_row, asked);
            enter();
        }
    };
    const auto flow_of = [&](uint32_t r) {
        Flow f;
        f.y = a.targets[r];
        f.lse = a.lse[r];
        f.gy = f.y < 0 ? 0.0f : f.y < (int64_t)n ? a.dlogp[r] : NAN;
        f.G = f.gy;
        f.gh = ENTROPY ? a.dentropy[r] : 0.0f;
        f.H = ENTROPY ? a.entropy[r] : 0.0f;
        f.still = f.lse == -INFINITY || (f.y < 0 && !ENTROPY && !TOP);
        return f;
    };
    if (lane == 0) {
        for (uint32_t d = 0; d < GRAD_DEPTH; d++) barrier_init(bar + d * 8, 1);
        barriers_ready();
        enter();
        for (uint32_t d = 0; d < GRAD_DEPTH; d++) ask(d);
    }
    uint32_t r = me / parts, part = me % parts, d = 0, turn = 0;
    bool gone = false;
    Flow next;
    if (r < rows) next = flow_of(r);
    __syncwarp();
    while (r < rows) {
        Flow f = next;
        const Row<T> row(reinterpret_cast<const T *>(base + r * pitch), n);
        T *out = static_cast<T *>(a.dlogits.p) + (size_t)r * a.dlogits.stride;
        const uint32_t whole_from = row.shift ? 1 : 0, whole_to = (row.n + row.shift) / V;
        const bool alike = ((reinterpret_cast<uintptr_t>(row.p) ^ reinterpret_cast<uintptr_t>(out)) & 15u) == 0;
        uint32_t r_next = r, part_next = part;
        on(r_next, part_next);
        if (r_next < rows) next = flow_of(r_next);
        if (TOP) {
            float sum = 0.0f;
            for (uint32_t i = lane; i < a.top; i += 32) sum += a.dtop[(size_t)r * a.top + i];
            f.G += warp_sum(sum);
        }
        const uint32_t to = min(part * run + run, pieces) * (32 * PACKS);
        for (uint32_t v0 = part * run * (32 * PACKS); v0 < to; v0 += 32 * PACKS) {
            const bool inside = v0 >= whole_from && v0 + 32 * PACKS <= whole_to;
            // whether the target or an alternative lies in this piece
            const int64_t first = row.first(v0), behind = first + 32 * PACKS * V;
            bool hit = f.y >= first && f.y < behind;
            if (TOP) {
                for (uint32_t i = lane; i < a.top; i += 32) {
                    const int64_t id = a.top_ids[(size_t)r * a.top + i];
                    hit = hit || (id >= first && id < behind);
                }
                hit = __any_sync(0xffffffffu, hit);
            }
            if (!gone && !copies_done(bar + d * 8, turn)) gone = true;
            const uint8_t *in = room + d * PIECE_BYTES + lane * 16;
            Pack<T, V> z[PACKS];
            if (inside) {
#pragma unroll
                for (int i = 0; i < PACKS; i++) z[i] = load_pack<T, V>(reinterpret_cast<const T *>(in + i * 512));
            } else {
#pragma unroll
                for (int i = 0; i < PACKS; i++) {
                    const uint32_t v = v0 + i * 32 + lane;
                    if (v >= whole_from && v < whole_to) z[i] = load_pack<T, V>(reinterpret_cast<const T *>(in + i * 512));
                    else if (v < row.vectors) z[i] = row.load(v);
                    else
#pragma unroll
                        for (int e = 0; e < V; e++) z[i].v[e] = from_f32<T>(0.0f);
                }
            }
            __syncwarp();
            if (lane == 0) ask(d);
            if (++d == GRAD_DEPTH) d = 0, turn ^= 1u;
#pragma unroll
            for (int i = 0; i < PACKS; i++) {
                const uint32_t v = v0 + i * 32 + lane;
                F2 g[V / 2];
#pragma unroll
                for (int e = 0; e < V / 2; e++) {
                    const F2 l = two_of(z[i], e) + F2(-f.lse);
                    if (ENTROPY) {
                        float2 lp = l.both();
                        lp.x = max_nan(lp.x, LEAST_LN);
                        lp.y = max_nan(lp.y, LEAST_LN);
                        const float2 t = (F2(lp.x, lp.y) * F2(LOG2E)).both();
                        g[e] = F2(-ex2(t.x), -ex2(t.y)) * fma2(F2(f.gh), F2(lp.x, lp.y) + F2(f.H), F2(f.G));
                    } else {
                        const float2 t = (l * F2(LOG2E)).both();
                        g[e] = F2(ex2(t.x), ex2(t.y)) * F2(-f.G);
                    }
                }
                if (hit) {
                    const int64_t j = row.first(v);
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        float more = j + e == f.y ? f.gy : 0.0f;
                        if (TOP)
                            for (uint32_t k = 0; k < a.top; k++)
                                if (a.top_ids[(size_t)r * a.top + k] == j + e) more += a.dtop[(size_t)r * a.top + k];
                        g[e / 2] = g[e / 2] + (e % 2 ? F2(0.0f, more) : F2(more, 0.0f));
                    }
                }
                Pack<T, V> o;
#pragma unroll
                for (int e = 0; e < V / 2; e++) set_two(o, e, f.still ? F2(0.0f) : g[e]);
                if (alike && (inside || (v >= whole_from && v < whole_to))) {
                    if (stream) __stcs(reinterpret_cast<uint4 *>(out + row.first(v)), *reinterpret_cast<const uint4 *>(&o));
                    else store_pack<T, V>(out + row.first(v), o);
                } else if (v < row.vectors) {
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        const int64_t j = row.first(v) + e;
                        if (j >= 0 && j < (int64_t)row.n) out[j] = o.v[e];
                    }
                }
            }
        }
        r = r_next;
        part = part_next;
    }
    if (gone) copies_lost(status);
}

template <class T>
cudaError_t log_probs_grad_of(const LogProbsGradArgs &a, int n_sm, int *status, cudaStream_t s) {
    const uint32_t pieces = (uint32_t)((a.vocab * sizeof(T) + 15 + PIECE_BYTES - 1) / PIECE_BYTES), bytes = GRAD_THREADS / 32 * GRAD_DEPTH * PIECE_BYTES;
    // Parts of two pieces, so that warps that run side by side read and write side by side, and results that no cache holds past the caches
    // (8192 x 32768 in bf16: parts of 16 pieces 219 us, of two 215; past the caches 211; with four blocks instead of six on an SM 170).
    const size_t most = (size_t)GRAD_BLOCKS * n_sm, warps = most * GRAD_THREADS / 32;
    const uint32_t run = a.rows * ((pieces + 1) / 2) < 4 * warps ? 1 : 2;
    const bool stream = a.rows * a.vocab * sizeof(T) > (size_t)64 << 20;
    const size_t blocks = (a.rows * ((pieces + run - 1) / run) + GRAD_THREADS / 32 - 1) / (GRAD_THREADS / 32);
    const auto kernel = a.top           ? (a.dentropy ? log_probs_grad_kernel<T, true, true> : log_probs_grad_kernel<T, false, true>)
                        : a.dentropy    ? log_probs_grad_kernel<T, true, false>
                                        : log_probs_grad_kernel<T, false, false>;
    const cudaError_t rc = allow_shared(reinterpret_cast<const void *>(kernel), bytes);
    if (rc != cudaSuccess) return rc;
    kernel<<<(unsigned)(blocks < most ? blocks : most), GRAD_THREADS, bytes, s>>>(a, pieces, run, stream, status);
    return FEDHE_LAUNCHED();
}

}  // namespace

cudaError_t launch_log_probs(const LogProbsArgs &a, int dtype, int n_sm, int *status, cudaStream_t s) {
    return dtype == HE_F32    ? log_probs_of<float>(a, n_sm, status, s)
           : dtype == HE_BF16 ? log_probs_of<__nv_bfloat16>(a, n_sm, status, s)
                              : log_probs_of<__half>(a, n_sm, status, s);
}

cudaError_t launch_log_probs_grad(const LogProbsGradArgs &a, int dtype, int n_sm, int *status, cudaStream_t s) {
    return dtype == HE_F32    ? log_probs_grad_of<float>(a, n_sm, status, s)
           : dtype == HE_BF16 ? log_probs_grad_of<__nv_bfloat16>(a, n_sm, status, s)
                              : log_probs_grad_of<__half>(a, n_sm, status, s);
}

}  // namespace fedhe
