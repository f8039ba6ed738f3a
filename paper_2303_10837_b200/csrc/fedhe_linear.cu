// A linear layer's entries of the sensitivity map:  S[o][i] = sum_k |sum_{t in k} dy[t][o] x[t][i]|  over the samples k, without the
// samples' gradients ever being in memory; every row a sample of its own:  S = |dy|^T |x|.
//
// A product of tiles on the tensor cores whose contracted index is the row.  Both operands lie in memory as the tensor cores want
// them with the contracted index second ("MN-major"), so tiles come by TMA and nothing is transposed.  A sample's product is summed in tensor
// memory; the epilogue's warps add its magnitudes to sums that they hold in registers, while the next sample goes to the other half of
// tensor memory.  Only the finished sums leave the chip.
//
// 16384 x 4096 x 1024 in 128 samples (bf16): 147 us, 0.94 PFLOP/s; every row alone, 8192 x 2048 x 2048 (fp16): 59 us, 1.17 PFLOP/s, and 29 for laying the
// magnitudes out.  Bounded by what passes between the roles: a sample's sums are in registers 1300 clocks after its last product, a stage's copies
// and products each some hundred clocks after what they wait for.
#include <cooperative_groups.h>
#include <cuda.h>

#include "fedhe_map.cuh"

namespace cg = cooperative_groups;

namespace fedhe {

namespace {

// Rows of a stage, at most.  What a role does for a stage takes it some 600 clocks of dependent instructions, so stages are large.
constexpr uint32_t DEPTH = 128;
constexpr uint32_t GROUP = 64;                          // columns of a swizzled group: 128 bytes of each row
constexpr uint32_t SLOTS = 16;                          // stages under way, at most
constexpr uint32_t RING_BYTES = 196608;
// Boxes of a copy have 128, 64, 32 or 16 rows.  A stage's rows are rounded up to sixteens, and three or seven of those to four or eight, which one
// box brings; then they are copied in as many boxes as their number has bits.
constexpr int BOXES = 4;
__device__ __forceinline__ uint32_t padded(uint32_t rows) {
    const uint32_t n = (rows + 15) / 16;
    return (n % 4 == 3 ? n + 1 : n) * 16;
}
struct Maps {
    CUtensorMap dy[BOXES], x[BOXES];
};
constexpr uint32_t MOST_N = 256;                        // inputs of a tile; its outputs are the 128 lanes of tensor memory of each block
// Tensor memory adds without rounding to nearest, so that a long sum of magnitudes loses about 2^-24 of itself for each step of 16 rows (8192
// rows in pieces of 512: 2.8e-6 off, of 128: 5.6e-7).  Pieces of so many rows are summed there, and their sums added in fp32.
// Where rows are samples of their own a piece costs no more than its epilogue; a sample's second piece waits for the first one's, so
// those are longer, and their terms of both signs lose less.
constexpr uint32_t PIECE = 512, PIECE_ALONE = 128;
// Warps by role: a stage's way through any of them takes some hundred clocks that nothing hides, so the work between copies and products
// is spread over eight.
constexpr uint32_t COPIES = 4, PRODUCTS = 4, CHECKS = 5, EPILOGUE = 8;      // how many copy; the first warp of the others
constexpr uint32_t THREADS = 512;
constexpr uint32_t STAGING = 128 * (MOST_N + 1) * 4;
constexpr uint32_t TRIES = 256;                         // of 10 ms at most

// ---- the hardware's instructions ----

// One lane of a warp, the same each time.  Instructions of one thread stand behind this and not behind a comparison of the lane: the
// compiler then knows that there is one, and needs no loop over threads around each (four products and their commit took 680 clocks so).
__device__ __forceinline__ bool elected() {
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes != 0;
}

__device__ __forceinline__ uint32_t smem_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t *b, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_at(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void block_meets() { asm volatile("barrier.sync 1, %0;" ::"n"(THREADS) : "memory"); }
// Registers of a warpgroup's threads: the epilogue's need those that the others leave.  At the launch 128 each, 4 * 128 = 2 * 48 + 2 * 208.
template <int N>
__device__ __forceinline__ void registers_less() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void registers_more() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
// Arrives at a barrier of the block `rank` of the cluster.  What it tells of was written by copies, or fenced for them and the tensor cores,
// so no fence of the cluster's scope is asked for here (with one at each of these and of the waits: 119 us instead of 95 for 8192 x 2048 x 2048).
__device__ __forceinline__ void bar_arrive(uint64_t *b, uint32_t rank) {
    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tmbarrier.arrive.shared::cluster.b64 _, [a];\n\t}" ::"r"(smem_at(b)),
                 "r"(rank)
                 : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t *b, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_at(b)), "r"(bytes) : "memory");
}
// By a whole warp; false after TRIES: something that should have come did not.
__device__ __forceinline__ bool bar_wait(uint64_t *b, uint32_t parity) {
    const uint32_t at = smem_at(b);
    for (uint32_t i = 0; i < TRIES; i++) {
        uint32_t done;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 0x989680;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done)
                     : "r"(at), "r"(parity)
                     : "memory");
        if (__all_sync(0xffffffffu, done)) return true;
    }
    return false;
}
// Copies a box to this block's shared memory; with CG = 2 the barrier may be the pair's other block's.
template <int CG>
__device__ __forceinline__ void tma_load(uint32_t to, const CUtensorMap *map, int32_t col, int32_t row, int32_t part, uint32_t bar) {
    if (CG == 1)
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(to), "l"(map),
                     "r"(col), "r"(row), "r"(part), "r"(bar)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(to), "l"(map),
                     "r"(col), "r"(row), "r"(part), "r"(bar)
                     : "memory");
}
__device__ __forceinline__ uint32_t mapped(uint32_t at, uint32_t rank) {      // to the block `rank` of the cluster
    uint32_t there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(rank));
    return there;
}
// An operand in shared memory whose rows (the contracted index) are 128 bytes of a group of 64 columns, swizzled in atoms of eight rows, which
// are 1024 bytes apart; groups are `ring` rows apart.
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t ring) {
    return (uint64_t)((at >> 4) & 0x3fff) | (uint64_t)(ring * 8) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
template <int CG>
__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add) {
    if (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                     "r"(what), "r"((uint32_t)add)
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                     "r"(what), "r"((uint32_t)add)
                     : "memory");
}
// the products issued so far arrive at a barrier when they are done, in both blocks of a pair
template <int CG>
__device__ __forceinline__ void commit(uint64_t *bar, uint16_t blocks) {
    if (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_at(bar)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_at(bar)), "h"(blocks)
                     : "memory");
}
template <int CG>
__device__ __forceinline__ void tmem_take(uint32_t *where) {
    if (CG == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_at(where)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_at(where)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
}
template <int CG>
__device__ __forceinline__ void tmem_give(uint32_t at) {
    if (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(at));
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(at));
}
__device__ __forceinline__ void tmem_order_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_order_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
#define REGS16(v, o)                                                                                                                          \
    "=f"(v[o + 0]), "=f"(v[o + 1]), "=f"(v[o + 2]), "=f"(v[o + 3]), "=f"(v[o + 4]), "=f"(v[o + 5]), "=f"(v[o + 6]), "=f"(v[o + 7]), "=f"(v[o + 8]), \
        "=f"(v[o + 9]), "=f"(v[o + 10]), "=f"(v[o + 11]), "=f"(v[o + 12]), "=f"(v[o + 13]), "=f"(v[o + 14]), "=f"(v[o + 15])
__device__ __forceinline__ void tmem_get32(uint32_t at, float (&v)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
                 : REGS16(v, 0), REGS16(v, 16)
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ void tmem_get64(uint32_t at, float (&v)[64]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];\n\ttcgen05.wait::ld.sync.aligned;"
                 : REGS16(v, 0), REGS16(v, 16), REGS16(v, 32), REGS16(v, 48)
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ void tmem_get16(uint32_t at, float (&v)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\ttcgen05.wait::ld.sync.aligned;"
                 : REGS16(v, 0)
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ void tmem_put16(uint32_t at, const float (&v)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};\n\ttcgen05.wait::st.sync.aligned;" ::"r"(at),
                 "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]),
                 "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
                 : "memory");
}
#undef REGS16

// ---- what every role of a block goes through: the stages of its samples, listed in shared memory ----

struct Stage {
    int32_t row;
    uint32_t what;           // rows (1 .. DEPTH), flags, and from PAIR on which pieces of fp32 values
    static constexpr uint32_t ROWS = 0xff, BEGINS = 1u << 8, ENDS = 1u << 9;           // a piece
    static constexpr uint32_t FIRST = 1u << 10, LAST = 1u << 11, PAIR = 12;            // piece of its sample
};
constexpr uint32_t LISTED = 1024;

// Where the list goes on: entry `at` of sample k.
struct Cursor {
    uint32_t k, end;         // samples
    uint32_t at;
    int32_t lo, hi;          // the rows of a block whose rows are samples of their own
};
// Entries of a sample of `count` rows in pieces of `piece` rows, each `pairs` times over.
__device__ __forceinline__ uint32_t entries_of(uint32_t count, uint32_t piece, uint32_t pairs) {
    const uint32_t whole = count / piece;
    return (whole * (piece / DEPTH) + (count % piece + DEPTH - 1) / DEPTH) * pairs;
}
__device__ __forceinline__ Stage entry_of(int32_t row, uint32_t count, uint32_t piece, uint32_t pairs, uint32_t j, bool alone) {
    const uint32_t per = piece / DEPTH * pairs, n = j / per, in = j % per, behind = n * piece;
    const uint32_t rows = min(piece, count - behind), stages = (rows + DEPTH - 1) / DEPTH, pair = in / stages, c = in % stages;
    uint32_t what = min(DEPTH, rows - c * DEPTH) | pair << Stage::PAIR;
    if (in == 0) what |= Stage::BEGINS;
    if (in + 1 == stages * pairs) what |= Stage::ENDS;
    if (alone || behind == 0) what |= Stage::FIRST;
    if (alone || behind + rows == count) what |= Stage::LAST;
    return Stage{row + (int32_t)(behind + c * DEPTH), what};
}
// The next entries, at most LISTED; by a warp.  What the offsets say is brought within the rows.
__device__ __forceinline__ uint32_t list_stages(Stage *list, Cursor &c, const int32_t *offsets, int32_t rows, uint32_t pairs) {
    const uint32_t lane = threadIdx.x & 31u;
    uint32_t n = 0;
    if (!offsets) {
        const uint32_t count = (uint32_t)(c.hi - c.lo), all = entries_of(count, PIECE_ALONE, pairs);
        n = min(LISTED, all - c.at);
        for (uint32_t i = lane; i < n; i += 32) list[i] = entry_of(c.lo, count, PIECE_ALONE, pairs, c.at + i, true);
        c.at += n;
        return n;
    }
    while (c.k < c.end && n < LISTED) {
        const uint32_t k = c.k + lane;
        int32_t lo = 0, count = 0;
        if (k < c.end) {
            lo = min(max(__ldg(offsets + k), 0), rows);
            count = min(max(__ldg(offsets + k + 1), lo), rows) - lo;
        }
        const uint32_t skip = lane == 0 ? c.at : 0, mine = entries_of((uint32_t)count, PIECE, pairs) - skip;
        uint32_t upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= (uint32_t)o) upto += v;
        }
        const uint32_t from = n + upto - mine, fit = from >= LISTED ? 0 : min(mine, LISTED - from);
        for (uint32_t i = 0; i < fit; i++) list[from + i] = entry_of(lo, (uint32_t)count, PIECE, pairs, skip + i, false);
        // the first sample that did not fit whole
        const uint32_t cut = __ballot_sync(0xffffffffu, fit < mine);
        const uint32_t total = __shfl_sync(0xffffffffu, upto, 31);
        if (cut) {
            const uint32_t who = __ffs(cut) - 1;
            c.at = __shfl_sync(0xffffffffu, skip + fit, who);
            c.k += who;
            return LISTED;
        }
        n += total;
        c.k = min(c.k + 32, c.end);
        c.at = 0;
    }
    return n;
}
// the first offset that is not below a row
__device__ __forceinline__ uint32_t first_at(const int32_t *offsets, uint32_t count, int64_t row) {
    uint32_t lo = 0, hi = count;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if ((int64_t)__ldg(offsets + mid) >= row) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

struct LinearJob {
    const int32_t *offsets;
    uint32_t samples, rows, inputs, outputs;
    uint32_t n, splits, tiles_i;      // inputs of a tile; blocks (or pairs) that share a tile's samples
    uint32_t ring, pairs, what;       // rows that shared memory holds; products of pieces of fp32 operands: 6, or 1; the instruction's descriptor
    bool accumulate, followed;        // followed: by a kernel of the same call
    float *weight;
    int *status;
};

// Which pieces of fp32 values are multiplied, the smallest products first: all of them down to 2^-16 of the whole.
__device__ __forceinline__ uint32_t piece_of_dy(uint32_t pair) { return (0x001120u >> (pair * 4)) & 3u; }   // 0 2 1 1 0 0 from pair 0 on
__device__ __forceinline__ uint32_t piece_of_x(uint32_t pair) { return (0x010102u >> (pair * 4)) & 3u; }    // 2 0 1 0 1 0

// Of a cluster of splits * CG blocks, CG blocks work on a tile of CG * 128 outputs and n inputs: each holds 128 outputs' columns of dy
// and n / CG inputs' columns of x, and the sums of its outputs.
// Rows go through shared memory in a ring, in which a stage takes as many as it has, rounded up to 16.
template <int CG>
__global__ void __launch_bounds__(THREADS, 1) linear_map_kernel(const __grid_constant__ Maps maps, const LinearJob job) {
    extern __shared__ uint8_t raw[];
    // A stage is full, in the block that issues the products, when that block's copying warps have arrived with what they and the other block's
    // copy, and when each block has cleared what came with a sample's last rows; `part`: the block's copies of those.
    __shared__ uint64_t full[SLOTS], part[SLOTS], empty[SLOTS], sum_full[2], sum_empty[2], drained;
    __shared__ uint32_t tmem_base, listed;
    __shared__ alignas(8) Stage list[LISTED + 1];
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid / 32, 0), lane = tid & 31u;
    const uint32_t rank = cluster.block_rank(), half = rank % CG, leader = rank - half, split = rank / CG;
    const uint32_t tile = blockIdx.x / (job.splits * CG);
    const uint32_t o0 = (tile / job.tiles_i) * 128 * CG + half * 128, i0 = (tile % job.tiles_i) * job.n;
    const uint32_t nb = job.n / CG, ib = i0 + half * nb;                       // x's columns in this block
    // groups of 64 columns that hold anything; what multiplies the others lies outside the result
    const uint32_t ga = o0 >= job.outputs ? 0 : min(2u, (job.outputs - o0 + GROUP - 1) / GROUP);
    const uint32_t gb = ib >= job.inputs ? 0 : min((nb + GROUP - 1) / GROUP, (job.inputs - ib + GROUP - 1) / GROUP);
    uint32_t ga_far = 0, gb_far = 0;                                           // of a pair's second block (asked for by its first)
    if (CG == 2) {
        ga_far = o0 + 128 >= job.outputs ? 0 : min(2u, (job.outputs - o0 - 128 + GROUP - 1) / GROUP);
        gb_far = ib + nb >= job.inputs ? 0 : min((nb + GROUP - 1) / GROUP, (job.inputs - ib - nb + GROUP - 1) / GROUP);
    }
    const uint32_t smem = (smem_at(raw) + 1023u) & ~1023u;
    const uint32_t pitch_group = job.ring * 128, shift_x = 2 * pitch_group;
    if (tid == 0) {
        for (uint32_t s = 0; s < SLOTS; s++) {
            bar_init(&full[s], COPIES + CG);
            bar_init(&part[s], COPIES);
            bar_init(&empty[s], 1);
        }
        for (int b = 0; b < 2; b++) {
            bar_init(&sum_full[b], 1);
            bar_init(&sum_empty[b], 8 * CG);
        }
        bar_init(&drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == PRODUCTS) tmem_take<CG>(&tmem_base);
    tmem_order_before();
    cluster.sync();
    tmem_order_after();
    const uint32_t tmem = tmem_base;
    before_is_done();                        // operands that were laid out
    if (job.followed) next_may_begin();

    Cursor next{0, 0, 0, 0, 0};
    const int64_t r0 = (int64_t)job.rows * split / job.splits, r1 = (int64_t)job.rows * (split + 1) / job.splits;
    if (warp == CHECKS) {
        if (job.offsets) {
            // a sample goes to the split in whose share of the rows it begins
            next.k = split == 0 ? 0 : first_at(job.offsets, job.samples, r0);
            next.end = split + 1 == job.splits ? job.samples : first_at(job.offsets, job.samples, r1);
        } else {
            next.lo = (int32_t)r0;
            next.hi = (int32_t)r1;
        }
    }
    bool well = true;
    if (warp < EPILOGUE) {
        registers_less<48>();
        uint32_t stage = 0;                  // of all so far
        uint32_t at = 0;                     // its first row in the ring
        uint32_t used = 0, held = 1, b = 0, parts = 0;
        for (;;) {
            if (warp == CHECKS) {
                const uint32_t n = list_stages(list, next, job.offsets, (int32_t)job.rows, job.pairs);
                if (lane == 0) listed = n;
            }
            block_meets();
            const uint32_t n = listed;
            if (n == 0) break;
            Stage e = list[0];
            if (warp < COPIES) {
                // copies of every second group of dy, and of x
                const bool of_dy = warp < 2;
                const uint32_t odd = warp & 1u, groups = of_dy ? ga : gb, to = smem + (of_dy ? 0 : shift_x);
                const uint32_t mine = (groups + 1 - odd) / 2, far = of_dy ? ga_far : gb_far, of_pair = mine + (far + 1 - odd) / 2;
                const int32_t col = (int32_t)(of_dy ? o0 : ib);
                const CUtensorMap *map = of_dy ? maps.dy : maps.x;
                uint32_t room = job.ring, oldest = 0;                          // the first stage of the list whose rows are not free yet
                for (uint32_t i = 0; well && i < n; i++, stage++) {
                    const uint32_t left = e.what & Stage::ROWS, pair = e.what >> Stage::PAIR, slot = stage % SLOTS, ends = left & 15u;
                    const int32_t plane = job.pairs == 1 ? 0 : (int32_t)(of_dy ? piece_of_dy(pair) : piece_of_x(pair));
                    const int32_t row = e.row;
                    const uint32_t rows = padded(left);
                    e = list[i + 1];
                    while (well && (room < rows || i - oldest >= SLOTS)) {
                        const uint32_t was = stage - (i - oldest);
                        well = bar_wait(&empty[was % SLOTS], was / SLOTS & 1u);
                        room += padded(list[oldest].what & Stage::ROWS);
                        oldest++;
                    }
                    if (!well) break;
                    room -= rows;
                    if (elected()) {
                        const uint32_t bar = ends ? smem_at(&part[slot]) : mapped(smem_at(&full[slot]), leader);
                        if (ends) bar_expect(&part[slot], mine * rows * 128);
                        else if (half == 0) bar_expect(&full[slot], of_pair * rows * 128);
                        for (uint32_t done = 0, r = at; done < rows;) {
                            const uint32_t fit = min(rows - done, job.ring - r), box = __clz((int)min(fit, DEPTH)) - 24, take = 128u >> box;   // fit: 16, 32, ...
                            for (uint32_t g = odd; g < groups; g += 2)
                                tma_load<CG>(to + g * pitch_group + r * 128, map + box, col + (int32_t)(g * GROUP), row + (int32_t)done, plane, bar);
                            done += take;
                            r = r + take == job.ring ? 0 : r + take;
                        }
                        if (ends && half == 0) bar_arrive(&full[slot], leader);
                    }
                    __syncwarp();
                    at += rows;
                    if (at >= job.ring) at -= job.ring;
                }
                for (; well && oldest < n; oldest++) {
                    const uint32_t was = stage - (n - oldest);
                    well = bar_wait(&empty[was % SLOTS], was / SLOTS & 1u);
                }
            } else if (warp == PRODUCTS) {
                if (half == 0)
                    for (uint32_t i = 0; well && i < n; i++, stage++) {
                        const uint32_t what = e.what, slot = stage % SLOTS, sixteens = ((what & Stage::ROWS) + 15) / 16;
                        e = list[i + 1];
                        const bool begins = what & Stage::BEGINS;
                        if (begins) {
                            if (what & Stage::FIRST) held ^= 1;
                            b = what & Stage::FIRST ? held : held ^ 1;
                            well = bar_wait(&sum_empty[b], (used >> b & 1u) ^ 1u);
                            used ^= 1u << b;
                        }
                        if (!well || !bar_wait(&full[slot], stage / SLOTS & 1u)) {
                            well = false;
                            break;
                        }
                        tmem_order_after();
                        if (elected()) {
                            const uint32_t d = tmem + b * MOST_N;
                            const uint64_t oa = operand(smem, job.ring), ob = operand(smem + shift_x, job.ring);
                            if (sixteens == DEPTH / 16 && at + DEPTH <= job.ring) {
#pragma unroll
                                for (uint32_t h = 0; h < DEPTH / 16; h++)
                                    multiply<CG>(d, oa + at * 8 + h * 128, ob + at * 8 + h * 128, job.what, !begins || h);
                            } else {
                                uint32_t r = at;
                                for (uint32_t h = 0; h < sixteens; h++) {
                                    multiply<CG>(d, oa + r * 8, ob + r * 8, job.what, !begins || h);
                                    r += 16;
                                    if (r == job.ring) r = 0;
                                }
                            }
                            commit<CG>(&empty[slot], (uint16_t)(3u << leader));
                            if (what & Stage::ENDS) commit<CG>(&sum_full[b], (uint16_t)(3u << leader));
                        }
                        __syncwarp();
                        at += padded(what & Stage::ROWS);
                        if (at >= job.ring) at -= job.ring;
                    }
            } else {
                // Rows of the next sample, or of none, that came with a sample's last ones count as zeros.  Three warps take the stages in turn; a lane
                // has 16 bytes of the rows of a group.
                for (uint32_t i = 0; well && i < n; i++, stage++) {
                    const uint32_t left = e.what & Stage::ROWS, slot = stage % SLOTS, over = left & 15u;
                    e = list[i + 1];
                    if (stage % (EPILOGUE - CHECKS) == warp - CHECKS) {
                        // The slot's last stage is done with, and with it the last phase of `part`: a warp that asks for the phase after one that
                        // is not over is told that it is.
                        if (stage >= SLOTS) well = bar_wait(&empty[slot], stage / SLOTS & 1u ^ 1u);
                        if (well && over) {
                            well = bar_wait(&part[slot], parts >> slot & 1u);
                            if (!well) break;
                            uint32_t from = at + left - over;    // the sample's last sixteen rows: the ring's end is a multiple of 16
                            if (from >= job.ring) from -= job.ring;
                            for (uint32_t g = lane / 8; g < 2 + nb / GROUP; g += 4) {
                                const uint32_t to = smem + g * pitch_group + from * 128 + lane % 8 * 16;
#pragma unroll
                                for (uint32_t r = 1; r < 16; r++)
                                    if (r >= over) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(to + r * 128), "r"(0) : "memory");
                            }
                            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                            __syncwarp();
                        }
                        if (well && elected()) bar_arrive(&full[slot], leader);
                        __syncwarp();
                    }
                    if (over) parts ^= 1u << slot;
                    at += padded(left);
                    if (at >= job.ring) at -= job.ring;
                }
            }
            block_meets();
        }
        if (warp == PRODUCTS) {
            // products under way use both blocks' memory
            if (half == 0 && elected()) commit<CG>(&drained, (uint16_t)(3u << leader));
            __syncwarp();
            if (!bar_wait(&drained, 0)) well = false;
        }
        // every copy that was waited for is there; after a wait that failed, copies under way get the time to end that they cannot need
        if (!well)
            for (int i = 0; i < 20; i++) __nanosleep(1000000);
        if (!well && lane == 0) atomicOr(job.status, STATUS_COPY);
        cluster.sync();                      // every product of the pair is done, and every sum read
        if (warp == PRODUCTS) {
            tmem_order_after();
            tmem_give<CG>(tmem);
        }
        cluster.sync();
        cluster.sync();
        return;
    }
    // the epilogue's warps: 32 lanes of tensor memory, half of a tile's columns
    registers_more<208>();
    float total[128];
#pragma unroll
    for (int e = 0; e < 128; e++) total[e] = 0.0f;
    const uint32_t cols = job.n / 2, mine = tmem + ((warp & 3u) << 21) + (warp - EPILOGUE) / 4 * cols;
    const auto free_place = [&](uint32_t b) {
        tmem_order_before();
        __syncwarp();
        if (elected()) bar_arrive(&sum_empty[b], leader);
        __syncwarp();
    };
    uint32_t used = 0, held = 1;
    for (;;) {
        block_meets();
        const uint32_t n = listed;
        if (n == 0) break;
        uint32_t now = list[0].what;
        for (uint32_t i = 0; well && i < n; i++) {
            const uint32_t what = now;
            now = list[i + 1].what;
            if (!(what & Stage::ENDS)) continue;
            const bool first = what & Stage::FIRST, last = what & Stage::LAST;
            if (first) held ^= 1;
            const uint32_t b = first ? held : held ^ 1;
            if (!bar_wait(&sum_full[b], used >> b & 1u)) {
                well = false;
                break;
            }
            used ^= 1u << b;
            tmem_order_after();
            const uint32_t at = mine + b * MOST_N;
            if (first && last) {
#pragma unroll
                for (int j = 0; j < 128; j += 64) {
                    if (j + 64 <= cols) {
                        float v[64];
                        tmem_get64(at + j, v);
                        if (j + 64 == cols) free_place(b);       // before what was read last is added
#pragma unroll
                        for (int e = 0; e < 64; e++) total[j + e] += fabsf(v[e]);
                    } else if (j < cols) {
                        float v[32];
                        tmem_get32(at + j, v);
                        free_place(b);
#pragma unroll
                        for (int e = 0; e < 32; e++) total[j + e] += fabsf(v[e]);
                    }
                }
            } else if (!first) {
                // a long sample: its first piece's place holds the sum of its pieces
#pragma unroll
                for (int j = 0; j < 128; j += 16)
                    if (j < cols) {
                        float v[16], u[16];
                        tmem_get16(at + j, v);
                        tmem_get16(mine + held * MOST_N + j, u);
#pragma unroll
                        for (int e = 0; e < 16; e++) u[e] += v[e];
                        if (last) {
#pragma unroll
                            for (int e = 0; e < 16; e++) total[j + e] += fabsf(u[e]);
                        } else {
                            tmem_put16(mine + held * MOST_N + j, u);
                        }
                    }
                free_place(b);
                if (last) free_place(held);
            }
        }
        block_meets();
    }
    if (!well && lane == 0) atomicOr(job.status, STATUS_COPY);
    cluster.sync();                          // every product of the pair is done: the stages' memory takes the sums
    float *sums = reinterpret_cast<float *>(raw + (smem - smem_at(raw)));
    const uint32_t pitch = job.n + 1;
    float *to = sums + ((warp & 3u) * 32 + lane) * pitch + (warp - EPILOGUE) / 4 * cols;
#pragma unroll
    for (int j = 0; j < 128; j += 32)
        if (j < cols)
#pragma unroll
            for (int e = 0; e < 32; e++) to[j + e] = total[j + e];
    cluster.sync();
    // the splits' sums, each block some outputs of its 128
    const uint32_t first = 128 * split / job.splits, behind = 128 * (split + 1) / job.splits;
    const uint32_t width = min(job.n, job.inputs - i0);
    for (uint32_t o = first + warp - EPILOGUE; o < behind; o += 8) {
        if (o0 + o >= job.outputs) break;
        float *out = job.weight + (size_t)(o0 + o) * job.inputs + i0;
        float v[MOST_N / 32];                // a row at once: loads from other blocks take long, stores should not wait for one another
#pragma unroll
        for (int j = 0; j < (int)MOST_N / 32; j++) v[j] = 0.0f;
        for (uint32_t f = 0; f < job.splits; f++) {
            const float *from = job.splits == 1 ? sums : cluster.map_shared_rank(sums, f * CG + half);
#pragma unroll
            for (int j = 0; j < (int)MOST_N / 32; j++)
                if (j * 32 < job.n) v[j] += from[o * pitch + j * 32 + lane];
        }
        if (job.accumulate)
#pragma unroll
            for (int j = 0; j < (int)MOST_N / 32; j++)
                if (j * 32 + lane < width) v[j] += out[j * 32 + lane];
#pragma unroll
        for (int j = 0; j < (int)MOST_N / 32; j++)
            if (j * 32 + lane < width) out[j * 32 + lane] = v[j];
    }
    cluster.sync();                          // nobody leaves while its memory is read
}

// ---- operands that TMA cannot take as they are ----

// The values v as the tensor cores take them: bf16 or fp16 as they are, fp32 as three bf16 pieces whose sum is v (each the rounding
// of what the pieces before it leave; below 2^-110 the last one ends at bf16's smallest step).  An infinity or a NaN is its own first piece: what it
// meets becomes NaN, since an infinity is multiplied by the other factor's smaller pieces too, which are 0 or of either sign.  Magnitudes where rows are samples of their own; those of dy
// are summed on the way, for the bias.
struct StageArgs {
    MatArg in[2];            // x, dy
    uint32_t width[2], pitch[2];
    uint16_t *out[2];
    uint32_t rows;
    bool magnitudes, half;   // half: 16-bit values are fp16
    float *sums;             // null, or [gridDim.y][3][width of dy], of which the first third is written
};
// Blocks take 32 packs of 8 columns and a run of rows; a thread stays with its columns.
constexpr int STAGE_WARPS = 8;
template <class T>
__global__ void __launch_bounds__(32 * STAGE_WARPS) stage_kernel(const StageArgs a) {
    constexpr int PIECES = sizeof(T) == 4 ? 3 : 1, AHEAD = sizeof(T) == 4 ? 2 : 4;
    __shared__ float met[STAGE_WARPS][8][32];
    const int m = blockIdx.z;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x / 32, width = a.width[m], pitch = a.pitch[m], c = (blockIdx.x * 32 + lane) * 8;
    const size_t plane = (size_t)a.rows * pitch;
    const uint32_t lo = (uint32_t)((uint64_t)a.rows * blockIdx.y / gridDim.y), hi = (uint32_t)((uint64_t)a.rows * (blockIdx.y + 1) / gridDim.y);
    const T *in = static_cast<const T *>(a.in[m].p) + c;
    uint16_t *out = a.out[m] + c;
    const bool wide = reinterpret_cast<uintptr_t>(a.in[m].p) % 16 == 0 && a.in[m].stride % (16 / sizeof(T)) == 0 && c + 8 <= width;
    const bool summed = m == 1 && a.sums;
    float sum[8] = {};
    if (c < pitch)
        for (uint32_t r0 = lo + warp; r0 < hi; r0 += STAGE_WARPS * AHEAD) {
            T v[AHEAD][8];
#pragma unroll
            for (int j = 0; j < AHEAD; j++) {
                const uint32_t r = r0 + j * STAGE_WARPS;
                if (r >= hi) break;
                const T *from = in + r * a.in[m].stride;
                if (wide) {
#pragma unroll
                    for (int q = 0; q < (int)sizeof(T) / 2; q++) reinterpret_cast<uint4 *>(v[j])[q] = reinterpret_cast<const uint4 *>(from)[q];
                } else {
#pragma unroll
                    for (int e = 0; e < 8; e++) v[j][e] = c + e < width ? from[e] : T(0);
                }
            }
#pragma unroll
            for (int j = 0; j < AHEAD; j++) {
                const uint32_t r = r0 + j * STAGE_WARPS;
                if (r >= hi) break;
                Pack<uint16_t, 8> o[PIECES];
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    if constexpr (PIECES == 1) {
                        o[0].v[e] = a.magnitudes ? v[j][e] & 0x7fffu : v[j][e];
                    } else {
                        float left = a.magnitudes ? fabsf(v[j][e]) : v[j][e];
                        if (summed) sum[e] += left;
#pragma unroll
                        for (int q = 0; q < 3; q++) {
                            __nv_bfloat16 b = __float2bfloat16_rn(left);
                            // what rounds up to infinity is cut instead
                            if (__hisinf(b) && !isinf(left)) b = __float2bfloat16_rz(left);
                            o[q].v[e] = __bfloat16_as_ushort(b);
                            left = isfinite(left) ? left - __bfloat162float(b) : 0.0f;
                        }
                    }
                }
                if constexpr (PIECES == 1) {
                    if (summed) {
#pragma unroll
                        for (int e = 0; e < 8; e++)
                            sum[e] += a.half ? __half2float(__ushort_as_half(o[0].v[e])) : __bfloat162float(__ushort_as_bfloat16(o[0].v[e]));
                    }
                }
#pragma unroll
                for (int q = 0; q < PIECES; q++) store_pack<uint16_t, 8>(out + q * plane + (size_t)r * pitch, o[q]);
            }
        }
    next_may_begin();
    if (!summed) return;
#pragma unroll
    for (int e = 0; e < 8; e++) met[warp][e][lane] = sum[e];
    __syncthreads();
    const uint32_t l = threadIdx.x / 8, e = threadIdx.x % 8, col = blockIdx.x * 256 + threadIdx.x;
    float all = 0.0f;
#pragma unroll
    for (int w = 0; w < STAGE_WARPS; w++) all += met[w][e][l];
    if (col < width) a.sums[(size_t)blockIdx.y * 3 * width + col] = all;
}

inline uint32_t pitch_of(size_t width) { return (uint32_t)((width + 7) / 8 * 8); }
inline size_t staged_words(size_t rows, size_t width, int dtype) { return (rows * pitch_of(width) * (dtype == HE_F32 ? 3 : 1) + 127) / 128 * 128; }

// ---- launch ----

using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                            const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

Encode tensor_map_encoder() {
    static const Encode got = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) f = nullptr;
        return reinterpret_cast<Encode>(f);
    }();
    return got;
}

// boxes of 64 columns and `box` rows of a matrix of 16-bit elements in `parts` planes
bool tensor_map(CUtensorMap &m, const void *p, size_t width, size_t rows, size_t stride, uint32_t parts, bool half, uint32_t box) {
    const Encode encode = tensor_map_encoder();
    if (!encode) return false;
    const cuuint64_t dims[3] = {width, rows, parts}, strides[2] = {stride * 2, parts == 1 ? stride * 2 : rows * stride * 2};
    const cuuint32_t boxes[3] = {GROUP, box, 1}, steps[3] = {1, 1, 1};
    return encode(&m, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(p), dims, strides, boxes, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr uint32_t SHARED = (RING_BYTES > STAGING ? RING_BYTES : STAGING) + 1024;
constexpr uint32_t MOST_CLUSTER = 8;

cudaError_t configure(cudaLaunchConfig_t &cfg, cudaLaunchAttribute (&at)[2], const void *kernel, uint32_t blocks, uint32_t cluster, bool early, cudaStream_t s) {
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SHARED;
    cfg.stream = s;
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {cluster, 1, 1};
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = early ? 2 : 1;
    return allow_shared(kernel, SHARED);
}

// Clusters of 1 to MOST_CLUSTER blocks that the GPU runs at once.  A cluster stays in a part of the GPU whose SMs it need not fill: of 148 SMs
// clusters of four have 132, of seven 105.  Asked for once by each host thread and device.
struct Clusters {
    int device = -1;
    int count[MOST_CLUSTER + 1];
};
cudaError_t clusters_at_once(const Clusters *&got) {
    thread_local Clusters known;
    int device = 0;
    cudaError_t rc = cudaGetDevice(&device);
    if (rc != cudaSuccess) return rc;
    got = &known;
    if (known.device == device) return cudaSuccess;
    for (uint32_t c = 1; c <= MOST_CLUSTER; c++) {
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute at[2];
        rc = configure(cfg, at, reinterpret_cast<const void *>(linear_map_kernel<1>), c, c, false, nullptr);
        if (rc == cudaSuccess) rc = cudaOccupancyMaxActiveClusters(&known.count[c], linear_map_kernel<1>, &cfg);
        if (rc != cudaSuccess) return rc;
    }
    known.device = device;
    return cudaSuccess;
}

// How a product is shared out: the blocks of a tile, its inputs, and how many share its samples.  The least of an estimate in clocks, fitted to the
// times of all choices at 17 shapes of 64 to 16384 rows and 128 to 8192 columns, where it is 0.8 % above the best on the mean (with as many clusters at
// once as SMs would hold, 40 %: 16384 x 640 x 640 in 512 samples takes 68 us in tiles of 256 shared by eight, 129 shared by seven).  Pairs read x half
// as often: 131 us for 16384 x 2048 x 2048 in 64 samples, 176 by single blocks; small maps have too few tiles for them.
struct Plan {
    uint32_t cg, n, splits;
};
Plan plan_of(const LinearMapArgs &a, uint32_t pairs, const Clusters &clusters) {
    Plan best{1, 64, 1};
    double least = 1e300;
    const size_t pieces = a.over == SumOver::SAMPLES ? (size_t)a.samples : (a.rows + PIECE_ALONE - 1) / PIECE_ALONE;
    for (uint32_t cg = 1; cg <= 2; cg++)
        for (uint32_t n = 64 * cg; n <= MOST_N; n += 64 * cg)
            for (uint32_t c = 1; c * cg <= MOST_CLUSTER; c++) {
                if (c > 1 && c > pieces) break;
                if (clusters.count[c * cg] < 1) continue;
                const double tiles = (double)((a.outputs + 128 * cg - 1) / (128 * cg)) * (double)((a.inputs + n - 1) / n);
                const double waves = ceil(tiles / clusters.count[c * cg]);
                // of a row: its products, or its bytes from L2; of a sample: its way through the epilogue; of a block: its beginning and end
                const double row = fmax(n / 32.0, (128.0 + n / cg) * 2 / 32), sample = 300 + 2.0 * n, block = 4000 + 8.0 * n + (c > 1 ? 1500 : 0);
                const double t = waves * ((double)a.rows / c * pairs * row + ceil((double)pieces / c) * sample + block);
                if (t < least) least = t, best = Plan{cg, n, c};
            }
    return best;
}

template <int CG>
cudaError_t launch(const Maps &maps, const LinearJob &job, uint32_t tiles, bool early, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    cudaError_t rc = configure(cfg, at, reinterpret_cast<const void *>(linear_map_kernel<CG>), tiles * job.splits * CG, job.splits * CG, early, s);
    if (rc != cudaSuccess) return rc;
    rc = cudaLaunchKernelEx(&cfg, linear_map_kernel<CG>, maps, job);
    return rc != cudaSuccess ? rc : FEDHE_LAUNCHED();
}

}  // namespace

bool linear_map_aligned(const MatArg &m, size_t width, int dtype) {
    return dtype != HE_F32 && reinterpret_cast<uintptr_t>(m.p) % 16 == 0 && m.stride % 8 == 0 && m.stride >= width;
}

size_t linear_map_work_bytes(size_t rows, size_t inputs, size_t outputs, int dtype, bool samples, bool aligned, bool bias, int n_sm) {
    size_t bytes = bias ? (column_sums_work_bytes(rows, outputs, n_sm) + 255) / 256 * 256 : 0;
    if (!samples || !aligned) bytes += (staged_words(rows, inputs, dtype) + staged_words(rows, outputs, dtype)) * 2;
    return bytes;
}

cudaError_t launch_linear_map(const LinearMapArgs &a, int dtype, int n_sm, int *status, cudaStream_t s) {
    const bool alone = a.over == SumOver::ROWS;
    // The bias's sums are made by a kernel that begins beside the product, on the SMs that it leaves and where its blocks have ended (16384 x 4096 x 1024 in
    // 128 samples: 151 us, 147 without the bias, 167 with its sums ahead of the product).
    const ColumnSumArgs column{a.dy, a.rows, a.outputs, alone ? SumOver::ALL : a.over, a.offsets, a.samples, a.accumulate, a.bias, a.work};
    if (!a.rows) {
        const cudaError_t rc = a.bias ? launch_column_sums(column, dtype, n_sm, false, s) : cudaSuccess;
        return rc != cudaSuccess || a.accumulate ? rc : cudaMemsetAsync(a.weight, 0, a.inputs * a.outputs * sizeof(float), s);
    }
    float *sums = static_cast<float *>(a.work);
    uint8_t *work = static_cast<uint8_t *>(a.work) + (a.bias ? (column_sums_work_bytes(a.rows, a.outputs, n_sm) + 255) / 256 * 256 : 0);
    size_t runs = 0;                                         // of the sums that laying out makes
    MatArg x = a.x, dy = a.dy;
    uint32_t parts = 1;
    if (alone || !linear_map_aligned(a.x, a.inputs, dtype) || !linear_map_aligned(a.dy, a.outputs, dtype)) {
        uint16_t *to = reinterpret_cast<uint16_t *>(work);
        const bool summed = alone && a.bias;
        const StageArgs g{{a.x, a.dy}, {(uint32_t)a.inputs, (uint32_t)a.outputs}, {pitch_of(a.inputs), pitch_of(a.outputs)}, {to, to + staged_words(a.rows, a.inputs, dtype)},
                          (uint32_t)a.rows, alone, dtype == HE_F16, summed ? sums : nullptr};
        const uint32_t columns = (g.pitch[0] > g.pitch[1] ? g.pitch[0] : g.pitch[1]) / 8;
        // as many runs as column_sums_work_bytes() has room for, at most; four blocks on an SM
        const size_t cols = (columns + 31) / 32, wanted = ((size_t)2 * n_sm + cols - 1) / cols, rows = (a.rows + STAGE_WARPS - 1) / STAGE_WARPS;
        runs = wanted < rows ? wanted : rows;
        if (runs > (size_t)n_sm) runs = n_sm;
        const dim3 grid((unsigned)cols, (unsigned)runs, 2);
        if (dtype == HE_F32) stage_kernel<float><<<grid, 32 * STAGE_WARPS, 0, s>>>(g);
        else stage_kernel<uint16_t><<<grid, 32 * STAGE_WARPS, 0, s>>>(g);
        const cudaError_t rc = FEDHE_LAUNCHED();
        if (rc != cudaSuccess) return rc;
        x = MatArg{g.out[0], g.pitch[0]};
        dy = MatArg{g.out[1], g.pitch[1]};
        parts = dtype == HE_F32 ? 3 : 1;
    }
    const bool laid_out = x.p != a.x.p;
    const uint32_t pairs = parts == 3 ? 6 : 1;
    const Clusters *clusters;
    const cudaError_t asked = clusters_at_once(clusters);
    if (asked != cudaSuccess) return asked;
    const Plan plan = plan_of(a, pairs, *clusters);
    Maps maps;
    const bool half = dtype == HE_F16;
    for (int i = 0; i < BOXES; i++)
        if (!tensor_map(maps.dy[i], dy.p, a.outputs, a.rows, dy.stride, parts, half, 128u >> i) ||
            !tensor_map(maps.x[i], x.p, a.inputs, a.rows, x.stride, parts, half, 128u >> i))
            return cudaErrorInvalidValue;
    LinearJob job{};
    job.offsets = alone ? nullptr : a.offsets;
    job.samples = a.samples;
    job.rows = (uint32_t)a.rows;
    job.inputs = (uint32_t)a.inputs;
    job.outputs = (uint32_t)a.outputs;
    job.n = plan.n;
    job.splits = plan.splits;
    job.tiles_i = (uint32_t)((a.inputs + plan.n - 1) / plan.n);
    job.ring = RING_BYTES / (128 * (2 + plan.n / plan.cg / GROUP)) / 16 * 16;
    job.pairs = pairs;
    // fp32 sums; both operands fp16 or bf16, with the contracted index second; n columns, 128 rows for each block
    const uint32_t type = half ? 0 : 1;
    job.what = 1u << 4 | type << 7 | type << 10 | 1u << 15 | 1u << 16 | (plan.n >> 3) << 17 | (128 * plan.cg >> 4) << 24;
    job.accumulate = a.accumulate;
    job.followed = a.bias != nullptr;
    job.weight = a.weight;
    job.status = status;
    const uint32_t tiles = (uint32_t)((a.outputs + 128 * plan.cg - 1) / (128 * plan.cg)) * job.tiles_i;
    const cudaError_t rc = plan.cg == 1 ? launch<1>(maps, job, tiles, laid_out, s) : launch<2>(maps, job, tiles, laid_out, s);
    if (rc != cudaSuccess || !a.bias) return rc;
    return alone ? launch_join_sums(sums, (uint32_t)runs, a.outputs, a.accumulate, a.bias, s) : launch_column_sums(column, dtype, n_sm, true, s);
}

}  // namespace fedhe
