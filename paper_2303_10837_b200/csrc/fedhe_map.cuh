// What the kernels of the sensitivity map share (fedhe_tokens.cu, fedhe_norm.cu, fedhe_linear.cu): element types, loads of
// rows at any alignment, sums over a warp.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "fedhe_kernels.cuh"
#include "fedhe_map.h"

namespace fedhe {

// Dynamic shared memory of a block, at most: all that there is less what the kernels hold besides (11 KB) and the system's 1 KB.
constexpr size_t MOST_SHARED = 216 << 10;
// A kernel's shared memory beyond 48 KB has to be allowed, for each device: asked for once by each host thread, and for the most that any call needs,
// so that no other thread's call lowers it.
inline cudaError_t allow_shared(const void *kernel, size_t bytes) {
    struct Allowed {
        const void *kernel;
        int device;
    };
    constexpr int PLACES = 64;
    thread_local Allowed known[PLACES] = {};
    int device = 0;
    if (bytes <= 32 << 10) return cudaSuccess;
    if (bytes > MOST_SHARED) return cudaErrorInvalidValue;
    const cudaError_t rc = cudaGetDevice(&device);
    if (rc != cudaSuccess) return rc;
    Allowed &a = known[(reinterpret_cast<uintptr_t>(kernel) / 16 + device * 7) % PLACES];
    if (a.kernel == kernel && a.device == device) return cudaSuccess;
    const cudaError_t set = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)MOST_SHARED);
    if (set == cudaSuccess) a = Allowed{kernel, device};
    return set;
}

// ---- a kernel that begins before the one ahead of it on the stream has ended ----
//
// Of the kernels that a call launches, the later ones may begin when every block of the one before has said next_may_begin(), and have to say
// before_is_done() ahead of using what it leaves; one block at least says that before it ends, so that what is behind the call on the stream finds all
// of it done (no more than one where there are others to come: blocks that wait keep their places).  A call's first kernel is launched as usual.
__device__ __forceinline__ void next_may_begin() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void before_is_done() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <class... P>
cudaError_t launch_early(bool early, void (*kernel)(P...), dim3 grid, uint32_t threads, size_t shared, cudaStream_t s, const P &...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = early ? 1 : 0;
    const cudaError_t rc = cudaLaunchKernelEx(&cfg, kernel, args...);
    return rc != cudaSuccess ? rc : FEDHE_LAUNCHED();
}

template <class T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

template <class T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// V elements that one access moves: 16 bytes, or a single element where rows are not aligned to that.
template <class T, int V>
struct alignas(V * sizeof(T)) Pack {
    T v[V];
};
template <class T>
constexpr int WIDE = 16 / sizeof(T);

template <class T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T *p) {
    return *reinterpret_cast<const Pack<T, V> *>(p);
}
template <class T, int V>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, V> &a) {
    *reinterpret_cast<Pack<T, V> *>(p) = a;
}

// a weight of a type that is known at run time (they are read once per thread block)
__device__ __forceinline__ float load_weight(const void *p, int dtype, size_t i) {
    return dtype == HE_F32    ? static_cast<const float *>(p)[i]
           : dtype == HE_BF16 ? to_f32(static_cast<const __nv_bfloat16 *>(p)[i])
                              : to_f32(static_cast<const __half *>(p)[i]);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Two fp32 values that one instruction works on.
struct F2 {
    unsigned long long v;
    F2() = default;
    __device__ __forceinline__ F2(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ explicit F2(float a) : F2(a, a) {}
    __device__ __forceinline__ float2 both() const {
        float2 r;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
        return r;
    }
    __device__ __forceinline__ float sum() const {
        const float2 r = both();
        return r.x + r.y;
    }
};
__device__ __forceinline__ F2 operator+(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 operator*(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// Elements 2 i and 2 i + 1 of a pack, of more than one.
template <class T, int V>
__device__ __forceinline__ F2 two_of(const Pack<T, V> &p, int i) { return F2(to_f32(p.v[2 * i]), to_f32(p.v[2 * i + 1])); }
template <int V>
__device__ __forceinline__ F2 two_of(const Pack<__nv_bfloat16, V> &p, int i) {
    const uint32_t w = reinterpret_cast<const uint32_t *>(&p)[i];
    return F2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <int V>
__device__ __forceinline__ F2 two_of(const Pack<__half, V> &p, int i) {
    const float2 v = __half22float2(reinterpret_cast<const __half2 *>(&p)[i]);
    return F2(v.x, v.y);
}
template <class T, int V>
__device__ __forceinline__ void set_two(Pack<T, V> &p, int i, F2 x) {
    const float2 v = x.both();
    p.v[2 * i] = from_f32<T>(v.x);
    p.v[2 * i + 1] = from_f32<T>(v.y);
}
template <int V>
__device__ __forceinline__ void set_two(Pack<__nv_bfloat16, V> &p, int i, F2 x) {
    const float2 v = x.both();
    reinterpret_cast<__nv_bfloat162 *>(&p)[i] = __floats2bfloat162_rn(v.x, v.y);
}
template <int V>
__device__ __forceinline__ void set_two(Pack<__half, V> &p, int i, F2 x) {
    const float2 v = x.both();
    reinterpret_cast<__half2 *>(&p)[i] = __floats2half2_rn(v.x, v.y);
}

// The larger one; NaN where one of them is.
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// ---- bulk copies to shared memory, and the barriers that tell of them (by their addresses there) ----

__device__ __forceinline__ uint32_t shared_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copies_begin(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
constexpr uint32_t COPY_TRIES = 256;             // of 10 ms at most
__device__ __forceinline__ bool copies_done(uint32_t bar, uint32_t parity) {
    for (uint32_t i = 0; i < COPY_TRIES; i++) {
        uint32_t done;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 0x989680;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done)
                     : "r"(bar), "r"(parity)
                     : "memory");
        if (done) return true;
    }
    return false;
}

// Copies that did not come in time have 20 ms more before their memory is given up.
static __device__ __noinline__ void copies_lost(int *status) {
    atomicOr(status, STATUS_COPY);
    for (int i = 0; i < 20; i++) __nanosleep(1000000);
}

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barriers_ready() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
// 16-byte aligned both, and a whole number of 16 bytes
__device__ __forceinline__ void bulk_copy(uint32_t to, uintptr_t from, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
}

// Where sample k ends that a row belongs to.  Offsets come from the caller's device memory: whatever they say, `k` stays below
// `count`, and rows that no sample holds have k == count.
struct SampleWalk {
    const int32_t *offsets;
    uint32_t count, k;
    int64_t begin, end;      // of sample k
    // the first sample that ends behind `row`; by a whole warp, whose lanes look at 32 places at once
    __device__ __forceinline__ void seek(const int32_t *off, uint32_t n, int64_t row) {
        offsets = off;
        count = n;
        uint32_t lo = 0, hi = n;
        while (lo < hi) {
            const uint32_t step = (hi - lo + 31) / 32, at = lo + (threadIdx.x & 31u) * step;
            const uint32_t before = __popc(__ballot_sync(0xffffffffu, at < hi && (int64_t)__ldg(off + min(at, n - 1) + 1) <= row));
            hi = min(hi, lo + before * step);
            if (before) lo += (before - 1) * step + 1;
            else hi = lo;
        }
        k = lo;
        bounds();
    }
    __device__ __forceinline__ void bounds() {
        begin = k < count ? (int64_t)__ldg(offsets + k) : INT64_MAX;
        end = k < count ? (int64_t)__ldg(offsets + k + 1) : INT64_MAX;
    }
    __device__ __forceinline__ void next(int64_t row) {      // the next one that ends behind `row`
        do {
            k++;
            bounds();
        } while (k < count && end <= row);
    }
};

}  // namespace fedhe
