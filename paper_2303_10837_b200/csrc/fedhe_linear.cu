// A linear layer's entries of the sensitivity map:  S[o][i] = sum_k |sum_{t in k} dy[t][o] x[t][i]|  over the samples k, without the
// samples' gradients ever being in memory; every row a sample of its own:  S = |dy|^T |x|.
#include "fedhe_map.cuh"

namespace fedhe {

namespace {

constexpr int TILE = 64, DEPTH = 16;

template <class T>
__global__ void __launch_bounds__(256) linear_map_kernel(const LinearMapArgs a) {
    __shared__ float g[DEPTH][TILE + 4], x[DEPTH][TILE + 4];
    const uint32_t tid = threadIdx.x, ty = tid / 16, tx = tid % 16;
    const size_t o0 = (size_t)blockIdx.y * TILE, i0 = (size_t)blockIdx.x * TILE;
    const bool rows_alone = a.over == SumOver::ROWS;
    float total[4][4] = {};
    const uint32_t samples = rows_alone ? 1 : a.samples;
    int64_t lo = 0, hi = 0;
    for (uint32_t k = 0; k < samples; k++) {
        if (rows_alone) {
            hi = (int64_t)a.rows;
        } else {                                         // whatever the offsets say, rows lie within the matrices
            lo = max((int64_t)a.offsets[k], hi);
            hi = min(max((int64_t)a.offsets[k + 1], lo), (int64_t)a.rows);
        }
        float acc[4][4] = {};
        for (int64_t r0 = lo; r0 < hi; r0 += DEPTH) {
            for (uint32_t i = tid; i < DEPTH * TILE; i += 256) {
                const int64_t r = r0 + i / TILE;
                const size_t c = i % TILE;
                float gv = 0.0f, xv = 0.0f;
                if (r < hi && o0 + c < a.outputs) gv = to_f32(static_cast<const T *>(a.dy.p)[(size_t)r * a.dy.stride + o0 + c]);
                if (r < hi && i0 + c < a.inputs) xv = to_f32(static_cast<const T *>(a.x.p)[(size_t)r * a.x.stride + i0 + c]);
                g[i / TILE][c] = rows_alone ? fabsf(gv) : gv;
                x[i / TILE][c] = rows_alone ? fabsf(xv) : xv;
            }
            __syncthreads();
#pragma unroll
            for (int d = 0; d < DEPTH; d++)
#pragma unroll
                for (int p = 0; p < 4; p++)
#pragma unroll
                    for (int q = 0; q < 4; q++) acc[p][q] = fmaf(g[d][ty * 4 + p], x[d][tx * 4 + q], acc[p][q]);
            __syncthreads();
        }
#pragma unroll
        for (int p = 0; p < 4; p++)
#pragma unroll
            for (int q = 0; q < 4; q++) total[p][q] += fabsf(acc[p][q]);
    }
#pragma unroll
    for (int p = 0; p < 4; p++)
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const size_t o = o0 + ty * 4 + p, i = i0 + tx * 4 + q;
            if (o < a.outputs && i < a.inputs) {
                float *d = a.weight + o * a.inputs + i;
                *d = a.accumulate ? *d + total[p][q] : total[p][q];
            }
        }
}

}  // namespace

size_t linear_map_work_bytes(const LinearMapArgs &a, int dtype, int n_sm) {
    (void)dtype;
    return a.bias ? column_sums_work_bytes(a.rows, a.outputs, n_sm) : 0;
}

cudaError_t launch_linear_map(const LinearMapArgs &a, int dtype, int n_sm, cudaStream_t s) {
    const dim3 grid(blocks_for(a.inputs, TILE), blocks_for(a.outputs, TILE));
    if (dtype == HE_F32) linear_map_kernel<float><<<grid, 256, 0, s>>>(a);
    else if (dtype == HE_BF16) linear_map_kernel<__nv_bfloat16><<<grid, 256, 0, s>>>(a);
    else linear_map_kernel<__half><<<grid, 256, 0, s>>>(a);
    const cudaError_t rc = FEDHE_LAUNCHED();
    if (rc != cudaSuccess || !a.bias) return rc;
    const ColumnSumArgs b{a.dy, a.rows, a.outputs, a.over, a.offsets, a.samples, a.accumulate, a.bias, a.work};
    return launch_column_sums(b, dtype, n_sm, s);
}

}  // namespace fedhe
