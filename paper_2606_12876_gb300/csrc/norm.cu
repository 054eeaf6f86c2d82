// RMS norm with the residual's addition (aq_rmsnorm): h = x + r, y = w h / sqrt(mean h^2 + eps).
//
// Bound: every element is read and written once, with five operations between: HBM for many rows,
// latency for one. A row stays in registers between the sum and the output, so nothing is read
// twice; threads take vectors of eight elements (16 or 32 bytes a load). Sums are fp32, over at
// most 64 elements in a thread and then pairwise over lanes and warps.
#include "kv.cuh"

namespace aq {
namespace {

constexpr int kMaxThreads = 1024;

struct NormArgs {
    const void *x, *residual, *weight;
    void *residual_out, *y;
    uint8_t* scales;
    long long x_stride;
    int rows, cols, x_dt, r_dt, w_dt, y_dt, scale_block, row_threads;
    float eps;
};

// A sum (or maximum) over the threads of each row: row_warps consecutive warps.
template <bool MAX>
__device__ __forceinline__ float row_reduce(float v, int row_warps, float* buf) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const float o = __shfl_xor_sync(~0u, v, d);
        v = MAX ? fmaxf(v, o) : v + o;
    }
    if (row_warps == 1) return v;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, first = warp / row_warps * row_warps;
    if (lane == 0) buf[warp] = v;
    __syncthreads();
    v = lane < row_warps ? buf[first + lane] : 0.0f;          // (sums and maxima of magnitudes: 0 is neutral)
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const float o = __shfl_xor_sync(~0u, v, d);
        v = MAX ? fmaxf(v, o) : v + o;
    }
    return v;
}

// row_threads (a multiple of 32) threads per row, VPT vectors of eight elements each.
template <int VPT>
__global__ void __launch_bounds__(kMaxThreads) norm_kernel(NormArgs a) {
    __shared__ float buf[2][kMaxThreads / 32];
    pdl_wait();
    pdl_launch_dependents();
    const int group = threadIdx.x / a.row_threads, t = threadIdx.x - group * a.row_threads;
    const int row = blockIdx.x * (blockDim.x / a.row_threads) + group;
    const bool live = row < a.rows;                            // the others take part in the barriers
    const int row_warps = a.row_threads >> 5;
    float h[VPT][8];
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int c = (v * a.row_threads + t) * 8;
        if (live && c < a.cols) {
            load8(a.x, (size_t)row * a.x_stride + c, a.x_dt, h[v]);
            if (a.residual) {
                float r[8];
                load8(a.residual, (size_t)row * a.cols + c, a.r_dt, r);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[v][j] += r[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(h[v][j], h[v][j], sum);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) h[v][j] = 0.0f;
        }
    }
    sum = row_reduce<false>(sum, row_warps, buf[0]);
    const float inv = rsqrtf(sum / (float)a.cols + a.eps);
    float row_max = 0.0f;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int c = (v * a.row_threads + t) * 8;
        const bool in = live && c < a.cols;
        float w[8] = {};
        if (in) {
            if (a.residual_out) store8(a.residual_out, (size_t)row * a.cols + c, a.r_dt, h[v]);
            load8(a.weight, c, a.w_dt, w);
        }
        float amax = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            h[v][j] = h[v][j] * inv * w[j];
            amax = fmaxf(amax, fabsf(h[v][j]));
        }
        if (a.y_dt != AQ_E4M3) {
            if (in) store8(a.y, (size_t)row * a.cols + c, a.y_dt, h[v]);
        } else if (a.scale_block == 32) {                      // four lanes hold a block
            amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 1));
            amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 2));
            const int e = e4m3_scale_exp(amax);
            if (in) {
                *(uint2*)((uint8_t*)a.y + (size_t)row * a.cols + c) = e4m3_pack8(h[v], pow2f(-e));
                if ((t & 3) == 0) a.scales[(size_t)row * (a.cols >> 5) + (c >> 5)] = (uint8_t)(e + 127);
            }
        } else {
            row_max = fmaxf(row_max, amax);
        }
    }
    if (a.y_dt == AQ_E4M3 && a.scale_block != 32) {
        row_max = row_reduce<true>(row_max, row_warps, buf[1]);
        const int e = e4m3_scale_exp(row_max);
        if (live && t == 0) a.scales[row] = (uint8_t)(e + 127);
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int c = (v * a.row_threads + t) * 8;
            if (live && c < a.cols) *(uint2*)((uint8_t*)a.y + (size_t)row * a.cols + c) = e4m3_pack8(h[v], pow2f(-e));
        }
    }
}

}  // namespace

aq_status launch_rmsnorm(int rows, int cols, const void* x, int x_dt, long long x_stride, const void* residual,
                         void* residual_out, int r_dt, const void* weight, int w_dt, float eps, void* y, int y_dt,
                         uint8_t* y_scales, int scale_block, cudaStream_t st) {
    NormArgs a = {x, residual, weight, residual_out, y, y_scales, x_stride, rows, cols, x_dt, r_dt, w_dt, y_dt,
                  scale_block, 0, eps};
    DeviceInfo di;
    if (aq_status e = device_info(&di); e != AQ_OK) return e;
    // Threads per row: with few rows as many as there are vectors (the row's latency is what
    // counts), with many rows four vectors a thread.
    const int vecs = cols / 8;
    int vpt = rows <= 2 * di.sms ? 1 : vecs <= 32 ? 1 : vecs <= 64 ? 2 : 4;
    while ((vecs + vpt - 1) / vpt > kMaxThreads) vpt *= 2;
    a.row_threads = (int)round_up((vecs + vpt - 1) / vpt, 32);
    const int per_cta = a.row_threads >= 256 || rows <= di.sms ? 1 : 256 / a.row_threads;
    const unsigned grid = (unsigned)((rows + (long long)per_cta - 1) / per_cta), block = a.row_threads * per_cta;
    if (vpt == 1) return launch_dependent(norm_kernel<1>, grid, block, 0, st, a);
    if (vpt == 2) return launch_dependent(norm_kernel<2>, grid, block, 0, st, a);
    if (vpt == 4) return launch_dependent(norm_kernel<4>, grid, block, 0, st, a);
    return launch_dependent(norm_kernel<8>, grid, block, 0, st, a);
}

}  // namespace aq
