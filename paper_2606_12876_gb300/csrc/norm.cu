// RMS norm with the residual's addition (aq_rmsnorm): h = x + r, y = w h / sqrt(mean h^2 + eps).
//
// Bound: every element is read and written once, with five operations between: HBM for many rows,
// latency for one. A row stays in registers between the sum and the output, so nothing is read
// twice (rows of more than 32768 columns are read again, through L2). Threads take vectors of eight
// elements; all loads of a thread, the weight's too, are issued before the first use, and h is
// written before the row's sum is known. Sums are fp32, over at most 32 elements in a thread (64 in
// rows that are read again) and then pairwise over lanes and warps.
//
// Measured on a GB300, bf16 with a bf16 residual: 4096 x 8192 in 42.9 us (6.26 TB/s of 6.79), 100000 x
// 128 in 15.4 us, 1 x 4096 in 2.2 us back to back.
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

// A sum (or maximum) over the threads of each row: row_threads consecutive ones, a power of two
// below 32 or whole warps. A CTA calls it once with each buffer.
template <bool MAX>
__device__ __forceinline__ float row_reduce(float v, int row_threads, float* buf) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const float o = __shfl_xor_sync(~0u, v, d);
        if (d < row_threads) v = MAX ? fmaxf(v, o) : v + o;
    }
    if (row_threads <= 32) return v;
    const int row_warps = row_threads >> 5;
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

// Eight output values at column c of a row: 16/32-bit, or E4M3 with the block's exponent e.
__device__ __forceinline__ void put(const NormArgs& a, size_t row, int c, const float (&y)[8], int e) {
    if (a.y_dt == AQ_E4M3) *(uint2*)((uint8_t*)a.y + row * a.cols + c) = e4m3_pack8(y, pow2f(-e));
    else store8(a.y, row * a.cols + c, a.y_dt, y);
}

// The exponent of a block of 32 columns, which four lanes hold; its first lane stores the scale.
__device__ __forceinline__ int block_scale(const NormArgs& a, size_t row, int c, bool in, float amax) {
    amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 2));
    const int e = e4m3_scale_exp(amax);
    if (in && (c & 31) == 0) a.scales[row * (a.cols >> 5) + (c >> 5)] = (uint8_t)(e + 127);
    return e;
}

__device__ __forceinline__ float max8(const float (&y)[8]) {
    float m = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(y[j]));
    return m;
}

// row_threads threads per row (see row_reduce), VPT vectors of eight elements each; XW, RW: x and
// the residual are fp32.
template <int VPT, bool XW, bool RW>
__global__ void __launch_bounds__(kMaxThreads) norm_kernel(const __grid_constant__ NormArgs a) {
    __shared__ float buf[2][kMaxThreads / 32];
    pdl_wait();
    pdl_launch_dependents();
    const int group = threadIdx.x / a.row_threads, t = threadIdx.x - group * a.row_threads;
    const size_t row = (size_t)blockIdx.x * (blockDim.x / a.row_threads) + group;
    const bool live = row < (size_t)a.rows;                    // the others take part in the barriers
    Raw<XW> x[VPT];
    Raw<RW> r[VPT];
    Raw<false> w[VPT];
    const bool narrow_w = a.w_dt != AQ_F32;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int c = (v * a.row_threads + t) * 8;
        if (live && c < a.cols) x[v].load(a.x, row * a.x_stride + c);
    }
    if (a.residual)
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int c = (v * a.row_threads + t) * 8;
            if (live && c < a.cols) r[v].load(a.residual, row * a.cols + c);
        }
    if (narrow_w)
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int c = (v * a.row_threads + t) * 8;
            if (live && c < a.cols) w[v].load(a.weight, c);
        }
    float h[VPT][8];
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int c = (v * a.row_threads + t) * 8;
        if (live && c < a.cols) {
            x[v].widen(a.x_dt, h[v]);
            if (a.residual) {
                float f[8];
                r[v].widen(a.r_dt, f);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[v][j] += f[j];
            }
            if (a.residual_out) store8(a.residual_out, row * a.cols + c, a.r_dt, h[v]);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(h[v][j], h[v][j], sum);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) h[v][j] = 0.0f;
        }
    }
    sum = row_reduce<false>(sum, a.row_threads, buf[0]);
    const float inv = rsqrtf(sum / (float)a.cols + a.eps);
    const bool by_row = a.y_dt == AQ_E4M3 && a.scale_block != 32;
    float row_max = 0.0f;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int c = (v * a.row_threads + t) * 8;
        const bool in = live && c < a.cols;
        if (in) {
            float f[8];
            if (narrow_w) w[v].widen(a.w_dt, f);
            else load8(a.weight, c, AQ_F32, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[v][j] = h[v][j] * inv * f[j];
        }
        int e = 0;
        if (a.y_dt == AQ_E4M3) {
            const float amax = max8(h[v]);
            if (by_row) row_max = fmaxf(row_max, amax);
            else e = block_scale(a, row, c, in, amax);
        }
        if (in && !by_row) put(a, row, c, h[v], e);
    }
    if (by_row) {
        row_max = row_reduce<true>(row_max, a.row_threads, buf[1]);
        const int e = e4m3_scale_exp(row_max);
        if (live && t == 0) a.scales[row] = (uint8_t)(e + 127);
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int c = (v * a.row_threads + t) * 8;
            if (live && c < a.cols) put(a, row, c, h[v], e);
        }
    }
}

// Rows that do not fit a CTA's registers: a CTA per row that reads it once for the sum, for a
// row's scale once more, and once for the output. h is written last, as it may replace x or the
// residual.
__global__ void __launch_bounds__(kMaxThreads) norm_long_kernel(const __grid_constant__ NormArgs a) {
    __shared__ float buf[2][kMaxThreads / 32];
    pdl_wait();
    pdl_launch_dependents();
    const size_t row = blockIdx.x;
    auto load_h = [&](int c, float (&h)[8]) {
        load8(a.x, row * a.x_stride + c, a.x_dt, h);
        if (a.residual) {
            float f[8];
            load8(a.residual, row * a.cols + c, a.r_dt, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] += f[j];
        }
    };
    auto scale = [&](int c, float inv, const float (&h)[8], float (&y)[8]) {
        load8(a.weight, c, a.w_dt, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = h[j] * inv * y[j];
    };
    float h[8], y[8], sum = 0.0f;
    for (int c = threadIdx.x * 8; c < a.cols; c += blockDim.x * 8) {
        load_h(c, h);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fmaf(h[j], h[j], sum);
    }
    sum = row_reduce<false>(sum, blockDim.x, buf[0]);
    const float inv = rsqrtf(sum / (float)a.cols + a.eps);
    const bool by_row = a.y_dt == AQ_E4M3 && a.scale_block != 32;
    int e = 0;
    if (by_row) {
        float row_max = 0.0f;
        for (int c = threadIdx.x * 8; c < a.cols; c += blockDim.x * 8) {
            load_h(c, h);
            scale(c, inv, h, y);
            row_max = fmaxf(row_max, max8(y));
        }
        e = e4m3_scale_exp(row_reduce<true>(row_max, blockDim.x, buf[1]));
        if (threadIdx.x == 0) a.scales[row] = (uint8_t)(e + 127);
    }
    for (int c0 = 0; c0 < a.cols; c0 += blockDim.x * 8) {      // (the same trips for all lanes of a block)
        const int c = c0 + threadIdx.x * 8;
        const bool in = c < a.cols;
        float amax = 0.0f;
        if (in) {
            load_h(c, h);
            scale(c, inv, h, y);
            amax = max8(y);
        }
        if (a.y_dt == AQ_E4M3 && !by_row) e = block_scale(a, row, c, in, amax);
        if (in) {
            if (a.residual_out) store8(a.residual_out, row * a.cols + c, a.r_dt, h);
            put(a, row, c, y, e);
        }
    }
}

template <int VPT>
aq_status launch(const NormArgs& a, unsigned grid, unsigned block, cudaStream_t st) {
    const bool xw = a.x_dt == AQ_F32, rw = a.residual && a.r_dt == AQ_F32;
    return launch_dependent(xw ? (rw ? norm_kernel<VPT, true, true> : norm_kernel<VPT, true, false>)
                               : (rw ? norm_kernel<VPT, false, true> : norm_kernel<VPT, false, false>),
                            grid, block, 0, st, a);
}

}  // namespace

aq_status launch_rmsnorm(int rows, int cols, const void* x, int x_dt, long long x_stride, const void* residual,
                         void* residual_out, int r_dt, const void* weight, int w_dt, float eps, void* y, int y_dt,
                         uint8_t* y_scales, int scale_block, cudaStream_t st) {
    NormArgs a = {x, residual, weight, residual_out, y, y_scales, x_stride, rows, cols, x_dt, r_dt, w_dt, y_dt,
                  scale_block, 0, eps};
    DeviceInfo di;
    if (aq_status e = device_info(&di); e != AQ_OK) return e;
    const int vecs = cols / 8;
    if (vecs > 4 * kMaxThreads) return launch_dependent(norm_long_kernel, (unsigned)rows, kMaxThreads, 0, st, a);
    // Threads per row. With few rows as many as there are vectors, as a row's latency is what
    // counts. With many rows each thread has four loads of each operand in flight (4096 x 8192
    // bf16 with residual: 42.8 us with four vectors a thread, 47.1 with two, 51.4 with one), two
    // vectors where one of them is fp32 (2047 x 4096 with an fp32 residual, 8-bit output: 15.9 us,
    // 23.1 with four, which spill 80 to 164 bytes in the 64 registers that 1024 threads leave; the
    // 16-bit form spills 20). Rows of 16385 to 32768 columns need four whatever the types are. Rows of
    // fewer than 32 vectors share a warp.
    int vpt = 1;
    if (vecs <= 32) {
        a.row_threads = 1;
        while (a.row_threads < vecs) a.row_threads *= 2;
    } else {
        if (rows > 2 * di.sms) vpt = vecs <= 64 || x_dt == AQ_F32 || (residual && r_dt == AQ_F32) ? 2 : 4;
        while ((vecs + vpt - 1) / vpt > kMaxThreads) vpt *= 2;
        a.row_threads = (int)round_up((vecs + vpt - 1) / vpt, 32);
    }
    const int per_cta = a.row_threads >= 256 || (rows <= di.sms && vecs > 32) ? 1 : 256 / a.row_threads;
    const unsigned grid = (unsigned)((rows + (long long)per_cta - 1) / per_cta);
    const unsigned block = (unsigned)round_up(a.row_threads * per_cta, 32);
    if (vpt == 1) return launch<1>(a, grid, block, st);
    if (vpt == 2) return launch<2>(a, grid, block, st);
    return launch<4>(a, grid, block, st);
}

}  // namespace aq
