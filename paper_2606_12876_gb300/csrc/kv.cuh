// Declarations shared by the paged key-value cache (kv_api.cu, kv_pages.cu, kv_attend.cu) and
// the RMS norm (norm.cu). Internal; not part of the ABI.
#pragma once

#include "aq_internal.cuh"

namespace aq {

// Power-of-two scale of a block of E4M3 values: the smallest exponent e with amax <= 448 * 2^e,
// kept in [-60, 60]. 448 = 1.75 * 2^8, so e is amax's exponent less 8, and one more where its
// significand is above 1.75. Dividing by 2^e is exact, so the code of a value depends on the
// value and the block's maximum alone. A larger amax (or an infinity) saturates; the bound
// leaves room for products of scales and softmax weights in fp32.
constexpr int kScaleExpMax = 60;
__device__ __forceinline__ int e4m3_scale_exp(float amax) {
    const uint32_t b = __float_as_uint(amax) & 0x7fffffffu;
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return min(max(e, -kScaleExpMax), kScaleExpMax);
}

// Two fp32 values to a pair of E4M3 codes (first value in the low byte), rounded to nearest
// even, saturating at +-448; NaN gives the NaN code.
__device__ __forceinline__ uint16_t e4m3_pair(float first, float second) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(second), "f"(first));
    return r;
}

// 16 bytes that are read once. A coherent load: the kernel ahead may have written them while this one
// was already waiting for it (launch_dependent).
__device__ __forceinline__ uint4 ld_once_v4(const void* p) {
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
                 : "l"(p));
    return r;
}

// Eight consecutive elements of dtype dt (AQ_F16, AQ_BF16, AQ_F32) at element index i, widened to
// fp32; 16-byte aligned. dt is the same for the whole grid, so the branches do not diverge.
__device__ __forceinline__ void load8(const void* p, size_t i, int dt, float (&f)[8]) {
    if (dt == AQ_F32) {
        const float4* q = (const float4*)((const float*)p + i);
        const float4 a = q[0], b = q[1];
        f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
    } else {
        const uint4 v = *(const uint4*)((const uint16_t*)p + i);
        if (dt == AQ_F16) unpack8<AQ_F16>(v, f);
        else unpack8<AQ_BF16>(v, f);
    }
}
// Eight elements as loaded, 16 or 32 bytes (WIDE: fp32), and their widening, apart from each other
// so that a run of loads is not broken by a branch on the type (dt is the same for all threads).
template <bool WIDE>
struct Raw {
    uint4 v[WIDE ? 2 : 1];
    __device__ __forceinline__ void load(const void* p, size_t i) {
        const uint4* q = (const uint4*)((const char*)p + i * (WIDE ? 4 : 2));
        v[0] = q[0];
        if constexpr (WIDE) v[1] = q[1];
    }
    __device__ __forceinline__ void widen(int dt, float (&f)[8]) const {
        if constexpr (WIDE) {
            const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(w[j]);
        } else if (dt == AQ_F16) {
            unpack8<AQ_F16>(v[0], f);
        } else {
            unpack8<AQ_BF16>(v[0], f);
        }
    }
};

__device__ __forceinline__ void store8(void* p, size_t i, int dt, const float (&f)[8]) {
    if (dt == AQ_F32) {
        float4* q = (float4*)((float*)p + i);
        q[0] = make_float4(f[0], f[1], f[2], f[3]);
        q[1] = make_float4(f[4], f[5], f[6], f[7]);
    } else {
        uint4 v;
        if (dt == AQ_F16)
            v = make_uint4(round_pack2<AQ_F16>(f[0], f[1]), round_pack2<AQ_F16>(f[2], f[3]),
                           round_pack2<AQ_F16>(f[4], f[5]), round_pack2<AQ_F16>(f[6], f[7]));
        else
            v = make_uint4(round_pack2<AQ_BF16>(f[0], f[1]), round_pack2<AQ_BF16>(f[2], f[3]),
                           round_pack2<AQ_BF16>(f[4], f[5]), round_pack2<AQ_BF16>(f[6], f[7]));
        *(uint4*)((uint16_t*)p + i) = v;
    }
}
// Eight values times `inv` (a power of two) as E4M3 codes.
__device__ __forceinline__ uint2 e4m3_pack8(const float (&f)[8], float inv) {
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        w[i] = (uint32_t)e4m3_pair(f[4 * i] * inv, f[4 * i + 1] * inv) |
               ((uint32_t)e4m3_pair(f[4 * i + 2] * inv, f[4 * i + 3] * inv) << 16);
    return make_uint2(w[0], w[1]);
}

// A launch that may start before the kernel ahead of it on the stream has finished (programmatic
// dependent launch); every kernel launched this way waits (pdl_wait) before its first access.
template <typename... KArgs, typename... Args>
inline aq_status launch_dependent(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st,
                                  Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cuda_ok(cudaLaunchKernelEx(&cfg, kern, (KArgs)args...), "cudaLaunchKernelEx");
}

// Scratch of the page operations, after the status block of their workspace.
struct KvScratch {
    unsigned int* status;
    int* ctl;      // [0] page pairs to copy, [1] 1 when the operation was carried out, [2] pages in use
    int* marks;    // [max_seqs]: the list entry that names a sequence
    int* prefix;   // [max_seqs + 1]: pages needed by the entries before
    int* count;    // [max_seqs]: an entry's length before the operation
    int* src;      // [num_pages] page pairs
    int* dst;      // [num_pages]
    int* moved;    // [num_pages]: where compaction moved a page
};
constexpr int kCtlInts = 64;
inline size_t kv_scratch_bytes(const aq_kv_cache& c) {
    return kWsStatusBytes + 4 * (kCtlInts + 3 * (size_t)c.max_seqs + 1 + 3 * (size_t)c.num_pages);
}
inline KvScratch kv_scratch(const aq_kv_cache& c, void* ws) {
    KvScratch s;
    s.status = (unsigned int*)ws;
    s.ctl = (int*)((char*)ws + kWsStatusBytes);
    s.marks = s.ctl + kCtlInts;
    s.prefix = s.marks + c.max_seqs;
    s.count = s.prefix + c.max_seqs + 1;
    s.src = s.count + c.max_seqs;
    s.dst = s.src + c.num_pages;
    s.moved = s.dst + c.num_pages;
    return s;
}

// ---- launchers (arguments already validated) ----
aq_status launch_kv_init(const aq_kv_cache& c, cudaStream_t st);
aq_status launch_kv_reserve(const aq_kv_cache& c, int n, const int* seqs, const int* counts, void* ws,
                            cudaStream_t st);
aq_status launch_kv_fork(const aq_kv_cache& c, int n, const int* src, const int* dst, void* ws, cudaStream_t st);
aq_status launch_kv_free(const aq_kv_cache& c, int n, const int* seqs, void* ws, cudaStream_t st);
aq_status launch_kv_compact(const aq_kv_cache& c, int* used, void* ws, cudaStream_t st);
aq_status launch_kv_copy_pages(const aq_kv_cache& c, int n, const int* src, const int* dst, void* ws,
                               cudaStream_t st);
aq_status launch_kv_write(const aq_kv_cache& c, int layer, int n, const int* seqs, const int* positions,
                          const void* k, const void* v, int x_dt, long long stride, void* ws, cudaStream_t st);
size_t kv_attend_ws_bytes(const aq_kv_cache& c, int q_heads);
aq_status launch_kv_attend(const aq_kv_cache& c, const DeviceInfo& di, int layer, int n, const int* seqs,
                           const void* q, int q_dt, long long q_stride, int q_heads, float scale, int window,
                           void* out, float* lse, void* ws, cudaStream_t st);
aq_status launch_rmsnorm(int rows, int cols, const void* x, int x_dt, long long x_stride, const void* residual,
                         void* residual_out, int r_dt, const void* weight, int w_dt, float eps, void* y, int y_dt,
                         uint8_t* y_scales, int scale_block, cudaStream_t st);

}  // namespace aq
