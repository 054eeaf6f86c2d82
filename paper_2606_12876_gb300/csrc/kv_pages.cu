// Pages of the key-value cache: allocation (aq_kv_reserve), sharing (aq_kv_fork), release
// (aq_kv_free), compaction (aq_kv_compact), plain copies (aq_kv_copy_pages), and the writes of new
// keys and values (aq_kv_write).
//
// All of the cache's bookkeeping lives on the device (tables, lengths, reference counts), so a
// decode loop that grows sequences, forks beams and drops them is ordered by its stream alone and
// can be captured in a CUDA graph. A page is free when its reference count is 0, and allocation
// takes the lowest free indices, in list order: counts are only added to and subtracted from, and
// every other decision is made in one CTA, so the outcome does not depend on scheduling. A page
// shared by several sequences is always full (a fork copies a partial last page), so no write
// ever needs to ask whether its page is shared.
#include <climits>

#include "kv.cuh"

namespace aq {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanPages = 16;         // reference counts a thread looks at per step
constexpr int kCopyThreads = 256;
constexpr int kCopyVecs = 4;           // 16-byte vectors a thread has in flight
constexpr int kCopyBytes = kCopyThreads * kCopyVecs * 16;

// Exclusive prefix sum of v over the CTA (kPlanThreads threads); *total gets the sum. Synchronises.
__device__ int block_scan(int v, int* total) {
    __shared__ int warp_sum[kPlanThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int s = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(~0u, s, d);
        if (lane >= d) s += o;
    }
    if (lane == 31) warp_sum[warp] = s;
    __syncthreads();
    int w = warp_sum[lane];                       // kPlanThreads / 32 == 32 warps
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(~0u, w, d);
        if (lane >= d) w += o;
    }
    const int before = warp ? __shfl_sync(~0u, w, warp - 1) : 0;
    *total = __shfl_sync(~0u, w, 31);
    __syncthreads();                              // warp_sum is written again by the next call
    return before + s - v;
}

__device__ __forceinline__ int pages_of(long long tokens, int page) { return (int)((tokens + page - 1) / page); }

// The reference counts of pages [at, at + kPlanPages) (past the pool: -1).
__device__ __forceinline__ void load_refs(const aq_kv_cache& c, int at, int (&r)[kPlanPages]) {
#pragma unroll
    for (int j = 0; j < kPlanPages; ++j) r[j] = at + j < c.num_pages ? c.refs[at + j] : -1;
}

// The `total` lowest free pages into list, in order; returns how many there were (at most total).
__device__ int find_free(const aq_kv_cache& c, int total, int* list) {
    int found = 0;
    for (int at = 0; at < c.num_pages && found < total; at += kPlanThreads * kPlanPages) {
        int r[kPlanPages], mine = 0, all;
        const int p0 = at + threadIdx.x * kPlanPages;
        load_refs(c, p0, r);
#pragma unroll
        for (int j = 0; j < kPlanPages; ++j) mine += r[j] == 0;
        int rank = found + block_scan(mine, &all);
#pragma unroll
        for (int j = 0; j < kPlanPages; ++j)
            if (r[j] == 0) {
                if (rank < total) list[rank] = p0 + j;
                ++rank;
            }
        found += all;
    }
    __syncthreads();
    return min(found, total);
}

// Reserve (FORK = false): entry i lengthens sequence a[i] (i when a is null) by b[i] tokens (1 when
// b is null). Fork (FORK = true): entry i makes the empty sequence b[i] a copy of a[i]; this
// kernel plans it and allocates the copies of partial last pages, kv_share_kernel does the rest.
// Nothing is changed unless every entry can be served. One CTA.
template <bool FORK>
__global__ void __launch_bounds__(kPlanThreads) kv_plan_kernel(aq_kv_cache c, KvScratch s, int n, const int* a,
                                                               const int* b) {
    __shared__ int bad;                           // the first error's status
    pdl_wait();
    if (threadIdx.x == 0) bad = 0, s.ctl[0] = 0, s.ctl[1] = 0;
    __syncthreads();
    const long long cap = (long long)c.max_pages * c.page_tokens;
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        const int from = a ? a[i] : i, seq = FORK ? b[i] : from;
        int err = 0;
        if ((unsigned)from >= (unsigned)c.max_seqs || (unsigned)seq >= (unsigned)c.max_seqs) {
            err = AQ_ERR_INVALID_ARG;
        } else {
            const int len = c.lens[from], add = FORK ? 0 : b ? b[i] : 1;
            if (len < 0 || add < 0 || (FORK && c.lens[seq] != 0)) err = AQ_ERR_INVALID_ARG;
            else if ((long long)len + add > cap || (long long)len + add > INT_MAX) err = AQ_ERR_CAPACITY;
            s.marks[seq] = i;
            s.count[i] = len;
        }
        if (err) atomicCAS(&bad, 0, err);
    }
    __syncthreads();
    // A sequence named twice keeps only one entry's mark. (Every thread has read `bad` before any
    // thread writes it again: the branches around the CTA-wide steps are taken by all or none.)
    int total = 0;
    const bool valid = !bad;
    __syncthreads();
    if (valid) {
        for (int at = 0; at < n; at += kPlanThreads) {
            const int i = at + threadIdx.x;
            int need = 0, all;
            if (i < n) {
                const int seq = FORK ? b[i] : a ? a[i] : i, len = s.count[i];
                if (s.marks[seq] != i) atomicCAS(&bad, 0, AQ_ERR_INVALID_ARG);
                need = FORK ? len % c.page_tokens != 0
                            : pages_of((long long)len + (b ? b[i] : 1), c.page_tokens) - pages_of(len, c.page_tokens);
            }
            const int before = block_scan(need, &all);
            if (i < n) s.prefix[i] = total + before;
            if (all > INT_MAX - total) {          // (the same for every thread)
                if (threadIdx.x == 0) atomicCAS(&bad, 0, AQ_ERR_CAPACITY);
                break;
            }
            total += all;
        }
        if (threadIdx.x == 0 && total > c.num_pages) atomicCAS(&bad, 0, AQ_ERR_CAPACITY);
        __syncthreads();
    }
    const bool search = !bad && total > 0;
    __syncthreads();
    if (search) {
        const int found = find_free(c, total, s.dst);
        if (threadIdx.x == 0 && found < total) bad = AQ_ERR_CAPACITY;
        __syncthreads();
    }
    if (bad) {
        if (threadIdx.x == 0) record_status(s.status, bad);
        return;
    }
    if (FORK) {
        for (int i = threadIdx.x; i < n; i += kPlanThreads) {
            const int len = s.count[i];
            if (len % c.page_tokens != 0) {
                const int k = s.prefix[i], last = len / c.page_tokens;
                s.src[k] = c.tables[(size_t)a[i] * c.max_pages + last];
                c.tables[(size_t)b[i] * c.max_pages + last] = s.dst[k];
                c.refs[s.dst[k]] = 1;
            }
            c.lens[b[i]] = len;
        }
        if (threadIdx.x == 0) s.ctl[0] = total, s.ctl[1] = 1;
    } else {
        for (int k = threadIdx.x; k < total; k += kPlanThreads) {
            int lo = 0, hi = n - 1;               // the last entry whose prefix is <= k
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (s.prefix[mid] <= k) lo = mid;
                else hi = mid - 1;
            }
            const int seq = a ? a[lo] : lo, at = pages_of(s.count[lo], c.page_tokens) + k - s.prefix[lo];
            c.tables[(size_t)seq * c.max_pages + at] = s.dst[k];
            c.refs[s.dst[k]] = 1;
        }
        for (int i = threadIdx.x; i < n; i += kPlanThreads) c.lens[a ? a[i] : i] = s.count[i] + (b ? b[i] : 1);
    }
}

// Copies pages src[i] -> dst[i] (keys, values and scales of every layer), i < count; the grid
// strides over pieces of kCopyBytes.
__device__ void copy_pages(const aq_kv_cache& c, int count, const int* src, const int* dst, unsigned int* status) {
    const int esz = c.dtype == AQ_E4M3 ? 1 : 2;
    const size_t page_bytes = (size_t)c.kv_heads * c.page_tokens * c.head_dim * esz;
    const size_t scale_bytes = (size_t)c.kv_heads * c.page_tokens;
    const int pieces = (int)((page_bytes + kCopyBytes - 1) / kCopyBytes);
    const size_t per_pair = (size_t)pieces * c.layers * 2, all = per_pair * count;
    for (size_t t = blockIdx.x; t < all; t += gridDim.x) {
        const int i = (int)(t / per_pair);
        int r = (int)(t - (size_t)i * per_pair);
        const int piece = r % pieces;
        r /= pieces;
        const int which = r & 1, layer = r >> 1;
        const int from = src[i], to = dst[i];
        if ((unsigned)from >= (unsigned)c.num_pages || (unsigned)to >= (unsigned)c.num_pages) {
            if (threadIdx.x == 0) record_status(status, AQ_ERR_INVALID_ARG);
            continue;
        }
        char* pool = (char*)(which ? c.v : c.k) + (size_t)layer * c.num_pages * page_bytes;
        const char* p = pool + (size_t)from * page_bytes;
        char* q = pool + (size_t)to * page_bytes;
        const size_t at = (size_t)piece * kCopyBytes + (size_t)threadIdx.x * 16;
        uint4 v[kCopyVecs];
#pragma unroll
        for (int j = 0; j < kCopyVecs; ++j)
            if (at + (size_t)j * kCopyThreads * 16 < page_bytes) v[j] = ld_stream_v4(p + at + (size_t)j * kCopyThreads * 16);
#pragma unroll
        for (int j = 0; j < kCopyVecs; ++j)
            if (at + (size_t)j * kCopyThreads * 16 < page_bytes) *(uint4*)(q + at + (size_t)j * kCopyThreads * 16) = v[j];
        if (esz == 1 && piece == 0) {
            uint8_t* sp = (uint8_t*)(which ? c.v_scales : c.k_scales) + (size_t)layer * c.num_pages * scale_bytes;
            const uint2* f = (const uint2*)(sp + (size_t)from * scale_bytes);
            uint2* g = (uint2*)(sp + (size_t)to * scale_bytes);
            for (size_t j = threadIdx.x; j < scale_bytes / 8; j += kCopyThreads) g[j] = f[j];
        }
    }
}

// Second half of a fork: the children take their parents' full pages (one reference more each),
// and the partial last pages are copied.
__global__ void __launch_bounds__(kCopyThreads) kv_share_kernel(aq_kv_cache c, KvScratch s, int n, const int* src,
                                                                const int* dst) {
    pdl_wait();
    if (!s.ctl[1]) return;
    for (int i = blockIdx.x; i < n; i += gridDim.x) {
        const int full = s.count[i] / c.page_tokens;
        const int* from = c.tables + (size_t)src[i] * c.max_pages;
        int* to = c.tables + (size_t)dst[i] * c.max_pages;
        for (int j = threadIdx.x; j < full; j += kCopyThreads) {
            const int p = from[j];
            to[j] = p;
            if ((unsigned)p < (unsigned)c.num_pages) atomicAdd(c.refs + p, 1);
            else record_status(s.status, AQ_ERR_INVALID_ARG);
        }
    }
    copy_pages(c, s.ctl[0], s.src, s.dst, s.status);
}

__global__ void __launch_bounds__(kCopyThreads) kv_copy_kernel(aq_kv_cache c, unsigned int* status, int n,
                                                               const int* src, const int* dst) {
    pdl_wait();
    copy_pages(c, n, src, dst, status);
}

// One CTA per listed sequence. The exchange of its length makes a sequence listed twice be freed
// once.
__global__ void __launch_bounds__(kCopyThreads) kv_free_kernel(aq_kv_cache c, unsigned int* status, const int* seqs) {
    __shared__ int shared_len;
    pdl_wait();
    const int seq = seqs ? seqs[blockIdx.x] : blockIdx.x;
    if ((unsigned)seq >= (unsigned)c.max_seqs) {
        if (threadIdx.x == 0) record_status(status, AQ_ERR_INVALID_ARG);
        return;
    }
    if (threadIdx.x == 0) shared_len = atomicExch(c.lens + seq, 0);
    __syncthreads();
    const int pages = min(pages_of(max(shared_len, 0), c.page_tokens), c.max_pages);
    int* row = c.tables + (size_t)seq * c.max_pages;
    for (int j = threadIdx.x; j < pages; j += kCopyThreads) {
        const int p = row[j];
        row[j] = -1;
        if ((unsigned)p < (unsigned)c.num_pages) atomicSub(c.refs + p, 1);
        else record_status(status, AQ_ERR_INVALID_ARG);
    }
}

// Plans a compaction: with U pages in use, the k-th used page at or above U goes to the k-th free
// page below U (there are equally many). One CTA.
__global__ void __launch_bounds__(kPlanThreads) kv_compact_plan_kernel(aq_kv_cache c, KvScratch s, int* used_out) {
    pdl_wait();
    constexpr int kStep = kPlanThreads * kPlanPages;
    int used = 0;
    for (int at = 0; at < c.num_pages; at += kStep) {
        int r[kPlanPages], mine = 0, all;
        load_refs(c, at + threadIdx.x * kPlanPages, r);
#pragma unroll
        for (int j = 0; j < kPlanPages; ++j) mine += r[j] > 0;
        block_scan(mine, &all);
        used += all;
    }
    int holes = 0, movers = 0;
    for (int at = 0; at < c.num_pages; at += kStep) {
        int r[kPlanPages], hole = 0, mover = 0, all;
        const int p0 = at + threadIdx.x * kPlanPages;
        load_refs(c, p0, r);
#pragma unroll
        for (int j = 0; j < kPlanPages; ++j) {
            hole += r[j] == 0 && p0 + j < used;
            mover += r[j] > 0 && p0 + j >= used;
        }
        int h = holes + block_scan(hole, &all);
        holes += all;
        int m = movers + block_scan(mover, &all);
        movers += all;
#pragma unroll
        for (int j = 0; j < kPlanPages; ++j) {
            if (r[j] == 0 && p0 + j < used) s.dst[h++] = p0 + j;
            if (r[j] > 0 && p0 + j >= used) s.src[m++] = p0 + j;
        }
    }
    __syncthreads();
    const int moves = min(holes, movers);         // equal unless a count is negative
    for (int k = threadIdx.x; k < moves; k += kPlanThreads) {
        const int from = s.src[k], to = s.dst[k];
        s.moved[from] = to;
        c.refs[to] = c.refs[from];
        c.refs[from] = 0;
    }
    if (threadIdx.x == 0) {
        s.ctl[0] = moves, s.ctl[2] = used;
        if (holes != movers) record_status(s.status, AQ_ERR_INVALID_ARG);
        if (used_out) *used_out = used;
    }
}

// Carries a compaction out: tables are rewritten, pages copied.
__global__ void __launch_bounds__(kCopyThreads) kv_compact_kernel(aq_kv_cache c, KvScratch s) {
    pdl_wait();
    const int used = s.ctl[2], moves = s.ctl[0];
    if (moves == 0) return;
    for (int seq = blockIdx.x; seq < c.max_seqs; seq += gridDim.x) {
        const int pages = min(pages_of(max(c.lens[seq], 0), c.page_tokens), c.max_pages);
        int* row = c.tables + (size_t)seq * c.max_pages;
        for (int j = threadIdx.x; j < pages; j += kCopyThreads) {
            const int p = row[j];
            if ((unsigned)p >= (unsigned)c.num_pages) record_status(s.status, AQ_ERR_INVALID_ARG);
            else if (p >= used) row[j] = s.moved[p];
        }
    }
    copy_pages(c, moves, s.src, s.dst, s.status);
}

__global__ void __launch_bounds__(kCopyThreads) kv_init_kernel(aq_kv_cache c) {
    pdl_wait();
    const size_t t = (size_t)blockIdx.x * kCopyThreads + threadIdx.x, step = (size_t)gridDim.x * kCopyThreads;
    for (size_t i = t; i < (size_t)c.max_seqs * c.max_pages; i += step) c.tables[i] = -1;
    for (size_t i = t; i < (size_t)c.max_seqs; i += step) c.lens[i] = 0;
    for (size_t i = t; i < (size_t)c.num_pages; i += step) c.refs[i] = 0;
}

// New keys and values into their slots. A group of `lanes` lanes (a power of two, at least
// head_dim / 8) takes one head of one token's key or value, eight elements a lane: one 16-byte
// load and store each for 16-bit types; for E4M3 the group's maximum gives the scale.
__global__ void __launch_bounds__(kCopyThreads) kv_write_kernel(aq_kv_cache c, int layer, int n, const int* seqs,
                                                                const int* positions, const void* k, const void* v,
                                                                int x_dt, long long stride, int lanes_log2,
                                                                unsigned int* status) {
    pdl_wait();
    const int lane = threadIdx.x & ((1 << lanes_log2) - 1);
    const int per_cta = kCopyThreads >> lanes_log2, slot0 = threadIdx.x >> lanes_log2;
    const size_t rows = (size_t)n * 2 * c.kv_heads;
    // Every thread makes the same number of trips: the shuffles below are warp-wide.
    for (size_t base = (size_t)blockIdx.x * per_cta; base < rows; base += (size_t)gridDim.x * per_cta) {
        const size_t r = base + slot0;
        const bool in = r < rows && lane * 8 < c.head_dim;
        const int head = (int)(r % c.kv_heads);
        const size_t tr = r / c.kv_heads;
        const int which = (int)(tr & 1);
        const long long i = (long long)(tr >> 1);
        float f[8] = {};
        size_t at = 0;
        bool ok = false;
        if (r < rows) {
            const int seq = seqs ? seqs[i] : (int)i;
            if ((unsigned)seq < (unsigned)c.max_seqs) {
                const int len = min((long long)c.lens[seq], (long long)c.max_pages * c.page_tokens);
                const int pos = positions ? positions[i] : len - 1;
                if (pos >= 0 && pos < len) {
                    const int page = c.tables[(size_t)seq * c.max_pages + pos / c.page_tokens];
                    if ((unsigned)page < (unsigned)c.num_pages) {
                        ok = true;
                        at = (((size_t)layer * c.num_pages + page) * c.kv_heads + head) * c.page_tokens +
                             pos % c.page_tokens;
                    }
                }
            }
            if (!ok && lane == 0) record_status(status, AQ_ERR_INVALID_ARG);
        }
        if (in && ok) load8(which ? v : k, (size_t)(i * stride + (long long)head * c.head_dim + lane * 8), x_dt, f);
        if (c.dtype == AQ_E4M3) {
            float amax = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(f[j]));
            for (int d = 1 << lanes_log2 >> 1; d > 0; d >>= 1) amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, d));
            const int e = e4m3_scale_exp(amax);
            if (in && ok) {
                *(uint2*)((uint8_t*)(which ? c.v : c.k) + at * c.head_dim + lane * 8) = e4m3_pack8(f, pow2f(-e));
                if (lane == 0) ((uint8_t*)(which ? c.v_scales : c.k_scales))[at] = (uint8_t)(e + 127);
            }
        } else if (in && ok) {
            store8(which ? c.v : c.k, at * c.head_dim + lane * 8, c.dtype, f);
        }
    }
}

// CTAs for the copying kernels: a few per SM, no more than there can be pieces.
aq_status copy_grid(const aq_kv_cache& c, long long pairs, int* grid) {
    DeviceInfo di;
    if (aq_status st = device_info(&di); st != AQ_OK) return st;
    const size_t page_bytes = (size_t)c.kv_heads * c.page_tokens * c.head_dim * (c.dtype == AQ_E4M3 ? 1 : 2);
    const size_t pieces = (page_bytes + kCopyBytes - 1) / kCopyBytes * c.layers * 2 * (size_t)pairs;
    const size_t most = (size_t)di.sms * 8;
    *grid = (int)(pieces < 1 ? 1 : pieces < most ? pieces : most);
    return AQ_OK;
}

}  // namespace

aq_status launch_kv_init(const aq_kv_cache& c, cudaStream_t st) {
    return launch_dependent(kv_init_kernel, 152, kCopyThreads, 0, st, c);
}

aq_status launch_kv_reserve(const aq_kv_cache& c, int n, const int* seqs, const int* counts, void* ws,
                            cudaStream_t st) {
    return launch_dependent(kv_plan_kernel<false>, 1, kPlanThreads, 0, st, c, kv_scratch(c, ws), n, seqs, counts);
}

aq_status launch_kv_fork(const aq_kv_cache& c, int n, const int* src, const int* dst, void* ws, cudaStream_t st) {
    const KvScratch s = kv_scratch(c, ws);
    int grid;
    if (aq_status e = copy_grid(c, n, &grid); e != AQ_OK) return e;
    if (aq_status e = launch_dependent(kv_plan_kernel<true>, 1, kPlanThreads, 0, st, c, s, n, src, dst); e != AQ_OK)
        return e;
    return launch_dependent(kv_share_kernel, grid, kCopyThreads, 0, st, c, s, n, src, dst);
}

aq_status launch_kv_free(const aq_kv_cache& c, int n, const int* seqs, void* ws, cudaStream_t st) {
    return launch_dependent(kv_free_kernel, n, kCopyThreads, 0, st, c, (unsigned int*)ws, seqs);
}

aq_status launch_kv_compact(const aq_kv_cache& c, int* used, void* ws, cudaStream_t st) {
    const KvScratch s = kv_scratch(c, ws);
    int grid;
    if (aq_status e = copy_grid(c, c.num_pages / 2 + 1, &grid); e != AQ_OK) return e;
    if (aq_status e = launch_dependent(kv_compact_plan_kernel, 1, kPlanThreads, 0, st, c, s, used); e != AQ_OK) return e;
    return launch_dependent(kv_compact_kernel, grid, kCopyThreads, 0, st, c, s);
}

aq_status launch_kv_copy_pages(const aq_kv_cache& c, int n, const int* src, const int* dst, void* ws,
                               cudaStream_t st) {
    int grid;
    if (aq_status e = copy_grid(c, n, &grid); e != AQ_OK) return e;
    return launch_dependent(kv_copy_kernel, grid, kCopyThreads, 0, st, c, (unsigned int*)ws, n, src, dst);
}

aq_status launch_kv_write(const aq_kv_cache& c, int layer, int n, const int* seqs, const int* positions,
                          const void* k, const void* v, int x_dt, long long stride, void* ws, cudaStream_t st) {
    DeviceInfo di;
    if (aq_status e = device_info(&di); e != AQ_OK) return e;
    int lanes_log2 = 1;
    while ((8 << lanes_log2) < c.head_dim) ++lanes_log2;
    const size_t per_cta = kCopyThreads >> lanes_log2, rows = (size_t)n * 2 * c.kv_heads;
    const size_t ctas = (rows + per_cta - 1) / per_cta, most = (size_t)di.sms * 8;
    return launch_dependent(kv_write_kernel, (unsigned)(ctas < most ? ctas : most), kCopyThreads, 0, st, c, layer, n,
                            seqs, positions, k, v, x_dt, stride, lanes_log2, (unsigned int*)ws);
}

}  // namespace aq
