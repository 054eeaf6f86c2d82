// Pages of the key-value cache: allocation (aq_kv_reserve), sharing (aq_kv_fork), release
// (aq_kv_free), compaction (aq_kv_compact), plain copies (aq_kv_copy_pages), and the writes of new
// keys and values (aq_kv_write).
//
// All of the cache's bookkeeping lives on the device (tables, lengths, reference counts), so a
// decode loop that grows sequences, forks beams and drops them is ordered by its stream alone and
// can be captured in a CUDA graph. A page is free when its reference count is 0, and allocation
// takes the lowest free indices, in list order: counts are only added to and subtracted from, and
// every other decision is made in one CTA, so the outcome does not depend on scheduling. A page
// shared by several sequences is always full (a fork copies a partial last page), so no write of a
// new token needs to ask whether its page is shared.
//
// Measured on a GB300: a compaction that moves 1000 of 4096 pages of 256 KB (524 MB of traffic) takes 82
// us, 75 of them the copies (6.9 TB/s); freeing, forking and lengthening 32 beams of about 1000 tokens
// (16 MB copied) 12.4 us, four kernels of 3 to 5 us that are dependent reads of the bookkeeping.
#include "kv.cuh"

namespace aq {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanPages = 16;         // reference counts a thread looks at per step
constexpr int kCopyThreads = 256;
constexpr int kCopyVecs = 4;           // 16-byte vectors a thread has in flight
constexpr int kCopyBytes = kCopyThreads * kCopyVecs * 16;

// Exclusive prefix sum of v over the CTA (kPlanThreads threads); *total gets the sum. Synchronises.
template <typename T>
__device__ T block_scan(T v, T* total) {
    __shared__ T warp_sum[kPlanThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    T s = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const T o = __shfl_up_sync(~0u, s, d);
        if (lane >= d) s += o;
    }
    if (lane == 31) warp_sum[warp] = s;
    __syncthreads();
    T w = warp_sum[lane];                         // kPlanThreads / 32 == 32 warps
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const T o = __shfl_up_sync(~0u, w, d);
        if (lane >= d) w += o;
    }
    const T before = __shfl_sync(~0u, w, warp ? warp - 1 : 0);
    *total = __shfl_sync(~0u, w, 31);
    __syncthreads();                              // warp_sum is written again by the next call
    return (warp ? before : 0) + s - v;
}

__device__ __forceinline__ int pages_of(long long tokens, int page) { return (int)((tokens + page - 1) / page); }

// The reference counts of pages [at, at + kPlanPages) (past the pool: -1), at a multiple of four.
__device__ __forceinline__ void load_refs(const aq_kv_cache& c, long long at, int (&r)[kPlanPages]) {
    if (at + kPlanPages <= c.num_pages && ((uintptr_t)c.refs & 15) == 0) {
#pragma unroll
        for (int j = 0; j < kPlanPages; j += 4) {
            const int4 v = *(const int4*)(c.refs + at + j);
            r[j] = v.x, r[j + 1] = v.y, r[j + 2] = v.z, r[j + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < kPlanPages; ++j) r[j] = at + j < c.num_pages ? c.refs[at + j] : -1;
    }
}

// The `total` lowest free pages into list, in order; returns how many there were (at most total).
// r: the counts of the first step, as load_refs gives them for this thread.
__device__ int find_free(const aq_kv_cache& c, int total, int* list, int (&r)[kPlanPages]) {
    int found = 0;
    for (long long at = 0; at < c.num_pages && found < total; at += kPlanThreads * kPlanPages) {
        int mine = 0, all;
        const long long p0 = at + threadIdx.x * kPlanPages;
        if (at > 0) load_refs(c, p0, r);
#pragma unroll
        for (int j = 0; j < kPlanPages; ++j) mine += r[j] == 0;
        int rank = found + block_scan<int>(mine, &all);
#pragma unroll
        for (int j = 0; j < kPlanPages; ++j)
            if (r[j] == 0) {
                if (rank < total) list[rank] = (int)(p0 + j);
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
// Nothing is changed unless every entry can be served. One CTA, up to kPlanThreads entries: a
// thread has one, in registers. The time is that of dependent reads of the bookkeeping (entry,
// length, last page; the reference counts are read meanwhile) and of a few barriers.
struct Entry {
    int from, seq, len, add, err;      // err: 0, or the status to record
};
template <bool FORK>
__device__ __forceinline__ Entry load_entry(const aq_kv_cache& c, int i, const int* a, const int* b) {
    Entry e;
    e.from = a ? a[i] : i;
    e.seq = FORK ? b[i] : e.from;
    e.add = FORK ? 0 : b ? b[i] : 1;
    e.len = 0, e.err = AQ_ERR_INVALID_ARG;
    if ((unsigned)e.from < (unsigned)c.max_seqs && (unsigned)e.seq < (unsigned)c.max_seqs) {
        e.len = c.lens[e.from];
        const int taken = FORK ? c.lens[e.seq] : 0;
        const long long len = (long long)e.len + e.add;
        if (e.len >= 0 && e.add >= 0 && taken == 0)
            e.err = len > (long long)c.max_pages * c.page_tokens ? AQ_ERR_CAPACITY : 0;
    }
    return e;
}
template <bool FORK>
__device__ __forceinline__ int pages_needed(const aq_kv_cache& c, const Entry& e) {
    return FORK ? e.len % c.page_tokens != 0
                : pages_of((long long)e.len + e.add, c.page_tokens) - pages_of(e.len, c.page_tokens);
}
// The status of a whole call (an invalid entry before a lack of pages), for every thread.
__device__ __forceinline__ int call_status(int err) {
    if (__syncthreads_or(err == AQ_ERR_INVALID_ARG)) return AQ_ERR_INVALID_ARG;
    return __syncthreads_or(err != 0) ? AQ_ERR_CAPACITY : 0;
}

template <bool FORK>
__global__ void __launch_bounds__(kPlanThreads) kv_plan_kernel(aq_kv_cache c, KvScratch s, int n, const int* a,
                                                               const int* b) {
    constexpr int kSlots = 2 * kPlanThreads;
    __shared__ int seen[kSlots];                  // the listed sequences + 1, hashed
    __shared__ int list[kPlanThreads];            // allocated pages (more of them: s.dst)
    __shared__ int prefix[kPlanThreads];          // pages of the entries before
    __shared__ int first[kPlanThreads];           // reserve: an entry's sequence and its first new table entry
    __shared__ int seqs[kPlanThreads];
    pdl_wait();
    pdl_launch_dependents();
    const int t = threadIdx.x;
    seen[t] = seen[t + kPlanThreads] = 0;
    int refs[kPlanPages];
    load_refs(c, t * kPlanPages, refs);
    Entry e = {0, 0, 0, 0, 0};
    if (t < n) e = load_entry<FORK>(c, t, a, b);
    const int need = t < n && e.err == 0 ? pages_needed<FORK>(c, e) : 0;
    int old = 0;                                  // fork: the partial page
    if (FORK && need) old = c.tables[(size_t)e.from * c.max_pages + e.len / c.page_tokens];
    __syncthreads();
    if (t < n && e.err != AQ_ERR_INVALID_ARG) {
        for (unsigned h = (unsigned)e.seq * 2654435761u >> 21;; h = (h + 1) & (kSlots - 1)) {
            const int was = atomicCAS(seen + h, 0, e.seq + 1);
            if (was == e.seq + 1) e.err = AQ_ERR_INVALID_ARG;
            if (was == 0 || was == e.seq + 1) break;
        }
    }
    int status = call_status(e.err), total = 0, before = 0;
    if (!status) {
        long long all;                            // (may pass 32 bits)
        before = (int)block_scan<long long>(need, &all);
        if (all > c.num_pages) status = AQ_ERR_CAPACITY;
        else total = (int)all;
    }
    int* const pages = total <= kPlanThreads ? list : s.dst;
    if (!status && total > 0 && find_free(c, total, pages, refs) < total) status = AQ_ERR_CAPACITY;
    if (t == 0) {
        s.ctl[0] = status ? 0 : total, s.ctl[1] = !status;
        if (status) record_status(s.status, status);
    }
    if (status) return;
    if (FORK) {
        if (t < n) {
            if (need) {
                const int page = list[before];
                s.src[before] = old;
                s.dst[before] = page;
                c.tables[(size_t)e.seq * c.max_pages + e.len / c.page_tokens] = page;
                c.refs[page] = 1;
            }
            s.count[t] = e.len;
            c.lens[e.seq] = e.len;
        }
        return;
    }
    if (t < n) {
        prefix[t] = before;
        seqs[t] = e.seq;
        first[t] = pages_of(e.len, c.page_tokens);
        c.lens[e.seq] = e.len + e.add;
    }
    __syncthreads();
    for (int k = t; k < total; k += kPlanThreads) {
        int lo = 0, hi = n - 1;                   // the last entry whose prefix is <= k
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (prefix[mid] <= k) lo = mid;
            else hi = mid - 1;
        }
        c.tables[(size_t)seqs[lo] * c.max_pages + first[lo] + k - prefix[lo]] = pages[k];
        c.refs[pages[k]] = 1;
    }
}

// The same for longer lists: what the one above keeps in registers and shared memory goes through
// the workspace, kPlanThreads entries at a time.
template <bool FORK>
__global__ void __launch_bounds__(kPlanThreads) kv_plan_long_kernel(aq_kv_cache c, KvScratch s, int n, const int* a,
                                                                    const int* b) {
    pdl_wait();
    pdl_launch_dependents();
    int err = 0;
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        const Entry e = load_entry<FORK>(c, i, a, b);
        if (e.err != AQ_ERR_INVALID_ARG) s.marks[e.seq] = i;
        s.count[i] = e.len;
        if (err != AQ_ERR_INVALID_ARG && e.err) err = e.err;
    }
    int status = call_status(err), total = 0;
    if (status != AQ_ERR_INVALID_ARG) {           // a sequence named twice keeps only one entry's mark
        bool twice = false;
        for (int i = threadIdx.x; i < n; i += kPlanThreads) twice |= s.marks[FORK ? b[i] : a ? a[i] : i] != i;
        if (__syncthreads_or(twice)) status = AQ_ERR_INVALID_ARG;
    }
    for (int at = 0; at < n && !status; at += kPlanThreads) {
        const int i = at + threadIdx.x;
        int need = 0;
        if (i < n) {
            Entry e;
            e.len = s.count[i], e.add = FORK ? 0 : b ? b[i] : 1;
            need = pages_needed<FORK>(c, e);
        }
        long long all;
        const long long before = block_scan<long long>(need, &all);
        if (i < n) s.prefix[i] = (int)(total + before);
        if (total + all > c.num_pages) status = AQ_ERR_CAPACITY;
        else total += (int)all;
    }
    __syncthreads();
    if (!status && total > 0) {
        int refs[kPlanPages];
        load_refs(c, threadIdx.x * kPlanPages, refs);
        if (find_free(c, total, s.dst, refs) < total) status = AQ_ERR_CAPACITY;
    }
    if (threadIdx.x == 0) {
        s.ctl[0] = status ? 0 : total, s.ctl[1] = !status;
        if (status) record_status(s.status, status);
    }
    if (status) return;
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
            if (at + (size_t)j * kCopyThreads * 16 < page_bytes) v[j] = ld_once_v4(p + at + (size_t)j * kCopyThreads * 16);
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
    pdl_launch_dependents();
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
    pdl_launch_dependents();
    copy_pages(c, n, src, dst, status);
}

// One CTA per listed sequence. The exchange of its length makes a sequence listed twice be freed
// once.
__global__ void __launch_bounds__(kCopyThreads) kv_free_kernel(aq_kv_cache c, unsigned int* status, const int* seqs) {
    __shared__ int shared_len;
    pdl_wait();
    pdl_launch_dependents();
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
    pdl_launch_dependents();
    constexpr int kStep = kPlanThreads * kPlanPages;
    int used = 0, r[kPlanPages];
    for (long long at = 0; at < c.num_pages; at += kStep) {
        int mine = 0, all;
        load_refs(c, at + threadIdx.x * kPlanPages, r);
#pragma unroll
        for (int j = 0; j < kPlanPages; ++j) mine += r[j] > 0;
        block_scan<int>(mine, &all);
        used += all;
    }
    int holes = 0, movers = 0;
    for (long long at = 0; at < c.num_pages; at += kStep) {
        int hole = 0, mover = 0, all;
        const long long p0 = at + threadIdx.x * kPlanPages;
        if (c.num_pages > kStep) load_refs(c, p0, r);          // (else they are still there)
#pragma unroll
        for (int j = 0; j < kPlanPages; ++j) {
            hole += r[j] == 0 && p0 + j < used;
            mover += r[j] > 0 && p0 + j >= used;
        }
        // both counts in one scan: a step has kStep < 2^16 pages
        const int both = block_scan<int>(hole << 16 | mover, &all);
        int h = holes + (int)((unsigned)both >> 16), m = movers + (both & 0xffff);
        holes += (int)((unsigned)all >> 16);
        movers += all & 0xffff;
#pragma unroll
        for (int j = 0; j < kPlanPages; ++j) {
            if (r[j] == 0 && p0 + j < used) s.dst[h++] = (int)(p0 + j);
            if (r[j] > 0 && p0 + j >= used) s.src[m++] = (int)(p0 + j);
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
    pdl_launch_dependents();
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
    pdl_launch_dependents();
    const size_t t = (size_t)blockIdx.x * kCopyThreads + threadIdx.x, step = (size_t)gridDim.x * kCopyThreads;
    for (size_t i = t; i < (size_t)c.max_seqs * c.max_pages; i += step) c.tables[i] = -1;
    for (size_t i = t; i < (size_t)c.max_seqs; i += step) c.lens[i] = 0;
    for (size_t i = t; i < (size_t)c.num_pages; i += step) c.refs[i] = 0;
}

// New keys and values into their slots. A CTA takes a few tokens (one per group of `lanes` lanes, a
// power of two that is at least head_dim / 8) and `heads` heads of their keys or of their values
// (even and odd blockIdx.y); a lane takes eight elements of a row: one 16-byte load and store each
// for 16-bit types; for E4M3 the group's maximum gives the scale. The tokens' slots are looked up
// once, three dependent reads, while the first UNDER_WAY rows are under way. Bound by HBM for
// prompts, by that chain for a decode step.
template <int UNDER_WAY, bool WIDE>
__global__ void __launch_bounds__(kCopyThreads) kv_write_kernel(aq_kv_cache c, int layer, int n, const int* seqs,
                                                                const int* positions, const void* k, const void* v,
                                                                int x_dt, long long stride, int lanes_log2, int heads,
                                                                unsigned int* status) {
    __shared__ long long slots[kCopyThreads / 2];  // of the first head's row in the pool, or -1
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & ((1 << lanes_log2) - 1), tok = threadIdx.x >> lanes_log2;
    const int per_cta = kCopyThreads >> lanes_log2;
    const long long i = (long long)blockIdx.x * per_cta + tok;
    const bool in = i < n && lane * 8 < c.head_dim, vals = blockIdx.y & 1;
    const int h0 = (blockIdx.y >> 1) * heads, count = min(heads, c.kv_heads - h0);
    const char* from = (const char*)(vals ? v : k) +
                       (i * stride + (long long)h0 * c.head_dim + lane * 8) * (WIDE ? 4 : 2);
    const size_t from_step = (size_t)c.head_dim * (WIDE ? 4 : 2);
    char* to = (char*)(vals ? c.v : c.k);
    uint8_t* scale = (uint8_t*)(vals ? c.v_scales : c.k_scales);
    const bool small = c.dtype == AQ_E4M3;
    const size_t to_step = (size_t)c.page_tokens * c.head_dim * (small ? 1 : 2);
    bool write = false;
    for (int h = 0; h < count; h += UNDER_WAY) {
        Raw<WIDE> x[UNDER_WAY] = {};
#pragma unroll
        for (int u = 0; u < UNDER_WAY; ++u) {
            if (in && h + u < count) x[u].load(from, 0);
            from += from_step;
        }
        if (h == 0) {                              // (the same for the whole CTA)
            const long long mine = (long long)blockIdx.x * per_cta + threadIdx.x;
            if (threadIdx.x < per_cta && mine < n) {
                const int seq = seqs ? seqs[mine] : (int)mine;
                int p = positions ? positions[mine] : -1;
                long long slot = -1;
                if ((unsigned)seq < (unsigned)c.max_seqs) {
                    const int len = (int)min((long long)c.lens[seq], (long long)c.max_pages * c.page_tokens);
                    if (!positions) p = len - 1;
                    if (p >= 0 && p < len) {
                        const int page = c.tables[(size_t)seq * c.max_pages + p / c.page_tokens];
                        if ((unsigned)page < (unsigned)c.num_pages)
                            slot = (((long long)layer * c.num_pages + page) * c.kv_heads + h0) * c.page_tokens +
                                   p % c.page_tokens;
                    }
                }
                if (slot < 0) record_status(status, AQ_ERR_INVALID_ARG);
                slots[threadIdx.x] = slot;
            }
            __syncthreads();
            const long long slot = i < n ? slots[tok] : -1;
            write = in && slot >= 0;
            to += (slot * c.head_dim + lane * 8) * (small ? 1 : 2);
            scale += slot;
        }
#pragma unroll
        for (int u = 0; u < UNDER_WAY; ++u) {
            const bool now = write && h + u < count;
            float f[8];
            x[u].widen(x_dt, f);
            if (small) {                           // (all lanes take part in the shuffles)
                float amax = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(f[j]));
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) {
                    const float o = __shfl_xor_sync(~0u, amax, d);
                    if (d < 1 << lanes_log2) amax = fmaxf(amax, o);
                }
                const int e = e4m3_scale_exp(amax);
                if (now) {
                    *(uint2*)to = e4m3_pack8(f, pow2f(-e));
                    if (lane == 0) *scale = (uint8_t)(e + 127);
                }
                scale += c.page_tokens;
            } else if (now) {
                store8(to, 0, c.dtype, f);
            }
            to += to_step;
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
    return launch_dependent(n <= kPlanThreads ? kv_plan_kernel<false> : kv_plan_long_kernel<false>, 1, kPlanThreads, 0, st,
                            c, kv_scratch(c, ws), n, seqs, counts);
}

aq_status launch_kv_fork(const aq_kv_cache& c, int n, const int* src, const int* dst, void* ws, cudaStream_t st) {
    const KvScratch s = kv_scratch(c, ws);
    int grid;
    if (aq_status e = copy_grid(c, n, &grid); e != AQ_OK) return e;
    if (aq_status e = launch_dependent(n <= kPlanThreads ? kv_plan_kernel<true> : kv_plan_long_kernel<true>, 1,
                                       kPlanThreads, 0, st, c, s, n, src, dst);
        e != AQ_OK)
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
    const long long per_cta = kCopyThreads >> lanes_log2, tokens = (n + per_cta - 1) / per_cta;
    // A CTA takes as many heads as leaves two CTAs per SM: all of them for prompts (8188 tokens of
    // 8 heads of 128, bf16 to E4M3: 12.2 us; with eight CTAs per SM 14.3), one for a decode step.
    long long heads = 2 * c.kv_heads * tokens / (2 * di.sms);
    heads = heads < 1 ? 1 : heads > c.kv_heads ? c.kv_heads : heads;
    const dim3 grid((unsigned)tokens, 2 * (unsigned)((c.kv_heads + heads - 1) / heads));
    const bool wide = x_dt == AQ_F32;
    return launch_dependent(heads > 1 ? (wide ? kv_write_kernel<4, true> : kv_write_kernel<4, false>)
                                      : (wide ? kv_write_kernel<1, true> : kv_write_kernel<1, false>), grid,
                            kCopyThreads, 0, st, c, layer, n, seqs, positions, k, v, x_dt, stride, lanes_log2,
                            (int)heads, (unsigned int*)ws);
}

}  // namespace aq
