// Attention of one new token per sequence over the paged key-value cache (aq_kv_attend).
//
//   s_t = scale * q . k_t for the cached tokens t the query sees (t >= L - window),
//   o = sum_t p_t v_t / sum_t p_t with p_t = exp(s_t - max), lse = max + ln sum_t p_t,
// in one pass over the cache with a running maximum and sum.
//
// Bound: every cached key and value is read once per 16 query heads of its kv head, 4 * head_dim
// bytes per token and head with 16-bit entries, for 4 * head_dim * (query heads per kv head)
// operations: a few operations per byte, so HBM is the limit and the work is arranged around
// keeping loads in flight.
//   - A tile is the up to 8 (or 16) query heads that share a kv head; above 16 there are several, each
//     of which reads the kv head's tokens for itself (48 heads of 128 over one kv head, 131072 tokens:
//     42.6 us, 16 heads 29.6). mma.sync m16n8k16 takes 16 cached tokens as rows and 8 heads as columns, S^T = K Q^T, then 16 head dimensions as rows,
//     O^T += V^T P^T: both big operands come straight from the copied tiles (ldmatrix), the
//     weights change from one form to the other by an 8x8 transpose in registers, and a column's
//     statistics are per-lane values. (At the copy bandwidth an SM receives 24 bytes a cycle,
//     which asks for about 100 multiply-adds a cycle of an 8-head tile; the legacy tensor path has
//     several times that, so tensor memory would add waits and nothing else.)
//   - The work is the list of all (sequence, tile) segments cut into chunks of CT tokens; every
//     warp takes an equal, contiguous share of the list whatever the sequences' lengths (a segment
//     counts SEG chunks more, for its query and its end), and runs through it with a ring of
//     asynchronous copies of its own that crosses segment ends: no CTA-wide step until the end.
//   - A segment that lies in one warp's share is written at once. Pieces of segments are merged
//     per CTA; of the CTAs that a segment crosses, the last to finish joins their partials, in the
//     order of the tokens, so the result does not depend on scheduling.
//
// Measured on a GB300 (copy peak 6.79 TB/s), medians in a CUDA graph: 48 sequences of 8192 to 32768
// tokens, 8 heads of 128, bf16 (3.5 GB): 511 us; one sequence of 131071 tokens, fp16: 87 us (6.2 TB/s);
// 64 sequences of 17 to 2048 tokens: 29.1 us; 64 query heads over an E4M3 cache of 380 MB: 70.4 us (5.4 TB/s). What a
// call costs beside its bytes, about 4 us until the first keys arrive (lengths, table, keys: three
// dependent reads) and 5 to 8 us to merge and join, is latency.
//
// Numbers: products of 16-bit values are accumulated in fp32 by the tensor cores; the statistics
// and accumulators are fp32. The weights p_t are rounded to the cache's 16-bit type for the
// product with V (a relative error of at most 2^-8 (bf16) or 2^-11 (fp16) of each, no more than
// the rounding of the 16-bit output); their sum is taken before that rounding. E4M3 entries widen
// exactly to fp16; the query is scaled to fp16's range by a power of two. A key's scale
// multiplies its score; a value's scale 2^b multiplies its weight, with the running maximum taken
// over s_t log2 e + b so that p_t 2^b stays in [0, 1]. fp16 weights are taken times 2^15, fp16's range
// above 1, so that those under a maximum keep their bits down to 2^-29 of it (with a maximum of 1
// they were subnormal below 2^-14 and 0 below 2^-25, which many tokens under one large weight
// notice); the output's division takes the factor back.
#include <atomic>
#include <climits>

#include "kv.cuh"

namespace aq {
namespace {

// One CTA per SM. The workspace is sized for the largest grid, so that its query needs no device.
constexpr int kMaxCtas = 160;
constexpr size_t kArrivedBytes = 2048;                       // three counters per CTA
static_assert(kArrivedBytes >= 3 * kMaxCtas * 4, "room for the counters");
constexpr int kSliceSeqs = 512;       // sequences per launch (their offsets sit in shared memory)
constexpr float kFp16Weights = 32768.0f;   // factor of fp16 weights (and so of their o)
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Sizes for a cache type, a padded head dimension HD (64, 128 or 256) and NH groups of 8 heads.
template <int DT, int HD, int NH>
struct Tile {
    static constexpr int ESZ = DT == AQ_E4M3 ? 1 : 2;
    static constexpr int RB = HD * ESZ;                      // bytes of a token's row
    static constexpr int PR = RB / 16;                       // 16-byte pieces of a row
    static constexpr int CT = RB == 64 ? 64 : RB == 128 ? 32 : 16;   // tokens per chunk
    static constexpr int KV = CT * RB;                       // bytes of a chunk's keys (or values)
    static constexpr int STAGE = 2 * KV + (ESZ == 1 ? 128 : 0);   // keys, values, scale bytes
    // Two stages a warp, 128 KB a CTA: with three the SMs' queues grow and some get their data
    // later than others (a 3.5 GB cache 530 us, with two 511). Registers: none spill but 16-head tiles at a
    // head dimension of 256 (255 registers, 92 bytes of stores in 16 bits, 134 in E4M3).
    static constexpr int NS = 2;
    static constexpr int ROWS = 8 * NH;                      // query heads of a tile
    static constexpr int OS = HD + 4;                        // floats from one row of a partial's o to the next
    static constexpr int PART = 2 * ROWS + ROWS * OS;        // floats of a partial: maxima, sums, o
    // a warp's ring, which takes its last piece in the end, then a place for its first piece
    static constexpr int RING = NS * STAGE > PART * 4 ? NS * STAGE : PART * 4;
    static constexpr int PER_WARP = (RING + PART * 4 + 127) / 128 * 128;
    static constexpr int WARPS_LOG2 = 8 * PER_WARP <= 210 * 1024 ? 3 : 2, WARPS = 1 << WARPS_LOG2;
    static constexpr int THREADS = 32 * WARPS;
    static constexpr int SMEM = WARPS * PER_WARP;
};
// Chunks that a segment's start and end count for in the shares (64 ragged sequences: 31.5 us with 1,
// 28.8 with 3, 28.8 with 6; many equal short ones lose a little with more).
constexpr int SEG = 3;

struct Args {
    const uint8_t *k, *v, *ks, *vs;   // the layer's pools
    const int *tables, *lens, *seqs;
    const void* q;
    void* out;
    float* lse;
    unsigned int* status;
    int* arrived;                     // CTAs that have left their partial, by segment or group; 0 between calls
    float* part;                      // [CTA][2][PART]: partials of segments that cross CTAs
    long long q_stride;
    float scale;
    float o_scale;                    // 1 / the weights' factor
    int n, q_heads, kv_heads, group, tiles_per_head, head_dim, page_log2, num_pages, max_seqs, max_pages, window, q_dt;
};

__device__ __forceinline__ void ldsm4(uint32_t a, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t a, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
template <bool BF>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (BF)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two E4M3 codes (low byte first) to a pair of fp16 values, exactly.
__device__ __forceinline__ uint32_t widen_e4m3x2(uint32_t w) {
    uint32_t d;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(d) : "h"((unsigned short)w));
    return d;
}
// The transpose of an 8x8 matrix of 16-bit values (a lane holds a pair of row lane / 4).
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}
// 16 bytes global -> shared; zeros when take is false (nothing is read then).
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool take) {
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(take ? 16 : 0)
                 : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const void* src, bool take) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(take ? 4 : 0) : "memory");
}

// 2^x to about 2 ulp; results below 2^-126 are 0.
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Byte offset of 16-byte piece c of row r in a tile of rows of PR pieces: eight rows read at one
// piece, or one row's eight pieces, touch all 32 banks.
template <int PR>
__device__ __forceinline__ uint32_t swz(int r, int c) {
    if constexpr (PR >= 8) return (uint32_t)(r * PR + (c ^ (r & 7))) * 16;
    else return (uint32_t)(r * PR + (c ^ ((r >> 1) & 3))) * 16;
}

// What sequence i of the launch has cached: its index, length (0 where it is invalid) and the
// first token that the window leaves.
__device__ __forceinline__ void seq_range(const Args& a, int i, int* seq, int* len, int* lo, bool report) {
    int s = a.seqs ? a.seqs[i] : i, l = 0, err = 0;
    if ((unsigned)s >= (unsigned)a.max_seqs) {
        s = 0, err = AQ_ERR_INVALID_ARG;
    } else {
        l = a.lens[s];
        const long long cap = (long long)a.max_pages << a.page_log2;
        if (l < 0 || l > cap) err = AQ_ERR_INVALID_ARG, l = l < 0 ? 0 : (int)cap;
    }
    if (err && report) record_status(a.status, err);
    *seq = s, *len = l;
    *lo = a.window > 0 && l > a.window ? l - a.window : 0;
}
// Chunks of a sequence: from the chunk of token lo to that of the last token.
template <int CT>
__device__ __forceinline__ int chunks_of(int len, int lo) {
    return len > 0 ? (len - 1) / CT - lo / CT + 1 : 0;
}

// a / b for non-negative a and positive b, in 32 bits where they fit.
__device__ __forceinline__ long long quotient(long long a, long long b) {
    return ((a | b) >> 32) == 0 ? (long long)((unsigned)a / (unsigned)b) : a / b;
}

// A place in the list of chunks. Positions count SEG for the start of every segment, then its
// chunks; base[i] is the position of entry i's first segment.
struct Place {
    int i, tile, seq, len, lo;        // entry, tile, and the entry's sequence and range
    int t;                            // first token of the chunk
    int left;                         // chunks of the segment from here on
    long long pos;
};

// The first chunk at or after position u (< the list's end; entry ranges as scanned).
template <int CT>
__device__ void place_at(const Args& a, const long long* base, const int2* range, const int* seq_of, long long u,
                         Place& p) {
    int lo = 0, hi = a.n - 1;
    while (lo < hi) {                 // the last entry that starts at or before u
        const int mid = (lo + hi + 1) >> 1;
        if (base[mid] <= u) lo = mid;
        else hi = mid - 1;
    }
    const int2 r = range[lo];
    const int chunks = chunks_of<CT>(r.x, r.y), per = chunks + SEG;
    const long long in = u - base[lo];
    const int tile = (int)quotient(in, per);
    const int c = max((int)(in - (long long)tile * per) - SEG, 0);
    p.i = lo, p.tile = tile, p.seq = seq_of[lo], p.len = r.x, p.lo = r.y;
    p.t = (r.y / CT + c) * CT;
    p.left = chunks - c;
    p.pos = base[lo] + (long long)tile * per + SEG + c;
}
__device__ __forceinline__ long long next_pos(const Place& p) { return p.pos + (p.left > 1 ? 1 : 1 + SEG); }

// To the next chunk of the list (there is one). True: it begins a segment.
template <int CT>
__device__ __forceinline__ bool advance(const Args& a, const int2* range, const int* seq_of, int tiles, Place& p) {
    p.pos = next_pos(p);
    if (--p.left > 0) {
        p.t += CT;
        return false;
    }
    if (++p.tile == tiles) {
        p.tile = 0;
        do {
            ++p.i;
        } while (p.i < a.n - 1 && range[p.i].x <= 0);
        p.seq = seq_of[p.i], p.len = range[p.i].x, p.lo = range[p.i].y;
    }
    p.left = chunks_of<CT>(p.len, p.lo);
    p.t = p.lo / CT * CT;
    return true;
}

// One segment as far as a warp has read it. A lane's columns are the heads 8 g + 2 (lane % 4) + x;
// m is the running maximum (of s_t log2 e + b), the same in a column's eight lanes; l the sum over
// the lane's own tokens. o[g][j][y] belongs to head column y & 1 and dimension dim_of(j, y >> 1).
template <int HD, int NH>
struct Acc {
    float o[NH][HD / 16][4];
    float m[NH][2], l[NH][2];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int g = 0; g < NH; ++g) {
#pragma unroll
            for (int j = 0; j < HD / 16; ++j)
#pragma unroll
                for (int y = 0; y < 4; ++y) o[g][j][y] = 0.0f;
            m[g][0] = m[g][1] = -INFINITY;
            l[g][0] = l[g][1] = 0.0f;
        }
    }
};
// E4M3 tiles take the even dimensions of 16 as rows 0..7 and the odd ones as rows 8..15.
template <int DT>
__device__ __forceinline__ int dim_of(int j, int half, int lane) {
    return DT == AQ_E4M3 ? 16 * j + 2 * (lane >> 2) + half : 16 * j + 8 * half + (lane >> 2);
}

// Over the eight lanes that share a column.
__device__ __forceinline__ float column_sum(float v) {
    v += __shfl_xor_sync(~0u, v, 4);
    v += __shfl_xor_sync(~0u, v, 8);
    return v + __shfl_xor_sync(~0u, v, 16);
}
__device__ __forceinline__ float column_max(float v) {
    v = fmaxf(v, __shfl_xor_sync(~0u, v, 4));
    v = fmaxf(v, __shfl_xor_sync(~0u, v, 8));
    return fmaxf(v, __shfl_xor_sync(~0u, v, 16));
}

// Two adjacent output elements of a query row.
__device__ __forceinline__ void store_out2(const Args& a, size_t q_row, int col, float v0, float v1) {
    uint32_t* o = (uint32_t*)((uint16_t*)a.out + q_row * a.head_dim + col);
    *o = a.q_dt == AQ_F16 ? round_pack2<AQ_F16>(v0, v1) : round_pack2<AQ_BF16>(v0, v1);
}
// 1 / sum; nothing seen (0) gives zeros, NaN stays NaN.
__device__ __forceinline__ float inverse_sum(float l) { return l > 0.0f ? 1.0f / l : l; }
__device__ __forceinline__ float lse_of(float m, float l) {
    return l > 0.0f ? kLn2 * (m + log2f(l)) : l == 0.0f ? -INFINITY : l;
}

// The query rows of a tile: first query head and how many there are.
template <int ROWS>
__device__ __forceinline__ void tile_rows(const Args& a, int tile, int* head0, int* rows) {
    const int kvh = tile / a.tiles_per_head, sub = tile - kvh * a.tiles_per_head;
    *head0 = kvh * a.group + sub * ROWS;
    *rows = min(ROWS, a.group - sub * ROWS);
}

// A finished segment to the output: the 16-bit values are transposed back to rows of heads.
template <int DT, int HD, int NH>
__device__ __forceinline__ void write_final(const Args& a, const Place& p, Acc<HD, NH>& acc, int lane) {
    int head0, rows;
    tile_rows<8 * NH>(a, p.tile, &head0, &rows);
    const int q = lane & 3;
#pragma unroll
    for (int g = 0; g < NH; ++g) {
        float inv[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const float l = column_sum(acc.l[g][x]);
            const int r = 8 * g + 2 * q + x;
            if (a.lse && lane < 4 && r < rows) a.lse[(size_t)p.i * a.q_heads + head0 + r] = lse_of(acc.m[g][x], l);
            inv[x] = inverse_sum(l) * a.o_scale;
        }
        const int r = 8 * g + (lane >> 2);
        uint16_t* out = (uint16_t*)a.out + ((size_t)p.i * a.q_heads + head0 + r) * a.head_dim;
#pragma unroll
        for (int j = 0; j < HD / 16; ++j) {
            const float* o = acc.o[g][j];
            uint32_t w0, w1;
            if (a.q_dt == AQ_F16) {
                w0 = round_pack2<AQ_F16>(o[0] * inv[0], o[1] * inv[1]);
                w1 = round_pack2<AQ_F16>(o[2] * inv[0], o[3] * inv[1]);
            } else {
                w0 = round_pack2<AQ_BF16>(o[0] * inv[0], o[1] * inv[1]);
                w1 = round_pack2<AQ_BF16>(o[2] * inv[0], o[3] * inv[1]);
            }
            w0 = transpose8x8(w0);
            w1 = transpose8x8(w1);
            if (r < rows && 16 * j < a.head_dim) {
                if constexpr (DT == AQ_E4M3) {
                    *(uint2*)(out + 16 * j + 4 * q) = make_uint2(prmt(w0, w1, 0x5410), prmt(w0, w1, 0x7632));
                } else {
                    *(uint32_t*)(out + 16 * j + 2 * q) = w0;
                    *(uint32_t*)(out + 16 * j + 8 + 2 * q) = w1;
                }
            }
        }
    }
}

// A partial: the rows' maxima, their sums, then o; rows past the real ones are left out.
template <int DT, int HD, int NH>
__device__ __forceinline__ void write_partial(const Args& a, int tile, const Acc<HD, NH>& acc, float* dst, int lane) {
    using T = Tile<DT, HD, NH>;
    int head0, rows;
    tile_rows<T::ROWS>(a, tile, &head0, &rows);
#pragma unroll
    for (int g = 0; g < NH; ++g)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const float l = column_sum(acc.l[g][x]);
            const int r = 8 * g + 2 * (lane & 3) + x;
            if (r >= rows) continue;
            if (lane < 4) dst[r] = acc.m[g][x], dst[T::ROWS + r] = l;
            float* o = dst + 2 * T::ROWS + r * T::OS;
#pragma unroll
            for (int j = 0; j < HD / 16; ++j) {
                o[dim_of<DT>(j, 0, lane)] = acc.o[g][j][x];
                o[dim_of<DT>(j, 1, lane)] = acc.o[g][j][2 + x];
            }
        }
}

// The factor that brings a partial with maximum m to maximum top.
__device__ __forceinline__ float rebase(float m, float top) { return m == -INFINITY ? 0.0f : exp2_fast(m - top); }

// Rows r0, r0 + 8 (while below `rows`; NH of them) of the `count` <= 32 partials of the list put
// together by a warp, in order, to output rows from q_row on, or to the partial dst (which may be one
// of the list: a row is read and written by one warp). A lane takes four columns, BATCH partials are
// under way at a time. OWN: the CTA's own pieces, in shared memory; otherwise partials of other
// CTAs, read through L2. Out of line: the main loop keeps its registers to itself.
template <bool OWN, int BATCH, int HD, int NH>
__device__ __noinline__ void merge_rows(const Args& a, const float* const* list, int count, int r0, int rows, size_t q_row,
                                        float* dst) {
    constexpr int ROWS = 8 * NH, OS = HD + 4;
    const int lane = threadIdx.x & 31;
    auto load = [](const float* q) { return OWN ? *q : __ldcg(q); };
    auto load4 = [](const float* q) { return OWN ? *(const float4*)q : __ldcg((const float4*)q); };
    const float* p = list[min(lane, count - 1)];
    int r[NH];                                       // (past the end: the first row again, not stored)
    float m[NH], l[NH];
#pragma unroll
    for (int g = 0; g < NH; ++g) {
        r[g] = r0 + 8 * g < rows ? r0 + 8 * g : r0;
        m[g] = load(p + r[g]), l[g] = load(p + ROWS + r[g]);
    }
    float4 v[NH][BATCH];
    const int col0 = 4 * (HD < 128 ? lane & (HD / 4 - 1) : lane);
    auto fetch = [&](int c, int y0) {                // (past the end: the last one again)
#pragma unroll
        for (int y = 0; y < BATCH; ++y) {
            const float* from = list[min(y0 + y, count - 1)] + 2 * ROWS + c + col0;
#pragma unroll
            for (int g = 0; g < NH; ++g) v[g][y] = load4(from + r[g] * OS);
        }
    };
    fetch(0, 0);                                     // before the maxima are known
    float f[NH], inv[NH];
#pragma unroll
    for (int g = 0; g < NH; ++g) {
        if (lane >= count) m[g] = -INFINITY, l[g] = 0.0f;
        float top = m[g];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
        f[g] = rebase(m[g], top == -INFINITY ? 0.0f : top);
        float sum = f[g] * l[g];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
        inv[g] = inverse_sum(sum) * a.o_scale;
        if (lane == 0 && r0 + 8 * g < rows) {
            if (dst) dst[r[g]] = top, dst[ROWS + r[g]] = sum;
            else if (a.lse) a.lse[q_row + r[g]] = lse_of(top, sum);
        }
    }
#pragma unroll 1
    for (int c = 0; c < HD; c += 128) {
        if (c > 0) fetch(c, 0);
        float4 o[NH];
#pragma unroll
        for (int g = 0; g < NH; ++g) o[g] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
        for (int y0 = 0;;) {
#pragma unroll
            for (int y = 0; y < BATCH; ++y)
#pragma unroll
                for (int g = 0; g < NH; ++g) {
                    const float fy = __shfl_sync(~0u, f[g], (y0 + y) & 31);
                    const float4 w = v[g][y];
                    if (y0 + y < count) o[g].x += fy * w.x, o[g].y += fy * w.y, o[g].z += fy * w.z, o[g].w += fy * w.w;
                }
            y0 += BATCH;
            if (y0 >= count) break;
            fetch(c, y0);
        }
#pragma unroll
        for (int g = 0; g < NH; ++g) {
            if (r0 + 8 * g >= rows) break;
            const int col = c + col0;
            if (dst) {
                *(float4*)(dst + 2 * ROWS + r[g] * OS + col) = o[g];
            } else if (col < a.head_dim) {
                store_out2(a, q_row + r[g], col, o[g].x * inv[g], o[g].y * inv[g]);
                store_out2(a, q_row + r[g], col + 2, o[g].z * inv[g], o[g].w * inv[g]);
            }
        }
    }
}

// Adds 1 to a counter; what the CTA wrote before (and a barrier) is seen by those that count later.
__device__ __forceinline__ int count_arrival(int* n) {
    int old;
    asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(old) : "l"(n) : "memory");
    return old;
}

// The query tile as B fragments (columns = query heads, k = head dimension), in the order of k that
// the keys' fragments come in, and each column's score factor: scale * log2 e, for E4M3 caches
// times the power of two that the row was divided by to fit fp16.
template <int DT, int HD, int NH>
__device__ __forceinline__ void load_query(const Args& a, const Place& p, int lane, uint32_t (&qf)[NH][HD / 16][2],
                                           float (&factor)[NH][2]) {
    int head0, rows;
    tile_rows<8 * NH>(a, p.tile, &head0, &rows);
    const int q = lane & 3;
#pragma unroll
    for (int g = 0; g < NH; ++g) {
        const int r = 8 * g + (lane >> 2);
        const bool real = r < rows;
        const uint16_t* row = (const uint16_t*)a.q + (size_t)p.i * a.q_stride + (size_t)(head0 + r) * a.head_dim;
        factor[g][0] = factor[g][1] = a.scale * kLog2e;
        if constexpr (DT != AQ_E4M3) {
#pragma unroll
            for (int ks = 0; ks < HD / 16; ++ks)
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    qf[g][ks][x] = real && 16 * ks < a.head_dim ? *(const uint32_t*)(row + 16 * ks + 8 * x + 2 * q) : 0u;
        } else {
            uint2 w[HD / 16];
            float top = 0.0f;
#pragma unroll
            for (int ks = 0; ks < HD / 16; ++ks)
                w[ks] = real && 16 * ks < a.head_dim ? *(const uint2*)(row + 16 * ks + 4 * q) : make_uint2(0, 0);
            auto widen = [&](const uint2& v, float (&f)[4]) {
                if (a.q_dt == AQ_F16) widen2<AQ_F16>(v.x, f[0], f[1]), widen2<AQ_F16>(v.y, f[2], f[3]);
                else widen2<AQ_BF16>(v.x, f[0], f[1]), widen2<AQ_BF16>(v.y, f[2], f[3]);
            };
#pragma unroll
            for (int ks = 0; ks < HD / 16; ++ks) {
                float f[4];
                widen(w[ks], f);
#pragma unroll
                for (int x = 0; x < 4; ++x) top = fmaxf(top, fabsf(f[x]));
            }
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
            const int e = min(max(exponent_of(top) - 14, -126), 112);    // |q| 2^-e < 2^15
            const float down = pow2f(-e), up = pow2f(e);
#pragma unroll
            for (int x = 0; x < 2; ++x) factor[g][x] *= __shfl_sync(~0u, up, 4 * (2 * q + x));
#pragma unroll
            for (int ks = 0; ks < HD / 16; ++ks) {
                float f[4];
                widen(w[ks], f);
                qf[g][ks][0] = round_pack2<AQ_F16>(f[0] * down, f[1] * down);
                qf[g][ks][1] = round_pack2<AQ_F16>(f[2] * down, f[3] * down);
            }
        }
    }
}

// Issues the copies of one chunk into a stage: the warp's lanes take 16-byte pieces, each of its
// token's page; tokens that are not seen become zeros (a weight of 0 times what happens to be
// there would not do). cur/nxt hold 32 table entries each, one a lane, from entry 32 * block on.
template <int DT, int HD>
struct Loader {
    using T = Tile<DT, HD, 1>;
    int cur, nxt, block, seq;

    __device__ __forceinline__ int entry(const Args& a, const Place& p, int b, int lane) const {
        const long long e = (long long)b * 32 + lane;
        return e << a.page_log2 < p.len ? a.tables[(size_t)p.seq * a.max_pages + e] : -1;
    }
    __device__ __forceinline__ void begin(const Args& a, const Place& p, int lane) {
        const int b = (p.t >> a.page_log2) >> 5;
        if (p.seq == seq && b == block) return;        // the next head of a short sequence
        block = b, seq = p.seq;
        cur = entry(a, p, block, lane);
        nxt = entry(a, p, block + 1, lane);
    }
    __device__ __forceinline__ void issue(const Args& a, const Place& p, uint32_t stage, int lane) {
        const int e0 = p.t >> a.page_log2;
        if (e0 >> 5 != block) {
            block = e0 >> 5;
            cur = nxt;
            nxt = entry(a, p, block + 1, lane);
        }
        const int kvh = p.tile / a.tiles_per_head;
        const int mask = (1 << a.page_log2) - 1;
        static_assert(T::PR <= 32, "a row is at most 32 pieces");
        constexpr int RPP = 32 / T::PR;                          // rows per pass, at most 8
        const int piece = lane % T::PR, row0 = lane / T::PR;
        const bool real = piece * 16 < a.head_dim * T::ESZ;
        const size_t row_bytes = (size_t)a.head_dim * T::ESZ;
        const bool full = p.t >= p.lo && p.t + T::CT <= p.len;
        if (mask >= 15 && full) {
            // all of the chunk is seen, and 16 rows that follow one another lie in one page
#pragma unroll
            for (int r1 = 0; r1 < T::CT; r1 += 16) {
                const int page = __shfl_sync(~0u, cur, ((p.t + r1) >> a.page_log2) & 31);
                const bool ok = (unsigned)page < (unsigned)a.num_pages;
                if (!ok) record_status(a.status, AQ_ERR_INVALID_ARG);
                const size_t row = (((size_t)(ok ? page : 0) * a.kv_heads + kvh) << a.page_log2) + ((p.t + r1) & mask) + row0;
                const size_t off = row * row_bytes + (real ? piece * 16 : 0);
                const uint8_t *k = a.k + off, *v = a.v + off;
#pragma unroll
                for (int r0 = 0; r0 < 16; r0 += RPP) {
                    const uint32_t d = stage + swz<T::PR>(r1 + r0 + row0, piece);
                    cp16(d, k + r0 * row_bytes, ok && real);
                    cp16(d + T::KV, v + r0 * row_bytes, ok && real);
                }
            }
        } else if (full) {
            // pages of eight tokens: a pass of at most eight rows has one
#pragma unroll
            for (int r0 = 0; r0 < T::CT; r0 += RPP) {
                const int page = __shfl_sync(~0u, cur, ((p.t + r0) >> a.page_log2) & 31);
                const bool ok = (unsigned)page < (unsigned)a.num_pages;
                if (!ok) record_status(a.status, AQ_ERR_INVALID_ARG);
                const size_t off =
                    ok && real ? ((((size_t)page * a.kv_heads + kvh) << a.page_log2) + ((p.t + r0) & mask) + row0) * row_bytes +
                                     piece * 16
                               : 0;
                const uint32_t d = stage + swz<T::PR>(r0 + row0, piece);
                cp16(d, a.k + off, ok && real);
                cp16(d + T::KV, a.v + off, ok && real);
            }
        } else {
#pragma unroll 1
            for (int r = row0; r < T::CT; r += RPP) {
                const int tok = p.t + r;
                const int page = __shfl_sync(~0u, cur, (tok >> a.page_log2) & 31);
                const bool in = tok >= p.lo && tok < p.len, ok = in && (unsigned)page < (unsigned)a.num_pages;
                if (in && !ok) record_status(a.status, AQ_ERR_INVALID_ARG);
                const size_t at = ok ? (((size_t)page * a.kv_heads + kvh) << a.page_log2) + (tok & mask) : 0;
                const size_t off = ok && real ? at * row_bytes + piece * 16 : 0;
                const uint32_t d = stage + swz<T::PR>(r, piece);
                cp16(d, a.k + off, ok && real);
                cp16(d + T::KV, a.v + off, ok && real);
            }
        }
        if constexpr (DT == AQ_E4M3) {
            // scale bytes, four tokens (of one page) a lane: keys' at 2 KV, values' at 2 KV + 64
            const int r = (lane & 15) * 4, tok = p.t + r;
            const int page = __shfl_sync(~0u, cur, (tok >> a.page_log2) & 31);
            // (four tokens at a time, unseen ones among them: their scores are masked)
            const bool ok = tok < p.len && (unsigned)page < (unsigned)a.num_pages;
            const size_t at = ok ? (((size_t)page * a.kv_heads + kvh) << a.page_log2) + (tok & mask) : 0;
            if (r < T::CT) {
                const bool vals = lane >= 16;
                cp4(stage + 2 * T::KV + (vals ? 64 : 0) + r, (vals ? a.vs : a.ks) + at, ok);
            }
        }
    }
};

// One chunk: scores, running maximum and sum, output.
template <int DT, int HD, int NH>
__device__ __forceinline__ void compute(const Place& p, uint32_t stage, int lane, const uint32_t (&qf)[NH][HD / 16][2],
                                        const float (&factor)[NH][2], Acc<HD, NH>& acc) {
    using T = Tile<DT, HD, NH>;
    constexpr bool BF = DT == AQ_BF16;
    constexpr int TT = T::CT / 16;                 // tiles of 16 tokens
    const int row = lane >> 2;                     // tokens of this lane in a tile: row and row + 8
    const int mi = lane >> 3, mr = lane & 7;       // this lane's matrix and row in an ldmatrix.x4
    float s[TT][NH][4];
#pragma unroll
    for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int g = 0; g < NH; ++g) s[tt][g][0] = s[tt][g][1] = s[tt][g][2] = s[tt][g][3] = 0.0f;
    if constexpr (DT != AQ_E4M3) {
#pragma unroll
        for (int ks = 0; ks < HD / 16; ++ks)
#pragma unroll
            for (int tt = 0; tt < TT; ++tt) {
                uint32_t k[4];
                ldsm4(stage + swz<T::PR>(tt * 16 + (mi & 1) * 8 + mr, 2 * ks + (mi >> 1)), k);
#pragma unroll
                for (int g = 0; g < NH; ++g) mma16816<BF>(s[tt][g], k, qf[g][ks][0], qf[g][ks][1]);
            }
    } else {
#pragma unroll
        for (int c = 0; c < HD / 16; c += 2)
#pragma unroll
            for (int tt = 0; tt < TT; ++tt) {
                uint32_t r[4];
                ldsm4(stage + swz<T::PR>(tt * 16 + (mi & 1) * 8 + mr, c + (mi >> 1)), r);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const uint32_t lo = r[2 * x], hi = r[2 * x + 1];
                    const uint32_t k[4] = {widen_e4m3x2(lo), widen_e4m3x2(hi), widen_e4m3x2(lo >> 16),
                                           widen_e4m3x2(hi >> 16)};
#pragma unroll
                    for (int g = 0; g < NH; ++g) mma16816<false>(s[tt][g], k, qf[g][c + x][0], qf[g][c + x][1]);
                }
            }
    }
    // base-2 scores, for E4M3 plus the value scale's exponent b; masked ones are -inf
    const bool edge = p.t < p.lo || p.t + T::CT > p.len;
    float vexp[TT][2], vfac[TT][2];                // b and 2^b times the weights' factor of the tokens' value scales
    float top[NH][2];
#pragma unroll
    for (int g = 0; g < NH; ++g) top[g][0] = top[g][1] = -INFINITY;
#pragma unroll
    for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int tok = p.t + tt * 16 + h * 8 + row;
            const bool out = edge && (tok < p.lo || tok >= p.len);
            float kf = 1.0f;
            if constexpr (DT == AQ_E4M3) {
                uint32_t kb, vb;
                const uint32_t at = stage + 2 * T::KV + tt * 16 + h * 8 + row;
                asm volatile("ld.shared.u8 %0, [%1];" : "=r"(kb) : "r"(at) : "memory");
                asm volatile("ld.shared.u8 %0, [%1];" : "=r"(vb) : "r"(at + 64) : "memory");
                kf = __uint_as_float(kb << 23);
                // (a bad page's bytes are 0; taken as -127, a piece of them alone would have sums beyond fp32)
                vexp[tt][h] = (float)max((int)vb - 127, -kScaleExpMax);
                vfac[tt][h] = out ? 0.0f : __uint_as_float(vb << 23) * kFp16Weights;   // (an unseen token's byte may be anything)
            }
#pragma unroll
            for (int g = 0; g < NH; ++g)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    float& v = s[tt][g][2 * h + x];
                    v = out ? -INFINITY : v * (DT == AQ_E4M3 ? factor[g][x] * kf : factor[g][x]);
                    if constexpr (DT == AQ_E4M3) v += vexp[tt][h];
                    top[g][x] = fmaxf(top[g][x], v);
                }
        }
    float sub[NH][2];
    bool moved = false;
#pragma unroll
    for (int g = 0; g < NH; ++g)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            top[g][x] = fmaxf(column_max(top[g][x]), acc.m[g][x]);
            moved |= top[g][x] > acc.m[g][x];
            sub[g][x] = top[g][x] == -INFINITY ? 0.0f : top[g][x];
        }
    if (__any_sync(~0u, moved)) {
#pragma unroll
        for (int g = 0; g < NH; ++g)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const float f = rebase(acc.m[g][x], sub[g][x]);
                acc.m[g][x] = top[g][x];
                acc.l[g][x] *= f;
#pragma unroll
                for (int j = 0; j < HD / 16; ++j) acc.o[g][j][x] *= f, acc.o[g][j][2 + x] *= f;
            }
    }
    // weights: p for the sum, p 2^b rounded to 16 bits for the product with V, as B fragments. E4M3: b is
    // taken off after the maximum, so that p 2^b is at most 1 however s + b was rounded.
    uint32_t w[TT][NH][2];
#pragma unroll
    for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int g = 0; g < NH; ++g)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float p0 = s[tt][g][2 * h] - sub[g][0], p1 = s[tt][g][2 * h + 1] - sub[g][1];
                if constexpr (DT == AQ_E4M3) p0 -= vexp[tt][h], p1 -= vexp[tt][h];
                p0 = exp2_fast(p0), p1 = exp2_fast(p1);
                acc.l[g][0] += p0;
                acc.l[g][1] += p1;
                if constexpr (DT == AQ_E4M3) p0 *= vfac[tt][h], p1 *= vfac[tt][h];
                if constexpr (DT == AQ_F16) p0 *= kFp16Weights, p1 *= kFp16Weights;
                w[tt][g][h] = transpose8x8(round_pack2<BF ? AQ_BF16 : AQ_F16>(p0, p1));
            }
    const uint32_t vt = stage + T::KV;
#pragma unroll
    for (int tt = 0; tt < TT; ++tt) {
        if constexpr (DT != AQ_E4M3) {
#pragma unroll
            for (int j = 0; j < HD / 16; ++j) {
                uint32_t v[4];
                ldsm4t(vt + swz<T::PR>(tt * 16 + (mi >> 1) * 8 + mr, 2 * j + (mi & 1)), v);
#pragma unroll
                for (int g = 0; g < NH; ++g) mma16816<BF>(acc.o[g][j], v, w[tt][g][0], w[tt][g][1]);
            }
        } else {
#pragma unroll
            for (int c = 0; c < HD / 16; c += 2) {
                uint32_t r[4];
                ldsm4t(vt + swz<T::PR>(tt * 16 + (mi & 1) * 8 + mr, c + (mi >> 1)), r);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const uint32_t lo = r[2 * x], hi = r[2 * x + 1];   // tokens 2q, 2q+1; + 8
                    const uint32_t v[4] = {widen_e4m3x2(prmt(lo, 0, 0x20)), widen_e4m3x2(prmt(lo, 0, 0x31)),
                                           widen_e4m3x2(prmt(hi, 0, 0x20)), widen_e4m3x2(prmt(hi, 0, 0x31))};
#pragma unroll
                    for (int g = 0; g < NH; ++g) mma16816<false>(acc.o[g][c + x], v, w[tt][g][0], w[tt][g][1]);
                }
            }
        }
    }
}

// Positions of the launch's n entries into base[0..n] (shared), their ranges and sequences;
// all threads. Each thread takes consecutive entries, so the sums stay in order.
template <int CT, int WARPS>
__device__ void scan_entries(const Args& a, int tiles, long long* base, int2* range, int* seq_of) {
    __shared__ long long warp_sum[WARPS];
    constexpr int PER = kSliceSeqs / (32 * WARPS);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long c[PER], mine = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int i = threadIdx.x * PER + j;
        c[j] = 0;
        if (i < a.n) {
            int seq, len, lo;
            seq_range(a, i, &seq, &len, &lo, blockIdx.x == 0);
            range[i] = make_int2(len, lo);
            seq_of[i] = seq;
            const int chunks = chunks_of<CT>(len, lo);
            c[j] = chunks ? (long long)(chunks + SEG) * tiles : 0;
        }
        mine += c[j];
    }
    long long s = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long o = __shfl_up_sync(~0u, s, d);
        if (lane >= d) s += o;
    }
    if (lane == 31) warp_sum[warp] = s;
    __syncthreads();
    long long at = s - mine;
    for (int w = 0; w < warp; ++w) at += warp_sum[w];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int i = threadIdx.x * PER + j;
        if (i < a.n) base[i] = at;
        at += c[j];
        if (i == a.n - 1) base[a.n] = at;
    }
    __syncthreads();
}

// Positions each warp takes.
__device__ __forceinline__ long long share_of(long long total, int warps) {
    const long long per = quotient(total + warps - 1, warps);
    return per < 1 ? 1 : per;
}

// A segment that crosses CTAs: the first of them, how many they are, its query rows.
struct Crossing {
    int j0, count, rows;
    size_t q_row;
    // CTAs that are joined at a time, and the first of CTA k's group.
    __device__ __forceinline__ int group() const { return count <= 32 ? count : 16; }
    __device__ __forceinline__ int first_of(int k) const { return count <= 32 ? 0 : k & ~15; }
};

template <int WARPS>
struct Shared {
    long long base[kSliceSeqs + 1];   // positions of the entries' first segments
    int2 range[kSliceSeqs];           // their lengths and first tokens seen
    int seq_of[kSliceSeqs];
    int piece_seg[2 * WARPS];         // segments of the warps' first and last pieces (-1: none)
    const float* list[WARPS][32];     // the partials that a warp puts together
    Crossing cross[2];
    bool last[2];
};

// What the CTA does after its warps' shares. Pieces of one segment are adjacent; the warps take the
// segments' rows in turn and merge their pieces. Of a segment that crosses CTAs (at most two of a
// CTA's do) that gives a partial (0: of the one that began before, 1: of the one that begins here),
// which come first: the segments that are the CTA's own are merged while its arrival is counted
// (a fence and an atomic through L2, one of each per CTA). The last CTA of a crossing segment to
// arrive joins the partials. Where there are many (few kv heads, one long sequence) groups of
// consecutive CTAs are joined first, in the same way, each into its first CTA's partial.
template <int DT, int HD, int NH>
__device__ __forceinline__ void finish(const Args& a, Shared<Tile<DT, HD, NH>::WARPS>& s, const uint8_t* ring, long long share,
                                       long long cta0, long long cta1) {
    using T = Tile<DT, HD, NH>;
    constexpr int kWarps = T::WARPS;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int tiles = a.kv_heads * a.tiles_per_head;
    const float** const list = s.list[warp];
    // Lane y holds piece y's segment: its rows, whether all of it is here, and if not its place
    // among the CTA's two crossing segments, its first CTA and how many it crosses.
    const int mine = lane < 2 * kWarps ? s.piece_seg[lane] : -1;
    const unsigned pieces = __ballot_sync(~0u, mine >= 0);
    int head0 = 0, rows = 0, entry = 0, j0 = 0, ctas = 0, which = 0;
    bool done = false;
    if (mine >= 0) {
        entry = mine / tiles;
        const int tile = mine - entry * tiles;
        const long long per = chunks_of<T::CT>(s.range[entry].x, s.range[entry].y) + SEG;
        const long long s0 = s.base[entry] + per * tile + SEG, s1 = s.base[entry] + per * (tile + 1);
        tile_rows<T::ROWS>(a, tile, &head0, &rows);
        done = s0 >= cta0 && s1 <= cta1;
        which = s0 < cta0 ? 0 : 1;
        if (!done) {
            j0 = (int)quotient(s0, share * kWarps);
            ctas = (int)quotient(s1 - 1, share * kWarps) - j0 + 1;
        }
    }
    const bool crossing = __any_sync(~0u, mine >= 0 && !done);
    int turn = 0;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
        const unsigned of_pass = __ballot_sync(~0u, mine >= 0 && done == (pass == 1));
#pragma unroll 1
        for (unsigned rest = of_pass; rest;) {
            const int y0 = __ffs(rest) - 1;
            const unsigned of_seg = __ballot_sync(~0u, mine == __shfl_sync(~0u, mine, y0));
            rest &= ~of_seg;
            const int seg_rows = __shfl_sync(~0u, rows, y0);
            int r = (warp - turn) & (kWarps - 1);
            const int first_rows = min(seg_rows, 8);   // (the others come with them)
            turn += first_rows;
            const size_t q_row = (size_t)__shfl_sync(~0u, entry, y0) * a.q_heads + __shfl_sync(~0u, head0, y0);
            const int w = __shfl_sync(~0u, which, y0);
            if (pass == 0 && threadIdx.x == y0) s.cross[w] = {j0, ctas, rows, q_row};
            if (r >= first_rows) continue;
            if (of_seg >> lane & 1)
                list[__popc(of_seg & ((1u << lane) - 1))] = (const float*)(ring + (lane >> 1) * T::PER_WARP) + (lane & 1 ? 0 : T::RING / 4);
            __syncwarp();
            float* const dst = pass == 1 ? nullptr : a.part + ((size_t)blockIdx.x * 2 + w) * T::PART;
            for (; r < first_rows; r += kWarps)
                merge_rows<true, 4, HD, NH>(a, list, __popc(of_seg), r, seg_rows, q_row, dst);
            __syncwarp();
        }
        if (pass == 0 && crossing) {
            __syncthreads();
            if (threadIdx.x < 2) {
                bool all = false;
                const Crossing x = s.cross[threadIdx.x];
                if (x.count > 0) {
                    const int k0 = x.first_of((int)blockIdx.x - x.j0);
                    int* n = a.arrived + 2 * (x.j0 + k0) + (k0 == 0 ? 1 : 0);
                    all = count_arrival(n) == min(x.group(), x.count - k0) - 1;
                    if (all) *n = 0;               // for the next call
                }
                s.last[threadIdx.x] = all;
            }
        }
    }
    if (!crossing) return;
    __syncthreads();
#pragma unroll 1
    for (int w = 0; w < 2; ++w) {
        if (!s.last[w]) continue;
        const Crossing x = s.cross[w];
        const int g = x.group();
        int k = x.first_of((int)blockIdx.x - x.j0), step = 1, members = min(g, x.count - k);
        bool final = g == x.count;
#pragma unroll 1
        while (true) {
            auto part = [&](int y) {
                const int j = k + y * step;
                return a.part + (size_t)((x.j0 + j) * 2 + (j == 0 ? 1 : 0)) * T::PART;
            };
            if (lane < members) list[lane] = part(lane);
            __syncwarp();
            float* const dst = final ? nullptr : part(0);
            for (int r = warp; r < min(x.rows, 8); r += kWarps) {
                if (members <= 4) merge_rows<false, 4, HD, NH>(a, list, members, r, x.rows, x.q_row, dst);
                else merge_rows<false, NH == 1 ? 20 : 16, HD, NH>(a, list, members, r, x.rows, x.q_row, dst);
            }
            __syncwarp();
            if (final) break;
            members = (x.count + g - 1) / g, step = g, k = 0, final = true;   // the groups' results
            __syncthreads();
            if (threadIdx.x == 0) {
                int* n = a.arrived + 2 * kMaxCtas + x.j0;
                s.last[w] = count_arrival(n) == members - 1;
                if (s.last[w]) *n = 0;
            }
            __syncthreads();
            if (!s.last[w]) break;
        }
    }
}

template <int DT, int HD, int NH>
__global__ void __launch_bounds__((Tile<DT, HD, NH>::THREADS), 1) kv_attend_kernel(const __grid_constant__ Args a) {
    using T = Tile<DT, HD, NH>;
    constexpr int kWarps = T::WARPS, kThreads = T::THREADS;
    extern __shared__ __align__(1024) uint8_t ring[];
    __shared__ Shared<kWarps> s;
    long long* const base = s.base;
    int2* const range = s.range;
    int* const seq_of = s.seq_of;
    int* const piece_seg = s.piece_seg;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int tiles = a.kv_heads * a.tiles_per_head;
    pdl_wait();
    scan_entries<T::CT, kWarps>(a, tiles, base, range, seq_of);
    pdl_launch_dependents();
    // entries that see nothing
    for (int i = blockIdx.x; i < a.n; i += gridDim.x)
        if (range[i].x <= 0) {
            uint32_t* o = (uint32_t*)((uint16_t*)a.out + (size_t)i * a.q_heads * a.head_dim);
            for (int j = threadIdx.x; j < a.q_heads * a.head_dim / 2; j += kThreads) o[j] = 0u;
            if (a.lse)
                for (int j = threadIdx.x; j < a.q_heads; j += kThreads) a.lse[(size_t)i * a.q_heads + j] = -INFINITY;
        }
    const long long total = base[a.n], share = share_of(total, gridDim.x * kWarps);
    const long long cta0 = min(total, share * kWarps * blockIdx.x), cta1 = min(total, cta0 + share * kWarps);
    const long long u0 = min(total, cta0 + share * warp), u1 = min(total, u0 + share);
    if (cta0 >= cta1) return;

    if (lane < 2) piece_seg[2 * warp + lane] = -1;
    if (threadIdx.x < 2) s.cross[threadIdx.x].count = 0;
    __syncwarp();
    Place at;
    if (u0 < u1) place_at<T::CT>(a, base, range, seq_of, u0, at);
    if (u0 < u1 && at.pos < u1) {
        const uint32_t stages = smem_u32(ring + warp * T::PER_WARP);
        Place in = at;
        bool more = true;                          // chunk `in` is still to be issued
        Loader<DT, HD> loader;
        loader.seq = -1;
        loader.begin(a, in, lane);
        int fill = 0;
        auto issue = [&]() {
            if (more) {
                loader.issue(a, in, stages + fill * T::STAGE, lane);
                more = next_pos(in) < u1;
                if (more && advance<T::CT>(a, range, seq_of, tiles, in)) loader.begin(a, in, lane);
            }
            if (++fill == T::NS) fill = 0;
            cp_async_commit();
        };
        uint32_t qf[NH][HD / 16][2];
        float factor[NH][2];
        Acc<HD, NH> acc;
        bool whole = at.t / T::CT == at.lo / T::CT;   // the segment begins in this warp's share
#pragma unroll 1
        for (int k = 0; k < T::NS - 1; ++k) issue();
        load_query<DT, HD, NH>(a, at, lane, qf, factor);
        acc.clear();
        int use = 0;
#pragma unroll 1
        while (true) {
            issue();
            cp_async_wait<T::NS - 1>();
            __syncwarp();
            compute<DT, HD, NH>(at, stages + use * T::STAGE, lane, qf, factor, acc);
            __syncwarp();
            if (++use == T::NS) use = 0;
            const bool last = next_pos(at) >= u1, ends = at.left == 1;
            if (!last && !ends) {
                at.t += T::CT;
                --at.left;
                ++at.pos;
                continue;
            }
            if (whole && ends) {
                write_final<DT, HD, NH>(a, at, acc, lane);
            } else {
                // The ring is free once the share's last chunk has been read (only empty groups
                // of copies are left then); an earlier piece has a place of its own.
                float* dst = (float*)(ring + warp * T::PER_WARP) + (last ? 0 : T::RING / 4);
                write_partial<DT, HD, NH>(a, at.tile, acc, dst, lane);
                if (lane == 0) piece_seg[2 * warp + last] = at.i * tiles + at.tile;
            }
            if (last) break;
            advance<T::CT>(a, range, seq_of, tiles, at);
            whole = true;
            load_query<DT, HD, NH>(a, at, lane, qf, factor);
            acc.clear();
        }
    }
    __syncthreads();
    finish<DT, HD, NH>(a, s, ring, share, cta0, cta1);
}

template <int DT, int HD, int NH>
size_t attend_ws() {
    using T = Tile<DT, HD, NH>;
    return kWsStatusBytes + kArrivedBytes + (size_t)kMaxCtas * 2 * T::PART * 4;
}

template <int DT, int HD, int NH>
aq_status attend(Args a, const DeviceInfo& di, int n, cudaStream_t st) {
    using T = Tile<DT, HD, NH>;
    static std::atomic<bool> have[64];             // (setting the attribute twice is harmless)
    int dev = 0;
    if (cudaError_t e = cudaGetDevice(&dev); e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
    if (!have[dev & 63]) {
        if (cudaError_t e = cudaFuncSetAttribute(kv_attend_kernel<DT, HD, NH>,
                                                 cudaFuncAttributeMaxDynamicSharedMemorySize, T::SMEM);
            e != cudaSuccess)
            return cuda_fail(e, "cudaFuncSetAttribute");
        have[dev & 63] = true;
    }
    const int ctas = di.sms < kMaxCtas ? di.sms : kMaxCtas;
    char* ws = (char*)a.status;
    a.arrived = (int*)(ws + kWsStatusBytes);
    a.part = (float*)(ws + kWsStatusBytes + kArrivedBytes);
    a.tiles_per_head = (a.group + T::ROWS - 1) / T::ROWS;
    for (int i0 = 0; i0 < n; i0 += kSliceSeqs) {
        Args s = a;
        s.n = n - i0 < kSliceSeqs ? n - i0 : kSliceSeqs;
        if (s.seqs) s.seqs += i0;
        else s.lens += i0, s.tables += (size_t)i0 * a.max_pages, s.max_seqs -= i0;
        s.q = (const uint16_t*)a.q + (size_t)i0 * a.q_stride;
        s.out = (uint16_t*)a.out + (size_t)i0 * a.q_heads * a.head_dim;
        if (s.lse) s.lse += (size_t)i0 * a.q_heads;
        if (aq_status e = launch_dependent(kv_attend_kernel<DT, HD, NH>, ctas, T::THREADS, T::SMEM, st, s); e != AQ_OK)
            return e;
    }
    return AQ_OK;
}

// Calls f<DT, HD, NH>() for the cache's type, the padded head dimension and one or two groups of
// eight query heads per tile.
#define AQ_KV_DISPATCH_HD(HD, f, ...)                                                       \
    (c.dtype == AQ_F16    ? (two ? f<AQ_F16, HD, 2>(__VA_ARGS__) : f<AQ_F16, HD, 1>(__VA_ARGS__))   \
     : c.dtype == AQ_BF16 ? (two ? f<AQ_BF16, HD, 2>(__VA_ARGS__) : f<AQ_BF16, HD, 1>(__VA_ARGS__)) \
                          : (two ? f<AQ_E4M3, HD, 2>(__VA_ARGS__) : f<AQ_E4M3, HD, 1>(__VA_ARGS__)))
#define AQ_KV_DISPATCH(f, ...)                                  \
    (c.head_dim <= 64    ? AQ_KV_DISPATCH_HD(64, f, __VA_ARGS__)  \
     : c.head_dim <= 128 ? AQ_KV_DISPATCH_HD(128, f, __VA_ARGS__) \
                         : AQ_KV_DISPATCH_HD(256, f, __VA_ARGS__))

}  // namespace

size_t kv_attend_ws_bytes(const aq_kv_cache& c, int q_heads) {
    const bool two = q_heads / c.kv_heads > 8;
    return AQ_KV_DISPATCH(attend_ws);
}

aq_status launch_kv_attend(const aq_kv_cache& c, const DeviceInfo& di, int layer, int n, const int* seqs,
                           const void* q, int q_dt, long long q_stride, int q_heads, float scale, int window,
                           void* out, float* lse, void* ws, cudaStream_t st) {
    Args a = {};
    const size_t rows = (size_t)c.num_pages * c.kv_heads * c.page_tokens;       // a layer's
    const size_t esz = c.dtype == AQ_E4M3 ? 1 : 2, off = (size_t)layer * rows;
    a.k = (const uint8_t*)c.k + off * c.head_dim * esz;
    a.v = (const uint8_t*)c.v + off * c.head_dim * esz;
    if (c.dtype == AQ_E4M3) {
        a.ks = (const uint8_t*)c.k_scales + off;
        a.vs = (const uint8_t*)c.v_scales + off;
    }
    a.tables = c.tables, a.lens = c.lens, a.seqs = seqs;
    a.q = q, a.q_dt = q_dt, a.q_stride = q_stride;
    a.out = out, a.lse = lse;
    a.status = (unsigned int*)ws;
    a.scale = scale;
    a.o_scale = c.dtype == AQ_BF16 ? 1.0f : 1.0f / kFp16Weights;
    a.q_heads = q_heads, a.kv_heads = c.kv_heads, a.group = q_heads / c.kv_heads;
    a.head_dim = c.head_dim;
    while ((1 << a.page_log2) < c.page_tokens) ++a.page_log2;
    a.num_pages = c.num_pages, a.max_seqs = c.max_seqs, a.max_pages = c.max_pages, a.window = window;
    const bool two = a.group > 8;
    return AQ_KV_DISPATCH(attend, a, di, n, st);
}

}  // namespace aq
