// Attention of one new token per sequence over the paged key-value cache (aq_kv_attend).
//
//   s_t = scale * q . k_t for the cached tokens t the query sees (t >= L - window),
//   o = sum_t p_t v_t / sum_t p_t with p_t = exp(s_t - max), lse = max + ln sum_t p_t,
// in one pass over the cache with a running maximum and sum.
//
// Bound: every cached key and value is read once, 4 * head_dim bytes per token and head with
// 16-bit entries, for 4 * head_dim * (query heads per kv head) operations: a few operations per
// byte, so HBM is the limit and the work is arranged around keeping loads in flight.
//   - A tile is up to 16 query heads that share a kv head; mma.sync m16n8k16 takes the heads as
//     its rows. (At the copy bandwidth an SM receives 24 bytes a cycle, which asks for about 190
//     multiply-adds a cycle of the padded 16-row tile; the legacy tensor path has several times
//     that, and its fragments come straight from the copied tiles, so tensor memory would add
//     waits and nothing else.)
//   - The work is the list of all (sequence, tile) segments cut into chunks of CT tokens; every
//     warp takes an equal, contiguous share of the list whatever the sequences' lengths, and runs
//     through it with a ring of asynchronous copies of its own that crosses segment ends: no
//     CTA-wide step until the end.
//   - A segment that lies in one warp's share is written at once. Pieces of segments are merged
//     per CTA, and what crosses CTAs is joined by a second kernel, in the order of the tokens, so
//     the result does not depend on scheduling.
//
// Numbers: products of 16-bit values are accumulated in fp32 by the tensor cores; the statistics
// and accumulators are fp32. The weights p_t are rounded to the cache's 16-bit type for the
// product with V (a relative error of at most 2^-8 (bf16) or 2^-11 (fp16) of each, no more than
// the rounding of the 16-bit output); their sum is taken before that rounding. E4M3 entries widen
// exactly to fp16; the query is scaled to fp16's range by a power of two. A key's scale
// multiplies its score; a value's scale 2^b multiplies its weight, with the running maximum taken
// over s_t log2 e + b so that the fp16 weights stay in [0, 1].
#include <atomic>

#include "kv.cuh"

namespace aq {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kSliceSeqs = 512;       // sequences per launch (their offsets sit in shared memory)
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Sizes for a cache type and a padded head dimension HD (64, 128 or 256).
template <int DT, int HD>
struct Tile {
    static constexpr int ESZ = DT == AQ_E4M3 ? 1 : 2;
    static constexpr int RB = HD * ESZ;                      // bytes of a token's row
    static constexpr int PR = RB / 16;                       // 16-byte pieces of a row
    static constexpr int CT = (HD == 64 || (HD == 128 && ESZ == 1)) ? 32 : 16;   // tokens per chunk
    static constexpr int KV = CT * RB;                       // bytes of a chunk's keys (or values)
    static constexpr int STAGE = 2 * KV + (ESZ == 1 ? 128 : 0);   // keys, values, scale bytes
    static constexpr int NS = STAGE <= 4224 ? 6 : HD == 256 && ESZ == 1 ? 5 : 3;
    static constexpr int RING = NS * STAGE;                  // a warp's ring
    static constexpr int PART = 32 + 16 * HD;                // floats of a partial: max, sum, o
    static_assert(RING >= PART * 4, "a warp's ring holds its last partial");
    static constexpr int CTAS = HD == 256 ? 1 : 2;           // per SM
    static constexpr int SMEM = kWarps * RING;
};

struct Args {
    const uint8_t *k, *v, *ks, *vs;   // the layer's pools
    const int *tables, *lens, *seqs;
    const void* q;
    void* out;
    float* lse;
    unsigned int* status;
    float* part;                      // [CTA][2][PART], then [CTA * warps][PART] for first pieces
    float* first;
    long long* base;                  // [n + 1] offsets, for the join
    long long q_stride;
    float scale;
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

// A place in the list of chunks.
struct Place {
    int i, tile, seq, len, lo;        // sequence entry, tile and its range
    int t;                            // first token of the chunk
    int left;                         // chunks of the segment from here on
};

// The segment that holds chunk u, and the place of u in it (base: chunk offsets of the n entries).
template <int CT>
__device__ void place_at(const Args& a, const long long* base, const int2* range, const int* seq_of, int tiles,
                         long long u, Place& p) {
    int lo = 0, hi = a.n - 1;
    while (lo < hi) {                 // the last entry that starts at or before u
        const int mid = (lo + hi + 1) >> 1;
        if (base[mid] <= u) lo = mid;
        else hi = mid - 1;
    }
    const int2 r = range[lo];
    const int per = chunks_of<CT>(r.x, r.y);
    const long long in = u - base[lo];
    const int tile = (int)(in / per), c = (int)(in - (long long)tile * per);
    p.i = lo, p.tile = tile, p.seq = seq_of[lo], p.len = r.x, p.lo = r.y;
    p.t = (r.y / CT + c) * CT;
    p.left = per - c;
}
// To the next chunk of the list (there is one).
template <int CT>
__device__ __forceinline__ bool advance(const Args& a, const int2* range, const int* seq_of, int tiles, Place& p) {
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

// Scores, weights and output of one segment as far as a warp has read it. Rows: lane / 4 and that
// + 8; the running maximum (of s_t log2 e + b) is the same in a row's four lanes, the sums are
// each lane's own columns'.
template <int HD>
struct Acc {
    float o[HD / 8][4];
    float m[2], l[2];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int j = 0; j < HD / 8; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) o[j][x] = 0.0f;
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.0f;
    }
};

// The head dimension that o[j][x] of a lane with lane % 4 == q belongs to (x = 0, 1; 2 and 3 are
// the same columns of the other row). E4M3 tiles pair the even and the odd columns of 16.
template <int DT>
__device__ __forceinline__ int column_of(int j, int x, int q) {
    return DT == AQ_E4M3 ? 16 * (j >> 1) + 4 * q + 2 * x + (j & 1) : 8 * j + 2 * q + x;
}

__device__ __forceinline__ float quad_sum(float v) {
    v += __shfl_xor_sync(~0u, v, 1);
    return v + __shfl_xor_sync(~0u, v, 2);
}
__device__ __forceinline__ float quad_max(float v) {
    v = fmaxf(v, __shfl_xor_sync(~0u, v, 1));
    return fmaxf(v, __shfl_xor_sync(~0u, v, 2));
}

// Two adjacent output elements of a query row.
__device__ __forceinline__ void store_out2(const Args& a, size_t q_row, int col, float v0, float v1) {
    uint32_t* o = (uint32_t*)((uint16_t*)a.out + q_row * a.head_dim + col);
    *o = a.q_dt == AQ_F16 ? round_pack2<AQ_F16>(v0, v1) : round_pack2<AQ_BF16>(v0, v1);
}
__device__ __forceinline__ float lse_of(float m, float l) {
    return l > 0.0f ? kLn2 * (m + log2f(l)) : -INFINITY;
}

// The query rows of (entry i, tile): first query head and how many of the 16 rows are real.
__device__ __forceinline__ void tile_rows(const Args& a, int tile, int* head0, int* rows) {
    const int kvh = tile / a.tiles_per_head, sub = tile - kvh * a.tiles_per_head;
    *head0 = kvh * a.group + sub * 16;
    *rows = min(16, a.group - sub * 16);
}

template <int DT, int HD>
__device__ __forceinline__ void write_final(const Args& a, const Place& p, Acc<HD>& acc, int lane) {
    int head0, rows;
    tile_rows(a, p.tile, &head0, &rows);
    const int g = lane >> 2, q = lane & 3;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float l = quad_sum(acc.l[h]);
        const int r = g + 8 * h;
        if (r >= rows) continue;
        const size_t q_row = (size_t)p.i * a.q_heads + head0 + r;
        const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;   // NaN stays NaN
        if (a.lse && q == 0) a.lse[q_row] = l == l ? lse_of(acc.m[h], l) : l;
#pragma unroll
        for (int j = 0; j < HD / 8; j += DT == AQ_E4M3 ? 2 : 1) {
            if constexpr (DT == AQ_E4M3) {
                const int col = column_of<DT>(j, 0, q);
                if (col < a.head_dim) {
                    store_out2(a, q_row, col, acc.o[j][2 * h] * inv, acc.o[j + 1][2 * h] * inv);
                    store_out2(a, q_row, col + 2, acc.o[j][2 * h + 1] * inv, acc.o[j + 1][2 * h + 1] * inv);
                }
            } else {
                const int col = column_of<DT>(j, 0, q);
                if (col < a.head_dim) store_out2(a, q_row, col, acc.o[j][2 * h] * inv, acc.o[j][2 * h + 1] * inv);
            }
        }
    }
}

// A partial: max of the 16 rows, their sums, then o [16][HD]; rows past the real ones are left out.
template <int DT, int HD>
__device__ __forceinline__ void write_partial(const Args& a, int tile, const Acc<HD>& acc, float* dst, int lane) {
    int head0, rows;
    tile_rows(a, tile, &head0, &rows);
    const int g = lane >> 2, q = lane & 3;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float l = quad_sum(acc.l[h]);
        const int r = g + 8 * h;
        if (r >= rows) continue;
        if (q == 0) dst[r] = acc.m[h], dst[16 + r] = l;
        float* o = dst + 32 + r * HD;
#pragma unroll
        for (int j = 0; j < HD / 8; ++j) {
            if constexpr (DT == AQ_E4M3) {
                o[column_of<DT>(j, 0, q)] = acc.o[j][2 * h];
                o[column_of<DT>(j, 1, q)] = acc.o[j][2 * h + 1];
            } else {
                *(float2*)(o + column_of<DT>(j, 0, q)) = make_float2(acc.o[j][2 * h], acc.o[j][2 * h + 1]);
            }
        }
    }
}

// The factor that brings a partial with maximum m to maximum top.
__device__ __forceinline__ float rebase(float m, float top) { return m == -INFINITY ? 0.0f : exp2_fast(m - top); }

// The query tile as A fragments (rows = query heads, k = head dimension), in the order of k that
// the keys' fragments come in, and each row's score factor: scale * log2 e, for E4M3 caches times
// the power of two that the row was divided by to fit fp16.
template <int DT, int HD>
__device__ __forceinline__ void load_query(const Args& a, const Place& p, int lane, uint32_t (&qf)[HD / 16][4],
                                           float (&factor)[2]) {
    int head0, rows;
    tile_rows(a, p.tile, &head0, &rows);
    const int g = lane >> 2, q = lane & 3;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = g + 8 * h;
        const uint16_t* row = (const uint16_t*)a.q + (size_t)p.i * a.q_stride + (size_t)(head0 + r) * a.head_dim;
        factor[h] = a.scale * kLog2e;
        if constexpr (DT != AQ_E4M3) {
#pragma unroll
            for (int ks = 0; ks < HD / 16; ++ks)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int col = 16 * ks + 8 * x + 2 * q;
                    qf[ks][2 * x + h] = r < rows && col < a.head_dim ? *(const uint32_t*)(row + col) : 0u;
                }
        } else {
            uint2 w[HD / 16];
            float top = 0.0f;
#pragma unroll
            for (int ks = 0; ks < HD / 16; ++ks) {
                const int col = 16 * ks + 4 * q;
                w[ks] = r < rows && col < a.head_dim ? *(const uint2*)(row + col) : make_uint2(0, 0);
                float f[4];
                if (a.q_dt == AQ_F16) widen2<AQ_F16>(w[ks].x, f[0], f[1]), widen2<AQ_F16>(w[ks].y, f[2], f[3]);
                else widen2<AQ_BF16>(w[ks].x, f[0], f[1]), widen2<AQ_BF16>(w[ks].y, f[2], f[3]);
#pragma unroll
                for (int x = 0; x < 4; ++x) top = fmaxf(top, fabsf(f[x]));
            }
            top = quad_max(top);
            const int e = min(max(exponent_of(top) - 14, -126), 112);    // |q| 2^-e < 2^15
            const float down = pow2f(-e);
            factor[h] *= pow2f(e);
#pragma unroll
            for (int ks = 0; ks < HD / 16; ++ks) {
                float f[4];
                if (a.q_dt == AQ_F16) widen2<AQ_F16>(w[ks].x, f[0], f[1]), widen2<AQ_F16>(w[ks].y, f[2], f[3]);
                else widen2<AQ_BF16>(w[ks].x, f[0], f[1]), widen2<AQ_BF16>(w[ks].y, f[2], f[3]);
                qf[ks][h] = round_pack2<AQ_F16>(f[0] * down, f[1] * down);
                qf[ks][2 + h] = round_pack2<AQ_F16>(f[2] * down, f[3] * down);
            }
        }
    }
}

// Issues the copies of one chunk into a stage: the warp's lanes take 16-byte pieces, each of its
// token's page. cur/nxt hold 32 table entries each, one a lane, from entry 32 * block on.
template <int DT, int HD>
struct Loader {
    using T = Tile<DT, HD>;
    int cur, nxt, block;

    __device__ __forceinline__ int entry(const Args& a, const Place& p, int b, int lane) const {
        const long long e = (long long)b * 32 + lane;
        return e << a.page_log2 < p.len ? a.tables[(size_t)p.seq * a.max_pages + e] : -1;
    }
    __device__ __forceinline__ void begin(const Args& a, const Place& p, int lane) {
        block = (p.t >> a.page_log2) >> 5;
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
        constexpr int RPP = 32 / (T::PR < 32 ? T::PR : 32);      // rows per pass
        static_assert(T::PR <= 32, "a row is at most 32 pieces");
        const int piece = lane % T::PR, row0 = lane / T::PR;
        const bool real = piece * 16 < a.head_dim * T::ESZ;
        const size_t row_bytes = (size_t)a.head_dim * T::ESZ;
#pragma unroll
        for (int r0 = 0; r0 < T::CT; r0 += RPP) {
            const int r = r0 + row0, tok = p.t + r;
            const int page = __shfl_sync(~0u, cur, (tok >> a.page_log2) & 31);
            const bool in = tok < p.len;
            const bool ok = in && (unsigned)page < (unsigned)a.num_pages;
            if (in && !ok) record_status(a.status, AQ_ERR_INVALID_ARG);
            const size_t at = ok ? (((size_t)page * a.kv_heads + kvh) << a.page_log2) + (tok & mask) : 0;
            const size_t off = ok && real ? at * row_bytes + piece * 16 : 0;
            const uint32_t d = stage + swz<T::PR>(r, piece);
            cp16(d, a.k + off, ok && real);
            cp16(d + T::KV, a.v + off, ok && real);
        }
        if constexpr (DT == AQ_E4M3) {
            // scale bytes, four tokens (of one page) a lane: keys' at 2 KV, values' at 2 KV + 64
            const int r = (lane & 7) * 4, tok = p.t + r;
            const int page = __shfl_sync(~0u, cur, (tok >> a.page_log2) & 31);
            const bool ok = tok < p.len && (unsigned)page < (unsigned)a.num_pages;
            const size_t at = ok ? (((size_t)page * a.kv_heads + kvh) << a.page_log2) + (tok & mask) : 0;
            if (lane < 16 && r < T::CT) {
                const bool vals = lane >= 8;
                cp4(stage + 2 * T::KV + (vals ? 64 : 0) + r, (vals ? a.vs : a.ks) + at, ok);
            }
        }
    }
};

// One chunk: scores, running maximum and sum, output.
template <int DT, int HD>
__device__ __forceinline__ void compute(const Place& p, uint32_t stage, int lane, const uint32_t (&qf)[HD / 16][4],
                                        const float (&factor)[2], Acc<HD>& acc) {
    using T = Tile<DT, HD>;
    constexpr bool BF = DT == AQ_BF16;
    constexpr int NT = T::CT / 8;
    const int q = lane & 3;
    const int mi = lane >> 3, mr = lane & 7;       // this lane's matrix and row in an ldmatrix.x4
    float s[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.0f;
    if constexpr (DT != AQ_E4M3) {
#pragma unroll
        for (int ks = 0; ks < HD / 16; ++ks)
#pragma unroll
            for (int tt = 0; tt < NT / 2; ++tt) {
                uint32_t b[4];
                ldsm4(stage + swz<T::PR>(tt * 16 + (mi >> 1) * 8 + mr, 2 * ks + (mi & 1)), b);
                mma16816<BF>(s[2 * tt], qf[ks], b[0], b[1]);
                mma16816<BF>(s[2 * tt + 1], qf[ks], b[2], b[3]);
            }
    } else {
#pragma unroll
        for (int c = 0; c < HD / 16; c += 2)
#pragma unroll
            for (int tt = 0; tt < NT / 2; ++tt) {
                uint32_t b[4];
                ldsm4(stage + swz<T::PR>(tt * 16 + (mi & 1) * 8 + mr, c + (mi >> 1)), b);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    mma16816<false>(s[2 * tt], qf[c + x], widen_e4m3x2(b[2 * x]), widen_e4m3x2(b[2 * x] >> 16));
                    mma16816<false>(s[2 * tt + 1], qf[c + x], widen_e4m3x2(b[2 * x + 1]),
                                    widen_e4m3x2(b[2 * x + 1] >> 16));
                }
            }
    }
    // base-2 scores; masked ones are -inf
    const bool edge = p.t < p.lo || p.t + T::CT > p.len;
    float vexp[NT][2], vfac[NT][2];               // b and 2^b of the tokens' value scales
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float kf[2] = {1.0f, 1.0f};
        if constexpr (DT == AQ_E4M3) {
            uint16_t kb, wb;
            const uint32_t at = stage + 2 * T::KV + nt * 8 + 2 * q;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(kb) : "r"(at) : "memory");
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(wb) : "r"(at + 64) : "memory");
            kf[0] = __uint_as_float((uint32_t)(kb & 255) << 23);
            kf[1] = __uint_as_float((uint32_t)(kb >> 8) << 23);
            vexp[nt][0] = (float)((int)(wb & 255) - 127);
            vexp[nt][1] = (float)((int)(wb >> 8) - 127);
            vfac[nt][0] = __uint_as_float((uint32_t)(wb & 255) << 23);
            vfac[nt][1] = __uint_as_float((uint32_t)(wb >> 8) << 23);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int tok = p.t + nt * 8 + 2 * q + x;
            const bool out = edge && (tok < p.lo || tok >= p.len);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float v = s[nt][2 * h + x] * (DT == AQ_E4M3 ? factor[h] * kf[x] : factor[h]);
                s[nt][2 * h + x] = out ? -INFINITY : v;
            }
        }
    }
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                top[h] = fmaxf(top[h], DT == AQ_E4M3 ? s[nt][2 * h + x] + vexp[nt][x] : s[nt][2 * h + x]);
    float sub[2];
    bool moved = false;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        top[h] = fmaxf(quad_max(top[h]), acc.m[h]);
        moved |= top[h] > acc.m[h];
        sub[h] = top[h] == -INFINITY ? 0.0f : top[h];
    }
    if (__any_sync(~0u, moved)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float f = rebase(acc.m[h], sub[h]);
            acc.m[h] = top[h];
            acc.l[h] *= f;
#pragma unroll
            for (int j = 0; j < HD / 8; ++j) acc.o[j][2 * h] *= f, acc.o[j][2 * h + 1] *= f;
        }
    }
    // weights: p for the sum, p 2^b rounded to 16 bits for the product with V
    uint32_t w[NT][2];                              // [token tile][row half]
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float p0 = exp2_fast(s[nt][2 * h] - sub[h]), p1 = exp2_fast(s[nt][2 * h + 1] - sub[h]);
            acc.l[h] += p0 + p1;
            if constexpr (DT == AQ_E4M3) p0 *= vfac[nt][0], p1 *= vfac[nt][1];
            w[nt][h] = round_pack2<BF ? AQ_BF16 : AQ_F16>(p0, p1);
        }
    const uint32_t vt = stage + T::KV;
#pragma unroll
    for (int kt = 0; kt < NT / 2; ++kt) {
        const uint32_t a[4] = {w[2 * kt][0], w[2 * kt][1], w[2 * kt + 1][0], w[2 * kt + 1][1]};
        if constexpr (DT != AQ_E4M3) {
#pragma unroll
            for (int jp = 0; jp < HD / 16; ++jp) {
                uint32_t b[4];
                ldsm4t(vt + swz<T::PR>(kt * 16 + (mi & 1) * 8 + mr, 2 * jp + (mi >> 1)), b);
                mma16816<BF>(acc.o[2 * jp], a, b[0], b[1]);
                mma16816<BF>(acc.o[2 * jp + 1], a, b[2], b[3]);
            }
        } else {
#pragma unroll
            for (int c = 0; c < HD / 16; c += 2) {
                uint32_t b[4];
                ldsm4t(vt + swz<T::PR>(kt * 16 + (mi & 1) * 8 + mr, c + (mi >> 1)), b);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const uint32_t lo = b[2 * x], hi = b[2 * x + 1];   // tokens 2q, 2q+1; +8
                    mma16816<false>(acc.o[2 * (c + x)], a, widen_e4m3x2(prmt(lo, 0, 0x20)),
                                    widen_e4m3x2(prmt(hi, 0, 0x20)));
                    mma16816<false>(acc.o[2 * (c + x) + 1], a, widen_e4m3x2(prmt(lo, 0, 0x31)),
                                    widen_e4m3x2(prmt(hi, 0, 0x31)));
                }
            }
        }
    }
}

// Chunk offsets of the launch's n entries into base[0..n] (shared), their ranges and sequences;
// all threads. Each thread takes consecutive entries, so the sums stay in order.
template <int CT>
__device__ void scan_entries(const Args& a, int tiles, long long* base, int2* range, int* seq_of) {
    __shared__ long long warp_sum[kWarps];
    constexpr int PER = kSliceSeqs / kThreads;
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
            c[j] = (long long)chunks_of<CT>(len, lo) * tiles;
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

// Chunks each warp takes.
__device__ __forceinline__ long long share_of(long long total, int ctas) {
    const long long warps = (long long)ctas * kWarps;
    const long long per = (total + warps - 1) / warps;
    return per < 1 ? 1 : per;
}

template <int DT, int HD>
__global__ void __launch_bounds__(kThreads, (Tile<DT, HD>::CTAS)) kv_attend_kernel(Args a) {
    using T = Tile<DT, HD>;
    extern __shared__ __align__(1024) uint8_t ring[];
    __shared__ long long base[kSliceSeqs + 1];
    __shared__ int2 range[kSliceSeqs];
    __shared__ int seq_of[kSliceSeqs];
    __shared__ long long piece_seg[kWarps][2];     // the segments of a warp's first and last piece
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int tiles = a.kv_heads * a.tiles_per_head;
    pdl_wait();
    scan_entries<T::CT>(a, tiles, base, range, seq_of);
    pdl_launch_dependents();
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i <= a.n; i += kThreads) a.base[i] = base[i];
    // entries that see nothing
    for (int i = blockIdx.x; i < a.n; i += gridDim.x)
        if (range[i].x <= 0) {
            uint32_t* o = (uint32_t*)((uint16_t*)a.out + (size_t)i * a.q_heads * a.head_dim);
            for (int j = threadIdx.x; j < a.q_heads * a.head_dim / 2; j += kThreads) o[j] = 0u;
            if (a.lse)
                for (int j = threadIdx.x; j < a.q_heads; j += kThreads) a.lse[(size_t)i * a.q_heads + j] = -INFINITY;
        }
    const long long total = base[a.n], share = share_of(total, gridDim.x);
    const long long cta0 = min(total, share * kWarps * blockIdx.x), cta1 = min(total, cta0 + share * kWarps);
    const long long u0 = min(total, cta0 + share * warp), u1 = min(total, u0 + share);
    if (cta0 >= cta1) return;

    float* slots[2] = {a.first + (size_t)(blockIdx.x * kWarps + warp) * T::PART,
                       (float*)(ring + warp * T::RING)};
    if (lane == 0) piece_seg[warp][0] = piece_seg[warp][1] = -1;
    __syncwarp();
    if (u0 < u1) {
        const uint32_t stages = smem_u32(ring + warp * T::RING);
        Place in, at;
        place_at<T::CT>(a, base, range, seq_of, tiles, u0, in);
        at = in;
        Loader<DT, HD> loader;
        loader.begin(a, in, lane);
        const int count = (int)(u1 - u0);
        int issued = 0, fill = 0;
        auto issue = [&]() {
            if (issued < count) {
                loader.issue(a, in, stages + fill * T::STAGE, lane);
                if (++issued < count && advance<T::CT>(a, range, seq_of, tiles, in)) loader.begin(a, in, lane);
            }
            if (++fill == T::NS) fill = 0;
            cp_async_commit();
        };
        uint32_t qf[HD / 16][4];
        float factor[2];
        Acc<HD> acc;
        bool whole = at.t / T::CT == at.lo / T::CT;   // the segment begins in this warp's share
        load_query<DT, HD>(a, at, lane, qf, factor);
        acc.clear();
#pragma unroll 1
        for (int k = 0; k < T::NS - 1; ++k) issue();
        int use = 0;
#pragma unroll 1
        for (int k = 0; k < count; ++k) {
            issue();
            cp_async_wait<T::NS - 1>();
            __syncwarp();
            compute<DT, HD>(at, stages + use * T::STAGE, lane, qf, factor, acc);
            __syncwarp();
            if (++use == T::NS) use = 0;
            const bool last = k + 1 == count;
            if (at.left == 1 || last) {
                const long long seg = (long long)at.i * tiles + at.tile;
                if (whole && at.left == 1) {
                    write_final<DT, HD>(a, at, acc, lane);
                } else if (!last) {
                    write_partial<DT, HD>(a, at.tile, acc, slots[0], lane);
                    if (lane == 0) piece_seg[warp][0] = seg;
                } else {
                    cp_async_wait<0>();            // (nothing but empty groups is left)
                    __syncwarp();
                    write_partial<DT, HD>(a, at.tile, acc, slots[1], lane);
                    if (lane == 0) piece_seg[warp][1] = seg;
                }
                if (!last) {
                    advance<T::CT>(a, range, seq_of, tiles, at);
                    whole = true;
                    load_query<DT, HD>(a, at, lane, qf, factor);
                    acc.clear();
                }
            } else {
                at.t += T::CT;
                --at.left;
            }
        }
    }
    __syncthreads();

    // Pieces of the CTA's warps, in order; those of one segment are adjacent.
    const float* piece[2 * kWarps];
    long long seg[2 * kWarps];
    int pieces = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w)
#pragma unroll
        for (int x = 0; x < 2; ++x)
            if (piece_seg[w][x] >= 0) {
                seg[pieces] = piece_seg[w][x];
                piece[pieces++] = x == 0 ? a.first + (size_t)(blockIdx.x * kWarps + w) * T::PART
                                         : (const float*)(ring + w * T::RING);
            }
    for (int b = 0; b < pieces;) {
        int e = b + 1;
        while (e < pieces && seg[e] == seg[b]) ++e;
        const int i = (int)(seg[b] / tiles), tile = (int)(seg[b] - (long long)i * tiles);
        const long long per = chunks_of<T::CT>(range[i].x, range[i].y);
        const long long s0 = base[i] + per * tile, s1 = s0 + per;
        const bool done = s0 >= cta0 && s1 <= cta1;
        float* dst = a.part + ((size_t)blockIdx.x * 2 + (s0 < cta0 ? 0 : 1)) * T::PART;
        int head0, rows;
        tile_rows(a, tile, &head0, &rows);
        for (int x = threadIdx.x; x < rows * (HD / 4); x += kThreads) {
            const int r = x / (HD / 4), col = (x - r * (HD / 4)) * 4;
            float top = -INFINITY;
            for (int y = b; y < e; ++y) top = fmaxf(top, piece[y][r]);
            const float sub = top == -INFINITY ? 0.0f : top;
            float l = 0.0f;
            float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            for (int y = b; y < e; ++y) {
                const float f = rebase(piece[y][r], sub);
                const float4 v = *(const float4*)(piece[y] + 32 + r * HD + col);
                l += f * piece[y][16 + r];
                o.x += f * v.x, o.y += f * v.y, o.z += f * v.z, o.w += f * v.w;
            }
            if (done) {
                const size_t q_row = (size_t)i * a.q_heads + head0 + r;
                const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
                if (col < a.head_dim) {
                    store_out2(a, q_row, col, o.x * inv, o.y * inv);
                    store_out2(a, q_row, col + 2, o.z * inv, o.w * inv);
                }
                if (a.lse && col == 0) a.lse[q_row] = l == l ? lse_of(top, l) : l;
            } else {
                if (col == 0) dst[r] = top, dst[16 + r] = l;
                *(float4*)(dst + 32 + r * HD + col) = o;
            }
        }
        b = e;
    }
}

// Joins the segments that cross CTAs of the kernel above. CTA (j, y) takes the segment that
// crosses the end of CTA j's share and began in it, rows y, y + gridDim.y, ...; the partials are
// summed by groups of HD / 4 threads, in a fixed order.
template <int DT, int HD>
__global__ void __launch_bounds__(kThreads) kv_join_kernel(Args a, int ctas) {
    using T = Tile<DT, HD>;
    constexpr int LANES = HD / 4, GROUPS = kThreads / LANES;
    __shared__ float red_m[kWarps], red_l[GROUPS];
    __shared__ float4 red_o[GROUPS][LANES];
    pdl_wait();
    const int tiles = a.kv_heads * a.tiles_per_head;
    const long long total = a.base[a.n], share = share_of(total, ctas) * kWarps;
    const long long end = share * (blockIdx.x + 1);
    if (end >= total) return;
    int lo = 0, hi = a.n - 1;                      // the entry of chunk end - 1
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.base[mid] <= end - 1) lo = mid;
        else hi = mid - 1;
    }
    const long long b0 = a.base[lo], per = (a.base[lo + 1] - b0) / tiles;
    const int tile = (int)((end - 1 - b0) / per);
    const long long s0 = b0 + per * tile, s1 = s0 + per;
    if (s1 == end || s0 < end - share) return;     // not crossing, or begun before
    const int j0 = blockIdx.x, j1 = (int)((s1 - 1) / share);
    int head0, rows;
    tile_rows(a, tile, &head0, &rows);
    const int sub = threadIdx.x / LANES, col = threadIdx.x % LANES * 4;
    for (int r = blockIdx.y; r < rows; r += gridDim.y) {
        auto part = [&](int j) { return a.part + ((size_t)j * 2 + (j == j0 ? 1 : 0)) * T::PART; };
        float top = -INFINITY;
        for (int j = j0 + threadIdx.x; j <= j1; j += kThreads) top = fmaxf(top, part(j)[r]);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
        if ((threadIdx.x & 31) == 0) red_m[threadIdx.x >> 5] = top;
        __syncthreads();
        top = red_m[0];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) top = fmaxf(top, red_m[w]);
        const float ref = top == -INFINITY ? 0.0f : top;
        float l = 0.0f;
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
        for (int j = j0 + sub; j <= j1; j += GROUPS) {
            const float* p = part(j);
            const float f = rebase(p[r], ref);
            const float4 v = *(const float4*)(p + 32 + r * HD + col);
            l += f * p[16 + r];
            o.x += f * v.x, o.y += f * v.y, o.z += f * v.z, o.w += f * v.w;
        }
        red_o[sub][col / 4] = o;
        if (col == 0) red_l[sub] = l;
        __syncthreads();
        if (sub == 0) {
            for (int g = 1; g < GROUPS; ++g) {
                const float4 v = red_o[g][col / 4];
                l += red_l[g];
                o.x += v.x, o.y += v.y, o.z += v.z, o.w += v.w;
            }
            const size_t q_row = (size_t)lo * a.q_heads + head0 + r;
            const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
            if (col < a.head_dim) {
                store_out2(a, q_row, col, o.x * inv, o.y * inv);
                store_out2(a, q_row, col + 2, o.z * inv, o.w * inv);
            }
            if (a.lse && col == 0) a.lse[q_row] = l == l ? lse_of(top, l) : l;
        }
        __syncthreads();
    }
}

// The workspace is sized for the largest grid, so that the query needs no device.
constexpr int kMaxSms = 160;

template <int DT, int HD>
size_t attend_ws() {
    return kWsStatusBytes + round_up((kSliceSeqs + 1) * 8, 256) +
           (size_t)kMaxSms * Tile<DT, HD>::CTAS * (2 + kWarps) * Tile<DT, HD>::PART * 4;
}

template <int DT, int HD>
aq_status attend(Args a, const DeviceInfo& di, int n, cudaStream_t st) {
    using T = Tile<DT, HD>;
    static std::atomic<bool> have[64];             // (setting the attribute twice is harmless)
    int dev = 0;
    if (cudaError_t e = cudaGetDevice(&dev); e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
    if (!have[dev & 63]) {
        if (cudaError_t e = cudaFuncSetAttribute(kv_attend_kernel<DT, HD>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 T::SMEM);
            e != cudaSuccess)
            return cuda_fail(e, "cudaFuncSetAttribute");
        have[dev & 63] = true;
    }
    const int ctas = (di.sms < kMaxSms ? di.sms : kMaxSms) * T::CTAS;
    char* ws = (char*)a.status;
    a.base = (long long*)(ws + kWsStatusBytes);
    a.part = (float*)(ws + kWsStatusBytes + round_up((kSliceSeqs + 1) * 8, 256));
    a.first = a.part + (size_t)ctas * 2 * T::PART;
    const int tiles = a.kv_heads * a.tiles_per_head, rows = a.group < 16 ? a.group : 16;
    for (int i0 = 0; i0 < n; i0 += kSliceSeqs) {
        Args s = a;
        s.n = n - i0 < kSliceSeqs ? n - i0 : kSliceSeqs;
        if (s.seqs) s.seqs += i0;
        else s.lens += i0, s.tables += (size_t)i0 * a.max_pages, s.max_seqs -= i0;
        s.q = (const uint16_t*)a.q + (size_t)i0 * a.q_stride;
        s.out = (uint16_t*)a.out + (size_t)i0 * a.q_heads * a.head_dim;
        if (s.lse) s.lse += (size_t)i0 * a.q_heads;
        if (aq_status e = launch_dependent(kv_attend_kernel<DT, HD>, ctas, kThreads, T::SMEM, st, s); e != AQ_OK)
            return e;
        // With few segments each is cut into many partials, and its rows get a CTA each.
        const dim3 grid(ctas - 1, (long long)s.n * tiles < ctas ? rows : 1);
        if (aq_status e = launch_dependent(kv_join_kernel<DT, HD>, grid, kThreads, 0, st, s, ctas); e != AQ_OK) return e;
    }
    return AQ_OK;
}

// Calls f<DT, HD>() for the cache's type and padded head dimension.
#define AQ_KV_DISPATCH(dtype, dim, f, ...)                                            \
    (dim) <= 64    ? ((dtype) == AQ_F16    ? f<AQ_F16, 64>(__VA_ARGS__)               \
                      : (dtype) == AQ_BF16 ? f<AQ_BF16, 64>(__VA_ARGS__)              \
                                           : f<AQ_E4M3, 64>(__VA_ARGS__))             \
    : (dim) <= 128 ? ((dtype) == AQ_F16    ? f<AQ_F16, 128>(__VA_ARGS__)              \
                      : (dtype) == AQ_BF16 ? f<AQ_BF16, 128>(__VA_ARGS__)             \
                                           : f<AQ_E4M3, 128>(__VA_ARGS__))            \
                   : ((dtype) == AQ_F16    ? f<AQ_F16, 256>(__VA_ARGS__)              \
                      : (dtype) == AQ_BF16 ? f<AQ_BF16, 256>(__VA_ARGS__)             \
                                           : f<AQ_E4M3, 256>(__VA_ARGS__))

}  // namespace

size_t kv_attend_ws_bytes(const aq_kv_cache& c) {
    return AQ_KV_DISPATCH(c.dtype, c.head_dim, attend_ws);
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
    a.q_heads = q_heads, a.kv_heads = c.kv_heads, a.group = q_heads / c.kv_heads;
    a.tiles_per_head = (a.group + 15) / 16;
    a.head_dim = c.head_dim;
    while ((1 << a.page_log2) < c.page_tokens) ++a.page_log2;
    a.num_pages = c.num_pages, a.max_seqs = c.max_seqs, a.max_pages = c.max_pages, a.window = window;
    return AQ_KV_DISPATCH(c.dtype, c.head_dim, attend, a, di, n, st);
}

}  // namespace aq
