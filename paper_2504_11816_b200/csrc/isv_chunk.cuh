// Parameter blocks and device helpers shared by the kernels on chunks of new tokens (isv_chunk_*).  Plain pointers and
// sizes; nothing here owns memory.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/isv.h"

namespace isv {
namespace chunk {

constexpr int kBT = 16;   // tokens of a page

// The cache, the sequences of a call and the rows that hold their new tokens.
struct CacheParams {
    uint16_t *pool;             // [n_pages][K|V][Hkv][16][D]
    const int32_t *table;       // [n_seqs][table_stride]
    const int32_t *lens;        // tokens of a sequence, the new ones included
    const int32_t *news;        // new tokens, or NULL: T of every sequence
    const int32_t *firsts;      // row of a sequence's first new token, or NULL: s * T
    uint32_t *status;
    int32_t table_stride, max_blocks, n_pages, n_seqs, n_rows, T, Hkv, Hq;
};

struct MergeRec;

struct AttnParams {
    CacheParams c;
    const uint16_t *q;          // [n_rows] rows of q_stride elements: [Hq][D]
    int64_t q_stride;
    const float *slopes;        // [Hq] or NULL
    const int32_t *prefixes;    // [n_seqs] or NULL
    uint16_t *out;              // [n_rows][Hq][D] or NULL
    float *out_f32;             // the same in fp32, or NULL
    int32_t window;             // 0: no limit
    float scale;                // of the scores
    float cap;                  // 0: scores are not capped
    // how the work is cut, and scratch
    int32_t GT, P;              // a visit serves GT of a KV head's query heads; P passes serve all of them
    int32_t tile_rows;          // rows of an item, as attn_tile_rows says
    int32_t TT, RT;             // tokens of a tile of (at most) 128 rows; items that a chunk of T tokens has at most, per KV head and pass
    float *part_o;              // partial results: [slot][D / 4][rows of an item] of four values, two slots a CTA
    float *part_ml;             // [slot][rows of an item] of (reference, sum)
    MergeRec *merges;           // [grid]: the item that begins in this CTA's range and ends in another's
    uint32_t spin_limit;        // polls of a barrier before a wait gives up
    int32_t drop_first_copy;    // failure injection: the first item's first barrier is armed without issuing one of its copies
};

// One sequence of a call, clamped to what the table row, T and the rows hold.
struct Seq {
    int len;                    // tokens in the cache
    int start;                  // position of the chunk's first token
    int n;                      // new tokens
    int first;                  // row of the first of them
};

// An item whose partial results are in slot 2 * first + 1 and in 2 * c for the CTAs c up to `last`.
struct MergeRec {
    int32_t n;                  // partial results, 0: none
    int32_t last, s, token0, kvh, pass;
    Seq q;
};

// Rows of an item for that many rows per KV head: a quarter, a half or the whole of a tile of 128, or two tiles.
inline int attn_tile_rows(long long rows) { return rows <= 32 ? 32 : rows <= 64 ? 64 : rows <= 128 ? 128 : 256; }
// Rows of partial results: two items of 256 rows a CTA.
inline size_t attn_part_rows(int grid) { return (size_t)2 * grid * 256; }
template <int D>
cudaError_t attn_configure(bool bf16);
template <int D>
cudaError_t launch_attn(const AttnParams &p, bool bf16, int grid, cudaStream_t st, const char **what);

__device__ __forceinline__ Seq seq_of(const CacheParams &c, int s, bool &bad) {
    Seq q;
    const int n = c.lens[s], most = c.max_blocks * kBT;
    q.len = min(max(n, 0), most);
    const int w = c.news ? c.news[s] : c.T;
    q.n = min(max(w, 0), min(c.T, q.len));
    q.start = q.len - q.n;
    const long long f = c.firsts ? (long long)c.firsts[s] : (long long)s * c.T;
    const int room = f < 0 || f >= c.n_rows ? 0 : c.n_rows - (int)f;
    q.first = room ? (int)f : 0;
    bad = n != q.len || w != q.n || q.n > room;
    q.n = min(q.n, room);
    return q;
}

// What a query at position p may look at: positions j < lim that are not below `low`, or are below `prefix`.
struct Sight {
    int lim, low, prefix;
    __device__ __forceinline__ bool sees(int j) const { return j < lim && (j >= low || j < prefix); }
};
__device__ __forceinline__ Sight sight_of(const AttnParams &a, int s, const Seq &q, int p) {
    Sight v;
    v.prefix = a.prefixes ? min(max(a.prefixes[s], 0), q.len) : 0;
    v.lim = min(q.len, max(p + 1, v.prefix));
    v.low = a.window > 0 ? max(0, p + 1 - a.window) : 0;
    return v;
}

// Where 16-byte chunk c of token t of a page stands in its row.
template <int D>
__device__ __forceinline__ int place(int c, int t) {
    return c < D / 64 * 8 ? c ^ (t & 7) : c;
}

template <bool BF16>
__device__ __forceinline__ float2 widen(uint32_t w) {
    if (BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}
// Two numbers rounded to 16 bits, the first in the low half.
template <bool BF16>
__device__ __forceinline__ uint32_t narrow(float lo, float hi) {
    if (BF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// A warp per (new token, query head): lanes take the 32 tokens of two pages for the scores, and pairs of dims for the
// sums, which are kept in 64 bits.
template <int D, bool BF16>
__device__ __noinline__ void attend_row(const AttnParams &a, int s, const Seq &q, int t, int h) {
    constexpr int J = (D / 2 + 31) / 32;
    const int lane = threadIdx.x & 31, kvh = h / (a.c.Hq / a.c.Hkv);
    const int p = q.start + t;
    const long long row = q.first + t;
    const Sight v = sight_of(a, s, q, p);
    const uint4 *qrow = reinterpret_cast<const uint4 *>(a.q + row * a.q_stride + h * D);
    const float slope = a.slopes ? a.slopes[h] : 0.f;
    float m = -INFINITY;
    double l = 0, o[J][2] = {};
    for (int j0 = (v.prefix ? 0 : v.low) / kBT * kBT; j0 < v.lim; j0 += 32) {
        const int j = j0 + lane, slot = j % kBT;
        int page = -1;
        if (j < v.lim) {
            page = a.c.table[(long long)s * a.c.table_stride + j / kBT];
            if (page != ISV_BLOCK_NONE && (page < 0 || page >= a.c.n_pages)) {
                atomicOr(a.c.status, ISV_STATUS_BAD_BLOCK_ID);
                page = -1;
            }
        }
        const bool seen = page >= 0 && v.sees(j);
        float x = -INFINITY;
        if (seen) {
            const uint4 *krow = reinterpret_cast<const uint4 *>(a.c.pool + (((long long)page * 2 * a.c.Hkv + kvh) * kBT + slot) * D);
            x = 0.f;
            for (int c = 0; c < D / 8; ++c) {
                const uint4 kw = krow[place<D>(c, slot)], qw = qrow[c];
                const uint32_t *kk = reinterpret_cast<const uint32_t *>(&kw), *qq = reinterpret_cast<const uint32_t *>(&qw);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 e = widen<BF16>(kk[i]), f = widen<BF16>(qq[i]);
                    x = fmaf(e.x, f.x, x);
                    x = fmaf(e.y, f.y, x);
                }
            }
            x *= a.scale;
            if (a.cap > 0.f) x = a.cap * tanhf(x / a.cap);
            x -= slope * fabsf((float)(p - j));
        }
        float top = x;
        for (int i = 16; i; i >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, i));
        unsigned left = __ballot_sync(~0u, seen);
        const float before = m;
        m = fmaxf(m, top);
        const double keep = before == -INFINITY ? 0.0 : (double)expf(before - m);
        const float e = seen ? expf(x - m) : 0.f;
        l *= keep;
#pragma unroll
        for (int i = 0; i < J; ++i) { o[i][0] *= keep; o[i][1] *= keep; }
        for (; left; left &= left - 1) {
            const int y = __ffs(left) - 1, pg = __shfl_sync(~0u, page, y), sl = (j0 + y) % kBT;
            const double w = (double)__shfl_sync(~0u, e, y);
            l += w;
            const uint32_t *vrow = reinterpret_cast<const uint32_t *>(a.c.pool + ((((long long)pg * 2 + 1) * a.c.Hkv + kvh) * kBT + sl) * D);
#pragma unroll
            for (int i = 0; i < J; ++i) {
                const int x2 = lane + 32 * i;
                if (x2 >= D / 2) continue;
                const float2 z = widen<BF16>(vrow[place<D>(x2 / 4, sl) * 4 + x2 % 4]);
                o[i][0] += w * z.x;
                o[i][1] += w * z.y;
            }
        }
    }
    const double inv = l != 0 ? 1.0 / l : 0.0;
#pragma unroll
    for (int i = 0; i < J; ++i) {
        const int x2 = lane + 32 * i;
        if (x2 >= D / 2) continue;
        const float e = l != 0 ? (float)(o[i][0] * inv) : 0.f, f = l != 0 ? (float)(o[i][1] * inv) : 0.f;
        const long long at = (row * a.c.Hq + h) * (D / 2) + x2;
        if (a.out) reinterpret_cast<uint32_t *>(a.out)[at] = narrow<BF16>(e, f);
        if (a.out_f32) reinterpret_cast<float2 *>(a.out_f32)[at] = make_float2(e, f);
    }
}

}  // namespace chunk
}  // namespace isv
