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
};

// One sequence of a call, clamped to what the table row, T and the rows hold.
struct Seq {
    int len;                    // tokens in the cache
    int start;                  // position of the chunk's first token
    int n;                      // new tokens
    int first;                  // row of the first of them
};
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

}  // namespace chunk
}  // namespace isv
