// Attention of chunks of new tokens over the paged cache (isv_chunk_attn, described in include/isv.h), on tcgen05.  Included by one
// source file per head_dim.
//
// Mathematics: per KV head the rows are the chunk's (token, query head) pairs, S = Q K^T and O = P V with P = 2^(S' - r) for the
// scaled, capped, biased and masked scores S' (base 2) and a row's running reference r; a row's sum l of P is kept in fp32, its
// O in tensor memory, and O / l is the result.  r follows the row's maximum only when that has passed it by 8 (fp16)
// or 40 (bf16), then O and l are scaled down once: the quotient does not depend on r.  fp16 weights are 2^7 times as large, so
// that they stay below 2^16 and down to 2^-21 of the largest are normal numbers.
//
// Work: an item is (sequence, NT tiles of 128 rows, KV head); its visits are the tiles of 128 tokens that some row of it sees.  All
// visits of all items form one list that is cut into equal ranges, one per persistent CTA, whatever the lengths; an item that
// crosses ranges leaves partial results, which a second small kernel merges in fixed order.
//
// A CTA: a producer warp copies the pages of K and V into a ring of tiles by TMA; one thread issues the products; NT groups of four
// warps turn scores into weights, one row per thread.  With NT = 2 the groups take turns with the tensor cores: while one
// computes its weights, the other's products run.  With NT = 1 the scores of the next visit are computed meanwhile.  Where a KV
// head has no more than 64 or 32 rows, the tile holds R = 2 or 4 copies of them, each for its share of a visit's columns (a warp
// reaches only its own quarter of tensor memory's lanes), and the weights meet as an operand in shared memory.
//
// Layout: the pool's rows hold their 16-byte chunks in the order that the 128-byte swizzle of tensor-core operands wants
// (chunk c of token t at c XOR t mod 8), so a page's 64-element half rows are copied by an unswizzled box of {64, 16} each and
// are operands as they land: K as the K-major B operand of Q K^T, V as the MN-major one of P V.  The last 16 elements of
// head_dim 80 are a box of their own with the 32-byte swizzle.  P goes back into the scores' columns of tensor memory as 16-bit
// numbers, the A operand of P V.
//
// Every wait is bounded (while a warp computes rows token by token, which ends, the count stops); on expiry the kernel flags the
// status word, waits for its copies (bounded), frees its tensor memory and returns.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cfloat>
#include <climits>

#include "isv_chunk.cuh"

namespace isv {
namespace chunk {

namespace {

constexpr int kTile = 128;             // rows of a tile, tokens of a visit
constexpr int kPages = kTile / kBT;
constexpr int kRecs = 8;               // visit records in flight (a ring of at most 10 tiles is less than 6 visits ahead of the products)
// Of 16 powers of two, those that are taken by a polynomial where weights are rounded to 16 bits and scores come as they are: the
// special-function unit does 4 a cycle and quarter of an SM.  A prompt of 8192 tokens, when this was
// settled: 0 625 us, 3 593, 5 594.
constexpr int kPoly = 3;
constexpr float kLog2e = 1.4426950408889634f;
// How far a row's maximum may pass its reference before the reference follows (and O is scaled): fp16 weights have to stay below 2^16;
// bf16's are as exact at 2^40 as at 1, and fp32 sums of 2^40 times values up to 2^70 do not overflow.  With heavy-tailed
// scores some row of a warp passes 2^8 in every second visit.
template <bool BF16>
__host__ __device__ constexpr float slack_of() { return BF16 ? 40.f : 8.f; }

__device__ __forceinline__ uint32_t s32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok)
                 : "r"(bar), "r"(parity)
                 : "memory");
    return ok;
}
// Whether the barrier's phase completed before the limit, and before another warp gave up (state below 0).  While warps compute rows
// token by token (their number above 0), which ends but may take long, a wait is not counted.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, uint32_t limit, const volatile int *state) {
    if (bar_try(bar, parity)) return true;
    for (uint32_t i = 0; i < limit; ++i) {
        if (bar_try(bar, parity)) return true;
        if ((i & 63) == 63) {
            const int now = *state;
            if (now < 0) return false;
            if (now > 0) i = 0;
        }
    }
    return false;
}

// A value that all lanes have alike, told to the compiler so: what is computed from it, and the branches on it, are the warp's.
__device__ __forceinline__ int same(int x) { return __shfl_sync(~0u, x, 0); }

__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}

// Shared-memory matrix descriptors.  K-major operands: 8-row groups are `stride` bytes apart.  MN-major: blocks of a swizzle
// row's elements are `lead` bytes apart, groups of 8 along K `stride` bytes.
__device__ __forceinline__ uint64_t desc(uint32_t addr, uint32_t lead, uint32_t stride, uint64_t layout) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(stride >> 4) << 32 | 1ull << 46 | layout << 61;
}
constexpr uint64_t kSwz128 = 2, kSwz32 = 6;

__host__ __device__ constexpr uint32_t instr_desc(bool bf16, bool b_mn_major, int n) {
    return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) |
           ((uint32_t)(kTile >> 4) << 24);
}
// The issuing warp runs these as a whole, so that operands stay in uniform registers, and each elects the thread that issues (a
// predicate of the lane's number instead costs 40 cycles an instruction: 64 users' drafts 156 us instead of 141, single tokens 118
// instead of 93).
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p, q;\nsetp.ne.b32 p, %4, 0;\nelect.sync _|q, 0xffffffff;\n@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p, q;\nsetp.ne.b32 p, %4, 0;\nelect.sync _|q, 0xffffffff;\n@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(
            d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile(
        "{\n.reg .pred q;\nelect.sync _|q, 0xffffffff;\n@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(bar)
        : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

__device__ __forceinline__ void tmem_ld32(uint32_t a, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
        "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
          "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]),
          "=r"(r[30]), "=r"(r[31])
        : "r"(a)
        : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t a, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(a)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t a, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(a),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t a, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
        "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(a),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
        "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// NaN if one of them is
__device__ __forceinline__ float max3(float x, float y, float z) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
    return r;
}
__device__ __forceinline__ float reciprocal(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint64_t pair(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ float2 unpair(uint64_t v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t both(float x) { return pair(x, x); }

// 2^x of two numbers without the special-function unit: x = n + f with |f| <= 1/2, a polynomial for 2^f whose constant is 1 (least
// largest relative error on that range, fitted: degree 3 1.0e-4, degree 4 2.8e-6), n added to its exponent.  For weights that are
// rounded to 16 bits next (2^-9 and 2^-12 of themselves).  -infinity gives 0; x is not above 127, and no NaN.
template <int DEGREE>
__device__ __forceinline__ float2 exp2_poly(uint64_t x) {
    const uint64_t magic = both(12582912.f);             // 1.5 * 2^23: a sum with it has the rounded x in its low bits
    const float2 v = unpair(x);
    x = pair(fmaxf(v.x, -127.f), fmaxf(v.y, -127.f));
    const uint64_t t = add2(x, magic);
    const uint64_t f = fma2(add2(t, both(-12582912.f)), both(-1.f), x);
    uint64_t y;
    if (DEGREE == 3) {
        y = fma2(both(0.05500892922282219f), f, both(0.24221095442771912f));
        y = fma2(y, f, both(0.6932829022407532f));
    } else {
        y = fma2(both(0.009582852944731712f), f, both(0.055906426161527634f));
        y = fma2(y, f, both(0.24024099111557007f));
        y = fma2(y, f, both(0.6931241750717163f));
    }
    y = fma2(y, f, both(1.f));
    const float2 z = unpair(y), n = unpair(t);
    return make_float2(__int_as_float(__float_as_int(z.x) + (__float_as_int(n.x) << 23)), __int_as_float(__float_as_int(z.y) + (__float_as_int(n.y) << 23)));
}
// tanh for |x| <= 1: an odd polynomial of degree 13 (least largest error, fitted: 2.0e-8)
__device__ __forceinline__ uint64_t tanh_poly(uint64_t x) {
    const uint64_t z = mul2(x, x);
    uint64_t y = fma2(both(0.0009637724724598229f), z, both(-0.005951281636953354f));
    y = fma2(y, z, both(0.019973283633589745f));
    y = fma2(y, z, both(-0.05326583608984947f));
    y = fma2(y, z, both(0.13319583237171173f));
    y = fma2(y, z, both(-0.33332130312919617f));
    y = fma2(y, z, both(0.9999997019767761f));
    return mul2(y, x);
}

// ---------------------------------------------------------------- how the work is cut

// `total` positions over n CTAs, the first `total mod n` of which get one more.
struct Cut {
    long long each, more;       // more: CTAs with each + 1
    __device__ Cut(long long total, int n) {
        // 64-bit division is a long way; nearly every total fits in 32
        if (total >> 31) each = total / n;
        else each = (int)total / n;
        more = total - each * n;
    }
    __device__ long long first(int c) const { return c * each + min((long long)c, more); }
    __device__ int cta_of(long long x) const {
        const long long border = more * (each + 1);
        if (x < border) return x >> 31 ? (int)(x / (each + 1)) : (int)x / (int)(each + 1);
        const long long y = x - border;
        return (int)more + (y >> 31 || each >> 31 ? (int)(y / each) : (int)y / (int)each);
    }
};

struct Item {
    int s, token0, kvh, pass;   // first token of the chunk in it
    int lo, hi;                 // its visits: tiles lo .. hi - 1 of 128 tokens
};
__device__ __forceinline__ void span_of(const AttnParams &a, int s, const Seq &q, int token0, int tokens, int &lo, int &hi) {
    const int last = min(token0 + tokens, q.n) - 1;
    const Sight first = sight_of(a, s, q, q.start + token0);
    lo = first.prefix > 0 ? 0 : first.low / kTile;
    hi = (min(q.len, max(q.start + last + 1, first.prefix)) + kTile - 1) / kTile;
}

// A visit's record, written by the producer for the warps that work on it.
struct Visit {
    int j0;                     // first token
    int pages;                  // bit i: page i is there
    int flags;
    int partial;                // tokens of the last page, 0: all 16
    int last_page;              // the page that is partial
    int s, token0, kvh, pass;
    int slot;                   // of the partial result, -1: the item is whole
    Seq q;
};
enum { FIRST = 1, LAST = 2, TWO = 4, END = 8 };

template <int D>
struct Shape {
    static constexpr int HALVES = D / 64, TAIL = D % 64;                          // of a row: 64 elements each, and the rest
    static constexpr int HALF_BYTES = kTile * 128, TAIL_BYTES = kTile * TAIL * 2;
    static constexpr int TILE = HALVES * HALF_BYTES + TAIL_BYTES;                 // a tile of Q, K or V
    // tiles of the ring: what fits beside two tiles of Q, or (R > 1) one and the weights
    static __host__ __device__ constexpr int slots(int R) { return D == 128 ? 5 : D == 80 ? (R > 1 ? 8 : 9) : 10; }
};
constexpr int kMisc = 1024;
constexpr int kWeights = 2 * 64 * 256;     // R > 1: weights of up to 64 rows as two 16-bit numbers each
constexpr int kExchange = 2 * kTile * 4;   // R > 1: maxima and sums that the copies of a row exchange
template <int D>
constexpr size_t smem_bytes(int R) {
    return 1024 + (size_t)((R > 1 ? 1 : 2) + Shape<D>::slots(R)) * Shape<D>::TILE + kMisc + (R > 1 ? kWeights + kExchange : 0);
}

// warps: NT groups of four for the weights, then the producer, the issuer of products, the loader of Q, and one that rests
template <int NT>
__host__ __device__ constexpr int threads_of() { return NT * 128 + 128; }
template <int D, bool BF16, int NT, int R, bool FINE, bool SHAPED>
__global__ void __launch_bounds__(threads_of<NT>(), 1)
attn_kernel(const __grid_constant__ CUtensorMap map_kv, const __grid_constant__ CUtensorMap map_kv_tail,
            const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_q_tail, const __grid_constant__ AttnParams a) {
    using SH = Shape<D>;
    constexpr int SLOTS = SH::slots(R), NTHREADS = threads_of<NT>(), NWARPS = NTHREADS / 32;
    constexpr int kProducer = NT * 4, kIssuer = NT * 4 + 1, kLoader = NT * 4 + 2;
    constexpr float kOffset = BF16 ? 0.f : 7.f;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (s32(smem_raw) & 1023u)) & 1023u);
    // the weights come first: what their operand's unused rows read is still shared memory of this CTA
    uint8_t *weights = smem, *q_tiles = smem + (R > 1 ? kWeights : 0), *ring = q_tiles + (R > 1 ? 1 : 2) * SH::TILE;
    uint8_t *misc = ring + SLOTS * SH::TILE;
    float *exchange = reinterpret_cast<float *>(misc + kMisc);      // [2][copy of the rows][row]
    Visit *recs = reinterpret_cast<Visit *>(misc);
    uint64_t *bars = reinterpret_cast<uint64_t *>(misc + kRecs * sizeof(Visit));
    uint64_t *full = bars, *empty = full + SLOTS, *rec_full = empty + SLOTS, *rec_read = rec_full + kRecs, *q_full = rec_read + kRecs, *q_empty = q_full + 2;
    uint64_t *s_full = q_empty + 2, *p_full = s_full + 2, *pv_done = p_full + 4, *drain = pv_done + 2, *x_full = drain + 1;   // p_full: [half of the tokens][2]
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(x_full + 1);
    int *state = reinterpret_cast<int *>(tmem_slot + 1);      // below 0: a wait ran out; above: warps that others wait for, however long
    static_assert(kRecs * sizeof(Visit) + (2 * SLOTS + 2 * kRecs + 14) * 8 + 8 <= kMisc, "");
    long long *sums = reinterpret_cast<long long *>(ring + (SLOTS - 1) * SH::TILE);   // until the first copies
    const int warp = same(threadIdx.x >> 5), lane = threadIdx.x & 31;
    auto give_up = [&]() { atomicOr(state, INT_MIN); };
    auto gave_up = [&]() { return *reinterpret_cast<const volatile int *>(state) < 0; };
    // Tiles in the order in which they are consumed.  NT = 2: K and V of a visit in turn.  NT = 1: the next visit's K before this one's V
    // (K0 K1 V0 K2 V1 ..), so that V does not wait in the ring for its weights.
    auto k_index = [](int v) -> uint32_t { return NT == 2 ? 2 * v : v == 0 ? 0 : 2 * v - 1; };
    auto v_index = [](int v) -> uint32_t { return NT == 2 ? 2 * v + 1 : 2 * v + 2; };

    if (threadIdx.x == 0) {
        for (int i = 0; i < SLOTS; ++i) {
            bar_init(s32(&full[i]), 1);
            bar_init(s32(&empty[i]), 1);
        }
        for (int i = 0; i < kRecs; ++i) {
            bar_init(s32(&rec_full[i]), 1);
            bar_init(s32(&rec_read[i]), NT == 2 ? 5 : 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(s32(&q_full[i]), 1);
            bar_init(s32(&q_empty[i]), 1);
            bar_init(s32(&s_full[i]), 1);
            bar_init(s32(&p_full[i]), 4);
            bar_init(s32(&p_full[2 + i]), 4);
            bar_init(s32(&pv_done[i]), 1);
        }
        bar_init(s32(drain), 1);
        bar_init(s32(x_full), 4);
        *state = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == kIssuer) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(s32(tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (warp == kProducer && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_kv) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
        if (SH::TAIL) {
            asm volatile("prefetch.tensormap [%0];" ::"l"(&map_kv_tail) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q_tail) : "memory");
        }
    }
    // nothing in global memory is touched before what was launched ahead is complete; then the kernel behind may enter
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---- the list of visits: a unit is (sequence, row tiles), each thread sums a run of units; an item counts one visit more
    // for what it costs by itself
    const int units = a.c.n_seqs * a.RT, group = a.c.Hkv * a.P;
    const int u_lo = (int)((long long)units * threadIdx.x / NTHREADS), u_hi = (int)((long long)units * (threadIdx.x + 1) / NTHREADS);
    auto weight = [&](int u, Seq &q, int &lo, int &hi) {   // of an item of unit u, 0: there is none
        const int s = u / a.RT, token0 = (u - s * a.RT) * NT * a.TT;
        bool bad;
        q = seq_of(a.c, s, bad);
        if (bad && token0 == 0 && blockIdx.x == 0) atomicOr(a.c.status, ISV_STATUS_BAD_LENGTH);
        if (token0 >= q.n) return 0;
        span_of(a, s, q, token0, NT * a.TT, lo, hi);
        return hi - lo + 1;
    };
    long long mine = 0;
    for (int u = u_lo; u < u_hi; ++u) {
        Seq q;
        int lo, hi;
        mine += weight(u, q, lo, hi);
    }
    mine *= group;
    long long up = mine;
#pragma unroll
    for (int i = 1; i < 32; i *= 2) {
        const long long z = __shfl_up_sync(~0u, up, i);
        if (lane >= i) up += z;
    }
    if (lane == 31) sums[NTHREADS + warp] = up;
    __syncthreads();
    long long base = 0, total = 0;
    for (int i = 0; i < NWARPS; ++i) {
        if (i < warp) base += sums[NTHREADS + i];
        total += sums[NTHREADS + i];
    }
    sums[threadIdx.x] = base + up - mine;
    fence_before();
    __syncthreads();
    fence_after();
    const int n_ctas = (int)min((long long)gridDim.x, total);
    const int cta = blockIdx.x;

    if (warp == kProducer) {
        // ---- walks the CTA's range, writes visit records, copies pages
        const Cut cut(total, max(n_ctas, 1));
        const long long f0 = cta < n_ctas ? cut.first(cta) : 0, f1 = cta < n_ctas ? cut.first(cta + 1) : 0;
        MergeRec rec{};
        int v = 0;              // visits so far
        uint32_t top = 0;       // tiles so far
        bool ok = true;
        int before_id = 0, before_kvh = 0;
        uint32_t before_pages = 0;
        auto slot_free = [&](uint32_t n) {
            ok = __all_sync(~0u, n < SLOTS || bar_wait(s32(&empty[n % SLOTS]), (n / SLOTS - 1) & 1, a.spin_limit, state));
        };
        // copies the pages of K (kv = 0) or V of a visit as tile n: a lane per copy (one lane for all takes twice as long)
        auto fetch = [&](uint32_t n, int kv, int id, uint32_t pages, int kvh, bool drop) {
            const uint32_t dst = s32(ring + (size_t)(n % SLOTS) * SH::TILE), bar = s32(&full[n % SLOTS]);
            if (lane == 0) bar_expect(bar, __popc(pages) * (SH::TILE / kPages));
            __syncwarp();
            const int page = lane & 7, piece = lane >> 3;     // piece: a half, or the tail
            const int trow = ((id * 2 + kv) * a.c.Hkv + kvh) * kBT;
            if ((pages >> page & 1) && !(drop && page == 0)) {
                if (piece < SH::HALVES) tma_2d(dst + piece * SH::HALF_BYTES + page * (kBT * 128), &map_kv, 64 * piece, trow, bar);
                else if (SH::TAIL && piece == SH::HALVES)
                    tma_2d(dst + SH::HALVES * SH::HALF_BYTES + page * (kBT * SH::TAIL * 2), &map_kv_tail, 64 * SH::HALVES, trow, bar);
            }
            top = n + 1;
        };
        // Record v may be written: the one before it in its place is read.  A visit whose tiles are used up has been read by those
        // who work on it; these may lag behind the ring: the loader, which only works at an item's begin, and the second group of
        // warps, which passes over items of one row tile.
        auto rec_free = [&]() {
            ok = ok && __all_sync(~0u, v < kRecs || bar_wait(s32(&rec_read[v % kRecs]), (v / kRecs - 1) & 1, a.spin_limit, state));
        };
        auto put_end = [&]() {
            rec_free();
            if (ok && lane == 0) {
                recs[v % kRecs].flags = END;
                bar_arrive(s32(&rec_full[v % kRecs]));
            }
        };
        if (f0 < f1) {
            // the run that holds f0: the last one that begins at or before it and is not empty
            int r = 0;
            for (int i = lane; i < NTHREADS; i += 32)
                if (sums[i] <= f0) r = max(r, i);
            r = __reduce_max_sync(~0u, r);
            long long at = sums[r];
            __syncwarp();
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // `sums` is read; copies may overwrite it
            bool recorded = false;
            for (int u = (int)((long long)units * r / NTHREADS); at < f1 && u < units && ok; ++u) {
                Seq q;
                int lo, hi;
                const int w = weight(u, q, lo, hi);
                if (w == 0 || at + (long long)w * group <= f0) {
                    at += (long long)w * group;
                    continue;
                }
                const int s = u / a.RT, token0 = (u - s * a.RT) * NT * a.TT;
                int i = at < f0 ? (int)((f0 - at) / w) : 0;
                at += (long long)i * w;
                for (; i < group && at < f1 && ok; ++i, at += w) {
                    // position 0 of an item stands for what it costs by itself, position 1 + i for visit i
                    const int b = (int)max(0ll, f0 - at - 1), e = (int)min((long long)w, f1 - at) - 1;
                    if (e <= b) continue;
                    const int kvh = i / a.P, pass = i - kvh * a.P;
                    const bool begins = b == 0, ends = e == w - 1;
                    const int slot = begins && ends ? -1 : 2 * cta + (begins ? 1 : 0);
                    if (begins && !ends) {
                        rec.last = cut.cta_of(at + w - 1);
                        rec.n = rec.last - cta + 1;
                        rec.s = s; rec.token0 = token0; rec.kvh = kvh; rec.pass = pass; rec.q = q;
                        // now: the record is this launch's, whatever becomes of the visits
                        if (lane == 0) a.merges[cta] = rec;
                        recorded = true;
                    }
                    const int tiles_rows = min(q.n - token0, NT * a.TT) > a.TT ? TWO : 0;
                    const int32_t *row = a.c.table + (long long)s * a.c.table_stride;
                    // page ids of four visits at a time, one batch ahead
                    auto page_at = [&](int tile) {
                        const int j = (lo + tile) * kPages + (lane & 7);
                        return tile < e && j * kBT < q.len ? row[j] : ISV_BLOCK_NONE;
                    };
                    int ids = page_at(b + lane / 8), next_ids = page_at(b + 4 + lane / 8);
                    for (int x = b; x < e; ++x, ++v) {
                        const int y = (x - b) & 3;
                        if (y == 0 && x > b) {
                            ids = next_ids;
                            next_ids = page_at(x + 4 + lane / 8);
                        }
                        const int j0 = (lo + x) * kTile;
                        const int id = __shfl_sync(~0u, ids, 8 * y + (lane & 7));
                        const bool there = id >= 0 && id < a.c.n_pages;
                        if (lane < 8 && !there && id != ISV_BLOCK_NONE) atomicOr(a.c.status, ISV_STATUS_BAD_BLOCK_ID);
                        const uint32_t pages = __ballot_sync(~0u, there) & 0xff;
                        slot_free(k_index(v));
                        rec_free();
                        if (!ok) break;
                        if (lane == 0) {
                            Visit &z = recs[v % kRecs];
                            z.j0 = j0; z.pages = pages;
                            z.flags = (x == b ? FIRST : 0) | (x == e - 1 ? LAST : 0) | tiles_rows;
                            const int left = q.len - j0;
                            z.partial = left < kTile ? left % kBT : 0;
                            z.last_page = left / kBT;
                            z.s = s; z.token0 = token0; z.kvh = kvh; z.pass = pass; z.slot = slot; z.q = q;
                            bar_arrive(s32(&rec_full[v % kRecs]));
                        }
                        fetch(k_index(v), 0, id, pages, kvh, a.drop_first_copy && at == 0 && x == 0);
                        if (NT == 1) {
                            if (v > 0) {
                                slot_free(v_index(v - 1));
                                if (!ok) break;
                                fetch(v_index(v - 1), 1, before_id, before_pages, before_kvh, false);
                            }
                            before_id = id; before_pages = pages; before_kvh = kvh;
                        } else {
                            slot_free(v_index(v));
                            if (!ok) break;
                            fetch(v_index(v), 1, id, pages, kvh, false);
                        }
                    }
                }
            }
            if (NT == 1 && ok && v > 0) {
                slot_free(v_index(v - 1));
                if (ok) fetch(v_index(v - 1), 1, before_id, before_pages, before_kvh, false);
            }
            if (lane == 0 && !recorded) a.merges[cta] = rec;
        } else if (lane == 0) {
            a.merges[cta] = rec;
        }
        if (ok) put_end();
        if (!ok) give_up();
        if (!ok || gave_up()) {
            // something gave up: the copies in flight land before the memory passes on
            for (uint32_t i = top > SLOTS ? top - SLOTS : 0; i < top; ++i)
                for (uint32_t k = 0; k < 1u << 16 && !bar_try(s32(&full[i % SLOTS]), (i / SLOTS) & 1); ++k) {}
        }
    } else if (warp == kLoader) {
        // ---- Q of each item: a box of the row tile's tokens and their GT heads
        if (lane == 0) {
            bool ok = true;
            int used[2] = {0, 0}, item = 0;
            for (int v = 0; ok; ++v) {
                if (!bar_wait(s32(&rec_full[v % kRecs]), (v / kRecs) & 1, a.spin_limit, state)) { ok = false; break; }
                const Visit z = recs[v % kRecs];
                bar_arrive(s32(&rec_read[v % kRecs]));
                if (z.flags & END) break;
                if (!(z.flags & FIRST)) continue;
                const int tiles = NT == 2 && (z.flags & TWO) ? 2 : 1;
                for (int i = 0; i < tiles && ok; ++i) {
                    const int buf = NT == 2 ? i : R > 1 ? 0 : item & 1;
                    if (used[buf] > 0 && !bar_wait(s32(&q_empty[buf]), (used[buf] - 1) & 1, a.spin_limit, state)) { ok = false; break; }
                    ++used[buf];
                    const uint32_t dst = s32(q_tiles + buf * SH::TILE), bar = s32(&q_full[buf]);
                    const int rows = a.GT * a.TT, head = z.kvh * (a.c.Hq / a.c.Hkv) + z.pass * a.GT, token = z.q.first + z.token0 + i * a.TT;
                    bar_expect(bar, R * rows * D * 2);
                    for (int y = 0; y < R; ++y) {
                        for (int h = 0; h < SH::HALVES; ++h)
                            tma_3d(dst + h * SH::HALF_BYTES + y * (kTile / R * 128), &map_q, 64 * h, head, token, bar);
                        if (SH::TAIL)
                            tma_3d(dst + SH::HALVES * SH::HALF_BYTES + y * (kTile / R * SH::TAIL * 2), &map_q_tail, 64 * SH::HALVES, head, token, bar);
                    }
                }
                ++item;
            }
            if (!ok) give_up();
            if (!ok || gave_up())
                for (int buf = 0; buf < 2; ++buf)
                    for (uint32_t k = 0; used[buf] > 0 && k < 1u << 16 && !bar_try(s32(&q_full[buf]), (used[buf] - 1) & 1); ++k) {}
        }
    } else if (warp == kIssuer) {
        // ---- the products, all issued by one thread in the order in which they run
        constexpr uint32_t idesc_s = instr_desc(BF16, false, kTile);
        constexpr uint32_t idesc_o = instr_desc(BF16, true, 64 * SH::HALVES), idesc_t = instr_desc(BF16, true, 16);
        constexpr uint32_t kTail = SH::HALVES * SH::HALF_BYTES;
        bool ok = true;
        int q_used[2] = {0, 0}, p_used[2] = {0, 0}, item = 0;
        uint32_t started[2] = {0, 0};
        const uint32_t q_base = s32(q_tiles), ring_base = s32(ring);
        auto wait = [&](uint64_t *bar, uint32_t parity) {
            ok = ok && __all_sync(~0u, bar_wait(s32(bar), parity, a.spin_limit, state));
        };
        // S of tile or buffer w of visit v
        auto scores = [&](int v, int flags, int w, bool release) {
            const int qb = NT == 2 ? w : R > 1 ? 0 : item & 1;
            const uint32_t ks = k_index(v) % SLOTS;
            const uint32_t qa = q_base + qb * SH::TILE, ka = ring_base + ks * SH::TILE;
            const uint64_t da = desc(qa, 16, 1024, kSwz128), db = desc(ka, 16, 1024, kSwz128);
#pragma unroll
            for (int h = 0; h < SH::HALVES; ++h)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    mma_ss(w * kTile, da + (h * SH::HALF_BYTES / 16 + 2 * k), db + (h * SH::HALF_BYTES / 16 + 2 * k), idesc_s, h + k > 0);
            if (SH::TAIL) mma_ss(w * kTile, desc(qa + kTail, 16, 256, kSwz32), desc(ka + kTail, 16, 256, kSwz32), idesc_s, 1);
            commit(s32(&s_full[w]));
            if (flags & LAST) commit(s32(&q_empty[qb]));
            if (release) commit(s32(&empty[ks]));
        };
        // O += P V of tile w of visit v, page after page; the weights come in two halves
        auto output = [&](int v, int flags, uint32_t pages, int w, bool release) {
            wait(&p_full[w], p_used[w] & 1);
            if (!ok) return;
            fence_after();
            const uint32_t vs = v_index(v) % SLOTS, va = ring_base + vs * SH::TILE;
            const int ow = NT == 2 ? w : 0;
            const uint32_t d = 2 * kTile + ow * kTile, p = w * kTile;
            const uint64_t db = desc(va, SH::HALF_BYTES, 1024, kSwz128), dt = desc(va + kTail, 16, 256, kSwz32);
            const uint64_t dp = desc(s32(weights), 16, 1024, kSwz128);
            uint32_t more = flags & FIRST ? 0 : started[ow];
            auto page = [&](int i) {
#pragma unroll
                for (int half = 0; half < (FINE ? 2 : 1); ++half) {
                    if (R > 1) {
                        const uint64_t pa = dp + half * (kWeights / 2 / 16) + (i / 4) * (kTile / R * 128 / 16) + 2 * (i % 4);
                        mma_ss(d, pa, db + i * (kBT * 128 / 16), idesc_o, more);
                        if (SH::TAIL) mma_ss(d + 64 * SH::HALVES, pa, dt + i * (kBT * SH::TAIL * 2 / 16), idesc_t, more);
                    } else {
                        const uint32_t pa = p + (i / 2) * 32 + (i % 2) * 8 + half * 16;
                        mma_ts(d, pa, db + i * (kBT * 128 / 16), idesc_o, more);
                        if (SH::TAIL) mma_ts(d + 64 * SH::HALVES, pa, dt + i * (kBT * SH::TAIL * 2 / 16), idesc_t, more);
                    }
                    more = 1;
                }
            };
            if (pages == 0xff) {
#pragma unroll
                for (int i = 0; i < kPages / 2; ++i) page(i);
            } else {
#pragma unroll 1
                for (uint32_t left = pages & 0xf; left; left &= left - 1) page(__ffs(left) - 1);
            }
            wait(&p_full[2 + w], p_used[w]++ & 1);
            if (!ok) return;
            fence_after();
            if (pages == 0xff) {
#pragma unroll
                for (int i = kPages / 2; i < kPages; ++i) page(i);
            } else {
#pragma unroll 1
                for (uint32_t left = pages & 0xf0; left; left &= left - 1) page(__ffs(left) - 1);
            }
            started[ow] = more;
            commit(s32(&pv_done[w]));
            if (release) commit(s32(&empty[vs]));
        };
        auto tile_ready = [&](uint32_t n) { wait(&full[n % SLOTS], (n / SLOTS) & 1); };
        auto q_ready = [&](int flags, int w) {
            if (!(flags & FIRST)) return;
            const int qb = NT == 2 ? w : R > 1 ? 0 : item & 1;
            wait(&q_full[qb], q_used[qb] & 1);
            ++q_used[qb];
        };
        wait(&rec_full[0], 0);
        int flags = same(ok ? recs[0].flags : END);
        uint32_t pages = same(recs[0].pages);
        ok = ok && same(*tmem_slot) == 0;       // all columns are ours: they are counted from 0
        if (ok && !(flags & END)) {
            tile_ready(0);
            q_ready(flags, 0);
            if (ok) {
                fence_after();
                scores(0, flags, 0, !(NT == 2 && (flags & TWO)));
            }
            if (NT == 2 && (flags & TWO)) {
                q_ready(flags, 1);
                if (ok) {
                    fence_after();
                    scores(0, flags, 1, true);
                }
            }
            for (int v = 0; ok; ++v) {
                wait(&rec_full[(v + 1) % kRecs], ((v + 1) / kRecs) & 1);
                if (!ok) break;
                const int next = same(recs[(v + 1) % kRecs].flags);
                const uint32_t next_pages = same(recs[(v + 1) % kRecs].pages);
                const bool more = !(next & END);
                if (NT == 1) {
                    // the next visit's scores go first if their tile is there
                    const int w = v & 1;
                    const uint32_t k_next = k_index(v + 1);
                    bool early = more && __all_sync(~0u, bar_try(s32(&full[k_next % SLOTS]), (k_next / SLOTS) & 1));
                    auto ahead = [&]() {
                        if (flags & LAST) ++item;
                        tile_ready(k_next);
                        q_ready(next, 0);
                        if (!ok) return;
                        fence_after();
                        scores(v + 1, next, w ^ 1, true);
                    };
                    if (early) ahead();
                    if (!ok) break;
                    tile_ready(v_index(v));
                    output(v, flags, pages, w, true);
                    if (!ok) break;
                    if (more && !early) ahead();
                } else {
                    const bool two = flags & TWO, next_two = more && (next & TWO);
                    tile_ready(v_index(v));
                    output(v, flags, pages, 0, !two);
                    if (more) {
                        tile_ready(k_index(v + 1));
                        q_ready(next, 0);
                        if (!ok) break;
                        fence_after();
                        scores(v + 1, next, 0, !next_two);
                    }
                    if (two) output(v, flags, pages, 1, true);
                    if (next_two) {
                        q_ready(next, 1);
                        if (!ok) break;
                        fence_after();
                        scores(v + 1, next, 1, true);
                    }
                }
                if (!more) break;
                flags = next;
                pages = next_pages;
            }
        }
        if (!ok) {
            give_up();
            commit(s32(drain));       // what was issued ends before tensor memory passes on
            for (uint32_t k = 0; k < 1u << 16 && !bar_try(s32(drain), 0); ++k) {}
        }
    } else if (warp < NT * 4) {
        // ---- weights: group w of four warps, one row of its tile per thread
        const int w = warp >> 2, r = threadIdx.x & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        bool ok = true;
        constexpr int ROWS = kTile / R, COLS = kTile / R;                      // of a copy
        const int rr = r % ROWS, part = r / ROWS, col0 = part * COLS;
        const int row_t = rr / a.GT, row_g = rr - row_t * a.GT, G = a.c.Hq / a.c.Hkv;
        uint32_t x_phase = 0;   // exchanges so far
        // what the copies of this thread's row hold of x; every warp takes part
        auto gather = [&](float x, float (&all)[R]) {
            float *at = exchange + (x_phase & 1) * kTile;
            at[r] = x;
            __syncwarp();
            if (lane == 0) bar_arrive(s32(x_full));
            ok = __all_sync(~0u, bar_wait(s32(x_full), x_phase & 1, a.spin_limit, state));
            ++x_phase;
            if (!ok) return;
#pragma unroll
            for (int i = 0; i < R; ++i) all[i] = at[i * ROWS + rr];
        };
        const float c = SHAPED ? kLog2e : a.scale * kLog2e;
        int used = 0;           // visits of this group
        int tok = 0, head = 0, pos = 0, s = 0;
        Seq q{};
        bool live = false, any_live = false;
        Sight sight{};
        float ref = -INFINITY, l = 0.f, slope = 0.f;
        for (int v = 0;; ++v) {
            ok = __all_sync(~0u, bar_wait(s32(&rec_full[v % kRecs]), (v / kRecs) & 1, a.spin_limit, state));
            if (!ok) break;
            const Visit &z = recs[v % kRecs];
            const int flags = z.flags;
            if (flags & END) break;
            auto read = [&]() {
                if (NT == 1 || w == 0) return;
                __syncwarp();
                if (lane == 0) bar_arrive(s32(&rec_read[v % kRecs]));
            };
            if (NT == 2 && w == 1 && !(flags & TWO)) {
                read();
                continue;
            }
            const int b = NT == 2 ? w : v & 1;                                // buffer of the scores
            const uint32_t phase = NT == 2 ? used & 1 : (v >> 1) & 1;
            if (flags & FIRST) {
                q = z.q;
                s = z.s;
                tok = z.token0 + w * a.TT + row_t;
                head = z.kvh * G + z.pass * a.GT + row_g;
                live = row_t < a.TT && tok < q.n && z.pass * a.GT + row_g < G;
                pos = q.start + tok;
                sight = sight_of(a, s, q, pos);
                slope = a.slopes && live ? a.slopes[head] : 0.f;
                ref = -INFINITY;
                l = 0.f;
                any_live = __any_sync(~0u, live);
            }
            const int j0 = z.j0, slot = z.slot, partial = w == 0 ? z.partial : 0, last_page = z.last_page;
            const uint32_t pages = z.pages;
            read();
            ok = __all_sync(~0u, bar_wait(s32(&s_full[b]), phase, a.spin_limit, state));
            if (!ok) break;
            fence_after();
            if (partial) {
                // rows of V behind the sequence's last token meet weights of 0; what stands there may be no number
                const uint32_t n = v_index(v);
                ok = __all_sync(~0u, bar_wait(s32(&full[n % SLOTS]), (n / SLOTS) & 1, a.spin_limit, state));
                if (!ok) break;
                if (pages >> last_page & 1) {
                    uint8_t *vt = ring + (size_t)(n % SLOTS) * SH::TILE;
                    const int rows = kBT - partial, first = last_page * kBT + partial;
                    for (int i = r; i < rows * 8 * SH::HALVES; i += 128)
                        *reinterpret_cast<uint4 *>(vt + (i / (rows * 8)) * SH::HALF_BYTES + (first + i % (rows * 8) / 8) * 128 + i % 8 * 16) =
                            make_uint4(0, 0, 0, 0);
                    if (SH::TAIL)
                        for (int i = r; i < rows * 2; i += 128)
                            *reinterpret_cast<uint4 *>(vt + SH::HALVES * SH::HALF_BYTES + (first + i / 2) * (SH::TAIL * 2) + i % 2 * 16) =
                                make_uint4(0, 0, 0, 0);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
            }
            if (any_live) {
                // two passes over the scores, a few columns at a time (a loop that holds a row's 128 scores in registers is so
                // long that fetching its instructions bounds it: 930 us against 590 on a prompt of 8192 tokens)
                const uint32_t cols = lanes + b * kTile + col0;
                const int j1 = j0 + col0;                                      // this thread's columns
                const bool all = pages == 0xff && sight.lim >= j0 + kTile && (sight.low <= j0 || sight.prefix >= j0 + kTile);
                const bool masked = !__all_sync(~0u, all || !live);
                float xa[32], xb[32];
                if (SHAPED) {
                    // scores that need more than a factor are made ready first, in place: a loop of its own is the least code
#pragma unroll 1
                    for (int k = 0; k < COLS / 32; ++k) {
                        const int at = j1 + 32 * k;
                        float (&y)[32] = xa;
                        tmem_ld32(cols + 32 * k, reinterpret_cast<uint32_t *>(y));
                        wait_ld();
                        if (a.cap > 0.f) {
                            const float in = a.scale / a.cap;
                            float most = 0.f;
#pragma unroll
                            for (int i = 0; i < 32; i += 2) most = max3(most, fabsf(y[i]), fabsf(y[i + 1]));
                            if (__all_sync(~0u, most * fabsf(in) <= 1.f || !live)) {
#pragma unroll
                                for (int i = 0; i < 32; i += 2) {
                                    const float2 z = unpair(mul2(tanh_poly(mul2(pair(y[i], y[i + 1]), both(in))), both(a.cap)));
                                    y[i] = z.x;
                                    y[i + 1] = z.y;
                                }
                            } else {
                                // cap tanh(z) = cap - 2 cap / (e^2z + 1): off by a few 2^-24 of the cap
#pragma unroll
                                for (int i = 0; i < 32; ++i) {
                                    const float e = exp2_fast(y[i] * (2.f * kLog2e * in));
                                    y[i] = fmaf(-2.f * a.cap, reciprocal(e + 1.f), a.cap);
                                }
                            }
                        }
                        if (a.slopes || !(a.cap > 0.f)) {
                            const uint64_t by = both(a.cap > 0.f ? 1.f : a.scale);
                            const float distance = (float)(pos - at);
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                const float2 z = unpair(mul2(pair(y[i], y[i + 1]), by));
                                y[i] = fmaf(-slope, fabsf(distance - (float)i), z.x);
                                y[i + 1] = fmaf(-slope, fabsf(distance - (float)(i + 1)), z.y);
                            }
                        }
                        if (masked) {
                            // bit i: token at + i is seen
                            auto below = [&](int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; };
                            const uint32_t here = pages >> ((at - j0) / kBT);
                            uint32_t seen = below(sight.lim - at) & (~below(sight.low - at) | below(sight.prefix - at));
                            seen &= (here & 1 ? 0xffffu : 0u) | (here & 2 ? 0xffff0000u : 0u);
#pragma unroll
                            for (int i = 0; i < 32; ++i) y[i] = seen >> i & 1 ? y[i] : -INFINITY;
                        }
                        tmem_st32(cols + 32 * k, reinterpret_cast<uint32_t *>(y));
                    }
                    wait_st();
                }
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                auto look = [&](float (&y)[32], int k) {
                    const int at = j1 + 32 * k;
                    if (!SHAPED && masked) {
                        // bit i: token at + i is seen
                        auto below = [&](int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; };
                        const uint32_t here = pages >> (2 * k + col0 / kBT);
                        uint32_t seen = below(sight.lim - at) & (~below(sight.low - at) | below(sight.prefix - at));
                        seen &= (here & 1 ? 0xffffu : 0u) | (here & 2 ? 0xffff0000u : 0u);
#pragma unroll
                        for (int i = 0; i < 32; ++i) y[i] = seen >> i & 1 ? y[i] : -INFINITY;
                    }
                    if (COLS > 32 && !SHAPED && masked) tmem_st32(cols + 32 * k, reinterpret_cast<uint32_t *>(y));
#pragma unroll
                    for (int i = 0; i < 32; i += 2) top[i / 2 & 3] = max3(top[i / 2 & 3], y[i], y[i + 1]);
                };
                tmem_ld32(cols, reinterpret_cast<uint32_t *>(xa));
#pragma unroll 1
                for (int k = 0; k < COLS / 32; k += 2) {
                    wait_ld();
                    if (COLS > 32) tmem_ld32(cols + 32 * (k + 1), reinterpret_cast<uint32_t *>(xb));
                    look(xa, k);
                    if (COLS > 32) {
                        wait_ld();
                        if (k + 2 < COLS / 32) tmem_ld32(cols + 32 * (k + 2), reinterpret_cast<uint32_t *>(xa));
                        look(xb, k + 1);
                    }
                }
                if (COLS > 32) {
                    if (!SHAPED && masked) wait_st();
                    tmem_ld32(cols, reinterpret_cast<uint32_t *>(xa));
                }
                float high = max3(top[0], top[1], max3(top[2], top[3], top[3])) * c;
                if (R > 1) {
                    float of[R];
                    gather(high, of);
                    if (!ok) break;
#pragma unroll
                    for (int i = 0; i < R; ++i) high = max3(high, high, of[i]);
                }
                float factor = 1.f;
                if (!(high <= FLT_MAX)) {
                    l = NAN;        // a score that is NaN or infinite: the row is computed token by token at the end
                } else if (ref == -INFINITY) {
                    ref = high;
                } else if (high > ref + slack_of<BF16>()) {
                    factor = exp2_fast(ref - high);
                    ref = high;
                }
                const uint32_t before = NT == 2 ? used - 1 : v - 1;            // the product before this one
                if (R > 1 && v > 0) {
                    // it has read the weights that are overwritten now
                    ok = __all_sync(~0u, bar_wait(s32(&pv_done[before & 1]), (before >> 1) & 1, a.spin_limit, state));
                    if (!ok) break;
                }
                if (__any_sync(~0u, factor != 1.f)) {
                    // O is scaled: the product before this one has to be in it
                    l *= factor;
                    ok = __all_sync(~0u, bar_wait(s32(&pv_done[NT == 2 ? w : before & 1]), (NT == 2 ? before : before >> 1) & 1, a.spin_limit, state));
                    if (!ok) break;
                    fence_after();
                    const uint32_t o = lanes + 2 * kTile + (NT == 2 ? w : 0) * kTile;
                    if (part == 0) {
#pragma unroll 1
                        for (int i = 0; i < D; i += 16) {
                            uint32_t y[16];
                            tmem_ld16(o + i, y);
                            wait_ld();
#pragma unroll
                            for (int k = 0; k < 16; ++k) y[k] = __float_as_uint(__uint_as_float(y[k]) * factor);
                            tmem_st16(o + i, y);
                        }
                        wait_st();
                    }
                }
                const float minus = ref == -INFINITY ? 0.f : kOffset - ref;
                const uint64_t cc = pair(c, c), mm = pair(minus, minus);
                uint64_t sum[2] = {pair(0.f, 0.f), pair(0.f, 0.f)};
                auto weigh = [&](const float (&y)[32], int k) {
                    uint32_t hi[16], lo[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const uint64_t e2 = fma2(pair(y[2 * i], y[2 * i + 1]), cc, mm);
                        const float2 e = unpair(e2);
                        const bool poly = NT == 2 && !FINE && !SHAPED && i * kPoly % 16 < kPoly;
                        const float2 p = poly ? exp2_poly<BF16 ? 3 : 4>(e2) : make_float2(exp2_fast(e.x), exp2_fast(e.y));
                        hi[i] = narrow<BF16>(p.x, p.y);
                        // the sum is that of the weights as they are used: a weight that is most of a row has no error then
                        const float2 h = widen<BF16>(hi[i]);
                        sum[i & 1] = add2(sum[i & 1], FINE ? pair(p.x, p.y) : pair(h.x, h.y));
                        if (FINE) lo[i] = narrow<BF16>(p.x - h.x, p.y - h.y);
                    }
                    if (R > 1) {
                        // rows of 64 columns with the 128-byte swizzle
                        const int col = col0 + 32 * k;
                        uint8_t *row = weights + (col / 64) * (ROWS * 128) + rr * 128;
#pragma unroll
                        for (int y4 = 0; y4 < 4; ++y4) {
                            const int chunk = (col % 64 / 8 + y4) ^ (rr & 7);
                            *reinterpret_cast<uint4 *>(row + chunk * 16) = make_uint4(hi[4 * y4], hi[4 * y4 + 1], hi[4 * y4 + 2], hi[4 * y4 + 3]);
                            if (FINE)
                                *reinterpret_cast<uint4 *>(row + kWeights / 2 + chunk * 16) =
                                    make_uint4(lo[4 * y4], lo[4 * y4 + 1], lo[4 * y4 + 2], lo[4 * y4 + 3]);
                        }
                    } else {
                        // in place of their scores
                        tmem_st16(cols + 32 * k, hi);
                        if (FINE) tmem_st16(cols + 32 * k + 16, lo);
                    }
                };
#pragma unroll 1
                for (int k = 0; k < COLS / 32; k += 2) {
                    if (COLS > 32) {
                        wait_ld();
                        tmem_ld32(cols + 32 * (k + 1), reinterpret_cast<uint32_t *>(xb));
                    }
                    weigh(xa, k);
                    if (COLS > 32) {
                        wait_ld();
                        if (k + 2 < COLS / 32) tmem_ld32(cols + 32 * (k + 2), reinterpret_cast<uint32_t *>(xa));
                        weigh(xb, k + 1);
                    }
                    if (R == 1 && k == 0) {
                        wait_st();
                        fence_before();
                        __syncwarp();
                        if (lane == 0) bar_arrive(s32(&p_full[b]));
                    }
                }
                const float2 total2 = unpair(add2(sum[0], sum[1]));
                l += total2.x + total2.y;
                if (R > 1) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                else wait_st();
            } else if (R > 1) {
                float of[R];
                gather(-INFINITY, of);
                if (!ok) break;
            }
            ++used;
            fence_before();
            __syncwarp();
            if (lane == 0) {
                if (R > 1 || !any_live) bar_arrive(s32(&p_full[b]));
                bar_arrive(s32(&p_full[2 + b]));
            }
            if (!(flags & LAST)) continue;

            // ---- the item's end: O / l, or a partial result
            ok = __all_sync(~0u, bar_wait(s32(&pv_done[b]), phase, a.spin_limit, state));
            if (!ok) break;
            if (R > 1) {
                float of[R];
                gather(l, of);
                if (!ok) break;
                if (any_live) {
                    l = 0.f;
#pragma unroll
                    for (int i = 0; i < R; ++i) l += of[i];
                }
            }
            if (!any_live || part > 0) continue;
            fence_after();
            const uint32_t o = lanes + 2 * kTile + (NT == 2 ? w : 0) * kTile;
            const bool some = l != 0.f;        // NaN is some
            const long long at = ((long long)(q.first + tok) * a.c.Hq + head) * D;
            const float inv = slot < 0 ? 1.f / l : 1.f;
            bool fine = !some || fabsf(l) <= FLT_MAX;
            constexpr int STEP = D == 80 ? 16 : 32;
#pragma unroll 1
            for (int i = 0; i < D; i += STEP) {
                uint32_t y[STEP];
#pragma unroll
                for (int k = 0; k < STEP; k += 16) tmem_ld16(o + i + k, y + k);
                wait_ld();
                float f[STEP];
#pragma unroll
                for (int k = 0; k < STEP; ++k) {
                    f[k] = some ? __uint_as_float(y[k]) * inv : 0.f;
                    fine = fine && fabsf(f[k]) <= FLT_MAX;
                }
                if (live && slot >= 0) {
                    float4 *dst = reinterpret_cast<float4 *>(a.part_o) + ((long long)slot * (D / 4) + i / 4) * (2 * kTile) + w * kTile + r;
#pragma unroll
                    for (int k = 0; k < STEP / 4; ++k) dst[k * (2 * kTile)] = make_float4(f[4 * k], f[4 * k + 1], f[4 * k + 2], f[4 * k + 3]);
                }
                if (live && slot < 0 && a.out_f32) {
#pragma unroll
                    for (int k = 0; k < STEP / 4; ++k)
                        reinterpret_cast<float4 *>(a.out_f32 + at + i)[k] = make_float4(f[4 * k], f[4 * k + 1], f[4 * k + 2], f[4 * k + 3]);
                }
                if (live && slot < 0 && a.out) {
#pragma unroll
                    for (int k = 0; k < STEP / 8; ++k)
                        reinterpret_cast<uint4 *>(a.out + at + i)[k] = make_uint4(narrow<BF16>(f[8 * k], f[8 * k + 1]), narrow<BF16>(f[8 * k + 2], f[8 * k + 3]),
                                                                                  narrow<BF16>(f[8 * k + 4], f[8 * k + 5]), narrow<BF16>(f[8 * k + 6], f[8 * k + 7]));
                }
                __syncwarp();
            }
            if (slot >= 0) {
                if (live) reinterpret_cast<float2 *>(a.part_ml)[(long long)slot * (2 * kTile) + w * kTile + r] =
                    make_float2(!some ? -INFINITY : fabsf(l) <= FLT_MAX ? ref : INFINITY, l);   // what is no number outweighs the rest
            } else {
                // sums that are no number: an infinity or NaN in a token that the row does not see (0 times that is NaN), or an
                // overflow of values near the type's largest.  Such a row is computed token by token.
                uint32_t odd = __ballot_sync(~0u, live && !fine);
                if (odd) {
                    if (lane == 0) atomicAdd(state, 1);
                    for (; odd; odd &= odd - 1) {
                        const int from = __ffs(odd) - 1;
                        attend_row<D, BF16>(a, s, q, __shfl_sync(~0u, tok, from), __shfl_sync(~0u, head, from));
                    }
                    if (lane == 0) atomicSub(state, 1);
                }
            }
            fence_before();
        }
        if (!ok) give_up();
    }

    fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && gave_up()) atomicOr(a.c.status, ISV_STATUS_WAIT_EXPIRED);
    if (warp == kIssuer) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(*tmem_slot) : "memory");
}

// ---------------------------------------------------------------- merging

// Partial results of items that crossed ranges.  CTA (record, group of 32 rows): a lane has one row, a warp kWide times four of its
// values, and kFly partial results are in flight together (bound by the latency of those rounds).  Items of few rows are cut into
// many partial results: a warp for every four values.  Items of 256 rows have two or three, in many CTAs: eight warps.
template <int D, int NT>
__host__ __device__ constexpr int merge_warps() { return NT == 1 ? D / 4 : 8; }
template <int D, bool BF16, int NT>
__global__ void __launch_bounds__(merge_warps<D, NT>() * 32) merge_kernel(const __grid_constant__ AttnParams a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const MergeRec m = a.merges[blockIdx.x];
    if (m.n == 0) return;
    const Seq q = m.q;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.y * 32 + lane;
    const int w = row / kTile, r = row % kTile, row_t = r / a.GT, row_g = r - row_t * a.GT, G = a.c.Hq / a.c.Hkv;
    const int tok = m.token0 + w * a.TT + row_t, head = m.kvh * G + m.pass * a.GT + row_g;
    const bool live = row_t < a.TT && tok < q.n && m.pass * a.GT + row_g < G;
    if (!__any_sync(~0u, live)) return;
    auto slot = [&](int i) { return (long long)(2 * ((int)blockIdx.x + i) + (i == 0 ? 1 : 0)); };
    const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml);
    constexpr int WARPS = merge_warps<D, NT>(), kWide = (D / 4 + WARPS - 1) / WARPS, kFly = NT == 1 ? 8 : 2;
    float at = -INFINITY, l = 0.f;        // the largest reference so far; sums relative to it
    float4 o[kWide];
#pragma unroll
    for (int c = 0; c < kWide; ++c) o[c] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < m.n; i += kFly) {
        float4 y[kFly][kWide];
        float2 z[kFly];
#pragma unroll
        for (int k = 0; k < kFly; ++k) {
            const long long from = slot(min(i + k, m.n - 1));
            z[k] = ml[from * (2 * kTile) + row];
#pragma unroll
            for (int c = 0; c < kWide; ++c)
                y[k][c] = reinterpret_cast<const float4 *>(a.part_o)[(from * (D / 4) + min(warp + c * WARPS, D / 4 - 1)) * (2 * kTile) + row];
        }
        float top = at;
#pragma unroll
        for (int k = 0; k < kFly; ++k) top = fmaxf(top, z[k].x);
        const float keep = at == -INFINITY ? 0.f : exp2_fast(at - top);
        const float to = top == -INFINITY ? 0.f : top;
        at = top;
        l *= keep;
#pragma unroll
        for (int c = 0; c < kWide; ++c) { o[c].x *= keep; o[c].y *= keep; o[c].z *= keep; o[c].w *= keep; }
#pragma unroll
        for (int k = 0; k < kFly; ++k) {
            const float f = exp2_fast(z[k].x - to);
            if (i + k < m.n && f != 0.f) {
                l = fmaf(f, z[k].y, l);
#pragma unroll
                for (int c = 0; c < kWide; ++c) {
                    o[c].x = fmaf(f, y[k][c].x, o[c].x); o[c].y = fmaf(f, y[k][c].y, o[c].y);
                    o[c].z = fmaf(f, y[k][c].z, o[c].z); o[c].w = fmaf(f, y[k][c].w, o[c].w);
                }
            }
        }
    }
    const float inv = l != 0.f ? 1.f / l : 0.f;
    bool fine = fabsf(l) <= FLT_MAX;
#pragma unroll
    for (int c = 0; c < kWide; ++c) {
        if (warp + c * WARPS >= D / 4) continue;
        float4 r4 = o[c];
        r4.x *= inv; r4.y *= inv; r4.z *= inv; r4.w *= inv;
        fine = fine && fabsf(r4.x) <= FLT_MAX && fabsf(r4.y) <= FLT_MAX && fabsf(r4.z) <= FLT_MAX && fabsf(r4.w) <= FLT_MAX;
        const long long to = ((long long)(q.first + tok) * a.c.Hq + head) * D + 4 * (warp + c * WARPS);
        if (live) {
            if (a.out) *reinterpret_cast<uint2 *>(a.out + to) = make_uint2(narrow<BF16>(r4.x, r4.y), narrow<BF16>(r4.z, r4.w));
            if (a.out_f32) *reinterpret_cast<float4 *>(a.out_f32 + to) = r4;
        }
    }
    // rows whose sums are no number (see the kernel above): every warp has its columns written before one recomputes the row
    __shared__ uint32_t odd_s;
    if (threadIdx.x == 0) odd_s = 0;
    __syncthreads();
    const uint32_t odd = __ballot_sync(~0u, live && !fine);
    if (lane == 0 && odd) atomicOr(&odd_s, odd);
    __syncthreads();
    int i = 0;
    for (uint32_t left = odd_s; left; left &= left - 1, ++i) {
        const int from = __ffs(left) - 1;
        const int t = __shfl_sync(~0u, tok, from), h = __shfl_sync(~0u, head, from);
        if (i % merge_warps<D, NT>() == warp) attend_row<D, BF16>(a, m.s, q, t, h);
    }
}

// ---------------------------------------------------------------- host side

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
    static const EncodeTiledFn fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        const bool ok = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess;
        return ok ? reinterpret_cast<EncodeTiledFn>(p) : nullptr;
    }();
    return fn;
}

bool encode(CUtensorMap *m, bool bf16, int rank, const void *base, const cuuint64_t *dims, const cuuint64_t *strides, const cuuint32_t *box,
            CUtensorMapSwizzle swizzle) {
    const cuuint32_t one[3] = {1, 1, 1};
    return encode_fn()(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank, const_cast<void *>(base), dims, strides,
                       box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool BF16, int NT, int R, bool FINE, bool SHAPED>
cudaError_t launch(const AttnParams &p, int grid, cudaStream_t st, const char **what) {
    CUtensorMap kv{}, kv_tail{}, q{}, q_tail{};
    if (!encode_fn()) { *what = "cuTensorMapEncodeTiled is not available from this driver"; return cudaErrorUnknown; }
    const cuuint64_t kv_dims[2] = {D, (cuuint64_t)p.c.n_pages * 2 * p.c.Hkv * kBT}, kv_strides[1] = {D * 2};
    const cuuint64_t q_dims[3] = {D, (cuuint64_t)p.c.Hq, (cuuint64_t)p.c.n_rows}, q_strides[2] = {D * 2, (cuuint64_t)p.q_stride * 2};
    const cuuint32_t kv_box[2] = {64, kBT}, q_box[3] = {64, (cuuint32_t)p.GT, (cuuint32_t)p.TT};
    const cuuint32_t kv_tail_box[2] = {16, kBT}, q_tail_box[3] = {16, (cuuint32_t)p.GT, (cuuint32_t)p.TT};
    bool ok = encode(&kv, BF16, 2, p.c.pool, kv_dims, kv_strides, kv_box, CU_TENSOR_MAP_SWIZZLE_NONE) &&
              encode(&q, BF16, 3, p.q, q_dims, q_strides, q_box, CU_TENSOR_MAP_SWIZZLE_128B);
    if (Shape<D>::TAIL)
        ok = ok && encode(&kv_tail, BF16, 2, p.c.pool, kv_dims, kv_strides, kv_tail_box, CU_TENSOR_MAP_SWIZZLE_32B) &&
             encode(&q_tail, BF16, 3, p.q, q_dims, q_strides, q_tail_box, CU_TENSOR_MAP_SWIZZLE_32B);
    if (!ok) { *what = "cuTensorMapEncodeTiled refused the pool or the rows of q"; return cudaErrorUnknown; }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads_of<NT>());
    cfg.dynamicSmemBytes = smem_bytes<D>(R);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, attn_kernel<D, BF16, NT, R, FINE, SHAPED>, kv, kv_tail, q, q_tail, p);
    // a table row that covers one visit: no item is cut
    if (e != cudaSuccess || p.c.max_blocks <= kPages) return e;
    cfg.gridDim = dim3(grid, NT * kTile / R / 32);
    cfg.blockDim = dim3(merge_warps<D, NT>() * 32);
    cfg.dynamicSmemBytes = 0;
    return cudaLaunchKernelEx(&cfg, merge_kernel<D, BF16, NT>, p);
}

template <int D, bool BF16, int NT, int R, bool FINE>
cudaError_t allow_as() {
    cudaError_t e = cudaFuncSetAttribute(attn_kernel<D, BF16, NT, R, FINE, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<D>(R));
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(attn_kernel<D, BF16, NT, R, FINE, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<D>(R));
    return e;
}
template <int D, bool BF16, int NT, int R>
cudaError_t allow() {
    const cudaError_t e = allow_as<D, BF16, NT, R, false>();
    return e == cudaSuccess ? allow_as<D, BF16, NT, R, true>() : e;
}
template <int D, bool BF16>
cudaError_t configure() {
    cudaError_t e = allow<D, BF16, 1, 4>();
    if (e == cudaSuccess) e = allow<D, BF16, 1, 2>();
    if (e == cudaSuccess) e = allow<D, BF16, 1, 1>();
    if (e == cudaSuccess) e = allow<D, BF16, 2, 1>();
    return e;
}
// FINE: weights enter their product as two 16-bit numbers, which keeps fp32's precision for one product more.  An fp32 output gets
// that.  A 16-bit output alone gets weights rounded to 16 bits, an error of the order of its own rounding: 64 users' drafts 131 ->
// 118 us, single tokens 90 -> 86; on prompts the tensor cores have half as much again to do for it.
template <int D, bool BF16, bool FINE, bool SHAPED>
cudaError_t pick_rows(const AttnParams &p, int grid, cudaStream_t st, const char **what) {
    switch (p.tile_rows) {
    case 32: return launch<D, BF16, 1, 4, FINE, SHAPED>(p, grid, st, what);
    case 64: return launch<D, BF16, 1, 2, FINE, SHAPED>(p, grid, st, what);
    case 128: return launch<D, BF16, 1, 1, FINE, SHAPED>(p, grid, st, what);
    default: return launch<D, BF16, 2, 1, FINE, SHAPED>(p, grid, st, what);
    }
}
template <int D, bool BF16, bool SHAPED>
cudaError_t pick_shape(const AttnParams &p, int grid, cudaStream_t st, const char **what) {
    return p.out_f32 ? pick_rows<D, BF16, true, SHAPED>(p, grid, st, what) : pick_rows<D, BF16, false, SHAPED>(p, grid, st, what);
}
// SHAPED: the scores need more than a positive factor.
template <int D, bool BF16>
cudaError_t pick(const AttnParams &p, int grid, cudaStream_t st, const char **what) {
    return p.cap > 0.f || p.slopes || !(p.scale > 0.f) ? pick_shape<D, BF16, true>(p, grid, st, what) : pick_shape<D, BF16, false>(p, grid, st, what);
}

}  // namespace

template <int D>
cudaError_t attn_configure(bool bf16) { return bf16 ? configure<D, true>() : configure<D, false>(); }
template <int D>
cudaError_t launch_attn(const AttnParams &p, bool bf16, int grid, cudaStream_t st, const char **what) {
    return bf16 ? pick<D, true>(p, grid, st, what) : pick<D, false>(p, grid, st, what);
}

}  // namespace chunk
}  // namespace isv
