// Decode attention over the 8-bit cache (isv_q8_attn; layout and formats: include/isv.h).
//
// Per (sequence, KV head) and block of 16 tokens, with q of the GT query heads that share the KV head:
//     S[token][head] = K q^T * (scale_K * log2(e) / sqrt(D)),  p = 2^(S - m),  l += p,  O[dim][head] += (V^T p) * scale_V
// with a running reference m per head, everything accumulated in fp32.  Both products run on the tensor cores
// (mma.m16n8k16, fp16 operands) with the cache as the 16-row operand and the query heads as the 8 columns: a
// visit of one block costs D / 16 instructions for the scores and D / 8 for the output however many of the 8
// columns are in use, half of what heads as rows would take.  8-bit codes are exact in fp16; q is brought into fp16
// by a power of two per head (exact but for elements 2^-32 below the largest).  p goes in as an fp16 value and its fp16
// remainder, scaled per block and head so that the block's largest weight lies near the top of fp16's range: a weight is then
// off by 2^-22 of itself, or by 2^-40 of the block's largest, however small the block's weights are next to another one's.  The
// block's product is scaled back, by scale_V too, as it is added to the output in fp32.  The codes lie in memory in the order of the operand
// registers, so a lane's operands are 16-byte shared-memory loads without conflicts and nothing is transposed.
//
// What bounds it is reading the cache.  All visits of all (sequence, KV head) pairs form one list that is cut into equal ranges,
// one per warp, whatever the lengths.  A warp streams its visits through a ring of its own (one bulk copy of
// a unit brings K, V and both scales).  A pair that several warps share leaves partial results that are merged in fixed
// order, first within the CTA in shared memory, then, for the pairs that cross CTAs, by the warp that arrives last.
//
// Measured on B200, a call in a captured graph (and among others through the Python binding): 256 sequences x 4111 tokens, 32
// query / 8 KV heads x 128, bf16, e4m3: 338 to 350 us, 6.4 to 6.2 TB/s (369 us); 32 x 1088 tokens, 32 heads x 128, fp16, int8:
// 61.5 us, 4.7 TB/s (62.1); one sequence of 8191 tokens, 32 / 8 heads: 13.6 us (13.6), of which the reading would take 2.6.
// In short calls about 10 us are look-up and first data, and merges.  What keeps fp32's precision (a block's own unit, products
// added in fp32, K's codes without an offset) takes 7 us of the 32 x 1088 tokens: 54.4 us without it.  There neither HBM (55 %)
// nor the issue slots (49 %) are full: with three warps a scheduler, a visit's chain of dependent steps is what is left.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "isv_q8.cuh"

namespace isv {
namespace q8 {
namespace {

constexpr float kMost = 3.402823466e38f;     // the largest number
constexpr float kNone = -kMost;              // reference of a head that has no score yet: the lowest number, so that no score lies below it
constexpr uint32_t kDrainLimit = 1u << 14;   // polls for each copy that may be in flight behind a lost one: tens of ms
constexpr float kSlack = 8.f;                // scores may exceed the reference by this much (log2) before it moves
constexpr float kLeast = -100.f;             // log2 of the smallest unit of a block's weights
constexpr int kFly = 10;                     // partial results that the last merge has in flight
// Visits below which fewer CTAs, and fewer warps of a CTA, take part: every CTA more is one more partial result to merge (one
// sequence of 4096 tokens, 8 heads on one KV head: 18.5 us on 148 CTAs, 11.4 on 32 when this was chosen, 11.8 now).
constexpr int kMinCtaVisits = 8, kMinVisits = 2;

__device__ __forceinline__ uint32_t s32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, uint32_t limit) {
    if (try_wait(bar, parity)) return true;
    for (uint32_t i = 1; i < limit; ++i) {
        if (try_wait(bar, parity)) return true;
        if (i > 256) __nanosleep(64);
    }
    return false;
}
__device__ __forceinline__ void arm(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_in(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void prefetch_l1(const void *p) { asm volatile("prefetch.global.L1 [%0];" ::"l"(p)); }
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <bool BF16>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same product alone.
template <bool BF16>
__device__ __forceinline__ void mma_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// acc += t * (f.x, f.y, f.x, f.y)
__device__ __forceinline__ void add_scaled(float (&acc)[4], const float (&t)[4], uint64_t f) {
    const float2 a = unpair(fma2(pair(t[0], t[1]), f, pair(acc[0], acc[1]))), b = unpair(fma2(pair(t[2], t[3]), f, pair(acc[2], acc[3])));
    acc[0] = a.x; acc[1] = a.y; acc[2] = b.x; acc[3] = b.y;
}
// 8x8 matrix of 16-bit values across the warp, transposed.
__device__ __forceinline__ uint32_t transpose(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// Four codes -> two pairs of fp16: (byte 0, byte 1) and (byte 2, byte 3).  Exact.
template <bool E4M3>
__device__ __forceinline__ void widen(uint32_t w, uint32_t &lo, uint32_t &hi) {
    if (E4M3) {
        asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.rn.f16x2.e4m3x2 %0, a;\ncvt.rn.f16x2.e4m3x2 %1, b;\n}\n" : "=r"(lo), "=r"(hi) : "r"(w));
    } else {
        // 0x6400 is 1024 in fp16, with a last place worth 1: 0x6400 + (code + 128) is 1152 + code
        const uint32_t u = w ^ 0x80808080u;
        const __half2 base = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));   // 1152
        uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
        const __half2 x = __hsub2(*reinterpret_cast<__half2 *>(&a), base), y = __hsub2(*reinterpret_cast<__half2 *>(&b), base);
        lo = *reinterpret_cast<const uint32_t *>(&x);
        hi = *reinterpret_cast<const uint32_t *>(&y);
    }
}

template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float x, float y) {   // x in the low half
    if (BF16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
    const __half2 v = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t x, uint32_t y) {
    const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&y));
    return *reinterpret_cast<const uint32_t *>(&m);
}
template <bool BF16>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
    return BF16 ? __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w)) : __half22float2(*reinterpret_cast<const __half2 *>(&w));
}
// x, y and what 16 bits lose of them
template <bool BF16>
__device__ __forceinline__ uint32_t split2(float &x, float &y) {
    const uint32_t w = pack2<BF16>(x, y);
    const float2 f = unpack2<BF16>(w);
    x -= f.x;
    y -= f.y;
    return w;
}

// ---- one warp's running state for the heads of a visit.  Lane 4 g + c holds, of each 16 x 8 score tile, tokens g and
// g + 8 of heads 2 c and 2 c + 1; of the output dims g * D / 8 .. of the same heads.
template <int D, int NT, bool BF16, bool E4M3>
struct State {
    static constexpr int KS = D / 16, MT = D / 16;
    static constexpr float kUp = 0x1p15f;   // weights of at most 2^0.25 become fp16 numbers at the top of its range
    float acc[NT][MT][4];
    float m[NT][2], l[NT][2];
    float vref, inv_vref;      // acc is in units of vref, a power of two not far below the largest scale of V seen
    uint32_t q[NT][KS][2];     // q as fp16 operand
    float qf[NT][2];           // what its scores have to be multiplied by

    // Raw q operand of k-steps 2 p, 2 p + 1 of head row `row` (16 bytes; the last 8 at head_dim 80).
    __device__ __forceinline__ static uint4 q_words(const uint16_t *row, int p, int c, bool valid) {
        uint4 w = make_uint4(0, 0, 0, 0);
        if (!valid) return w;
        if (p < D / 32) return *reinterpret_cast<const uint4 *>(row + 32 * p + 8 * c);
        const uint2 h = *reinterpret_cast<const uint2 *>(row + 32 * p + 4 * c);
        w.x = h.x; w.y = h.y;
        return w;
    }

    __device__ __forceinline__ void start(const uint16_t *q0, int GT, float scale_log2, int lane) {
        const int g = lane >> 2, c = lane & 3;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const bool valid = nt * 8 + g < GT;
            const uint16_t *row = q0 + (size_t)(nt * 8 + g) * D;
            uint4 w[(KS + 1) / 2];
#pragma unroll
            for (int p = 0; p < (KS + 1) / 2; ++p) w[p] = q_words(row, p, c, valid);
            float f = scale_log2;
            if (BF16) {   // by a power of two to the top of fp16's range: eight bits of bf16 are exact from 2^-32 of the largest on
                float top = 0.f;
#pragma unroll
                for (int p = 0; p < (KS + 1) / 2; ++p)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 v = unpack2<true>((&w[p].x)[i]);
                        top = fmaxf(top, fmaxf(fabsf(v.x), fabsf(v.y)));
                    }
                top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
                top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
                int e = (int)(__float_as_uint(top) >> 23) - 127;
                e = e == 128 ? 0 : max(e, -100);   // not finite, or so small that f would leave the normal range
                const float up = __uint_as_float((uint32_t)(127 + 15 - e) << 23);
                f *= __uint_as_float((uint32_t)(127 - 15 + e) << 23);
#pragma unroll
                for (int p = 0; p < (KS + 1) / 2; ++p)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 v = unpack2<true>((&w[p].x)[i]);
                        (&w[p].x)[i] = pack2<false>(v.x * up, v.y * up);
                    }
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                q[nt][ks][0] = (&w[ks / 2].x)[2 * (ks % 2)];
                q[nt][ks][1] = (&w[ks / 2].x)[2 * (ks % 2) + 1];
            }
            qf[nt][0] = __shfl_sync(~0u, f, 8 * c);        // head 2 c is row 2 c: lanes 8 c ..
            qf[nt][1] = __shfl_sync(~0u, f, 8 * c + 4);
#pragma unroll
            for (int i = 0; i < 2; ++i) { m[nt][i] = kNone; l[nt][i] = 0.f; }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[nt][mt][i] = 0.f;
        }
        vref = 0.f;
        inv_vref = 0.f;
    }

    // Brings acc into units in which values of scale vs do not come near the end of fp32's range.  Units only grow: smaller
    // values have all of fp32's exponents below, where larger ones, enlarged by a smaller unit, could overflow.
    __device__ __forceinline__ void refer(float vs) {
        if (!(vs > vref * 0x1p40f)) return;
        const float now = fmaxf(__uint_as_float(__float_as_uint(vs) & 0x7f800000u), 0x1p-126f);
        const float f = vref / now;
        vref = now;
        inv_vref = 1.f / now;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[nt][mt][i] *= f;
    }

    // Scores of a tile -> weights p, as p = s * unit with a unit of the block per head in which its largest weight is between
    // 2^-0.25 and 2^0.25 (unless that is below 2^-100); moves the reference where a score exceeds it by more than kSlack.
    __device__ __forceinline__ void weigh(float (&s)[NT][4], float (&unit)[NT][2]) {
        bool over = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) over = over || s[nt][i] - m[nt][i & 1] > kSlack;
        if (__any_sync(~0u, over)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float top = fmaxf(s[nt][i], s[nt][i + 2]);
                    top = fmaxf(top, __shfl_xor_sync(~0u, top, 4));
                    top = fmaxf(top, __shfl_xor_sync(~0u, top, 8));
                    top = fmaxf(top, __shfl_xor_sync(~0u, top, 16));
                    top = fmaxf(top, m[nt][i]);
                    const float f = ex2(m[nt][i] - top);
                    m[nt][i] = top;
                    l[nt][i] *= f;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) { acc[nt][mt][i] *= f; acc[nt][mt][i + 2] *= f; }
                }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][i] -= m[nt][i & 1];
            // the unit's exponent needs no more than bf16's bits: two heads in one register; a NaN is left to the weights
            uint32_t top2 = pack2<true>(fmaxf(fmaxf(s[nt][0], s[nt][2]), kLeast), fmaxf(fmaxf(s[nt][1], s[nt][3]), kLeast));
#pragma unroll
            for (int o = 4; o < 32; o *= 2) top2 = max_bf16x2(top2, __shfl_xor_sync(~0u, top2, o));
            const float top[2] = {__uint_as_float(top2 << 16), __uint_as_float(top2 & 0xffff0000u)};
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][i] = ex2(s[nt][i] - top[i & 1]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                unit[nt][i] = ex2(top[i]);
                l[nt][i] = fmaf(s[nt][i] + s[nt][i + 2], unit[nt][i], l[nt][i]);
            }
        }
    }

    // One complete block; `unit` in shared memory.
    __device__ __forceinline__ void visit(const uint8_t *unit, int lane) {
        const float2 scale = *reinterpret_cast<const float2 *>(unit + 2 * kBT * D);
        float s[NT][4], odd[NT][4];        // two sums: half the length of the chain of dependent instructions
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][i] = odd[nt][i] = 0.f;
#pragma unroll
        for (int p = 0; p < (KS + 1) / 2; ++p) {
            uint32_t w[4];
            load4(unit, p, lane, w);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (2 * p + i >= KS) break;
                uint32_t a0, a1, a2, a3;
                widen<E4M3>(w[2 * i], a0, a2);
                widen<E4M3>(w[2 * i + 1], a1, a3);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma<false>(i ? odd[nt] : s[nt], a0, a1, a2, a3, q[nt][2 * p + i][0], q[nt][2 * p + i][1]);
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // the factor may overflow where no product does
                const float f = qf[nt][i & 1] * scale.x;
                s[nt][i] = (s[nt][i] + odd[nt][i]) * (f > kMost ? kMost : f);
            }
        float unit_p[NT][2];
        weigh(s, unit_p);
        refer(scale.y);
        const float vr = scale.y * inv_vref * (1.f / kUp);
        uint32_t hi[NT][2], lo[NT][2];
        uint64_t back[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float x = s[nt][2 * i] * kUp, y = s[nt][2 * i + 1] * kUp;
                hi[nt][i] = transpose(split2<false>(x, y));
                lo[nt][i] = transpose(pack2<false>(x, y));
            }
            back[nt] = pair(unit_p[nt][0] * vr, unit_p[nt][1] * vr);
        }
#pragma unroll
        for (int p = 0; p < (MT + 1) / 2; ++p) {
            uint32_t w[4];
            load4(unit + kBT * D, p, lane, w);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (2 * p + i >= MT) break;
                uint32_t a0, a1, a2, a3;
                widen<E4M3>(w[2 * i], a0, a2);
                widen<E4M3>(w[2 * i + 1], a1, a3);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float t[4];
                    mma_first<false>(t, a0, a1, a2, a3, hi[nt][0], hi[nt][1]);
                    mma<false>(t, a0, a1, a2, a3, lo[nt][0], lo[nt][1]);
                    add_scaled(acc[nt][2 * p + i], t, back[nt]);
                }
            }
        }
    }
    __device__ __forceinline__ static void load4(const uint8_t *part, int p, int lane, uint32_t (&w)[4]) {
        if (p < D / 32) {
            const uint4 v = *reinterpret_cast<const uint4 *>(part + 512 * p + 16 * lane);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
            const uint2 v = *reinterpret_cast<const uint2 *>(part + 512 * p + 8 * lane);
            w[0] = v.x; w[1] = v.y; w[2] = w[3] = 0;
        }
    }

    // A pair of 16-bit numbers with zeros for infinities and NaN.
    __device__ __forceinline__ static uint32_t numbers(uint32_t w) {
        return w & ~__vcmpgeu2(w & 0x7fff7fffu, BF16 ? 0x7f807f80u : 0x7c007c00u);
    }

    // The open block: n (1 .. 15) rows in 16 bits at k, v (global memory); later rows are not read.  Weights go in as
    // as many 16-bit terms as fp32 has bits for.
    __device__ __forceinline__ void open_block(const uint16_t *k, const uint16_t *v, int n, const uint16_t *q0, int GT,
                                               float scale_log2, int lane) {
        const int g = lane >> 2, c = lane & 3;
        if (128 * lane < n * D * 2) {      // the rows of V arrive while the scores are taken
            prefetch_l1(reinterpret_cast<const uint8_t *>(k) + 128 * lane);
            prefetch_l1(reinterpret_cast<const uint8_t *>(v) + 128 * lane);
        }
        float s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][i] = 0.f;
#pragma unroll
        for (int p = 0; p < (KS + 1) / 2; ++p) {
            const uint4 a = q_words(k + (size_t)g * D, p, c, g < n), b = q_words(k + (size_t)(g + 8) * D, p, c, g + 8 < n);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                uint4 w;                   // q as it is (in fp16 the operand in use, in bf16 that one is scaled)
                if (BF16) w = q_words(q0 + (size_t)(nt * 8 + g) * D, p, c, nt * 8 + g < GT);
                else {
                    const uint32_t (&x)[2] = q[nt][2 * p], (&y)[2] = q[nt][(2 * p + 1) % KS];
                    w = make_uint4(x[0], x[1], y[0], y[1]);
                }
                mma<BF16>(s[nt], a.x, b.x, a.y, b.y, w.x, w.y);
                if (2 * p + 1 < KS) mma<BF16>(s[nt], a.z, b.z, a.w, b.w, w.z, w.w);
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][i] = g + 8 * (i >> 1) < n ? s[nt][i] * scale_log2 : -INFINITY;   // weight 0
        float unit_p[NT][2];
        weigh(s, unit_p);
        uint32_t w[4][MT];     // dims g * D / 8 + 2 mt, + 1 of tokens 2 c, 2 c + 1, 2 c + 8, 2 c + 9
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int tok = 2 * c + (j & 1) + 8 * (j >> 1);
            const uint32_t *row = reinterpret_cast<const uint32_t *>(v + (size_t)tok * D + g * (D / 8));
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) w[j][mt] = tok < n ? row[mt] : 0u;
        }
        // bf16 needs nothing for the weights; where the values are near an end of its range, their products stay off it
        float up = kUp;
        constexpr uint32_t kInf = BF16 ? 0x7f80u : 0x7c00u;
        uint32_t top2 = 0;     // the largest magnitude
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) top2 = __vmaxu2(top2, w[j][mt] & 0x7fff7fffu);
        top2 = __reduce_max_sync(~0u, max(top2 & 0xffffu, top2 >> 16));
        const bool finite = top2 < kInf;
        if (BF16) {
            const float top = __uint_as_float(min(top2, kInf - 1) << 16);
            up = top > 0x1p100f ? 0x1p-8f : top < 0x1p-60f ? 0x1p60f : 1.f;
            refer(top);
        } else {
            refer(1.f);
        }
        constexpr int TERMS = BF16 ? 3 : 2;
        uint32_t t[TERMS][NT][2];
        uint64_t back[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float x = s[nt][2 * i] * up, y = s[nt][2 * i + 1] * up;
#pragma unroll
                for (int j = 0; j < TERMS; ++j) t[j][nt][i] = transpose(split2<BF16>(x, y));
            }
            const float f = inv_vref / up;
            back[nt] = pair(unit_p[nt][0] * f, unit_p[nt][1] * f);
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const uint32_t a0 = __byte_perm(w[0][mt], w[1][mt], 0x5410), a1 = __byte_perm(w[0][mt], w[1][mt], 0x7632);
            const uint32_t a2 = __byte_perm(w[2][mt], w[3][mt], 0x5410), a3 = __byte_perm(w[2][mt], w[3][mt], 0x7632);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float sum[4];
                mma_first<BF16>(sum, a0, a1, a2, a3, t[0][nt][0], t[0][nt][1]);
#pragma unroll
                for (int j = 1; j < TERMS; ++j) {
                    if (finite) mma<BF16>(sum, a0, a1, a2, a3, t[j][nt][0], t[j][nt][1]);
                    // an infinity has met the weight's first term and meets no remainder: that may be 0 or negative
                    else mma<BF16>(sum, numbers(a0), numbers(a1), numbers(a2), numbers(a3), t[j][nt][0], t[j][nt][1]);
                }
                add_scaled(acc[nt][mt], sum, back[nt]);
            }
        }
    }

    // Sums over the lanes that share a head.
    __device__ __forceinline__ void finish() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                l[nt][i] += __shfl_xor_sync(~0u, l[nt][i], 4);
                l[nt][i] += __shfl_xor_sync(~0u, l[nt][i], 8);
                l[nt][i] += __shfl_xor_sync(~0u, l[nt][i], 16);
            }
        if (vref == 0.f) vref = 1.f;
    }
};

// Two neighbouring output values of one head.
template <bool BF16>
__device__ __forceinline__ void store2(const AttnParams &p, size_t at, float x, float y) {
    if (p.out_f32) *reinterpret_cast<float2 *>(p.out_f32 + at) = make_float2(x, y);
    if (p.out) *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(p.out) + at) = pack2<BF16>(x, y);
}

// The first n (at most N) of some records into a running result.  A record is (m, l) and J pairs of output values, which are
// those of its own tokens alone, divided by its l: their means stay inside the range of V, where a sum over a long history
// could pass the largest number.
template <int N, int J>
__device__ __forceinline__ void merge(const float2 (&ml)[N], const float2 (&v)[N][J], int n, float &m, float &l, float2 (&o)[J]) {
    float top = m, w[N];
#pragma unroll
    for (int i = 0; i < N; ++i) top = i < n ? fmaxf(top, ml[i].x) : top;
    const float f = l * ex2(m - top);
    m = top;
    l = f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        w[i] = i < n ? ex2(ml[i].x - top) * ml[i].y : 0.f;
        l += w[i];
    }
    const float part = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int j = 0; j < J; ++j) { o[j].x *= f * part; o[j].y *= f * part; }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < n)   // and not where w is 0: a NaN stays one
#pragma unroll
            for (int j = 0; j < J; ++j) { o[j].x += w[i] * part * v[i][j].x; o[j].y += w[i] * part * v[i][j].y; }
}

// A visit as the producing lane writes it down for the whole warp.
struct Visit {
    int32_t seq, group;        // sequence, head group
    int32_t flags;             // below; the tail's row count in the upper bits
    int32_t pad;
};
enum { COPY = 1, OPEN = 2, FIRST = 4, LAST = 8, HEAD = 16, END = 32 };   // FIRST/LAST of the warp's part of an item; HEAD/END of the item itself

// Warps of a CTA: as many as the registers allow without spills that cost more than the warps bring (32 sequences x 1088
// tokens x 32 heads x 128: 61.4 us with 12, 65.3 with 11, and 16 spilled up to 90 bytes in the loop; with two tiles 12 instead of
// 8 at head_dim 64 and 80: 2 sequences of 7000 to 15287 tokens, 384 / 32 heads x 80, 57.7 -> 47.8); ring: 130 to 150 KB in flight
// per SM.
template <int D, int NT>
struct Shape {
    static constexpr int NW = NT == 2 ? (D == 128 ? 8 : 12) : D == 128 ? 12 : 16;
    static constexpr int UNIT = unit_bytes(D);
    static constexpr int ST = (D == 128 && NT == 1 ? 149 << 10 : 132 << 10) / (NW * UNIT);
    static constexpr int HT = 8 * NT;
    static constexpr int REC = HT * D / 2;     // pairs of output values in a record
    static_assert(ST >= 2 && ST <= 8, "ring depth");
    static_assert(REC * 8 <= ST * UNIT, "a record fits a warp's part of the ring");
};

template <int D, int NT, bool BF16, bool E4M3>
__global__ void __launch_bounds__(Shape<D, NT>::NW * 32, 1) attn_kernel(const __grid_constant__ AttnParams p) {
    using SH = Shape<D, NT>;
    constexpr int NW = SH::NW, UNIT = SH::UNIT, ST = SH::ST, HT = SH::HT, THREADS = NW * 32;
    extern __shared__ __align__(128) uint8_t smem[];
    uint8_t *ring = smem;                                                       // [NW][ST] units
    float2 *early = reinterpret_cast<float2 *>(ring + (size_t)NW * ST * UNIT);  // [NW][REC]: records left before a warp's end
    Visit *visits = reinterpret_cast<Visit *>(early + NW * SH::REC);            // [NW][ST]
    uint64_t *bars = reinterpret_cast<uint64_t *>(visits + NW * ST);            // [NW][ST]
    int *prefix = reinterpret_cast<int *>(bars + NW * ST);                      // [n_seqs + 1] visits of a head group before a sequence
    uint8_t *open = reinterpret_cast<uint8_t *>(prefix + p.c.n_seqs + 1);       // [n_seqs] rows of the open block
    __shared__ int scan[NW];
    __shared__ int rec_item[NW][2];            // items of which the warps left a partial result (flat: sequence, group)
    __shared__ float2 rec_ml[NW][2][HT];       // their m and l
    __shared__ int run_item[NW + 1], run_first[NW + 2], n_runs;
    __shared__ int list[2 * NW];               // records in order: 2 * warp + which
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int G = p.c.Hkv * p.P;               // head groups of a sequence

    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---- visits before each sequence: one per block, one without data at the front of each item, which is about what starting
    // and finishing an item costs, and one behind an open block, which costs two (32 ragged rows of 0 to 1152 tokens, 32
    // heads of 80: 42 us without, 36.8 with the first, 31.3 with both when chosen, 31.4 now); sequences without any block get their zeros
    uint32_t bad = 0;
    int carry = 0;
    for (int s0 = 0; s0 < p.c.n_seqs; s0 += THREADS) {
        const int s = s0 + tid;
        int nb = 0;
        if (s < p.c.n_seqs) {
            bool b;
            const int len = seq_len(p.c, s, b);
            nb = len ? (len + kBT - 1) / kBT + 1 + (len % kBT != 0) : 0;
            open[s] = (uint8_t)(len % kBT);
            if (b) bad |= ISV_STATUS_BAD_LENGTH;
        }
        int x = nb;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int y = __shfl_up_sync(~0u, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) scan[warp] = x;
        __syncthreads();
        int before = carry;
        for (int w = 0; w < NW; ++w) {
            if (w < warp) before += scan[w];
            carry += scan[w];
        }
        if (s < p.c.n_seqs) prefix[s] = before + x - nb;
        __syncthreads();
    }
    if (tid == 0) prefix[p.c.n_seqs] = carry;
    if (lane < 2) rec_item[warp][lane] = -1;
    if (lane < ST) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(s32(&bars[warp * ST + lane])) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    for (int s = blockIdx.x; s < p.c.n_seqs; s += gridDim.x)
        if (prefix[s] == prefix[s + 1])
            for (int x = 2 * tid; x < p.Hq * D; x += 2 * THREADS) store2<BF16>(p, (size_t)s * p.Hq * D + x, 0.f, 0.f);

    // range of part i of n: the first `rest` parts are one longer
    const int total = carry * G;               // below 2^31: the host checks
    // An item of V visits over C CTAs takes about V / C * 0.1 us of reading and C * 0.07 us of merging: C = 1.2 sqrt(V) has
    // the shortest sum (one sequence on one KV head: 65536 tokens 21.1 -> 18.1 us, 21041 tokens x 80 17.0 -> 12.6 when chosen;
    // 19.1 and 13.4 now).
    int cap = (int)gridDim.x;
    const long long reach = (long long)total * p.c.n_seqs * G;
    if (reach < (long long)gridDim.x * gridDim.x) cap = min(cap, p.c.n_seqs * G + (int)(1.2f * sqrtf((float)reach)));   // items * (1 + 1.2 sqrt(V))
    const int ctas = total ? min(cap, max(1, total / kMinCtaVisits)) : 0;
    if ((int)blockIdx.x >= ctas) {
        if (bad && blockIdx.x == 0) atomicOr(p.c.status, bad);
        return;
    }
    const int share = total / ctas, rest = total - share * ctas;
    auto cta_at = [&](int c) { return share * c + min(c, rest); };
    const int cta_beg = cta_at(blockIdx.x), cta_end = cta_at(blockIdx.x + 1), cta_n = cta_end - cta_beg;
    const int warps = min(NW, max(1, cta_n / kMinVisits));
    const int mine = cta_n / warps, more = cta_n - mine * warps;
    const int beg = warp < warps ? cta_beg + mine * warp + min(warp, more) : 0;
    const int end = warp < warps ? beg + mine + (warp < more ? 1 : 0) : 0;

    // ---- producer: 32 visits at a time are looked up, one per lane
    uint64_t my_src = 0;
    Visit my_visit{};
    auto look_up = [&](int v) {
        my_src = 0;
        if (v >= end) return;
        int lo = 0, hi = p.c.n_seqs;           // the last sequence whose visits begin at or before v
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (prefix[mid] * G <= v) lo = mid; else hi = mid;
        }
        const int nb = prefix[lo + 1] - prefix[lo];
        const int r = v - prefix[lo] * G, group = r / nb, at = r - group * nb, blk = at - 1;
        int flags = (v == beg || at == 0 ? FIRST : 0) | (v == end - 1 || at == nb - 1 ? LAST : 0) | (at == 0 ? HEAD : 0) |
                    (at == nb - 1 ? END : 0);
        if (blk < 0) {
        } else if (blk < nb - 1 - 2 * (open[lo] != 0)) {
            const int page = p.c.table[(size_t)lo * p.c.table_stride + blk];
            if (page >= 0 && page < p.c.n_pages) {
                my_src = reinterpret_cast<uint64_t>(p.c.pool) + ((uint64_t)page * p.c.Hkv + group / p.P) * UNIT;
                flags |= COPY;
            } else if (page != ISV_BLOCK_NONE) {
                bad |= ISV_STATUS_BAD_BLOCK_ID;
            }
        } else if (blk < nb - 2) {
            flags |= OPEN | open[lo] << 8;
        }
        my_visit = Visit{lo, group, flags, 0};
    };
    int next = beg;
    bool lost = false;                         // a copy did not arrive in time: the range is walked to its end without its data
    auto produce = [&](int slot) {             // the next visit into this slot of the ring
        if (next >= end) return;
        const int i = (next - beg) & 31;
        if (i == 0) look_up(next + lane);
        const uint64_t src = __shfl_sync(~0u, my_src, i);
        if (lane == i) visits[warp * ST + slot] = my_visit;
        if (lane == 0 && src && !lost) {
            const uint32_t bar = s32(&bars[warp * ST + slot]);
            arm(bar, UNIT);
            if (!(p.drop_first_copy && next == 1)) copy_in(s32(ring + (size_t)(warp * ST + slot) * UNIT), reinterpret_cast<const void *>(src), UNIT, bar);
        }
        ++next;
    };

    // ---- consumer
    State<D, NT, BF16, E4M3> st;
    const uint16_t *q0 = p.q;
    uint32_t phases = 0;
    int slot = 0;
    bool whole = false;
    // the first ST turns only fill the ring
#pragma unroll 1
    for (int v = beg - ST; v < end; ++v) {
        Visit t{};
        if (v >= beg) t = visits[warp * ST + slot];
        if (t.flags & FIRST) {
            q0 = p.q + ((size_t)t.seq * p.Hq + (size_t)t.group * p.GT) * D;
            st.start(q0, p.GT, p.scale_log2, lane);
            whole = t.flags & HEAD;
        }
        if (t.flags & COPY) {
            // all lanes have to agree: what a lane alone had seen arrive would split the warp at the next vote
            if (!lost && !__all_sync(~0u, wait(s32(&bars[warp * ST + slot]), (phases >> slot) & 1u, p.spin_limit))) {
                // the copies in flight get one more bounded chance, so that none lands in memory used for something else
#pragma unroll 1
                for (int i = 0; i < ST && i < end - v; ++i) {
                    const int x = (slot + i) % ST;
                    if (visits[warp * ST + x].flags & COPY) wait(s32(&bars[warp * ST + x]), (phases >> x) & 1u, kDrainLimit);
                }
                __syncwarp();
                lost = true;
                bad |= ISV_STATUS_WAIT_EXPIRED;
            }
            if (!lost) {
                phases ^= 1u << slot;
                st.visit(ring + (size_t)(warp * ST + slot) * UNIT, lane);
            }
        } else if (t.flags & OPEN) {
            const uint16_t *k = reinterpret_cast<const uint16_t *>(p.c.tails) + ((size_t)t.seq * 2 * p.c.Hkv + t.group / p.P) * kBT * D;
            st.open_block(k, k + (size_t)p.c.Hkv * kBT * D, t.flags >> 8, q0, p.GT, p.scale_log2, lane);
        }
        __syncwarp();
        produce(slot);
        if (t.flags & LAST) {
            st.finish();
            const int g = lane >> 2, c = lane & 3;
            if (whole && (t.flags & END)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int h = nt * 8 + 2 * c + i;
                        const float f = st.l[nt][i] == 0.f ? 0.f : st.vref / st.l[nt][i];
                        if (h < p.GT) {
                            const size_t at = ((size_t)t.seq * p.Hq + (size_t)t.group * p.GT + h) * D + g * (D / 8);
#pragma unroll
                            for (int mt = 0; mt < D / 16; ++mt) store2<BF16>(p, at + 2 * mt, st.acc[nt][mt][i] * f, st.acc[nt][mt][i + 2] * f);
                        }
                    }
            } else {
                // an item that begins before this warp's range leaves record 0, any other record 1
                const int which = whole ? 1 : 0;
                if (lane == 0) rec_item[warp][which] = t.seq * G + t.group;
                // a later record is this warp's last: its part of the ring is no longer in use
                float2 *o = which ? reinterpret_cast<float2 *>(ring + (size_t)warp * ST * UNIT) : early + warp * SH::REC;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (g == 0) rec_ml[warp][which][nt * 8 + 2 * c + i] = make_float2(st.m[nt][i], st.l[nt][i]);
                        const float f = st.l[nt][i] == 0.f ? 0.f : st.vref / st.l[nt][i];
#pragma unroll
                        for (int mt = 0; mt < D / 16; ++mt)
                            o[((nt * 2 + i) * (D / 16) + mt) * 32 + c * 8 + g] = make_float2(st.acc[nt][mt][i] * f, st.acc[nt][mt][i + 2] * f);
                    }
            }
        }
        slot = slot + 1 == ST ? 0 : slot + 1;
        __syncwarp();
    }
    if (bad) atomicOr(p.c.status, bad);
    __syncthreads();

    // ---- partial results of this CTA: consecutive records of one item form a run
    if (warp == 0) {
        const int w = lane;                    // warps' records in order, two a lane
        const int i0 = w < warps ? rec_item[w][0] : -1, i1 = w < warps ? rec_item[w][1] : -1;
        const unsigned h0 = __ballot_sync(~0u, i0 >= 0), h1 = __ballot_sync(~0u, i1 >= 0), below = (1u << w) - 1u;
        const int n0 = __popc(h0 & below) + __popc(h1 & below), n1 = n0 + (i0 >= 0);
        if (i0 >= 0) list[n0] = 2 * w;
        if (i1 >= 0) list[n1] = 2 * w + 1;
        // an item begins a run where its own first record is: the records of an item are neighbours in the list
        const int total_recs = __popc(h0) + __popc(h1);
        __syncwarp();
        const int r = lane < total_recs ? list[lane] : 0;
        const int item = lane < total_recs ? rec_item[r >> 1][r & 1] : -1;
        int before = __shfl_up_sync(~0u, item, 1);
        if (lane == 0) before = -1;
        const bool first = item >= 0 && item != before;
        const unsigned f = __ballot_sync(~0u, first);
        const int run = __popc(f & below);
        if (first) { run_item[run] = item; run_first[run] = lane; }
        if (lane == 0) { n_runs = __popc(f); run_first[__popc(f)] = total_recs; }
    }
    __syncthreads();
    if (n_runs == 0) return;
    // A warp merges one head of one run: lane i holds the pairs i, i + 32 of the head, in the order (tile, g): output dims
    // g * D / 8 + 2 tile, + 1.
    constexpr int MT = D / 16, PAIRS = D / 2, J = (PAIRS + 31) / 32;
    auto cta_of = [&](int v) {                 // CTA whose range holds visit v
        const int longer = rest * (share + 1);
        return v < longer ? v / (share + 1) : rest + (v - longer) / share;
    };
    auto span = [&](int item, int &b, int &e) {
        const int s = item / G, nb = prefix[s + 1] - prefix[s];
        b = prefix[s] * G + (item - s * G) * nb;
        e = b + nb;
    };
    auto put = [&](int item, int h, const float2 (&o)[J]) {
        const size_t at = ((size_t)item * p.GT + h) * D;       // item * GT + h: the flat query head
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int u = lane + 32 * j;
            if (u < PAIRS) store2<BF16>(p, at + (u % 8) * (D / 8) + 2 * (u / 8), o[j].x, o[j].y);
        }
    };
    // An item that crosses CTAs (only the first and the last of a CTA may): its CTAs' results meet in memory, and the warp
    // that brings a head's last one merges them.  The ticket is that of the item's first CTA, in which no other item
    // continues into the next.  A warp has at most 2 * 16 / 8 + 1 such heads; lane i keeps the i-th, and all their tickets
    // are drawn at once.
    int mine_x = 0, crossing = 0;
#pragma unroll 1
    for (int x = warp; x < n_runs * p.GT; x += NW) {
        const int run = x / p.GT, h = x - run * p.GT;
        const int r0 = run_first[run], r1 = run_first[run + 1], item = run_item[run];
        const int place = ((h >> 3) * 2 + (h & 1)) * MT * 32 + ((h & 7) >> 1) * 8 + lane % 8 + lane / 8 * 32;
        float m = kNone, l = 0.f;
        float2 o[J];
#pragma unroll
        for (int j = 0; j < J; ++j) o[j] = make_float2(0.f, 0.f);
#pragma unroll 1
        for (int r = r0; r < r1; r += 4) {
            float2 ml[4], v[4][J];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int rec = list[min(r + i, r1 - 1)], w = rec >> 1;
                const float2 *from = rec & 1 ? reinterpret_cast<const float2 *>(ring + (size_t)w * ST * UNIT) : early + w * SH::REC;
                ml[i] = rec_ml[w][rec & 1][h];
#pragma unroll
                for (int j = 0; j < J; ++j) v[i][j] = lane + 32 * j < PAIRS ? from[place + 128 * j] : make_float2(0.f, 0.f);
            }
            merge(ml, v, r1 - r, m, l, o);
        }
        int b, e;
        span(item, b, e);
        if (b >= cta_beg && e <= cta_end) {
            put(item, h, o);
            continue;
        }
        const int slot = blockIdx.x * 2 + (b > cta_beg ? 1 : 0);
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (lane + 32 * j < PAIRS) __stcg(reinterpret_cast<float2 *>(p.part_o) + (size_t)slot * SH::REC + h * PAIRS + lane + 32 * j, o[j]);
        if (lane == 0) __stcg(reinterpret_cast<float2 *>(p.part_ml) + slot * HT + h, make_float2(m, l));
        if (lane == crossing) mine_x = x;
        ++crossing;
    }
    if (crossing == 0) return;
    __threadfence();
    __syncwarp();
    bool last = false;
    if (lane < crossing) {
        const int run = mine_x / p.GT, h = mine_x - run * p.GT;
        int b, e;
        span(run_item[run], b, e);
        const int c0 = cta_of(b);
        int *ticket = p.tickets + c0 * HT + h;
        last = atomicAdd(ticket, 1) == cta_of(e - 1) - c0;
        if (last) *ticket = 0;
        __threadfence();
    }
    unsigned todo = __ballot_sync(~0u, last);
#pragma unroll 1
    for (; todo; todo &= todo - 1) {
        const int x = __shfl_sync(~0u, mine_x, __ffs(todo) - 1), run = x / p.GT, h = x - run * p.GT, item = run_item[run];
        int b, e;
        span(item, b, e);
        const int c0 = cta_of(b), n = cta_of(e - 1) - c0 + 1, first_slot = b == cta_at(c0) ? 0 : 1;
        float m = kNone, l = 0.f;
        float2 o[J];
#pragma unroll
        for (int j = 0; j < J; ++j) o[j] = make_float2(0.f, 0.f);
#pragma unroll 1
        for (int i = 0; i < n; i += kFly) {
            float2 ml[kFly], v[kFly][J];
#pragma unroll
            for (int y = 0; y < kFly; ++y) {
                const int z = min(i + y, n - 1), at = (c0 + z) * 2 + (z == 0 ? first_slot : 0);
                ml[y] = __ldcg(reinterpret_cast<const float2 *>(p.part_ml) + at * HT + h);
#pragma unroll
                for (int j = 0; j < J; ++j)
                    v[y][j] = lane + 32 * j < PAIRS ? __ldcg(reinterpret_cast<const float2 *>(p.part_o) + (size_t)at * SH::REC + h * PAIRS + lane + 32 * j)
                                                    : make_float2(0.f, 0.f);
            }
            merge(ml, v, n - i, m, l, o);
        }
        put(item, h, o);
    }
}

template <int D, int NT, bool BF16, bool E4M3>
cudaError_t configure(size_t smem) {
    return cudaFuncSetAttribute(attn_kernel<D, NT, BF16, E4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
}
template <int D, int NT, bool BF16, bool E4M3>
cudaError_t launch(const AttnParams &p, int grid, size_t smem, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(Shape<D, NT>::NW * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;   // see the kernel's griddepcontrol pair
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attn_kernel<D, NT, BF16, E4M3>, p);
}

// Calls f with the template arguments of a case.
template <int D, int NT, typename F>
cudaError_t pick_types(bool bf16, bool e4m3, F f) {
    if (bf16) return e4m3 ? f.template operator()<D, NT, true, true>() : f.template operator()<D, NT, true, false>();
    return e4m3 ? f.template operator()<D, NT, false, true>() : f.template operator()<D, NT, false, false>();
}
template <typename F>
cudaError_t pick(int D, int GT, bool bf16, bool e4m3, F f) {
    if (GT <= 8) {
        if (D == 64) return pick_types<64, 1>(bf16, e4m3, f);
        if (D == 80) return pick_types<80, 1>(bf16, e4m3, f);
        return pick_types<128, 1>(bf16, e4m3, f);
    }
    if (D == 64) return pick_types<64, 2>(bf16, e4m3, f);
    if (D == 80) return pick_types<80, 2>(bf16, e4m3, f);
    return pick_types<128, 2>(bf16, e4m3, f);
}
struct Configure {
    size_t smem;
    template <int D, int NT, bool BF16, bool E4M3>
    cudaError_t operator()() const { return configure<D, NT, BF16, E4M3>(smem); }
};
struct Launch {
    const AttnParams &p;
    int grid;
    size_t smem;
    cudaStream_t st;
    template <int D, int NT, bool BF16, bool E4M3>
    cudaError_t operator()() const { return launch<D, NT, BF16, E4M3>(p, grid, smem, st); }
};

}  // namespace

int attn_head_rows(int GT) { return GT <= 8 ? 8 : 16; }
int attn_slots(int grid) { return 2 * grid; }

template <int D, int NT>
size_t smem_of(int max_seqs) {
    using SH = Shape<D, NT>;
    return SH::NW * (SH::ST * (SH::UNIT + sizeof(Visit) + 8) + SH::REC * 8) + 4 * ((size_t)max_seqs + 1) + max_seqs;
}
size_t attn_smem(int D, int GT, int max_seqs) {
    if (GT <= 8) return D == 64 ? smem_of<64, 1>(max_seqs) : D == 80 ? smem_of<80, 1>(max_seqs) : smem_of<128, 1>(max_seqs);
    return D == 64 ? smem_of<64, 2>(max_seqs) : D == 80 ? smem_of<80, 2>(max_seqs) : smem_of<128, 2>(max_seqs);
}
cudaError_t attn_configure(int D, int GT, bool bf16, bool e4m3, size_t smem) { return pick(D, GT, bf16, e4m3, Configure{smem}); }
cudaError_t launch_attn(const AttnParams &p, int D, bool bf16, bool e4m3, int grid, size_t smem, cudaStream_t st) {
    return pick(D, p.GT, bf16, e4m3, Launch{p, grid, smem, st});
}

}  // namespace q8
}  // namespace isv
