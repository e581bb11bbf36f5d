// The KV cache held in 8 bits: the handle, and storing new tokens (quantisation of complete blocks).  Layout, formats and
// the treatment of open blocks are described in include/isv.h; the attention kernel is in isv_q8_attn.cu.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>

#include "../../include/isv.h"
#include "isv_kernels.cuh"
#include "isv_q8.cuh"

namespace isv {
int set_error(int code, const char *msg);
}

namespace {

using isv::q8::add2;
using isv::q8::AttnParams;
using isv::q8::CacheParams;
using isv::q8::fma2;
using isv::q8::kBT;
using isv::q8::mul2;
using isv::q8::pair;
using isv::q8::seq_len;
using isv::q8::unit_bytes;
using isv::q8::unpair;

int err(int code, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return isv::set_error(code, buf);
}

// Makes a device current for the length of a call.
struct OnDevice {
    int before = -1;
    cudaError_t e;
    explicit OnDevice(int dev) {
        e = cudaGetDevice(&before);
        if (e == cudaSuccess && before != dev) e = cudaSetDevice(dev);
        else if (e == cudaSuccess) before = -1;
    }
    ~OnDevice() {
        if (before >= 0) cudaSetDevice(before);
    }
};

constexpr uint32_t kSpinLimit = 1u << 22;   // polls before a wait of the attention kernel gives up, unless isv_q8_set_wait_limit says otherwise
constexpr int kWriteThreads = 128;
constexpr int kStaticSmem = 4096;   // room for what the attention kernel declares besides its dynamic shared memory

struct WriteParams {
    CacheParams c;
    const int32_t *new_lens;    // NULL = T
    const uint16_t *k, *v;
    int64_t seq_stride, token_stride;
    int32_t T, blocks;          // blocks: how many blocks T tokens can touch
};

// ---- quantisation
//
// A code is the rounding of the exact quotient x / s.  The kernel multiplies by 1 / s: that product is off by at most
// 2^-23 of its value, so its rounding is the right one unless it lies that close to the border m between two codes.  There the
// sign of x - m * s decides, which one fused multiply-add gives exactly (m has at most eight bits; the caller keeps x
// and s in the normal range): 0 is a tie.  Ties are common, x = absmax / 2 is one for int8, and with eight bits of bf16 so
// are others: nearly every word of a block has one.

constexpr float kMagic = 12582912.f;   // 1.5 * 2^23: adding it rounds to an integer, which is then in the low bits

// e4m3 keeps three bits behind the leading one, and below 2^-6 the steps that it has at 2^-6: |q|, below 2^-6 raised by 2^-6,
// has its borders where the last 20 bits are 0x80000.
__device__ __forceinline__ float raised(float q) {
    const float a = fabsf(q);
    return a < 0x1p-6f ? a + 0x1p-6f : a;
}
template <bool E4M3>
__device__ __forceinline__ bool near_border(float q) {
    if (E4M3) return ((__float_as_uint(raised(q)) - 0x7fffcu) & 0xfffffu) <= 8u;
    return fabsf(q - ((q + kMagic) - kMagic)) > 0.49998f;             // |q| <= 127: off by at most 1.6e-5
}
// A number that rounds as x / s does, where q = x * (1 / s) lies near a border.
template <bool E4M3>
__device__ __forceinline__ float settle(float q, float x, float s) {
    if (!near_border<E4M3>(q)) return q;
    if (E4M3) {
        const float low = fabsf(q) < 0x1p-6f ? 0x1p-6f : 0.f;
        const uint32_t border = (__float_as_uint(raised(q)) & 0xfff00000u) | 0x80000u;
        const float e = __fmaf_rn(-(__uint_as_float(border) - low), s, fabsf(x));
        const float y = __uint_as_float(border + (e > 0.f ? 0x1000u : e < 0.f ? ~0xfffu : 0u)) - low;
        return copysignf(y, q);
    }
    const float m = ((q - 0.5f) + kMagic) - kMagic + 0.5f, e = __fmaf_rn(-m, s, x);
    return e > 0.f ? m + 0.25f : e < 0.f ? m - 0.25f : m;
}

__device__ __forceinline__ uint32_t low_bytes(const float2 (&r)[2]) {
    return __byte_perm(__byte_perm(__float_as_uint(r[0].x), __float_as_uint(r[0].y), 0x0040),
                       __byte_perm(__float_as_uint(r[1].x), __float_as_uint(r[1].y), 0x0040), 0x5410);
}
// Four numbers -> four codes, in the bytes of a word.
template <bool E4M3>
__device__ __forceinline__ uint32_t codes_of(const float2 (&q)[2]) {
    uint32_t w;
    if (E4M3) {
        asm("{\n.reg .b16 a, b;\ncvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\ncvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\nmov.b32 %0, {a, b};\n}\n"
            : "=r"(w) : "f"(q[0].x), "f"(q[0].y), "f"(q[1].x), "f"(q[1].y));
    } else {
        const float2 r[2] = {make_float2(q[0].x + kMagic, q[0].y + kMagic), make_float2(q[1].x + kMagic, q[1].y + kMagic)};
        w = low_bytes(r);
    }
    return w;
}
// The four int8 codes of numbers some of which may lie next to a border.  A call of its own: inlined sixteen times it made the
// kernel's code so long that a prompt of 16 x 1024 tokens x 32 heads took 109 us instead of 86.  With e4m3 it is inlined:
// nearly every word needs it, and an append of one token to 256 sequences takes 8.6 us instead of 10.4.
__device__ __noinline__ uint32_t int8_settled(float a, float b, float c, float d, float s, float inv) {
    const float2 q[2] = {make_float2(settle<false>(a * inv, a, s), settle<false>(b * inv, b, s)),
                         make_float2(settle<false>(c * inv, c, s), settle<false>(d * inv, d, s))};
    return codes_of<false>(q);
}
// up: the power of two by which numbers and scale are multiplied, for blocks so small that the arithmetic would leave the
// normal range (s and inv have it already).
template <bool E4M3>
__device__ __forceinline__ uint32_t encode(const float2 (&x)[2], float s, float inv, float up) {
    const uint64_t inv2 = pair(inv, inv);
    bool close = up != 1.f;
    float2 q[2], r[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint64_t v = pair(x[i].x, x[i].y);
        if (E4M3) {
            q[i] = unpair(mul2(v, inv2));
            close = close || near_border<true>(q[i].x) || near_border<true>(q[i].y);
        } else {   // t: rounded to the integer n, which is in its low bits; d: how far the quotient is from n
            const uint64_t t = fma2(v, inv2, pair(kMagic, kMagic)), n = add2(t, pair(-kMagic, -kMagic));
            const float2 d = unpair(fma2(v, inv2, mul2(n, pair(-1.f, -1.f))));
            r[i] = unpair(t);
            close = close || fabsf(d.x) > 0.49998f || fabsf(d.y) > 0.49998f;
        }
    }
    if (!E4M3) return close ? int8_settled(x[0].x * up, x[0].y * up, x[1].x * up, x[1].y * up, s, inv) : low_bytes(r);
    if (close)
#pragma unroll
        for (int i = 0; i < 2; ++i)
            q[i] = make_float2(settle<true>(x[i].x * up * inv, x[i].x * up, s), settle<true>(x[i].y * up * inv, x[i].y * up, s));
    return codes_of<true>(q);
}

template <bool BF16>
__device__ __forceinline__ float half_of(uint32_t w, int i) {   // the low (0) or high (1) 16-bit number of a word
    if (BF16) return __uint_as_float(i ? w & 0xffff0000u : w << 16);
    return __half2float(__ushort_as_half((unsigned short)(i ? w >> 16 : w & 0xffffu)));
}

// Quantises a complete block's K (V = false) or V part: `row(t)` is the address of token t's row, `unit` the block's place.
// A lane's loads are the 16-bit rows in the order in which the page wants its codes: lane 4 g + c takes tokens g, g + 8 of K,
// 8 dims at a time, and dims g * D / 8 .. of tokens 2 c, 2 c + 1, 2 c + 8, 2 c + 9 of V; what it writes are 16-byte pieces, 512
// contiguous bytes of the warp.
template <int D, bool BF16, bool E4M3, bool V, typename Rows>
__device__ __forceinline__ void quantise(Rows row, uint8_t *unit, int lane) {
    constexpr int MT = D / 16, P = D / 32, REST = D % 32 ? 1 : 0;
    const int g = lane >> 2, c = lane & 3;
    // r[2 * MT * i + ..]: K: the lane's words of token g + 8 i; V: r[MT * j + ..]: those of the lane's j-th token
    uint32_t r[4 * MT];
    if (!V) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint16_t *at = row(g + 8 * i);
#pragma unroll
            for (int x = 0; x < P; ++x) {
                const uint4 w = *reinterpret_cast<const uint4 *>(at + 32 * x + 8 * c);
                r[2 * MT * i + 4 * x] = w.x; r[2 * MT * i + 4 * x + 1] = w.y; r[2 * MT * i + 4 * x + 2] = w.z; r[2 * MT * i + 4 * x + 3] = w.w;
            }
            if (REST) {
                const uint2 w = *reinterpret_cast<const uint2 *>(at + 32 * P + 4 * c);
                r[2 * MT * i + 4 * P] = w.x; r[2 * MT * i + 4 * P + 1] = w.y;
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint16_t *at = row(2 * c + (j & 1) + 8 * (j >> 1)) + g * (D / 8);
            if (D % 64 == 0) {
#pragma unroll
                for (int x = 0; x < MT / 4; ++x) {
                    const uint4 w = *reinterpret_cast<const uint4 *>(at + 8 * x);
                    r[MT * j + 4 * x] = w.x; r[MT * j + 4 * x + 1] = w.y; r[MT * j + 4 * x + 2] = w.z; r[MT * j + 4 * x + 3] = w.w;
                }
            } else {
#pragma unroll
                for (int x = 0; x < MT; ++x) r[MT * j + x] = *reinterpret_cast<const uint32_t *>(at + 2 * x);
            }
        }
    }
    uint32_t top2 = 0;                                   // magnitudes of 16-bit floats order like their bits
#pragma unroll
    for (int x = 0; x < 4 * MT; ++x) top2 = __vmaxu2(top2, r[x] & 0x7fff7fffu);
#pragma unroll
    for (int o = 16; o; o /= 2) top2 = __vmaxu2(top2, __shfl_xor_sync(~0u, top2, o));
    const uint32_t bits = max(top2 & 0xffffu, top2 >> 16);
    const float top = half_of<BF16>(bits, 0);
    const bool odd = bits >= (BF16 ? 0x7f80u : 0x7c00u); // an infinity or a NaN: codes of 0 and the scale NaN
    const float scale = odd ? __int_as_float(0x7fffffff) : __fdiv_rn(top, E4M3 ? 448.f : 127.f);
    const float up = top < 0x1p-60f ? 0x1p64f : 1.f, s_up = scale * up;
    const bool zeros = odd || top == 0.f;
    const float inv = zeros ? 0.f : __fdiv_rn(1.f, s_up);
    uint8_t *part = unit + (V ? kBT * D : 0);
#pragma unroll
    for (int x = 0; x < P + REST; ++x) {
        uint32_t w[4] = {0, 0, 0, 0};
        if (!zeros) {
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int t = 2 * x + y / 2, i = y & 1;  // K: k-step t, token g + 8 i; V: tile t, dim 2 t + i of the lane's
                if (t >= MT) continue;
                float2 n[2];
                if (V) {
                    n[0] = make_float2(half_of<BF16>(r[t], i), half_of<BF16>(r[MT + t], i));
                    n[1] = make_float2(half_of<BF16>(r[2 * MT + t], i), half_of<BF16>(r[3 * MT + t], i));
                } else {
                    const uint32_t a = r[2 * MT * i + 2 * t], b = r[2 * MT * i + 2 * t + 1];
                    n[0] = make_float2(half_of<BF16>(a, 0), half_of<BF16>(a, 1));
                    n[1] = make_float2(half_of<BF16>(b, 0), half_of<BF16>(b, 1));
                }
                w[y] = encode<E4M3>(n, s_up, inv, up);
            }
        }
        if (x < P) *reinterpret_cast<uint4 *>(part + 512 * x + 16 * lane) = make_uint4(w[0], w[1], w[2], w[3]);
        else *reinterpret_cast<uint2 *>(part + 512 * x + 8 * lane) = make_uint2(w[0], w[1]);
    }
    if (lane == 0) {
        float *tags = reinterpret_cast<float *>(unit + 2 * kBT * D);
        tags[V] = scale;
        tags[2 + V] = 0.f;
    }
}

// A warp per (sequence, block that its new tokens touch, KV head, K or V).  Measured on B200: 16 prompts of 1024 tokens on
// average, 32 heads x 128, fp16 to int8: 86.7 us, 4.6 TB/s of rows read and codes written, with 57 % of the issue slots and
// 50 % of HBM busy, so bound by latency (a warp has nothing in flight while it encodes); one token for each of 256 sequences, 8 heads x 128, bf16 to e4m3: 9.1 us, the latency of the blocks it completes (2.4
// where none is).
template <int D, bool BF16, bool E4M3>
__global__ void __launch_bounds__(kWriteThreads) write_kernel(const __grid_constant__ WriteParams p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const int task = blockIdx.x * (kWriteThreads / 32) + threadIdx.x / 32, s = blockIdx.y;
    const int kv = task & 1, bi = (task >> 1) / p.c.Hkv, h = (task >> 1) - bi * p.c.Hkv;
    if (bi >= p.blocks) return;
    bool bad;
    const int len = seq_len(p.c, s, bad);
    const int asked = p.new_lens ? p.new_lens[s] : p.T;
    const int n_new = min(max(asked, 0), min(p.T, len));
    if ((bad || n_new != asked) && task == 0 && lane == 0) atomicOr(p.c.status, ISV_STATUS_BAD_LENGTH);
    const int start = len - n_new, b = start / kBT + bi, last = (len - 1) / kBT;
    if (n_new == 0 || b > last) return;
    uint16_t *tail = reinterpret_cast<uint16_t *>(p.c.tails) + (((size_t)s * 2 + kv) * p.c.Hkv + h) * kBT * D;
    const uint16_t *src = (kv ? p.v : p.k) + s * p.seq_stride + (size_t)h * D;
    if ((b + 1) * kBT <= len) {
        const int page = p.c.table[(size_t)s * p.c.table_stride + b];
        if (page < 0 || page >= p.c.n_pages) {
            if (lane == 0) atomicOr(p.c.status, ISV_STATUS_BAD_BLOCK_ID);
        } else {
            auto row = [&](int t) {                      // rows before `start` wait in the tail slot
                const int pos = b * kBT + t;
                return pos < start ? tail + t * D : src + (pos - start) * p.token_stride;
            };
            uint8_t *unit = p.c.pool + ((size_t)page * p.c.Hkv + h) * unit_bytes(D);
            if (kv) quantise<D, BF16, E4M3, true>(row, unit, lane);
            else quantise<D, BF16, E4M3, false>(row, unit, lane);
        }
    }
    // ---- the open block's new rows into the tail slot.  Where the first block completes with rows from the tail slot, its warp
    // stores them, after it has read those.
    if (len % kBT == 0 || (start % kBT == 0 ? b != last : bi != 0)) return;
    __syncwarp();
    const int from = max(start, last * kBT);
    for (int i = lane; i < (len - from) * (D / 8); i += 32) {
        const int x = i % (D / 8), t = i / (D / 8) + from;
        const uint4 w = *reinterpret_cast<const uint4 *>(src + (t - start) * p.token_stride + 8 * x);
        *reinterpret_cast<uint4 *>(tail + (t - last * kBT) * D + 8 * x) = w;
    }
}

template <int D>
cudaError_t launch_write(const WriteParams &p, bool bf16, bool e4m3, dim3 grid, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kWriteThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;   // see the kernel's griddepcontrol pair
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (bf16) return e4m3 ? cudaLaunchKernelEx(&cfg, write_kernel<D, true, true>, p) : cudaLaunchKernelEx(&cfg, write_kernel<D, true, false>, p);
    return e4m3 ? cudaLaunchKernelEx(&cfg, write_kernel<D, false, true>, p) : cudaLaunchKernelEx(&cfg, write_kernel<D, false, false>, p);
}

}  // namespace

struct isv_q8 {
    isv_q8_desc d{};
    int device = 0;
    int GT = 1, P = 1;            // query heads of a visit, visits that share a block
    int grid = 1;
    int smem_optin = 0;
    uint32_t *status = nullptr;
    float *part_o = nullptr, *part_ml = nullptr;   // the attention's partial results
    int32_t *tickets = nullptr;
    std::atomic<uint32_t> wait_polls{kSpinLimit};
    std::atomic<int32_t> lost_copies{0};           // failure injection: attention launches still to lose a copy
};

namespace {

bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

// The checks that both calls share.
int check_cache(const char *who, const isv_q8 *h, const void *pool, int32_t n_pages, const void *tails, const int32_t *table,
                int32_t stride, int32_t max_blocks, const int32_t *lens, int32_t n_seqs) {
    if (!h) return err(ISV_EINVAL, "null handle");
    if (!pool || !tails || !table || !lens) return err(ISV_EINVAL, "%s: pool, tails, table and lengths are required", who);
    if (misaligned(pool) || misaligned(tails)) return err(ISV_EINVAL, "%s: pool and tails must be 16-byte aligned", who);
    if (n_seqs < 0 || n_seqs > h->d.max_seqs) return err(ISV_EINVAL, "%s: n_seqs (%d) must be in [0, %d]", who, n_seqs, h->d.max_seqs);
    // the longest length that a row of max_blocks allows, 16 * max_blocks + 15, is rounded up to whole blocks in 32 bits
    if (n_pages < 1 || max_blocks < 1 || stride < max_blocks || max_blocks >= (1 << 27) - 1)
        return err(ISV_EINVAL, "%s: bad page count (%d) or table row (%d entries, stride %d)", who, n_pages, max_blocks, stride);
    return ISV_OK;
}

CacheParams cache_params(const isv_q8 *h, const void *pool, int32_t n_pages, const void *tails, const int32_t *table,
                         int32_t stride, int32_t max_blocks, const int32_t *lens, int32_t n_seqs) {
    CacheParams c{};
    c.pool = static_cast<uint8_t *>(const_cast<void *>(pool));
    c.tails = static_cast<uint8_t *>(const_cast<void *>(tails));
    c.table = table; c.lens = lens; c.status = h->status;
    c.table_stride = stride; c.max_blocks = max_blocks; c.n_pages = n_pages; c.n_seqs = n_seqs; c.Hkv = h->d.kv_heads;
    return c;
}

}  // namespace

extern "C" {

int isv_q8_sizes(int32_t kv_heads, int32_t head_dim, uint64_t *page_bytes, uint64_t *tail_bytes) {
    if (kv_heads < 1 || (head_dim != 64 && head_dim != 80 && head_dim != 128))
        return err(ISV_EINVAL, "isv_q8_sizes: kv_heads >= 1 and head_dim 64/80/128 only");
    if (page_bytes) *page_bytes = (uint64_t)kv_heads * unit_bytes(head_dim);
    if (tail_bytes) *tail_bytes = (uint64_t)kv_heads * 2 * kBT * head_dim * 2;
    return ISV_OK;
}

int isv_q8_free(isv_q8 *h) {
    if (!h) return err(ISV_EINVAL, "null handle");
    OnDevice on(h->device);
    cudaDeviceSynchronize();   // calls may have been made on any stream
    cudaFree(h->status);
    cudaFree(h->part_o);
    cudaFree(h->part_ml);
    cudaFree(h->tickets);
    delete h;
    return ISV_OK;
}

int isv_q8_create(isv_q8 **out, const isv_q8_desc *desc) {
    if (!out) return err(ISV_EINVAL, "out is null");
    *out = nullptr;
    if (!desc) return err(ISV_EINVAL, "desc is null");
    if (desc->kv_heads < 1 || desc->q_heads < 1 || desc->q_heads % desc->kv_heads != 0)
        return err(ISV_EINVAL, "isv_q8_create: q_heads must be a positive multiple of kv_heads");
    if (desc->q_heads > 65536) return err(ISV_EINVAL, "isv_q8_create: at most 65536 query heads");
    if (desc->head_dim != 64 && desc->head_dim != 80 && desc->head_dim != 128)
        return err(ISV_EINVAL, "isv_q8_create: head_dim 64/80/128 only");
    if ((desc->dtype != ISV_F16 && desc->dtype != ISV_BF16) || (desc->format != ISV_Q8_INT8 && desc->format != ISV_Q8_E4M3))
        return err(ISV_EINVAL, "isv_q8_create: dtype f16/bf16, format int8/e4m3 only");
    if (desc->max_seqs < 1 || desc->max_seqs > 4096 || desc->max_ctas < 0)
        return err(ISV_EINVAL, "isv_q8_create: max_seqs must be in [1, 4096], max_ctas not negative");
    isv_q8 *h = new (std::nothrow) isv_q8();
    if (!h) return err(ISV_EINVAL, "out of host memory");
    h->d = *desc;
    const int G = desc->q_heads / desc->kv_heads, D = desc->head_dim;
    h->GT = isv::group_heads(G);
    h->P = G / h->GT;
    int sms = 0;
    cudaError_t e = cudaGetDevice(&h->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, h->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->smem_optin, cudaDevAttrMaxSharedMemoryPerBlockOptin, h->device);
    h->grid = desc->max_ctas > 0 ? std::min(desc->max_ctas, sms) : sms;   // one CTA per SM
    if (e == cudaSuccess && isv::q8::attn_smem(D, h->GT, desc->max_seqs) + kStaticSmem > (size_t)h->smem_optin) {
        delete h;
        return err(ISV_EINVAL, "isv_q8_create: shared memory too small for this shape");
    }
    const size_t rows = (size_t)isv::q8::attn_slots(h->grid) * isv::q8::attn_head_rows(h->GT);
    if (e == cudaSuccess) e = isv::q8::attn_configure(D, h->GT, desc->dtype == ISV_BF16, desc->format == ISV_Q8_E4M3, h->smem_optin - kStaticSmem);
    if (e == cudaSuccess) e = cudaMalloc((void **)&h->status, 4);
    if (e == cudaSuccess) e = cudaMemset(h->status, 0, 4);
    if (e == cudaSuccess) e = cudaMalloc((void **)&h->part_o, rows * D * 4);
    if (e == cudaSuccess) e = cudaMalloc((void **)&h->part_ml, rows * 2 * 4);
    const size_t tickets = (size_t)h->grid * isv::q8::attn_head_rows(h->GT) * 4;
    if (e == cudaSuccess) e = cudaMalloc((void **)&h->tickets, tickets);
    if (e == cudaSuccess) e = cudaMemset(h->tickets, 0, tickets);
    if (e == cudaSuccess) e = cudaDeviceSynchronize();   // the zeros are there before any stream's first call
    if (e != cudaSuccess) {
        cudaGetLastError();
        isv_q8_free(h);
        return err(e == cudaErrorMemoryAllocation ? ISV_ENOMEM_DEVICE : ISV_ECUDA, "isv_q8_create: %s", cudaGetErrorString(e));
    }
    *out = h;
    return ISV_OK;
}

int isv_q8_write(isv_q8 *h, void *pool_dev, int32_t n_pages, void *tails_dev, const int32_t *block_table_dev,
                 int32_t table_stride, int32_t max_blocks_per_seq, const int32_t *seq_lens_dev,
                 const int32_t *new_lens_dev, const void *k_dev, const void *v_dev, int64_t seq_stride,
                 int64_t token_stride, int32_t n_seqs, int32_t T, void *stream) {
    int rc = check_cache("isv_q8_write", h, pool_dev, n_pages, tails_dev, block_table_dev, table_stride, max_blocks_per_seq,
                         seq_lens_dev, n_seqs);
    if (rc) return rc;
    if (!k_dev || !v_dev || misaligned(k_dev) || misaligned(v_dev))
        return err(ISV_EINVAL, "isv_q8_write: k and v must be non-null, 16-byte aligned");
    if (T < 0 || T > (1 << 30)) return err(ISV_EINVAL, "isv_q8_write: bad T (%d)", T);
    if (seq_stride % 8 || token_stride % 8 || seq_stride < 0 || token_stride < 0)
        return err(ISV_EINVAL, "isv_q8_write: strides must be non-negative multiples of 8 elements");
    if (n_seqs == 0 || T == 0) return ISV_OK;
    WriteParams p{};
    p.c = cache_params(h, pool_dev, n_pages, tails_dev, block_table_dev, table_stride, max_blocks_per_seq, seq_lens_dev, n_seqs);
    p.new_lens = new_lens_dev;
    p.k = static_cast<const uint16_t *>(k_dev);
    p.v = static_cast<const uint16_t *>(v_dev);
    p.seq_stride = seq_stride; p.token_stride = token_stride; p.T = T;
    p.blocks = (T + kBT - 2) / kBT + 1;
    const bool bf16 = h->d.dtype == ISV_BF16, e4m3 = h->d.format == ISV_Q8_E4M3;
    const long long tasks = 2ll * p.blocks * h->d.kv_heads, per = kWriteThreads / 32;
    if (tasks >= (1ll << 31) - per) return err(ISV_EINVAL, "isv_q8_write: T * kv_heads too large");
    const dim3 grid((unsigned)((tasks + per - 1) / per), (unsigned)n_seqs);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    OnDevice on(h->device);
    if (on.e != cudaSuccess) return err(ISV_ECUDA, "isv_q8_write: %s", cudaGetErrorString(on.e));
    const cudaError_t e = h->d.head_dim == 64   ? launch_write<64>(p, bf16, e4m3, grid, st)
                          : h->d.head_dim == 80 ? launch_write<80>(p, bf16, e4m3, grid, st)
                                                : launch_write<128>(p, bf16, e4m3, grid, st);
    return e == cudaSuccess ? ISV_OK : err(ISV_ECUDA, "isv_q8_write: %s", cudaGetErrorString(e));
}

int isv_q8_attn(isv_q8 *h, const void *pool_dev, int32_t n_pages, const void *tails_dev, const int32_t *block_table_dev,
                int32_t table_stride, int32_t max_blocks_per_seq, const int32_t *seq_lens_dev, const void *q_dev,
                void *out_dev, float *out_f32_dev, int32_t n_seqs, void *stream) {
    int rc = check_cache("isv_q8_attn", h, pool_dev, n_pages, tails_dev, block_table_dev, table_stride, max_blocks_per_seq,
                         seq_lens_dev, n_seqs);
    if (rc) return rc;
    if (!q_dev || (!out_dev && !out_f32_dev)) return err(ISV_EINVAL, "isv_q8_attn: q and one output are required");
    if (misaligned(q_dev) || misaligned(out_dev) || misaligned(out_f32_dev))
        return err(ISV_EINVAL, "isv_q8_attn: q and outputs must be 16-byte aligned");
    if (n_seqs == 0) return ISV_OK;
    const long long groups = (long long)h->d.kv_heads * h->P;
    if (((long long)max_blocks_per_seq + 3) * n_seqs * groups >= (1ll << 31))
        return err(ISV_EINVAL, "isv_q8_attn: n_seqs * blocks * heads too large");
    AttnParams p{};
    p.c = cache_params(h, pool_dev, n_pages, tails_dev, block_table_dev, table_stride, max_blocks_per_seq, seq_lens_dev, n_seqs);
    p.q = static_cast<const uint16_t *>(q_dev);
    p.out = out_dev; p.out_f32 = out_f32_dev;
    p.part_o = h->part_o; p.part_ml = h->part_ml; p.tickets = h->tickets;
    p.Hq = h->d.q_heads; p.P = h->P; p.GT = h->GT;
    p.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)h->d.head_dim));
    p.spin_limit = h->wait_polls.load();
    if (h->lost_copies.load() > 0) p.drop_first_copy = h->lost_copies.fetch_sub(1) > 0;
    OnDevice on(h->device);
    if (on.e != cudaSuccess) return err(ISV_ECUDA, "isv_q8_attn: %s", cudaGetErrorString(on.e));
    cudaError_t e = isv::q8::launch_attn(p, h->d.head_dim, h->d.dtype == ISV_BF16, h->d.format == ISV_Q8_E4M3, h->grid,
                                         isv::q8::attn_smem(h->d.head_dim, h->GT, n_seqs), static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? ISV_OK : err(ISV_ECUDA, "isv_q8_attn: %s", cudaGetErrorString(e));
}

int isv_q8_status(isv_q8 *h, void *stream, uint32_t *status_out) {
    if (!h || !status_out) return err(ISV_EINVAL, "null argument");
    OnDevice on(h->device);
    if (on.e != cudaSuccess) return err(ISV_ECUDA, "isv_q8_status: %s", cudaGetErrorString(on.e));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaMemcpyAsync(status_out, h->status, 4, cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e == cudaSuccess && *status_out) {
        e = cudaMemsetAsync(h->status, 0, 4, st);
        if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    }
    if (e != cudaSuccess) return err(ISV_ECUDA, "isv_q8_status: %s", cudaGetErrorString(e));
    if (*status_out) return err(ISV_EDEVICE_STATUS, "a call on the 8-bit cache reported status 0x%x", *status_out);
    return ISV_OK;
}

int isv_q8_set_wait_limit(isv_q8 *h, uint32_t polls) {
    if (!h) return err(ISV_EINVAL, "null handle");
    h->wait_polls = polls ? polls : kSpinLimit;
    return ISV_OK;
}

int isv_q8_inject_lost_copy(isv_q8 *h, int32_t launches) {
    if (!h) return err(ISV_EINVAL, "null handle");
    if (launches < 0) return err(ISV_EINVAL, "launches must not be negative");
    h->lost_copies = launches;
    return ISV_OK;
}

}  // extern "C"
