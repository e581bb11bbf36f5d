// The KV cache held in 8 bits: the handle, and storing new tokens (quantisation of complete blocks).  Layout, formats and
// the treatment of open blocks are described in include/isv.h; the attention kernel is in isv_q8_attn.cu.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <algorithm>
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

using isv::q8::AttnParams;
using isv::q8::CacheParams;
using isv::q8::kBT;
using isv::q8::seq_len;
using isv::q8::unit_bytes;

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

struct WriteParams {
    CacheParams c;
    const int32_t *new_lens;    // NULL = T
    const uint16_t *k, *v;
    int64_t seq_stride, token_stride;
    int32_t T, blocks;          // blocks: how many blocks T tokens can touch
    int32_t bf16, e4m3;
};

__device__ __forceinline__ float to_f32(uint16_t b, int bf16) {
    return bf16 ? __bfloat162float(__ushort_as_bfloat16(b)) : __half2float(__ushort_as_half(b));
}

// Byte of (token, dim) inside a unit's K part and inside its V part.
__device__ __forceinline__ int k_byte(int t, int x, int d) {
    const int whole = d / 32;
    const int p = x / 32, h = t / 8, g = t % 8;
    if (p < whole) {
        const int c = (x % 32) / 8, i = (x % 8) / 4, j = x % 4;
        return 512 * p + 16 * (4 * g + c) + 8 * i + 4 * h + j;
    }
    const int r = x - 32 * whole;
    return 512 * whole + 8 * (4 * g + r / 4) + 4 * h + r % 4;
}
__device__ __forceinline__ int v_byte(int t, int x, int d) {
    const int whole = d / 32;
    const int g = x / (d / 8), r = x % (d / 8), tile = r / 2, h = r % 2;
    const int c = (t % 8) / 2, j = t % 2 + 2 * (t / 8), lane = 4 * g + c;
    if (tile < 2 * whole) return 512 * (tile / 2) + 16 * lane + 8 * (tile % 2) + 4 * h + j;
    return 512 * whole + 8 * lane + 4 * h + j;
}

// x / s rounded so that a later rounding to fewer bits gives what it gives for the exact quotient: the fp32
// quotient, and where that is inexact and its last bit is 0 the neighbour on the side of the exact value ("round
// to odd").  The residual is exact: x has at most 11 significant bits and the caller keeps s and x in the normal range.
// Quotients below 2^-20 become the code 0 whatever their last bits.
__device__ __forceinline__ float quotient_to_odd(float x, float s) {
    const float q = __fdiv_rn(x, s);
    const float r = __fmaf_rn(-q, s, x);
    uint32_t b = __float_as_uint(q);
    if (fabsf(q) > 0x1p-20f && r != 0.f && !(b & 1u)) b += ((r > 0.f) == (q > 0.f)) ? 1u : ~0u;   // away from zero, or toward it
    return __uint_as_float(b);
}
__device__ __forceinline__ uint8_t encode(float q, int e4m3) {
    if (e4m3) return (uint8_t)__nv_cvt_float_to_fp8(q, __NV_SATFINITE, __NV_E4M3);
    return (uint8_t)(int8_t)max(-127, min(127, __float2int_rn(q)));
}

// One thread per (sequence, head) walks the blocks that the new tokens touch.
__global__ void write_kernel(WriteParams p, int D) {
    const int id = blockIdx.x * blockDim.x + threadIdx.x;
    if (id >= p.c.n_seqs * p.c.Hkv) return;
    const int s = id / p.c.Hkv, h = id % p.c.Hkv;
    bool bad;
    const int len = seq_len(p.c, s, bad);
    const int asked = p.new_lens ? p.new_lens[s] : p.T;
    const int n_new = min(max(asked, 0), min(p.T, len));
    if (bad || n_new != asked) atomicOr(p.c.status, ISV_STATUS_BAD_LENGTH);
    if (n_new == 0) return;
    const int start = len - n_new;
    for (int b = start / kBT; b <= (len - 1) / kBT; ++b) {
        const bool complete = (b + 1) * kBT <= len;
        uint8_t *unit = nullptr;
        if (complete) {
            const int page = p.c.table[(size_t)s * p.c.table_stride + b];
            if (page < 0 || page >= p.c.n_pages) {
                atomicOr(p.c.status, ISV_STATUS_BAD_BLOCK_ID);
                continue;
            }
            unit = p.c.pool + ((size_t)page * p.c.Hkv + h) * unit_bytes(D);
        }
        for (int kv = 0; kv < 2; ++kv) {
            uint16_t *tail = reinterpret_cast<uint16_t *>(p.c.tails) + (((size_t)s * 2 + kv) * p.c.Hkv + h) * kBT * D;
            const uint16_t *src = (kv ? p.v : p.k) + s * p.seq_stride + (size_t)h * D;
            auto row = [&](int t) {
                const int pos = b * kBT + t;
                return pos < start ? tail + t * D : src + (pos - start) * p.token_stride;
            };
            if (!complete) {
                for (int t = 0; b * kBT + t < len; ++t)
                    if (b * kBT + t >= start)
                        for (int x = 0; x < D; ++x) tail[t * D + x] = row(t)[x];
                continue;
            }
            float top = 0.f;
            bool odd = false;
            for (int t = 0; t < kBT; ++t)
                for (int x = 0; x < D; ++x) {
                    const float a = fabsf(to_f32(row(t)[x], p.bf16));
                    odd = odd || !(a <= 3.4e38f);
                    top = fmaxf(top, a);
                }
            // tiny blocks are scaled by a power of two so that the quotients' steps stay in the normal range
            const float scale = odd ? __int_as_float(0x7fffffff) : __fdiv_rn(top, p.e4m3 ? 448.f : 127.f);
            const float up = top < 0x1p-60f ? 0x1p64f : 1.f;
            for (int t = 0; t < kBT; ++t)
                for (int x = 0; x < D; ++x) {
                    const float q = odd || top == 0.f ? 0.f : quotient_to_odd(to_f32(row(t)[x], p.bf16) * up, scale * up);
                    unit[kv * kBT * D + (kv ? v_byte(t, x, D) : k_byte(t, x, D))] = encode(q, p.e4m3);
                }
            float *tags = reinterpret_cast<float *>(unit + 2 * kBT * D);
            tags[kv] = scale;
            tags[2 + kv] = 0.f;
        }
    }
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
    if (n_pages < 1 || max_blocks < 1 || stride < max_blocks || max_blocks >= (1 << 27))
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
    if (e == cudaSuccess && isv::q8::attn_smem(D, h->GT, desc->max_seqs) + 1024 > (size_t)h->smem_optin) {
        delete h;
        return err(ISV_EINVAL, "isv_q8_create: shared memory too small for this shape");
    }
    const size_t rows = (size_t)isv::q8::attn_slots(h->GT, h->grid) * isv::q8::attn_head_rows(h->GT);
    if (e == cudaSuccess) e = isv::q8::attn_configure(D, h->GT, desc->dtype == ISV_BF16, desc->format == ISV_Q8_E4M3, h->smem_optin - 1024);
    if (e == cudaSuccess) e = cudaMalloc((void **)&h->status, 4);
    if (e == cudaSuccess) e = cudaMemset(h->status, 0, 4);
    if (e == cudaSuccess) e = cudaMalloc((void **)&h->part_o, rows * D * 4);
    if (e == cudaSuccess) e = cudaMalloc((void **)&h->part_ml, rows * 2 * 4);
    if (e == cudaSuccess) e = cudaMalloc((void **)&h->tickets, (size_t)h->grid * 4);
    if (e == cudaSuccess) e = cudaMemset(h->tickets, 0, (size_t)h->grid * 4);
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
    p.bf16 = h->d.dtype == ISV_BF16; p.e4m3 = h->d.format == ISV_Q8_E4M3;
    OnDevice on(h->device);
    if (on.e != cudaSuccess) return err(ISV_ECUDA, "isv_q8_write: %s", cudaGetErrorString(on.e));
    write_kernel<<<(n_seqs * h->d.kv_heads + 63) / 64, 64, 0, static_cast<cudaStream_t>(stream)>>>(p, h->d.head_dim);
    cudaError_t e = cudaGetLastError();
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
    if (((long long)max_blocks_per_seq + 1) * n_seqs * groups >= (1ll << 31))
        return err(ISV_EINVAL, "isv_q8_attn: n_seqs * blocks * heads too large");
    AttnParams p{};
    p.c = cache_params(h, pool_dev, n_pages, tails_dev, block_table_dev, table_stride, max_blocks_per_seq, seq_lens_dev, n_seqs);
    p.q = static_cast<const uint16_t *>(q_dev);
    p.out = out_dev; p.out_f32 = out_f32_dev;
    p.part_o = h->part_o; p.part_ml = h->part_ml; p.tickets = h->tickets;
    p.Hq = h->d.q_heads; p.P = h->P; p.GT = h->GT;
    p.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)h->d.head_dim));
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

}  // extern "C"
