// Chunks of new tokens over a caller-owned 16-bit paged cache (described in include/isv.h): the handle, and the kernel
// that stores a chunk with the position rotation applied on the way.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>

#include "isv_chunk.cuh"

namespace isv {
int set_error(int code, const char *msg);
}

namespace {

using namespace isv::chunk;

int err(int code, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return isv::set_error(code, buf);
}

// Makes a handle's device current for the length of a call.
struct OnDevice {
    int before = -1;
    cudaError_t e;
    explicit OnDevice(int device) {
        e = cudaGetDevice(&before);
        if (e == cudaSuccess && before != device) e = cudaSetDevice(device);
        else before = -1;
    }
    ~OnDevice() {
        if (before >= 0) cudaSetDevice(before);
    }
};

// ---------------------------------------------------------------- storing a chunk

constexpr int kWriteThreads = 256;
constexpr uint32_t kSpinLimit = 1u << 22;   // polls before a wait of the attention kernel gives up, unless isv_chunk_set_wait_limit says otherwise

struct WriteParams {
    CacheParams c;
    const uint16_t *k, *v, *q;      // rows of kv_stride / q_stride elements; q may be NULL
    uint16_t *q_out;                // rows of q_out_stride elements (q itself: in place)
    int64_t kv_stride, q_stride, q_out_stride;
    const float *freq;              // [rotary / 2] radians per position
    const int32_t *positions;       // [axes][n_rows] or NULL: the place in the sequence
    const uint8_t *axis;            // [rotary / 2] or NULL: axis 0
    int32_t rotary, adjacent, axes;
    float magnitude;
};

// Angle = position * frequency.  The product of a 32-bit whole number and an fp32 number has 55 bits at most; it is taken
// in 64 bits and reduced to a fraction of a turn there (2^-53 of up to 2^29 turns is 2^-24 of a turn), so that far
// positions keep their angle; the sine and cosine of the fraction are fp32.
__device__ __forceinline__ float2 turn(int position, float freq, float magnitude) {
    const double turns = (double)position * (double)freq * 0.15915494309189533577;
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    return make_float2(c * magnitude, s * magnitude);
}

// One thread of the grid per 32 bytes of a token's head: the two 16-byte chunks that the rotation pairs (or, behind the
// rotated part and in V, two adjacent ones).
template <int D, bool BF16>
__global__ void __launch_bounds__(kWriteThreads) write_kernel(const WriteParams p) {
    constexpr int UNITS = D / 16;
    const int s = blockIdx.y;
    bool bad;
    const Seq q = seq_of(p.c, s, bad);
    if (bad && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(p.c.status, ISV_STATUS_BAD_LENGTH);
    const int heads = (p.q ? p.c.Hq : 0) + 2 * p.c.Hkv;
    const long long at = (long long)blockIdx.x * kWriteThreads + threadIdx.x;
    const int u = (int)(at % UNITS);
    const long long th = at / UNITS;
    const int t = (int)(th / heads), h = (int)(th % heads);
    if (t >= q.n) return;
    const int pos = q.start + t, row = q.first + t, slot = pos % kBT;
    const bool is_v = h >= p.c.Hkv && h < 2 * p.c.Hkv, is_q = h >= 2 * p.c.Hkv;
    const bool turned = !is_v && u < p.rotary / 16;
    const int c0 = turned && !p.adjacent ? u : 2 * u, c1 = turned && !p.adjacent ? u + p.rotary / 16 : 2 * u + 1;
    const uint16_t *src = is_q   ? p.q + row * p.q_stride + (h - 2 * p.c.Hkv) * D
                          : is_v ? p.v + row * p.kv_stride + (h - p.c.Hkv) * D
                                 : p.k + row * p.kv_stride + h * D;
    uint4 x[2] = {reinterpret_cast<const uint4 *>(src)[c0], reinterpret_cast<const uint4 *>(src)[c1]};
    if (turned) {
        uint32_t *w0 = reinterpret_cast<uint32_t *>(&x[0]), *w1 = reinterpret_cast<uint32_t *>(&x[1]);
        float2 cs[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int pair = 8 * u + i;
            const int axis = p.axis ? min((int)p.axis[pair], p.axes - 1) : 0;
            cs[i] = turn(p.positions ? p.positions[(long long)axis * p.c.n_rows + row] : pos, p.freq[pair], p.magnitude);
        }
        if (p.adjacent) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint32_t &w = i < 4 ? w0[i] : w1[i - 4];
                const float2 v = widen<BF16>(w);
                w = narrow<BF16>(v.x * cs[i].x - v.y * cs[i].y, v.y * cs[i].x + v.x * cs[i].y);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 a = widen<BF16>(w0[i]), b = widen<BF16>(w1[i]), e = cs[2 * i], f = cs[2 * i + 1];
                w0[i] = narrow<BF16>(a.x * e.x - b.x * e.y, a.y * f.x - b.y * f.y);
                w1[i] = narrow<BF16>(b.x * e.x + a.x * e.y, b.y * f.x + a.y * f.y);
            }
        }
    }
    if (is_q) {
        uint4 *dst = reinterpret_cast<uint4 *>(p.q_out + row * p.q_out_stride + (h - 2 * p.c.Hkv) * D);
        dst[c0] = x[0];
        dst[c1] = x[1];
        return;
    }
    const int page = p.c.table[(long long)s * p.c.table_stride + pos / kBT];
    if (page < 0 || page >= p.c.n_pages) {
        if (h == 0 && u == 0) atomicOr(p.c.status, ISV_STATUS_BAD_BLOCK_ID);
        return;
    }
    // heads of K, then of V: the order of a page's tiles
    uint4 *dst = reinterpret_cast<uint4 *>(p.c.pool + (((long long)page * 2 * p.c.Hkv + h) * kBT + slot) * D);
    dst[place<D>(c0, slot)] = x[0];
    dst[place<D>(c1, slot)] = x[1];
}

bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

}  // namespace

struct isv_chunk {
    isv_chunk_desc d{};
    int device = 0;
    int grid = 1;                       // of the attention kernel
    int GT = 1, P = 1;                  // query heads per visit, passes
    uint32_t *status = nullptr;
    float *part_o = nullptr, *part_ml = nullptr;
    MergeRec *merges = nullptr;
    std::atomic<uint32_t> wait_polls{kSpinLimit};
    std::atomic<int32_t> lost_copies{0};
};

namespace {

int check_call(const char *who, const isv_chunk *h, const void *pool, int32_t n_pages, const int32_t *table, int32_t stride,
               int32_t max_blocks, const int32_t *lens, const int32_t *firsts, int32_t n_rows, int32_t n_seqs, int32_t T) {
    if (!h) return err(ISV_EINVAL, "null handle");
    if (!pool || !table || !lens) return err(ISV_EINVAL, "%s: pool, table and lengths are required", who);
    if (misaligned(pool)) return err(ISV_EINVAL, "%s: the pool must be 16-byte aligned", who);
    if (n_seqs < 0 || n_seqs > h->d.max_seqs) return err(ISV_EINVAL, "%s: n_seqs (%d) must be in [0, %d]", who, n_seqs, h->d.max_seqs);
    // the longest length that a row of max_blocks allows is counted in 32 bits, with a whole tile to spare
    if (n_pages < 1 || max_blocks < 1 || stride < max_blocks || max_blocks >= (1 << 27) - 64)
        return err(ISV_EINVAL, "%s: bad page count (%d) or table row (%d entries, stride %d)", who, n_pages, max_blocks, stride);
    // rows of the pool's tiles are counted in 32 bits
    if ((long long)n_pages * 2 * h->d.kv_heads * kBT >= (1ll << 31)) return err(ISV_EINVAL, "%s: too many pages (%d)", who, n_pages);
    if (T < 0 || (long long)T * h->d.q_heads >= (1ll << 30)) return err(ISV_EINVAL, "%s: bad T (%d)", who, T);
    if (n_rows < 0) return err(ISV_EINVAL, "%s: bad n_rows (%d)", who, n_rows);
    if (!firsts && (long long)n_seqs * T > n_rows)
        return err(ISV_EINVAL, "%s: n_rows (%d) must be at least n_seqs * T without row_starts", who, n_rows);
    return ISV_OK;
}

CacheParams cache_params(const isv_chunk *h, const void *pool, int32_t n_pages, const int32_t *table, int32_t stride,
                         int32_t max_blocks, const int32_t *lens, const int32_t *news, const int32_t *firsts, int32_t n_rows,
                         int32_t n_seqs, int32_t T) {
    CacheParams c{};
    c.pool = static_cast<uint16_t *>(const_cast<void *>(pool));
    c.table = table; c.lens = lens; c.news = news; c.firsts = firsts; c.status = h->status;
    c.table_stride = stride; c.max_blocks = max_blocks; c.n_pages = n_pages; c.n_seqs = n_seqs; c.n_rows = n_rows; c.T = T;
    c.Hkv = h->d.kv_heads; c.Hq = h->d.q_heads;
    return c;
}

template <int D>
cudaError_t launch_write(const WriteParams &p, bool bf16, dim3 grid, cudaStream_t st) {
    if (bf16) write_kernel<D, true><<<grid, kWriteThreads, 0, st>>>(p);
    else write_kernel<D, false><<<grid, kWriteThreads, 0, st>>>(p);
    return cudaGetLastError();
}
}  // namespace

extern "C" {

int isv_chunk_free(isv_chunk *h) {
    if (!h) return err(ISV_EINVAL, "null handle");
    OnDevice on(h->device);
    cudaDeviceSynchronize();   // calls may have been made on any stream
    cudaFree(h->status);
    cudaFree(h->part_o);
    cudaFree(h->part_ml);
    cudaFree(h->merges);
    delete h;
    return ISV_OK;
}

int isv_chunk_create(isv_chunk **out, const isv_chunk_desc *desc) {
    if (!out) return err(ISV_EINVAL, "out is null");
    *out = nullptr;
    if (!desc) return err(ISV_EINVAL, "desc is null");
    if (desc->kv_heads < 1 || desc->q_heads < 1 || desc->q_heads % desc->kv_heads != 0)
        return err(ISV_EINVAL, "isv_chunk_create: q_heads must be a positive multiple of kv_heads");
    if (desc->q_heads > 65536) return err(ISV_EINVAL, "isv_chunk_create: at most 65536 query heads");
    if (desc->head_dim != 64 && desc->head_dim != 80 && desc->head_dim != 128)
        return err(ISV_EINVAL, "isv_chunk_create: head_dim 64/80/128 only");
    if (desc->dtype != ISV_F16 && desc->dtype != ISV_BF16) return err(ISV_EINVAL, "isv_chunk_create: dtype f16/bf16 only");
    if (desc->max_seqs < 1 || desc->max_seqs > 4096 || desc->max_ctas < 0)
        return err(ISV_EINVAL, "isv_chunk_create: max_seqs must be in [1, 4096], max_ctas not negative");
    if (desc->rotary_dim < 0 || desc->rotary_dim > desc->head_dim || desc->rotary_dim % 16)
        return err(ISV_EINVAL, "isv_chunk_create: rotary_dim (%d) must be a multiple of 16 up to head_dim", desc->rotary_dim);
    if (desc->rotary_pairs != ISV_ROTARY_HALVES && desc->rotary_pairs != ISV_ROTARY_ADJACENT)
        return err(ISV_EINVAL, "isv_chunk_create: rotary_pairs must be ISV_ROTARY_HALVES or ISV_ROTARY_ADJACENT");
    if (desc->rotary_axes < 1 || desc->rotary_axes > 4) return err(ISV_EINVAL, "isv_chunk_create: rotary_axes must be in [1, 4]");
    if (!std::isfinite(desc->scale) || !std::isfinite(desc->softcap) || desc->softcap < 0)
        return err(ISV_EINVAL, "isv_chunk_create: scale and softcap must be finite, softcap not negative");
    isv_chunk *h = new (std::nothrow) isv_chunk();
    if (!h) return err(ISV_EINVAL, "out of host memory");
    h->d = *desc;
    // a row tile holds tokens with GT heads each; more than a tile's rows of heads are served in equal passes
    const int G = desc->q_heads / desc->kv_heads;
    h->P = (G + 127) / 128;
    h->GT = (G + h->P - 1) / h->P;
    int sms = 0;
    cudaError_t e = cudaGetDevice(&h->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, h->device);
    h->grid = desc->max_ctas > 0 ? std::min(desc->max_ctas, sms) : sms;   // one CTA per SM
    const size_t rows = attn_part_rows(h->grid);
    if (e == cudaSuccess) e = attn_configure(desc->head_dim, desc->dtype == ISV_BF16);
    if (e == cudaSuccess) e = cudaMalloc((void **)&h->status, 4);
    if (e == cudaSuccess) e = cudaMemset(h->status, 0, 4);
    if (e == cudaSuccess) e = cudaMalloc((void **)&h->part_o, rows * desc->head_dim * 4);
    if (e == cudaSuccess) e = cudaMalloc((void **)&h->part_ml, rows * 2 * 4);
    if (e == cudaSuccess) e = cudaMalloc((void **)&h->merges, h->grid * sizeof(MergeRec));
    if (e == cudaSuccess) e = cudaDeviceSynchronize();   // the zeros are there before any stream's first call
    if (e != cudaSuccess) {
        cudaGetLastError();
        isv_chunk_free(h);
        return err(e == cudaErrorMemoryAllocation ? ISV_ENOMEM_DEVICE : ISV_ECUDA, "isv_chunk_create: %s", cudaGetErrorString(e));
    }
    *out = h;
    return ISV_OK;
}

int isv_chunk_write(isv_chunk *h, void *pool_dev, int32_t n_pages, const int32_t *block_table_dev, int32_t table_stride,
                    int32_t max_blocks_per_seq, const int32_t *seq_lens_dev, const int32_t *new_lens_dev,
                    const int32_t *row_starts_dev, int32_t n_rows, const void *k_dev, const void *v_dev, int64_t kv_stride,
                    const void *q_dev, int64_t q_stride, void *q_out_dev, const float *inv_freq_dev,
                    const int32_t *positions_dev, const uint8_t *pair_axis_dev, float magnitude, int32_t n_seqs, int32_t T,
                    void *stream) {
    const char *who = "isv_chunk_write";
    int rc = check_call(who, h, pool_dev, n_pages, block_table_dev, table_stride, max_blocks_per_seq, seq_lens_dev, row_starts_dev,
                        n_rows, n_seqs, T);
    if (rc) return rc;
    if (!k_dev || !v_dev || misaligned(k_dev) || misaligned(v_dev)) return err(ISV_EINVAL, "%s: k and v must be non-null, 16-byte aligned", who);
    if (misaligned(q_dev) || misaligned(q_out_dev)) return err(ISV_EINVAL, "%s: q and q_out must be 16-byte aligned", who);
    if (!q_dev && q_out_dev) return err(ISV_EINVAL, "%s: q_out without q", who);
    const int64_t kv_row = (int64_t)h->d.kv_heads * h->d.head_dim, q_row = (int64_t)h->d.q_heads * h->d.head_dim;
    if (kv_stride % 8 || kv_stride < kv_row || (q_dev && (q_stride % 8 || q_stride < q_row)))
        return err(ISV_EINVAL, "%s: strides must be multiples of 8 elements that hold a token's heads", who);
    if (h->d.rotary_dim > 0 && !inv_freq_dev) return err(ISV_EINVAL, "%s: inv_freq is required", who);
    if (!positions_dev && pair_axis_dev) return err(ISV_EINVAL, "%s: pair_axis without positions", who);
    if (!std::isfinite(magnitude)) return err(ISV_EINVAL, "%s: magnitude must be finite", who);
    if (n_seqs == 0 || T == 0) return ISV_OK;
    WriteParams p{};
    p.c = cache_params(h, pool_dev, n_pages, block_table_dev, table_stride, max_blocks_per_seq, seq_lens_dev, new_lens_dev, row_starts_dev,
                       n_rows, n_seqs, T);
    p.k = static_cast<const uint16_t *>(k_dev);
    p.v = static_cast<const uint16_t *>(v_dev);
    p.q = static_cast<const uint16_t *>(q_dev);
    p.q_out = q_out_dev ? static_cast<uint16_t *>(q_out_dev) : const_cast<uint16_t *>(p.q);
    p.kv_stride = kv_stride; p.q_stride = q_stride; p.q_out_stride = q_out_dev ? q_row : q_stride;
    p.freq = inv_freq_dev; p.positions = positions_dev; p.axis = pair_axis_dev;
    p.rotary = h->d.rotary_dim; p.adjacent = h->d.rotary_pairs == ISV_ROTARY_ADJACENT; p.axes = h->d.rotary_axes;
    p.magnitude = magnitude;
    const long long units = (long long)T * ((q_dev ? h->d.q_heads : 0) + 2 * h->d.kv_heads) * (h->d.head_dim / 16);
    const dim3 grid((unsigned)((units + kWriteThreads - 1) / kWriteThreads), (unsigned)n_seqs);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    OnDevice on(h->device);
    if (on.e != cudaSuccess) return err(ISV_ECUDA, "%s: %s", who, cudaGetErrorString(on.e));
    const bool bf16 = h->d.dtype == ISV_BF16;
    const cudaError_t e = h->d.head_dim == 64   ? launch_write<64>(p, bf16, grid, st)
                          : h->d.head_dim == 80 ? launch_write<80>(p, bf16, grid, st)
                                                : launch_write<128>(p, bf16, grid, st);
    return e == cudaSuccess ? ISV_OK : err(ISV_ECUDA, "%s: %s", who, cudaGetErrorString(e));
}

int isv_chunk_attn(isv_chunk *h, const void *pool_dev, int32_t n_pages, const int32_t *block_table_dev, int32_t table_stride,
                   int32_t max_blocks_per_seq, const int32_t *seq_lens_dev, const int32_t *new_lens_dev,
                   const int32_t *row_starts_dev, int32_t n_rows, const void *q_dev, int64_t q_stride, const float *slopes_dev,
                   const int32_t *prefix_lens_dev, int32_t window, void *out_dev, float *out_f32_dev, int32_t n_seqs, int32_t T,
                   void *stream) {
    const char *who = "isv_chunk_attn";
    int rc = check_call(who, h, pool_dev, n_pages, block_table_dev, table_stride, max_blocks_per_seq, seq_lens_dev, row_starts_dev,
                        n_rows, n_seqs, T);
    if (rc) return rc;
    if (!q_dev || (!out_dev && !out_f32_dev)) return err(ISV_EINVAL, "%s: q and one output are required", who);
    if (misaligned(q_dev) || misaligned(out_dev) || misaligned(out_f32_dev))
        return err(ISV_EINVAL, "%s: q and outputs must be 16-byte aligned", who);
    if (q_stride % 8 || q_stride < (int64_t)h->d.q_heads * h->d.head_dim)
        return err(ISV_EINVAL, "%s: the stride of q must be a multiple of 8 elements that holds a token's heads", who);
    if (window < 0) return err(ISV_EINVAL, "%s: window must not be negative", who);
    if (n_seqs == 0 || T == 0) return ISV_OK;
    AttnParams p{};
    p.c = cache_params(h, pool_dev, n_pages, block_table_dev, table_stride, max_blocks_per_seq, seq_lens_dev, new_lens_dev, row_starts_dev,
                       n_rows, n_seqs, T);
    p.q = static_cast<const uint16_t *>(q_dev);
    p.q_stride = q_stride;
    p.slopes = slopes_dev; p.prefixes = prefix_lens_dev; p.window = window;
    p.out = static_cast<uint16_t *>(out_dev); p.out_f32 = out_f32_dev;
    p.scale = h->d.scale != 0.f ? h->d.scale : (float)(1.0 / std::sqrt((double)h->d.head_dim));
    p.cap = h->d.softcap;
    p.GT = h->GT; p.P = h->P;
    p.tile_rows = attn_tile_rows((long long)T * h->GT);
    p.TT = std::min(p.tile_rows, 128) / h->GT;
    const int tokens = p.tile_rows / std::min(p.tile_rows, 128) * p.TT;
    p.RT = (T + tokens - 1) / tokens;
    if ((long long)n_seqs * p.RT >= (1ll << 31)) return err(ISV_EINVAL, "%s: n_seqs * T too large", who);
    p.part_o = h->part_o; p.part_ml = h->part_ml; p.merges = h->merges;
    p.spin_limit = h->wait_polls.load();
    if (h->lost_copies.load() > 0) p.drop_first_copy = h->lost_copies.fetch_sub(1) > 0;
    OnDevice on(h->device);
    if (on.e != cudaSuccess) return err(ISV_ECUDA, "%s: %s", who, cudaGetErrorString(on.e));
    const char *what = nullptr;
    const cudaError_t e = launch_attn(p, h->d.head_dim, h->d.dtype == ISV_BF16, h->grid, static_cast<cudaStream_t>(stream), &what);
    return e == cudaSuccess ? ISV_OK : err(ISV_ECUDA, "%s: %s", who, what ? what : cudaGetErrorString(e));
}

int isv_chunk_status(isv_chunk *h, void *stream, uint32_t *status_out) {
    if (!h || !status_out) return err(ISV_EINVAL, "null argument");
    OnDevice on(h->device);
    if (on.e != cudaSuccess) return err(ISV_ECUDA, "isv_chunk_status: %s", cudaGetErrorString(on.e));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaMemcpyAsync(status_out, h->status, 4, cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e == cudaSuccess && *status_out) {
        e = cudaMemsetAsync(h->status, 0, 4, st);
        if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    }
    if (e != cudaSuccess) return err(ISV_ECUDA, "isv_chunk_status: %s", cudaGetErrorString(e));
    if (*status_out) return err(ISV_EDEVICE_STATUS, "a call on a chunk reported status 0x%x", *status_out);
    return ISV_OK;
}

int isv_chunk_set_wait_limit(isv_chunk *h, uint32_t polls) {
    if (!h) return err(ISV_EINVAL, "null handle");
    h->wait_polls = polls ? polls : kSpinLimit;
    return ISV_OK;
}

int isv_chunk_inject_lost_copy(isv_chunk *h, int32_t launches) {
    if (!h) return err(ISV_EINVAL, "null handle");
    if (launches < 0) return err(ISV_EINVAL, "launches must not be negative");
    h->lost_copies = launches;
    return ISV_OK;
}

}  // extern "C"
