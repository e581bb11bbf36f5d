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
constexpr int kWriteTokens = 16;       // of a CTA, at most
constexpr int kWriteAhead = 2;         // units of a thread whose loads are in flight (4: more registers, fewer CTAs, 194 us instead of 143)
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
    int32_t tokens;                 // of a CTA
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

// A CTA takes a few tokens of one sequence.  The unit of work is 32 bytes of a token's head: the two 16-byte chunks that the rotation
// pairs (or, behind the rotated part and in V, two adjacent ones).  The first units' loads are in flight while the tokens' sines
// and cosines are computed, once for all heads, into shared memory.  Bound by HBM on prompts, by one chain of loads (lengths, rows,
// page) on single tokens.
template <int D, bool BF16>
__global__ void __launch_bounds__(kWriteThreads) write_kernel(const WriteParams p) {
    constexpr int UNITS = D / 16;
    __shared__ float2 turns[kWriteTokens * D / 2];      // [token][pair]
    __shared__ int pages[kWriteTokens];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int s = blockIdx.y, t0 = blockIdx.x * p.tokens;
    bool bad;
    const Seq q = seq_of(p.c, s, bad);
    if (bad && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(p.c.status, ISV_STATUS_BAD_LENGTH);
    const int n = min(p.tokens, q.n - t0);
    if (n <= 0) return;
    const int heads = (p.q ? p.c.Hq : 0) + 2 * p.c.Hkv, per_token = heads * UNITS, units = n * per_token;
    const int row0 = q.first + t0, pos0 = q.start + t0;

    struct Unit {
        int t, h, c0, c1;       // token, head (of K, V, Q in this order), chunks
        bool turned;
    };
    auto unit_at = [&](int i) {
        Unit z;
        z.t = i / per_token;
        const int y = i - z.t * per_token, u = y % UNITS;
        z.h = y / UNITS;
        z.turned = (z.h < p.c.Hkv || z.h >= 2 * p.c.Hkv) && u < p.rotary / 16;
        const bool halves = z.turned && !p.adjacent;
        z.c0 = halves ? u : 2 * u;
        z.c1 = halves ? u + p.rotary / 16 : 2 * u + 1;
        return z;
    };
    auto load = [&](int i, uint4 (&x)[2]) {
        const Unit z = unit_at(i);
        const long long row = row0 + z.t;
        const uint16_t *src = z.h >= 2 * p.c.Hkv ? p.q + row * p.q_stride + (z.h - 2 * p.c.Hkv) * D
                              : z.h >= p.c.Hkv   ? p.v + row * p.kv_stride + (z.h - p.c.Hkv) * D
                                                 : p.k + row * p.kv_stride + z.h * D;
        x[0] = reinterpret_cast<const uint4 *>(src)[z.c0];
        x[1] = reinterpret_cast<const uint4 *>(src)[z.c1];
    };
    uint4 x[kWriteAhead][2];
#pragma unroll
    for (int k = 0; k < kWriteAhead; ++k)
        if (threadIdx.x + k * kWriteThreads < units) load(threadIdx.x + k * kWriteThreads, x[k]);

    const int pairs = p.rotary / 2;
    for (int i = threadIdx.x; i < n * pairs; i += kWriteThreads) {
        const int t = i / pairs, y = i - t * pairs;
        const int axis = p.axis ? min((int)p.axis[y], p.axes - 1) : 0;
        turns[t * (D / 2) + y] = turn(p.positions ? p.positions[(long long)axis * p.c.n_rows + row0 + t] : pos0 + t, p.freq[y], p.magnitude);
    }
    if (threadIdx.x < n) {
        const int page = p.c.table[(long long)s * p.c.table_stride + (pos0 + threadIdx.x) / kBT];
        const bool there = page >= 0 && page < p.c.n_pages;
        if (!there) atomicOr(p.c.status, ISV_STATUS_BAD_BLOCK_ID);
        pages[threadIdx.x] = there ? page : -1;
    }
    __syncthreads();

    for (int base = threadIdx.x; base < units; base += kWriteAhead * kWriteThreads) {
#pragma unroll
        for (int k = 0; k < kWriteAhead; ++k) {
            const int i = base + k * kWriteThreads;
            if (i >= units) break;
            const Unit z = unit_at(i);
            uint4 y[2] = {x[k][0], x[k][1]};
            if (i + kWriteAhead * kWriteThreads < units) load(i + kWriteAhead * kWriteThreads, x[k]);
            if (z.turned) {
                uint32_t *w0 = reinterpret_cast<uint32_t *>(&y[0]), *w1 = reinterpret_cast<uint32_t *>(&y[1]);
                const int u = p.adjacent ? z.c0 / 2 : z.c0;
                const float4 *cs = reinterpret_cast<const float4 *>(turns + z.t * (D / 2) + 8 * u);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float4 f = cs[e];                 // cos, sin of two pairs
                    if (p.adjacent) {
                        uint32_t &a = e < 2 ? w0[2 * e] : w1[2 * e - 4], &b = e < 2 ? w0[2 * e + 1] : w1[2 * e - 3];
                        const float2 v = widen<BF16>(a), w = widen<BF16>(b);
                        a = narrow<BF16>(v.x * f.x - v.y * f.y, v.y * f.x + v.x * f.y);
                        b = narrow<BF16>(w.x * f.z - w.y * f.w, w.y * f.z + w.x * f.w);
                    } else {
                        const float2 v = widen<BF16>(w0[e]), w = widen<BF16>(w1[e]);
                        w0[e] = narrow<BF16>(v.x * f.x - w.x * f.y, v.y * f.z - w.y * f.w);
                        w1[e] = narrow<BF16>(w.x * f.x + v.x * f.y, w.y * f.z + v.y * f.w);
                    }
                }
            }
            uint4 *dst;
            int c0 = z.c0, c1 = z.c1;
            if (z.h >= 2 * p.c.Hkv) {
                dst = reinterpret_cast<uint4 *>(p.q_out + (long long)(row0 + z.t) * p.q_out_stride + (z.h - 2 * p.c.Hkv) * D);
            } else {
                if (pages[z.t] < 0) continue;
                // heads of K, then of V: the order of a page's tiles
                const int slot = (pos0 + z.t) % kBT;
                dst = reinterpret_cast<uint4 *>(p.c.pool + (((long long)pages[z.t] * 2 * p.c.Hkv + z.h) * kBT + slot) * D);
                c0 = place<D>(c0, slot);
                c1 = place<D>(c1, slot);
            }
            dst[c0] = y[0];
            dst[c1] = y[1];
        }
    }
}

bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

}  // namespace

struct isv_chunk {
    isv_chunk_desc d{};
    int device = 0;
    int sms = 1, grid = 1;              // of the device, of the attention kernel
    int GT = 1, P = 1;                  // query heads per visit, passes
    char *memory = nullptr;             // all of what follows
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

template <int D, bool BF16>
cudaError_t launch_write_as(const WriteParams &p, dim3 grid, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kWriteThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;   // see the kernel's griddepcontrol pair
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, write_kernel<D, BF16>, p);
}
template <int D>
cudaError_t launch_write(const WriteParams &p, bool bf16, dim3 grid, cudaStream_t st) {
    return bf16 ? launch_write_as<D, true>(p, grid, st) : launch_write_as<D, false>(p, grid, st);
}

}  // namespace

extern "C" {

int isv_chunk_free(isv_chunk *h) {
    if (!h) return err(ISV_EINVAL, "null handle");
    OnDevice on(h->device);
    cudaDeviceSynchronize();   // calls may have been made on any stream
    cudaFree(h->memory);
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
    h->sms = std::max(1, sms);
    h->grid = desc->max_ctas > 0 ? std::min(desc->max_ctas, h->sms) : h->sms;   // one CTA per SM
    const size_t rows = attn_part_rows(h->grid);
    const bool bf16 = desc->dtype == ISV_BF16;
    if (e == cudaSuccess)
        e = desc->head_dim == 64 ? attn_configure<64>(bf16) : desc->head_dim == 80 ? attn_configure<80>(bf16) : attn_configure<128>(bf16);
    const size_t o_bytes = rows * desc->head_dim * 4, ml_bytes = rows * 2 * 4, rec_bytes = (h->grid * sizeof(MergeRec) + 255) / 256 * 256;
    if (e == cudaSuccess) e = cudaMalloc((void **)&h->memory, o_bytes + ml_bytes + rec_bytes + 256);
    if (e == cudaSuccess) {
        h->part_o = reinterpret_cast<float *>(h->memory);
        h->part_ml = reinterpret_cast<float *>(h->memory + o_bytes);
        h->merges = reinterpret_cast<MergeRec *>(h->memory + o_bytes + ml_bytes);
        h->status = reinterpret_cast<uint32_t *>(h->memory + o_bytes + ml_bytes + rec_bytes);
        e = cudaMemset(h->status, 0, 4);
    }
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
    if (q_dev && q_out_dev == q_dev && q_stride != q_row) return err(ISV_EINVAL, "%s: q_out is q, but q has another stride (NULL turns q in place)", who);
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
    // about six units a thread (fewer, and the tokens' sines weigh), but not less than six CTAs an SM
    const long long per_token = (long long)((q_dev ? h->d.q_heads : 0) + 2 * h->d.kv_heads) * (h->d.head_dim / 16);
    const long long most = std::min<long long>(6 * kWriteThreads / per_token, (long long)n_seqs * T / (6 * h->sms));
    p.tokens = (int)std::min<long long>(kWriteTokens, std::max<long long>(1, most));
    const dim3 grid((unsigned)((T + p.tokens - 1) / p.tokens), (unsigned)n_seqs);
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
    if (out_dev == q_dev || out_f32_dev == q_dev || out_dev == out_f32_dev) return err(ISV_EINVAL, "%s: outputs overlap nothing", who);
    if (q_stride % 8 || q_stride < (int64_t)h->d.q_heads * h->d.head_dim)
        return err(ISV_EINVAL, "%s: the stride of q must be a multiple of 8 elements that holds a token's heads", who);
    if (window < 0) return err(ISV_EINVAL, "%s: window must not be negative", who);
    if (n_seqs == 0 || T == 0 || n_rows == 0) return ISV_OK;
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
    const bool bf16 = h->d.dtype == ISV_BF16;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = h->d.head_dim == 64   ? launch_attn<64>(p, bf16, h->grid, st, &what)
                          : h->d.head_dim == 80 ? launch_attn<80>(p, bf16, h->grid, st, &what)
                                                : launch_attn<128>(p, bf16, h->grid, st, &what);
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
