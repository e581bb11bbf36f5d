// Decode linear layers with 4-bit weights and a 16-bit scale per (row, group of k): y = x . w^T for a few tokens.
//
// The product is bound by reading the weights, half a byte each, and what the SMs have to do per byte is large: turning
// eight nibbles into 16-bit numbers takes about ten instructions, so the multiplications must not cost any.  They run on
// mma.m16n8k16 with 16 weight rows as the rows and 8 tokens as the columns (one token takes as long as eight; tcgen05 would want the widened weights
// in shared memory, i.e. a store and a load more per weight).  Nibbles become numbers by placing them in the mantissa of
// 1024 (fp16) or 128 (bf16) and subtracting: exact, as are the products; sums are fp32 and a group's sum is scaled once.
//
// isv_linear4_create lays the weights out in operand order: blocks of 32 rows, per block all of K in chunks of 32, per
// chunk 16 bytes for each lane of a warp, so a warp's loads are 512 contiguous bytes and need no shared memory.  A CTA
// takes one block of rows and its warps share K in steps of 128; where there are few blocks a cluster of CTAs shares a block's K
// and adds up through distributed shared memory.  The order of all sums is fixed.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <new>

#include "../../include/isv.h"

namespace cg = cooperative_groups;

namespace isv {
int set_error(int code, const char *msg);
}

namespace {

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

constexpr int kRows = 32;      // rows of a block
constexpr int kChunk = 32;     // k of a chunk: two steps of the matrix instruction
constexpr int kStep = 128;     // k of a warp's step: four chunks
constexpr int kWarps = 8;
constexpr int kMaxCluster = 8;

struct Linear4Params {
    const uint4 *w;            // [blocks][chunks][32 lanes]
    const uint2 *scales;       // [blocks][K / group][8]: rows g, g + 8, g + 16, g + 24
    const uint16_t *x;
    uint16_t *y;
    float *y_f32;
    int32_t M, N, K;
};

struct PackParams {
    const uint8_t *w;          // [N][K / 2]
    const uint16_t *s;         // [N][K / group]
    uint32_t *w_out;
    uint16_t *s_out;
    int32_t N, K, group, blocks;
};

// Word i of a lane (4 g + c) in a chunk: row tile i / 2, k-step i % 2.  Its nibble 4 e + r belongs to operand register r:
// row g + 8 * (r % 2) of the tile, k = 8 c + 4 (i % 2) + 2 (r / 2) + e of the chunk.  Rows from N on are zeros.
__global__ void pack_kernel(PackParams p) {
    const long long words = (long long)p.blocks * (p.K / kChunk) * 128, scales = (long long)p.blocks * kRows * (p.K / p.group);
    const long long stride = (long long)gridDim.x * blockDim.x, at = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    for (long long id = at; id < words; id += stride) {
        const int i = (int)(id & 3), lane = (int)(id >> 2) & 31, g = lane >> 2, c = lane & 3;
        const int chunk = (int)((id >> 7) % (p.K / kChunk));
        const int block = (int)((id >> 7) / (p.K / kChunk));
        uint32_t w = 0;
        for (int n = 0; n < 8; ++n) {
            const int r = n & 3, e = n >> 2;
            const long long row = (long long)block * kRows + (i >> 1) * 16 + g + 8 * (r & 1);
            const int k = chunk * kChunk + 8 * c + 4 * (i & 1) + 2 * (r >> 1) + e;
            uint32_t u = 8;
            if (row < p.N) {
                const uint8_t b = p.w[row * (p.K / 2) + k / 2];
                u = k & 1 ? b >> 4 : b & 15;
            }
            w |= u << (4 * n);
        }
        p.w_out[id] = w;
    }
    for (long long id = at; id < scales; id += stride) {   // [block][group][g][4]
        const int i = (int)(id & 3), g = (int)(id >> 2) & 7;
        const int group = (int)((id >> 5) % (p.K / p.group));
        const long long row = (id >> 5) / (p.K / p.group) * kRows + g + 8 * i;
        p.s_out[id] = row < p.N ? p.s[row * (p.K / p.group) + group] : 0;
    }
}

template <bool BF16>
__device__ __forceinline__ float to_f32(uint32_t b) {
    return BF16 ? __uint_as_float(b << 16) : __half2float(__ushort_as_half((unsigned short)b));
}

template <bool BF16>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Eight nibbles u -> four pairs of u - 8.
template <bool BF16>
__device__ __forceinline__ void widen(uint32_t w, uint32_t (&a)[4]) {
    if (BF16) {
        const __nv_bfloat162 base = __floats2bfloat162_rn(136.f, 136.f);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            uint32_t v = ((w >> (4 * r)) & 0x000f000fu) | 0x43004300u;          // 128 + u
            const __nv_bfloat162 d = __hsub2(*reinterpret_cast<__nv_bfloat162 *>(&v), base);
            a[r] = *reinterpret_cast<const uint32_t *>(&d);
        }
    } else {
        const __half2 base = __floats2half2_rn(1032.f, 1032.f), part = __floats2half2_rn(0.0625f, 0.0625f),
                      base16 = __floats2half2_rn(-72.f, -72.f);
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
            const uint32_t v = w >> (4 * r);
            uint32_t even = (v & 0x000f000fu) | 0x64006400u, odd = (v & 0x00f000f0u) | 0x64006400u;   // 1024 + u, 1024 + 16 u
            const __half2 x = __hsub2(*reinterpret_cast<__half2 *>(&even), base);
            const __half2 y = __hfma2(*reinterpret_cast<__half2 *>(&odd), part, base16);
            a[r] = *reinterpret_cast<const uint32_t *>(&x);
            a[r + 1] = *reinterpret_cast<const uint32_t *>(&y);
        }
    }
}

// NT tiles of 8 tokens; blockIdx.y counts passes of 8 * NT tokens.
template <int NT, int GROUP, bool BF16>
__global__ void __launch_bounds__(kWarps * 32) linear4_kernel(const __grid_constant__ Linear4Params p) {
    constexpr int CHUNKS = kStep / kChunk, PER = GROUP / kChunk;       // chunks of a step, of a group
    constexpr int COLS = 8 * NT, PITCH = kRows + 1;
    __shared__ float sums[kWarps][COLS][PITCH];
    cg::cluster_group cluster = cg::this_cluster();
    const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const int block = blockIdx.x / cs, m0 = blockIdx.y * COLS;
    const int chunks = p.K / kChunk, groups = p.K / GROUP;
    const int steps = (p.K + kStep - 1) / kStep;
    const int end = (int)((long long)steps * (rank + 1) / cs);
    const uint4 *w = p.w + (size_t)block * chunks * 32 + lane;
    const uint2 *scales = p.scales + (size_t)block * groups * 8 + g;

    uint4 next[CHUNKS];
    auto fetch = [&](int step) {
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int chunk = step * CHUNKS + i;
            next[i] = step < end && chunk < chunks ? __ldg(w + (size_t)chunk * 32) : make_uint4(0x88888888u, 0x88888888u, 0x88888888u, 0x88888888u);
        }
    };
    int step = (int)((long long)steps * rank / cs) + warp;
    fetch(step);               // the weights do not change: they are on their way before the predecessor has ended
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    float total[2][NT][4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) total[t][nt][i] = 0.f;
    for (; step < end; step += kWarps) {
        uint4 now[CHUNKS];
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) now[i] = next[i];
        uint4 x[CHUNKS][NT];
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int m = m0 + nt * 8 + g, chunk = step * CHUNKS + i;
                x[i][nt] = m < p.M && chunk < chunks ? *reinterpret_cast<const uint4 *>(p.x + (size_t)m * p.K + chunk * kChunk + 8 * c)
                                                     : make_uint4(0, 0, 0, 0);
            }
        uint2 sc[CHUNKS / PER];
#pragma unroll
        for (int i = 0; i < CHUNKS / PER; ++i) {
            const int group = step * (CHUNKS / PER) + i;
            sc[i] = group < groups ? __ldg(scales + (size_t)group * 8) : make_uint2(0, 0);
        }
        fetch(step + kWarps);
#pragma unroll
        for (int i0 = 0; i0 < CHUNKS / PER; ++i0) {
            float part[2][NT][4];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) part[t][nt][i] = 0.f;
#pragma unroll
            for (int i = i0 * PER; i < (i0 + 1) * PER; ++i) {
                const uint32_t words[4] = {now[i].x, now[i].y, now[i].z, now[i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t a[4];
                    widen<BF16>(words[j], a);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        mma<BF16>(part[j >> 1][nt], a, j & 1 ? x[i][nt].z : x[i][nt].x, j & 1 ? x[i][nt].w : x[i][nt].y);
                }
            }
            const float s[4] = {to_f32<BF16>(sc[i0].x & 0xffffu), to_f32<BF16>(sc[i0].x >> 16), to_f32<BF16>(sc[i0].y & 0xffffu),
                                to_f32<BF16>(sc[i0].y >> 16)};
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) total[t][nt][i] += part[t][nt][i] * s[2 * t + (i >> 1)];
        }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[warp][nt * 8 + 2 * c + (i & 1)][t * 16 + g + 8 * (i >> 1)] = total[t][nt][i];
    if (cs > 1) cluster.sync(); else __syncthreads();
    const int cols = min(COLS, p.M - m0);
    // the CTAs of a cluster share the outputs; each adds the warps of all of them in order
    for (int o = rank * kWarps * 32 + threadIdx.x; o < cols * kRows; o += cs * kWarps * 32) {
        const int m = o / kRows, r = o % kRows, n = block * kRows + r;
        float v = 0.f;
        for (int k = 0; k < cs; ++k) {
            const float *other = cs > 1 ? cluster.map_shared_rank(&sums[0][0][0], k) : &sums[0][0][0];
#pragma unroll
            for (int i = 0; i < kWarps; ++i) v += other[(i * COLS + m) * PITCH + r];
        }
        if (n < p.N) {
            const size_t at = (size_t)(m0 + m) * p.N + n;
            if (p.y_f32) p.y_f32[at] = v;
            if (p.y) p.y[at] = BF16 ? __bfloat16_as_ushort(__float2bfloat16(v)) : __half_as_ushort(__float2half(v));
        }
    }
    if (cs > 1) cluster.sync();   // nobody leaves while its sums may be read
}

template <int NT, int GROUP>
cudaError_t launch(const Linear4Params &p, bool bf16, const cudaLaunchConfig_t &cfg) {
    return bf16 ? cudaLaunchKernelEx(&cfg, linear4_kernel<NT, GROUP, true>, p) : cudaLaunchKernelEx(&cfg, linear4_kernel<NT, GROUP, false>, p);
}
template <int NT>
cudaError_t launch(const Linear4Params &p, int group, bool bf16, const cudaLaunchConfig_t &cfg) {
    if (group == 32) return launch<NT, 32>(p, bf16, cfg);
    if (group == 64) return launch<NT, 64>(p, bf16, cfg);
    return launch<NT, 128>(p, bf16, cfg);
}

}  // namespace

struct isv_linear4 {
    int N = 0, K = 0, group = 0, max_M = 0, device = 0, blocks = 0, cluster = 1;
    bool bf16 = false;
    uint32_t *w = nullptr;
    uint16_t *scales = nullptr;
};

extern "C" {

int isv_linear4_free(isv_linear4 *l) {
    if (!l) return err(ISV_EINVAL, "null handle");
    OnDevice on(l->device);
    cudaDeviceSynchronize();   // calls may have been made on any stream
    cudaFree(l->w);
    cudaFree(l->scales);
    delete l;
    return ISV_OK;
}

int isv_linear4_create(isv_linear4 **out, const void *w4_dev, const void *scales_dev, int32_t N, int32_t K, int32_t group,
                       int32_t dtype, int32_t max_M, void *stream) {
    if (!out) return err(ISV_EINVAL, "out is null");
    *out = nullptr;
    if (!w4_dev || !scales_dev) return err(ISV_EINVAL, "isv_linear4_create: weights and scales are required");
    if (reinterpret_cast<uintptr_t>(scales_dev) & 1u) return err(ISV_EINVAL, "isv_linear4_create: scales must be 2-byte aligned");
    if (group != 32 && group != 64 && group != 128) return err(ISV_EINVAL, "isv_linear4_create: group (%d) must be 32, 64 or 128", group);
    if (N < 1 || N > (1 << 24)) return err(ISV_EINVAL, "isv_linear4_create: bad N (%d)", N);
    if (K < group || K % group != 0 || K > (1 << 20)) return err(ISV_EINVAL, "isv_linear4_create: K (%d) must be a multiple of the group (%d)", K, group);
    if (max_M < 1 || max_M > 64) return err(ISV_EINVAL, "isv_linear4_create: max_M (%d) must be in [1, 64]", max_M);
    if (dtype != ISV_F16 && dtype != ISV_BF16) return err(ISV_EINVAL, "dtype must be ISV_F16 or ISV_BF16");
    isv_linear4 *l = new (std::nothrow) isv_linear4();
    if (!l) return err(ISV_EINVAL, "out of host memory");
    l->N = N; l->K = K; l->group = group; l->max_M = max_M; l->bf16 = dtype == ISV_BF16;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    l->blocks = (N + kRows - 1) / kRows;
    int sms = 0;
    cudaError_t e = cudaGetDevice(&l->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, l->device);
    // few blocks of rows: several CTAs share the K of one, while each of their warps keeps two steps
    while (l->cluster < kMaxCluster && l->blocks * l->cluster < 2 * sms && K >= 2 * l->cluster * 2 * kWarps * kStep) l->cluster *= 2;
    if (e == cudaSuccess) e = cudaMalloc((void **)&l->w, (size_t)l->blocks * kRows * (K / 2));
    if (e == cudaSuccess) e = cudaMalloc((void **)&l->scales, (size_t)l->blocks * kRows * (K / group) * 2);
    if (e == cudaSuccess) {
        const PackParams p = {static_cast<const uint8_t *>(w4_dev), static_cast<const uint16_t *>(scales_dev), l->w, l->scales, N, K, group, l->blocks};
        pack_kernel<<<8 * sms, 256, 0, st>>>(p);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) {
        cudaGetLastError();
        isv_linear4_free(l);
        return err(e == cudaErrorMemoryAllocation ? ISV_ENOMEM_DEVICE : ISV_ECUDA, "isv_linear4_create: %s", cudaGetErrorString(e));
    }
    *out = l;
    return ISV_OK;
}

int isv_linear4_forward(isv_linear4 *l, const void *x_dev, void *y_dev, float *y_f32_dev, int32_t M, void *stream) {
    if (!l) return err(ISV_EINVAL, "null handle");
    if (!x_dev || (!y_dev && !y_f32_dev)) return err(ISV_EINVAL, "x and one of y / y_f32 must be given");
    if (reinterpret_cast<uintptr_t>(x_dev) & 15u) return err(ISV_EINVAL, "x must be 16-byte aligned");
    if (M < 1 || M > l->max_M) return err(ISV_EINVAL, "M (%d) must be in [1, %d]", M, l->max_M);
    if ((reinterpret_cast<uintptr_t>(y_dev) & 1u) || (reinterpret_cast<uintptr_t>(y_f32_dev) & 3u))
        return err(ISV_EINVAL, "outputs must be aligned to their elements");
    Linear4Params p{};
    p.w = reinterpret_cast<const uint4 *>(l->w); p.scales = reinterpret_cast<const uint2 *>(l->scales); p.x = static_cast<const uint16_t *>(x_dev);
    p.y = static_cast<uint16_t *>(y_dev); p.y_f32 = y_f32_dev;
    p.M = M; p.N = l->N; p.K = l->K;
    OnDevice on(l->device);
    if (on.e != cudaSuccess) return err(ISV_ECUDA, "isv_linear4_forward: %s", cudaGetErrorString(on.e));
    const int nt = M <= 8 ? 1 : M <= 16 ? 2 : 4;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(l->blocks * l->cluster), (unsigned)((M + 8 * nt - 1) / (8 * nt)));
    cfg.blockDim = dim3(kWarps * 32);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;   // see the kernel's griddepcontrol pair
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)l->cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t e = nt == 1   ? launch<1>(p, l->group, l->bf16, cfg)
                          : nt == 2 ? launch<2>(p, l->group, l->bf16, cfg)
                                    : launch<4>(p, l->group, l->bf16, cfg);
    return e == cudaSuccess ? ISV_OK : err(ISV_ECUDA, "isv_linear4_forward: %s", cudaGetErrorString(e));
}

}  // extern "C"
