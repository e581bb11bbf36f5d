// Decode linear layers with 4-bit weights and a 16-bit scale per (row, group of k): y = x . w^T for a few tokens.
//
// The product is bound by reading the weights, half a byte each, and what the SMs have to do per byte is large: turning
// eight nibbles into 16-bit numbers takes nine instructions (fp16) or eleven (bf16), so the multiplications must not cost
// any.  They run on mma.m16n8k16 with 16 weight rows as the rows and 8 tokens as the columns (one token takes as long as eight; tcgen05 would want the widened weights
// in shared memory, i.e. a store and a load more per weight).  Nibbles become numbers by placing them in the mantissa of
// 1024 (fp16) or 128 (bf16) and subtracting: exact, as are the products; sums are fp32 and a group's sum is scaled once.
//
// isv_linear4_create lays the weights out in operand order: blocks of 32 rows, per block all of K in steps of 128 (padded with
// zeros), per step 64 bytes for each lane of a warp and behind them the step's scales: one bulk copy of contiguous memory.
// A warp streams its steps through a ring of its own in shared memory, so that the bytes in flight do not cost
// registers.  The warps of a CTA share a row block's K; where there are few blocks a cluster of CTAs does, and adds
// up through distributed shared memory.  The order of all sums is fixed.
//
// Measured on B200 (a call in a captured graph): 32000 x 4096 at one token 16.9 us (4.1 TB/s of weights and scales), 22016 x
// 4096 13.0, 4096 x 4096 5.8; 4096 x 11008 at 16 tokens 12.7; 22016 x 4096 at 32 tokens 45.5.  About 3.5 us are fixed; the
// rest is 59 ns a step and SM, where HBM would allow 50.  Issue slots are busy to 60 %, HBM to 35 % of its peak: what is
// left is latency, a warp's chain of wait, conversions and products.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
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
constexpr uint32_t kSpinLimit = 1u << 22;    // polls before a wait gives up (Linear4Params::spin_limit overrides it)
constexpr uint32_t kDrainLimit = 1u << 14;   // for each copy that may be in flight behind a lost one: tens of ms

__host__ __device__ constexpr int step_bytes(int group) { return kRows * kStep / 2 + kRows * (kStep / group) * 2; }

struct Linear4Params {
    const uint8_t *w;          // [blocks][steps][step_bytes]: weights [4 chunks][32 lanes][16], scales [groups][8][4] (rows g, g + 8, ..)
    const uint16_t *x;
    uint16_t *y;
    float *y_f32;
    uint32_t *status;
    int32_t M, N, K, blocks;
    uint32_t spin_limit;       // polls of a barrier before a wait gives up
    int32_t drop_first_copy;   // failure injection: warp 0 of CTA 0 arms its first slot without issuing the copy
};

struct PackParams {
    const uint8_t *w;          // [N][K / 2]
    const uint16_t *s;         // [N][K / group]
    uint8_t *out;
    int32_t N, K, group, blocks, steps;
};

// Word i of a lane (4 g + c) in a chunk: row tile i / 2, k-step i % 2.  Its nibble 4 e + r belongs to operand register r:
// row g + 8 * (r % 2) of the tile, k = 8 c + 4 (i % 2) + 2 (r / 2) + e of the chunk.  Rows from N and k from K on are zeros.
__global__ void pack_kernel(PackParams p) {
    const int words = kRows * kStep / 8, halves = kRows * (kStep / p.group), bytes = step_bytes(p.group);
    for (long long id = blockIdx.x; id < (long long)p.blocks * p.steps; id += gridDim.x) {
        const int step = (int)(id % p.steps);
        const long long row0 = id / p.steps * kRows;
        uint8_t *out = p.out + (size_t)id * bytes;
        for (int t = threadIdx.x; t < words; t += blockDim.x) {
            const int i = t & 3, lane = (t >> 2) & 31, g = lane >> 2, c = lane & 3, chunk = t >> 7;
            uint32_t w = 0;
            for (int n = 0; n < 8; ++n) {
                const int r = n & 3, e = n >> 2;
                const long long row = row0 + (i >> 1) * 16 + g + 8 * (r & 1);
                const int k = step * kStep + chunk * kChunk + 8 * c + 4 * (i & 1) + 2 * (r >> 1) + e;
                uint32_t u = 8;
                if (row < p.N && k < p.K) {
                    const uint8_t b = p.w[row * (p.K / 2) + k / 2];
                    u = k & 1 ? b >> 4 : b & 15;
                }
                w |= u << (4 * n);
            }
            reinterpret_cast<uint32_t *>(out)[t] = w;
        }
        for (int t = threadIdx.x; t < halves; t += blockDim.x) {
            const int i = t & 3, g = (t >> 2) & 7, group = step * (kStep / p.group) + (t >> 5);
            const long long row = row0 + g + 8 * i;
            reinterpret_cast<uint16_t *>(out + kRows * kStep / 2)[t] = row < p.N && group < p.K / p.group ? p.s[row * (p.K / p.group) + group] : 0;
        }
    }
}

__device__ __forceinline__ uint32_t s32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, uint32_t limit) {
    for (uint32_t i = 0; i < limit; ++i) {
        uint32_t ok;
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return true;
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

// (x & mask) | bits in one instruction (two immediate operands would make it two)
__device__ __forceinline__ uint32_t mask_or(uint32_t x, uint32_t mask, uint32_t bits) {
    uint32_t y;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(y) : "r"(x), "r"(mask), "r"(bits));
    return y;
}

// Eight nibbles u -> four pairs of u - 8.
template <bool BF16>
__device__ __forceinline__ void widen(uint32_t w, uint32_t (&a)[4]) {
    if (BF16) {
        const __nv_bfloat162 base = __floats2bfloat162_rn(136.f, 136.f);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            uint32_t v = mask_or(w >> (4 * r), 0x000f000fu, 0x43004300u);       // 128 + u
            const __nv_bfloat162 d = __hsub2(*reinterpret_cast<__nv_bfloat162 *>(&v), base);
            a[r] = *reinterpret_cast<const uint32_t *>(&d);
        }
    } else {
        const __half2 base = __floats2half2_rn(1032.f, 1032.f), part = __floats2half2_rn(0.0625f, 0.0625f),
                      base16 = __floats2half2_rn(-72.f, -72.f);
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
            const uint32_t v = w >> (4 * r);
            uint32_t even = mask_or(v, 0x000f000fu, 0x64006400u), odd = mask_or(v, 0x00f000f0u, 0x64006400u);   // 1024 + u, 1024 + 16 u
            const __half2 x = __hsub2(*reinterpret_cast<__half2 *>(&even), base);
            const __half2 y = __hfma2(*reinterpret_cast<__half2 *>(&odd), part, base16);
            a[r] = *reinterpret_cast<const uint32_t *>(&x);
            a[r + 1] = *reinterpret_cast<const uint32_t *>(&y);
        }
    }
}

template <int NT, int RW>
struct Shape {
    static constexpr int COLS = 8 * NT, KW = kWarps / RW, TILE = kRows * RW, PITCH = TILE + 1;
    static constexpr int BUF = NT == 4 ? 1 : 2;                        // two buffers of sums: one barrier a tile
    static constexpr int SUMS = KW * COLS * PITCH;
    // what registers and shared memory allow: CTAs of an SM, and steps that a warp has in flight (about 150 KB an SM)
    static constexpr int RESIDENT = NT == 1 ? 3 : 2, RING = NT == 1 ? 3 : 4;
    static constexpr size_t smem(int group) { return (size_t)kWarps * RING * (step_bytes(group) + 8) + (size_t)BUF * SUMS * 4; }
};

// NT tiles of 8 tokens, RW blocks of rows side by side in a CTA (its other warps share K); blockIdx.y counts passes of 8 * NT
// tokens.  CTAs (clusters) walk the row tiles, and a warp's ring goes on across the border between two of them.
template <int NT, int RW, int GROUP, bool BF16>
__global__ void __launch_bounds__(kWarps * 32, Shape<NT, RW>::RESIDENT) linear4_kernel(const __grid_constant__ Linear4Params p) {
    using SH = Shape<NT, RW>;
    constexpr int CHUNKS = kStep / kChunk, GROUPS = kStep / GROUP, PER = GROUP / kChunk;
    constexpr int COLS = SH::COLS, KW = SH::KW, TILE = SH::TILE, PITCH = SH::PITCH, BUF = SH::BUF, BYTES = step_bytes(GROUP);
    extern __shared__ __align__(128) uint8_t smem[];
    uint8_t *ring = smem;                                              // [kWarps][RING][BYTES]
    uint64_t *bars = reinterpret_cast<uint64_t *>(ring + kWarps * SH::RING * BYTES);
    float *sums = reinterpret_cast<float *>(bars + kWarps * SH::RING);    // [BUF][KW][COLS][PITCH]
    cg::cluster_group cluster = cg::this_cluster();
    const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const int rw = warp % RW, kw = warp / RW, m0 = blockIdx.y * COLS;
    const int steps = (p.K + kStep - 1) / kStep, tiles = (p.blocks + RW - 1) / RW, stride = gridDim.x / cs;
    const int first = steps * rank / cs + kw;
    int end = steps * (rank + 1) / cs;

    uint8_t *mine = ring + warp * SH::RING * BYTES;
    const uint32_t bar0 = s32(bars + warp * SH::RING);
    if (lane < SH::RING) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar0 + 8 * lane) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncwarp();
    int next_tile = blockIdx.x / cs, next_step = first;
    const uint8_t *next = p.w + ((size_t)(next_tile * RW + rw) * steps + first) * BYTES;
    bool fetching = first < end && next_tile * RW + rw < p.blocks;
    auto fetch = [&](int slot, bool drop) {
        if (!fetching) return;
        if (lane == 0) {
            arm(bar0 + 8 * slot, BYTES);
            if (!drop) copy_in(s32(mine + slot * BYTES), next, BYTES, bar0 + 8 * slot);
        }
        next_step += KW;
        next += KW * BYTES;
        if (next_step >= end) {
            next_step = first;
            next_tile += stride;
            next = p.w + ((size_t)(next_tile * RW + rw) * steps + first) * BYTES;
            fetching = next_tile * RW + rw < p.blocks;
        }
    };
#pragma unroll 1
    for (int i = 0; i < SH::RING; ++i) fetch(i, p.drop_first_copy && i + warp + blockIdx.x + blockIdx.y == 0);   // the weights do not change: they are on their way before the predecessor has ended
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // x of one chunk, loaded one chunk ahead (a whole step of it would cost 32 tokens the second CTA of an SM)
    uint4 x[NT];
    const uint16_t *xs = p.x + (size_t)(m0 + g) * p.K + 8 * c;
    auto load_x = [&](uint4 (&to)[NT], int k) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
            to[nt] = m0 + nt * 8 + g < p.M && k < p.K ? *reinterpret_cast<const uint4 *>(xs + (size_t)nt * 8 * p.K + k) : make_uint4(0, 0, 0, 0);
    };
    load_x(x, first * kStep);
    int slot = 0;
    uint32_t phase = 0;
    int turn = 0;
    for (int tile = blockIdx.x / cs; tile < tiles; tile += stride, turn ^= BUF - 1) {
        float total[2][NT][4];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) total[t][nt][i] = 0.f;
#pragma unroll 1
        for (int step = first; step < end && tile * RW + rw < p.blocks; step += KW) {
            const int after = (step + KW < end ? step + KW : first) * kStep;
            if (!__all_sync(~0u, wait(bar0 + 8 * slot, phase, p.spin_limit))) {
                // A copy did not arrive in time: the warp issues no more of them, gives those in flight one more bounded
                // chance, so that none lands in memory that is somebody else's by then (a slot without one takes the whole
                // limit too), and goes on to the barriers ahead with sums that are incomplete.
#pragma unroll 1
                for (int i = 0; i < SH::RING; ++i) {
                    wait(bar0 + 8 * slot, phase, kDrainLimit);
                    if (++slot == SH::RING) { slot = 0; phase ^= 1u; }
                }
                if (lane == 0) atomicOr(p.status, ISV_STATUS_WAIT_EXPIRED);
                fetching = false;
                end = 0;           // no further step, in this tile or another
                break;
            }
            const uint8_t *in = mine + slot * BYTES;
#pragma unroll
            for (int i0 = 0; i0 < GROUPS; ++i0) {
                float part[2][NT][4];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) part[t][nt][i] = 0.f;
#pragma unroll
                for (int i = i0 * PER; i < (i0 + 1) * PER; ++i) {
                    uint4 next_x[NT];
                    load_x(next_x, i + 1 < CHUNKS ? step * kStep + (i + 1) * kChunk : after);
                    const uint4 w = *reinterpret_cast<const uint4 *>(in + 512 * i + 16 * lane);
                    const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t a[4];
                        widen<BF16>(words[j], a);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            mma<BF16>(part[j >> 1][nt], a, j & 1 ? x[nt].z : x[nt].x, j & 1 ? x[nt].w : x[nt].y);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) x[nt] = next_x[nt];
                }
                const uint2 sc = *reinterpret_cast<const uint2 *>(in + kRows * kStep / 2 + 64 * i0 + 8 * g);
                const float s[4] = {to_f32<BF16>(sc.x & 0xffffu), to_f32<BF16>(sc.x >> 16), to_f32<BF16>(sc.y & 0xffffu), to_f32<BF16>(sc.y >> 16)};
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) total[t][nt][i] += part[t][nt][i] * s[2 * t + (i >> 1)];
            }
            __syncwarp();
            fetch(slot, false);
            if (++slot == SH::RING) { slot = 0; phase ^= 1u; }
        }
        float *mine_sums = sums + turn * SH::SUMS;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    mine_sums[(kw * COLS + nt * 8 + 2 * c + (i & 1)) * PITCH + rw * kRows + t * 16 + g + 8 * (i >> 1)] = total[t][nt][i];
        if (cs > 1) cluster.sync(); else __syncthreads();
        const int cols = min(COLS, p.M - m0);
        // the CTAs of a cluster share the outputs; each adds the warps of all of them in order
        for (int o = rank * kWarps * 32 + threadIdx.x; o < cols * TILE; o += cs * kWarps * 32) {
            const int m = o / TILE, r = o % TILE, n = tile * TILE + r;
            float v = 0.f;
            for (int k = 0; k < cs; ++k) {
                const float *other = mine_sums;
                if (cs > 1) other = cluster.map_shared_rank(other, k);
#pragma unroll
                for (int i = 0; i < KW; ++i) v += other[(i * COLS + m) * PITCH + r];
            }
            if (n < p.N) {
                const size_t at = (size_t)(m0 + m) * p.N + n;
                if (p.y_f32) p.y_f32[at] = v;
                if (p.y) p.y[at] = BF16 ? __bfloat16_as_ushort(__float2bfloat16(v)) : __half_as_ushort(__float2half(v));
            }
        }
        if (BUF == 1) { if (cs > 1) cluster.sync(); else __syncthreads(); }
    }
    if (cs > 1) cluster.sync();   // nobody leaves while its sums may be read
}

template <int NT, int RW, int GROUP>
cudaError_t launch(const Linear4Params &p, bool bf16, cudaLaunchConfig_t cfg) {
    cfg.dynamicSmemBytes = Shape<NT, RW>::smem(GROUP);
    return bf16 ? cudaLaunchKernelEx(&cfg, linear4_kernel<NT, RW, GROUP, true>, p)
                : cudaLaunchKernelEx(&cfg, linear4_kernel<NT, RW, GROUP, false>, p);
}
template <int NT, int RW, int GROUP>
cudaError_t configure(bool bf16) {
    const int smem = (int)Shape<NT, RW>::smem(GROUP);
    return bf16 ? cudaFuncSetAttribute(linear4_kernel<NT, RW, GROUP, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)
                : cudaFuncSetAttribute(linear4_kernel<NT, RW, GROUP, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
}
template <int NT, int RW>
cudaError_t configure(int group, bool bf16) {
    return group == 32 ? configure<NT, RW, 32>(bf16) : group == 64 ? configure<NT, RW, 64>(bf16) : configure<NT, RW, 128>(bf16);
}
cudaError_t configure(int group, bool bf16) {
    cudaError_t e = configure<1, 1>(group, bf16);
    if (e == cudaSuccess) e = configure<2, 1>(group, bf16);
    if (e == cudaSuccess) e = configure<4, 1>(group, bf16);
    if (e == cudaSuccess) e = configure<1, 4>(group, bf16);
    if (e == cudaSuccess) e = configure<2, 4>(group, bf16);
    if (e == cudaSuccess) e = configure<4, 4>(group, bf16);
    return e;
}
template <int NT, int RW>
cudaError_t launch(const Linear4Params &p, int group, bool bf16, const cudaLaunchConfig_t &cfg) {
    if (group == 32) return launch<NT, RW, 32>(p, bf16, cfg);
    if (group == 64) return launch<NT, RW, 64>(p, bf16, cfg);
    return launch<NT, RW, 128>(p, bf16, cfg);
}

}  // namespace

struct isv_linear4 {
    int N = 0, K = 0, group = 0, max_M = 0, device = 0, blocks = 0, sms = 0;
    bool bf16 = false;
    std::atomic<uint32_t> wait_polls{kSpinLimit};
    std::atomic<int32_t> lost_copies{0};      // failure injection: launches still to lose a copy
    uint8_t *w = nullptr;
    uint32_t *status = nullptr;
};

extern "C" {

int isv_linear4_free(isv_linear4 *l) {
    if (!l) return err(ISV_EINVAL, "null handle");
    OnDevice on(l->device);
    cudaDeviceSynchronize();   // calls may have been made on any stream
    cudaFree(l->w);
    cudaFree(l->status);
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
    l->sms = sms;
    const int steps = (K + kStep - 1) / kStep;
    if (e == cudaSuccess) e = configure(group, l->bf16);
    if (e == cudaSuccess) e = cudaMalloc((void **)&l->w, (size_t)l->blocks * steps * step_bytes(group));
    if (e == cudaSuccess) e = cudaMalloc((void **)&l->status, 4);
    if (e == cudaSuccess) e = cudaMemsetAsync(l->status, 0, 4, st);
    if (e == cudaSuccess) {
        const PackParams p = {static_cast<const uint8_t *>(w4_dev), static_cast<const uint16_t *>(scales_dev), l->w, N, K, group, l->blocks, steps};
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
    p.w = l->w; p.status = l->status; p.x = static_cast<const uint16_t *>(x_dev);
    p.y = static_cast<uint16_t *>(y_dev); p.y_f32 = y_f32_dev;
    p.M = M; p.N = l->N; p.K = l->K; p.blocks = l->blocks;
    p.spin_limit = l->wait_polls.load();
    if (l->lost_copies.load() > 0) p.drop_first_copy = l->lost_copies.fetch_sub(1) > 0;
    OnDevice on(l->device);
    if (on.e != cudaSuccess) return err(ISV_ECUDA, "isv_linear4_forward: %s", cudaGetErrorString(on.e));
    const int nt = M <= 8 ? 1 : M <= 16 ? 2 : 4;
    // From five tokens on x is as much traffic as a block's weights: four blocks then share what a CTA reads of it,
    // if enough CTAs are left.
    const int rw = M > 4 && l->blocks >= l->sms / 8 ? 4 : 1;
    const int tiles = (l->blocks + rw - 1) / rw, steps = (l->K + kStep - 1) / kStep;
    // Clusters of any size up to 8 share a tile's K.  A round of tiles takes the steps of a warp and about one and a half
    // steps' time for its start and its sums (with 32 columns of sums eight, and one more for each CTA); the size with the shortest sum of rounds is
    // taken.  Against a cluster of 1 throughout: 4096 x 11008 at one token 12.2 -> 9.1 us, 2560 x 10240 8.0 -> 6.2; against
    // as many CTAs as are resident: 22016 x 4096 at 16 tokens 25.8 -> 23.7.
    const int room = (nt == 1 ? Shape<1, 1>::RESIDENT : nt == 2 ? Shape<2, 1>::RESIDENT : Shape<4, 1>::RESIDENT) * l->sms;
    const int kw = kWarps / rw;
    int cluster = 1;
    long long best = 0;
    for (int cs = 1; cs <= kMaxCluster && cs <= std::min(steps, room); ++cs) {
        const long long rounds = (tiles + room / cs - 1) / (room / cs), cost = rounds * (2 * ((steps + cs * kw - 1) / (cs * kw)) + (nt == 4 ? 16 + 2 * cs : 3));
        if (cs == 1 || cost < best) { best = cost; cluster = cs; }
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(std::min(tiles, std::max(1, room / cluster)) * cluster), (unsigned)((M + 8 * nt - 1) / (8 * nt)));
    cfg.blockDim = dim3(kWarps * 32);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;   // see the kernel's griddepcontrol pair
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cudaError_t e;
    if (rw == 1) e = nt == 1 ? launch<1, 1>(p, l->group, l->bf16, cfg) : nt == 2 ? launch<2, 1>(p, l->group, l->bf16, cfg) : launch<4, 1>(p, l->group, l->bf16, cfg);
    else e = nt == 1 ? launch<1, 4>(p, l->group, l->bf16, cfg) : nt == 2 ? launch<2, 4>(p, l->group, l->bf16, cfg) : launch<4, 4>(p, l->group, l->bf16, cfg);
    return e == cudaSuccess ? ISV_OK : err(ISV_ECUDA, "isv_linear4_forward: %s", cudaGetErrorString(e));
}

int isv_linear4_status(isv_linear4 *l, void *stream, uint32_t *status_out) {
    if (!l || !status_out) return err(ISV_EINVAL, "null argument");
    OnDevice on(l->device);
    if (on.e != cudaSuccess) return err(ISV_ECUDA, "isv_linear4_status: %s", cudaGetErrorString(on.e));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaMemcpyAsync(status_out, l->status, 4, cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e == cudaSuccess && *status_out) {
        e = cudaMemsetAsync(l->status, 0, 4, st);
        if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    }
    if (e != cudaSuccess) return err(ISV_ECUDA, "isv_linear4_status: %s", cudaGetErrorString(e));
    if (*status_out) return err(ISV_EDEVICE_STATUS, "the 4-bit linear kernel reported status 0x%x", *status_out);
    return ISV_OK;
}

int isv_linear4_set_wait_limit(isv_linear4 *l, uint32_t polls) {
    if (!l) return err(ISV_EINVAL, "null handle");
    l->wait_polls = polls ? polls : kSpinLimit;
    return ISV_OK;
}

int isv_linear4_inject_lost_copy(isv_linear4 *l, int32_t launches) {
    if (!l) return err(ISV_EINVAL, "null handle");
    if (launches < 0) return err(ISV_EINVAL, "launches must not be negative");
    l->lost_copies = launches;
    return ISV_OK;
}

}  // extern "C"
