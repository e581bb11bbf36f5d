// Parameter blocks and launchers of the 8-bit cache's kernels.  Plain pointers and sizes; nothing here owns memory.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/isv.h"

namespace isv {
namespace q8 {

constexpr int kBT = 16;   // tokens of a page

// Bytes of one (page, KV head): codes of K and V, two scales, padding to 16.
__host__ __device__ constexpr int unit_bytes(int d) { return 2 * kBT * d + 16; }

struct CacheParams {
    uint8_t *pool;              // [n_pages][Hkv] units
    uint8_t *tails;             // [n_seqs][K|V][Hkv][16][D] 16-bit
    const int32_t *table;       // [n_seqs][table_stride]
    const int32_t *lens;
    uint32_t *status;
    int32_t table_stride, max_blocks, n_pages, n_seqs, Hkv;
};

struct AttnParams {
    CacheParams c;
    const uint16_t *q;          // [n_seqs][Hq][D]
    void *out;
    float *out_f32;
    float *part_o;              // partial results of items that cross CTAs: [slot][values of a visit's heads], two slots a CTA
    float *part_ml;             // [slot][heads of a visit][m, l]
    int32_t *tickets;           // [grid][heads of a visit], zero between launches
    int32_t Hq, P, GT;          // Hq = Hkv * P * GT; a visit serves GT query heads
    float scale_log2;           // log2(e) / sqrt(D)
    uint32_t spin_limit;        // polls of a barrier before a wait gives up
    int32_t drop_first_copy;    // failure injection: the second visit of all, the first block's, is armed without issuing its copy
};

// Tokens of sequence s, clamped to what its table row and its tail slot hold.
__device__ __forceinline__ int seq_len(const CacheParams &c, int s, bool &bad) {
    const int n = c.lens[s], most = c.max_blocks * kBT + kBT - 1;
    bad = n < 0 || n > most;
    return min(max(n, 0), most);
}

// Two fp32 numbers in one register pair: the multiplications and additions below take one instruction for both.
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
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// a * b + c
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

// Shape of the attention kernel that serves GT query heads per visit at head_dim D.
int attn_head_rows(int GT);                                        // GT rounded up to whole tiles of 8
int attn_slots(int grid);                                          // partial results of a launch
size_t attn_smem(int D, int GT, int max_seqs);
cudaError_t attn_configure(int D, int GT, bool bf16, bool e4m3, size_t smem);
cudaError_t launch_attn(const AttnParams &p, int D, bool bf16, bool e4m3, int grid, size_t smem, cudaStream_t st);

}  // namespace q8
}  // namespace isv
