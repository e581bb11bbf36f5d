// Verification of drafted tokens against the target model's probabilities (isv_draft_verify, described in include/isv.h).
//
// Draft i of a sequence is kept while u_i q_i(x_i) < p_i(x_i) (exact in 64 bits: 24-bit factors).  At the first one that
// is not kept the next token comes from the residual max(p - q, 0), behind the last draft from p itself: the lowest index
// whose running sum exceeds u times the total.  Which index that is hangs on sums over a whole vocabulary, so these are
// taken in 64 bits (in 32 bits, neighbouring tokens of probability 1e-5 would trade places in one call of a hundred).
//
// A cluster of up to eight CTAs does a sequence.  Every warp owns a contiguous part of the row and sums it once, group by group;
// the parts' totals are exchanged through distributed shared memory; the warp whose part holds the crossing finds the group
// in its sums and walks that group alone again.  So the row is read from HBM once, and nothing is kept but the groups' sums.
// Bound by a chain of dependent loads (counts, drafts, their probabilities, the row, the group), then by HBM.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdio>

#include "../../include/isv.h"

namespace cg = cooperative_groups;

namespace isv {
int set_error(int code, const char *msg);
}

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCtas = 8;            // of a cluster (the portable maximum)
constexpr int kMaxDraft = 1024;
constexpr int kGroups = 64;            // groups of a warp's part, at most

int err(int code, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return isv::set_error(code, buf);
}

struct Params {
    const void *target, *draft;        // rows of V probabilities
    const int32_t *firsts;             // target row of a sequence's first draft, or NULL: s * (K + 1)
    const int32_t *drafted, *counts;   // [n_seqs][K], [n_seqs]
    const float *u;                    // [n_seqs][K + 1]
    const int32_t *lens;
    int32_t *tokens, *accepted, *lens_out;
    uint32_t *status;
    int32_t V, K, n_rows, ctas;
};

template <typename T>
__device__ __forceinline__ float number(T x);
template <>
__device__ __forceinline__ float number<float>(float x) { return x; }
template <>
__device__ __forceinline__ float number<__half>(__half x) { return __half2float(x); }
template <>
__device__ __forceinline__ float number<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }

// A probability: what is negative or no number counts as 0.
template <typename T>
__device__ __forceinline__ float chance(T x) { return fmaxf(number<T>(x), 0.f); }

// E adjacent probabilities from index i on; those at `end` and behind it are 0.
template <typename T, bool VEC, int E>
__device__ __forceinline__ void load(const T *row, int i, int end, float (&x)[E]) {
    if (VEC && i + E <= end) {
        const uint4 w = *reinterpret_cast<const uint4 *>(row + i);
        const T *e = reinterpret_cast<const T *>(&w);
#pragma unroll
        for (int y = 0; y < E; ++y) x[y] = chance<T>(e[y]);
        return;
    }
#pragma unroll
    for (int y = 0; y < E; ++y) x[y] = i + y < end ? chance<T>(row[i + y]) : 0.f;
}

// What a lane holds of a row before it is used: 16 bytes of adjacent probabilities, or (rows that are not aligned) elements that
// lie 32 apart, so that a warp's loads are contiguous either way.
template <typename T, bool VEC>
struct Batch {
    static constexpr int E = 16 / sizeof(T), DEEP = VEC ? 4 : 16 / E;       // loads in flight: 4 of 16 bytes, or 16 of an element
    static constexpr int STEP = 32 * E * DEEP;                              // elements of a warp's batch
    uint4 w[VEC ? DEEP : 1];
    T e[VEC ? 1 : DEEP * E];
    __device__ __forceinline__ static int index(int i0, int lane, int d, int y) {
        return VEC ? i0 + (d * 32 + lane) * E + y : i0 + (d * E + y) * 32 + lane;
    }
    __device__ __forceinline__ void load(const T *row, int i0, int lane, int end) {
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            if constexpr (VEC) {
                // a row's length is a multiple of E here: a vector is inside or behind
                w[d] = index(i0, lane, d, 0) < end ? *reinterpret_cast<const uint4 *>(row + index(i0, lane, d, 0)) : make_uint4(0, 0, 0, 0);
            } else {
#pragma unroll
                for (int y = 0; y < E; ++y) e[d * E + y] = index(i0, lane, d, y) < end ? row[index(i0, lane, d, y)] : T(0.f);
            }
        }
    }
    __device__ __forceinline__ float at(int d, int y) const {
        return chance<T>(VEC ? reinterpret_cast<const T *>(&w[d])[y] : e[d * E + y]);
    }
};

// Weight of one token in the residual: what the target gives it beyond the draft.
__device__ __forceinline__ double beyond(float p, float q) {
    const double r = (double)p - (double)q;
    return r > 0 ? r : 0.0;
}

// A sum as an fp32 number and what its roundings left.
struct Sum {
    float hi = 0.f, lo = 0.f;
    // x + rest, |rest| far below |x|
    __device__ __forceinline__ void add(float x, float rest) {
        const float t = __fadd_rn(hi, x), z = __fsub_rn(t, hi);
        lo = __fadd_rn(lo, __fadd_rn(__fadd_rn(__fsub_rn(hi, __fsub_rn(t, z)), __fsub_rn(x, z)), rest));
        hi = t;
    }
    // what the target gives beyond the draft, exactly: the difference and its rounding
    __device__ __forceinline__ void add_beyond(float p, float q) {
        const bool more = p > q;
        const float d = __fsub_rn(p, q), rest = __fsub_rn(__fsub_rn(p, d), q);
        add(more ? d : 0.f, more ? rest : 0.f);
    }
};
__device__ __forceinline__ double warp_sum(Sum x) {
#pragma unroll
    for (int i = 16; i; i >>= 1) {
        const float hi = __shfl_xor_sync(~0u, x.hi, i), lo = __shfl_xor_sync(~0u, x.lo, i);
        // both lanes add the smaller number to the larger, so that they get the same bits
        Sum y;
        y.hi = fmaxf(x.hi, hi);
        y.lo = __fadd_rn(x.lo, lo);
        y.add(fminf(x.hi, hi), 0.f);
        x = y;
    }
    return (double)x.hi + (double)x.lo;
}

__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int i = 16; i; i >>= 1) x += __shfl_xor_sync(~0u, x, i);
    return x;
}

// Of n weights get(0) .. get(n - 1): the first whose running sum, from `start` on, passes the border; the last one with any weight, if
// rounding (or u >= 1) lets none do so; -1 if there is none.  `before` becomes the sum ahead of it.  A lane has a few in a row.
template <typename Get>
__device__ __forceinline__ int crossing(int n, Get get, double start, double border, double &before) {
    const int lane = threadIdx.x & 31, each = (n + 31) / 32, lo = lane * each, hi = min(n, lo + each);
    double mine = 0;
    for (int i = lo; i < hi; ++i) mine += get(i);
    double up = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const double z = __shfl_up_sync(~0u, up, d);
        if (lane >= d) up += z;
    }
    double at = start + (up - mine), ahead = 0;
    int hit = 0x7fffffff, any = -1;
    for (int i = lo; i < hi; ++i) {
        const double w = get(i);
        if (w > 0 && hit == 0x7fffffff) {
            any = i;
            ahead = at;
            if (at + w > border) hit = i;
        }
        at += w;
    }
    const int first = __reduce_min_sync(~0u, hit), last = __reduce_max_sync(~0u, any);
    const int found = first != 0x7fffffff ? first : last;
    before = __shfl_sync(~0u, ahead, found < 0 ? 0 : found / each);
    return found;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, 2) verify_kernel(const Params p) {
    constexpr int E = 16 / sizeof(T);
    cg::cluster_group cluster = cg::this_cluster();
    __shared__ int took_s, refused_s, row_s, bad_s, owner_s;
    __shared__ double border_s, before_s;
    __shared__ double totals[kMaxCtas * kWarps][2];   // of each warp's part: residual, target
    __shared__ double groups[kWarps][kGroups];        // of each group of this CTA's parts
    const int s = blockIdx.x / p.ctas, rank = blockIdx.x % p.ctas;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const T *target = static_cast<const T *>(p.target), *draft = static_cast<const T *>(p.draft);

    if (warp == 0) {
        const int count = p.counts[s];
        int n = min(max(count, 0), p.K);
        const long long first = p.firsts ? (long long)p.firsts[s] : (long long)s * (p.K + 1);
        const int room = first < 0 || first >= p.n_rows ? 0 : p.n_rows - (int)first;
        uint32_t bad = n != count || n + 1 > room ? ISV_STATUS_BAD_LENGTH : 0;
        n = min(n, room - 1);
        int took = 0;
        for (int i0 = 0; i0 < n; i0 += 32) {
            const int i = i0 + lane;
            bool keep = false;
            if (i < n) {
                const int x = p.drafted[(long long)s * p.K + i];
                const float u = p.u[(long long)s * (p.K + 1) + i];
                if (x < 0 || x >= p.V) {
                    bad |= ISV_STATUS_BAD_TOKEN;
                } else {
                    const double px = chance<T>(target[(first + i) * p.V + x]);
                    const double qx = draft ? (double)chance<T>(draft[((long long)s * p.K + i) * p.V + x]) : 1.0;
                    keep = (double)u * qx < px;
                }
            }
            const unsigned not_kept = __ballot_sync(~0u, !keep);
            took += not_kept ? __ffs(not_kept) - 1 : 32;
            if (not_kept) break;
        }
        took = min(took, max(n, 0));
        bad = __reduce_or_sync(~0u, bad);
        if (lane == 0) {
            took_s = took;
            refused_s = took < n;
            row_s = room > 0 ? (int)first + took : -1;
            bad_s = bad;
        }
    }
    __syncthreads();
    const int took = took_s;
    const bool refused = refused_s, some = row_s >= 0;
    const float u_last = p.u[(long long)s * (p.K + 1) + p.K];
    const int x = refused ? p.drafted[(long long)s * p.K + took] : -1;
    const T *prow = some ? target + (long long)row_s * p.V : nullptr;
    const T *qrow = refused && draft ? draft + ((long long)s * p.K + took) * p.V : nullptr;

    // this warp's part of the row: whole steps of a warp, so that vector loads stay aligned
    const int parts = p.ctas * kWarps, steps = (p.V + 32 * E - 1) / (32 * E);
    const int part = rank * kWarps + warp;
    const int lo = (int)((long long)steps * part / parts) * 32 * E, hi = min(p.V, (int)((long long)steps * (part + 1) / parts) * 32 * E);
    using Rows = Batch<T, VEC>;
    int kind = refused ? 0 : 1;         // 0: from the residual, 1: from the target
    auto weight = [&](float target, float draft_, int i) {
        return kind == 1 ? beyond(target, 0.f) : qrow ? beyond(target, draft_) : i == x ? 0.0 : beyond(target, 0.f);
    };
    const int batches = (hi - lo + Rows::STEP - 1) / Rows::STEP, per_group = max(1, (batches + kGroups - 1) / kGroups) * Rows::STEP;
    for (;; kind = 1) {
        double part_sum = 0;
        for (int g = 0; lo + g * per_group < hi && some; ++g) {
            const int end = min(hi, lo + (g + 1) * per_group);
            Sum sum;
            for (int i0 = lo + g * per_group; i0 < end; i0 += Rows::STEP) {
                Rows a, b;
                a.load(prow, i0, lane, hi);
                if (kind == 0 && qrow) b.load(qrow, i0, lane, hi);
#pragma unroll
                for (int d = 0; d < Rows::DEEP; ++d)
#pragma unroll
                    for (int y = 0; y < E; ++y) {
                        const bool left_out = kind == 0 && !qrow && Rows::index(i0, lane, d, y) == x;
                        sum.add_beyond(left_out ? 0.f : a.at(d, y), kind == 0 && qrow ? b.at(d, y) : 0.f);
                    }
            }
            const double group_sum = warp_sum(sum);
            if (lane == 0) groups[warp][g] = group_sum;
            part_sum += group_sum;
        }
        if (lane < p.ctas) cluster.map_shared_rank(totals, lane)[part][kind] = part_sum;
        cluster.sync();
        // one warp adds up, and finds the part that holds the crossing
        if (warp == 0) {
            double mine = 0;
            for (int i = lane; i < parts; i += 32) mine += totals[i][kind];
            const double total = warp_sum(mine);
            double before = 0;
            const double border = (double)u_last * total;
            const int owner = total > 0 ? crossing(parts, [&](int i) { return totals[i][kind]; }, 0.0, border, before) : -1;
            if (lane == 0) {
                owner_s = owner;
                border_s = border;
                before_s = before;
            }
        }
        __syncthreads();
        if (kind == 1 || owner_s >= 0) break;
        // nothing is left of the target beyond the draft: the same with the target alone
    }
    const double border = border_s, before = before_s;
    const int owner = owner_s;
    if (part == owner) {
        const int n = (hi - lo + per_group - 1) / per_group;
        double run = before;
        const int g = n > 1 ? crossing(n, [&](int i) { return groups[warp][i]; }, before, border, run) : 0;
        const int end = min(hi, lo + (g + 1) * per_group);
        constexpr int W = 16 / E;       // steps whose loads are in flight
        int token = -1, last = -1;
        for (int i0 = lo + g * per_group; i0 < end && token < 0; i0 += W * 32 * E) {
            float a[W][E], b[W][E];
#pragma unroll
            for (int k = 0; k < W; ++k) {
                load<T, VEC, E>(prow, i0 + (k * 32 + lane) * E, end, a[k]);
                if (qrow && kind == 0) load<T, VEC, E>(qrow, i0 + (k * 32 + lane) * E, end, b[k]);
            }
#pragma unroll
            for (int k = 0; k < W; ++k) {
                if (token >= 0 || i0 + k * 32 * E >= end) continue;
                const int i = i0 + (k * 32 + lane) * E;
                double w[E], mine = 0;
#pragma unroll
                for (int y = 0; y < E; ++y) {
                    w[y] = i + y < end ? weight(a[k][y], qrow && kind == 0 ? b[k][y] : 0.f, i + y) : 0.0;
                    mine += w[y];
                }
                double up = mine;
#pragma unroll
                for (int d = 1; d < 32; d *= 2) {
                    const double z = __shfl_up_sync(~0u, up, d);
                    if (lane >= d) up += z;
                }
                double c = run + (up - mine);
                run += __shfl_sync(~0u, up, 31);
                int hit = 0x7fffffff, any = -1;
#pragma unroll
                for (int y = 0; y < E; ++y) {
                    c += w[y];
                    if (w[y] > 0) {
                        any = i + y;
                        if (c > border) hit = min(hit, i + y);
                    }
                }
                hit = __reduce_min_sync(~0u, hit);
                last = max(last, __reduce_max_sync(~0u, any));
                if (hit != 0x7fffffff) token = hit;
            }
        }
        if (lane == 0) p.tokens[(long long)s * (p.K + 1) + took] = token >= 0 ? token : last;
    }
    if (rank == 0) {
        for (int i = threadIdx.x; i <= p.K; i += kThreads)
            if (i != took || owner < 0)
                p.tokens[(long long)s * (p.K + 1) + i] = i < took ? p.drafted[(long long)s * p.K + i] : -1;
        if (threadIdx.x == 0) {
            const int n = min(max(p.counts[s], 0), p.K);
            p.accepted[s] = took;
            if (p.lens_out) p.lens_out[s] = p.lens[s] - n + took;
            const uint32_t bad = bad_s | (owner < 0 ? ISV_STATUS_BAD_TOKEN : 0);
            if (bad && p.status) atomicOr(p.status, bad);
        }
    }
    cluster.sync();   // no CTA leaves while another may still write its totals there
}

template <typename T, bool VEC>
cudaError_t launch(const Params &p, int n_seqs, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(n_seqs * p.ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = p.ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, verify_kernel<T, VEC>, p);
}

}  // namespace

extern "C" int isv_draft_verify(const void *target_dev, const int32_t *row_starts_dev, int32_t n_rows, const void *draft_dev,
                                int32_t vocab, int32_t dtype, const int32_t *drafted_dev, const int32_t *n_draft_dev,
                                const float *uniforms_dev, const int32_t *seq_lens_dev, int32_t n_seqs, int32_t max_draft,
                                int32_t *tokens_dev, int32_t *accepted_dev, int32_t *lens_out_dev, uint32_t *status_dev,
                                void *stream) {
    const char *who = "isv_draft_verify";
    if (!target_dev || !drafted_dev || !n_draft_dev || !uniforms_dev || !tokens_dev || !accepted_dev)
        return err(ISV_EINVAL, "%s: target, drafted tokens, their counts, uniforms, tokens and accepted are required", who);
    if (lens_out_dev && !seq_lens_dev) return err(ISV_EINVAL, "%s: lens_out without seq_lens", who);
    if (dtype != ISV_F16 && dtype != ISV_BF16 && dtype != ISV_F32) return err(ISV_EINVAL, "%s: dtype f16/bf16/f32 only", who);
    const uintptr_t size = dtype == ISV_F32 ? 4 : 2, both = reinterpret_cast<uintptr_t>(target_dev) | reinterpret_cast<uintptr_t>(draft_dev);
    if (both % size) return err(ISV_EINVAL, "%s: probabilities must be aligned to their elements", who);
    if (vocab < 1 || vocab > (1 << 30)) return err(ISV_EINVAL, "%s: bad vocab (%d)", who, vocab);
    if (max_draft < 1 || max_draft > kMaxDraft) return err(ISV_EINVAL, "%s: max_draft (%d) must be in [1, %d]", who, max_draft, kMaxDraft);
    if (n_seqs < 0 || n_seqs > (1 << 20)) return err(ISV_EINVAL, "%s: bad n_seqs (%d)", who, n_seqs);
    if (n_rows < 0) return err(ISV_EINVAL, "%s: bad n_rows (%d)", who, n_rows);
    if (!row_starts_dev && (long long)n_seqs * (max_draft + 1) > n_rows)
        return err(ISV_EINVAL, "%s: n_rows (%d) must be at least n_seqs * (max_draft + 1) without row_starts", who, n_rows);
    if (n_seqs == 0) return ISV_OK;
    Params p{};
    p.target = target_dev; p.draft = draft_dev; p.firsts = row_starts_dev; p.drafted = drafted_dev; p.counts = n_draft_dev;
    p.u = uniforms_dev; p.lens = seq_lens_dev; p.tokens = tokens_dev; p.accepted = accepted_dev; p.lens_out = lens_out_dev;
    p.status = status_dev; p.V = vocab; p.K = max_draft; p.n_rows = n_rows;
    // As many CTAs a sequence as keep the GPU at two CTAs an SM, and a few thousand tokens a CTA.
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return err(ISV_ECUDA, "%s: %s", who, cudaGetErrorString(e));
    p.ctas = 1;
    while (p.ctas < kMaxCtas && (long long)n_seqs * p.ctas * 2 <= 2 * sms && vocab / (p.ctas * 2) >= 2048) p.ctas *= 2;
    const bool vec = both % 16 == 0 && vocab * size % 16 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == ISV_F32) e = vec ? launch<float, true>(p, n_seqs, st) : launch<float, false>(p, n_seqs, st);
    else if (dtype == ISV_F16) e = vec ? launch<__half, true>(p, n_seqs, st) : launch<__half, false>(p, n_seqs, st);
    else e = vec ? launch<__nv_bfloat16, true>(p, n_seqs, st) : launch<__nv_bfloat16, false>(p, n_seqs, st);
    return e == cudaSuccess ? ISV_OK : err(ISV_ECUDA, "%s: %s", who, cudaGetErrorString(e));
}
