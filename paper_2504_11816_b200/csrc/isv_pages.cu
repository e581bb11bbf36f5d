// Operations on the pages of a caller-owned paged cache (described in include/isv.h): copying pages, and the three
// operations on block tables (fork, resize, compact).
//
// The table operations need to know which pages are free.  That is derived each time from the table itself: every
// entry that a row's length covers sets its bit in a bitmap of the pool.  One thread-block cluster does a whole
// operation in one launch: each CTA marks the entries of its share of the rows in a bitmap of its own in shared
// memory, each CTA then takes one slice of the pages, ORs the others' bitmaps for it through distributed shared
// memory and counts; the exclusive prefix of those counts gives every page its rank among the free (or live)
// pages, and a rank says which table entry a free page goes to.  There are no atomics whose order matters.
// Bound by the latency of five phases that depend on one another (rows, marks, union, ranks, assignment), 1 to 2 us each:
// resize of 512 rows x 256 blocks in a pool of 65536 pages 8.7 us on B200; eight CTAs of 1024 threads (of 512: 10.7).
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdarg>
#include <cstdio>

#include "../../include/isv.h"

namespace cg = cooperative_groups;

namespace isv {
int set_error(int code, const char *msg);
}

namespace {

constexpr int kBT = 16;
constexpr int kCtas = 8;           // CTAs of the cluster (the portable maximum)
constexpr int kThreads = 1024;
constexpr int kMaxRows = 4096;
constexpr int kMaxDevices = 64;
constexpr int kCopyThreads = 256, kCopyUnroll = 4;
constexpr unsigned kCopyMaxGrid = 1u << 20;   // CTAs of a copy along x: the kernel's 32-bit counter of items takes that many past the last

int err(int code, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return isv::set_error(code, buf);
}

enum TableOp { FORK, RESIZE, COMPACT };

struct TableParams {
    const int32_t *table, *lens;
    const int32_t *other;        // FORK: parents; RESIZE: new lengths
    int32_t *table_out, *lens_out;
    int32_t *src, *dst, *counts; // FORK: copy pairs; COMPACT: moves and counts
    uint32_t *status;
    int32_t n_rows, n_in, stride, max_blocks, open_in_pool, n_pages, max_moves;
    int32_t words, slice;        // bitmap words in all, and of one CTA's slice
    int32_t row_threads;         // threads (a power of two) that share a row
};

__device__ __forceinline__ int blocks_of(const TableParams &p, int len, uint32_t &bad) {
    if (len < 0) { bad |= ISV_STATUS_BAD_LENGTH; return 0; }
    const int b = len / kBT + (p.open_in_pool && len % kBT ? 1 : 0);
    if (b > p.max_blocks) { bad |= ISV_STATUS_BAD_LENGTH; return p.max_blocks; }
    return b;
}

// What an operation does with a row: blocks [0, min(lo, hi)) stay, blocks [lo, hi) get fresh pages, blocks from hi on
// become ISV_BLOCK_NONE.
struct Row {
    int lo, hi;
};

// Exclusive prefix sums of one value per thread over the CTA; returns the thread's prefix, `total` the sum.
__device__ __forceinline__ int block_scan(int v, int *warp_sums, int &total) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int y = __shfl_up_sync(~0u, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();                       // the previous scan's readers are done
    if (lane == 31) warp_sums[w] = x;
    __syncthreads();
    if (w == 0) {
        int s = warp_sums[lane];
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int y = __shfl_up_sync(~0u, s, o);
            if (lane >= o) s += y;
        }
        warp_sums[lane] = s;
    }
    __syncthreads();
    total = warp_sums[31];
    return x - v + (w ? warp_sums[w - 1] : 0);
}

template <int OP>
__global__ void __launch_bounds__(kThreads, 1) table_kernel(TableParams p) {
    extern __shared__ uint32_t smem[];
    __shared__ int warp_sums[32];
    __shared__ int slice_live[kCtas];          // live pages of every slice: each CTA tells all
    uint32_t *bits = smem;                                              // [words]: this CTA's marks
    uint32_t *fin = bits + p.words;                                     // [slice]: all marks of this CTA's slice
    int *before = reinterpret_cast<int *>(fin + p.slice);               // [slice]: live pages of the slice before the word
    int *need = before + p.slice;                                       // [n_rows + 1]: fresh pages before row r
    int *rows_hi = need + p.n_rows + 1;                                 // [n_rows]: Row::hi; FORK: 2 * hi + (hi - lo)
    int *rows_lo = rows_hi + p.n_rows;                                  // RESIZE [n_rows]: Row::lo
    int *first = rows_lo;                                               // FORK [n_in]: first row that continues a parent
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), tid = threadIdx.x;
    uint32_t bad = 0;

    for (int i = tid; i < p.words; i += kThreads) bits[i] = 0;
    if (OP == FORK)
        for (int i = tid; i < p.n_in; i += kThreads) first[i] = p.n_rows;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    auto parent_of = [&](int r) {
        const int q = p.other[r];
        if (q >= 0 && q < p.n_in) return q;
        if (q != ISV_BLOCK_NONE) bad |= ISV_STATUS_BAD_BLOCK_ID;
        return -1;
    };
    if (OP == FORK) {
        __syncthreads();
        for (int r = tid; r < p.n_rows; r += kThreads) {
            const int q = parent_of(r);
            if (q >= 0) atomicMin(&first[q], r);
        }
        __syncthreads();
    }
    // every CTA has the whole list of rows
    for (int r = tid; r < p.n_rows; r += kThreads) {
        if (OP == FORK) {
            const int from = parent_of(r), len = from < 0 ? 0 : p.lens[from], hi = blocks_of(p, len, bad);
            int own = 0;             // 1: the row gets a page of its own for its open block
            if (hi > 0 && p.open_in_pool && len % kBT && len / kBT < p.max_blocks && first[from] < r) {
                const int page = p.table[(size_t)from * p.stride + hi - 1];
                own = page >= 0 && page < p.n_pages;
            }
            rows_hi[r] = 2 * hi + own;
        } else {
            rows_hi[r] = blocks_of(p, OP == RESIZE ? p.other[r] : p.lens[r], bad);
            if (OP == RESIZE) rows_lo[r] = blocks_of(p, p.lens[r], bad);
        }
    }
    __syncthreads();
    auto row_of = [&](int r) {
        const int x = rows_hi[r];
        return OP == FORK ? Row{x / 2 - (x & 1), x / 2} : OP == RESIZE ? Row{rows_lo[r], x} : Row{x, x};
    };

    // ---- marks; FORK also copies the kept entries to the new table
    const int per = kCtas * kThreads / p.row_threads;
    const int at = rank * kThreads + tid;
    for (int r = at / p.row_threads; r < p.n_rows; r += per) {
        const Row w = row_of(r);
        const int keep = min(w.lo, w.hi);
        const int32_t *from = p.table + (size_t)(OP == FORK ? (keep ? p.other[r] : 0) : r) * p.stride;
        for (int j = at % p.row_threads; j < keep; j += 4 * p.row_threads) {
            int id[4];                 // four loads in flight
#pragma unroll
            for (int i = 0; i < 4; ++i) id[i] = j + i * p.row_threads < keep ? from[j + i * p.row_threads] : ISV_BLOCK_NONE;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (OP == FORK && j + i * p.row_threads < keep) p.table_out[(size_t)r * p.stride + j + i * p.row_threads] = id[i];
                if (id[i] >= 0 && id[i] < p.n_pages) atomicOr(&bits[id[i] >> 5], 1u << (id[i] & 31));
                else if (id[i] != ISV_BLOCK_NONE) bad |= ISV_STATUS_BAD_BLOCK_ID;
            }
        }
    }
    cluster.barrier_arrive();              // this CTA's marks are there; what follows does not need the others'
    // ---- fresh pages before each row
    int wanted = 0;
    if (OP != COMPACT) {
        const int each = (p.n_rows + kThreads - 1) / kThreads;
        int sum = 0;
        for (int r = tid * each; r < min(tid * each + each, p.n_rows); ++r) {
            const Row w = row_of(r);
            sum += max(0, w.hi - w.lo);
        }
        // A pool has at most ISV_PAGES_MAX pages, so a demand beyond that is counted as that: the scan stays below 2^30, where
        // long tables could ask for more than 2^31 entries.  Prefixes below n_pages, the only ones that matter, are exact.
        int x = block_scan(min(sum, ISV_PAGES_MAX), warp_sums, wanted);
        for (int r = tid * each; r < min(tid * each + each, p.n_rows); ++r) {
            const Row w = row_of(r);
            need[r] = x;
            x += max(0, w.hi - w.lo);
        }
        if (tid == 0) need[p.n_rows] = wanted;
    }
    cluster.barrier_wait();

    // ---- this CTA's slice of the pool: all marks, and the live pages before each word
    const int each = (p.slice + kThreads - 1) / kThreads;
    int sum = 0;
    for (int i = 0; i < each; ++i) {
        const int k = tid * each + i, word = rank * p.slice + k;
        if (k >= p.slice) break;
        uint32_t v = 0;
        if (word < p.words)
            for (int c = 0; c < kCtas; ++c) v |= cluster.map_shared_rank(bits, c)[word];
        fin[k] = v;
        sum += __popc(v);
    }
    int total;
    int x = block_scan(sum, warp_sums, total);
    for (int i = 0; i < each; ++i) {
        const int k = tid * each + i;
        if (k >= p.slice) break;
        before[k] = x;
        x += __popc(fin[k]);
    }
    if (tid < kCtas) cluster.map_shared_rank(slice_live, tid)[rank] = total;
    __syncthreads();
    cluster.barrier_arrive();
    // ---- meanwhile, entries that depend on no rank (all marks have been taken)
    if (OP != COMPACT)
        for (int r = at / p.row_threads; r < p.n_rows; r += per) {
            const Row w = row_of(r);
            for (int j = w.hi + at % p.row_threads; j < p.max_blocks; j += p.row_threads) p.table_out[(size_t)r * p.stride + j] = ISV_BLOCK_NONE;
            if (OP == FORK && at % p.row_threads == 0) {
                const int from = parent_of(r);
                p.lens_out[r] = from < 0 ? 0 : p.lens[from];
                if (w.hi == w.lo) p.src[r] = p.dst[r] = ISV_BLOCK_NONE;
            }
        }
    cluster.barrier_wait();
    int base = 0, live = 0;                // live pages before this slice, and in all
    for (int c = 0; c < kCtas; ++c) {
        if (c < rank) base += slice_live[c];
        live += slice_live[c];
    }
    const int first_id = rank * p.slice * 32;
    const int ids = max(0, min(p.slice * 32, p.n_pages - first_id));

    if (OP != COMPACT) {
        // ---- free pages to the entries that need them
        const int free_pages = p.n_pages - live;
        for (int i = tid; i < ids; i += kThreads) {
            const int k = i >> 5, id = first_id + i;
            const int r = id - (base + before[k] + __popc(fin[k] & ((1u << (i & 31)) - 1u)));   // rank among the free pages
            if ((fin[k] >> (i & 31)) & 1u) continue;
            if (r >= wanted) break;        // ranks only grow
            int lo = 0, hi = p.n_rows;     // the last row with need[row] <= r and room for it
            while (hi - lo > 1) {
                const int m = (lo + hi) / 2;
                if (need[m] <= r) lo = m; else hi = m;
            }
            const Row w = row_of(lo);
            p.table_out[(size_t)lo * p.stride + w.lo + (r - need[lo])] = id;
            if (OP == FORK) {
                p.src[lo] = p.table[(size_t)p.other[lo] * p.stride + w.lo];
                p.dst[lo] = id;
            }
        }
        // ---- too few: the last entries in order stay without a page
        if (wanted > free_pages) {
            bad |= ISV_STATUS_NO_PAGES;
            for (int r = at / p.row_threads; r < p.n_rows; r += per) {
                const Row w = row_of(r);
                const int lacking = w.lo + max(0, free_pages - need[r]);    // first block of the row without a page
                for (int j = lacking + at % p.row_threads; j < w.hi; j += p.row_threads) p.table_out[(size_t)r * p.stride + j] = ISV_BLOCK_NONE;
                if (OP == FORK && at % p.row_threads == 0 && w.hi > w.lo && lacking <= w.lo) p.src[r] = p.dst[r] = ISV_BLOCK_NONE;
            }
        }
    } else {
        auto live_before = [&](int id) {   // over the whole pool
            const int c = (id >> 5) / p.slice, k = (id >> 5) % p.slice;
            int n = 0;
            for (int i = 0; i < c; ++i) n += slice_live[i];
            if (c < kCtas)
                n += cluster.map_shared_rank(before, c)[k] + __popc(cluster.map_shared_rank(fin, c)[k] & ((1u << (id & 31)) - 1u));
            return n;
        };
        const int below = live >= p.n_pages ? live : live_before(live);   // live pages that stay
        const int moves = live - below;
        for (int i = tid; i < ids; i += kThreads) {
            const int k = i >> 5, id = first_id + i;
            const int lb = base + before[k] + __popc(fin[k] & ((1u << (i & 31)) - 1u));
            const bool is_live = (fin[k] >> (i & 31)) & 1u;
            if (!is_live && id < live) p.dst[id - lb] = id;
            if (is_live && id >= live) p.src[lb - below] = id;
        }
        for (uint32_t i = moves + rank * kThreads + tid; i < (uint32_t)p.max_moves; i += kCtas * kThreads) p.src[i] = p.dst[i] = ISV_BLOCK_NONE;
        if (rank == 0 && tid == 0) { p.counts[0] = live; p.counts[1] = moves; }
        cluster.sync();                    // all moves are in place
        for (int r = at / p.row_threads; r < p.n_rows; r += per) {
            const int keep = row_of(r).hi;
            for (int j = at % p.row_threads; j < p.max_blocks; j += p.row_threads) {
                int id = ISV_BLOCK_NONE;
                if (j < keep) {
                    id = p.table[(size_t)r * p.stride + j];
                    if (id >= live && id < p.n_pages) id = __ldcg(&p.dst[live_before(id) - below]);
                }
                p.table_out[(size_t)r * p.stride + j] = id;
            }
        }
    }
    if (bad && p.status) atomicOr(p.status, bad);
    if (OP == COMPACT) cluster.sync();     // nobody leaves while its shared memory may be read
}

struct CopyParams {
    uint4 *dst;
    const uint4 *src;
    const int32_t *src_ids, *dst_ids, *n_dev;
    uint32_t *status;
    uint64_t dst_stride, src_stride;       // 16-byte units
    int32_t page;                          // 16-byte units of a page
    int32_t pieces;                        // of a page
    int32_t n, n_dst, n_src, layers;
};

// Each CTA takes pieces of pages: 16 KB, so that a thread has four loads in flight (128 KB an SM), and a few pages fill the
// machine.  Bound by HBM: 434 MB in 75 us on B200 (1656 pages of 64 KB in two layers, read and written), 5.8 TB/s.
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const __grid_constant__ CopyParams p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int n = p.n_dev ? min(p.n, max(0, *p.n_dev)) : p.n;
    const uint32_t items = (uint32_t)n * (uint32_t)p.pieces;               // the host checks that they, and a grid more, fit
    for (uint32_t layer = blockIdx.y; layer < (uint32_t)p.layers; layer += gridDim.y)   // unsigned: the last step may pass 2^31
        for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
            const int i = (int)(item / (uint32_t)p.pieces), piece = (int)(item - (uint32_t)i * (uint32_t)p.pieces);
            const int s = p.src_ids[i], d = p.dst_ids ? p.dst_ids[i] : i;
            if (s < 0 || s >= p.n_src || d < 0 || d >= p.n_dst) {
                if (s != ISV_BLOCK_NONE && d != ISV_BLOCK_NONE && threadIdx.x == 0 && p.status)
                    atomicOr(p.status, ISV_STATUS_BAD_BLOCK_ID);
                continue;
            }
            const uint4 *from = p.src + layer * p.src_stride + (size_t)s * p.page;
            uint4 *to = p.dst + layer * p.dst_stride + (size_t)d * p.page;
            uint4 v[kCopyUnroll];
            const int x = piece * kCopyThreads * kCopyUnroll + threadIdx.x;
#pragma unroll
            for (int k = 0; k < kCopyUnroll; ++k)
                if (x + k * kCopyThreads < p.page) v[k] = from[x + k * kCopyThreads];
#pragma unroll
            for (int k = 0; k < kCopyUnroll; ++k)
                if (x + k * kCopyThreads < p.page) to[x + k * kCopyThreads] = v[k];
        }
}

size_t table_smem(const TableParams &p, int op) {
    const size_t last = op == FORK ? p.n_in : op == RESIZE ? p.n_rows : 0;
    return 4ull * ((size_t)p.words + 2 * (size_t)p.slice + 2 * (size_t)p.n_rows + 1 + last);
}

template <int OP>
int launch_table(const char *who, TableParams &p, void *stream) {
    p.words = (p.n_pages + 31) / 32;
    p.slice = (p.words + kCtas - 1) / kCtas;
    int rows = 1;
    while (rows < p.n_rows) rows *= 2;
    p.row_threads = std::max(8, kCtas * kThreads / rows);
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return err(ISV_ECUDA, "%s: %s", who, cudaGetErrorString(e));
    static std::atomic<bool> ready[kMaxDevices];
    if (dev >= kMaxDevices || !ready[dev].load()) {
        TableParams most = p;
        most.words = ISV_PAGES_MAX / 32;
        most.slice = most.words / kCtas;
        most.n_rows = most.n_in = kMaxRows;
        e = cudaFuncSetAttribute(table_kernel<OP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)table_smem(most, OP));
        if (e != cudaSuccess) return err(ISV_ECUDA, "%s: %s", who, cudaGetErrorString(e));
        if (dev < kMaxDevices) ready[dev].store(true);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kCtas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = table_smem(p, OP);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;   // see the kernel's griddepcontrol pair
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kCtas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, table_kernel<OP>, p);
    return e == cudaSuccess ? ISV_OK : err(ISV_ECUDA, "%s: %s", who, cudaGetErrorString(e));
}

int check_table(const char *who, const void *table, const void *lens, int32_t n_rows, int32_t stride, int32_t max_blocks,
                int32_t open_in_pool, int32_t n_pages) {
    if (!table || !lens) return err(ISV_EINVAL, "%s: table and lengths are required", who);
    if (n_rows < 0 || n_rows > kMaxRows) return err(ISV_EINVAL, "%s: rows (%d) must be in [0, %d]", who, n_rows, kMaxRows);
    if (max_blocks < 1 || max_blocks >= (1 << 27) || stride < max_blocks)
        return err(ISV_EINVAL, "%s: bad table row (%d entries, stride %d)", who, max_blocks, stride);
    if (open_in_pool != 0 && open_in_pool != 1) return err(ISV_EINVAL, "%s: open_in_pool must be 0 or 1", who);
    if (n_pages < 1) return err(ISV_EINVAL, "%s: bad page count (%d)", who, n_pages);
    if (n_pages > ISV_PAGES_MAX) return err(ISV_ECAPACITY, "%s: at most %d pages (%d)", who, ISV_PAGES_MAX, n_pages);
    return ISV_OK;
}

// Two device ranges, in 32-bit words.
bool overlap(const void *a, size_t na, const void *b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && na && nb && x < y + 4 * nb && y < x + 4 * na;
}

}  // namespace

extern "C" {

int isv_pages_copy(void *dst_pool_dev, int32_t n_dst_pages, const void *src_pool_dev, int32_t n_src_pages,
                   uint64_t page_bytes, int32_t layers, uint64_t dst_layer_stride, uint64_t src_layer_stride,
                   const int32_t *src_ids_dev, const int32_t *dst_ids_dev, int32_t n, const int32_t *n_dev,
                   uint32_t *status_dev, void *stream) {
    if (!dst_pool_dev || !src_pool_dev || !src_ids_dev) return err(ISV_EINVAL, "isv_pages_copy: pools and source ids are required");
    if ((reinterpret_cast<uintptr_t>(dst_pool_dev) | reinterpret_cast<uintptr_t>(src_pool_dev) | page_bytes | dst_layer_stride |
         src_layer_stride) & 15u)
        return err(ISV_EINVAL, "isv_pages_copy: pools, page_bytes and layer strides must be multiples of 16 bytes");
    if (page_bytes == 0 || page_bytes >= (1ull << 34) || n_dst_pages < 1 || n_src_pages < 1 || layers < 1 || n < 0)
        return err(ISV_EINVAL, "isv_pages_copy: bad page size, page counts (%d, %d), layers (%d) or n (%d)", n_dst_pages,
                   n_src_pages, layers, n);
    if (layers > 1 && (dst_layer_stride < page_bytes * n_dst_pages || src_layer_stride < page_bytes * n_src_pages))
        return err(ISV_EINVAL, "isv_pages_copy: a layer stride is smaller than the layer's pages");
    if (n == 0) return ISV_OK;
    CopyParams p{};
    p.dst = static_cast<uint4 *>(dst_pool_dev); p.src = static_cast<const uint4 *>(src_pool_dev);
    p.src_ids = src_ids_dev; p.dst_ids = dst_ids_dev; p.n_dev = n_dev; p.status = status_dev;
    p.dst_stride = dst_layer_stride / 16; p.src_stride = src_layer_stride / 16; p.page = (int32_t)(page_bytes / 16);
    p.n = n; p.n_dst = n_dst_pages; p.n_src = n_src_pages; p.layers = layers;
    p.pieces = (p.page + kCopyThreads * kCopyUnroll - 1) / (kCopyThreads * kCopyUnroll);
    if ((unsigned long long)n * (unsigned)p.pieces >= (1ull << 32) - kCopyMaxGrid) return err(ISV_EINVAL, "isv_pages_copy: n * page_bytes too large");
    const unsigned items = (unsigned)n * (unsigned)p.pieces, rows = (unsigned)std::min(layers, 65535);
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return err(ISV_ECUDA, "isv_pages_copy: %s", cudaGetErrorString(e));
    const unsigned room = std::min(8u * (unsigned)sms, kCopyMaxGrid);   // about 8 CTAs an SM
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(std::max(1u, std::min(items, room / std::min(rows, room))), rows);
    cfg.blockDim = dim3(kCopyThreads);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;   // see the kernel's griddepcontrol pair
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, copy_kernel, p);
    return e == cudaSuccess ? ISV_OK : err(ISV_ECUDA, "isv_pages_copy: %s", cudaGetErrorString(e));
}

int isv_pages_fork(const int32_t *block_table_dev, const int32_t *lens_dev, int32_t n_rows, const int32_t *parent_dev,
                   int32_t *table_out_dev, int32_t *lens_out_dev, int32_t n_rows_out, int32_t table_stride,
                   int32_t max_blocks_per_seq, int32_t open_in_pool, int32_t n_pages, int32_t *copy_src_dev,
                   int32_t *copy_dst_dev, uint32_t *status_dev, void *stream) {
    int rc = check_table("isv_pages_fork", block_table_dev, lens_dev, n_rows, table_stride, max_blocks_per_seq, open_in_pool, n_pages);
    if (!rc && (!parent_dev || !table_out_dev || !lens_out_dev || !copy_src_dev || !copy_dst_dev))
        rc = err(ISV_EINVAL, "isv_pages_fork: parents, outputs and copy lists are required");
    if (!rc && (n_rows_out < 0 || n_rows_out > kMaxRows))
        rc = err(ISV_EINVAL, "isv_pages_fork: rows (%d) must be in [0, %d]", n_rows_out, kMaxRows);
    if (rc) return rc;
    const void *at[8] = {block_table_dev, lens_dev, parent_dev, table_out_dev, lens_out_dev, copy_src_dev, copy_dst_dev, status_dev};
    const size_t in = (size_t)n_rows, o = (size_t)n_rows_out, st = (size_t)table_stride;
    const size_t size[8] = {in * st, in, o, o * st, o, o, o, 1};
    for (int i = 0; i < 8; ++i)
        for (int j = std::max(i + 1, 3); j < 8; ++j)   // an output with anything
            if (overlap(at[i], size[i], at[j], size[j])) return err(ISV_EINVAL, "isv_pages_fork: the arrays must not overlap");
    if (n_rows_out == 0) return ISV_OK;
    TableParams p{};
    p.table = block_table_dev; p.lens = lens_dev; p.other = parent_dev;
    p.table_out = table_out_dev; p.lens_out = lens_out_dev; p.src = copy_src_dev; p.dst = copy_dst_dev; p.status = status_dev;
    p.n_rows = n_rows_out; p.n_in = n_rows; p.stride = table_stride; p.max_blocks = max_blocks_per_seq;
    p.open_in_pool = open_in_pool; p.n_pages = n_pages;
    return launch_table<FORK>("isv_pages_fork", p, stream);
}

int isv_pages_resize(int32_t *block_table_dev, const int32_t *lens_dev, const int32_t *new_lens_dev, int32_t n_rows,
                     int32_t table_stride, int32_t max_blocks_per_seq, int32_t open_in_pool, int32_t n_pages,
                     uint32_t *status_dev, void *stream) {
    int rc = check_table("isv_pages_resize", block_table_dev, lens_dev, n_rows, table_stride, max_blocks_per_seq, open_in_pool, n_pages);
    if (!rc && !new_lens_dev) rc = err(ISV_EINVAL, "isv_pages_resize: new lengths are required");
    if (rc) return rc;
    if (overlap(block_table_dev, (size_t)n_rows * table_stride, lens_dev, n_rows) ||
        overlap(block_table_dev, (size_t)n_rows * table_stride, new_lens_dev, n_rows))
        return err(ISV_EINVAL, "isv_pages_resize: the arrays must not overlap");
    if (n_rows == 0) return ISV_OK;
    TableParams p{};
    p.table = block_table_dev; p.table_out = block_table_dev; p.lens = lens_dev; p.other = new_lens_dev; p.status = status_dev;
    p.n_rows = p.n_in = n_rows; p.stride = table_stride; p.max_blocks = max_blocks_per_seq;
    p.open_in_pool = open_in_pool; p.n_pages = n_pages;
    return launch_table<RESIZE>("isv_pages_resize", p, stream);
}

int isv_pages_compact(const int32_t *block_table_dev, const int32_t *lens_dev, int32_t n_rows, int32_t table_stride,
                      int32_t max_blocks_per_seq, int32_t open_in_pool, int32_t n_pages, int32_t *table_out_dev,
                      int32_t *src_ids_dev, int32_t *dst_ids_dev, int32_t max_moves, int32_t *counts_dev,
                      uint32_t *status_dev, void *stream) {
    int rc = check_table("isv_pages_compact", block_table_dev, lens_dev, n_rows, table_stride, max_blocks_per_seq, open_in_pool, n_pages);
    if (!rc && (!table_out_dev || !src_ids_dev || !dst_ids_dev || !counts_dev))
        rc = err(ISV_EINVAL, "isv_pages_compact: outputs are required");
    if (!rc && max_moves < n_pages / 2)
        rc = err(ISV_EINVAL, "isv_pages_compact: max_moves (%d) must be at least n_pages / 2 (%d)", max_moves, n_pages / 2);
    if (rc) return rc;
    const void *at[7] = {block_table_dev, lens_dev, table_out_dev, src_ids_dev, dst_ids_dev, counts_dev, status_dev};
    const size_t in = (size_t)n_rows, st = (size_t)table_stride, m = (size_t)max_moves;
    const size_t size[7] = {in * st, in, in * st, m, m, 2, 1};
    for (int i = 0; i < 7; ++i)
        for (int j = std::max(i + 1, 2); j < 7; ++j)
            if (!(i == 0 && j == 2 && at[0] == at[2]) && overlap(at[i], size[i], at[j], size[j]))
                return err(ISV_EINVAL, "isv_pages_compact: the arrays must not overlap (table_out may be the table itself)");
    TableParams p{};
    p.table = block_table_dev; p.table_out = table_out_dev; p.lens = lens_dev; p.src = src_ids_dev; p.dst = dst_ids_dev;
    p.counts = counts_dev; p.status = status_dev; p.max_moves = max_moves;
    p.n_rows = p.n_in = n_rows; p.stride = table_stride; p.max_blocks = max_blocks_per_seq;
    p.open_in_pool = open_in_pool; p.n_pages = n_pages;
    return launch_table<COMPACT>("isv_pages_compact", p, stream);
}

}  // extern "C"
