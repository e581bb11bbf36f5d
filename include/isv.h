/*
 * isv.h - decode attention over a paged KV cache that is split between GPU HBM
 * and pinned host memory (KV cache offloading), for NVIDIA B200 (sm_100a).
 *
 * The library executes the computation whose time the InferSave cost model
 * predicts per layer and decode step (paper Section IV-C, Eq. 6):
 *     T_dec = CTCF(T_compute^d) + T_trans^d
 * i.e. the self-attention part of T_compute^d (4 * BS * ctx * h1 flops) over a
 * KV cache of which the fraction C_off (Section IV-B) lives in CPU memory and
 * must cross the host link (T_trans^d) every step.
 *
 * Conventions
 *   - All entry points return 0 (ISV_OK) or a negative ISV_E* code; the text of
 *     the last error of the calling thread is available from isv_last_error().
 *     Nothing aborts, throws across the boundary or traps on the device.
 *   - "device" pointers are CUDA device addresses on the GPU that was current
 *     when the handle was created; "host" pointers are ordinary CPU addresses.
 *   - Work is enqueued on the handle's compute stream (and on internal copy
 *     streams) and is asynchronous unless a function says it synchronises.
 *     Caller-owned buffers must stay valid until that work has completed.
 *   - K/V/q/out elements are 16-bit (fp16 or bf16, chosen at allocation);
 *     arithmetic is fp32.
 *   - KV pool layout, per physical layer and pool (HBM pool, host pool):
 *         [block][K|V][kv_head][block_tokens][head_dim]
 *     so one (block, K-or-V, head) tile is contiguous.  Inside a tile the row
 *     of token t (head_dim elements) is stored as 16-byte chunks, and chunk c
 *     sits at chunk position c XOR (t mod 8) of that row (head_dim 80: chunks
 *     0..7 only; chunks 8 and 9 stay in place): the arrangement
 *     that lets the tensor-core path load eight tokens at once without
 *     shared-memory bank conflicts.  isv_kv_fill / isv_kv_append / isv_kv_gather
 *     apply it; only a caller that builds a pool itself
 *     (isv_attn_decode_static) has to.
 *   - Block table entry (int32): ISV_BLOCK_NONE = not allocated; otherwise the
 *     physical block id, with ISV_BLOCK_HOST_BIT set when the block belongs to
 *     the host pool.  The block that holds a sequence's newest token is kept in
 *     GPU memory even when it is host-flagged (it is still being written); it
 *     is copied to the host pool when it becomes full.
 */
#ifndef ISV_H
#define ISV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define ISV_OK               0
#define ISV_EINVAL          (-1)   /* bad argument                                   */
#define ISV_ENOMEM_DEVICE   (-2)   /* cudaMalloc refused                             */
#define ISV_ENOMEM_PINNED   (-3)   /* pinned host allocation refused (by the system, or because it  */
                                   /* exceeds the environment variable ISV_PINNED_LIMIT_BYTES)      */
#define ISV_ECAPACITY       (-4)   /* sequence or pool would exceed its capacity     */
#define ISV_ECUDA           (-5)   /* a CUDA runtime call failed                     */
#define ISV_ETIMEOUT        (-6)   /* a host-side wait exceeded isv_set_host_timeout */
#define ISV_EDEVICE_STATUS  (-7)   /* a kernel reported a problem (see status bits)  */
#define ISV_ENODEVICE       (-8)   /* compute requested on a plan-only handle        */

#define ISV_F16   0
#define ISV_BF16  1
#define ISV_F32   2    /* isv_draft_verify only */

#define ISV_BLOCK_NONE      (-1)
#define ISV_BLOCK_HOST_BIT  (1 << 30)

/* bits of the device status word (isv_step_times.status, isv_sync, isv_linear_status) */
#define ISV_STATUS_BAD_BLOCK_ID  1u   /* a table entry pointed outside its pool; block skipped */
#define ISV_STATUS_WAIT_EXPIRED  2u   /* a bounded wait inside a kernel gave up                */
#define ISV_STATUS_BAD_LENGTH    4u   /* a device-side sequence length was negative or exceeded */
                                      /* the table row; it was clamped to what the row covers  */
#define ISV_STATUS_NO_PAGES      8u   /* isv_pages_*: fewer free pages than were needed        */
#define ISV_STATUS_BAD_TOKEN     16u  /* isv_draft_verify: a drafted token outside the vocabulary, or no probability */

typedef struct isv_kv isv_kv;   /* opaque; created by isv_kv_alloc, destroyed by isv_kv_free */

/*
 * Problem statement of one cache (paper Table II: model shape, batch size,
 * input/output lengths, precision; Section IV-B: offload ratio).
 */
typedef struct {
    int32_t  layers;             /* logical layers (n)                                          */
    int32_t  phys_layers;        /* physical KV slabs; 0 = layers.  Logical layer l uses slab   */
                                 /* l % phys_layers (lets a benchmark hold fewer slabs than     */
                                 /* layers; layers sharing a slab overwrite each other's data)  */
    int32_t  q_heads;            /* query heads; multiple of kv_heads                           */
    int32_t  kv_heads;
    int32_t  head_dim;           /* 64, 80 (OPT-2.7B, the paper's main model: h1 2560 / 32) or 128 */
    int32_t  block_tokens;       /* tokens per KV block; 16                                     */
    int32_t  dtype;              /* ISV_F16 or ISV_BF16                                         */
    float    offload_frac;       /* C_off in [0, 1]: of every prefix of j blocks of a sequence, */
                                 /* floor(j * C_off) are host-resident                          */
    int32_t  max_seqs;           /* capacity in sequences (BS), <= 4096                         */
    int32_t  max_tokens_per_seq; /* capacity per sequence (L_in + L_out)                        */
    uint64_t perm_seed;          /* 0 = physical block ids handed out in order; otherwise they  */
                                 /* follow a seeded permutation (host pool ids stay compact)    */
    uint64_t chunk_bytes;        /* staging chunk size; 0 = 128 MiB or a layer's host pool if smaller */
    int32_t  ring_depth;         /* staging ring buffers; 0 = 3                                 */
    int32_t  max_ctas;           /* cap on the resident kernel's grid; 0 = one CTA per SM.      */
                                 /* The KV blocks are cut evenly over the grid's warps, so this */
                                 /* also sets into how many splits a sequence falls             */
    int32_t  plan_only;          /* 1 = host bookkeeping only: no CUDA call is made, no memory  */
                                 /* is allocated, compute entry points return ISV_ENODEVICE     */
    void    *compute_stream;     /* cudaStream_t to enqueue on, or NULL = library creates one   */
                                 /* (the legacy default stream, handle 0, cannot be passed)     */
} isv_kv_desc;

/* Sizes the library derived from a description (filled by isv_kv_info). */
typedef struct {
    uint64_t block_bytes;        /* one block: 2 * kv_heads * block_tokens * head_dim * 2 B     */
    uint64_t kv_bytes_per_token; /* K and V of one token in one layer                           */
    int32_t  max_blocks_per_seq;
    int32_t  hbm_blocks;         /* HBM pool capacity per physical layer, in blocks             */
    int32_t  host_blocks;        /* host pool capacity per physical layer, in blocks            */
    int32_t  hbm_blocks_used;
    int32_t  host_blocks_used;
    uint64_t hbm_pool_bytes;     /* all physical layers, tail slots included                    */
    uint64_t host_pool_bytes;    /* all physical layers                                         */
    uint64_t scratch_bytes;      /* split partials, running state, staging ring                 */
    int32_t  phys_layers;
    int32_t  max_ctas;
    int32_t  ring_depth;
    int32_t  sm_count;
    uint64_t chunk_bytes;
    uint64_t kernel_launches;    /* kernels this handle has launched since it was created       */
} isv_kv_info_t;

/*
 * Per-layer timing of the most recent decode of that layer, and what the
 * paper's terms are for it: h2d_ms is T_trans^d, attn_resident_ms +
 * attn_offloaded_ms + merge_ms is the self-attention part of T_compute^d,
 * total_ms is T_dec without the linear layers.  Byte counters: bytes_resident
 * and bytes_offloaded are the KV bytes the attention had to read from HBM and
 * to fetch over the host link; bytes_offloaded equals the first term of the
 * T_trans^d numerator, C_off * 2 * L * h1 * Precision * BS, counted per block.
 * bytes_staged is what the copy engine actually moved (whole chunks).
 */
typedef struct {
    float    append_ms;           /* 0 when the append was fused into the attention kernel */
    float    h2d_ms;
    float    attn_resident_ms;
    float    attn_offloaded_ms;
    float    merge_ms;
    float    total_ms;
    uint64_t bytes_resident;
    uint64_t bytes_offloaded;
    uint64_t bytes_staged;
    uint64_t bytes_appended;
    int32_t  n_chunks;
    uint32_t status;
} isv_step_times;

/* ---- lifetime ---------------------------------------------------------- */

/* Allocates pools (HBM, pinned host), block tables, scratch, staging ring,
 * streams and events on the current device.  Synchronous.  *out is NULL on
 * failure.  The handle must be used from one host thread at a time. */
int isv_kv_alloc(isv_kv **out, const isv_kv_desc *desc);

/* Waits for all work of the handle, then frees everything it owns. */
int isv_kv_free(isv_kv *h);

/* Forgets all sequences (lengths 0, all blocks free).  Synchronises. */
int isv_kv_reset(isv_kv *h);

int isv_kv_info(isv_kv *h, isv_kv_info_t *out);

/* ---- loading and appending (the KV cache of Section II-A) --------------- */

/* Prompt load for one layer (prefill's KV, not timed): k, v are device arrays
 * [n_seqs][T][kv_heads][head_dim]; lens_host[s] <= T tokens of sequence s are
 * kept and replace what the layer held for s.  Blocks are allocated by the
 * residency rule on first use and shared by all layers.  Synchronises. */
int isv_kv_fill(isv_kv *h, int32_t layer, const void *k_dev, const void *v_dev,
                const int32_t *lens_host, int32_t n_seqs, int32_t T);

/* The same load without the final wait: returns once the work is enqueued (k_dev and v_dev must stay valid
 * until isv_sync or isv_fill_timing).  Resident blocks are written by a kernel; the complete host-resident
 * blocks - the share C_off of the prompt's KV that the paper's prefill stage stores to CPU memory,
 * T_trans^p = C_off * 2 * (L_in + 1) * h1 * Precision * BS / BW_gpu->cpu (Section IV-C) - are packed into
 * the staging ring in host-block order and stored by device-to-host copies on the write-back stream, so
 * that the store overlaps whatever the caller computes next (the paper's Eq. 5 takes the max of both). */
int isv_kv_fill_async(isv_kv *h, int32_t layer, const void *k_dev, const void *v_dev,
                      const int32_t *lens_host, int32_t n_seqs, int32_t T);

/* Timing of the latest isv_kv_fill / isv_kv_fill_async: store_ms is the measured T_trans^p of that layer
 * (first to last device-to-host copy), bytes_stored its numerator counted per block.  Synchronises. */
typedef struct {
    float    pack_ms;          /* kernels: resident blocks, tails, packing of host blocks */
    float    store_ms;         /* device-to-host copies, first start to last end          */
    float    total_ms;         /* start of the load to the end of its last copy           */
    uint64_t bytes_stored;     /* KV bytes written to the host pool                       */
    uint64_t bytes_resident;   /* KV bytes written to GPU memory                          */
    int32_t  n_copies;
} isv_fill_times;
int isv_fill_timing(isv_kv *h, isv_fill_times *out);

/* Appends one token to sequences 0..n_seqs-1 of one layer at that layer's
 * current lengths (the cache growth of one decode step): k, v are device
 * arrays [n_seqs][kv_heads][head_dim].  K and V are written by one kernel; the
 * copy is bit-exact.  ISV_ECAPACITY if a sequence is full. */
int isv_kv_append(isv_kv *h, int32_t layer, const void *k_dev, const void *v_dev,
                  int32_t n_seqs);

/* ---- decode attention (self-attention term of T_compute^d; T_trans^d) ---- */

/* out[s][h][:] = softmax(q[s][h] . K_s^T / sqrt(head_dim)) V_s over the
 * layer's current tokens of sequence s (the newest token included), for
 * s < n_seqs.  q_dev: [n_seqs][q_heads][head_dim] 16-bit; out_dev (same shape
 * and dtype) and out_f32_dev (fp32) may each be NULL but not both.  Query head
 * h reads KV head h / (q_heads / kv_heads).  A sequence of length 0 yields
 * zeros.  Host-resident blocks are streamed through the staging ring on the
 * copy stream while the resident blocks are processed; partial results are
 * combined by a log-sum-exp merge.
 * block_table_dev / seq_lens_dev: NULL = the library's own (normal use).  If
 * given, they replace the library's device arrays for the resident kernel
 * (same format, row stride as isv_block_table_dev reports) and must agree with
 * the library's bookkeeping on lengths and on host-resident entries. */
int isv_attn_decode(isv_kv *h, int32_t layer, const void *q_dev, void *out_dev,
                    float *out_f32_dev, const int32_t *block_table_dev,
                    const int32_t *seq_lens_dev, int32_t n_seqs);

/* isv_kv_append followed by isv_attn_decode for one layer, as one kernel: the
 * resident attention kernel also stores the new token's K/V rows and advances
 * the lengths, and attends to the new token straight from k_dev / v_dev, so
 * the step needs one launch per layer instead of two.  Same arguments and
 * result as the two calls (up to fp32 summation order). */
int isv_decode_layer(isv_kv *h, int32_t layer, const void *q_dev, const void *k_dev, const void *v_dev,
                     void *out_dev, float *out_f32_dev, int32_t n_seqs);

/* Second design point for the offloaded part: with on = 1 the host-resident blocks are not staged
 * through the ring by the copy engine; the attention kernel's bulk copies read them in place from the
 * mapped pinned pool, over the host link.  No HBM staging traffic and no copy-engine work, but the link
 * is driven by SM-issued reads.  Results are the same; isv_step_timing then reports h2d_ms = 0 and the
 * link time inside attn_offloaded_ms.  Off by default. */
int isv_set_zero_copy(isv_kv *h, int32_t on);

/* One decode step of all layers: the result of isv_decode_layer for l in 0..layers-1.
 * Device arrays: q, out (16-bit) and out_f32 (fp32) [layers][n_seqs][q_heads][head_dim];
 * k, v [layers][n_seqs][kv_heads][head_dim].  out_dev and out_f32_dev may each be NULL, not both.
 * Because all layers' inputs are handed over at once, the resident attention (and the appends) of up to
 * phys_layers consecutive layers run as ONE launch whose work list spans those layers: the start-up and
 * the tail of a launch are then paid once per step instead of once per layer, which matters when a
 * layer's KV is read in under 100 microseconds.  With offloaded blocks each layer's staged launches and
 * merge follow that launch, and the copy engine's queue is filled for all of them at once.  (Layers that
 * share a physical slab are never put into one launch.  With offload_frac = 0 and per-layer timing on it
 * is one launch per layer.)  A caller whose layers depend on one another (a real model) uses
 * isv_decode_layer per layer. */
int isv_decode_step(isv_kv *h, const void *q_dev, const void *k_dev, const void *v_dev,
                    void *out_dev, float *out_f32_dev, int32_t n_seqs);

/* The same step with HOST buffers of the same shapes (pinned memory gives
 * asynchronous copies): inputs are copied to library-owned device buffers a
 * few layers at a time on a copy stream while earlier layers compute, and
 * each group's result is copied back as soon as it is ready.  Returns after
 * the whole result is in out_host (synchronises).  The first call on a handle
 * allocates the device buffers for one step's q, k, v and out (cudaMalloc,
 * counted in isv_kv_info's scratch_bytes) and a copy stream; make it outside
 * any region that must not allocate. */
int isv_decode_step_host(isv_kv *h, const void *q_host, const void *k_host,
                         const void *v_host, void *out_host, int32_t n_seqs);

/* ---- inspection --------------------------------------------------------- */

/* Logical-order copy of one sequence's K and V of one layer to host arrays
 * [len][kv_heads][head_dim] (capacity max_tokens_per_seq rows each).
 * Bit-exact; synchronises. */
int isv_kv_gather(isv_kv *h, int32_t layer, int32_t seq, void *k_host, void *v_host,
                  int32_t *len_out);

/* Library-maintained device arrays: table [max_seqs][*row_stride] int32 and
 * one layer's lengths [max_seqs] int32.  NULL on a plan-only handle. */
const int32_t *isv_block_table_dev(isv_kv *h, int32_t *row_stride);
const int32_t *isv_seq_lens_dev(isv_kv *h, int32_t layer);

/* Host copies of the same (work on plan-only handles too). */
int isv_block_table_host(isv_kv *h, int32_t *out, int32_t n_seqs, int32_t row_stride);
int isv_seq_lens_host(isv_kv *h, int32_t layer, int32_t *out, int32_t n_seqs);

/* KV bytes a decode of this layer over n_seqs sequences would read now:
 * resident (HBM) and offloaded (host link) algorithmic bytes, the bytes the
 * staging engine would copy, and its chunk count.  Any pointer may be NULL. */
int isv_plan_bytes(isv_kv *h, int32_t layer, int32_t n_seqs, uint64_t *bytes_resident,
                   uint64_t *bytes_offloaded, uint64_t *bytes_staged, int32_t *n_chunks);

/* ---- timing (feeds the terms of Eq. 6) ----------------------------------- */

/* Turns event recording per layer on or off (off by default: events cost a
 * little on short steps). */
int isv_set_timing(isv_kv *h, int32_t on);

/* Times of the latest decode of `layer`, or with layer = -1 the sums over all
 * layers (total_ms then spans first layer start to last layer end).
 * Synchronises.  Times are 0 where timing was off. */
int isv_step_timing(isv_kv *h, int32_t layer, isv_step_times *out);

/* Waits for everything enqueued by the handle; returns ISV_EDEVICE_STATUS if
 * a kernel flagged a problem since the last call (bits in *status_out). */
int isv_sync(isv_kv *h, uint32_t *status_out);

/* ---- failure handling ----------------------------------------------------- */

/* (The paper treats only predicted out-of-memory, Algorithm 1's "Unsuitable" case, which isv_kv_alloc's
 * ISV_ENOMEM_* codes mirror; it has no counterpart for what follows.  These calls keep a lost transfer or
 * a stuck stream from turning into a hang: every wait of the library, on the device and on the host, can
 * be given a limit, and running into it is reported as a status or an error code with the handle intact.) */

/* Limit, in seconds, of every host-side wait of this handle (isv_sync, isv_step_timing, isv_kv_fill,
 * isv_fill_timing, isv_kv_gather, isv_decode_step_host): a wait that exceeds it returns ISV_ETIMEOUT
 * and leaves the work enqueued, so the caller can wait again, report, or tear down.  0 (the default)
 * waits without limit.  The wait polls the stream instead of blocking in the driver. */
int isv_set_host_timeout(isv_kv *h, double seconds);

/* Limit of a device-side wait for a K/V copy, in polls of its barrier (0 = the built-in default, about
 * 4 million polls, i.e. seconds).  A warp whose wait runs out sets ISV_STATUS_WAIT_EXPIRED, gives its
 * other copies one more bounded chance to land and leaves the kernel; the handle stays usable and the
 * next isv_sync / isv_step_timing returns ISV_EDEVICE_STATUS once and clears the state.  The outputs of
 * that launch are incomplete. */
int isv_set_wait_limit(isv_kv *h, uint32_t polls);

/* Failure injection for tests of the path above: in each of the next `launches` resident attention
 * launches one warp arms the barrier of its first K tile without issuing the copy, as if the transfer
 * had been lost; its wait then runs out after the limit set by isv_set_wait_limit.  Nothing faults
 * and nothing hangs. */
int isv_inject_lost_copy(isv_kv *h, int32_t launches);

/* Measures pinned host<->device copy bandwidth on the current device: `bytes`
 * per copy, best of `reps`, CUDA events.  This is the measured host-link rate
 * that T_trans^d's BW_cpu->gpu stands for.  Allocates and frees its buffers. */
int isv_link_probe(uint64_t bytes, int32_t reps, double *h2d_gbs, double *d2h_gbs);

/* ---- decode linear layers (linear-layer term of T_compute^d) -------------- */

/* y = x . w^T for a batch of M <= max_M <= 256 tokens: the QKV / output / MLP projections whose
 * flops the paper counts as BS * (8 h1^2 + 4 h1 h2) per layer (Section IV-C, T_compute^d).  At
 * decode batch sizes the product is bound by reading w once from HBM; it runs on the tensor cores
 * (tcgen05, fp32 accumulation in tensor memory) so that the arithmetic keeps up with that read.
 *   w_dev  [N][K] 16-bit row-major (the usual weight layout), N and K multiples of 128;
 *          must stay valid and unchanged while the handle lives
 *   x_dev  [M][K] 16-bit;  y_dev [M][N] 16-bit and / or y_f32_dev [M][N] fp32 (one may be NULL)
 * isv_linear_create allocates split-K scratch and encodes the weight's tensor map (synchronous);
 * isv_linear_forward enqueues the streaming kernel and, where tiles of the output are shared by
 * several CTAs, a small kernel that adds their partial sums, on `stream` (asynchronous, no host
 * wait); isv_linear_status waits for the stream and returns ISV_EDEVICE_STATUS if a bounded wait
 * inside the kernel expired. */
typedef struct isv_linear isv_linear;
int isv_linear_create(isv_linear **out, const void *w_dev, int32_t N, int32_t K, int32_t dtype,
                      int32_t max_M, void *stream);
int isv_linear_forward(isv_linear *l, const void *x_dev, void *y_dev, float *y_f32_dev, int32_t M);
int isv_linear_status(isv_linear *l, uint32_t *status_out);
int isv_linear_free(isv_linear *l);

/* ---- decode attention for callers that cannot allocate ------------------- */

/* Size of the fixed device array that holds this entry point's scratch.  Every
 * GPU on which the library is loaded keeps this much memory until the process
 * exits, whether or not the entry point is ever called. */
#define ISV_STATIC_SCRATCH_BYTES (8u << 20)

/* (The paper has no counterpart for this call: it is a packaging variant of
 * isv_attn_decode's resident kernel, added for deployment reasons.)
 *
 * Some callers may not call cudaMalloc: a serving process that has handed all
 * of its GPU memory to a framework's caching allocator, a latency-critical
 * loop in which an allocation would stall the device, a plugin that is given
 * pointers and a stream and nothing else.  This call is for them.  It makes no
 * cudaMalloc / cudaFree / cudaHostAlloc and uses no allocating library call;
 * it needs no handle.  The caller owns and passes every buffer:
 *   kv_pool_dev      KV pool in the library's layout,
 *                    [n_pool_blocks][K|V][kv_heads][block_tokens][head_dim], 16-bit,
 *                    with the 16-byte chunks of each token row permuted as
 *                    described under "KV pool layout" above
 *   block_table_dev  int32 [n_seqs][table_stride]: pool block ids in logical
 *                    order (ISV_BLOCK_NONE or host-flagged entries are skipped;
 *                    ids outside the pool are skipped and flagged)
 *   seq_lens_dev     int32 [n_seqs]: tokens to attend; at most
 *                    max_blocks_per_seq * block_tokens each (the table rows must
 *                    cover them)
 *   q_dev            [n_seqs][q_heads][head_dim] 16-bit
 *   out_dev / out_f32_dev   same shape, 16-bit / fp32; either may be NULL, not both
 *   status_dev       optional uint32 the kernel ORs ISV_STATUS_* bits into
 *                    (the caller clears it); NULL = not reported
 *   stream           cudaStream_t the work is enqueued on (asynchronous)
 * max_ctas: cap on the kernel's grid, 0 = one CTA per SM.
 * The split kernel's partial results and arrival counters live in one fixed
 * device array of ISV_STATIC_SCRATCH_BYTES:
 *   n_seqs * (q_heads / heads per warp) * 4 B of counters
 *   + 2 * warps in the grid * heads per warp * (head_dim + 2) * 4 B of partials.
 * When the partials of a full grid do not fit, the grid is cut down to the
 * CTAs whose partials do (the kernel divides the work among the CTAs it
 * gets).  A shape that leaves no room for a single CTA is refused with
 * ISV_ECAPACITY and a message; nothing runs then.
 * All calls on a GPU share that array and it keeps the previous call's
 * contents; each call zeroes the counters it needs on `stream` first.  Two
 * calls whose GPU work overlaps (different streams, or different threads
 * without ordering) race on it: order them on one stream or with events.
 * The first call on each device looks up the array's device address
 * (cudaGetSymbolAddress) and the device limits; make that first call with the
 * device current and before starting any stream capture. */
int isv_attn_decode_static(const void *kv_pool_dev, int32_t n_pool_blocks,
                           const int32_t *block_table_dev, int32_t table_stride,
                           const int32_t *seq_lens_dev, int32_t n_seqs, int32_t max_blocks_per_seq,
                           int32_t q_heads, int32_t kv_heads, int32_t head_dim, int32_t block_tokens,
                           int32_t dtype, int32_t max_ctas, const void *q_dev, void *out_dev,
                           float *out_f32_dev, uint32_t *status_dev, void *stream);

/* ---- a KV cache held in 8 bits -------------------------------------------- */

/* (The paper keeps K and V in the model's 16-bit precision; a cache in 8 bits halves both the memory term
 * and the bandwidth term of its decode model.  These calls stand beside isv_attn_decode_static: the caller
 * owns every buffer, nothing is offloaded.)
 *
 * A page holds one block of 16 tokens.  Every (page, KV head, K or V) has a scale of its own:
 *     ISV_Q8_INT8   scale = absmax / 127, code = x / scale rounded to the nearest integer
 *     ISV_Q8_E4M3   scale = absmax / 448, code = x / scale rounded to the nearest e4m3 value
 * absmax is taken over the block's 16 x head_dim values; scale is the fp32 rounding of the quotient and the
 * code is the rounding (ties to even) of the exact quotient x / scale.  A block of zeros has scale 0.  A
 * block with an infinity or a NaN has scale NaN, and so has every result that reads it.
 * Only complete blocks are quantised.  The open block of a sequence (its last n mod 16 tokens) stays in 16
 * bits in the sequence's tail slot until it is complete; it is then rounded once and its page never changes
 * again, so sequences may share complete pages.
 *
 * Page layout: [kv_head][16 * head_dim codes of K | 16 * head_dim codes of V | fp32 scale of K | fp32 scale
 * of V | 8 unused bytes].  The codes are stored in the order in which a warp's lanes feed them to the tensor
 * cores.  With D = head_dim and P = D / 32 (rounded down), byte b < 512 * P of a part belongs to
 *     lane = (b mod 512) / 16, g = lane / 4, c = lane mod 4, p = b / 512, i = (b mod 16) / 8,
 *     h = (b mod 8) / 4, j = b mod 4;
 * the last 256 bytes at head_dim 80 belong to lane = (b - 512 * P) / 8, p = P, i = 0 and the same h and j:
 *     K: token g + 8 * h,                           dim 32 * p + 8 * c + 4 * i + j  (32 * P + 4 * c + j in the last 256)
 *     V: token 2 * c + (j mod 2) + 8 * (j / 2),     dim g * (D / 8) + 2 * (2 * p + i) + h
 * Tail slots: [sequence][K|V][kv_head][16][head_dim] 16-bit, rows in order; rows from n mod 16 on are never
 * read. */
#define ISV_Q8_INT8  0
#define ISV_Q8_E4M3  1

typedef struct {
    int32_t q_heads;             /* query heads; multiple of kv_heads                           */
    int32_t kv_heads;
    int32_t head_dim;            /* 64, 80 or 128                                               */
    int32_t dtype;               /* ISV_F16 or ISV_BF16: q, k, v, tails and the 16-bit output   */
    int32_t format;              /* ISV_Q8_INT8 or ISV_Q8_E4M3                                  */
    int32_t max_seqs;            /* sequences per call, <= 4096                                 */
    int32_t max_ctas;            /* cap on the attention kernel's grid; 0 = one CTA per SM      */
} isv_q8_desc;

typedef struct isv_q8 isv_q8;

/* Bytes of one page and of one sequence's tail slot.  Needs no GPU. */
int isv_q8_sizes(int32_t kv_heads, int32_t head_dim, uint64_t *page_bytes, uint64_t *tail_bytes);

/* Allocates the attention's scratch and a status word on the current device (synchronous).  The handle
 * holds no cache: any number of layers and pools may be used with it.  Calls on one handle share its
 * scratch: order them on one stream or with events (one handle per stream or captured graph that may
 * overlap another).  Calls run on the handle's device, whichever is current. */
int isv_q8_create(isv_q8 **out, const isv_q8_desc *desc);
int isv_q8_free(isv_q8 *h);

/* Stores new tokens of one layer: a prompt, a chunk of one, or one token per sequence.  Sequence s has
 * seq_lens_dev[s] tokens after the call; its last new_lens_dev[s] <= T of them are rows 0 .. of
 *     k_dev, v_dev + s * seq_stride + t * token_stride, each [kv_heads][head_dim] 16-bit
 * (strides in elements, multiples of 8).  new_lens_dev NULL = T new tokens for every sequence.  Blocks that
 * are complete afterwards are quantised into the page that block_table_dev ([n_seqs][table_stride],
 * max_blocks_per_seq <= table_stride entries of a row are used, at most 2^27 - 2) names; the rest goes to the tail slot
 * tails_dev[s].  A sequence with no new token keeps everything.  Page ids outside [0, n_pages) are skipped
 * and flagged (ISV_STATUS_BAD_BLOCK_ID), also ISV_BLOCK_NONE; lengths are clamped to what the table row
 * and the tail slot hold, 16 * max_blocks_per_seq + 15, and new lengths to [0, min(T, length)], and flagged
 * (ISV_STATUS_BAD_LENGTH).  Asynchronous on `stream`; may be captured into a CUDA graph. */
int isv_q8_write(isv_q8 *h, void *pool_dev, int32_t n_pages, void *tails_dev, const int32_t *block_table_dev,
                 int32_t table_stride, int32_t max_blocks_per_seq, const int32_t *seq_lens_dev,
                 const int32_t *new_lens_dev, const void *k_dev, const void *v_dev, int64_t seq_stride,
                 int64_t token_stride, int32_t n_seqs, int32_t T, void *stream);

/* out[s][h][:] = softmax(q[s][h] . K_s^T / sqrt(head_dim)) V_s over the seq_lens_dev[s] tokens of sequence s,
 * as isv_attn_decode: complete blocks from their pages, the open block from its tail slot.  A sequence of
 * length 0 yields zeros.  q_dev [n_seqs][q_heads][head_dim] 16-bit; out_dev (16-bit) and out_f32_dev (fp32),
 * same shape, may each be NULL, not both.  A block without a page (ISV_BLOCK_NONE) is left out and not
 * flagged; other ids outside [0, n_pages) are left out and flagged.  fp32 arithmetic, except that over complete
 * blocks bf16 rows of q are exact from 2^-32 of their largest element on and smaller elements are rounded to
 * 2^-39 of the power of two below it; the same inputs give the same bits.  pool, tails, q and outputs are
 * 16-byte aligned.  With g query heads per KV head and t the largest divisor of g up to 16, the cache is read
 * g / t times (17 times for g = 17); n_seqs * (max_blocks_per_seq + 3) * kv_heads * g / t must be below 2^31.
 * Asynchronous on `stream`; may be captured. */
int isv_q8_attn(isv_q8 *h, const void *pool_dev, int32_t n_pages, const void *tails_dev,
                const int32_t *block_table_dev, int32_t table_stride, int32_t max_blocks_per_seq,
                const int32_t *seq_lens_dev, const void *q_dev, void *out_dev, float *out_f32_dev,
                int32_t n_seqs, void *stream);

/* Waits for `stream` and returns ISV_EDEVICE_STATUS (and clears the status) if a call on this handle
 * flagged a problem since the last query. */
int isv_q8_status(isv_q8 *h, void *stream, uint32_t *status_out);
/* As isv_set_wait_limit and isv_inject_lost_copy, for the attention's copies: `polls` of a barrier before a wait gives up
 * (0 = the built-in default), and launches in which the first block of the first sequence (if that has 16 tokens or more)
 * is armed without issuing its copy.  A warp whose wait runs out issues no more copies, gives those in flight one more
 * bounded chance to land and goes on without data; the launch ends with incomplete outputs, isv_q8_status reports it
 * once, and the handle stays usable. */
int isv_q8_set_wait_limit(isv_q8 *h, uint32_t polls);
int isv_q8_inject_lost_copy(isv_q8 *h, int32_t launches);

/* ---- pages of a paged cache ------------------------------------------------ */

/* (The paper has no counterpart: it treats the cache as one growing array per sequence.)  For callers that
 * own their pool and block table (isv_attn_decode_static, isv_q8_*).  All state is the table and the lengths:
 * a page is live if some row names it in the blocks its length covers, and free otherwise; there are no
 * reference counts to keep and nothing to release.  Rows may share pages.
 *   block_table_dev  int32 [n_rows][table_stride]; the first max_blocks_per_seq entries of a row are used
 *   lens_dev         int32 [n_rows] tokens; a length covers ceil(n / 16) blocks, or floor(n / 16) where the
 *                    open block has no page (open_in_pool = 0: the 8-bit cache)
 *   n_pages          pages of the pool, at most ISV_PAGES_MAX; ids outside [0, n_pages) are kept as they are,
 *                    and flagged with ISV_STATUS_BAD_BLOCK_ID unless ISV_BLOCK_NONE
 *   status_dev       optional uint32 into which ISV_STATUS_* bits are ORed
 * A row that is shortened (isv_pages_resize) to end inside a complete block: where it shares that page, the
 * caller gives it one of its own, or its next tokens go into the shared one; with open_in_pool = 0 the tokens
 * that it keeps of the block are stored again, since its tail slot does not hold them.
 * Free pages are handed out lowest id first.  Lengths that are negative or not covered by max_blocks_per_seq
 * are clamped and flagged (ISV_STATUS_BAD_LENGTH).  n_rows <= 4096.  All calls are asynchronous on `stream`,
 * use no memory but what they are given, run on the current device, and may be captured into a CUDA graph.
 * Results do not depend on scheduling. */
#define ISV_PAGES_MAX (1 << 20)

/* Copies whole pages: src_ids_dev[i] of src_pool to dst_ids_dev[i] of dst_pool (NULL = page i) for i < n, in
 * each of `layers` slabs that lie a layer stride apart.  page_bytes and the strides are multiples of 16.
 * n_dev (optional, device) lowers n to *n_dev.  An id of ISV_BLOCK_NONE on either side skips the pair; other
 * ids outside the pool are skipped and flagged.  The pools may be the same; a page that is both source and
 * destination of one call, or twice a destination, ends up with unspecified contents. */
int isv_pages_copy(void *dst_pool_dev, int32_t n_dst_pages, const void *src_pool_dev, int32_t n_src_pages,
                   uint64_t page_bytes, int32_t layers, uint64_t dst_layer_stride, uint64_t src_layer_stride,
                   const int32_t *src_ids_dev, const int32_t *dst_ids_dev, int32_t n, const int32_t *n_dev,
                   uint32_t *status_dev, void *stream);

/* Row s of the new table (table_out_dev, lens_out_dev; n_rows_out rows, same stride) continues old row
 * parent_dev[s]: the same row again (keep), another one (reorder), one that several rows name (fork), or
 * ISV_BLOCK_NONE for an empty row.  Old rows that nobody continues are freed.  Entries behind a row's blocks
 * become ISV_BLOCK_NONE; lens_out_dev[s] is the parent's length as it was, also where that had to be clamped.
 * Where rows continue the same parent and its last block is open (open_in_pool = 1
 * and length mod 16 not 0), the first of them keeps that page and every other one gets a fresh page, in row
 * order; copy_src_dev[s], copy_dst_dev[s] is then the pair for isv_pages_copy, else ISV_BLOCK_NONE twice.
 * Fresh pages may be pages of freed rows.  Without enough free pages the last rows' entries become
 * ISV_BLOCK_NONE (ISV_STATUS_NO_PAGES).  A parent outside [0, n_rows) other than ISV_BLOCK_NONE gives an empty
 * row (ISV_STATUS_BAD_BLOCK_ID).  The arrays must not overlap. */
int isv_pages_fork(const int32_t *block_table_dev, const int32_t *lens_dev, int32_t n_rows, const int32_t *parent_dev,
                   int32_t *table_out_dev, int32_t *lens_out_dev, int32_t n_rows_out, int32_t table_stride,
                   int32_t max_blocks_per_seq, int32_t open_in_pool, int32_t n_pages, int32_t *copy_src_dev,
                   int32_t *copy_dst_dev, uint32_t *status_dev, void *stream);

/* Grows and shrinks rows in place, from lens_dev to new_lens_dev (neither is written): blocks that a longer
 * row adds get free pages, in the order of rows and blocks; blocks behind the new length are freed, their
 * entries become ISV_BLOCK_NONE.  Length 0 frees a row.  Without enough free pages the last blocks in that
 * order become ISV_BLOCK_NONE (ISV_STATUS_NO_PAGES).  A page freed by this call may be handed out by it. */
int isv_pages_resize(int32_t *block_table_dev, const int32_t *lens_dev, const int32_t *new_lens_dev, int32_t n_rows,
                     int32_t table_stride, int32_t max_blocks_per_seq, int32_t open_in_pool, int32_t n_pages,
                     uint32_t *status_dev, void *stream);

/* Renames live pages so that they are exactly the ids [0, counts[0]): the i-th live page from counts[0] on
 * takes the i-th free id below it.  table_out_dev (may be block_table_dev itself) gets the new ids, with
 * ISV_BLOCK_NONE behind every row's blocks; src_ids_dev[i] -> dst_ids_dev[i], i < counts[1], are the moves for
 * isv_pages_copy (sources and destinations are disjoint), filled up with ISV_BLOCK_NONE to max_moves, which
 * must be at least n_pages / 2.  counts_dev: int32 [2]. */
int isv_pages_compact(const int32_t *block_table_dev, const int32_t *lens_dev, int32_t n_rows, int32_t table_stride,
                      int32_t max_blocks_per_seq, int32_t open_in_pool, int32_t n_pages, int32_t *table_out_dev,
                      int32_t *src_ids_dev, int32_t *dst_ids_dev, int32_t max_moves, int32_t *counts_dev,
                      uint32_t *status_dev, void *stream);

/* ---- decode linear layers with 4-bit weights -------------------------------- */

/* y = x . w^T as isv_linear_*, with w[n][k] = (u[n][k] - 8) * scale[n][k / group] and u in 0 .. 15, for M <= max_M
 * <= 64 tokens: a quarter of the weight bytes that bound a decode step's linear layers at small batches.
 *   w4_dev      uint8 [N][K / 2]: u[n][2 i] in the low and u[n][2 i + 1] in the high four bits of byte i
 *   scales_dev  [N][K / group] 16-bit of `dtype`; group 32, 64 or 128, K a multiple of it; N >= 1
 *   x_dev [M][K] 16-bit, 16-byte aligned;  y_dev [M][N] 16-bit and / or y_f32_dev [M][N] fp32 (one may be NULL)
 * isv_linear4_create lays the weights out anew in memory of its own (on `stream`, then waits for it): w4_dev and
 * scales_dev may be freed afterwards.  isv_linear4_forward is asynchronous on the stream it is given, keeps no
 * state between calls (calls may overlap) and may be captured; it runs on the handle's device.  Products are
 * exact and summed in fp32; the scale is applied to each group's sum. */
typedef struct isv_linear4 isv_linear4;
int isv_linear4_create(isv_linear4 **out, const void *w4_dev, const void *scales_dev, int32_t N, int32_t K,
                       int32_t group, int32_t dtype, int32_t max_M, void *stream);
int isv_linear4_forward(isv_linear4 *l, const void *x_dev, void *y_dev, float *y_f32_dev, int32_t M, void *stream);
/* Waits for `stream` and returns ISV_EDEVICE_STATUS (and clears the status) if a bounded wait inside a kernel
 * of this handle expired since the last query. */
int isv_linear4_status(isv_linear4 *l, void *stream, uint32_t *status_out);
/* As isv_set_wait_limit and isv_inject_lost_copy, for the copies of weights of this handle: `polls` of a barrier before
 * a wait gives up (0 = the built-in default), and launches in which one warp arms a barrier without issuing its copy.  A
 * warp whose wait runs out issues no more copies, gives those in flight one more bounded chance to land, and leaves
 * its sums incomplete; the launch ends, isv_linear4_status reports it once, and the handle stays usable. */
int isv_linear4_set_wait_limit(isv_linear4 *l, uint32_t polls);
int isv_linear4_inject_lost_copy(isv_linear4 *l, int32_t launches);
int isv_linear4_free(isv_linear4 *l);

/* ---- chunks of new tokens over a caller-owned paged cache --------------------- */

/* (The paper has no counterpart: its prefill stage stores keys and values that are given, and its decode stage attends
 * with one query per sequence.)  For callers that own their pool and block table (isv_attn_decode_static, isv_pages_*):
 * a chunk of a prompt, drafted tokens that the model is to check, or one token per sequence is stored with the position
 * rotation applied on the way (isv_chunk_write), its queries attend to the cache and to one another (isv_chunk_attn), and
 * what of a draft holds is decided (isv_draft_verify), whose lengths isv_pages_resize takes.
 *
 * The pool is [n_pages][K|V][kv_heads][16 tokens][head_dim] 16-bit in the order described under "KV pool layout" above,
 * one layer of it.  Sequence s has seq_lens_dev[s] tokens, the new ones included; its last new_lens_dev[s] <= T of them
 * (NULL = T of every sequence) are the chunk, at positions seq_lens_dev[s] - new_lens_dev[s] and on.  Their q, k, v and
 * outputs are rows row_starts_dev[s] and on (NULL = s * T) of arrays of n_rows rows, which no two sequences share; rows of no
 * sequence have no influence and are not written.  Row strides are in elements, multiples of 8, and hold at least a token's
 * heads: q, k and v may be parts of one array.
 * Lengths are clamped to what the table row holds (16 * max_blocks_per_seq), new lengths to [0, min(T, length)] and to the
 * rows there are, and flagged (ISV_STATUS_BAD_LENGTH).  All pointers but block tables, lengths, starts, prefixes, slopes,
 * frequencies and positions (aligned to their elements) are 16-byte aligned. */
#define ISV_ROTARY_HALVES    0   /* element i turns with element i + rotary_dim / 2 */
#define ISV_ROTARY_ADJACENT  1   /* element 2 i turns with element 2 i + 1          */

typedef struct {
    int32_t q_heads;             /* query heads; multiple of kv_heads                           */
    int32_t kv_heads;
    int32_t head_dim;            /* 64, 80 or 128                                               */
    int32_t dtype;               /* ISV_F16 or ISV_BF16                                         */
    int32_t max_seqs;            /* sequences per call, <= 4096                                 */
    int32_t max_ctas;            /* cap on the attention kernel's grid; 0 = one CTA per SM      */
    int32_t rotary_dim;          /* leading elements of a head that are turned: a multiple of   */
                                 /* 16 up to head_dim, 0 = none                                 */
    int32_t rotary_pairs;        /* ISV_ROTARY_HALVES or ISV_ROTARY_ADJACENT                    */
    int32_t rotary_axes;         /* position axes, 1 to 4                                       */
    float   scale;               /* of the scores; 0 = 1 / sqrt(head_dim)                       */
    float   softcap;             /* cap of the scores; 0 = none                                 */
} isv_chunk_desc;

typedef struct isv_chunk isv_chunk;

/* Allocates the attention's scratch and a status word on the current device (synchronous).  The handle holds no cache:
 * any number of layers and pools may be used with it.  isv_chunk_attn calls on one handle share its scratch: order them
 * on one stream or with events (one handle per stream or captured graph that may overlap another).  Calls run on the
 * handle's device, whichever is current. */
int isv_chunk_create(isv_chunk **out, const isv_chunk_desc *desc);
int isv_chunk_free(isv_chunk *h);

/* Stores the chunk's keys and values of one layer and turns its keys and queries:
 *     angle_i = position * inv_freq_dev[i],  i < rotary_dim / 2
 *     (a, b)  ->  (a cos - b sin, b cos + a sin) * magnitude    for the i-th pair of each head of k and q
 * computed in fp32 (the angle in 64 bits) and rounded once.  V is stored as it is.
 *   k_dev, v_dev     rows of kv_stride elements, [kv_heads][head_dim] each
 *   q_dev            rows of q_stride elements, [q_heads][head_dim] each; NULL = there are no queries to turn
 *   q_out_dev        [n_rows][q_heads][head_dim]; NULL = q_dev is turned in place
 *   inv_freq_dev     fp32 [rotary_dim / 2], radians per position
 *   positions_dev    int32 [rotary_axes][n_rows]: positions to turn by; NULL = the token's position in its sequence
 *   pair_axis_dev    uint8 [rotary_dim / 2]: which axis pair i goes by (images and video: time, height, width; values
 *                    beyond the last axis mean the last); NULL = axis 0
 *   magnitude        factor on the turned elements, 1 for none
 * A token whose block has no page (ISV_BLOCK_NONE or an id outside [0, n_pages)) is not stored, and flagged
 * (ISV_STATUS_BAD_BLOCK_ID); its query is turned all the same.  Inputs, pool and q_out must not overlap, and no two sequences
 * store into one page.
 * Asynchronous on `stream`; may be captured into a CUDA graph; calls may overlap. */
int isv_chunk_write(isv_chunk *h, void *pool_dev, int32_t n_pages, const int32_t *block_table_dev, int32_t table_stride,
                    int32_t max_blocks_per_seq, const int32_t *seq_lens_dev, const int32_t *new_lens_dev,
                    const int32_t *row_starts_dev, int32_t n_rows, const void *k_dev, const void *v_dev, int64_t kv_stride,
                    const void *q_dev, int64_t q_stride, void *q_out_dev, const float *inv_freq_dev,
                    const int32_t *positions_dev, const uint8_t *pair_axis_dev, float magnitude, int32_t n_seqs, int32_t T,
                    void *stream);

/* out[row][h] = softmax over the visible j of score(j), times V:
 *     x = (q . K_j) * scale;  if softcap > 0: x = softcap * tanh(x / softcap);  score(j) = x - slopes_dev[h] * |p - j|
 * for the query at position p of its sequence, p the chunk's first position and on.  Visible are the tokens with
 *     j <= p and (window = 0 or p - j < window), and those with j < prefix_lens_dev[s]
 * (a prefix that all queries see, later ones too), as far as they exist.  slopes_dev: fp32 [q_heads], or NULL;
 * prefix_lens_dev: int32 [n_seqs], or NULL.  Query head h reads KV head h / (q_heads / kv_heads).  out_dev (16-bit) and
 * out_f32_dev (fp32) are [n_rows][q_heads][head_dim], may each be NULL, not both, and overlap nothing.  A block without a page
 * (ISV_BLOCK_NONE) is left out and not flagged; other ids outside [0, n_pages) are left out and flagged.  A query that
 * sees nothing yields zeros.  What stands in invisible tokens, infinities and NaN too, changes nothing.
 * Scores, sums and statistics are fp32.  The softmax weights meet V as 16-bit numbers (an error of the order of the output's own
 * rounding) if out_f32_dev is NULL, and with fp32's precision if it is given.  The same inputs give the same bits.
 * A row whose sums are not finite (an infinity or NaN among the tokens of its tile, values near the type's largest) is computed
 * again, token by token: correctly, but slowly.
 * Asynchronous on `stream`; may be captured. */
int isv_chunk_attn(isv_chunk *h, const void *pool_dev, int32_t n_pages, const int32_t *block_table_dev, int32_t table_stride,
                   int32_t max_blocks_per_seq, const int32_t *seq_lens_dev, const int32_t *new_lens_dev,
                   const int32_t *row_starts_dev, int32_t n_rows, const void *q_dev, int64_t q_stride, const float *slopes_dev,
                   const int32_t *prefix_lens_dev, int32_t window, void *out_dev, float *out_f32_dev, int32_t n_seqs, int32_t T,
                   void *stream);

/* Waits for `stream` and returns ISV_EDEVICE_STATUS (and clears the status) if a call on this handle flagged a problem
 * since the last query. */
int isv_chunk_status(isv_chunk *h, void *stream, uint32_t *status_out);
/* As isv_set_wait_limit and isv_inject_lost_copy, for the attention's copies: `polls` of a barrier before a wait gives up
 * (0 = the built-in default), and launches in which the first page that is to be read is expected and not copied.  A CTA
 * in which a wait runs out gives the copies in flight one more bounded chance to land and leaves; the launch ends with
 * incomplete outputs, isv_chunk_status reports it once, and the handle stays usable. */
int isv_chunk_set_wait_limit(isv_chunk *h, uint32_t polls);
int isv_chunk_inject_lost_copy(isv_chunk *h, int32_t launches);

/* Which drafted tokens the target model's probabilities let stand, and the token behind them, so that the result is
 * distributed as the target's own tokens (given uniforms in [0, 1) that are independent of everything else).  With
 * n = n_draft_dev[s] <= max_draft drafts x_0 .. x_(n-1), target rows p_0 .. p_n and draft rows q_0 .. q_(n-1):
 *     a = the first i < n for which u_i * q_i(x_i) < p_i(x_i) does not hold, or n
 *     next token: drawn from max(p_a - q_a, 0) where a < n (from p_a if that is 0 everywhere), from p_n where a = n
 * A draw takes the lowest index whose running sum exceeds u * total, with u = uniforms[s][max_draft].  Sums are taken in
 * 64 bits (long ones as pairs of fp32 numbers); probabilities that are negative or NaN count as 0, and need not sum to 1.  They
 * are finite.
 *   target_dev     rows of vocab probabilities: rows row_starts_dev[s] .. + n (NULL = from s * (max_draft + 1) on) of n_rows
 *   draft_dev      [n_seqs][max_draft][vocab]; NULL = the drafts were certain (looked up, or the draft's best token):
 *                  q_i is 1 at x_i and 0 elsewhere.  dtype of both: ISV_F32, ISV_F16 or ISV_BF16
 *   drafted_dev    int32 [n_seqs][max_draft];  n_draft_dev int32 [n_seqs];  uniforms_dev fp32 [n_seqs][max_draft + 1]
 *   tokens_dev     int32 [n_seqs][max_draft + 1]: the a drafts that stand, the next token, then -1
 *   accepted_dev   int32 [n_seqs]: a
 *   lens_out_dev   int32 [n_seqs] or NULL: seq_lens_dev[s] - n + a, the length to keep (isv_pages_resize) of a cache in
 *                  which all n drafts stand
 *   status_dev     optional uint32 into which ISV_STATUS_* bits are ORed
 * A drafted token outside [0, vocab) does not stand (ISV_STATUS_BAD_TOKEN).  Where all of a row's probabilities are 0 the
 * next token is -1 (ISV_STATUS_BAD_TOKEN).  Counts outside [0, max_draft] and rows that are not there are clamped and
 * flagged (ISV_STATUS_BAD_LENGTH); a sequence without any row gets no token.  max_draft <= 1024.  Probabilities are aligned
 * to their elements; outputs overlap nothing, but lens_out_dev may be seq_lens_dev.  Uses no memory but what it is given and
 * runs on the current device; asynchronous on `stream`; may be captured; results do not depend on scheduling. */
int isv_draft_verify(const void *target_dev, const int32_t *row_starts_dev, int32_t n_rows, const void *draft_dev,
                     int32_t vocab, int32_t dtype, const int32_t *drafted_dev, const int32_t *n_draft_dev,
                     const float *uniforms_dev, const int32_t *seq_lens_dev, int32_t n_seqs, int32_t max_draft,
                     int32_t *tokens_dev, int32_t *accepted_dev, int32_t *lens_out_dev, uint32_t *status_dev, void *stream);

/* Text of the calling thread's last error; valid until its next call. */
const char *isv_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* ISV_H */
