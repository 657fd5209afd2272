/*
 * gva.h -- C ABI of the B200 (sm_100a) Grouped Value Attention decode library.
 *
 * One decode step of GVA with decoupled RoPE (Algorithm 1 of the paper) is three calls:
 *
 *   gva_absorb_query   q~_h = q^nope_h M_h^T  and  q^rope_h <- q^rope_h R_t^T      (Eq. absorb; Alg. 1)
 *   gva_append_cache   V_{1:t,g} <- [V_{1:t-1,g}; v_{t,g}],  k^rope_t = (.) R_t^T  (Eq. krope;  Alg. 1)
 *   gva_decode         s_j = q~_h v_{j,g(h)}^T + q^rope_h (k^rope_j)^T,
 *                      o_h = softmax(s / sqrt(d_qk)) V_{1:t,g(h)},  d_qk = d_c + d_r   (Section 3.3; Alg. 1)
 *
 * plus gqa_decode, a matched GQA decode over cached K and V (Section 2 / Section 3.4), built the
 * same way, as the reference point for the cache-bytes comparison N_GVA/N_GQA = 1/2 + d_r/(2 G d_h).
 *
 * Names: d_v = value width (paper d_h), d_c = content-key width (paper d_n), d_r = RoPE width,
 * H query heads, G value groups, head h reads group g(h) = h / (H/G).
 *
 * Conventions
 *   - All pointers are DEVICE pointers unless a parameter is marked [host].  The library allocates
 *     no device memory, keeps no caller pointer after a call returns, and never synchronises: every
 *     call enqueues work on `stream` (a cudaStream_t passed as void*; NULL = default stream).
 *   - Weights (the maps M, the packed projections W_in and W_o) are constants to the kernels: gva_absorb_query,
 *     gva_decode_step and the projections are launched as programmatic dependents of the kernel that precedes them in
 *     the stream and request their weights before they wait for that kernel's completion (all other inputs are read
 *     after the wait).  The kernel enqueued immediately before such a call must therefore not be the one that writes
 *     the weights it uses: write them by a copy, or by any earlier kernel.  (The library's own kernels never write weights.)
 *   - Return value: a gva_status detected on the host before/at launch.  Conditions only the device
 *     can see (a page id outside [0, num_pages), a sequence longer than its block table) are
 *     recorded once in *dev_status (caller-zeroed int32 on the device; may be NULL) as
 *     code | (sequence_index << 8); the offending work is skipped and the kernel ends normally.
 *   - RoPE: pairs (2i, 2i+1) of the d_r-wide slice are rotated by the angle pos * base^(-2i/d_r)
 *     (y[2i] = x[2i] cos a - x[2i+1] sin a, y[2i+1] = x[2i] sin a + x[2i+1] cos a), evaluated in fp64.
 *   - Cache layout ("pools"): v_pool [num_pages][G][page_size][d_v], kr_pool [num_pages][page_size][d_r],
 *     element type = cfg.cache_dtype.  Logical page j of sequence b is block_table[b*max_pages_per_seq + j];
 *     block_table == NULL means contiguous: page j of sequence b is b*max_pages_per_seq + j.
 *     Slots at or beyond seq_lens[b] and block-table entries beyond ceil(seq_lens[b]/page_size) are never
 *     read by gva_decode (they may hold NaN / -1).
 */
#ifndef GVA_H_
#define GVA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    GVA_OK = 0,
    GVA_ERR_INVALID_ARG = 1,  /* null pointer, negative size, misaligned pointer                         */
    GVA_ERR_UNSUPPORTED = 2,  /* shape / dtype / page size outside the instantiated kernels              */
    GVA_ERR_WORKSPACE = 3,    /* workspace smaller than gva_decode_workspace_bytes()                     */
    GVA_ERR_CUDA = 4,         /* a CUDA runtime/driver call failed (launch error, no sm_100 device, ...) */
    GVA_ERR_BAD_PAGE = 5,     /* [device] block-table entry outside [0, num_pages) in the live range     */
    GVA_ERR_SEQ_LEN = 6,      /* [device] seq_len < 0 or beyond max_pages_per_seq * page_size            */
    GVA_ERR_TIMEOUT = 7,      /* [device] a bounded wait on an asynchronous copy expired                 */
    GVA_ERR_STATIC_LIMIT = 8, /* gva_decode_static: the request needs more than GVA_STATIC_SCRATCH_BYTES  */
    GVA_ERR_NO_ROOM = 9,      /* [device] gva_assign_pages: not enough free pages or rows for a sequence  */
    GVA_ERR_TREE = 10         /* [device] a node's parent is not a node before it, or a tree has more nodes than max_q_len */
} gva_status;

/* Element type of the cache pools.  GVA_E4M3 stores every cache element as one byte (sign, 4 exponent bits with bias 7,
 * 3 mantissa bits; no infinities, 0x7F / 0xFF = NaN, largest finite 448): appends round to nearest even and saturate
 * at +-448, decode widens the codes exactly and computes as for the other types.  The paper stores 16-bit caches; the
 * 8-bit cache is this library's extension of its byte accounting (Section 3.4) and halves the bytes per token again.
 * It is built for (d_v, d_r) = (64, 16), (64, 0), (128, 32), (128, 0), G <= 8, pages of a multiple of 64 tokens, with the
 * tensor-core kernel only:
 * gva_absorb_query, gva_append_cache, gva_append_chunk, gva_decode, gva_decode_step, gva_decode_step_host,
 * gva_decode_static, gqa_decode (keys and values as e4m3 codes), the projections, gva_layer_step and (with a positional
 * slice, d_r > 0) gva_decode_tokens / gva_decode_tokens_ragged serve it, and so do gva_prefill and gva_decode_multi (the
 * byte tiles are widened to f16 in shared memory; queries and weights are then f16 instead of bf16), gva_append_cache_at, gva_append_rows,
 * gqa_append, gva_attention_weights, gva_evict and gva_tree_commit; gva_decode_tree serves it on CUDA cores. */
typedef enum { GVA_F32 = 0, GVA_BF16 = 1, GVA_E4M3 = 2 } gva_dtype;

/* Which decode kernel gva_decode launches.  AUTO = tensor-core kernel when the cache is bf16 or e4m3,
 * CUDA-core (FMA) kernel for an f32 cache.  FMA / MMA force one (MMA with an f32 cache and
 * FMA with an e4m3 cache are GVA_ERR_UNSUPPORTED). */
typedef enum { GVA_KERNEL_AUTO = 0, GVA_KERNEL_FMA = 1, GVA_KERNEL_MMA = 2 } gva_kernel;

typedef struct {
    int32_t H, G;          /* query heads, value groups; H % G == 0 and H/G == 4                          */
    int32_t d_v;           /* value width: 64 or 128                                                      */
    int32_t d_c;           /* content-key width (only gva_absorb_query uses it): 1..256                   */
    int32_t d_r;           /* RoPE width: 16 or 24 with d_v = 64 (the paper's two tested widths), 32 with d_v = 128;
                              0 = value-only cache without a positional slice (Section 3.4: a cache of values alone is
                              half of matched GQA's): kr_pool, q_r and kr_new are then unused and may be NULL, scale = 1/sqrt(d_c) */
    int32_t page_size;     /* tokens per page, a multiple of 32                                           */
    int32_t cache_dtype;   /* gva_dtype                                                                   */
    int32_t kernel;        /* gva_kernel                                                                  */
    double rope_base;      /* 10000.0                                                                     */
    float softmax_scale;   /* 0 => 1/sqrt(d_c + d_r)                                                      */
    int32_t reserved;      /* set to 0                                                                    */
} gva_config;

typedef struct {
    void *v_pool;               /* [num_pages][G][page_size][d_v]   16-byte aligned                        */
    void *kr_pool;              /* [num_pages][page_size][d_r]      16-byte aligned                        */
    const int32_t *block_table; /* [B][max_pages_per_seq] or NULL (contiguous)                             */
    int32_t num_pages;
    int32_t max_pages_per_seq;
} gva_cache;

typedef struct {
    void *k_pool;               /* [num_pages][G][page_size][d_h]  keys, already rotated                    */
    void *v_pool;               /* [num_pages][G][page_size][d_h]                                           */
    const int32_t *block_table;
    int32_t num_pages;
    int32_t max_pages_per_seq;
} gqa_cache;

typedef struct gva_handle gva_handle; /* opaque host-side state: config, device properties, last launch geometry */

/* Create / destroy a handle for one head configuration on one device.  Validates cfg
 * (GVA_ERR_UNSUPPORTED / GVA_ERR_INVALID_ARG), checks that `device` is compute capability 10.x
 * (GVA_ERR_CUDA otherwise) and raises the kernels' shared-memory limits.  Makes `device` current.
 *
 * One handle, one stream at a time.  Besides its host-side state a handle owns a few words of DEVICE-side
 * scheduling state inside the library image (the counters through which the thread blocks of a decode
 * kernel share out the tail of the cache stream).  Decode calls on one handle -- gva_decode, gqa_decode,
 * gva_decode_step(_host), gva_decode_static, gva_decode_tokens, gva_layer_step -- must therefore be
 * stream-ordered with respect to one another: issue them on one stream, or order the streams with events.
 * Two such calls that may overlap on the GPU race on those words even if their workspaces differ (wrong
 * partition of the work, hence wrong results; never a fault).  Use one handle per concurrent stream; handles
 * are cheap (no device allocation).  The handle is not thread-safe either: one host thread at a time.
 * gva_destroy only after the last call on the handle has finished on the device. */
int gva_create(gva_handle **out, const gva_config *cfg, int device);
int gva_destroy(gva_handle *h);

/* Bytes of scratch gva_decode / gqa_decode need for B sequences of at most max_seq_len tokens with
 * the given num_splits (same meaning as in gva_decode).  Holds the split-KV partial results
 * (unnormalised output, running max and sum per partition and head).  0 on invalid arguments. */
size_t gva_decode_workspace_bytes(const gva_handle *h, int B, int max_seq_len, int num_splits);

/* Eq. absorb and the query-side rotation of Algorithm 1.
 *   q_c   [B][H][d_c] f32   content ("nope") query slices
 *   q_r   [B][H][d_r] f32   positional query slices, unrotated
 *   M     [H][d_v][d_c] f32 reconstruction maps, row-major (M_h in R^{d_h x d_n}; K_h = V_g(h) M_h)
 *   q_pos [B] i32           query positions t (0-based)
 *   q_abs [B][H][d_v+d_r] f32 out:  [:d_v] = q_c M_h^T  (q~[i] = sum_j q_c[j] M_h[i][j]),
 *                                   [d_v:] = q_r R_t^T */
int gva_absorb_query(gva_handle *h, const float *q_c, const float *q_r, const float *M,
                     const int32_t *q_pos, float *q_abs, int B, void *stream);

/* Algorithm 1's cache append for one new token per sequence.
 *   v_new  [B][G][d_v] f32   new value rows;  kr_new [B][d_r] f32 unrotated positional key (x_t W_r)
 *   pos    [B] i32           0-based position t of the new token
 * Writes, for each b, rows (page = block_table[b][t/page_size], slot = t % page_size):
 *   v_pool[page][g][slot][:] = cast(v_new[b][g][:]),  kr_pool[page][slot][:] = cast(kr_new[b] R_t^T)
 * cast = round-to-nearest-even to the cache dtype (from the fp64 rotation for k^rope); no other byte
 * of the pools changes.  pos < 0 or beyond the block table -> GVA_ERR_SEQ_LEN in *dev_status, bad
 * page id -> GVA_ERR_BAD_PAGE; that sequence is skipped. */
int gva_append_cache(gva_handle *h, const gva_cache *cache, const float *v_new, const float *kr_new,
                     const int32_t *pos, int B, int32_t *dev_status, void *stream);

/* Decode attention over the cache (the score and softmax-value lines of Algorithm 1) for B
 * sequences, query heads sharing each value group's stream.
 *   q_abs    [B][H][d_v+d_r] f32  from gva_absorb_query
 *   seq_lens [B] i32              number of cached tokens attended (positions 0..seq_len-1)
 *   out      [B][H][d_v] f32      o_h;  seq_len == 0 gives 0
 *   lse      [B][H] f32 or NULL   natural log of sum_j exp(scale * s_j); -inf for seq_len == 0
 *   workspace / workspace_bytes   scratch of at least gva_decode_workspace_bytes(h, B, max_seq_len, num_splits),
 *                                 256-byte aligned; contents are overwritten; calls sharing it must be
 *                                 stream-ordered
 *   max_seq_len                   upper bound on seq_lens[] (sizes the launch; a longer sequence is
 *                                 still computed correctly as long as it fits its block table)
 *   num_splits                    0: the cache stream is cut into equal contiguous ranges of tiles, one
 *                                 per resident thread block (ranges may cross sequence boundaries);
 *                                 n >= 1: every sequence is cut into exactly n ranges.
 * Partial results are merged by log-sum-exp weights in a second kernel.  For fixed arguments the
 * result is bitwise reproducible from run to run.  Calls on one handle must be stream-ordered (see gva_create).
 * The call may be captured into a CUDA graph (after one call outside the capture, which sizes the handle's scheduling
 * state) and replayed with different contents of its device buffers: every call leaves the scheduling words as it
 * found them, and nothing on the device depends on the call's number changing between replays. */
int gva_decode(gva_handle *h, const gva_cache *cache, const float *q_abs, const int32_t *seq_lens,
               float *out, float *lse, void *workspace, size_t workspace_bytes, int B, int max_seq_len,
               int num_splits, int32_t *dev_status, void *stream);

/* gva_decode for callers that cannot allocate device memory.  (The paper has no counterpart: this
 * entry point exists for the library's users, not for the method.)
 *
 * Who this is for: code that runs where cudaMalloc is off limits -- inside a serving loop whose memory
 * pool was sized and frozen at start-up, under a framework allocator that forbids side allocations, or
 * in a plug-in that is handed tensors but no allocator.  Such callers cannot provide the split-KV
 * workspace gva_decode asks for, so here the partial results live in a fixed array compiled into the
 * library (GVA_STATIC_SCRATCH_BYTES of device memory, held by every GPU that loads the library until
 * the process exits).  Inputs and outputs are still the caller's, with the same meaning, layout and
 * error rules as gva_decode; neither this call nor anything it uses calls cudaMalloc, cudaFree or an
 * allocating library routine.
 *
 *  - Limit: if gva_decode_workspace_bytes(h, B, max_seq_len, num_splits) exceeds
 *    GVA_STATIC_SCRATCH_BYTES the call launches nothing and returns GVA_ERR_STATIC_LIMIT.  At num_splits = 0
 *    the need grows with the batch (one partial record per sequence on top of a few per thread block), not
 *    with the context length: on a B200 the five workloads of the benchmark take 2.5 to 5.5 MB (for example
 *    B = 32 sequences of 32768 tokens, H = 16, d_v = 64: 5.1 MB; B = 64, H = 32, d_v = 128: 3.5 MB), and
 *    H = 16, d_v = 64 fits up to about B = 2700.  With num_splits = n the need is B * n records of
 *    H * (d_v + 2) * 4 bytes each.
 *  - Set-up: the first call on each device looks up the array's device address (once per device; the
 *    handle's device must be the current device, otherwise GVA_ERR_INVALID_ARG).  Make that first
 *    call outside any stream capture.
 *  - Sharing: every call on a device uses the same array, and it keeps whatever the previous call left.
 *    Nothing needs clearing -- each call writes every word it later reads -- but two calls that may run
 *    at the same time on one GPU (different streams, different handles, different threads) race on it:
 *    keep calls to this entry point stream-ordered per device. */
#define GVA_STATIC_SCRATCH_BYTES (16u << 20)
int gva_decode_static(gva_handle *h, const gva_cache *cache, const float *q_abs, const int32_t *seq_lens,
                      float *out, float *lse, int B, int max_seq_len, int num_splits, int32_t *dev_status,
                      void *stream);

/* Matched GQA decode (two cached streams): s_j = q_h K_{j,g(h)}^T / sqrt(d_h), o_h = softmax(s) V_{g(h)},
 * with d_h = cfg.d_v, q [B][H][d_h] f32 already rotated, K cached already rotated.  Same paging,
 * splitting, workspace and error rules as gva_decode.  cfg.d_c, cfg.d_r and cfg.softmax_scale are
 * ignored (scale = 1/sqrt(d_h)). */
int gqa_decode(gva_handle *h, const gqa_cache *cache, const float *q, const int32_t *seq_lens, float *out,
               float *lse, void *workspace, size_t workspace_bytes, int B, int max_seq_len, int num_splits,
               int32_t *dev_status, void *stream);

/* One whole decode step on device buffers: the same results, bit for bit, as gva_absorb_query ->
 * gva_append_cache -> gva_decode called in that order (Algorithm 1 from the split queries to the
 * per-head outputs), in two launches instead of four: absorb and append run in one kernel, and the
 * decode kernel starts its bookkeeping and its first cache loads while that kernel computes.
 *   pos      [B] i32  position t of the new token: the append slot and the query position
 *   seq_lens [B] i32  tokens attended (normally t + 1, so the query sees its own token)
 *   q_abs    [B][H][d_v+d_r] f32  written by the call (the absorbed queries), then read by the decode
 *   other arguments as in the three separate calls.
 * Because the decode kernel reads seq_lens, pos, the block table and cache tiles other than the one
 * receiving the new token before the fused front kernel has finished, those must not be outputs of
 * that same call; everything enqueued on the stream before the call is complete before any of it is read. */
int gva_decode_step(gva_handle *h, const gva_cache *cache, const float *M, const float *q_c, const float *q_r,
                    const float *v_new, const float *kr_new, const int32_t *pos, const int32_t *seq_lens,
                    float *q_abs, float *out, float *lse, void *workspace, size_t workspace_bytes, int B,
                    int max_seq_len, int num_splits, int32_t *dev_status, void *stream);

/* One whole decode step (Algorithm 1 from the split queries to the per-head outputs) for callers whose
 * per-step tensors live in HOST memory: copies the step's inputs to the device, runs
 * gva_decode_step, and copies the outputs back, all enqueued on
 * `stream`; the caller synchronises the stream before reading out_host.  The cache and the maps M stay
 * resident on the device (they are state, not per-step input).
 *   [host] q_c_host [B][H][d_c], q_r_host [B][H][d_r], v_new_host [B][G][d_v], kr_new_host [B][d_r] f32,
 *          pos_host [B] i32 (position t of the new token = query position), seq_lens_host [B] i32
 *          (tokens attended, normally t + 1).  If the four float inputs and out_host are all pinned
 *          (page-locked, device-mapped) memory the kernels read and write them in place over the
 *          interconnect and only pos and seq_lens are brought to the device (by a one-block kernel when they are
 *          pinned too, else by two copies); otherwise every buffer is staged through
 *          `scratch` with cudaMemcpyAsync (pageable memory makes those copies synchronous).
 *   [host] out_host [B][H][d_v] f32
 *   M                device, as in gva_absorb_query
 *   scratch          device, at least gva_step_scratch_bytes(h, B, max_seq_len, num_splits) bytes, 256-byte aligned;
 *                    holds the staged inputs, q_abs, out and the decode workspace.
 * Bytes moved per call: host->device B*(H*(d_c+d_r) + G*d_v + d_r)*4 + 8*B, device->host B*H*d_v*4. */
size_t gva_step_scratch_bytes(const gva_handle *h, int B, int max_seq_len, int num_splits);
int gva_decode_step_host(gva_handle *h, const gva_cache *cache, const float *M, const float *q_c_host,
                         const float *q_r_host, const float *v_new_host, const float *kr_new_host,
                         const int32_t *pos_host, const int32_t *seq_lens_host, float *out_host, void *scratch,
                         size_t scratch_bytes, int B, int max_seq_len, int num_splits, int32_t *dev_status,
                         void *stream);

/* ---- The projections around the attention (Algorithm 1: q_t = x_t W_Q, v_t = x_t W_V, k^rope_t = (x_t W_r) R_t^T;
 * then the heads side by side through the output projection), with the maps folded into the query projection:
 * because M_h is fixed at inference, q~_h = (x W_Q^{nope,h}) M_h^T = x (W_Q^{nope,h} M_h^T)  (Eq. absorb), so
 * one product with a packed weight matrix yields the absorbed queries directly and gva_absorb_query drops out.
 *
 * Packed input projection W_in: bf16 [d_model][N_in], N_in = gva_input_width() = H*(d_v+d_r) + G*d_v + d_r,
 * columns per head h: d_v folded content columns (W_Q^{nope,h} M_h^T), then d_r positional-query columns;
 * then the G*d_v value columns; then the d_r positional-key columns.  d_model must be a multiple of 128. */
int gva_input_width(const gva_handle *h);

/* [host] Offline packing of one layer's input projection: folds the maps in fp64 and rounds every entry once to
 * bf16.  W_q_nope [d_model][H][d_c], W_q_rope [d_model][H][d_r], W_v [d_model][G][d_v], W_r [d_model][d_r],
 * M [H][d_v][d_c] f32 (host); W_in [d_model][N_in] bf16 bit patterns (host, caller uploads it).  With a value-only
 * cache (d_r = 0) there are no positional columns: W_q_rope and W_r are unused and may be NULL. */
int gva_pack_input_weights(const gva_handle *h, const float *W_q_nope, const float *W_q_rope, const float *W_v,
                           const float *W_r, const float *M, int d_model, uint16_t *W_in);
/* [host] f32 -> bf16 bit patterns, nearest even (for the output projection W_o). */
int gva_pack_bf16(const float *src, uint16_t *dst, size_t n);

/* x [B][d_model] f32 -> q_abs [B][H][d_v+d_r] f32 (positional slice rotated at pos[b]) and the cache append of the
 * new token at pos[b], in one kernel.  The appended rows are bit for bit what gva_append_cache writes when it is given
 * the kernel's own f32 products as v_new / kr_new (value rows rounded once to the cache dtype, k^rope rotated in fp64
 * and rounded once); against products accumulated in higher precision they can differ by one unit in the last place
 * of the cache dtype.  Same device-side error rules as gva_append_cache. */
int gva_project_in(gva_handle *h, const gva_cache *cache, const float *x, const void *W_in, int d_model,
                   const int32_t *pos, float *q_abs, int B, int32_t *dev_status, void *stream);
/* attn [B][H*d_v] f32 (heads concatenated, as gva_decode writes them) x W_o bf16 [H*d_v][d_model] -> y [B][d_model] f32. */
int gva_project_out(gva_handle *h, const float *attn, const void *W_o, int d_model, float *y, int B, void *stream);
/* A whole layer's decode step from the hidden state: gva_project_in -> gva_decode -> gva_project_out. */
int gva_layer_step(gva_handle *h, const gva_cache *cache, const float *x, const void *W_in, const void *W_o,
                   int d_model, const int32_t *pos, const int32_t *seq_lens, float *q_abs, float *attn, float *y,
                   void *workspace, size_t workspace_bytes, int B, int max_seq_len, int num_splits,
                   int32_t *dev_status, void *stream);

/* ---- Several new tokens per sequence: prefill and chunked prefill (the paper's multi-token form: ordinary causal
 * attention whose scores keep the content + positional split, Section 3.3 and the remark after Algorithm 1), computed in the
 * absorbed form of Eq. absorb.  Sequence b has ctx_lens[b] tokens cached already and q_len_b = cu_q[b+1] - cu_q[b]
 * new tokens; new token i of sequence b is input row cu_q[b] + i, sits at position t = ctx_lens[b] + i and attends
 * to positions 0..t.  The order of calls is Algorithm 1's, once per chunk instead of once per token:
 *   gva_absorb_query(B := n_q, q_pos[row] = position of the row)  ->  gva_append_chunk  ->  gva_prefill.
 *   cu_q [B+1] i32 (cu_q[0] = 0, non-decreasing), ctx_lens [B] i32, n_q = cu_q[B] rows in all. */

/* Algorithm 1's append for every new token of the chunk: row n of v_new [n_q][G][d_v] / kr_new [n_q][d_r] (unrotated)
 * is written at its position exactly as gva_append_cache writes one token (same rounding, same error rules). */
int gva_append_chunk(gva_handle *h, const gva_cache *cache, const float *v_new, const float *kr_new,
                     const int32_t *cu_q, const int32_t *ctx_lens, int B, int n_q, int32_t *dev_status, void *stream);

/* Causal attention of the chunk over the cache, which must already hold the chunk's own tokens.
 *   q_abs [n_q][H][d_v+d_r] f32  from gva_absorb_query;  out [n_q][H][d_v] f32;  lse [n_q][H] f32 or NULL
 *   max_q_len                    upper bound on the q_len_b (sizes the launch; longer chunks are cut off)
 * bf16 or e4m3 cache, page_size a multiple of 64, (d_v, d_r) = (64, 16), (64, 24) (bf16 only), (128, 32), (64, 0) or
 * (128, 0); otherwise GVA_ERR_UNSUPPORTED.
 * Runs on the tensor cores with bf16 operands (the absorbed query and the softmax weights are rounded to bf16,
 * accumulation is f32), so results carry bf16-level error: |out - exact| <= 2e-2 for unit-variance data.
 * Device-side errors as in gva_decode; a thread block that meets one stops and leaves its rows of out unwritten. */
int gva_prefill(gva_handle *h, const gva_cache *cache, const float *q_abs, const int32_t *cu_q,
                const int32_t *ctx_lens, float *out, float *lse, int B, int max_q_len, int32_t *dev_status,
                void *stream);

/* Decode of several new tokens per sequence over a long cached context (speculative / multi-token decode; not in the
 * paper -- Algorithm 1 applied to q_len_b tokens at once, i.e. gva_prefill's computation) with split-KV: every block of
 * 32 query tokens is handled by several thread blocks, each over a contiguous range of 64-token tiles, and a second
 * kernel merges their partial results by log-sum-exp weights, so that small batches still fill the GPU.
 *   arguments as gva_prefill, plus
 *   n_q                          cu_q[B]: query rows in all (sizes the merge)
 *   max_seq_len                  upper bound on ctx_lens[b] + q_len_b
 *   num_splits                   0 = enough splits for two thread blocks per SM; n >= 1 = exactly n (at most one per tile, 64)
 *   workspace / workspace_bytes  at least gva_decode_multi_workspace_bytes(...) bytes, 256-byte aligned
 * Same support, tolerance and error rules as gva_prefill. */
size_t gva_decode_multi_workspace_bytes(const gva_handle *h, int B, int n_q, int max_q_len, int max_seq_len,
                                        int num_splits);
int gva_decode_multi(gva_handle *h, const gva_cache *cache, const float *q_abs, const int32_t *cu_q,
                     const int32_t *ctx_lens, float *out, float *lse, void *workspace, size_t workspace_bytes, int B,
                     int n_q, int max_q_len, int max_seq_len, int num_splits, int32_t *dev_status, void *stream);

/* Decode of q_len = 2 .. 8 new tokens per sequence at the single-token kernel's cache-stream rate (speculative /
 * multi-token decode; not in the paper -- Algorithm 1 applied to q_len tokens at once).  The split-KV tensor-core decode
 * kernel of gva_decode carries the 4 * q_len (head, token) pairs of a value group as its MMA columns, so the cache is
 * streamed once for all of them.  Every sequence has exactly q_len new tokens, already appended.
 *   q_abs    [B * q_len][H][d_v+d_r] f32  row b * q_len + i = new token i of sequence b (from gva_absorb_query)
 *   seq_lens [B] i32                      tokens attended by the LAST new token; new token i attends seq_lens[b] - (q_len-1-i)
 *   out      [B * q_len][H][d_v] f32, lse [B * q_len][H] f32 or NULL
 *   workspace                             at least gva_decode_tokens_workspace_bytes(...) bytes, 256-byte aligned
 * q_len 2 .. 4: bf16 cache with (d_v, d_r) = (64, 16), (64, 24) (pages of a multiple of 64 tokens), (64, 0), (128, 32) or
 * (128, 0), and the e4m3 cache with a positional slice; q_len 5 .. 8: bf16 cache with d_v = 64, d_r = 16, 24 or 0, G <= 4
 * and pages of a multiple of 64 tokens; tensor-core kernel only; otherwise GVA_ERR_UNSUPPORTED.  The queries enter the score product as two bf16 numbers each (hi + lo), the
 * softmax weights as one (the 8-bit cache: f16 instead of bf16), accumulation is f32: |out - exact| <= 2e-2 whatever
 * the size of the scores. */
size_t gva_decode_tokens_workspace_bytes(const gva_handle *h, int B, int q_len, int max_seq_len, int num_splits);
int gva_decode_tokens(gva_handle *h, const gva_cache *cache, const float *q_abs, const int32_t *seq_lens, float *out,
                      float *lse, void *workspace, size_t workspace_bytes, int B, int q_len, int max_seq_len,
                      int num_splits, int32_t *dev_status, void *stream);

/* The same with a different number of new tokens per sequence (a batch in which some sequences verify eight draft
 * tokens, some two, some none): sequence b has q_len_b = cu_q[b+1] - cu_q[b] new tokens, 0 <= q_len_b <= max_q_len <= 8,
 * already appended; its rows of q_abs / out / lse are cu_q[b] .. cu_q[b+1] - 1 (cu_q [B + 1] i32, cu_q[0] = 0,
 * non-decreasing).  seq_lens[b] = tokens attended by the last new token of b; new token i attends
 * seq_lens[b] - (q_len_b - 1 - i).  Workspace: gva_decode_tokens_workspace_bytes(h, B, max(max_q_len, 2), ...).
 * Caches and shapes as gva_decode_tokens for the given max_q_len.  Same accuracy. */
int gva_decode_tokens_ragged(gva_handle *h, const gva_cache *cache, const float *q_abs, const int32_t *cu_q,
                             const int32_t *seq_lens, float *out, float *lse, void *workspace, size_t workspace_bytes, int B,
                             int max_q_len, int max_seq_len, int num_splits, int32_t *dev_status, void *stream);

/* ---- A cache that is kept small: 4-bit values, gathered attention weights, eviction --------------------------------
 * (Not in the paper, which stores 16-bit values and keeps every token: this library's extension of its byte accounting,
 * Section 3.4.)  All calls below want the handle's device to be the current one (GVA_ERR_INVALID_ARG otherwise), use no
 * state of the handle on the device, and may be captured into CUDA graphs and replayed; calls on different streams may
 * overlap as long as they share no workspace, no output and no page that one of them writes.  Any of the head shapes of
 * gva_create is served, with every page size.
 *
 * The 4-bit cache.  A value row x[0 .. d_v) of one token and group is held as d_v codes of 4 bits and two f16 numbers:
 *     lowest z = the largest f16 <= min x,   step s = the smallest f16 with z + 15 s >= max x,
 *     code c = the number of k in 0 .. 14 with x >= z + (k + 1/2) s,   value = z + s c,   hence |value - x| <= s / 2.
 * Elements beyond +-65504 are clamped first; a row with a NaN anywhere reads as NaN (and attention that sees it gives NaN, however
 * the sequence is split); a row of one value has s = 0.
 * Positional keys are bf16.  A token takes G (d_v / 2 + 4) + 2 d_r bytes: 176 against the bf16 cache's 544 with H = 16,
 * G = 4, d_v = 64, d_r = 16.  The calls take a handle with cache_dtype = GVA_BF16 (GVA_ERR_UNSUPPORTED otherwise), which
 * serves bf16 caches beside it: gva_q4_widen brings tokens into bf16 pages for the calls that have no 4-bit form
 * (gva_prefill, gva_decode_tokens, gva_decode_multi). */
typedef struct {
    void *v_pool;               /* [num_pages][G][page_size][d_v / 2] bytes: dim 2 i low, dim 2 i + 1 high nibble; 16-byte aligned */
    void *sz_pool;              /* [num_pages][G][page_size] pairs of f16 (step, lowest)                   16-byte aligned */
    void *kr_pool;              /* [num_pages][page_size][d_r] bf16; unused with d_r = 0                   16-byte aligned */
    const int32_t *block_table; /* [B][max_pages_per_seq] or NULL (contiguous)                             */
    int32_t num_pages;
    int32_t max_pages_per_seq;
} gva_q4_cache;

/* gva_append_cache where the slot is not the position (a cache that has lost tokens to gva_evict, any cache type):
 *   slots [B] i32   slot of the new token, normally the number of tokens the sequence holds
 *   pos   [B] i32   position its key is rotated to; < 0 -> GVA_ERR_SEQ_LEN in *dev_status, the sequence is skipped
 * With slots == pos it writes what gva_append_cache writes. */
int gva_append_cache_at(gva_handle *h, const gva_cache *cache, const float *v_new, const float *kr_new, const int32_t *slots,
                        const int32_t *pos, int B, int32_t *dev_status, void *stream);

/* Append of one new token per sequence to the 4-bit cache: arguments and device-side errors as gva_append_cache_at. */
int gva_q4_append(gva_handle *h, const gva_q4_cache *cache, const float *v_new, const float *kr_new, const int32_t *slots,
                  const int32_t *pos, int B, int32_t *dev_status, void *stream);

/* Append of a chunk of new tokens per sequence to the 4-bit cache: rows and errors as gva_append_chunk (row cu_q[b] + i goes
 * to slot ctx_lens[b] + i); the key of that row is rotated to position first_pos[b] + i (first_pos NULL: to its slot).
 * Rows at or beyond cu_q[B] are not read. */
int gva_q4_append_chunk(gva_handle *h, const gva_q4_cache *cache, const float *v_new, const float *kr_new, const int32_t *cu_q,
                        const int32_t *ctx_lens, const int32_t *first_pos, int B, int n_q, int32_t *dev_status, void *stream);

/* Slots starts[b] .. seq_lens[b] - 1 (starts NULL: from 0) of every sequence as rows of a bf16 cache with the same page size,
 * same slots: value rows z + s c, rounded to f32 and then to bf16, positional rows as they are.  Nothing else of the bf16 cache changes.
 * max_seq_len sizes the launch (longer sequences are widened whole, those beyond either block table to its end, with
 * GVA_ERR_SEQ_LEN).  The two caches must not share memory. */
int gva_q4_widen(gva_handle *h, const gva_q4_cache *cache, const gva_cache *wide, const int32_t *starts, const int32_t *seq_lens,
                 int B, int max_seq_len, int32_t *dev_status, void *stream);

/* Decode attention over the 4-bit cache: arguments, splitting, outputs and errors as gva_decode (a tile whose page is bad
 * counts as empty).  Content queries and softmax weights enter the products as two f16 numbers each (22 bits), positional queries as
 * three bf16 numbers, accumulation is f32: measured against 64 bits the result is as far off as that of f32 arithmetic on the cached
 * values (1.3e-7 of its size over 1 M tokens, 1.1e-7 in f32).  Bitwise reproducible for fixed arguments.
 * Workspace: at least gva_q4_decode_workspace_bytes(h, B, max_seq_len, num_splits) bytes, 256-byte aligned. */
size_t gva_q4_decode_workspace_bytes(const gva_handle *h, int B, int max_seq_len, int num_splits);
int gva_q4_decode(gva_handle *h, const gva_q4_cache *cache, const float *q_abs, const int32_t *seq_lens, float *out, float *lse,
                  void *workspace, size_t workspace_bytes, int B, int max_seq_len, int num_splits, int32_t *dev_status, void *stream);

/* The attention every cached token has received, added up:
 *   weights_out[b][t] = decay * weights_in[b][t] + sum over the new rows r of sequence b that see slot t, and over all
 *                       heads, of exp(scale * score(r, head, t) - lse[r][head]),        t < seq_lens[b]
 * i.e. the softmax weights of the attention whose lse is given (where lse is -inf nothing is added, whatever q_abs holds there).
 * Queries enter the score products as three bf16 numbers each (24 bits) over a bf16 cache, as two f16 numbers (22 bits) over e4m3 and
 * 4 bits (there the positional part as three bf16), accumulation is f32; over an f32 cache all is f32.  Measured against 64 bits: 2e-7
 * of the weights, 1e-7 in plain f32 arithmetic.
 *   q_abs [rows][H][d_v+d_r], lse [rows][H] f32   as the attention call had and returned them
 *   cu_q  [B + 1] i32 or NULL    rows cu_q[b] .. cu_q[b+1] - 1 belong to sequence b, row i of q_len_b sees seq_lens[b] -
 *                                (q_len_b - 1 - i) slots; rows beyond the first max_q_len add nothing.  NULL: one row per sequence
 *   decay                        >= 0, finite; 0: weights_in is not read
 *   weights_in / weights_out     [B][stride] f32, stride >= max_seq_len; weights_in may be NULL (zeros) or weights_out itself
 * Slots at or beyond seq_lens[b] keep what weights_out held.  seq_lens[b] < 0, beyond the block table or beyond stride ->
 * GVA_ERR_SEQ_LEN, the sequence is skipped; a slot whose page is bad gets decay * weights_in.  Any cache type. */
int gva_attention_weights(gva_handle *h, const gva_cache *cache, const float *q_abs, const float *lse, const int32_t *cu_q,
                          const int32_t *seq_lens, float decay, const float *weights_in, float *weights_out, int stride, int B,
                          int max_q_len, int max_seq_len, int32_t *dev_status, void *stream);
int gva_q4_attention_weights(gva_handle *h, const gva_q4_cache *cache, const float *q_abs, const float *lse, const int32_t *cu_q,
                             const int32_t *seq_lens, float decay, const float *weights_in, float *weights_out, int stride, int B,
                             int max_q_len, int max_seq_len, int32_t *dev_status, void *stream);

/* Eviction: of sequence b's seq_lens[b] tokens the n = min(keep[b], seq_lens[b]) first in this order stay -- tokens at
 * positions < sinks or >= next_pos[b] - recent before all others (as if their weight were +inf), then by weight from large
 * to small (NaN counts as -inf), then by slot from low to high.  Survivors in slots below n stay where they are; the i-th
 * survivor behind them moves to the i-th slot below n that has become free, rows bit for bit.  The order of tokens in the
 * cache carries no meaning (keys are rotated already), so no more than that is moved; afterwards the sequence has n tokens
 * in slots 0 .. n - 1 and goes on growing with gva_append_cache_at / gva_q4_append (slot n, its own position).
 *   weights_in / weights_out       [B][stride] f32, as from gva_attention_weights; stride >= max_seq_len
 *   positions_in / positions_out   [B][stride] i32: position of the token in each slot; positions_in NULL: its slot.  Each
 *                                  pair may be one buffer or two that do not overlap
 *                                  for slots t < seq_lens[b] the outputs get what now is in the slot, 0 and -1 for t >= n;
 *                                  slots at or beyond seq_lens[b] are left as they were
 *   keep [B] i32, next_pos [B] i32 (position of the sequence's next token; NULL if recent = 0)
 *   new_lens [B] i32               n; may be seq_lens itself
 *   max_seq_len                    upper bound on seq_lens[] (here a longer sequence is an error), 2^30 at most
 *   workspace                      gva_evict_workspace_bytes(h, B, max_seq_len) bytes, 256-byte aligned
 * Pages must belong to one sequence only.  keep[b] < 0 or a bad length -> GVA_ERR_SEQ_LEN, a bad page in the live range of a
 * sequence that would lose tokens -> GVA_ERR_BAD_PAGE: that sequence stays as it is (a bad length: its outputs too), with
 * new_lens[b] = seq_lens[b].  Any cache type. */
size_t gva_evict_workspace_bytes(const gva_handle *h, int B, int max_seq_len);
int gva_evict(gva_handle *h, const gva_cache *cache, const float *weights_in, const int32_t *positions_in, const int32_t *seq_lens,
              const int32_t *keep, const int32_t *next_pos, int sinks, int recent, float *weights_out, int32_t *positions_out,
              int32_t *new_lens, int stride, void *workspace, size_t workspace_bytes, int B, int max_seq_len, int32_t *dev_status,
              void *stream);
int gva_q4_evict(gva_handle *h, const gva_q4_cache *cache, const float *weights_in, const int32_t *positions_in, const int32_t *seq_lens,
                 const int32_t *keep, const int32_t *next_pos, int sinks, int recent, float *weights_out, int32_t *positions_out,
                 int32_t *new_lens, int stride, void *workspace, size_t workspace_bytes, int B, int max_seq_len, int32_t *dev_status,
                 void *stream);

/* ---- A step with drafted tokens: pages and slots, rows by slot map, attention of a tree, commit -----------------------
 * (Not in the paper, whose steps add one token: this library's calls for serving programs that draft several continuations of
 * every sequence as a tree, look at all of them in one step and keep the path the model agrees with.)  One step in order:
 *   gva_assign_pages -> gva_tree_masks -> gva_absorb_query(q_pos = positions) -> (its queries to bf16) -> gva_append_rows -> gva_decode_tree ->
 *   (its output to f32) -> gva_project_out and the rest of the model -> gva_tree_commit;
 * the two conversions are the caller's, and over an f32 cache there are none: gva_decode_tree takes and gives 16-bit numbers where its
 * neighbours take and give f32 (what that costs is said there);
 * the first and gqa_append serve single tokens and prompts as well.  All of them want the handle's device to be the current
 * one (GVA_ERR_INVALID_ARG otherwise), use no state of the handle on the device, and may be captured into CUDA graphs and
 * replayed; calls on different streams may overlap as long as they share no workspace, no output and no page that one of them
 * writes.  B is 8192 at most; num_pages * page_size is below 2^31. */

/* Pages for the tokens that sequences are about to get, pages back from those that need fewer, and a position and a slot for every
 * new row.  The free pages are a ring of num_pages entries: free_in / free_out [2] = (entry of the first free page, how many there
 * are); pages are taken from its front in the order of sequences and returned to its end.
 *   used     [B] i32   tokens that sequence b holds
 *   want     [B] i32   tokens it is to have room for: used + new rows; fewer than used (0 once it is done) returns its pages
 *   pages_in / pages_out [B] i32   pages in its row of the block table, before and after: ceil(want / page_size) afterwards
 *   block_table [B][max_pages_per_seq]   entries pages_in[b] and on are filled in for pages taken; nothing else in it changes
 *   new_lens [B]       want[b], or used[b] where the sequence was not served
 *   cu_q     [B + 1]   rows cu_q[b] .. cu_q[b+1] - 1 are the new tokens of b, max(want - used, 0) of them
 *   positions, slots [max_rows]   of every row: its position used[b] + i, and its place page * page_size + position % page_size
 *                      (-1 if that page is none of the pool: GVA_ERR_BAD_PAGE, the row will not be cached).  Rows at or beyond cu_q[B] are left as they were
 * pages_out may be pages_in, new_lens may be used, free_out may be free_in; nothing else overlaps.
 * Sequences that grow are served in order as long as free pages and rows suffice: the first that does not fit, and all growing
 * ones after it, stay as they are (GVA_ERR_NO_ROOM with the index of one of them).  Pages returned by a call are there for the next one.
 * used < 0, want < 0, pages_in outside [0, max_pages_per_seq], used beyond those pages or want beyond the block table -> GVA_ERR_SEQ_LEN,
 * the sequence stays as it is.  A ring state outside its range -> GVA_ERR_BAD_PAGE, everything stays as it is; more pages returned
 * than the ring has room for -> GVA_ERR_BAD_PAGE, those beyond it are lost; a returned page that is none of the pool -> GVA_ERR_BAD_PAGE, it
 * is lost too.  Pages must belong to one sequence only. */
int gva_assign_pages(gva_handle *h, const int32_t *used, const int32_t *want, const int32_t *pages_in, int32_t *pages_out, int32_t *block_table,
                     int max_pages_per_seq, int num_pages, int32_t *free_ring, const int32_t *free_in, int32_t *free_out, int32_t *new_lens,
                     int32_t *cu_q, int32_t *positions, int32_t *slots, int max_rows, int B, int32_t *dev_status, void *stream);

/* What the nodes of trees see of one another.  Row cu_q[b] + i is node i of sequence b's tree; its parent is a node before it, or
 * -1: a first token behind the context.
 *   parents   [rows] i32   number of the parent within the tree, below the node's own; or -1
 *   mask      [rows][mask_words] u32   bit j of a row (bit j % 32 of word j / 32) is set iff node j is the row's node or one of its ancestors
 *   positions [rows] i32 or NULL   ctx_lens[b] + number of ancestors
 * mask_words >= ceil(max_q_len / 32), 8 at most; max_q_len = nodes of a tree at most, 256 at most.  A tree with a bad parent or more
 * than max_q_len nodes -> GVA_ERR_TREE, its rows are left as they were. */
int gva_tree_masks(gva_handle *h, const int32_t *parents, const int32_t *cu_q, const int32_t *ctx_lens, uint32_t *mask, int mask_words,
                   int32_t *positions, int B, int max_q_len, int32_t *dev_status, void *stream);

/* How far a rotation turns: pair i of d_rot / 2 by position * f_i, with f_i from base^(-2 i / d_rot):
 *   GVA_ROPE_PLAIN    f_i
 *   GVA_ROPE_LINEAR   f_i / factor                                  (positions closer together)
 *   GVA_ROPE_BASE     with base * factor^(d_rot / (d_rot - 2)) for base: the slowest pair by 1 / factor, the fastest as it was
 *   GVA_ROPE_PARTS    f_i (g + (1 - g) / factor), g = (original_len f_i / 2 pi - low) / (high - low) held to [0, 1]: pairs that turn
 *                     more than `high` times over the original context stay, those below `low` turns are divided
 * Pair i is elements (2 i, 2 i + 1) (GVA_ROPE_PAIRS) or (i, i + d_rot / 2) (GVA_ROPE_HALVES) of the first d_rot; what is rotated is
 * multiplied by magnitude.  factor >= 1 (unused with PLAIN); original_len > 0 and 0 <= low < high with PARTS, unused otherwise. */
typedef enum { GVA_ROPE_PAIRS = 0, GVA_ROPE_HALVES = 1 } gva_rope_layout;
typedef enum { GVA_ROPE_PLAIN = 0, GVA_ROPE_LINEAR = 1, GVA_ROPE_BASE = 2, GVA_ROPE_PARTS = 3 } gva_rope_scaling;
typedef struct {
    int32_t layout;        /* gva_rope_layout                                                            */
    int32_t d_rot;         /* elements of a head that turn, even                                         */
    int32_t scaling;       /* gva_rope_scaling                                                           */
    int32_t original_len;  /* context that PARTS counts turns over                                       */
    double base, factor, low, high;
    float magnitude;       /* 1                                                                          */
    int32_t reserved;      /* set to 0                                                                   */
} gva_rope;
/* [host] The f_i of a rotation: d_rot / 2 numbers. */
int gva_rope_frequencies(const gva_rope *rope, double *inv_freq);
/* [host] The rotation of the positional slice, for every call on this handle from now on that rotates one (absorb, appends of every kind,
 * the projections, the fused steps); after gva_create it is PAIRS, PLAIN with cfg.rope_base.  d_rot = cfg.d_r, PAIRS and magnitude 1 only
 * (GVA_ERR_UNSUPPORTED otherwise).  Calls that were captured before keep the rotation they were captured with. */
int gva_set_rope(gva_handle *h, const gva_rope *rope);
/* [host] The rotation of gqa_append on this handle; after gva_create it is PAIRS, PLAIN with cfg.rope_base over the whole head.
 * d_rot a multiple of 8, cfg.d_v at most (GVA_ERR_UNSUPPORTED otherwise). */
int gqa_set_rope(gva_handle *h, const gva_rope *rope);

/* Rows of the matched GQA cache by slot map: keys are rotated to their positions and written with their values, queries are
 * rotated for gqa_decode.  Any mixture of sequences, of single tokens and prompts.
 *   q [n][H][d_h], k_new, v_new [n][G][d_h] f32   with q_stride, k_stride, v_stride elements from row to row (multiples of 4, so that one
 *                      packed projection [n][H + 2 G][d_h] serves all three); q and q_out may both be NULL
 *   pos, slots [n] i32 position and place page * page_size + slot of every row; slots < 0: a padded row, of which nothing is cached
 *   q_out [n][H][d_h] f32   rotated queries of all rows, padded ones too; may be q where q_stride = H d_h
 * The angle is reduced to a fraction of a turn in fp64, sine and cosine are f32, and so are the two products and the sum of an element;
 * keys and values are rounded once to the cache dtype (nearest even; e4m3 saturates).  All pointers are 16-byte aligned
 * (pos and slots 4).  A slot beyond the pool -> GVA_ERR_BAD_PAGE, pos < 0 with a slot -> GVA_ERR_SEQ_LEN, each with the row's
 * number (2^23 - 1 from there on) in the place of a sequence's: that row is not cached.  Two rows with the same slot leave either's elements.  cache->block_table
 * and max_pages_per_seq are not used. */
int gqa_append(gva_handle *h, const gqa_cache *cache, const float *q, int64_t q_stride, const float *k_new, int64_t k_stride,
               const float *v_new, int64_t v_stride, const int32_t *pos, const int32_t *slots, float *q_out, int n,
               int32_t *dev_status, void *stream);

/* Rows of the GVA cache by slot map, any cache type: v_new [n][G][d_v], kr_new [n][d_r] f32 as gva_append_chunk takes them, pos, slots
 * and errors as gqa_append.  A row is bit for bit what gva_append_cache_at writes for that slot and position. */
int gva_append_rows(gva_handle *h, const gva_cache *cache, const float *v_new, const float *kr_new, const int32_t *pos, const int32_t *slots,
                    int n, int32_t *dev_status, void *stream);

/* Attention of drafted tokens over the cache, which already holds them: sequence b has ctx_lens[b] tokens of context in slots
 * 0 .. ctx - 1 and its n_b = cu_q[b+1] - cu_q[b] nodes in slots ctx .. ctx + n_b - 1.  Node i sees the whole context and those nodes j whose
 * bit is set in its row of the mask (gva_tree_masks, or any other mask: a chain, a prompt's causal order, none of the nodes).
 *   q    [n_q][H][d_v+d_r]   absorbed queries with their rotated positional slice; bf16, or f32 over an f32 cache
 *   mask [n_q][mask_words] u32, mask_words >= ceil(max_q_len / 32); bits at or beyond n_b are ignored
 *   out  [n_q][H][d_v]       of q's type: rounded once.  A row that sees nothing gives 0
 *   lse  [n_q][H] f32 or NULL   natural logarithm; -inf for a row that sees nothing
 *   n_q                      rows that q, mask, out and lse hold: at least cu_q[B]
 *   max_q_len, max_seq_len   upper bounds on n_b (256 at most) and on ctx_lens[b] + n_b (2^30 at most)
 *   num_splits               0: all sequences' tiles in a row are cut into equal ranges; n: every 32 nodes' tiles into n ranges (64 at most)
 * Over a bf16 cache the products are taken of the bf16 numbers as they are, accumulated in f32; softmax weights enter the value product
 * rounded to bf16 (2^-8 at most, as the output; their sum is taken before), everything else is f32: over a thousand tokens and more the output is
 * as far off as its own rounding makes it (1.7e-3 of its size), over a hundred 1.1 times.  Over e4m3 and f32 caches all is f32 but the type of
 * queries and output; these caches are served on CUDA cores (1 M tokens of 80, 16 nodes: 12.3 ms, over bf16 0.16 ms).
 * That is the error for the queries as they are given.  Rounding f32 queries to bf16 is one of its own, 2^-8 sum |q k| scale of a score at
 * most: with queries of 1, 5 and 30 times the unit scale outputs were 2.5e-3, 4.4e-3 and 1.0e-2 of their size (3e-3, 4e-2 and 2.4e-1 of a
 * unit at most) from those of f32 queries.  The calls that take f32 queries (gva_decode_tokens and gva_decode_multi for
 * chains, this one over an f32 cache) stay within 2e-2 of a unit at any scale.
 * Bitwise reproducible for fixed arguments.  What is cached for a node does not reach rows that do not see it, not even infinities and NaN;
 * a row that sees a node with an infinity or NaN among a group's values has NaN in the heads of that group, in those elements or in all.
 * n_b < 0 or > max_q_len, rows outside [0, n_q), ctx_lens[b] < 0, or ctx_lens[b] + n_b beyond max_seq_len or the block table -> GVA_ERR_SEQ_LEN, the
 * sequence's rows are left as they were; tokens of a page outside the pool count as absent (GVA_ERR_BAD_PAGE).  Rows at or beyond cu_q[B] are left as they were.
 * Workspace: at least gva_decode_tree_workspace_bytes(...) bytes, 256-byte aligned: a record of 128 rows x G for every 32 nodes of every
 * sequence and some more (32 sequences of 16 narrow nodes 9 MB; 256 of 64 wide ones 282 MB). */
size_t gva_decode_tree_workspace_bytes(const gva_handle *h, int B, int n_q, int max_q_len, int max_seq_len, int num_splits);
int gva_decode_tree(gva_handle *h, const gva_cache *cache, const void *q, const uint32_t *mask, int mask_words, const int32_t *cu_q,
                    const int32_t *ctx_lens, void *out, float *lse, void *workspace, size_t workspace_bytes, int B, int n_q, int max_q_len,
                    int max_seq_len, int num_splits, int32_t *dev_status, void *stream);

/* The drafts that the model agrees with become part of their sequences.  Node 0 of a tree is the token that was chosen last, so it stays; of a
 * node that stays the first child whose token is the one chosen after it stays too.
 *   parents [rows] as gva_tree_masks;  tokens [rows] i32 the drafted tokens;  chosen [rows] i32 what the model says after each node
 *   path     [rows]   row cu_q[b] + k: the k-th node that stays (0 first), -1 behind the last
 *   new_lens [B]      ctx_lens[b] + number of nodes that stay; may be ctx_lens
 *   last     [B]      the token chosen after the last of them (the next tree's node 0), -1 for a sequence without nodes
 * Their rows move to slots ctx, ctx + 1, ... bit for bit (any cache type), so that slots are positions again; the slots behind them
 * hold what is left of the tree and are the next append's.  A bad tree (see gva_tree_masks) -> GVA_ERR_TREE, ctx_lens[b] < 0 or a tree beyond
 * the block table -> GVA_ERR_SEQ_LEN, a bad page among the rows that move -> GVA_ERR_BAD_PAGE: nothing of that sequence moves, new_lens[b] =
 * ctx_lens[b], last[b] = -1 and its path is -1. */
int gva_tree_commit(gva_handle *h, const gva_cache *cache, const int32_t *parents, const int32_t *tokens, const int32_t *chosen, const int32_t *cu_q,
                    const int32_t *ctx_lens, int32_t *path, int32_t *new_lens, int32_t *last, int B, int max_q_len, int32_t *dev_status, void *stream);

/* Geometry of the most recent gva_decode / gqa_decode launch on this handle (reporting only):
 * number of split-KV partitions launched (thread blocks of the decode kernel). */
int gva_last_num_splits(const gva_handle *h);
/* 1 = CUDA-core (FMA) kernel, 2 = tensor-core (MMA) kernel, 0 = none yet. */
int gva_last_kernel(const gva_handle *h);
/* Tokens per tile of the kernel chosen by the last launch (the unit in which ranges are cut). */
int gva_last_tile_tokens(const gva_handle *h);

const char *gva_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* GVA_H_ */
