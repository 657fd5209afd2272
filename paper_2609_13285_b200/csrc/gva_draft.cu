// Host side of the calls around a step with drafted tokens (include/gva.h): pages and slots, rows by slot map with their
// rotation, attention of a tree, and its commit.  As in gva_api.cu, nothing here allocates device memory or synchronises.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "gva_pages.cuh"
#include "gva_rows.cuh"
#include "gva_tree_mma.cuh"
#include "gva_handle.cuh"

using namespace gva;

namespace {
inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

int rope_status(const gva_rope *r) {
    if (!r || (r->layout != GVA_ROPE_PAIRS && r->layout != GVA_ROPE_HALVES) || r->scaling < GVA_ROPE_PLAIN || r->scaling > GVA_ROPE_PARTS)
        return GVA_ERR_INVALID_ARG;
    if (r->d_rot <= 0 || r->d_rot % 2 != 0 || !(r->base > 1.0) || !std::isfinite(r->base) || !(r->magnitude > 0.f) || !std::isfinite(r->magnitude))
        return GVA_ERR_INVALID_ARG;
    if (r->scaling != GVA_ROPE_PLAIN && (!(r->factor >= 1.0) || !std::isfinite(r->factor))) return GVA_ERR_INVALID_ARG;
    if (r->scaling == GVA_ROPE_BASE && r->d_rot < 4) return GVA_ERR_INVALID_ARG;
    if (r->scaling == GVA_ROPE_PARTS && (r->original_len <= 0 || !(r->low >= 0.0) || !(r->high > r->low) || !std::isfinite(r->high)))
        return GVA_ERR_INVALID_ARG;
    return GVA_OK;
}
int check_gqa(const gva_handle *h, const gqa_cache *cache) {
    if (!h || !cache || !cache->k_pool || !cache->v_pool || cache->num_pages <= 0) return GVA_ERR_INVALID_ARG;
    if (!aligned(cache->k_pool, 16) || !aligned(cache->v_pool, 16)) return GVA_ERR_INVALID_ARG;
    return check_device(h);
}
// Slots are numbers of 32 bits.
bool slots_fit(const gva_handle *h, int num_pages) { return (long long)num_pages * h->cfg.page_size <= 0x7fffffffll; }
int element_bytes(const gva_handle *h) { return h->cfg.cache_dtype == GVA_E4M3 ? 1 : h->cfg.cache_dtype == GVA_BF16 ? 2 : 4; }
uint32_t inverse_of(int per_row) { return (uint32_t)(((1ull << 32) + per_row - 1) / per_row); }

// Rows of a block: as few as still fill the GPU a few times over, `most` at most.
int rows_per_block(const gva_handle *h, int n, int most) { return (int)std::min<long long>(most, std::max<long long>(1, n / (4 * h->sm_count))); }

// ---- the tree's launch ----
struct TreePlan {
    int tile, strips, ranges, num_splits;
    long long records;
    size_t smem, rec_o, rec_ml, total;       // shared memory of a block; workspace: entries, records, their maxima and sums
};
int tree_status(const gva_handle *h, int B, int n_q, int max_q_len, int max_seq_len, int num_splits) {
    if (!h || B < 0 || n_q < 0 || max_q_len < 0 || max_seq_len < 0 || num_splits < 0) return GVA_ERR_INVALID_ARG;
    if (B > 8192 || max_q_len > kTreeMost || num_splits > 64 || max_seq_len > (1 << 30)) return GVA_ERR_UNSUPPORTED;
    const long long strips = ceil_div(max_q_len, kStripNodes) * B;
    if (strips * std::max<long long>(ceil_div(max_seq_len, kTreeFmaTile), num_splits) >= (1ll << 30)) return GVA_ERR_UNSUPPORTED;   // (tiles are counted in 32 bits)
    return GVA_OK;
}
TreePlan tree_plan(const gva_handle *h, int B, int max_q_len, int max_seq_len, int num_splits) {
    const gva_config &c = h->cfg;
    TreePlan t;
    t.strips = (int)std::max<long long>(1, ceil_div(max_q_len, kStripNodes));
    t.tile = c.cache_dtype == GVA_BF16 ? tree_mma_tile(c.d_v) : kTreeFmaTile;
    const long long tiles = std::max<long long>(1, ceil_div(max_seq_len, t.tile)), all = (long long)std::max(B, 1) * t.strips;
    // Short sequences: one piece per strip, which writes its result itself -- there is nothing to merge.  us, in one piece / in ranges, 8 nodes:
    //   narrow heads, 500 tokens (4 tiles)  1 sequence 10.5 / 12.0   8: 10.8 / 13.7   64: 18.9 / 26.9;   800 tokens (7)   12.6 / 13.3   13.0 / 17.8   23.6 / 32.3
    //   wide heads, 200 tokens (4 tiles)    1 sequence 13.0 / 16.3   8: 13.7 / 18.7   64: 43.3 / 53.7;   800 tokens (13)  16.3 / 16.3   17.1 / 26.5   58.5 / 66.6
    // Four tiles stay clear of the border, which one long sequence among short ones moves down.  The bound decides, not the lengths: a call
    // captured with a larger one takes ranges.
    t.num_splits = num_splits > 0 ? num_splits : tiles <= 4 ? 1 : 0;
    num_splits = t.num_splits;
    const bool mma = c.cache_dtype == GVA_BF16;
    const TreeMma k = tree_mma(c);
    const int room = std::max(1, h->sm_count / c.G);
    t.ranges = (int)std::min<long long>(all * (num_splits > 0 ? num_splits : tiles), room);
    t.records = num_splits == 1 ? 0 : num_splits > 0 ? all * num_splits : t.ranges + all;
    // (never more blocks on an SM than its 512 columns of tensor memory serve: one)
    t.smem = mma ? std::max(k.fixed + (size_t)B * 4, (size_t)h->smem_per_sm / 2) : tree_fma_smem(B, c.d_v, c.d_r);
    t.rec_o = t.num_splits == 1 ? 0 : align_up((size_t)all * sizeof(int4), 256);
    t.rec_ml = t.rec_o + align_up((size_t)t.records * c.G * kStripRows * c.d_v * 4, 256);
    t.total = std::max<size_t>(256, t.rec_ml + align_up((size_t)t.records * c.G * kStripRows * 2 * 4, 256));
    return t;
}
using TreeFmaFn = void (*)(TreeParams, int);
TreeFmaFn tree_fma(const gva_config &c) {
    const bool wide = c.d_v == 128;
    if (c.cache_dtype == GVA_F32) return wide ? tree_fma_kernel<float, float, 128> : tree_fma_kernel<float, float, 64>;
    return wide ? tree_fma_kernel<uint8_t, __nv_bfloat16, 128> : tree_fma_kernel<uint8_t, __nv_bfloat16, 64>;
}
}  // namespace

extern "C" {

int gva_rope_frequencies(const gva_rope *rope, double *inv_freq) {
    const int rc = rope_status(rope);
    if (rc != GVA_OK) return rc;
    if (!inv_freq) return GVA_ERR_INVALID_ARG;
    rope_frequencies(*rope, inv_freq);
    return GVA_OK;
}

int gva_set_rope(gva_handle *h, const gva_rope *rope) {
    if (!h) return GVA_ERR_INVALID_ARG;
    const int rc = rope_status(rope);
    if (rc != GVA_OK) return rc;
    if (rope->layout != GVA_ROPE_PAIRS || rope->d_rot != h->cfg.d_r || rope->magnitude != 1.f) return GVA_ERR_UNSUPPORTED;
    rope_frequencies(*rope, h->rope.inv_freq);
    return GVA_OK;
}

int gqa_set_rope(gva_handle *h, const gva_rope *rope) {
    if (!h) return GVA_ERR_INVALID_ARG;
    const int rc = rope_status(rope);
    if (rc != GVA_OK) return rc;
    if (rope->d_rot % 8 != 0 || rope->d_rot > h->cfg.d_v) return GVA_ERR_UNSUPPORTED;
    h->head_rope = head_rope(*rope);
    return GVA_OK;
}

int gqa_append(gva_handle *h, const gqa_cache *cache, const float *q, int64_t q_stride, const float *k_new, int64_t k_stride,
               const float *v_new, int64_t v_stride, const int32_t *pos, const int32_t *slots, float *q_out, int n,
               int32_t *dev_status, void *stream) {
    const int rc = check_gqa(h, cache);
    if (rc != GVA_OK) return rc;
    if (n < 0) return GVA_ERR_INVALID_ARG;
    if (n == 0) return GVA_OK;
    const gva_config &c = h->cfg;
    if (!k_new || !v_new || !pos || !slots || (q != nullptr) != (q_out != nullptr)) return GVA_ERR_INVALID_ARG;
    if (k_stride < (int64_t)c.G * c.d_v || v_stride < (int64_t)c.G * c.d_v || (q && q_stride < (int64_t)c.H * c.d_v)) return GVA_ERR_INVALID_ARG;
    if (k_stride % 4 != 0 || v_stride % 4 != 0 || (q && q_stride % 4 != 0)) return GVA_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(q_out, 16) || !aligned(pos, 4) || !aligned(slots, 4))
        return GVA_ERR_INVALID_ARG;
    if (q == q_out && q && q_stride != (int64_t)c.H * c.d_v) return GVA_ERR_INVALID_ARG;
    if (!slots_fit(h, cache->num_pages)) return GVA_ERR_UNSUPPORTED;
    GqaAppendParams p;
    std::memset(&p, 0, sizeof(p));
    p.k_pool = cache->k_pool; p.v_pool = cache->v_pool;
    p.q = q; p.k_new = k_new; p.v_new = v_new;
    p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride;
    p.q_out = q_out; p.pos = pos; p.slots = slots; p.dev_status = dev_status;
    p.n = n; p.H = q ? c.H : 0; p.G = c.G; p.d = c.d_v; p.P = c.page_size; p.num_pages = cache->num_pages;
    p.rows = rows_per_block(h, n, kGqaRows);
    p.per_row_inv = inverse_of((p.H + 2 * c.G) * c.d_v / 8);
    auto fn = c.cache_dtype == GVA_E4M3 ? gqa_append_kernel<uint8_t> : c.cache_dtype == GVA_BF16 ? gqa_append_kernel<__nv_bfloat16> : gqa_append_kernel<float>;
    return launched(launch_pdl(fn, dim3((unsigned)ceil_div(n, p.rows)), dim3(kRowsThreads), 0, static_cast<cudaStream_t>(stream), p, h->head_rope));
}

int gva_append_rows(gva_handle *h, const gva_cache *cache, const float *v_new, const float *kr_new, const int32_t *pos, const int32_t *slots,
                    int n, int32_t *dev_status, void *stream) {
    const int rc = check_plain(h, cache);
    if (rc != GVA_OK) return rc;
    if (n < 0) return GVA_ERR_INVALID_ARG;
    if (n == 0) return GVA_OK;
    const gva_config &c = h->cfg;
    if (!v_new || (c.d_r > 0 && !kr_new) || !pos || !slots || !aligned(v_new, 4) || !aligned(kr_new, 4) || !aligned(pos, 4) || !aligned(slots, 4))
        return GVA_ERR_INVALID_ARG;
    if (!slots_fit(h, cache->num_pages)) return GVA_ERR_UNSUPPORTED;
    AppendRowsParams p;
    std::memset(&p, 0, sizeof(p));
    p.v_pool = cache->v_pool; p.kr_pool = cache->kr_pool;
    p.v_new = v_new; p.kr_new = kr_new; p.pos = pos; p.slots = slots; p.dev_status = dev_status;
    p.n = n; p.G = c.G; p.d_v = c.d_v; p.d_r = c.d_r; p.P = c.page_size; p.num_pages = cache->num_pages;
    p.rows = rows_per_block(h, n, 16);
    p.per_row_inv = inverse_of(c.G * c.d_v / 8);
    p.vec = aligned(v_new, 16) ? 1 : 0;
    auto fn = c.cache_dtype == GVA_E4M3 ? append_rows_kernel<uint8_t> : c.cache_dtype == GVA_BF16 ? append_rows_kernel<__nv_bfloat16> : append_rows_kernel<float>;
    return launched(launch_pdl(fn, dim3((unsigned)ceil_div(n, p.rows)), dim3(kRowsThreads), 0, static_cast<cudaStream_t>(stream), p, h->rope));
}

int gva_assign_pages(gva_handle *h, const int32_t *used, const int32_t *want, const int32_t *pages_in, int32_t *pages_out, int32_t *block_table,
                     int max_pages_per_seq, int num_pages, int32_t *free_ring, const int32_t *free_in, int32_t *free_out, int32_t *new_lens,
                     int32_t *cu_q, int32_t *positions, int32_t *slots, int max_rows, int B, int32_t *dev_status, void *stream) {
    if (!h || B < 0 || max_rows < 0 || max_pages_per_seq <= 0 || num_pages <= 0) return GVA_ERR_INVALID_ARG;
    if (!free_ring || !free_in || !free_out || !cu_q) return GVA_ERR_INVALID_ARG;
    if (B > 0 && (!used || !want || !pages_in || !pages_out || !block_table || !new_lens)) return GVA_ERR_INVALID_ARG;
    if (max_rows > 0 && (!positions || !slots)) return GVA_ERR_INVALID_ARG;
    for (const void *x : {(const void *)used, (const void *)want, (const void *)pages_in, (const void *)pages_out, (const void *)block_table, (const void *)free_ring,
                          (const void *)free_in, (const void *)free_out, (const void *)new_lens, (const void *)cu_q, (const void *)positions, (const void *)slots})
        if (!aligned(x, 4)) return GVA_ERR_INVALID_ARG;
    if (B > kAssignItems * 1024 || !slots_fit(h, num_pages)) return GVA_ERR_UNSUPPORTED;
    int rc = check_device(h);
    if (rc != GVA_OK) return rc;
    AssignParams p;
    std::memset(&p, 0, sizeof(p));
    p.used = used; p.want = want; p.pages_in = pages_in; p.pages_out = pages_out; p.block_table = block_table; p.ring = free_ring;
    p.free_in = free_in; p.free_out = free_out; p.new_lens = new_lens; p.cu_q = cu_q; p.positions = positions; p.slots = slots;
    p.dev_status = dev_status;
    p.max_pages = max_pages_per_seq; p.num_pages = num_pages; p.max_rows = max_rows; p.B = B; p.P = h->cfg.page_size;
    // Up to 8192 rows the kernel's threads have one row each, in a cluster of up to eight blocks; more rows get a kernel of their own
    // (in the cluster and apart, us: 5000 rows of 256 trees 6.8 and 12.3, 0.2 M rows of 48 prompts 33 and 9.3).
    p.rows_here = max_rows <= 8192 ? 1 : 0;
    // As many threads as rows, or as pages taken (at least), up to the cluster's.  How many pages come back is not known here: 8769 of them
    // from 111 of 1000 sequences take 14.1 us in the one block of a call for 1000 rows, 8.2 in the eight of one for 8000.
    const int work = (int)std::max<long long>(B, p.rows_here ? max_rows : std::max<long long>(1024, ceil_div(max_rows, p.P)));
    const int threads = work <= 128 ? 128 : work <= 256 ? 256 : work <= 512 ? 512 : 1024;
    const int blocks = work <= 1024 ? 1 : work <= 2048 ? 2 : work <= 4096 ? 4 : 8;
    const size_t smem = (size_t)6 * B * 4;
    void (*const fn)(AssignParams) = B <= threads ? assign_pages_kernel<1> : assign_pages_kernel<kAssignItems>;
    rc = allow_smem(h, reinterpret_cast<const void *>(fn), smem);
    if (rc != GVA_OK) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = blocks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    rc = launched(cudaLaunchKernelEx(&cfg, fn, p));
    if (rc != GVA_OK || p.rows_here) return rc;
    return launched(launch_pdl(assign_rows_kernel, dim3((unsigned)ceil_div(max_rows, kAssignRows)), dim3(kAssignRowThreads), 0, cfg.stream, p));
}

int gva_tree_masks(gva_handle *h, const int32_t *parents, const int32_t *cu_q, const int32_t *ctx_lens, uint32_t *mask, int mask_words,
                   int32_t *positions, int B, int max_q_len, int32_t *dev_status, void *stream) {
    if (!h || B < 0 || max_q_len < 0 || mask_words < 0) return GVA_ERR_INVALID_ARG;
    if (B == 0 || max_q_len == 0) return GVA_OK;
    if (!parents || !cu_q || !mask || (positions && !ctx_lens) || mask_words * 32ll < max_q_len) return GVA_ERR_INVALID_ARG;
    if (!aligned(parents, 4) || !aligned(cu_q, 4) || !aligned(ctx_lens, 4) || !aligned(mask, 4) || !aligned(positions, 4)) return GVA_ERR_INVALID_ARG;
    if (B > 8192 || max_q_len > kTreeMost || mask_words > kTreeMost / 32) return GVA_ERR_UNSUPPORTED;
    const int rc = check_device(h);
    if (rc != GVA_OK) return rc;
    const TreeMaskParams p{parents, cu_q, ctx_lens, mask, positions, dev_status, mask_words, max_q_len};
    const int threads = max_q_len <= 32 ? 32 : max_q_len <= 64 ? 64 : max_q_len <= 128 ? 128 : 256;
    return launched(launch_pdl(tree_masks_kernel, dim3(B), dim3(threads), 0, static_cast<cudaStream_t>(stream), p));
}

size_t gva_decode_tree_workspace_bytes(const gva_handle *h, int B, int n_q, int max_q_len, int max_seq_len, int num_splits) {
    if (tree_status(h, B, n_q, max_q_len, max_seq_len, num_splits) != GVA_OK) return 0;
    return tree_plan(h, B, max_q_len, max_seq_len, num_splits).total;
}

int gva_decode_tree(gva_handle *h, const gva_cache *cache, const void *q, const uint32_t *mask, int mask_words, const int32_t *cu_q,
                    const int32_t *ctx_lens, void *out, float *lse, void *workspace, size_t workspace_bytes, int B, int n_q, int max_q_len,
                    int max_seq_len, int num_splits, int32_t *dev_status, void *stream) {
    int rc = tree_status(h, B, n_q, max_q_len, max_seq_len, num_splits);
    if (rc == GVA_OK) rc = check_plain(h, cache);
    if (rc != GVA_OK) return rc;
    if (mask_words < 0) return GVA_ERR_INVALID_ARG;
    if (B == 0 || n_q == 0 || max_q_len == 0 || max_seq_len == 0) return GVA_OK;
    if (!q || !mask || !cu_q || !ctx_lens || !out || mask_words * 32ll < max_q_len) return GVA_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(mask, 4) || !aligned(cu_q, 4) || !aligned(ctx_lens, 4) || !aligned(lse, 4)) return GVA_ERR_INVALID_ARG;
    if (h->cfg.cache_dtype == GVA_BF16 && (uint64_t)cache->num_pages * h->cfg.G * h->cfg.page_size >= (1ull << 31)) return GVA_ERR_UNSUPPORTED;
    const TreePlan plan = tree_plan(h, B, max_q_len, max_seq_len, num_splits);
    if (!workspace || workspace_bytes < plan.total) return GVA_ERR_WORKSPACE;
    if (!aligned(workspace, 256)) return GVA_ERR_INVALID_ARG;
    const gva_config &c = h->cfg;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    TreeParams p;
    std::memset(&p, 0, sizeof(p));
    p.q = q; p.mask = mask; p.cu_q = cu_q; p.ctx_lens = ctx_lens; p.block_table = cache->block_table;
    p.v_pool = cache->v_pool; p.kr_pool = cache->kr_pool; p.out = out; p.lse = lse; p.dev_status = dev_status;
    p.entries = reinterpret_cast<int4 *>(ws);
    p.rec_o = reinterpret_cast<float *>(ws + plan.rec_o);
    p.rec_ml = reinterpret_cast<float *>(ws + plan.rec_ml);
    p.B = B; p.H = c.H; p.G = c.G; p.P = c.page_size; p.num_pages = cache->num_pages; p.max_pages = cache->max_pages_per_seq; p.words = mask_words;
    p.n_q = n_q; p.max_q_len = max_q_len; p.max_seq_len = max_seq_len;
    p.tile = plan.tile; p.strips = plan.strips; p.ranges = plan.ranges; p.num_splits = plan.num_splits;
    p.scale_log2 = h->scale * kLog2e;
    if (plan.smem > (size_t)h->smem_optin) return GVA_ERR_UNSUPPORTED;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const dim3 grid(plan.ranges * c.G);
    if (c.cache_dtype == GVA_BF16) {
        const TreeMma k = tree_mma(c);
        CUtensorMap tm_v, tm_k;
        if (!tree_maps(c, h->mma, p, k.drp, &tm_v, &tm_k)) return GVA_ERR_CUDA;
        rc = allow_smem(h, reinterpret_cast<const void *>(k.fn), plan.smem);
        if (rc != GVA_OK) return rc;
        rc = launched(launch_pdl(k.fn, grid, dim3(k.threads), plan.smem, s, p, tm_v, tm_k));
    } else {
        const TreeFmaFn fn = tree_fma(c);
        rc = allow_smem(h, reinterpret_cast<const void *>(fn), plan.smem);
        if (rc != GVA_OK) return rc;
        rc = launched(launch_pdl(fn, grid, dim3(kTreeFmaThreads), plan.smem, s, p, c.d_r));
    }
    if (rc != GVA_OK || plan.num_splits == 1) return rc;
    // Many pieces a strip: a block per node with the pieces side by side; few: a warp per node.  us, side by side / by warps, 4000 tokens:
    //   narrow heads (37 ranges), 8 nodes   1 sequence 13.8 / 17.5   2: 14.1 / 15.3   4: 15.7 / 15.6   5: 20.5 / 20.6   8: 23.3 / 21.6
    //                             32 nodes  1 sequence 16.7 / 20.4   2: 18.1 / 18.8   4: 21.8 / 19.5   5: 29.7 / 26.7   8: 35.0 / 28.8
    //   wide heads (18 ranges), 8 nodes     1 sequence 19.3 / 22.3   2: 21.0 / 23.0   3: 22.2 / 23.5   8: 37.7 / 35.5
    //   narrow, 4 (16) sequences in splits  4 splits 16.4 / 16.1 (30.6 / 26.2)   8: 15.4 / 15.2 (39.7 / 36.7)   16: 19.2 / 20.3 (51.6 / 50.5)
    const bool wide = plan.ranges >= 8 * plan.strips * B || plan.num_splits >= 8;
    const int nodes = std::min(max_q_len, kStripNodes);
    const dim3 merge_grid((unsigned)(B * plan.strips), c.H, wide ? nodes : (nodes + 7) / 8);
#define GVA_MERGE(OT_, DV_) (wide ? tree_merge_kernel<OT_, DV_, true> : tree_merge_kernel<OT_, DV_, false>)
    auto merge = c.cache_dtype == GVA_F32 ? (c.d_v == 64 ? GVA_MERGE(float, 64) : GVA_MERGE(float, 128))
                                          : (c.d_v == 64 ? GVA_MERGE(__nv_bfloat16, 64) : GVA_MERGE(__nv_bfloat16, 128));
#undef GVA_MERGE
    return launched(launch_pdl(merge, merge_grid, dim3(256), 0, s, p));
}

int gva_tree_commit(gva_handle *h, const gva_cache *cache, const int32_t *parents, const int32_t *tokens, const int32_t *chosen, const int32_t *cu_q,
                    const int32_t *ctx_lens, int32_t *path, int32_t *new_lens, int32_t *last, int B, int max_q_len, int32_t *dev_status, void *stream) {
    const int rc = check_plain(h, cache);
    if (rc != GVA_OK) return rc;
    if (B < 0 || max_q_len < 0) return GVA_ERR_INVALID_ARG;
    if (B == 0) return GVA_OK;
    if (!cu_q || !ctx_lens || !new_lens || !last || !parents || !tokens || !chosen || !path) return GVA_ERR_INVALID_ARG;
    if (!aligned(parents, 4) || !aligned(tokens, 4) || !aligned(chosen, 4) || !aligned(cu_q, 4) || !aligned(ctx_lens, 4) || !aligned(path, 4) || !aligned(new_lens, 4) ||
        !aligned(last, 4))
        return GVA_ERR_INVALID_ARG;
    if (B > 8192 || max_q_len > kTreeMost) return GVA_ERR_UNSUPPORTED;
    const gva_config &c = h->cfg;
    TreeCommitParams p;
    std::memset(&p, 0, sizeof(p));
    p.v_pool = static_cast<uint8_t *>(cache->v_pool);
    p.kr_pool = c.d_r > 0 ? static_cast<uint8_t *>(cache->kr_pool) : nullptr;
    p.block_table = cache->block_table; p.parents = parents; p.tokens = tokens; p.chosen = chosen; p.cu_q = cu_q; p.ctx_lens = ctx_lens;
    p.path = path; p.new_lens = new_lens; p.last = last; p.dev_status = dev_status;
    p.v_bytes = c.d_v * element_bytes(h); p.kr_bytes = c.d_r * element_bytes(h);
    p.G = c.G; p.P = c.page_size; p.num_pages = cache->num_pages; p.max_pages = cache->max_pages_per_seq; p.most = max_q_len;
    return launched(launch_pdl(tree_commit_kernel, dim3(B), dim3(kCommitThreads), 0, static_cast<cudaStream_t>(stream), p));
}

}  // extern "C"
