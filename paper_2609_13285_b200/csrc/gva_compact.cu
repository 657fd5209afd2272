// Host side of the calls that keep a cache small (include/gva.h): the 4-bit cache, gathered attention weights, eviction.
// As in gva_api.cu, nothing here allocates device memory or synchronises.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "gva_evict.cuh"
#include "gva_q4_decode.cuh"
#include "gva_weights.cuh"
#include "gva_handle.cuh"

using namespace gva;

namespace {
int check_q4(const gva_handle *h, const gva_q4_cache *cache) {
    if (!h || !cache) return GVA_ERR_INVALID_ARG;
    if (h->cfg.cache_dtype != GVA_BF16) return GVA_ERR_UNSUPPORTED;
    if (!cache->v_pool || !cache->sz_pool || (h->cfg.d_r > 0 && !cache->kr_pool)) return GVA_ERR_INVALID_ARG;
    if (cache->num_pages <= 0 || cache->max_pages_per_seq <= 0) return GVA_ERR_INVALID_ARG;
    if (!aligned(cache->v_pool, 16) || !aligned(cache->sz_pool, 16) || !aligned(cache->kr_pool, 16) || !aligned(cache->block_table, 4))
        return GVA_ERR_INVALID_ARG;
    return check_device(h);
}
Q4Pools q4_pools(const gva_q4_cache *c) {
    return Q4Pools{static_cast<uint8_t *>(c->v_pool), static_cast<__half2 *>(c->sz_pool), static_cast<uint16_t *>(c->kr_pool),
                   c->block_table, c->num_pages, c->max_pages_per_seq};
}
int append_q4(gva_handle *h, const gva_q4_cache *cache, const float *v_new, const float *kr_new, const int32_t *cu_q,
              const int32_t *slot0, const int32_t *pos0, int B, int n_q, int rows, int32_t *dev_status, void *stream) {
    if (!v_new || (h->cfg.d_r > 0 && !kr_new) || !aligned(v_new, 4) || !aligned(kr_new, 4) || !aligned(slot0, 4) || !aligned(pos0, 4))
        return GVA_ERR_INVALID_ARG;
    const gva_config &c = h->cfg;
    AppendQ4Params p;
    std::memset(&p, 0, sizeof(p));
    p.c = q4_pools(cache);
    p.v_new = v_new; p.kr_new = kr_new; p.cu_q = cu_q; p.slot0 = slot0; p.pos0 = pos0;
    p.B = B; p.n_q = n_q; p.G = c.G; p.d_r = c.d_r; p.P = c.page_size; p.rows = rows;
    p.per_row_inv = (uint32_t)(((1u << 20) + c.G * c.d_v / 8 - 1) / (c.G * c.d_v / 8));
    p.vec = aligned(v_new, 16) ? 1 : 0;
    p.dev_status = dev_status;
    return launched(launch_pdl(c.d_v == 64 ? append_q4_kernel<64> : append_q4_kernel<128>, dim3((n_q + rows - 1) / rows), dim3(kAppendQ4Threads), 0,
                               static_cast<cudaStream_t>(stream), p, h->rope));
}

// (lengths may be up to 2^31 - 1: a rounding up in 32 bits would overflow)
inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// ---- 4-bit decode: which kernel, which grid ----
using Q4DecodeFn = void (*)(DecodeParams, Q4Launch);
struct Q4Kernel {
    Q4DecodeFn fn;
    int tile;
    size_t stage;
};
template <int DV, int DR, int TILE>
Q4Kernel q4_kernel_t(int G) {
    constexpr int FEW = q4_consumers(DV, 1), MANY = q4_consumers(DV, 8);
    return Q4Kernel{q4_consumers(DV, G) == FEW ? decode_q4_kernel<DV, DR, TILE, FEW> : decode_q4_kernel<DV, DR, TILE, MANY>, TILE,
                    (size_t)Q4Traits<DV, DR, TILE>::stage_bytes(G)};
}
Q4Kernel q4_kernel(const gva_config &c) {
    const bool t64 = c.page_size % 64 == 0;              // a tile lies in one page
#define GVA_Q4(DV_, DR_) (t64 ? q4_kernel_t<DV_, DR_, 64>(c.G) : q4_kernel_t<DV_, DR_, 32>(c.G))
    if (c.d_v == 64) return c.d_r == 16 ? GVA_Q4(64, 16) : c.d_r == 24 ? GVA_Q4(64, 24) : GVA_Q4(64, 0);
    return c.d_r == 32 ? GVA_Q4(128, 32) : GVA_Q4(128, 0);
#undef GVA_Q4
}
// Ring of up to four slots per team in `room` bytes: a multiple of the teams and of the producers (see produce_tiles).
void ring(int teams, size_t stage, size_t room, int *nstage, int *producers) {
    const int slots = (int)std::min<size_t>(4 * teams, room / stage);
    *nstage = std::max(teams == 1 ? 2 : teams, slots / teams * teams);
    *producers = kQ4Producers;
    while (*nstage % *producers != 0) --*producers;
}
// The launch for B sequences of at most max_seq_len tokens.  num_splits = 0: where every sequence is a few tiles at most, one
// block per sequence, which writes the result itself -- there is nothing to merge; else the balanced partition, one
// block per SM with as many teams as there are tiles for.  num_splits >= 1: blocks of one team, num_splits per sequence.
// One block each against balanced, us, narrow heads (G = 4, d_v = 64): in tiles of 64 tokens 64 x 256 9.2 / 11.6, 64 x 512 12.4 / 12.3,
// 64 x 640 15.0 / 12.7; of 32 64 x 128 9.2 / 11.8, 64 x 256 9.6 / 11.7, 64 x 384 12.3 / 11.8; 200 sequences of 512 15.4 / 19.1 and 17.4 / 20.7.
// Wide heads (G = 8, d_v = 128): 8 x 128 11.5 / 11.9, 8 x 256 16.1 / 12.0, 64 x 128 13.3 / 14.4, 64 x 256 21.4 / 17.2, 200 x 512 39.6 / 46.3:
// there two tiles would be the better border.  The rule goes by max_seq_len, as every launch does: a captured graph that allows for long
// sequences takes the balanced form for short ones too.
struct Q4Plan {
    Q4Kernel k;
    int num_splits, grid, teams, nstage, producers, n_rec;
    size_t smem, rec_o, rec_ml, total;                   // shared memory of a block; workspace: segments, records, maxima and sums
};
Q4Plan q4_plan(const gva_handle *h, int B, int max_seq_len, int num_splits) {
    Q4Plan p;
    p.k = q4_kernel(h->cfg);
    const long long tiles = ceil_div(max_seq_len, p.k.tile);
    p.num_splits = num_splits > 0 ? num_splits : tiles <= (B >= h->sm_count ? 8 : 4) ? 1 : 0;
    if (p.num_splits > 0) {
        p.teams = 1;
        p.grid = B * p.num_splits;
        p.n_rec = p.grid;
    } else {
        p.grid = (int)std::min<long long>(tiles * B, h->sm_count);
        p.teams = (int)std::min<long long>(q4_consumers(h->cfg.d_v, h->cfg.G) / h->cfg.G, std::max(1ll, ceil_div(tiles * B, p.grid)));
        p.n_rec = (p.grid + B) * p.teams;
    }
    // the ring takes what the SM holds (one block per SM) or a third of it
    const size_t room = (p.num_splits > 0 ? (size_t)h->smem_per_sm / 3 : (size_t)h->smem_optin) - (size_t)(B + 1) * 4 - 2048;
    ring(p.teams, p.k.stage, room, &p.nstage, &p.producers);
    p.smem = p.nstage * p.k.stage + Q4Traits<64, 0, 32>::tail_bytes(B, p.nstage);
    p.rec_o = align_up((size_t)B * sizeof(int2), 256);
    p.rec_ml = p.rec_o + align_up((size_t)p.n_rec * h->cfg.H * h->cfg.d_v * 4, 256);
    p.total = p.rec_ml + align_up((size_t)p.n_rec * h->cfg.H * 2 * 4, 256);
    return p;
}

// ---- gathered weights: which kernel ----
struct WeightKernel {
    void (*fn)(WeightParams, WeightLaunch);
    int tile;
    size_t stage;
};
template <int KIND, int DV, int DR, int TILE>
WeightKernel weight_kernel_t(int G, bool multi) {
    return WeightKernel{multi ? weights_mma_kernel<KIND, DV, DR, TILE, true> : weights_mma_kernel<KIND, DV, DR, TILE, false>, TILE,
                        (size_t)WeightTraits<KIND, DV, DR, TILE>::stage_bytes(G)};
}
WeightKernel weight_kernel(int kind, const gva_config &c, bool multi) {
    // a tile lies in one page; the bf16 tile of wide heads is kept to 32 tokens, so that a ring of several fits
    const bool t64 = c.page_size % 64 == 0;
#define GVA_W(KIND_, DV_, DR_) (t64 ? weight_kernel_t<KIND_, DV_, DR_, 64>(c.G, multi) : weight_kernel_t<KIND_, DV_, DR_, 32>(c.G, multi))
#define GVA_W_SHAPES(KIND_) \
    if (c.d_v == 64 && c.d_r == 16) return GVA_W(KIND_, 64, 16); \
    if (c.d_v == 64 && c.d_r == 0) return GVA_W(KIND_, 64, 0)
    if (kind == kCacheQ4) {
        GVA_W_SHAPES(kCacheQ4);
        if (c.d_v == 64) return GVA_W(kCacheQ4, 64, 24);
        return c.d_r == 32 ? GVA_W(kCacheQ4, 128, 32) : GVA_W(kCacheQ4, 128, 0);
    }
    if (kind == kCacheBf16) {
        GVA_W_SHAPES(kCacheBf16);
        if (c.d_v == 64) return GVA_W(kCacheBf16, 64, 24);
        return c.d_r == 32 ? weight_kernel_t<kCacheBf16, 128, 32, 32>(c.G, multi) : weight_kernel_t<kCacheBf16, 128, 0, 32>(c.G, multi);
    }
    if (c.d_v == 64) return c.d_r == 16 ? weight_kernel_t<kCacheE4m3, 64, 16, 64>(c.G, multi) : weight_kernel_t<kCacheE4m3, 64, 0, 64>(c.G, multi);   // pages of 64 k tokens
    return c.d_r == 32 ? weight_kernel_t<kCacheE4m3, 128, 32, 64>(c.G, multi) : weight_kernel_t<kCacheE4m3, 128, 0, 64>(c.G, multi);
#undef GVA_W_SHAPES
#undef GVA_W
}

int attention_weights(gva_handle *h, WeightParams p, int kind, const float *q_abs, const float *lse, const int32_t *cu_q,
                      const int32_t *seq_lens, float decay, const float *weights_in, float *weights_out, int stride, int B,
                      int max_q_len, int max_seq_len, int32_t *dev_status, void *stream) {
    if (B < 0 || max_q_len < 0 || max_seq_len < 0 || stride < 0) return GVA_ERR_INVALID_ARG;
    if (B == 0 || max_seq_len == 0) return GVA_OK;
    if (!q_abs || !lse || !seq_lens || !weights_out || stride < max_seq_len || !(decay >= 0.f) || std::isinf(decay)) return GVA_ERR_INVALID_ARG;
    if (!aligned(q_abs, 16) || !aligned(lse, 4) || !aligned(cu_q, 4) || !aligned(seq_lens, 4) || !aligned(weights_in, 4) || !aligned(weights_out, 4))
        return GVA_ERR_INVALID_ARG;
    if (B > 8192 || B * (ceil_div(stride, 32) + 1) >= (1ll << 30)) return GVA_ERR_UNSUPPORTED;     // (tiles are counted in 32 bits)
    const gva_config &c = h->cfg;
    p.q = q_abs; p.lse = lse; p.cu_q = cu_q; p.seq_lens = seq_lens; p.decay = decay; p.w_in = decay > 0.f ? weights_in : nullptr; p.w_out = weights_out;
    p.stride = stride; p.B = B; p.max_q_len = max_q_len; p.H = c.H; p.G = c.G; p.P = c.page_size;
    p.scale = h->scale;
    p.dev_status = dev_status;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (kind == kCacheF32)
        return launched(launch_pdl(c.d_v == 64 ? weights_f32_kernel<64> : weights_f32_kernel<128>, dim3((unsigned)ceil_div(max_seq_len, kWeightTile), B),
                                   dim3(256), 0, s, p, c.d_r));
    const bool multi = cu_q != nullptr && max_q_len > 1;
    const WeightKernel k = weight_kernel(kind, c, multi);
    const long long tiles = B * ceil_div(max_seq_len, k.tile);
    const int grid = (int)std::min<long long>(tiles, h->sm_count);
    WeightLaunch l;
    l.teams = std::max(1, kWeightConsumers / c.G);
    l.split = 1;
    if (multi) {                                         // as many teams on the same tiles as there are pairs of rows for
        l.split = l.teams;
        while (l.split > (max_q_len + 1) / 2 || l.teams % l.split != 0) --l.split;
    } else {
        l.teams = (int)std::min<long long>(l.teams, (tiles + grid - 1) / grid);
    }
    const int leads = l.teams / l.split;
    // beside the ring: lengths, barriers and the sums of up to four tiles per team
    const size_t tail = (size_t)(B + 1) * 4 + 2048 + (size_t)l.teams * 4 * c.G * k.tile * 4;
    ring(leads, k.stage, (size_t)h->smem_optin - tail, &l.nstage, &l.producers);
    l.batch = l.nstage / leads;
    const int sums = multi ? l.batch * l.teams : 2 * l.teams;
    const size_t smem = l.nstage * k.stage + WeightTraits<kCacheQ4, 64, 0, 32>::tail_bytes(B, l.nstage, sums, c.G) + (size_t)sums * c.G * (k.tile - 32) * 4;
    if (smem > (size_t)h->smem_optin) return GVA_ERR_UNSUPPORTED;
    const int rc = allow_smem(h, reinterpret_cast<const void *>(k.fn), smem);
    if (rc != GVA_OK) return rc;
    return launched(launch_pdl(k.fn, dim3(grid), dim3(32 * (l.teams * c.G + l.producers)), smem, s, p, l));
}

// Blocks per sequence of the eviction's selection: as many as leave the device with about one block per SM, eight (the
// portable cluster size) at most.  Short sequences need them for the moves alone.
int evict_cluster(const gva_handle *h, int B) {
    int c = 1;
    while (c < 8 && 2 * c * B <= h->sm_count) c *= 2;
    return c;
}
// The kernels count slots in 32 bits, ahead of the one in hand.
constexpr int kEvictMost = 1 << 30;
size_t evict_workspace(int B, int max_seq_len) {
    const size_t stride = ((size_t)max_seq_len / 2 + 64) / 64 * 64;
    return align_up((size_t)B * 4, 256) + 2 * align_up((size_t)B * stride * 4, 256);
}
int evict(gva_handle *h, const int32_t *block_table, int num_pages, int max_pages, MovePools pools, const float *weights_in,
          const int32_t *positions_in, const int32_t *seq_lens, const int32_t *keep, const int32_t *next_pos, int sinks, int recent,
          float *weights_out, int32_t *positions_out, int32_t *new_lens, int stride, void *workspace, size_t workspace_bytes, int B,
          int max_seq_len, int32_t *dev_status, void *stream) {
    if (B < 0 || max_seq_len < 0 || stride < 0 || sinks < 0 || recent < 0) return GVA_ERR_INVALID_ARG;
    if (B == 0) return GVA_OK;
    if (!weights_in || !seq_lens || !keep || (recent > 0 && !next_pos) || !weights_out || !positions_out || !new_lens || stride < max_seq_len)
        return GVA_ERR_INVALID_ARG;
    if (!aligned(weights_in, 4) || !aligned(positions_in, 4) || !aligned(seq_lens, 4) || !aligned(keep, 4) || !aligned(next_pos, 4) ||
        !aligned(weights_out, 4) || !aligned(positions_out, 4) || !aligned(new_lens, 4))
        return GVA_ERR_INVALID_ARG;
    if (B > 8192 || max_seq_len > kEvictMost) return GVA_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < evict_workspace(B, max_seq_len)) return GVA_ERR_WORKSPACE;
    if (!aligned(workspace, 256)) return GVA_ERR_INVALID_ARG;
    EvictParams p;
    std::memset(&p, 0, sizeof(p));
    p.w_in = weights_in; p.pos_in = positions_in; p.seq_lens = seq_lens; p.keep = keep; p.next_pos = recent > 0 ? next_pos : nullptr;
    p.sinks = sinks; p.recent = recent; p.w_out = weights_out; p.pos_out = positions_out; p.new_lens = new_lens;
    p.stride = stride; p.B = B; p.max_seq_len = max_seq_len; p.P = h->cfg.page_size; p.num_pages = num_pages; p.max_pages = max_pages;
    p.block_table = block_table;
    p.move_stride = (int)(((size_t)max_seq_len / 2 + 64) / 64 * 64);
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    p.n_moves = reinterpret_cast<int32_t *>(ws);
    p.holes = reinterpret_cast<int32_t *>(ws + align_up((size_t)B * 4, 256));
    p.sources = reinterpret_cast<int32_t *>(ws + align_up((size_t)B * 4, 256) + align_up((size_t)B * p.move_stride * 4, 256));
    p.dev_status = dev_status;
    // few moves: the cluster that has chosen moves the rows too, which saves a launch and its look-ups (three sequences of 1100 to
    // 1500 tokens: 18.7 us with two launches, 14.4 with one; 31 with one and a single block per sequence)
    int C = evict_cluster(h, B);
    const int here = max_seq_len / 2 <= kEvictMoveHere * kMoveBatch * C ? 1 : 0;
    if (max_seq_len <= kEvictAlone && !here) C = 1;
    const int alone = max_seq_len <= kEvictAlone ? 1 : 0;
    const int per_block = ((max_seq_len + (alone ? 1 : C) - 1) / (alone ? 1 : C) + 1023) / 1024 * 1024;
    const int held = std::min(per_block, kEvictKeysMax);
    const size_t smem = (size_t)held * 4;
    int rc = allow_smem(h, reinterpret_cast<const void *>(evict_select_kernel), smem);
    if (rc != GVA_OK) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(B * C);
    cfg.blockDim = dim3(kEvictThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = C;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    rc = launched(cudaLaunchKernelEx(&cfg, evict_select_kernel, p, pools, h->cfg.G, held, alone, here));
    if (rc != GVA_OK || here) return rc;
    const int blocks = std::max(1, std::min((max_seq_len / 2 + 31) / 32, (8 * h->sm_count + B - 1) / B));
    return launched(launch_pdl(evict_move_kernel, dim3(blocks, B), dim3(kMoveThreads), 0, static_cast<cudaStream_t>(stream), p, pools, h->cfg.G));
}
}  // namespace

extern "C" {

int gva_q4_append(gva_handle *h, const gva_q4_cache *cache, const float *v_new, const float *kr_new, const int32_t *slots,
                  const int32_t *pos, int B, int32_t *dev_status, void *stream) {
    int rc = check_q4(h, cache);
    if (rc != GVA_OK) return rc;
    if (B < 0) return GVA_ERR_INVALID_ARG;
    if (B == 0) return GVA_OK;
    if (!slots || !pos) return GVA_ERR_INVALID_ARG;
    return append_q4(h, cache, v_new, kr_new, nullptr, slots, pos, B, B, 1, dev_status, stream);
}

int gva_q4_append_chunk(gva_handle *h, const gva_q4_cache *cache, const float *v_new, const float *kr_new, const int32_t *cu_q,
                        const int32_t *ctx_lens, const int32_t *first_pos, int B, int n_q, int32_t *dev_status, void *stream) {
    int rc = check_q4(h, cache);
    if (rc != GVA_OK) return rc;
    if (B < 0 || n_q < 0) return GVA_ERR_INVALID_ARG;
    if (B == 0 || n_q == 0) return GVA_OK;
    if (!cu_q || !aligned(cu_q, 4) || !ctx_lens) return GVA_ERR_INVALID_ARG;
    // rows of a block: up to four shares of eight elements per thread, as long as that leaves four blocks per SM (990 rows of
    // 4 x 64: 6.7 us with 32 rows to a block, 5.7 with one)
    const int most = append_q4_rows(h->cfg.d_v) / h->cfg.G;
    const int rows = std::max(1, std::min(most, n_q / (4 * h->sm_count)));
    return append_q4(h, cache, v_new, kr_new, cu_q, ctx_lens, first_pos ? first_pos : ctx_lens, B, n_q, rows, dev_status, stream);
}

int gva_q4_widen(gva_handle *h, const gva_q4_cache *cache, const gva_cache *wide, const int32_t *starts, const int32_t *seq_lens,
                 int B, int max_seq_len, int32_t *dev_status, void *stream) {
    int rc = check_q4(h, cache);
    if (rc == GVA_OK) rc = check_plain(h, wide);
    if (rc != GVA_OK) return rc;
    if (B < 0 || max_seq_len < 0) return GVA_ERR_INVALID_ARG;
    if (B == 0 || max_seq_len == 0) return GVA_OK;
    if (!seq_lens || !aligned(starts, 4) || !aligned(seq_lens, 4)) return GVA_ERR_INVALID_ARG;
    if (B > 65535) return GVA_ERR_UNSUPPORTED;
    const gva_config &c = h->cfg;
    WidenParams p;
    std::memset(&p, 0, sizeof(p));
    p.c = q4_pools(cache);
    p.v = static_cast<uint16_t *>(wide->v_pool);
    p.kr = static_cast<uint16_t *>(wide->kr_pool);
    p.block_table = wide->block_table;
    p.num_pages = wide->num_pages;
    p.max_pages = wide->max_pages_per_seq;
    p.starts = starts;
    p.seq_lens = seq_lens;
    p.G = c.G; p.d_v = c.d_v; p.d_r = c.d_r; p.P = c.page_size;
    p.dev_status = dev_status;
    return launched(launch_pdl(widen_q4_kernel, dim3((unsigned)ceil_div(max_seq_len, kWidenTokens), B), dim3(256), 0,
                               static_cast<cudaStream_t>(stream), p));
}

size_t gva_q4_decode_workspace_bytes(const gva_handle *h, int B, int max_seq_len, int num_splits) {
    if (check_common(h, B, max_seq_len, num_splits) != GVA_OK) return 0;
    return q4_plan(h, std::max(B, 1), max_seq_len, num_splits).total;
}

int gva_q4_decode(gva_handle *h, const gva_q4_cache *cache, const float *q_abs, const int32_t *seq_lens, float *out, float *lse,
                  void *workspace, size_t workspace_bytes, int B, int max_seq_len, int num_splits, int32_t *dev_status, void *stream) {
    int rc = check_common(h, B, max_seq_len, num_splits);
    if (rc == GVA_OK) rc = check_q4(h, cache);
    if (rc != GVA_OK) return rc;
    if (B == 0) return GVA_OK;
    if (!q_abs || !seq_lens || !out || !aligned(q_abs, 16) || !aligned(out, 16) || !aligned(seq_lens, 4) || !aligned(lse, 4)) return GVA_ERR_INVALID_ARG;
    const Q4Plan plan = q4_plan(h, B, max_seq_len, num_splits);
    if (!workspace || workspace_bytes < plan.total) return GVA_ERR_WORKSPACE;
    if (!aligned(workspace, 256)) return GVA_ERR_INVALID_ARG;
    if (plan.smem > (size_t)h->smem_optin) return GVA_ERR_UNSUPPORTED;
    const gva_config &c = h->cfg;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    DecodeParams p;
    std::memset(&p, 0, sizeof(p));
    p.seq_lens = seq_lens;
    p.block_table = cache->block_table;
    p.q = q_abs;
    p.out = out;
    p.lse = lse;
    p.rec_o = reinterpret_cast<float *>(ws + plan.rec_o);
    p.rec_ml = reinterpret_cast<float *>(ws + plan.rec_ml);
    p.dev_status = dev_status;
    p.B = B; p.H = c.H; p.G = c.G; p.P = c.page_size;
    p.num_pages = cache->num_pages;
    p.max_pages = cache->max_pages_per_seq;
    p.num_splits = plan.num_splits;
    p.scale_log2 = h->scale * kLog2e;
    Q4Launch l;
    l.pools = q4_pools(cache);
    l.teams = plan.teams;
    l.nstage = plan.nstage;
    l.producers = plan.producers;
    l.segments = plan.num_splits > 0 ? nullptr : reinterpret_cast<int2 *>(ws);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    rc = allow_smem(h, reinterpret_cast<const void *>(plan.k.fn), plan.smem);
    if (rc != GVA_OK) return rc;
    rc = launched(launch_pdl(plan.k.fn, dim3(plan.grid), dim3(32 * (plan.teams * c.G + plan.producers)), plan.smem, s, p, l));
    if (rc != GVA_OK || plan.num_splits == 1) return rc;
    const MergeParams m{p.rec_o, p.rec_ml, l.segments, out, lse, c.H, plan.num_splits, plan.teams};
    const int records = plan.num_splits > 0 ? plan.num_splits : (plan.grid / B + 2) * plan.teams;      // of a sequence, about
    int threads = 64;
    while (threads < 1024 && threads / (c.d_v / 4) * 4 < records) threads *= 2;
    const size_t smem = (size_t)(threads / (c.d_v / 4)) * (c.d_v + 2) * 4;
    return launched(c.d_v == 64 ? launch_pdl(merge_records_kernel<64>, dim3(B, c.H), dim3(threads), smem, s, m)
                                : launch_pdl(merge_records_kernel<128>, dim3(B, c.H), dim3(threads), smem, s, m));
}

int gva_attention_weights(gva_handle *h, const gva_cache *cache, const float *q_abs, const float *lse, const int32_t *cu_q,
                          const int32_t *seq_lens, float decay, const float *weights_in, float *weights_out, int stride, int B,
                          int max_q_len, int max_seq_len, int32_t *dev_status, void *stream) {
    const int rc = check_plain(h, cache);
    if (rc != GVA_OK) return rc;
    WeightParams p;
    std::memset(&p, 0, sizeof(p));
    p.v = cache->v_pool; p.kr = cache->kr_pool;
    p.block_table = cache->block_table; p.num_pages = cache->num_pages; p.max_pages = cache->max_pages_per_seq;
    const int kind = h->cfg.cache_dtype == GVA_E4M3 ? kCacheE4m3 : h->cfg.cache_dtype == GVA_BF16 ? kCacheBf16 : kCacheF32;
    return attention_weights(h, p, kind, q_abs, lse, cu_q, seq_lens, decay, weights_in, weights_out, stride, B, max_q_len, max_seq_len, dev_status, stream);
}

int gva_q4_attention_weights(gva_handle *h, const gva_q4_cache *cache, const float *q_abs, const float *lse, const int32_t *cu_q,
                             const int32_t *seq_lens, float decay, const float *weights_in, float *weights_out, int stride, int B,
                             int max_q_len, int max_seq_len, int32_t *dev_status, void *stream) {
    const int rc = check_q4(h, cache);
    if (rc != GVA_OK) return rc;
    WeightParams p;
    std::memset(&p, 0, sizeof(p));
    p.v = cache->v_pool; p.sz = static_cast<const __half2 *>(cache->sz_pool); p.kr = cache->kr_pool;
    p.block_table = cache->block_table; p.num_pages = cache->num_pages; p.max_pages = cache->max_pages_per_seq;
    return attention_weights(h, p, kCacheQ4, q_abs, lse, cu_q, seq_lens, decay, weights_in, weights_out, stride, B, max_q_len, max_seq_len, dev_status, stream);
}

size_t gva_evict_workspace_bytes(const gva_handle *h, int B, int max_seq_len) {
    if (!h || B < 0 || max_seq_len < 0 || B > 8192 || max_seq_len > kEvictMost) return 0;
    return evict_workspace(B, max_seq_len);
}

int gva_evict(gva_handle *h, const gva_cache *cache, const float *weights_in, const int32_t *positions_in, const int32_t *seq_lens,
              const int32_t *keep, const int32_t *next_pos, int sinks, int recent, float *weights_out, int32_t *positions_out,
              int32_t *new_lens, int stride, void *workspace, size_t workspace_bytes, int B, int max_seq_len, int32_t *dev_status,
              void *stream) {
    const int rc = check_plain(h, cache);
    if (rc != GVA_OK) return rc;
    const int elem = h->cfg.cache_dtype == GVA_E4M3 ? 1 : h->cfg.cache_dtype == GVA_BF16 ? 2 : 4;
    const MovePools pools{static_cast<uint8_t *>(cache->v_pool), h->cfg.d_r > 0 ? static_cast<uint8_t *>(cache->kr_pool) : nullptr, nullptr,
                          h->cfg.d_v * elem, h->cfg.d_r * elem};
    return evict(h, cache->block_table, cache->num_pages, cache->max_pages_per_seq, pools, weights_in, positions_in, seq_lens, keep, next_pos,
                 sinks, recent, weights_out, positions_out, new_lens, stride, workspace, workspace_bytes, B, max_seq_len, dev_status, stream);
}

int gva_q4_evict(gva_handle *h, const gva_q4_cache *cache, const float *weights_in, const int32_t *positions_in, const int32_t *seq_lens,
                 const int32_t *keep, const int32_t *next_pos, int sinks, int recent, float *weights_out, int32_t *positions_out,
                 int32_t *new_lens, int stride, void *workspace, size_t workspace_bytes, int B, int max_seq_len, int32_t *dev_status,
                 void *stream) {
    const int rc = check_q4(h, cache);
    if (rc != GVA_OK) return rc;
    const MovePools pools{static_cast<uint8_t *>(cache->v_pool), h->cfg.d_r > 0 ? static_cast<uint8_t *>(cache->kr_pool) : nullptr,
                          static_cast<uint32_t *>(cache->sz_pool), h->cfg.d_v / 2, h->cfg.d_r * 2};
    return evict(h, cache->block_table, cache->num_pages, cache->max_pages_per_seq, pools, weights_in, positions_in, seq_lens, keep, next_pos,
                 sinks, recent, weights_out, positions_out, new_lens, stride, workspace, workspace_bytes, B, max_seq_len, dev_status, stream);
}

}  // extern "C"
