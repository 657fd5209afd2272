// Attention of a tree of drafted tokens over the paged GVA cache (gva_decode_tree), sm_100a.
//
// Sequence b has ctx_lens[b] tokens cached and behind them the n_b nodes of its tree; node i sees all of the context and
// those nodes whose bit is set in its mask row:
//     s_ij = q~_i,h . v_j,g + q^rope_i,h . k^rope_j,   o_i,h = softmax_j(s_ij / sqrt(d_qk)) V_g,   j < ctx or bit (j - ctx).
//
// Work: a sequence's nodes are cut into strips of at most 32 (x 4 heads of a group = 128 rows, the M of one MMA), the strip's
// cache into tiles of 64 or 128 tokens.  All strips' tiles in a row, sequence by sequence, are the flat list; it is cut into equal
// ranges, each of which G neighbouring blocks share, one per value group (they read the same positional keys).  A piece = what
// a range holds of one strip.  A strip in one piece is written at once; the pieces of others leave unnormalised (O, m, l)
// records that tree_merge_kernel joins.
#pragma once

#include "gva_prefill.cuh"

namespace gva {

constexpr int kStripNodes = 32, kStripRows = kStripNodes * kHeadsPerGroup;

struct TreeParams {
    const void *q;               // [n_q][H][d_v + d_r]
    const uint32_t *mask;        // [n_q][words]
    const int32_t *cu_q, *ctx_lens, *block_table;
    const void *v_pool, *kr_pool;
    void *out;                   // [n_q][H][d_v]
    float *lse;                  // [n_q][H], nullable
    int32_t *dev_status;
    int4 *entries;               // workspace [B][strips]: a strip's first record, its records, first node, nodes -- for the merge
    float *rec_o, *rec_ml;       // workspace records [..][G][128][d_v], [..][G][128][2]
    int B, H, G, P, num_pages, max_pages, words;
    int n_q, max_q_len, max_seq_len;
    int tile;                    // tokens of a tile
    int strips;                  // of a sequence at most
    int ranges;                  // balanced form: ranges of the flat list; uniform form: blocks (of a group) that share the pieces
    int num_splits;              // 0: balanced; n: every strip in n pieces
    float scale_log2;            // softmax scale * log2(e)
};

// A sequence as the kernels see it: nodes (0 where there is nothing to do), cached tokens and the strips and tiles that makes.
struct TreeSeq {
    int r0, n, ctx, total, strips, tiles, per_strip;
};
__device__ __forceinline__ TreeSeq tree_seq(const TreeParams &p, int b, bool say) {
    TreeSeq s;
    s.r0 = p.cu_q[b];
    s.n = p.cu_q[b + 1] - s.r0;
    s.ctx = p.ctx_lens[b];
    const long long total = (long long)s.ctx + s.n;
    const bool fine = s.n >= 0 && s.n <= p.max_q_len && s.r0 >= 0 && s.r0 <= p.n_q - s.n && s.ctx >= 0 && total <= p.max_seq_len && total <= (long long)p.max_pages * p.P;
    if (!fine && say) report_error(p.dev_status, GVA_ERR_SEQ_LEN, b);
    if (!fine) s.n = 0;
    s.total = (int)total;
    s.strips = (s.n + kStripNodes - 1) / kStripNodes;
    s.tiles = s.n > 0 ? (s.total + p.tile - 1) / p.tile : 0;
    s.per_strip = s.strips > 0 ? (s.n + s.strips - 1) / s.strips : 0;     // nodes, shared out evenly
    return s;
}
// s_off[b] = units before sequence b: tiles of all its strips (balanced) or strips (uniform).  By every thread of the block.
__device__ __forceinline__ void tree_offsets(const TreeParams &p, int *s_off) {
    const int tid = threadIdx.x, nt = blockDim.x;
    for (int b = tid; b < p.B; b += nt) {
        const TreeSeq s = tree_seq(p, b, blockIdx.x == 0);
        s_off[b + 1] = p.num_splits > 0 ? s.strips : s.strips * s.tiles;
    }
    if (tid == 0) s_off[0] = 0;
    __syncthreads();
    if (tid < 32) {
        const int per = (p.B + 31) / 32, start = 1 + tid * per, end = min(start + per, p.B + 1);
        int sum = 0;
        for (int i = start; i < end; ++i) sum += s_off[i];
        int x = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (tid >= o) x += y;
        }
        int base = x - sum;
        for (int i = start; i < end; ++i) {
            base += s_off[i];
            s_off[i] = base;
        }
    }
    __syncthreads();
}

struct TreePiece {
    TreeSeq s;
    int b, strip, n0, nv;        // first node of the strip and how many it has
    int lo, hi;                  // tiles of the piece
    int rec;                     // record it leaves, -1: it is the whole strip and writes its result
};
// The pieces of block group c, in order.
struct TreePieces {
    int x, end, step;
    __device__ __forceinline__ TreePieces(const TreeParams &p, const int *s_off, int c) {
        const int total = s_off[p.B];
        if (p.num_splits > 0) {
            x = c;
            end = total * p.num_splits;
            step = p.ranges;
        } else {
            const int n = partitions_in_use(total, p.ranges);
            // range_begin() in 32 bits: floor(c total / n) = c floor(total / n) + floor(c (total mod n) / n)
            const int whole = n > 0 ? total / n : 0, rest = total - whole * n;
            x = c < n ? c * whole + c * rest / n : 0;
            end = c < n ? (c + 1) * whole + (c + 1) * rest / n : 0;
            step = c;
        }
    }
    __device__ __noinline__ bool next(const TreeParams &p, const int *s_off, TreePiece &t) {      // (rare, and large)
        if (x >= end) return false;
        if (p.num_splits > 0) {
            const int strip = x / p.num_splits, k = x - strip * p.num_splits;
            t.b = seq_of_tile(s_off, p.B, strip);
            t.s = tree_seq(p, t.b, false);
            t.strip = strip - s_off[t.b];
            t.lo = k * t.s.tiles / p.num_splits;                          // (2^24 tiles and 64 splits at most)
            t.hi = (k + 1) * t.s.tiles / p.num_splits;
            t.rec = p.num_splits == 1 ? -1 : (t.b * p.strips + t.strip) * p.num_splits + k;
            x += step;
        } else {
            t.b = seq_of_tile(s_off, p.B, x);
            t.s = tree_seq(p, t.b, false);
            const int rel = x - s_off[t.b];
            t.strip = rel / t.s.tiles;
            t.lo = rel - t.strip * t.s.tiles;
            t.hi = min(t.s.tiles, t.lo + end - x);
            t.rec = t.lo == 0 && t.hi == t.s.tiles ? -1 : step + t.b * p.strips + t.strip;
            x += t.hi - t.lo;
        }
        t.n0 = t.strip * t.s.per_strip;
        t.nv = min(t.s.per_strip, t.s.n - t.n0);
        return true;
    }
};
__device__ __forceinline__ long long tree_page(const TreeParams &p, int b, int j) {
    return p.block_table ? (long long)p.block_table[(size_t)b * p.max_pages + j] : (long long)b * p.max_pages + j;
}
// Which of the 64 tokens from `base` on (counted from the tree's first node; below 0 is context) a mask row shows.
__device__ __forceinline__ uint64_t tree_window(const uint32_t *row, int words, int base) {
    const int o = max(base, 0), w = o >> 5, sh = o & 31;
    const uint32_t a = w < words ? row[w] : 0, b = w + 1 < words ? row[w + 1] : 0, c = w + 2 < words ? row[w + 2] : 0;
    const uint64_t bits = (uint64_t)__funnelshift_r(a, b, sh) | ((uint64_t)__funnelshift_r(b, c, sh) << 32);
    if (base >= 0) return bits;
    return base <= -64 ? ~0ull : (bits << -base) | ((1ull << -base) - 1);
}
template <typename OT>
__device__ __forceinline__ void store_out4(OT *dst, float a, float b, float c, float d) {
    if constexpr (sizeof(OT) == 2) *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_bf16(a, b), pack_bf16(c, d));
    else *reinterpret_cast<float4 *>(dst) = make_float4(a, b, c, d);
}
__device__ __forceinline__ size_t record_row(const TreeParams &p, int rec, int g, int row) { return ((size_t)rec * p.G + g) * kStripRows + row; }
// What a row has come to: its part of the output, by 4 elements, and its log-sum-exp.  A row that saw nothing is 0 and -inf.
__device__ __forceinline__ float tree_inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }
__device__ __forceinline__ float tree_lse(float m, float l) { return (m + log2f(l)) * kLn2; }

// What the merge has to know of every strip, shared out among nt threads of each block of the attention kernel, so that a block of the
// merge finds its work in one trip to memory: it is a chain of trips and little else.
__device__ __forceinline__ void tree_publish(const TreeParams &p, const int *s_off, int tid, int nt) {
    if (p.num_splits == 1) return;
    const int total = s_off[p.B], n = p.num_splits > 0 ? 0 : partitions_in_use(total, p.ranges);
    for (int e = blockIdx.x * nt + tid; e < p.B * p.strips; e += gridDim.x * nt) {
        const int b = e / p.strips, strip = e - b * p.strips;
        const TreeSeq s = tree_seq(p, b, false);
        int4 x = make_int4(0, 0, 0, 0);
        if (strip < s.strips) {
            const int n0 = strip * s.per_strip;
            if (p.num_splits > 0) {
                x = make_int4(e * p.num_splits, p.num_splits, s.r0 + n0, min(s.per_strip, s.n - n0));
            } else {
                const int lo = s_off[b] + strip * s.tiles, c0 = range_owner(lo, total, n), c1 = range_owner(lo + s.tiles - 1, total, n);
                x = make_int4(c0 + e, c0 == c1 ? 0 : c1 - c0 + 1, s.r0 + n0, min(s.per_strip, s.n - n0));
            }
        }
        p.entries[e] = x;
    }
}

// ---- CUDA cores: f32 and e4m3 caches ------------------------------------------------------------------------
// 256 threads, two per row: each scores 16 of 32 tokens, holds half of the row's output in registers.  All 128 rows of a strip are computed,
// whatever it holds, and nothing is loaded ahead: this is the simple form, bound by its f32 products.  us over e4m3 and f32: 32 x 32768 narrow
// tokens, 16 nodes 12270 and 12400 (their bytes 44 and 175); 16 x 32768 wide, 8 nodes 19940 and 19710; 200 x 300, 8 nodes 738 and 798; 7 x 2000, 16 nodes 154
// and 161; 1 x 97 43 and 45.
constexpr int kTreeFmaThreads = 256, kTreeFmaTokens = 32, kTreeFmaTile = 64;
inline size_t tree_fma_smem(int B, int d_v, int d_r) {
    return (size_t)(kStripRows + kTreeFmaTokens) * (d_v + d_r + 4) * 4 + (size_t)kStripRows * (kTreeFmaTokens + 1) * 4 + (size_t)(B + 1) * 4;
}
__device__ __forceinline__ float tree_element(const float *p) { return *p; }
__device__ __forceinline__ float tree_element(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ float tree_element(const uint8_t *p) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(*p, __NV_E4M3)));
}
template <typename CT, typename QT, int DV>
__global__ void __launch_bounds__(kTreeFmaThreads)
tree_fma_kernel(TreeParams p, int d_r) {
    grid_dependency_launch();
    extern __shared__ float s_f[];
    const int d = DV + d_r, ld = d + 4;
    float *s_q = s_f, *s_k = s_q + kStripRows * ld, *s_p = s_k + kTreeFmaTokens * ld;
    int *s_off = reinterpret_cast<int *>(s_p + kStripRows * (kTreeFmaTokens + 1));
    grid_dependency_wait();
    tree_offsets(p, s_off);
    const int tid = threadIdx.x, c = blockIdx.x / p.G, g = blockIdx.x % p.G;
    tree_publish(p, s_off, tid, kTreeFmaThreads);
    const CT *v_pool = static_cast<const CT *>(p.v_pool), *kr_pool = static_cast<const CT *>(p.kr_pool);
    const QT *q = static_cast<const QT *>(p.q);
    QT *out = static_cast<QT *>(p.out);
    const int row = tid >> 1, half = tid & 1, tok = row >> 2, h = g * kHeadsPerGroup + (row & 3);
    TreePieces pieces(p, s_off, c);
    TreePiece t;
    while (pieces.next(p, s_off, t)) {
        const bool live = tok < t.nv;
        const size_t node = (size_t)t.s.r0 + t.n0 + (live ? tok : 0);
        __syncthreads();
        for (int i = half; i < d; i += 2) s_q[row * ld + i] = live ? tree_element(q + (node * p.H + h) * d + i) : 0.f;
        float m = -INFINITY, l = 0.f, acc[DV / 2];
#pragma unroll
        for (int i = 0; i < DV / 2; ++i) acc[i] = 0.f;
        for (int t0 = t.lo * kTreeFmaTile; t0 < min(t.hi * kTreeFmaTile, t.s.total); t0 += kTreeFmaTokens) {
            const long long page = tree_page(p, t.b, t0 / p.P);           // 32 tokens lie in one page
            if (page < 0 || page >= p.num_pages) {                        // counts as empty
                if (tid == 0) report_error(p.dev_status, GVA_ERR_BAD_PAGE, t.b);
                continue;
            }
            __syncthreads();
            const int slot0 = t0 % p.P, nk = min(kTreeFmaTokens, t.s.total - t0);
            for (int i = tid; i < kTreeFmaTokens * DV; i += kTreeFmaThreads) {
                const int k = i / DV, e = i % DV;
                s_k[k * ld + e] = k < nk ? tree_element(v_pool + (((size_t)page * p.G + g) * p.P + slot0 + k) * DV + e) : 0.f;
            }
            for (int i = tid; i < kTreeFmaTokens * d_r; i += kTreeFmaThreads) {
                const int k = i / d_r, e = i % d_r;
                s_k[k * ld + DV + e] = k < nk ? tree_element(kr_pool + ((size_t)page * p.P + slot0 + k) * d_r + e) : 0.f;
            }
            __syncthreads();
            const uint64_t see = live ? tree_window(p.mask + node * p.words, p.words, t0 - t.s.ctx) : 0;
            float x[kTreeFmaTokens / 2], top = -INFINITY;
#pragma unroll
            for (int j = 0; j < kTreeFmaTokens / 2; ++j) x[j] = 0.f;
            for (int e = 0; e < d; e += 4) {
                const float4 a = *reinterpret_cast<const float4 *>(s_q + row * ld + e);
#pragma unroll
                for (int j = 0; j < kTreeFmaTokens / 2; ++j) {
                    const float4 b = *reinterpret_cast<const float4 *>(s_k + (2 * j + half) * ld + e);
                    x[j] = fmaf(a.x, b.x, fmaf(a.y, b.y, fmaf(a.z, b.z, fmaf(a.w, b.w, x[j]))));
                }
            }
#pragma unroll
            for (int j = 0; j < kTreeFmaTokens / 2; ++j) {
                const int k = 2 * j + half;
                x[j] = k < nk && ((see >> k) & 1) ? x[j] * p.scale_log2 : -INFINITY;
                top = fmaxf(top, x[j]);
            }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            const float m_new = fmaxf(m, top), ref = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = m == -INFINITY ? 0.f : exp2f(m - ref);
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < kTreeFmaTokens / 2; ++j) {
                const float e = exp2f(x[j] - ref);
                s_p[row * (kTreeFmaTokens + 1) + 2 * j + half] = e;
                sum += e;
            }
            l = l * alpha + sum + __shfl_xor_sync(0xffffffffu, sum, 1);
            m = m_new;
#pragma unroll
            for (int i = 0; i < DV / 2; ++i) acc[i] *= alpha;
            __syncwarp();
            for (int k = 0; k < nk; ++k) {
                if (!((see >> k) & 1)) continue;                          // (a token out of sight may hold anything)
                const float w = s_p[row * (kTreeFmaTokens + 1) + k];
                const float *v = s_k + k * ld + half * (DV / 2);
#pragma unroll
                for (int i = 0; i < DV / 2; i += 4) {
                    const float4 y = *reinterpret_cast<const float4 *>(v + i);
                    acc[i] = fmaf(w, y.x, acc[i]);
                    acc[i + 1] = fmaf(w, y.y, acc[i + 1]);
                    acc[i + 2] = fmaf(w, y.z, acc[i + 2]);
                    acc[i + 3] = fmaf(w, y.w, acc[i + 3]);
                }
            }
            __syncwarp();
        }
        if (!live) continue;
        if (t.rec < 0) {
            const float inv = tree_inverse(l);
            QT *dst = out + (node * p.H + h) * DV + half * (DV / 2);
#pragma unroll
            for (int i = 0; i < DV / 2; i += 4) store_out4(dst + i, acc[i] * inv, acc[i + 1] * inv, acc[i + 2] * inv, acc[i + 3] * inv);
            if (p.lse && half == 0) p.lse[node * p.H + h] = tree_lse(m, l);
        } else {
            const size_t r = record_row(p, t.rec, g, row);
            float *dst = p.rec_o + r * DV + half * (DV / 2);
#pragma unroll
            for (int i = 0; i < DV / 2; i += 4) *reinterpret_cast<float4 *>(dst + i) = make_float4(acc[i], acc[i + 1], acc[i + 2], acc[i + 3]);
            if (half == 0) *reinterpret_cast<float2 *>(p.rec_ml + r * 2) = make_float2(m, l);
        }
    }
}

// ---- merge -----------------------------------------------------------------------------------------------------
// A block per strip and head and eight nodes of it, a warp each; or (WIDE: few strips in many pieces) one node, the pieces side by side:
// DV / 4 threads read a piece's row.  In both the pieces' weights are made first, one by each lane or thread.
template <typename OT, int DV, bool WIDE>
__global__ void __launch_bounds__(256)
tree_merge_kernel(TreeParams p) {
    grid_dependency_launch();
    constexpr int kMost = 256;                                            // pieces whose weights are held at a time (WIDE)
    __shared__ float s_w[WIDE ? kMost : 1], s_part[WIDE ? 8 : 1], s_o[WIDE ? 256 / (DV / 4) : 1][WIDE ? DV : 1];
    grid_dependency_wait();
    const int4 e = p.entries[blockIdx.x];
    const int h = blockIdx.y, g = h / kHeadsPerGroup, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, count = e.y;
    const int tok = WIDE ? blockIdx.z : blockIdx.z * 8 + warp;
    if (count == 0 || tok >= e.w) return;
    const size_t step = (size_t)p.G * kStripRows, r0 = record_row(p, e.x, g, tok * kHeadsPerGroup + h % kHeadsPerGroup);   // from a piece's row to the next one's
    const size_t row = (size_t)(e.z + tok) * p.H + h;
    OT *out = static_cast<OT *>(p.out) + row * DV;
    // (log-sum-exp over the pieces: every lane has the pieces lane, lane + 32, ...)
    float m = -INFINITY, l = 0.f;
    for (int k = lane; k < count; k += 32) m = fmaxf(m, p.rec_ml[(r0 + k * step) * 2]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float ref = m == -INFINITY ? 0.f : m;
    auto weight = [&](int k) {                                            // 0: an empty piece, which left its O unwritten
        const float2 ml = *reinterpret_cast<const float2 *>(p.rec_ml + (r0 + k * step) * 2);
        const float w = ml.y == 0.f ? 0.f : fast_exp2(ml.x - ref);
        l = fmaf(w, ml.y, l);
        return w;
    };
    if constexpr (WIDE) {
        constexpr int PT = DV / 4, PP = 256 / PT;                         // threads of a row, pieces side by side
        const int c = threadIdx.x % PT, pp = threadIdx.x / PT;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k0 = 0; k0 < count; k0 += kMost) {
            __syncthreads();
            if (k0 + (int)threadIdx.x < count) s_w[threadIdx.x] = weight(k0 + threadIdx.x);
            __syncthreads();
            const int n = min(kMost, count - k0);
#pragma unroll 4
            for (int k = pp; k < n; k += PP) {
                const float w = s_w[k];
                if (w == 0.f) continue;
                const float4 x = *reinterpret_cast<const float4 *>(p.rec_o + (r0 + (k0 + k) * step) * DV + c * 4);
                acc.x = fmaf(w, x.x, acc.x);
                acc.y = fmaf(w, x.y, acc.y);
                acc.z = fmaf(w, x.z, acc.z);
                acc.w = fmaf(w, x.w, acc.w);
            }
        }
        *reinterpret_cast<float4 *>(&s_o[pp][c * 4]) = acc;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        if (lane == 0) s_part[warp] = l;
        __syncthreads();
        if (threadIdx.x >= PT) return;
        l = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) l += s_part[i];
        acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < PP; ++i) {
            const float4 x = *reinterpret_cast<const float4 *>(&s_o[i][c * 4]);
            acc = make_float4(acc.x + x.x, acc.y + x.y, acc.z + x.z, acc.w + x.w);
        }
        const float inv = tree_inverse(l);
        store_out4(out + c * 4, acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    } else {
        constexpr int E = DV / 32;
        float acc[E];
#pragma unroll
        for (int i = 0; i < E; ++i) acc[i] = 0.f;
        for (int k0 = 0; k0 < count; k0 += 32) {
            const float own = k0 + lane < count ? weight(k0 + lane) : 0.f;
            const int n = min(32, count - k0);
#pragma unroll 4
            for (int k = 0; k < n; ++k) {
                const float w = __shfl_sync(0xffffffffu, own, k);
                if (w == 0.f) continue;
#pragma unroll
                for (int i = 0; i < E; i += 2) {
                    const float2 x = *reinterpret_cast<const float2 *>(p.rec_o + (r0 + (k0 + k) * step) * DV + lane * E + i);
                    acc[i] = fmaf(w, x.x, acc[i]);
                    acc[i + 1] = fmaf(w, x.y, acc[i + 1]);
                }
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        const float inv = tree_inverse(l);
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            if constexpr (sizeof(OT) == 2) *reinterpret_cast<uint32_t *>(out + lane * E + i) = pack_bf16(acc[i] * inv, acc[i + 1] * inv);
            else *reinterpret_cast<float2 *>(out + lane * E + i) = make_float2(acc[i] * inv, acc[i + 1] * inv);
        }
    }
    if (p.lse && (WIDE ? threadIdx.x : lane) == 0) p.lse[row] = tree_lse(m, l);
}

}  // namespace gva
