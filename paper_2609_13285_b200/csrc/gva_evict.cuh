// Eviction of the cached tokens that have gathered the least attention.
#pragma once

#include <cooperative_groups.h>

#include "gva_q4.cuh"

namespace gva {

// ---- eviction -------------------------------------------------------------------------------------------------------
// A token counts by its weight; those at positions below `sinks` or within the last `recent` positions count as +inf, a
// NaN as -inf.  The keep[b] first in the order (weight descending, slot ascending) stay.  Attention does not care in which
// order the cache holds its tokens (their positional keys are rotated already), so nothing is shifted: with n = min(keep,
// len), survivors in slots below n stay where they are, and the i-th survivor behind n goes to the i-th free slot before n.
// Sources and targets are disjoint, so the moves need no order among themselves.
//
// select: one cluster of blocks per sequence -- or, where the keys of a sequence fit one block's shared memory with room to spare, its
// first block alone -- finds the n-th key by a radix select (digits of 11, 11 and 10 bits from the top, histograms in
// shared memory summed over the cluster), counts the ties that still fit, and writes weights and
// positions of the slots that stay, zero and -1 for those that leave, and the lists of free slots and of survivors to move.
// move: blocks copy the rows of the moves in 16-byte pieces, weights and positions with them.
constexpr int kEvictThreads = 1024;
constexpr int kEvictBins = 2048;
// Sequences up to this length: one block selects, since a cluster has histograms to read from one another and to meet for them.  One
// block against a cluster, us for a 4-bit eviction to three quarters: 1 x 1536 tokens 13.6 / 19.9, 1 x 4096 16.7 / 21.7,
// 1 x 8192 21.6 / 21.6; 3 x 4096 17.1 / 22.2, 3 x 8192 22.7 / 22.9; 32 x 4096 20.0 / 21.6, 32 x 6000 23.0 / 22.9, 32 x 8192 26.4 / 24.4.
constexpr int kEvictAlone = 8192;
constexpr int kEvictMoveHere = 2;        // up to so many batches of moves per block: rows are moved by the selecting cluster
constexpr int kEvictKeysMax = 32768;     // keys of one block that are kept in shared memory; beyond, they are made again

struct EvictParams {
    const float *w_in;
    const int32_t *pos_in;       // nullable: position = slot
    const int32_t *seq_lens, *keep, *next_pos;
    int sinks, recent;
    float *w_out;
    int32_t *pos_out, *new_lens;
    int stride, B, max_seq_len, P, num_pages, max_pages;
    const int32_t *block_table;
    int32_t *n_moves;            // [B]
    int32_t *holes, *sources;    // [B][move_stride]
    int move_stride;
    int32_t *dev_status;
};

// Order-preserving image of the weight: larger key = more worth keeping.
__device__ __forceinline__ uint32_t evict_key(float w) {
    if (w != w) w = -INFINITY;
    const uint32_t u = __float_as_uint(w + 0.f);             // -0 counts as 0
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
constexpr uint32_t kEvictKeyInf = 0xff800000u;               // evict_key(+inf)

// One cached row of a pool: G segments of v_bytes and sz, a page's slots apart, and one of kr_bytes.
struct MovePools {
    uint8_t *v, *kr;             // kr: nullable
    uint32_t *sz;                // 4-bit only, else NULL
    int v_bytes, kr_bytes;       // bytes of a value row of one group, of a positional row (multiples of 16)
};
// A block looks up kMoveBatch moves at a time, and its threads then copy their pieces, four of a thread's in flight at once.
constexpr int kMoveThreads = 256, kMoveBatch = 64;
struct MoveScratch {
    uint32_t to[kMoveBatch], from[kMoveBatch], page_to[kMoveBatch], page_from[kMoveBatch];
};
// Batches first, first + stride, ... of the n moves of sequence b; every thread of a block of NT calls it.
template <int NT>
__device__ __forceinline__ void move_rows(const EvictParams &p, const MovePools &c, int G, int b, int n, int first, int stride, MoveScratch &s) {
    const int tid = threadIdx.x;
    const uint32_t pv = c.v_bytes / 16, values = G * pv, pk = c.kr ? c.kr_bytes / 16 : 0, per = values + pk + (c.sz ? G : 0);
    for (int i0 = first * kMoveBatch; i0 < n; i0 += stride * kMoveBatch) {
        const int here = min(kMoveBatch, n - i0);
        if (tid < here) {
            const int to = p.holes[(size_t)b * p.move_stride + i0 + tid], from = p.sources[(size_t)b * p.move_stride + i0 + tid];
            const size_t table = (size_t)b * p.max_pages, row = (size_t)b * p.stride;
            s.page_to[tid] = (uint32_t)(p.block_table ? (size_t)p.block_table[table + to / p.P] : table + to / p.P);
            s.page_from[tid] = (uint32_t)(p.block_table ? (size_t)p.block_table[table + from / p.P] : table + from / p.P);
            s.to[tid] = to % p.P;
            s.from[tid] = from % p.P;
            p.w_out[row + to] = p.w_in[row + from];          // (the two may be one buffer: sources lie behind all targets)
            p.w_out[row + from] = 0.f;
            p.pos_out[row + to] = p.pos_in ? p.pos_in[row + from] : from;
            p.pos_out[row + from] = -1;
        }
        __syncthreads();
        constexpr int U = 4;
        for (uint32_t e0 = tid; e0 < here * per; e0 += U * NT) {
            uint4 x[U];
            uint8_t *dst[U];
            int size[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t e = e0 + u * NT, m = e / per, k = e - m * per;
                size[u] = 0;
                if (e < here * per) {
                    const size_t to = s.page_to[m], from = s.page_from[m];
                    if (k < values) {
                        const uint32_t g = k / pv, piece = k - g * pv;
                        x[u] = *reinterpret_cast<const uint4 *>(c.v + ((from * G + g) * p.P + s.from[m]) * c.v_bytes + 16 * piece);
                        dst[u] = c.v + ((to * G + g) * p.P + s.to[m]) * c.v_bytes + 16 * piece;
                        size[u] = 16;
                    } else if (k < values + pk) {
                        x[u] = *reinterpret_cast<const uint4 *>(c.kr + (from * p.P + s.from[m]) * c.kr_bytes + 16 * (k - values));
                        dst[u] = c.kr + (to * p.P + s.to[m]) * c.kr_bytes + 16 * (k - values);
                        size[u] = 16;
                    } else {
                        const uint32_t g = k - values - pk;
                        x[u].x = c.sz[(from * G + g) * p.P + s.from[m]];
                        dst[u] = reinterpret_cast<uint8_t *>(c.sz + (to * G + g) * p.P + s.to[m]);
                        size[u] = 4;
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (size[u] == 16) *reinterpret_cast<uint4 *>(dst[u]) = x[u];
                else if (size[u] == 4) *reinterpret_cast<uint32_t *>(dst[u]) = x[u].x;
            }
        }
        __syncthreads();
    }
}

__global__ void __launch_bounds__(kMoveThreads)
evict_move_kernel(EvictParams p, MovePools c, int G) {
    grid_dependency_launch();
    __shared__ MoveScratch s;
    grid_dependency_wait();
    move_rows<kMoveThreads>(p, c, G, blockIdx.y, p.n_moves[blockIdx.y], blockIdx.x, gridDim.x, s);
}

// keys_in_smem: keys of a block that fit; alone: the cluster's first block selects; here: the cluster moves the rows itself
__global__ void __launch_bounds__(kEvictThreads)
evict_select_kernel(EvictParams p, MovePools pools, int G, int keys_in_smem, int alone, int here) {
    namespace cg = cooperative_groups;
    grid_dependency_launch();
    extern __shared__ uint32_t s_keys[];                     // [keys_in_smem]
    __shared__ __align__(8) int s_hists[3][kEvictBins];      // one per digit: a pass needs no second meeting of the cluster
    __shared__ int s_warp[3][32];
    __shared__ int4 s_runs[32];                              // per warp: over first, tie first, over last, tie last
    __shared__ int4 s_share;                                 // their sums, read by the other blocks of the cluster
    __shared__ int s_digit[3], s_rest[3], s_bad;
    __shared__ MoveScratch s_move;
    cg::cluster_group cluster = cg::this_cluster();
    const int blocks = (int)cluster.num_blocks(), block = (int)cluster.block_rank();
    const int C = alone ? 1 : blocks, rank = alone ? 0 : block;          // who selects
    auto meet = [&]() {
        if (alone) __syncthreads();
        else cluster.sync();
    };
    const int b = blockIdx.x / blocks, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int kWarps = kEvictThreads / 32;
    static_assert(kWarps == 32, "a lane per warp");
    if (tid == 0) s_bad = 0;
    for (int i = tid; i < 3 * kEvictBins; i += kEvictThreads) (&s_hists[0][0])[i] = 0;
    grid_dependency_wait();
    if (alone && block > 0) {                                // waits for the lists, then helps to move
        if (!here) return;
        cluster.sync();
        move_rows<kEvictThreads>(p, pools, G, b, *(volatile int *)(p.n_moves + b), block, blocks, s_move);
        return;
    }
    __syncthreads();
    const int len_in = p.seq_lens[b], keep_in = p.keep[b], next = p.next_pos ? p.next_pos[b] : 0;
    bool bad = len_in < 0 || len_in > p.max_seq_len || (long long)len_in > (long long)p.max_pages * p.P;
    const int len = bad ? 0 : len_in;
    if ((bad || keep_in < 0) && rank == 0 && tid == 0) report_error(p.dev_status, GVA_ERR_SEQ_LEN, b);
    const float *w = p.w_in + (size_t)b * p.stride;
    const int32_t *pos = p.pos_in ? p.pos_in + (size_t)b * p.stride : nullptr;
    float *w_out = p.w_out + (size_t)b * p.stride;
    int32_t *pos_out = p.pos_out + (size_t)b * p.stride;
    // this block's slots: a multiple of 32 per warp, warps one after the other
    const int per_block = ((len + C - 1) / C + 1023) / 1024 * 1024;
    const int lo = min(len, rank * per_block), hi = min(len, lo + per_block);
    const bool loses = !bad && keep_in >= 0 && keep_in < len;            // (a negative budget: the sequence stays as it is)
    auto make_key = [&](float weight, int at) -> uint32_t {
        const bool safe = at < p.sinks || (p.recent > 0 && (long long)at >= (long long)next - p.recent);
        return safe ? kEvictKeyInf : evict_key(weight);
    };
    const bool held = per_block <= keys_in_smem;
    // every page of the live range has to be there before a row is moved; asked for ahead of the keys
    const int n_pages = loses && p.block_table ? (len + p.P - 1) / p.P : 0;
    const int32_t *table = p.block_table + (size_t)b * p.max_pages;
    const int page = tid < n_pages ? table[tid] : 0;
    if (held && loses) {
        constexpr int U = 8;                                 // a thread's weights and positions are asked for eight at a time
        for (int t0 = lo + tid; t0 < hi; t0 += U * kEvictThreads) {
            float ww[U];
            int at[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int t = min(t0 + u * kEvictThreads, hi - 1);
                ww[u] = w[t];
                at[u] = pos ? pos[t] : t;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int t = t0 + u * kEvictThreads;
                if (t < hi) s_keys[t - lo] = make_key(ww[u], at[u]);
            }
        }
    }
    if (page < 0 || page >= p.num_pages) s_bad = 1;
    for (int j = tid + kEvictThreads; j < n_pages; j += kEvictThreads)
        if (table[j] < 0 || table[j] >= p.num_pages) s_bad = 1;
    if (loses && !p.block_table && (long long)b * p.max_pages + (len + p.P - 1) / p.P > p.num_pages) s_bad = 1;
    __syncthreads();
    if (s_bad) {
        if (rank == 0 && tid == 0) report_error(p.dev_status, GVA_ERR_BAD_PAGE, b);
        bad = true;
    }
    const int keep = bad || !loses ? len : keep_in;
    if (keep == len) {                                       // nothing leaves (uniform over the cluster)
        for (int t = lo + tid; t < hi; t += kEvictThreads) {
            if (w_out != w) w_out[t] = w[t];
            if (pos_out != pos) pos_out[t] = pos ? pos[t] : t;
        }
        meet();                                              // everyone has read the lengths: new_lens may be seq_lens
        if (rank == 0 && tid == 0) {
            p.new_lens[b] = bad ? len_in : keep;
            p.n_moves[b] = 0;
        }
        if (alone && here) cluster.sync();
        return;
    }
    auto key_of = [&](int t) -> uint32_t { return held ? s_keys[t - lo] : make_key(w[t], pos ? pos[t] : t); };

    // ---- the key of rank `keep`, from the top digit down ----
    uint32_t prefix = 0, mask = 0;
    int want = keep;                                         // this many are still to be found among the keys with this prefix
    const bool none = keep == 0;
    for (int pass = 0; pass < 3 && !none; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11, bins = 1 << bits;
        int *s_hist = s_hists[pass];
        for (int t0 = lo; t0 < hi; t0 += kEvictThreads) {
            const int t = t0 + tid;
            uint32_t key = 0;
            bool on = t < hi;
            if (on) key = key_of(t);
            on = on && (key & mask) == prefix;
            const int digit = (key >> shift) & (bins - 1);
            // equal digits across the warp (runs of equal weights) are counted once
            const uint32_t live = __ballot_sync(0xffffffffu, on);
            if (live == 0) continue;
            const int lead = __ffs(live) - 1;
            const int first = __shfl_sync(0xffffffffu, digit, lead);
            if (__all_sync(0xffffffffu, !on || digit == first)) {
                if (lane == lead) atomicAdd(&s_hist[digit], __popc(live));
            } else if (on) {
                atomicAdd(&s_hist[digit], 1);
            }
        }
        meet();
        // bins from the top: thread i takes bins 2 i and 2 i + 1 counted from the top
        int n0 = 0, n1 = 0;
        const int i0 = bins - 1 - 2 * tid, i1 = i0 - 1;
        if (i1 >= 0) {
#pragma unroll 8
            for (int c = 0; c < C; ++c) {
                const int2 n = *reinterpret_cast<const int2 *>(cluster.map_shared_rank(s_hist, c) + i1);
                n0 += n.y;
                n1 += n.x;
            }
        }
        int incl = n0 + n1;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        if (lane == 31) s_warp[pass][warp] = incl;
        __syncthreads();
        int sums = s_warp[pass][lane];                       // (kWarps = 32)
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, sums, o);
            if (lane >= o) sums += y;
        }
        const int before_warp = warp ? __shfl_sync(0xffffffffu, sums, max(warp - 1, 0)) : 0;
        const int above = before_warp + incl - (n0 + n1);    // keys in bins above i0
        if (above < want && above + n0 + n1 >= want) {
            const bool second = above + n0 < want;
            s_digit[pass] = second ? i1 : i0;
            s_rest[pass] = want - above - (second ? n0 : 0);
        }
        __syncthreads();
        prefix |= (uint32_t)s_digit[pass] << shift;
        mask |= (uint32_t)(bins - 1) << shift;
        want = s_rest[pass];
    }

    // ---- one count of the block's slots: before `keep` and behind it, above the key and equal to it.  Ties stay in slot order, so
    //      how many of a run of slots do follows from how many ties lie before it ----
    const int rows = per_block / kWarps;                     // slots of a warp
    const int w_lo = min(hi, lo + warp * rows), w_hi = min(hi, w_lo + rows);
    int over_first = 0, tie_first = 0, over_last = 0, tie_last = 0;
    for (int t0 = w_lo; t0 < w_hi; t0 += 32) {
        const int t = t0 + lane;
        const uint32_t key = t < w_hi && !none ? key_of(t) : 0;
        const uint32_t over = __ballot_sync(0xffffffffu, !none && t < w_hi && key > prefix), tie = __ballot_sync(0xffffffffu, !none && t < w_hi && key == prefix);
        const uint32_t first = t0 + 32 <= keep ? 0xffffffffu : t0 >= keep ? 0u : (1u << (keep - t0)) - 1;
        over_first += __popc(over & first);
        tie_first += __popc(tie & first);
        over_last += __popc(over & ~first);
        tie_last += __popc(tie & ~first);
    }
    // (slots before `keep`, what stays of them) for a run with so many ties before it
    auto stays_first = [&](int of, int tf, int before) { return of + min(tf, max(0, want - before)); };
    auto stays_last = [&](int ol, int tf, int tl, int before) { return ol + min(tl, max(0, want - before - tf)); };
    if (lane == 0) s_runs[warp] = make_int4(over_first, tie_first, over_last, tie_last);
    __syncthreads();
    int4 run = s_runs[lane];                                 // lane i: warp i's
    if (warp == 0) {
        const int4 sum = make_int4(__reduce_add_sync(0xffffffffu, run.x), __reduce_add_sync(0xffffffffu, run.y),
                                   __reduce_add_sync(0xffffffffu, run.z), __reduce_add_sync(0xffffffffu, run.w));
        if (lane == 0) s_share = sum;
    }
    meet();
    int tie_base = 0, hole_base = 0, source_base = 0, all_holes = 0;
    {
        int ties = 0;
        for (int c = 0; c < C; ++c) {
            const int4 o = alone ? s_share : *cluster.map_shared_rank(&s_share, c);
            const int c_lo = min(len, c * per_block), c_hi = min(len, c_lo + per_block);
            const int holes = max(0, min(c_hi, keep) - c_lo) - stays_first(o.x, o.y, ties), sources = stays_last(o.z, o.y, o.w, ties);
            if (c < rank) {
                hole_base += holes;
                source_base += sources;
                tie_base += o.y + o.w;
            }
            all_holes += holes;
            ties += o.y + o.w;
        }
    }
    {   // the block's warps: lane i holds warp i's ties before, free slots and moving survivors
        int ties = run.y + run.w;
        const int own = ties;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, ties, o);
            if (lane >= o) ties += y;
        }
        ties += tie_base - own;
        const int i_lo = min(hi, lo + lane * rows), i_hi = min(hi, i_lo + rows);
        int holes = max(0, min(i_hi, keep) - i_lo) - stays_first(run.x, run.y, ties), sources = stays_last(run.z, run.y, run.w, ties);
        const int own_holes = holes, own_sources = sources;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, holes, o), z = __shfl_up_sync(0xffffffffu, sources, o);
            if (lane >= o) {
                holes += y;
                sources += z;
            }
        }
        hole_base += __shfl_sync(0xffffffffu, holes - own_holes, warp);
        source_base += __shfl_sync(0xffffffffu, sources - own_sources, warp);
        tie_base = __shfl_sync(0xffffffffu, ties, warp);
    }
    if (rank == 0 && tid == 0) {
        p.n_moves[b] = all_holes;
        p.new_lens[b] = keep;                                // (everyone has read the lengths)
    }
    {
        int seen = tie_base;
        constexpr int U = 4;
        for (int t00 = w_lo; t00 < w_hi; t00 += 32 * U) {
            float ww[U];
            int at[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {                    // what stays where it is, asked for ahead of the decisions
                const int t = t00 + 32 * u + lane;
                if (t < keep && t < w_hi) {
                    if (w_out != w) ww[u] = w[t];
                    if (pos_out != pos) at[u] = pos ? pos[t] : t;
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int t = t00 + 32 * u + lane;
                const uint32_t key = t < w_hi ? key_of(t) : 0, below = (1u << lane) - 1;
                const uint32_t tie = __ballot_sync(0xffffffffu, !none && t < w_hi && key == prefix);
                const bool kept = !none && t < w_hi && (key > prefix || (key == prefix && seen + __popc(tie & below) < want));
                const bool hole = t < w_hi && t < keep && !kept, source = kept && t >= keep;
                const uint32_t hm = __ballot_sync(0xffffffffu, hole), sm = __ballot_sync(0xffffffffu, source);
                if (hole) p.holes[(size_t)b * p.move_stride + hole_base + __popc(hm & below)] = t;
                if (source) p.sources[(size_t)b * p.move_stride + source_base + __popc(sm & below)] = t;
                if (kept && t < keep) {
                    if (w_out != w) w_out[t] = ww[u];
                    if (pos_out != pos) pos_out[t] = at[u];
                } else if (t < w_hi && t >= keep && !kept) { // leaves; the slot is behind the new end
                    w_out[t] = 0.f;
                    pos_out[t] = -1;
                }
                hole_base += __popc(hm);
                source_base += __popc(sm);
                seen += __popc(tie);
            }
        }
    }
    if (!alone || here) cluster.sync();                      // no block leaves while another still reads its shared memory; lists complete
    if (here) move_rows<kEvictThreads>(p, pools, G, b, all_holes, block, blocks, s_move);
}

}  // namespace gva
