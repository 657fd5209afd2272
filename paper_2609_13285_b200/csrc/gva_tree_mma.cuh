// gva_decode_tree over a bf16 cache on the 5th-generation tensor cores (tcgen05 + tensor memory), sm_100a.
//
// A block (one per SM) works on one value group: the strip's 128 rows (32 nodes x 4 heads) are the M of every MMA, a tile of 128
// (d_v = 128: 64) cached tokens is the N of the score product and the K of the value product, so one tile in shared memory feeds both.
//   NWG = 2 (3) groups of 4 warps   softmax: tile t is group t % NWG's, a thread owns a row = a lane of tensor memory
//   4 more warps          issuer of the value products, issuer of the score products (owns the tensor memory), two loaders
//   S[t % NWG] = Q K^T (Q from tensor memory)  ->  weights as bf16 pairs in P[t % NWG]  ->  O += P V
// What bounds it is neither bytes nor a pipe but every role's chain of steps per tile: a wait that is complete already takes 150
// cycles, an MMA 40 to 60 to issue, a tile in all some 600 for each issuer and 1500 and more for the softmax.  Hence large tiles for
// narrow heads (1 M tokens, 16 nodes, the same pools every pass: tiles of 128 and two groups 147 - 154 us = 0.57 - 0.60 of the bytes' time, of 64 and
// four groups 179; wide heads, 16 x 32768, 8 nodes: tiles of 64 and three groups 239 - 243 us = 0.70, of 128 and two 267), and several tiles side by side.  They
// share one O, so they share the rows' softmax references too: those go from tile to tile through shared memory in the tiles' order
// (`turn`), which is a short step as long as no maximum moves one.  Sums stay with each group, relative to the reference they were made with.
// Few nodes leave rows of the MMA unused, and its time is the same: up to 16 nodes are laid out twice, and each copy weighs its half
// of every tile's tokens and has zeros for the others -- a sequence of its own, joined with the other at the end.  What is issued is
// the same for 1 to 32 nodes: 155 GFLOP for 1 M narrow tokens, 95 us at the measured rate, more than the 87 us of their bytes.
// The weights are rounded to bf16 because the value product's operands have one type and the values are bf16; in two parts they would cost
// a second product.  It adds half as much error to the output as its own rounding does where a hundred tokens share the weight, and less the
// more there are.  Their sums are of what is rounded, before it is, in f32.
// The running number of a tile over the block's pieces decides its stage, its group and every barrier's phase; loader and query run
// ahead over pieces.
// Rules as in the prefill kernel: tcgen05.ld / .st never sit in a per-lane branch; no barrier is waited on by parity two phases
// late; every wait is bounded.
#pragma once

#include "gva_tree.cuh"
#include "gva_waits.cuh"

namespace gva {

// 16 consecutive f32 columns of this thread's tensor-memory lane.
__device__ __forceinline__ void tmem_ld16(uint32_t addr, float (&v)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]),
                   "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
                 : "r"(addr)
                 : "memory");
    tmem_ld_wait();
}
__device__ __forceinline__ bool elect_one() {
    uint32_t yes;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(yes));
    return yes != 0;
}

constexpr int tree_mma_tile(int d_v) { return d_v == 64 ? 128 : 64; }
template <int DV, int DR>
struct TreeTraits {
    static constexpr int TILE = tree_mma_tile(DV), HALF = TILE / 2;    // tokens of a tile, and of what a copy of two weighs
    static constexpr int NWG = DV == 64 ? 2 : 3;
    static constexpr int NSTAGE = DV == 64 ? 6 : 8;
    static constexpr int BOXES = DV / 64;
    static constexpr int DRP = (DR + 15) / 16 * 16;              // d_r = 24 occupies 32: the box reads zeros behind the row
    static constexpr int KR_ROW = DRP * 2;
    static constexpr int VBOX_BYTES = TILE * 128;
    static constexpr int V_BYTES = BOXES * VBOX_BYTES;
    static constexpr int KR_BYTES = TILE * KR_ROW;
    static constexpr int STAGE_BYTES = V_BYTES + ((KR_BYTES + 1023) & ~1023);
    // Tensor memory columns: scores and weights of each group, O, the query.
    static constexpr int TMEM_COLS = 512;
    static constexpr int COL_S = 0, COL_P = NWG * TILE, COL_O = COL_P + NWG * TILE / 2, COL_Q = COL_O + DV;
    static_assert(COL_Q + (DV + DRP) / 2 <= TMEM_COLS, "scores, weights, O and the query must fit the allocation");
    static constexpr int SOFTMAX = NWG * 128, THREADS = SOFTMAX + 128;
    static constexpr int PART = 32, JOIN_LD = 36;                // columns of O at a time in the join of copies; f32 of a row there, padded
    static constexpr int OFF_JOIN = NSTAGE * STAGE_BYTES;
    static constexpr int OFF_REF = OFF_JOIN + NWG * (kStripRows / 2) * JOIN_LD * 4;
    static constexpr int OFF_SUM = OFF_REF + 3 * kStripRows * 4, OFF_BAR = OFF_SUM + 2 * SOFTMAX * 4;
    static constexpr int N_BARS = 2 * NSTAGE + 8 * NWG + 6;
    static constexpr int OFF_WORDS = OFF_BAR + N_BARS * 8;       // tensor-memory address, abort flag, a flag per stage, bad rows of a group's tile
    static constexpr int OFF_SEQ = OFF_WORDS + (2 + NSTAGE + 8 * NWG) * 4;
    static constexpr size_t smem_bytes(int B) { return 1024 + OFF_SEQ + (size_t)(B + 1) * 4; }
};

template <int DV, int DR>
__global__ void __launch_bounds__(TreeTraits<DV, DR>::THREADS, 1)
tree_mma_kernel(TreeParams p, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_k) {
    using T = TreeTraits<DV, DR>;
    constexpr int NS = T::NSTAGE, NWG = T::NWG, KS_V = DV / 16, KS_S = KS_V + T::DRP / 16, KS_O = T::TILE / 16;
    constexpr uint32_t kAll = 0xffffffffu;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int c = blockIdx.x / p.G, g = blockIdx.x - c * p.G;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t s_base = smem_u32(smem), bar0 = s_base + T::OFF_BAR;
    auto kv_full = [&](int st) { return bar0 + 8u * st; };                            // by the stage
    auto kv_empty = [&](int st) { return bar0 + 8u * (NS + st); };
    auto s_full = [&](int w) { return bar0 + 8u * (2 * NS + w); };                    // by the group
    auto s_free = [&](int w) { return bar0 + 8u * (2 * NS + NWG + w); };
    auto p_full = [&](int w) { return bar0 + 8u * (2 * NS + 2 * NWG + w); };
    auto met = [&](int w) { return bar0 + 8u * (2 * NS + 3 * NWG + w); };
    auto turn = [&](int w, int quarter) { return bar0 + 8u * (2 * NS + 4 * NWG + 4 * w + quarter); };
    const uint32_t bar1 = bar0 + 8u * (2 * NS + 8 * NWG);
    const uint32_t q_ready = bar1, o_full = bar1 + 8, o_free = bar1 + 16, met_all = bar1 + 24, drain_o = bar1 + 32, drain_s = bar1 + 40;
    uint32_t *s_tmem = reinterpret_cast<uint32_t *>(smem + T::OFF_WORDS);
    volatile int *s_abort = reinterpret_cast<volatile int *>(s_tmem + 1);
    volatile uint32_t *s_flag = s_tmem + 2, *s_bad = s_tmem + 2 + NS;
    volatile float *s_ref = reinterpret_cast<volatile float *>(smem + T::OFF_REF), *s_sum = reinterpret_cast<volatile float *>(smem + T::OFF_SUM);
    int *s_off = reinterpret_cast<int *>(smem + T::OFF_SEQ);

    if (tid == 0) {
        for (int i = 0; i < NS; ++i) {
            mbar_init(kv_full(i), 1);
            mbar_init(kv_empty(i), 1);
        }
        for (int w = 0; w < NWG; ++w) {
            mbar_init(s_full(w), 2);                    // the score product, and its issuer (who has seen the stage's flag)
            mbar_init(s_free(w), 4);                    // one arrival per warp: 32 lanes' would be handled one after the other
            mbar_init(p_full(w), 4);
            mbar_init(met(w), 4);
            for (int i = 0; i < 4; ++i) mbar_init(turn(w, i), 1);
        }
        mbar_init(q_ready, 4);
        mbar_init(o_full, 1);
        mbar_init(o_free, 4 * NWG);
        mbar_init(met_all, 4 * NWG);
        mbar_init(drain_o, 1);
        mbar_init(drain_s, 1);
        *s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        asm volatile("prefetch.tensormap [%0];\n" ::"l"(reinterpret_cast<uint64_t>(&tm_v)) : "memory");
        asm volatile("prefetch.tensormap [%0];\n" ::"l"(reinterpret_cast<uint64_t>(&tm_k)) : "memory");
    }
    if (warp == 4 * NWG + 1) {
        tmem_alloc(smem_u32(s_tmem), T::TMEM_COLS);
        tmem_relinquish();
    }
    grid_dependency_wait();
    tree_offsets(p, s_off);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *s_tmem;
    TreePieces pieces(p, s_off, c);
    TreePiece pc = {};
    uint32_t n_pc = 0;                                  // running number of a piece
    int refs_at = 0;                                    // its references: n_pc % 3 * kStripRows
    int st = 0;                                         // stage of a tile, and the parity of its round through the ring
    uint32_t ph = 0;
    auto advance = [&](int by) {
        st += by;
        if (st >= NS) {
            st -= NS;
            ph ^= 1u;
        }
    };
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) { return warp_wait(bar, parity & 1u, s_abort); };
    // Arrivals of whole warps, by one lane: the barrier unit takes lanes one after the other.
    auto arrive = [&](uint32_t bar) {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
    };

    if (warp < 4 * NWG) {
        // ========================================= softmax: one row per thread =========================================
        const int w = warp >> 2, quarter = warp & 3, r = tid & (kStripRows - 1), hl = lane & 3, h = g * kHeadsPerGroup + hl;
        const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16), o_addr = lane_base + T::COL_O;
        const uint32_t s_addr = lane_base + T::COL_S + w * T::TILE, p_addr = lane_base + T::COL_P + w * (T::TILE / 2);
        float *s_join = reinterpret_cast<float *>(smem + T::OFF_JOIN) + w * (kStripRows / 2) * T::JOIN_LD;
        uint32_t n_tiles = 0;                           // tiles that this group has had: the next one's number is n_tiles * NWG + w
        advance(w);                                     // (its first tile's stage)
        int st_own = 0;                                 // stage and phase of the tile before
        uint32_t ph_own = 0;
        uint32_t n_met = 0;
        // The group's warps meet; false: one of them has given up.  (Not a hardware barrier, on which the others would wait for good.)
        auto meet = [&]() {
            arrive(met(w));
            return wait(met(w), n_met++);
        };
        // A row's node of a piece: its copy, whether there is one, its number.
        auto copies_of = [](const TreePiece &x) { return x.nv <= 16 ? 2 : 1; };
        auto node_of = [&](const TreePiece &x) { return (quarter & (4 / copies_of(x) - 1)) * 8 + (lane >> 2); };
        // The next piece with any tile; one without (more splits than tiles) weighs nothing in the merge.
        auto next_piece = [&](TreePiece &x) {
            while (pieces.next(p, s_off, x)) {
                if (x.lo < x.hi) return true;
                if (w == 0 && r / 4 < x.nv) *reinterpret_cast<float2 *>(p.rec_ml + record_row(p, x.rec, g, r) * 2) = make_float2(-INFINITY, 0.f);
            }
            return false;
        };
        // The query's rows into tensor memory, once the score products before are done, and fresh references.  (Three sets of those: while
        // this group is at piece k and prepares k + 1, others may still read those of k - 1, but not of k - 2, since all have met at k - 1's end.)
        auto next_refs = [&]() { return refs_at == 2 * kStripRows ? 0 : refs_at + kStripRows; };
        auto stage_query = [&](const TreePiece &x, int refs_of, uint32_t last_tile, bool any) {
            const int tok = node_of(x);
            const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(p.q) +
                                                               (((size_t)x.s.r0 + x.n0 + min(tok, x.nv - 1)) * p.H + h) * (DV + DR));
            constexpr int N = (DV + T::DRP) / 8, HALF = (N + 1) / 2;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint4 v[HALF];
#pragma unroll
                for (int i = 0; i < HALF; ++i) {
                    const int at = half * HALF + i;
                    v[i] = tok < x.nv && at * 8 < DV + DR ? __ldg(src + at) : make_uint4(0, 0, 0, 0);
                }
                if (half == 0) {
                    if (any && !wait(s_full(last_tile % NWG), last_tile / NWG)) return false;
                    tc_fence_after();
                }
#pragma unroll
                for (int i = 0; i < HALF; ++i) {
                    if (half * HALF + i >= N) continue;
                    const int at = half * HALF + i;
                    const uint32_t words[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                    tmem_st4_nowait(lane_base + T::COL_Q + at * 4, words);
                }
            }
            s_ref[refs_of + r] = -INFINITY;
            tmem_st_wait();
            tc_fence_before();
            arrive(q_ready);
            return true;
        };
        float sum = 0.f, sum_ref = -INFINITY;           // this group's sum, and the reference it is relative to
        bool poison = false;
        // A tile that drafted tokens, the sequence's end or a bad page reach into: which of its tokens the row sees.  Value rows that P
        // multiplies by 0 must not be NaN or infinite: those behind the end and of bad pages become zeros, and so do drafted tokens' rows
        // with such an element (a row that sees one is made NaN at the end instead).
        auto edge_tile = [&](int st, int t0, uint32_t flag, bool live, size_t node, int half0, int halves, uint64_t (&bits)[2]) -> bool {
            volatile uint32_t *bad_rows = s_bad + w * 8 + (n_tiles & 1) * 4;         // (two sets: a slow reader of the tile before)
            unsigned char *v = smem + st * T::STAGE_BYTES + r * 128;
            const bool mine = r < T::TILE, zero = mine && (t0 + r >= pc.s.total || ((flag >> quarter) & 1));
            bool bad = false;
            if (mine && !zero && t0 + r >= pc.s.ctx) {
#pragma unroll 1
                for (int bx = 0; bx < T::BOXES; ++bx)
#pragma unroll 2
                    for (int i = 0; i < 8; ++i) {
                        const uint4 x = *reinterpret_cast<const uint4 *>(v + bx * T::VBOX_BYTES + i * 16);
                        auto odd = [](uint32_t y) { return (y & 0x7f80u) == 0x7f80u || (y & 0x7f800000u) == 0x7f800000u; };
                        bad |= odd(x.x) || odd(x.y) || odd(x.z) || odd(x.w);
                    }
            }
            if (zero || bad)
#pragma unroll 1
                for (int bx = 0; bx < T::BOXES; ++bx)
#pragma unroll 2
                    for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4 *>(v + bx * T::VBOX_BYTES + i * 16) = make_uint4(0, 0, 0, 0);
            const uint32_t all = __ballot_sync(kAll, bad);
            if (lane == 0) bad_rows[quarter] = all;
            fence_async_smem();
            if (!meet()) return false;
#pragma unroll 1
            for (int k = 0; k < halves; ++k) {
                const int from = (half0 + k) * T::HALF, n = pc.s.total - t0 - from;  // tokens of this half of the tile
                uint64_t seen = live ? tree_window(p.mask + node * p.words, p.words, t0 + from - pc.s.ctx) : 0, bad_here = 0;
                if (n < 64) seen = n <= 0 ? 0 : seen & ((1ull << n) - 1);
#pragma unroll
                for (int i = 0; i < T::HALF / 32; ++i) {
                    const int word = (half0 + k) * (T::HALF / 32) + i;
                    if ((flag >> word) & 1) seen &= ~(0xffffffffull << (32 * i));
                    bad_here |= (uint64_t)bad_rows[word] << (32 * i);
                }
                poison |= (seen & bad_here) != 0;
                if (k == 0) bits[0] = seen;
                else bits[1] = seen;
            }
            return true;
        };

        auto store_words = [](uint32_t addr, const uint32_t (&x)[T::HALF / 2]) {
            if constexpr (T::HALF == 64) tmem_st32u_nowait(addr, x);
            else tmem_st16_nowait(addr, x);
        };
        if (w == NWG - 1) tree_publish(p, s_off, r, kStripRows);     // (its first tile comes last)
        bool have = next_piece(pc);
        uint32_t t_base = 0;                            // running number of the piece's first tile
        if (have && w == 0) ok = stage_query(pc, 0, 0, false);
        while (have && ok) {
            const int copies = copies_of(pc), copy = quarter * copies / 4, tok = node_of(pc);
            const bool live = tok < pc.nv;
            const size_t node = (size_t)pc.s.r0 + pc.n0 + (live ? tok : 0), row_h = node * p.H + h;
            if (copies > 1) {                           // the other copy's tokens weigh nothing
                const uint32_t none[T::HALF / 2] = {};
                store_words(p_addr + (1 - copy) * (T::HALF / 2), none);
                tmem_st_wait();
            }
            sum = 0.f;
            sum_ref = -INFINITY;
            poison = false;
            const uint32_t t_end = t_base + (uint32_t)(pc.hi - pc.lo);
            const int first = pc.lo, ctx = pc.s.ctx, halves = 2 / copies, half0 = copy;   // (halves of a tile that this copy weighs)
            for (; n_tiles * NWG + w < t_end; ++n_tiles) {
                const int t = (int)(n_tiles * NWG) + w, t0 = (first + (int)(t - t_base)) * T::TILE;
                if (!wait(s_full(w), n_tiles)) { ok = false; break; }
                tc_fence_after();
                // The row's scores, half a tile at a time: of two halves the first is loaded again for its weights.
                const uint32_t flag = s_flag[st];
                float s[T::HALF], m_tile = -INFINITY;
                auto load = [&](int half) {
                    if constexpr (T::HALF == 64) {
                        float lo[32], hi[32];
                        tmem_ld32_nowait(s_addr + half * 64, lo);
                        tmem_ld32_nowait(s_addr + half * 64 + 32, hi);
                        tmem_ld_wait();
#pragma unroll
                        for (int k = 0; k < 32; ++k) { s[k] = lo[k]; s[32 + k] = hi[k]; }
                    } else {
                        tmem_ld32(s_addr + half * 32, s);
                    }
                };
                auto free_scores = [&]() {              // the score product after the next NWG - 1 may have their place
                    tc_fence_before();
                    arrive(s_free(w));
                };
                load(half0);
                if (halves == 1) free_scores();
                const bool edge = t0 + T::TILE > ctx || flag != 0;                   // the same for the whole block
                uint64_t bits[2] = {~0ull, ~0ull};
                if (edge && !edge_tile(st, t0, flag, live, node, half0, halves, bits)) { ok = false; break; }
                auto hide = [&](uint64_t seen) {
#pragma unroll
                    for (int j = 0; j < T::HALF; j += 32) {
                        const uint32_t word = (uint32_t)(seen >> j);
#pragma unroll
                        for (int k = 0; k < 32; ++k) s[j + k] = (word >> k) & 1 ? s[j + k] : -INFINITY;
                    }
                };
#pragma unroll 1
                for (int i = 0;;) {
                    if (edge) hide(i == 0 ? bits[0] : bits[1]);
                    float mx[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) mx[k] = max3(s[k], s[k + 4], s[k + 8]);
#pragma unroll
                    for (int j = 12; j + 8 <= T::HALF; j += 8)
#pragma unroll
                        for (int k = 0; k < 4; ++k) mx[k] = max3(mx[k], s[j + k], s[j + 4 + k]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) mx[k] = fmaxf(mx[k], s[T::HALF - 4 + k]);
                    m_tile = max3(m_tile, fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                    if (++i == halves) break;
                    load(i);
                }
                m_tile *= p.scale_log2;
                // The reference as the tile before leaves it.  It moves only when a tile's maximum exceeds it by more than 2^8: weights stay
                // below 256, the quotient is the same, and O in tensor memory is rescaled only then, once the value product before is done.
                // (tcgen05.ld / .st take whole warps: rows that stay multiply by 1.)  Asked for together: whether the group's weights
                // before (long done, mostly) have been used.
                const int w1 = w == 0 ? NWG - 1 : w - 1;
                const uint32_t turn1 = w == 0 ? n_tiles - 1 : n_tiles;
                if (t > 0 && !(n_tiles == 0 ? wait(turn(w1, quarter), turn1)
                                            : warp_wait(turn(w1, quarter), turn1 & 1u, kv_empty(st_own), ph_own, s_abort))) { ok = false; break; }
                float ref = s_ref[refs_at + r];
                const bool move = m_tile > ref + kRescaleLog2;
                if (__any_sync(kAll, move)) {
                    if ((uint32_t)t != t_base) {
                        const int before = st == 0 ? NS - 1 : st - 1;                // stage of the tile before, and its phase
                        if (!wait(kv_empty(before), st == 0 ? ph ^ 1u : ph)) { ok = false; break; }
                        tc_fence_after();
                        const float alpha = move ? fast_exp2(ref - m_tile) : 1.f;
#pragma unroll 1
                        for (int part = 0; part < DV / 16; ++part) {
                            float o[16];
                            uint32_t words[16];
                            tmem_ld16(o_addr + part * 16, o);
#pragma unroll
                            for (int i = 0; i < 16; ++i) words[i] = __float_as_uint(o[i] * alpha);
                            tmem_st16_nowait(o_addr + part * 16, words);
                        }
                        tmem_st_wait();
                        tc_fence_before();
                    }
                    if (move) s_ref[refs_at + r] = ref = m_tile;
                }
                arrive(turn(w, quarter));
                tc_fence_after();
                if (sum_ref != ref) {
                    sum *= fast_exp2(sum_ref - ref);
                    sum_ref = ref;
                }
                const float nm = ref == -INFINITY ? 0.f : -ref;                      // nothing seen yet: all weights 0, not NaN
                const uint64_t sc2 = f2_pack(p.scale_log2, p.scale_log2), nm2 = f2_pack(nm, nm);
                uint64_t sum2[2] = {f2_pack(0.f, 0.f), f2_pack(0.f, 0.f)};
#pragma unroll 1
                for (int i = halves - 1;;) {
                    uint32_t pk[T::HALF / 2];
#pragma unroll
                    for (int k = 0; k < T::HALF; k += 2) {
                        float a, b;
                        f2_unpack(f2_fma(f2_pack(s[k], s[k + 1]), sc2, nm2), a, b);
                        a = fast_exp2(a);
                        b = fast_exp2(b);
                        sum2[(k >> 1) & 1] = f2_add(sum2[(k >> 1) & 1], f2_pack(a, b));
                        pk[k >> 1] = pack_bf16(a, b);
                    }
                    store_words(p_addr + (half0 + i) * (T::HALF / 2), pk);
                    if (--i < 0) break;
                    load(i);
                    free_scores();
                    if (edge) hide(bits[0]);
                }
                float sa, sb;
                f2_unpack(f2_add(sum2[0], sum2[1]), sa, sb);
                sum += sa + sb;
                tmem_st_wait();
                tc_fence_before();
                arrive(p_full(w));
                st_own = st;
                ph_own = ph;
                advance(NWG);
            }
            TreePiece nx;
            const bool more = next_piece(nx);
            if (ok && more && w == 0) ok = stage_query(nx, next_refs(), t_end - 1, true);
            ok = ok && wait(o_full, n_pc);
            if (!__all_sync(kAll, ok)) { ok = false; break; }
            // All value products are done, so all references are final: sums relative to them from every group, then the copies' shares.
            volatile float *refs = s_ref + refs_at, *sums = s_sum + (n_pc & 1) * T::SOFTMAX;
            const float own_ref = refs[r];
            sums[tid] = poison ? __int_as_float(0x7fc00000) : sum == 0.f ? 0.f : sum * fast_exp2(sum_ref - own_ref);
            arrive(met_all);
            if (!wait(met_all, n_pc)) { ok = false; break; }
            float m = -INFINITY, l = 0.f, share = 1.f;
            {
                const int rows = kStripRows / copies, r0 = r & (rows - 1);
                for (int k = 0; k < copies; ++k) m = fmaxf(m, refs[r0 + k * rows]);
                const float ref = m == -INFINITY ? 0.f : m;
                for (int k = 0; k < copies; ++k) {
                    float x = 0.f;
#pragma unroll
                    for (int i = 0; i < NWG; ++i) x += sums[i * kStripRows + r0 + k * rows];
                    l += x == 0.f ? 0.f : fast_exp2(refs[r0 + k * rows] - ref) * x;
                }
                if (copies > 1) share = own_ref == -INFINITY ? 0.f : fast_exp2(own_ref - ref);
            }
            const size_t rec = pc.rec >= 0 ? record_row(p, pc.rec, g, live ? tok * kHeadsPerGroup + hl : 0) : 0;
            if (w == 0 && live && copy == 0) {
                if (pc.rec >= 0) *reinterpret_cast<float2 *>(p.rec_ml + rec * 2) = make_float2(m, l);
                else if (p.lse) p.lse[row_h] = tree_lse(m, l);
            }
            const float inv = (pc.rec < 0 ? tree_inverse(l) : 1.f) * share;
            tc_fence_after();
#pragma unroll 1
            for (int part = w; part < DV / T::PART; part += NWG) {
                float o[T::PART];
                tmem_ld32(o_addr + part * T::PART, o);
#pragma unroll
                for (int i = 0; i < T::PART; ++i) o[i] *= inv;
                if (copies > 1) {
                    if (copy > 0)
#pragma unroll
                        for (int i = 0; i < T::PART; i += 4)
                            *reinterpret_cast<float4 *>(s_join + (r - kStripRows / 2) * T::JOIN_LD + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                    if (!meet()) { ok = false; break; }
                    if (copy == 0)
#pragma unroll
                        for (int i = 0; i < T::PART; i += 4) {
                            const float4 x = *reinterpret_cast<const float4 *>(s_join + r * T::JOIN_LD + i);
                            o[i] += x.x;
                            o[i + 1] += x.y;
                            o[i + 2] += x.z;
                            o[i + 3] += x.w;
                        }
                    if (part + NWG < DV / T::PART && !meet()) { ok = false; break; }     // (else the next piece's meetings do)
                }
                if (live && copy == 0) {
                    if (pc.rec < 0) {
                        uint4 *dst = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.out) + row_h * DV + part * T::PART);
#pragma unroll
                        for (int i = 0; i < T::PART; i += 8)
                            dst[i / 8] = make_uint4(pack_bf16(o[i], o[i + 1]), pack_bf16(o[i + 2], o[i + 3]), pack_bf16(o[i + 4], o[i + 5]), pack_bf16(o[i + 6], o[i + 7]));
                    } else {
                        float4 *dst = reinterpret_cast<float4 *>(p.rec_o + rec * DV + part * T::PART);
#pragma unroll
                        for (int i = 0; i < T::PART; i += 4) dst[i / 4] = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                    }
                }
            }
            tc_fence_before();
            arrive(o_free);
            t_base = t_end;
            ++n_pc;
            refs_at = next_refs();
            pc = nx;
            have = more;
        }
    } else {
        int t = 0;                                      // running number of a tile
        if (warp >= 4 * NWG + 2) {
            // ========================== loaders: of even and of odd tiles; a lane per box ==========================
            const int rows = p.P % 64 == 0 ? 64 : 32, boxes = T::TILE / rows;      // a box of that many rows lies in one page
            const uint64_t stream = l2_policy_evict_first();
            const uint32_t box_bytes = (uint32_t)rows * (T::BOXES * 128 + T::KR_ROW);
            while (ok && pieces.next(p, s_off, pc)) {
                for (int base = pc.lo; base < pc.hi && ok; base += 32 / boxes) {
                    // rows of the pools where a lane's box begins; -1: a bad page, -2: nothing there
                    int v0 = -2, k0 = 0;
                    const int at = base * T::TILE + lane * rows;
                    if (base + lane / boxes < pc.hi && at < pc.s.total) {
                        const int j = at / p.P, slot = at - j * p.P;
                        const long long page = tree_page(p, pc.b, j);
                        const bool bad = page < 0 || page >= p.num_pages;
                        if (bad) report_error(p.dev_status, GVA_ERR_BAD_PAGE, pc.b);
                        v0 = bad ? -1 : ((int)page * p.G + g) * p.P + slot;
                        k0 = (int)page * p.P + slot;
                    }
                    const uint32_t bad_boxes = __ballot_sync(kAll, v0 == -1), good_boxes = __ballot_sync(kAll, v0 >= 0);
                    const int n = min(32 / boxes, pc.hi - base);
                    for (int i = 0; i < n; ++i, ++t, advance(1)) {
                        if ((t ^ warp) & 1) continue;
                        if (t >= NS && !wait(kv_empty(st), ph ^ 1u)) { ok = false; break; }
                        const uint32_t mine = (1u << boxes) - 1, full = kv_full(st), dst = s_base + st * T::STAGE_BYTES;
                        const uint32_t bad = (bad_boxes >> (i * boxes)) & mine, good = (good_boxes >> (i * boxes)) & mine;
                        if (elect_one()) {
                            // the flag: a bit for 32 tokens
                            s_flag[st] = rows == 32 ? bad : (bad & 1 ? 3u : 0u) | (bad & 2 ? 12u : 0u);
                            if (good == 0) mbar_arrive(full);
                            else mbar_expect_tx(full, __popc(good) * box_bytes);
                        }
                        __syncwarp();                   // (what is expected is known before any of it comes)
                        const int k = lane - i * boxes; // a lane fetches the box that it has looked up
                        if (k >= 0 && k < boxes && v0 >= 0) {
#pragma unroll
                            for (int bx = 0; bx < T::BOXES; ++bx) tma_load_2d_stream(dst + bx * T::VBOX_BYTES + k * rows * 128, &tm_v, bx * 64, v0, full, stream);
                            if constexpr (DR > 0) tma_load_2d(dst + T::V_BYTES + k * rows * T::KR_ROW, &tm_k, 0, k0, full);
                        }
                        __syncwarp();
                    }
                }
            }
            // copies in flight must land before the block's shared memory is released
            if (!ok || __any_sync(kAll, *s_abort)) {
                bool landed = true;                     // (the last tile of every stage, the other loader's too, which may never have been asked for)
                for (int k = 0; k < min(t, NS) && landed; ++k) landed = warp_wait(kv_full(k), ((t - 1 - k) / NS) & 1, nullptr);
            }
        } else if (warp < 4 * NWG + 2) {
            // ================================= MMA issuers: a warp per product, one elected lane issues =================================
            constexpr uint32_t hi128 = (1024u >> 4) | (1u << 14) | ((uint32_t)kSwz128 << 29);    // (descriptors as in the prefill kernel)
            constexpr uint32_t hikr = ((8u * T::KR_ROW) >> 4) | (1u << 14) | ((uint32_t)(T::KR_ROW == 32 ? kSwz32 : kSwz64) << 29);
            constexpr uint32_t lo_k = (16u >> 4) << 16, lo_mn = ((uint32_t)T::VBOX_BYTES >> 4) << 16;
            const uint32_t a_st = (s_base & 0x3FFFFu) >> 4;
            auto mk = [](uint32_t lo, uint32_t hi) { return (uint64_t)lo | ((uint64_t)hi << 32); };
            int w = 0;
            uint32_t round = 0;                         // t = round * NWG + w
            if (warp == 4 * NWG + 1) {
                constexpr uint32_t idesc = umma_idesc(kStripRows, T::TILE, false);
                while (ok && pieces.next(p, s_off, pc)) {
                    if (pc.lo >= pc.hi) continue;
                    if (!wait(q_ready, n_pc)) { ok = false; break; }
                    ++n_pc;
                    const int first = pc.lo, end = pc.hi;
                    for (int j = first; j < end; ++j, ++t, advance(1)) {
                        if (!(round == 0 ? wait(kv_full(st), ph) : warp_wait(kv_full(st), ph, s_free(w), (round - 1) & 1u, s_abort))) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t vb = a_st + (uint32_t)st * (T::STAGE_BYTES >> 4), d = tmem + T::COL_S + w * T::TILE;
                        if (elect_one()) {
#pragma unroll
                            for (int ks = 0; ks < KS_S; ++ks) {
                                const uint32_t off = ks < KS_V ? ((ks >> 2) * T::VBOX_BYTES + (ks & 3) * 32) >> 4 : (T::V_BYTES >> 4) + (uint32_t)(ks - KS_V) * 2;
                                const uint64_t k_desc = mk((vb + off) | lo_k, ks < KS_V ? hi128 : hikr);
                                umma_bf16_ts(d, tmem + T::COL_Q + ks * 8, k_desc, idesc, ks > 0);
                            }
                            umma_commit(s_full(w));
                            mbar_arrive(s_full(w));
                        }
                        __syncwarp();
                        if (++w == NWG) { w = 0; ++round; }
                    }
                }
            } else {
                constexpr uint32_t idesc = umma_idesc(kStripRows, DV, true);
                while (ok && pieces.next(p, s_off, pc)) {
                    if (pc.lo >= pc.hi) continue;
                    const int first = pc.lo, end = pc.hi;
                    for (int j = first; j < end; ++j, ++t, advance(1)) {
                        // every row has stored its weights of tile t and finished any rescaling of O; of a new piece, the one before has been read
                        if (!wait(p_full(w), round)) { ok = false; break; }
                        if (j == first && n_pc > 0 && !wait(o_free, n_pc - 1)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t vb = a_st + (uint32_t)st * (T::STAGE_BYTES >> 4), a = tmem + T::COL_P + w * (T::TILE / 2);
                        if (elect_one()) {
#pragma unroll
                            for (int ks = 0; ks < KS_O; ++ks)
                                umma_bf16_ts(tmem + T::COL_O, a + ks * 8, mk((vb + ks * (16 * 128 >> 4)) | lo_mn, hi128), idesc, (j > first || ks > 0) ? 1u : 0u);
                            umma_commit(kv_empty(st));
                            if (j + 1 == end) umma_commit(o_full);
                        }
                        __syncwarp();
                        if (++w == NWG) { w = 0; ++round; }
                    }
                    ++n_pc;
                }
            }
            // nothing issued here may still be running (or about to signal a barrier) when the block ends
            if (t > 0) {
                const uint32_t dr = warp == 4 * NWG + 1 ? drain_s : drain_o;
                if (elect_one()) umma_commit(dr);
                __syncwarp();
                warp_wait(dr, 0, nullptr);
            }
        }
    }
    if (!ok && lane == 0 && !*s_abort) {
        report_error(p.dev_status, GVA_ERR_TIMEOUT, pc.b);
        *s_abort = 1;
    }
    tc_fence_before();
    grid_dependency_launch();
    __syncthreads();
    if (warp == 4 * NWG + 1) {
        tc_fence_after();
        tmem_dealloc(tmem, T::TMEM_COLS);
    }
}

// ---- host ------------------------------------------------------------------------------------------------------
using TreeMmaFn = void (*)(TreeParams, CUtensorMap, CUtensorMap);
struct TreeMma {
    TreeMmaFn fn;
    int threads, drp;
    size_t fixed;                    // shared memory without the offsets of sequences
};
template <int DV, int DR>
TreeMma tree_mma_t() { return TreeMma{tree_mma_kernel<DV, DR>, TreeTraits<DV, DR>::THREADS, TreeTraits<DV, DR>::DRP, TreeTraits<DV, DR>::smem_bytes(0)}; }
inline TreeMma tree_mma(const gva_config &c) {
    if (c.d_v == 64) return c.d_r == 16 ? tree_mma_t<64, 16>() : c.d_r == 24 ? tree_mma_t<64, 24>() : tree_mma_t<64, 0>();
    return c.d_r == 32 ? tree_mma_t<128, 32>() : tree_mma_t<128, 0>();
}
// Maps of the values (boxes of 64 dims by the tokens that lie in one page) and of the positional keys.
inline bool tree_maps(const gva_config &c, const MmaHostState &st, const TreeParams &p, int drp, CUtensorMap *v, CUtensorMap *k) {
    const uint32_t rows = c.page_size % 64 == 0 ? 64 : 32;
    if (!encode_map(st, v, p.v_pool, c.d_v, (uint64_t)p.num_pages * c.G * c.page_size, 64, rows, CU_TENSOR_MAP_SWIZZLE_128B)) return false;
    if (c.d_r == 0) {
        *k = *v;                     // (never used)
        return true;
    }
    return encode_map(st, k, p.kr_pool, c.d_r, (uint64_t)p.num_pages * c.page_size, drp, rows, drp == 16 ? CU_TENSOR_MAP_SWIZZLE_32B : CU_TENSOR_MAP_SWIZZLE_64B);
}

}  // namespace gva
