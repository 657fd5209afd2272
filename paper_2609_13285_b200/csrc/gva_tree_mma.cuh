// gva_decode_tree over a bf16 cache on the 5th-generation tensor cores (tcgen05 + tensor memory), sm_100a.
//
// A block works on one value group: the strip's 128 rows (32 nodes x 4 heads) are the M of every MMA, a tile of 64 cached tokens
// is the N of the score product and the K of the value product, so one tile in shared memory feeds both.
//   warps 0-3   softmax: a thread owns a row = a lane of tensor memory
//   warp 4      issues the value products, warp 5 the score products (and owns the tensor memory), warp 6 fetches the tiles
// The running number of a tile over the block's pieces decides its stage, its score buffer and every barrier's phase; the loader runs
// ahead over pieces, so the ring does not drain where a sequence ends.
//   S[t & 1] = Q K^T (Q from tensor memory)  ->  weights as bf16 pairs over the first half of the row's S  ->  O += P V
// Rules as in the prefill kernel: tcgen05.ld / .st never sit in a per-lane branch; no barrier is waited on by parity two phases
// late; every wait is bounded.
#pragma once

#include "gva_tree.cuh"

namespace gva {

constexpr int kTreeMmaThreads = 224;
template <int DV, int DR>
struct TreeTraits {
    static constexpr int NSTAGE = DV == 64 ? 6 : 5;
    static constexpr int BOXES = DV / 64;
    static constexpr int DRP = (DR + 15) / 16 * 16;              // d_r = 24 occupies 32: the box reads zeros behind the row
    static constexpr int KR_ROW = DRP * 2;
    static constexpr int VBOX_BYTES = kTreeTile * 128;
    static constexpr int V_BYTES = BOXES * VBOX_BYTES;
    static constexpr int KR_BYTES = kTreeTile * KR_ROW;
    static constexpr int STAGE_BYTES = V_BYTES + ((KR_BYTES + 1023) & ~1023);
    // Tensor memory: two score buffers, O, the query.  d_v = 64: 256 columns, two blocks on an SM; d_v = 128: 336 of 512, one block.
    static constexpr int TMEM_COLS = DV == 64 ? 256 : 512, BLOCKS_PER_SM = 512 / TMEM_COLS;
    static constexpr int COL_S = 0, COL_O = 2 * kTreeTile, COL_Q = COL_O + DV;
    static_assert(COL_Q + (DV + DRP) / 2 <= TMEM_COLS, "scores, O and the query must fit the allocation");
    static constexpr int OFF_BAR = NSTAGE * STAGE_BYTES, N_BARS = 2 * NSTAGE + 8;
    static constexpr int OFF_WORDS = OFF_BAR + N_BARS * 8;      // tensor-memory address, abort flag, 4 words of bad rows, a flag per stage
    static constexpr int OFF_SEQ = OFF_WORDS + (6 + NSTAGE) * 4;
    static constexpr size_t smem_bytes(int B) { return 1024 + OFF_SEQ + (size_t)(B + 1) * 4; }
};

template <int DV, int DR>
__global__ void __launch_bounds__(kTreeMmaThreads, TreeTraits<DV, DR>::BLOCKS_PER_SM)
tree_mma_kernel(TreeParams p, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_k) {
    using T = TreeTraits<DV, DR>;
    constexpr int NS = T::NSTAGE, KS_V = DV / 16, KS_S = KS_V + T::DRP / 16, KS_O = kTreeTile / 16;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int c = blockIdx.x / p.G, g = blockIdx.x - c * p.G;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t s_base = smem_u32(smem), bar0 = s_base + T::OFF_BAR;
    auto kv_full = [&](int s) { return bar0 + 8u * s; };
    auto kv_empty = [&](int s) { return bar0 + 8u * (NS + s); };
    auto s_full = [&](int t) { return bar0 + 8u * (2 * NS + (t & 1)); };
    auto p_full = [&](int t) { return bar0 + 8u * (2 * NS + 2 + (t & 1)); };      // (one per score buffer: see the prefill kernel)
    const uint32_t q_ready = bar0 + 8u * (2 * NS + 4), o_full = bar0 + 8u * (2 * NS + 5), drain_o = bar0 + 8u * (2 * NS + 6), drain_s = bar0 + 8u * (2 * NS + 7);
    uint32_t *s_tmem = reinterpret_cast<uint32_t *>(smem + T::OFF_WORDS);
    volatile int *s_abort = reinterpret_cast<volatile int *>(s_tmem + 1);
    volatile uint32_t *s_bad = s_tmem + 2, *s_flag = s_tmem + 6;
    int *s_off = reinterpret_cast<int *>(smem + T::OFF_SEQ);

    if (tid == 0) {
        for (int s = 0; s < NS; ++s) {
            mbar_init(kv_full(s), 1);
            mbar_init(kv_empty(s), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(s_full(i), 1);
            mbar_init(p_full(i), kStripRows);
        }
        mbar_init(q_ready, kStripRows);
        mbar_init(o_full, 1);
        mbar_init(drain_o, 1);
        mbar_init(drain_s, 1);
        *s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        asm volatile("prefetch.tensormap [%0];\n" ::"l"(reinterpret_cast<uint64_t>(&tm_v)) : "memory");
        asm volatile("prefetch.tensormap [%0];\n" ::"l"(reinterpret_cast<uint64_t>(&tm_k)) : "memory");
    }
    if (warp == 5) {
        tmem_alloc(smem_u32(s_tmem), T::TMEM_COLS);
        tmem_relinquish();
    }
    grid_dependency_wait();
    tree_offsets(p, s_off);
    if (blockIdx.x == 0)
        for (int b = tid; b <= p.B; b += kTreeMmaThreads) p.offsets[b] = s_off[b];
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *s_tmem;
    TreePieces pieces(p, s_off, c);
    TreePiece pc;
    int t = 0;                                          // running number of a tile, and of a piece that has any
    uint32_t n_pc = 0;
    bool ok = true;

    if (warp < 4) {
        // ========================================= softmax: one row per thread =========================================
        const uint32_t lane_base = tmem + ((uint32_t)(warp * 32) << 16), o_addr = lane_base + T::COL_O;
        while (ok && pieces.next(p, s_off, pc)) {
            // Up to 16 nodes are two warps' rows.  The second block on an SM (its tensor memory starts at column 256) takes the lanes of
            // the upper two warps for them, so that the two blocks' softmax runs on different quarters of the SM.
            const int lw = warp - ((tmem & 0xffffu) >= 256 && pc.nv <= 16 ? 2 : 0);
            const bool dead = lw < 0 || lw * 8 >= pc.nv;
            const int tok = lw * 8 + (lane >> 2), h = g * kHeadsPerGroup + (lane & 3);
            const bool live = !dead && tok < pc.nv;
            const size_t node = (size_t)pc.s.r0 + pc.n0 + (live ? tok : 0), row_h = node * p.H + h;
            const size_t rec = pc.rec >= 0 ? record_row(p, pc.rec, g, live ? tok * kHeadsPerGroup + (lane & 3) : 0) : 0;
            if (pc.lo >= pc.hi) {                       // more splits than tiles: weighs nothing in the merge
                if (live) *reinterpret_cast<float2 *>(p.rec_ml + rec * 2) = make_float2(-INFINITY, 0.f);
                continue;
            }
            // (the last score product of the piece before has been waited for: nothing reads the old query any more)
            if (!dead) {
                const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(p.q) + row_h * (DV + DR));
                uint4 x[(DV + T::DRP) / 8];
#pragma unroll
                for (int i = 0; i < (DV + T::DRP) / 8; ++i) x[i] = live && i * 8 < DV + DR ? __ldg(src + i) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < (DV + T::DRP) / 8; ++i) {
                    const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
                    tmem_st4_nowait(lane_base + T::COL_Q + i * 4, w);
                }
                tmem_st_wait();
                tc_fence_before();
            }
            mbar_arrive(q_ready);
            float m_run = -INFINITY, l_run = 0.f;       // softmax reference (log2 domain) and sum relative to it
            bool poison = false;
            for (int j = pc.lo; j < pc.hi; ++j, ++t) {
                const int st = t % NS, t0 = j * kTreeTile;
                if (!__all_sync(0xffffffffu, mbar_wait_spin(s_full(t), (t >> 1) & 1, s_abort))) { ok = false; break; }
                // (complete since before the score product; waited for by every thread because it also publishes the stage's flag)
                if (!__all_sync(0xffffffffu, mbar_wait_spin(kv_full(st), (t / NS) & 1, s_abort))) { ok = false; break; }
                const uint32_t flag = s_flag[st];
                const bool edge = t0 + kTreeTile > pc.s.ctx || flag != 0;            // the same for the whole block
                uint64_t bits = ~0ull;
                if (edge) {
                    // Value rows that P multiplies by 0 must not be NaN or infinite: those behind the end and of bad pages become zeros, and
                    // so do drafted tokens' rows with such an element (a row that sees one is made NaN at the end instead).
                    if (tid < kTreeTile) {
                        unsigned char *v = smem + st * T::STAGE_BYTES + tid * 128;
                        bool zero = t0 + tid >= pc.s.total || ((flag >> (tid >> 5)) & 1), bad = false;
                        if (!zero && t0 + tid >= pc.s.ctx) {
#pragma unroll
                            for (int bx = 0; bx < T::BOXES; ++bx)
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    const uint4 x = *reinterpret_cast<const uint4 *>(v + bx * T::VBOX_BYTES + i * 16);
                                    auto odd = [](uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; };
                                    bad |= odd(x.x) || odd(x.y) || odd(x.z) || odd(x.w);
                                }
                        }
                        if (zero || bad)
#pragma unroll
                            for (int bx = 0; bx < T::BOXES; ++bx)
#pragma unroll
                                for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4 *>(v + bx * T::VBOX_BYTES + i * 16) = make_uint4(0, 0, 0, 0);
                        const uint32_t all = __ballot_sync(0xffffffffu, bad);
                        if (lane == 0) s_bad[(t & 1) * 2 + warp] = all;              // (two sets: a slow reader of the tile before)
                    }
                    fence_async_smem();
                    asm volatile("bar.sync 1, 128;\n" ::: "memory");
                    if (live) {
                        bits = tree_window(p.mask + node * p.words, p.words, t0 - pc.s.ctx);
                        const int n = pc.s.total - t0;
                        if (n < kTreeTile) bits &= (1ull << n) - 1;
                        if (flag & 1) bits &= ~0xffffffffull;
                        if (flag & 2) bits &= 0xffffffffull;
                        poison |= (bits & (s_bad[(t & 1) * 2] | ((uint64_t)s_bad[(t & 1) * 2 + 1] << 32))) != 0;
                    }
                }
                if (dead) {                             // keeps the protocol going; nothing reads its rows
                    mbar_arrive(p_full(t));
                    continue;
                }
                tc_fence_after();
                const uint32_t s_addr = lane_base + T::COL_S + (t & 1) * kTreeTile;
                float s[kTreeTile];
                {
                    float lo[32], hi[32];
                    tmem_ld32_nowait(s_addr, lo);
                    tmem_ld32_nowait(s_addr + 32, hi);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 32; ++i) { s[i] = lo[i]; s[32 + i] = hi[i]; }
                }
                if (edge) {
                    const uint32_t b0 = (uint32_t)bits, b1 = (uint32_t)(bits >> 32);
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        s[i] = (b0 >> i) & 1 ? s[i] : -INFINITY;
                        s[32 + i] = (b1 >> i) & 1 ? s[32 + i] : -INFINITY;
                    }
                }
                uint32_t pk[kTreeTile / 2];
                float tile_sum = 0.f;
                auto weights = [&](float m_ref) {       // and their sum, relative to the reference
                    const float nm = m_ref == -INFINITY ? 0.f : -m_ref;              // nothing seen yet: all weights 0, not NaN
                    const uint64_t sc2 = f2_pack(p.scale_log2, p.scale_log2), nm2 = f2_pack(nm, nm);
                    uint64_t sum2[2] = {f2_pack(0.f, 0.f), f2_pack(0.f, 0.f)};
#pragma unroll
                    for (int i = 0; i < kTreeTile; i += 2) {
                        float a, b;
                        f2_unpack(f2_fma(f2_pack(s[i], s[i + 1]), sc2, nm2), a, b);
                        a = fast_exp2(a);
                        b = fast_exp2(b);
                        sum2[(i >> 1) & 1] = f2_add(sum2[(i >> 1) & 1], f2_pack(a, b));
                        pk[i >> 1] = pack_bf16(a, b);
                    }
                    float sa, sb;
                    f2_unpack(f2_add(sum2[0], sum2[1]), sa, sb);
                    tile_sum = sa + sb;
                };
                // As in the prefill kernel: weights against the present reference while the maximum is reduced; a tile whose maximum
                // exceeds it by more than 2^8 is done again.
                if (j > pc.lo) weights(m_run);
                float mx[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) mx[k] = max3(s[k], s[k + 4], s[k + 8]);
#pragma unroll
                for (int i = 12; i + 8 <= kTreeTile; i += 8)
#pragma unroll
                    for (int k = 0; k < 4; ++k) mx[k] = max3(mx[k], s[i + k], s[i + 4 + k]);
#pragma unroll
                for (int k = 0; k < 4; ++k) mx[k] = fmaxf(mx[k], s[kTreeTile - 4 + k]);
                const float m_tile = max3(mx[0], mx[1], fmaxf(mx[2], mx[3])) * p.scale_log2;
                const bool move = m_tile > m_run + kRescaleLog2;
                if (j == pc.lo || __any_sync(0xffffffffu, move)) {
                    float alpha = 1.f;
                    if (move) {
                        alpha = fast_exp2(m_run - m_tile);
                        l_run *= alpha;
                        m_run = m_tile;
                    }
                    if (j > pc.lo) {                    // the piece's O so far, once the value product before has landed
                        if (!__all_sync(0xffffffffu, mbar_wait_spin(kv_empty((t - 1) % NS), ((t - 1) / NS) & 1, s_abort))) { ok = false; break; }
                        tc_fence_after();
                        const uint64_t al2 = f2_pack(alpha, alpha);
#pragma unroll
                        for (int part = 0; part < DV / 32; ++part) {
                            float o[32];
                            tmem_ld32_nowait(o_addr + part * 32, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 32; i += 2) f2_unpack(f2_mul(f2_pack(o[i], o[i + 1]), al2), o[i], o[i + 1]);
                            tmem_st32(o_addr + part * 32, o);
                        }
                    }
                    weights(m_run);
                }
                tmem_st32u_nowait(s_addr, pk);
                l_run += tile_sum;
                tmem_st_wait();
                tc_fence_before();
                mbar_arrive(p_full(t));
            }
            if (ok && !__all_sync(0xffffffffu, mbar_wait_spin(o_full, n_pc & 1, s_abort))) ok = false;
            ++n_pc;
            if (!ok || dead) continue;
            tc_fence_after();
            if (poison) l_run = __int_as_float(0x7fc00000);
            const float inv = pc.rec < 0 ? tree_inverse(l_run) : 1.f;
#pragma unroll
            for (int part = 0; part < DV / 32; ++part) {
                float o[32];
                tmem_ld32_nowait(o_addr + part * 32, o);
                tmem_ld_wait();
                if (live) {
                    if (pc.rec < 0) {
                        uint4 *dst = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.out) + row_h * DV + part * 32);
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
                            dst[i / 8] = make_uint4(pack_bf16(o[i] * inv, o[i + 1] * inv), pack_bf16(o[i + 2] * inv, o[i + 3] * inv),
                                                    pack_bf16(o[i + 4] * inv, o[i + 5] * inv), pack_bf16(o[i + 6] * inv, o[i + 7] * inv));
                    } else {
                        float4 *dst = reinterpret_cast<float4 *>(p.rec_o + rec * DV + part * 32);
#pragma unroll
                        for (int i = 0; i < 32; i += 4) dst[i / 4] = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                    }
                }
            }
            if (live) {
                if (pc.rec >= 0) *reinterpret_cast<float2 *>(p.rec_ml + rec * 2) = make_float2(m_run, l_run);
                else if (p.lse) p.lse[row_h] = tree_lse(m_run, l_run);
            }
        }
        if (!ok && !*s_abort) {
            report_error(p.dev_status, GVA_ERR_TIMEOUT, pc.b);
            *s_abort = 1;
        }
        tc_fence_before();
    } else if (warp == 6) {
        // ==================================== loader: one lane issues, all look pages up ====================================
        const bool whole = p.P % kTreeTile == 0;        // a tile lies in one page; else its two halves do, each in its own
        const uint64_t stream = l2_policy_evict_first();
        while (ok && pieces.next(p, s_off, pc)) {
            for (int base = pc.lo; base < pc.hi && ok; base += 32) {
                int page0 = -1, page1 = -1;             // (-2: a half behind the sequence's end)
                if (base + lane < pc.hi) {
                    const int t0 = (base + lane) * kTreeTile;
                    auto look = [&](int at) {
                        const long long page = tree_page(p, pc.b, at / p.P);
                        return page < 0 || page >= p.num_pages ? -1 : (int)page;
                    };
                    page0 = look(t0);
                    if (!whole) page1 = t0 + 32 < pc.s.total ? look(t0 + 32) : -2;
                    if (page0 == -1 || (!whole && page1 == -1)) report_error(p.dev_status, GVA_ERR_BAD_PAGE, pc.b);
                }
                const int n = min(32, pc.hi - base);
                for (int i = 0; i < n && ok; ++i, ++t) {
                    const int pg0 = __shfl_sync(0xffffffffu, page0, i), pg1 = __shfl_sync(0xffffffffu, page1, i);
                    if (lane == 0) {
                        const int st = t % NS;
                        if (t >= NS) ok = mbar_wait_sleepy(kv_empty(st), ((t / NS) - 1) & 1, s_abort);
                        if (ok) {
                            const int at = ((base + i) * kTreeTile) % p.P;
                            const uint32_t dst = s_base + st * T::STAGE_BYTES;
                            s_flag[st] = whole ? (pg0 < 0 ? 3u : 0u) : (pg0 < 0 ? 1u : 0u) | (pg1 == -1 ? 2u : 0u);
                            const int boxes = (pg0 >= 0 ? 1 : 0) + (!whole && pg1 >= 0 ? 1 : 0);
                            const uint32_t bytes = (uint32_t)(T::V_BYTES + T::KR_BYTES) / (whole ? 1 : 2) * boxes;
                            if (boxes == 0) mbar_arrive(kv_full(st));
                            else mbar_expect_tx(kv_full(st), bytes);
                            auto fetch = [&](int page, int slot, int row) {
#pragma unroll
                                for (int bx = 0; bx < T::BOXES; ++bx)
                                    tma_load_2d_stream(dst + bx * T::VBOX_BYTES + row * 128, &tm_v, bx * 64, (page * p.G + g) * p.P + slot, kv_full(st), stream);
                                if constexpr (DR > 0) tma_load_2d(dst + T::V_BYTES + row * T::KR_ROW, &tm_k, 0, page * p.P + slot, kv_full(st));
                            };
                            if (pg0 >= 0) fetch(pg0, at, 0);
                            if (!whole && pg1 >= 0) fetch(pg1, (at + 32) % p.P, 32);
                        }
                    }
                    ok = __shfl_sync(0xffffffffu, ok, 0);
                }
            }
        }
        if (lane == 0) {
            if (!ok && !*s_abort) {
                report_error(p.dev_status, GVA_ERR_TIMEOUT, pc.b);
                *s_abort = 1;
            }
            // copies in flight must land before the block's shared memory is released
            for (int k = max(0, t - NS); k < t; ++k)
                for (int it = 0; it < kDrainPolls && !mbar_try_wait(kv_full(k % NS), (k / NS) & 1); ++it) {}
        }
    } else if (lane == 0) {
        // ======================================= MMA issuers: one thread per product =======================================
        constexpr uint32_t hi128 = (1024u >> 4) | (1u << 14) | ((uint32_t)kSwz128 << 29);        // (descriptors as in the prefill kernel)
        constexpr uint32_t hikr = ((8u * T::KR_ROW) >> 4) | (1u << 14) | ((uint32_t)(T::KR_ROW == 32 ? kSwz32 : kSwz64) << 29);
        constexpr uint32_t lo_k = (16u >> 4) << 16, lo_mn = ((uint32_t)T::VBOX_BYTES >> 4) << 16;
        const uint32_t a_st = (s_base & 0x3FFFFu) >> 4;
        auto mk = [](uint32_t lo, uint32_t hi) { return (uint64_t)lo | ((uint64_t)hi << 32); };
        int issued = 0;
        if (warp == 5) {
            constexpr uint32_t idesc = umma_idesc(kStripRows, kTreeTile, false);
            while (ok && pieces.next(p, s_off, pc)) {
                if (pc.lo >= pc.hi) continue;
                if (!mbar_wait_spin(q_ready, n_pc & 1, s_abort)) { ok = false; break; }
                ++n_pc;
                for (int j = pc.lo; j < pc.hi; ++j, ++t) {
                    // S[t & 1] also holds the weights of tile t - 2: its value product must have completed
                    if (!mbar_wait_spin(kv_full(t % NS), (t / NS) & 1, s_abort)) { ok = false; break; }
                    if (t >= 2 && !mbar_wait_spin(kv_empty((t - 2) % NS), ((t - 2) / NS) & 1, s_abort)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t vb = a_st + (uint32_t)(t % NS) * (T::STAGE_BYTES >> 4), d = tmem + T::COL_S + (t & 1) * kTreeTile;
#pragma unroll
                    for (int ks = 0; ks < KS_S; ++ks) {
                        const uint32_t off = ks < KS_V ? ((ks >> 2) * T::VBOX_BYTES + (ks & 3) * 32) >> 4 : (T::V_BYTES >> 4) + (uint32_t)(ks - KS_V) * 2;
                        umma_bf16_ts(d, tmem + T::COL_Q + ks * 8, mk((vb + off) | lo_k, ks < KS_V ? hi128 : hikr), idesc, ks > 0);
                    }
                    umma_commit(s_full(t));
                    issued = 1;
                }
            }
        } else {
            constexpr uint32_t idesc = umma_idesc(kStripRows, DV, true);
            while (ok && pieces.next(p, s_off, pc)) {
                if (pc.lo >= pc.hi) continue;
                for (int j = pc.lo; j < pc.hi; ++j, ++t) {
                    // every row has stored its weights of tile t and finished any rescaling of O
                    if (!mbar_wait_spin(p_full(t), (t >> 1) & 1, s_abort)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t vb = a_st + (uint32_t)(t % NS) * (T::STAGE_BYTES >> 4);
#pragma unroll
                    for (int ks = 0; ks < KS_O; ++ks)
                        umma_bf16_ts(tmem + T::COL_O, tmem + T::COL_S + (t & 1) * kTreeTile + ks * 8, mk((vb + ks * (16 * 128 >> 4)) | lo_mn, hi128), idesc,
                                     (j > pc.lo || ks > 0) ? 1u : 0u);
                    umma_commit(kv_empty(t % NS));
                    issued = 1;
                }
                if (ok) umma_commit(o_full);
            }
        }
        if (!ok && !*s_abort) {
            report_error(p.dev_status, GVA_ERR_TIMEOUT, pc.b);
            *s_abort = 1;
        }
        // nothing issued by this thread may still be running (or about to signal a barrier) when the block ends
        if (issued) {
            const uint32_t dr = warp == 5 ? drain_s : drain_o;
            umma_commit(dr);
            for (int it = 0; it < kDrainPolls * 16 && !mbar_try_wait(dr, 0); ++it) {}
        }
        tc_fence_before();
    }
    grid_dependency_launch();
    __syncthreads();
    if (warp == 5) {
        tc_fence_after();
        tmem_dealloc(tmem, T::TMEM_COLS);
    }
}

// ---- host ------------------------------------------------------------------------------------------------------
using TreeMmaFn = void (*)(TreeParams, CUtensorMap, CUtensorMap);
struct TreeMma {
    TreeMmaFn fn;
    int blocks_per_sm, drp;
    size_t fixed;                    // shared memory without the offsets of sequences
};
template <int DV, int DR>
TreeMma tree_mma_t() { return TreeMma{tree_mma_kernel<DV, DR>, TreeTraits<DV, DR>::BLOCKS_PER_SM, TreeTraits<DV, DR>::DRP, TreeTraits<DV, DR>::smem_bytes(0)}; }
inline TreeMma tree_mma(const gva_config &c) {
    if (c.d_v == 64) return c.d_r == 16 ? tree_mma_t<64, 16>() : c.d_r == 24 ? tree_mma_t<64, 24>() : tree_mma_t<64, 0>();
    return c.d_r == 32 ? tree_mma_t<128, 32>() : tree_mma_t<128, 0>();
}
// Maps of the values (boxes of 64 dims by a tile or half a tile) and of the positional keys.
inline bool tree_maps(const gva_config &c, const MmaHostState &st, const TreeParams &p, int drp, CUtensorMap *v, CUtensorMap *k) {
    const uint32_t rows = c.page_size % kTreeTile == 0 ? kTreeTile : kTreeTile / 2;
    if (!encode_map(st, v, p.v_pool, c.d_v, (uint64_t)p.num_pages * c.G * c.page_size, 64, rows, CU_TENSOR_MAP_SWIZZLE_128B)) return false;
    if (c.d_r == 0) {
        *k = *v;                     // (never used)
        return true;
    }
    return encode_map(st, k, p.kr_pool, c.d_r, (uint64_t)p.num_pages * c.page_size, drp, rows, drp == 16 ? CU_TENSOR_MAP_SWIZZLE_32B : CU_TENSOR_MAP_SWIZZLE_64B);
}

}  // namespace gva
