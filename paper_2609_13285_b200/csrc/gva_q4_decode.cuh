// Split-KV decode over the 4-bit cache on the tensor cores (mma.sync m16n8k16, f16 in, f32 accumulate).
//
// With value = z + s c (gva_q4.cuh) the score of token t and its share of the output are
//     q . v_t = s_t (q . c_t) + z_t sum(q),          sum_t p_t v_t = sum_t (p_t s_t) c_t + sum_t p_t z_t,
// so the products run over the codes and step and lowest come in afterwards, per token, in f32.
//
// Codes as MMA operands.  Score: four bits in the middle of a 16-bit half word, the rest zero, are an f16 subnormal, c 2^-22 at bits 2
// to 5 and c 2^-18 at bits 6 to 9.  Two shifts and four masks widen a word of eight codes, and the powers of two are undone
// in the query.  Tensor cores multiply subnormals exactly but align products by their nominal exponent 2^-14, which costs
// the sum as many of its bits as the code stands below: 8 and 4 here (without the shift up, at bits 0 and 4, a score
// was off by 8e-7, rms).  The output cannot take that, nor the offset of codes that are all positive, which over T tokens
// cancels to T^-1/2 of its size (3e-5 measured).  So there the codes are centred, c - 8, and made normal numbers: one
// subtraction per two codes more, and
//     sum_t p_t v_t = sum_t (p_t s_t) (c_t - 8) + sum_t p_t (z_t + 8 s_t).
//
// Both products need the contraction index in pairs inside a register: dims for the score, tokens for the output.  A lane
// therefore reads the tile twice, as whole words: for the score the d_v / 4 dims [c d_v / 4, ...) of its two token rows
// (c = lane % 4), for the output eight dims of four tokens, whose words two byte permutes interleave into token pairs.  The
// order of dims inside the score's contraction and of dims over the output's rows is free, so no transposing load is needed.
// Tokens stand in the order rowmap() in both, which keeps the two access patterns free of bank conflicts for d_v = 64.
//
// Precision: query and softmax weight enter as two f16 numbers (hi + lo, the 4 heads x 2 are the 8 MMA columns), each scaled
// by a power of two so that neither overflows nor loses bits to f16's range: per head for the query, and for the weights
// p s by the largest step seen so far, which is followed like the running maximum.
//
// Blocks.  One block per SM streams a contiguous range of tiles through a ring of bulk copies: up to four producer warps, and
// teams of G consumer warps, one warp per group, 12 to 16 consumers in all.  Team k takes tiles k, k + teams, ..., keeps its own
// running softmax and writes its own partial records, so results do not depend on who is faster; a team that the
// scheduler favours meets the end of the ring and waits there for the others, which evens them out (four blocks per SM with
// equal ranges each ended between 45 and 69 us on the 1 M token batch, median 57).  All waits are bounded.
#pragma once

#include "gva_decode_mma.cuh"
#include "gva_q4.cuh"

namespace gva {

template <int DV_, int DR_, int TILE_>
struct Q4Traits {
    static constexpr int DV = DV_, DR = DR_, TILE = TILE_;
    static constexpr int ROW = DV / 2;                       // bytes of codes per token and group
    static constexpr int V_BYTES = TILE * ROW, SZ_BYTES = TILE * 4, KR_ROW = DR * 2, KR_BYTES = TILE * KR_ROW;
    static constexpr int WORDS = DV / 32;                    // words of a row a lane takes for the score: two k-steps each
    static constexpr int KSTEPS = DV / 16;
    static constexpr int MT = DV / 16;
    static constexpr int CHUNKS = TILE / 16;
    static constexpr int DQ = DV + DR;
    __host__ __device__ static constexpr int stage_bytes(int G) { return G * (V_BYTES + SZ_BYTES) + KR_BYTES; }
    __host__ __device__ static constexpr int tail_bytes(int B, int nstage) { return nstage * 32 + 16 + (B + 1) * 4; }
};

__device__ __forceinline__ int rowmap(int r) { return r ^ ((r >> 2) & 1); }

// A copy of whole 16-byte pieces that nobody else reads: evict-first in L2.
__device__ __forceinline__ void bulk_load_stream(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar, uint64_t pol) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;\n" ::"r"(dst),
        "l"(src), "r"(bytes), "r"(bar), "l"(pol)
        : "memory");
}
__device__ __forceinline__ void mma_f16_q4(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// c = a b from nothing
__device__ __forceinline__ void mma_f16_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_bf16_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t pack_half2(float x, float y) {
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// (x0, x1) -> {hi, lo} f16 pairs of each
__device__ __forceinline__ void split_pair_f16(float x0, float x1, uint32_t &s0, uint32_t &s1) {
    const __half2 h = __floats2half2_rn(x0, x1);
    const float2 f = __half22float2(h);
    const uint32_t hu = *reinterpret_cast<const uint32_t *>(&h), lu = pack_half2(x0 - f.x, x1 - f.y);
    s0 = __byte_perm(hu, lu, 0x5410);
    s1 = __byte_perm(hu, lu, 0x7632);
}
// hi (part 0) or lo (part 1) of x as f16 bits; hi, mid, lo (part 2) as bf16 bits
__device__ __forceinline__ uint32_t part_f16(float x, int part) {
    const __half hi = __float2half_rn(x);
    return __half_as_ushort(part ? __float2half_rn(x - __half2float(hi)) : hi);
}
__device__ __forceinline__ uint32_t part_bf16(float x, int part) {
    __nv_bfloat16 y = __float2bfloat16_rn(x);
    for (int i = 0; i < part; ++i) {
        x -= __bfloat162float(y);
        y = __float2bfloat16_rn(x);
    }
    return __bfloat16_as_ushort(y);
}

__device__ __forceinline__ uint32_t and_or(uint32_t x, uint32_t mask, uint32_t bits) {      // one instruction, its constants in registers
    uint32_t y;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;\n" : "=r"(y) : "r"(x), "r"(mask), "r"(bits));
    return y;
}
// Two codes as signed f16 numbers c - 8: 1024 + c (or 64 + c, one nibble up) by masks, less 1032 (72), exactly.
__device__ __forceinline__ uint32_t centred_low(uint32_t x) {
    const uint32_t y = and_or(x, 0x000f000fu, 0x64006400u), off = 0x64086408u;
    const __half2 d = __hsub2(*reinterpret_cast<const __half2 *>(&y), *reinterpret_cast<const __half2 *>(&off));
    return *reinterpret_cast<const uint32_t *>(&d);
}
__device__ __forceinline__ uint32_t centred_high(uint32_t x) {
    const uint32_t y = and_or(x, 0x00f000f0u, 0x54005400u), off = 0x54805480u;
    const __half2 d = __hsub2(*reinterpret_cast<const __half2 *>(&y), *reinterpret_cast<const __half2 *>(&off));
    return *reinterpret_cast<const uint32_t *>(&d);
}

constexpr uint32_t kCodeLow = 0x003c003cu, kCodeHigh = 0x03c003c0u;

// One group's four queries as the score product's B fragments, for the MMA column n = lane / 4 = 2 head + {hi, lo}, scaled
// by `factor` (softmax scale and log2 e).  Content: q 2^-e 2^10 with |q 2^-e| <= 1, times 16 where the code stands in the low
// nibble; unscale = 2^(e + 8) of the head whose scores this lane holds (lane % 4); sum = sum of that head's content query.
// Position: the keys are bf16 and so are the query's parts, of which two carry 16 bits only (2^-17 of every term); the third
// stands in r2, in the hi columns, for one more MMA per 16 tokens.
template <class T>
struct Q4Query {
    uint32_t v[T::KSTEPS][2];
    uint32_t r[T::DR > 0 ? (T::DR + 15) / 16 : 1][2], r2[T::DR > 0 ? (T::DR + 15) / 16 : 1][2];
    float unscale, sum;
};
template <class T>
__device__ __forceinline__ void load_q4_query(Q4Query<T> &out, const float *q /* first of the group's four heads */, float factor, int lane) {
    const int n = lane >> 2, c = lane & 3, head = n >> 1, part = n & 1;
    const float *src = q + (size_t)head * T::DQ;
    float v[T::DV / 4];
    float top = 0.f, sum = 0.f;
#pragma unroll
    for (int i = 0; i < T::DV / 16; ++i) {                   // dims c DV / 4 + 4 i ..
        const float4 x = *reinterpret_cast<const float4 *>(src + c * (T::DV / 4) + 4 * i);
        v[4 * i] = x.x * factor; v[4 * i + 1] = x.y * factor; v[4 * i + 2] = x.z * factor; v[4 * i + 3] = x.w * factor;
    }
#pragma unroll
    for (int i = 0; i < T::DV / 4; ++i) {
        top = fmaxf(top, fabsf(v[i]));
        sum += v[i];
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));  // over the four lanes that share this column
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    // 2^e >= top, with e held inside what keeps 2^-e 2^14 and 2^(e + 8) finite
    int e = (int)((__float_as_uint(top) >> 23) & 255u) - 126;
    e = min(max(e, -100), 110);
    const float down = __uint_as_float((uint32_t)(127 - e + 10) << 23), down16 = 16.f * down;
#pragma unroll
    for (int w = 0; w < T::WORDS; ++w) {
        const float *x = v + 8 * w;
        out.v[2 * w][0] = part_f16(x[0] * down16, part) | (part_f16(x[4] * down16, part) << 16);
        out.v[2 * w][1] = part_f16(x[1] * down, part) | (part_f16(x[5] * down, part) << 16);
        out.v[2 * w + 1][0] = part_f16(x[2] * down16, part) | (part_f16(x[6] * down16, part) << 16);
        out.v[2 * w + 1][1] = part_f16(x[3] * down, part) | (part_f16(x[7] * down, part) << 16);
    }
    // from the column's lanes to the lanes that hold the head's scores: lane % 4 = head, columns 2 head and 2 head + 1 alike
    const float up = __uint_as_float((uint32_t)(127 + e + 8) << 23);       // c 2^-22 x q 2^-e 2^14 = c q 2^-(e + 8)
    out.unscale = __shfl_sync(0xffffffffu, up, 8 * c);
    out.sum = __shfl_sync(0xffffffffu, sum, 8 * c);
    if constexpr (T::DR > 0) {
        const float *r = src + T::DV;
        constexpr int FULL = T::DR / 16;
        auto pair = [&](const float *x, int pt) { return part_bf16(x[0] * factor, pt) | (part_bf16(x[1] * factor, pt) << 16); };
#pragma unroll
        for (int k = 0; k < FULL; ++k) {
            const float *x = r + 16 * k + 2 * c;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                out.r[k][i] = pair(x + 8 * i, part);
                out.r2[k][i] = part ? 0u : pair(x + 8 * i, 2);
            }
        }
        if constexpr (T::DR % 16 == 8) {
            const float *x = r + 16 * FULL + 2 * c;
            out.r[FULL][0] = pair(x, part);
            out.r2[FULL][0] = part ? 0u : pair(x, 2);
        }
    }
}

// Content and positional products of two 16-token chunks with one group's queries, side by side so that neither waits for the
// other's MMAs.  acc: codes (to be multiplied by unscale and the token's step), rot: positional part, in f32; columns hi and
// lo of head lane % 4 in [0], [1] for token row rowmap(lane / 4) and in [2], [3] for that row + 8.  v: this lane's share of the
// first chunk's low token row; kr: shared-memory address of the lane's row and piece of the first chunk (kr_lane()).
template <class T>
__device__ __forceinline__ uint32_t kr_lane(int lane) {      // matrices: (low rows | high rows) x (first | second 16 bytes)
    return (uint32_t)((rowmap(lane & 7) + 8 * ((lane >> 3) & 1)) * T::KR_ROW + 16 * (lane >> 4));
}
template <class T>
__device__ __forceinline__ void score_q4(const unsigned char *v, uint32_t kr, const Q4Query<T> &q, float (&acc)[2][4], float (&rot)[2][4]) {
    uint32_t lo[2][T::WORDS], hi[2][T::WORDS];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const unsigned char *row = v + k * 16 * T::ROW;
#pragma unroll
        for (int w = 0; w < T::WORDS; w += 2) {
            const uint2 a = *reinterpret_cast<const uint2 *>(row + 4 * w), b = *reinterpret_cast<const uint2 *>(row + 8 * T::ROW + 4 * w);
            lo[k][w] = a.x; lo[k][w + 1] = a.y; hi[k][w] = b.x; hi[k][w + 1] = b.y;
        }
    }
    if constexpr (T::DR == 0) {
#pragma unroll
        for (int k = 0; k < 2; ++k) rot[k][0] = rot[k][1] = rot[k][2] = rot[k][3] = 0.f;
    } else {
        constexpr int FULL = T::DR / 16;
        uint32_t f[2][FULL][4];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int u = 0; u < FULL; ++u) ldsm_x4(kr + k * 16 * T::KR_ROW + 32 * u, f[k][u]);
#pragma unroll
        for (int u = 0; u < FULL; ++u)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (u == 0) mma_bf16_first(rot[k], f[k][u], q.r2[u][0], q.r2[u][1]);
                else mma_bf16(rot[k], f[k][u], q.r2[u][0], q.r2[u][1]);
            }
        if constexpr (T::DR % 16 == 8) {                     // the last 8 dims lie apart
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uint32_t t[2];
                ldsm_x2(kr + k * 16 * T::KR_ROW + 32 * FULL, t);             // lanes 0 .. 15 give the rows
                mma_bf16_k8(rot[k], t, q.r2[FULL][0]);
                mma_bf16_k8(rot[k], t, q.r[FULL][0]);
            }
        }
#pragma unroll
        for (int u = 0; u < FULL; ++u)
#pragma unroll
            for (int k = 0; k < 2; ++k) mma_bf16(rot[k], f[k][u], q.r[u][0], q.r[u][1]);
    }
#pragma unroll
    for (int w = 0; w < T::WORDS; ++w) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t l = lo[k][w] << 2, h = hi[k][w] << 2;
            const uint32_t a0 = l & kCodeLow, a1 = h & kCodeLow, a2 = l & kCodeHigh, a3 = h & kCodeHigh;
            if (w == 0) mma_f16_first(acc[k], a0, a1, a2, a3, q.v[2 * w][0], q.v[2 * w][1]);
            else mma_f16_q4(acc[k], a0, a1, a2, a3, q.v[2 * w][0], q.v[2 * w][1]);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t l = lo[k][w] >> 6, h = hi[k][w] >> 6;
            mma_f16_q4(acc[k], l & kCodeLow, h & kCodeLow, l & kCodeHigh, h & kCodeHigh, q.v[2 * w + 1][0], q.v[2 * w + 1][1]);
        }
    }
}

// The producer's wait for a free slot of the ring: it is ahead by the whole ring and polls without hurry, so as to leave the
// issue slots to the consumers (measured: a tenth of all instructions were its polls).  Bounded like mbar_wait_bounded.
__device__ __forceinline__ bool mbar_wait_relaxed(uint32_t bar, uint32_t parity, volatile int *abort_flag) {
    const unsigned long long t0 = global_timer_ns();
    for (;;) {
        uint32_t ok;
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}\n"
            : "=r"(ok)
            : "r"(bar), "r"(parity), "r"(100000u)            // may sleep in hardware for 100 us
            : "memory");
        if (ok) return true;
        if (*abort_flag || global_timer_ns() - t0 > kWaitLimitNs) return false;
    }
}

// What the producer tells the consumers about a stage.
struct TileMeta {
    int b, t0, n_valid, len;     // sequence, first slot, live tokens (none if the page is bad), tokens of the sequence
};

// One of `n_producers` producer warps: takes every n_producers-th of the flat tiles [lo, hi), 32 look-ups at a time (a lane
// each), and fills their slots of the ring.  nstage is a multiple of n_producers, so that a slot is always filled by the same warp:
// the parity that a wait goes by tells a slot's turn from the one before, not from the one before that.  copy(stage, page, first slot, full barrier, lane) starts the copies, any lane any of
// them; bytes = what they add up to.  (One warp needs about 1050 cycles a tile -- the issue of a bulk copy is slow, not
// its flight -- against some 600 that sixteen consumer warps need: 89 us on the 1 M token batch.)
template <int TILE, class Copy>
__device__ __forceinline__ void produce_tiles(int producer, int n_producers, int nstage, const int *s_off, const int32_t *seq_lens,
                                              const int32_t *block_table, int B, int P, int num_pages, int max_pages, int32_t *dev_status, int lo,
                                              int hi, uint64_t *full_bar, uint64_t *empty_bar, TileMeta *s_meta, volatile int *s_abort,
                                              uint32_t bytes, Copy copy) {
    const int lane = threadIdx.x & 31, n_mine = (hi - lo - producer + n_producers - 1) / n_producers;
    int issued = 0, st = producer, parity = 1;               // slot; parity of its empty barrier's phase to wait for
    bool ok = true;
    for (int base = 0; base < n_mine && ok; base += 32) {
        const int f = lo + producer + (base + lane) * n_producers;
        int b = 0, t0 = 0, n_valid = 0, len = 0;
        long long page = 0;
        if (f < hi) {
            b = seq_of_tile(s_off, B, f);
            t0 = (f - s_off[b]) * TILE;
            len = seq_lens[b];
            page = block_table ? (long long)block_table[(size_t)b * max_pages + t0 / P] : (long long)b * max_pages + t0 / P;
            n_valid = min(TILE, len - t0);
            if (page < 0 || page >= num_pages) {
                report_error(dev_status, GVA_ERR_BAD_PAGE, b);
                page = 0;                                    // there is one; what is read of it counts for nothing
                n_valid = 0;
            }
        }
        const int slot = t0 % P, n = min(32, n_mine - base);
        for (int i = 0; i < n; ++i, ++issued) {
            const int pg = (int)__shfl_sync(0xffffffffu, (int)page, i), sl = __shfl_sync(0xffffffffu, slot, i);
            const int t = __shfl_sync(0xffffffffu, t0, i), nv = __shfl_sync(0xffffffffu, n_valid, i), bb = __shfl_sync(0xffffffffu, b, i), ln = __shfl_sync(0xffffffffu, len, i);
            const uint32_t bar = smem_u32(&full_bar[st]);
            int good = 1;
            if (lane == 0) {
                if (mbar_wait_relaxed(smem_u32(&empty_bar[st]), parity, s_abort)) {
                    s_meta[st] = TileMeta{bb, t, nv, ln};
                    mbar_expect_tx(bar, bytes);
                } else {
                    if (!*s_abort) report_error(dev_status, GVA_ERR_TIMEOUT, bb);
                    *s_abort = 1;
                    good = 0;
                }
            }
            good = __shfl_sync(0xffffffffu, good, 0);
            if (!good) {
                ok = false;
                break;
            }
            copy(st, (size_t)pg, sl, bar, lane);
            st += n_producers;
            if (st >= nstage) {
                st -= nstage;
                parity ^= 1;
            }
        }
    }
    if (!ok && lane == 0) {                                  // every copy in flight must land before the shared memory is released
        for (int i = max(0, issued - nstage / n_producers); i < issued; ++i) {
            const int at = producer + i * n_producers;
            for (int it = 0; it < kDrainPolls; ++it)
                if (mbar_try_wait(smem_u32(&full_bar[at % nstage]), (at / nstage) & 1)) break;
        }
    }
}

// The copies of one 4-bit tile into a stage: value rows of every group, their (step, lowest) pairs, positional rows.  A page
// that is one tile has all groups side by side: one copy each.
template <class T>
__device__ __forceinline__ void copy_q4_tile(uint32_t base, const Q4Pools &c, int G, int P, size_t page, int slot, uint32_t bar, uint64_t pol, int lane) {
    if (P == T::TILE) {
        if (lane == 0) bulk_load_stream(base, c.v + page * G * T::V_BYTES, G * T::V_BYTES, bar, pol);
        if (lane == 1) bulk_load_stream(base + G * T::V_BYTES, c.sz + page * G * T::TILE, G * T::SZ_BYTES, bar, pol);
    } else if (lane < G) {
        bulk_load_stream(base + lane * T::V_BYTES, c.v + ((page * G + lane) * P + slot) * T::ROW, T::V_BYTES, bar, pol);
    } else if (lane < 2 * G) {
        const int g = lane - G;
        bulk_load_stream(base + G * T::V_BYTES + g * T::SZ_BYTES, c.sz + (page * G + g) * P + slot, T::SZ_BYTES, bar, pol);
    }
    if (T::DR > 0 && lane == 31)
        bulk_load_stream(base + G * (T::V_BYTES + T::SZ_BYTES), c.kr + (page * P + slot) * T::DR, T::KR_BYTES, bar, pol);
}

// What the launch adds to DecodeParams.
struct Q4Launch {
    Q4Pools pools;
    int teams, producers, nstage;   // nstage: a multiple of both, see produce_tiles (a team likewise finds only its own tiles in a slot)
    int2 *segments;              // per sequence: first record group and their number, for the merge (balanced partition only)
};
constexpr int kQ4Producers = 4;           // producer warps of a block at most
// Consumer warps of a block at most: 12, which leaves a thread 128 registers, where that is three teams or more, else 16 with 96
// (1 M tokens, G = 4: 66.3 us with 12, 67.8 with 16, 75.4 with 8; 0.55 M tokens of wide heads, G = 8: 142.7 with 8, 136.7 with 16).
__host__ __device__ constexpr int q4_consumers(int d_v, int G) { return d_v == 64 && G <= 4 ? 12 : 16; }

template <int DV, int DR, int TILE, int CONSUMERS>
__global__ void __launch_bounds__(32 * (CONSUMERS + kQ4Producers), 1)
decode_q4_kernel(DecodeParams p, Q4Launch L) {
    using T = Q4Traits<DV, DR, TILE>;
    grid_dependency_launch();
    extern __shared__ __align__(128) unsigned char smem[];
    const int G = p.G, H = p.H, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, nstage = L.nstage;
    const int stage_bytes = T::stage_bytes(G);
    unsigned char *tail = smem + (size_t)nstage * stage_bytes;
    uint64_t *full_bar = reinterpret_cast<uint64_t *>(tail), *empty_bar = full_bar + nstage;
    TileMeta *s_meta = reinterpret_cast<TileMeta *>(empty_bar + nstage);
    volatile int *s_abort = reinterpret_cast<volatile int *>(s_meta + nstage);
    int *s_off = reinterpret_cast<int *>(s_meta + nstage) + 4;
    if (tid == 0) {
        for (int s = 0; s < nstage; ++s) {
            mbar_init(smem_u32(&full_bar[s]), 1);
            mbar_init(smem_u32(&empty_bar[s]), G);
        }
        *s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    grid_dependency_wait();
    compute_tile_offsets<TILE>(p, s_off);                    // ends with a barrier
    const BlockRange rg = block_range(p, s_off);
    if (L.segments && blockIdx.x == 0) {
        const int total = s_off[p.B], n_eff = partitions_in_use(total, gridDim.x);
        for (int b = tid; b < p.B; b += blockDim.x) {
            int2 seg = make_int2(0, 0);
            if (s_off[b + 1] > s_off[b]) {
                const int c0 = range_owner(s_off[b], total, n_eff), c1 = range_owner(s_off[b + 1] - 1, total, n_eff);
                seg = make_int2(c0 + b, c1 - c0 + 1);
            }
            L.segments[b] = seg;
        }
    }
    // the result itself is written where a block has the whole sequence and one team
    const bool direct = p.num_splits == 1;
    if (rg.lo >= rg.hi) {
        if (p.num_splits > 0) {                              // an empty split
            const int b = blockIdx.x / p.num_splits;
            if (direct) {
                for (int i = tid; i < H * DV; i += blockDim.x) p.out[(size_t)b * H * DV + i] = 0.f;
                if (p.lse)
                    for (int i = tid; i < H; i += blockDim.x) p.lse[(size_t)b * H + i] = -INFINITY;
            } else {
                for (int i = tid; i < H; i += blockDim.x) *reinterpret_cast<float2 *>(p.rec_ml + ((size_t)rg.rec_fixed * H + i) * 2) = make_float2(-INFINITY, 0.f);
            }
        }
        return;
    }
    if (warp >= G * L.teams) {
        const uint64_t pol = l2_policy_evict_first();
        produce_tiles<TILE>(warp - G * L.teams, L.producers, nstage, s_off, p.seq_lens, p.block_table, p.B, p.P, p.num_pages, p.max_pages, p.dev_status, rg.lo, rg.hi,
                            full_bar, empty_bar, s_meta, s_abort, (uint32_t)stage_bytes,
                            [&](int st, size_t page, int slot, uint32_t bar, int ln) {
                                copy_q4_tile<T>(smem_u32(smem + (size_t)st * stage_bytes), L.pools, G, p.P, page, slot, bar, pol, ln);
                            });
    } else {
        const int team = warp / G, g = warp - team * G, c = lane & 3, r8 = lane >> 2;
        const int tok_lo = rowmap(r8), tok_hi = tok_lo + 8;
        const int ta = rowmap(2 * c), tb = rowmap(2 * c + 1);            // tokens of the output product's k = 2 c, 2 c + 1 (+ 8)
        const int head = g * kHeadsPerGroup + c;
        Q4Query<T> q;
        float oacc[T::MT][4];
        float m_run = -INFINITY, l_run = 0.f, z_run = 0.f, step_ref = 0.f, lift = 0.f;   // all sums carry the factor 2^lift
        int cur_b = -1, next_b = rg.b_first;                 // sequence in hand; first one this team has not accounted for yet
        auto record = [&](int b) { return (size_t)((rg.rec_fixed >= 0 ? rg.rec_fixed : (int)blockIdx.x + b) * L.teams + team) * H + head; };
        // this team's part of the sequence in hand: one partial record, or the result
        auto flush = [&]() {
            float l = l_run, z = z_run;
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
                l += __shfl_xor_sync(0xffffffffu, l, o);
                z += __shfl_xor_sync(0xffffffffu, z, o);
            }
            const size_t at = direct ? (size_t)cur_b * H + head : record(cur_b);
            const float norm = direct ? (l != 0.f ? 1.f / l : 0.f) : fast_exp2(-lift);               // (a power of two: exact)
            float *dst = (direct ? p.out : p.rec_o) + at * DV;
#pragma unroll
            for (int h = 0; h < DV / 64; ++h) {
                float o[8];
#pragma unroll
                for (int mt = 0; mt < 4; ++mt) {             // rows r8 and r8 + 8 of m-tile mt: dims 8 word + 2 mt and + 1
                    o[2 * mt] = (oacc[4 * h + mt][0] + oacc[4 * h + mt][1] + z) * norm;
                    o[2 * mt + 1] = (oacc[4 * h + mt][2] + oacc[4 * h + mt][3] + z) * norm;
                }
                *reinterpret_cast<float4 *>(dst + 64 * h + 8 * r8) = make_float4(o[0], o[1], o[2], o[3]);
                *reinterpret_cast<float4 *>(dst + 64 * h + 8 * r8 + 4) = make_float4(o[4], o[5], o[6], o[7]);
            }
            if (r8 == 0) {
                if (!direct) *reinterpret_cast<float2 *>(p.rec_ml + at * 2) = make_float2(m_run, l * norm);
                else if (p.lse) p.lse[at] = (m_run + (log2f(l) - lift)) * kLn2;
            }
        };
        // sequences [next_b, to) of the block's range of which this team got no tile
        auto mark_empty = [&](int to) {
            for (; next_b < to; ++next_b)
                if (r8 == 0) *reinterpret_cast<float2 *>(p.rec_ml + record(next_b) * 2) = make_float2(-INFINITY, 0.f);
        };
        auto begin = [&](int b) {                            // sequence b is in hand from here
            if (!direct) mark_empty(b);
            cur_b = b;
            next_b = b + 1;
            load_q4_query<T>(q, p.q + ((size_t)b * H + g * kHeadsPerGroup) * T::DQ, p.scale_log2, lane);
            m_run = -INFINITY;
            l_run = z_run = step_ref = lift = 0.f;
#pragma unroll
            for (int mt = 0; mt < T::MT; ++mt)
#pragma unroll
                for (int e = 0; e < 4; ++e) oacc[mt][e] = 0.f;
        };
        const int n_tiles = rg.hi - rg.lo;
        if (team < n_tiles) begin(seq_of_tile(s_off, p.B, rg.lo + team));    // its query is fetched while the first tiles fly
#pragma unroll 1
        for (int i = team, st = team, parity = 0; i < n_tiles; i += L.teams) {
            if (!mbar_wait_bounded(smem_u32(&full_bar[st]), parity, s_abort)) {
                if (!*s_abort && lane == 0) report_error(p.dev_status, GVA_ERR_TIMEOUT, cur_b);
                *s_abort = 1;
                break;
            }
            const TileMeta meta = s_meta[st];
            if (meta.b != cur_b) {
                flush();
                begin(meta.b);
            }
            const unsigned char *stage = smem + (size_t)st * stage_bytes;
            const unsigned char *vt = stage + (size_t)g * T::V_BYTES;
            const __half2 *szt = reinterpret_cast<const __half2 *>(stage + (size_t)G * T::V_BYTES + (size_t)g * T::SZ_BYTES);
            const uint32_t krt = smem_u32(stage + (size_t)G * (T::V_BYTES + T::SZ_BYTES)) + kr_lane<T>(lane);

            // ---- scores (log2 units) of this lane's head and token rows ----
            float x[T::CHUNKS][2], step[T::CHUNKS][2], mid[T::CHUNKS][2];
            float top = -INFINITY, smax = 0.f;
#pragma unroll
            for (int kk = 0; kk < T::CHUNKS; kk += 2) {
                float acc[2][4], rot[2][4];
                score_q4<T>(vt + (kk * 16 + tok_lo) * T::ROW + c * (T::ROW / 4), krt + kk * 16 * T::KR_ROW, q, acc, rot);
#pragma unroll
                for (int k = kk; k < kk + 2; ++k) {
                    const float2 a = __half22float2(szt[k * 16 + tok_lo]), b = __half22float2(szt[k * 16 + tok_hi]);
                    const float *s = acc[k - kk], *r = rot[k - kk];
                    step[k][0] = a.x; mid[k][0] = fmaf(8.f, a.x, a.y); step[k][1] = b.x; mid[k][1] = fmaf(8.f, b.x, b.y);
                    x[k][0] = fmaf((s[0] + s[1]) * q.unscale, a.x, fmaf(a.y, q.sum, r[0] + r[1]));
                    x[k][1] = fmaf((s[2] + s[3]) * q.unscale, b.x, fmaf(b.y, q.sum, r[2] + r[3]));
                }
            }
            if (meta.n_valid < TILE) {                       // (what stands behind the sequence may be anything)
#pragma unroll
                for (int k = 0; k < T::CHUNKS; ++k) {
                    if (k * 16 + tok_lo >= meta.n_valid) { x[k][0] = -INFINITY; step[k][0] = mid[k][0] = 0.f; }
                    if (k * 16 + tok_hi >= meta.n_valid) { x[k][1] = -INFINITY; step[k][1] = mid[k][1] = 0.f; }
                }
            }
#pragma unroll
            for (int k = 0; k < T::CHUNKS; ++k) {
                top = fmaxf(top, fmaxf(x[k][0], x[k][1]));
                smax = fmaxf(smax, fmaxf(step[k][0], step[k][1]));
            }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
            const float m_new = fmaxf(m_run, top);
            if (__any_sync(0xffffffffu, m_new != m_run || smax > step_ref)) {    // rare once maximum and largest step have settled
                float f = m_run == -INFINITY ? 0.f : fast_exp2(m_run - m_new);
                const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(smax));     // steps are not negative
                if (__uint_as_float(most) > step_ref) {
                    const int e = min(max((int)(most >> 23) - 126, -30), 60);                    // 2^e > the largest step
                    const float to = (float)(10 - e);
                    f *= fast_exp2(to - lift);
                    lift = to;
                    step_ref = __uint_as_float((uint32_t)(127 + e) << 23);
                }
                l_run *= f;
                z_run *= f;
#pragma unroll
                for (int mt = 0; mt < T::MT; ++mt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) oacc[mt][e] *= f;
            }
            m_run = m_new;
            const float base = m_new != -INFINITY ? m_new - lift : 0.f;          // keeps (-inf) - (-inf) out of the exponent

            // ---- softmax weights times steps, as B fragments of the output product ----
            uint32_t pb0[T::CHUNKS], pb1[T::CHUNKS];
#pragma unroll
            for (int k = 0; k < T::CHUNKS; ++k) {
                const float p0 = fast_exp2(x[k][0] - base), p1 = fast_exp2(x[k][1] - base);
                l_run += p0 + p1;
                z_run = fmaf(p0, mid[k][0], fmaf(p1, mid[k][1], z_run));
                uint32_t s0, s1;
                split_pair_f16(p0 * step[k][0], p1 * step[k][1], s0, s1);
                pb0[k] = movmatrix_trans(s0);
                pb1[k] = movmatrix_trans(s1);
            }
            // ---- O^T += C_tile^T . (P s)^T.  A tile's products are summed from nothing and added to the running output in f32: the
            //      MMA's own accumulation truncates, which over hundreds of steps came to 1.3e-6 of an output whose terms cancel ----
#pragma unroll
            for (int h = 0; h < DV / 64; ++h) {              // words lane / 4 and, for d_v = 128, lane / 4 + 8
                uint32_t half[2][T::CHUNKS][2];              // [low | high half words][chunk][pair of tokens], interleaved by token
#pragma unroll
                for (int k = 0; k < T::CHUNKS; ++k)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const unsigned char *row = vt + k * 16 * T::ROW + r8 * 4 + 32 * h;
                        const uint32_t w0 = *reinterpret_cast<const uint32_t *>(row + (ta + 8 * u) * T::ROW);
                        const uint32_t w1 = *reinterpret_cast<const uint32_t *>(row + (tb + 8 * u) * T::ROW);
                        half[0][k][u] = __byte_perm(w0, w1, 0x5410);
                        half[1][k][u] = __byte_perm(w0, w1, 0x7632);
                    }
#pragma unroll
                for (int u = 0; u < 4; u += 2) {             // dims 8 word + 2 u .. + 2 u + 3
                    float acc[2][4];
#pragma unroll
                    for (int k = 0; k < T::CHUNKS; ++k)
#pragma unroll
                        for (int v = 0; v < 2; ++v) {
                            const uint32_t e0 = half[u / 2][k][0], e1 = half[u / 2][k][1], f0 = v ? e0 >> 8 : e0, f1 = v ? e1 >> 8 : e1;
                            if (k == 0) mma_f16_first(acc[v], centred_low(f0), centred_high(f0), centred_low(f1), centred_high(f1), pb0[k], pb1[k]);
                            else mma_f16_q4(acc[v], centred_low(f0), centred_high(f0), centred_low(f1), centred_high(f1), pb0[k], pb1[k]);
                        }
#pragma unroll
                    for (int v = 0; v < 2; ++v)
#pragma unroll
                        for (int e = 0; e < 4; ++e) oacc[4 * h + u + v][e] += acc[v][e];
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&empty_bar[st]));
            st += L.teams;
            if (st >= nstage) {
                st -= nstage;
                parity ^= 1;
            }
        }
        if (cur_b >= 0) flush();
        if (!direct) mark_empty(rg.rec_fixed >= 0 ? (cur_b < 0 ? rg.b_first + 1 : next_b) : seq_of_tile(s_off, p.B, rg.hi - 1) + 1);
    }
    __syncthreads();                                         // shared memory stays until every warp is done with it
}

}  // namespace gva
