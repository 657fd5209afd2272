// What every cached token has gathered of the attention.
#pragma once

#include <type_traits>

#include "gva_q4_decode.cuh"

namespace gva {

// ---- gathered weights -----------------------------------------------------------------------------------------------
// w_out[b][t] = decay w_in[b][t] + sum over the new rows r of b that see t, and all heads, of exp(score(r, h, t) - lse[r][h]).
struct WeightParams {
    const void *v;               // value pool of the cache's type (4-bit: codes)
    const __half2 *sz;           // 4-bit only
    const void *kr;
    const int32_t *block_table;
    int num_pages, max_pages;
    const float *q, *lse;        // [rows][H][d_v + d_r], [rows][H]
    const int32_t *cu_q;         // nullable: one row per sequence
    const int32_t *seq_lens;
    float decay;
    const float *w_in;           // nullable
    float *w_out;
    int stride, B, max_q_len, H, G, P;
    float scale;
    int32_t *dev_status;
};

enum WeightCache { kCacheF32 = 0, kCacheBf16 = 1, kCacheE4m3 = 2, kCacheQ4 = 3 };

// ---- f32 caches: one warp per token, d_v / 32 dims per lane, on the CUDA cores (a cache type for comparisons) ----
constexpr int kWeightTile = 64;
template <int DV>
__global__ void __launch_bounds__(256)
weights_f32_kernel(WeightParams p, int DR) {
    grid_dependency_launch();
    grid_dependency_wait();
    const int b = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n_warps = blockDim.x >> 5;
    const int len = p.seq_lens[b];
    if (len < 0 || (long long)len > (long long)p.max_pages * p.P || len > p.stride) {
        if (blockIdx.x == 0 && threadIdx.x == 0) report_error(p.dev_status, GVA_ERR_SEQ_LEN, b);
        return;
    }
    const int row0 = p.cu_q ? p.cu_q[b] : b;
    const int rows = p.cu_q ? min(max(p.cu_q[b + 1] - row0, 0), p.max_q_len) : 1;
    const int DQ = DV + DR;
    constexpr int E = DV / 32;
    for (long long t0 = (long long)blockIdx.x * kWeightTile; t0 < len; t0 += (long long)gridDim.x * kWeightTile) {
        for (int t = (int)t0 + warp; t < min((long long)len, t0 + kWeightTile); t += n_warps) {
            const int page = locate_page(p.block_table, p.num_pages, p.max_pages, p.P, b, t, p.dev_status);
            float total = 0.f;
            if (page >= 0) {
                const int slot = t % p.P;
                float k = 0.f;
                if (lane < DR) k = static_cast<const float *>(p.kr)[((size_t)page * p.P + slot) * DR + lane];
                for (int g = 0; g < p.G; ++g) {
                    const size_t row = ((size_t)page * p.G + g) * p.P + slot;
                    float v[E];
                    for (int e = 0; e < E; ++e) v[e] = static_cast<const float *>(p.v)[row * DV + lane * E + e];
                    for (int r = 0; r < rows; ++r) {
                        if (t >= len - (rows - 1 - r)) continue;
                        for (int j = 0; j < kHeadsPerGroup; ++j) {
                            const int h = g * kHeadsPerGroup + j;
                            const float *q = p.q + ((size_t)(row0 + r) * p.H + h) * DQ;
                            float x = lane < DR ? q[DV + lane] * k : 0.f;
                            for (int e = 0; e < E; ++e) x = fmaf(q[lane * E + e], v[e], x);
                            for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
                            const float lse = p.lse[(size_t)(row0 + r) * p.H + h];
                            if (lse != -INFINITY) total += exp2f(fmaf(x, p.scale, -lse) * kLog2e);
                        }
                    }
                }
            }
            if (lane == 0) {
                const size_t i = (size_t)b * p.stride + t;
                p.w_out[i] = p.w_in ? fmaf(p.decay, p.w_in[i], total) : total;
            }
        }
    }
}

// ---- bf16, e4m3 and 4-bit caches: the score half of the decode kernels on the tensor cores ----
// Blocks, teams, ring and producers as in decode_q4_kernel; a team's warps hold one group each.  Scores come out of the
// MMAs with the sum over a head's {hi, lo} columns in one lane; every lane adds up the weights of its head over the new
// rows, four lanes join the group's heads, and the team's groups meet in shared memory (two buffers, one named barrier per
// tile), where they are added in a fixed order.  A row's queries are kept in registers while a sequence has only
// one; several rows are loaded for every tile, from L1.
//   bf16 : values as they lie, queries as bf16 hi + lo (and lo's rest for the positional part, as in the 4-bit kernel)
//   e4m3 : codes widened to f16 exactly, queries as f16 hi + lo, scaled by a power of two per head
// A lane reads the d_v / 4 neighbouring dims [lane % 4 * d_v / 4, ...) of its rows in 16-byte loads: as in the 4-bit kernel the
// order of dims inside the contraction is free.
template <int KIND, int DV_, int DR_, int TILE_>
struct WeightTraits {
    static constexpr int DV = DV_, DR = DR_, TILE = TILE_;
    static constexpr int ROW = KIND == kCacheQ4 ? DV / 2 : KIND == kCacheBf16 ? 2 * DV : DV;
    static constexpr int V_BYTES = TILE * ROW, SZ_BYTES = KIND == kCacheQ4 ? TILE * 4 : 0;
    static constexpr int KR_ROW = KIND == kCacheE4m3 ? DR : 2 * DR, KR_BYTES = TILE * KR_ROW;
    static constexpr int CHUNKS = TILE / 16, DQ = DV + DR;
    __host__ __device__ static constexpr int stage_bytes(int G) { return G * (V_BYTES + SZ_BYTES) + KR_BYTES; }
    __host__ __device__ static constexpr int tail_bytes(int B, int nstage, int teams, int G) {
        return nstage * 32 + 16 + teams * 2 * G * TILE * 4 + (B + 1) * 4;
    }
};

// Queries of a group as B fragments for values that need no step: k-step j of the content holds the lane's dims 4 j .. 4 j + 3.
template <int KIND, class T>
struct PlainQuery {
    uint32_t v[T::DV / 16][2];
    uint32_t r[T::DR > 0 ? (T::DR + 15) / 16 : 1][2], r2[KIND == kCacheBf16 && T::DR > 0 ? (T::DR + 15) / 16 : 1][2];
    float unscale;
};
template <int KIND, class T>
__device__ __forceinline__ void load_query(PlainQuery<KIND, T> &out, const float *q, float factor, int lane) {
    const int n = lane >> 2, c = lane & 3, head = n >> 1, part = n & 1;
    const float *src = q + (size_t)head * T::DQ, *rot = src + T::DV;
    float v[T::DV / 4];
#pragma unroll
    for (int i = 0; i < T::DV / 16; ++i) {
        const float4 x = *reinterpret_cast<const float4 *>(src + c * (T::DV / 4) + 4 * i);
        v[4 * i] = x.x * factor; v[4 * i + 1] = x.y * factor; v[4 * i + 2] = x.z * factor; v[4 * i + 3] = x.w * factor;
    }
    constexpr int FULL = T::DR / 16;
    if constexpr (KIND == kCacheBf16) {
        auto pair = [&](float a, float b, int pt) { return part_bf16(a, pt) | (part_bf16(b, pt) << 16); };
#pragma unroll
        for (int j = 0; j < T::DV / 16; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) out.v[j][i] = pair(v[4 * j + 2 * i], v[4 * j + 2 * i + 1], part);
        out.unscale = 1.f;
#pragma unroll
        for (int k = 0; k < FULL; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) {                    // the natural order: ldmatrix
                const float *x = rot + 16 * k + 8 * i + 2 * c;
                out.r[k][i] = pair(x[0] * factor, x[1] * factor, part);
                out.r2[k][i] = part ? 0u : pair(x[0] * factor, x[1] * factor, 2);
            }
        if constexpr (T::DR % 16 == 8) {
            const float *x = rot + 16 * FULL + 2 * c;
            out.r[FULL][0] = pair(x[0] * factor, x[1] * factor, part);
            out.r2[FULL][0] = part ? 0u : pair(x[0] * factor, x[1] * factor, 2);
        }
    } else {
        float w[T::DR > 0 ? T::DR / 4 : 1];
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < T::DV / 4; ++i) top = fmaxf(top, fabsf(v[i]));
#pragma unroll
        for (int i = 0; i < T::DR / 4; ++i) {
            w[i] = rot[c * (T::DR / 4) + i] * factor;
            top = fmaxf(top, fabsf(w[i]));
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        int e = (int)((__float_as_uint(top) >> 23) & 255u) - 126;
        e = min(max(e, -100), 120);
        const float down = __uint_as_float((uint32_t)(127 - e + 6) << 23);
        auto pair = [&](float a, float b) { return part_f16(a * down, part) | (part_f16(b * down, part) << 16); };
#pragma unroll
        for (int j = 0; j < T::DV / 16; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) out.v[j][i] = pair(v[4 * j + 2 * i], v[4 * j + 2 * i + 1]);
#pragma unroll
        for (int k = 0; k < FULL; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) out.r[k][i] = pair(w[4 * k + 2 * i], w[4 * k + 2 * i + 1]);
        out.unscale = __shfl_sync(0xffffffffu, __uint_as_float((uint32_t)(127 + e - 6) << 23), 8 * c);
    }
}
template <int KIND, class T>
__device__ __forceinline__ void load_query(Q4Query<T> &out, const float *q, float factor, int lane) { load_q4_query<T>(out, q, factor, lane); }

__device__ __forceinline__ void e4m3_words(uint32_t x, uint32_t &lo, uint32_t &hi) {      // four codes -> f16 pairs, exactly
    asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}\n" : "=r"(lo), "=r"(hi) : "r"(x));
}

// Scores of two chunks (rows tok_lo and tok_lo + 8 of each), sum over the query's parts, in log2 units.
template <int KIND, class T>
__device__ __forceinline__ void score_plain(const unsigned char *v, const unsigned char *kr_row, uint32_t kr, int c, const PlainQuery<KIND, T> &q, float (&x)[2][2]) {
    float acc[2][4];
    if constexpr (KIND == kCacheBf16) {
#pragma unroll
        for (int j = 0; j < T::DV / 32; ++j) {
            uint4 a[2], b[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                a[k] = *reinterpret_cast<const uint4 *>(v + k * 16 * T::ROW + 16 * j);
                b[k] = *reinterpret_cast<const uint4 *>(v + k * 16 * T::ROW + 8 * T::ROW + 16 * j);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t f[4] = {a[k].x, b[k].x, a[k].y, b[k].y};
                if (j == 0) mma_bf16_first(acc[k], f, q.v[2 * j][0], q.v[2 * j][1]);
                else mma_bf16(acc[k], f, q.v[2 * j][0], q.v[2 * j][1]);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t f[4] = {a[k].z, b[k].z, a[k].w, b[k].w};
                mma_bf16(acc[k], f, q.v[2 * j + 1][0], q.v[2 * j + 1][1]);
            }
        }
        constexpr int FULL = T::DR / 16;
#pragma unroll
        for (int u = 0; u < FULL; ++u) {
            uint32_t f[2][4];
#pragma unroll
            for (int k = 0; k < 2; ++k) ldsm_x4(kr + k * 16 * T::KR_ROW + 32 * u, f[k]);
#pragma unroll
            for (int k = 0; k < 2; ++k) mma_bf16(acc[k], f[k], q.r2[u][0], q.r2[u][1]);
#pragma unroll
            for (int k = 0; k < 2; ++k) mma_bf16(acc[k], f[k], q.r[u][0], q.r[u][1]);
        }
        if constexpr (T::DR % 16 == 8) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uint32_t t[2];
                ldsm_x2(kr + k * 16 * T::KR_ROW + 32 * FULL, t);
                mma_bf16_k8(acc[k], t, q.r2[FULL][0]);
                mma_bf16_k8(acc[k], t, q.r[FULL][0]);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < T::DV / 64; ++j) {
            uint4 a[2], b[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                a[k] = *reinterpret_cast<const uint4 *>(v + k * 16 * T::ROW + 16 * j);
                b[k] = *reinterpret_cast<const uint4 *>(v + k * 16 * T::ROW + 8 * T::ROW + 16 * j);
            }
#pragma unroll
            for (int w = 0; w < 4; ++w)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t lo = w == 0 ? a[k].x : w == 1 ? a[k].y : w == 2 ? a[k].z : a[k].w;
                    const uint32_t hi = w == 0 ? b[k].x : w == 1 ? b[k].y : w == 2 ? b[k].z : b[k].w;
                    uint32_t f[4];
                    e4m3_words(lo, f[0], f[2]);
                    e4m3_words(hi, f[1], f[3]);
                    if (j == 0 && w == 0) mma_f16_first(acc[k], f[0], f[1], f[2], f[3], q.v[4 * j + w][0], q.v[4 * j + w][1]);
                    else mma_f16_q4(acc[k], f[0], f[1], f[2], f[3], q.v[4 * j + w][0], q.v[4 * j + w][1]);
                }
        }
#pragma unroll
        for (int u = 0; u < T::DR / 16; ++u)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const unsigned char *row = kr_row + k * 16 * T::KR_ROW + c * (T::DR / 4) + 4 * u;
                uint32_t f[4];
                e4m3_words(*reinterpret_cast<const uint32_t *>(row), f[0], f[2]);
                e4m3_words(*reinterpret_cast<const uint32_t *>(row + 8 * T::KR_ROW), f[1], f[3]);
                mma_f16_q4(acc[k], f[0], f[1], f[2], f[3], q.r[u][0], q.r[u][1]);
            }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        x[k][0] = (acc[k][0] + acc[k][1]) * q.unscale;
        x[k][1] = (acc[k][2] + acc[k][3]) * q.unscale;
    }
}

struct WeightLaunch {
    int teams, producers, nstage;   // see Q4Launch
};
constexpr int kWeightConsumers = 16;

template <int KIND, int DV, int DR, int TILE>
__global__ void __launch_bounds__(32 * (kWeightConsumers + kQ4Producers), 1)
weights_mma_kernel(WeightParams w, WeightLaunch L) {
    using T = WeightTraits<KIND, DV, DR, TILE>;
    using QT = Q4Traits<DV, DR, TILE>;
    grid_dependency_launch();
    extern __shared__ __align__(128) unsigned char smem[];
    const int G = w.G, H = w.H, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, nstage = L.nstage;
    const int stage_bytes = T::stage_bytes(G);
    unsigned char *tail = smem + (size_t)nstage * stage_bytes;
    uint64_t *full_bar = reinterpret_cast<uint64_t *>(tail), *empty_bar = full_bar + nstage;
    TileMeta *s_meta = reinterpret_cast<TileMeta *>(empty_bar + nstage);
    volatile int *s_abort = reinterpret_cast<volatile int *>(s_meta + nstage);
    float *s_sum = reinterpret_cast<float *>(s_meta + nstage) + 4;                       // [team][2][G][TILE]
    int *s_off = reinterpret_cast<int *>(s_sum + L.teams * 2 * G * TILE);
    if (tid == 0) {
        for (int s = 0; s < nstage; ++s) {
            mbar_init(smem_u32(&full_bar[s]), 1);
            mbar_init(smem_u32(&empty_bar[s]), G);
        }
        *s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    grid_dependency_wait();
    DecodeParams p;                                          // what the partition looks at
    p.seq_lens = w.seq_lens;
    p.dev_status = w.dev_status;
    p.B = w.B;
    p.P = w.P;
    p.max_pages = w.max_pages;
    p.num_splits = 0;
    compute_tile_offsets<TILE>(p, s_off, min((long long)w.max_pages * w.P, (long long)w.stride));    // ends with a barrier
    const BlockRange rg = block_range(p, s_off);
    if (rg.lo >= rg.hi) return;
    if (warp >= G * L.teams) {
        const uint64_t pol = l2_policy_evict_first();
        produce_tiles<TILE>(warp - G * L.teams, L.producers, nstage, s_off, w.seq_lens, w.block_table, w.B, w.P, w.num_pages, w.max_pages,
                            w.dev_status, rg.lo, rg.hi, full_bar, empty_bar, s_meta, s_abort, (uint32_t)stage_bytes,
                            [&](int st, size_t page, int slot, uint32_t bar, int ln) {
                                const uint32_t base = smem_u32(smem + (size_t)st * stage_bytes);
                                const unsigned char *v = static_cast<const unsigned char *>(w.v), *kr = static_cast<const unsigned char *>(w.kr);
                                if (w.P == TILE) {           // a page that is one tile has all groups side by side
                                    if (ln == 0) bulk_load_stream(base, v + page * G * T::V_BYTES, G * T::V_BYTES, bar, pol);
                                    if (KIND == kCacheQ4 && ln == 1) bulk_load_stream(base + G * T::V_BYTES, w.sz + page * G * TILE, G * T::SZ_BYTES, bar, pol);
                                } else if (ln < G) {
                                    bulk_load_stream(base + ln * T::V_BYTES, v + ((page * G + ln) * w.P + slot) * T::ROW, T::V_BYTES, bar, pol);
                                } else if (KIND == kCacheQ4 && ln < 2 * G) {
                                    const int g = ln - G;
                                    bulk_load_stream(base + G * T::V_BYTES + g * T::SZ_BYTES, w.sz + (page * G + g) * w.P + slot, T::SZ_BYTES, bar, pol);
                                }
                                if (DR > 0 && ln == 31) bulk_load_stream(base + G * (T::V_BYTES + T::SZ_BYTES), kr + (page * w.P + slot) * T::KR_ROW, T::KR_BYTES, bar, pol);
                            });
    } else {
        const int team = warp / G, g = warp - team * G, c = lane & 3, r8 = lane >> 2;
        const int tok_lo = rowmap(r8), tok_hi = tok_lo + 8, head = g * kHeadsPerGroup + c;
        using Query = std::conditional_t<KIND == kCacheQ4, Q4Query<QT>, PlainQuery<KIND, T>>;
        Query q;
        float *sums = s_sum + team * 2 * G * TILE;
        int cur_b = -1, row0 = 0, rows = 0, buf = 0;
        float off = 0.f;                                     // -lse in log2 units of the row in hand
        auto take_row = [&](int r) {
            load_query<KIND>(q, w.q + ((size_t)(row0 + r) * H + g * kHeadsPerGroup) * T::DQ, w.scale * kLog2e, lane);
            const float lse = w.lse[(size_t)(row0 + r) * H + head];
            off = lse == -INFINITY ? -INFINITY : -lse * kLog2e;
        };
        const int n_tiles = rg.hi - rg.lo;
        bool dead = false;                                   // a wait ran out: only the team's barriers are still kept
#pragma unroll 1
        for (int i = team, st = team, parity = 0; i < n_tiles; i += L.teams) {
            if (!dead && !mbar_wait_bounded(smem_u32(&full_bar[st]), parity, s_abort)) {
                if (!*s_abort && lane == 0) report_error(w.dev_status, GVA_ERR_TIMEOUT, cur_b < 0 ? 0 : cur_b);
                *s_abort = 1;
                dead = true;
            }
            const TileMeta meta = dead ? TileMeta{cur_b, 0, 0, 0} : s_meta[st];
            if (meta.b != cur_b) {
                cur_b = meta.b;
                row0 = w.cu_q ? w.cu_q[cur_b] : cur_b;
                rows = w.cu_q ? min(max(w.cu_q[cur_b + 1] - row0, 0), w.max_q_len) : 1;
                if (rows == 1) take_row(0);
            }
            const unsigned char *stage = smem + (size_t)st * stage_bytes;
            const unsigned char *vt = stage + (size_t)g * T::V_BYTES;
            const __half2 *szt = reinterpret_cast<const __half2 *>(stage + (size_t)G * T::V_BYTES + (size_t)g * T::SZ_BYTES);
            const unsigned char *krt = stage + (size_t)G * (T::V_BYTES + T::SZ_BYTES);
            float sum[T::CHUNKS][2];
#pragma unroll
            for (int k = 0; k < T::CHUNKS; ++k) sum[k][0] = sum[k][1] = 0.f;
#pragma unroll 1
            for (int r = 0; r < rows && !dead; ++r) {
                if (rows > 1) take_row(r);
                const int lim = min(meta.n_valid, meta.len - (rows - 1 - r) - meta.t0);   // tokens of the tile this row sees
                if (lim <= 0) continue;
#pragma unroll
                for (int kk = 0; kk < T::CHUNKS; kk += 2) {
                    float x[2][2];
                    const uint32_t kr = smem_u32(krt) + kk * 16 * T::KR_ROW + kr_lane<QT>(lane);      // (bf16 rows only)
                    const unsigned char *v = vt + (kk * 16 + tok_lo) * T::ROW + c * (T::ROW / 4);
                    if constexpr (KIND == kCacheQ4) {
                        float acc[2][4], rot[2][4];
                        score_q4<QT>(v, kr, q, acc, rot);
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float2 a = __half22float2(szt[(kk + k) * 16 + tok_lo]), b = __half22float2(szt[(kk + k) * 16 + tok_hi]);
                            x[k][0] = fmaf((acc[k][0] + acc[k][1]) * q.unscale, a.x, fmaf(a.y, q.sum, rot[k][0] + rot[k][1]));
                            x[k][1] = fmaf((acc[k][2] + acc[k][3]) * q.unscale, b.x, fmaf(b.y, q.sum, rot[k][2] + rot[k][3]));
                        }
                    } else {
                        score_plain<KIND, T>(v, krt + (kk * 16 + tok_lo) * T::KR_ROW, kr, c, q, x);
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float p0 = fast_exp2(x[k][0] + off), p1 = fast_exp2(x[k][1] + off);
                        // (what stands behind the sequence may be anything, a NaN included)
                        sum[kk + k][0] += (kk + k) * 16 + tok_lo < lim ? p0 : 0.f;
                        sum[kk + k][1] += (kk + k) * 16 + tok_hi < lim ? p1 : 0.f;
                    }
                }
            }
            __syncwarp();
            if (lane == 0 && !dead) mbar_arrive(smem_u32(&empty_bar[st]));
            // the group's four heads, then the groups
            float *mine = sums + (buf * G + g) * TILE;
#pragma unroll
            for (int k = 0; k < T::CHUNKS; ++k)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float t = sum[k][e];
                    t += __shfl_xor_sync(0xffffffffu, t, 1);
                    t += __shfl_xor_sync(0xffffffffu, t, 2);
                    if (c == 0) mine[k * 16 + (e ? tok_hi : tok_lo)] = t;
                }
            if (G > 1) asm volatile("bar.sync %0, %1;\n" ::"r"(1 + team), "r"(32 * G) : "memory");   // (at most 8 teams then)
            else __syncwarp();
            const int here = min(TILE, meta.len - meta.t0);
            for (int t = g * 32 + lane; t < here; t += 32 * G) {
                float total = 0.f;
                for (int k = 0; k < G; ++k) total += sums[(buf * G + k) * TILE + t];
                const size_t at = (size_t)cur_b * w.stride + meta.t0 + t;
                w.w_out[at] = w.w_in ? fmaf(w.decay, w.w_in[at], total) : total;
            }
            buf ^= 1;
            st += L.teams;
            if (st >= nstage) {
                st -= nstage;
                parity ^= 1;
            }
        }
    }
    __syncthreads();                                         // shared memory stays until every warp is done with it
}

}  // namespace gva
