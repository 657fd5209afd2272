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

// ---- f32 caches: one warp per token, d_v / 32 dims per lane, on the CUDA cores (a cache type for comparisons: 1 M tokens, narrow shape,
//      1236 us against 175 of bytes, bound by five shuffles per head) ----
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
    const int q_len = p.cu_q ? p.cu_q[b + 1] - row0 : 1, rows = min(max(q_len, 0), p.max_q_len);
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
                        if (t >= len - (q_len - 1 - r)) continue;
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
// tile), where they are added in a fixed order.  A single row's queries stay in registers while the sequence lasts.
//   bf16 : values as they lie, queries as three bf16 parts, of which two carry 16 bits only (1.1e-6 of the weights, measured): the
//          third stands in the hi columns of MMAs of its own
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
    // sums: two tiles per team, or one per slot of the ring
    __host__ __device__ static constexpr int tail_bytes(int B, int nstage, int sums, int G) {
        return nstage * 32 + 32 + sums * G * TILE * 4 + (B + 1) * 4;
    }
};

// Queries of a group as B fragments for values that need no step: k-step j of the content holds the lane's dims 4 j .. 4 j + 3.
template <int KIND, class T>
struct PlainQuery {
    uint32_t v[T::DV / 16][2], v2[KIND == kCacheBf16 ? T::DV / 16 : 1][2];
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
            for (int i = 0; i < 2; ++i) {
                out.v[j][i] = pair(v[4 * j + 2 * i], v[4 * j + 2 * i + 1], part);
                out.v2[j][i] = part ? 0u : pair(v[4 * j + 2 * i], v[4 * j + 2 * i + 1], 2);
            }
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
        float low[2][4];                                     // the third parts, apart: see score_pair
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
                if (j == 0) mma_bf16_first(low[k], f, q.v2[2 * j][0], q.v2[2 * j][1]);
                else mma_bf16(low[k], f, q.v2[2 * j][0], q.v2[2 * j][1]);
                if (j == 0) mma_bf16_first(acc[k], f, q.v[2 * j][0], q.v[2 * j][1]);
                else mma_bf16(acc[k], f, q.v[2 * j][0], q.v[2 * j][1]);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t f[4] = {a[k].z, b[k].z, a[k].w, b[k].w};
                mma_bf16(low[k], f, q.v2[2 * j + 1][0], q.v2[2 * j + 1][1]);
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
            for (int k = 0; k < 2; ++k) mma_bf16(low[k], f[k], q.r2[u][0], q.r2[u][1]);
#pragma unroll
            for (int k = 0; k < 2; ++k) mma_bf16(acc[k], f[k], q.r[u][0], q.r[u][1]);
        }
        if constexpr (T::DR % 16 == 8) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uint32_t t[2];
                ldsm_x2(kr + k * 16 * T::KR_ROW + 32 * FULL, t);
                mma_bf16_k8(low[k], t, q.r2[FULL][0]);
                mma_bf16_k8(acc[k], t, q.r[FULL][0]);
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[k][i] += low[k][i];
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

// ---- several new rows per sequence ----
// Two rows at a time: the eight MMA columns are 2 rows x 4 heads, and the query's parts go in as MMAs of their own on the same
// values, so that whatever widening the values need is done once for both rows; both parts of a query are made by the
// lane that holds its column, which is a quarter of the instructions that filling columns {hi, lo} takes.  A pair of rows is
// loaded once for several tiles -- 32 lanes read 32 cache lines apart, from L2, since the ring leaves L1 no room --: the teams
// take all tiles of the ring together and split the rows where there are enough, adding up in shared memory.  The blocks'
// ranges of tiles are cut by the rows that see them.
template <int KIND, class T>
struct PairQuery {
    uint32_t hi[T::DV / 16][2], lo[T::DV / 16][2], low[KIND == kCacheBf16 ? T::DV / 16 : 1][2];     // (bf16: three parts)
    uint32_t rhi[T::DR > 0 ? (T::DR + 15) / 16 : 1][2], rlo[T::DR > 0 ? (T::DR + 15) / 16 : 1][2], rlow[KIND != kCacheE4m3 && T::DR > 0 ? (T::DR + 15) / 16 : 1][2];
    float unscale[2], sum[2], off[2];                        // of this lane's score columns 2 c, 2 c + 1
};
__device__ __forceinline__ void parts_f16(float a, float b, uint32_t &hi, uint32_t &lo) {
    const __half2 h = __floats2half2_rn(a, b);
    const float2 f = __half22float2(h);
    hi = *reinterpret_cast<const uint32_t *>(&h);
    lo = pack_half2(a - f.x, b - f.y);
}
__device__ __forceinline__ void parts_bf16(float a, float b, uint32_t &hi, uint32_t &lo, uint32_t &low) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    const float2 f = __bfloat1622float2(h);
    const __nv_bfloat162 l = __floats2bfloat162_rn(a - f.x, b - f.y);
    const float2 g = __bfloat1622float2(l);
    const __nv_bfloat162 r = __floats2bfloat162_rn(a - f.x - g.x, b - f.y - g.y);
    hi = *reinterpret_cast<const uint32_t *>(&h);
    lo = *reinterpret_cast<const uint32_t *>(&l);
    low = *reinterpret_cast<const uint32_t *>(&r);
}
// q: row r's first head of the group; second: the row after it exists
template <int KIND, class T>
__device__ __forceinline__ void load_pair(PairQuery<KIND, T> &out, const float *q, const float *lse, int H, bool second, float factor, int lane) {
    const int n = lane >> 2, c = lane & 3, row = second ? n >> 2 : 0, head = n & 3;
    const float *src = q + ((size_t)row * H + head) * T::DQ, *rot = src + T::DV;
    constexpr int FULL = T::DR / 16;
    float v[T::DV / 4];
    float top = 0.f, sum = 0.f;
#pragma unroll
    for (int i = 0; i < T::DV / 16; ++i) {
        const float4 x = *reinterpret_cast<const float4 *>(src + c * (T::DV / 4) + 4 * i);
        v[4 * i] = x.x * factor; v[4 * i + 1] = x.y * factor; v[4 * i + 2] = x.z * factor; v[4 * i + 3] = x.w * factor;
    }
    float up = 1.f;
    if constexpr (KIND == kCacheBf16) {
#pragma unroll
        for (int j = 0; j < T::DV / 16; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) parts_bf16(v[4 * j + 2 * i], v[4 * j + 2 * i + 1], out.hi[j][i], out.lo[j][i], out.low[j][i]);
    } else {
        float w[KIND == kCacheE4m3 && T::DR > 0 ? T::DR / 4 : 1];
#pragma unroll
        for (int i = 0; i < T::DV / 4; ++i) {
            top = fmaxf(top, fabsf(v[i]));
            sum += v[i];
        }
        if constexpr (KIND == kCacheE4m3) {
#pragma unroll
            for (int i = 0; i < T::DR / 4; ++i) {
                w[i] = rot[c * (T::DR / 4) + i] * factor;
                top = fmaxf(top, fabsf(w[i]));
            }
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        int e = (int)((__float_as_uint(top) >> 23) & 255u) - 126;
        e = min(max(e, -100), 110);
        if constexpr (KIND == kCacheQ4) {                    // as in load_q4_query
            const float down = __uint_as_float((uint32_t)(127 - e + 10) << 23), down16 = 16.f * down;
            up = __uint_as_float((uint32_t)(127 + e + 8) << 23);
#pragma unroll
            for (int i = 0; i < T::DV / 32; ++i) {
                const float *x = v + 8 * i;
                parts_f16(x[0] * down16, x[4] * down16, out.hi[2 * i][0], out.lo[2 * i][0]);
                parts_f16(x[1] * down, x[5] * down, out.hi[2 * i][1], out.lo[2 * i][1]);
                parts_f16(x[2] * down16, x[6] * down16, out.hi[2 * i + 1][0], out.lo[2 * i + 1][0]);
                parts_f16(x[3] * down, x[7] * down, out.hi[2 * i + 1][1], out.lo[2 * i + 1][1]);
            }
        } else {
            const float down = __uint_as_float((uint32_t)(127 - e + 6) << 23);
            up = __uint_as_float((uint32_t)(127 + e - 6) << 23);
#pragma unroll
            for (int j = 0; j < T::DV / 16; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) parts_f16(v[4 * j + 2 * i] * down, v[4 * j + 2 * i + 1] * down, out.hi[j][i], out.lo[j][i]);
#pragma unroll
            for (int k = 0; k < FULL; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i) parts_f16(w[4 * k + 2 * i] * down, w[4 * k + 2 * i + 1] * down, out.rhi[k][i], out.rlo[k][i]);
        }
    }
    if constexpr (KIND != kCacheE4m3) {                      // bf16 positional keys, in the natural order
#pragma unroll
        for (int k = 0; k < FULL; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float2 x = *reinterpret_cast<const float2 *>(rot + 16 * k + 8 * i + 2 * c);
                parts_bf16(x.x * factor, x.y * factor, out.rhi[k][i], out.rlo[k][i], out.rlow[k][i]);
            }
        if constexpr (T::DR % 16 == 8) {
            const float2 x = *reinterpret_cast<const float2 *>(rot + 16 * FULL + 2 * c);
            parts_bf16(x.x * factor, x.y * factor, out.rhi[FULL][0], out.rlo[FULL][0], out.rlow[FULL][0]);
        }
    }
    const float l = lse[row * H + head], shift = l == -INFINITY ? -INFINITY : -l * kLog2e;
#pragma unroll
    for (int i = 0; i < 2; ++i) {                            // from the column's lanes to the lanes that hold its scores
        out.unscale[i] = __shfl_sync(0xffffffffu, up, 8 * c + 4 * i);
        out.sum[i] = __shfl_sync(0xffffffffu, sum, 8 * c + 4 * i);
        out.off[i] = __shfl_sync(0xffffffffu, shift, 8 * c + 4 * i);
    }
}

// Scores of one chunk: x[0], x[1]: token row tok_lo, columns 2 c, 2 c + 1; x[2], x[3]: the row eight further.
template <int KIND, class T>
__device__ __forceinline__ void score_pair(const unsigned char *v, const unsigned char *kr_row, uint32_t kr, const __half2 *sz /* of row tok_lo */, int c, const PairQuery<KIND, T> &q, float (&x)[4]) {
    // The low parts have an accumulator of their own: every MMA truncates its sum to what it is aligned to, the largest of its terms.  Over
    // codes that is 2^-14, the exponent that a subnormal counts for, which cuts up to eight bits more off.  (Eight rows, 700 tokens,
    // against 64 bits, rms: 4 bits 3.5e-7 -> 1.6e-7, bf16 3.9e-7 -> 2.1e-7, e4m3 3.6e-7 -> 1.9e-7.  Two short chains of MMAs are also
    // faster than a long one: 1 M tokens in 4 bits 410 -> 384 us, bf16 483 -> 451, e4m3 398 -> 364.)
    float acc[4], acc_lo[4];
    auto mma = [&](float (&to)[4], bool first, const uint32_t (&f)[4], const uint32_t (&b)[2]) {
        if constexpr (KIND == kCacheBf16) {
            if (first) mma_bf16_first(to, f, b[0], b[1]);
            else mma_bf16(to, f, b[0], b[1]);
        } else {
            if (first) mma_f16_first(to, f[0], f[1], f[2], f[3], b[0], b[1]);
            else mma_f16_q4(to, f[0], f[1], f[2], f[3], b[0], b[1]);
        }
    };
    auto both = [&](bool first, const uint32_t (&f)[4], int j) {
        if constexpr (KIND == kCacheBf16) mma(acc_lo, first, f, q.low[j]);
        mma(acc_lo, first && KIND != kCacheBf16, f, q.lo[j]);
        mma(acc, first, f, q.hi[j]);
    };
    if constexpr (KIND == kCacheQ4) {
#pragma unroll
        for (int w = 0; w < T::DV / 32; w += 2) {
            const uint2 a = *reinterpret_cast<const uint2 *>(v + 4 * w), b = *reinterpret_cast<const uint2 *>(v + 8 * T::ROW + 4 * w);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t lo = u ? a.y : a.x, hi = u ? b.y : b.x;
                const uint32_t l = lo << 2, h = hi << 2, l6 = lo >> 6, h6 = hi >> 6;
                both(w + u == 0, {l & kCodeLow, h & kCodeLow, l & kCodeHigh, h & kCodeHigh}, 2 * (w + u));
                both(false, {l6 & kCodeLow, h6 & kCodeLow, l6 & kCodeHigh, h6 & kCodeHigh}, 2 * (w + u) + 1);
            }
        }
    } else if constexpr (KIND == kCacheBf16) {
#pragma unroll
        for (int j = 0; j < T::DV / 32; ++j) {
            const uint4 a = *reinterpret_cast<const uint4 *>(v + 16 * j), b = *reinterpret_cast<const uint4 *>(v + 8 * T::ROW + 16 * j);
            both(j == 0, {a.x, b.x, a.y, b.y}, 2 * j);
            both(false, {a.z, b.z, a.w, b.w}, 2 * j + 1);
        }
    } else {
#pragma unroll
        for (int j = 0; j < T::DV / 64; ++j) {
            const uint4 a = *reinterpret_cast<const uint4 *>(v + 16 * j), b = *reinterpret_cast<const uint4 *>(v + 8 * T::ROW + 16 * j);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t f[4];
                e4m3_words(w == 0 ? a.x : w == 1 ? a.y : w == 2 ? a.z : a.w, f[0], f[2]);
                e4m3_words(w == 0 ? b.x : w == 1 ? b.y : w == 2 ? b.z : b.w, f[1], f[3]);
                both(j == 0 && w == 0, f, 4 * j + w);
            }
        }
    }
    constexpr int FULL = T::DR / 16;
    if constexpr (KIND == kCacheE4m3) {
#pragma unroll
        for (int u = 0; u < FULL; ++u) {
            const unsigned char *row = kr_row + c * (T::DR / 4) + 4 * u;
            uint32_t f[4];
            e4m3_words(*reinterpret_cast<const uint32_t *>(row), f[0], f[2]);
            e4m3_words(*reinterpret_cast<const uint32_t *>(row + 8 * T::KR_ROW), f[1], f[3]);
            mma(acc_lo, false, f, q.rlo[u]);
            mma(acc, false, f, q.rhi[u]);
        }
    } else {
        float rot[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < FULL; ++u) {
            uint32_t f[4];
            ldsm_x4(kr + 32 * u, f);
            mma_bf16(rot, f, q.rlow[u][0], q.rlow[u][1]);
            mma_bf16(rot, f, q.rlo[u][0], q.rlo[u][1]);
            mma_bf16(rot, f, q.rhi[u][0], q.rhi[u][1]);
        }
        if constexpr (T::DR % 16 == 8) {
            uint32_t t[2];
            ldsm_x2(kr + 32 * FULL, t);
            mma_bf16_k8(rot, t, q.rlow[FULL][0]);
            mma_bf16_k8(rot, t, q.rlo[FULL][0]);
            mma_bf16_k8(rot, t, q.rhi[FULL][0]);
        }
        if constexpr (KIND == kCacheQ4) {
            const float2 a = __half22float2(sz[0]), b = __half22float2(sz[8]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 z = i < 2 ? a : b;
                x[i] = fmaf((acc[i] + acc_lo[i]) * q.unscale[i & 1], z.x, fmaf(z.y, q.sum[i & 1], rot[i]));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = (acc[i] + (acc_lo[i] + rot[i])) * q.unscale[i & 1];
        }
        return;
    }
    if constexpr (KIND == kCacheE4m3) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (acc[i] + acc_lo[i]) * q.unscale[i & 1];
    }
}

// The block's range of the tile list when a tile costs (rows + 1) / 2 + 1: block c of n takes the tiles whose cost starts in
// [c, c + 1) total / n.  Called by one whole warp.
__device__ __forceinline__ void weighted_range(const int *s_off, const int32_t *cu_q, int B, int max_q_len, int lane, int *out_lo, int *out_hi) {
    auto weight = [&](int b) { return (min(max(cu_q[b + 1] - cu_q[b], 0), max_q_len) + 1) / 2 + 1; };
    long long total = 0;
    for (int b = lane; b < B; b += 32) total += (long long)(s_off[b + 1] - s_off[b]) * weight(b);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    int edge[2] = {s_off[B], s_off[B]};
    long long before = 0;
    for (int base = 0; base < B; base += 32) {
        const int b = base + lane;
        const int w = b < B ? weight(b) : 1, tiles = b < B ? s_off[b + 1] - s_off[b] : 0;
        const long long mine = (long long)tiles * w;
        long long incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        const long long start = before + incl - mine;
#pragma unroll
        for (int e = 0; e < 2; ++e) {                        // the first tile whose cost starts at or behind x
            const long long x = ((long long)blockIdx.x + e) * total / gridDim.x;
            const bool here = mine > 0 && x <= start + mine - w;     // (the first such sequence has it)
            const int at = here ? s_off[b] + (int)((max(x - start, 0ll) + w - 1) / w) : 0;
            const uint32_t who = __ballot_sync(0xffffffffu, here);
            if (who) edge[e] = min(edge[e], __shfl_sync(0xffffffffu, at, __ffs(who) - 1));
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
    }
    *out_lo = edge[0];
    *out_hi = edge[1];
}

struct WeightLaunch {
    int teams, producers, nstage;   // see Q4Launch
    int split;                      // several rows: teams that share their tiles and split the rows; 1 otherwise
    int batch;                      // several rows: tiles that such teams take at once, nstage / (teams / split)
};
constexpr int kWeightConsumers = 16;      // warps of a block (12 with more registers: 56.2 against 50.4 us on the 1 M token batch, 81.0 against 80.6 with 32 rows)

template <int KIND, int DV, int DR, int TILE, bool MULTI>
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
    int *s_edge = reinterpret_cast<int *>(s_meta + nstage) + 4;
    float *s_sum = reinterpret_cast<float *>(s_edge + 4);                                // [team][2 or batch][G][TILE]
    int *s_off = reinterpret_cast<int *>(s_sum + (MULTI ? L.batch : 2) * L.teams * G * TILE);
    if (tid == 0) {
        for (int s = 0; s < nstage; ++s) {
            mbar_init(smem_u32(&full_bar[s]), 1);
            mbar_init(smem_u32(&empty_bar[s]), G * L.split);
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
    BlockRange rg;
    if constexpr (MULTI) {
        if (warp == 0) {
            int lo, hi;
            weighted_range(s_off, w.cu_q, w.B, w.max_q_len, lane, &lo, &hi);
            if (lane == 0) {
                s_edge[0] = lo;
                s_edge[1] = hi;
            }
        }
        __syncthreads();
        rg.lo = s_edge[0];
        rg.hi = s_edge[1];
    } else {
        rg = block_range(p, s_off);
    }
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
        using Single = std::conditional_t<KIND == kCacheQ4, Q4Query<QT>, PlainQuery<KIND, T>>;
        std::conditional_t<MULTI, PairQuery<KIND, T>, Single> q;
        const int part = MULTI ? team % L.split : 0, lead = MULTI ? team / L.split : team, leads = L.teams / L.split;   // rows' part, tiles' part
        const int GS = G * L.split;                          // partial sums per token
        float *sums = s_sum + lead * (MULTI ? L.batch : 2) * GS * TILE;
        int cur_b = -1, row0 = 0, q_len = 0, rows = 0, buf = 0;
        float off = 0.f;                                     // -lse in log2 units (one row)
        const int n_tiles = rg.hi - rg.lo;
        bool dead = false;                                   // a wait ran out: only the team's barriers are still kept
        if constexpr (MULTI) {
            // the tiles of one round stand in slots lead, lead + leads, ... of the ring, all of it
#pragma unroll 1
            for (int i0 = lead, parity = 0; i0 < n_tiles; i0 += leads * L.batch, parity ^= 1) {
                const int n = min(L.batch, (n_tiles - i0 + leads - 1) / leads);
                for (int t = lane; t < n * TILE; t += 32) sums[(t / TILE * GS + part * G + g) * TILE + t % TILE] = 0.f;
                __syncwarp();
                for (int j = 0; j < n && !dead; ++j)
                    if (!mbar_wait_bounded(smem_u32(&full_bar[lead + j * leads]), parity, s_abort)) {
                        if (!*s_abort && lane == 0) report_error(w.dev_status, GVA_ERR_TIMEOUT, 0);
                        *s_abort = 1;
                        dead = true;
                    }
#pragma unroll 1
                for (int j0 = 0; j0 < n && !dead;) {         // tiles [j0, j1) of one sequence
                    const int b = s_meta[lead + j0 * leads].b;
                    int j1 = j0 + 1;
                    while (j1 < n && s_meta[lead + j1 * leads].b == b) ++j1;
                    row0 = w.cu_q[b];
                    const int q_len = w.cu_q[b + 1] - row0;
                    rows = min(max(q_len, 0), w.max_q_len);
#pragma unroll 1
                    for (int r = 2 * part; r < rows; r += 2 * L.split) {
                        const bool second = r + 1 < rows;
                        const size_t at = (size_t)(row0 + r) * H + g * kHeadsPerGroup;
                        load_pair<KIND, T>(q, w.q + at * T::DQ, w.lse + at, H, second, w.scale * kLog2e, lane);
#pragma unroll 1
                        for (int j = j0; j < j1; ++j) {
                            const int st = lead + j * leads;
                            const TileMeta meta = s_meta[st];
                            // tokens of the tile that this lane's row sees; the later row sees one more
                            const int seen = meta.len - (q_len - 1 - r) - meta.t0;
                            if (min(meta.n_valid, seen + 1) <= 0) continue;
                            const int lim = c < 2 ? min(meta.n_valid, seen) : second ? min(meta.n_valid, seen + 1) : 0;
                            const unsigned char *stage = smem + (size_t)st * stage_bytes;
                            const unsigned char *vt = stage + (size_t)g * T::V_BYTES;
                            const __half2 *szt = reinterpret_cast<const __half2 *>(stage + (size_t)G * T::V_BYTES + (size_t)g * T::SZ_BYTES);
                            const unsigned char *krt = stage + (size_t)G * (T::V_BYTES + T::SZ_BYTES);
                            float *mine = sums + (j * GS + part * G + g) * TILE;
#pragma unroll
                            for (int k = 0; k < T::CHUNKS; ++k) {
                                float x[4];
                                score_pair<KIND, T>(vt + (k * 16 + tok_lo) * T::ROW + c * (T::ROW / 4), krt + (k * 16 + tok_lo) * T::KR_ROW,
                                                    smem_u32(krt) + k * 16 * T::KR_ROW + kr_lane<QT>(lane), szt + k * 16 + tok_lo, c, q, x);
                                // (scores may be anything, a NaN included, behind the sequence and where a head has no lse)
                                auto weight = [&](float s, int i) { return q.off[i] == -INFINITY ? 0.f : fast_exp2(s + q.off[i]); };
                                float p0 = weight(x[0], 0) + weight(x[1], 1), p1 = weight(x[2], 0) + weight(x[3], 1);
                                p0 = k * 16 + tok_lo < lim ? p0 : 0.f;
                                p1 = k * 16 + tok_hi < lim ? p1 : 0.f;
                                p0 += __shfl_xor_sync(0xffffffffu, p0, 1);       // the group's heads and the two rows
                                p1 += __shfl_xor_sync(0xffffffffu, p1, 1);
                                p0 += __shfl_xor_sync(0xffffffffu, p0, 2);
                                p1 += __shfl_xor_sync(0xffffffffu, p1, 2);
                                if (c < 2) mine[k * 16 + (c ? tok_hi : tok_lo)] += c ? p1 : p0;
                            }
                        }
                    }
                    j0 = j1;
                }
                if (GS > 1) asm volatile("bar.sync %0, %1;\n" ::"r"(1 + lead), "r"(32 * GS) : "memory");   // (at most 8 of them then)
                else __syncwarp();
                for (int j = 0; j < n && !dead; ++j) {
                    const TileMeta meta = s_meta[lead + j * leads];
                    const int here = min(TILE, meta.len - meta.t0);
                    for (int t = (part * G + g) * 32 + lane; t < here; t += 32 * GS) {
                        float total = 0.f;
                        for (int k = 0; k < GS; ++k) total += sums[(j * GS + k) * TILE + t];
                        const size_t at = (size_t)meta.b * w.stride + meta.t0 + t;
                        w.w_out[at] = w.w_in ? fmaf(w.decay, w.w_in[at], total) : total;
                    }
                }
                if (GS > 1) asm volatile("bar.sync %0, %1;\n" ::"r"(1 + lead), "r"(32 * GS) : "memory");   // the sums may be cleared again
                else __syncwarp();
                if (lane == 0 && !dead)
                    for (int j = 0; j < n; ++j) mbar_arrive(smem_u32(&empty_bar[lead + j * leads]));
            }
        } else {
        auto begin = [&](int b) {                            // sequence b is in hand from here
            cur_b = b;
            row0 = w.cu_q ? w.cu_q[b] : b;
            q_len = w.cu_q ? w.cu_q[b + 1] - row0 : 1;
            rows = min(max(q_len, 0), w.max_q_len);          // 0 or 1
            if (rows == 1) {
                load_query<KIND>(q, w.q + ((size_t)row0 * H + g * kHeadsPerGroup) * T::DQ, w.scale * kLog2e, lane);
                const float lse = w.lse[(size_t)row0 * H + head];
                off = lse == -INFINITY ? -INFINITY : -lse * kLog2e;
            }
        };
        if (team < n_tiles) begin(seq_of_tile(s_off, w.B, rg.lo + team));        // its query is fetched while the first tiles fly
#pragma unroll 1
        for (int i = team, st = team, parity = 0; i < n_tiles; i += L.teams) {
            if (!dead && !mbar_wait_bounded(smem_u32(&full_bar[st]), parity, s_abort)) {
                if (!*s_abort && lane == 0) report_error(w.dev_status, GVA_ERR_TIMEOUT, cur_b < 0 ? 0 : cur_b);
                *s_abort = 1;
                dead = true;
            }
            const TileMeta meta = dead ? TileMeta{cur_b, 0, 0, 0} : s_meta[st];
            if (meta.b != cur_b) begin(meta.b);
            const unsigned char *stage = smem + (size_t)st * stage_bytes;
            const unsigned char *vt = stage + (size_t)g * T::V_BYTES;
            const __half2 *szt = reinterpret_cast<const __half2 *>(stage + (size_t)G * T::V_BYTES + (size_t)g * T::SZ_BYTES);
            const unsigned char *krt = stage + (size_t)G * (T::V_BYTES + T::SZ_BYTES);
            float sum[T::CHUNKS][2];
#pragma unroll
            for (int k = 0; k < T::CHUNKS; ++k) sum[k][0] = sum[k][1] = 0.f;
            if (rows > 0 && !dead) {
                // (q_len > 1 where max_q_len cuts it off; a head without an lse adds nothing, not even a NaN score's NaN)
                const int lim = off == -INFINITY ? 0 : min(meta.n_valid, meta.len - (q_len - 1) - meta.t0);
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
                        sum[kk + k][0] = (kk + k) * 16 + tok_lo < lim ? p0 : 0.f;
                        sum[kk + k][1] = (kk + k) * 16 + tok_hi < lim ? p1 : 0.f;
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
    }
    __syncthreads();                                         // shared memory stays until every warp is done with it
}

}  // namespace gva
