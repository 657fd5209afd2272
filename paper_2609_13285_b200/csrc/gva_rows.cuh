// Appends by slot map: row r of a batch goes to slot slots[r] % P of page slots[r] / P, rotated to position pos[r], whatever
// sequence it belongs to.  A slot below 0 is a padded row: nothing of it is cached.
//
// Both kernels are bound by memory: f32 rows in, cache rows (and rotated queries) out, each byte once.  A thread moves pieces
// of eight elements (two 16-byte loads; one 16-byte store into a bf16 page) and has the loads of four pieces in flight.  65536 rows of
// 32 + 16 heads of 128 into bf16 pages, half of each head rotated: 438 - 456 us, 6.5 - 6.75 TB/s, the rate of a copy; one row 4.0 us, a launch.
// GVA rows (their rotation in fp64), us, and TB/s: 65536 of 8 x 128 + 32 into bf16, e4m3, f32 pages 76, 71, 100 (5.5, 4.9, 5.5); of 4 x 64 + 16 37, 37, 39 (2.9, 2.4,
// 3.6: the fp64 chains of 8 pairs a row); 8192 of them 7.6, 7.5, 7.8; 500 4.1 - 4.3.
#pragma once

#include "gva_rope.cuh"

namespace gva {

constexpr int kRowsThreads = 256;
constexpr int kRowsBatch = 4;                       // pieces of eight elements that a thread has in flight

// Eight (or 4 + 4) consecutive elements of a cache row.
template <typename CT>
__device__ __forceinline__ void store4(CT *dst, const float4 &x) {
    if constexpr (sizeof(CT) == 1) {
        *reinterpret_cast<uint32_t *>(dst) = (uint32_t)float_to_e4m3_bits(x.x) | ((uint32_t)float_to_e4m3_bits(x.y) << 8) |
                                             ((uint32_t)float_to_e4m3_bits(x.z) << 16) | ((uint32_t)float_to_e4m3_bits(x.w) << 24);
    } else if constexpr (sizeof(CT) == 2) {
        *reinterpret_cast<uint2 *>(dst) = make_uint2((uint32_t)float_to_bf16_bits(x.x) | ((uint32_t)float_to_bf16_bits(x.y) << 16),
                                                     (uint32_t)float_to_bf16_bits(x.z) | ((uint32_t)float_to_bf16_bits(x.w) << 16));
    } else {
        *reinterpret_cast<float4 *>(dst) = x;
    }
}
template <typename CT>
__device__ __forceinline__ void store8(CT *dst, const float4 &a, const float4 &b) {
    if constexpr (sizeof(CT) == 2) {
        *reinterpret_cast<uint4 *>(dst) = make_uint4((uint32_t)float_to_bf16_bits(a.x) | ((uint32_t)float_to_bf16_bits(a.y) << 16),
                                                     (uint32_t)float_to_bf16_bits(a.z) | ((uint32_t)float_to_bf16_bits(a.w) << 16),
                                                     (uint32_t)float_to_bf16_bits(b.x) | ((uint32_t)float_to_bf16_bits(b.y) << 16),
                                                     (uint32_t)float_to_bf16_bits(b.z) | ((uint32_t)float_to_bf16_bits(b.w) << 16));
    } else {
        store4(dst, a);
        store4(dst + 4, b);
    }
}

// ---- grouped values with their positional key --------------------------------------------------------------
struct AppendRowsParams {
    void *v_pool, *kr_pool;
    const float *v_new, *kr_new;     // [n][G][d_v], [n][d_r]
    const int32_t *pos, *slots;      // [n]
    int32_t *dev_status;
    int n, G, d_v, d_r, P, num_pages, rows;     // rows per block
    uint32_t per_row_inv;            // ceil(2^32 / pieces of a row)
    int vec;                         // v_new is 16-byte aligned
};

// Reports row r as it does a sequence; a status word has 23 bits for the number, the last of which stands for all rows behind it too.
__device__ __forceinline__ void report_row(int32_t *dev_status, int code, int r) { report_error(dev_status, code, min(r, (1 << 23) - 1)); }
// The slot of a row: < 0 where nothing is to be written.
__device__ __forceinline__ int row_slot(const int32_t *slots, const int32_t *pos, int r, int P, int num_pages, int32_t *dev_status, bool say) {
    const int s = slots[r];
    if (s < 0) return -1;
    if (s / P >= num_pages) {
        if (say) report_row(dev_status, GVA_ERR_BAD_PAGE, r);
        return -1;
    }
    if (pos[r] < 0) {
        if (say) report_row(dev_status, GVA_ERR_SEQ_LEN, r);
        return -1;
    }
    return s;
}

// The positional key is rotated in fp64 and rounded once, so a row is bit for bit what gva_append_cache writes.
template <typename CT>
__global__ void __launch_bounds__(kRowsThreads)
append_rows_kernel(AppendRowsParams p, RopeTable rope) {
    grid_dependency_launch();
    grid_dependency_wait();
    const int r0 = blockIdx.x * p.rows, rows = min(p.rows, p.n - r0);
    const int n_v = p.G * p.d_v, per_row = n_v / 8, sh = p.d_v == 64 ? 3 : 4;
    CT *v_pool = static_cast<CT *>(p.v_pool), *kr_pool = static_cast<CT *>(p.kr_pool);
    // the rotations first: their fp64 chains run while the value rows are on their way
    const int pairs = p.d_r / 2;
    for (int i = threadIdx.x; i < rows * kMaxRopePairs; i += kRowsThreads) {
        const int r = r0 + i / kMaxRopePairs, k = i % kMaxRopePairs;
        if (k >= pairs) continue;
        const int s = row_slot(p.slots, p.pos, r, p.P, p.num_pages, p.dev_status, false);
        if (s < 0) continue;
        double y0, y1;
        rope_pair((double)p.kr_new[(size_t)r * p.d_r + 2 * k], (double)p.kr_new[(size_t)r * p.d_r + 2 * k + 1], p.pos[r], rope.inv_freq[k], y0, y1);
        CT *dst = kr_pool + (size_t)s * p.d_r + 2 * k;           // pages follow one another: slot s is row s of the pool
        if constexpr (sizeof(CT) == 1) {
            *reinterpret_cast<uint16_t *>(dst) = (uint16_t)(double_to_e4m3_bits(y0) | (double_to_e4m3_bits(y1) << 8));
        } else if constexpr (sizeof(CT) == 2) {
            *reinterpret_cast<uint32_t *>(dst) = (uint32_t)double_to_bf16_bits(y0) | ((uint32_t)double_to_bf16_bits(y1) << 16);
        } else {
            *reinterpret_cast<float2 *>(dst) = make_float2(__double2float_rn(y0), __double2float_rn(y1));
        }
    }
    const int pieces = rows * per_row;
    for (int base = threadIdx.x; base < pieces; base += kRowsThreads * kRowsBatch) {
        float4 a[kRowsBatch], b[kRowsBatch];
        int slot[kRowsBatch];
#pragma unroll
        for (int u = 0; u < kRowsBatch; ++u) {
            const int e = base + u * kRowsThreads;
            slot[u] = -1;
            if (e >= pieces) continue;
            const int r = (int)__umulhi((uint32_t)e, p.per_row_inv);
            const float *src = p.v_new + ((size_t)r0 * n_v + (size_t)e * 8);
            if (p.vec) {
                a[u] = *reinterpret_cast<const float4 *>(src);
                b[u] = *reinterpret_cast<const float4 *>(src + 4);
            } else {
                a[u] = make_float4(src[0], src[1], src[2], src[3]);
                b[u] = make_float4(src[4], src[5], src[6], src[7]);
            }
            slot[u] = row_slot(p.slots, p.pos, r0 + r, p.P, p.num_pages, p.dev_status, e == r * per_row);
        }
#pragma unroll
        for (int u = 0; u < kRowsBatch; ++u) {
            if (slot[u] < 0) continue;
            const int e = base + u * kRowsThreads;
            const int r = (int)__umulhi((uint32_t)e, p.per_row_inv), i = e - r * per_row;
            const int g = i >> sh, d = (i & ((1 << sh) - 1)) * 8;
            const int page = slot[u] / p.P, at = slot[u] - page * p.P;
            store8(v_pool + (((size_t)page * p.G + g) * p.P + at) * p.d_v + d, a[u], b[u]);
        }
    }
}

// ---- keys and values of the matched GQA cache, and the queries ----------------------------------------------
struct GqaAppendParams {
    void *k_pool, *v_pool;
    const float *q, *k_new, *v_new;                // rows of H d_h, G d_h, G d_h elements (q may be null)
    long long q_stride, k_stride, v_stride;        // elements from row to row
    float *q_out;                                  // [n][H][d_h]
    const int32_t *pos, *slots;
    int32_t *dev_status;
    int n, H, G, d, P, num_pages, rows;            // H = 0 without queries; rows per block, kGqaRows at most
    uint32_t per_row_inv;                          // ceil(2^32 / pieces of a row)
};
constexpr int kGqaRows = 4;

// A piece is eight elements of a head: four pairs, neighbours or (halves) four elements and the four half a rotation away.
// The angle of a pair goes by position alone, so a block computes the cosines and sines of its rows once, for all their heads:
// the turn pos f / 2 pi and its fraction in fp64, what is left in f32 (2^-25 of a half-turn, 1e-7 radians).
template <typename CT>
__global__ void __launch_bounds__(kRowsThreads)
gqa_append_kernel(GqaAppendParams p, HeadRope rope) {
    grid_dependency_launch();
    __shared__ __align__(16) float2 s_turn[kGqaRows][kMaxHeadPairs];
    grid_dependency_wait();
    const int r0 = blockIdx.x * p.rows, rows = min(p.rows, p.n - r0);
    const int sh = p.d == 64 ? 3 : 4;                                     // pieces of a head, as a shift
    const int heads = p.H + 2 * p.G, per_row = heads << sh;
    const int turned = rope.d_rot / 8;                                    // pieces of a head that turn
    const int half = rope.halves ? rope.d_rot / 2 : 4;                    // from the first four elements to the second
    CT *k_pool = static_cast<CT *>(p.k_pool), *v_pool = static_cast<CT *>(p.v_pool);
    const int pieces = rows * per_row;
    bool first = true;
    for (int base = 0; base < pieces; base += kRowsThreads * kRowsBatch) {
        float4 a[kRowsBatch], b[kRowsBatch];
#pragma unroll
        for (int u = 0; u < kRowsBatch; ++u) {
            const int e = base + u * kRowsThreads + threadIdx.x;
            if (e >= pieces) continue;
            const int r = (int)__umulhi((uint32_t)e, p.per_row_inv), i = e - r * per_row;
            const int h = i >> sh, c = i & ((1 << sh) - 1);
            const float *row = h < p.H         ? p.q + (size_t)(r0 + r) * p.q_stride + h * p.d
                               : h < p.H + p.G ? p.k_new + (size_t)(r0 + r) * p.k_stride + (h - p.H) * p.d
                                               : p.v_new + (size_t)(r0 + r) * p.v_stride + (h - p.H - p.G) * p.d;
            const bool apart = rope.halves && c < turned && h < p.H + p.G;
            const int at = apart ? c * 4 : c * 8;
            a[u] = *reinterpret_cast<const float4 *>(row + at);
            b[u] = *reinterpret_cast<const float4 *>(row + at + (apart ? half : 4));
        }
        if (first) {                                                      // (the same for the whole block)
            first = false;
            for (int i = threadIdx.x; i < rows * kMaxHeadPairs; i += kRowsThreads) {
                const int r = i / kMaxHeadPairs, k = i % kMaxHeadPairs;
                if (k >= rope.d_rot / 2) continue;
                const double t = (double)p.pos[r0 + r] * rope.turns[k];
                float s, co;
                sincospif((float)(2.0 * (t - rint(t))), &s, &co);
                s_turn[r][k] = make_float2(co * rope.magnitude, s * rope.magnitude);
            }
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < kRowsBatch; ++u) {
            const int e = base + u * kRowsThreads + threadIdx.x;
            if (e >= pieces) continue;
            const int r = (int)__umulhi((uint32_t)e, p.per_row_inv), i = e - r * per_row;
            const int h = i >> sh, c = i & ((1 << sh) - 1);
            float4 x = a[u], y = b[u];
            const bool turn = c < turned && h < p.H + p.G;
            if (turn) {
                const float4 t0 = *reinterpret_cast<const float4 *>(&s_turn[r][4 * c]), t1 = *reinterpret_cast<const float4 *>(&s_turn[r][4 * c + 2]);
                auto rot = [](float &u0, float &u1, float co, float s) {
                    const float v0 = fmaf(u0, co, -u1 * s), v1 = fmaf(u0, s, u1 * co);
                    u0 = v0;
                    u1 = v1;
                };
                if (rope.halves) {
                    rot(x.x, y.x, t0.x, t0.y);
                    rot(x.y, y.y, t0.z, t0.w);
                    rot(x.z, y.z, t1.x, t1.y);
                    rot(x.w, y.w, t1.z, t1.w);
                } else {
                    rot(x.x, x.y, t0.x, t0.y);
                    rot(x.z, x.w, t0.z, t0.w);
                    rot(y.x, y.y, t1.x, t1.y);
                    rot(y.z, y.w, t1.z, t1.w);
                }
            }
            const bool apart = rope.halves && turn;
            const int at = apart ? c * 4 : c * 8;
            if (h < p.H) {
                float *dst = p.q_out + ((size_t)(r0 + r) * p.H + h) * p.d + at;
                *reinterpret_cast<float4 *>(dst) = x;
                *reinterpret_cast<float4 *>(dst + (apart ? half : 4)) = y;
                continue;
            }
            const int s = row_slot(p.slots, p.pos, r0 + r, p.P, p.num_pages, p.dev_status, h == p.H && c == 0);
            if (s < 0) continue;
            const int page = s / p.P, g = (h - p.H) % p.G;
            CT *dst = (h < p.H + p.G ? k_pool : v_pool) + (((size_t)page * p.G + g) * p.P + (s - page * p.P)) * p.d + at;
            if (apart) {
                store4(dst, x);
                store4(dst + half, y);
            } else {
                store8(dst, x, y);
            }
        }
    }
}

}  // namespace gva
