// The 4-bit cache: how rows enter it, how they leave it as bf16, and the pieces its readers share.
//
// A value row x[0 .. d_v) of one token and group is held as d_v codes of 4 bits and two f16 numbers,
//     lowest z = the largest f16 <= min x,      step s = the smallest f16 with z + 15 s >= max x,
//     code c = the number of k in 0 .. 14 with x >= z + (k + 1/2) s,      value = z + s c,
// so that |value - x| <= s / 2 for every x: z is rounded down and s up, hence the codes always cover the row.  Elements
// beyond +-65504 are clamped first; a row with a NaN anywhere reads as NaN.  A row of one value has s = 0.
// Byte i of a row holds dims 2 i (low nibble) and 2 i + 1 (high nibble).  Positional keys are bf16, as in the bf16 cache.
#pragma once

#include "gva_rope.cuh"

namespace gva {

struct Q4Pools {
    uint8_t *v;                  // [num_pages][G][P][d_v / 2]
    __half2 *sz;                 // [num_pages][G][P] (step, lowest)
    uint16_t *kr;                // [num_pages][P][d_r] bf16
    const int32_t *block_table;  // nullable
    int num_pages, max_pages;
};

// Page of slot t of sequence b, or -1 after reporting why there is none.
__device__ __forceinline__ int locate_page(const int32_t *block_table, int num_pages, int max_pages, int P, int b, int t, int32_t *dev_status) {
    if (t < 0 || t / P >= max_pages) {
        report_error(dev_status, GVA_ERR_SEQ_LEN, b);
        return -1;
    }
    const long long page = block_table ? (long long)block_table[(size_t)b * max_pages + t / P] : (long long)b * max_pages + t / P;
    if (page < 0 || page >= num_pages) {
        report_error(dev_status, GVA_ERR_BAD_PAGE, b);
        return -1;
    }
    return (int)page;
}

// ---- append -----------------------------------------------------------------------------------------------------
// d_v / 8 neighbouring lanes hold one value row, eight elements each (two 16-byte loads), reduce minimum and maximum with
// shuffles, and each writes its eight codes as one 32-bit word.  A block takes as many input rows as give every thread four such
// shares, asks for all of them at once and looks up where they go while they are quantised (65536 rows of 8 x 128: 72 us, 4.4 TB/s
// of rows in and codes out; issue slots 69 % busy with some 190 instructions per share and warp, no pipe above 46 %).  Its threads rotate the positional pairs in fp64.
// All comparisons against the borders z + (k + 1/2) s are exact in f32: 15 s and (k + 1/2) s have at most 16 significant
// bits, and "x - z >= T" for an f32 number T holds exactly if it holds for x - z rounded down (max - z <= 15 s: up).
struct AppendQ4Params {
    Q4Pools c;
    const float *v_new, *kr_new;
    const int32_t *cu_q;        // nullable: one row per sequence
    const int32_t *slot0;       // per sequence: slot of its first row
    const int32_t *pos0;        // per sequence: position of its first row
    int B, n_q, G, d_r, P, rows;
    uint32_t per_row_inv;       // ceil(2^20 / (G d_v / 8)): shares of a block (< 1024) are told apart into rows by a product
    int vec;                    // v_new is 16-byte aligned
    int32_t *dev_status;
};
constexpr int kAppendQ4Threads = 256;
constexpr int kAppendQ4Shares = 4;        // shares of eight elements per thread
// Rows of a block at most (G = 1), and the positional pairs that many rows can bring: 128 x 12 with d_v = 64, 64 x 16 with 128.
__host__ __device__ constexpr int append_q4_rows(int d_v) { return kAppendQ4Threads * kAppendQ4Shares / (d_v / 8); }
template <int DV>
constexpr int kAppendQ4Pairs = append_q4_rows(DV) * widest_rope(DV) / 2;

// The codes of eight elements (z <= x, x - z <= 15 s).  A code is the integer nearest to (x - z) / s, read out of the mantissa after
// adding 2^23; the quotient is off by less than 3e-6, so a code is right unless its remainder comes within 2e-5 of a half:
// those elements (one in 25000) are compared with their border as above.
__device__ __forceinline__ uint32_t quantise8(const float (&x)[8], float z, float s) {
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;\n" : "=f"(inv) : "f"(s));
    if (!(s > 0.f)) inv = 0.f;
    float c[8], edge = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float d = __fsub_rd(x[i], z);                  // >= 0
        c[i] = __fsub_rn(__fmaf_rn(d, inv, 8388608.f), 8388608.f);
        edge = fmaxf(edge, fabsf(__fmaf_rn(d, inv, -c[i])));
    }
    if (edge > 0.5f - 2e-5f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = __fsub_rd(x[i], z);
            if (d < (c[i] - 0.5f) * s) c[i] -= 1.f;          // (a product of <= 5 by 11 bits: exact)
            else if (d >= (c[i] + 0.5f) * s) c[i] += 1.f;
            c[i] = fminf(fmaxf(c[i], 0.f), 15.f);
        }
    }
    // four codes as one number below 2^16, again in the mantissa
    const float lo = fmaf(4096.f, c[3], fmaf(256.f, c[2], fmaf(16.f, c[1], c[0]))) + 8388608.f;
    const float hi = fmaf(4096.f, c[7], fmaf(256.f, c[6], fmaf(16.f, c[5], c[4]))) + 8388608.f;
    return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x5410);
}
// The smallest f16 number s with 15 s >= d, for 0 <= d <= 15 * 65504: from the product with 1 / 15, which is at most one step off;
// 15 s is exact in f32.
__device__ __forceinline__ __half step_for(float d) {
    uint32_t u = __half_as_ushort(__float2half_ru(d * 0.066666667f));
    if (15.f * __half2float(__ushort_as_half((unsigned short)u)) < d) ++u;
    const uint32_t less = u > 0 ? u - 1 : 0;
    if (15.f * __half2float(__ushort_as_half((unsigned short)less)) >= d) u = less;
    return __ushort_as_half((unsigned short)u);
}
__device__ __forceinline__ float max_nan(float a, float b) {         // NaN if either is
    float y;
    asm("max.NaN.f32 %0, %1, %2;\n" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

template <int DV>
__global__ void __launch_bounds__(kAppendQ4Threads)
append_q4_kernel(const __grid_constant__ AppendQ4Params p, const __grid_constant__ RopeTable rope) {     // (tables are indexed where they lie)
    grid_dependency_launch();
    constexpr int ROWS = append_q4_rows(DV);
    __shared__ int s_page[ROWS], s_slot[ROWS], s_pos[ROWS];  // page -1: the row is not written
    __shared__ uint32_t s_key[kAppendQ4Pairs<DV>];           // rotated pairs, bf16
    static_assert(ROWS <= kAppendQ4Threads, "a thread per row");
    grid_dependency_wait();
    const int tid = threadIdx.x, n0 = blockIdx.x * p.rows;
    const int total = p.cu_q ? min(p.n_q, p.cu_q[p.B]) : p.n_q;
    constexpr int L = DV / 8;                                // lanes per value row
    const int per_row = p.G * L;
    // a row of G d_v elements is per_row shares side by side: share e of the block lies at 8 e
    const int n_shares = min(p.rows, total - n0) * per_row;
    const float *src = p.v_new + (size_t)n0 * per_row * 8;
    float x[kAppendQ4Shares][8];
#pragma unroll
    for (int u = 0; u < kAppendQ4Shares; ++u) {
        const int e = u * kAppendQ4Threads + tid;
        if (e < n_shares) {
            if (p.vec) {
                const float4 a = *reinterpret_cast<const float4 *>(src + 8 * (size_t)e), b = *reinterpret_cast<const float4 *>(src + 8 * (size_t)e + 4);
                x[u][0] = a.x; x[u][1] = a.y; x[u][2] = a.z; x[u][3] = a.w;
                x[u][4] = b.x; x[u][5] = b.y; x[u][6] = b.z; x[u][7] = b.w;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[u][i] = src[8 * (size_t)e + i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] = 0.f;
        }
    }
    int my_b = -1, my_t = 0;                                 // this thread's row, if it has one: sequence and slot
    if (tid < p.rows && n0 + tid < total) {
        const int n = n0 + tid;
        int b = n, i = 0;
        if (p.cu_q) {
            int lo = 0, hi = p.B - 1;                        // largest b with cu_q[b] <= n (empty sequences repeat an offset)
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (p.cu_q[mid] <= n) lo = mid;
                else hi = mid - 1;
            }
            b = lo;
            i = n - p.cu_q[b];
        }
        const int slot0 = p.slot0[b], pos0 = p.pos0[b];
        const long long t = (long long)slot0 + i, at = (long long)pos0 + i;
        if (slot0 < 0 || pos0 < 0 || t > 0x7fffffff || at > 0x7fffffff) {
            report_error(p.dev_status, GVA_ERR_SEQ_LEN, b);
        } else {
            my_b = b;
            my_t = (int)t;
        }
        s_pos[tid] = (int)at;
    }
    uint32_t word[kAppendQ4Shares];
    __half2 sz[kAppendQ4Shares];
#pragma unroll
    for (int u = 0; u < kAppendQ4Shares; ++u) {
        if (u * kAppendQ4Threads >= n_shares) break;         // (the whole block)
        float mn = x[u][0], mx = x[u][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) {
            mn = fminf(mn, x[u][i]);
            mx = max_nan(mx, x[u][i]);
        }
#pragma unroll
        for (int o = 1; o < L; o <<= 1) {
            mn = fminf(mn, __shfl_xor_sync(0xffffffffu, mn, o));
            mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        }
        const bool nan = mx != mx;
        if (!(mn >= -65504.f && mx <= 65504.f)) {            // (rare) what is beyond f16, and rows with a NaN, which are marked below
            mn = fminf(fmaxf(mn, -65504.f), 65504.f);
            mx = nan ? mn : fminf(fmaxf(mx, -65504.f), 65504.f);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] = nan ? mn : fminf(fmaxf(x[u][i], -65504.f), 65504.f);
        }
        const __half zh = __float2half_rd(mn);
        const float z = __half2float(zh);
        const __half sh = step_for(__fsub_ru(mx, z));
        word[u] = quantise8(x[u], z, __half2float(sh));
        sz[u] = __halves2half2(sh, zh);
        if (nan) {
            word[u] = 0;
            sz[u] = __halves2half2(__float2half(0.f), __ushort_as_half(0x7fff));
        }
    }
    __syncthreads();
    // pages by the first threads, positional pairs by the last
    if (tid < p.rows) {
        s_page[tid] = my_b >= 0 ? locate_page(p.c.block_table, p.c.num_pages, p.c.max_pages, p.P, my_b, my_t, p.dev_status) : -1;
        s_slot[tid] = my_t % p.P;
    }
    const int pairs = p.d_r / 2, n_pairs = min(p.rows, total - n0) * pairs;
    for (int e = kAppendQ4Threads - 1 - tid; e < n_pairs; e += kAppendQ4Threads) {
        const int r = e / pairs, k = e - r * pairs;
        const float *x = p.kr_new + (size_t)n0 * p.d_r + 2 * (size_t)e;
        double y0, y1;
        rope_pair((double)x[0], (double)x[1], s_pos[r], rope.inv_freq[k], y0, y1);
        s_key[e] = (uint32_t)double_to_bf16_bits(y0) | ((uint32_t)double_to_bf16_bits(y1) << 16);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kAppendQ4Shares; ++u) {
        const int e = u * kAppendQ4Threads + tid;
        const int r = (int)(((uint32_t)e * p.per_row_inv) >> 20), l = e & (L - 1), g = (e - r * per_row) >> (L == 8 ? 3 : 4);
        if (e < n_shares && s_page[r] >= 0) {
            const size_t row = ((size_t)s_page[r] * p.G + g) * p.P + s_slot[r];
            *reinterpret_cast<uint32_t *>(p.c.v + row * (DV / 2) + 4 * l) = word[u];
            if (l == 0) p.c.sz[row] = sz[u];
        }
    }
    for (int e = tid; e < n_pairs; e += kAppendQ4Threads) {
        const int r = e / pairs, k = e - r * pairs;
        if (s_page[r] >= 0) *reinterpret_cast<uint32_t *>(p.c.kr + ((size_t)s_page[r] * p.P + s_slot[r]) * p.d_r + 2 * k) = s_key[e];
    }
}

// ---- widen ------------------------------------------------------------------------------------------------------
// Slots [starts[b], seq_lens[b]) of every sequence as bf16 rows of another cache: z + s c rounded to f32, then to bf16.  A block
// takes 64 slots of one sequence; d_v / 8 lanes widen one row, 4 bytes in and 16 bytes out per lane, neighbouring slots of
// a group one after the other, so that reads and writes run through a page's rows in order; four shares of a thread are asked
// for at a time (64 K tokens of wide heads: 46 us, 3.9 TB/s; one share at a time 76).
constexpr int kWidenTokens = 64;
struct WidenParams {
    Q4Pools c;
    uint16_t *v, *kr;            // bf16 pools
    const int32_t *block_table;  // of the bf16 cache; nullable
    int num_pages, max_pages;
    const int32_t *starts, *seq_lens;
    int G, d_v, d_r, P;
    int32_t *dev_status;
};
__global__ void __launch_bounds__(256)
widen_q4_kernel(WidenParams p) {
    grid_dependency_launch();
    __shared__ int s_src[kWidenTokens], s_dst[kWidenTokens], s_slot[kWidenTokens];
    grid_dependency_wait();
    const int b = blockIdx.y, tid = threadIdx.x;
    const int start = p.starts ? p.starts[b] : 0, len_in = p.seq_lens[b];
    const long long room = (long long)min(p.c.max_pages, p.max_pages) * p.P;     // slots that both block tables have
    if (start < 0 || len_in < 0 || len_in > room) {
        if (blockIdx.x == 0 && tid == 0) report_error(p.dev_status, GVA_ERR_SEQ_LEN, b);
        if (start < 0 || len_in < 0) return;
    }
    const int len = (int)min((long long)len_in, room);
    const int shift = p.d_v == 64 ? 3 : 4, L = 1 << shift;   // lanes per row
    for (long long t0 = start + (long long)blockIdx.x * kWidenTokens; t0 < len; t0 += (long long)gridDim.x * kWidenTokens) {
        const int n = (int)min((long long)kWidenTokens, len - t0);
        if (tid < n) {
            const int t = (int)t0 + tid;
            const int a = locate_page(p.c.block_table, p.c.num_pages, p.c.max_pages, p.P, b, t, p.dev_status);
            const int d = locate_page(p.block_table, p.num_pages, p.max_pages, p.P, b, t, p.dev_status);
            s_src[tid] = d < 0 ? -1 : a;
            s_dst[tid] = d;
            s_slot[tid] = t % p.P;
        }
        __syncthreads();
        // item e: lane e % L of row (g, k); k runs fastest among rows, kWidenTokens places to a group
        constexpr int U = 4;
        const int items = p.G * kWidenTokens << shift;
        for (int e0 = tid; e0 < items; e0 += U * 256) {
            uint32_t word[U];
            __half2 sz[U];
            bool on[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int e = e0 + u * 256, k = (e >> shift) % kWidenTokens, g = (e >> shift) / kWidenTokens;
                on[u] = e < items && k < n && s_src[k] >= 0;
                word[u] = 0;
                if (on[u]) {
                    const size_t row = ((size_t)s_src[k] * p.G + g) * p.P + s_slot[k];
                    word[u] = *reinterpret_cast<const uint32_t *>(p.c.v + row * (p.d_v / 2) + 4 * (e & (L - 1)));
                    sz[u] = p.c.sz[row];
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (!on[u]) continue;
                const int e = e0 + u * 256, k = (e >> shift) % kWidenTokens, g = (e >> shift) / kWidenTokens;
                const float2 q = __half22float2(sz[u]);
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)                  // the code as a float: 2^23 + c less 2^23
                    y[i] = fmaf(__uint_as_float(((word[u] >> (4 * i)) & 15u) | 0x4b000000u) - 8388608.f, q.x, q.y);
                uint32_t out[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
                    out[i] = *reinterpret_cast<const uint32_t *>(&h);
                }
                const size_t to = (((size_t)s_dst[k] * p.G + g) * p.P + s_slot[k]) * p.d_v + 8 * (e & (L - 1));
                *reinterpret_cast<uint4 *>(p.v + to) = make_uint4(out[0], out[1], out[2], out[3]);
            }
        }
        const int pieces = p.d_r / 8;                        // 16-byte pieces of a positional row
        for (int e = tid; e < n * pieces; e += blockDim.x) {
            const int k = e / pieces, i = e % pieces;
            if (s_src[k] < 0) continue;
            reinterpret_cast<uint4 *>(p.kr)[((size_t)s_dst[k] * p.P + s_slot[k]) * pieces + i] =
                reinterpret_cast<const uint4 *>(p.c.kr)[((size_t)s_src[k] * p.P + s_slot[k]) * pieces + i];
        }
        __syncthreads();
    }
}

// ---- merge of split-KV partials -----------------------------------------------------------------------------------
// Records of sequence b: segments[b] = (first group of records, groups), as the decode kernel's block 0 has written it, or
// num_splits groups from b num_splits on; a group is one record per team.  One block per (sequence, head).  d_v / 4
// lanes read one record's output in 16-byte pieces, the other threads other records, each under its own running maximum, so
// that a record costs one trip to memory; the parts are then joined in a fixed order.
struct MergeParams {
    const float *rec_o, *rec_ml;   // [n_rec][H][d_v], [n_rec][H][2]
    const int2 *segments;
    float *out, *lse;
    int H, num_splits, teams;
};
template <int DV>
__global__ void __launch_bounds__(1024)
merge_records_kernel(MergeParams p) {
    grid_dependency_launch();
    constexpr int L = DV / 4;
    extern __shared__ float s_part[];                        // [parts][DV] outputs, [parts] maxima, [parts] sums
    const int b = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, parts = blockDim.x / L, part = tid / L, l = tid % L;
    float *s_m = s_part + parts * DV, *s_l = s_m + parts;
    grid_dependency_wait();
    const int2 seg = p.num_splits > 0 ? make_int2(b * p.num_splits, p.num_splits) : p.segments[b];
    const int first = seg.x * p.teams, count = seg.y * p.teams;
    float m = -INFINITY, sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int U = 4;                                     // records in flight per thread
    for (int r0 = part; r0 < count; r0 += U * parts) {
        float2 ml[U];
        float4 o[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = r0 + u * parts;
            const size_t rh = (size_t)(first + min(r, count - 1)) * p.H + h;
            ml[u] = *reinterpret_cast<const float2 *>(p.rec_ml + rh * 2);
            o[u] = *reinterpret_cast<const float4 *>(p.rec_o + rh * DV + 4 * l);
            if (r >= count) ml[u] = make_float2(-INFINITY, 0.f);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // an empty range: its output is not written.  (Where all scores are NaN the maximum is -inf too, but the sum is NaN, which
            // from here on stays in sum and outputs: 0 NaN = NaN)
            if (ml[u].x == -INFINITY && ml[u].y == 0.f) continue;
            const float top = fmaxf(m, ml[u].x), f = exp2f(m - top), w = exp2f(ml[u].x - top);
            m = top;
            acc.x = fmaf(w, o[u].x, acc.x * f);
            acc.y = fmaf(w, o[u].y, acc.y * f);
            acc.z = fmaf(w, o[u].z, acc.z * f);
            acc.w = fmaf(w, o[u].w, acc.w * f);
            sum = fmaf(w, ml[u].y, sum * f);
        }
    }
    *reinterpret_cast<float4 *>(s_part + part * DV + 4 * l) = acc;
    if (l == 0) {
        s_m[part] = m;
        s_l[part] = sum;
    }
    __syncthreads();
    for (int d = tid; d < DV; d += blockDim.x) {
        float top = -INFINITY, o = 0.f, t = 0.f;
        for (int k = 0; k < parts; ++k) top = fmaxf(top, s_m[k]);
        for (int k = 0; k < parts; ++k) {
            const float w = s_m[k] == -INFINITY ? 0.f : exp2f(s_m[k] - top);
            o = fmaf(w, s_part[k * DV + d], o);
            t = fmaf(w, s_l[k], t);
        }
        p.out[((size_t)b * p.H + h) * DV + d] = t != 0.f ? o / t : 0.f;
        if (d == 0 && p.lse) p.lse[(size_t)b * p.H + h] = (top + log2f(t)) * kLn2;
    }
}

}  // namespace gva
