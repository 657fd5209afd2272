// RoPE in fp64 and the roundings of an append.
#pragma once

#include "gva_common.cuh"

namespace gva {

constexpr int kMaxRopePairs = 16;   // d_r <= 32

// The head widths that gva_create serves: of a value row and of the positional slice beside it.
struct HeadWidths {
    int d_v, d_r;
};
constexpr HeadWidths kHeadWidths[] = {{64, 16}, {64, 24}, {64, 0}, {128, 32}, {128, 0}};
constexpr bool serves_widths(int d_v, int d_r) {
    for (const HeadWidths &w : kHeadWidths)
        if (w.d_v == d_v && w.d_r == d_r) return true;
    return false;
}
constexpr int widest_rope(int d_v) {
    int most = 0;
    for (const HeadWidths &w : kHeadWidths)
        if (w.d_v == d_v && w.d_r > most) most = w.d_r;
    return most;
}

struct RopeTable {
    double inv_freq[kMaxRopePairs];   // base^(-2i/d_r), computed once on the host in fp64
};

// fp64 -> bf16, round to nearest even without double rounding: truncate to f32 toward zero, fold
// everything that was cut off into the f32's last mantissa bit (round to odd), then round that
// f32 to 8 significant bits.  f32 keeps 16 more bits than bf16, so the two-step result equals the
// direct rounding of the fp64 value.
__device__ __forceinline__ uint16_t double_to_bf16_bits(double x) {
    float f = __double2float_rz(x);
    uint32_t u = __float_as_uint(f);
    if ((double)f != x && (u & 0x7f800000u) != 0x7f800000u) u |= 1u;
    if ((u & 0x7fffffffu) > 0x7f800000u) return (uint16_t)((u >> 16) | 0x40);   // NaN stays NaN
    u += 0x7fffu + ((u >> 16) & 1u);
    return (uint16_t)(u >> 16);
}
__device__ __forceinline__ uint16_t float_to_bf16_bits(float f) {
    return __bfloat16_as_ushort(__float2bfloat16_rn(f));
}
// 8-bit e4m3 codes: round to nearest even, finite overflow and infinity saturate to +-448, NaN stays NaN
__device__ __forceinline__ uint8_t float_to_e4m3_bits(float f) { return (uint8_t)__nv_cvt_float_to_fp8(f, __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ uint8_t double_to_e4m3_bits(double x) { return (uint8_t)__nv_cvt_double_to_fp8(x, __NV_SATFINITE, __NV_E4M3); }

// One pair of y = x R_pos^T in fp64.
__device__ __forceinline__ void rope_pair(double x0, double x1, int pos, double inv_freq, double &y0, double &y1) {
    double s, c;
    sincos((double)pos * inv_freq, &s, &c);
    y0 = x0 * c - x1 * s;
    y1 = x0 * s + x1 * c;
}

}  // namespace gva
