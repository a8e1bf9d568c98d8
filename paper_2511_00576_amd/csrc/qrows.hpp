// Rows of the 8-bit cache (eva_qcache): d e4m3 codes and one exponent byte,
// value = code 2^(byte - 127).  The exponent is the smallest whose power of
// two brings the row's largest finite magnitude to 448, e4m3's largest value,
// or below.  A power of two scales exactly both ways, so a code differs from
// the row's value by its one rounding, half a step (2^-4 of an entry: 3 mantissa
// bits), and rows of the same values have the same codes wherever they are
// quantised; a row's small entries lose nothing more, since the codes have
// exponents of their own, until they are subnormal, below 2^-6 of the row's power
// of two, where half a step is 2^-10 of that (so from 2^-13 of the row's largest, which
// lies in (224, 448], every code is a normal one).
#pragma once

#include "eva_device.hpp"
#include "eva_kernels.hpp"

namespace eva {

// 16 slots of one feature are 16 contiguous bytes: row r, feature f of a
// transposed value array lies at byte (r / 16) 16 D + 16 f + r % 16.
constexpr int kQTile = 16;
template <int D>
__host__ __device__ __forceinline__ size_t qt_index(int f, int r) {
    return (size_t)(r >> 4) * (kQTile * D) + (size_t)f * kQTile + (r & 15);
}

__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < INFINITY; }

// Exponent byte of a row whose largest finite magnitude is amax.  At most 119 + 127:
// a scale meets softmax weights of up to 2^kTreeTau = 2^8, and 2^127 is the last power of two.
// Magnitudes past 464 2^119 = 3.08e38 round past the last code, 448, to NaN, e4m3's
// own conversion.
__device__ __forceinline__ uint32_t q_exponent(float amax) {
    if (amax == 0.f) return 127;
    // amax = m 2^e, 1/2 <= m < 1: 448 = 7/8 2^9
    const int e = __builtin_amdgcn_frexp_expf(amax) - 9 + (__builtin_amdgcn_frexp_mantf(amax) > 0.875f ? 1 : 0);
    return (uint32_t)(min(max(e, -126), 119) + 127);
}
__device__ __forceinline__ float q_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Codes of eight features; inv = 2^-(byte - 127).  Values that are not finite
// become e4m3's NaN.
__device__ __forceinline__ u32x2 q_codes(const float x[8], float inv) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = is_finite(x[i]) ? x[i] * inv : __uint_as_float(0x7fc00000u);
    u32x2 w;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        int v = 0;
        v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h], y[4 * h + 1], v, false);
        v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h + 2], y[4 * h + 3], v, true);
        w[h] = (uint32_t)v;
    }
    return w;
}
__device__ __forceinline__ float q_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// One row held by D / 8 neighbouring lanes of eight features: its exponent
// byte (in every lane) and this lane's codes.
template <int D>
__device__ __forceinline__ uint32_t q_row(const float x[8], u32x2& codes) {
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, is_finite(x[i]) ? fabsf(x[i]) : 0.f);
#pragma unroll
    for (int off = 1; off < D / 8; off <<= 1) amax = fmaxf(amax, __shfl_xor(amax, off, 64));
    const uint32_t byte = q_exponent(amax);
    codes = q_codes(x, q_inverse(byte));
    return byte;
}

// Value of one code.
__device__ __forceinline__ float q_value(uint32_t code, float scale) {
    return __builtin_amdgcn_cvt_f32_fp8((int)code, 0) * scale;
}
// Two codes (the low or high half of w) as bf16, exactly.
template <bool HI>
__device__ __forceinline__ uint32_t q_bf16x2(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, HI));
}
// Eight codes as a matrix-core operand fragment.
__device__ __forceinline__ bf16x8 q_bf16x8(uint32_t lo, uint32_t hi) {
    return __builtin_bit_cast(bf16x8, u32x4{q_bf16x2<false>(lo), q_bf16x2<true>(lo), q_bf16x2<false>(hi), q_bf16x2<true>(hi)});
}

// Whether one of 16 codes is a NaN.
__device__ __forceinline__ bool q_has_nan(const u32x4& w) {
    uint32_t x = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) x |= (w[i] & 0x7f7f7f7fu) + 0x01010101u;  // bit 7 of a byte: it is 0x7f
    return (x & 0x80808080u) != 0;
}
// 16 exponent bytes of which some may be stale: 255, an infinite scale, becomes
// 254 (no row has it), so that a weight of zero stays zero.
__device__ __forceinline__ u32x4 q_finite_scales(u32x4 w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] ^= (((w[i] & 0x7f7f7f7fu) + 0x01010101u) & w[i] & 0x80808080u) >> 7;
    return w;
}

// Eight bf16 features as fp32.
__device__ __forceinline__ void unpack8(const u32x4& w, float out[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        out[2 * i] = bf16_lo(w[i]);
        out[2 * i + 1] = bf16_hi(w[i]);
    }
}
__device__ __forceinline__ void row8(const bf16* p, float out[8]) { unpack8(*reinterpret_cast<const u32x4*>(p), out); }

// Rows of a chunk in the 8-bit ring.
template <int D>
struct QRingChunk {
    const uint8_t* k;   // this (b, g): [R][D]
    const uint8_t* vt;  // [R / 16][D][16]
    const uint8_t* ke;  // [R]
    const uint8_t* ve;
    long long pos0;
    int R;
    __device__ int slot(int r) const { return (int)((pos0 + r) % R); }
};

}  // namespace eva
