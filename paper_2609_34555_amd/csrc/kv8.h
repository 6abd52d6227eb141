// kv8.h -- the 8-bit KV block: its layout and the hardware's conversions between e4m3
// codes and 16-bit or fp32 values.
//
// The keys of one head in one block share the scale 2^e, and so do its values: a code c
// (e4m3: sign, 4 bits of exponent, 3 of mantissa; up to 448, subnormals down to 2^-9, 0x7F
// NaN) stands for c * 2^e.  A block is num_kv_heads regions of 256 * bs bytes, then the
// scales:
//   keys    [bs][128]           a byte per channel
//   values  [bs/8][16][8][8]    channel c of token t at [t / 8][c % 16][c / 16][t % 8]
//   scales  [num_kv_heads][2]   bytes e + 127 of keys and values, padded to 128 bytes
// so that a lane's MFMA operands are whole 16-byte loads (of a key row 32 channels, of the
// values 8 tokens of 8 channels 16 apart) and every region begins on a 128-byte line.
#pragma once

#include "pulse_internal.h"

namespace pulse {

// Offsets within a head's region of a block of bs tokens, and within the block.
__host__ __device__ constexpr int kv8_values(int bs) { return 128 * bs; }
__host__ __device__ constexpr int kv8_head_bytes(int bs) { return 256 * bs; }
__host__ __device__ constexpr int64_t kv8_scales(int64_t heads, int bs) { return heads * kv8_head_bytes(bs); }
__host__ __device__ constexpr int64_t kv8_block_bytes(int64_t heads, int bs) {
    return kv8_scales(heads, bs) + (2 * heads + 127) / 128 * 128;
}

// Exponents of a scale: every product of a code and 2^e is a value of the 16-bit type (a bf16 normal, an fp16 of at
// most 57344 and a multiple of 2^-24).
template <int DT>
struct Kv8Range {
    static constexpr int lo = DT == PULSE_BF16 ? -100 : -15, hi = DT == PULSE_BF16 ? 119 : 7;
};

// 2^e as fp32, for e in -126 .. 127.
__device__ inline float kv8_pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Exponent for values whose largest finite magnitude is `top`: the least e with top <= 448 * 2^e, within the range.
// (A floating format loses nothing to an unused factor of two but at its subnormal end, so a scale that is a power of
// two costs no accuracy, and codes change to another scale exactly above that end.)
template <int DT>
__device__ inline int kv8_exponent(float top) {
    const uint32_t u = __float_as_uint(top);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return min(max(e, Kv8Range<DT>::lo), Kv8Range<DT>::hi);
}

// Two values as the codes of a byte pair: nearest, ties to even, saturated at 448 (an fp16 beyond 57344); infinities and
// NaN become NaN.
__device__ inline uint32_t kv8_encode(float a, float b) {
    const float inf = INFINITY;
    a = fabsf(a) < inf ? __builtin_amdgcn_fmed3f(a, -448.f, 448.f) : __uint_as_float(0x7FC00000u);
    b = fabsf(b) < inf ? __builtin_amdgcn_fmed3f(b, -448.f, 448.f) : __uint_as_float(0x7FC00000u);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xFFFFu;
}

// Codes of half SEL of w (0: low), times `scale`, as two 16-bit values (exact).
template <int DT, int SEL>
__device__ inline uint32_t kv8_decode(uint32_t w, float scale) {
    if constexpr (DT == PULSE_BF16)
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, SEL));
    else
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, SEL));
}

// Eight codes as an MFMA operand.
template <int DT>
__device__ inline typename Mfma<DT>::vec kv8_decode8(u32x2 w, float scale) {
    const u32x4 v = {kv8_decode<DT, 0>(w[0], scale), kv8_decode<DT, 1>(w[0], scale), kv8_decode<DT, 0>(w[1], scale),
                     kv8_decode<DT, 1>(w[1], scale)};
    return __builtin_bit_cast(typename Mfma<DT>::vec, v);
}

// Four codes under another scale: times `factor`, rounded again.
__device__ inline uint32_t kv8_rescale4(uint32_t w, float factor) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    return kv8_encode(a[0] * factor, a[1] * factor) | kv8_encode(b[0] * factor, b[1] * factor) << 16;
}

}  // namespace pulse
