// kv4.h -- the 4-bit KV block: its layout and the hardware's conversions between
// e2m1 codes and 16-bit or fp32 values.
//
// The 128 channels of a token's key (or value) are four groups of 32.  A group is 32 e2m1
// codes (sign and 0, .5, 1, 1.5, 2, 3, 4, 6) and one byte e + 127 of its scale 2^e (255: NaN).
// A block is num_kv_heads regions of 136 * bs bytes, one per KV head:
//   keys    [bs][64]            byte i of a token: channel 2i in the low half, 2i + 1 in the high
//   values  [bs/8][16][8]       words of 32 bits; word [o][c % 16][c / 16] holds channel c of tokens
//                               8o .. 8o + 7, token 8o in the lowest 4 bits
//   key scales [bs][4], value scales [4][bs]
// so that a lane's MFMA operands are whole 16-byte loads: of a key row the 32 channels of one
// group, under one scale; of the values 8 tokens of 8 channels 16 apart.
#pragma once

#include "pulse_internal.h"

namespace pulse {

constexpr int kGroup = 32;                     // channels under one scale
constexpr int kGroups = kHeadDim / kGroup;     // scales of a token's key or value
constexpr int kKv4Nan = 255;

// Offsets within a head's region of a block of bs tokens.
__host__ __device__ constexpr int kv4_values(int bs) { return 64 * bs; }
__host__ __device__ constexpr int kv4_key_scales(int bs) { return 128 * bs; }
__host__ __device__ constexpr int kv4_value_scales(int bs) { return 132 * bs; }
__host__ __device__ constexpr int kv4_head_bytes(int bs) { return 136 * bs; }

// 2^e of a scale byte as fp32 (byte 0 as 0, byte 255 as infinity).
__device__ inline float kv4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Scale byte for a group whose largest magnitude is `top`: the least e with top <= 7 * 2^e (a value
// between 6 and 7 is nearer to 6 than the next scale's step would round the others), kept where every
// product of a code and 2^e is a value of the 16-bit type.
template <int DT>
__device__ inline uint32_t kv4_scale_byte(float top) {
    const uint32_t u = __float_as_uint(top);
    if (u >= 0x7F800000u) return kKv4Nan;
    const int e = (int)(u >> 23) - 127 - 2 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    const int lo = DT == PULSE_BF16 ? -100 : -23, hi = DT == PULSE_BF16 ? 125 : 13;
    return (uint32_t)(min(max(e, lo), hi) + 127);
}

// Two values over `scale` as codes in the lowest byte: nearest, ties to the even code, saturated at 6.
__device__ inline uint32_t kv4_encode(float a, float b, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, a, b, scale, 0) & 0xFFu;
}

// Codes of byte SEL of w, times `scale`, as two 16-bit values (exact).
template <int DT, int SEL>
__device__ inline uint32_t kv4_decode(uint32_t w, float scale) {
    if constexpr (DT == PULSE_BF16)
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
    else
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, SEL));
}

// Eight codes as an MFMA operand.
template <int DT>
__device__ inline typename Mfma<DT>::vec kv4_decode8(uint32_t w, float scale) {
    const u32x4 v = {kv4_decode<DT, 0>(w, scale), kv4_decode<DT, 1>(w, scale), kv4_decode<DT, 2>(w, scale),
                     kv4_decode<DT, 3>(w, scale)};
    return __builtin_bit_cast(typename Mfma<DT>::vec, v);
}

}  // namespace pulse
