// Codes of the paged cache in 8 bits (gfx950): e4m3 and int8, in units of a power of two whose byte is
// 127 + its exponent, the exponent field of the fp32 number it is.
#pragma once

#include "mf_device.h"
#include "paged_attn.h"

namespace mf {

__device__ __forceinline__ float power_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// The largest magnitude that is held: its codes, and what they are rounded up to, are finite in the type.
template <bool BF16, bool INT8>
constexpr float kHeld = INT8 ? (BF16 ? 127 * 0x1p121f : 65024.f) : BF16 ? 240 * 0x1p120f : 61440.f;
// The least byte: fp16 has no smaller step (int8) and e4m3's steps of 2^-9 units are no smaller; in bf16 every value that is held is
// normal.
template <bool BF16, bool INT8>
constexpr uint32_t kLeastByte = BF16 ? 127 - 110 : INT8 ? 127 - 24 : 127 - 15;

// The least power of two, as its byte, that takes magnitudes up to `top` to codes: 448 = 1.75 * 2^8, 127 = 1.984375 * 2^6.
template <bool BF16, bool INT8>
__device__ __forceinline__ uint32_t byte_for(float top) {
  const uint32_t u = __builtin_bit_cast(uint32_t, fminf(top, kHeld<BF16, INT8>));
  const int byte = (int)((u + (INT8 ? 0x01ffffu : 0x1fffffu)) >> 23) - (INT8 ? 6 : 8);
  return (uint32_t)max(byte, (int)kLeastByte<BF16, INT8>);
}

// Four values in units of the scale (magnitudes within the codes', or NaN) as codes, to nearest, ties to even.
template <bool INT8>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  if constexpr (INT8) {
    // (1.5 * 2^23: the sum's last bits are the whole number; NaN is held as 0)
    auto whole = [](float x) { return __builtin_bit_cast(uint32_t, (x != x ? 0.f : x) + 12582912.f); };
    const uint32_t lo = __builtin_amdgcn_perm(whole(b), whole(a), 0x0c0c0400u), hi = __builtin_amdgcn_perm(whole(d), whole(c), 0x04000c0cu);
    return lo | hi;
  } else {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
  }
}

// Two pairs of the type as codes in units of 1 / inverse.
template <bool BF16, bool INT8>
__device__ __forceinline__ uint32_t encode_pairs(uint32_t xy, uint32_t zw, float inverse) {
  auto held = [&](uint32_t bits) {
    const float x = to_float<BF16>(bits), y = fminf(fmaxf(x, -kHeld<BF16, INT8>), kHeld<BF16, INT8>);
    return (x != x ? x : y) * inverse;
  };
  return encode4<INT8>(held(xy & 0xffffu), held(xy >> 16), held(zw & 0xffffu), held(zw >> 16));
}

// Four codes as fp32 values.
template <bool INT8>
__device__ __forceinline__ f32x4 decode4(uint32_t codes, float scale) {
  if constexpr (INT8) {
    const int x = (int)codes;
    return (f32x4){(float)(int8_t)x * scale, (float)(int8_t)(x >> 8) * scale, (float)(int8_t)(x >> 16) * scale, (float)(x >> 24) * scale};
  } else {
    const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, true);
    return (f32x4){lo.x, lo.y, hi.x, hi.y};
  }
}

// Four int8 codes as whole numbers of the type, in two pairs.
template <bool BF16>
__device__ __forceinline__ u32x2 whole_pairs(uint32_t codes) {
  if constexpr (BF16) {
    // (a number of 7 bits has no more in fp32 than in its upper half)
    const f32x4 x = decode4<true>(codes, 1.f);
    auto pair = [](float a, float b) { return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u); };
    return (u32x2){pair(x[0], x[1]), pair(x[2], x[3])};
  } else {
    // 0x64 above the code + 128 is 1024 + that; its difference from 1152 is the code.
    const uint32_t u = codes ^ 0x80808080u;
    const half2_t zero = {(_Float16)1152.f, (_Float16)1152.f};
    return (u32x2){__builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - zero),
                   __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - zero)};
  }
}

// Four codes as values of the type, exactly, in two pairs.
template <bool BF16, bool INT8>
__device__ __forceinline__ u32x2 decode_pairs(uint32_t codes, float scale) {
  if constexpr (!INT8) {
    if constexpr (BF16)
      return (u32x2){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true))};
    else
      return (u32x2){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, true))};
  } else if constexpr (BF16) {
    const f32x4 x = decode4<true>(codes, scale);
    return (u32x2){pack2<true>(x[0], x[1]), pack2<true>(x[2], x[3])};
  } else {
    const u32x2 x = whole_pairs<false>(codes);
    const half2_t s = {(_Float16)scale, (_Float16)scale};
    auto scaled = [&](uint32_t pair) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, pair) * s); };
    return (u32x2){scaled(x.x), scaled(x.y)};
  }
}

}  // namespace mf
