// Tiles of the fp8 (E4M3) cache that take new tokens: the rule that
// sf_kv_store_fp8 states in sf_decode_attn.h, for one wave per tile. Shared by
// the store of new tokens and by the moves of an eviction.
//
// A lane holds the same 16-byte pieces of a tile as in the attention kernels,
// D / 64 of them, each 16 codes. Of a key tile piece p of lane (grp, col) is
// slot col, dims 64 p + 8 grp + e (e < 8) and 64 p + 32 + 8 grp + e - 8; of a
// value tile code 4 j + e is slot 4 grp + e, dim 64 p + 16 j + col.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sf {

typedef uint32_t tile_u32x4 __attribute__((ext_vector_type(4)));
typedef float tile_f32x2 __attribute__((ext_vector_type(2)));

// The smallest maximum that a scale is made from: 448 / 2^-100 and 2^-100 / 448
// are normal fp32 numbers, so neither a factor nor a scale is 0, infinite or
// subnormal (values below 2^-110 become code 0).
constexpr float kFp8SmallestMax = 0x1p-100f;

__device__ __forceinline__ float fp8_value(uint32_t codes, int byte) {
  switch (byte) {   // the byte is part of the instruction
    case 0: return __builtin_amdgcn_cvt_f32_fp8(int(codes), 0);
    case 1: return __builtin_amdgcn_cvt_f32_fp8(int(codes), 1);
    case 2: return __builtin_amdgcn_cvt_f32_fp8(int(codes), 2);
    default: return __builtin_amdgcn_cvt_f32_fp8(int(codes), 3);
  }
}

// Four values to codes, round to nearest even.
__device__ __forceinline__ uint32_t fp8_codes(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true));
}

// Byte mask of this lane's words for the slots in `slots` (bit t: slot t): the
// same for every word of a piece (all bytes of a key piece are slot col; byte
// e of a value word is slot 4 grp + e).
__device__ __forceinline__ uint32_t fp8_slot_bytes(uint32_t slots, bool is_v, int lane) {
  if (!is_v) return (slots >> (lane & 15)) & 1u ? 0xFFFFFFFFu : 0u;
  const uint32_t four = (slots >> (4 * (lane >> 4))) & 15u;
  return (four & 1u ? 0xFFu : 0u) | (four & 2u ? 0xFF00u : 0u) | (four & 4u ? 0xFF0000u : 0u) |
         (four & 8u ? 0xFF000000u : 0u);
}

// Scale of a tile that takes new values whose largest magnitude is top, the
// power of two that its held codes are divided by, and the factor of the new ones.
struct Fp8Scale {
  float scale, factor;
  int shift;
};
__device__ __forceinline__ Fp8Scale fp8_new_scale(float scale, bool used, float top) {
  Fp8Scale r = {1.f, 1.f, 0};
  if (!used) {
    if (top > 0.f) {
      const float m = fmaxf(top, kFp8SmallestMax);
      r.scale = __fdiv_rn(m, 448.f);
      r.factor = __fdiv_rn(448.f, m);
    }
    return r;
  }
  const float ratio = __fdiv_rn(top, __fmul_rn(448.f, scale));
  if (ratio > 1.f) {   // ceil(log2 ratio), from its bits
    const uint32_t b = __builtin_bit_cast(uint32_t, ratio);
    r.shift = int(b >> 23) - 127 + ((b & 0x7FFFFFu) ? 1 : 0);
  }
  r.scale = __builtin_amdgcn_ldexpf(scale, r.shift);
  r.factor = __fdiv_rn(1.f, r.scale);
  return r;
}

// Stores a tile: `old` is what it holds (with `read`; else nothing of it is
// kept), of which the bytes set in keep belong to held slots, old_scale its
// scale, and x the values of the slots whose bytes are set in fresh (16 per
// piece, in the order of the codes; 0 elsewhere). The whole wave calls it. Lanes
// whose pieces stay as they are write nothing: a single token then touches a
// quarter of the tile.
template <int D>
__device__ __forceinline__ void fp8_store_tile(const tile_u32x4 (&old)[D / 64], bool read, uint32_t keep,
                                               const float (&x)[D / 64][16], uint32_t fresh, float old_scale,
                                               uint8_t* tile, float* scale, int lane) {
  constexpr int kPieces = D / 64;
  tile_u32x4 codes[kPieces];
#pragma unroll
  for (int p = 0; p < kPieces; ++p) codes[p] = old[p] & keep;
  uint32_t any = 0;
  float top = 0.f;
#pragma unroll
  for (int p = 0; p < kPieces; ++p) {
#pragma unroll
    for (int j = 0; j < 4; ++j) any |= codes[p][j] & 0x7F7F7F7Fu;
#pragma unroll
    for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(x[p][e]));
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
  const Fp8Scale s = fp8_new_scale(old_scale, __any(any != 0), top);
#pragma unroll
  for (int p = 0; p < kPieces; ++p) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t w = codes[p][j];
      if (s.shift > 0)   // wave-uniform, rare
        w = fp8_codes(__builtin_amdgcn_ldexpf(fp8_value(w, 0), -s.shift), __builtin_amdgcn_ldexpf(fp8_value(w, 1), -s.shift),
                      __builtin_amdgcn_ldexpf(fp8_value(w, 2), -s.shift), __builtin_amdgcn_ldexpf(fp8_value(w, 3), -s.shift));
      const uint32_t n = fp8_codes(x[p][4 * j] * s.factor, x[p][4 * j + 1] * s.factor, x[p][4 * j + 2] * s.factor,
                                   x[p][4 * j + 3] * s.factor);
      codes[p][j] = (w & ~fresh) | (n & fresh);
    }
  }
  if (!read) {   // wave-uniform
#pragma unroll
    for (int p = 0; p < kPieces; ++p) *reinterpret_cast<tile_u32x4*>(tile + 1024 * p + 16 * lane) = codes[p];
  } else {
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      const tile_u32x4 changed = codes[p] ^ old[p];
      if ((changed[0] | changed[1] | changed[2] | changed[3]) != 0)
        *reinterpret_cast<tile_u32x4*>(tile + 1024 * p + 16 * lane) = codes[p];
    }
  }
  if (lane == 0 && (!read || s.scale != old_scale)) *scale = s.scale;
}

}  // namespace sf
