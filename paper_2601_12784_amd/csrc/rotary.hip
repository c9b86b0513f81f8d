// Rotary positions: queries and keys turned by their positions, alone or on
// the way into the pages of a bf16 cache (sf_rotary, sf_rotary_store).
//
// Angles. A turn is 2^64 units, so position * (units per position) modulo 2^64
// is the angle's fraction of a turn with no rounding at all; its nearest quarter
// turn is an addition and a shift, what is left of it lies within an eighth of a
// turn, and sine and cosine there are short polynomials. An angle in fp32 would be off by
// 2^-24 of itself: 0.008 at position 131072.
//
// Memory bounds it: every element is read and written once. A thread
// takes 16 dims (8 pairs, two 16-byte pieces) of one token, forms their sines and cosines
// once and walks over heads with them. Values take the transposition that their
// page layout asks for in registers: a thread reads two dims of 16 tokens
// and writes 2 x 32 contiguous bytes.
//
// Measured: 8192 tokens of 32 + 8 heads of 128 38 us = 4.4 TB/s, the tokens of 32 prompts into their
// pages 230 us = 4.5 TB/s (a copy of 4 GiB here: 4.6). Few tokens alone are bound by the launch (3 us) and the host; the 512
// of a step with their store by reads that wait for each other (list row over PCIe, block table, keys, then values: 11 us
// where the bytes take 2) and by values of 2 bytes 32 bytes apart, as the layout has them.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sf_internal.h"

namespace sf {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(4))) const int32_t* const_i32_ptr;
__device__ __forceinline__ const_i32_ptr as_constant(const int32_t* p) { return (const_i32_ptr)(p); }

constexpr int kThreads = 256;
constexpr int kBatch = 2;   // heads whose loads a thread has in flight together

struct Turn {
  float cos, sin;
};

// Sine and cosine of phase 2^-64 turns, times m. The polynomials are the Taylor
// series to x^9 and x^8: for |x| <= pi/4 the next terms are below 2e-9 and 2.5e-8.
__device__ __forceinline__ Turn turn_of(uint64_t phase, float m) {
  const uint64_t up = phase + (uint64_t(1) << 61);
  const uint32_t quarter = uint32_t(up >> 62);
  const int32_t rest = int32_t(uint32_t((phase - (up & (uint64_t(3) << 62))) >> 32));   // 2^-32 turns, within 2^29
  const float x = float(rest) * 1.46291807926715968e-9f;                               // 2 pi 2^-32
  const float y = x * x;
  const float s = x * (1.f + y * (-1.f / 6 + y * (1.f / 120 + y * (-1.f / 5040 + y * (1.f / 362880)))));
  const float c = 1.f + y * (-0.5f + y * (1.f / 24 + y * (-1.f / 720 + y * (1.f / 40320))));
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return {(quarter == 1 || quarter == 2) ? -a * m : a * m, quarter >= 2 ? -b * m : b * m};
}

__device__ __forceinline__ float low(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

struct Pieces {
  u32x4 x, y;
};

// The turn of a pair, with its two fused products named: left to the compiler, another copy of the loop fused the others,
// and where the sum nearly cancels a head's bits followed from the launch's shape.
__device__ __forceinline__ float first_of(float a, float b, const Turn& t) { return __builtin_fmaf(a, t.cos, -(b * t.sin)); }
__device__ __forceinline__ float second_of(float a, float b, const Turn& t) { return __builtin_fmaf(b, t.cos, a * t.sin); }

// The two pieces' 8 pairs: (x[i], y[i]) in the half layout, neighbours in the
// interleaved one.
template <bool kInterleaved>
__device__ __forceinline__ Pieces turned(const Pieces& p, const Turn* t) {
  Pieces r;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if constexpr (kInterleaved) {
      const Turn t0 = t[w], t1 = t[4 + w];
      const float a0 = low(p.x[w]), b0 = high(p.x[w]), a1 = low(p.y[w]), b1 = high(p.y[w]);
      r.x[w] = pack(first_of(a0, b0, t0), second_of(a0, b0, t0));
      r.y[w] = pack(first_of(a1, b1, t1), second_of(a1, b1, t1));
    } else {
      const Turn t0 = t[2 * w], t1 = t[2 * w + 1];
      const float a0 = low(p.x[w]), a1 = high(p.x[w]), b0 = low(p.y[w]), b1 = high(p.y[w]);
      r.x[w] = pack(first_of(a0, b0, t0), first_of(a1, b1, t1));
      r.y[w] = pack(second_of(a0, b0, t0), second_of(a1, b1, t1));
    }
  }
  return r;
}

// A page's tokens as a workgroup works on them.
struct Tile {
  int tokens;     // 1 .. 16
  int64_t row0;   // query row of the first
  int slot0;      // its slot (storing)
  int64_t page;   // (storing)
};

template <int D, bool kStore, bool kInterleaved>
__device__ __forceinline__ void turn_tile(const RotaryArgs& a, const Tile& t, int first_pos, int part, int parts) {
  constexpr int kUnits = D / 16;
  const int unit = int(threadIdx.x) % kUnits, rest = int(threadIdx.x) / kUnits;
  const int tok = rest % t.tokens, lane = rest / t.tokens, lanes = kThreads / kUnits / t.tokens;
  if (lane >= lanes) return;
  const int heads = a.num_q_heads + a.num_kv_heads;
  const int64_t row = t.row0 + tok;
  const int32_t pos = kStore ? first_pos + tok : a.positions[row];
  const bool turns = unit < a.rotary_dim / 16;
  const int dx = !kInterleaved && turns ? 8 * unit : 16 * unit;
  const int dy = !kInterleaved && turns ? a.rotary_dim / 2 + 8 * unit : 16 * unit + 8;
  Turn turn[8];
  if (turns) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn[i] = turn_of(uint64_t(int64_t(pos)) * a.turns[8 * unit + i], a.magnitude);
  }
  const int step = lanes * parts;
  for (int h0 = part * lanes + lane; h0 < heads; h0 += kBatch * step) {
    Pieces p[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int h = h0 + b * step;
      if (h >= heads) break;
      const uint16_t* src = h < a.num_q_heads ? a.q + row * a.q_stride + h * D : a.k + row * a.k_stride + (h - a.num_q_heads) * D;
      p[b].x = *reinterpret_cast<const u32x4*>(src + dx);
      p[b].y = *reinterpret_cast<const u32x4*>(src + dy);
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int h = h0 + b * step;
      if (h >= heads) break;
      const Pieces r = turns ? turned<kInterleaved>(p[b], turn) : p[b];
      if (h < a.num_q_heads || !kStore) {
        uint16_t* dst = h < a.num_q_heads ? a.q_out + row * a.q_out_stride + h * D
                                          : a.k_out + row * a.k_out_stride + (h - a.num_q_heads) * D;
        *reinterpret_cast<u32x4*>(dst + dx) = r.x;
        *reinterpret_cast<u32x4*>(dst + dy) = r.y;
      } else {
        // K tile [D/8][16][8]
        uint16_t* tile = a.k_pool + (t.page * a.num_kv_heads + (h - a.num_q_heads)) * (kPage * D) + (t.slot0 + tok) * 8;
        *reinterpret_cast<u32x4*>(tile + dx * kPage) = r.x;
        *reinterpret_cast<u32x4*>(tile + dy * kPage) = r.y;
      }
    }
  }
}

// Values of a page's tokens into its V tiles [D][16].
template <int D>
__device__ __forceinline__ void store_values(const RotaryArgs& a, const Tile& t, int part, int parts) {
  constexpr int kPairs = D / 2;
  const uint16_t* src = a.v + t.row0 * a.v_stride;
  uint16_t* page = a.v_pool + t.page * a.num_kv_heads * (kPage * D);
  if (t.tokens == kPage) {
    for (int i = part * kThreads + int(threadIdx.x); i < a.num_kv_heads * kPairs; i += parts * kThreads) {
      const int at = 2 * i;   // (head, dim) in a token's row
      uint32_t w[kPage];
#pragma unroll
      for (int k = 0; k < kPage; ++k) w[k] = *reinterpret_cast<const uint32_t*>(src + k * a.v_stride + at);
      u32x4 even[2], odd[2];
#pragma unroll
      for (int k = 0; k < kPage / 2; ++k) {
        even[k / 4][k % 4] = __builtin_amdgcn_perm(w[2 * k + 1], w[2 * k], 0x05040100u);
        odd[k / 4][k % 4] = __builtin_amdgcn_perm(w[2 * k + 1], w[2 * k], 0x07060302u);
      }
      u32x4* dst = reinterpret_cast<u32x4*>(page + size_t(at) * kPage);
      dst[0] = even[0];
      dst[1] = even[1];
      dst[2] = odd[0];
      dst[3] = odd[1];
    }
    return;
  }
  const int n = a.num_kv_heads * kPairs;
  for (int i = part * kThreads + int(threadIdx.x); i < n * t.tokens; i += parts * kThreads) {
    const int tok = i / n, at = 2 * (i % n);
    const uint32_t w = *reinterpret_cast<const uint32_t*>(src + tok * a.v_stride + at);
    uint16_t* dst = page + size_t(at) * kPage + t.slot0 + tok;
    dst[0] = uint16_t(w);
    dst[kPage] = uint16_t(w >> 16);
  }
}

template <int D, bool kInterleaved>
__global__ __launch_bounds__(kThreads) void rotary_store_kernel(RotaryArgs a) {
  const const_i32_ptr row = as_constant(a.rows) + size_t(blockIdx.x) * kItemInts;
  const int seq = row[0], pb = row[1], np = row[2], first = row[3], end = row[4], qrow = row[5], pos0 = row[6];
  const int part = int(blockIdx.y), parts = int(gridDim.y);
  const int opened = a.new_pages ? as_constant(a.new_pages)[seq] : -1;
  const int last = (end - 1) / kPage;
  const size_t entry0 = size_t(seq) * a.bt_stride;
  for (int pg = pb; pg < pb + np; ++pg) {
    const bool fresh = pg == last && opened >= 0;
    const int page = fresh ? opened : as_constant(a.block_table)[entry0 + pg];
    const int lo = max(first, pg * kPage), hi = min(end, (pg + 1) * kPage);
    const Tile t = {hi - lo, int64_t(qrow) + (lo - first), lo - pg * kPage, page};
    turn_tile<D, true, kInterleaved>(a, t, pos0 + (lo - first), part, parts);
    store_values<D>(a, t, part, parts);
    if (fresh && part == 0 && threadIdx.x == 0) a.block_table[entry0 + pg] = page;
  }
}

template <int D, bool kInterleaved>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a, int per_tile) {
  const int64_t row0 = int64_t(blockIdx.x) * per_tile;
  const Tile t = {int(min(int64_t(per_tile), a.num_tokens - row0)), row0, 0, 0};
  turn_tile<D, false, kInterleaved>(a, t, 0, int(blockIdx.y), int(gridDim.y));
}

template <int D, bool kInterleaved>
hipError_t launch(const RotaryArgs& a, hipStream_t stream) {
  const int heads = a.num_q_heads + a.num_kv_heads;
  // tokens that share a workgroup's tile: all of a page's, or in the plain form one, four of many (28 + 4 heads of 128, one,
  // four and sixteen to a tile: 8192 tokens 31.0, 29.8 and 30.9 us, 17000 54.9, 56.2 and 63.2, 32768 100, 101 and 111),
  // and sixteen where a launch would have 2^32 threads
  const int per_tile = a.rows ? kPage : a.num_tokens > 1 << 24 ? 16 : a.num_tokens >= 4096 ? 4 : 1;
  const int64_t tiles = a.rows ? a.num_rows : (int64_t(a.num_tokens) + per_tile - 1) / per_tile;
  // few tiles: their heads are split over workgroups
  const int lanes = kThreads / (D / 16) / (a.rows && a.num_tokens <= a.num_rows ? 1 : per_tile);
  const int most = (heads + lanes - 1) / lanes;
  const int parts = int(max(int64_t(1), min(int64_t(most), 1024 / tiles)));
  const dim3 grid{uint32_t(tiles), uint32_t(parts), 1};
  if (a.rows)
    rotary_store_kernel<D, kInterleaved><<<grid, kThreads, 0, stream>>>(a);
  else
    rotary_kernel<D, kInterleaved><<<grid, kThreads, 0, stream>>>(a, per_tile);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream) {
  if (a.head_dim == 128) return a.interleaved ? launch<128, true>(a, stream) : launch<128, false>(a, stream);
  return a.interleaved ? launch<64, true>(a, stream) : launch<64, false>(a, stream);
}

}  // namespace sf
