// gfx950 kernels of a decode step whose sequences share their first tokens in
// groups: several trajectories sampled from one prompt.
//
// A prompt's pages are read once for all members. Their query rows (members times
// the g query heads of a KV head) fill tiles of 16 matrix-core columns, two
// per wave, so a K or V operand that a wave has loaded meets up to 32 rows; a prompt with
// more rows has several waves walk the same pages side by side, each with its own 32. What a sequence
// has to itself is a walk with the g rows of one sequence. Per block of two pages (32 keys) and tile,
//
//   S^T[16 keys][16 rows] = K Q^T per page   (D/32) v_mfma_f32_16x16x32_bf16 each
//   weights 2^(z - m), the row's reference m moved only when a block's weights grow past 2^kHeadroom
//   O^T[D][16 rows]      += V^T P^T           (D/16) x 2 MFMAs, P as two bf16 parts (16 bits of each weight)
//
// A sequence's own operands come straight from memory to registers (the page layouts are the
// operands' own), a prompt's through LDS, which all waves of its workgroup read; two waves per SIMD. A wave
// (worker) walks an equal share of the pages; its results are rows of normalized
// output with their log-sum-exp, which a second launch joins per (sequence, KV head).
//
// What bounds it: own pages memory (16 prompts of 2048 tokens with 16 samples each, 484 MB in all: 102 us, of which
// the merge is 6), prompts with hundreds of rows the matrix and the vector work of their blocks, which eight waves in
// step hardly overlap (32760 tokens under 64 samples of 8 x 4 heads: 89 us; matrix cores busy 27 % of it, vector units 30). Without LDS, every
// wave reading the prompt's pages for itself, these took 210 and 165 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "sf_internal.h"

namespace sf {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(4))) const int32_t* const_i32_ptr;
typedef __attribute__((address_space(4))) const float* const_f32_ptr;

constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kHeadroom = 1024.f;   // most that a lane's eight weights of a block may sum to

__device__ __forceinline__ const_i32_ptr as_constant(const int32_t* p) { return (const_i32_ptr)(p); }

__device__ __forceinline__ f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
__device__ __forceinline__ float low_bf16(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }
template <bool kHigh>
__device__ __forceinline__ uint32_t widen2(uint32_t codes4) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes4, 1.0f, kHigh));
}

struct Item {
  int seq0, source, kvh, pb, pe, end, slot, row0, rows, blocks, split, member, within;
};

// Lane's position in the MFMA layouts.
struct Lane {
  int col, grp;
  int lane;
  // Hidden from the compiler, which else forms every address part of every kind of item before the first
  // one and keeps them all (35 registers more than there are).
  __device__ __forceinline__ Lane() {
    lane = int(__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)));
    asm volatile("" : "+v"(lane));
    col = lane & 15;
    grp = lane >> 4;
  }
  // x of the lane with another bit of its number
  __device__ __forceinline__ float across(float x, int bit) const {
    return __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute((lane ^ bit) << 2, __builtin_bit_cast(int, x)));
  }
};

// Keys and values of a block of two pages as they come from memory: bf16
// operands, or fp8 codes with their scales.
template <int D, bool kFp8>
struct Keys;
template <int D, bool kFp8>
struct Values;
template <int D>
struct Keys<D, false> {
  u32x4 k[2][D / 32];
};
template <int D>
struct Values<D, false> {
  u32x4 v[D / 16];
};
template <int D>
struct Keys<D, true> {
  u32x4 k[2][D / 64];
  float scale[2];
};
template <int D>
struct Values<D, true> {
  u32x4 v[2][D / 64];
  float scale[2];
};

template <int D, bool kFp8>
struct Source {
  const char* k_pool;
  const char* v_pool;
  const_f32_ptr k_scale, v_scale;
  const_i32_ptr bt;
  int hkv, kvh, pe;
  int k_off, v_off;   // this lane's bytes inside a tile

  __device__ __forceinline__ Source(const SharedArgs& a, const Item& it, const Lane& l) {
    k_pool = reinterpret_cast<const char*>(a.k_pool);
    v_pool = reinterpret_cast<const char*>(a.v_pool);
    k_scale = (const_f32_ptr)a.k_scale;
    v_scale = (const_f32_ptr)a.v_scale;
    bt = as_constant(a.block_table) + size_t(it.source) * a.bt_stride;
    hkv = a.num_kv_heads;
    kvh = it.kvh;
    pe = it.pe;
    k_off = kFp8 ? (l.grp * kPage + l.col) * 16 : (l.grp * kPage + l.col) * 16;
    v_off = kFp8 ? (l.grp * kPage + l.col) * 16 : (l.col * kPage + 4 * l.grp) * 2;
  }
  __device__ __forceinline__ size_t tile(int page) const {
    return (size_t(page) * hkv + kvh) * size_t(kPage * D * (kFp8 ? 1 : 2));
  }
};

struct Pages {
  int p0, p1;
};
template <int D, bool kFp8>
__device__ __forceinline__ Pages pages_at(const Source<D, kFp8>& s, int pg) {
  Pages p;
  p.p0 = s.bt[pg];
  p.p1 = pg + 1 < s.pe ? s.bt[pg + 1] : p.p0;   // masked
  return p;
}

// No other wave reads these bytes.
template <class T>
__device__ __forceinline__ T load(const char* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const T*>(p));
}

template <int D, bool kFp8>
__device__ __forceinline__ void load_keys(const Source<D, kFp8>& s, Pages p, Keys<D, kFp8>& b) {
  const char* k0 = s.k_pool + s.tile(p.p0) + s.k_off;
  const char* k1 = s.k_pool + s.tile(p.p1) + s.k_off;
  constexpr int kN = kFp8 ? D / 64 : D / 32;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    b.k[0][i] = load<u32x4>(k0 + 1024 * i);
    b.k[1][i] = load<u32x4>(k1 + 1024 * i);
  }
  if constexpr (kFp8) {
    b.scale[0] = s.k_scale[size_t(p.p0) * s.hkv + s.kvh];
    b.scale[1] = s.k_scale[size_t(p.p1) * s.hkv + s.kvh];
  }
}

template <int D, bool kFp8>
__device__ __forceinline__ void load_values(const Source<D, kFp8>& s, Pages p, Values<D, kFp8>& b) {
  const char* v0 = s.v_pool + s.tile(p.p0) + s.v_off;
  const char* v1 = s.v_pool + s.tile(p.p1) + s.v_off;
  if constexpr (kFp8) {
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      b.v[0][i] = load<u32x4>(v0 + 1024 * i);
      b.v[1][i] = load<u32x4>(v1 + 1024 * i);
    }
    b.scale[0] = s.v_scale[size_t(p.p0) * s.hkv + s.kvh];
    b.scale[1] = s.v_scale[size_t(p.p1) * s.hkv + s.kvh];
  } else {
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      const u32x2 x = load<u32x2>(v0 + 512 * j);
      const u32x2 y = load<u32x2>(v1 + 512 * j);
      b.v[j] = u32x4{x[0], x[1], y[0], y[1]};
    }
  }
}

// K operand of page h for dims 32 kb ..; V^T operand for dims 16 jb .. (fp8: widened, exact).
template <int D, bool kFp8>
__device__ __forceinline__ u32x4 key_operand(const Keys<D, kFp8>& b, int h, int kb) {
  if constexpr (!kFp8) return b.k[h][kb];
  else {
    const u32x4 w = b.k[h][kb / 2];
    const uint32_t lo = w[2 * (kb % 2)], hi = w[2 * (kb % 2) + 1];
    return u32x4{widen2<false>(lo), widen2<true>(lo), widen2<false>(hi), widen2<true>(hi)};
  }
}
template <int D, bool kFp8>
__device__ __forceinline__ u32x4 value_operand(const Values<D, kFp8>& b, int jb) {
  if constexpr (!kFp8) return b.v[jb];
  else {
    const uint32_t p0 = b.v[0][jb / 4][jb % 4], p1 = b.v[1][jb / 4][jb % 4];
    return u32x4{widen2<false>(p0), widen2<true>(p0), widen2<false>(p1), widen2<true>(p1)};
  }
}

// Key of a block that a lane's weight e belongs to: 0 .. 3 are slots 4 grp + e
// of the first page, 4 .. 7 of the second.
__device__ __forceinline__ int key_at(int grp, int e) { return (e < 4 ? 0 : kPage - 4) + 4 * grp + e; }

// Slots past the end may hold anything, and a zero weight times NaN is NaN: their
// keys (token col of either page) and values (tokens 4 grp .. + 3) become zeros.
template <int D>
__device__ __forceinline__ void drop_past(Keys<D, false>& k, Values<D, false>& v, int valid, const Lane& l) {
  const u32x4 none = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    k.k[0][i] = l.col < valid ? k.k[0][i] : none;
    k.k[1][i] = kPage + l.col < valid ? k.k[1][i] : none;
  }
  u32x4 mask;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    mask[i] = (key_at(l.grp, 2 * i) < valid ? 0x0000FFFFu : 0u) | (key_at(l.grp, 2 * i + 1) < valid ? 0xFFFF0000u : 0u);
#pragma unroll
  for (int j = 0; j < D / 16; ++j) v.v[j] &= mask;
}
template <int D>
__device__ __forceinline__ void drop_past(Keys<D, true>& k, Values<D, true>& v, int valid, const Lane& l) {
  const u32x4 none = {0u, 0u, 0u, 0u};
  uint32_t mask[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int n = valid - h * kPage - 4 * l.grp;
    mask[h] = n >= 4 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
  }
#pragma unroll
  for (int i = 0; i < D / 64; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      k.k[h][i] = h * kPage + l.col < valid ? k.k[h][i] : none;
      v.v[h][i] &= mask[h];
    }
}

// A tile's weights of one block: the P^T operand as two bf16 parts.
struct Weights {
  u32x4 hi, lo;
};

template <int D>
struct Tile {
  f32x4 o[D / 16];   // O[row col][16 jb + 4 grp + i]
  float m;           // reference, log2 units
  float sum;         // this lane's share of the weights' sum
};

__device__ __forceinline__ float sum8(const float* p) {
  return ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
}

// c0, c1: factors of the two pages' scores in log2 units; v0, v1: value scales (fp8).
// A lane's sum of weights bounds each of them; until one passes the headroom (the first
// block's does: m is -inf) lanes of a row need not agree on its maximum, and nothing is exchanged. Only the rows
// that passed it move their reference: a row's bits are its own, whatever the other sequences' rows of its tile hold.
template <int D, bool kFp8>
__device__ __forceinline__ Weights weigh(Tile<D>& t, const f32x4& s0, const f32x4& s1, float c0, float c1, float v0, float v1,
                                         int valid, const Lane& l) {
  float z[8], p[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    z[e] = s0[e] * c0;
    z[4 + e] = s1[e] * c1;
  }
  if (valid < 2 * kPage) {
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = key_at(l.grp, e) < valid ? z[e] : -__builtin_inff();
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) p[e] = exp2_fast(z[e] - t.m);
  float part = sum8(p);
  float past = part <= kHeadroom ? 0.f : 1.f;
  if (__any(past != 0.f)) {
    past = fmaxf(past, l.across(past, 16));
    past = fmaxf(past, l.across(past, 32));
    const bool moves = past != 0.f;   // (every row without a reference so far does)
    float top = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
    top = fmaxf(top, l.across(top, 16));
    top = fmaxf(top, l.across(top, 32));
    const float m = moves ? fmaxf(t.m, top) : t.m;
    const float ref = m == -__builtin_inff() ? 0.f : m;   // no key with a finite score so far
    const float keep = moves ? exp2_fast(t.m - ref) : 1.f;
    t.m = m;
    t.sum *= keep;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) t.o[j] *= keep;
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = exp2_fast(z[e] - ref);
    part = sum8(p);
  }
  t.sum += part;
  Weights w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = p[2 * i], b = p[2 * i + 1];
    if constexpr (kFp8) {
      a *= i < 2 ? v0 : v1;
      b *= i < 2 ? v0 : v1;
    }
    const uint32_t hi = pack_bf16(a, b);
    w.hi[i] = hi;
    w.lo[i] = pack_bf16(a - low_bf16(hi), b - high_bf16(hi));
  }
  return w;
}

// A wave's rows: their queries as the B operand of S^T = K Q^T, and results so far.
template <int D, int kTiles>
struct Rows {
  u32x4 q[kTiles][D / 32];
  Tile<D> tile[kTiles];

  __device__ __forceinline__ void begin(const SharedArgs& a, const Item& it, const Lane& l) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int r = 16 * t + l.col;
      const bool ok = r < it.rows;
      const int row = it.within + (ok ? r : 0);   // below 16 + 32
      const int member = row * a.group_inverse >> 16, head = row - member * a.group;
      const uint16_t* src = a.q + (size_t(it.member + member) * a.num_q_heads + it.kvh * a.group + head) * D + 8 * l.grp;
#pragma unroll
      for (int kb = 0; kb < D / 32; ++kb) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(src + 32 * kb);
        q[t][kb] = ok ? x : u32x4{0u, 0u, 0u, 0u};
      }
#pragma unroll
      for (int j = 0; j < D / 16; ++j) tile[t].o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
      tile[t].m = -__builtin_inff();
      tile[t].sum = 0.f;
    }
  }

  __device__ __forceinline__ void finish(const SharedArgs& a, const Item& it, const Lane& l) const {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      float total = tile[t].sum + l.across(tile[t].sum, 16);
      total += l.across(total, 32);
      const float inv = total > 0.f ? 1.f / total : 0.f;
      const float lse = total > 0.f ? tile[t].m + __log2f(total) : -__builtin_inff();
      const int r = 16 * t + l.col;
      if (r >= it.rows) continue;
      if (it.slot >= 0) {
        float* dst = a.part_o + size_t(it.slot + r) * D + 4 * l.grp;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) *reinterpret_cast<f32x4*>(dst + 16 * j) = tile[t].o[j] * inv;
        if (l.grp == 0) a.part_lse[it.slot + r] = lse;
        continue;
      }
      // a sequence's only segment: its rows are the heads
      const size_t row = size_t(it.seq0) * a.num_q_heads + it.kvh * a.group + r;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) {
        const f32x4 o = tile[t].o[j] * inv;
        const size_t at = row * D + 16 * j + 4 * l.grp;
        if (a.out_bf16)
          *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + at) = u32x2{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
        else
          *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at) = o;
      }
      if (a.lse && l.grp == 0) a.lse[row] = lse * kLn2;
    }
  }
};

// O^T += V^T P^T over a block; value(j) is the operand of dims 16 j ... Products of one
// accumulator are kept apart, each would wait for the one before it.
template <int D, int kTiles, class Value>
__device__ __forceinline__ void accumulate(Rows<D, kTiles>& rows, const Weights* w, Value value) {
#pragma unroll
  for (int j = 0; j < D / 16; j += 2) {
    const u32x4 v0 = value(j), v1 = value(j + 1);
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      rows.tile[t].o[j] = mfma_bf16(v0, w[t].hi, rows.tile[t].o[j]);
      rows.tile[t].o[j + 1] = mfma_bf16(v1, w[t].hi, rows.tile[t].o[j + 1]);
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      rows.tile[t].o[j] = mfma_bf16(v0, w[t].lo, rows.tile[t].o[j]);
      rows.tile[t].o[j + 1] = mfma_bf16(v1, w[t].lo, rows.tile[t].o[j + 1]);
    }
  }
}

// One segment with kTiles tiles of rows that no other wave shares. kBufs blocks of
// registers: with one, a block's keys are requested once the scores of the block before
// it are formed and its values once those before it are used, so each waits behind half a
// block's work; with more, the block kBufs - 1 ahead is requested.
template <int D, int kTiles, bool kFp8>
__device__ __forceinline__ void walk(const SharedArgs& a, const Item& it) {
  constexpr int kBufs = kFp8 ? 3 : 1;
  constexpr int kAhead = kBufs == 1 ? 1 : kBufs - 1;   // blocks
  const Lane l;
  const Source<D, kFp8> src(a, it, l);
  Keys<D, kFp8> keys[kBufs];
  Values<D, kFp8> values[kBufs];
#pragma unroll
  for (int b = 0; b < kAhead; ++b) {
    if (it.pb + 2 * b >= it.pe) break;
    const Pages p = pages_at(src, it.pb + 2 * b);
    load_keys(src, p, keys[b]);
    load_values(src, p, values[b]);
  }
  Rows<D, kTiles> rows;
  rows.begin(a, it, l);

  // Block at pg from kc, vc; the one kAhead blocks on loads into kn, vn (kBufs = 1: the same).
  auto step = [&](int pg, Keys<D, kFp8>& kc, Values<D, kFp8>& vc, Keys<D, kFp8>& kn, Values<D, kFp8>& vn) {
    const bool more = pg + 2 * kAhead < it.pe;
    Pages next = {0, 0};
    if (more) {
      next = pages_at(src, pg + 2 * kAhead);
      if constexpr (kBufs > 1) load_keys(src, next, kn);
    }
    const int valid = min(it.end - pg * kPage, pg + 1 < it.pe ? 2 * kPage : kPage);
    if (valid < 2 * kPage) drop_past(kc, vc, valid, l);   // a segment's last block
    f32x4 s0[kTiles], s1[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) s0[t] = s1[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < D / 32; ++kb) {
      const u32x4 k0 = key_operand(kc, 0, kb), k1 = key_operand(kc, 1, kb);
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        s0[t] = mfma_bf16(k0, rows.q[t][kb], s0[t]);
        s1[t] = mfma_bf16(k1, rows.q[t][kb], s1[t]);
      }
    }
    float c0 = a.scale_log2, c1 = a.scale_log2, v0 = 1.f, v1 = 1.f;
    if constexpr (kFp8) {
      c0 *= kc.scale[0];
      c1 *= kc.scale[1];
      v0 = vc.scale[0];
      v1 = vc.scale[1];
    }
    if constexpr (kBufs == 1) {
      __builtin_amdgcn_sched_barrier(0);   // into the same registers: not ahead of their last use
      if (more) load_keys(src, next, kn);
    } else if (more) {
      load_values(src, next, vn);
    }
    Weights w[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) w[t] = weigh<D, kFp8>(rows.tile[t], s0[t], s1[t], c0, c1, v0, v1, valid, l);
    accumulate(rows, w, [&](int j) { return value_operand(vc, j); });
    if constexpr (kBufs == 1) {
      __builtin_amdgcn_sched_barrier(0);
      if (more) load_values(src, next, vn);
    }
  };
  for (int pg = it.pb; pg < it.pe; pg += 2 * kBufs) {
#pragma unroll
    for (int b = 0; b < kBufs; ++b) {
      if (pg + 2 * b >= it.pe) break;
      step(pg + 2 * b, keys[b], values[b], keys[(b + kAhead) % kBufs], values[(b + kAhead) % kBufs]);
    }
  }
  rows.finish(a, it, l);
}

// A prompt's segment, by all eight waves of a workgroup: 8 / kSplits of them hold its
// rows (32 each), and the kSplits sets of them go through its key blocks in turns. The keys
// and values of a step (kSplits blocks) are read from memory once, into registers four
// blocks ahead, and pass through LDS (fp8: widened on the way), two steps of it in turns, one barrier a
// step. V in LDS: dim d owns 64 bytes, four 16-byte slots, and slot g ^ swizzle(d) holds tokens 4g .. 4g + 3
// of both pages: the P.V operand of a lane is one read, and 8 lanes of it meet 8 banks' groups.
template <int D>
struct Stage {
  static constexpr int kTile = kPage * D;         // elements of a page's K or V
  static constexpr int kBlock = 4 * kTile;        // K of two pages, then V of both
  static constexpr int kRing = 8 * kBlock;        // two steps of at most four blocks
};
__device__ __forceinline__ int v_swizzle(int d) { return (d >> 1) & 3; }

template <int D, bool kFp8, int kSplits>
__device__ __forceinline__ void walk_together(const SharedArgs& a, const Item& it, int wave, uint16_t* lds, f32x4* lds_scale) {
  constexpr int kTiles = kSharedTiles;
  constexpr int kAhead = 4 / kSplits;               // steps in registers
  constexpr int kTile = Stage<D>::kTile;
  constexpr int kChunks = kTile * (kFp8 ? 1 : 2) / 1024;   // of 1 KiB in a page's K or V
  constexpr int kMine = kChunks > 1 ? kChunks / 2 : 1;     // of a wave
  const Lane l;
  const int lane = l.lane;
  const Source<D, kFp8> src(a, it, l);
  const int blocks = (it.pe - it.pb + 1) / 2, steps = (blocks + kSplits - 1) / kSplits;

  // Staging: waves 2t and 2t + 1 move tile t of a block (K of its first page, of its second, V of both).
  // Loads are issued whether a step exists or not (the last one's again): the waits count them.
  const int part = wave >> 1, chunk0 = min((wave & 1) * kMine, kChunks - kMine);
  const bool stager = (wave & 1) * kMine < kChunks;
  const char* const pool = part < 2 ? src.k_pool : src.v_pool;
  const const_f32_ptr pool_scale = part < 2 ? src.k_scale : src.v_scale;
  struct Staged {
    u32x4 x[kSplits][kMine];
    float scale[kSplits];
  };
  Staged held[kAhead];
  int page[kSplits];   // of the step to be fetched next
  auto find = [&](int step) {
#pragma unroll
    for (int b = 0; b < kSplits; ++b) {
      const int pg = it.pb + 2 * min(step * kSplits + b, blocks - 1);
      page[b] = src.bt[min(pg + (part & 1), it.pe - 1)];
    }
  };
  auto fetch = [&](Staged& s, int step) {
#pragma unroll
    for (int b = 0; b < kSplits; ++b) {
      const char* p = pool + src.tile(page[b]) + (chunk0 * 64 + lane) * 16;
#pragma unroll
      for (int c = 0; c < kMine; ++c) s.x[b][c] = *reinterpret_cast<const u32x4*>(p + 1024 * c);
      if constexpr (kFp8) s.scale[b] = pool_scale[size_t(page[b]) * src.hkv + src.kvh];
    }
    find(step + 1);
  };
  auto put = [&](const Staged& s, int step) {
    if (!stager) return;
    // (a ring of 128 KiB is more than an address reaches: the parts' addresses are formed anew rather than all kept)
    int lane = l.lane;
    if constexpr (kSplits == 4) asm volatile("" : "+v"(lane));
#pragma unroll
    for (int b = 0; b < kSplits; ++b) {
      const int slot = (step & 1) * kSplits + b;
      uint16_t* const L = lds + slot * Stage<D>::kBlock;
      if constexpr (kFp8) {
        if (lane == 0 && !(wave & 1)) reinterpret_cast<float*>(lds_scale + slot)[part] = s.scale[b];
      }
#pragma unroll
      for (int c = 0; c < kMine; ++c) {
        const u32x4 x = s.x[b][c];
        const int chunk = chunk0 + c;
        if constexpr (kFp8) {
          if (part < 2) {   // dims 64 chunk + 8 grp .. + 7 of token col, and those 32 further
            uint16_t* dst = L + part * kTile + ((8 * chunk + l.grp) * kPage + l.col) * 8;
            *reinterpret_cast<u32x4*>(dst) = u32x4{widen2<false>(x[0]), widen2<true>(x[0]), widen2<false>(x[1]), widen2<true>(x[1])};
            *reinterpret_cast<u32x4*>(dst + 4 * kPage * 8) =
                u32x4{widen2<false>(x[2]), widen2<true>(x[2]), widen2<false>(x[3]), widen2<true>(x[3])};
          } else {          // tokens 4 grp .. + 3 of dims 64 chunk + 16 j + col
            const int d = 64 * chunk + l.col;
            uint16_t* dst = L + 2 * kTile + d * 32 + (l.grp ^ v_swizzle(d)) * 8 + (part - 2) * 4;
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<u32x2*>(dst + j * 16 * 32) = u32x2{widen2<false>(x[j]), widen2<true>(x[j])};
          }
        } else if (part < 2) {
          *reinterpret_cast<u32x4*>(L + part * kTile + (chunk * 64 + lane) * 8) = x;
        } else {            // tokens 8 h .. + 7 of dim d
          const int d = chunk * 32 + (lane >> 1), h = lane & 1;
          uint16_t* row = L + 2 * kTile + d * 32 + (part - 2) * 4;
          *reinterpret_cast<u32x2*>(row + ((2 * h) ^ v_swizzle(d)) * 8) = u32x2{x[0], x[1]};
          *reinterpret_cast<u32x2*>(row + ((2 * h + 1) ^ v_swizzle(d)) * 8) = u32x2{x[2], x[3]};
        }
      }
    }
  };

  Rows<D, kTiles> rows;
  auto compute = [&](int step) {
    const int block = step * kSplits + it.split;
    if (block >= blocks) return;
    const int slot = (step & 1) * kSplits + it.split;
    const uint16_t* const L = lds + slot * Stage<D>::kBlock;
    float c0 = a.scale_log2, c1 = a.scale_log2, v0 = 1.f, v1 = 1.f;
    if constexpr (kFp8) {
      const f32x4 sc = lds_scale[slot];
      c0 *= sc[0];
      c1 *= sc[1];
      v0 = sc[2];
      v1 = sc[3];
    }
    const int valid = it.pb + 2 * block + 1 < it.pe ? 2 * kPage : kPage;
    f32x4 s0[kTiles], s1[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) s0[t] = s1[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < D / 32; ++kb) {
      const int at = ((4 * kb + l.grp) * kPage + l.col) * 8;
      const u32x4 k0 = *reinterpret_cast<const u32x4*>(L + at);
      const u32x4 k1 = *reinterpret_cast<const u32x4*>(L + kTile + at);
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        s0[t] = mfma_bf16(k0, rows.q[t][kb], s0[t]);
        s1[t] = mfma_bf16(k1, rows.q[t][kb], s1[t]);
      }
    }
    Weights w[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) w[t] = weigh<D, kFp8>(rows.tile[t], s0[t], s1[t], c0, c1, v0, v1, valid, l);
    const int vat = 2 * kTile + l.col * 32 + (l.grp ^ v_swizzle(l.col)) * 8;
    accumulate(rows, w, [&](int j) { return *reinterpret_cast<const u32x4*>(L + vat + j * 16 * 32); });
  };

  find(0);
#pragma unroll
  for (int j = 0; j < kAhead; ++j) fetch(held[j], j);
  rows.begin(a, it, l);
  put(held[0], 0);
  fetch(held[0], kAhead);
  __syncthreads();
  constexpr int kUnroll = kAhead > 2 ? kAhead : 2;
  for (int i = 0; i < steps; i += kUnroll) {
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      if (i + j >= steps) break;
      put(held[(j + 1) % kAhead], i + j + 1);
      fetch(held[(j + 1) % kAhead], i + j + 1 + kAhead);
      compute(i + j);
      __syncthreads();
    }
  }
  rows.finish(a, it, l);
}

__device__ __forceinline__ Item item_at(const_i32_ptr row) {
  return {row[2], row[3], row[4], row[5], row[6], row[7], row[8], row[9], row[10], row[11], row[12], row[13], row[14]};
}

template <int D, bool kFp8, int kWG>
__global__ __launch_bounds__(64 * kWG) __attribute__((amdgpu_waves_per_eu(2, 2))) void shared_attn_kernel(SharedArgs a) {
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int worker = int(blockIdx.x) * kWG + wave;
  // the side job: merge rows to the device
  for (int64_t i = int64_t(blockIdx.x) * (64 * kWG) + int(threadIdx.x); i < a.copy_ints; i += int64_t(gridDim.x) * (64 * kWG))
    a.copy_dst[i] = a.copy_src[i];
  if (worker >= a.num_workers) return;
  const const_i32_ptr head = as_constant(a.workers) + size_t(worker) * kSharedInts;
  const int first = head[0], count = head[1];
  for (int i = 0; i < count; ++i) {
    const Item it = item_at(i == 0 ? head : as_constant(a.items) + size_t(first + i) * kSharedInts);
    if constexpr (kWG == kSharedWaves) {
      // the same for all waves of the workgroup, as many items and steps
      if (it.blocks) {
        __shared__ __attribute__((aligned(16))) uint16_t lds[Stage<D>::kRing];
        __shared__ f32x4 lds_scale[8];
        if (it.blocks == 8) walk_together<D, kFp8, 1>(a, it, wave, lds, lds_scale);
        else if (it.blocks == 4) walk_together<D, kFp8, 2>(a, it, wave, lds, lds_scale);
        else walk_together<D, kFp8, 4>(a, it, wave, lds, lds_scale);
        continue;
      }
    }
    walk<D, 1, kFp8>(a, it);
  }
}

// One workgroup per (sequence, KV head): its parts and those of its prompt.
__global__ __launch_bounds__(256) void shared_merge_kernel(SharedArgs a) {
  const const_i32_ptr row = as_constant(a.merge_rows) + size_t(blockIdx.x) * kSharedMergeInts;
  const int seq = row[0], kvh = row[1], own = row[2], own_parts = row[3], pre = row[4], pre_parts = row[5], stride = row[6];
  const int g = a.group, d4n = a.head_dim / 4;
  for (int i = int(threadIdx.x); i < g * d4n; i += int(blockDim.x)) {
    const int h = i / d4n, d4 = i - h * d4n;
    float top = -__builtin_inff(), sum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](size_t at) {
      const float lse = a.part_lse[at];
      const f32x4 o = *reinterpret_cast<const f32x4*>(a.part_o + at * a.head_dim + 4 * d4);
      const float m = fmaxf(top, lse);
      const float ref = m == -__builtin_inff() ? 0.f : m;
      const float keep = exp2_fast(top - ref), w = exp2_fast(lse - ref);
      acc = acc * keep + o * w;
      sum = sum * keep + w;
      top = m;
    };
#pragma unroll 4
    for (int c = 0; c < pre_parts; ++c) add(size_t(pre) + size_t(c) * stride + h);
#pragma unroll 4
    for (int c = 0; c < own_parts; ++c) add(size_t(own) + size_t(c) * g + h);
    const f32x4 o = acc * (sum > 0.f ? 1.f / sum : 0.f);
    const size_t r = size_t(seq) * a.num_q_heads + kvh * g + h;
    if (a.out_bf16)
      *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + r * a.head_dim + 4 * d4) =
          u32x2{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
    else
      *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + r * a.head_dim + 4 * d4) = o;
    if (a.lse && d4 == 0) a.lse[r] = sum > 0.f ? (top + __log2f(sum)) * kLn2 : -__builtin_inff();
  }
}

template <int D, bool kFp8>
void launch_walks(const SharedArgs& a, hipStream_t stream) {
  if (a.workers_per_group == kSharedWaves)
    hipLaunchKernelGGL((shared_attn_kernel<D, kFp8, kSharedWaves>), dim3((a.num_workers + kSharedWaves - 1) / kSharedWaves),
                       dim3(64 * kSharedWaves), 0, stream, a);
  else
    hipLaunchKernelGGL((shared_attn_kernel<D, kFp8, 1>), dim3(a.num_workers), dim3(64), 0, stream, a);
}

}  // namespace

hipError_t launch_shared(const SharedArgs& a, hipStream_t stream) {
  if (a.num_workers > 0) {
    if (a.head_dim == 128) a.k_scale ? launch_walks<128, true>(a, stream) : launch_walks<128, false>(a, stream);
    else a.k_scale ? launch_walks<64, true>(a, stream) : launch_walks<64, false>(a, stream);
  }
  if (a.num_merge > 0) hipLaunchKernelGGL(shared_merge_kernel, dim3(a.num_merge), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sf
