// Sampling with temperature, top-k, top-p and min-p from given uniform numbers.
//
// Each row asks which index a running sum crosses a share of the whole at, and
// the answer must not depend on the order of the sums: weights are rounded to
// multiples of 2^-44 of the largest (fp64 arithmetic, whose fma runs at the rate of an unpacked fp32 one
// here) and added as integers, by atomics too.
//
// The first launch reads the logits once, a chunk per workgroup: the chunk's largest
// logit, the sum of its weights relative to it and, where there are cuts, the largest
// logit of every 64. The second, a workgroup per row, joins the chunks' sums. Without cuts it
// then knows the chunk of the drawn index, and reads that again.
//
// With cuts, the kept entries are the first ones in the order of falling logits, and
// the groups' largest logits bound where that order can end (Bound below): if
// no more than 4096 entries lie above the bound, only their groups are read again, the
// entries are sorted in LDS and every cut is a position there. A row left open by
// that takes one of two ways. A top-p of everything, a min-p too, is found by all of the row's chunks at once, in two
// launches: sums by 2048 equal steps of the logit, then the entries of the step in which the share is
// reached, which a third one sorts. The rest (a top-k of thousands) is read whole by the third's workgroup.
// Rows that are done cost those launches a workgroup each that ends at once.
//
// Measured: 256 rows of 131072 bf16 without cuts 34 + 11 us, where reading them takes 15: an entry
// costs the first launch some thirty vector instructions (13 of them fp64), which is 25 us of that
// work alone. 192 rows of 200003 fp32 with mixed cuts (33 us to read): 47 + 62 + 19 + 22 + 23, the second bound by its
// slowest workgroup (thousands of entries near a cut, read again and sorted). The step forms of the
// flat rows by one workgroup each instead took 460 us, sorting networks for the lists 120 more.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "sf_internal.h"

namespace sf {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kChunkThreads = 256;
constexpr int kDrawThreads = 256;
constexpr int kCutThreads = 512;   // two waves per SIMD
constexpr int kRowThreads = 512;
constexpr int kBins = kSampleBins;
constexpr int kBinBits = 11;
static_assert(kBins == 1 << kBinBits, "bins");
constexpr int kUnitBits = 44;
constexpr double kUnit = 0x1p-44;
constexpr int kList = kSampleList;   // entries that are sorted
constexpr int kGroup = kSampleGroup;
constexpr float kNone = -__builtin_inff();

enum Type { kF32 = 0, kBF16 = 1, kF16 = 2 };

template <int kType>
struct Elem {
  static constexpr int kBytes = kType == kF32 ? 4 : 2;
  static constexpr int kPer = 16 / kBytes;   // logits of a 16-byte piece
};

// A NaN counts as no entry.
__device__ __forceinline__ float clean(float x) { return fmaxf(x, kNone); }

// (A bit cast of a vector's element itself takes the vector's first.)
__device__ __forceinline__ float value32(uint32_t bits) { return __builtin_bit_cast(float, bits); }
template <int kType>
__device__ __forceinline__ float value16(uint32_t bits) {
  if constexpr (kType == kBF16) return __builtin_bit_cast(float, bits << 16);
  return float(__builtin_bit_cast(_Float16, uint16_t(bits)));
}

template <int kType>
__device__ __forceinline__ void values(u32x4 w, float* x) {
#pragma unroll
  for (int i = 0; i < Elem<kType>::kPer; ++i) {
    if constexpr (kType == kF32)
      x[i] = clean(value32(w[i]));
    else
      x[i] = clean(value16<kType>(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xFFFFu));
  }
}

// Some pieces of a row: all loads first, so that they are in flight together.
template <int kCount, class Row, class At>
__device__ __forceinline__ void load_all(const Row& r, float (&x)[kCount][Row::kPer], At at) {
  u32x4 w[kCount];
#pragma unroll
  for (int j = 0; j < kCount; ++j) w[j] = r.raw(at(j));
#pragma unroll
  for (int j = 0; j < kCount; ++j) values<Row::kElem>(w[j], x[j]);
}

// A row of logits as 16-byte pieces at 16-byte addresses: piece p holds
// entries p * kPer - lead .. + kPer - 1, of which the first and the last pieces
// may lack some.
template <int kType>
struct Row {
  static constexpr int kElem = kType, kPer = Elem<kType>::kPer;
  const char* base;
  int lead;
  int vocab;
  int pieces;

  __device__ __forceinline__ Row(const SampleArgs& a, int row) {
    constexpr int kPer = Elem<kType>::kPer, kBytes = Elem<kType>::kBytes;
    const char* at = static_cast<const char*>(a.logits) + int64_t(row) * a.row_stride * kBytes;
    const int off = int(reinterpret_cast<uintptr_t>(at) & 15);
    base = at - off;
    lead = off / kBytes;
    vocab = a.vocab;
    pieces = (vocab + lead + kPer - 1) / kPer;
  }
  __device__ __forceinline__ int first(int p) const { return p * Elem<kType>::kPer - lead; }
  // A piece as it lies in memory; entries that it lacks, or past the last piece, are -inf.
  __device__ __forceinline__ u32x4 raw(int p) const {
    constexpr int kPer = Elem<kType>::kPer, kBytes = Elem<kType>::kBytes;
    constexpr uint32_t kLeast = kType == kF32 ? 0xFF800000u : kType == kBF16 ? 0xFF80FF80u : 0xFC00FC00u;
    const int lo = first(p);
    u32x4 w = {kLeast, kLeast, kLeast, kLeast};
    if (lo >= 0 && lo + kPer <= vocab) {
      w = *reinterpret_cast<const u32x4*>(base + int64_t(p) * 16);
    } else if (p < pieces) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (lo + i >= 0 && lo + i < vocab) {
          const char* at = base + int64_t(p) * 16 + i * kBytes;
          if constexpr (kType == kF32)
            w[i] = *reinterpret_cast<const uint32_t*>(at);
          else
            w[i / 2] = i & 1 ? (w[i / 2] & 0xFFFFu) | uint32_t(*reinterpret_cast<const uint16_t*>(at)) << 16
                             : (w[i / 2] & 0xFFFF0000u) | *reinterpret_cast<const uint16_t*>(at);
        }
    }
    return w;
  }
  __device__ __forceinline__ void load(int p, float* x) const { values<kType>(raw(p), x); }
};

// 2^(i / 32), i < 32, in LDS: 64 lanes read it without a conflict.
struct Powers {
  double at[32];
};
__constant__ const double kPowers[32] = {
    0x1.0000000000000p+0, 0x1.059b0d3158574p+0, 0x1.0b5586cf9890fp+0, 0x1.11301d0125b51p+0,
    0x1.172b83c7d517bp+0, 0x1.1d4873168b9aap+0, 0x1.2387a6e756238p+0, 0x1.29e9df51fdee1p+0,
    0x1.306fe0a31b715p+0, 0x1.371a7373aa9cbp+0, 0x1.3dea64c123422p+0, 0x1.44e086061892dp+0,
    0x1.4bfdad5362a27p+0, 0x1.5342b569d4f82p+0, 0x1.5ab07dd485429p+0, 0x1.6247eb03a5585p+0,
    0x1.6a09e667f3bcdp+0, 0x1.71f75e8ec5f74p+0, 0x1.7a11473eb0187p+0, 0x1.82589994cce13p+0,
    0x1.8ace5422aa0dbp+0, 0x1.93737b0cdc5e5p+0, 0x1.9c49182a3f090p+0, 0x1.a5503b23e255dp+0,
    0x1.ae89f995ad3adp+0, 0x1.b7f76f2fb5e47p+0, 0x1.c199bdd85529cp+0, 0x1.cb720dcef9069p+0,
    0x1.d5818dcfba487p+0, 0x1.dfc97337b9b5fp+0, 0x1.ea4afa2a490dap+0, 0x1.f50765b6e4540p+0,
};
__device__ __forceinline__ void make_powers(Powers& t) {
  if (threadIdx.x < 32) t.at[threadIdx.x] = kPowers[threadIdx.x];
}

// 2^(y + shift), -1000 < y + shift: the nearest multiple of 1/32 comes off by adding
// 1.5 2^47, its whole part goes back as an addition to the exponent, and what is left,
// within 1/64, enters the Taylor series to f^5 (the next term is below 2^-48).
__device__ __forceinline__ double exp2_of(const Powers& t, double y, int shift) {
  const double m = y + 0x1.8p47;
  const int n = int(uint32_t(__builtin_bit_cast(uint64_t, m)));
  const double f = y - (m - 0x1.8p47);
  double p = 0.00133335581464284434;
  p = __builtin_fma(p, f, 0.00961812910762847716);
  p = __builtin_fma(p, f, 0.05550410866482157995);
  p = __builtin_fma(p, f, 0.24022650695910071233);
  p = __builtin_fma(p, f, 0.69314718055994530942);
  p = __builtin_fma(p, f, 1.0) * t.at[n & 31];
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  u32x2 bits = __builtin_bit_cast(u32x2, p);
  bits.y += (uint32_t(n) << 15 & 0xFFF00000u) + (uint32_t(shift) << 20);
  return __builtin_bit_cast(double, bits);
}

// Weights of logits relative to a largest one: exp((l - top) / T), 1 / (T ln 2) in rate.
struct Scale {
  const Powers& powers;
  float top;
  double rate;
  __device__ __forceinline__ Scale(const Powers& t, float largest, double r) : powers(t), top(largest), rate(r) {}
  __device__ __forceinline__ double exponent(float l) const { return (double(l) - double(top)) * rate; }
  // In units of 2^-44, rounded, with the bits of 2^52 above them. (max takes its other operand for the NaN of -inf * 0.)
  __device__ __forceinline__ uint64_t raw_units(float l) const {
    return __builtin_bit_cast(uint64_t, exp2_of(powers, fmax(exponent(l), -62.0), kUnitBits) + 0x1p52);   // the sum's last bit is one unit
  }
  static constexpr uint64_t kRaw = 0x4330000000000000ull;
  __device__ __forceinline__ uint64_t units(float l) const {
    if (top == __builtin_inff()) return l == top ? uint64_t(1) << kUnitBits : 0;
    return raw_units(l) - kRaw;
  }
  __device__ __forceinline__ double weight(float l) const {
    if (top == __builtin_inff()) return l == top ? 1.0 : 0.0;
    if (l == kNone) return 0.0;
    const double y = exponent(l);
    return y > -1000.0 ? exp2_of(powers, y, 0) : 0.0;
  }
};

__device__ __forceinline__ bool greedy(float t) { return !(t > 0.f); }
__device__ __forceinline__ float temperature_of(const SampleArgs& a, int row) { return a.temperature ? a.temperature[row] : 1.f; }
__device__ __forceinline__ double rate_of(float t) { return 1.44269504088896340736 / (greedy(t) ? 1.0 : double(t)); }

// Rising keys for rising logits, above 0 for every finite one and +inf; -0 is 0 (equal logits have equal keys).
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
  return x == kNone ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
  return value32(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}

__device__ __forceinline__ uint64_t join(uint32_t lo, uint32_t hi) { return uint64_t(lo) | uint64_t(hi) << 32; }
__device__ __forceinline__ uint64_t shuffle_xor(uint64_t x, int m) {
  return join(uint32_t(__shfl_xor(int(uint32_t(x)), m)), uint32_t(__shfl_xor(int(uint32_t(x >> 32)), m)));
}
__device__ __forceinline__ uint64_t shuffle_up(uint64_t x, int n) {
  return join(uint32_t(__shfl_up(int(uint32_t(x)), n)), uint32_t(__shfl_up(int(uint32_t(x >> 32)), n)));
}
__device__ __forceinline__ uint64_t shuffle(uint64_t x, int lane) {
  return join(uint32_t(__shfl(int(uint32_t(x)), lane)), uint32_t(__shfl(int(uint32_t(x >> 32)), lane)));
}
__device__ __forceinline__ uint64_t wave_sum(uint64_t x) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) x += shuffle_xor(x, m);
  return x;
}
__device__ __forceinline__ uint32_t wave_sum(uint32_t x) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) x += uint32_t(__shfl_xor(int(x), m));
  return x;
}
// Inclusive sums over the wave's lanes.
__device__ __forceinline__ uint64_t wave_scan(uint64_t x) {
  const int lane = int(threadIdx.x) & 63;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const uint64_t y = shuffle_up(x, m);
    x += lane >= m ? y : 0;
  }
  return x;
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  const int lane = int(threadIdx.x) & 63;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const uint32_t y = uint32_t(__shfl_up(int(x), m));
    x += lane >= m ? y : 0;
  }
  return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) x = fmaxf(x, __shfl_xor(x, m));
  return x;
}

// Maximum over each kLanes (8 or 16) neighbouring lanes, in all of them.
template <int kLanes>
__device__ __forceinline__ float neighbours_max(float x) {
  auto across = [](float v, auto control) {
    return value32(uint32_t(__builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(control)::value, 0xF, 0xF, true)));
  };
  x = fmaxf(x, across(x, std::integral_constant<int, 0xB1>{}));    // lanes 1 0 3 2
  x = fmaxf(x, across(x, std::integral_constant<int, 0x4E>{}));    // lanes 2 3 0 1
  x = fmaxf(x, across(x, std::integral_constant<int, 0x141>{}));   // eight lanes mirrored
  if constexpr (kLanes == 16) x = fmaxf(x, across(x, std::integral_constant<int, 0x140>{}));   // sixteen
  return x;
}

template <int kType, int kChunk, bool kGroups>
__global__ __launch_bounds__(kChunkThreads) void sample_chunk_kernel(SampleArgs a) {
  constexpr int kPer = Elem<kType>::kPer;
  constexpr int kPieces = kChunk / kPer / kChunkThreads;   // of a thread
  constexpr int kWaves = kChunkThreads / 64;
  constexpr int kLanes = kGroup / kPer;                    // whose pieces are a group
  __shared__ float tops[kWaves];
  __shared__ int ats[kWaves];
  __shared__ uint64_t sums[kWaves];
  __shared__ Powers powers;
  const int row = int(blockIdx.x) / a.num_chunks, chunk = int(blockIdx.x) % a.num_chunks;
  const Row<kType> r(a, row);
  const int tid = int(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const int p0 = chunk * (kChunk / kPer) + tid;
  float x[kPieces][kPer];
  load_all(r, x, [&](int j) { return p0 + j * kChunkThreads; });
  make_powers(powers);
  if constexpr (kGroups) {
    if (blockIdx.x == 0 && tid == 0) *a.taken = 0;
  }
  float top = kNone;
#pragma unroll
  for (int j = 0; j < kPieces; ++j) {
    float most = x[j][0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) most = fmaxf(most, x[j][i]);
    top = fmaxf(top, most);
    if constexpr (kGroups) {
      most = neighbours_max<kLanes>(most);
      if (tid % kLanes == 0) a.groups[size_t(blockIdx.x) * (kChunk / kGroup) + (j * kChunkThreads + tid) / kLanes] = most;
    }
  }
  top = wave_max(top);
  if (lane == 0) tops[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, tops[w]);
  const float t = temperature_of(a, row);
  const Scale s(powers, top, rate_of(t));
  uint64_t sum = 0;
  if (top == __builtin_inff()) {
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
#pragma unroll
      for (int i = 0; i < kPer; ++i) sum += s.units(x[j][i]);
  } else if (top != kNone) {
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
#pragma unroll
      for (int i = 0; i < kPer; ++i) sum += s.raw_units(x[j][i]);
    sum -= uint64_t(kPieces * kPer) * Scale::kRaw;   // modulo 2^64
  }
  sum = wave_sum(sum);
  int at = INT32_MAX;
  if (greedy(t)) {
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (x[j][i] == top && top != kNone) at = min(at, r.first(p0 + j * kChunkThreads) + i);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) at = min(at, __shfl_xor(at, m));
  }
  if (lane == 0) {
    sums[wave] = sum;
    ats[wave] = at;
  }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kWaves; ++w) {
      sum += sums[w];
      at = min(at, ats[w]);
    }
    a.chunks[blockIdx.x] = SampleChunk{top, at, sum};
  }
}

// What a row's chunks say together, in a wave's lanes: chunk 64 i + lane is
// element i of each array.
constexpr int kMaxChunks = SF_SAMPLE_MAX_VOCAB / kSampleSmallChunk + 1;
constexpr int kPerLane = (kMaxChunks + 63) / 64;
struct Whole {
  float top;
  double total;                // of the weights relative to top, in units
  double before[kPerLane];     // of the chunks before it
  double part[kPerLane];       // its own
};
__device__ __forceinline__ Whole join_chunks(const SampleArgs& a, int row, double rate, const Powers& powers) {
  const SampleChunk* chunks = a.chunks + int64_t(row) * a.num_chunks;
  const int lane = int(threadIdx.x) & 63;
  SampleChunk c[kPerLane];
  Whole w;
  w.top = kNone;
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    c[i] = 64 * i + lane < a.num_chunks ? chunks[64 * i + lane] : SampleChunk{kNone, INT32_MAX, 0};
    w.top = fmaxf(w.top, c[i].top);
  }
  w.top = wave_max(w.top);
  const Scale s(powers, w.top, rate);
  w.total = 0.0;
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    w.before[i] = w.part[i] = 0.0;
    if (64 * i >= a.num_chunks) continue;
    w.part[i] = c[i].top == kNone ? 0.0 : double(c[i].sum) * s.weight(c[i].top);
    double scan = w.part[i];
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      const double y = __shfl_up(scan, m);
      scan += lane >= m ? y : 0.0;
    }
    w.before[i] = w.total + scan - w.part[i];
    w.total += __shfl(scan, 63);
  }
  return w;
}

// A row's results: a token's logit and what stays of the weights.
__device__ __forceinline__ void finish(const SampleArgs& a, int row, float top, double total, int token, float l, double kept) {
  const float t = temperature_of(a, row);
  a.token[row] = token;
  const double y = top == __builtin_inff() ? 0.0 : (double(l) - double(top)) / (greedy(t) ? 1.0 : double(t));
  if (a.logprob) a.logprob[row] = token < 0 ? kNone : float(y - log(total * kUnit));
  if (a.kept) a.kept[row] = token < 0 ? 0.f : float(kept / total);
}

__device__ __forceinline__ double uniform_of(const SampleArgs& a, int row) {
  const float u = a.uniform[row];
  return u > 0.f ? fmin(double(u), 1.0 - 0x1p-24) : 0.0;
}

// Rows that need no threshold: the largest logit (T = 0), or a draw from all
// entries. True if the row was one (by all of the workgroup's threads alike).
struct Drawn {
  int chunk;
  float top, chunk_top;
  double total, want;
  uint64_t waves[kRowThreads / 64];
  Powers powers;
};
template <int kType, int kThreads>
__device__ __forceinline__ void draw_row(const SampleArgs& a, int row, Drawn& sh) {
  constexpr int kPer = Elem<kType>::kPer;
  const int tid = int(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const Row<kType> r(a, row);
  const float t = temperature_of(a, row);
  const double rate = rate_of(t);
  const SampleChunk* chunks = a.chunks + int64_t(row) * a.num_chunks;
  make_powers(sh.powers);
  __syncthreads();
  if (wave == 0) {
    const Whole w = join_chunks(a, row, rate, sh.powers);
    int chunk = -1;
    if (w.top == kNone) {
      if (lane == 0) finish(a, row, w.top, 1.0, -1, 0.f, 0.0);
    } else if (greedy(t)) {
      int at = INT32_MAX;
      for (int c = lane; c < a.num_chunks; c += 64)
        if (chunks[c].top == w.top) at = min(at, chunks[c].at);
#pragma unroll
      for (int m = 1; m < 64; m *= 2) at = min(at, __shfl_xor(at, m));
      if (lane == 0) finish(a, row, w.top, w.total, at, w.top, 0x1p44);
    } else {
      // the last chunk before which no more than the draw's share lies
      const double target = uniform_of(a, row) * w.total;
      double before = 0.0;
#pragma unroll
      for (int i = 0; i < kPerLane; ++i)
        if (w.part[i] > 0.0 && w.before[i] <= target) {
          chunk = 64 * i + lane;
          before = w.before[i];
        }
      int last = chunk;
#pragma unroll
      for (int m = 1; m < 64; m *= 2) last = max(last, __shfl_xor(last, m));
      if (chunk == last) {
        const SampleChunk c = chunks[chunk];
        const Scale s(sh.powers, w.top, rate);
        sh.top = w.top;
        sh.chunk_top = c.top;
        sh.total = w.total;
        // (below the sum as a double holds it, which is some thread's end: c.sum - 1 is c.sum again beyond 2^53)
        const double sum = double(c.sum), below = __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, sum) - 1);
        sh.want = fmin((target - before) / s.weight(c.top), below);
      }
      chunk = last;
    }
    if (lane == 0) sh.chunk = chunk;
  }
  __syncthreads();
  const int chunk = sh.chunk;
  if (chunk < 0) return;
  const Scale cs(sh.powers, sh.chunk_top, rate);
  const double want = sh.want;
  // thread by thread in index order
  constexpr int kRun = kSampleChunk / kPer / kThreads;
  const int n = a.chunk / kPer, run = (n + kThreads - 1) / kThreads;
  uint64_t sum = 0;
  float x[kRun][kPer];
  load_all(r, x, [&](int j) { return j < run && tid * run + j < n ? chunk * n + tid * run + j : r.pieces; });   // (nothing behind the last)
  uint64_t part[kRun];   // a piece's
#pragma unroll
  for (int j = 0; j < kRun; ++j) {
    part[j] = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) part[j] += cs.units(x[j][i]);
    sum += part[j];
  }
  const uint64_t scan = wave_scan(sum);
  if (lane == 63) sh.waves[wave] = scan;
  __syncthreads();
  uint64_t at = scan - sum;
  for (int w = 0; w < wave; ++w) at += sh.waves[w];
  if (!(double(at) <= want && want < double(at + sum))) return;
  float y[kPer];   // the piece that holds the draw
  int piece = -1;
#pragma unroll
  for (int j = 0; j < kRun; ++j) {
    if (piece < 0 && double(at + part[j]) > want) {
      piece = j;
#pragma unroll
      for (int i = 0; i < kPer; ++i) y[i] = x[j][i];
    }
    if (piece < 0) at += part[j];
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const bool was = double(at) > want;
    at += cs.units(y[i]);
    if (!was && double(at) > want) finish(a, row, sh.top, sh.total, r.first(chunk * n + tid * run + piece) + i, y[i], sh.total);
  }
}

template <int kType>
__global__ __launch_bounds__(kDrawThreads) void sample_draw_kernel(SampleArgs a) {
  __shared__ Drawn sh;
  draw_row<kType, kDrawThreads>(a, int(blockIdx.x), sh);
}

// What a workgroup that looks for a threshold shares. kThreads: its threads.
template <int kThreads>
struct Shared {
  static constexpr int kWaves = kThreads / 64;
  union {
    Drawn drawn;
    struct {
      uint64_t mass[kBins];
      uint32_t count[kBins];
    };
  };
  uint64_t list[kList];          // entries: key, then the complement of the index (falling order is the ranks')
  uint64_t spare[kList];
  uint64_t wave_mass[64];
  uint32_t wave_count[64];
  Powers powers;
  float top;
  double total;
  // found by one thread
  int bin;
  int found;
  uint32_t above_count;
  uint64_t above_mass;
  uint32_t listed;
};

// The entries that stay: keys above `key`, and the first `ties` of those equal to it.
struct Cut {
  uint32_t key;
  uint32_t ties;
  uint64_t mass;     // sum of what stays
};

__device__ __forceinline__ uint64_t entry_of(uint32_t key, int index) { return join(~uint32_t(index), key); }
__device__ __forceinline__ int index_of(uint64_t entry) { return int(~uint32_t(entry)); }
__device__ __forceinline__ uint32_t key_of(uint64_t entry) { return uint32_t(entry >> 32); }

// Sum and count of the threads before this one in the workgroup (exclusive); *all_*: of all of them.
template <int kThreads>
__device__ __forceinline__ void block_scan(Shared<kThreads>& sh, uint64_t mass, uint32_t count, uint64_t* mass_before,
                                           uint32_t* count_before, uint64_t* all_mass, uint32_t* all_count) {
  const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
  const uint64_t m = wave_scan(mass);
  const uint32_t c = wave_scan(count);
  __syncthreads();
  if (lane == 63) {
    sh.wave_mass[wave] = m;
    sh.wave_count[wave] = c;
  }
  __syncthreads();
  uint64_t mb = m - mass, ma = 0;
  uint32_t cb = c - count, ca = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    mb += w < wave ? sh.wave_mass[w] : 0;
    cb += w < wave ? sh.wave_count[w] : 0;
    ma += sh.wave_mass[w];
    ca += sh.wave_count[w];
  }
  *mass_before = mb;
  *count_before = cb;
  *all_mass = ma;
  *all_count = ca;
}

// Sorts list[0 .. n) into falling order (n <= kList, no two alike). All threads. bin_of(entry), below kBins, does not
// fall from an entry to a smaller one: a count by bins places each entry to within its bin, whose others say the rest
// (4096 entries: 6 us, where the network below takes 50). Few entries are their own bin, and a bin of
// more than kCrowd, say of equal logits, leaves all to a sorting network.
constexpr int kCrowd = 256;
template <int kThreads, class BinOf>
__device__ __forceinline__ void sort_list(Shared<kThreads>& sh, int n, BinOf bin_of) {
  constexpr int kMine = kBins / kThreads, kPos = kList / kThreads;
  const int tid = int(threadIdx.x);
  __syncthreads();
  if (n <= kCrowd) {
    const uint64_t e = sh.list[tid < n ? tid : 0];
    int rank = 0;
    if ((tid & ~63) < n)
      for (int i = 0; i < n; ++i) rank += sh.list[i] > e;
    __syncthreads();
    if (tid < n) sh.list[rank] = e;
    __syncthreads();
    return;
  }
  for (int b = tid; b < kBins; b += kThreads) sh.count[b] = 0;
  if (tid == 0) sh.bin = 0;
  __syncthreads();
  uint32_t slot[kPos];
#pragma unroll
  for (int j = 0; j < kPos; ++j)
    if (tid + j * kThreads < n) slot[j] = atomicAdd(&sh.count[bin_of(sh.list[tid + j * kThreads])], 1u);
  __syncthreads();
  uint32_t c[kMine], mine = 0, most = 0;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    mine += c[i] = sh.count[kMine * tid + i];
    most = max(most, c[i]);
  }
  uint32_t before, all;
  uint64_t unused, unused2;
  if (most > kCrowd) sh.bin = 1;
  block_scan(sh, 0, mine, &unused, &before, &unused2, &all);
  if (sh.bin == 0) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      sh.count[kMine * tid + i] = before;   // the bin's first place
      before += c[i];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPos; ++j)
      if (tid + j * kThreads < n) {
        const uint64_t e = sh.list[tid + j * kThreads];
        sh.spare[sh.count[bin_of(e)] + slot[j]] = e;
      }
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
      const uint64_t e = sh.spare[i];
      const int b = bin_of(e), first = int(sh.count[b]), end = b + 1 < kBins ? int(sh.count[b + 1]) : n;
      int rank = first;
      for (int q = first; q < end; ++q) rank += sh.spare[q] > e;
      sh.list[rank] = e;
    }
    __syncthreads();
    return;
  }
  int size = 64;
  while (size < n) size *= 2;
  for (int i = n + tid; i < size; i += kThreads) sh.list[i] = 0;
  __syncthreads();
  for (int k = 2; k <= size; k *= 2)
    for (int j = k / 2; j > 0; j /= 2) {
      for (int p = tid; p < size / 2; p += kThreads) {
        const int lo = 2 * p - (p & (j - 1)), hi = lo + j;
        const uint64_t x = sh.list[lo], y = sh.list[hi];
        const bool falling = (lo & k) == 0;
        if (falling ? x < y : x > y) {
          sh.list[lo] = y;
          sh.list[hi] = x;
        }
      }
      __syncthreads();
    }
}

// Steps of the logit from the row's largest down to the bound: rounding keeps the order.
struct Steps {
  float top, per;
  __device__ __forceinline__ Steps(float largest, float bound)
      : top(largest), per(largest - bound > 0.f && largest - bound < __builtin_inff() ? float(kBins) / (largest - bound) : 0.f) {}
  __device__ __forceinline__ int of(float l) const { return int(fminf((top - l) * per, float(kBins - 1))); }
};

// Entries that lie in one step, mostly: by 2048 steps of that.
template <int kThreads>
__device__ __forceinline__ void sort_step(Shared<kThreads>& sh, int n, const Steps& steps) {
  const float first = n > 0 ? float(steps.of(logit_of(key_of(sh.list[0])))) : 0.f;
  sort_list(sh, n, [&](uint64_t e) {
    const float part = (steps.top - logit_of(key_of(e))) * steps.per - first;
    return int(fminf(fmaxf(part * float(kBins), 0.f), float(kBins - 1)));
  });
}

// Counts and sums by ranges of keys or steps of the logit, in falling order.
template <int kThreads>
__device__ __forceinline__ void clear_bins(Shared<kThreads>& sh) {
  for (int b = int(threadIdx.x); b < kBins; b += kThreads) {
    sh.mass[b] = 0;
    sh.count[b] = 0;
  }
  __syncthreads();
}
template <int kThreads>
__device__ __forceinline__ void add_to_bin(Shared<kThreads>& sh, int b, uint64_t units) {
  atomicAdd(&sh.count[b], 1u);
  atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[b]), (unsigned long long)(units));
}
// The bin that completes the first `most` entries (most > 0), or at which the
// sum reaches `share` (most = 0); -1: none. above_*: of what lies before it.
template <int kThreads>
__device__ __forceinline__ int crossing_bin(Shared<kThreads>& sh, uint32_t most, double share, uint32_t* above_count, uint64_t* above) {
  constexpr int kMine = kBins / kThreads;
  if (threadIdx.x == 0) sh.bin = -1;
  __syncthreads();
  const int b0 = kMine * int(threadIdx.x);
  uint64_t m[kMine], mass = 0;
  uint32_t c[kMine], count = 0;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    mass += m[i] = sh.mass[b0 + i];
    count += c[i] = sh.count[b0 + i];
  }
  uint64_t mb, unused64;
  uint32_t cb, unused;
  block_scan(sh, mass, count, &mb, &cb, &unused64, &unused);
  mb += *above;
  cb += *above_count;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const bool here = most ? cb < most && cb + c[i] >= most
                           : c[i] > 0 && double(mb) < share && double(mb + m[i]) >= share;
    if (here) {
      sh.bin = b0 + i;
      sh.above_count = cb;
      sh.above_mass = mb;
    }
    mb += m[i];
    cb += c[i];
  }
  __syncthreads();
  const int bin = sh.bin;
  if (bin >= 0) {
    *above_count = sh.above_count;
    *above = sh.above_mass;
  }
  __syncthreads();
  return bin;
}

// One row with cuts. Bound: no entry below it stays, and none below it enters the sums that say which do.
//   top-k: the k-th largest of the groups' largest logits (k entries at least are no smaller);
//   top-p of everything: entries with less than (1 - p) of the whole's mean weight sum to less than (1 - p) of the whole;
//   min-p: its own limit, where no top-k has to sum what lies below.
template <int kType>
__global__ __launch_bounds__(kCutThreads) void sample_cut_kernel(SampleArgs a) {
  constexpr int kPer = Elem<kType>::kPer;
  __shared__ Shared<kCutThreads> sh;
  constexpr int kPos = kList / kCutThreads;   // neighbouring positions of a thread
  const int row = int(blockIdx.x), tid = int(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const float t = temperature_of(a, row);
  const int k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.f;
  const double low = a.min_p && a.min_p[row] > 0.f ? fmin(double(a.min_p[row]), 1.0) : 0.0;
  const bool cut_k = k > 0 && k < a.vocab, cut_p = p < 1.f;
  if (greedy(t) || (!cut_k && !cut_p && low == 0.0)) {
    if (tid == 0) a.rows[row].open = 0;
    draw_row<kType, kCutThreads>(a, row, sh.drawn);
    return;
  }
  const Row<kType> r(a, row);
  const double rate = rate_of(t);
  make_powers(sh.powers);
  if (tid == 0) a.rows[row].open = 0;
  __syncthreads();
  if (wave == 0) {
    const Whole w = join_chunks(a, row, rate, sh.powers);
    if (lane == 0) {
      sh.top = w.top;
      sh.total = w.total;
      sh.listed = 0;
    }
  }
  __syncthreads();
  const float top = sh.top;
  const double total = sh.total;
  if (top == kNone) {
    if (tid == 0) finish(a, row, top, 1.0, -1, 0.f, 0.0);
    return;
  }
  const Scale s(sh.powers, top, rate);
  const uint32_t top_key = key_of(top);
  const float* groups = a.groups + size_t(row) * a.num_chunks * (a.chunk / kGroup);
  const int num_groups = (r.pieces * kPer + kGroup - 1) / kGroup;

  // the bound
  float bound = -__FLT_MAX__;
  auto at_weight = [&](double w) {   // a logit of no more than this weight
    const double l = double(top) + log2(w) / rate;
    return float(l - 1e-6 * (fabs(l) + fabs(double(top))) - 1e-30);
  };
  if (top == __builtin_inff()) {
    bound = top;
  } else if (cut_k) {
    // by key ranges of the groups' largest logits, as refine()
    uint32_t lo = key_of(-__FLT_MAX__), hi = top_key, above_count = 0;
    uint64_t above = 0;
    for (;;) {
      const uint32_t range = hi - lo;
      const int bits = range ? 32 - __builtin_clz(range) : 0;
      const int shift = max(0, bits - 11);
      clear_bins(sh);
      for (int g = tid; g < num_groups; g += kCutThreads) {
        const uint32_t key = key_of(groups[g]);
        if (key >= lo && key <= hi) atomicAdd(&sh.count[(hi - key) >> shift], 1u);
      }
      const int bin = crossing_bin(sh, uint32_t(k), 0.0, &above_count, &above);
      if (bin < 0) break;
      hi -= uint32_t(bin) << shift;
      lo = hi - lo >= (1u << shift) ? hi - ((1u << shift) - 1u) : lo;
      bound = logit_of(lo);
      if (shift <= 13) break;   // near enough
    }
    if (!cut_p && low > 0.0) bound = fmaxf(bound, at_weight(low));
  } else {
    if (cut_p) bound = fmaxf(bound, at_weight(fmax(0.0, 1.0 - double(p)) * total * kUnit / double(a.vocab)));
    if (low > 0.0) bound = fmaxf(bound, at_weight(low));
  }
  bound = fminf(fmaxf(bound, at_weight(0x1p-60)), top);   // (weights below it are none)

  // the entries above it, if the list holds them
  uint32_t near = 0;
  for (int g = tid; g < num_groups; g += kCutThreads) near += groups[g] >= bound;
  uint64_t unused64, unused_sum;
  uint32_t near_before, num_near;
  block_scan(sh, 0, near, &unused64, &near_before, &unused_sum, &num_near);
  if (num_near <= kBins) {
    uint32_t* const ids = sh.count;
    for (int g = tid; g < num_groups; g += kCutThreads)
      if (groups[g] >= bound) ids[near_before++] = uint32_t(g);
    __syncthreads();
    constexpr int kPieces = kGroup / kPer;
    constexpr int kDeep = kType == kF32 ? 8 : 4;   // loads in flight
    for (uint32_t w0 = 0; w0 < num_near * kPieces; w0 += kCutThreads * kDeep) {
      const uint32_t i0 = w0 + uint32_t(tid);
      float x[kDeep][kPer];
      int piece[kDeep];
#pragma unroll
      for (int d = 0; d < kDeep; ++d) {
        const uint32_t i = i0 + uint32_t(d) * kCutThreads;
        piece[d] = i < num_near * kPieces ? int(ids[i / kPieces]) * kPieces + int(i % kPieces) : r.pieces;   // (nothing behind the last)
      }
      load_all(r, x, [&](int d) { return piece[d]; });
      uint32_t mine = 0;
#pragma unroll
      for (int d = 0; d < kDeep; ++d)
#pragma unroll
        for (int j = 0; j < kPer; ++j) mine += x[d][j] >= bound;
      const uint32_t upto = wave_scan(mine);
      uint32_t at = 0;
      if (lane == 63) at = atomicAdd(&sh.listed, upto);
      at = uint32_t(__shfl(int(at), 63)) + upto - mine;
      if (mine == 0) continue;
#pragma unroll
      for (int d = 0; d < kDeep; ++d)
#pragma unroll
        for (int j = 0; j < kPer; ++j)
          if (x[d][j] >= bound) {
            if (at < kList) sh.list[at] = entry_of(key_of(x[d][j]), r.first(piece[d]) + j);
            ++at;
          }
    }
    __syncthreads();
    const int n = int(sh.listed);
    if (n <= kList) {
      const Steps steps(top, bound);
      sort_list(sh, n, [&](uint64_t e) { return steps.of(logit_of(key_of(e))); });
      const int p0 = kPos * tid;
      uint64_t w[kPos], sum = 0;
      uint32_t heavy = 0;   // entries of at least the least weight, the first ones
#pragma unroll
      for (int i = 0; i < kPos; ++i) {
        w[i] = 0;
        if (p0 + i < n) {
          const float l = logit_of(key_of(sh.list[p0 + i]));
          w[i] = s.units(l);
          heavy += low == 0.0 || s.weight(l) >= low;
        }
        sum += w[i];
      }
      uint64_t before, list_sum;
      uint32_t heavy_before, all_heavy;
      block_scan(sh, sum, heavy, &before, &heavy_before, &list_sum, &all_heavy);
      int stays = int(all_heavy);
      if (cut_k) stays = min(stays, k);
      if (tid == 0) {
        sh.above_mass = list_sum;
        sh.found = 0;
      }
      __syncthreads();
      // the first k's sum, then how many entries have less than the share before them
      if (cut_k && k < n && k - 1 >= p0 && k - 1 < p0 + kPos) {
        uint64_t x = before;
        for (int i = 0; i <= k - 1 - p0; ++i) x += w[i];
        sh.above_mass = x;
      }
      __syncthreads();
      if (cut_p) {
        const double share = fmax(double(p) * (cut_k ? double(sh.above_mass) : total), 1.0);
        uint32_t mine = 0;
        uint64_t x = before;
#pragma unroll
        for (int i = 0; i < kPos; ++i) {
          if (p0 + i < n && double(x) < share) ++mine;
          x += w[i];
        }
        mine = wave_sum(mine);
        if (lane == 0) atomicAdd(&sh.found, int(mine));
        __syncthreads();
        stays = min(stays, sh.found);
      }
      // what stays in index order: index, then place in the list
      __syncthreads();
      uint64_t entry[kPos];
#pragma unroll
      for (int i = 0; i < kPos; ++i) {
        const int q = p0 + i;
        entry[i] = q < stays ? sh.list[q] : 0;
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kPos; ++i)
        if (p0 + i < stays) sh.list[p0 + i] = join(key_of(entry[i]), ~uint32_t(index_of(entry[i])));   // falling: index rising
      __syncthreads();
      const int shift = max(0, 32 - __builtin_clz(uint32_t(a.vocab)) - kBinBits);
      sort_list(sh, stays, [&](uint64_t e) { return int(~uint32_t(e >> 32) >> shift); });
      sum = 0;
#pragma unroll
      for (int i = 0; i < kPos; ++i) {
        w[i] = p0 + i < stays ? s.units(logit_of(uint32_t(sh.list[p0 + i]))) : 0;
        sum += w[i];
      }
      uint64_t kept;
      uint32_t unused, unused_count;
      block_scan(sh, sum, 0, &before, &unused, &kept, &unused_count);
      const double target = uniform_of(a, row) * double(kept);
#pragma unroll
      for (int i = 0; i < kPos; ++i) {
        const bool was = double(before) > target;
        before += w[i];
        if (!was && w[i] > 0 && double(before) > target) {
          const uint64_t e = sh.list[p0 + i];
          finish(a, row, top, total, int(~uint32_t(e >> 32)), logit_of(uint32_t(e)), double(kept));
        }
      }
      return;
    }
  }

  // left to the launches behind this one
  // (which rows get a place may differ from run to run; what they give does not)
  if (tid == 0) {
    const uint32_t place = cut_k ? uint32_t(a.places) : atomicAdd(a.taken, 1u);
    sh.found = place < uint32_t(a.places) ? int(place) + 1 : -1;
    a.rows[row] = SampleRow{total, 0, top, bound, sh.found, 0};
  }
  __syncthreads();
  const int open = sh.found;
  if (open > 0)
    for (int b = tid; b < kBins; b += kCutThreads) a.bins[size_t(open - 1) * kBins + b] = 0;
}

// The slow way, of a row with a top-k of more entries than the list holds, or with as many near
// a cut: read whole by one workgroup, in 64 runs, once per cut and twice for the draw.
constexpr int kRuns = 64;
constexpr int kWaveRuns = kRuns / (kRowThreads / 64);
template <int kType>
__device__ __forceinline__ int run_begin(const Row<kType>& r, int run) {
  const int per = (r.pieces + kRuns - 1) / kRuns;
  return min(r.pieces, run * per);
}
// Calls use(logit, index) for every entry of a run, in the wave that takes it.
template <int kType, class Use>
__device__ __forceinline__ void for_run(const Row<kType>& r, int run, Use use) {
  constexpr int kPer = Elem<kType>::kPer, kDeep = 4;   // loads in flight
  const int end = run_begin(r, run + 1);
  for (int p = run_begin(r, run) + (int(threadIdx.x) & 63); p < end; p += 64 * kDeep) {
    float x[kDeep][kPer];
    load_all(r, x, [&](int d) { return p + 64 * d < end ? p + 64 * d : r.pieces; });   // (nothing behind the last)
#pragma unroll
    for (int d = 0; d < kDeep; ++d)
#pragma unroll
      for (int i = 0; i < kPer; ++i) use(x[d][i], r.first(p + 64 * d) + i);
  }
}
template <int kType, class Use>
__device__ __forceinline__ void for_each(const Row<kType>& r, Use use) {
  const int wave = int(threadIdx.x) >> 6;
#pragma nounroll
  for (int i = 0; i < kWaveRuns; ++i) for_run(r, kWaveRuns * wave + i, use);
}

template <int kType>
__device__ __forceinline__ void whole_row(const SampleArgs& a, int row, const SampleRow& st, Shared<kRowThreads>& sh) {
  constexpr int kPer = Elem<kType>::kPer;
  constexpr int kPos = kList / kRowThreads;
  const int tid = int(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const float t = temperature_of(a, row);
  const int k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.f;
  const double low = a.min_p && a.min_p[row] > 0.f ? fmin(double(a.min_p[row]), 1.0) : 0.0;
  const bool cut_k = k > 0 && k < a.vocab, cut_p = p < 1.f;
  const Row<kType> r(a, row);
  const double rate = rate_of(t);
  make_powers(sh.powers);
  __syncthreads();
  const float top = st.top, bound = st.bound;   // (the chunks' sums may be those of what stays by now)
  const Scale s(sh.powers, top, rate);
  const Steps steps(top, bound);

  Cut cut = {0, 0, 0};   // nothing is cut: every key is above 0
  double whole = st.total;
  // Top-k, then top-p of what it leaves. Ranges: equal steps of the logit first; the one in
  // which the cut falls is sorted, or, of more entries than the list, refined by keys (three times for 32 bits).
  for (int by_p = cut_k ? 0 : 1; by_p < (cut_p ? 2 : 1); ++by_p) {
    const uint32_t most = by_p ? 0u : uint32_t(k);
    // no share lies before the first, so it always stays; entries behind the k-th do not reach the share
    const double share = by_p ? fmax(double(p) * whole, 1.0) : 0.0;
    uint32_t above_count = 0, lo = max(cut.key, 1u), hi = key_of(top);
    uint64_t above = 0;
    int shift = -1;        // by steps
    bool found = false;
    Cut next = cut;
#pragma nounroll
    for (;;) {
      clear_bins(sh);
      for_each(r, [&](float l, int) {
        const uint32_t key = key_of(l);
        if (l >= bound && key >= lo && key <= hi) add_to_bin(sh, shift < 0 ? steps.of(l) : int((hi - key) >> shift), s.units(l));
      });
      const int bin = crossing_bin(sh, most, share, &above_count, &above);
      if (bin < 0) break;
      const uint32_t count = sh.count[bin];
      const uint64_t mass = sh.mass[bin];
      if (shift == 0) {    // one key
        const uint64_t w = mass / count;
        next.key = hi - uint32_t(bin);
        next.ties = most ? most - above_count : w ? uint32_t(fmin(double(count), ceil((share - double(above)) / double(w)))) : count;
        next.mass = above + next.ties * w;
        found = true;
        break;
      }
      if (count <= kList) {
        if (tid == 0) {
          sh.listed = 0;
          sh.found = -1;
        }
        __syncthreads();
        for_each(r, [&](float l, int index) {
          const uint32_t key = key_of(l);
          if (l >= bound && key >= lo && key <= hi && (shift < 0 ? steps.of(l) : int((hi - key) >> shift)) == bin)
            sh.list[atomicAdd(&sh.listed, 1u)] = entry_of(key, index);
        });
        __syncthreads();
        sort_step(sh, int(count), steps);
        const int n = int(count), p0 = kPos * tid;
        uint64_t sum = 0;
#pragma unroll
        for (int i = 0; i < kPos; ++i) sum += p0 + i < n ? s.units(logit_of(key_of(sh.list[p0 + i]))) : 0;
        uint64_t before, unused64;
        uint32_t unused, unused2;
        block_scan(sh, sum, 0, &before, &unused, &unused64, &unused2);
        before += above;
#pragma unroll
        for (int i = 0; i < kPos; ++i) {
          const int q = p0 + i;
          const uint64_t w = q < n ? s.units(logit_of(key_of(sh.list[q]))) : 0;
          const bool last = q < n && (most ? above_count + uint32_t(q) + 1 == most
                                           : double(before) < share && (double(before + w) >= share || q + 1 == n));
          before += w;
          if (last) {
            sh.found = q;
            sh.above_mass = before;
          }
        }
        __syncthreads();
        // entries equal to the last one that stays
        const int at = sh.found;
        next.key = key_of(sh.list[at]);
        next.mass = sh.above_mass;
        uint32_t ties = 0;
#pragma unroll
        for (int i = 0; i < kPos; ++i) ties += p0 + i <= at && key_of(sh.list[p0 + i]) == next.key;
        block_scan(sh, 0, ties, &unused64, &unused, &before, &next.ties);
        found = true;
        break;
      }
      // by keys from here on, all of them the first time
      if (shift < 0) {
        above_count = 0;
        above = 0;
      } else {
        hi -= uint32_t(bin) << shift;
        lo = hi - lo >= (1u << shift) ? hi - ((1u << shift) - 1u) : lo;
      }
      shift = max(0, (hi > lo ? 32 - __builtin_clz(hi - lo) : 0) - 11);
      __syncthreads();
    }
    __syncthreads();
    if (found) {
      if (next.key == cut.key) next.ties = min(next.ties, cut.ties);
      cut = next;
      whole = double(cut.mass);
    }
  }

  // what stays, run by run
  uint64_t tie_units = 0;
#pragma nounroll
  for (int i = 0; i < kWaveRuns; ++i) {
    uint64_t sum = 0;
    uint32_t ties = 0;
    for_run(r, kWaveRuns * wave + i, [&](float l, int) {
      const uint32_t key = key_of(l);
      if (l < bound || key < cut.key || key == 0 || (low > 0.0 && s.weight(l) < low)) return;
      const uint64_t w = s.units(l);
      if (key > cut.key) {
        sum += w;
      } else {
        ++ties;
        tie_units = w;
      }
    });
    sum = wave_sum(sum);
    ties = wave_sum(ties);
    if (lane == 0) {
      sh.wave_mass[kWaveRuns * wave + i] = sum;
      sh.wave_count[kWaveRuns * wave + i] = ties;
    }
  }
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const uint64_t y = shuffle_xor(tie_units, m);
    tie_units = tie_units > y ? tie_units : y;
  }
  if (lane == 0) sh.mass[wave] = tie_units;
  __syncthreads();
  for (int w = 0; w < kRowThreads / 64; ++w) tie_units = tie_units > sh.mass[w] ? tie_units : sh.mass[w];
  // lane i of every wave: run i
  const uint32_t seen = wave_scan(sh.wave_count[lane]) - sh.wave_count[lane];
  const uint32_t left = cut.ties > seen ? cut.ties - seen : 0;
  const uint64_t in_run = sh.wave_mass[lane] + uint64_t(min(left, sh.wave_count[lane])) * tie_units;
  const uint64_t upto = wave_scan(in_run), kept = shuffle(upto, 63);
  const double target = uniform_of(a, row) * double(kept);
  const uint64_t holds = __ballot(double(upto - in_run) <= target && target < double(upto));
  const int run = __builtin_ctzll(holds);   // (some run does: target < kept)
  if (wave != 0) return;
  // the run that holds the draw
  uint64_t cum = shuffle(upto - in_run, run);
  uint32_t tie = uint32_t(__shfl(int(seen), run));
  const int end = run_begin(r, run + 1);
  for (int q0 = run_begin(r, run); q0 < end; q0 += 64) {
    float x[kPer];
    uint64_t w[kPer], lane_sum = 0;
    uint32_t is_tie = 0, mine_ties = 0;
    const int q = q0 + lane;
    r.load(q < end ? q : r.pieces, x);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      // Selects of values formed for all lanes: with a branch around the weight, hipcc left the weight's bits in
      // w[i] of lanes that it sent away (ROCm 7.2.0; a draw then fell to an entry below the least weight).
      const uint32_t key = key_of(x[i]);
      const uint64_t units = s.units(x[i]);
      bool in = (x[i] >= bound) & (key >= cut.key) & (key != 0);
      if (low > 0.0) in &= !(s.weight(x[i]) < low);
      const bool tie = in & (key == cut.key);
      w[i] = in ? units : 0;
      is_tie |= uint32_t(tie) << i;
      mine_ties += tie;
    }
    uint32_t rank = tie + wave_scan(mine_ties) - mine_ties;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (is_tie >> i & 1) {
        if (rank >= cut.ties) w[i] = 0;
        ++rank;
      }
      lane_sum += w[i];
    }
    const uint64_t scan = wave_scan(lane_sum);
    uint64_t at = cum + scan - lane_sum;
    if (double(at) <= target && target < double(at + lane_sum)) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const bool was = double(at) > target;
        at += w[i];
        if (!was && double(at) > target) finish(a, row, top, st.total, r.first(q) + i, x[i], double(kept));
      }
    }
    cum += shuffle(scan, 63);
    tie += wave_sum(mine_ties);
    if (double(cum) > target) return;
  }
}

// Rows without a top-k that keep more than the list holds, by three launches over all of the row's chunks:
// sums by equal steps of the logit; the step in which the share is reached, whose entries are
// listed, with the sums of what lies above it by chunk; the order of the listed ones, which is the cut, and the draw.
struct Crossing {
  int bin;          // kBins: nowhere
  uint64_t above;   // the sum before it
};
__device__ __forceinline__ double share_of(const SampleArgs& a, int row, double whole) {
  const float p = a.top_p ? a.top_p[row] : 1.f;
  return p < 1.f ? fmax(double(p) * whole, 1.0) : __builtin_inf();   // no share lies before the first, so it always stays
}
__device__ __forceinline__ double least_of(const SampleArgs& a, int row) {
  return a.min_p && a.min_p[row] > 0.f ? fmin(double(a.min_p[row]), 1.0) : 0.0;
}
template <int kType, int kChunk>
__global__ __launch_bounds__(kChunkThreads) void sample_bins_kernel(SampleArgs a) {
  constexpr int kPer = Elem<kType>::kPer;
  constexpr int kPieces = kChunk / kPer / kChunkThreads;
  __shared__ uint64_t mass[kBins];
  __shared__ Powers powers;
  const int row = int(blockIdx.x) / a.num_chunks, chunk = int(blockIdx.x) % a.num_chunks, tid = int(threadIdx.x);
  const SampleRow st = a.rows[row];
  if (st.open <= 0) return;
  const Row<kType> r(a, row);
  float x[kPieces][kPer];
  load_all(r, x, [&](int j) { return chunk * (kChunk / kPer) + tid + j * kChunkThreads; });
  make_powers(powers);
  for (int b = tid; b < kBins; b += kChunkThreads) mass[b] = 0;
  __syncthreads();
  const Scale s(powers, st.top, rate_of(temperature_of(a, row)));
  const Steps steps(st.top, st.bound);
#pragma unroll
  for (int j = 0; j < kPieces; ++j)
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const uint64_t w = s.units(x[j][i]);
      if (x[j][i] >= st.bound && w) atomicAdd(reinterpret_cast<unsigned long long*>(&mass[steps.of(x[j][i])]), (unsigned long long)(w));
    }
  __syncthreads();
  for (int b = tid; b < kBins; b += kChunkThreads)
    if (mass[b]) atomicAdd(reinterpret_cast<unsigned long long*>(a.bins + size_t(st.open - 1) * kBins + b), (unsigned long long)(mass[b]));
}

template <int kType, int kChunk>
__global__ __launch_bounds__(kChunkThreads) void sample_collect_kernel(SampleArgs a) {
  constexpr int kPer = Elem<kType>::kPer;
  constexpr int kPieces = kChunk / kPer / kChunkThreads;
  constexpr int kWaves = kChunkThreads / 64, kMine = kBins / kChunkThreads;
  __shared__ uint64_t sums[kWaves];
  __shared__ Crossing found;
  __shared__ Powers powers;
  const int row = int(blockIdx.x) / a.num_chunks, chunk = int(blockIdx.x) % a.num_chunks;
  const int tid = int(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const SampleRow st = a.rows[row];
  if (st.open <= 0) return;
  const Row<kType> r(a, row);
  float x[kPieces][kPer];
  load_all(r, x, [&](int j) { return chunk * (kChunk / kPer) + tid + j * kChunkThreads; });
  // the crossing, by every chunk for itself
  const uint64_t* bins = a.bins + size_t(st.open - 1) * kBins + kMine * tid;
  uint64_t m[kMine], mine = 0;
#pragma unroll
  for (int i = 0; i < kMine; ++i) mine += m[i] = bins[i];
  const uint64_t scan = wave_scan(mine);
  if (lane == 63) sums[wave] = scan;
  if (tid == 0) found.bin = kBins;
  make_powers(powers);
  __syncthreads();
  uint64_t before = scan - mine;
  for (int w = 0; w < wave; ++w) before += sums[w];
  const double share = share_of(a, row, st.total);
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    if (double(before) < share && double(before + m[i]) >= share) {
      found.bin = kMine * tid + i;
      found.above = before;
      if (chunk == 0) a.rows[row].above = before;
    }
    before += m[i];
  }
  __syncthreads();
  const int bin = found.bin;
  const Scale s(powers, st.top, rate_of(temperature_of(a, row)));
  const Steps steps(st.top, st.bound);
  const double low = least_of(a, row);
  uint64_t sum = 0;
#pragma unroll
  for (int j = 0; j < kPieces; ++j)
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const float l = x[j][i];
      const uint64_t w = s.units(l);
      const bool in = l >= st.bound && w;
      const int b = steps.of(l);
      if (in && b < bin && (low == 0.0 || s.weight(l) >= low)) sum += w;
      if (in && b == bin) {
        const uint32_t at = atomicAdd(&a.rows[row].listed, 1u);
        if (at < kList) a.lists[size_t(st.open - 1) * kList + at] = entry_of(key_of(l), r.first(chunk * (kChunk / kPer) + tid + j * kChunkThreads) + i);
      }
    }
  sum = wave_sum(sum);
  __syncthreads();
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kWaves; ++w) sum += sums[w];
    a.chunks[blockIdx.x].sum = sum;   // what stays of the chunk for certain
  }
}

template <int kType>
__global__ __launch_bounds__(kRowThreads) void sample_finish_kernel(SampleArgs a) {
  constexpr int kPer = Elem<kType>::kPer;
  constexpr int kPos = kList / kRowThreads;
  __shared__ Shared<kRowThreads> sh;
  const int row = int(blockIdx.x), tid = int(threadIdx.x);
  const SampleRow st = a.rows[row];
  if (st.open == 0) return;
  if (st.open < 0 || st.listed > kList) {
    whole_row<kType>(a, row, st, sh);
    return;
  }
  const Row<kType> r(a, row);
  const float top = st.top;
  make_powers(sh.powers);
  const int n = int(st.listed), p0 = kPos * tid;
  for (int i = tid; i < n; i += kRowThreads) sh.list[i] = a.lists[size_t(st.open - 1) * kList + i];
  // sums of what stays by chunk, joined below by the listed entries'
  uint64_t* const by_chunk = sh.mass;
  for (int c = tid; c < kMaxChunks; c += kRowThreads) by_chunk[c] = c < a.num_chunks ? a.chunks[size_t(row) * a.num_chunks + c].sum : 0;
  __syncthreads();
  sort_step(sh, n, Steps(top, st.bound));
  const Scale s(sh.powers, top, rate_of(temperature_of(a, row)));
  const double low = least_of(a, row), share = share_of(a, row, st.total);
  uint64_t w[kPos], sum = 0;
#pragma unroll
  for (int i = 0; i < kPos; ++i) {
    w[i] = p0 + i < n ? s.units(logit_of(key_of(sh.list[p0 + i]))) : 0;
    sum += w[i];
  }
  uint64_t before, all;
  uint32_t unused, unused2;
  if (tid == 0) sh.found = -1;
  block_scan(sh, sum, 0, &before, &unused, &all, &unused2);
  before += st.above;
#pragma unroll
  for (int i = 0; i < kPos; ++i) {
    if (p0 + i < n && double(before) < share) {
      atomicMax(&sh.found, p0 + i);
      const float l = logit_of(key_of(sh.list[p0 + i]));
      if (low == 0.0 || s.weight(l) >= low)
        atomicAdd(reinterpret_cast<unsigned long long*>(&by_chunk[(index_of(sh.list[p0 + i]) + r.lead) / a.chunk]), (unsigned long long)(w[i]));
    }
    before += w[i];
  }
  __syncthreads();
  const uint64_t last = n > 0 ? sh.list[sh.found] : 0;   // entries from it on stay
  // the chunk that holds the draw
  const uint64_t mine = tid < kMaxChunks ? by_chunk[tid] : 0;
  uint64_t kept;
  block_scan(sh, mine, 0, &before, &unused, &kept, &unused2);
  const double target = uniform_of(a, row) * double(kept);
  if (double(before) <= target && target < double(before + mine)) {
    sh.bin = tid;
    sh.above_mass = before;
  }
  __syncthreads();
  const int chunk = sh.bin;
  const uint64_t base = sh.above_mass;
  const int pieces = a.chunk / kPer, run = (pieces + kRowThreads - 1) / kRowThreads;
  constexpr int kRun = kSampleChunk / kPer / kRowThreads;
  float x[kRun][kPer];
  uint64_t units[kRun][kPer];
  sum = 0;
  auto piece_of = [&](int j) {
    const int q = tid * run + j;
    return j < run && q < pieces ? chunk * pieces + q : r.pieces;   // (nothing behind the last)
  };
  load_all(r, x, piece_of);
#pragma unroll
  for (int j = 0; j < kRun; ++j) {
    const int piece = piece_of(j);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const float l = x[j][i];
      const bool in = l >= st.bound && l != kNone && entry_of(key_of(l), r.first(piece) + i) >= last && (low == 0.0 || s.weight(l) >= low);
      units[j][i] = in ? s.units(l) : 0;
      sum += units[j][i];
    }
  }
  block_scan(sh, sum, 0, &before, &unused, &all, &unused2);
  before += base;
  if (!(double(before) <= target && target < double(before + sum))) return;
#pragma unroll
  for (int j = 0; j < kRun; ++j)
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const bool was = double(before) > target;
      before += units[j][i];
      if (!was && double(before) > target) finish(a, row, top, st.total, r.first(chunk * pieces + tid * run + j) + i, x[j][i], double(kept));
    }
}

template <int kType, int kChunk>
void launch_chunks(const SampleArgs& a, hipStream_t stream) {
  const dim3 grid{uint32_t(a.num_rows) * uint32_t(a.num_chunks), 1, 1};
  if (a.groups)
    hipLaunchKernelGGL((sample_chunk_kernel<kType, kChunk, true>), grid, dim3(kChunkThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((sample_chunk_kernel<kType, kChunk, false>), grid, dim3(kChunkThreads), 0, stream, a);
}

// The rows that the sorted list did not do.
template <int kType, int kChunk>
void launch_open(const SampleArgs& a, hipStream_t stream) {
  const dim3 grid{uint32_t(a.num_rows) * uint32_t(a.num_chunks), 1, 1};
  if (a.top_p || a.min_p) {
    hipLaunchKernelGGL((sample_bins_kernel<kType, kChunk>), grid, dim3(kChunkThreads), 0, stream, a);
    hipLaunchKernelGGL((sample_collect_kernel<kType, kChunk>), grid, dim3(kChunkThreads), 0, stream, a);
  }
  hipLaunchKernelGGL(sample_finish_kernel<kType>, dim3(uint32_t(a.num_rows)), dim3(kRowThreads), 0, stream, a);
}

template <int kType>
hipError_t launch(const SampleArgs& a, hipStream_t stream) {
  if (a.chunk == kSampleChunk)
    launch_chunks<kType, kSampleChunk>(a, stream);
  else
    launch_chunks<kType, kSampleSmallChunk>(a, stream);
  if (a.groups)
    hipLaunchKernelGGL(sample_cut_kernel<kType>, dim3(uint32_t(a.num_rows)), dim3(kCutThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(sample_draw_kernel<kType>, dim3(uint32_t(a.num_rows)), dim3(kDrawThreads), 0, stream, a);
  if (a.groups) {
    if (a.chunk == kSampleChunk)
      launch_open<kType, kSampleChunk>(a, stream);
    else
      launch_open<kType, kSampleSmallChunk>(a, stream);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, int32_t dtype, hipStream_t stream) {
  switch (dtype) {
    case kF32: return launch<kF32>(a, stream);
    case kBF16: return launch<kBF16>(a, stream);
    default: return launch<kF16>(a, stream);
  }
}

}  // namespace sf
