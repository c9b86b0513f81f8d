// Sampling with temperature, top-k, top-p and min-p from given uniform numbers.
//
// Each row asks which index a running sum crosses a share of the whole at, and
// the answer must not depend on the order of the sums: weights are rounded to
// multiples of 2^-44 of the largest (fp64 arithmetic, whose fma runs at the rate of an unpacked fp32 one
// here) and added as integers, by atomics too.
//
// Two launches. The first reads the logits once, a chunk per workgroup: the
// chunk's largest logit, the sum of its weights relative to it and, where there are cuts, the
// largest logit of every 64. The second, a workgroup per row, joins the chunks'
// sums. Without cuts it then knows the chunk of the drawn index, and reads that again.
// With cuts, the kept entries are the first ones in the order of falling logits, and
// the groups' largest logits bound where that order can end (Bound below): if
// no more than 4096 entries lie above the bound, only their groups are read again, the
// entries are sorted in LDS and every cut is a position there. Else the row is read
// again: one pass for counts and sums by 2048 equal steps of the logit, one that
// sorts the entries of the step in which the cut falls, one for the sums of what stays by runs of the row and
// one over the run of the draw.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "sf_internal.h"

namespace sf {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kChunkThreads = 256;
constexpr int kDrawThreads = 256;
constexpr int kRowThreads = 512;    // two waves per SIMD: nothing may spill (below)
constexpr int kRowWaves = kRowThreads / 64;
constexpr int kBins = 2048;
constexpr int kUnitBits = 44;
constexpr double kUnit = 0x1p-44;
constexpr int kList = 4096;        // entries that are sorted
constexpr int kPos = kList / kRowThreads;   // neighbouring ones of a thread
constexpr int kGroup = kSampleGroup;
constexpr float kNone = -__builtin_inff();

enum Type { kF32 = 0, kBF16 = 1, kF16 = 2 };

template <int kType>
struct Elem {
  static constexpr int kBytes = kType == kF32 ? 4 : 2;
  static constexpr int kPer = 16 / kBytes;   // logits of a 16-byte piece
};

// A NaN counts as no entry, and -0 as 0 (equal logits have equal keys).
__device__ __forceinline__ float clean(float x) { return x == x ? x + 0.f : kNone; }

// (A bit cast of a vector's element itself takes the vector's first.)
__device__ __forceinline__ float value32(uint32_t bits) { return __builtin_bit_cast(float, bits); }
template <int kType>
__device__ __forceinline__ float value16(uint32_t bits) {
  if constexpr (kType == kBF16) return __builtin_bit_cast(float, bits << 16);
  return float(__builtin_bit_cast(_Float16, uint16_t(bits)));
}

// A row of logits as 16-byte pieces at 16-byte addresses: piece p holds
// entries p * kPer - lead .. + kPer - 1, of which the first and the last pieces
// may lack some.
template <int kType>
struct Row {
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
  // Entries that a piece lacks, or past the last piece, are -inf.
  __device__ __forceinline__ void load(int p, float* x) const {
    constexpr int kPer = Elem<kType>::kPer, kBytes = Elem<kType>::kBytes;
    const int lo = first(p);
    if (lo >= 0 && lo + kPer <= vocab) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(base + int64_t(p) * 16);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if constexpr (kType == kF32)
          x[i] = clean(value32(w[i]));
        else
          x[i] = clean(value16<kType>(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xFFFFu));
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      x[i] = kNone;
      if (lo + i >= 0 && lo + i < vocab) {
        const char* at = base + int64_t(p) * 16 + i * kBytes;
        if constexpr (kType == kF32)
          x[i] = clean(*reinterpret_cast<const float*>(at));
        else
          x[i] = clean(value16<kType>(*reinterpret_cast<const uint16_t*>(at)));
      }
    }
  }
};

// 2^f, |f| <= 1/2: the Taylor series to f^11 (the next term is below 2^-47).
__device__ __forceinline__ double exp2_part(double f) {
  double p = 4.4455382718708114976e-10;
  p = __builtin_fma(p, f, 7.0549116208011233299e-9);
  p = __builtin_fma(p, f, 1.0178086009239699728e-7);
  p = __builtin_fma(p, f, 1.3215486790144309488e-6);
  p = __builtin_fma(p, f, 1.5252733804059840280e-5);
  p = __builtin_fma(p, f, 0.00015403530393381610);
  p = __builtin_fma(p, f, 0.00133335581464284434);
  p = __builtin_fma(p, f, 0.00961812910762847716);
  p = __builtin_fma(p, f, 0.05550410866482157995);
  p = __builtin_fma(p, f, 0.24022650695910071233);
  p = __builtin_fma(p, f, 0.69314718055994530942);
  return __builtin_fma(p, f, 1.0);
}

// 2^(y + shift) for -1000 < y + shift: the nearest whole number comes off by adding
// 1.5 2^52, and goes back as an addition to the exponent.
__device__ __forceinline__ double exp2_of(double y, int shift) {
  const double t = y + 0x1.8p52;
  const int n = int(uint32_t(__builtin_bit_cast(uint64_t, t))) + shift;
  const double p = exp2_part(y - (t - 0x1.8p52));
  return __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, p) + (uint64_t(uint32_t(n << 20)) << 32));
}

// Weights of logits relative to a largest one: exp((l - top) / T), 1 / (T ln 2) in rate.
struct Scale {
  float top;
  double rate;
  __device__ __forceinline__ double exponent(float l) const { return (double(l) - double(top)) * rate; }
  // In units of 2^-44, rounded, with the bits of 2^52 above them. (max takes its other operand for the NaN of -inf * 0.)
  __device__ __forceinline__ uint64_t raw_units(float l) const {
    const double y = fmax(exponent(l), -62.0);
    return __builtin_bit_cast(uint64_t, exp2_of(y, kUnitBits) + 0x1p52);   // the sum's last bit is one unit
  }
  static constexpr uint64_t kRaw = 0x4330000000000000ull;
  __device__ __forceinline__ uint64_t units(float l) const {
    if (top == __builtin_inff()) return l == top ? uint64_t(1) << kUnitBits : 0;
    return raw_units(l) - kRaw;
  }
  __device__ __forceinline__ double weight(float l) const {
    if (top == __builtin_inff()) return l == top ? 1.0 : 0.0;
    const double y = exponent(l);
    return y > -1000.0 ? exp2_of(y, 0) : 0.0;
  }
};

__device__ __forceinline__ bool greedy(float t) { return !(t > 0.f); }
__device__ __forceinline__ float temperature_of(const SampleArgs& a, int row) { return a.temperature ? a.temperature[row] : 1.f; }
__device__ __forceinline__ double rate_of(float t) { return 1.44269504088896340736 / (greedy(t) ? 1.0 : double(t)); }

// Rising keys for rising logits, above 0 for every finite one and +inf.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x);
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
  const int row = int(blockIdx.x) / a.num_chunks, chunk = int(blockIdx.x) % a.num_chunks;
  const Row<kType> r(a, row);
  const int tid = int(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const int p0 = chunk * (kChunk / kPer) + tid;
  float x[kPieces][kPer];
#pragma unroll
  for (int j = 0; j < kPieces; ++j) r.load(p0 + j * kChunkThreads, x[j]);
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
  const Scale s = {top, rate_of(t)};
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
__device__ __forceinline__ Whole join_chunks(const SampleArgs& a, int row, double rate) {
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
  const Scale s = {w.top, rate};
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
};
template <int kType, int kThreads>
__device__ __forceinline__ void draw_row(const SampleArgs& a, int row, Drawn& sh) {
  constexpr int kPer = Elem<kType>::kPer;
  const int tid = int(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const Row<kType> r(a, row);
  const float t = temperature_of(a, row);
  const double rate = rate_of(t);
  const SampleChunk* chunks = a.chunks + int64_t(row) * a.num_chunks;
  if (wave == 0) {
    const Whole w = join_chunks(a, row, rate);
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
        const Scale s = {w.top, rate};
        sh.top = w.top;
        sh.chunk_top = c.top;
        sh.total = w.total;
        sh.want = fmin((target - before) / s.weight(c.top), double(c.sum) - 1.0);
      }
      chunk = last;
    }
    if (lane == 0) sh.chunk = chunk;
  }
  __syncthreads();
  const int chunk = sh.chunk;
  if (chunk < 0) return;
  const Scale cs = {sh.chunk_top, rate};
  const double want = sh.want;
  // thread by thread in index order
  constexpr int kRun = kSampleChunk / kPer / kThreads;
  const int n = a.chunk / kPer, run = (n + kThreads - 1) / kThreads;
  uint64_t sum = 0;
#pragma unroll
  for (int j = 0; j < kRun; ++j) {
    const int q = tid * run + j;
    if (j >= run || q >= n) break;
    float x[kPer];
    r.load(chunk * n + q, x);
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum += cs.units(x[i]);
  }
  const uint64_t scan = wave_scan(sum);
  if (lane == 63) sh.waves[wave] = scan;
  __syncthreads();
  uint64_t at = scan - sum;
  for (int w = 0; w < wave; ++w) at += sh.waves[w];
  if (double(at) <= want && want < double(at + sum)) {
    for (int j = 0; j < run; ++j) {
      float x[kPer];
      r.load(chunk * n + tid * run + j, x);
      for (int i = 0; i < kPer; ++i) {
        at += cs.units(x[i]);
        if (double(at) > want) {
          finish(a, row, sh.top, sh.total, r.first(chunk * n + tid * run + j) + i, x[i], sh.total);
          return;
        }
      }
    }
  }
}

template <int kType>
__global__ __launch_bounds__(kDrawThreads) void sample_draw_kernel(SampleArgs a) {
  __shared__ Drawn sh;
  draw_row<kType, kDrawThreads>(a, int(blockIdx.x), sh);
}

// What a workgroup that looks for a threshold shares.
struct Shared {
  union {
    Drawn drawn;
    struct {
      uint64_t mass[kBins];
      uint32_t count[kBins];
    };
  };
  uint64_t list[kList];          // entries: key, then the complement of the index (falling order is the ranks')
  uint64_t wave_mass[kRowWaves];
  uint32_t wave_count[kRowWaves];
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

// Sum and count of the threads before this one in the workgroup (exclusive).
__device__ __forceinline__ void block_scan(Shared& sh, uint64_t mass, uint32_t count, uint64_t* mass_before, uint32_t* count_before) {
  const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
  const uint64_t m = wave_scan(mass);
  const uint32_t c = wave_scan(count);
  __syncthreads();
  if (lane == 63) {
    sh.wave_mass[wave] = m;
    sh.wave_count[wave] = c;
  }
  __syncthreads();
  uint64_t mb = m - mass;
  uint32_t cb = c - count;
  for (int w = 0; w < wave; ++w) {
    mb += sh.wave_mass[w];
    cb += sh.wave_count[w];
  }
  *mass_before = mb;
  *count_before = cb;
}

// Sorts list[0 .. n) into falling order (n <= kList; behind it, up to the next power of two, zeros). All threads.
__device__ __forceinline__ void sort_list(uint64_t* list, int n) {
  const int tid = int(threadIdx.x);
  int size = 64;
  while (size < n) size *= 2;
  for (int i = n + tid; i < size; i += kRowThreads) list[i] = 0;
  __syncthreads();
  for (int k = 2; k <= size; k *= 2)
    for (int j = k / 2; j > 0; j /= 2) {
      for (int p = tid; p < size / 2; p += kRowThreads) {
        const int lo = 2 * p - (p & (j - 1)), hi = lo + j;
        const uint64_t x = list[lo], y = list[hi];
        const bool falling = (lo & k) == 0;
        if (falling ? x < y : x > y) {
          list[lo] = y;
          list[hi] = x;
        }
      }
      __syncthreads();
    }
}

// Calls use(logit, index) for every entry of the row, from the thread that holds it: the waves take runs of the row.
template <int kType>
struct Runs {
  int begin, end;
  __device__ __forceinline__ explicit Runs(const Row<kType>& r) {
    const int wave = int(threadIdx.x) >> 6, per = (r.pieces + kRowWaves - 1) / kRowWaves;
    begin = wave * per;
    end = min(r.pieces, begin + per);
  }
};
template <int kType, class Use>
__device__ __forceinline__ void for_each(const Row<kType>& r, Use use) {
  constexpr int kPer = Elem<kType>::kPer, kDeep = 4;
  const Runs<kType> run(r);
  for (int p = run.begin + (int(threadIdx.x) & 63); p < run.end; p += 64 * kDeep) {
    float x[kDeep][kPer];
#pragma unroll
    for (int d = 0; d < kDeep; ++d) {
      if (p + 64 * d < run.end) r.load(p + 64 * d, x[d]);
    }
#pragma unroll
    for (int d = 0; d < kDeep; ++d) {
      if (p + 64 * d >= run.end) break;
#pragma unroll
      for (int i = 0; i < kPer; ++i) use(x[d][i], r.first(p + 64 * d) + i);
    }
  }
}

// Counts and sums by 2048 ranges of keys from lo on, each 2^shift wide.
template <int kType>
__device__ __forceinline__ void clear_bins(Shared& sh) {
  for (int b = int(threadIdx.x); b < kBins; b += kRowThreads) {
    sh.mass[b] = 0;
    sh.count[b] = 0;
  }
  if (threadIdx.x == 0) sh.bin = -1;
  __syncthreads();
}
__device__ __forceinline__ void add_to_bin(Shared& sh, int b, uint64_t units) {
  atomicAdd(&sh.count[b], 1u);
  atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[b]), (unsigned long long)(units));
}
// The bin, bins in falling order of logits, that completes the first `most` entries (most > 0), or at which the
// sum reaches `share` (most = 0); -1: none. above_*: of what lies before it.
__device__ __forceinline__ int crossing_bin(Shared& sh, uint32_t most, double share, uint32_t* above_count, uint64_t* above) {
  constexpr int kMine = kBins / kRowThreads;
  __syncthreads();
  const int b0 = kMine * int(threadIdx.x);
  uint64_t m[kMine], mass = 0;
  uint32_t c[kMine], count = 0;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    mass += m[i] = sh.mass[b0 + i];
    count += c[i] = sh.count[b0 + i];
  }
  uint64_t mb;
  uint32_t cb;
  block_scan(sh, mass, count, &mb, &cb);
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
  return bin;
}

// The cut by repeated refinement of key ranges (three times for 32 bits): for steps
// of the logit that hold more entries than the list.
template <int kType>
__device__ __forceinline__ Cut refine(Shared& sh, const Row<kType>& r, const Scale& s, uint32_t top_key, Cut within, uint32_t most, double share) {
  uint32_t lo = max(within.key, 1u), hi = top_key, above_count = 0;
  uint64_t above = 0;
  for (;;) {
    const uint32_t range = hi - lo;
    const int bits = range ? 32 - __builtin_clz(range) : 0;
    const int shift = max(0, bits - 11);
    clear_bins<kType>(sh);
    for_each(r, [&](float l, int) {
      const uint32_t key = key_of(l);
      if (key >= lo && key <= hi) add_to_bin(sh, int((hi - key) >> shift), s.units(l));
    });
    const int bin = crossing_bin(sh, most, share, &above_count, &above);
    if (bin < 0) {
      __syncthreads();
      return within;
    }
    const uint64_t mass = sh.mass[bin];
    const uint32_t count = sh.count[bin];
    __syncthreads();
    hi -= uint32_t(bin) << shift;
    if (shift == 0) {
      const uint64_t w = mass / count;
      uint32_t ties = count;
      if (most)
        ties = most - above_count;
      else if (w > 0)
        ties = uint32_t(fmin(double(count), ceil((share - double(above)) / double(w))));
      if (hi == within.key) ties = min(ties, within.ties);
      return {hi, ties, above + ties * w};
    }
    lo = hi - lo >= (1u << shift) ? hi - ((1u << shift) - 1u) : lo;
  }
}

// Steps of the logit from the row's largest down to the bound: rounding keeps the order.
struct Steps {
  float top, per;
  __device__ __forceinline__ int of(float l) const { return int(fminf((top - l) * per, float(kBins - 1))); }
};

// The cut by equal steps of the logit; the bins hold the row's counts and sums.
// The step in which it falls is sorted. *spoiled: the bins are gone.
template <int kType>
__device__ __forceinline__ Cut select(Shared& sh, const Row<kType>& r, const Scale& s, const Steps& steps, uint32_t top_key, float bound, Cut within,
                      uint32_t most, double share, bool* spoiled) {
  uint32_t above_count = 0;
  uint64_t above = 0;
  if (threadIdx.x == 0) {
    sh.bin = -1;
    sh.listed = 0;
    sh.found = -1;
  }
  const int bin = crossing_bin(sh, most, share, &above_count, &above);
  if (bin < 0) {
    __syncthreads();
    return within;
  }
  const uint32_t count = sh.count[bin];
  __syncthreads();
  if (count > kList) {
    *spoiled = true;
    return refine(sh, r, s, top_key, within, most, share);
  }
  for_each(r, [&](float l, int index) {
    if (l >= bound && l != kNone && steps.of(l) == bin) sh.list[atomicAdd(&sh.listed, 1u)] = entry_of(key_of(l), index);
  });
  __syncthreads();
  sort_list(sh.list, int(count));
  // positions of the list
  const int n = int(count), p0 = kPos * int(threadIdx.x);
  uint64_t w[kPos], sum = 0;
#pragma unroll
  for (int i = 0; i < kPos; ++i) {
    w[i] = p0 + i < n ? s.units(logit_of(key_of(sh.list[p0 + i]))) : 0;
    sum += w[i];
  }
  uint64_t before;
  uint32_t unused;
  block_scan(sh, sum, 0, &before, &unused);
  before += above;
#pragma unroll
  for (int i = 0; i < kPos; ++i) {
    const int p = p0 + i;
    const bool last = p < n && (most ? above_count + uint32_t(p) + 1 == most
                                     : double(before) < share && (double(before + w[i]) >= share || p + 1 == n));
    before += w[i];
    if (last && (most || atomicMax(&sh.found, p) < p)) {
      sh.found = p;
      sh.above_mass = before;
    }
  }
  __syncthreads();
  // entries equal to the last one that stays
  const int at = sh.found;
  const uint32_t key = key_of(sh.list[at]);
  uint32_t ties = 0;
#pragma unroll
  for (int i = 0; i < kPos; ++i) ties += p0 + i <= at && key_of(sh.list[p0 + i]) == key;
  uint64_t unused64;
  const uint64_t mass = sh.above_mass;
  block_scan(sh, 0, ties, &unused64, &unused);
  ties = 0;
  for (int v = 0; v < kRowWaves; ++v) ties += sh.wave_count[v];
  __syncthreads();
  return {key, ties, mass};
}

// (With 1024 threads, and so 128 registers, values that outlive a divergent block were
// stored to memory before its end, by the lanes still active alone.)
// One row with cuts. Bound: no entry below it stays, and none below it enters the sums that say which do.
//   top-k: the k-th largest of the groups' largest logits (k entries at least are no smaller);
//   top-p of everything: entries with less than (1 - p) of the whole's mean weight sum to less than (1 - p) of the whole;
//   min-p: its own limit, where no top-k has to sum what lies below.
template <int kType>
__global__ __launch_bounds__(kRowThreads) void sample_cut_kernel(SampleArgs a) {
  constexpr int kPer = Elem<kType>::kPer;
  __shared__ Shared sh;
  const int row = int(blockIdx.x), tid = int(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const float t = temperature_of(a, row);
  const int k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.f;
  const double low = a.min_p && a.min_p[row] > 0.f ? fmin(double(a.min_p[row]), 1.0) : 0.0;
  const bool cut_k = k > 0 && k < a.vocab, cut_p = p < 1.f;
  if (greedy(t) || (!cut_k && !cut_p && low == 0.0)) {
    draw_row<kType, kRowThreads>(a, row, sh.drawn);
    return;
  }
  const Row<kType> r(a, row);
  const double rate = rate_of(t);
  if (wave == 0) {
    const Whole w = join_chunks(a, row, rate);
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
  const Scale s = {top, rate};
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
      clear_bins<kType>(sh);
      for (int g = tid; g < num_groups; g += kRowThreads) {
        const uint32_t key = key_of(groups[g]);
        if (key >= lo && key <= hi) atomicAdd(&sh.count[(hi - key) >> shift], 1u);
      }
      const int bin = crossing_bin(sh, uint32_t(k), 0.0, &above_count, &above);
      __syncthreads();
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
  for (int g = tid; g < num_groups; g += kRowThreads) near += groups[g] >= bound;
  uint64_t unused64;
  uint32_t near_before;
  block_scan(sh, 0, near, &unused64, &near_before);
  uint32_t num_near = 0;
  for (int w = 0; w < kRowWaves; ++w) num_near += sh.wave_count[w];
  __syncthreads();
  if (num_near <= kBins) {
    uint32_t* const ids = sh.count;
    for (int g = tid; g < num_groups; g += kRowThreads)
      if (groups[g] >= bound) ids[near_before++] = uint32_t(g);
    __syncthreads();
    constexpr int kPieces = kGroup / kPer;
    for (uint32_t i = uint32_t(tid); i < num_near * kPieces; i += kRowThreads) {
      const int piece = int(ids[i / kPieces]) * kPieces + int(i % kPieces);
      float x[kPer];
      r.load(piece, x);
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (x[j] >= bound && x[j] != kNone) {
          const uint32_t at = atomicAdd(&sh.listed, 1u);
          if (at < kList) sh.list[at] = entry_of(key_of(x[j]), r.first(piece) + j);
        }
    }
    __syncthreads();
    const int n = int(sh.listed);
    if (n <= kList) {
      sort_list(sh.list, n);
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
      uint64_t before;
      uint32_t heavy_before;
      block_scan(sh, sum, heavy, &before, &heavy_before);
      int stays = 0;
      uint64_t list_sum = 0;
      for (int v = 0; v < kRowWaves; ++v) {
        stays += int(sh.wave_count[v]);
        list_sum += sh.wave_mass[v];
      }
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
      sort_list(sh.list, stays);
      sum = 0;
#pragma unroll
      for (int i = 0; i < kPos; ++i) {
        w[i] = p0 + i < stays ? s.units(logit_of(uint32_t(sh.list[p0 + i]))) : 0;
        sum += w[i];
      }
      uint32_t unused;
      block_scan(sh, sum, 0, &before, &unused);
      uint64_t kept = 0;
      for (int v = 0; v < kRowWaves; ++v) kept += sh.wave_mass[v];
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

  // the whole row again
  Cut cut = {0, 0, 0};   // nothing is cut: every key is above 0
  if (cut_k || cut_p) {
    const float span = top - bound;
    const Steps steps = {top, span > 0.f && span < __builtin_inff() ? float(kBins) / span : 0.f};
    auto fill = [&] {
      clear_bins<kType>(sh);
      for_each(r, [&](float l, int) {
        if (l >= bound && l != kNone) add_to_bin(sh, steps.of(l), s.units(l));
      });
      __syncthreads();
    };
    double whole = total;
    bool filled = false;
    for (int by_p = cut_k ? 0 : 1; by_p < (cut_p ? 2 : 1); ++by_p) {   // top-k, then top-p of what it leaves
      if (!filled) fill();
      filled = true;
      // no share lies before the first, so it always stays; entries behind the k-th do not reach the share
      bool spoiled = false;
      Cut next = select(sh, r, s, steps, top_key, bound, cut, by_p ? 0u : uint32_t(k), by_p ? fmax(double(p) * whole, 1.0) : 0.0, &spoiled);
      filled = !spoiled;
      if (next.key == cut.key) next.ties = min(next.ties, cut.ties);
      if (next.key) {
        cut = next;
        whole = double(cut.mass);
      }
    }
  }
  // what stays, wave by wave
  const Runs<kType> run(r);
  uint64_t sum = 0, tie_units = 0;
  uint32_t ties = 0;
  for_each(r, [&](float l, int) {
    const uint32_t key = key_of(l);
    if (key < cut.key || key == 0 || (low > 0.0 && s.weight(l) < low)) return;
    const uint64_t w = s.units(l);
    if (key > cut.key) {
      sum += w;
    } else {
      ++ties;
      tie_units = w;
    }
  });
  sum = wave_sum(sum);
  const uint32_t wave_ties = wave_sum(ties);
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const uint64_t y = shuffle_xor(tie_units, m);
    tie_units = tie_units > y ? tie_units : y;
  }
  __syncthreads();
  if (lane == 0) {
    sh.wave_mass[wave] = sum;
    sh.wave_count[wave] = wave_ties;
    sh.mass[wave] = tie_units;
  }
  __syncthreads();
  for (int w = 0; w < kRowWaves; ++w) tie_units = tie_units > sh.mass[w] ? tie_units : sh.mass[w];
  uint64_t kept = 0, before_me = 0, in_me = 0;
  uint32_t seen = 0, ties_before = 0;
  for (int w = 0; w < kRowWaves; ++w) {
    const uint32_t left = cut.ties > seen ? cut.ties - seen : 0;
    const uint64_t here = sh.wave_mass[w] + uint64_t(min(left, sh.wave_count[w])) * tie_units;
    if (w == wave) {
      before_me = kept;
      ties_before = seen;
      in_me = here;
    }
    kept += here;
    seen += sh.wave_count[w];
  }
  const double target = uniform_of(a, row) * double(kept);
  if (!(double(before_me) <= target && target < double(before_me + in_me))) return;
  // this wave's run holds the draw
  uint64_t cum = before_me;
  uint32_t tie = ties_before;
  for (int q0 = run.begin; q0 < run.end; q0 += 64) {
    float x[kPer];
    uint64_t w[kPer];
    uint32_t is_tie = 0, mine_ties = 0;
    const int q = q0 + lane;
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = kNone;
    if (q < run.end) r.load(q, x);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const uint32_t key = key_of(x[i]);
      const bool in = key >= cut.key && key != 0 && !(low > 0.0 && s.weight(x[i]) < low);
      w[i] = in ? s.units(x[i]) : 0;
      if (in && key == cut.key) {
        is_tie |= 1u << i;
        ++mine_ties;
      }
    }
    uint32_t rank = tie + wave_scan(mine_ties) - mine_ties;
    uint64_t lane_sum = 0;
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
        if (!was && double(at) > target) finish(a, row, top, total, r.first(q) + i, x[i], double(kept));
      }
    }
    cum += shuffle(scan, 63);
    tie += wave_sum(mine_ties);
    if (double(cum) > target) return;
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

template <int kType>
hipError_t launch(const SampleArgs& a, hipStream_t stream) {
  if (a.chunk == kSampleChunk)
    launch_chunks<kType, kSampleChunk>(a, stream);
  else
    launch_chunks<kType, kSampleSmallChunk>(a, stream);
  if (a.groups)
    hipLaunchKernelGGL(sample_cut_kernel<kType>, dim3(uint32_t(a.num_rows)), dim3(kRowThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(sample_draw_kernel<kType>, dim3(uint32_t(a.num_rows)), dim3(kDrawThreads), 0, stream, a);
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
