// Sampling with temperature, top-k, top-p and min-p from given uniform numbers.
//
// Each row asks which index a running sum crosses a share of the whole at, and
// the answer must not depend on the order of the sums: weights are rounded to
// multiples of 2^-44 of the largest (fp64 arithmetic, which runs at the rate of unpacked fp32 here) and
// added as integers, by atomics too.
//
// Two launches. The first reads the logits once, a chunk per workgroup: the
// chunk's largest logit and the sum of its weights relative to it. The second, a
// workgroup per row, joins the chunks' sums. Without cuts it then knows the
// chunk of the drawn index, and reads that chunk again. With cuts it
// looks for the logit at which they fall: the kept entries are the first ones in
// the order of falling logits, so one threshold (an order-preserving integer key)
// and a number of entries equal to it describe them. The threshold comes from
// histograms of counts and weights over 2048 key ranges, refined until a range
// is one key (three times for 32 bits).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sf_internal.h"

namespace sf {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kChunkThreads = 256;
constexpr int kRowThreads = 1024;
constexpr int kRowWaves = kRowThreads / 64;
constexpr int kBins = 2048;
constexpr int kUnitBits = 44;
constexpr double kUnit = 0x1p-44;
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

// 2^y for y <= 0: the Taylor series of 2^f to f^11, |f| <= 1/2 (the next term is below 2^-47).
__device__ __forceinline__ double exp2_of(double y, int shift = 0) {
  constexpr double kC[12] = {1.0,
                             0.69314718055994530942,
                             0.24022650695910071233,
                             0.05550410866482157995,
                             0.00961812910762847716,
                             0.00133335581464284434,
                             0.00015403530393381610,
                             1.5252733804059840280e-5,
                             1.3215486790144309488e-6,
                             1.0178086009239699728e-7,
                             7.0549116208011233299e-9,
                             4.4455382718708114976e-10};
  const double n = __builtin_rint(y), f = y - n;
  double p = kC[11];
#pragma unroll
  for (int i = 10; i >= 0; --i) p = __builtin_fma(p, f, kC[i]);
  return __builtin_ldexp(p, int(n) + shift);
}

// Weights of logits relative to a largest one: exp((l - top) / T), 1 / T ln 2 in rate.
struct Scale {
  float top;
  double rate;
  __device__ __forceinline__ double exponent(float l) const { return (double(l) - double(top)) * rate; }
  // In units of 2^-44, rounded.
  __device__ __forceinline__ uint64_t units(float l) const {
    if (top == __builtin_inff() || l == top) return l == top ? uint64_t(1) << kUnitBits : 0;
    if (l == kNone) return 0;
    const double y = exponent(l);
    if (!(y > -46.0)) return 0;
    const double w = exp2_of(y, kUnitBits) + 0x1p52;   // the sum's last bit is one unit
    return __builtin_bit_cast(uint64_t, w) & ((uint64_t(1) << 52) - 1);
  }
  __device__ __forceinline__ double weight(float l) const {
    if (top == __builtin_inff() || l == top) return l == top ? 1.0 : 0.0;
    if (l == kNone) return 0.0;
    const double y = exponent(l);
    return y > -1000.0 ? exp2_of(y) : 0.0;
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

__device__ __forceinline__ uint64_t shuffle_xor(uint64_t x, int m) {
  return uint64_t(uint32_t(__shfl_xor(int(uint32_t(x)), m))) | uint64_t(uint32_t(__shfl_xor(int(uint32_t(x >> 32)), m))) << 32;
}
__device__ __forceinline__ uint64_t shuffle_up(uint64_t x, int n) {
  return uint64_t(uint32_t(__shfl_up(int(uint32_t(x)), n))) | uint64_t(uint32_t(__shfl_up(int(uint32_t(x >> 32)), n))) << 32;
}
template <class T>
__device__ __forceinline__ T wave_sum(T x);
template <>
__device__ __forceinline__ uint64_t wave_sum(uint64_t x) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) x += shuffle_xor(x, m);
  return x;
}
template <>
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

template <int kType, int kChunk>
__global__ __launch_bounds__(kChunkThreads) void sample_chunk_kernel(SampleArgs a) {
  constexpr int kPer = Elem<kType>::kPer;
  constexpr int kPieces = kChunk / kPer / kChunkThreads;   // of a thread
  constexpr int kWaves = kChunkThreads / 64;
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
  for (int j = 0; j < kPieces; ++j)
#pragma unroll
    for (int i = 0; i < kPer; ++i) top = fmaxf(top, x[j][i]);
#pragma unroll
  for (int m = 1; m < 64; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, tops[w]);
  int at = INT32_MAX;
  uint64_t sum = 0;
  if (top != kNone) {
    const float t = temperature_of(a, row);
    const Scale s = {top, rate_of(t)};
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        sum += s.units(x[j][i]);
        if (x[j][i] == top) at = min(at, r.first(p0 + j * kChunkThreads) + i);
      }
  }
  sum = wave_sum(sum);
#pragma unroll
  for (int m = 1; m < 64; m *= 2) at = min(at, __shfl_xor(at, m));
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

// What a workgroup of the second launch shares.
struct Shared {
  uint64_t mass[kBins];
  uint32_t count[kBins];
  uint64_t wave_mass[kRowWaves];
  uint32_t wave_count[kRowWaves];
  double wave_part[kRowWaves];
  float wave_top[kRowWaves];
  // found by one thread
  int bin;
  uint32_t above_count;
  uint64_t above_mass;
  double before;
};

// The entries that stay: keys above `key`, and the first `ties` of those equal to it.
struct Cut {
  uint32_t key;
  uint32_t ties;
  uint64_t mass;     // sum of what stays
};

// Sum and count of the lanes before this one in the workgroup (exclusive).
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

// The entry that completes the first `most` ones (most > 0), or before which, of all
// with keys >= floor, at least `share` lies (most = 0). Returns no cut if there is none.
template <int kType>
__device__ Cut select(Shared& sh, const Row<kType>& r, const Scale& s, uint32_t top_key, Cut within, uint32_t most, double share) {
  const int tid = int(threadIdx.x), wave = tid >> 6, lane = tid & 63;
  const int per_wave = (r.pieces + kRowWaves - 1) / kRowWaves;
  uint32_t lo = max(within.key, 1u), hi = top_key, above_count = 0;
  uint64_t above = 0;
  for (;;) {
    const uint32_t range = hi - lo;
    const int bits = range ? 32 - __builtin_clz(range) : 0;
    const int shift = max(0, bits - 11);
    for (int b = tid; b < kBins; b += kRowThreads) {
      sh.mass[b] = 0;
      sh.count[b] = 0;
    }
    if (tid == 0) sh.bin = -1;
    __syncthreads();
    const int end = min(r.pieces, (wave + 1) * per_wave);
    for (int p = wave * per_wave + lane; p < end; p += 64) {
      float x[Elem<kType>::kPer];
      r.load(p, x);
#pragma unroll
      for (int i = 0; i < Elem<kType>::kPer; ++i) {
        const uint32_t key = key_of(x[i]);
        if (key < lo || key > hi) continue;
        const int b = int((key - lo) >> shift);
        atomicAdd(&sh.count[b], 1u);
        atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[b]), (unsigned long long)(s.units(x[i])));
      }
    }
    __syncthreads();
    // from the top: thread t takes bins kBins - 1 - 2t and the one below
    const int b1 = kBins - 1 - 2 * tid, b0 = b1 - 1;
    const uint64_t m1 = sh.mass[b1], m0 = sh.mass[b0];
    const uint32_t c1 = sh.count[b1], c0 = sh.count[b0];
    uint64_t mb;
    uint32_t cb;
    block_scan(sh, m1 + m0, c1 + c0, &mb, &cb);
    mb += above;
    cb += above_count;
    auto crosses = [&](uint64_t m_before, uint32_t c_before, uint64_t m, uint32_t c) {
      if (most) return c_before < most && c_before + c >= most;
      return c > 0 && double(m_before) < share && double(m_before + m) >= share;
    };
    if (crosses(mb, cb, m1, c1)) {
      sh.bin = b1;
      sh.above_count = cb;
      sh.above_mass = mb;
    } else if (crosses(mb + m1, cb + c1, m0, c0)) {
      sh.bin = b0;
      sh.above_count = cb + c1;
      sh.above_mass = mb + m1;
    }
    __syncthreads();
    const int bin = sh.bin;
    above_count = sh.above_count;
    above = sh.above_mass;
    if (bin < 0) {
      __syncthreads();
      return within;
    }
    const uint64_t mass = sh.mass[bin];
    const uint32_t count = sh.count[bin];
    __syncthreads();
    lo += uint32_t(bin) << shift;
    if (shift == 0) {
      const uint64_t w = mass / count;
      uint32_t ties = count;
      if (most)
        ties = most - above_count;
      else if (w > 0)
        ties = uint32_t(fmin(double(count), ceil((share - double(above)) / double(w))));
      if (lo == within.key) ties = min(ties, within.ties);
      return {lo, ties, above + ties * w};
    }
    hi = min(hi, lo + ((1u << shift) - 1u));
  }
}

// One row. The chunks' sums are joined; with cuts, the threshold is looked for;
// then the waves, each over its own run of the row, sum what stays, and the one
// in whose run the draw falls walks it.
template <int kType>
__global__ __launch_bounds__(kRowThreads) void sample_row_kernel(SampleArgs a) {
  constexpr int kPer = Elem<kType>::kPer;
  __shared__ Shared sh;
  const int row = int(blockIdx.x), tid = int(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const Row<kType> r(a, row);
  const float t = temperature_of(a, row);
  const double rate = rate_of(t);
  const SampleChunk* chunks = a.chunks + int64_t(row) * a.num_chunks;
  const SampleChunk mine = tid < a.num_chunks ? chunks[tid] : SampleChunk{kNone, 0, 0};
  float top = mine.top;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
  if (lane == 0) sh.wave_top[wave] = top;
  __syncthreads();
  for (int w = 0; w < kRowWaves; ++w) top = fmaxf(top, sh.wave_top[w]);
  if (top == kNone) {
    if (tid == 0) {
      a.token[row] = -1;
      if (a.logprob) a.logprob[row] = kNone;
      if (a.kept) a.kept[row] = 0.f;
    }
    return;
  }
  const Scale s = {top, rate};
  // the chunk's sum relative to the row's largest logit, and the sums before it
  const double part = mine.top == kNone ? 0.0 : double(mine.sum) * s.weight(mine.top);
  double scan = part;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const double y = __shfl_up(scan, m);
    scan += lane >= m ? y : 0.0;
  }
  if (lane == 63) sh.wave_part[wave] = scan;
  __syncthreads();
  double total = 0.0, before = scan - part;
  for (int w = 0; w < kRowWaves; ++w) {
    if (w == wave) before += total;
    total += sh.wave_part[w];
  }
  auto finish = [&](int token, float l, double kept) {
    a.token[row] = token;
    const double y = top == __builtin_inff() ? 0.0 : (double(l) - double(top)) / (greedy(t) ? 1.0 : double(t));
    if (a.logprob) a.logprob[row] = float(y - log(total * kUnit));
    if (a.kept) a.kept[row] = float(kept / total);
  };
  if (greedy(t)) {
    int at = mine.top == top ? mine.at : INT32_MAX;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) at = min(at, __shfl_xor(at, m));
    if (lane == 0) sh.wave_count[wave] = uint32_t(at);
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kRowWaves; ++w) at = min(at, int(sh.wave_count[w]));
      finish(at, top, 0x1p44);
    }
    return;
  }
  const float u0 = a.uniform[row];
  const double u = u0 > 0.f ? fmin(double(u0), 1.0 - 0x1p-24) : 0.0;
  const int k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.f;
  const double low = a.min_p && a.min_p[row] > 0.f ? fmin(double(a.min_p[row]), 1.0) : 0.0;
  const bool cut_k = k > 0 && k < a.vocab, cut_p = p < 1.f;

  if (!cut_k && !cut_p && low == 0.0) {
    // the last chunk before which no more than the draw's share lies
    const double target = u * total;
    if (tid == 0) sh.bin = -1;
    __syncthreads();
    if (part > 0.0 && before <= target) atomicMax(&sh.bin, tid);
    __syncthreads();
    if (sh.bin == tid) sh.before = before;
    __syncthreads();
    const int chunk = sh.bin;
    const SampleChunk c = chunks[chunk];
    const Scale cs = {c.top, rate};
    const double want = fmin((target - sh.before) / s.weight(c.top), double(c.sum) - 1.0);
    // thread by thread in index order, kRun pieces each
    const int n = a.chunk / kPer, run = (n + kRowThreads - 1) / kRowThreads;
    uint64_t sum = 0;
    for (int j = 0; j < run; ++j) {
      const int q = tid * run + j;
      if (q >= n) break;
      float x[kPer];
      r.load(chunk * n + q, x);
#pragma unroll
      for (int i = 0; i < kPer; ++i) sum += cs.units(x[i]);
    }
    uint64_t mb;
    uint32_t unused;
    block_scan(sh, sum, 0, &mb, &unused);
    if (double(mb) <= want && want < double(mb + sum)) {
      for (int j = 0; j < run; ++j) {
        float x[kPer];
        r.load(chunk * n + tid * run + j, x);
        for (int i = 0; i < kPer; ++i) {
          mb += cs.units(x[i]);
          if (double(mb) > want) {
            finish(r.first(chunk * n + tid * run + j) + i, x[i], total);
            return;
          }
        }
      }
    }
    return;
  }

  const uint32_t top_key = key_of(top);
  Cut cut = {0, 0, 0};   // nothing is cut: every key is above 0
  double whole = total;
  if (cut_k) {
    cut = select<kType>(sh, r, s, top_key, cut, uint32_t(k), 0.0);
    if (cut.key) whole = double(cut.mass);
  }
  if (cut_p) {
    // no share lies before the first, so it always stays
    const double share = fmax(double(p) * whole, 1.0);
    cut = select<kType>(sh, r, s, top_key, cut, 0, share);
  }
  // what stays, wave by wave
  const int per_wave = (r.pieces + kRowWaves - 1) / kRowWaves;
  const int begin = wave * per_wave, end = min(r.pieces, begin + per_wave);
  uint64_t sum = 0, tie_units = 0;
  uint32_t ties = 0;
  for (int q = begin + lane; q < end; q += 64) {
    float x[kPer];
    r.load(q, x);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const uint32_t key = key_of(x[i]);
      if (key < cut.key || key == 0) continue;
      if (low > 0.0 && s.weight(x[i]) < low) continue;
      if (key > cut.key) {
        sum += s.units(x[i]);
      } else {
        ++ties;
        tie_units = s.units(x[i]);
      }
    }
  }
  sum = wave_sum(sum);
  const uint32_t wave_ties = wave_sum(ties);
#pragma unroll
  for (int m = 1; m < 64; m *= 2) tie_units = max(tie_units, shuffle_xor(tie_units, m));
  __syncthreads();
  if (lane == 0) {
    sh.wave_mass[wave] = sum;
    sh.wave_count[wave] = wave_ties;
    sh.mass[wave] = tie_units;
  }
  __syncthreads();
  for (int w = 0; w < kRowWaves; ++w) tie_units = max(tie_units, sh.mass[w]);
  uint64_t kept = 0, before_me = 0;
  uint32_t seen = 0, ties_before = 0;
  uint64_t in_me = 0;
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
  const double target = u * double(kept);
  if (!(double(before_me) <= target && target < double(before_me + in_me))) return;
  // this wave's run holds the draw
  uint64_t cum = before_me;
  uint32_t tie = ties_before;
  for (int q0 = begin; q0 < end; q0 += 64) {
    float x[kPer];
    uint64_t w[kPer];
    uint32_t is_tie = 0, mine_ties = 0;
    const int q = q0 + lane;
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = kNone;
    if (q < end) r.load(q, x);
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
    const uint64_t scan_sum = wave_scan(lane_sum);
    uint64_t at = cum + scan_sum - lane_sum;
    if (double(at) <= target && target < double(at + lane_sum)) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const bool was = double(at) > target;
        at += w[i];
        if (!was && double(at) > target) finish(r.first(q) + i, x[i], double(kept));
      }
    }
    const int last = 63;
    cum += uint64_t(uint32_t(__shfl(int(uint32_t(scan_sum)), last))) | uint64_t(uint32_t(__shfl(int(uint32_t(scan_sum >> 32)), last))) << 32;
    tie += wave_sum(mine_ties);
    if (double(cum) > target) return;
  }
}

template <int kType>
hipError_t launch(const SampleArgs& a, hipStream_t stream) {
  const dim3 grid{uint32_t(a.num_rows) * uint32_t(a.num_chunks), 1, 1};
  if (a.chunk == kSampleChunk)
    hipLaunchKernelGGL((sample_chunk_kernel<kType, kSampleChunk>), grid, dim3(kChunkThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((sample_chunk_kernel<kType, kSampleSmallChunk>), grid, dim3(kChunkThreads), 0, stream, a);
  hipLaunchKernelGGL(sample_row_kernel<kType>, dim3(uint32_t(a.num_rows)), dim3(kRowThreads), 0, stream, a);
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
