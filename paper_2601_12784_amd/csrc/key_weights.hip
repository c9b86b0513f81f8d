// Attention weights of cached keys, summed over the query rows that read them.
//
// A cache of bounded size keeps the keys that its queries attend to most. What
// it goes by is, for every cached key t of a (sequence, KV head),
//   w[t] += sum over rows (new token j, query head h of the group) with t <= P + j
//           of exp(scale q[j,h].K[t] - lse[j,h])
// with the rows' lse known from the attention that ran before. That is a score
// product without its P.V half, and the sum runs over rows, not keys, so the
// work is cut by keys: a wave keeps 64 keys (four pages) in registers as MFMA A
// operands and takes the rows 16 at a time,
//   S^T[16 keys][16 rows] = K Q^T    (D/32) v_mfma_f32_16x16x32_bf16 per page
//   w[key] += 2^(S^T c - lse2)       one fma, exp2 and add per score
// and no sum crosses waves: no atomics, the same bits on every run. A lane's
// partial sums (its row column) are joined once at the end, by a butterfly that
// halves the values at every step and leaves one key per lane.
//
// Two kernels. A decode step has one row tile per (sequence, KV head) and is
// bound by reading K once: key_weights_step_kernel holds the queries and streams
// the keys (long-tail batch, 704k tokens, 28/4 heads, D = 128, bf16: 124 us = 6.0 TB/s of
// a plain read's 6.85; fp8 73 us = 5.2 TB/s). Prompts, or their last rows, are bound by matrix and
// vector work: key_weights_rows_kernel holds the keys and streams the rows through LDS (every row of
// 32 long-tail prompts, 2.27 TFLOP: 2.44 ms = 0.93 PFLOP/s; the last 32 rows of 16
// prompts, fp8: 72 us). Counted per SIMD, 16 rows and 64 keys take 536 cycles: 16 MFMAs
// (256) and 63 vector instructions, 16 of them exponentials of two issue slots (316). The
// two hardly overlap. Work items, and the parts that long walks are cut into, are the host
// plan's; key_weights_merge_kernel adds the parts of a cut item in order.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sf_internal.h"

namespace sf {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(4))) const int32_t* const_i32_ptr;
typedef __attribute__((address_space(4))) const float* const_f32_ptr;

__device__ __forceinline__ const_i32_ptr as_constant(const int32_t* p) { return (const_i32_ptr)(p); }
__device__ __forceinline__ f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}
template <bool kHigh>
__device__ __forceinline__ uint32_t widen2(uint32_t codes4) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes4, 1.0f, kHigh));
}

constexpr int kWaves = 4;
constexpr int kTiles = kWeightPages;   // pages (16-key tiles) a wave holds
constexpr float kLog2e = 1.44269504088896340736f;

// Adds a key's sum to what it had, and gives a key that is weighed for the
// first time its position.
__device__ __forceinline__ void finish_key(const WeightArgs& a, const_i32_ptr row, int key, float sum) {
  const int len = row[7], held = row[10];
  if (key >= len) return;
  const int page = as_constant(a.block_table)[size_t(row[0]) * a.bt_stride + key / kPage];
  const size_t at = (size_t(page) * a.num_kv_heads + row[1]) * kPage + key % kPage;
  a.w_out[at] = (key < held ? a.w_in[at] : 0.f) + sum;
  if (a.positions && key >= held) a.positions[at] = row[11] + (key - held);
}

// 64 keys as they come from the pool: operands (bf16) or codes (fp8), and what
// turns each page's raw scores into log2 units.
template <int D, bool kFp8>
struct Keys {
  static constexpr int kPieces = kFp8 ? D / 64 : D / 32;
  u32x4 x[kTiles][kPieces];
  float c[kTiles];
  int page[kTiles];   // wave-uniform

  // Pages pg .. pg + 3 of the sequence (one at or past `end` repeats the first: its keys are not stored).
  __device__ __forceinline__ void load(const WeightArgs& a, const_i32_ptr bt, int kvh, int pg, int end, int lane) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      page[i] = bt[pg + i < end ? pg + i : pg];
      const size_t tile = size_t(page[i]) * a.num_kv_heads + kvh;
      // a piece is 1 KiB over the wave in either format
      const uint8_t* src = reinterpret_cast<const uint8_t*>(a.k_pool) + tile * size_t(kPieces * 1024) + lane * 16;
#pragma unroll
      for (int p = 0; p < kPieces; ++p)
        x[i][p] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + 1024 * p));
      c[i] = a.scale_log2;
      if constexpr (kFp8) c[i] *= ((const_f32_ptr)a.k_scale)[tile];
    }
  }
  // The A operand of page i for dims 32 kb .. + 31: codes are widened here (exact).
  __device__ __forceinline__ u32x4 operand(int i, int kb) const {
    if constexpr (!kFp8) return x[i][kb];
    const u32x4 w = x[i][kb / 2];
    const uint32_t lo = w[2 * (kb % 2)], hi = w[2 * (kb % 2) + 1];
    return u32x4{widen2<false>(lo), widen2<true>(lo), widen2<false>(hi), widen2<true>(hi)};
  }
};

// Sums over the 16 row columns: every step hands half of the values to the
// partner lane and keeps the other half, until lane (grp, col) holds that of
// the key 16 i + 4 grp + e, 4 i + e = col.
template <int kHalf>
__device__ __forceinline__ void join_half(float* v, int col) {
  const bool upper = (col & kHalf) != 0;
#pragma unroll
  for (int j = 0; j < kHalf; ++j) {
    const float keep = upper ? v[j + kHalf] : v[j];
    const float give = upper ? v[j] : v[j + kHalf];
    v[j] = keep + __shfl_xor(give, kHalf);
  }
}
__device__ __forceinline__ float join_columns(const f32x4* acc, int col) {
  float v[16];
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * i + e] = acc[i][e];
  join_half<8>(v, col);
  join_half<4>(v, col);
  join_half<2>(v, col);
  join_half<1>(v, col);
  return v[0];
}

// A row that is not there, or whose lse is not finite, adds nothing whatever its
// queries hold (their products may be NaN).
__device__ __forceinline__ bool row_counts(float lse, bool there) {
  return there && __builtin_fabsf(lse) < __builtin_inff();
}

// At most 16 rows per (sequence, KV head), bound by reading the keys: every wave
// streams an equal share of all keys, cut into segments of one (sequence, KV head)
// each, 64 keys at a time, the next 64 requested before these are used (16 KiB in
// flight per wave at D = 128, bf16; eight waves per CU). Queries, lse and the
// weights that the keys had come with them, so one segment runs into the next. Wave
// w starts with row w; a row names the one that follows it, which is requested with the
// segment's first keys: the list may lie in host memory. The results wait in LDS
// and are stored once the wave has no more keys or LDS is full: stored as they
// come, 64 bytes here and there in the middle of the read stream, they cost 21 us of the
// long-tail batch's 133 (0.72 GB of keys, 11 MB of weights). The stash is as large as two
// workgroups per CU allow, 39 blocks per wave: batches of 22 and 26 blocks per wave
// take the same with 24 (125 and 151 us), one of 65 takes 375 us against 384 (fp8 211, 218).
constexpr int kStashBlockBytes = kWaves * (64 * 8 + 4);   // a sum and a page per lane, a KV head
constexpr int kStash = (160 << 10) / 2 / kStashBlockBytes;

template <int D, bool kFp8>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void key_weights_step_kernel(WeightArgs a) {
  constexpr int KB = D / 32;
  const int lane = int(threadIdx.x) & 63;
  const int col = lane & 15;
  const int grp = lane >> 4;
  const int wave = int(blockIdx.x) * kWaves + __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  __shared__ float sum_lds[kWaves][kStash][64];
  __shared__ int page_lds[kWaves][kStash][64];   // -1: the lane has no key
  __shared__ int kvh_lds[kWaves][kStash];
  const int here = wave - int(blockIdx.x) * kWaves;
  if (wave >= a.steps) return;
  struct Segment {
    int seq, kvh, page, end, tokens, len, prefix, qrow, held, first_pos, next;
  };
  Segment seg;
  {
    const const_i32_ptr row = as_constant(a.items) + size_t(wave) * kWeightInts;
    seg = {row[0], row[1], row[2], row[3], row[5], row[7], row[8], row[9], row[10], row[11], row[12]};
  }
  int row_ints = 0;   // lane i: int i % 16 of the row that follows
  auto request_row = [&]() {
    row_ints = a.items[size_t(seg.next >= 0 ? seg.next : wave) * kWeightInts + col];
  };
  const int dt = int((uint32_t(col) * a.inv_group) >> 16);   // this lane's row: token, head of the group
  const int head = col - dt * a.group;
  // This lane's key of a block, after the sums are joined: slot 4 grp + col % 4 of page col / 4.
  const int my_tile = col >> 2, my_slot = 4 * grp + (col & 3);

  struct Block {
    Keys<D, kFp8> k;
    u32x4 q[KB];
    float lse, before;
    int page, end, tokens, len, prefix, held, first_pos, kvh;
  };
  auto page_of = [&](const Block& b) {
    return my_tile == 0 ? b.k.page[0] : my_tile == 1 ? b.k.page[1] : my_tile == 2 ? b.k.page[2] : b.k.page[3];
  };
  auto slot_of = [&](int page, int kvh) { return (size_t(page) * a.num_kv_heads + kvh) * kPage + my_slot; };
  int stashed = 0;
  auto flush = [&]() {
    for (int i = 0; i < stashed; ++i) {
      const int page = page_lds[here][i][lane];
      if (page >= 0) a.w_out[slot_of(page, kvh_lds[here][i])] = sum_lds[here][i][lane];
    }
    stashed = 0;
  };
  auto load = [&](Block& b) {
    b.k.load(a, as_constant(a.block_table) + size_t(seg.seq) * a.bt_stride, seg.kvh, seg.page, seg.end, lane);
    b.page = seg.page;
    b.end = seg.end;
    b.tokens = seg.tokens;
    b.len = seg.len;
    b.prefix = seg.prefix;
    b.held = seg.held;
    b.first_pos = seg.first_pos;
    b.kvh = seg.kvh;
    const bool ok = dt < seg.tokens;
    const size_t r = (size_t(seg.qrow) + size_t(ok ? dt : 0)) * a.num_q_heads + size_t(seg.kvh) * a.group + size_t(ok ? head : 0);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) b.q[kb] = *reinterpret_cast<const u32x4*>(a.q + r * D + 8 * grp + 32 * kb);
    b.lse = a.lse[r];
    b.before = a.w_in[slot_of(page_of(b), b.kvh)];   // for a page past the end: another's, unused
  };
  auto advance = [&]() {
    seg.page += kTiles;
    if (seg.page < seg.end) return true;
    if (seg.next < 0) return false;
    auto field = [&](int i) { return __builtin_amdgcn_readlane(row_ints, i); };
    seg = {field(0), field(1), field(2), field(3), field(5), field(7), field(8), field(9), field(10), field(11), field(12)};
    request_row();
    return true;
  };
  auto weigh = [&](const Block& b) {
    f32x4 s[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < kTiles; ++i) s[i] = mfma_bf16(b.k.operand(i, kb), b.q[kb], s[i]);
    const float lse2 = b.lse * kLog2e;
    const int limit = row_counts(b.lse, dt < b.tokens) ? b.prefix + dt : -1;
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][e], b.k.c[i], -lse2));
        s[i][e] = (b.page + i) * kPage + 4 * grp + e <= limit ? p : 0.f;
      }
    const float sum = join_columns(s, col);
    const int key = (b.page + my_tile) * kPage + my_slot;
    const bool there = b.page + my_tile < b.end && key < b.len;
    if (stashed == kStash) flush();
    sum_lds[here][stashed][lane] = (key < b.held ? b.before : 0.f) + sum;
    page_lds[here][stashed][lane] = there ? page_of(b) : -1;
    if (lane == 0) kvh_lds[here][stashed] = b.kvh;
    ++stashed;
    if (a.positions && there && key >= b.held) a.positions[slot_of(page_of(b), b.kvh)] = b.first_pos + (key - b.held);
  };
  Block even, odd;
  load(even);
  request_row();
  while (true) {
    if (!advance()) {
      weigh(even);
      break;
    }
    load(odd);
    weigh(even);
    if (!advance()) {
      weigh(odd);
      break;
    }
    load(even);
    weigh(odd);
  }
  flush();
}

// Any number of rows: an item's 256 keys (64 per wave) stay in registers, its
// rows pass through LDS 64 at a time, double buffered, one barrier per 64. Each
// wave fetches one of a block's four row tiles into registers while the block
// before is computed, in the operand's own order (lane (grp, col): dims 8 grp ..
// of row col), so writing and reading LDS are whole 1 KiB rows without conflicts.
// Three waves per SIMD and a plain loop: two waves with the next tile's products issued
// ahead by hand took 2.44 ms on the prompts above, four waves spill.
constexpr int kBlockTiles = kWaves;
constexpr int kBlockRows = 16 * kBlockTiles;

template <int D, bool kFp8>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(3, 3))) void key_weights_rows_kernel(WeightArgs a) {
  constexpr int KB = D / 32;
  __shared__ u32x4 q_lds[2][kBlockTiles][KB][64];
  __shared__ float lse_lds[2][kBlockRows];
  __shared__ int limit_lds[2][kBlockRows];
  const const_i32_ptr row = as_constant(a.items) + size_t(blockIdx.x) * kWeightInts;
  const int seq = row[0], kvh = row[1], page_begin = row[2], page_end = row[3], tok_begin = row[4], tok_end = row[5];
  const int slot = row[6], prefix = row[8], qrow0 = row[9];
  const int lane = int(threadIdx.x) & 63;
  const int col = lane & 15;
  const int grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int g = a.group;
  const const_i32_ptr bt = as_constant(a.block_table) + size_t(seq) * a.bt_stride;
  const int pg = page_begin + wave * kTiles;
  const bool mine = pg < page_end;

  // operands of this wave's keys (codes are widened once)
  u32x4 k[kTiles][KB];
  float c[kTiles];
  {
    Keys<D, kFp8> raw;
    raw.load(a, bt, kvh, mine ? pg : page_begin, page_end, lane);
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      c[i] = raw.c[i];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) k[i][kb] = raw.operand(i, kb);
    }
  }

  // The row this lane fetches: row 16 wave + col of a block, by (token, head).
  const int rows = (tok_end - tok_begin) * g;
  const int blocks = (rows + kBlockRows - 1) / kBlockRows;
  int tok = tok_begin + (16 * wave + col) / g;
  int head = (16 * wave + col) % g;
  const int tok_step = kBlockRows / g, head_step = kBlockRows % g;
  u32x4 pre[KB];
  float pre_lse;   // as loaded: whatever looked at it here would wait for the loads before it
  bool pre_ok;
  int pre_limit;
  auto fetch = [&]() {
    const bool ok = tok < tok_end;
    const size_t r = (size_t(qrow0) + size_t(ok ? tok : tok_begin)) * a.num_q_heads + size_t(kvh) * g + size_t(ok ? head : 0);
    const uint16_t* src = a.q + r * D + 8 * grp;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) pre[kb] = *reinterpret_cast<const u32x4*>(src + 32 * kb);
    pre_lse = a.lse[r];
    pre_ok = ok;
    pre_limit = prefix + tok;
    tok += tok_step;
    head += head_step;
    if (head >= g) {
      head -= g;
      ++tok;
    }
  };
  // A row that does not count has queries 0 and lse +inf: its weights are 0. A mask by its
  // lse in the loop below took 7 to 11 % longer.
  auto put = [&](int buffer) {
    const bool counts = row_counts(pre_lse, pre_ok);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) q_lds[buffer][wave][kb][lane] = counts ? pre[kb] : u32x4{0, 0, 0, 0};
    if (grp == 0) {
      lse_lds[buffer][16 * wave + col] = counts ? pre_lse * kLog2e : __builtin_inff();
      limit_lds[buffer][16 * wave + col] = pre_limit;
    }
  };

  f32x4 acc[kTiles];
#pragma unroll
  for (int i = 0; i < kTiles; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int key0 = pg * kPage;
  // Rows (of the item) before `blind` see none of the wave's keys, from `clear` on all of them.
  const int64_t before = int64_t(key0) - prefix - tok_begin;
  const int blind = int(min(max(before * g, int64_t(0)), int64_t(rows)));
  const int clear = int(min(max((before + kTiles * kPage - 1) * g, int64_t(0)), int64_t(rows)));
  auto block = [&](int buffer, int row0) {
#pragma unroll 1
    for (int t = 0; t < kBlockTiles; ++t) {
      const int r0 = row0 + 16 * t;
      if (r0 >= rows || r0 + 15 < blind) continue;
      f32x4 s[kTiles];
#pragma unroll
      for (int i = 0; i < kTiles; ++i) s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const u32x4 q = q_lds[buffer][t][kb][lane];
#pragma unroll
        for (int i = 0; i < kTiles; ++i) s[i] = mfma_bf16(k[i][kb], q, s[i]);
      }
      const float lse2 = lse_lds[buffer][16 * t + col];
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][e], c[i], -lse2));
      if (r0 < clear) {
        const int limit = limit_lds[buffer][16 * t + col];
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[i][e] = key0 + kPage * i + 4 * grp + e <= limit ? s[i][e] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][e] += s[i][e];
    }
  };
  fetch();
  put(0);
  // Every load so far has come: without this the first use of the keys, in the
  // loop, would wait for the rows just requested.
  __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
  __syncthreads();
  for (int b = 0; b < blocks; ++b) {
    if (b + 1 < blocks) fetch();
    if (mine) block(b & 1, b * kBlockRows);
    if (b + 1 < blocks) put((b + 1) & 1);
    __syncthreads();
  }

  const float sum = join_columns(acc, col);
  const int key = key0 + kPage * (col >> 2) + 4 * grp + (col & 3);
  if (pg + (col >> 2) >= page_end) return;
  if (slot >= 0)
    a.part[size_t(slot) * a.part_keys + (key - page_begin * kPage)] = sum;
  else
    finish_key(a, row, key, sum);
}

// Adds the parts of a cut item, in order: a thread per key.
__global__ __launch_bounds__(256) void key_weights_merge_kernel(WeightArgs a) {
  const const_i32_ptr row = as_constant(a.merge_rows) + size_t(blockIdx.x) * kWeightInts;
  const int page_begin = row[2];
  const int keys = (row[3] - page_begin) * kPage;
  const int first = row[4];
  const int n = row[5];
  for (int i = threadIdx.x; i < keys; i += 256) {
    float sum = 0.f;
    for (int p = 0; p < n; ++p) sum += a.part[size_t(first + p) * a.part_keys + i];
    finish_key(a, row, page_begin * kPage + i, sum);
  }
}

template <int D>
void (*pick_kernel(const WeightArgs& a))(WeightArgs) {
  if (a.steps) return a.k_scale ? key_weights_step_kernel<D, true> : key_weights_step_kernel<D, false>;
  return a.k_scale ? key_weights_rows_kernel<D, true> : key_weights_rows_kernel<D, false>;
}

}  // namespace

hipError_t launch_key_weights(const WeightArgs& a, hipStream_t stream) {
  if (a.num_items == 0) return hipSuccess;
  const dim3 grid(a.steps ? (a.steps + kWaves - 1) / kWaves : a.num_items), block(64 * kWaves);
  void (*kernel)(WeightArgs) = a.head_dim == 128 ? pick_kernel<128>(a) : pick_kernel<64>(a);
  hipLaunchKernelGGL(kernel, grid, block, 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.num_merge == 0) return e;
  hipLaunchKernelGGL(key_weights_merge_kernel, dim3(a.num_merge), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sf
