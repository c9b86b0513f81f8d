// Eviction from a paged cache by accumulated attention weight.
//
// Each (sequence, KV head) keeps n of its L cached keys. Softmax attention does
// not depend on the order of its keys (their positions are in the keys), so
// nothing is compacted: a kept key in the first n slots stays where it is, and
// the i-th kept key behind them moves into the i-th freed slot. That moves at
// most min(n, L - n) tokens, for a cache that gives up a page at a time 16 of
// n, where keeping the order would move nearly all of them; and in an 8-bit
// cache a token is rounded again only when it moves. The positions array keeps
// what the slot no longer says.
//
// Selection, one workgroup per (sequence, KV head), a thread per page: the n-th
// largest key of (weight, lowest slot first) by four passes of 8 bits over the
// weights' order-preserving integers, then for every page of the first n slots
// the freed slots' mask and number, and the list of kept slots behind. Bound by
// latency: 14 us for 64 sequences of 2112 tokens, 20 + 27 us for the long-tail batch
// (256 sequences, up to 16384 tokens; four KV heads each). Sixteen copies of the counters
// took as long.
// Moves, a wave per (page, KV head, keys or values) of the first n slots:
// gathers its page's new tokens. Bound by memory at tile granularity; a bf16 value tile is
// dim-major, so a token's values are 2 bytes of D 32-byte rows, and a page with
// one freed slot reads and writes its whole tile: the long-tail batch halved takes
// 450 us for 2.2 GB of tiles (0.72 GB of tokens); 64 sequences of 2112 fp8 tokens cut to
// 2048, at one or two tokens per tile and most of them with none, 27 us, of which waves wait more than
// half (full stores of their tiles 33).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fp8_tile.h"
#include "sf_internal.h"

namespace sf {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x8 __attribute__((ext_vector_type(8), aligned(16)));
typedef __attribute__((address_space(4))) const int32_t* const_i32_ptr;
__device__ __forceinline__ const_i32_ptr as_constant(const int32_t* p) { return (const_i32_ptr)(p); }

// Sequence row of the work list: L, n, first page of the moves' masks, first
// entry of the moves' sources (both of KV head 0), end (next position), sequence, 0, 0;
// the long sequences first
constexpr int kRowInts = kItemInts;

template <int kThreads>
struct BlockScan {
  int32_t wave_sum[kThreads / 64];
};

// Exclusive prefix sum of x over the workgroup's threads, and the total.
template <int kThreads>
__device__ __forceinline__ int block_scan(int x, BlockScan<kThreads>& lds, int& total) {
  const int lane = int(threadIdx.x) & 63;
  const int wave = int(threadIdx.x) >> 6;
  int incl = x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int y = __shfl_up(incl, off);
    if (lane >= off) incl += y;
  }
  __syncthreads();   // the sums of the scan before have been read
  if (lane == 63) lds.wave_sum[wave] = incl;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) before += lds.wave_sum[w];
    total += lds.wave_sum[w];
  }
  return before + incl - x;
}

// Integers in the order of the weights: a protected position above all, NaN below all.
__device__ __forceinline__ uint32_t rank_key(float w, int pos, int sinks, int recent_from) {
  if (pos < sinks || pos >= recent_from) return 0xFFFFFFFFu;
  if (w != w) return 0u;
  const uint32_t b = __builtin_bit_cast(uint32_t, w + 0.f);   // -0 is 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

constexpr int kSelectShort = kEvictLong / kPage, kSelectLong = 1024;   // threads

template <int kThreads>
__global__ __launch_bounds__(kThreads) void evict_select_kernel(EvictArgs a) {
  __shared__ int32_t hist[256];
  __shared__ int32_t found[2];
  __shared__ BlockScan<kThreads> scan;
  // Side job: the rows to device memory, 16 bytes per thread and turn, requested
  // before and stored after all else.
  const i32x4* copy_src = reinterpret_cast<const i32x4*>(a.rows);
  i32x4* copy_dst = reinterpret_cast<i32x4*>(a.late_rows);
  const int copies = a.late_rows ? (a.num_seqs + a.num_moves) * (kRowInts / 4) : 0;
  int64_t copy_at = int64_t(blockIdx.x) * kThreads + int(threadIdx.x);
  const i32x4 copied = copy_src[copy_at < copies ? copy_at : 0];
  auto finish = [&]() {
    if (copy_at < copies) copy_dst[copy_at] = copied;
    const int64_t stride = int64_t(gridDim.x) * kThreads;
    for (copy_at += stride; copy_at < copies; copy_at += stride) copy_dst[copy_at] = copy_src[copy_at];
  };
  const int kvh = int(blockIdx.x) % a.num_kv_heads;
  const const_i32_ptr row =
      as_constant(a.rows) + size_t((kThreads == kSelectLong ? 0 : a.num_long) + int(blockIdx.x) / a.num_kv_heads) * kRowInts;
  const int len = row[0];
  const int n = row[1];
  const int seq = row[5];
  if (n == 0) return finish();
  const int keep_pages = (n + kPage - 1) / kPage;
  uint32_t* holes = a.holes + 2 * (size_t(row[2]) + size_t(kvh) * keep_pages);
  const int tid = int(threadIdx.x);
  if (n == len) {   // nothing to give up
    for (int p = tid; p < keep_pages; p += kThreads) holes[2 * p] = holes[2 * p + 1] = 0;
    return finish();
  }
  int32_t* tails = a.tails + size_t(row[3]) + size_t(kvh) * min(n, len - n);
  const int recent_from = a.recent > 0 ? row[4] - a.recent : INT32_MAX;
  const int pages = (len + kPage - 1) / kPage;
  const const_i32_ptr bt = as_constant(a.block_table) + size_t(seq) * a.bt_stride;

  // The 16 keys of page p (0 past the end of the sequence: counted nowhere).
  auto load = [&](int p, uint32_t* key) {
    const size_t at = (size_t(bt[p]) * a.num_kv_heads + kvh) * kPage;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 w = *reinterpret_cast<const f32x4*>(a.w_in + at + 4 * q);
      const i32x4 pos = *reinterpret_cast<const i32x4*>(a.pos_in + at + 4 * q);
#pragma unroll
      for (int e = 0; e < 4; ++e) key[4 * q + e] = rank_key(w[e], pos[e], a.sinks, recent_from);
    }
  };
  uint32_t cached[kPage];   // of this thread's first page
  if (tid < pages) load(tid, cached);

  // The n-th largest key, 8 bits at a time from the top.
  uint32_t prefix = 0;
  int want = n;   // keys still to be found among those with this prefix
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int p = tid; p < pages; p += kThreads) {
      uint32_t key[kPage];
      if (p == tid) {
#pragma unroll
        for (int j = 0; j < kPage; ++j) key[j] = cached[j];
      } else {
        load(p, key);
      }
      const int valid = min(len - p * kPage, kPage);
#pragma unroll
      for (int j = 0; j < kPage; ++j)
        if (j < valid && (shift == 24 || (key[j] >> ((shift + 8) & 31)) == (prefix >> ((shift + 8) & 31))))
          atomicAdd(&hist[(key[j] >> shift) & 255u], 1);
    }
    __syncthreads();
    // keys with a larger digit than d, by a scan from the top
    if (tid < 64) {
      int four[4], sum = 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) sum += four[q] = hist[255 - (4 * tid + q)];
      int incl = sum;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(incl, off);
        if (tid >= off) incl += y;
      }
      int above = incl - sum;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (above < want && above + four[q] >= want) {   // exactly one digit
          found[0] = 255 - (4 * tid + q);
          found[1] = above;
        }
        above += four[q];
      }
    }
    __syncthreads();
    prefix |= uint32_t(found[0]) << shift;
    want -= found[1];
  }

  // Keys above the threshold stay, and the first `want` equal ones.
  int equal_before = 0, hole_before = 0, tail_before = 0;
  for (int base = 0; base < pages; base += kThreads) {
    const int p = base + tid;
    uint32_t key[kPage];
    int valid = 0;
    if (p < pages) {
      if (base == 0) {
#pragma unroll
        for (int j = 0; j < kPage; ++j) key[j] = cached[j];
      } else {
        load(p, key);
      }
      valid = min(len - p * kPage, kPage);
    }
    uint32_t above = 0, equal = 0;
#pragma unroll
    for (int j = 0; j < kPage; ++j) {
      if (j >= valid) break;
      above |= uint32_t(key[j] > prefix) << j;
      equal |= uint32_t(key[j] == prefix) << j;
    }
    int total;
    int rank = equal_before + block_scan<kThreads>(__popc(equal), scan, total);
    equal_before += total;
    uint32_t kept = above;
    for (uint32_t m = equal; m != 0; m &= m - 1, ++rank)
      if (rank < want) kept |= m & (0u - m);
    const uint32_t all = (1u << valid) - 1u;
    const int front = min(max(n - p * kPage, 0), valid);   // slots of this page among the first n
    const uint32_t front_mask = (1u << front) - 1u;
    const uint32_t hole = all & front_mask & ~kept;
    uint32_t tail = kept & ~front_mask;
    const int hole_at = hole_before + block_scan<kThreads>(__popc(hole), scan, total);
    hole_before += total;
    int tail_at = tail_before + block_scan<kThreads>(__popc(tail), scan, total);
    tail_before += total;
    if (p < keep_pages) {
      holes[2 * p] = hole;
      holes[2 * p + 1] = uint32_t(hole_at);
    }
    for (; tail != 0; tail &= tail - 1) tails[tail_at++] = p * kPage + __ffs(tail) - 1;
  }
  finish();
}

constexpr int kMoveWaves = 4;
constexpr int kMoveRun = kMaxRun;   // pages of a row, at most
constexpr int kFewTokens = 2;

// An fp8 tile that takes one or two tokens (set in mask) and keeps its scale: a lane
// has dims lane and 64 + lane of each token, where the full store has 16 or 32 values of
// which an eighth or less are new. False, with nothing written, where the scale
// must change.
template <int D>
__device__ __forceinline__ bool move_few_fp8(uint8_t* pool, const float* scales, size_t dst_tile, int hkv, int kvh, bool is_v,
                                             uint32_t held, uint32_t mask, int src_page, int src_slot, int lane) {
  constexpr int kPieces = D / 64;
  const int slots[2] = {__ffs(mask) - 1, 31 - __clz(mask)};   // alike for one token, which is then moved twice
  // byte of (slot, dim 64 p + lane): 1024 p + of_lane + of_slot (fp8_tile.h)
  const int of_lane = is_v ? 16 * (lane & 15) + 4 * (lane >> 4) : 256 * ((lane >> 3) & 3) + 8 * (lane >> 5) + (lane & 7);
  auto of_slot = [&](int s) { return is_v ? 256 * (s >> 2) + (s & 3) : 16 * s; };
  uint8_t* dst = pool + dst_tile * (kPage * D);
  uint32_t raw[2][kPieces];
  float s[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const size_t tile = size_t(__builtin_amdgcn_readlane(src_page, slots[i])) * hkv + kvh;
    const uint8_t* from = pool + tile * (kPage * D) + of_slot(__builtin_amdgcn_readlane(src_slot, slots[i])) + of_lane;
    s[i] = scales[tile];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) raw[i][p] = from[1024 * p];
  }
  tile_u32x4 codes[kPieces];
#pragma unroll
  for (int p = 0; p < kPieces; ++p) codes[p] = *reinterpret_cast<const tile_u32x4*>(dst + 1024 * p + 16 * lane);
  const float scale = scales[dst_tile];
  uint32_t any = 0;
#pragma unroll
  for (int p = 0; p < kPieces; ++p) any |= codes[p][0] | codes[p][1] | codes[p][2] | codes[p][3];
  any &= fp8_slot_bytes(held, is_v, lane) & 0x7F7F7F7Fu;
  float x[2][kPieces], top = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      x[i][p] = fp8_value(raw[i][p], 0) * s[i];
      top = fmaxf(top, fabsf(x[i][p]));
    }
  // fp8_new_scale's shift is 0 where the quotient rounds to at most 1, which is where top <= 448 scale
  if (!__any(any != 0) || __any(top > __fmul_rn(448.f, scale))) return false;
  const float factor = __fdiv_rn(1.f, scale);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t n = fp8_codes(x[i][0] * factor, x[i][kPieces - 1] * factor, 0.f, 0.f);
#pragma unroll
    for (int p = 0; p < kPieces; ++p) dst[1024 * p + of_slot(slots[i]) + of_lane] = uint8_t(n >> (8 * p));
  }
  return true;
}

// One tile of page pg (pool page `page`). Lane t (every 16 lanes alike): slot t
// takes the token of slot `source` of the sequence, in pool page src_page, if its bit is set in mask.
template <int D, bool kFp8>
__device__ __forceinline__ void move_tile(const EvictArgs& a, int pg, int kvh, bool is_v, int len, int n, uint32_t mask,
                                          int source, int page, int src_page, int lane) {
  constexpr int kPieces = D / 64;
  const int col = lane & 15;
  const int grp = lane >> 4;
  const int hkv = a.num_kv_heads;
  const bool moved = (mask >> col) & 1u;
  const int src_slot = moved ? source % kPage : col;
  const size_t dst_tile = size_t(page) * hkv + kvh;
  const size_t src_tile = size_t(src_page) * hkv + kvh;
  if (!is_v && lane < kPage && pg * kPage + lane < n && (mask != 0 || a.w_out != a.w_in || a.pos_out != a.pos_in)) {
    const size_t from = src_tile * kPage + src_slot, to = dst_tile * kPage + lane;
    const float w = a.w_in[from];
    const int32_t pos = a.pos_in[from];
    a.w_out[to] = w;
    a.pos_out[to] = pos;
  }
  if (mask == 0) return;
  if constexpr (kFp8) {
    uint8_t* pool = static_cast<uint8_t*>(is_v ? a.v_pool : a.k_pool);
    float* scales = is_v ? a.v_scale : a.k_scale;
    uint8_t* dst = pool + dst_tile * (kPage * D);
    const uint32_t live = (1u << min(len - pg * kPage, kPage)) - 1u;
    if (__popc(mask) <= kFewTokens && live == 0xFFFFu &&
        move_few_fp8<D>(pool, scales, dst_tile, hkv, kvh, is_v, ~mask, mask, src_page, src_slot, lane))
      return;
    tile_u32x4 codes[kPieces];
    float x[kPieces][16];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      codes[p] = *reinterpret_cast<const tile_u32x4*>(dst + 1024 * p + 16 * lane);
#pragma unroll
      for (int e = 0; e < 16; ++e) x[p][e] = 0.f;
    }
    const float old_scale = scales[dst_tile];
    if (!is_v) {
      if (moved) {
        const float s = scales[src_tile];
        const uint8_t* from = pool + src_tile * (kPage * D) + (grp * kPage + src_slot) * 16;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
          const tile_u32x4 w = *reinterpret_cast<const tile_u32x4*>(from + 1024 * p);
#pragma unroll
          for (int e = 0; e < 16; ++e) x[p][e] = fp8_value(w[e >> 2], e & 3) * s;
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int t = 4 * grp + e;
        const int from_slot = __shfl(src_slot, t);
        const int from_page = __shfl(src_page, t);
        if (!((mask >> t) & 1u)) continue;
        const size_t tile = size_t(from_page) * hkv + kvh;
        const float s = scales[tile];
        const uint8_t* from = pool + tile * (kPage * D) + ((from_slot >> 2) * kPage + col) * 16;
        const int shift = 8 * (from_slot & 3);
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
          const tile_u32x4 w = *reinterpret_cast<const tile_u32x4*>(from + 1024 * p);
#pragma unroll
          for (int j = 0; j < 4; ++j) x[p][4 * j + e] = fp8_value(w[j] >> shift, 0) * s;
        }
      }
    }
    fp8_store_tile<D>(codes, true, fp8_slot_bytes(live & ~mask, is_v, lane), x, fp8_slot_bytes(mask, is_v, lane),
                      old_scale, dst, scales + dst_tile, lane);
  } else if (!is_v) {
    // Keys: a lane's pieces are all of slot col, from its own tile or the
    // token's; the tile goes out whole (16 bytes here and there would be read
    // and written as whole lines all the same).
    uint16_t* pool = static_cast<uint16_t*>(a.k_pool);
    u32x4 v[D / 32];
#pragma unroll
    for (int p = 0; p < D / 32; ++p)
      v[p] = *reinterpret_cast<const u32x4*>(pool + src_tile * (kPage * D) + ((4 * p + grp) * kPage + src_slot) * 8);
#pragma unroll
    for (int p = 0; p < D / 32; ++p)
      *reinterpret_cast<u32x4*>(pool + dst_tile * (kPage * D) + (64 * p + lane) * 8) = v[p];
  } else {
    // Values: a lane takes whole dims (32-byte rows of 16 slots). Every tile
    // that tokens come from is read once, the next one requested before the
    // tokens of this one are picked out: their slots are the same for all
    // lanes, so they are register indexes. (Read token by token, two bytes of
    // each row, the long-tail batch's moves took 562 us.)
    uint16_t* pool = static_cast<uint16_t*>(a.v_pool);
    uint16_t* dst = pool + dst_tile * (kPage * D) + lane * kPage;
    u32x8 row[kPieces], from[kPieces], next[kPieces];
    auto read = [&](const uint16_t* tile, u32x8* x) {
#pragma unroll
      for (int p = 0; p < kPieces; ++p) x[p] = *reinterpret_cast<const u32x8*>(tile + 64 * p * kPage);
    };
    auto tile_of = [&](uint32_t m) {   // of the lowest slot in m
      const int t = __ffs(m) - 1;
      return pool + (size_t(__builtin_amdgcn_readlane(src_page, t)) * hkv + kvh) * (kPage * D) + lane * kPage;
    };
    // the slots whose tokens come from the same page as that of the lowest one
    auto same_page = [&](uint32_t m) {
      const int page_of = __builtin_amdgcn_readlane(src_page, __ffs(m) - 1);
      return uint32_t(__ballot(src_page == page_of) & 0xFFFFu) & m;
    };
    uint32_t left = __builtin_amdgcn_readfirstlane(mask);
    read(dst, row);
    read(tile_of(left), from);
    while (left != 0) {
      const uint32_t now = same_page(left);
      left &= ~now;
      if (left != 0) read(tile_of(left), next);
      for (uint32_t m = now; m != 0; m &= m - 1) {
        const int t = __ffs(m) - 1;
        const int s = __builtin_amdgcn_readlane(src_slot, t);
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
          const uint32_t x = (s & 1 ? from[p][s >> 1] >> 16 : from[p][s >> 1] & 0xFFFFu);
          const uint32_t w = row[p][t >> 1];
          row[p][t >> 1] = t & 1 ? (w & 0xFFFFu) | (x << 16) : (w & 0xFFFF0000u) | x;
        }
      }
#pragma unroll
      for (int p = 0; p < kPieces; ++p) from[p] = next[p];
    }
#pragma unroll
    for (int p = 0; p < kPieces; ++p) *reinterpret_cast<u32x8*>(dst + 64 * p * kPage) = row[p];
  }
}

// Of an fp8 cache the page that holds slot n keeps both freed slots and
// sources of other pages' moves, which must read its codes by the scale that
// they have; it is left to a launch of its own behind the others (kBoundary).
template <int D, bool kFp8, bool kBoundary>
__global__ __launch_bounds__(64 * kMoveWaves) void evict_move_kernel(EvictArgs a) {
  const int lane = int(threadIdx.x) & 63;
  const int col = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int hkv = a.num_kv_heads;
  // A row has all that its workgroup needs.
  const const_i32_ptr item = as_constant(a.late_rows ? a.late_rows : a.rows) + (kBoundary ? size_t(blockIdx.x) : size_t(a.num_seqs) + blockIdx.x) * kRowInts;
  int seq, pb, np, len, n, hole_base, tail_base;
  if constexpr (kBoundary) {
    seq = item[5];
    len = item[0];
    n = item[1];
    hole_base = item[2];
    tail_base = item[3];
    pb = n / kPage;
    np = 1;
    if (n % kPage == 0 || n == len) return;
  } else {
    seq = item[0];
    pb = item[1];
    np = item[2];
    len = item[3];
    n = item[4];
    hole_base = item[5];
    tail_base = item[6];
  }
  const int keep_pages = (n + kPage - 1) / kPage;
  const const_i32_ptr bt = as_constant(a.block_table) + size_t(seq) * a.bt_stride;
  const int moves = min(n, len - n);
  // A wave takes one (KV head, keys or values) of all the run's pages. What it
  // takes to find the tokens (freed slots, sources, their pages: three dependent
  // reads) is requested for all of them before the first tile is moved.
  for (int rem = int(blockIdx.y) * kMoveWaves + wave; rem < hkv * 2; rem += int(gridDim.y) * kMoveWaves) {
    const bool is_v = rem >= hkv;
    const int kvh = is_v ? rem - hkv : rem;
    const const_i32_ptr hole = (const_i32_ptr)(a.holes) + 2 * (size_t(hole_base) + size_t(kvh) * keep_pages + pb);
    const int32_t* tails = a.tails + size_t(tail_base) + size_t(kvh) * moves;
    uint32_t masks[kMoveRun];
    int sources[kMoveRun], pages[kMoveRun], source_pages[kMoveRun];
#pragma unroll
    for (int j = 0; j < kMoveRun; ++j) {
      const bool here = j < np && !(kFp8 && !kBoundary && n < len && (pb + j + 1) * kPage > n);
      masks[j] = here ? uint32_t(hole[2 * j]) : 0u;
      pages[j] = bt[j < np ? pb + j : pb];
      // Lane t (every 16 lanes alike): the slot that slot t's token comes from.
      const bool moved = (masks[j] >> col) & 1u;
      sources[j] = moved ? tails[hole[2 * j + 1] + __popc(masks[j] & ((1u << col) - 1u))] : 0;
    }
#pragma unroll
    for (int j = 0; j < kMoveRun; ++j)
      source_pages[j] = (masks[j] >> col) & 1u ? a.block_table[size_t(seq) * a.bt_stride + sources[j] / kPage] : pages[j];
#pragma unroll
    for (int j = 0; j < kMoveRun; ++j) {
      if (j >= np) break;
      if (kFp8 && !kBoundary && n < len && (pb + j + 1) * kPage > n) continue;
      move_tile<D, kFp8>(a, pb + j, kvh, is_v, len, n, masks[j], sources[j], pages[j], source_pages[j], lane);
    }
  }
}

template <int D, bool kFp8>
hipError_t launch_moves(const EvictArgs& a, hipStream_t stream) {
  const int groups = (2 * a.num_kv_heads + kMoveWaves - 1) / kMoveWaves;
  const int gy = groups < 65535 ? groups : 65535;
  if (a.num_moves > 0) {
    hipLaunchKernelGGL((evict_move_kernel<D, kFp8, false>), dim3(a.num_moves, gy), dim3(64 * kMoveWaves), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!kFp8 || !a.boundary) return hipSuccess;
  hipLaunchKernelGGL((evict_move_kernel<D, kFp8, true>), dim3(a.num_seqs, gy), dim3(64 * kMoveWaves), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_evict(const EvictArgs& a, hipStream_t stream) {
  if (a.num_moves == 0) return hipSuccess;
  // A thread keeps its first page's keys in registers, and reads the others
  // again at each of the five passes: sequences of more pages than a small
  // workgroup has threads go to a launch of large ones (long-tail batch, both on
  // 256 threads 64 us, both on 1024 63).
  if (a.num_long < a.num_seqs)
    hipLaunchKernelGGL(evict_select_kernel<kSelectShort>, dim3((a.num_seqs - a.num_long) * a.num_kv_heads), dim3(kSelectShort),
                       0, stream, a);
  if (a.num_long > 0) {
    EvictArgs b = a;
    if (a.num_long < a.num_seqs) b.late_rows = nullptr;   // the launch before has copied them
    hipLaunchKernelGGL(evict_select_kernel<kSelectLong>, dim3(a.num_long * a.num_kv_heads), dim3(kSelectLong), 0, stream, b);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.k_scale) return a.head_dim == 128 ? launch_moves<128, true>(a, stream) : launch_moves<64, true>(a, stream);
  return a.head_dim == 128 ? launch_moves<128, false>(a, stream) : launch_moves<64, false>(a, stream);
}

}  // namespace sf
