// Store of new tokens into an fp8 (E4M3) cache: the growing form of the
// per-page quantizer. Every decode step adds one token per running trajectory
// (App. B.1) and every (re-)prefill a block of them (Sec. 2.3); here their
// keys and values go straight into the 8-bit pages.
//
// A (page, KV head) tile has one scale, and a page fills over up to 16 calls,
// so the scale is not final when the first token comes. It grows by powers of
// two (fp8_tile.h): dividing an E4M3 code by 2^k only moves its exponent, exact
// until it becomes subnormal, so a token keeps the rounding of its own store
// where a scale made anew from each maximum would round all held tokens again
// at every growth.
//
// One wave per tile, which it reads (where it holds tokens), requantizes in
// registers and writes in 16-byte pieces, the changed ones: whole fresh pages
// go out as 1 KiB per wave store. Values of new tokens are read two
// bytes at a time (16 lanes, 32 contiguous bytes per token), which is not what
// bounds it: memory is. 95,330 tokens of 32 prompts (28/4 heads, D = 128; 195 MB in,
// 98 MB out) take 62 us (56 at best) = 4.7 TB/s, a 4 GiB device copy's rate; one token of
// 512 sequences 10 us, latency. With the reads of a lane's four slots behind branches
// the prompts took 68 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fp8_tile.h"
#include "sf_internal.h"

namespace sf {
namespace {

typedef __attribute__((address_space(4))) const int32_t* const_i32_ptr;
__device__ __forceinline__ const_i32_ptr as_constant(const int32_t* p) { return (const_i32_ptr)(p); }
__device__ __forceinline__ float bf16_value(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }

constexpr int kWaves = 4;

template <int D>
__global__ __launch_bounds__(64 * kWaves) void kv_store_fp8_kernel(Store8Args a) {
  constexpr int kPieces = D / 64;
  // 64 bits: a launch of up to 2^24 rows, times the heads' groups, has more threads than 2^31
  int64_t i0 = (int64_t(blockIdx.y) * gridDim.x + blockIdx.x) * (64 * kWaves) + int(threadIdx.x);
  const int copied = i0 < a.copy_ints ? a.copy_src[i0] : 0;
  const const_i32_ptr row = as_constant(a.rows) + size_t(blockIdx.x) * kItemInts;
  const int seq = row[0];
  const int pb = row[1];
  const int np = row[2];
  const int first = row[3];
  const int end = row[4];
  const int qrow = row[5];
  const int lane = int(threadIdx.x) & 63;
  const int col = lane & 15;
  const int grp = lane >> 4;
  const int hkv = a.num_kv_heads;
  const size_t tok_stride = size_t(hkv) * D;
  const size_t entry0 = size_t(seq) * a.bt_stride;
  const int last = (end - 1) / kPage;
  const int fresh_page = a.new_pages ? as_constant(a.new_pages)[seq] : -1;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  for (int i = int(blockIdx.y) * kWaves + wave; i < np * hkv * 2; i += int(gridDim.y) * kWaves) {
    const int pg = pb + i / (2 * hkv);
    const int rem = i % (2 * hkv);
    const bool is_v = rem >= hkv;
    const int kvh = is_v ? rem - hkv : rem;
    const bool opened = pg == last && fresh_page >= 0;
    const int page = opened ? fresh_page : as_constant(a.block_table)[entry0 + pg];
    const int lo = max(first, pg * kPage), hi = min(end, (pg + 1) * kPage);   // positions stored here
    const int s0 = lo - pg * kPage, s1 = hi - pg * kPage;
    const uint32_t held_slots = (1u << s0) - 1u;
    const uint32_t new_slots = ((1u << s1) - 1u) & ~held_slots;
    const size_t tile = (size_t(page) * hkv + kvh) * size_t(kPage * D);
    uint8_t* dst = (is_v ? a.v_pool : a.k_pool) + tile;
    float* scale = (is_v ? a.v_scale : a.k_scale) + size_t(page) * hkv + kvh;
    tile_u32x4 codes[kPieces];
    float old_scale = 1.f;
#pragma unroll
    for (int p = 0; p < kPieces; ++p) codes[p] = tile_u32x4{0u, 0u, 0u, 0u};
    if (s0 > 0) {
#pragma unroll
      for (int p = 0; p < kPieces; ++p) codes[p] = *reinterpret_cast<const tile_u32x4*>(dst + 1024 * p + 16 * lane);
      old_scale = *scale;
    }
    // new-token row of slot s0; slot s is row s - s0
    const uint16_t* src = (is_v ? a.v_new : a.k_new) + size_t(qrow + (lo - first)) * tok_stride + size_t(kvh) * D;
    // Slots without a new token read the nearest one that has: without branches
    // all of a lane's reads are in flight at once.
    float x[kPieces][16];
    if (is_v) {
      uint16_t raw[kPieces][16];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint16_t* v = src + size_t(min(max(4 * grp + e, s0), s1 - 1) - s0) * tok_stride + col;
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
#pragma unroll
          for (int j = 0; j < 4; ++j) raw[p][4 * j + e] = v[64 * p + 16 * j];
      }
#pragma unroll
      for (int p = 0; p < kPieces; ++p)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int s = 4 * grp + (e & 3);
          x[p][e] = s >= s0 && s < s1 ? bf16_value(raw[p][e]) : 0.f;
        }
    } else {
      const bool there = col >= s0 && col < s1;
      const uint16_t* k = src + size_t(min(max(col, s0), s1 - 1) - s0) * tok_stride + 8 * grp;
      tile_u32x4 raw[kPieces][2];
#pragma unroll
      for (int p = 0; p < kPieces; ++p)
#pragma unroll
        for (int h = 0; h < 2; ++h) raw[p][h] = *reinterpret_cast<const tile_u32x4*>(k + 64 * p + 32 * h);
#pragma unroll
      for (int p = 0; p < kPieces; ++p)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const uint32_t w = raw[p][e >> 3][(e >> 1) & 3];
          x[p][e] = there ? bf16_value(e & 1 ? w >> 16 : w & 0xFFFFu) : 0.f;
        }
    }
    fp8_store_tile<D>(codes, s0 > 0, fp8_slot_bytes(held_slots, is_v, lane), x, fp8_slot_bytes(new_slots, is_v, lane),
                      old_scale, dst, scale, lane);
    if (opened && rem == 0 && lane == 0) a.block_table[entry0 + pg] = page;
  }
  if (i0 < a.copy_ints) a.copy_dst[i0] = copied;
  const int64_t stride = int64_t(gridDim.x) * gridDim.y * (64 * kWaves);
  for (i0 += stride; i0 < a.copy_ints; i0 += stride) a.copy_dst[i0] = a.copy_src[i0];
}

}  // namespace

hipError_t launch_store_fp8(const Store8Args& a, hipStream_t stream) {
  if (a.num_rows == 0) return hipSuccess;
  // one wave per tile of a single page; the waves of a run of pages loop
  const int groups = (2 * a.num_kv_heads + kWaves - 1) / kWaves;
  const dim3 grid(a.num_rows, groups < 65535 ? groups : 65535), block(64 * kWaves);
  if (a.head_dim == 128)
    hipLaunchKernelGGL(kv_store_fp8_kernel<128>, grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL(kv_store_fp8_kernel<64>, grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace sf
