// Attention weights of cached keys, summed over the query rows that read them.
//
// A cache of bounded size keeps the keys that its queries attend to most. What
// it goes by is, for every cached key t of a (sequence, KV head),
//   w[t] += sum over rows (new token j, query head h of the group) with t <= P + j
//           of exp(scale q[j,h].K[t] - lse[j,h])
// with the rows' lse known from the attention that ran before. That is a score
// product without its P.V half, and the sum runs over rows, not keys, so the
// work is cut by keys: a wave keeps 64 keys (four pages) in registers as MFMA A
// operands and walks the rows, 16 at a time,
//   S^T[16 keys][16 rows] = K Q^T    (D/32) v_mfma_f32_16x16x32_bf16 per page
//   w[key] += 2^(S^T c - lse2)       one fma, exp2 and add per score
// and no sum crosses waves: no atomics, the same bits on every run. A lane's
// partial sums (its row column) are joined once at the end of the walk, by a
// butterfly that halves the values at every step and leaves one key per lane.
//
// One row per sequence (a decode step) is bound by reading K once; the rows of
// a whole prompt by the exponentials (quarter rate: 24 vector cycles per 16 of
// matrix work). Work items, and the parts that long walks are cut into, are the
// host plan's; key_weights_merge_kernel adds the parts of a cut item in order.
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

// Rows of a tile: this lane's query row and its lse in log2 units (+inf, weight
// 0, for a row past the walk's end and for one whose lse is not finite).
template <int D>
struct RowTile {
  u32x4 q[D / 32];
  float lse2;
};

template <int D, bool kFp8>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 4))) void key_weights_kernel(WeightArgs a) {
  constexpr int KB = D / 32;
  const const_i32_ptr row = as_constant(a.items) + size_t(blockIdx.x) * kWeightInts;
  const int seq = row[0];
  const int kvh = row[1];
  const int page_begin = row[2];
  const int page_end = row[3];
  const int tok_begin = row[4];
  const int tok_end = row[5];
  const int slot = row[6];
  const int prefix = row[8];
  const int qrow0 = row[9];
  const int lane = int(threadIdx.x) & 63;
  const int col = lane & 15;
  const int grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int g = a.group;
  const int hkv = a.num_kv_heads;
  const uint32_t inv_g = a.inv_group;   // floor(x / g) = x * inv_g >> 16 for x < 32
  const const_i32_ptr bt = as_constant(a.block_table) + size_t(seq) * a.bt_stride;

  // Row tiles are 16 rows (token-major over the group's heads) from token `tok`, head `rem`.
  struct At {
    int tok, rem;
  };
  auto next = [&](At at) {
    const int x = at.rem + 16, dt = int((uint32_t(x) * inv_g) >> 16);
    return At{at.tok + dt, x - dt * g};
  };
  auto load_rows = [&](RowTile<D>& t, At at) {
    const int x = at.rem + col, dt = int((uint32_t(x) * inv_g) >> 16);
    const bool ok = at.tok + dt < tok_end;
    const size_t head_row = (size_t(qrow0) + size_t(ok ? at.tok + dt : tok_begin)) * a.num_q_heads + size_t(kvh) * g +
                            size_t(ok ? x - dt * g : 0);
    const uint16_t* q = a.q + head_row * D + 8 * grp;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) t.q[kb] = *reinterpret_cast<const u32x4*>(q + 32 * kb);
    const float l = a.lse[head_row];
    t.lse2 = ok && __builtin_fabsf(l) < __builtin_inff() ? l * kLog2e : __builtin_inff();
  };

  for (int pg = page_begin + wave * kTiles; pg < page_end; pg += kWaves * kTiles) {
    u32x4 k[kTiles][KB];
    float c[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      const int page = bt[pg + i < page_end ? pg + i : pg];   // a page past the end repeats the first, unused
      const size_t tile = (size_t(page) * hkv + kvh) * size_t(kPage * D);
      c[i] = a.scale_log2;
      if constexpr (kFp8) {
        const uint8_t* src = reinterpret_cast<const uint8_t*>(a.k_pool) + tile + lane * 16;
#pragma unroll
        for (int p = 0; p < D / 64; ++p) {
          const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + 1024 * p));
          k[i][2 * p] = u32x4{widen2<false>(w[0]), widen2<true>(w[0]), widen2<false>(w[1]), widen2<true>(w[1])};
          k[i][2 * p + 1] = u32x4{widen2<false>(w[2]), widen2<true>(w[2]), widen2<false>(w[3]), widen2<true>(w[3])};
        }
        c[i] *= ((const_f32_ptr)a.k_scale)[size_t(page) * hkv + kvh];
      } else {
        const uint16_t* src = a.k_pool + tile + lane * 8;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
          k[i][kb] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + 512 * kb));
      }
    }
    f32x4 acc[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int key0 = pg * kPage;
    const int tok_first = max(tok_begin, key0 - prefix);   // rows before it see none of these keys
    auto step = [&](const RowTile<D>& t, At at) {
      f32x4 s[kTiles];
#pragma unroll
      for (int i = 0; i < kTiles; ++i) s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < kTiles; ++i) s[i] = mfma_bf16(k[i][kb], t.q[kb], s[i]);
      if (prefix + at.tok >= key0 + kTiles * kPage - 1) {   // every row sees every key
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            acc[i][e] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][e], c[i], -t.lse2));
      } else {
        const int limit = prefix + at.tok + int((uint32_t(at.rem + col) * inv_g) >> 16);   // the row's own position
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][e], c[i], -t.lse2));
            acc[i][e] += key0 + kPage * i + 4 * grp + e <= limit ? p : 0.f;
          }
      }
    };
    At at = {tok_first, 0};
    if (at.tok < tok_end) {
      RowTile<D> even, odd;
      load_rows(even, at);
      while (true) {
        At then = next(at);
        if (then.tok < tok_end) load_rows(odd, then);
        step(even, at);
        if (then.tok >= tok_end) break;
        at = next(then);
        if (at.tok < tok_end) load_rows(even, at);
        step(odd, then);
        if (at.tok >= tok_end) break;
      }
    }

    // Sums over the 16 row columns: every step hands half of the values to the
    // partner lane and keeps the other half, until lane (grp, col) holds the
    // value col = 4 i + e of key 16 i + 4 grp + e.
    float v[16];
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * i + e] = acc[i][e];
#pragma unroll
    for (int half = 8; half >= 1; half >>= 1) {
      const bool upper = (col & half) != 0;
#pragma unroll
      for (int j = 0; j < half; ++j) {
        const float keep = upper ? v[j + half] : v[j];
        const float give = upper ? v[j] : v[j + half];
        v[j] = keep + __shfl_xor(give, half);
      }
    }
    const int key = key0 + kPage * (col >> 2) + 4 * grp + (col & 3);
    if (pg + (col >> 2) < page_end) {
      if (slot >= 0)
        a.part[size_t(slot) * a.part_keys + (key - page_begin * kPage)] = v[0];
      else
        finish_key(a, row, key, v[0]);
    }
  }
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

}  // namespace

hipError_t launch_key_weights(const WeightArgs& a, hipStream_t stream) {
  if (a.num_items == 0) return hipSuccess;
  const dim3 grid(a.num_items), block(64 * kWaves);
  void (*kernel)(WeightArgs) = a.head_dim == 128 ? (a.k_scale ? key_weights_kernel<128, true> : key_weights_kernel<128, false>)
                                                 : (a.k_scale ? key_weights_kernel<64, true> : key_weights_kernel<64, false>);
  hipLaunchKernelGGL(kernel, grid, block, 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.num_merge == 0) return e;
  hipLaunchKernelGGL(key_weights_merge_kernel, dim3(a.num_merge), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sf
