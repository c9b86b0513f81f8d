// Rotary positions: frequencies, the plan of the storing form, and the entry
// points. The rules are stated in sf_decode_attn.h.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>

#include "sf_internal.h"

static_assert(sizeof(sf_rotary_desc) == 16, "sf_rotary_desc layout is part of the ABI");
static_assert(sizeof(sf_rotary_scaling) == 32, "sf_rotary_scaling layout is part of the ABI");

using namespace sf;

namespace {

constexpr int32_t kMaxTokens = 1 << 30;     // per sequence, as the fp8 store's
constexpr int64_t kMaxRows = 1 << 23;       // workgroups of 256 threads: 2^32 threads are too many for a launch
constexpr int32_t kMaxTurned = 1 << 27;     // tokens of a call, of so many 16 to a workgroup
constexpr uint64_t kRotaryKey = 0x526f74617279ull;   // tells this plan's info from the fp8 store's

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
int32_t pages_of(int32_t tokens) { return (tokens + kPage - 1) / kPage; }

// One page per row has the most parallelism; a long list is cheaper to make and
// read in runs of four.
constexpr int64_t kSinglePages = 2048;

sf_status check_rotary(const sf_rotary_desc* r) {
  if (!r || (r->interleaved | 1) != 1 || !std::isfinite(r->magnitude)) return SF_ERR_INVALID_ARG;
  if (r->head_dim != 64 && r->head_dim != 128) return SF_ERR_UNSUPPORTED;
  if (r->rotary_dim < 16 || r->rotary_dim > r->head_dim) return SF_ERR_INVALID_ARG;
  return r->rotary_dim % 16 == 0 ? SF_OK : SF_ERR_UNSUPPORTED;
}

bool good_rows(const void* p, int64_t stride, int64_t heads, int32_t d) {
  return p && aligned16(p) && stride >= heads * d && stride % 8 == 0;
}

RotaryArgs rotary_args(const sf_rotary_desc* r, int32_t hq, int32_t hkv, const uint64_t* turns, const void* q,
                       int64_t q_stride, void* q_out, int64_t q_out_stride, const void* k, int64_t k_stride) {
  RotaryArgs a = {};
  a.head_dim = r->head_dim;
  a.rotary_dim = r->rotary_dim;
  a.interleaved = r->interleaved != 0;
  a.magnitude = r->magnitude;
  a.turns = turns;
  a.num_q_heads = q ? hq : 0;
  a.num_kv_heads = k ? hkv : 0;
  a.q = static_cast<const uint16_t*>(q);
  a.q_stride = q_stride;
  a.q_out = static_cast<uint16_t*>(q_out);
  a.q_out_stride = q_out_stride;
  a.k = static_cast<const uint16_t*>(k);
  a.k_stride = k_stride;
  return a;
}

}  // namespace

extern "C" sf_status sf_rotary_frequencies(int32_t rotary_dim, double base, const sf_rotary_scaling* scaling,
                                           double* freq_host) {
  if (!freq_host || rotary_dim < 2 || rotary_dim % 2 != 0 || !(base > 0.0) || !std::isfinite(base))
    return SF_ERR_INVALID_ARG;
  if (scaling && (!(scaling->factor > 0.0) || !std::isfinite(scaling->factor) || !(scaling->trained_length >= 0.0) ||
                  !std::isfinite(scaling->trained_length) ||
                  (scaling->trained_length > 0.0 &&
                   (!(scaling->low_turns < scaling->high_turns) || !std::isfinite(scaling->high_turns - scaling->low_turns)))))
    return SF_ERR_INVALID_ARG;
  const double two_pi = 6.283185307179586476925;
  for (int32_t i = 0; i < rotary_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rotary_dim);
    if (scaling) {
      double stay = 0.0;
      if (scaling->trained_length > 0.0) {
        const double r = scaling->trained_length * f / two_pi;
        stay = std::min(1.0, std::max(0.0, (r - scaling->low_turns) / (scaling->high_turns - scaling->low_turns)));
      }
      f = stay * f + (1.0 - stay) * f / scaling->factor;
    }
    if (!std::isfinite(f)) return SF_ERR_INVALID_ARG;
    freq_host[i] = f;
  }
  return SF_OK;
}

extern "C" sf_status sf_rotary_turns(const double* freq_host, int32_t n, uint64_t* turns_host) {
  if (n < 0 || (n > 0 && (!freq_host || !turns_host))) return SF_ERR_INVALID_ARG;
  for (int32_t i = 0; i < n; ++i) {
    if (!std::isfinite(freq_host[i])) return SF_ERR_INVALID_ARG;
    // long double holds 64 bits: the quotient is off by half a unit of 2^-64 where |f| < 2 pi
    const long double t = static_cast<long double>(freq_host[i]) / 6.283185307179586476925286766559L;
    const long double part = t - std::floor(t);                       // [0, 1], rounded
    const long double units = std::nearbyint(part * 18446744073709551616.0L);
    turns_host[i] = units >= 18446744073709551616.0L ? 0 : static_cast<uint64_t>(units);   // a whole turn is none
  }
  return SF_OK;
}

extern "C" sf_status sf_rotary(const sf_rotary_desc* rotary, int32_t num_tokens, int32_t num_q_heads,
                               int32_t num_kv_heads, const uint64_t* turns, const int32_t* positions, const void* q,
                               int64_t q_stride, void* q_out, int64_t q_out_stride, const void* k, int64_t k_stride,
                               void* k_out, int64_t k_out_stride, void* stream) {
  const sf_status st = check_rotary(rotary);
  if (st != SF_OK) return st;
  if (num_tokens < 0 || num_q_heads < 0 || num_kv_heads < 0 || num_q_heads > 1 << 16 || num_kv_heads > 1 << 16)
    return SF_ERR_INVALID_ARG;
  if (num_tokens > kMaxTurned) return SF_ERR_UNSUPPORTED;
  if (num_tokens == 0 || (!q && !k)) return SF_OK;
  const int32_t d = rotary->head_dim;
  if (!turns || !positions || !aligned8(turns) || !aligned4(positions)) return SF_ERR_INVALID_ARG;
  if (q && (!good_rows(q, q_stride, num_q_heads, d) || !good_rows(q_out, q_out_stride, num_q_heads, d)))
    return SF_ERR_INVALID_ARG;
  if (k && (!good_rows(k, k_stride, num_kv_heads, d) || !good_rows(k_out, k_out_stride, num_kv_heads, d)))
    return SF_ERR_INVALID_ARG;
  if ((q == q_out && q && q_stride != q_out_stride) || (k == k_out && k && k_stride != k_out_stride))
    return SF_ERR_INVALID_ARG;
  RotaryArgs a = rotary_args(rotary, num_q_heads, num_kv_heads, turns, q, q_stride, q_out, q_out_stride, k, k_stride);
  if (a.num_q_heads + a.num_kv_heads == 0) return SF_OK;
  a.k_out = static_cast<uint16_t*>(k_out);
  a.k_out_stride = k_out_stride;
  a.positions = positions;
  a.num_tokens = num_tokens;
  return launch_rotary(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SF_OK : SF_ERR_HIP;
}

extern "C" sf_status sf_rotary_store_plan(const sf_attn_desc* desc, const int32_t* seq_lens_host,
                                          const int32_t* q_lens_host, const int32_t* first_pos_host, int32_t* work_host,
                                          uint64_t work_capacity_bytes, sf_store_info* info) {
  if (!info) return SF_ERR_INVALID_ARG;
  const sf_status st = validate_desc(desc);
  if (st != SF_OK) return st;
  const int32_t n = desc->num_seqs;
  if (n > 0 && !seq_lens_host) return SF_ERR_INVALID_ARG;
  auto news = [&](int32_t s) { return q_lens_host ? q_lens_host[s] : int32_t(seq_lens_host[s] > 0); };
  auto touched = [&](int32_t s) {
    return news(s) == 0 ? 0 : pages_of(seq_lens_host[s]) - (seq_lens_host[s] - news(s)) / kPage;
  };
  int64_t pages = 0, rows = 0, tokens = 0;
  for (int32_t s = 0; s < n; ++s) {
    const int32_t L = seq_lens_host[s], e = news(s);
    if (L < 0 || e < 0 || L < e || L > kMaxTokens || int64_t(L) > int64_t(kPage) * desc->block_table_stride)
      return SF_ERR_INVALID_ARG;
    if (L > 0 && desc->num_pages == 0) return SF_ERR_INVALID_ARG;
    tokens += q_lens_host ? e : 1;
    if (tokens > INT32_MAX) return SF_ERR_INVALID_ARG;
    if (first_pos_host && (first_pos_host[s] < 0 || first_pos_host[s] > INT32_MAX - news(s))) return SF_ERR_INVALID_ARG;
    pages += touched(s);
  }
  const int32_t run = pages > kSinglePages ? kMaxRun : 1;
  for (int32_t s = 0; s < n; ++s) rows += (touched(s) + run - 1) / run;
  if (rows >= kMaxRows) return SF_ERR_UNSUPPORTED;
  info->num_rows = int32_t(rows);
  info->num_q_rows = int32_t(tokens);
  info->work_bytes = uint64_t(rows) * kItemInts * 4;
  info->desc_key = desc_key(desc) ^ kRotaryKey;
  if (!work_host) return SF_OK;
  if (work_capacity_bytes < info->work_bytes) return SF_ERR_CAPACITY;
  int32_t qrow = 0;
  for (int32_t s = 0; s < n; qrow += q_lens_host ? q_lens_host[s] : 1, ++s) {
    const int32_t first = seq_lens_host[s] - news(s), begin = first / kPage, end = begin + touched(s);
    for (int32_t p = begin; p < end; p += run) {
      const int32_t row[kItemInts] = {s,    p, std::min(run, end - p), first, seq_lens_host[s], qrow,
                                      first_pos_host ? first_pos_host[s] : first, 0};
      std::memcpy(work_host, row, sizeof row);
      work_host += kItemInts;
    }
  }
  return SF_OK;
}

extern "C" sf_status sf_rotary_store(const sf_attn_desc* desc, const sf_rotary_desc* rotary, const sf_store_info* info,
                                     const int32_t* work_host, int32_t* work_dev, const uint64_t* turns, const void* q,
                                     int64_t q_stride, void* q_out, int64_t q_out_stride, const void* k_new,
                                     int64_t k_stride, const void* v_new, int64_t v_stride, const int32_t* new_pages,
                                     void* k_pool, void* v_pool, int32_t* block_table, void* stream) {
  sf_status st = validate_desc(desc);
  if (st != SF_OK || (rotary && (st = check_rotary(rotary)) != SF_OK)) return st;
  const sf_rotary_desc none = {desc->head_dim, 0, 0, 1.f};
  if (!rotary) rotary = &none;
  if (!info || rotary->head_dim != desc->head_dim) return SF_ERR_INVALID_ARG;
  if (info->desc_key != (desc_key(desc) ^ kRotaryKey) || info->num_rows < 0 || info->num_q_rows < 0 ||
      info->work_bytes != uint64_t(info->num_rows) * kItemInts * 4)
    return SF_ERR_PLAN_MISMATCH;
  if (info->num_rows == 0) return SF_OK;
  const int32_t hq = desc->num_q_heads, hkv = desc->num_kv_heads, d = desc->head_dim;
  if (!work_dev || (rotary->rotary_dim && (!turns || !aligned8(turns))) || !k_pool || !v_pool || !block_table) return SF_ERR_INVALID_ARG;
  if (!aligned16(work_dev) || !aligned16(k_pool) || !aligned16(v_pool) || !aligned4(block_table) ||
      (new_pages && !aligned4(new_pages)))
    return SF_ERR_INVALID_ARG;
  if (!good_rows(k_new, k_stride, hkv, d) || !good_rows(v_new, v_stride, hkv, d)) return SF_ERR_INVALID_ARG;
  if (q && (!good_rows(q, q_stride, hq, d) || !good_rows(q_out, q_out_stride, hq, d) ||
            (q == q_out && q_stride != q_out_stride)))
    return SF_ERR_INVALID_ARG;
  RotaryArgs a = rotary_args(rotary, hq, hkv, turns, q, q_stride, q_out, q_out_stride, k_new, k_stride);
  a.rows = work_dev;
  a.num_rows = info->num_rows;
  a.v = static_cast<const uint16_t*>(v_new);
  a.v_stride = v_stride;
  a.new_pages = new_pages;
  a.k_pool = static_cast<uint16_t*>(k_pool);
  a.v_pool = static_cast<uint16_t*>(v_pool);
  a.block_table = block_table;
  a.bt_stride = desc->block_table_stride;
  a.num_tokens = info->num_q_rows;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (work_host && hipMemcpyAsync(work_dev, work_host, info->work_bytes, hipMemcpyHostToDevice, s) != hipSuccess)
    return SF_ERR_HIP;
  return launch_rotary(a, s) == hipSuccess ? SF_OK : SF_ERR_HIP;
}
