// A cache of bounded size: host planners and entry points of the store into
// an fp8 cache, the weights of cached keys and the eviction that goes by them.
// The rules are stated in sf_decode_attn.h next to their plan functions.
#include <algorithm>
#include <climits>
#include <cstdint>
#include <cstring>
#include <vector>

#include "sf_internal.h"

static_assert(sizeof(sf_store_info) == 24, "sf_store_info layout is part of the ABI");
static_assert(sizeof(sf_weights_info) == 48, "sf_weights_info layout is part of the ABI");
static_assert(sizeof(sf_evict_info) == 56, "sf_evict_info layout is part of the ABI");

using namespace sf;

namespace {

constexpr int32_t kMaxTokens = 1 << 30;   // per sequence: token and page numbers stay far from 2^31
constexpr int64_t kMaxGroups = 1 << 22;   // workgroups of 1024 threads (4 times as many of 256): 2^32 threads are too many for a launch

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
int32_t pages_of(int32_t tokens) { return (tokens + kPage - 1) / kPage; }
sf_status from_hip(hipError_t e) { return e == hipSuccess ? SF_OK : SF_ERR_HIP; }

// Pages per work-list row: one wave per tile has the most parallelism, and a
// long list is cheaper to make and read in runs of four.
constexpr int64_t kSinglePages = 2048;
int32_t run_of(int64_t pages) { return pages > kSinglePages ? kMaxRun : 1; }

void put_row(int32_t*& at, int32_t a, int32_t b, int32_t c, int32_t d, int32_t e, int32_t f, int32_t g = 0) {
  const int32_t row[kItemInts] = {a, b, c, d, e, f, g, 0};
  std::memcpy(at, row, sizeof row);
  at += kItemInts;
}

sf_status check_lengths(const sf_attn_desc* desc, const int32_t* seq_lens, const int32_t* q_lens, int64_t* rows) {
  const sf_status st = check_extend_lengths(desc, seq_lens, q_lens, rows);
  if (st != SF_OK) return st;
  for (int32_t s = 0; s < desc->num_seqs; ++s)
    if (seq_lens[s] > kMaxTokens) return SF_ERR_INVALID_ARG;
  return SF_OK;
}

}  // namespace

// ---------------------------------------------------------------------------
// store into an fp8 cache
// ---------------------------------------------------------------------------
extern "C" sf_status sf_kv_store_fp8_plan(const sf_attn_desc* desc, const int32_t* seq_lens_host,
                                          const int32_t* q_lens_host, int32_t* work_host, uint64_t work_capacity_bytes,
                                          sf_store_info* info) {
  if (!info) return SF_ERR_INVALID_ARG;
  int64_t tokens = 0;
  sf_status st = check_lengths(desc, seq_lens_host, q_lens_host, &tokens);
  if (st != SF_OK) return st;
  const int32_t* news = q_lens_host;
  auto touched = [&](int32_t s) {
    return news[s] == 0 ? 0 : pages_of(seq_lens_host[s]) - (seq_lens_host[s] - news[s]) / kPage;
  };
  int64_t pages = 0, rows = 0;
  for (int32_t s = 0; s < desc->num_seqs; ++s) pages += touched(s);
  const int32_t run = run_of(pages);
  for (int32_t s = 0; s < desc->num_seqs; ++s) rows += (touched(s) + run - 1) / run;
  if (rows >= 4 * kMaxGroups) return SF_ERR_UNSUPPORTED;
  info->num_rows = int32_t(rows);
  info->num_q_rows = int32_t(tokens);
  info->work_bytes = uint64_t(rows) * kItemInts * 4;
  info->desc_key = desc_key(desc);
  if (!work_host) return SF_OK;
  if (work_capacity_bytes < info->work_bytes) return SF_ERR_CAPACITY;
  int32_t qrow = 0;
  for (int32_t s = 0; s < desc->num_seqs; qrow += news[s++]) {
    const int32_t first = seq_lens_host[s] - news[s], begin = first / kPage, end = begin + touched(s);
    for (int32_t p = begin; p < end; p += run)
      put_row(work_host, s, p, std::min(run, end - p), first, seq_lens_host[s], qrow);
  }
  return SF_OK;
}

sf_status sf::store8_args(const sf_attn_desc* desc, const int32_t* work_dev, const void* k_new, const void* v_new,
                          const int32_t* new_pages, void* k_pool8, void* v_pool8, float* k_scale, float* v_scale,
                          int32_t* block_table, Store8Args* args) {
  if (!work_dev || !k_new || !v_new || !k_pool8 || !v_pool8 || !k_scale || !v_scale || !block_table)
    return SF_ERR_INVALID_ARG;
  if (!aligned16(work_dev) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(k_pool8) || !aligned16(v_pool8) ||
      !aligned4(k_scale) || !aligned4(v_scale) || !aligned4(block_table) || (new_pages && !aligned4(new_pages)))
    return SF_ERR_INVALID_ARG;
  Store8Args a = {};
  a.rows = work_dev;
  a.k_new = static_cast<const uint16_t*>(k_new);
  a.v_new = static_cast<const uint16_t*>(v_new);
  a.new_pages = new_pages;
  a.k_pool = static_cast<uint8_t*>(k_pool8);
  a.v_pool = static_cast<uint8_t*>(v_pool8);
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.block_table = block_table;
  a.num_kv_heads = desc->num_kv_heads;
  a.head_dim = desc->head_dim;
  a.bt_stride = desc->block_table_stride;
  *args = a;
  return SF_OK;
}

extern "C" sf_status sf_kv_store_fp8(const sf_attn_desc* desc, const sf_store_info* info, const int32_t* work_host,
                                     int32_t* work_dev, const void* k_new, const void* v_new, const int32_t* new_pages,
                                     void* k_pool8, void* v_pool8, float* k_scale, float* v_scale, int32_t* block_table,
                                     void* stream) {
  sf_status st = validate_desc(desc);
  if (st != SF_OK) return st;
  if (!info) return SF_ERR_INVALID_ARG;
  if (info->desc_key != desc_key(desc) || info->num_rows < 0 || info->num_q_rows < 0 ||
      info->work_bytes != uint64_t(info->num_rows) * kItemInts * 4)
    return SF_ERR_PLAN_MISMATCH;
  if (info->num_rows == 0) return SF_OK;
  Store8Args a;
  if ((st = store8_args(desc, work_dev, k_new, v_new, new_pages, k_pool8, v_pool8, k_scale, v_scale, block_table, &a)) !=
      SF_OK)
    return st;
  a.num_rows = info->num_rows;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (work_host && hipMemcpyAsync(work_dev, work_host, info->work_bytes, hipMemcpyHostToDevice, s) != hipSuccess)
    return SF_ERR_HIP;
  return from_hip(launch_store_fp8(a, s));
}

// ---------------------------------------------------------------------------
// weights of cached keys
// ---------------------------------------------------------------------------
namespace {

// A decode step (at most 16 query rows per (sequence, KV head), one row tile) is
// bound by reading the keys: the pairs' keys, in blocks of four pages laid end to end,
// are cut into equal slices, one per wave, two waves per SIMD (one takes as long, three
// per two SIMDs 10 % longer).
// Other calls are made of items, a block of 16 pages of one (sequence, KV head), whose cost is
// the walk over its query rows, 16 per tile. Walks longer than about an eighth of a
// compute unit's share are cut into parts, so that no walk is longer than the rest.
constexpr int32_t kItemPages = 4 * kWeightPages;
constexpr int32_t kStepRows = 16;
constexpr int64_t kStepWavesPerCu = 8;
constexpr int64_t kItemsPerCu = 8;
constexpr int64_t kShortestPart = 8;   // row tiles

// Calls f(sequence, first page, end page, first token that sees the block, parts) for every item.
template <class F>
void for_weight_items(const sf_attn_desc* d, const int32_t* lens, const int32_t* news, int64_t part_tokens, F f) {
  for (int32_t s = 0; s < d->num_seqs; ++s) {
    if (news[s] == 0) continue;
    const int32_t pages = pages_of(lens[s]), prefix = lens[s] - news[s];
    for (int32_t p = 0; p < pages; p += kItemPages) {
      const int32_t t0 = std::max(0, p * kPage - prefix);
      f(s, p, std::min(pages, p + kItemPages), t0, int32_t((news[s] - t0 + part_tokens - 1) / part_tokens));
    }
  }
}

struct WeightRow {
  int32_t v[kWeightInts];
};

// What the rows of a sequence have in common.
struct WeightSeqs {
  const int32_t *lens, *news, *held, *pos;
  WeightRow row(int32_t s, int32_t h, int32_t pb, int32_t pe, int32_t t0, int32_t t1, int32_t slot, int64_t qrow) const {
    const int32_t from = held ? held[s] : lens[s] - news[s];
    return {{s, h, pb, pe, t0, t1, slot, lens[s], lens[s] - news[s], int32_t(qrow), from, pos ? pos[s] : from}};
  }
};

int32_t blocks_of(int32_t tokens) { return (pages_of(tokens) + kWeightPages - 1) / kWeightPages; }

// A decode step's rows: wave w's first segment is row w, the others follow the
// first `waves` rows. Returns the number of rows; work may be NULL.
int64_t plan_weight_steps(const sf_attn_desc* d, const WeightSeqs& q, int64_t blocks, int64_t waves, int32_t* work) {
  int64_t extra = waves, done = 0, wave = 0, qrow = 0;
  int64_t cut = blocks / waves, rest = 0;   // the wave's end, floor(blocks (wave + 1) / waves), stepped without divisions
  const int64_t step = blocks / waves, over = blocks % waves;
  rest = over;
  int64_t at = 0, last = -1;   // row of the next segment; the wave's last row so far
  for (int32_t s = 0; s < d->num_seqs; qrow += q.news[s++]) {
    if (q.news[s] == 0) continue;
    const int32_t pages = pages_of(q.lens[s]), n = blocks_of(q.lens[s]);
    for (int32_t h = 0; h < d->num_kv_heads; ++h)
      for (int32_t b = 0; b < n;) {
        const int32_t take = int32_t(std::min<int64_t>(n - b, cut - done));
        if (work) {
          WeightRow r = q.row(s, h, b * kWeightPages, std::min(pages, (b + take) * kWeightPages), 0, q.news[s], -1, qrow);
          r.v[12] = -1;
          std::memcpy(work + at * kWeightInts, &r, sizeof r);
          if (last >= 0) work[last * kWeightInts + 12] = int32_t(at);
        }
        b += take;
        done += take;
        if (done == cut) {   // the next wave starts
          at = ++wave;
          last = -1;
          cut += step;
          if ((rest += over) >= waves) {
            rest -= waves;
            ++cut;
          }
        } else {
          last = at;
          at = extra++;
        }
      }
  }
  return extra;
}

}  // namespace

extern "C" sf_status sf_key_weights_plan(const sf_attn_desc* desc, const int32_t* seq_lens_host,
                                         const int32_t* q_lens_host, const int32_t* held_lens_host,
                                         const int32_t* first_pos_host, const sf_plan_opts* opts, int32_t* work_host,
                                         uint64_t work_capacity_bytes, sf_weights_info* info) {
  if (!info) return SF_ERR_INVALID_ARG;
  int64_t tokens = 0;
  sf_status st = check_lengths(desc, seq_lens_host, q_lens_host, &tokens);
  if (st != SF_OK) return st;
  if (opts && opts->num_cus < 0) return SF_ERR_INVALID_ARG;
  const WeightSeqs q = {seq_lens_host, q_lens_host, held_lens_host, first_pos_host};
  const int32_t *lens = seq_lens_host, *news = q_lens_host;
  const int64_t g = desc->num_q_heads / desc->num_kv_heads, hkv = desc->num_kv_heads;
  const int64_t cus = opts && opts->num_cus > 0 ? opts->num_cus : kDefaultNumCus;
  int64_t blocks = 0, most = 0;
  for (int32_t s = 0; s < desc->num_seqs; ++s) {
    const int32_t held = held_lens_host ? held_lens_host[s] : lens[s] - news[s];
    const int32_t pos = first_pos_host ? first_pos_host[s] : held;
    if (held < 0 || held > lens[s] || pos < 0 || int64_t(pos) + (lens[s] - held) > INT32_MAX) return SF_ERR_INVALID_ARG;
    if (news[s] == 0) continue;
    blocks += blocks_of(lens[s]) * hkv;
    most = std::max<int64_t>(most, news[s] * g);
  }
  info->num_items = info->num_merge = info->num_slots = info->steps = 0;
  info->item_pages = kItemPages;
  info->num_q_rows = int32_t(tokens);
  info->work_bytes = info->workspace_bytes = 0;
  info->desc_key = desc_key(desc);
  if (blocks == 0) return SF_OK;

  if (most <= kStepRows) {
    const int64_t waves = std::min({kStepWavesPerCu * cus, blocks, kMaxGroups});
    const int64_t rows = plan_weight_steps(desc, q, blocks, waves, nullptr);
    if (rows > INT32_MAX / kWeightInts) return SF_ERR_UNSUPPORTED;
    info->num_items = int32_t(rows);
    info->steps = int32_t(waves);
    info->work_bytes = uint64_t(rows) * kWeightInts * 4;
    if (!work_host) return SF_OK;
    if (work_capacity_bytes < info->work_bytes) return SF_ERR_CAPACITY;
    plan_weight_steps(desc, q, blocks, waves, work_host);
    return SF_OK;
  }

  int64_t tiles = 0;
  for_weight_items(desc, lens, news, INT32_MAX,
                   [&](int32_t s, int32_t, int32_t, int32_t t0, int32_t) { tiles += ((news[s] - t0) * g + 15) / 16; });
  const int64_t part = std::max(kShortestPart, tiles * hkv / (kItemsPerCu * cus));
  const int64_t part_tokens = std::max<int64_t>(1, part * 16 / g);
  int64_t items = 0, merges = 0, slots = 0;
  for_weight_items(desc, lens, news, part_tokens, [&](int32_t, int32_t, int32_t, int32_t, int32_t parts) {
    items += parts * hkv;
    if (parts > 1) merges += hkv, slots += parts * hkv;
  });
  if (std::max(items, merges) >= kMaxGroups) return SF_ERR_UNSUPPORTED;
  info->num_items = int32_t(items);
  info->num_merge = int32_t(merges);
  info->num_slots = int32_t(slots);
  info->work_bytes = uint64_t(items + merges) * kWeightInts * 4;
  info->workspace_bytes = uint64_t(slots) * kItemPages * kPage * 4;
  if (!work_host) return SF_OK;
  if (work_capacity_bytes < info->work_bytes) return SF_ERR_CAPACITY;
  // Items with the most row tiles first (a counting sort; equal ones keep the order sequence, block, KV head, part).
  auto tiles_of = [&](int64_t n) { return size_t((n * g + 15) / 16); };
  auto part_begin = [](int32_t t0, int64_t span, int32_t i, int32_t parts) { return t0 + int32_t(span * i / parts); };
  std::vector<int64_t> at;
  try {
    at.assign(tiles_of(std::min(part_tokens, tokens)) + 1, 0);
  } catch (...) {
    return SF_ERR_CAPACITY;
  }
  for_weight_items(desc, lens, news, part_tokens, [&](int32_t s, int32_t, int32_t, int32_t t0, int32_t parts) {
    for (int32_t i = 0; i < parts; ++i)
      at[tiles_of(part_begin(t0, news[s] - t0, i + 1, parts) - part_begin(t0, news[s] - t0, i, parts))] += hkv;
  });
  for (int64_t i = int64_t(at.size()) - 1, sum = 0; i >= 0; --i) {
    const int64_t n = at[size_t(i)];
    at[size_t(i)] = sum;
    sum += n;
  }
  int32_t* merge = work_host + items * kWeightInts;
  int32_t slot = 0, last = 0;
  int64_t qrow = 0;
  for_weight_items(desc, lens, news, part_tokens, [&](int32_t s, int32_t pb, int32_t pe, int32_t t0, int32_t parts) {
    for (; last < s; ++last) qrow += news[last];
    for (int32_t h = 0; h < hkv; ++h) {
      if (parts > 1) {
        const WeightRow r = q.row(s, h, pb, pe, slot, parts, -1, qrow);
        std::memcpy(merge, &r, sizeof r);
        merge += kWeightInts;
      }
      const int64_t span = news[s] - t0;
      for (int32_t i = 0; i < parts; ++i) {
        const WeightRow r = q.row(s, h, pb, pe, part_begin(t0, span, i, parts), part_begin(t0, span, i + 1, parts),
                                  parts > 1 ? slot++ : -1, qrow);
        std::memcpy(work_host + at[tiles_of(r.v[5] - r.v[4])]++ * kWeightInts, &r, sizeof r);
      }
    }
  });
  return SF_OK;
}

sf_status sf::weight_args(const sf_attn_desc* desc, const sf_weights_info* info, const int32_t* work_dev, const void* q,
                          const float* lse, const void* k_pool, const float* k_scale, const int32_t* block_table,
                          const float* weights, float* weights_out, int32_t* positions, void* workspace,
                          WeightArgs* args) {
  if (!work_dev || !q || !lse || !k_pool || !block_table || !weights || !weights_out) return SF_ERR_INVALID_ARG;
  if (!aligned16(work_dev) || !aligned16(q) || !aligned4(lse) || !aligned16(k_pool) || !aligned4(k_scale) ||
      !aligned4(block_table) || !aligned16(weights) || !aligned16(weights_out) || !aligned16(positions) ||
      (info->workspace_bytes && (!workspace || !aligned16(workspace))))
    return SF_ERR_INVALID_ARG;
  WeightArgs a = {};
  a.items = work_dev;
  a.num_items = info->num_items;
  a.steps = info->steps;
  a.merge_rows = work_dev + int64_t(info->num_items) * kWeightInts;
  a.num_merge = info->num_merge;
  a.q = static_cast<const uint16_t*>(q);
  a.lse = lse;
  a.k_pool = static_cast<const uint16_t*>(k_pool);
  a.k_scale = k_scale;
  a.block_table = block_table;
  a.w_in = weights;
  a.w_out = weights_out;
  a.positions = positions;
  a.part = static_cast<float*>(workspace);
  a.part_keys = info->item_pages * kPage;
  a.num_q_heads = desc->num_q_heads;
  a.num_kv_heads = desc->num_kv_heads;
  a.group = desc->num_q_heads / desc->num_kv_heads;
  a.inv_group = uint32_t((65536 + a.group - 1) / a.group);
  a.head_dim = desc->head_dim;
  a.bt_stride = desc->block_table_stride;
  a.scale_log2 = float(double(desc->softmax_scale) * 1.4426950408889634074);
  *args = a;
  return SF_OK;
}

extern "C" sf_status sf_key_weights(const sf_attn_desc* desc, const sf_weights_info* info, const int32_t* work_host,
                                    int32_t* work_dev, const void* q, const float* lse, const void* k_pool,
                                    const float* k_scale, const int32_t* block_table, const float* weights,
                                    float* weights_out, int32_t* positions, void* workspace, uint64_t workspace_bytes,
                                    void* stream) {
  sf_status st = validate_desc(desc);
  if (st != SF_OK) return st;
  if (!info) return SF_ERR_INVALID_ARG;
  if (info->desc_key != desc_key(desc) || info->num_items < 0 || info->num_merge < 0 || info->num_slots < 0 ||
      info->steps < 0 || info->steps > info->num_items || (info->steps > 0 && info->num_merge > 0) || info->item_pages != kItemPages ||
      info->work_bytes != (uint64_t(info->num_items) + info->num_merge) * kWeightInts * 4 ||
      info->workspace_bytes != uint64_t(info->num_slots) * info->item_pages * kPage * 4)
    return SF_ERR_PLAN_MISMATCH;
  if (info->num_items == 0) return SF_OK;
  WeightArgs a;
  if ((st = weight_args(desc, info, work_dev, q, lse, k_pool, k_scale, block_table, weights, weights_out, positions,
                        workspace, &a)) != SF_OK)
    return st;
  if (workspace_bytes < info->workspace_bytes) return SF_ERR_CAPACITY;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (work_host && hipMemcpyAsync(work_dev, work_host, info->work_bytes, hipMemcpyHostToDevice, s) != hipSuccess)
    return SF_ERR_HIP;
  return from_hip(launch_key_weights(a, s));
}

// ---------------------------------------------------------------------------
// eviction
// ---------------------------------------------------------------------------
namespace {
constexpr int64_t kBusyPage = 4;   // tokens that a kept page takes, on average and at most
}  // namespace

extern "C" sf_status sf_kv_evict_plan(const sf_attn_desc* desc, const int32_t* seq_lens_host,
                                      const int32_t* keep_lens_host, const int32_t* ends_host, int32_t sinks,
                                      int32_t recent, int32_t* work_host, uint64_t work_capacity_bytes,
                                      sf_evict_info* info) {
  if (!info) return SF_ERR_INVALID_ARG;
  sf_status st = validate_desc(desc);
  if (st != SF_OK) return st;
  if (sinks < 0 || recent < 0 || (desc->num_seqs > 0 && (!seq_lens_host || !keep_lens_host))) return SF_ERR_INVALID_ARG;
  const int64_t hkv = desc->num_kv_heads;
  int64_t pages = 0, tails = 0;
  for (int32_t s = 0; s < desc->num_seqs; ++s) {
    const int32_t L = seq_lens_host[s], end = ends_host ? ends_host[s] : L;
    if (L < 0 || L > kMaxTokens || int64_t(L) > int64_t(kPage) * desc->block_table_stride ||
        (L > 0 && desc->num_pages == 0) || end < L)
      return SF_ERR_INVALID_ARG;
    const int32_t n = std::min(keep_lens_host[s], L);
    if (n < 0 || n < std::min<int64_t>(L, int64_t(sinks) + recent)) return SF_ERR_INVALID_ARG;
    pages += pages_of(n);
    tails += std::min(n, L - n);
  }
  // Where most pages take several tokens their moves are the work, and every
  // wave has one tile; runs pay where most pages have little to do (us with runs of 1, 2
  // and 4: long-tail batch halved 494, 505, 522; 64 x 2112 to 2048 76, 46, 40).
  const int32_t run = tails >= kBusyPage * pages ? 1 : run_of(pages);
  int64_t moves = 0;
  int32_t num_long = 0;
  bool boundary = false;
  for (int32_t s = 0; s < desc->num_seqs; ++s) {
    const int32_t n = std::min(keep_lens_host[s], seq_lens_host[s]);
    moves += (pages_of(n) + run - 1) / run;
    num_long += seq_lens_host[s] > kEvictLong;
    boundary = boundary || (n < seq_lens_host[s] && n % kPage != 0);
  }
  if (pages * hkv > INT32_MAX / 2 || tails * hkv > INT32_MAX || int64_t(desc->num_seqs) * hkv >= kMaxGroups ||
      moves >= 4 * kMaxGroups)
    return SF_ERR_UNSUPPORTED;
  info->num_seqs = desc->num_seqs;
  info->num_moves = int32_t(moves);
  info->sinks = sinks;
  info->recent = recent;
  info->boundary = boundary ? 1 : 0;
  info->hole_pages = int32_t(pages * hkv);
  info->num_long = num_long;
  info->reserved = 0;
  info->work_bytes = (uint64_t(desc->num_seqs) + uint64_t(moves)) * kItemInts * 4;
  info->workspace_bytes = align256(uint64_t(pages) * hkv * 8) + uint64_t(tails) * hkv * 4;
  info->desc_key = desc_key(desc);
  if (!work_host) return SF_OK;
  if (work_capacity_bytes < info->work_bytes) return SF_ERR_CAPACITY;
  int32_t *long_row = work_host, *row = work_host + int64_t(num_long) * kItemInts, *move = work_host + int64_t(desc->num_seqs) * kItemInts;
  int64_t hole = 0, tail = 0;
  for (int32_t s = 0; s < desc->num_seqs; ++s) {
    const int32_t L = seq_lens_host[s], n = std::min(keep_lens_host[s], L), np = pages_of(n);
    put_row(L > kEvictLong ? long_row : row, L, n, int32_t(hole), int32_t(tail), ends_host ? ends_host[s] : L, s);
    for (int32_t p = 0; p < np; p += run) put_row(move, s, p, std::min(run, np - p), L, n, int32_t(hole), int32_t(tail));
    hole += np * hkv;
    tail += std::min(n, L - n) * hkv;
  }
  return SF_OK;
}

sf_status sf::evict_args(const sf_attn_desc* desc, const sf_evict_info* info, const int32_t* work_dev, void* k_pool,
                         void* v_pool, float* k_scale, float* v_scale, const int32_t* block_table, const float* weights,
                         const int32_t* positions, float* weights_out, int32_t* positions_out, void* workspace,
                         EvictArgs* args) {
  if ((k_scale == nullptr) != (v_scale == nullptr)) return SF_ERR_INVALID_ARG;
  if (!work_dev || !k_pool || !v_pool || !block_table || !weights || !positions || !weights_out || !positions_out ||
      !workspace)
    return SF_ERR_INVALID_ARG;
  if (!aligned16(work_dev) || !aligned16(k_pool) || !aligned16(v_pool) || !aligned4(k_scale) || !aligned4(v_scale) ||
      !aligned4(block_table) || !aligned16(weights) || !aligned16(positions) || !aligned16(weights_out) ||
      !aligned16(positions_out) || !aligned16(workspace))
    return SF_ERR_INVALID_ARG;
  EvictArgs a = {};
  a.rows = work_dev;
  a.num_seqs = info->num_seqs;
  a.num_moves = info->num_moves;
  a.boundary = info->boundary != 0;
  a.num_long = info->num_long;
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.block_table = block_table;
  a.w_in = weights;
  a.pos_in = positions;
  a.w_out = weights_out;
  a.pos_out = positions_out;
  a.holes = static_cast<uint32_t*>(workspace);
  a.tails = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + align256(uint64_t(info->hole_pages) * 8));
  a.sinks = info->sinks;
  a.recent = info->recent;
  a.num_kv_heads = desc->num_kv_heads;
  a.head_dim = desc->head_dim;
  a.bt_stride = desc->block_table_stride;
  *args = a;
  return SF_OK;
}

sf_status sf::run_evict(const sf_attn_desc* desc, const sf_evict_info* info, const int32_t* work_host, int32_t* work_dev,
                        void* k_pool, void* v_pool, float* k_scale, float* v_scale, const int32_t* block_table,
                        const float* weights, const int32_t* positions, float* weights_out, int32_t* positions_out,
                        void* workspace, uint64_t workspace_bytes, void* stream, int32_t* late_rows) {
  sf_status st = validate_desc(desc);
  if (st != SF_OK) return st;
  if (!info) return SF_ERR_INVALID_ARG;
  if (info->desc_key != desc_key(desc) || info->num_seqs != desc->num_seqs || info->num_moves < 0 || info->sinks < 0 ||
      info->recent < 0 || info->hole_pages < 0 || info->num_long < 0 || info->num_long > info->num_seqs || info->reserved != 0 ||
      info->work_bytes != (uint64_t(info->num_seqs) + uint64_t(info->num_moves)) * kItemInts * 4 ||
      info->workspace_bytes < align256(uint64_t(info->hole_pages) * 8))
    return SF_ERR_PLAN_MISMATCH;
  if (info->num_moves == 0) return SF_OK;
  EvictArgs a;
  if ((st = evict_args(desc, info, work_dev, k_pool, v_pool, k_scale, v_scale, block_table, weights, positions,
                       weights_out, positions_out, workspace, &a)) != SF_OK)
    return st;
  if (workspace_bytes < info->workspace_bytes) return SF_ERR_CAPACITY;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (work_host && hipMemcpyAsync(work_dev, work_host, info->work_bytes, hipMemcpyHostToDevice, s) != hipSuccess)
    return SF_ERR_HIP;
  a.late_rows = late_rows;
  return from_hip(launch_evict(a, s));
}

extern "C" sf_status sf_kv_evict(const sf_attn_desc* desc, const sf_evict_info* info, const int32_t* work_host,
                                 int32_t* work_dev, void* k_pool, void* v_pool, float* k_scale, float* v_scale,
                                 const int32_t* block_table, const float* weights, const int32_t* positions,
                                 float* weights_out, int32_t* positions_out, void* workspace, uint64_t workspace_bytes,
                                 void* stream) {
  return run_evict(desc, info, work_host, work_dev, k_pool, v_pool, k_scale, v_scale, block_table, weights, positions,
                   weights_out, positions_out, workspace, workspace_bytes, stream, nullptr);
}
