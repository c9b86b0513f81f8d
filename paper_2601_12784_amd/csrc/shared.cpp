// A decode step of groups that share their first tokens: host planner and
// entry points. The rule is stated in sf_decode_attn.h.
#include <algorithm>
#include <climits>
#include <cstdint>
#include <cstring>
#include <new>
#include <vector>

#include "sf_internal.h"

static_assert(sizeof(sf_shared_info) == 48, "sf_shared_info layout is part of the ABI");

using namespace sf;

namespace {

constexpr int32_t kMinChunk = 4;   // pages per wave, at least
constexpr int64_t kSegmentPages = 2;   // what a segment's start costs, in pages
constexpr uint64_t kSharedKey = 0x536861726564ull;
constexpr int64_t kMaxMerge = int64_t(1) << 23;   // workgroups of 256 threads: 2^32 threads are too many for a launch

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
int32_t pages_of(int32_t tokens) { return (tokens + kPage - 1) / kPage; }

// Waves of a workgroup that hold a prompt's rows together, of `blocks` in all, and
// the sets of them that take its key blocks in turns.
int32_t blocks_together(int32_t blocks) { return std::min(blocks, kSharedWaves); }
int32_t splits_of(int32_t blocks) { return blocks == 1 ? 1 : kSharedWaves / blocks_together(blocks); }

// What a page costs, ns of one wave. One that a wave reads for itself (a prompt of one block, too): its latency, where
// waves of prompts leave memory to spare. One prompt of 32760 tokens with 64 members (32/8 heads) at 1450, 1700 and
// 2450: 95, 89 and 93 us; 8 of 8000 with 8 (40/8, fp8) at 900, 1000 and 1300: 84, 81 and 85.
double own_cost(const sf_attn_desc& d, bool fp8) { return fp8 ? 1000 : d.head_dim == 64 ? 950 : 1700; }
// Of a prompt whose rows several waves hold: the time of its blocks of rows on their waves' matrix and vector units, at least
// the staging by eight waves. Head dim 64 at 0.45, 0.63 and 1.0 of it (14/2 heads, prompts x members: 16 x 16 of 2048 tokens,
// 8 x 40 of 4000, 1 x 256 of 4000): 49, 74 and 61 us; 46, 61 and 53; 43, 65 and 47. Own pages there in fp8 at 700, 1000 and
// 1400: 46, 58 and 45 us; 44, 60 and 45; 46, 67 and 56.
double page_cost(const sf_attn_desc& d, int32_t blocks, bool fp8) {
  if (blocks == 1) return own_cost(d, fp8);
  return std::max(2000.0, (fp8 ? 1300 : 980) * (d.head_dim == 64 ? 0.63 : 1.0) * blocks);
}
// Own pages take up to kShort times their latency where all bytes at kBytesPerNs take longer than all waves' work;
// prompts, read ahead further, feel that less. 16 prompts of 2048 tokens with 16 members (28/4; half as much work
// as bytes) at 1.45 and 1.3: 109 and 102 us.
constexpr double kShort = 1.3, kBytesPerNs = 5000;

// A group whose prompt is read once.
struct Prompt {
  int32_t first;     // sequence of row 0
  int32_t source;    // its block-table row
  int32_t pages;
  int32_t rows;
  int32_t tiles;
  int32_t blocks;
  int64_t start;     // first page of its KV head 0 in its track
  int64_t unit;      // index of its KV head 0 among all prompts' units
};

// Prompts with the same number of blocks, laid end to end, KV head by KV head.
struct Track {
  int32_t blocks;
  int64_t pages = 0;
  double cost = 0;         // ns of all waves
  int64_t columns = 0;     // runs; blocks > 1: of workgroups
  std::vector<int32_t> prompts;
};

struct Unit {
  int32_t base;    // partial row of its part 0
  int32_t parts;
};

// Runs [at(j), at(j + 1)) of `pages` pages, j < columns.
struct Runs {
  int64_t pages, columns;
  int64_t at(int64_t j) const { return pages * j / columns; }
  int64_t of(int64_t page) const { return ((page + 1) * columns - 1) / pages; }
  int32_t parts(int64_t begin, int64_t end) const { return int32_t(of(end - 1) - of(begin) + 1); }
};

struct Scratch {
  std::vector<Prompt> prompts;
  std::vector<Track> tracks;
  std::vector<Unit> units;       // of prompts
  std::vector<int32_t> prompt_of;    // per sequence: index, -1
  std::vector<Unit> own;         // per (sequence, KV head)
  std::vector<int64_t> start;    // per sequence: its first place among the own pages'
};

void put_fields(int32_t* row, int32_t seq0, int32_t source, int32_t kvh, int32_t pb, int32_t pe, int32_t end, int32_t slot,
                int32_t row0, int32_t rows, int32_t group, int32_t together = 0, int32_t split = 0) {
  const int32_t f[kSharedInts] = {0, 0, seq0, source, kvh, pb, pe, end, slot, row0, rows, together, split,
                                  seq0 + row0 / group, row0 % group, 0};
  std::memcpy(row, f, sizeof f);
}

sf_status plan(const sf_attn_desc* desc, const int32_t* lens, int32_t num_groups, const int32_t* offsets,
               const int32_t* shared, bool fp8, const sf_plan_opts* opts, int32_t* work, uint64_t capacity,
               sf_shared_info* info) {
  sf_status st = validate_desc(desc);
  if (st != SF_OK) return st;
  const int32_t n = desc->num_seqs, hkv = desc->num_kv_heads, g = desc->num_q_heads / hkv;
  if (!info || num_groups < 0 || (n > 0 && !lens) || (num_groups > 0 && (!offsets || !shared))) return SF_ERR_INVALID_ARG;
  if (num_groups == 0 ? n != 0 : offsets[0] != 0 || offsets[num_groups] != n) return SF_ERR_INVALID_ARG;
  int32_t cus = kDefaultNumCus, least = kMinChunk;
  if (opts) {
    if (opts->num_cus < 0 || opts->min_chunk_pages < 0) return SF_ERR_INVALID_ARG;
    if (opts->num_cus) cus = opts->num_cus;
    if (opts->min_chunk_pages) least = opts->min_chunk_pages;
  }
  if (cus > 1 << 20) return SF_ERR_INVALID_ARG;
  for (int32_t i = 0; i < num_groups; ++i)
    if (offsets[i + 1] < offsets[i] || offsets[i + 1] > n || shared[i] < 0) return SF_ERR_INVALID_ARG;
  for (int32_t s = 0; s < n; ++s) {
    if (lens[s] < 0 || int64_t(lens[s]) > int64_t(kPage) * desc->block_table_stride || lens[s] > INT32_MAX - kPage)
      return SF_ERR_INVALID_ARG;
    if (lens[s] > 0 && desc->num_pages == 0) return SF_ERR_INVALID_ARG;
  }
  if (int64_t(n) * hkv >= kMaxMerge || int64_t(n) * desc->num_q_heads > INT32_MAX / kPage) return SF_ERR_UNSUPPORTED;

  static thread_local Scratch t;
  t.prompts.clear();
  t.prompt_of.assign(size_t(n), -1);
  t.start.resize(size_t(n));
  t.tracks.clear();
  int64_t num_units = 0;
  for (int32_t i = 0; i < num_groups; ++i) {
    int32_t first = -1, last = -1, live = 0;
    for (int32_t s = offsets[i]; s < offsets[i + 1]; ++s) {
      if (lens[s] == 0) continue;
      if (lens[s] < shared[i]) return SF_ERR_INVALID_ARG;
      if (first < 0) first = s;
      last = s;
      ++live;
    }
    const int32_t pages = shared[i] / kPage;
    if (live < 2 || pages == 0) continue;
    Prompt p = {};
    p.first = p.source = first;
    p.pages = pages;
    p.rows = (last - first + 1) * g;
    p.tiles = (p.rows + 15) / 16;
    p.blocks = (p.tiles + kSharedTiles - 1) / kSharedTiles;
    if (p.tiles > 1) p.blocks = std::max(p.blocks, 2);
    p.blocks = p.blocks > 4 ? (p.blocks + kSharedWaves - 1) / kSharedWaves * kSharedWaves : p.blocks > 2 ? 4 : p.blocks;
    p.unit = num_units;
    num_units += hkv;
    for (int32_t s = first; s <= last; ++s)
      if (lens[s] > 0) t.prompt_of[s] = int32_t(t.prompts.size());
    auto track = std::find_if(t.tracks.begin(), t.tracks.end(), [&](const Track& x) { return x.blocks == p.blocks; });
    if (track == t.tracks.end()) {
      t.tracks.push_back({});
      track = t.tracks.end() - 1;
      track->blocks = p.blocks;
    }
    p.start = track->pages;
    track->pages += int64_t(pages) * hkv;
    track->cost += double(pages) * hkv * page_cost(*desc, p.blocks, fp8);
    track->prompts.push_back(int32_t(t.prompts.size()));
    t.prompts.push_back(p);
  }
  // many blocks first: a prompt's blocks then fill whole workgroups
  std::sort(t.tracks.begin(), t.tracks.end(), [](const Track& x, const Track& y) { return x.blocks > y.blocks; });
  // What sequences have to themselves, end to end: of each (sequence, KV head), kSegmentPages places for its start, then its pages.
  int64_t own_pages = 0, own_places = 0;
  for (int32_t s = 0; s < n; ++s) {
    const int32_t pages = pages_of(lens[s]) - (t.prompt_of[s] >= 0 ? t.prompts[t.prompt_of[s]].pages : 0);
    t.start[s] = own_places;
    own_pages += int64_t(pages) * hkv;
    if (pages) own_places += (pages + kSegmentPages) * hkv;
  }
  const double own_work = double(own_places) * own_cost(*desc, fp8);
  double alone_work = own_work, all_work = own_work, all_pages = double(own_pages);
  for (const Track& x : t.tracks) {
    all_work += x.cost;
    if (x.blocks == 1) alone_work += x.cost;
    all_pages += double(x.pages);
  }
  const double bytes = all_pages * kPage * desc->head_dim * (fp8 ? 2 : 4);
  const double at_memory = bytes / kBytesPerNs * kSharedWaves * cus;   // ns of all waves
  const double slower = all_work > 0.0 ? std::min(kShort, std::max(1.0, at_memory / all_work)) : 1.0;
  for (Track& x : t.tracks)
    if (x.blocks == 1) x.cost *= slower;
  const double cost = all_work + alone_work * (slower - 1.0);
  // waves: two per SIMD, fewer rather than thinner runs
  const int64_t waves = std::max<int64_t>(1, std::min<int64_t>(int64_t(kSharedWaves) * cus, int64_t(cost / (own_cost(*desc, fp8) * least))));
  // Prompts of several blocks take whole workgroups, the first ones; the other
  // waves (prompts of one block, then the sequences' own pages) are spread over the rest.
  int64_t groups = 0, alone = 0;
  for (Track& x : t.tracks) {
    const double share = double(waves) * x.cost / cost;
    if (x.blocks == 1) {
      x.columns = std::max<int64_t>(1, std::min<int64_t>(x.pages, int64_t(share)));
      alone += x.columns;
    } else {
      const int32_t each = (x.blocks + kSharedWaves - 1) / kSharedWaves;
      x.columns = std::max<int64_t>(1, std::min<int64_t>(x.pages, int64_t(share / kSharedWaves / each)));
      // Runs that end with every KV head's pages spare a second start: 27 for each of 8 KV heads 89 us, 221 for all 8 95.
      const int64_t units = int64_t(x.prompts.size()) * hkv, over = x.columns % units;
      const bool alike = x.pages == units * t.prompts[size_t(x.prompts[0])].pages;   // (or none is cut right but by chance)
      if (alike && over * 32 <= x.columns && x.columns > over) x.columns -= over;
      groups += x.columns * each;
    }
  }
  const int64_t own_columns =
      own_pages == 0 ? 0 : std::max<int64_t>(1, std::min(own_pages, waves - groups * kSharedWaves - alone));
  alone += own_columns;
  const bool whole = groups > 0 || alone > cus;
  const int64_t alone_groups = std::max((alone + kSharedWaves - 1) / kSharedWaves, std::min(alone, std::max<int64_t>(0, cus - groups)));
  const int64_t workers = whole ? (groups + alone_groups) * kSharedWaves : alone;

  // parts and partial rows
  int64_t rows = 0, items = 0, merges = 0;
  t.units.resize(size_t(num_units));
  for (const Track& x : t.tracks) {
    const Runs runs = {x.pages, x.columns};
    for (int32_t i : x.prompts) {
      const Prompt& p = t.prompts[i];
      for (int32_t h = 0; h < hkv; ++h) {
        const int64_t begin = p.start + int64_t(h) * p.pages;
        const int32_t parts = runs.parts(begin, begin + p.pages);
        const int32_t splits = splits_of(x.blocks);
        t.units[size_t(p.unit + h)] = {int32_t(std::min<int64_t>(rows, INT32_MAX)), parts * splits};
        rows += int64_t(parts) * splits * p.rows;
        items += int64_t(parts) * splits * p.blocks;
      }
    }
  }
  const Runs own_runs = {own_places, own_columns};
  t.own.resize(size_t(n) * hkv);
  for (int32_t s = 0; s < n; ++s) {
    const bool has_prompt = t.prompt_of[s] >= 0;
    const int32_t pages = pages_of(lens[s]) - (has_prompt ? t.prompts[t.prompt_of[s]].pages : 0);
    for (int32_t h = 0; h < hkv; ++h) {
      Unit& u = t.own[size_t(s) * hkv + h];
      const int64_t begin = t.start[s] + h * (pages + kSegmentPages) + kSegmentPages;
      u.parts = pages ? own_runs.parts(begin, begin + pages) : 0;
      u.base = -1;
      items += u.parts;
      if (u.parts == 1 && !has_prompt) continue;
      u.base = int32_t(std::min<int64_t>(rows, INT32_MAX));
      rows += int64_t(u.parts) * g;
      ++merges;
    }
  }
  if (rows > INT32_MAX || items > INT32_MAX / kSharedInts || workers > INT32_MAX / kSharedInts) return SF_ERR_UNSUPPORTED;
  info->num_workers = int32_t(workers);
  info->num_work = int32_t(items);
  info->num_merge = int32_t(merges);
  info->num_rows = int32_t(rows);
  info->workers_per_group = whole ? kSharedWaves : 1;
  info->reserved = 0;
  info->work_bytes = uint64_t(workers + items) * kSharedInts * 4 + uint64_t(merges) * kSharedMergeInts * 4;
  info->workspace_bytes = rows ? align256(uint64_t(rows) * desc->head_dim * 4) + uint64_t(rows) * 4 : 0;
  info->desc_key = desc_key(desc) ^ kSharedKey;
  if (!work) return SF_OK;
  if (capacity < info->work_bytes) return SF_ERR_CAPACITY;

  int32_t* const table = work;
  int32_t* const list = work + workers * kSharedInts;
  int32_t* merge = list + items * kSharedInts;
  int32_t item = 0;
  int64_t worker = 0;
  auto close_worker = [&](int32_t first) {
    int32_t* row = table + worker * kSharedInts;
    if (item > first)
      std::memcpy(row, list + int64_t(first) * kSharedInts, kSharedInts * 4);
    else
      std::memset(row, 0, kSharedInts * 4);
    row[0] = first;
    row[1] = item - first;
    ++worker;
  };
  // Waves alone go to every workgroup of theirs in turn, as many as fit one behind the other.
  const int64_t per_group = whole && alone_groups ? (alone + alone_groups - 1) / alone_groups : 1;
  int64_t lonely = 0;
  auto next_alone = [&] {
    if (whole && ++lonely == per_group) {
      for (; worker % kSharedWaves; lonely = 0) close_worker(item);
      lonely = 0;
    }
  };
  for (const Track& x : t.tracks) {
    const Runs runs = {x.pages, x.columns};
    const int32_t together = x.blocks == 1 ? 0 : blocks_together(x.blocks), splits = splits_of(x.blocks);
    auto emit = [&](int64_t col, int32_t block, int32_t split) {
      const int32_t first = item;
      int64_t page = runs.at(col);
      const int64_t end = runs.at(col + 1);
      size_t lo = 0, hi = x.prompts.size();   // the prompt that holds the page
      while (hi - lo > 1) {
        const size_t mid = (lo + hi) / 2;
        if (t.prompts[x.prompts[mid]].start <= page) lo = mid;
        else hi = mid;
      }
      for (; page < end; ++lo) {
        const Prompt& p = t.prompts[x.prompts[lo]];
        const int32_t row0 = int32_t(int64_t(p.tiles) * block / p.blocks) * 16;
        const int32_t row1 = std::min(p.rows, int32_t(int64_t(p.tiles) * (block + 1) / p.blocks) * 16);
        while (page < end && page < p.start + int64_t(p.pages) * hkv) {
          const int32_t h = int32_t((page - p.start) / p.pages);
          const int64_t begin = p.start + int64_t(h) * p.pages;
          const int64_t stop = std::min(end, begin + p.pages);
          const int32_t part = int32_t(col - runs.of(begin)) * splits + split;
          put_fields(list + int64_t(item++) * kSharedInts, p.first, p.source, h, int32_t(page - begin), int32_t(stop - begin),
                     p.pages * kPage, t.units[size_t(p.unit + h)].base + part * p.rows + row0, row0, row1 - row0, g,
                     together, split);
          page = stop;
        }
      }
      close_worker(first);
    };
    if (x.blocks == 1) {
      for (int64_t c = 0; c < x.columns; ++c) {
        emit(c, 0, 0);
        next_alone();
      }
      continue;
    }
    // Workgroups go round the eight XCDs: a run of several workgroups takes every eighth,
    // so that they find each other's pages in one L2.
    const int32_t each = (x.blocks + kSharedWaves - 1) / kSharedWaves;
    for (int64_t c0 = 0; c0 < x.columns; c0 += 8)
      for (int32_t k = 0; k < each; ++k)
        for (int64_t c = c0; c < std::min(x.columns, c0 + 8); ++c)
          for (int32_t w = 0; w < kSharedWaves; ++w) emit(c, k * kSharedWaves + w % together, w / together);
  }
  if (own_columns > 0) {
    int64_t col = 0;
    int32_t first = item;
    auto close_until = [&](int64_t place) {
      for (; col < own_columns && own_runs.at(col + 1) <= place; ++col) {
        close_worker(first);
        next_alone();
        first = item;
      }
    };
    for (int32_t s = 0; s < n; ++s) {
      const int32_t skip = t.prompt_of[s] >= 0 ? t.prompts[t.prompt_of[s]].pages : 0;
      const int32_t pages = pages_of(lens[s]) - skip;
      for (int32_t h = 0; h < hkv && pages > 0; ++h) {
        const Unit& u = t.own[size_t(s) * hkv + h];
        const int64_t begin = t.start[s] + h * (pages + kSegmentPages) + kSegmentPages, end = begin + pages;
        int64_t at = begin;
        close_until(at);
        for (int32_t part = 0; at < end; ++part) {
          const int64_t stop = std::min(end, own_runs.at(col + 1));
          put_fields(list + int64_t(item++) * kSharedInts, s, s, h, skip + int32_t(at - begin), skip + int32_t(stop - begin),
                     lens[s], u.base < 0 ? -1 : u.base + part * g, 0, g, g);
          at = stop;
          close_until(at);
        }
      }
    }
  }
  while (worker < workers) close_worker(item);
  for (int32_t s = 0; s < n; ++s) {
    const Prompt* p = t.prompt_of[s] >= 0 ? &t.prompts[t.prompt_of[s]] : nullptr;
    for (int32_t h = 0; h < hkv; ++h) {
      const Unit& u = t.own[size_t(s) * hkv + h];
      if (u.base < 0) continue;
      const Unit* q = p ? &t.units[size_t(p->unit + h)] : nullptr;
      const int32_t row[kSharedMergeInts] = {s, h, u.base, u.parts, q ? q->base + (s - p->first) * g : 0, q ? q->parts : 0,
                                             q ? p->rows : 0, 0};
      std::memcpy(merge, row, sizeof row);
      merge += kSharedMergeInts;
    }
  }
  return SF_OK;
}

}  // namespace

extern "C" sf_status sf_shared_attn_plan(const sf_attn_desc* desc, const int32_t* seq_lens_host, int32_t num_groups,
                                         const int32_t* group_offsets_host, const int32_t* shared_lens_host, int32_t fp8,
                                         const sf_plan_opts* opts, int32_t* work_host, uint64_t work_capacity_bytes,
                                         sf_shared_info* info) {
  if ((fp8 | 1) != 1) return SF_ERR_INVALID_ARG;
  try {
    return plan(desc, seq_lens_host, num_groups, group_offsets_host, shared_lens_host, fp8 != 0, opts, work_host,
                work_capacity_bytes, info);
  } catch (const std::bad_alloc&) {
    return SF_ERR_HIP;
  }
}

sf_status sf::run_shared(const sf_attn_desc* desc, const sf_shared_info* info, const int32_t* work_host, int32_t* work_dev,
                         const void* q, const void* k_pool, const void* v_pool, const float* k_scale,
                         const float* v_scale, const int32_t* block_table, void* out, int32_t out_bf16, float* lse,
                         void* workspace, uint64_t workspace_bytes, void* stream, int32_t* late_rows) {
  const sf_status st = validate_desc(desc);
  if (st != SF_OK) return st;
  if (!info || (out_bf16 | 1) != 1) return SF_ERR_INVALID_ARG;
  if (info->desc_key != (desc_key(desc) ^ kSharedKey) || info->num_workers < 0 || info->num_work < 0 || info->num_merge < 0 ||
      info->num_rows < 0 || (info->workers_per_group != 1 && info->workers_per_group != kSharedWaves) ||
      info->work_bytes != (uint64_t(info->num_workers) + uint64_t(info->num_work)) * kSharedInts * 4 +
                              uint64_t(info->num_merge) * kSharedMergeInts * 4 ||
      info->workspace_bytes !=
          (info->num_rows ? align256(uint64_t(info->num_rows) * desc->head_dim * 4) + uint64_t(info->num_rows) * 4 : 0))
    return SF_ERR_PLAN_MISMATCH;
  if (info->num_workers == 0 && info->num_merge == 0) return SF_OK;
  if (!work_dev || !q || !block_table || !out || (desc->num_pages > 0 && (!k_pool || !v_pool))) return SF_ERR_INVALID_ARG;
  if (!aligned16(work_dev) || !aligned16(q) || !aligned16(k_pool) || !aligned16(v_pool) || !aligned16(out) ||
      !aligned4(block_table) || !aligned4(lse) || !aligned16(workspace))
    return SF_ERR_INVALID_ARG;
  if ((k_scale == nullptr) != (v_scale == nullptr) || !aligned4(k_scale) || !aligned4(v_scale)) return SF_ERR_INVALID_ARG;
  if (workspace_bytes < info->workspace_bytes || (info->workspace_bytes && !workspace)) return SF_ERR_CAPACITY;
  SharedArgs a = {};
  a.workers = work_dev;
  a.items = work_dev + int64_t(info->num_workers) * kSharedInts;
  a.num_workers = info->num_workers;
  a.workers_per_group = info->workers_per_group;
  a.merge_rows = a.items + int64_t(info->num_work) * kSharedInts;
  a.num_merge = info->num_merge;
  if (late_rows) {
    a.copy_src = a.merge_rows;
    a.copy_dst = late_rows;
    a.copy_ints = info->num_merge * kSharedMergeInts;
    a.merge_rows = late_rows;
  }
  a.q = static_cast<const uint16_t*>(q);
  a.k_pool = static_cast<const uint16_t*>(k_pool);
  a.v_pool = static_cast<const uint16_t*>(v_pool);
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.block_table = block_table;
  a.out = out;
  a.out_bf16 = out_bf16 != 0;
  a.lse = lse;
  a.part_o = static_cast<float*>(workspace);
  a.part_lse = reinterpret_cast<float*>(static_cast<char*>(workspace) + align256(uint64_t(info->num_rows) * desc->head_dim * 4));
  a.num_q_heads = desc->num_q_heads;
  a.num_kv_heads = desc->num_kv_heads;
  a.group = desc->num_q_heads / desc->num_kv_heads;
  a.group_inverse = 65536 / a.group + 1;
  a.head_dim = desc->head_dim;
  a.bt_stride = desc->block_table_stride;
  a.scale_log2 = float(double(desc->softmax_scale) * 1.4426950408889634074);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (work_host && hipMemcpyAsync(work_dev, work_host, info->work_bytes, hipMemcpyHostToDevice, s) != hipSuccess)
    return SF_ERR_HIP;
  return launch_shared(a, s) == hipSuccess ? SF_OK : SF_ERR_HIP;
}

extern "C" sf_status sf_shared_attn(const sf_attn_desc* desc, const sf_shared_info* info, const int32_t* work_host,
                                    int32_t* work_dev, const void* q, const void* k_pool, const void* v_pool,
                                    const float* k_scale, const float* v_scale, const int32_t* block_table, void* out,
                                    int32_t out_bf16, float* lse, void* workspace, uint64_t workspace_bytes, void* stream) {
  return sf::run_shared(desc, info, work_host, work_dev, q, k_pool, v_pool, k_scale, v_scale, block_table, out, out_bf16,
                        lse, workspace, workspace_bytes, stream, nullptr);
}
