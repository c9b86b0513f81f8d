// Sampling: entry points. The rules are stated in sf_decode_attn.h.
#include <algorithm>
#include <cstdint>

#include "sf_internal.h"

static_assert(sizeof(sf_sample_desc) == 24, "sf_sample_desc layout is part of the ABI");

using namespace sf;

namespace {

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

sf_status check_sample(const sf_sample_desc* d) {
  if (!d || d->num_rows < 0 || d->vocab < 1 || d->row_stride < d->vocab || d->reserved != 0) return SF_ERR_INVALID_ARG;
  if (d->dtype < 0 || d->dtype > 2 || d->vocab > SF_SAMPLE_MAX_VOCAB) return SF_ERR_UNSUPPORTED;
  // a launch takes fewer than 2^32 threads, a grid's second dimension 2^16 - 1 blocks
  if (int64_t(d->num_rows) * sample_chunks(*d) >= (int64_t(1) << 24) || d->num_rows >= 1 << 22) return SF_ERR_UNSUPPORTED;
  return SF_OK;
}

}  // namespace

// Elements per workgroup of the first launch: long chunks read with the fewest
// instructions, short ones give a few rows enough workgroups. Rows of 131072 bf16 with a top-p, short and long:
// 8 rows 81 and 85 us, 24 106 and 102, 40 123 and 106, 128 224 and 175 (without cuts 19, 19, 20 and 30, all within 1.3).
int32_t sf::sample_chunk(const sf_sample_desc& d) {
  return int64_t(d.num_rows) * d.vocab >= int64_t(512) * kSampleChunk ? kSampleChunk : kSampleSmallChunk;
}

// A row may start inside a 16-byte piece, which is one more.
int32_t sf::sample_chunks(const sf_sample_desc& d) {
  const int32_t per = d.dtype == 0 ? 4 : 8;
  const int32_t pieces = (d.vocab + per - 1) / per + 1, chunk = sample_chunk(d) / per;
  return (pieces + chunk - 1) / chunk;
}

namespace {

// The workspace: chunks, rows, a counter, bins and lists, groups.
struct Layout {
  uint64_t rows, taken, bins, lists, groups, bytes;
  int32_t places;
  explicit Layout(const sf_sample_desc& d) {
    const uint64_t n = uint64_t(d.num_rows), chunks = n * uint64_t(sample_chunks(d));
    rows = align256(chunks * sizeof(SampleChunk));
    taken = align256(rows + n * sizeof(SampleRow));
    bins = taken + 256;
    places = std::min(d.num_rows, kSamplePlaces);
    lists = bins + uint64_t(places) * kSampleBins * 8;
    groups = lists + uint64_t(places) * kSampleList * 8;
    bytes = groups + chunks * uint64_t(sample_chunk(d) / kSampleGroup) * 4;
  }
};

}  // namespace

extern "C" sf_status sf_sample_workspace(const sf_sample_desc* desc, uint64_t* bytes) {
  const sf_status st = check_sample(desc);
  if (st != SF_OK) return st;
  if (!bytes) return SF_ERR_INVALID_ARG;
  *bytes = Layout(*desc).bytes;
  return SF_OK;
}

extern "C" sf_status sf_sample(const sf_sample_desc* desc, const void* logits, const float* temperature,
                               const int32_t* top_k, const float* top_p, const float* min_p, const float* uniform,
                               int32_t* token, float* logprob, float* kept, void* workspace, uint64_t workspace_bytes,
                               void* stream) {
  uint64_t need = 0;
  const sf_status st = sf_sample_workspace(desc, &need);
  if (st != SF_OK) return st;
  if (desc->num_rows == 0) return SF_OK;
  if (!logits || !uniform || !token || !workspace) return SF_ERR_INVALID_ARG;
  if (!aligned(logits, desc->dtype == 0 ? 4 : 2) || !aligned(workspace, 16) || !aligned(temperature, 4) ||
      !aligned(top_k, 4) || !aligned(top_p, 4) || !aligned(min_p, 4) || !aligned(uniform, 4) || !aligned(token, 4) ||
      !aligned(logprob, 4) || !aligned(kept, 4))
    return SF_ERR_INVALID_ARG;
  if (workspace_bytes < need) return SF_ERR_CAPACITY;
  SampleArgs a = {};
  a.logits = logits;
  a.num_rows = desc->num_rows;
  a.vocab = desc->vocab;
  a.row_stride = desc->row_stride;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.uniform = uniform;
  a.token = token;
  a.logprob = logprob;
  a.kept = kept;
  a.chunk = sample_chunk(*desc);
  a.num_chunks = sample_chunks(*desc);
  char* ws = static_cast<char*>(workspace);
  const Layout at(*desc);
  a.chunks = reinterpret_cast<SampleChunk*>(ws);
  if (top_k || top_p || min_p) {
    a.rows = reinterpret_cast<SampleRow*>(ws + at.rows);
    a.places = at.places;
    a.taken = reinterpret_cast<uint32_t*>(ws + at.taken);
    a.bins = reinterpret_cast<uint64_t*>(ws + at.bins);
    a.lists = reinterpret_cast<uint64_t*>(ws + at.lists);
    a.groups = reinterpret_cast<float*>(ws + at.groups);
  }
  return launch_sample(a, desc->dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? SF_OK : SF_ERR_HIP;
}
