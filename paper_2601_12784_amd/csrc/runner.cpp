// Native per-step runner: plan -> attention (-> merge) in one call.
//
// A rollout instance runs one batched decode step after another (App. B.1:
// each step generates one token per running trajectory), so the host work
// between two steps is on the critical path once the kernels are short:
// small batches, late steps of a long-tail batch, an fp8 cache. This object
// keeps that work native. It owns a ring of pinned host buffers that the
// planner writes into and the kernels read in place (mapped host memory,
// zero-copy), the split-K workspace, and a few events:
//   - a slot is rewritten only after the step that read it has ended;
//   - nothing else orders the steps, so the host plans step i + 1 while the
//     kernels of step i run.
// An event recorded on the stream after every step delayed the next step's
// first launch by ~4.4 us (the marker's own dispatch; 2 % of a long-tail
// step), so one event marks a run of kMarkEvery steps on one stream instead;
// the ring holds kRing > kMarkEvery slots, so the run that holds a slot's
// last step is always marked before the slot comes round again.
// A separate upload (a copy stream, a device work list and a cross-stream
// wait) cost more per step than the kernels' in-place reads of the list, and
// how much more depended on whether the two streams shared a hardware queue.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <new>

#include "sf_internal.h"

static_assert(sizeof(sf_runner_memory) == 56, "sf_runner_memory layout is part of the ABI");
static_assert(sizeof(sf_runner_extras) == 56, "sf_runner_extras layout is part of the ABI");

namespace {

constexpr int kRing = 32;
constexpr int kMarkEvery = 16;
constexpr int kMarks = 4;
// Without a store launch to copy the rows, a copy launch (about 4 us) pays from
// about two rounds of workgroups on, each starting with a read over PCIe.
constexpr int kExtendCopyParts = 512;
const hipStream_t kNoStream = reinterpret_cast<hipStream_t>(~uintptr_t(0));   // no call yet
static_assert(kMarkEvery < kRing, "a slot's last step must be marked before the slot comes round again");

struct Pinned {
  int32_t* ptr = nullptr;          // host address (the planner writes here)
  const int32_t* dev = nullptr;    // the same memory as the kernels address it
  uint64_t bytes = 0;
  uint64_t last_step = 0;          // the step that last read it
  bool used = false;
  bool in_arena = false;           // part of sf_runner::arena, not an allocation of its own
};

// An event recorded on one stream after steps [begin, end), all on that stream.
struct Mark {
  hipEvent_t ev = nullptr;
  uint64_t begin = 0, end = 0;
  bool valid = false;
};

// Memory lent by sf_runner_extend's caller. Every few calls (a run: half the
// slots) the last launch of the call completes an event, which stands for the
// calls since the event before. Nothing is recorded on a stream after the call
// that was given it, so the caller may destroy it between calls: where calls
// without an event have to be waited for (the next call is on another stream,
// other memory comes, the runner goes), the device is. A runner that has seen
// two streams gives every call its event. (On every call of a single stream the
// events cost up to 2 us: three prompts of up to 61 tokens 16.4 against 14.4.)
struct Lent {
  void* pinned = nullptr;
  const char* pinned_dev = nullptr;   // the same memory as the kernels address it
  int32_t slots = 0;
  uint64_t slot_bytes = 0;
  void* device = nullptr;             // of the last call that lent it for longer than the call
  uint64_t device_bytes = 0;
  uint64_t next = 0;                  // slots go round
  hipEvent_t done[kRing] = {};        // created with the first call of the slot that takes one
  bool used[kRing] = {};              // a call whose end has not been waited for read the slot
  int event[kRing] = {};              // the slot whose event stands for that call; -1: none yet
  int unmarked = 0;                   // calls without an event so far
  bool streams = false;               // calls came on more than one stream
  hipStream_t last_stream = kNoStream;   // of the last call (compared, never used)
};

}  // namespace

struct sf_runner {
  sf_attn_desc shape;      // heads, head_dim, page size (per-step fields are overwritten)
  sf_plan_opts opts;
  int device = 0;
  Pinned ring[kRing];
  void* arena = nullptr;   // one allocation that sf_runner_reserve cut into slots
  Mark marks[kMarks];
  uint64_t num_marks = 0;  // marks recorded so far (the next one reuses marks[num_marks % kMarks])
  uint64_t unmarked = 0;   // steps [unmarked, steps) have no mark yet
  hipStream_t last_stream = nullptr;
  hipEvent_t order = nullptr;   // on the last stream, for a call on another
  void* workspace = nullptr;
  uint64_t workspace_bytes = 0;
  Lent lent;
  uint64_t steps = 0;
  sf_plan_info last;
};

namespace {

// Records a mark after the unmarked steps, on the stream they ran on. The
// mark it reuses is waited for first, so a recycled event never stands for
// steps of another run.
sf_status mark_steps(sf_runner* r) {
  if (r->unmarked == r->steps) return SF_OK;
  Mark& m = r->marks[r->num_marks % kMarks];
  if (m.valid && hipEventSynchronize(m.ev) != hipSuccess) return SF_ERR_HIP;
  m.valid = false;
  if (hipEventRecord(m.ev, r->last_stream) != hipSuccess) return SF_ERR_HIP;
  m.begin = r->unmarked;
  m.end = r->steps;
  m.valid = true;
  r->unmarked = r->steps;
  ++r->num_marks;
  return SF_OK;
}

// Returns once step u (< steps) has ended on the GPU.
sf_status wait_step(sf_runner* r, uint64_t u) {
  if (u >= r->unmarked) {
    sf_status st = mark_steps(r);
    if (st != SF_OK) return st;
  }
  for (auto& m : r->marks)
    if (m.valid && m.begin <= u && u < m.end) return hipEventSynchronize(m.ev) == hipSuccess ? SF_OK : SF_ERR_HIP;
  return SF_OK;  // its mark was waited for and reused: the step has ended
}

// Returns once every step so far has ended.
sf_status wait_all(sf_runner* r) {
  sf_status st = mark_steps(r);
  for (auto& m : r->marks)
    if (m.valid && hipEventSynchronize(m.ev) != hipSuccess) st = SF_ERR_HIP;
  return st;
}

// Called only when no step in flight reads the slot (its last step has ended).
sf_status grow_pinned(Pinned& p, uint64_t bytes) {
  if (p.bytes >= bytes) return SF_OK;
  if (p.ptr && !p.in_arena && hipHostFree(p.ptr) != hipSuccess) return SF_ERR_HIP;
  p.in_arena = false;
  p.ptr = nullptr;
  p.dev = nullptr;
  p.bytes = 0;
  const uint64_t want = bytes + bytes / 4 + 4096;
  if (hipHostMalloc(reinterpret_cast<void**>(&p.ptr), want, hipHostMallocDefault) != hipSuccess) return SF_ERR_HIP;
  void* dev = nullptr;
  if (hipHostGetDevicePointer(&dev, p.ptr, 0) != hipSuccess) {
    (void)hipHostFree(p.ptr);
    p.ptr = nullptr;
    return SF_ERR_HIP;
  }
  p.dev = static_cast<const int32_t*>(dev);
  p.bytes = want;
  return SF_OK;
}

// The workspace grows only when nothing in flight can still use it: growing
// waits for the runner's steps and the stream (sf_runner_reserve does it
// ahead of the steps).
sf_status grow_device(sf_runner* r, void** ptr, uint64_t* have, uint64_t bytes, hipStream_t main) {
  if (*have >= bytes) return SF_OK;
  sf_status st = wait_all(r);
  if (st != SF_OK) return st;
  if (hipStreamSynchronize(main) != hipSuccess) return SF_ERR_HIP;
  if (*ptr && hipFree(*ptr) != hipSuccess) return SF_ERR_HIP;
  *ptr = nullptr;
  *have = 0;
  const uint64_t want = bytes + bytes / 4 + 4096;
  if (hipMalloc(ptr, want) != hipSuccess) return SF_ERR_HIP;
  *have = want;
  return SF_OK;
}

bool same_shape(const sf_runner* r, const sf_attn_desc* desc) {
  return desc->num_q_heads == r->shape.num_q_heads && desc->num_kv_heads == r->shape.num_kv_heads &&
         desc->head_dim == r->shape.head_dim && desc->page_size == r->shape.page_size;
}

bool capturing(hipStream_t stream) {
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  return hipStreamIsCapturing(stream, &status) == hipSuccess && status != hipStreamCaptureStatusNone;
}

// A call on another stream than the last one comes after the runner's calls so
// far on the device, too: all of them share the workspace, and an eviction's lists
// there are indexes. Where either stream is being captured the wait would tie the
// graph to work outside of it, or that work to the graph.
sf_status follow_last_stream(sf_runner* r, hipStream_t main) {
  if (r->steps == 0 || main == r->last_stream) return SF_OK;
  if (capturing(main) || capturing(r->last_stream)) return mark_steps(r);   // a mark stands for steps of one stream
  // an event of its own: unlike the marks' it publishes what the calls wrote
  if (mark_steps(r) == SF_OK && hipEventRecord(r->order, r->last_stream) == hipSuccess &&
      hipStreamWaitEvent(main, r->order, 0) == hipSuccess)
    return SF_OK;
  // the caller may have destroyed the last stream: the device is waited for
  (void)hipGetLastError();
  if (hipDeviceSynchronize() != hipSuccess) return SF_ERR_HIP;
  for (auto& p : r->ring) p.used = false;
  r->unmarked = r->steps;
  return SF_OK;
}

// Takes the next ring slot for a call on `main`: after the step that last read
// it has ended.
sf_status open_slot(sf_runner* r, hipStream_t main, Pinned** slot) {
  Pinned& pin = r->ring[r->steps % kRing];
  sf_status st = pin.used ? wait_step(r, pin.last_step) : SF_OK;
  if (st != SF_OK) return st;
  pin.used = false;
  if ((st = follow_last_stream(r, main)) != SF_OK) return st;
  *slot = &pin;
  return SF_OK;
}

// Counts a call whose launches may have been enqueued and read the slot, with
// what they returned.
sf_status close_slot(sf_runner* r, hipStream_t main, Pinned& pin, sf_status st) {
  pin.used = true;
  pin.last_step = r->steps;
  r->last_stream = main;
  ++r->steps;
  if (r->steps - r->unmarked >= kMarkEvery && mark_steps(r) != SF_OK) {
    // Without the mark nothing orders a later rewrite of these slots after
    // the steps' reads: wait for the stream instead.
    (void)hipStreamSynchronize(main);
    for (auto& p : r->ring) p.used = false;
    r->unmarked = r->steps;
    if (st == SF_OK) st = SF_ERR_HIP;
  }
  return st;
}

// Slots are reused by waiting on the host, which a graph's replays would not.
sf_status not_capturing(hipStream_t main) {
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(main, &status) != hipSuccess) return SF_ERR_HIP;
  return status == hipStreamCaptureStatusNone ? SF_OK : SF_ERR_UNSUPPORTED;
}

// Makes the runner's device current for a call, and the caller's again after it.
struct OnDevice {
  int before = -1;
  sf_status st = SF_OK;
  explicit OnDevice(int device) {
    int now = device;
    if (hipGetDevice(&now) != hipSuccess || (now != device && hipSetDevice(device) != hipSuccess)) st = SF_ERR_HIP;
    if (st == SF_OK && now != device) before = now;
  }
  ~OnDevice() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

// A call of a runner besides its steps: plan(work, capacity) into the next slot
// (grown and planned again if it is too small; bytes() afterwards are what the
// slot must hold), `workspace` bytes, then launch(slot as the kernels address it).
template <class Plan, class Bytes, class Workspace, class Launch>
sf_status run_in_slot(sf_runner* r, hipStream_t main, Plan plan, Bytes bytes, Workspace workspace, Launch launch) {
  const OnDevice on(r->device);
  if (on.st != SF_OK) return on.st;
  sf_status st = not_capturing(main);
  Pinned* pin = nullptr;
  if (st != SF_OK || (st = open_slot(r, main, &pin)) != SF_OK) return st;
  st = plan(pin->ptr, pin->bytes);
  if (st == SF_ERR_CAPACITY || (st == SF_OK && pin->bytes < bytes())) {
    if ((st = grow_pinned(*pin, bytes())) != SF_OK) return st;
    st = plan(pin->ptr, pin->bytes);
  }
  if (st != SF_OK) return st;
  if (bytes() == 0) return SF_OK;
  if ((st = grow_device(r, &r->workspace, &r->workspace_bytes, workspace(), main)) != SF_OK) return st;
  return close_slot(r, main, *pin, launch(pin->ptr, pin->dev));
}

// Waits for the device where calls have no event.
sf_status wait_unmarked(Lent& l) {
  if (l.unmarked == 0) return SF_OK;
  if (hipDeviceSynchronize() != hipSuccess) return SF_ERR_HIP;
  std::fill(l.used, l.used + kRing, false);
  l.unmarked = 0;
  return SF_OK;
}

// Returns once the call that last read the lent slot has ended.
sf_status wait_slot(Lent& l, int slot) {
  if (!l.used[slot]) return SF_OK;
  if (l.event[slot] < 0) return wait_unmarked(l);
  if (hipEventSynchronize(l.done[l.event[slot]]) != hipSuccess) return SF_ERR_HIP;
  l.used[slot] = false;
  return SF_OK;
}

// Returns once every call on the lent memory has ended.
sf_status wait_lent(Lent& l) {
  sf_status st = wait_unmarked(l);
  for (int i = 0; i < kRing; ++i)
    if (wait_slot(l, i) != SF_OK) st = SF_ERR_HIP;
  return st;
}

}  // namespace

extern "C" sf_status sf_runner_create(const sf_attn_desc* shape, const sf_plan_opts* opts, sf_runner** out) {
  if (!out) return SF_ERR_INVALID_ARG;
  *out = nullptr;
  if (!shape) return SF_ERR_INVALID_ARG;
  sf_attn_desc probe = *shape;
  probe.num_seqs = 0;
  probe.block_table_stride = probe.block_table_stride > 0 ? probe.block_table_stride : 1;
  probe.num_pages = probe.num_pages >= 0 ? probe.num_pages : 0;
  sf_status st = sf::validate_desc(&probe);
  if (st != SF_OK) return st;
  if (opts && (opts->xcd_parity_skew < -sf::kMaxParitySkew || opts->xcd_parity_skew > sf::kMaxParitySkew))
    return SF_ERR_INVALID_ARG;
  sf_runner* r = new (std::nothrow) sf_runner();
  if (!r) return SF_ERR_HIP;
  r->shape = probe;
  if (opts) r->opts = *opts;
  else std::memset(&r->opts, 0, sizeof r->opts);
  if (hipGetDevice(&r->device) != hipSuccess) {
    delete r;
    return SF_ERR_HIP;
  }
  // The events only order the host's reuse of a slot after the GPU's reads
  // of it; they publish no GPU writes, so they skip the system-scope fence.
  for (auto& m : r->marks)
    if (hipEventCreateWithFlags(&m.ev, hipEventDisableTiming | hipEventDisableSystemFence) != hipSuccess)
      st = SF_ERR_HIP;
  if (hipEventCreateWithFlags(&r->order, hipEventDisableTiming) != hipSuccess) st = SF_ERR_HIP;
  if (st != SF_OK) {
    sf_runner_destroy(r);
    return st;
  }
  *out = r;
  return SF_OK;
}

// Teardown cannot report errors: every call is made, whatever the others return.
extern "C" void sf_runner_destroy(sf_runner* r) {
  if (!r) return;
  // a garbage collector may be here with any device current
  int current = r->device;
  (void)hipGetDevice(&current);
  if (current != r->device) (void)hipSetDevice(r->device);
  // Steps not yet marked ran on the caller's stream, which may be gone by
  // now: nothing is recorded on it here, the device is waited for instead.
  if (r->unmarked < r->steps) (void)hipDeviceSynchronize();
  for (auto& m : r->marks) {
    if (m.ev && m.valid) (void)hipEventSynchronize(m.ev);
    if (m.ev) (void)hipEventDestroy(m.ev);
  }
  if (r->order) (void)hipEventDestroy(r->order);
  (void)wait_lent(r->lent);
  for (auto ev : r->lent.done)
    if (ev) (void)hipEventDestroy(ev);
  for (auto& p : r->ring)
    if (p.ptr && !p.in_arena) (void)hipHostFree(p.ptr);
  if (r->arena) (void)hipHostFree(r->arena);
  if (r->workspace) {
    (void)hipDeviceSynchronize();
    (void)hipFree(r->workspace);
  }
  if (current != r->device) (void)hipSetDevice(current);
  delete r;
}

extern "C" sf_status sf_runner_step(sf_runner* r, const sf_attn_desc* desc, const int32_t* seq_lens_host,
                                    const void* q, const void* k_pool, const void* v_pool,
                                    const int32_t* block_table, float* out, float* lse,
                                    const sf_runner_extras* extras, void* stream, sf_plan_info* info_out) {
  if (!r || !desc || (desc->num_seqs > 0 && !seq_lens_host)) return SF_ERR_INVALID_ARG;
  if (!same_shape(r, desc)) return SF_ERR_INVALID_ARG;
  const bool fp8 = extras && extras->k_scale;
  const bool store = fp8 && extras->k_new;   // an appending step over an fp8 cache: stored, then attended
  const bool append = extras && extras->k_new && !store;
  if (append && !lse) return SF_ERR_INVALID_ARG;
  hipStream_t main = static_cast<hipStream_t>(stream);

  // 1. plan into the next ring slot (after the step that last read it has
  //    ended); grow it and plan again only if the plan does not fit
  Pinned* slot = nullptr;
  sf_status st = open_slot(r, main, &slot);
  if (st != SF_OK) return st;
  Pinned& pin = *slot;
  // Appending: after the work list, copies of the rows the merge launch acts
  // on (pairs with one segment and len > 0, at most one per item), then
  // new_pages. The work list ends with the combine rows, so the merge
  // launch's rows are one contiguous range, which the attention launch
  // copies to device memory (RowCopy). Over an fp8 cache: the rows of the
  // store launch (one per sequence with a token), then new_pages.
  const uint64_t pages_bytes = append || store ? (uint64_t(desc->num_seqs) * 4 + 31) / 32 * 32 : 0;
  sf_plan_info info;
  const sf::StepKind kind = fp8 ? sf::StepKind::kFp8 : append ? sf::StepKind::kAppend : sf::StepKind::kPlain;
  st = sf::decode_plan_runner(desc, seq_lens_host, &r->opts, kind, pin.ptr, pin.bytes, &info);
  auto need = [&]() {
    return info.work_bytes + pages_bytes + (append ? uint64_t(info.num_work) : store ? uint64_t(desc->num_seqs) : 0) * 32;
  };
  if (st == SF_ERR_CAPACITY || (st == SF_OK && pin.bytes < need())) {
    if ((st = grow_pinned(pin, need())) != SF_OK) return st;
    st = sf::decode_plan_runner(desc, seq_lens_host, &r->opts, kind, pin.ptr, pin.bytes, &info);
  }
  if (st != SF_OK) return st;
  const bool shared = info.workers_per_group > sf::kSharedGroups;
  if (shared) info.workers_per_group -= sf::kSharedGroups;
  int32_t num_single = 0;
  uint64_t pages_off = info.work_bytes;
  if (append && desc->num_seqs > 0) {
    if (!extras->new_pages_host) return SF_ERR_INVALID_ARG;
    char* base = reinterpret_cast<char*>(pin.ptr);
    const int32_t* items = pin.ptr + sf::table_rows(info.num_workers) * sf::kItemInts;
    int32_t* singles = reinterpret_cast<int32_t*>(base + info.work_bytes);
    for (int32_t i = 0; i < info.num_work; ++i) {
      const int32_t* row = items + int64_t(i) * sf::kItemInts;
      if (row[7] == 1 && row[4] > 0)
        std::memcpy(singles + int64_t(num_single++) * sf::kItemInts, row, sf::kItemInts * 4);
    }
    pages_off = info.work_bytes + uint64_t(num_single) * 32;
    std::memcpy(base + pages_off, extras->new_pages_host, uint64_t(desc->num_seqs) * 4);
  }
  int32_t num_store = 0;
  if (store && desc->num_seqs > 0) {
    if (!extras->new_pages_host) return SF_ERR_INVALID_ARG;
    char* base = reinterpret_cast<char*>(pin.ptr);
    int32_t* row = reinterpret_cast<int32_t*>(base + info.work_bytes);
    for (int32_t s = 0; s < desc->num_seqs; ++s) {
      const int32_t L = seq_lens_host[s];
      if (L <= 0) continue;
      const int32_t r8[sf::kItemInts] = {s, (L - 1) / sf::kPage, 1, L - 1, L, s, 0, 0};
      std::memcpy(row + int64_t(num_store++) * sf::kItemInts, r8, sizeof r8);
    }
    pages_off = info.work_bytes + uint64_t(num_store) * 32;
    std::memcpy(base + pages_off, extras->new_pages_host, uint64_t(desc->num_seqs) * 4);
  }
  if (info_out) *info_out = info;
  r->last = info;
  if (info.num_workers == 0) return SF_OK;
  sf::Store8Args store_args = {};
  if (num_store > 0) {
    const char* base = reinterpret_cast<const char*>(pin.dev);
    if ((st = sf::check_step_args(desc, &info, pin.dev, q, k_pool, v_pool, block_table, out, lse, nullptr, nullptr,
                                  nullptr, extras->k_scale, extras->v_scale)) != SF_OK ||
        (st = sf::store8_args(desc, reinterpret_cast<const int32_t*>(base + info.work_bytes), extras->k_new,
                              extras->v_new, reinterpret_cast<const int32_t*>(base + pages_off),
                              const_cast<void*>(k_pool), const_cast<void*>(v_pool), const_cast<float*>(extras->k_scale),
                              const_cast<float*>(extras->v_scale), const_cast<int32_t*>(block_table), &store_args)) != SF_OK)
      return st;
    store_args.num_rows = num_store;
  }

  // 2. workspace (grown only while idle): the partial results, then the
  //    device copy of what the merge launch reads from the ring: the combine
  //    rows and, appending, the single rows and new_pages (contiguous there)
  const uint64_t rows_off = sf::align256(info.workspace_bytes);
  const int64_t rows_ints = (int64_t(info.num_combine) + (append ? num_single : 0)) * sf::kItemInts;
  const int64_t copy_ints = rows_ints + (append && desc->num_seqs > 0 ? int64_t(pages_bytes / 4) : 0);
  if ((st = grow_device(r, &r->workspace, &r->workspace_bytes, rows_off + uint64_t(copy_ints) * 4, main)) != SF_OK)
    return st;
  int32_t* work = const_cast<int32_t*>(pin.dev);
  const sf::RowCopy copy = {work + (sf::table_rows(info.num_workers) + info.num_work) * sf::kItemInts,
                            reinterpret_cast<int32_t*>(static_cast<char*>(r->workspace) + rows_off),
                            int32_t(copy_ints), append ? int32_t(info.num_combine) * sf::kItemInts : -1,
                            append && desc->num_seqs > 0 ? int32_t(rows_ints) : -1};
  const sf::RowCopy* cp = copy_ints > 0 ? &copy : nullptr;

  // 3. kernels on the caller's stream (the caller's events, if any, take the
  //    attention kernel's own start and end times)
  void* ev0 = extras ? extras->attn_start : nullptr;
  void* ev1 = extras ? extras->attn_end : nullptr;
  // From here on a launch may have been enqueued that reads the slot, so the
  // step counts (and is marked in its turn) whatever the launches return.
  if (append) {
    const char* wbase = reinterpret_cast<const char*>(work);
    st = sf::decode_attn_append_rows(desc, &info, work, q, extras->k_new, extras->v_new,
                                     reinterpret_cast<const int32_t*>(wbase + pages_off),
                                     reinterpret_cast<const int32_t*>(wbase + info.work_bytes), num_single,
                                     const_cast<void*>(k_pool), const_cast<void*>(v_pool),
                                     const_cast<int32_t*>(block_table), out, lse, r->workspace,
                                     r->workspace_bytes, stream, cp, ev0, ev1, shared);
  } else {
    if (num_store > 0 && sf::launch_store_fp8(store_args, main) != hipSuccess) return close_slot(r, main, pin, SF_ERR_HIP);
    st = sf::decode_attn_rows(desc, &info, work, q, k_pool, v_pool, fp8 ? extras->k_scale : nullptr,
                              fp8 ? extras->v_scale : nullptr, block_table, out, lse, r->workspace,
                              r->workspace_bytes, stream, cp, ev0, ev1, shared, store);
  }
  return close_slot(r, main, pin, st);
}

extern "C" sf_status sf_runner_store_fp8(sf_runner* r, const sf_attn_desc* desc, const int32_t* seq_lens_host,
                                         const int32_t* q_lens_host, const void* k_new, const void* v_new,
                                         const int32_t* new_pages_host, void* k_pool8, void* v_pool8, float* k_scale,
                                         float* v_scale, int32_t* block_table, void* stream) {
  if (!r || !desc || !same_shape(r, desc)) return SF_ERR_INVALID_ARG;
  hipStream_t main = static_cast<hipStream_t>(stream);
  sf_store_info info = {};
  const uint64_t pages_bytes = new_pages_host && desc->num_seqs > 0 ? (uint64_t(desc->num_seqs) * 4 + 31) / 32 * 32 : 0;
  return run_in_slot(
      r, main,
      [&](int32_t* work, uint64_t bytes) {
        return sf_kv_store_fp8_plan(desc, seq_lens_host, q_lens_host, work, bytes, &info);
      },
      [&] { return info.num_rows > 0 ? info.work_bytes + pages_bytes : 0; }, [] { return uint64_t(0); },
      [&](int32_t* host, const int32_t* dev) {
        const int32_t* pages = nullptr;
        if (pages_bytes) {
          std::memcpy(host + info.work_bytes / 4, new_pages_host, uint64_t(desc->num_seqs) * 4);
          pages = dev + info.work_bytes / 4;
        }
        return sf_kv_store_fp8(desc, &info, nullptr, const_cast<int32_t*>(dev), k_new, v_new, pages, k_pool8, v_pool8,
                               k_scale, v_scale, block_table, stream);
      });
}

extern "C" sf_status sf_runner_shared(sf_runner* r, const sf_attn_desc* desc, const int32_t* seq_lens_host,
                                      int32_t num_groups, const int32_t* group_offsets_host,
                                      const int32_t* shared_lens_host, const void* q, const void* k_pool,
                                      const void* v_pool, const float* k_scale, const float* v_scale,
                                      const int32_t* block_table, void* out, int32_t out_bf16, float* lse, void* stream) {
  if (!r || !desc || !same_shape(r, desc)) return SF_ERR_INVALID_ARG;
  sf_shared_info info = {};
  auto merge_bytes = [&] { return uint64_t(info.num_merge) * sf::kSharedMergeInts * 4; };
  return run_in_slot(
      r, static_cast<hipStream_t>(stream),
      [&](int32_t* work, uint64_t bytes) {
        return sf_shared_attn_plan(desc, seq_lens_host, num_groups, group_offsets_host, shared_lens_host, k_scale != nullptr,
                                   &r->opts, work, bytes, &info);
      },
      [&] { return info.work_bytes; },
      // the merge rows' device copy lies behind the call's own workspace
      [&] { return sf::align256(info.workspace_bytes) + merge_bytes(); },
      [&](int32_t*, const int32_t* dev) {
        char* rows = static_cast<char*>(r->workspace) + sf::align256(info.workspace_bytes);
        return sf::run_shared(desc, &info, nullptr, const_cast<int32_t*>(dev), q, k_pool, v_pool, k_scale, v_scale,
                              block_table, out, out_bf16, lse, r->workspace, r->workspace_bytes, stream,
                              info.num_workers > 0 ? reinterpret_cast<int32_t*>(rows) : nullptr);
      });
}

extern "C" sf_status sf_runner_rotary_store(sf_runner* r, const sf_attn_desc* desc, const sf_rotary_desc* rotary,
                                            const int32_t* seq_lens_host, const int32_t* q_lens_host,
                                            const int32_t* first_pos_host, const uint64_t* turns, const void* q,
                                            int64_t q_stride, void* q_out, int64_t q_out_stride, const void* k_new,
                                            int64_t k_stride, const void* v_new, int64_t v_stride,
                                            const int32_t* new_pages_host, void* k_pool, void* v_pool,
                                            int32_t* block_table, void* stream) {
  if (!r || !desc || !same_shape(r, desc)) return SF_ERR_INVALID_ARG;
  sf_store_info info = {};
  const uint64_t pages_bytes = new_pages_host && desc->num_seqs > 0 ? (uint64_t(desc->num_seqs) * 4 + 31) / 32 * 32 : 0;
  return run_in_slot(
      r, static_cast<hipStream_t>(stream),
      [&](int32_t* work, uint64_t bytes) {
        return sf_rotary_store_plan(desc, seq_lens_host, q_lens_host, first_pos_host, work, bytes, &info);
      },
      [&] { return info.num_rows > 0 ? info.work_bytes + pages_bytes : 0; }, [] { return uint64_t(0); },
      [&](int32_t* host, const int32_t* dev) {
        const int32_t* pages = nullptr;
        if (pages_bytes) {
          std::memcpy(host + info.work_bytes / 4, new_pages_host, uint64_t(desc->num_seqs) * 4);
          pages = dev + info.work_bytes / 4;
        }
        return sf_rotary_store(desc, rotary, &info, nullptr, const_cast<int32_t*>(dev), turns, q, q_stride, q_out,
                               q_out_stride, k_new, k_stride, v_new, v_stride, pages, k_pool, v_pool, block_table, stream);
      });
}

extern "C" sf_status sf_runner_key_weights(sf_runner* r, const sf_attn_desc* desc, const int32_t* seq_lens_host,
                                           const int32_t* q_lens_host, const int32_t* held_lens_host,
                                           const int32_t* first_pos_host, const void* q, const float* lse,
                                           const void* k_pool, const float* k_scale, const int32_t* block_table,
                                           const float* weights, float* weights_out, int32_t* positions, void* stream) {
  if (!r || !desc || !same_shape(r, desc)) return SF_ERR_INVALID_ARG;
  sf_weights_info info = {};
  return run_in_slot(
      r, static_cast<hipStream_t>(stream),
      [&](int32_t* work, uint64_t bytes) {
        return sf_key_weights_plan(desc, seq_lens_host, q_lens_host, held_lens_host, first_pos_host, &r->opts, work,
                                   bytes, &info);
      },
      [&] { return info.work_bytes; }, [&] { return info.workspace_bytes; },
      [&](int32_t*, const int32_t* dev) {
        return sf_key_weights(desc, &info, nullptr, const_cast<int32_t*>(dev), q, lse, k_pool, k_scale, block_table,
                              weights, weights_out, positions, r->workspace, r->workspace_bytes, stream);
      });
}

// Every workgroup of an eviction's moves begins with a row, which the ring's host
// memory gives late: the selection, which waits most of its time, copies the list to the device.
// Up to this size: 8, 64, 200 and 480 sequences of 2112 fp8 tokens take 20.4, 39.8, 96.4 and 259 us with the
// copy (32 to 495 KiB) and 22.8, 44.5, 104.7 and 279 without; the long-tail batch (700 KiB) 507 and 495.
constexpr uint64_t kLateBytes = 512 << 10;

extern "C" sf_status sf_runner_evict(sf_runner* r, const sf_attn_desc* desc, const int32_t* seq_lens_host,
                                     const int32_t* keep_lens_host, const int32_t* ends_host, int32_t sinks,
                                     int32_t recent, void* k_pool, void* v_pool, float* k_scale, float* v_scale,
                                     const int32_t* block_table, const float* weights, const int32_t* positions,
                                     float* weights_out, int32_t* positions_out, void* stream) {
  if (!r || !desc || !same_shape(r, desc)) return SF_ERR_INVALID_ARG;
  sf_evict_info info = {};
  return run_in_slot(
      r, static_cast<hipStream_t>(stream),
      [&](int32_t* work, uint64_t bytes) {
        return sf_kv_evict_plan(desc, seq_lens_host, keep_lens_host, ends_host, sinks, recent, work, bytes, &info);
      },
      [&] { return info.num_moves > 0 ? info.work_bytes : 0; },
      // the copy lies behind the call's own workspace
      [&] { return sf::align256(info.workspace_bytes) + info.work_bytes; },
      [&](int32_t*, const int32_t* dev) {
        char* rows = info.work_bytes <= kLateBytes ? static_cast<char*>(r->workspace) + sf::align256(info.workspace_bytes) : nullptr;
        return sf::run_evict(desc, &info, nullptr, const_cast<int32_t*>(dev), k_pool, v_pool, k_scale, v_scale,
                             block_table, weights, positions, weights_out, positions_out, r->workspace,
                             r->workspace_bytes, stream, reinterpret_cast<int32_t*>(rows));
      });
}

// Extend attention, in memory that the caller lends: the pinned part is cut
// into slots that the plans go round, the device part is the workspace.
static sf_status runner_extend(sf_runner* r, const sf_attn_desc* desc, const int32_t* seq_lens_host,
                               const int32_t* q_lens_host, const void* q, const void* k_new,
                               const void* v_new, void* k_pool, void* v_pool, const int32_t* block_table,
                               float* out, float* lse, sf_runner_memory* memory, void* stream,
                               sf_extend_info* info_out, float* k_scale = nullptr, float* v_scale = nullptr,
                               bool out_bf16 = false) {
  if (!r || !desc || !info_out || !memory) return SF_ERR_INVALID_ARG;
  if (!same_shape(r, desc)) return SF_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(memory->pinned) | reinterpret_cast<uintptr_t>(memory->device)) & 15u)
    return SF_ERR_INVALID_ARG;
  hipStream_t main = static_cast<hipStream_t>(stream);
  // Slots are reused by waiting for events on the host, which a graph's
  // replays would not: a capturing stream is left to sf_extend_attn.
  sf_status st = not_capturing(main);
  if (st != SF_OK) return st;

  // Other memory than the last call's: nothing may still use either.
  const bool per_call = memory->device_per_call == 1;
  Lent& lent = r->lent;
  const uint64_t slot_bytes = memory->slots > 0 ? memory->pinned_bytes / memory->slots / 32 * 32 : 0;
  if (!per_call && (lent.device != memory->device || lent.device_bytes != memory->device_bytes)) {
    if ((st = wait_lent(lent)) != SF_OK) return st;
    lent.device = memory->device;
    lent.device_bytes = memory->device_bytes;
  }
  if (lent.pinned != memory->pinned || lent.slots != memory->slots || lent.slot_bytes != slot_bytes) {
    if ((st = wait_lent(lent)) != SF_OK) return st;
    if (memory->slots < 0 || memory->slots > kRing || (memory->pinned == nullptr) != (memory->slots == 0))
      return SF_ERR_INVALID_ARG;
    void* dev = nullptr;
    if (memory->pinned && hipHostGetDevicePointer(&dev, memory->pinned, 0) != hipSuccess) return SF_ERR_HIP;
    lent.pinned = memory->pinned;
    lent.pinned_dev = static_cast<const char*>(dev);
    lent.slots = memory->slots;
    lent.slot_bytes = slot_bytes;
    lent.next = 0;
  }
  const int slot = lent.slots > 0 ? lent.next % lent.slots : 0;
  if ((st = wait_slot(lent, slot)) != SF_OK) return st;

  const bool store = k_new != nullptr;
  sf::ExtendPlan plan;
  try {
    int32_t* work = reinterpret_cast<int32_t*>(static_cast<char*>(lent.pinned) + uint64_t(slot) * lent.slot_bytes);
    st = sf::extend_plan_parts(desc, seq_lens_host, q_lens_host, r->opts.num_cus, store, work, lent.slot_bytes,
                               &plan, info_out);
  } catch (const std::bad_alloc&) {
    return SF_ERR_HIP;
  }
  if (st != SF_OK && st != SF_ERR_CAPACITY) return st;
  // Device memory: partial results, then the device copy of the part and
  // merge rows. The store launch makes that copy, or a launch of its own where
  // enough workgroups would otherwise read their row over PCIe.
  const uint64_t row_ints = (uint64_t(plan.num_parts) + plan.num_merge) * sf::kItemInts;
  if (row_ints > INT32_MAX) return SF_ERR_INVALID_ARG;
  const uint64_t lse_off = sf::align256(uint64_t(plan.num_slots) * plan.rows * desc->head_dim * 4);
  const uint64_t rows_off = lse_off + sf::align256(uint64_t(plan.num_slots) * plan.rows * 4);
  const bool copy = store || plan.num_parts > kExtendCopyParts;
  const uint64_t device_bytes = rows_off + (copy ? row_ints * 4 : 0);
  memory->need_slot = plan.bytes();
  memory->need_device = device_bytes;
  if (st == SF_ERR_CAPACITY || memory->device_bytes < device_bytes) return SF_ERR_CAPACITY;
  if (plan.num_parts == 0) return SF_OK;
  const int32_t* work_dev = reinterpret_cast<const int32_t*>(lent.pinned_dev + uint64_t(slot) * lent.slot_bytes);
  sf::ExtendArgs a;
  if ((st = sf::extend_args(desc, work_dev, q, k_new, v_new, k_pool, v_pool, block_table, out, lse, &a)) != SF_OK)
    return st;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.out_bf16 = out_bf16;
  sf::Store8Args store8 = {};
  if (k_scale && store &&
      (st = sf::store8_args(desc, work_dev, k_new, v_new, nullptr, k_pool, v_pool, k_scale, v_scale,
                            const_cast<int32_t*>(block_table), &store8)) != SF_OK)
    return st;
  // Calls of another stream may still use the device memory: they are waited
  // for (calls on one stream are in order by themselves).
  if (main != lent.last_stream && lent.last_stream != kNoStream) {
    lent.streams = true;
    if ((st = wait_lent(lent)) != SF_OK) return st;
  }
  lent.last_stream = main;
  // The events skip HIP's system-scope fence, as the marks do.
  const bool mark = lent.streams || lent.unmarked + 1 >= lent.slots / 2;
  if (mark && !lent.done[slot] &&
      hipEventCreateWithFlags(&lent.done[slot], hipEventDisableTiming | hipEventDisableSystemFence) != hipSuccess) {
    lent.done[slot] = nullptr;
    return SF_ERR_HIP;
  }
  char* ws = static_cast<char*>(memory->device);
  a.parts = true;
  a.num_items = plan.num_parts;
  a.part_rows = plan.rows;
  a.part_o = reinterpret_cast<float*>(ws);
  a.part_lse = reinterpret_cast<float*>(ws + lse_off);
  a.num_merge = plan.num_merge;
  a.num_store = plan.num_store;
  a.store_rows = work_dev + row_ints;
  if (copy) {
    a.copy_src = work_dev;
    a.copy_dst = reinterpret_cast<int32_t*>(ws + rows_off);
    a.copy_ints = int32_t(row_ints);
    a.items = a.copy_dst;
  }
  a.merge_rows = a.items + int64_t(plan.num_parts) * sf::kItemInts;
  hipError_t launched = hipSuccess;
  if (k_scale && store) {   // a store launch of its own, with the same rows and side job
    store8.rows = a.store_rows;
    store8.num_rows = plan.num_store;
    store8.copy_src = a.copy_src;
    store8.copy_dst = a.copy_dst;
    store8.copy_ints = a.copy_ints;
    a.k_new = a.v_new = nullptr;
    a.num_store = a.copy_ints = 0;
    launched = sf::launch_store_fp8(store8, main);
  }
  if (launched == hipSuccess) launched = sf::launch_extend(a, main, mark ? lent.done[slot] : nullptr);
  if (launched != hipSuccess) {
    // An earlier launch of the call may read the slot, with no event behind it.
    (void)hipStreamSynchronize(main);
    return SF_ERR_HIP;
  }
  lent.used[slot] = true;
  lent.event[slot] = -1;
  ++lent.unmarked;
  if (mark) {
    for (int i = 0; i < kRing; ++i)
      if (lent.used[i] && lent.event[i] < 0) lent.event[i] = slot;
    lent.unmarked = 0;
  }
  ++lent.next;
  return SF_OK;
}

extern "C" sf_status sf_runner_extend(sf_runner* r, const sf_attn_desc* desc, const int32_t* seq_lens_host,
                                      const int32_t* q_lens_host, const void* q, const void* k_new,
                                      const void* v_new, void* k_pool, void* v_pool, const int32_t* block_table,
                                      float* out, float* lse, sf_runner_memory* memory, void* stream,
                                      sf_extend_info* info_out) {
  return runner_extend(r, desc, seq_lens_host, q_lens_host, q, k_new, v_new, k_pool, v_pool, block_table, out, lse,
                       memory, stream, info_out);
}

extern "C" sf_status sf_runner_extend_fp8(sf_runner* r, const sf_attn_desc* desc, const int32_t* seq_lens_host,
                                          const int32_t* q_lens_host, const void* q, const void* k_new,
                                          const void* v_new, void* k_pool8, void* v_pool8, const int32_t* block_table,
                                          void* out, float* lse, sf_runner_memory* memory, void* stream,
                                          sf_extend_info* info_out, float* k_scale, float* v_scale, int32_t out_bf16) {
  if (!k_scale || !v_scale || ((reinterpret_cast<uintptr_t>(k_scale) | reinterpret_cast<uintptr_t>(v_scale)) & 3u) ||
      (out_bf16 | 1) != 1)
    return SF_ERR_INVALID_ARG;
  return runner_extend(r, desc, seq_lens_host, q_lens_host, q, k_new, v_new, k_pool8, v_pool8, block_table,
                       static_cast<float*>(out), lse, memory, stream, info_out, k_scale, v_scale, out_bf16 != 0);
}

namespace {

sf_status reserve(sf_runner* r, const sf::ReserveBytes& need, hipStream_t main) {
  sf_status st = grow_device(r, &r->workspace, &r->workspace_bytes, need.device, main);
  if (st != SF_OK) return st;
  const uint64_t slot = need.slot;
  bool small = false;
  for (auto& p : r->ring) small = small || p.bytes < slot;
  if (!small) return SF_OK;
  // The slots that are too small come from one allocation (32 of their own take
  // 30 us each), once no step in flight reads the old ones. A slot leaves an
  // arena only for more bytes than the arena's slots have, so where any slot is
  // too small, all of an earlier arena's are.
  if ((st = wait_all(r)) != SF_OK) return st;
  void* ptr = nullptr;
  void* dev = nullptr;
  if (hipHostMalloc(&ptr, slot * kRing, hipHostMallocDefault) != hipSuccess) return SF_ERR_HIP;
  if (hipHostGetDevicePointer(&dev, ptr, 0) != hipSuccess) {
    (void)hipHostFree(ptr);
    return SF_ERR_HIP;
  }
  for (int i = 0; i < kRing; ++i) {
    Pinned& p = r->ring[i];
    if (p.bytes >= slot) continue;
    if (p.ptr && !p.in_arena && hipHostFree(p.ptr) != hipSuccess) st = SF_ERR_HIP;
    p = Pinned{};
    p.ptr = reinterpret_cast<int32_t*>(static_cast<char*>(ptr) + slot * i);
    p.dev = reinterpret_cast<const int32_t*>(static_cast<const char*>(dev) + slot * i);
    p.bytes = slot;
    p.in_arena = true;
  }
  if (r->arena && hipHostFree(r->arena) != hipSuccess) st = SF_ERR_HIP;
  r->arena = ptr;
  return st;
}

}  // namespace

extern "C" sf_status sf_runner_reserve(sf_runner* r, uint64_t workspace_bytes, uint64_t work_bytes,
                                       int32_t max_num_seqs, void* stream) {
  if (!r || max_num_seqs < 0) return SF_ERR_INVALID_ARG;
  // A smaller batch, or a step of another kind, may be planned in another way
  // than the batch reserved for and take more than it.
  return reserve(r, sf::reserve_bytes(&r->shape, &r->opts, workspace_bytes, work_bytes, max_num_seqs, -1),
                 static_cast<hipStream_t>(stream));
}

extern "C" sf_status sf_runner_reserve_batch(sf_runner* r, const int32_t* seq_lens_host, int32_t num_seqs, void* stream) {
  if (!r || num_seqs < 0 || (num_seqs > 0 && !seq_lens_host)) return SF_ERR_INVALID_ARG;
  int64_t pages = 0;
  for (int32_t s = 0; s < num_seqs; ++s) {
    if (seq_lens_host[s] < 0) return SF_ERR_INVALID_ARG;
    pages += (int64_t(seq_lens_host[s]) + sf::kPage - 1) / sf::kPage;
  }
  // Room for the batch to grow: the bounds stop at the planner's workers soon.
  return reserve(r, sf::reserve_bytes(&r->shape, &r->opts, 0, 0, num_seqs, 2 * (pages + num_seqs) * r->shape.num_kv_heads),
                 static_cast<hipStream_t>(stream));
}
