// C-ABI entry points that touch the device: table upload, execute, reduce.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <limits>
#include <map>
#include <mutex>
#include <new>
#include <utility>
#include <vector>

#include "kernels.h"
#include "plan_internal.h"

namespace {

thread_local int g_last_hip_error = 0;

int hip_fail(hipError_t e) {
  g_last_hip_error = static_cast<int>(e);
  return CLEAVE_EHIP;
}

#define CLEAVE_HIP(expr)                         \
  do {                                           \
    hipError_t e__ = (expr);                     \
    if (e__ != hipSuccess) return hip_fail(e__); \
  } while (0)

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

void free_verify_device(cleave::VerifyTables* v) {
  if (!v) return;
  void* ptrs[] = {v->d_row_segs, v->d_col_segs, v->d_task_row_seg, v->d_task_col_seg,
                  v->d_items, v->d_task_first_item, v->d_agg_items, v->d_agg_first_item,
                  v->d_agg_item_sums, v->d_proj, v->d_item_sums};
  for (void* q : ptrs)
    if (q) (void)hipFree(q);
  v->d_row_segs = v->d_col_segs = nullptr;
  v->d_task_row_seg = v->d_task_col_seg = v->d_task_first_item = v->d_agg_first_item = nullptr;
  v->d_items = v->d_agg_items = nullptr;
  v->d_proj = v->d_item_sums = v->d_agg_item_sums = nullptr;
}

void free_subset_ring(cleave::SubsetRing* r) {
  if (r->d_ring) (void)hipFree(r->d_ring);
  if (r->d_captured) (void)hipFree(r->d_captured);
  for (const auto& f : r->in_flight) (void)hipEventDestroy(f.done);
  for (hipEvent_t e : r->idle_events) (void)hipEventDestroy(e);
  r->d_ring = r->d_captured = nullptr;
  r->in_flight.clear();
  r->idle_events.clear();
  r->max_items = r->pos = r->captured_used = 0;
}

void free_device_tables(cleave_plan* p) {
  free_verify_device(p->verify);
  if (p->d_tasks) (void)hipFree(p->d_tasks);
  for (int c = 0; c < cleave::kNumTileClasses; ++c)
    if (p->d_items[c]) (void)hipFree(p->d_items[c]);
  if (p->d_reduce_items) (void)hipFree(p->d_reduce_items);
  free_subset_ring(&p->subset);
  p->d_tasks = nullptr;
  if (p->d_items_fine) (void)hipFree(p->d_items_fine);
  p->d_items_fine = nullptr;
  for (int list = 0; list < cleave::kNumTileClasses + 1; ++list) {
    if (p->d_wg_ranges[list]) (void)hipFree(p->d_wg_ranges[list]);
    p->d_wg_ranges[list] = nullptr;
    p->wg_ranges_grid[list] = 0;
  }
  p->d_items[0] = p->d_items[1] = nullptr;
  p->d_reduce_items = nullptr;
  p->device = -1;
}

template <typename T>
int upload_vector(const std::vector<T>& v, T** dst) {
  *dst = nullptr;
  if (v.empty()) return CLEAVE_OK;
  hipError_t e = hipMalloc(reinterpret_cast<void**>(dst), v.size() * sizeof(T));
  if (e == hipErrorOutOfMemory) return CLEAVE_ENOMEM;
  if (e != hipSuccess) return hip_fail(e);
  CLEAVE_HIP(hipMemcpy(*dst, v.data(), v.size() * sizeof(T), hipMemcpyHostToDevice));
  return CLEAVE_OK;
}

// The current device's stream for kernels of an upload: made by the first upload
// that needs it, held until the process ends.
constexpr int kMaxDevices = 64;
std::mutex g_upload_mu;
hipStream_t g_upload_stream[kMaxDevices] = {};
int upload_stream(hipStream_t* out) {
  int dev = 0;
  CLEAVE_HIP(hipGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices) return CLEAVE_EINVAL;
  std::lock_guard<std::mutex> lock(g_upload_mu);
  if (!g_upload_stream[dev]) CLEAVE_HIP(hipStreamCreateWithFlags(&g_upload_stream[dev], hipStreamNonBlocking));
  *out = g_upload_stream[dev];
  return CLEAVE_OK;
}

// The aggregation's table, from the tasks already on the device and the tile list
// (which goes behind the records).  The kernel that writes it is on the device's
// own upload stream, so that neither it nor the caller's wait for it stands
// behind work that the program has on the null stream (on that stream, preparing
// three plans of 16384 x 13824 beside their operands took 12.7 ms, 10.5 without),
// and the caller waits behind its other uploads, which overlap it.  A short table
// is written by the host and copied (2 ns a record; launch and wait cost 25 us).
constexpr int64_t kHostRecords = 8192;
int make_reduce_table(cleave_plan* p, hipStream_t* used) {
  *used = nullptr;
  if (p->reduce_runs <= kHostRecords) {
    try {
      std::vector<cleave::ReduceItem> records;
      records.reserve(static_cast<size_t>(p->reduce_runs));
      for (const cleave::ReduceTile& tile : p->reduce_tiles) {
        const cleave_task& t = p->tasks[tile.task];
        const uint64_t block = static_cast<uint64_t>(t.m_len) * t.n_len;
        for (uint64_t e = 0; e < block; e += tile.run) records.push_back(cleave::make_reduce_item(t, e, tile.run));
      }
      return upload_vector(records, &p->d_reduce_items);
    } catch (const std::bad_alloc&) {
      return CLEAVE_ENOMEM;
    }
  }
  const int64_t n_tiles = static_cast<int64_t>(p->reduce_tiles.size());
  const size_t records = static_cast<size_t>(p->reduce_runs) * sizeof(cleave::ReduceItem);
  const size_t listed = p->reduce_tiles.size() * sizeof(cleave::ReduceTile);
  unsigned char* table = nullptr;
  const hipError_t e = hipMalloc(reinterpret_cast<void**>(&table), records + listed);
  if (e == hipErrorOutOfMemory) return CLEAVE_ENOMEM;
  if (e != hipSuccess) return hip_fail(e);
  p->d_reduce_items = reinterpret_cast<cleave::ReduceItem*>(table);
  cleave::ReduceTile* tiles = reinterpret_cast<cleave::ReduceTile*>(table + records);
  CLEAVE_HIP(hipMemcpy(tiles, p->reduce_tiles.data(), listed, hipMemcpyHostToDevice));
  hipStream_t stream = nullptr;
  const int rc = upload_stream(&stream);
  if (rc != CLEAVE_OK) return rc;
  CLEAVE_HIP(cleave::launch_expand_reduce(p->d_tasks, tiles, n_tiles, p->d_reduce_items, stream));
  *used = stream;
  return CLEAVE_OK;
}

// Work-list memory of cleave_execute_noalloc: a fixed array in the code
// object, one copy per GPU the library runs on, held until the process ends
// (768 KB).  In host code the name is only a handle for hipGetSymbolAddress;
// the address that kernels and copies use is g_static_scratch[device].
constexpr int64_t kStaticScratchItems = 16384;
static __device__ __align__(256) __attribute__((used))
unsigned char scratch[kStaticScratchItems * sizeof(cleave::WorkItem)];

// Once per device and process: the execute kernels' dynamic-LDS limits, the
// CU count and the address of this device's copy of `scratch`.  Done when a
// plan's tables are uploaded, so that no launch has to.
std::mutex g_device_mu;
int g_device_cus[kMaxDevices] = {};   // 0 = not initialised
cleave::WorkItem* g_static_scratch[kMaxDevices] = {};

int ensure_device_ready(int dev, int* cus) {
  if (dev < 0 || dev >= kMaxDevices) return CLEAVE_EINVAL;
  std::lock_guard<std::mutex> lock(g_device_mu);
  if (g_device_cus[dev] == 0) {
    CLEAVE_HIP(cleave::configure_execute_kernels());
    CLEAVE_HIP(cleave::configure_execute_direct_kernels());
    void* ptr = nullptr;   // `dev` is the current device: its copy of the array
    CLEAVE_HIP(hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch)));
    g_static_scratch[dev] = static_cast<cleave::WorkItem*>(ptr);
    int n = 0;
    CLEAVE_HIP(hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev));
    g_device_cus[dev] = std::max(n, 1);
  }
  if (cus) *cus = g_device_cus[dev];
  return CLEAVE_OK;
}

// The kernels with an epilogue likewise, when a plan of cleave_plan_linear's is uploaded, or by the first cleave_linear: they would
// cost who only executes another 4 ms.
bool g_linear_ready[kMaxDevices] = {};

int ensure_linear_ready(int dev) {
  if (dev < 0 || dev >= kMaxDevices) return CLEAVE_EINVAL;
  std::lock_guard<std::mutex> lock(g_device_mu);
  if (g_linear_ready[dev]) return CLEAVE_OK;
  CLEAVE_HIP(cleave::configure_linear_general_kernels());
  CLEAVE_HIP(cleave::configure_linear_direct_kernels());
  CLEAVE_HIP(cleave::configure_linear_8bit_kernels());
  g_linear_ready[dev] = true;
  return CLEAVE_OK;
}

// And the gated product's and its gradient's.
bool g_gated_ready[kMaxDevices] = {};

int ensure_gated_ready(int dev) {
  if (dev < 0 || dev >= kMaxDevices) return CLEAVE_EINVAL;
  std::lock_guard<std::mutex> lock(g_device_mu);
  if (g_gated_ready[dev]) return CLEAVE_OK;
  CLEAVE_HIP(cleave::configure_gated_direct_kernels());
  CLEAVE_HIP(cleave::configure_gated_8bit_kernels());
  CLEAVE_HIP(cleave::configure_gated_grad_kernels());
  g_gated_ready[dev] = true;
  return CLEAVE_OK;
}

constexpr int kSubsetEvents = 16;

int allocate_subset_ring(cleave_plan* p) {
  cleave::SubsetRing& r = p->subset;
  r.max_items = static_cast<int64_t>(std::max(p->items[0].size() + p->items[1].size(), p->items_fine.size()));
  if (r.max_items == 0) return CLEAVE_OK;
  const size_t item_bytes = static_cast<size_t>(r.max_items) * sizeof(cleave::WorkItem);
  hipError_t e = hipMalloc(reinterpret_cast<void**>(&r.d_ring), 2 * item_bytes);
  if (e == hipSuccess) e = hipMalloc(reinterpret_cast<void**>(&r.d_captured), item_bytes);
  if (e == hipErrorOutOfMemory) return CLEAVE_ENOMEM;
  if (e != hipSuccess) return hip_fail(e);
  try {
    r.idle_events.reserve(kSubsetEvents);
    r.in_flight.reserve(kSubsetEvents);
  } catch (const std::bad_alloc&) {
    return CLEAVE_ENOMEM;
  }
  for (int i = 0; i < kSubsetEvents; ++i) {
    hipEvent_t ev = nullptr;
    CLEAVE_HIP(hipEventCreateWithFlags(&ev, hipEventDisableTiming));
    r.idle_events.push_back(ev);
  }
  return CLEAVE_OK;
}

bool cut_small(const cleave_plan* plan, int cus);

int ensure_uploaded(cleave_plan* p) {
  int dev = 0;
  CLEAVE_HIP(hipGetDevice(&dev));
  if (p->device == dev) return CLEAVE_OK;
  if (p->device >= 0) free_device_tables(p);
  int rc = ensure_device_ready(dev, nullptr);
  if (rc == CLEAVE_OK && p->linear) rc = ensure_linear_ready(dev);
  if (rc == CLEAVE_OK && p->gated) rc = ensure_gated_ready(dev);
  if (rc == CLEAVE_OK && p->gated && p->pairs && p->uniform_splits > 1) rc = ensure_linear_ready(dev);
  if (rc != CLEAVE_OK) return rc;
  rc = upload_vector(p->tasks, &p->d_tasks);
  hipStream_t writing = nullptr;
  if (rc == CLEAVE_OK) rc = make_reduce_table(p, &writing);
  // The three work-item lists; items of unequal length get a balanced workgroup
  // schedule for this device's grid (the host lists keep their canonical order for
  // the next device).  Full launches of the general kernel run the third list, the
  // fast kernel's only where it cuts large blocks small.
  int cus = 0;
  if (rc == CLEAVE_OK) rc = ensure_device_ready(dev, &cus);
  for (int list = 0; rc == CLEAVE_OK && list < cleave::kNumTileClasses + 1; ++list) {
    const bool fine = list == cleave::kNumTileClasses;
    const int cls = fine ? cleave::kTileSmall : list;
    const std::vector<cleave::WorkItem>& host = fine ? p->items_fine : p->items[list];
    cleave::WorkItem** dst = fine ? &p->d_items_fine : &p->d_items[list];
    const int64_t resident = static_cast<int64_t>(cus) * cleave::direct_workgroups_per_cu(
                                                                cls == cleave::kTileLarge ? cleave::kDirectLarge : cleave::kDirectSmall);
    const int grid = static_cast<int>(std::min<int64_t>(static_cast<int64_t>(host.size()), resident));
    std::vector<uint32_t> ranges;
    try {
      std::vector<cleave::WorkItem> scheduled;
      if (!fine || cut_small(p, cus)) scheduled = cleave::scheduled_list(host, grid, fine, &ranges);
      rc = upload_vector(ranges.empty() ? host : scheduled, dst);
    } catch (const std::bad_alloc&) {
      rc = CLEAVE_ENOMEM;
    }
    if (rc == CLEAVE_OK && !ranges.empty()) {
      rc = upload_vector(ranges, &p->d_wg_ranges[list]);
      p->wg_ranges_grid[list] = grid;
    }
  }
  if (rc == CLEAVE_OK) rc = allocate_subset_ring(p);
  if (writing) {   // the tables are read on any stream next (and freed on an error)
    const hipError_t e = hipStreamSynchronize(writing);
    if (e != hipSuccess && rc == CLEAVE_OK) rc = hip_fail(e);
  }
  if (rc != CLEAVE_OK) {
    free_device_tables(p);
    return rc;
  }
  p->device = dev;
  return CLEAVE_OK;
}

int compute_units(int* out) {
  int dev = 0;
  CLEAVE_HIP(hipGetDevice(&dev));
  return ensure_device_ready(dev, out);
}

// A slice of `total` work items for a subset launch on `stream`.  Eager
// launches take the next slice of the ring (waiting, on the host, only for
// earlier launches that still read the slice: none unless the ring has
// wrapped onto unfinished work); launches under stream capture take a slice
// of the second buffer that is never handed out again.  No allocation.
int acquire_subset_slice(cleave::SubsetRing& r, int64_t total, bool capturing, cleave::WorkItem** out,
                         int64_t* begin) {
  if (total > r.max_items) return CLEAVE_EINVAL;   // cannot happen for distinct task ids
  if (capturing) {
    if (r.captured_used + total > r.max_items) return CLEAVE_ENOMEM;
    *out = r.d_captured + r.captured_used;
    *begin = -1;
    r.captured_used += total;
    return CLEAVE_OK;
  }
  if (r.pos + total > 2 * r.max_items) r.pos = 0;
  const int64_t b = r.pos, e = r.pos + total;
  // launches retire in order per stream, not across streams: check every record
  for (size_t i = 0; i < r.in_flight.size();) {
    const auto f = r.in_flight[i];
    const bool overlaps = f.begin < e && b < f.end;
    hipError_t q = overlaps ? hipEventSynchronize(f.done) : hipEventQuery(f.done);
    if (q == hipSuccess) {
      r.idle_events.push_back(f.done);
      r.in_flight.erase(r.in_flight.begin() + static_cast<std::ptrdiff_t>(i));
    } else if (q == hipErrorNotReady) {
      ++i;
    } else {
      return hip_fail(q);
    }
  }
  *out = r.d_ring + b;
  *begin = b;
  r.pos = e;
  return CLEAVE_OK;
}

// Marks the slice [begin, begin + total) as read by what has been enqueued on
// `stream` so far.
int release_subset_slice(cleave::SubsetRing& r, int64_t begin, int64_t total, hipStream_t stream) {
  if (begin < 0) return CLEAVE_OK;   // captured: never reused
  if (r.idle_events.empty()) {
    // every event is attached to a launch still in flight: wait for the oldest
    const auto f = r.in_flight.front();
    CLEAVE_HIP(hipEventSynchronize(f.done));
    r.in_flight.erase(r.in_flight.begin());
    r.idle_events.push_back(f.done);
  }
  hipEvent_t ev = r.idle_events.back();
  r.idle_events.pop_back();
  const hipError_t e = hipEventRecord(ev, stream);
  if (e != hipSuccess) {
    r.idle_events.push_back(ev);
    return hip_fail(e);
  }
  r.in_flight.push_back({begin, begin + total, ev});
  return CLEAVE_OK;
}

const char* kernel_name(int dtype, const cleave::GeneralLoads& how, int transA, int transB) {
  static const char* names[2][6][4] = {
      {{"execute_f32_128x128_nn", "execute_f32_128x128_nt", "execute_f32_128x128_tn", "execute_f32_128x128_tt"},
       {"execute_f32_64x64_nn", "execute_f32_64x64_nt", "execute_f32_64x64_tn", "execute_f32_64x64_tt"},
       {"none", "none", "none", "none"},
       {"execute_f32_64x64_quarters_nn", "execute_f32_64x64_quarters_nt", "execute_f32_64x64_quarters_tn",
        "execute_f32_64x64_quarters_tt"},
       {"execute_f32_element", "execute_f32_element", "execute_f32_element", "execute_f32_element"},
       {"execute_f32_64x64_lone_nn", "execute_f32_64x64_lone_nt", "execute_f32_64x64_lone_tn", "execute_f32_64x64_lone_tt"}},
      {{"execute_bf16_128x128_nn", "execute_bf16_128x128_nt", "execute_bf16_128x128_tn", "execute_bf16_128x128_tt"},
       {"execute_bf16_64x64_nn", "execute_bf16_64x64_nt", "execute_bf16_64x64_tn", "execute_bf16_64x64_tt"},
       {"none", "execute_bf16_256x256_nt", "none", "none"},
       {"none", "none", "none", "none"},
       {"execute_bf16_element", "execute_bf16_element", "execute_bf16_element", "execute_bf16_element"},
       {"execute_bf16_64x64_lone_nn", "execute_bf16_64x64_lone_nt", "execute_bf16_64x64_lone_tn",
        "execute_bf16_64x64_lone_tt"}}};
  const int row = how.a_elements || how.b_elements ? 4 : how.tile == cleave::kTileWide4 ? cleave::kTileWide : how.tile;
  return names[dtype == CLEAVE_BF16 ? 1 : 0][row][(transA ? 2 : 0) + (transB ? 1 : 0)];
}

const char* direct_kernel_name(cleave::DirectShape shape, int transA, int transB) {
  static const char* names[4][4] = {
      {"execute_direct_bf16_256x256_nn", "execute_direct_bf16_256x256_nt",
       "execute_direct_bf16_256x256_tn", "execute_direct_bf16_256x256_tt"},
      {"execute_direct_bf16_128x128_nn", "execute_direct_bf16_128x128_nt",
       "execute_direct_bf16_128x128_tn", "execute_direct_bf16_128x128_tt"},
      {"execute_direct_bf16_128x128_deep_nn", "execute_direct_bf16_128x128_deep_nt",
       "execute_direct_bf16_128x128_deep_tn", "execute_direct_bf16_128x128_deep_tt"},
      {"execute_direct_bf16_64x64_nn", "execute_direct_bf16_64x64_nt",
       "execute_direct_bf16_64x64_tn", "execute_direct_bf16_64x64_tt"}};
  return names[shape][(transA ? 2 : 0) + (transB ? 1 : 0)];
}

// The kernels with an epilogue.
const char* linear_kernel_name(int dtype, const cleave::GeneralLoads& how, int transA, int transB) {
  static const char* names[2][2][4] = {
      {{"linear_f32_128x128_nn", "linear_f32_128x128_nt", "linear_f32_128x128_tn", "linear_f32_128x128_tt"},
       {"linear_f32_64x64_nn", "linear_f32_64x64_nt", "linear_f32_64x64_tn", "linear_f32_64x64_tt"}},
      {{"linear_bf16_128x128_nn", "linear_bf16_128x128_nt", "linear_bf16_128x128_tn", "linear_bf16_128x128_tt"},
       {"linear_bf16_64x64_nn", "linear_bf16_64x64_nt", "linear_bf16_64x64_tn", "linear_bf16_64x64_tt"}}};
  const bool bf16 = dtype == CLEAVE_BF16;
  if (how.a_elements || how.b_elements) return bf16 ? "linear_bf16_element" : "linear_f32_element";
  return names[bf16 ? 1 : 0][how.tile == cleave::kTileLone ? 1 : 0][(transA ? 2 : 0) + (transB ? 1 : 0)];
}

// which: a gated product of bf16, of e4m3, the gradient
const char* gated_kernel_name(cleave::DirectShape shape, int which, int transB) {
  static const char* names[4][3][2] = {
      {{"gated_direct_bf16_256x128_nn", "gated_direct_bf16_256x128_nt"}, {"none", "none"},
       {"gated_grad_direct_bf16_256x256_nn", "gated_grad_direct_bf16_256x256_nt"}},
      {{"gated_direct_bf16_128x64_nn", "gated_direct_bf16_128x64_nt"}, {"none", "gated_direct_e4m3_128x64_nt"},
       {"gated_grad_direct_bf16_128x128_nn", "gated_grad_direct_bf16_128x128_nt"}},
      {{"gated_direct_bf16_128x64_deep_nn", "gated_direct_bf16_128x64_deep_nt"}, {"none", "gated_direct_e4m3_128x64_deep_nt"},
       {"gated_grad_direct_bf16_128x128_deep_nn", "gated_grad_direct_bf16_128x128_deep_nt"}},
      {{"gated_direct_bf16_64x32_nn", "gated_direct_bf16_64x32_nt"}, {"none", "gated_direct_e4m3_64x32_nt"},
       {"gated_grad_direct_bf16_64x64_nn", "gated_grad_direct_bf16_64x64_nt"}}};
  return names[shape][which][transB ? 1 : 0];
}

const char* linear_direct_kernel_name(cleave::DirectShape shape, bool e4m3, int transB) {
  static const char* names[4][3] = {   // (8-bit operands: no large shape, and B is N x K)
      {"linear_direct_bf16_256x256_nn", "linear_direct_bf16_256x256_nt", "none"},
      {"linear_direct_bf16_128x128_nn", "linear_direct_bf16_128x128_nt", "linear_direct_e4m3_128x128_nt"},
      {"linear_direct_bf16_128x128_deep_nn", "linear_direct_bf16_128x128_deep_nt", "linear_direct_e4m3_128x128_deep_nt"},
      {"linear_direct_bf16_64x64_nn", "linear_direct_bf16_64x64_nt", "linear_direct_e4m3_64x64_nt"}};
  return names[shape][e4m3 ? 2 : transB ? 1 : 0];
}

}  // namespace

int cleave::record_hip_error(hipError_t e) { return hip_fail(e); }

extern "C" int cleave_last_hip_error(void) { return g_last_hip_error; }

extern "C" int cleave_version(void) { return 107; }

namespace {

int upload_gated(cleave_plan* plan);

}  // namespace

extern "C" int cleave_plan_upload(cleave_plan* plan) {
  if (!plan) return CLEAVE_EINVAL;
  return plan->gated ? upload_gated(plan) : ensure_uploaded(plan);
}

extern "C" void cleave_plan_destroy(cleave_plan* plan) {
  if (!plan) return;
  cleave_plan_destroy(plan->fused);
  if (plan->device >= 0) free_device_tables(plan);
  delete plan->verify;
  delete plan;
}

namespace {

// How a batched call finds its members' matrices (element offsets from the
// base pointers); all zero for a plain plan.
struct BatchLayout {
  cleave::BatchShape shape{0, 0};
  cleave::MemberOffsets a{}, b{};
  cleave::MemberOffsets c{};   // assemble mode and reduce only
};

// Every member offset is a multiple of `e` elements.
bool offsets_multiple_of(const cleave::MemberOffsets& at, const cleave::BatchShape& shape, int64_t e) {
  if (shape.n_group == 0) return at.outer % e == 0 && at.inner % e == 0;
  for (uint32_t g = 0; g < shape.n_group; ++g)
    if (at.table[g] % e != 0) return false;
  return true;
}

BatchLayout strided_layout(int64_t n_inner, int64_t a_outer, int64_t a_inner, int64_t b_outer,
                           int64_t b_inner, int64_t c_outer, int64_t c_inner) {
  BatchLayout bl;
  bl.shape.batch_inner = static_cast<uint32_t>(n_inner);
  bl.a.outer = a_outer;
  bl.a.inner = a_inner;
  bl.b.outer = b_outer;
  bl.b.inner = b_inner;
  bl.c.outer = c_outer;
  bl.c.inner = c_inner;
  return bl;
}

// Grouped launch: members given by one pointer each.  list[0] becomes the base
// pointer, the others element offsets from it.
int group_offsets(const void* const* list, int64_t n, int elem_bytes, cleave::MemberOffsets* at,
                  const void** base) {
  if (!list || n < 1 || n > cleave::kMaxGroup) return CLEAVE_EINVAL;
  for (int64_t g = 0; g < n; ++g)
    if (!list[g] || !aligned(list[g], elem_bytes)) return CLEAVE_EINVAL;
  *base = list[0];
  for (int64_t g = 0; g < n; ++g)
    at->table[g] = (reinterpret_cast<intptr_t>(list[g]) - reinterpret_cast<intptr_t>(list[0])) / elem_bytes;
  return CLEAVE_OK;
}

// Assemble mode: blocks go to their place in C instead of the partial buffer.
struct AssembleTarget {
  void* C = nullptr;
  int64_t ldc = 0;
  int out_dtype = CLEAVE_F32;
};

// The work items of a full launch whose chunk starts below the returned k leave
// through non-temporal stores.  An output that the cache cannot hold pushes its own
// first part (and the operands) out of it, and the next launch waits for those
// write-backs; a streamed one goes to memory without them.  One that it can hold is
// read from there by whoever comes next.
//   Assembled outputs: see streamed_output.
//   Partial blocks of uniform plans (their items run chunk by chunk): execute +
// reduce over plain, all chunks but the last streamed / all of them streamed:
//   blocks of a chunk x chunks
//    67 MB x 4   1.031, 0.998 / 1.043, 1.005      67 MB x 8   0.893, 0.894 / 0.907, 0.901
//   134 MB x 2   1.034, 0.992 / 1.033, 0.991     134 MB x 4   0.884, 0.927 / 0.904, 0.920
//   134 MB x 8   0.911, 0.975 / 0.862, 0.992     180 MB x 2   0.969, 0.955 / 0.979, 0.954
//   180 MB x 4   0.945, 0.980 / 0.925, 0.965     180 MB x 8   0.984, 0.978 / 0.922, 0.988
//   268 MB x 4   1.001, 0.986 / 0.921, 1.005     268 MB x 8   0.968, 0.984 / 0.988, 0.981
//   336 MB x 2   0.976, 0.985 / 1.029, 1.002     336 MB x 8   0.955, 0.974 / 0.959, 0.967
//   453 MB x 2   0.989, 0.991 / 1.012, 0.996     453 MB x 4   0.967, 0.980 / 0.971, 0.980
//   453 MB x 8   0.981 / 0.971                   537 MB x 2   1.011, 1.007 / 1.025, 1.015
//   537 MB x 4   0.977, 0.989 / 0.974, 0.982     537 MB x 8   0.972 / 0.958
//   906 MB x 2   0.985, 0.991 / 0.970, 0.981     906 MB x 8   0.891 / 0.879
// (chunks of 512 and of 1024 elements, 1024 alone where one figure is given).  537 MB x 2
// (8192 x 16384) loses 1 % in every form, again in a second run (1.016, 1.010); beside it
// 528 MB x 2 0.998, 1.011, 604 MB x 2 0.985, 0.993, so no line by size leaves it out.
// Batched, grouped and explicit plans have not been measured and keep plain stores.  Short
// chains, whose launches are bound by the stores themselves, lose: linear layers, us,
// plain / streamed, chunks of 48 elements 292 / 302, of 63 494 / 512, of 82 525 / 531, of
// 200 639 / 651; of 476 1703 / 1612.
uint32_t streamed_below(const cleave_plan* plan, const AssembleTarget& asm_to) {
  const int64_t members = std::max<int64_t>(plan->batch, 1);
  const int64_t outputs = plan->M * plan->N * members;
  if (asm_to.C) {
    const int64_t bytes = outputs * (asm_to.out_dtype == CLEAVE_BF16 ? 2 : 4);
    return cleave::streamed_output(bytes, plan->batch > 0) ? static_cast<uint32_t>(plan->K) : 0;
  }
  const int64_t splits = plan->uniform_splits;
  if (splits < 2 || 4 * plan->partial_elems < cleave::kCacheBytes / 4 * 5) return 0;
  const int64_t chunk = (plan->K + splits - 1) / splits;
  if (chunk < 6 * int64_t{cleave::kDirectKStep}) return 0;
  const bool all = 4 * outputs >= 3 * cleave::kCacheBytes || (4 * outputs >= cleave::kCacheBytes / 2 * 3 && splits >= 4);
  return static_cast<uint32_t>(all ? plan->K : (splits - 1) * chunk);
}

// Where the work items of a subset go: one list per tile class, in the caller's
// order (the layout of the plan's own lists).
struct SubsetLayout {
  bool fine = false;                               // every block cut into small-class sub-tiles
  int64_t counts[cleave::kNumTileClasses] = {};    // work items per class
  int64_t steps[cleave::kNumTileClasses] = {};     // their whole K steps, together
  cleave::ListShape shapes[cleave::kNumTileClasses];
  int64_t total() const { return counts[0] + counts[1]; }
};

// Validates the ids (range, no repeats) and sizes the lists.  Uses the plan's
// own stamp array for the repeat check: no allocation.  Caller holds subset.mu.
// The cut depends on the ids alone, not on which kernel runs the items (the
// general one cuts large items into its workgroup tiles itself), so neither do
// the work-list memory a subset takes and the limit on it.
int layout_subset(cleave_plan* plan, const int64_t* task_ids, int64_t n_ids, int cus, SubsetLayout* out) {
  const int64_t n_tasks = static_cast<int64_t>(plan->tasks.size());
  if (++plan->seen_generation == 0) {   // wrapped: start over with clean stamps
    std::fill(plan->seen_stamp.begin(), plan->seen_stamp.end(), 0u);
    plan->seen_generation = 1;
  }
  size_t large_items = 0;
  for (int64_t i = 0; i < n_ids; ++i) {
    const int64_t id = task_ids[i];
    if (id < 0 || id >= n_tasks || plan->seen_stamp[id] == plan->seen_generation) return CLEAVE_EINVAL;
    plan->seen_stamp[id] = plan->seen_generation;
    const cleave::SubTiling st = cleave::sub_tiling(plan->tasks[id], false);
    if (st.cls == cleave::kTileLarge) large_items += st.count();
  }
  // Few large items would leave most CUs idle: cut everything small instead
  // (the bits do not depend on the cut).
  out->fine = large_items > 0 && large_items <= static_cast<size_t>(cus) / 2;
  for (int64_t i = 0; i < n_ids; ++i) {
    const cleave_task& t = plan->tasks[task_ids[i]];
    const cleave::SubTiling st = cleave::sub_tiling(t, out->fine);
    out->counts[st.cls] += st.count();
    out->steps[st.cls] += int64_t{st.count()} * (t.k_len / cleave::kDirectKStep);
    out->shapes[st.cls].add(t);
  }
  return CLEAVE_OK;
}

// Enqueues the kernels that write the subset's work items to `out`; the
// (task, destination) pairs are built on the stack, one launch's worth at a time.
int expand_subset(const cleave_plan* plan, const int64_t* task_ids, int64_t n_ids,
                  const SubsetLayout& layout, cleave::WorkItem* out, hipStream_t stream) {
  int64_t next[cleave::kNumTileClasses] = {0, layout.counts[0]};
  cleave::ExpandArgs ea{};
  ea.tasks = plan->d_tasks;
  ea.out = out;
  ea.fine = layout.fine ? 1u : 0u;
  for (int64_t i = 0; i < n_ids; ++i) {
    const cleave_task& t = plan->tasks[task_ids[i]];
    const cleave::SubTiling st = cleave::sub_tiling(t, layout.fine);
    int64_t& at = next[st.cls];
    ea.entries[ea.n_entries++] = {static_cast<uint32_t>(task_ids[i]), static_cast<uint32_t>(at)};
    at += st.count();
    if (ea.n_entries == cleave::kSubsetEntriesPerLaunch || i + 1 == n_ids) {
      CLEAVE_HIP(cleave::launch_expand_subset(ea, stream));
      ea.n_entries = 0;
    }
  }
  return CLEAVE_OK;
}

// Workgroup tile of the general kernel for `items` 128 x 128 work items.  The
// 64 x 64 tile gives four times as many workgroups, four of them per CU
// instead of two, at twice the LDS traffic per flop.  fp32 MFMAs leave the LDS
// mostly idle, so there the narrow tile wins unless the wide one's workgroups fill
// their rounds of the CUs to 15/16 (from four rounds on it runs whether or not).  us, wide /
// narrow, layouts NN, NT, TN: 32 steps, 256 items 71 / 68, 70 / 67, 72 / 69, 480 items
// 125 / 129, 123 / 127, 127 / 129, 704 items 183 / 182, 184 / 177, 183 / 183, 768 items 184 /
// 196, 185 / 191, 184 / 195, 896 items 246 / 227, 242 / 226, 249 / 229; 12 steps, 480 items
// 52.7 / 54.1, 52.3 / 54.0, 53.5 / 55.1, 768 items 76.4 / 81.2, 76.3 / 81.9, 77.4 / 80.9.
// The wide tile multiplies all of an item, the narrow one the 64 x 64 parts that hold
// something (`list.parts64` in all): with small blocks there is less to win.  Below four
// rounds it runs from four fifths on, from there on from a half.  fp32, 1024 of K, by what
// the items hold: 960 items 0.56 246 / 230, 242 / 225, 248 / 231; 720 items 0.88 183 / 186,
// 184 / 183, 183 / 187; 512 items of 64 x 64 blocks (0.25, 512 of K) 64 / 22, 64 / 21, 66 / 22;
// 1024 items 0.25 244 / 68, 241 / 67, 248 / 68, 0.52 246 / 246, 242 / 241, 248 / 246; 2048 items
// 0.5 252 / 136, 251 / 134, 255 / 135; 2560 items 0.56 314 / 316, 314 / 308, 318 / 318, with 256
// of K 97 / 102, 97 / 102, 100 / 106.
// bf16 MFMAs do not: narrow only while the wide tile leaves half of the CUs without a
// workgroup (11 steps, 128 items 14.6 / 12.6, 13.7 / 12.4, 14.5 / 12.4, 192 items 15.2 /
// 17.4, 15.1 / 17.7, 15.5 / 17.4; 3 to 6 steps, 64 items 9.6 / 7.1, 192 items 9.5 / 10.0).
// Few fp32 items run as quarters of the 64 x 64 tile, up to two on each CU: a wave's
// chain of matrix instructions is what such a launch takes, and a quarter's is a
// quarter as long (with four times the waves, half as many products per load).
// Execute alone, us, 64 x 64 / quarters, operands in L2, layouts NN, NT, TN, TT (64 x 64 as it
// runs: the form that reads ahead from eight steps on): 16 items of 32 of K 4.0 / 3.9, 3.8 / 3.8,
// 4.1 / 3.8, 4.1 / 3.9, of 128 5.9 / 4.8, 5.7 / 4.9, 6.0 / 4.4, 6.0 / 4.8, of 512 12.4 / 8.1, 12.2 / 8.6,
// 12.5 / 7.0, 12.2 / 8.1, of 2048 37 / 20.9, 37 / 22.9, 37 / 17.2, 37 / 21.2; 32 items of 32 4.1 / 4.4,
// 3.9 / 4.4, 4.3 / 4.2, 4.2 / 4.4, of 64 4.8 / 4.7, 4.6 / 4.7, 4.9 / 4.5, 4.8 / 4.7, of 96 5.5 / 5.3,
// 5.2 / 5.3, 5.6 / 5.0, 5.5 / 5.1, of 128 6.1 / 5.7, 5.9 / 5.9, 6.2 / 5.3, 6.1 / 5.6, of 160 6.8 / 6.1,
// 6.6 / 6.4, 6.9 / 5.7, 6.8 / 6.1, of 256 8.4 / 7.3, 8.2 / 7.7, 8.6 / 6.6, 8.3 / 7.3, of 1024 20.9 / 16.6,
// 20.8 / 19.0, 21.0 / 14.3, 20.8 / 17.0 (20 and 24 items as 32); 40 items of 256 8.5 / 8.6, 8.3 / 9.5,
// 8.7 / 7.9, 8.4 / 8.6, of 1024 21.0 / 21.2, 21.0 / 24.3, 21.3 / 19.1, 21.0 / 21.8; 64 of 512 13.1 / 15.5,
// 13.0 / 17.4, 13.2 / 13.9, 13.1 / 15.6.  With two on a CU, beyond 16 items, only chunks from 128
// elements on, of two K-contiguous operands (whose fragments take twice the reads) from 256.  That
// is on the safe side: the lines were drawn on forms of both that read nothing ahead, and below them the
// quarters now gain too, from 160 on in NT, from 64 on in NN and TT (1 to 6 %), at any length in TN (2 to 15 %).
// `whole`: that many 256 x 256 items of a subset (full launches of this kernel run
// the all-small list), with `steps` whole K steps between them, that the kernel
// could take as they are (bf16, both operands K-contiguous: six
// fragment reads for eight products instead of eight).  They win when their
// rounds are nearly full and their chains long enough to cover a start and end
// alone on a CU (us, 128 / 256: 17 steps, 256 items 57 / 50, 1024 items 230 / 193, 688 items 144 / 132,
// 576 items, the third round a quarter full, 116 / 127; 5 steps, 1024 items
// 92.7 / 92.6, 688 items 59 / 66).
cleave::ExecuteTile general_tile(int dtype, bool both_k, int64_t items, const cleave::ListShape& list, int64_t whole,
                                 int64_t steps, int cus) {
  const int64_t places = (whole + cus - 1) / cus * cus;
  if (whole > 0 && whole * 8 >= places * 7 && steps >= 16 * whole) return cleave::kTileHuge;
  if (dtype == CLEAVE_F32 && 8 * items <= cus && (16 * items <= cus || list.longest >= (both_k ? 256u : 128u)))
    return cleave::kTileQuarter;
  if (dtype == CLEAVE_BF16) return 2 * items <= cus ? cleave::kTileNarrow : cleave::kTileWide;
  const int64_t places_wide = (items + cus - 1) / cus * cus;
  const bool wide = items >= int64_t{4} * cus
                        ? list.parts64 > 2 * items
                        : items > cus && 16 * items >= 15 * places_wide && 5 * list.parts64 >= 16 * items;
  return wide ? cleave::kTileWide : cleave::kTileNarrow;
}

// Shape of the direct kernel for `items` work items of a class.  Small items run as 64 x 64
// parts while a part has a place of its own, two on each CU (an item is four of them): there
// parts win at every chain length.  From there to one item per CU the deep ring does.  Time
// against 128 x 128 items with two stages, operands in L2 / from HBM, the largest of three
// layouts, by K steps per item (256 CUs):
//                    2 steps      4            8            16           24           48
//    16 items parts  0.65 / 0.65  0.63 / 0.63  0.60 / 0.60  0.57 / 0.51  0.56 / 0.45  0.54 / 0.42
//             deep   0.85 / 0.85  0.88 / 0.88  0.91 / 0.88  0.94 / 0.81  0.95 / 0.75  0.98 / 0.75
//    64 items parts  0.70 / 0.70  0.67 / 0.67  0.64 / 0.62  0.61 / 0.56  0.59 / 0.53  0.49 / 0.48
//             deep   0.87 / 0.86  0.89 / 0.88  0.92 / 0.86  0.94 / 0.83  0.96 / 0.83  0.81 / 0.79
//   128 items parts  0.78 / 0.78  0.78 / 0.79  0.79 / 0.80  0.77 / 0.79  0.78 / 0.78  0.77 / 0.78
//             deep   0.88 / 0.86  0.89 / 0.91  0.92 / 0.88  0.94 / 0.85  0.95 / 0.84  0.80 / 0.81
//   130 items parts  0.92 / 0.95  0.94 / 0.94  0.98 / 0.93  1.01 / 0.88  0.88 / 0.89  0.86 / 0.81
//             deep   0.88 / 0.87  0.91 / 0.91  0.92 / 0.86  0.93 / 0.80  0.78 / 0.78  0.72 / 0.72
//   160 items parts  0.97 / 0.98  0.98 / 0.98  1.02 / 0.98  0.98 / 0.91  0.96 / 0.92  0.95 / 0.93
//             deep   0.88 / 0.88  0.91 / 0.90  0.92 / 0.87  0.93 / 0.83  0.90 / 0.76  0.78 / 0.73
//   224 items deep   0.89 / 0.89  0.92 / 0.91  0.92 / 0.88  0.93 / 0.82  0.83 / 0.76  0.83 / 0.74
//   256 items deep   0.90 / 0.90  0.92 / 0.92  0.93 / 0.87  0.91 / 0.80  0.83 / 0.76  0.85 / 0.73
// (Before its last steps were copies with constant waits the ring took 1.09 to 1.14 of the two-stage time
// with operands in L2 at 4 and 8 steps, and ran from 16 on only.)  Two such launches at a time, on
// two streams, 4 to 24 steps: deep 0.87 to 0.98 of two stages with 136 or 160 items each, 0.95 to 1.02
// with 192, 1.11 to 1.17 with 256, when a CU would have held a two-stage workgroup of each.
cleave::DirectShape direct_shape(int cls, int64_t items, int cus) {
  if (cls == cleave::kTileLarge) return cleave::kDirectLarge;
  if (items * 2 <= cus) return cleave::kDirectParts;
  return items <= cus ? cleave::kDirectDeep : cleave::kDirectSmall;
}

// Whether a full launch of the direct kernel cuts every block into small sub-tiles:
// four times as many items, two workgroups per CU.  They cost more per product
// (twice the operand traffic into LDS, 1.1-1.25 times the time from four full
// rounds on), but a round is a quarter as much work, so they win where large items
// leave much of the last round's CUs idle.  The bits do not depend on the cut.
// Time of the small cut over the large one's, operands and blocks as the launch
// before left them in the caches / not in any cache (256 CUs, items of equal
// length; of three layouts and of square outputs and ones 1024 wide, where cold
// operands cost the small cut most, the one with the largest product of the two):
//            2 steps      4            8            12           16           24
//   136      0.88 / 0.89  0.94 / 1.00  0.98 / 1.08  1.01 / 1.14  1.02 / 1.19  1.07 / 1.25
//   192      0.91 / 0.92  0.89 / 0.98  0.95 / 1.07  0.96 / 1.18  0.96 / 1.20  0.97 / 1.33
//   224      0.98 / 0.97  0.93 / 1.12  0.97 / 1.33  1.01 / 1.45  1.04 / 1.48  1.05 / 1.51
//   272      0.81 / 0.94  0.74 / 1.06  0.75 / 1.10  0.78 / 1.11  0.78 / 1.12  0.80 / 1.13
//   288      0.81 / 0.94  0.75 / 1.09  0.76 / 1.11  0.78 / 1.15  0.80 / 1.13  0.82 / 1.16
//   320      0.86 / 0.97  0.84 / 1.02  0.81 / 1.04  0.79 / 1.12  0.81 / 1.13  0.81 / 1.15
//   352      0.92 / 1.09  0.90 / 1.19  0.87 / 1.21  0.88 / 1.25  0.90 / 1.21  0.90 / 1.23
//   384      0.89 / 1.05  0.93 / 1.16  0.89 / 1.25  0.90 / 1.24  0.92 / 1.23  0.91 / 1.25
//   544      0.89 / 1.01  0.83 / 1.13  0.88 / 1.12  0.86 / 1.21  0.86 / 1.18  0.85 / 1.21
//   576      0.89 / 1.05  0.84 / 1.14  0.88 / 1.22  0.91 / 1.24  0.89 / 1.23  1.04 / 1.30
//   640      0.92 / 1.18  0.93 / 1.22  0.94 / 1.32  0.96 / 1.33  0.95 / 1.25  1.23 / 1.33
// Chains of 64 steps: 272 items 0.87 / 0.94, 288 0.87 / 1.02.  Where some blocks are
// small anyway (a rim of the output), cutting all of them also saves the launch for
// those, and wins further out (few: 4 to 40 small items; many: as many as large ones):
//            2 steps      4            8            12           16           24
//   136 few  0.69 / 0.71  0.73 / 0.81  0.77 / 0.88  0.83 / 0.98  0.86 / 1.00  0.92 / 1.04
//   136 many 0.64 / 0.66  0.64 / 0.74  0.66 / 0.79  0.70 / 0.80  0.75 / 0.86  0.80 / 0.87
//   192 few  0.82 / 0.86  0.81 / 0.95  0.86 / 0.98  0.89 / 1.02  0.91 / 1.06  0.94 / 1.11
//   192 many 0.70 / 0.79  0.71 / 0.84  0.74 / 0.90  0.76 / 0.91  0.80 / 0.96  0.84 / 0.99
//   224 few  0.78 / 0.82  0.75 / 0.93  0.81 / 1.08  0.86 / 1.11  0.88 / 1.16  0.92 / 1.24
//   224 many 0.72 / 0.83  0.74 / 0.90  0.79 / 1.02  0.86 / 1.07  0.96 / 1.16  1.02 / 1.21
//   272 few  0.70 / 0.78  0.65 / 0.84  0.67 / 0.92  0.71 / 0.97  0.74 / 0.99  0.78 / 0.99
//   272 many 0.67 / 0.79  0.66 / 0.86  0.67 / 0.86  0.70 / 0.86  0.71 / 0.83  0.71 / 0.84
//   288 few  0.68 / 0.79  0.65 / 0.88  0.68 / 0.94  0.72 / 0.96  0.75 / 0.97  0.79 / 1.01
//   288 many 0.69 / 0.77  0.67 / 0.85  0.68 / 0.91  0.71 / 0.87  0.72 / 0.84  0.73 / 0.84
//   320 few  0.79 / 0.90  0.78 / 0.96  0.80 / 1.01  0.82 / 0.98  0.83 / 1.01  0.84 / 1.05
//   320 many 0.72 / 0.84  0.71 / 0.90  0.77 / 0.90  0.79 / 0.93  0.81 / 0.94  0.83 / 0.97
//   352 few  0.79 / 0.94  0.79 / 1.05  0.78 / 1.04  0.80 / 1.08  0.83 / 1.10  0.84 / 1.14
//   352 many 0.75 / 0.86  0.74 / 0.92  0.74 / 0.97  0.85 / 0.93  0.80 / 1.00  0.85 / 1.00
//   384 few  0.77 / 0.92  0.82 / 1.03  0.82 / 1.12  0.89 / 1.19  0.93 / 1.21  0.97 / 1.26
//   384 many 0.77 / 0.93  0.81 / 1.04  0.84 / 1.04  0.88 / 1.04  0.89 / 1.04  0.89 / 1.07
//   544 few  0.79 / 0.91  0.74 / 1.06  0.80 / 1.13  0.82 / 1.16  0.84 / 1.17  0.88 / 1.21
//   544 many 0.76 / 0.83  0.72 / 0.94  0.80 / 0.96  0.79 / 0.97  0.79 / 0.98  0.94 / 0.98
//   576 few  0.84 / 0.98  0.83 / 1.09  0.91 / 1.18  0.91 / 1.20  0.93 / 1.21  0.96 / 1.27
//   576 many 0.79 / 0.91  0.78 / 1.00  0.88 / 1.02  0.86 / 1.05  0.97 / 1.04  1.01 / 1.05
//   640 few  0.85 / 1.03  0.83 / 1.13  0.92 / 1.23  0.92 / 1.25  0.95 / 1.33  1.25 / 1.37
//   640 many 0.82 / 0.96  0.81 / 1.04  0.88 / 1.10  0.98 / 1.11  1.05 / 1.11  1.12 / 1.07
// Operands are rarely as cold as that in a layer's pass: beside a rim of an eighth to
// a half of the large items its launches gain to the further lines (passes of layers
// and linears whose launches lie between the two, small / large cut: 208 items and 52
// small of 17 steps 1908 / 1960, 224 and 108 of 24 2468 / 2513, 522 and 154 of 20 1992
// / 2034, 528 and 96 of 18 1226 / 1244, 576 and 196 of 18 490 / 508 us).  Beside fewer
// they do not (one product, three sets of operands in turn: 224 and 8 of 20 steps 83 /
// 69, 384 and 8 of 12 104 / 93, 544 and 8 of 24 211 / 187, 576 and 8 of 10 142 / 127,
// 640 and 8 of 5 123 / 110 with an output 1024 wide; square 0.94 to 1.07).
// Lists with items of other lengths among them keep the balanced schedule of
// both classes: rounds say nothing about those (caches as above: 320 items of 3
// and 1 steps 1.12 / 1.06; 16 steps and a few of 8, 269 items 1.04 / 1.15, 286
// items 0.84 / 0.96).
bool cut_small(const cleave_plan* plan, int cus) {
  const int64_t n = static_cast<int64_t>(plan->items[cleave::kTileLarge].size());
  if (n == 0) return false;
  if (2 * n <= cus) return true;
  const int64_t steps = plan->large_steps, over = n % cus;
  const bool equal = steps - plan->large_steps_least <= 1;   // but for a shorter last chunk
  const int64_t rim = static_cast<int64_t>(plan->items[cleave::kTileSmall].size());
  if (!equal || rim > n) return false;
  const bool few = 8 * rim < n, many = 2 * rim > n;
  switch (n / cus) {
    case 0:
      if (rim > 0) return (4 * n <= 3 * cus && steps <= 24) || (8 * n <= 7 * cus && steps <= (few || many ? 12 : 24));
      return 4 * n <= 3 * cus && steps <= 4;
    case 1:
      if (over == 0) return false;
      if (8 * over <= cus) return true;
      if (rim > 0) return (8 * over <= 3 * cus && steps <= 24) || (2 * over <= cus && steps <= (few ? 8 : 12));
      return 4 * over <= cus && steps <= 16;
    case 2:
      if (over == 0) return false;
      if (rim > 0 && few)
        return (8 * over <= cus && steps <= 16) || (4 * over <= cus && steps <= 8) || (2 * over <= cus && steps <= 4);
      if (rim > 0) return (4 * over <= cus && steps <= 24) || (2 * over <= cus && steps <= 8);
      return 8 * over <= cus && steps <= 8;
    default: return false;
  }
}

int execute_impl(cleave_plan* plan, const int64_t* task_ids, int64_t n_ids, const void* A,
                 int64_t lda, int transA, const void* B, int64_t ldb, int transB, int dtype,
                 float* partials, const BatchLayout& bl, void* hip_stream,
                 const AssembleTarget& asm_to = AssembleTarget{}, bool static_scratch = false,
                 const cleave::LinearArgs* linear = nullptr, const cleave::GatedArgs* gated = nullptr) {
  if (!plan || !A || !B || (!partials && !asm_to.C)) return CLEAVE_EINVAL;
  const bool two = gated && gated->b_up;   // a gated product: the plan's columns are both operands'
  if (dtype != CLEAVE_F32 && dtype != CLEAVE_BF16) return CLEAVE_EINVAL;
  if (plan->pairs && !linear && !gated) return CLEAVE_EINVAL;   // a plan of 8-bit operands
  if ((transA != 0 && transA != 1) || (transB != 0 && transB != 1)) return CLEAVE_EINVAL;
  if ((task_ids == nullptr) != (n_ids == 0) || n_ids < 0) return CLEAVE_EINVAL;
  if (lda < (transA ? plan->M : plan->K) || ldb < (transB ? plan->K : two ? plan->N / 2 : plan->N)) return CLEAVE_EINVAL;
  const int eb = dtype == CLEAVE_BF16 ? 2 : 4;
  if (!aligned(A, eb) || !aligned(B, eb) || !aligned(partials, 4)) return CLEAVE_EINVAL;   // null partials: assemble mode
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);

  int cus = 0;
  int rc = compute_units(&cus);
  if (rc != CLEAVE_OK) return rc;
  int dev = 0;
  CLEAVE_HIP(hipGetDevice(&dev));
  if (static_scratch) {
    // this entry point never allocates: the tables must be on the device already
    if (plan->device != dev) return CLEAVE_EINVAL;
  } else {
    rc = ensure_uploaded(plan);
    if (rc != CLEAVE_OK) return rc;
  }

  // The direct kernel: bf16, every 16 bytes that it fetches (8 elements along the
  // operand's rows as stored) belong to one chunk and one tile and lie on a
  // 16-byte boundary; rows of the output in whole eights.  An operand stored
  // with the inner dimension across its rows takes any chunk, the other kind any
  // tile row.  Chunks that end within a K step against the general kernel (us):
  // 4096 x 4096 x 4128 in 4 splits 230 / 175, 4096 x 8192 x 1032 101 / 71, 8192 x
  // 3072 x 800 in 4 126 / 98, 512 x 512 x 200 5.2 / 4.4; odd chunks of two operands
  // with the inner dimension across, 3000 x 2504 x 3001 in 4 77 / 54; odd rows, 3001
  // x 2504 x 1024 in 4 37 / 30.
  const int e = 16 / eb;
  // (The epilogue's stores take any number of columns, and its kernels read A along K.)
  // (Who asks for a gated product has seen to that.)
  const bool direct =
      gated || (dtype == CLEAVE_BF16 && (plan->all_n_mult8 || (linear && transB)) && !(linear && transA) &&
                (transA ? plan->all_m_mult8 : plan->all_k_mult8) && (!transB || plan->all_k_mult8) && lda % e == 0 && ldb % e == 0 &&
                aligned(A, 16) && aligned(B, 16) &&
                // in-tile byte offsets are kept in 32 bits
                lda * eb < (int64_t{1} << 22) && ldb * eb < (int64_t{1} << 22) &&
                offsets_multiple_of(bl.a, bl.shape, e) && offsets_multiple_of(bl.b, bl.shape, e));
  // 8-bit operands have no general kernel, and partial blocks leave theirs in whole eights of columns (cleave_linear
  // refuses what would come here otherwise, and cleave_plan_linear does not plan it).
  if (plan->pairs && (!direct || (!asm_to.C && !plan->all_n_mult8))) return CLEAVE_EINVAL;
  // An operand of the general kernel's 16-byte loads needs that much between the start of a
  // stored row and the end of any chunk (K-contiguous) or row (otherwise), and
  // in-tile byte offsets (up to 128 rows) that fit 32 bits.
  const bool a_elements = (transA ? plan->M : plan->min_k_end) < e || lda * eb >= (int64_t{1} << 25);
  const bool b_elements = (transB ? plan->min_k_end : plan->N) < e || ldb * eb >= (int64_t{1} << 25);

  const cleave::WorkItem* d_lists[cleave::kNumTileClasses] = {plan->d_items[0], plan->d_items[1]};
  int64_t counts[cleave::kNumTileClasses] = {static_cast<int64_t>(plan->items[0].size()),
                                             static_cast<int64_t>(plan->items[1].size())};
  int64_t steps[cleave::kNumTileClasses] = {plan->items_steps[0], plan->items_steps[1]};   // whole K steps of a list's items
  cleave::ListShape shapes[cleave::kNumTileClasses] = {plan->shape, plan->shape};   // (the general kernel runs all tasks, or a subset)
  // which of the plan's lists a class runs from (-1: a subset's own list)
  int list_of[cleave::kNumTileClasses] = {task_ids ? -1 : 0, task_ids ? -1 : 1};
  // (8-bit operands have no large shape)
  if (!task_ids && (!direct || plan->pairs || cut_small(plan, cus))) {
    list_of[cleave::kTileSmall] = cleave::kNumTileClasses;
    d_lists[cleave::kTileLarge] = nullptr;
    counts[cleave::kTileLarge] = 0;
    d_lists[cleave::kTileSmall] = plan->d_items_fine;
    counts[cleave::kTileSmall] = static_cast<int64_t>(plan->items_fine.size());
    steps[cleave::kTileSmall] = plan->items_steps[cleave::kNumTileClasses];
  }
  // Subset launches: the work-item lists are written on the device, from the
  // task records, into a slice of memory the plan set aside when its tables
  // were uploaded -- stream-ordered, no host wait, no copy, no allocation.
  std::unique_lock<std::mutex> subset_lock;
  int64_t slice_begin = -1, slice_total = 0;
  if (task_ids) {
    subset_lock = std::unique_lock<std::mutex>(plan->subset.mu);
    SubsetLayout layout;
    rc = layout_subset(plan, task_ids, n_ids, cus, &layout);
    if (rc != CLEAVE_OK) return rc;
    slice_total = layout.total();
    cleave::WorkItem* slice = nullptr;
    if (static_scratch) {
      // the device's fixed array, from its start: whatever an earlier call left there is overwritten
      if (slice_total > kStaticScratchItems) return CLEAVE_ELIMIT;
      slice = g_static_scratch[dev];
    } else {
      hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
      CLEAVE_HIP(hipStreamIsCapturing(stream, &capture));
      rc = acquire_subset_slice(plan->subset, slice_total, capture != hipStreamCaptureStatusNone, &slice,
                                &slice_begin);
      if (rc != CLEAVE_OK) return rc;
    }
    rc = expand_subset(plan, task_ids, n_ids, layout, slice, stream);
    if (rc != CLEAVE_OK) {
      if (!static_scratch) (void)release_subset_slice(plan->subset, slice_begin, slice_total, stream);
      return rc;
    }
    int64_t pos = 0;
    for (int c = 0; c < cleave::kNumTileClasses; ++c) {
      d_lists[c] = slice + pos;
      steps[c] = layout.steps[c];
      shapes[c] = layout.shapes[c];
      counts[c] = layout.counts[c];
      pos += counts[c];
    }
  }

  // whatever has been enqueued reads the slice: mark it even if a later launch fails
  const auto launch_failed = [&](hipError_t e) {
    if (task_ids && !static_scratch) (void)release_subset_slice(plan->subset, slice_begin, slice_total, stream);
    return hip_fail(e);
  };
  int64_t most = -1;
  for (int c = 0; c < cleave::kNumTileClasses; ++c) {
    if (counts[c] == 0) continue;
    cleave::ExecuteArgs args{};
    args.items = d_lists[c];
    args.n_items = counts[c];
    args.A = A;
    args.B = B;
    args.lda = lda;
    args.ldb = ldb;
    args.transA = transA;
    args.transB = transB;
    args.partials = partials;
    args.batch = bl.shape;
    args.a_at = bl.a;
    args.b_at = bl.b;
    args.c_at = bl.c;
    args.C = asm_to.C;
    args.M = plan->M;
    args.N = plan->N;
    args.K = plan->K;
    args.ldc = asm_to.ldc;
    args.stream_below_k = task_ids ? 0 : streamed_below(plan, asm_to);
    args.c_bf16 = asm_to.out_dtype == CLEAVE_BF16 ? 1 : 0;
    const bool large = c == cleave::kTileLarge;
    if (direct) {
      // Persistent workgroups, as many as the chip holds at once: each walks
      // the item list with the grid as stride and fetches the head of its next
      // item while it stores the current one.
      const cleave::DirectShape shape = direct_shape(c, counts[c], cus);
      const int64_t resident = static_cast<int64_t>(cus) * cleave::direct_workgroups_per_cu(shape);
      const int grid = static_cast<int>(std::min<int64_t>(counts[c], resident));
      // items of unequal length: the schedule made for this grid when the tables were uploaded
      const int list = list_of[c];
      args.wg_ranges = (list >= 0 && plan->wg_ranges_grid[list] == grid)
                           ? plan->d_wg_ranges[list] : nullptr;
      if (args.wg_ranges && list == cleave::kNumTileClasses) args.items += counts[c];   // behind the list as laid out
      const hipError_t he = two && plan->pairs ? cleave::launch_gated_8bit(args, *gated, shape, plan->chunk_tails, grid, stream)
                            : two       ? cleave::launch_gated_direct(args, *gated, shape, plan->chunk_tails, grid, stream)
                            : gated     ? cleave::launch_gated_grad_direct(args, *gated, shape, plan->chunk_tails, grid, stream)
                            : plan->pairs ? cleave::launch_linear_8bit(args, *linear, shape, plan->chunk_tails, grid, stream)
                            : linear    ? cleave::launch_linear_direct(args, *linear, shape, plan->chunk_tails, grid, stream)
                                        : cleave::launch_execute_direct(args, shape, plan->chunk_tails, grid, stream);
      if (he != hipSuccess) return launch_failed(he);
      if (counts[c] > most)
        plan->last_kernel = gated ? gated_kernel_name(shape, two ? plan->pairs : 2, transB)
                            : linear ? linear_direct_kernel_name(shape, plan->pairs, transB) : direct_kernel_name(shape, transA, transB);
    } else {
      // in-tile byte offsets (256 rows) stay within 32 bits
      const bool by_k = !transA && transB && !a_elements && !b_elements && lda * eb < (int64_t{1} << 24) &&
                        ldb * eb < (int64_t{1} << 24);
      const int64_t items = counts[c] * (large ? 4 : 1);
      cleave::GeneralLoads how{
          general_tile(dtype, !transA && transB, items, shapes[c], large && dtype == CLEAVE_BF16 && by_k ? counts[c] : 0,
                       steps[c], cus),
          a_elements, b_elements, shapes[c], cus};
      if (how.tile == cleave::kTileWide && cleave::four_waves(dtype, transA, transB, items, shapes[c], cus))
        how.tile = cleave::kTileWide4;
      if (how.tile == cleave::kTileNarrow && cleave::runs_lone(dtype, c, counts[c], shapes[c], cus))
        how.tile = cleave::kTileLone;
      if (linear)   // (two tiles serve an epilogue)
        how.tile = how.tile == cleave::kTileLone || how.tile == cleave::kTileQuarter || how.tile == cleave::kTileNarrow
                       ? cleave::kTileLone
                       : cleave::kTileWide4;
      const hipError_t he = linear ? cleave::launch_linear_general(args, *linear, dtype, c, how, stream)
                                   : cleave::launch_execute(args, dtype, c, how, stream);
      if (he != hipSuccess) return launch_failed(he);
      if (counts[c] > most)
        plan->last_kernel = linear ? linear_kernel_name(dtype, how, transA, transB) : kernel_name(dtype, how, transA, transB);
    }
    most = std::max(most, counts[c]);
  }
  if (task_ids && !static_scratch) return release_subset_slice(plan->subset, slice_begin, slice_total, stream);
  return CLEAVE_OK;
}

}  // namespace

extern "C" int cleave_execute(cleave_plan* plan, const int64_t* task_ids, int64_t n_ids,
                              const void* A, int64_t lda, int transA, const void* B, int64_t ldb,
                              int transB, int dtype, float* partials, void* hip_stream) {
  if (plan && plan->batch > 0) return CLEAVE_EINVAL;   // batched plans use the batched call
  return execute_impl(plan, task_ids, n_ids, A, lda, transA, B, ldb, transB, dtype, partials,
                      BatchLayout{}, hip_stream);
}

extern "C" int cleave_execute_noalloc(cleave_plan* plan, const int64_t* task_ids, int64_t n_ids,
                                      const void* A, int64_t lda, int transA, const void* B,
                                      int64_t ldb, int transB, int dtype, float* partials,
                                      void* hip_stream) {
  if (plan && plan->batch > 0) return CLEAVE_EINVAL;
  return execute_impl(plan, task_ids, n_ids, A, lda, transA, B, ldb, transB, dtype, partials,
                      BatchLayout{}, hip_stream, AssembleTarget{}, true);
}

extern "C" int cleave_execute_batched(cleave_plan* plan, const int64_t* task_ids, int64_t n_ids,
                                      const void* A, int64_t lda, int transA, int64_t a_outer,
                                      int64_t a_inner, const void* B, int64_t ldb, int transB,
                                      int64_t b_outer, int64_t b_inner, int64_t n_inner, int dtype,
                                      float* partials, void* hip_stream) {
  if (!plan || plan->batch < 1) return CLEAVE_EINVAL;
  if (n_inner < 1 || n_inner > std::numeric_limits<uint32_t>::max() || plan->batch % n_inner != 0)
    return CLEAVE_EINVAL;
  if (a_outer < 0 || a_inner < 0 || b_outer < 0 || b_inner < 0) return CLEAVE_EINVAL;
  return execute_impl(plan, task_ids, n_ids, A, lda, transA, B, ldb, transB, dtype, partials,
                      strided_layout(n_inner, a_outer, a_inner, b_outer, b_inner, 0, 0), hip_stream);
}

extern "C" int cleave_execute_grouped(cleave_plan* plan, const int64_t* task_ids, int64_t n_ids,
                                      int64_t n_members, const void* const* A_list, int64_t lda,
                                      int transA,
                                      const void* const* B_list, int64_t ldb, int transB, int dtype,
                                      float* partials, void* hip_stream) {
  if (!plan || plan->batch < 1 || plan->batch > cleave::kMaxGroup || n_members != plan->batch)
    return CLEAVE_EINVAL;
  if (dtype != CLEAVE_F32 && dtype != CLEAVE_BF16) return CLEAVE_EINVAL;
  const int eb = dtype == CLEAVE_BF16 ? 2 : 4;
  BatchLayout bl;
  bl.shape.n_group = static_cast<uint32_t>(plan->batch);
  const void* A = nullptr;
  const void* B = nullptr;
  int rc = group_offsets(A_list, plan->batch, eb, &bl.a, &A);
  if (rc != CLEAVE_OK) return rc;
  rc = group_offsets(B_list, plan->batch, eb, &bl.b, &B);
  if (rc != CLEAVE_OK) return rc;
  return execute_impl(plan, task_ids, n_ids, A, lda, transA, B, ldb, transB, dtype, partials, bl,
                      hip_stream);
}

extern "C" int cleave_execute_assemble(cleave_plan* plan, const int64_t* task_ids, int64_t n_ids,
                                       const void* A, int64_t lda, int transA, int64_t a_outer,
                                       int64_t a_inner, const void* B, int64_t ldb, int transB,
                                       int64_t b_outer, int64_t b_inner, int64_t n_inner, int dtype,
                                       void* C, int64_t ldc, int64_t c_outer, int64_t c_inner,
                                       int out_dtype, void* hip_stream) {
  if (!plan || !C) return CLEAVE_EINVAL;
  if (out_dtype != CLEAVE_F32 && out_dtype != CLEAVE_BF16) return CLEAVE_EINVAL;
  if (ldc < plan->N || !aligned(C, out_dtype == CLEAVE_BF16 ? 2 : 4)) return CLEAVE_EINVAL;
  // a block is the finished output only if its task covers the whole inner dimension
  for (const cleave_task& t : plan->tasks)
    if (t.ksplit_cnt != 1) return CLEAVE_EINVAL;
  BatchLayout bl;
  if (plan->batch > 0) {
    if (n_inner < 1 || n_inner > std::numeric_limits<uint32_t>::max() || plan->batch % n_inner != 0)
      return CLEAVE_EINVAL;
    if (a_outer < 0 || a_inner < 0 || b_outer < 0 || b_inner < 0 || c_outer < 0 || c_inner < 0)
      return CLEAVE_EINVAL;
    bl = strided_layout(n_inner, a_outer, a_inner, b_outer, b_inner, c_outer, c_inner);
  } else if (n_inner != 0 || a_outer || a_inner || b_outer || b_inner || c_outer || c_inner) {
    return CLEAVE_EINVAL;   // strides belong to batched plans
  }
  AssembleTarget to;
  to.C = C;
  to.ldc = ldc;
  to.out_dtype = out_dtype;
  return execute_impl(plan, task_ids, n_ids, A, lda, transA, B, ldb, transB, dtype, nullptr, bl,
                      hip_stream, to);
}

namespace {

// Which operator consumes the aggregated values.
struct ReduceEpilogue {
  const void* residual = nullptr;          // C = sum + residual
  const cleave::AdamArgs* adam = nullptr;  // Adam update of adam->w (C unused)
  const cleave::AdamGroupOffsets* adam_group = nullptr;   // with adam: one set of arrays per member
};

int reduce_impl(cleave_plan* plan, const float* partials, void* C, int64_t ldc, int out_dtype,
                const BatchLayout& bl, void* hip_stream,
                const ReduceEpilogue& epi = ReduceEpilogue{}, bool members_aligned = true) {
  if (!plan || plan->pairs || !partials || !C) return CLEAVE_EINVAL;   // (pairs: a plan of 8-bit operands)
  if (out_dtype != CLEAVE_F32 && out_dtype != CLEAVE_BF16) return CLEAVE_EINVAL;
  if (ldc < plan->N) return CLEAVE_EINVAL;
  const int ob = out_dtype == CLEAVE_BF16 ? 2 : 4;
  if (!aligned(partials, 4) || !aligned(C, ob)) return CLEAVE_EINVAL;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);

  int rc = ensure_uploaded(plan);
  if (rc != CLEAVE_OK) return rc;

  bool vec = plan->all_n_mult4 && ldc % 4 == 0 && aligned(partials, 16) && aligned(C, 4 * ob) &&
             offsets_multiple_of(bl.c, bl.shape, 4) && members_aligned;
  if (epi.residual) vec = vec && aligned(epi.residual, 4 * ob);
  if (epi.adam)
    vec = vec && aligned(epi.adam->m, 16) && aligned(epi.adam->v, 16) &&
          (!epi.adam->w_bf16 || aligned(epi.adam->w_bf16, 8));
  cleave::ReduceArgs args{};
  args.items = plan->d_reduce_items;
  args.n_items = plan->reduce_runs;
  args.partials = partials;
  args.C = C;
  args.ldc = ldc;
  args.batch = bl.shape;
  args.c_at = bl.c;
  // one workgroup per reduce item (the kernel loops only if the grid is capped)
  const int grid = static_cast<int>(std::min<int64_t>(args.n_items, int64_t{1} << 20));
  if (epi.adam && epi.adam_group) {
    CLEAVE_HIP(cleave::launch_reduce_adam_grouped(args, *epi.adam, *epi.adam_group, vec, grid, stream));
  } else if (epi.adam) {
    CLEAVE_HIP(cleave::launch_reduce_adam(args, *epi.adam, vec, grid, stream));
  } else if (epi.residual) {
    CLEAVE_HIP(cleave::launch_reduce_residual(args, epi.residual, out_dtype, vec, grid, stream));
  } else {
    CLEAVE_HIP(cleave::launch_reduce(args, out_dtype, vec, grid, stream));
  }
  return CLEAVE_OK;
}

}  // namespace

extern "C" int cleave_reduce_residual(cleave_plan* plan, const float* partials, const void* R,
                                      void* C, int64_t ldc, int out_dtype, void* hip_stream) {
  if (!R || (plan && plan->batch > 0)) return CLEAVE_EINVAL;
  if (out_dtype != CLEAVE_F32 && out_dtype != CLEAVE_BF16) return CLEAVE_EINVAL;
  if (!aligned(R, out_dtype == CLEAVE_BF16 ? 2 : 4)) return CLEAVE_EINVAL;
  ReduceEpilogue epi;
  epi.residual = R;
  return reduce_impl(plan, partials, C, ldc, out_dtype, BatchLayout{}, hip_stream, epi);
}

extern "C" int cleave_reduce_adam(cleave_plan* plan, const float* partials, float* w, float* m,
                                  float* v, void* w_bf16, int64_t ld, float lr, float beta1,
                                  float beta2, float eps, float weight_decay, int64_t step,
                                  void* hip_stream) {
  if (!w || !m || !v || (plan && plan->batch > 0)) return CLEAVE_EINVAL;
  if (step < 1 || !(beta1 >= 0.0f && beta1 < 1.0f) || !(beta2 >= 0.0f && beta2 < 1.0f) ||
      !(eps >= 0.0f) || !(lr == lr) || !(weight_decay == weight_decay))
    return CLEAVE_EINVAL;
  if (!aligned(m, 4) || !aligned(v, 4) || !aligned(w_bf16, 2)) return CLEAVE_EINVAL;
  cleave::AdamArgs h{};
  h.w = w;
  h.m = m;
  h.v = v;
  h.w_bf16 = static_cast<uint16_t*>(w_bf16);
  h.lr = lr;
  h.beta1 = beta1;
  h.beta2 = beta2;
  h.eps = eps;
  h.weight_decay = weight_decay;
  h.inv_bias1 = static_cast<float>(1.0 / (1.0 - std::pow(static_cast<double>(beta1), static_cast<double>(step))));
  h.inv_bias2 = static_cast<float>(1.0 / (1.0 - std::pow(static_cast<double>(beta2), static_cast<double>(step))));
  ReduceEpilogue epi;
  epi.adam = &h;
  // the fp32 master weight takes C's place in the common checks (pointer, leading dimension)
  return reduce_impl(plan, partials, w, ld, CLEAVE_F32, BatchLayout{}, hip_stream, epi);
}

extern "C" int cleave_reduce_adam_grouped(cleave_plan* plan, const float* partials, int64_t n_members,
                                          float* const* w_list, float* const* m_list,
                                          float* const* v_list, void* const* w_bf16_list, int64_t ld,
                                          float lr, float beta1, float beta2, float eps,
                                          float weight_decay, int64_t step, void* hip_stream) {
  if (!plan || plan->batch < 1 || plan->batch > cleave::kMaxGroup || n_members != plan->batch)
    return CLEAVE_EINVAL;
  if (!w_list || !m_list || !v_list) return CLEAVE_EINVAL;
  if (step < 1 || !(beta1 >= 0.0f && beta1 < 1.0f) || !(beta2 >= 0.0f && beta2 < 1.0f) ||
      !(eps >= 0.0f) || !(lr == lr) || !(weight_decay == weight_decay))
    return CLEAVE_EINVAL;
  cleave::AdamGroupOffsets at{};
  bool all16 = true;
  for (int64_t g = 0; g < n_members; ++g) {
    if (!w_list[g] || !m_list[g] || !v_list[g] || (w_bf16_list && !w_bf16_list[g])) return CLEAVE_EINVAL;
    if (!aligned(w_list[g], 4) || !aligned(m_list[g], 4) || !aligned(v_list[g], 4) ||
        (w_bf16_list && !aligned(w_bf16_list[g], 2)))
      return CLEAVE_EINVAL;
    all16 = all16 && aligned(w_list[g], 16) && aligned(m_list[g], 16) && aligned(v_list[g], 16) &&
            (!w_bf16_list || aligned(w_bf16_list[g], 8));
    at.w[g] = w_list[g] - w_list[0];
    at.m[g] = m_list[g] - m_list[0];
    at.v[g] = v_list[g] - v_list[0];
    at.w_bf16[g] = w_bf16_list ? static_cast<uint16_t*>(w_bf16_list[g]) - static_cast<uint16_t*>(w_bf16_list[0]) : 0;
  }
  cleave::AdamArgs h{};
  h.w = w_list[0];
  h.m = m_list[0];
  h.v = v_list[0];
  h.w_bf16 = w_bf16_list ? static_cast<uint16_t*>(w_bf16_list[0]) : nullptr;
  h.lr = lr;
  h.beta1 = beta1;
  h.beta2 = beta2;
  h.eps = eps;
  h.weight_decay = weight_decay;
  h.inv_bias1 = static_cast<float>(1.0 / (1.0 - std::pow(static_cast<double>(beta1), static_cast<double>(step))));
  h.inv_bias2 = static_cast<float>(1.0 / (1.0 - std::pow(static_cast<double>(beta2), static_cast<double>(step))));
  ReduceEpilogue epi;
  epi.adam = &h;
  epi.adam_group = &at;
  BatchLayout bl;
  bl.shape.n_group = static_cast<uint32_t>(plan->batch);   // c_at stays zero: every array has its own table
  // reduce_impl's vector-path test looks at h's (member 0's) arrays; the members must agree
  // (a member whose arrays are not 16-byte aligned sends the whole launch down the element path)
  return reduce_impl(plan, partials, h.w, ld, CLEAVE_F32, bl, hip_stream, epi, all16);
}

extern "C" int cleave_reduce(cleave_plan* plan, const float* partials, void* C, int64_t ldc,
                             int out_dtype, void* hip_stream) {
  if (plan && plan->batch > 0) return CLEAVE_EINVAL;
  return reduce_impl(plan, partials, C, ldc, out_dtype, BatchLayout{}, hip_stream);
}

extern "C" int cleave_reduce_batched(cleave_plan* plan, const float* partials, void* C, int64_t ldc,
                                     int64_t c_outer, int64_t c_inner, int64_t n_inner,
                                     int out_dtype, void* hip_stream) {
  if (!plan || plan->batch < 1) return CLEAVE_EINVAL;
  if (n_inner < 1 || n_inner > std::numeric_limits<uint32_t>::max() || plan->batch % n_inner != 0)
    return CLEAVE_EINVAL;
  if (c_outer < 0 || c_inner < 0) return CLEAVE_EINVAL;
  return reduce_impl(plan, partials, C, ldc, out_dtype,
                     strided_layout(n_inner, 0, 0, 0, 0, c_outer, c_inner), hip_stream);
}

extern "C" int cleave_reduce_grouped(cleave_plan* plan, const float* partials, int64_t n_members,
                                     void* const* C_list, int64_t ldc, int out_dtype,
                                     void* hip_stream) {
  if (!plan || plan->batch < 1 || plan->batch > cleave::kMaxGroup || n_members != plan->batch)
    return CLEAVE_EINVAL;
  if (out_dtype != CLEAVE_F32 && out_dtype != CLEAVE_BF16) return CLEAVE_EINVAL;
  BatchLayout bl;
  bl.shape.n_group = static_cast<uint32_t>(plan->batch);
  const void* C = nullptr;
  const int rc = group_offsets(C_list, plan->batch, out_dtype == CLEAVE_BF16 ? 2 : 4, &bl.c, &C);
  if (rc != CLEAVE_OK) return rc;
  return reduce_impl(plan, partials, const_cast<void*>(C), ldc, out_dtype, bl, hip_stream);
}

// ---- linear product ------------------------------------------------------------

namespace {

// Splits of K for products whose tiles alone leave CUs idle: a second launch joins them (3 to 4 us with the partial sums'
// way), so only chains of some length are split.  The chunks are whole sixteen bytes of the operands (`e` elements)
// where K is.
//   Few rows: up to 128 groups of 64 columns leave CUs without one, 257 to 384 give two to some and one to the others; where a
// row of K has 5 KB or more those split, to one per CU, these in two.  One row, bf16, us, 1, 2, 4 splits, the weights from
// memory / from the caches: K x N = 4096 x 4096 20, 16, 13 / 12, 12, 9, 4096 x 5632 22, 17, 17 / 14, 13, 8192 x 8192 40, 32, 32 / 24, 25,
// stored N x K 46, 33, 35 / 34, 28, 4096 x 22016 49, 42, 43 / 34, 32; 4096 x 8192 21, 20, 19 / 14, 16, N x K 25, 19, 21 / 18, 16; as they
// are 4096 x 11008 21, 25, 23 / 17.6, 20, 2048 x 6144 12.2, 11.7, 12.1 / 7.0, 7.7, 5120 x 27648 62, 65, 60 / 51, 53.
//   Tiles, us, 1, 2, 4, 8 splits: bf16, 64 x 512 x 11008 32.5, 20.6, 13.6, 14.2, 128 x 768 x 3072 11.8, 10.5, 9.1, 12.2, 300 x 512 x
// 4096 14.8, 12.7, 10.3, 14.4, 64 x 4096 x 4096 16.8, 15.0, 15.3, 19.7, 500 x 1024 x 4096 15.4, 14.3, 15.3, 19.1, 256 x 4096 x 4096
// 17.5, 21.7, 21.0, 26.0, 64 x 4096 x 1024 6.7, 9.2, 9.8, 15.2; where two splits make one 128 x 128 item per CU, 64 x 11008 x
// 4096 29.1, 23.2, 24.7, 29.5, 128 x 11008 x 4096 29.3, 24.9, 27.9, 33.3, 256 x 8192 x 4096 29.3, 28.1, 30.9, 39.2.
//   fp32 is bound by its products: a 64 x 64 part takes 17.6 ns per k alone on its CU, two on one CU twice that, so the
// time is the most parts that a CU gets times their chunks, and the join with the partial sums' way.  Up to three parts per CU,
// beyond which the last round counts for little, the least of one to four splits is taken, us, 1, 2, 3, 4 splits: 64 x 4096 x 4096 71, 42, 32, 28, 500 x 1000 x 1000 24, 19, 22, 21, 1590 x 313 x 3890 75, 50,
// 58, 50, 162 x 2752 x 7768 136, 122, 92, 101, 1300 x 1226 x 4793 153, 158, 139, 150, 3835 x 704 x 3904 250, 195, 179, 186,
// 1000 x 1000 x 4000, a part per CU as it is, 73, 81, 78, 77.
struct Fp32Splits {
  int64_t splits, workgroups;
};
Fp32Splits fp32_splits(int64_t M, int64_t N, int64_t K) {
  constexpr int64_t kCUs = 256;
  const int64_t parts = ((M + 63) / 64) * ((N + 63) / 64);
  int64_t best = 1;
  double least = 0.0;
  const int64_t most = parts <= 3 * kCUs ? std::min<int64_t>(4, K / 256) : 1;
  for (int64_t S = 1; S <= std::max<int64_t>(most, 1); ++S) {
    const int64_t chunk = (K + S - 1) / S;
    double us = 0.0176 * static_cast<double>((parts * S + kCUs - 1) / kCUs * chunk);
    if (S > 1) us += 4.0 + 2.0 * 16384.0 * static_cast<double>(parts * S) / 4.5e6;
    if (S > 1 && us >= least) continue;
    least = us;
    best = S;
  }
  return {best, parts * best};
}
int64_t linear_splits(int64_t M, int64_t N, int64_t K, int64_t e, bool pairs) {
  constexpr int64_t kCUs = 256;
  if (pairs && M > cleave::kFewRows && N % 8 != 0) return 1;   // (partial blocks leave the 8-bit kernel in whole eights)
  int64_t want = 1;
  if (M <= cleave::kFewRows) {
    const int64_t groups = (N + 63) / 64;
    if (K * 16 / e >= 5120) {
      if (groups <= kCUs / 2) want = std::min<int64_t>({kCUs / groups, K / (32 * e), 16});
      else if (groups > kCUs && groups <= kCUs / 2 * 3) want = 2;
    }
  } else {
    const int64_t parts = ((M + 63) / 64) * ((N + 63) / 64);
    const int64_t items = ((M + 127) / 128) * ((N + 127) / 128);
    if (e == 4) return fp32_splits(M, N, K).splits;
    if (K >= 3000 && parts <= 48) want = 4;
    else if (K >= 3000 && (parts <= kCUs / 2 || (items > kCUs / 4 && items <= kCUs / 2))) want = 2;
  }
  for (int64_t S = want; S > 1; --S) {
    const int64_t chunk = (K + S - 1) / S;
    // (what takes chunks of any length anyway, or cuts its own, is split at any)
    if ((S - 1) * chunk < K && (chunk % e == 0 || K % e != 0 || e == 4 || M <= cleave::kFewRows)) return S;
  }
  return 1;
}

bool linear_dtype(int dtype) { return dtype == CLEAVE_F32 || dtype == CLEAVE_BF16 || dtype == CLEAVE_E4M3; }

}  // namespace

extern "C" int cleave_plan_linear(int64_t M, int64_t N, int64_t K, int dtype, cleave_plan** out) {
  if (!linear_dtype(dtype) || !out || M < 1 || N < 1 || K < 1) return CLEAVE_EINVAL;
  constexpr int64_t kMost = std::numeric_limits<int32_t>::max();
  if (M > kMost || N > kMost || K > kMost) return CLEAVE_EINVAL;
  const bool pairs = dtype == CLEAVE_E4M3;
  if (pairs && K % 16 != 0) return CLEAVE_EINVAL;
  const int64_t k = pairs ? K / 2 : K;
  // (fp32 in tiles of one part each where several go to a CU: parts of larger tiles that hold nothing would take their turn
  // among them.  us, 64 x 64 / 256 x 256: 167 x 1226 x 4793 in 4 splits 35 / 51, 162 x 2752 x 7768 in 3 92 / 126; in one split, and
  // few parts, which are quartered, 2048 x 2048 x 2048 147 / 137, 124 x 768 x 2432 in 4 19 / 16)
  const Fp32Splits parts = dtype == CLEAVE_F32 ? fp32_splits(M, N, K) : Fp32Splits{1, 0};
  const int64_t tile = M <= cleave::kFewRows                        ? cleave::kSmallTileRows
                       : parts.splits > 1 && parts.workgroups > 128 ? 64
                                                                    : cleave::kLargeTileRows;
  const int rc = cleave_plan_uniform(M, N, k, tile, tile,
                                     static_cast<int32_t>(linear_splits(M, N, k, dtype == CLEAVE_F32 ? 4 : 8, pairs)), 0, out);
  if (rc != CLEAVE_OK) return rc;
  (*out)->linear = true;
  (*out)->for_fp32 = dtype == CLEAVE_F32;
  (*out)->pairs = pairs;
  return CLEAVE_OK;
}

extern "C" int64_t cleave_linear_workspace(const cleave_plan* plan) {
  if (!plan || plan->batch > 0) return CLEAVE_EINVAL;
  return plan->uniform_splits == 1 ? 0 : plan->partial_elems;
}

extern "C" int cleave_linear(cleave_plan* plan, const cleave_linear_args* a, void* hip_stream) {
  if (!plan || !a || plan->batch > 0 || !linear_dtype(a->dtype)) return CLEAVE_EINVAL;
  const bool e4m3 = a->dtype == CLEAVE_E4M3;
  if (plan->pairs != e4m3 || !a->A || !a->B || !a->C) return CLEAVE_EINVAL;
  if ((a->transA != 0 && a->transA != 1) || (a->transB != 0 && a->transB != 1)) return CLEAVE_EINVAL;
  if (a->out_dtype != CLEAVE_F32 && a->out_dtype != CLEAVE_BF16) return CLEAVE_EINVAL;
  if (a->act < CLEAVE_ACT_NONE || a->act > CLEAVE_ACT_SILU || (a->act_grad != 0 && a->act_grad != 1)) return CLEAVE_EINVAL;
  if (a->act_grad && (a->bias || (a->act != CLEAVE_ACT_NONE && !a->preact))) return CLEAVE_EINVAL;
  if (e4m3 != (a->scale_a != nullptr) || e4m3 != (a->scale_b != nullptr)) return CLEAVE_EINVAL;
  const int ob = a->out_dtype == CLEAVE_BF16 ? 2 : 4, eb = e4m3 ? 1 : a->dtype == CLEAVE_BF16 ? 2 : 4;
  const int64_t M = plan->M, N = plan->N, K = e4m3 ? 2 * plan->K : plan->K;
  if (a->lda < (a->transA ? M : K) || a->ldb < (a->transB ? K : N) || a->ldc < N || (a->residual && a->ldr < N) ||
      (a->preact && a->ldz < N))
    return CLEAVE_EINVAL;
  if (!aligned(a->A, eb) || !aligned(a->B, eb) || !aligned(a->C, ob) || !aligned(a->residual, ob) || !aligned(a->preact, ob) ||
      !aligned(a->bias, 4) || !aligned(a->scale_a, 4) || !aligned(a->scale_b, 4) || !aligned(a->partials, 4))
    return CLEAVE_EINVAL;
  // in place: the same elements at the same places, and not two outputs
  if ((a->residual == a->C && M > 1 && a->ldr != a->ldc) || (a->preact == a->C && (!a->act_grad || (M > 1 && a->ldz != a->ldc))))
    return CLEAVE_EINVAL;
  if (e4m3 && (a->transA || !a->transB || !aligned(a->A, 16) || !aligned(a->B, 16) || a->lda % 16 || a->ldb % 16 ||
               a->lda >= int64_t{1} << 22 || a->ldb >= int64_t{1} << 22))
    return CLEAVE_EINVAL;
  const int64_t splits = plan->uniform_splits;
  const bool joined = splits != 1;
  const void* const z = a->act_grad ? nullptr : a->preact;   // an output
  if (joined && (!a->partials || !cleave::apart({a->partials}, {a->A, a->B, a->C, a->preact, a->residual, a->bias, a->scale_a, a->scale_b})))
    return CLEAVE_EINVAL;
  if (!cleave::apart({a->C, z}, {a->A, a->B, a->bias, a->scale_a, a->scale_b})) return CLEAVE_EINVAL;

  cleave::LinearArgs epi{};
  epi.bias = a->bias;
  epi.scale_a = a->scale_a;
  epi.scale_b = a->scale_b;
  epi.residual = a->residual;
  epi.preact = a->act_grad && a->act == CLEAVE_ACT_NONE ? nullptr : a->preact;
  epi.ldr = a->ldr;
  epi.ldz = a->ldz;
  epi.act = a->act;
  epi.grad = a->act_grad;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  int rc = ensure_uploaded(plan);
  if (rc == CLEAVE_OK) rc = ensure_linear_ready(plan->device);
  if (rc != CLEAVE_OK) return rc;

  // (a launch has fewer than 2^32 threads)
  const bool few_rows = M <= cleave::kFewRows && !a->transA && splits >= 1 && N <= int64_t{1} << 27;
  // (its chunks end on whole lines of 128 bytes; the last ones may be short, or empty, which leaves zeros)
  const int64_t line = 128 / eb, chunk = few_rows ? ((K + splits - 1) / splits + line - 1) / line * line : 0;
  AssembleTarget to;
  to.C = joined ? nullptr : a->C;
  to.ldc = a->ldc;
  to.out_dtype = a->out_dtype;
  if (few_rows) {
    cleave::ExecuteArgs args{};
    args.A = a->A;
    args.B = a->B;
    args.lda = a->lda;
    args.ldb = a->ldb;
    args.transB = a->transB;
    args.partials = a->partials;
    args.C = a->C;
    args.ldc = a->ldc;
    args.c_bf16 = a->out_dtype == CLEAVE_BF16;
    args.M = M;
    args.N = N;
    args.K = K;
    CLEAVE_HIP(cleave::launch_linear_few_rows(args, epi, a->dtype, static_cast<int>(splits), chunk, stream));
    plan->last_kernel = "linear_few_rows";
  } else {
    // (nothing to do behind the sums: the blocks themselves)
    const bool bare = !e4m3 && (joined || (!epi.bias && !epi.residual && !epi.preact && epi.act == CLEAVE_ACT_NONE));
    rc = execute_impl(plan, nullptr, 0, a->A, e4m3 ? a->lda / 2 : a->lda, a->transA, a->B, e4m3 ? a->ldb / 2 : a->ldb, a->transB,
                      e4m3 ? CLEAVE_BF16 : a->dtype, joined ? a->partials : nullptr, BatchLayout{}, hip_stream, to, false,
                      bare ? nullptr : &epi);
    if (rc != CLEAVE_OK) return rc;
  }
  if (!joined) return CLEAVE_OK;
  cleave::ReduceArgs args{};
  args.items = few_rows ? nullptr : plan->d_reduce_items;
  args.n_items = plan->reduce_runs;
  args.partials = a->partials;
  args.C = a->C;
  args.ldc = a->ldc;
  CLEAVE_HIP(cleave::launch_linear_join(args, epi, M, N, static_cast<int>(splits), a->out_dtype,
                                        plan->all_n_mult4 && aligned(a->partials, 16), stream));
  return CLEAVE_OK;
}

// ---- gated product ---------------------------------------------------------------

namespace {

// Few rows are read as cleave_linear reads them.
bool gated_few_rows(int64_t M, int64_t N) { return M <= cleave::kFewRows && N <= int64_t{1} << 27; }

// What the direct kernel takes of bf16 operands (in units of it: pairs of e4m3): whole sixteen bytes, in-tile offsets of 32 bits.
constexpr int64_t kMostPitch = (int64_t{1} << 21) - 8;
bool whole_operand(const void* p, int64_t ld) { return aligned(p, 16) && ld % 8 == 0 && ld <= kMostPitch; }

// bf16 operands that are not whole are laid out again, in the workspace, in rows of whole sixteen bytes, zeros behind their ends (one pass
// over what is not whole), for the direct kernel, where there are rows enough that the way through the general kernel
// and fp32 partial blocks takes longer.  us, general / laid out, weights of K x N stored so where nothing else is said:
//   gated, whole K  4096 x 11007: 512, 800, 1024, 1999, 4096 rows 146 / 169, 242 / 250, 286 / 252, 564 / 371, 1058 / 641
//                   1000 x 2500: 800, 1999, 4096 rows 30 / 30, 45.5 / 42.5, 78 / 70
//                   2048 x 4100: 800, 1200, 2048 rows 49 / 48, 68 / 73, 112 / 79
//   gated, odd K    4097 x 11008: 200, 400, 800 rows 107 / 91, 151 / 102, 260 / 202 (stored N x K 135 / 147, 192 / 171, 308 / 271)
//                   1001 x 2500: 18.9 / 21.4, 24.3 / 23.0, 32.3 / 30.0
//   gradient, odd K 4097 x 11008: 200, 400, 800, 2048 rows 60 / 51, 102 / 71, 150 / 150, 299 / 234 (N x K 74 / 78, 125 / 109, 183 / 171, 347 / 262)
//                   2049 x 4096: 200, 400, 800 rows 20.5 / 14.9, 29.0 / 24.8, 37.9 / 31.3
//   gradient, odd N (the output's rows cost the direct kernel's stores more than the join's)
//                   4096 x 11007: 800, 1024, 1999, 4096 rows 149 / 199, 159 / 178, 299 / 293, 572 / 440
//                   2048 x 4100: 1200, 2048, 4096 rows 49 / 49, 71 / 73, 126 / 91; 2048 x 2500: 33 / 40, 49 / 49, 77 / 84
//                   1000 x 2500: 4096 rows 56 / 71
int64_t eights(int64_t n) { return (n + 7) / 8 * 8; }
bool packs(int64_t M, int64_t N, int64_t K) {
  return M >= (K % 8 != 0 ? 384 : 768) && eights(N) <= kMostPitch && eights(K) <= kMostPitch;
}
bool packs_grad(int64_t M, int64_t N, int64_t K) {
  return (N % 8 == 0 ? M >= 384 : M >= 2048 && K >= 2048) && eights(N) <= kMostPitch && eights(K) <= kMostPitch;
}
// Floats of the workspace: A and `weights` operands B, in either layout, from a 16-byte boundary on.
int64_t packed_floats(int64_t M, int64_t N, int64_t K, int64_t weights) {
  return (M * eights(K) + weights * std::max(N * eights(K), K * eights(N))) / 2 + 4;
}

// What calls of the plan need on the device: few rows nothing, but for the direct kernel.
int upload_gated(cleave_plan* plan) {
  if (gated_few_rows(plan->M, plan->N)) return plan->fused ? ensure_uploaded(plan->fused) : CLEAVE_OK;
  if (plan->fused) {
    const int rc = ensure_uploaded(plan->fused);
    if (rc != CLEAVE_OK || plan->pairs || packs(plan->M, plan->N, plan->K)) return rc;
  }
  return ensure_uploaded(plan);
}

// The operands of a call on the direct kernel, laid out again where they are not whole.
struct Operands {
  const void* a;
  const void* b[2];
  int64_t lda, ldb;
};
hipError_t pack_operands(Operands& o, int weights, int64_t M, int64_t N, int64_t K, int transB, float* workspace, hipStream_t stream) {
  unsigned char* at = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(workspace) + 15) / 16 * 16);
  cleave::PackArgs args{};
  const auto add = [&](const void* from, int64_t ld, int64_t rows, int64_t cols) -> const void* {
    cleave::PackMatrix& m = args.matrices[args.count++];
    m = {from, at, ld, rows, cols};
    at += rows * eights(cols) * 2;
    return m.to;
  };
  if (K % 8 != 0 || !whole_operand(o.a, o.lda)) {
    o.a = add(o.a, o.lda, M, K);
    o.lda = eights(K);
  }
  bool whole = (transB ? K : N) % 8 == 0;
  for (int w = 0; w < weights; ++w) whole = whole && whole_operand(o.b[w], o.ldb);
  if (!whole) {
    const int64_t rows = transB ? N : K, cols = transB ? K : N;
    for (int w = 0; w < weights; ++w) o.b[w] = add(o.b[w], o.ldb, rows, cols);
    o.ldb = eights(cols);
  }
  return cleave::launch_pack(args, stream);
}

// Splits of K for few rows: a workgroup has 64 columns of both weights, so up to 128 of them leave CUs without one; where a
// row of K has 2 KB or more they are split, to one per CU, and joined by a second launch.  (`k` elements of `bytes`: pairs of e4m3.)  One
// row, bf16, K x N, us:
//   weights from memory, 1, 2, 4, 8 splits
//     split           4096 x 4096 26, 21, 18.7, 19.5; 11008 x 4096 58, 47, 38.3, 39.8; 2048 x 5632 21, 16.1, 17.1, 15.6;
//                     8192 x 8192 76, 51.6, 53.7, 54.7
//     not split       4096 x 11008 36.1, 40, 36.9, 38.5; 5120 x 13824 54.4, 61, 62, 58.0; 1024 x 12000 13.9, 17.8, 18.0, 19;
//                     768 x 2048 7.1, 9.3, 9.2, 10
//   weights from the caches, one / as here (4 to 7)
//                     1024 x 64 6.9 / 6.6; 1024 x 4096 8.8 / 9.3 (stored N x K 10.9 / 9.3); 1408 x 1062 10.9 / 9.4; 2016 x 2048 13.4 / 10.3
int64_t gated_few_splits(int64_t N, int64_t k, int64_t bytes) {
  constexpr int64_t kCUs = 256;
  const int64_t groups = (N + 63) / 64;
  if (groups > kCUs / 2 || k * bytes < 2048) return 1;
  for (int64_t S = std::min<int64_t>({kCUs / groups, k * bytes / 512, 16}); S > 1; --S)
    if ((S - 1) * ((k + S - 1) / S) < k) return S;
  return 1;
}

// Splits of K for more rows, `k` in elements of two bytes.  Few items of 128 x 128: what takes least by the time of a K step (up to 64
// items run as a part a CU, up to 128 as two, up to 256 as one item; K x N's half tiles of 32 columns are half lines, which only whole
// products have) and of the join (5 us, and both products' partial blocks written and read at 4.5 TB/s).  Otherwise as many as fill the CUs
// with large tiles.  bf16, weights from memory, columns x K, us, stored K x N / N x K, unsplit; 2; 4 splits:
//   17 rows      2560 x 5120 52 / 25; 34 / 27; 19 / 19, 4096 x 11008 91 / 51; 61 / 53; 48 / 40, 5632 x 2048 34 / 18; 17 / 17; 19 / 19,
//                2816 x 1024 8.5 / 7.0; 10.6 / 10.6; 10.8 / 10.2
//   128 rows     4096 x 4096 39 / 23; 32 / 27; 28 / 27, 2048 x 2048 15.6 / 11.4; 12.3 / 12.6; 14.9 / 14.1
//   256 rows     2048 x 5632 50 / 30; 38 / 34; 27 / 26, 4096 x 2048 27 / 20; 22 / 22; 27 / 25
//   1289 rows    192 x 2880 15.1 / 12.3; not measured; 17.2 / 17.9
//   large tiles  256 rows, 11008 x 4096 83 / 78; 67 / 67; 90 / 87; 512 rows, 4096 x 11008 118 / 109; 120 / 119; 96 / 92, 8192 x 4096 86 / 77;
//                73 / 77; 94 / 94, 5632 x 4096 63 / 62; 67 / 66; 83 / 81; 1159 rows, 1920 x 9920 134 / 131; 152 / 178
//   e4m3         17 rows, 1024 x 4096 14.8; 12.0; 9.3, 2048 x 5632 18.8; 14.1; 13.3, 4096 x 4096 15.7; 16.3; 18.2; 256 rows, 2048 x 2048
//                10.5; 15.8; 20.3
// Not split, and not measured split: 129 to 255 items (of up to 128 rows more than 8192 columns, of up to 256 more than 4096: unsplit they
// take 1.3 to 3.0 times what their bytes do), and 33 and more of e4m3 (whose 0.25 us a K step are less than unsplit calls take, 0.34 with
// the launch).
int64_t gated_splits(int64_t M, int64_t N, int64_t k, bool pairs) {
  constexpr int64_t kCUs = 256;
  const int64_t items = ((M + 127) / 128) * ((2 * N + 127) / 128), large = ((M + 255) / 256) * ((2 * N + 255) / 256);
  const auto whole = [&](int64_t S) { return (k + S - 1) / S % 8 == 0 && (S - 1) * ((k + S - 1) / S) < k; };   // (chunks in sixteen bytes)
  if (items <= (pairs ? kCUs / 8 : kCUs / 2)) {
    int64_t best = 1;
    double least = 0.0;
    for (int64_t S = 1; S <= 4 && items * S <= kCUs; ++S) {
      if (S > 1 && !whole(S)) continue;
      const double step = S == 1                   ? (pairs ? 0.25 : items <= kCUs / 4 ? 0.3 : 0.65)
                          : items * S <= kCUs / 4  ? 0.25
                          : items * S <= kCUs / 2  ? 0.52
                                                   : 0.6;
      double us = step * static_cast<double>(k) / static_cast<double>(64 * S);
      if (S > 1) us += 5.0 + 8.0 * static_cast<double>(S * M * 2 * N) / 4.5e6;
      if (S > 1 && us >= least) continue;
      least = us;
      best = S;
    }
    return best;
  }
  if (pairs || items < kCUs || large > kCUs / 2) return 1;
  const int64_t S = large <= kCUs / 4 ? 4 : 2;
  return k >= 2048 * S && whole(S) && large * S >= (M <= 256 ? 160 : 192) ? S : 1;
}

// Few rows of whole bf16 operands that the direct kernel takes in less time, though its tiles are mostly empty: short K, whose loads it
// has on their way sooner, where every part has a CU; and long rows of K stored N x K, of which it reads whole lines, where 129 to 192 CUs
// have an item each.  us, weights from memory, N x K sizes, few rows / direct:
//   short K, stored K x N and N x K, one row (16)
//     taken      768 x 768 7.0, 8.7 (8.1, 10.2) / 6.3, 6.2 (6.4, 6.2); 4096 x 1024 9.3, 9.4 (10.5, 10.3) / 8.5, 7.1 (8.9, 7.2);
//                4096 x 256 5.0, 5.2 (5.7, 6.0) / 5.2, 5.1 (5.3, 5.1)
//     not taken  5632 x 1024 10.2, 10.9 / 14.5, 9.5; 2816 x 2048 10.9, 11.8 / 12.8, 11.0
//   long rows, stored N x K, one row (16)
//     taken      8448 x 4096 42.9 (48.9) / 35.8 (35.1); 10240 x 4096 48.1 (50.4) / 39.4 (40.0); 12288 x 4096 51.6 (52.2) / 46.2 (46.2);
//                8448 x 8192 88.2 (95.5) / 66.4 (66.8); 11008 x 8192 93.9 (99.4) / 75.5 (76.8); 12288 x 8192 97.3 (102.4) / 76.2 (76.7)
//     not taken  8192 x 8192 65 / 67; 16384 x 4096 57 / 64; (13824 x 4096 50.4 (53.5) / 46.4 (45.9) and, stored K x N, 11008 x 4096 43 (44)
//                / 40 (41), 11008 x 8192 80 (84) / 74 (77) would gain; 8192 x 8192 so 60 / 111)
enum FewDirect { kFewNever, kFewByColumn, kFewAlways };   // ByColumn: stored N x K
FewDirect gated_few_direct(int64_t N, int64_t K) {
  constexpr int64_t kCUs = 256;
  const int64_t items = (2 * N + 127) / 128;
  if (K % 8 != 0) return kFewNever;
  if (items <= kCUs / 4) return K <= 1024 ? kFewAlways : kFewNever;
  return items > kCUs / 2 && items <= kCUs / 4 * 3 && K >= 4096 ? kFewByColumn : kFewNever;
}

bool floats_aligned(const float* const* list, int n) {
  for (int k = 0; k < n; ++k)
    if (!aligned(list[k], 4)) return false;
  return true;
}

// The few-rows launch's operands: K is cut into chunks that end on whole lines of 128 bytes (the last ones may be short, or
// empty, which leaves zeros).
cleave::ExecuteArgs few_rows_args(int64_t M, int64_t N, int64_t K, int eb, int64_t splits, int64_t* chunk) {
  const int64_t line = 128 / eb;
  *chunk = ((K + splits - 1) / splits + line - 1) / line * line;
  cleave::ExecuteArgs args{};
  args.M = M;
  args.N = N;
  args.K = K;
  return args;
}

}  // namespace

extern "C" int cleave_plan_gated(int64_t M, int64_t N, int64_t K, int dtype, cleave_plan** out) {
  if (!linear_dtype(dtype) || !out || M < 1 || N < 1 || K < 1) return CLEAVE_EINVAL;
  constexpr int64_t kMost = std::numeric_limits<int32_t>::max();
  if (M > kMost || N > kMost / 2 || K > kMost) return CLEAVE_EINVAL;
  const bool pairs = dtype == CLEAVE_E4M3;
  if (pairs && K % 16 != 0) return CLEAVE_EINVAL;
  const int64_t k = pairs ? K / 2 : K;
  const bool few = gated_few_rows(M, N);
  // (partial blocks leave the 8-bit kernel in whole eights of columns; what the general kernel takes is split as one product of both
  // operands' columns)
  const int64_t splits = few                                      ? gated_few_splits(N, k, dtype == CLEAVE_F32 ? 4 : 2)
                         : pairs && N % 8 != 0                    ? 1
                         : dtype == CLEAVE_F32 || k % 8 != 0      ? linear_splits(M, 2 * N, k, dtype == CLEAVE_F32 ? 4 : 8, pairs)
                                                                  : gated_splits(M, N, k, pairs);
  const int64_t tile = M <= cleave::kFewRows ? cleave::kSmallTileRows
                       : dtype == CLEAVE_F32 && splits > 1 && fp32_splits(M, 2 * N, K).workgroups > 128 ? 64
                                                                                                       : cleave::kLargeTileRows;
  cleave_plan* plan = nullptr;
  int rc = cleave_plan_batched(M, N, k, tile, tile, static_cast<int32_t>(splits), 2, &plan);
  if (rc != CLEAVE_OK) return rc;
  plan->gated = true;
  plan->for_fp32 = dtype == CLEAVE_F32;
  plan->pairs = pairs;
  plan->uniform_splits = splits;
  const FewDirect few_direct = few && dtype == CLEAVE_BF16 ? gated_few_direct(N, K) : kFewNever;
  if ((few ? few_direct != kFewNever : splits == 1) && dtype != CLEAVE_F32 && (pairs || (eights(N) <= kMostPitch && eights(K) <= kMostPitch))) {
    rc = cleave_plan_uniform(M, 2 * N, k, cleave::kLargeTileRows, cleave::kLargeTileCols, 1, 0, &plan->fused);
    if (rc != CLEAVE_OK) {
      cleave_plan_destroy(plan);
      return rc;
    }
    plan->fused->gated = true;
    plan->fused->pairs = pairs;
  }
  *out = plan;
  return CLEAVE_OK;
}

extern "C" int64_t cleave_gated_workspace(const cleave_plan* plan, int whole) {
  if (!plan || !plan->gated || plan->batch != 2 || (whole != 0 && whole != 1)) return CLEAVE_EINVAL;
  if (gated_few_rows(plan->M, plan->N)) {
    const bool direct = plan->fused && whole && gated_few_direct(plan->N, plan->K) == kFewAlways;
    return direct || plan->uniform_splits == 1 ? 0 : plan->partial_elems;
  }
  if (plan->fused && (plan->pairs || whole)) return 0;
  if (plan->fused && packs(plan->M, plan->N, plan->K)) return packed_floats(plan->M, plan->N, plan->K, 2);
  return plan->partial_elems;
}

extern "C" int cleave_linear_gated(cleave_plan* plan, const cleave_gated_args* a, void* hip_stream) {
  if (!plan || !a || !plan->gated || plan->batch != 2 || !linear_dtype(a->dtype)) return CLEAVE_EINVAL;
  const bool e4m3 = a->dtype == CLEAVE_E4M3;
  if (plan->pairs != e4m3 || plan->for_fp32 != (a->dtype == CLEAVE_F32) || !a->A || !a->B_gate || !a->B_up || !a->C) return CLEAVE_EINVAL;
  if ((a->transB != 0 && a->transB != 1) || (a->out_dtype != CLEAVE_F32 && a->out_dtype != CLEAVE_BF16)) return CLEAVE_EINVAL;
  if (a->act < CLEAVE_ACT_NONE || a->act > CLEAVE_ACT_SILU) return CLEAVE_EINVAL;
  if (e4m3 != (a->scale_a != nullptr) || e4m3 != (a->scale_gate != nullptr) || e4m3 != (a->scale_up != nullptr)) return CLEAVE_EINVAL;
  const int ob = a->out_dtype == CLEAVE_BF16 ? 2 : 4, eb = e4m3 ? 1 : a->dtype == CLEAVE_BF16 ? 2 : 4;
  const int64_t M = plan->M, N = plan->N, K = e4m3 ? 2 * plan->K : plan->K;
  if (a->lda < K || a->ldb < (a->transB ? K : N) || a->ldc < N || (a->gate && a->ld_gate < N) || (a->up && a->ld_up < N))
    return CLEAVE_EINVAL;
  const float* const vectors[] = {a->scale_a, a->scale_gate, a->scale_up, a->bias_gate, a->bias_up, a->partials};
  if (!aligned(a->A, eb) || !aligned(a->B_gate, eb) || !aligned(a->B_up, eb) || !aligned(a->C, ob) || !aligned(a->gate, ob) ||
      !aligned(a->up, ob) || !floats_aligned(vectors, 6))
    return CLEAVE_EINVAL;
  if (!cleave::apart({a->C, a->gate, a->up}, {a->A, a->B_gate, a->B_up, a->bias_gate, a->bias_up, a->scale_a, a->scale_gate, a->scale_up}))
    return CLEAVE_EINVAL;
  if (e4m3 && (!a->transB || !aligned(a->A, 16) || !aligned(a->B_gate, 16) || !aligned(a->B_up, 16) || a->lda % 16 || a->ldb % 16 ||
               a->lda >= int64_t{1} << 22 || a->ldb >= int64_t{1} << 22))
    return CLEAVE_EINVAL;
  cleave::GatedArgs epi{};
  epi.b_up = a->B_up;
  epi.bias_gate = a->bias_gate;
  epi.bias_up = a->bias_up;
  epi.scale_a = a->scale_a;
  epi.scale_gate = a->scale_gate;
  epi.scale_up = a->scale_up;
  epi.gate = a->gate;
  epi.up = a->up;
  epi.ld_gate = a->ld_gate;
  epi.ld_up = a->ld_up;
  epi.act = a->act;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const int64_t splits = plan->uniform_splits;
  const bool few = gated_few_rows(M, N);
  const bool whole = e4m3 || (a->dtype == CLEAVE_BF16 && K % 8 == 0 && (a->transB || N % 8 == 0) && whole_operand(a->A, a->lda) &&
                              whole_operand(a->B_gate, a->ldb) && whole_operand(a->B_up, a->ldb));
  const bool fused = plan->fused && (few ? whole && (a->transB || gated_few_direct(N, K) == kFewAlways) : whole || packs(M, N, K));
  if (!(fused && whole) && (!few || splits > 1) &&
      (!a->partials || !cleave::apart({a->partials}, {a->A, a->B_gate, a->B_up, a->C, a->gate, a->up, a->bias_gate, a->bias_up, a->scale_a,
                                                      a->scale_gate, a->scale_up})))
    return CLEAVE_EINVAL;
  if (fused) {
    AssembleTarget to;
    to.C = a->C;
    to.ldc = a->ldc;
    to.out_dtype = a->out_dtype;
    int rc = ensure_uploaded(plan->fused);
    if (rc != CLEAVE_OK) return rc;
    Operands o{a->A, {a->B_gate, a->B_up}, e4m3 ? a->lda / 2 : a->lda, e4m3 ? a->ldb / 2 : a->ldb};
    if (!whole) CLEAVE_HIP(pack_operands(o, 2, M, N, K, a->transB, a->partials, stream));
    epi.b_up = o.b[1];
    rc = execute_impl(plan->fused, nullptr, 0, o.a, o.lda, 0, o.b[0], o.ldb, a->transB, CLEAVE_BF16, nullptr, BatchLayout{}, hip_stream,
                      to, false, nullptr, &epi);
    plan->last_kernel = plan->fused->last_kernel;
    return rc;
  }
  cleave::ReduceArgs join{};
  join.partials = a->partials;
  join.C = a->C;
  join.ldc = a->ldc;
  const bool vec = N % 4 == 0 && aligned(a->partials, 16);
  if (few) {
    int64_t chunk = 0;
    cleave::ExecuteArgs args = few_rows_args(M, N, K, eb, splits, &chunk);
    args.A = a->A;
    args.B = a->B_gate;
    args.lda = a->lda;
    args.ldb = a->ldb;
    args.transB = a->transB;
    args.partials = a->partials;
    args.C = a->C;
    args.ldc = a->ldc;
    args.c_bf16 = a->out_dtype == CLEAVE_BF16;
    CLEAVE_HIP(cleave::launch_gated_few_rows(args, epi, a->dtype, static_cast<int>(splits), chunk, stream));
    plan->last_kernel = "gated_few_rows";
    if (splits == 1) return CLEAVE_OK;
    CLEAVE_HIP(cleave::launch_gated_join(join, epi, N, M, N, static_cast<int>(splits), a->out_dtype, vec, stream));
    return CLEAVE_OK;
  }
  // both products' partial blocks, then one pass over them
  const void* const Bs[2] = {a->B_gate, a->B_up};
  BatchLayout bl;
  bl.shape.n_group = 2;
  const void* B = nullptr;
  int rc = group_offsets(Bs, 2, e4m3 ? 2 : eb, &bl.b, &B);
  if (rc == CLEAVE_OK) rc = ensure_uploaded(plan);
  const cleave::LinearArgs none{};   // (what the blocks of 8-bit operands go through)
  if (rc == CLEAVE_OK)
    rc = execute_impl(plan, nullptr, 0, a->A, e4m3 ? a->lda / 2 : a->lda, 0, B, e4m3 ? a->ldb / 2 : a->ldb, a->transB,
                      e4m3 ? CLEAVE_BF16 : a->dtype, a->partials, bl, hip_stream, AssembleTarget{}, false, e4m3 ? &none : nullptr);
  if (rc != CLEAVE_OK) return rc;
  // (a long table of runs begins with the last member's)
  const bool up_first = plan->tasks[plan->reduce_tiles[0].task].gemm_id != 0;
  join.n_items = plan->reduce_runs / 2;
  join.items = plan->d_reduce_items + (up_first ? join.n_items : 0);
  CLEAVE_HIP(cleave::launch_gated_join(join, epi, plan->partial_elems / 2, M, N, static_cast<int>(splits), a->out_dtype,
                                       plan->all_n_mult4 && vec, stream));
  return CLEAVE_OK;
}

extern "C" int64_t cleave_gated_grad_workspace(const cleave_plan* plan, int whole) {
  if (!plan || !plan->linear || plan->pairs || (whole != 0 && whole != 1)) return CLEAVE_EINVAL;
  if (!gated_few_rows(plan->M, plan->N) && plan->uniform_splits == 1 && !plan->for_fp32) {
    if (whole) return 0;
    if (packs_grad(plan->M, plan->N, plan->K)) return packed_floats(plan->M, plan->N, plan->K, 1);
  }
  return plan->partial_elems;
}

extern "C" int cleave_linear_gated_grad(cleave_plan* plan, const cleave_gated_grad_args* a, void* hip_stream) {
  if (!plan || !a || !plan->linear || plan->pairs || a->dtype != (plan->for_fp32 ? CLEAVE_F32 : CLEAVE_BF16)) return CLEAVE_EINVAL;
  if (!a->A || !a->B || !a->gate || !a->up || !a->dgate || !a->dup) return CLEAVE_EINVAL;
  if ((a->transB != 0 && a->transB != 1) || (a->out_dtype != CLEAVE_F32 && a->out_dtype != CLEAVE_BF16)) return CLEAVE_EINVAL;
  if (a->act < CLEAVE_ACT_NONE || a->act > CLEAVE_ACT_SILU) return CLEAVE_EINVAL;
  const int ob = a->out_dtype == CLEAVE_BF16 ? 2 : 4, eb = a->dtype == CLEAVE_BF16 ? 2 : 4;
  const int64_t M = plan->M, N = plan->N, K = plan->K;
  if (a->lda < K || a->ldb < (a->transB ? K : N) || a->ld_gate < N || a->ld_up < N || a->ld_dgate < N || a->ld_dup < N)
    return CLEAVE_EINVAL;
  if (!aligned(a->A, eb) || !aligned(a->B, eb) || !aligned(a->gate, ob) || !aligned(a->up, ob) || !aligned(a->dgate, ob) ||
      !aligned(a->dup, ob) || !aligned(a->partials, 4))
    return CLEAVE_EINVAL;
  // in place: each over its own argument, the same elements at the same places
  if (a->dgate == a->dup || a->dgate == a->up || a->dup == a->gate || a->dgate == a->A || a->dgate == a->B || a->dup == a->A ||
      a->dup == a->B ||
      (a->dgate == a->gate && M > 1 && a->ld_dgate != a->ld_gate) || (a->dup == a->up && M > 1 && a->ld_dup != a->ld_up))
    return CLEAVE_EINVAL;
  cleave::GatedArgs epi{};
  epi.gate = const_cast<void*>(a->gate);
  epi.up = const_cast<void*>(a->up);
  epi.second = a->dup;
  epi.ld_gate = a->ld_gate;
  epi.ld_up = a->ld_up;
  epi.ld_second = a->ld_dup;
  epi.act = a->act;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const int64_t splits = plan->uniform_splits;
  const bool few = gated_few_rows(M, N);
  const bool whole = a->dtype == CLEAVE_BF16 && K % 8 == 0 && (a->transB || N % 8 == 0) && whole_operand(a->A, a->lda) &&
                     whole_operand(a->B, a->ldb);
  const bool fused = !few && splits == 1 && !plan->for_fp32 && (whole || packs_grad(M, N, K));
  if (!(fused && whole) && (!a->partials || !cleave::apart({a->partials}, {a->A, a->B, a->gate, a->up, a->dgate, a->dup})))
    return CLEAVE_EINVAL;
  int rc = ensure_uploaded(plan);
  if (rc == CLEAVE_OK) rc = ensure_gated_ready(plan->device);
  if (rc != CLEAVE_OK) return rc;
  if (fused) {
    AssembleTarget to;
    to.C = a->dgate;
    to.ldc = a->ld_dgate;
    to.out_dtype = a->out_dtype;
    Operands o{a->A, {a->B, nullptr}, a->lda, a->ldb};
    if (!whole) CLEAVE_HIP(pack_operands(o, 1, M, N, K, a->transB, a->partials, stream));
    return execute_impl(plan, nullptr, 0, o.a, o.lda, 0, o.b[0], o.ldb, a->transB, a->dtype, nullptr, BatchLayout{}, hip_stream, to,
                        false, nullptr, &epi);
  }
  if (few) {   // (the sums themselves, also where there is one chunk)
    int64_t chunk = 0;
    cleave::ExecuteArgs args = few_rows_args(M, N, K, eb, splits, &chunk);
    args.A = a->A;
    args.B = a->B;
    args.lda = a->lda;
    args.ldb = a->ldb;
    args.transB = a->transB;
    args.partials = a->partials;
    args.C = a->partials;
    args.ldc = N;
    CLEAVE_HIP(cleave::launch_linear_few_rows(args, cleave::LinearArgs{}, a->dtype, static_cast<int>(splits), chunk, stream));
    plan->last_kernel = "linear_few_rows";
  } else {
    rc = execute_impl(plan, nullptr, 0, a->A, a->lda, 0, a->B, a->ldb, a->transB, a->dtype, a->partials, BatchLayout{}, hip_stream);
    if (rc != CLEAVE_OK) return rc;
  }
  cleave::ReduceArgs join{};
  join.items = few ? nullptr : plan->d_reduce_items;
  join.n_items = plan->reduce_runs;
  join.partials = a->partials;
  join.C = a->dgate;
  join.ldc = a->ld_dgate;
  CLEAVE_HIP(cleave::launch_gated_grad_join(join, epi, M, N, static_cast<int>(splits), a->out_dtype,
                                            plan->all_n_mult4 && N % 4 == 0 && aligned(a->partials, 16), stream));
  return CLEAVE_OK;
}

#ifndef CLEAVE_AGG_ELEMS
#define CLEAVE_AGG_ELEMS 8192
#endif

namespace {

// Host tables of the returned-block check (built once per plan) and their
// device copies plus scratch (once per device the plan is used on).
int ensure_verify_tables_host(cleave_plan* p) {
  using cleave::Segment;
  if (!p->verify) {
    cleave::VerifyTables* v = new (std::nothrow) cleave::VerifyTables;
    if (!v) return CLEAVE_ENOMEM;
    try {
      std::map<std::pair<uint32_t, uint32_t>, uint32_t> rows, cols;
      // Elements of a partial block per bilinear item: runs long enough to stream, as
      // short as the last round of workgroups needs.  us, runs of 8 K / 16 K / 32 K: 17 M
      // elements in all 23.4 / 20.1 / 21.8, 67 M 71.8 / 64.4 / 67.4, behind the launch that
      // wrote them 189.4 / 187.9 / 191.4, 134 M 113 / 101 / 104, 180 M 174 / 139 / 144, 268 M
      // 208 / 185 / 188; 451 M in 8 splits of 4 MiB blocks 421 / 336 / 330.
      const uint32_t kElemsPerItem = p->partial_elems >= (int64_t{384} << 20) ? 32768u : 16384u;
      v->task_first_item.push_back(0);
      for (const cleave_task& t : p->tasks) {
        auto ri = rows.emplace(std::make_pair(t.m0, t.m_len), static_cast<uint32_t>(rows.size()));
        if (ri.second) v->row_segs.push_back(Segment{t.m0, t.m_len});
        v->task_row_seg.push_back(ri.first->second);
        auto ci = cols.emplace(std::make_pair(t.n0, t.n_len), static_cast<uint32_t>(cols.size()));
        if (ci.second) v->col_segs.push_back(Segment{t.n0, t.n_len});
        v->task_col_seg.push_back(ci.first->second);
        const uint32_t rows_per = std::max<uint32_t>(1, kElemsPerItem / t.n_len);
        for (uint32_t r0 = 0; r0 < t.m_len; r0 += rows_per)
          v->items.push_back(cleave::make_verify_item(t, r0, std::min(rows_per, t.m_len - r0)));
        v->max_ksplit = std::max(v->max_ksplit, t.ksplit_cnt);
        if (v->items.size() > std::numeric_limits<uint32_t>::max()) {
          delete v;
          return CLEAVE_EINVAL;
        }
        v->task_first_item.push_back(static_cast<uint32_t>(v->items.size()));
      }
      for (const std::vector<Segment>* segs : {&v->row_segs, &v->col_segs})
        for (const Segment& sg : *segs) {
          v->segs_mult8 &= ((sg.start | sg.len) % 8 == 0);
          v->segs_mult4 &= ((sg.start | sg.len) % 4 == 0);
        }
    } catch (const std::bad_alloc&) {
      delete v;
      return CLEAVE_ENOMEM;
    }
    p->verify = v;
  }
  return CLEAVE_OK;
}

int ensure_verify_tables(cleave_plan* p) {
  int rc = ensure_verify_tables_host(p);
  if (rc != CLEAVE_OK) return rc;
  cleave::VerifyTables* v = p->verify;
  if (v->d_items || p->tasks.empty()) return CLEAVE_OK;
  rc = upload_vector(v->row_segs, &v->d_row_segs);
  if (rc == CLEAVE_OK) rc = upload_vector(v->col_segs, &v->d_col_segs);
  if (rc == CLEAVE_OK) rc = upload_vector(v->task_row_seg, &v->d_task_row_seg);
  if (rc == CLEAVE_OK) rc = upload_vector(v->task_col_seg, &v->d_task_col_seg);
  if (rc == CLEAVE_OK) rc = upload_vector(v->task_first_item, &v->d_task_first_item);
  if (rc == CLEAVE_OK) rc = upload_vector(v->items, &v->d_items);
  if (rc == CLEAVE_OK) {
    const size_t members = p->batch > 0 ? static_cast<size_t>(p->batch) : 1;
    const size_t proj = 2 * (v->row_segs.size() + v->col_segs.size()) * static_cast<size_t>(p->K) * members;
    hipError_t e = hipMalloc(reinterpret_cast<void**>(&v->d_proj), proj * sizeof(double));
    if (e == hipSuccess)
      e = hipMalloc(reinterpret_cast<void**>(&v->d_item_sums), v->items.size() * sizeof(double));
    if (e == hipErrorOutOfMemory) rc = CLEAVE_ENOMEM;
    else if (e != hipSuccess) rc = hip_fail(e);
  }
  if (rc != CLEAVE_OK) free_verify_device(v);
  return rc;
}

// Tables of the fused check + aggregation (first fused call on the plan, after
// ensure_verify_tables): runs of rows of ~kAggElemsPerItem output elements.
int ensure_aggregate_tables(cleave_plan* p) {
  cleave::VerifyTables* v = p->verify;
  if (v->d_agg_items || p->tasks.empty()) return CLEAVE_OK;
  if (v->agg_first_item.empty()) {
    try {
      constexpr uint32_t kAggElemsPerItem = CLEAVE_AGG_ELEMS;
      uint64_t slots = 0;
      v->agg_first_item.push_back(0);
      for (const cleave_task& t : p->tasks) {
        const uint32_t rows_per = std::max<uint32_t>(1, kAggElemsPerItem / t.n_len);
        const uint32_t runs = (t.m_len + rows_per - 1) / rows_per;
        for (uint32_t j = 0; t.ksplit_idx == 0 && j < runs; ++j) {
          const uint32_t r0 = j * rows_per;
          cleave::VerifyItem item = cleave::make_verify_item(t, r0, std::min(rows_per, t.m_len - r0));
          item.slot = static_cast<uint32_t>(slots) + j;
          item.slot_step = runs;
          v->agg_items.push_back(item);
        }
        slots += runs;
        if (slots > std::numeric_limits<uint32_t>::max()) {
          v->agg_items.clear();
          v->agg_first_item.clear();
          return CLEAVE_EINVAL;
        }
        v->agg_first_item.push_back(static_cast<uint32_t>(slots));
      }
    } catch (const std::bad_alloc&) {
      v->agg_items.clear();
      v->agg_first_item.clear();
      return CLEAVE_ENOMEM;
    }
  }
  int rc = upload_vector(v->agg_items, &v->d_agg_items);
  if (rc == CLEAVE_OK) rc = upload_vector(v->agg_first_item, &v->d_agg_first_item);
  if (rc == CLEAVE_OK) {
    const hipError_t e = hipMalloc(reinterpret_cast<void**>(&v->d_agg_item_sums),
                                   static_cast<size_t>(v->agg_first_item.back()) * sizeof(double));
    if (e == hipErrorOutOfMemory) rc = CLEAVE_ENOMEM;
    else if (e != hipSuccess) rc = hip_fail(e);
  }
  if (rc != CLEAVE_OK) {
    for (void* q : {static_cast<void*>(v->d_agg_items), static_cast<void*>(v->d_agg_first_item),
                    static_cast<void*>(v->d_agg_item_sums)})
      if (q) (void)hipFree(q);
    v->d_agg_items = nullptr;
    v->d_agg_first_item = nullptr;
    v->d_agg_item_sums = nullptr;
  }
  return rc;
}

}  // namespace

namespace {

// Where the fused pass writes the aggregated output (C == nullptr: check only).
struct AggregateTarget {
  void* C = nullptr;
  int64_t ldc = 0;
  int out_dtype = CLEAVE_F32;
};

int verify_impl(cleave_plan* plan, const void* A, int64_t lda, int transA, const void* B, int64_t ldb,
                int transB, int dtype, const float* partials, const float* r, const float* s, double tol,
                double* lhs, double* rhs, double* scale, int32_t* accept, const BatchLayout& bl,
                void* hip_stream, const AggregateTarget& agg = AggregateTarget{}) {
  if (!plan || !A || !B || !partials || !r || !s || !accept) return CLEAVE_EINVAL;
  if (plan->pairs) return CLEAVE_EINVAL;   // a plan of 8-bit operands
  if (dtype != CLEAVE_F32 && dtype != CLEAVE_BF16) return CLEAVE_EINVAL;
  if ((transA != 0 && transA != 1) || (transB != 0 && transB != 1)) return CLEAVE_EINVAL;
  if (lda < (transA ? plan->M : plan->K) || ldb < (transB ? plan->K : plan->N)) return CLEAVE_EINVAL;
  if (!(tol >= 0.0)) return CLEAVE_EINVAL;   // also refuses NaN
  const int eb = dtype == CLEAVE_BF16 ? 2 : 4;
  if (!aligned(A, eb) || !aligned(B, eb) || !aligned(partials, 4) || !aligned(r, 4) ||
      !aligned(s, 4) || !aligned(accept, 4) || !aligned(lhs, 8) || !aligned(rhs, 8) ||
      !aligned(scale, 8))
    return CLEAVE_EINVAL;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);

  int rc = ensure_uploaded(plan);
  if (rc != CLEAVE_OK) return rc;
  rc = ensure_verify_tables(plan);
  if (rc != CLEAVE_OK) return rc;
  cleave::VerifyTables* v = plan->verify;
  if (plan->tasks.empty()) return CLEAVE_OK;

  const int64_t K = plan->K;
  const bool batched = plan->batch > 0;
  const int n_members = batched ? static_cast<int>(plan->batch) : 1;
  const int e = 16 / eb;   // elements per 16-byte load
  const bool segs_ok = e == 8 ? v->segs_mult8 : v->segs_mult4;
  const size_t row_proj = v->row_segs.size() * static_cast<size_t>(K) * static_cast<size_t>(n_members);
  const size_t col_proj = v->col_segs.size() * static_cast<size_t>(K) * static_cast<size_t>(n_members);
  double* U = v->d_proj;
  double* U_abs = U + row_proj;
  double* V = U_abs + row_proj;
  double* V_abs = V + col_proj;

  // op(A)[i][k]: stored M x K (transA = 0) -> the summed row index strides;
  // stored K x M (transA = 1) -> it is contiguous.  op(B)[k][j]: stored K x N
  // (transB = 0) -> the summed column index is contiguous; stored N x K -> it
  // strides.
  const bool a_contig = transA != 0;
  const bool b_contig = transB == 0;
  // members' probe vectors follow each other: r is n_members x M, s is n_members x N
  const int64_t r_stride = batched ? plan->M : 0, s_stride = batched ? plan->N : 0;
  const bool a_vec = aligned(A, 16) && lda % e == 0 && offsets_multiple_of(bl.a, bl.shape, e) &&
                     (a_contig ? (segs_ok && aligned(r, 16) && r_stride % 4 == 0) : K % e == 0);
  const bool b_vec = aligned(B, 16) && ldb % e == 0 && offsets_multiple_of(bl.b, bl.shape, e) &&
                     (b_contig ? (segs_ok && aligned(s, 16) && s_stride % 4 == 0) : K % e == 0);
  const bool p_vec = plan->all_n_mult4 && aligned(partials, 16) && aligned(s, 16) && s_stride % 4 == 0;
  cleave::VerifyPassArgs pass{};
  pass.A = cleave::ProjectArgs{A, lda, v->d_row_segs, static_cast<int>(v->row_segs.size()), r, U, U_abs, K,
                               n_members, r_stride, bl.shape, bl.a};
  pass.B = cleave::ProjectArgs{B, ldb, v->d_col_segs, static_cast<int>(v->col_segs.size()), s, V, V_abs, K,
                               n_members, s_stride, bl.shape, bl.b};
  pass.bil = cleave::BilinearArgs{v->d_items, static_cast<int64_t>(v->items.size()),
                                  partials, r, s, v->d_item_sums, batched ? 1 : 0, r_stride, s_stride};
  const uint32_t* first_item = v->d_task_first_item;
  const double* item_sums = v->d_item_sums;
  if (agg.C) {
    rc = ensure_aggregate_tables(plan);
    if (rc != CLEAVE_OK) return rc;
    first_item = v->d_agg_first_item;
    item_sums = v->d_agg_item_sums;
    const int ob = agg.out_dtype == CLEAVE_BF16 ? 2 : 4;
    const bool c_vec = agg.ldc % 4 == 0 && aligned(agg.C, 4 * ob);
    cleave::VerifyReducePassArgs fused{};
    fused.A = pass.A;
    fused.B = pass.B;
    fused.bil = pass.bil;
    fused.bil.item_sums = v->d_agg_item_sums;
    fused.agg = cleave::AggregateArgs{v->d_agg_items, static_cast<int64_t>(v->agg_items.size()), agg.C, agg.ldc, agg.out_dtype == CLEAVE_BF16 ? 1 : 0,
                                      agg.out_dtype == CLEAVE_F32 && cleave::streamed_sum(plan->M * plan->N, plan->partial_elems)};
    CLEAVE_HIP(cleave::launch_verify_reduce_pass(fused, dtype, a_contig, b_contig,
                                                 a_vec && b_vec && p_vec && c_vec, stream));
  } else {
    CLEAVE_HIP(cleave::launch_verify_pass(pass, dtype, a_contig, b_contig, a_vec && b_vec && p_vec, stream));
  }

  cleave::VerdictArgs va{plan->d_tasks, static_cast<int64_t>(plan->tasks.size()),
                         v->d_task_row_seg, v->d_task_col_seg, first_item,
                         item_sums, U, U_abs, V, V_abs, K, batched ? 1 : 0,
                         static_cast<int>(v->row_segs.size()), static_cast<int>(v->col_segs.size()),
                         tol, lhs, rhs, scale, accept};
  CLEAVE_HIP(cleave::launch_verdict(va, stream));
  return CLEAVE_OK;
}

}  // namespace

extern "C" int cleave_verify(cleave_plan* plan, const void* A, int64_t lda, int transA,
                             const void* B, int64_t ldb, int transB, int dtype,
                             const float* partials, const float* r, const float* s, double tol,
                             double* lhs, double* rhs, double* scale, int32_t* accept,
                             void* hip_stream) {
  if (plan && plan->batch > 0) return CLEAVE_EINVAL;   // batched plans use the batched / grouped calls
  return verify_impl(plan, A, lda, transA, B, ldb, transB, dtype, partials, r, s, tol, lhs, rhs, scale,
                     accept, BatchLayout{}, hip_stream);
}

extern "C" int cleave_verify_reduce(cleave_plan* plan, const void* A, int64_t lda, int transA,
                                    const void* B, int64_t ldb, int transB, int dtype,
                                    const float* partials, const float* r, const float* s, double tol,
                                    double* lhs, double* rhs, double* scale, int32_t* accept,
                                    void* C, int64_t ldc, int out_dtype, void* hip_stream) {
  if (!plan || plan->batch > 0 || !C) return CLEAVE_EINVAL;
  if (out_dtype != CLEAVE_F32 && out_dtype != CLEAVE_BF16) return CLEAVE_EINVAL;
  if (ldc < plan->N || !aligned(C, out_dtype == CLEAVE_BF16 ? 2 : 4)) return CLEAVE_EINVAL;
  int rc = ensure_verify_tables_host(plan);
  if (rc != CLEAVE_OK) return rc;
  if (plan->verify->max_ksplit > static_cast<uint32_t>(cleave::kMaxFusedSplits)) {
    // more splits per tile than the fused pass carries: the two passes one after the other
    rc = verify_impl(plan, A, lda, transA, B, ldb, transB, dtype, partials, r, s, tol, lhs, rhs, scale,
                     accept, BatchLayout{}, hip_stream);
    if (rc != CLEAVE_OK) return rc;
    return reduce_impl(plan, partials, C, ldc, out_dtype, BatchLayout{}, hip_stream);
  }
  AggregateTarget agg;
  agg.C = C;
  agg.ldc = ldc;
  agg.out_dtype = out_dtype;
  return verify_impl(plan, A, lda, transA, B, ldb, transB, dtype, partials, r, s, tol, lhs, rhs, scale,
                     accept, BatchLayout{}, hip_stream, agg);
}

extern "C" int cleave_verify_batched(cleave_plan* plan, const void* A, int64_t lda, int transA,
                                     int64_t a_outer, int64_t a_inner, const void* B, int64_t ldb,
                                     int transB, int64_t b_outer, int64_t b_inner, int64_t n_inner,
                                     int dtype, const float* partials, const float* r, const float* s,
                                     double tol, double* lhs, double* rhs, double* scale,
                                     int32_t* accept, void* hip_stream) {
  if (!plan || plan->batch < 1) return CLEAVE_EINVAL;
  if (n_inner < 1 || n_inner > std::numeric_limits<uint32_t>::max() || plan->batch % n_inner != 0)
    return CLEAVE_EINVAL;
  if (a_outer < 0 || a_inner < 0 || b_outer < 0 || b_inner < 0) return CLEAVE_EINVAL;
  return verify_impl(plan, A, lda, transA, B, ldb, transB, dtype, partials, r, s, tol, lhs, rhs, scale,
                     accept, strided_layout(n_inner, a_outer, a_inner, b_outer, b_inner, 0, 0), hip_stream);
}

extern "C" int cleave_verify_grouped(cleave_plan* plan, int64_t n_members, const void* const* A_list,
                                     int64_t lda, int transA, const void* const* B_list, int64_t ldb,
                                     int transB, int dtype, const float* partials, const float* r,
                                     const float* s, double tol, double* lhs, double* rhs,
                                     double* scale, int32_t* accept, void* hip_stream) {
  if (!plan || plan->batch < 1 || plan->batch > cleave::kMaxGroup || n_members != plan->batch)
    return CLEAVE_EINVAL;
  if (dtype != CLEAVE_F32 && dtype != CLEAVE_BF16) return CLEAVE_EINVAL;
  const int eb = dtype == CLEAVE_BF16 ? 2 : 4;
  BatchLayout bl;
  bl.shape.n_group = static_cast<uint32_t>(plan->batch);
  const void* A = nullptr;
  const void* B = nullptr;
  int rc = group_offsets(A_list, plan->batch, eb, &bl.a, &A);
  if (rc != CLEAVE_OK) return rc;
  rc = group_offsets(B_list, plan->batch, eb, &bl.b, &B);
  if (rc != CLEAVE_OK) return rc;
  return verify_impl(plan, A, lda, transA, B, ldb, transB, dtype, partials, r, s, tol, lhs, rhs, scale,
                     accept, bl, hip_stream);
}
