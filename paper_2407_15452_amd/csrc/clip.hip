// gs_clip_grads: the norm of many tensors taken together, and all of them scaled down to a limit.
//
//   norm = sqrt(sum over tensors and elements of x^2);  x <- x * (max_norm / norm) where norm > max_norm
//
// Both passes run over the same units of work (32 KB of one tensor each), dealt in ranges to a fixed number of workgroups, and
// are bound by memory: squares of 512 MB of bf16 in 89 us (5.8 TB/s), 301 fp32 tensors of 80 MB in all 16 and 29 us.  The squares are summed in fp64 (fp32 would overflow from 1.8e19 on and lose small tensors next to large
// ones); every workgroup leaves one partial sum and the second pass adds them in order, so the same tensors give the same
// bits on every run.  The second pass runs backwards: what the first one read last is still in the caches.
// Addresses and sizes travel in the kernel arguments (nothing is copied to the device): of up to kPerLaunch tensors in those of
// the two passes, of more in those of small kernels that write them to a table in the workspace first (301 tensors of 80 MB in
// all: three launches for each pass took 82 us).

#include <cmath>

#include "common.h"

namespace gs {
namespace {

constexpr int kThreads = 256;
constexpr int kPieces = 8;                     // 16-byte pieces per lane and unit: that many loads in flight
constexpr int kUnit = kThreads * kPieces;      // pieces per unit: 32 KB
constexpr int kMaxGroups = 1024;               // four workgroups per compute unit
constexpr int kPerLaunch = 112;                // the arguments stay below 4 KB

struct Item {
  void* data;
  void* out;
  int64_t count;
  uint32_t first_unit;
  int32_t dtype;
};
struct Items {
  Item item[kPerLaunch];
  int32_t items;
};
struct Pass {
  const Item* table;                           // or null: in the arguments
  int32_t items;
  uint32_t units;
  double* parts;                               // one per workgroup of the first pass
  int32_t num_parts;
  double max_norm;
  double* norm_out;
};
static_assert(sizeof(Items) + sizeof(Pass) <= 4096, "kernel arguments");

// The item that holds `unit`, by a whole wave: 64 places at a time.
template <bool TABLE>
__device__ __forceinline__ int find_item(const Items& list, const Pass& a, uint32_t unit) {
  int lo = 0, n = a.items;                     // the last of items lo .. lo + n - 1 that begins at or before `unit`; lo does
  const int lane = threadIdx.x & 63;
  while (n > 1) {
    const int part = (n + 63) / 64, at = lane * part;
    const bool before = at < n && (TABLE ? a.table[lo + at].first_unit : list.item[lo + at].first_unit) <= unit;
    const int last = 63 - __clzll((long long)__ballot(before));
    lo += last * part;
    n = min(part, n - last * part);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// elements in front of the first 16-byte boundary
template <typename T>
__device__ __forceinline__ int64_t head_of(const T* p, int64_t count) {
  const int64_t h = (int64_t)((16 - ((uintptr_t)p & 15)) & 15) / (int64_t)sizeof(T);
  return h < count ? h : count;
}

struct F32Value {
  typedef float elem;
  static __device__ __forceinline__ float get(float x) { return x; }
  static __device__ __forceinline__ float put(float x) { return x; }
};
template <typename H>
struct HalfValue {
  typedef uint16_t elem;
  static __device__ __forceinline__ float get(uint16_t x) { return H::lo(x); }
  static __device__ __forceinline__ uint16_t put(float x) { return (uint16_t)H::round(x); }
};

template <typename V>
__device__ __forceinline__ double piece_squares(uint4 w) {
  constexpr int per = 16 / (int)sizeof(typename V::elem);
  typename V::elem e[per];
  __builtin_memcpy(e, &w, 16);
  double s = 0.0;
#pragma unroll
  for (int k = 0; k < per; ++k) {
    const double x = (double)V::get(e[k]);
    s = fma(x, x, s);
  }
  return s;
}
// In fp64: a factor far below 1 would lose its bits in fp32, where norms of 1e40 exist.  (16-bit formats: through fp32, which
// moves a result only within 2^-24 of the middle between two of the format's numbers.)
template <typename V>
__device__ __forceinline__ typename V::elem scaled(typename V::elem x, double factor) {
  return V::put((float)((double)V::get(x) * factor));
}
template <typename V>
__device__ __forceinline__ uint4 piece_scaled(uint4 w, double factor) {
  constexpr int per = 16 / (int)sizeof(typename V::elem);
  typename V::elem e[per];
  __builtin_memcpy(e, &w, 16);
#pragma unroll
  for (int k = 0; k < per; ++k) e[k] = scaled<V>(e[k], factor);
  __builtin_memcpy(&w, e, 16);
  return w;
}

template <typename V>
__device__ double unit_squares(const Item& it, uint32_t unit) {
  typedef typename V::elem elem;
  constexpr int per = 16 / (int)sizeof(elem);
  const elem* x = static_cast<const elem*>(it.data);
  const int64_t head = head_of(x, it.count);
  const int64_t pieces = (it.count - head) / per;
  const uint4* body = reinterpret_cast<const uint4*>(x + head);
  const int64_t first = (int64_t)unit * kUnit + threadIdx.x;
  uint4 w[kPieces];
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    const int64_t p = first + (int64_t)k * kThreads;
    w[k] = p < pieces ? body[p] : make_uint4(0, 0, 0, 0);
  }
  double s = 0.0;
#pragma unroll
  for (int k = 0; k < kPieces; ++k) s += piece_squares<V>(w[k]);
  if (unit == 0) {                             // what lies in front of the first whole piece and after the last
    const int64_t tail = head + pieces * per;
    const int64_t rest = head + (it.count - tail);
    if ((int64_t)threadIdx.x < rest) {
      const int64_t at = (int64_t)threadIdx.x < head ? (int64_t)threadIdx.x : tail + ((int64_t)threadIdx.x - head);
      const double v = (double)V::get(x[at]);
      s = fma(v, v, s);
    }
  }
  return s;
}

template <typename V>
__device__ void unit_scaled(const Item& it, uint32_t unit, double factor, bool copy) {
  typedef typename V::elem elem;
  constexpr int per = 16 / (int)sizeof(elem);
  const elem* x = static_cast<const elem*>(it.data);
  elem* y = static_cast<elem*>(it.out);
  const int64_t head = head_of(x, it.count);
  const int64_t pieces = (it.count - head) / per;
  const int64_t tail = head + pieces * per;
  if ((((uintptr_t)x ^ (uintptr_t)y) & 15) == 0) {
    const uint4* from = reinterpret_cast<const uint4*>(x + head);
    uint4* to = reinterpret_cast<uint4*>(y + head);
    const int64_t first = (int64_t)unit * kUnit + threadIdx.x;
    uint4 w[kPieces];
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      const int64_t p = first + (int64_t)k * kThreads;
      w[k] = p < pieces ? from[p] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      const int64_t p = first + (int64_t)k * kThreads;
      if (p < pieces) to[p] = copy ? w[k] : piece_scaled<V>(w[k], factor);
    }
  } else {                                     // the two lie differently: element by element
    const int64_t from = head + (int64_t)unit * kUnit * per;
    const int64_t end = min(from + (int64_t)kUnit * per, tail);
    for (int64_t i = from + threadIdx.x; i < end; i += kThreads) y[i] = copy ? x[i] : scaled<V>(x[i], factor);
  }
  if (unit == 0) {
    const int64_t rest = head + (it.count - tail);
    if ((int64_t)threadIdx.x < rest) {
      const int64_t at = (int64_t)threadIdx.x < head ? (int64_t)threadIdx.x : tail + ((int64_t)threadIdx.x - head);
      y[at] = copy ? x[at] : scaled<V>(x[at], factor);
    }
  }
}

// sum over the workgroup, the same in every lane
__device__ double group_sum(double s) {
  __shared__ double wave_sum[kThreads / 64];
#pragma unroll
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d, 64);
  if ((threadIdx.x & 63) == 0) wave_sum[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) s += wave_sum[w];
  __syncthreads();
  return s;
}

// this workgroup's units: body(item, unit of the item)
template <bool TABLE, typename Body>
__device__ __forceinline__ void for_units(const Items& list, const Pass& a, uint32_t group, Body body) {
  const uint32_t per = a.units / gridDim.x, more = a.units % gridDim.x;
  const uint32_t first = group * per + min(group, more), last = first + per + (group < more ? 1 : 0);
  if (first >= last) return;
  int at = find_item<TABLE>(list, a, first);
  uint32_t end = 0;
  Item it;
  for (uint32_t u = first; u < last; ++u) {
    if (u == first || u >= end) {
      if (u != first) ++at;
      it = TABLE ? a.table[at] : list.item[at];
      end = at + 1 < a.items ? (TABLE ? a.table[at + 1].first_unit : list.item[at + 1].first_unit) : a.units;
    }
    body(it, u - it.first_unit);
  }
}

template <bool TABLE>
__global__ __launch_bounds__(kThreads) void squares_kernel(Items list, Pass a) {
  double s = 0.0;
  for_units<TABLE>(list, a, blockIdx.x, [&](const Item& it, uint32_t unit) {
    if (it.dtype == GS_F32) s += unit_squares<F32Value>(it, unit);
    else if (it.dtype == GS_BF16) s += unit_squares<HalfValue<bf16_t>>(it, unit);
    else s += unit_squares<HalfValue<f16_t>>(it, unit);
  });
  s = group_sum(s);
  if (threadIdx.x == 0) a.parts[blockIdx.x] = s;
}

template <bool TABLE>
__global__ __launch_bounds__(kThreads) void clip_kernel(Items list, Pass a) {
  double s = 0.0;
  for (int32_t k = threadIdx.x; k < a.num_parts; k += kThreads) s += a.parts[k];
  const double norm = sqrt(group_sum(s));
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm_out = norm;
  // a norm that is no number, or infinite, says that some gradient is: nothing is scaled by it
  const bool reached = norm > a.max_norm && norm < INFINITY;
  const double factor = reached ? a.max_norm / norm : 1.0;
  for_units<TABLE>(list, a, gridDim.x - 1 - blockIdx.x, [&](const Item& it, uint32_t unit) {
    if (!reached && it.out == it.data) return;
    if (it.dtype == GS_F32) unit_scaled<F32Value>(it, unit, factor, !reached);
    else if (it.dtype == GS_BF16) unit_scaled<HalfValue<bf16_t>>(it, unit, factor, !reached);
    else unit_scaled<HalfValue<f16_t>>(it, unit, factor, !reached);
  });
}

__global__ __launch_bounds__(kThreads) void table_kernel(Items list, Item* to) {
  for (int k = threadIdx.x; k < list.items; k += kThreads) to[k] = list.item[k];
}

int64_t elem_bytes(int32_t dtype) { return dtype == GS_F32 ? 4 : 2; }
// the next kPerLaunch tensors that are not empty, from `at` on; returns where the ones after them begin
int32_t fill_items(const gs_tensor* list, int32_t num_tensors, int32_t at, Items& to, uint32_t& units) {
  to.items = 0;
  while (at < num_tensors && to.items < kPerLaunch) {
    const gs_tensor& t = list[at++];
    if (t.count == 0) continue;
    to.item[to.items++] = Item{t.data, t.out ? t.out : t.data, t.count, units, t.dtype};
    units += (uint32_t)std::max<int64_t>(1, ceil_div(ceil_div(t.count * elem_bytes(t.dtype), 16), kUnit));
  }
  return at;
}

struct ClipPlan {
  double* parts;
  Item* table;
  size_t bytes;
};
ClipPlan plan_clip(void* ws, int64_t num_tensors) {
  ClipPlan p{};
  Carver c(ws);
  p.parts = c.take<double>(kMaxGroups);
  if (num_tensors > kPerLaunch) p.table = c.take<Item>((size_t)num_tensors);
  p.bytes = c.used;
  return p;
}

template <bool TABLE>
int32_t run_passes(const Items& list, const Pass& a, bool norm_alone, hipStream_t stream) {
  const unsigned groups = (unsigned)a.num_parts;
  if (groups > 0) {
    squares_kernel<TABLE><<<groups, kThreads, 0, stream>>>(list, a);
    GS_LAUNCH_CHECK();
  }
  Pass second = a;
  if (norm_alone) second.units = 0;
  clip_kernel<TABLE><<<norm_alone ? 1 : groups, kThreads, 0, stream>>>(list, second);
  GS_LAUNCH_CHECK();
  return GS_OK;
}

}  // namespace
}  // namespace gs

using namespace gs;

extern "C" size_t gs_clip_grads_workspace_bytes(int32_t num_tensors) {
  return num_tensors < 0 ? 0 : plan_clip(nullptr, num_tensors).bytes;
}

extern "C" int32_t gs_clip_grads(const gs_tensor* list, int32_t num_tensors, double max_norm, double* norm_out, void* ws,
                                 size_t ws_bytes, void* stream_) {
  hipStream_t stream = (hipStream_t)stream_;
  if (num_tensors < 0 || (num_tensors > 0 && !list) || !norm_out || !(max_norm >= 0.0)) return GS_EINVAL;
  if (!ws || !aligned(ws, 256)) return GS_EINVAL;
  int64_t total = 0;
  bool elsewhere = false;
  for (int32_t i = 0; i < num_tensors; ++i) {
    const gs_tensor& t = list[i];
    if (t.dtype != GS_F32 && t.dtype != GS_BF16 && t.dtype != GS_F16) return GS_EINVAL;
    if (t.count < 0 || t.count > ((int64_t)1 << 40)) return GS_EINVAL;
    if (t.count == 0) continue;
    if (!t.data || !aligned(t.data, (size_t)elem_bytes(t.dtype)) || !aligned(t.out, (size_t)elem_bytes(t.dtype))) return GS_EINVAL;
    if (t.out && t.out != t.data) elsewhere = true;
    total += t.count;
    if (total > ((int64_t)1 << 40)) return GS_EINVAL;
  }
  const ClipPlan p = plan_clip(ws, num_tensors);
  if (ws_bytes < p.bytes) return GS_EWORKSPACE;
  Items items;
  uint32_t units = 0;
  int32_t count = 0;
  int32_t at = fill_items(list, num_tensors, 0, items, units);
  const bool table = at < num_tensors;
  while (table && items.items > 0) {
    table_kernel<<<1, kThreads, 0, stream>>>(items, p.table + count);
    GS_LAUNCH_CHECK();
    count += items.items;
    at = fill_items(list, num_tensors, at, items, units);
  }
  const bool norm_alone = units == 0 || (!elsewhere && std::isinf(max_norm));
  const Pass a{p.table, table ? count : items.items, units, p.parts, (int32_t)std::min<uint32_t>(units, kMaxGroups), max_norm, norm_out};
  return table ? run_passes<true>(items, a, norm_alone, stream) : run_passes<false>(items, a, norm_alone, stream);
}
