// gs_beam_select: the best continuations of a group's walks over all of them and all nodes.  gs_beam_reorder: what is kept for the
// walks follows.
//
//   p_bj = logp_b + s_bj - log sum_i exp(s_bi);  of a group, the `width` first by p, then lower b, larger s, lower j
//
// Inside a row the order is that of the scores, so that the width best of a row, or of a part of it, are known without its sum.
// A workgroup holds a part of a row in registers: one read gives its largest score, the sum of its weights below that (fp64, for
// comparisons across rows: an fp32 sum would exchange neighbours of different walks) and its width best, in order.  One workgroup a
// group then adds the parts' sums and joins the lists.
//
// The width best without a sort: of the largest score of each lane, the width-th largest is a lower bound of what can be taken,
// and little more than `width` scores reach it.  Those go to a list, where each one's place is the number of larger ones.  Where too
// many reach it (equal scores), the best is taken out `width` times instead.

#include "weigh.h"

namespace gs {
namespace {

constexpr int kMostWidth = 256;
constexpr int kPartThreads = 256;
constexpr int kJoinThreads = 512;
constexpr int kPartList = 1024;                // scores that may reach the bound
constexpr int kJoinList = 2048;
static_assert(kPartThreads >= kMostWidth && kJoinThreads >= kMostWidth, "a lane each for the bound");

struct SelectArgs {
  const void* scores;
  int64_t groups, rows, n;
  int32_t beams, width;
  const float* logp;
  const uint8_t* ended;                        // or null
  int32_t parts;                               // of a row
  int64_t part_len;
  uint64_t* keys;                              // [rows][parts][width]: a part's best, in order
  int32_t* counts;                             // [rows][parts]: how many these are
  float* tops;                                 // largest score
  double* sums;                                // of exp(s - top)
  int32_t *parents, *nodes;
  float* logp_out;
};

// larger for an earlier place in the order: score, then node
__device__ __forceinline__ uint64_t place_of(uint32_t key, uint32_t node) { return (uint64_t)key << 32 | (uint32_t)~node; }

// the same order for fp64 values; 0: no candidate (-infinity or NaN)
__device__ __forceinline__ uint64_t key64_of(double p) {
  if (!(p > -INFINITY)) return 0;
  const uint64_t b = (uint64_t)__double_as_longlong(p == 0.0 ? 0.0 : p);
  return (b >> 63) ? ~b : (b | 0x8000000000000000ull);
}
__device__ __forceinline__ double value_of(uint64_t key) {
  return __longlong_as_double((long long)((key >> 63) ? (key & 0x7fffffffffffffffull) : ~key));
}

__device__ __forceinline__ uint64_t wave_most(uint64_t v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = max(v, (uint64_t)__shfl_xor((unsigned long long)v, d, 64));
  return v;
}

// The width-th largest of a value of each lane, 0 if there are fewer than `width` above 0: a lower bound of the width-th largest
// of all, if each lane's value is one of them.
template <int THREADS, typename K>
__device__ __forceinline__ K bound_of(K own, int width, K* all, K* bound) {
  all[threadIdx.x] = own;
  if (threadIdx.x == 0) *bound = 0;
  __syncthreads();
  int before = 0;
  for (int t = 0; t < THREADS; ++t) before += all[t] > own || (all[t] == own && t < (int)threadIdx.x);
  if (before == width - 1) *bound = own;
  __syncthreads();
  return *bound;
}

struct PartShared {
  double powers[kPowers];
  float wave_top[kPartThreads / 64];
  double wave_sum[kPartThreads / 64];
  uint32_t lane_top[kPartThreads];
  uint32_t bound;
  uint32_t listed;
  uint64_t list[kPartList];
  uint64_t wave_best[2][kPartThreads / 64];
};

template <typename V, int LOADS>
__global__ __launch_bounds__(kPartThreads) void part_kernel(SelectArgs a) {
  typedef typename V::elem elem;
  constexpr int kPer = 16 / (int)sizeof(elem);
  __shared__ PartShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t row = blockIdx.x / (uint32_t)a.parts, part = blockIdx.x - row * (uint32_t)a.parts;
  const int64_t slot = (int64_t)blockIdx.x;
  if (!(a.logp[row] > -INFINITY) || (a.ended && a.ended[row])) {      // not looked at
    if (tid == 0) a.counts[slot] = 0, a.tops[slot] = -INFINITY, a.sums[slot] = 0.0;
    return;
  }
  fill_powers(sh.powers);
  if (tid == 0) sh.listed = 0;
  const int64_t from = (int64_t)part * a.part_len;
  const int len = (int)min(a.n - from, a.part_len), whole = len / kPer;      // of 16 bytes
  const elem* base = static_cast<const elem*>(a.scores) + (int64_t)row * a.n + from;
  float s[LOADS][kPer];
  {
    uint4 w[LOADS];
#pragma unroll
    for (int e = 0; e < LOADS; ++e) {
      const int p = e * kPartThreads + tid;
      if (p < whole) __builtin_memcpy(&w[e], base + (int64_t)p * kPer, 16);
    }
#pragma unroll
    for (int e = 0; e < LOADS; ++e) {
      const int p = e * kPartThreads + tid;
      elem x[kPer];
      __builtin_memcpy(x, &w[e], 16);
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const float v = V::get(x[k]);
        s[e][k] = p < whole && v > -INFINITY ? v : -INFINITY;
      }
      if (p == whole)
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
          if (p * kPer + k >= len) break;
          const float v = V::get(base[(int64_t)p * kPer + k]);
          s[e][k] = v > -INFINITY ? v : -INFINITY;
        }
    }
  }
  float own = -INFINITY;
#pragma unroll
  for (int e = 0; e < LOADS; ++e)
#pragma unroll
    for (int k = 0; k < kPer; ++k) own = fmaxf(own, s[e][k]);
  float top = own;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  if (lane == 0) sh.wave_top[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPartThreads / 64; ++w) top = fmaxf(top, sh.wave_top[w]);
  if (!(top > -INFINITY)) {                      // nothing there
    if (tid == 0) a.counts[slot] = 0, a.tops[slot] = -INFINITY, a.sums[slot] = 0.0;
    return;
  }

  const Weigh weigh(top, 1.0f, sh.powers);
  double sum = 0.0;
#pragma unroll
  for (int e = 0; e < LOADS; ++e)
#pragma unroll
    for (int k = 0; k < kPer; ++k) sum += weigh(s[e][k]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
  if (lane == 0) sh.wave_sum[wave] = sum;

  const uint32_t bound = bound_of<kPartThreads>(key_of(own), a.width, sh.lane_top, &sh.bound);
  const float least = bound ? score_of(bound) : -INFINITY;
  int reach = 0;
#pragma unroll
  for (int e = 0; e < LOADS; ++e)
#pragma unroll
    for (int k = 0; k < kPer; ++k) reach += s[e][k] >= least && s[e][k] > -INFINITY;
  if (reach > 0) {
    uint32_t to = atomicAdd(&sh.listed, (uint32_t)reach);
#pragma unroll
    for (int e = 0; e < LOADS; ++e)
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if (s[e][k] >= least && s[e][k] > -INFINITY) {
          if (to < kPartList) sh.list[to] = place_of(key_of(s[e][k]), (uint32_t)(from + (e * kPartThreads + tid) * kPer + k));
          ++to;
        }
  }
  __syncthreads();
  const int listed = (int)sh.listed;
  uint64_t* keys = a.keys + slot * a.width;
  if (listed <= kPartList) {
    for (int c = tid; c < listed; c += kPartThreads) {
      const uint64_t place = sh.list[c];
      int before = 0;
      for (int o = 0; o < listed; ++o) before += sh.list[o] > place;
      if (before < a.width) keys[before] = place;
    }
  } else {
    uint64_t last = ~0ull, best = ~0ull;
    for (int taken = 0; taken < a.width; ++taken) {         // listed > width: there are as many
      if (best >= last) {
        best = 0;
#pragma unroll
        for (int e = 0; e < LOADS; ++e)
#pragma unroll
          for (int k = 0; k < kPer; ++k)
            if (s[e][k] > -INFINITY) {
              const uint64_t place = place_of(key_of(s[e][k]), (uint32_t)(from + (e * kPartThreads + tid) * kPer + k));
              if (place < last) best = max(best, place);
            }
      }
      const uint64_t most = wave_most(best);
      if (lane == 0) sh.wave_best[taken & 1][wave] = most;
      __syncthreads();
      last = 0;
#pragma unroll
      for (int w = 0; w < kPartThreads / 64; ++w) last = max(last, sh.wave_best[taken & 1][w]);
      if (tid == 0) keys[taken] = last;
    }
  }
  if (tid == 0) {
    double all = 0.0;
#pragma unroll
    for (int w = 0; w < kPartThreads / 64; ++w) all += sh.wave_sum[w];
    a.counts[slot] = min(listed, a.width);
    a.tops[slot] = top;
    a.sums[slot] = all;
  }
}

// a candidate's place in the order of its group: larger p, lower row, earlier in the row
struct Place {
  uint64_t p, in_row;
  uint32_t row;
  __device__ __forceinline__ bool before(const Place& o) const {
    return p != o.p ? p > o.p : row != o.row ? row < o.row : in_row > o.in_row;
  }
};

struct JoinShared {
  float top[kMostWidth];                       // by walk of the group
  float logp[kMostWidth];
  double log_sum[kMostWidth];                  // log sum exp(s - top)
  uint8_t state[kMostWidth];                   // 0: no walk, 1: one, 2: one that has ended
  uint64_t lane_top[kJoinThreads];
  uint64_t bound;
  uint32_t listed;
  uint64_t p[kJoinList], in_row[kJoinList];
  uint32_t row[kJoinList];
  Place wave_best[2][kJoinThreads / 64];
};

__global__ __launch_bounds__(kJoinThreads) void join_kernel(SelectArgs a) {
  __shared__ JoinShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t group = blockIdx.x, first_row = group * a.beams;
  if (tid == 0) sh.listed = 0;
  for (int b = wave; b < a.beams; b += kJoinThreads / 64) {        // a wave adds a row's parts, in a fixed order
    const int64_t slot = (first_row + b) * a.parts;
    float top = -INFINITY;
    for (int part = lane; part < a.parts; part += 64) top = fmaxf(top, a.tops[slot + part]);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    double sum = 0.0;
    for (int part = lane; part < a.parts; part += 64) {
      const float t = a.tops[slot + part];
      if (t > -INFINITY) sum += a.sums[slot + part] * (t == top ? 1.0 : exp((double)t - (double)top));
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
    if (lane == 0) {
      const float logp = a.logp[first_row + b];
      sh.top[b] = top;
      sh.logp[b] = logp;
      sh.log_sum[b] = log(sum);
      sh.state[b] = !(logp > -INFINITY) ? 0 : a.ended && a.ended[first_row + b] ? 2 : 1;
    }
  }
  __syncthreads();

  const int64_t lists = (int64_t)a.beams * a.parts;
  auto size_of = [&](int b, int part) {        // candidates of a list
    return sh.state[b] == 1 ? a.counts[(first_row + b) * a.parts + part] : sh.state[b] == 2 && part == 0 ? 1 : 0;
  };
  auto place_at = [&](int b, int part, int t) {
    Place c{0, 0, (uint32_t)b};
    if (sh.state[b] == 2) {
      c.p = key64_of((double)sh.logp[b]);
    } else {
      c.in_row = a.keys[((first_row + b) * a.parts + part) * a.width + t];
      const float s = score_of((uint32_t)(c.in_row >> 32));
      c.p = key64_of((double)sh.logp[b] + ((s == sh.top[b] ? 0.0 : (double)s - (double)sh.top[b]) - sh.log_sum[b]));
    }
    return c;
  };

  uint64_t own = 0;
  for (int64_t l = tid; l < lists; l += kJoinThreads) {
    const int b = (int)(l / a.parts), part = (int)(l - (int64_t)b * a.parts);
    if (size_of(b, part) > 0) own = max(own, place_at(b, part, 0).p);
  }
  const uint64_t bound = max(bound_of<kJoinThreads>(own, a.width, sh.lane_top, &sh.bound), (uint64_t)1);
  for (int64_t l = tid; l < lists; l += kJoinThreads) {
    const int b = (int)(l / a.parts), part = (int)(l - (int64_t)b * a.parts), size = size_of(b, part);
    for (int t = 0; t < size; ++t) {
      const Place c = place_at(b, part, t);
      if (c.p < bound) break;
      const uint32_t to = atomicAdd(&sh.listed, 1u);
      if (to < kJoinList) sh.p[to] = c.p, sh.in_row[to] = c.in_row, sh.row[to] = c.row;
    }
  }
  __syncthreads();

  auto write = [&](int at, const Place& c) {
    const int64_t to = group * a.width + at;
    const bool there = c.p != 0;
    a.parents[to] = there ? (int32_t)c.row : -1;
    a.nodes[to] = there && sh.state[c.row] == 1 ? (int32_t)~(uint32_t)c.in_row : -1;
    a.logp_out[to] = there ? (float)value_of(c.p) : -INFINITY;
  };
  const int listed = (int)sh.listed;
  if (listed <= kJoinList) {
    for (int c = tid; c < listed; c += kJoinThreads) {
      const Place own{sh.p[c], sh.in_row[c], sh.row[c]};
      int before = 0;
      for (int o = 0; o < listed; ++o) before += Place{sh.p[o], sh.in_row[o], sh.row[o]}.before(own);
      if (before < a.width) write(before, own);
    }
    for (int at = listed + tid; at < a.width; at += kJoinThreads) write(at, Place{0, 0, 0});
    return;
  }
  // The best is taken out `width` times; a lane looks again through its own lists only where it was its own.
  Place last{~0ull, ~0ull, 0}, best = last;
  for (int taken = 0; taken < a.width; ++taken) {
    if (!last.before(best)) {
      best = Place{0, 0, 0};
      for (int64_t l = tid; l < lists; l += kJoinThreads) {
        const int b = (int)(l / a.parts), part = (int)(l - (int64_t)b * a.parts), size = size_of(b, part);
        for (int t = 0; t < size; ++t) {
          const Place c = place_at(b, part, t);
          if (c.p == 0 || !last.before(c)) continue;
          if (c.before(best)) best = c;
          break;
        }
      }
    }
    Place most = best;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      Place o;
      o.p = (uint64_t)__shfl_xor((unsigned long long)most.p, d, 64);
      o.in_row = (uint64_t)__shfl_xor((unsigned long long)most.in_row, d, 64);
      o.row = (uint32_t)__shfl_xor((int)most.row, d, 64);
      if (o.before(most)) most = o;
    }
    if (lane == 0) sh.wave_best[taken & 1][wave] = most;
    __syncthreads();
    last = sh.wave_best[taken & 1][0];
    for (int w = 1; w < kJoinThreads / 64; ++w)
      if (sh.wave_best[taken & 1][w].before(last)) last = sh.wave_best[taken & 1][w];
    if (tid == 0) write(taken, last);
  }
}

struct SelectPlan {
  int loads;
  int32_t parts;
  int64_t part_len;
  uint64_t* keys;
  int32_t* counts;
  float* tops;
  double* sums;
  size_t bytes;
};

SelectPlan plan_select(void* ws, int64_t groups, int32_t beams, int64_t n, int32_t width, int32_t dtype) {
  SelectPlan p{};
  const int64_t per = dtype == GS_F32 ? 4 : 8, rows = groups * beams;
  // Few rows: parts small enough that every compute unit has one.
  p.loads = dtype == GS_F32 ? 16 : 8;
  while (p.loads > 2 && rows * ceil_div(n, per * kPartThreads * p.loads) < 512) p.loads /= 2;
  p.part_len = per * kPartThreads * p.loads;
  p.parts = (int32_t)ceil_div(n, p.part_len);
  Carver carve(ws);
  p.keys = carve.take<uint64_t>((size_t)rows * p.parts * width);
  p.counts = carve.take<int32_t>((size_t)rows * p.parts);
  p.tops = carve.take<float>((size_t)rows * p.parts);
  p.sums = carve.take<double>((size_t)rows * p.parts);
  p.bytes = carve.used;
  return p;
}

bool dtype_known(int32_t dtype) { return dtype == GS_F32 || dtype == GS_BF16 || dtype == GS_F16; }
constexpr int64_t kMostRows = ((int64_t)1 << 22) - 1;
// before the products that they bound
bool select_shape_ok(int64_t groups, int32_t beams, int64_t n, int32_t width, int32_t dtype) {
  return groups >= 0 && groups <= (int64_t)INT32_MAX && beams >= 1 && beams <= kMostWidth && width >= 1 && width <= kMostWidth && n >= 1 &&
         n <= (int64_t)INT32_MAX && dtype_known(dtype);
}

template <typename V>
void launch_parts(const SelectArgs& a, int loads, unsigned grid, hipStream_t s) {
  if (loads == 16) part_kernel<V, 16><<<dim3(grid), kPartThreads, 0, s>>>(a);
  if (loads == 8) part_kernel<V, 8><<<dim3(grid), kPartThreads, 0, s>>>(a);
  if (loads == 4) part_kernel<V, 4><<<dim3(grid), kPartThreads, 0, s>>>(a);
  if (loads == 2) part_kernel<V, 2><<<dim3(grid), kPartThreads, 0, s>>>(a);
}

}  // namespace

// ---- gs_beam_reorder ----------------------------------------------------------
namespace {

constexpr int kCopyThreads = 256;
constexpr int kStates = 64;                    // of one launch
constexpr int kAhead = 4;                      // pieces of a lane in flight
constexpr int kStripe = 4096;                  // pieces of a group that a workgroup holds, in place

struct ReorderArgs {
  struct State {
    const char* data;
    char* out;
    int64_t row_bytes, append_at;
    int32_t piece;                             // bytes: 16, 4 or 1
    int32_t first;                             // workgroup
  };
  State state[kStates];
  int32_t num_states, beams, width;
  int64_t groups;
  const int32_t *parents, *nodes;
};

// The node goes into its piece of the row, or is written alone where the row stays.
template <typename P>
__device__ __forceinline__ void put_node(P* row, int64_t append_at, int32_t node) {
  *reinterpret_cast<int32_t*>(reinterpret_cast<char*>(row) + append_at) = node;
}

// One state, to another buffer: row by row, `lanes` lanes along a row (a power of two), kAhead pieces each.
template <typename P>
__device__ void copy_rows(const ReorderArgs& a, const ReorderArgs::State& st, int64_t at) {
  const int64_t pieces = st.row_bytes / (int64_t)sizeof(P), rows = a.groups * a.width;
  int shift = 0;
  while ((1 << shift) < kCopyThreads && (1 << shift) < pieces) ++shift;
  const int lanes = 1 << shift, rows_at_once = kCopyThreads >> shift;
  const int64_t chunks = (pieces + (int64_t)lanes * kAhead - 1) / ((int64_t)lanes * kAhead);
  const int64_t block_row = at / chunks, chunk = at - block_row * chunks;
  const int64_t r = block_row * rows_at_once + (threadIdx.x >> shift);
  if (r >= rows) return;
  const int64_t group = r / a.width;
  const int32_t parent = a.parents[r];
  if (parent < 0 || parent >= a.beams) return;
  const P* from = reinterpret_cast<const P*>(st.data + (group * a.beams + parent) * st.row_bytes);
  P* to = reinterpret_cast<P*>(st.out + r * st.row_bytes);
  const int64_t first = chunk * lanes * kAhead + (threadIdx.x & (lanes - 1));
  P x[kAhead];
#pragma unroll
  for (int e = 0; e < kAhead; ++e)
    if (first + e * lanes < pieces) x[e] = from[first + e * lanes];
#pragma unroll
  for (int e = 0; e < kAhead; ++e) {
    const int64_t p = first + e * lanes;
    if (p >= pieces) break;
    to[p] = x[e];
    if (st.append_at >= 0 && st.append_at / (int64_t)sizeof(P) == p) put_node(to, st.append_at, a.nodes[r]);   // after its piece, by its lane
  }
}

// One state in place: a workgroup has a stripe of a group's rows, all of them, reads what moves and then writes it.
template <typename P>
__device__ void move_rows(const ReorderArgs& a, const ReorderArgs::State& st, int64_t at, uint4* lds) {
  P* held = reinterpret_cast<P*>(lds);
  const int64_t pieces = st.row_bytes / (int64_t)sizeof(P);
  int shift = 6;
  while ((a.beams << shift) > kStripe) --shift;
  const int wide = 1 << shift;
  const int64_t stripes = (pieces + wide - 1) / wide, group = at / stripes, first = (at - group * stripes) * wide;
  const int total = a.beams << shift;
  const int32_t* parents = a.parents + group * a.beams;
  char* rows = st.out + group * a.beams * st.row_bytes;
  for (int t = threadIdx.x; t < total; t += kCopyThreads) {
    const int k = t >> shift;
    const int64_t p = first + (t & (wide - 1));
    const int32_t parent = parents[k];
    if (parent >= 0 && parent < a.beams && parent != k && p < pieces) held[t] = reinterpret_cast<const P*>(rows + parent * st.row_bytes)[p];
  }
  __syncthreads();
  for (int t = threadIdx.x; t < total; t += kCopyThreads) {
    const int k = t >> shift;
    const int64_t p = first + (t & (wide - 1));
    const int32_t parent = parents[k];
    if (parent < 0 || parent >= a.beams || p >= pieces) continue;
    P* row = reinterpret_cast<P*>(rows + k * st.row_bytes);
    if (parent != k) row[p] = held[t];
    if (st.append_at >= 0 && st.append_at / (int64_t)sizeof(P) == p) put_node(row, st.append_at, a.nodes[group * a.beams + k]);
  }
}

template <bool IN_PLACE>
__global__ __launch_bounds__(kCopyThreads) void reorder_kernel(ReorderArgs a) {
  __shared__ uint4 lds[IN_PLACE ? kStripe : 1];
  int s = 0;
  while (s + 1 < a.num_states && (int)blockIdx.x >= a.state[s + 1].first) ++s;
  const ReorderArgs::State& st = a.state[s];
  const int64_t at = (int64_t)blockIdx.x - st.first;
  if (IN_PLACE) {
    if (st.piece == 16) move_rows<uint4>(a, st, at, lds);
    else if (st.piece == 4) move_rows<uint32_t>(a, st, at, lds);
    else move_rows<uint8_t>(a, st, at, lds);
  } else {
    if (st.piece == 16) copy_rows<uint4>(a, st, at);
    else if (st.piece == 4) copy_rows<uint32_t>(a, st, at);
    else copy_rows<uint8_t>(a, st, at);
  }
}

// workgroups of a state
int64_t copy_blocks(int64_t pieces, int64_t rows) {
  int64_t lanes = 1;
  while (lanes < kCopyThreads && lanes < pieces) lanes *= 2;
  return ceil_div(rows, kCopyThreads / lanes) * ceil_div(pieces, lanes * kAhead);
}
int64_t move_blocks(int64_t pieces, int64_t groups, int32_t beams) {
  int64_t wide = 64;
  while (wide * beams > kStripe) wide /= 2;
  return groups * ceil_div(pieces, wide);
}

bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a_bytes > 0 && b_bytes > 0 && x < y + (uintptr_t)b_bytes && y < x + (uintptr_t)a_bytes;
}

}  // namespace
}  // namespace gs

using namespace gs;

extern "C" size_t gs_beam_select_workspace_bytes(int64_t groups, int32_t beams, int64_t n, int32_t width, int32_t dtype) {
  if (!select_shape_ok(groups, beams, n, width, dtype) || groups * beams > kMostRows) return 0;
  return std::max<size_t>(plan_select(nullptr, std::max<int64_t>(groups, 1), beams, n, width, dtype).bytes, 256);
}

extern "C" int32_t gs_beam_select(const void* scores, int64_t groups, int32_t beams, int64_t n, int32_t dtype, const float* logp,
                                  const uint8_t* ended, int32_t width, int32_t* parents_out, int32_t* nodes_out, float* logp_out, void* ws,
                                  size_t ws_bytes, void* stream) {
  if (!select_shape_ok(groups, beams, n, width, dtype) || !ws || !aligned(ws, 256)) return GS_EINVAL;
  if (!aligned(scores, dtype == GS_F32 ? 4 : 2) || !aligned(logp, 4) || !aligned(parents_out, 4) || !aligned(nodes_out, 4) || !aligned(logp_out, 4))
    return GS_EINVAL;
  if (groups > 0 && (!scores || !logp || !parents_out || !nodes_out || !logp_out)) return GS_EINVAL;
  if (groups * beams > kMostRows) return GS_EOVERFLOW;
  if (groups == 0) return GS_OK;
  const SelectPlan p = plan_select(ws, groups, beams, n, width, dtype);
  if (ws_bytes < p.bytes) return GS_EWORKSPACE;
  const int64_t grid = groups * beams * p.parts;
  if (grid > (int64_t)INT32_MAX) return GS_EOVERFLOW;
  const SelectArgs a{scores, groups, groups * beams, n, beams, width, logp, ended, p.parts, p.part_len, p.keys, p.counts, p.tops, p.sums, parents_out,
                     nodes_out, logp_out};
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == GS_F32) launch_parts<ScoreF32>(a, p.loads, (unsigned)grid, s);
  if (dtype == GS_BF16) launch_parts<ScoreHalf<bf16_t>>(a, p.loads, (unsigned)grid, s);
  if (dtype == GS_F16) launch_parts<ScoreHalf<f16_t>>(a, p.loads, (unsigned)grid, s);
  GS_LAUNCH_CHECK();
  join_kernel<<<dim3((unsigned)groups), kJoinThreads, 0, s>>>(a);
  GS_LAUNCH_CHECK();
  return GS_OK;
}

extern "C" int32_t gs_beam_reorder(const gs_state* list, int32_t num_states, int64_t groups, int32_t beams, int32_t width,
                                   const int32_t* parents, const int32_t* nodes, void* stream) {
  if (num_states < 0 || (num_states > 0 && !list) || groups < 0 || groups > (int64_t)INT32_MAX || beams < 1 || beams > kMostWidth || width < 1 ||
      width > kMostWidth)
    return GS_EINVAL;
  if (groups > 0 && (!parents || !aligned(parents, 4) || !aligned(nodes, 4))) return GS_EINVAL;
  if (groups * std::max(beams, width) > kMostRows) return GS_EOVERFLOW;
  const int64_t rows_in = groups * beams, rows_out = groups * width;
  for (int i = 0; i < num_states; ++i) {
    const gs_state& x = list[i];
    const bool in_place = !x.out || x.out == x.data;
    if (x.row_bytes < 0 || x.row_bytes >= ((int64_t)1 << 40) || (in_place && beams != width && x.row_bytes > 0)) return GS_EINVAL;
    if (x.row_bytes > 0 && groups > 0 && !x.data) return GS_EINVAL;
    if (x.append_at < -1 || (x.append_at >= 0 && (x.append_at % 4 != 0 || x.append_at + 4 > x.row_bytes || x.row_bytes % 4 != 0 || !nodes ||
                                                  !aligned(x.data, 4) || !aligned(x.out, 4))))
      return GS_EINVAL;
  }
  for (int i = 0; i < num_states; ++i)         // what is written overlaps nothing else
    for (int j = 0; j < num_states; ++j) {
      const gs_state &x = list[i], &y = list[j];
      const bool in_place = !x.out || x.out == x.data, other_in_place = !y.out || y.out == y.data;
      const void* out = in_place ? x.data : x.out;
      if (!(i == j && in_place) && overlap(out, rows_out * x.row_bytes, y.data, rows_in * y.row_bytes)) return GS_EINVAL;
      if (i != j && !other_in_place && overlap(out, rows_out * x.row_bytes, y.out, rows_out * y.row_bytes)) return GS_EINVAL;
    }
  if (groups == 0) return GS_OK;
  for (int in_place = 0; in_place < 2; ++in_place) {
    ReorderArgs a{};
    a.beams = beams, a.width = width, a.groups = groups, a.parents = parents, a.nodes = nodes;
    int64_t blocks = 0;
    auto launch = [&]() -> int32_t {
      if (a.num_states == 0) return GS_OK;
      if (in_place) reorder_kernel<true><<<dim3((unsigned)blocks), kCopyThreads, 0, (hipStream_t)stream>>>(a);
      else reorder_kernel<false><<<dim3((unsigned)blocks), kCopyThreads, 0, (hipStream_t)stream>>>(a);
      GS_LAUNCH_CHECK();
      a.num_states = 0, blocks = 0;
      return GS_OK;
    };
    for (int i = 0; i < num_states; ++i) {
      const gs_state& x = list[i];
      if ((!x.out || x.out == x.data) != (in_place == 1) || x.row_bytes == 0) continue;
      void* out = in_place ? x.data : x.out;
      int piece = 1;
      for (int size : {4, 16})
        if (aligned(x.data, size) && aligned(out, size) && x.row_bytes % size == 0) piece = size;
      const int64_t pieces = x.row_bytes / piece, more = in_place ? move_blocks(pieces, groups, beams) : copy_blocks(pieces, rows_out);
      if (more > (int64_t)INT32_MAX) return GS_EOVERFLOW;
      if (a.num_states == kStates || blocks + more > (int64_t)INT32_MAX) {
        const int32_t rc = launch();
        if (rc != GS_OK) return rc;
      }
      a.state[a.num_states++] = ReorderArgs::State{static_cast<const char*>(x.data), static_cast<char*>(out), x.row_bytes, x.append_at, piece, (int32_t)blocks};
      blocks += more;
    }
    const int32_t rc = launch();
    if (rc != GS_OK) return rc;
  }
  return GS_OK;
}
