// gs_sample_scores: one node per row of scores, by temperature, top-k, top-p and min-p, from given random numbers.
//
//   order: score descending, index ascending among equal scores;  e_j = exp((s_j - max) / temperature) in fp64
//   top-k: the first k;  top-p: those of them with sum of e before < top_p * sum of e;  min-p: e_j >= min_p
//   answer: the smallest index j with  sum_{i <= j, kept} e_i > u * sum_{kept} e
//
// The row is never sorted.  A score becomes a 32-bit key of the same order, and a histogram over 2048 equal steps of the score
// between the row's least and greatest (scores spread over them; over the bits of a float they would not) says in which step
// the cut of top-k or top-p lies.  With top-k the nodes from that step up go to a short list, which is sorted and holds all
// there is to decide; with top-p alone only that step's nodes do, while the weights of those above are added by pieces of the
// index, so that the answer is looked for in one piece.  Weights are added as integers (multiples of 2^-62, in two halves of 31
// bits): neither the order of the atomics nor the shape of the launch changes a sum.  Comparisons near a border are why nothing
// here is fp32: an error of 1e-7 of the sum would move the answer to a neighbour for one row in ten at a million nodes.
//
// A list that would be too long (thousands of nodes of one step: k in the thousands, or equal scores) is not made: histograms of
// the key inside the step, and of the index among equal keys, go down to the cut instead, over the whole row each time.
//
// Two routes.  Row by row: one workgroup does all of it.  Split: where rows are long and fewer than the compute units need,
// three passes over the scores by several workgroups a row (least and greatest; histogram; list and pieces), and one workgroup
// a row finishes.
//
// Measured: 64 rows of 1 M fp32 scores, every filter: 45 us for the least and greatest (5.7 TB/s), 57 histogram, 9 plan, 45 list,
// 30 to finish (a chain of small steps in one workgroup a row).  256 rows of 100,003 bf16 scores, top-p alone: 19, 51, 9, 33, 22:
// the histogram weighs every score and adds it with three LDS atomics, the list weighs what lies above the cut.  One row of 10,000:
// 16 us, latency of its steps.  Cuts among more nodes than a list takes are one workgroup's, which reads the whole row for every
// level: 64 rows of 1 M, top-k of 10,000, 1.5 of 1.6 ms in all, with top-p 3.7 of 3.9; one such row 1.15 of 1.18 ms, where plain
// operations, which sort it, take 0.48.

#include "weigh.h"

namespace gs {
namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 2048;
constexpr int kAhead = 4;                      // 16-byte loads per lane in flight
constexpr int kListMost = 2 * kBins;           // elements of a row that may go to its list: room for two values of a 16-bit
                                               // format, which a step may hold, in rows of a million nodes
constexpr int kSplitGroups = 2048;             // of one launch: eight per compute unit, where each has kSplitMany scores at least;
constexpr int kSplitMany = 24576;              // half as many where not: a workgroup's histogram costs 40 KB of LDS and its sums
constexpr int kPartLeast = 2048;                // scores per part at least: what one histogram along the index takes
constexpr int kSplitLeast = 8192;              // scores per workgroup at least, of few rows

struct SampleArgs {
  const void* scores;
  int64_t rows, n;
  const float* uniforms;
  const float* temperature;                    // each of the four: [rows] or null
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* ids;
  float* probs;                                // or null
};

// A row's parameters, as the filters see them.
struct RowLimits {
  float temperature, top_p;
  double min_p, u;
  int64_t k;
  bool by_k, by_p;
  __device__ __forceinline__ RowLimits(const SampleArgs& a, int64_t r) {
    temperature = a.temperature ? a.temperature[r] : 1.0f;
    k = a.top_k ? a.top_k[r] : 0;
    top_p = a.top_p ? a.top_p[r] : 1.0f;
    min_p = a.min_p && a.min_p[r] > 0.0f ? fmin((double)a.min_p[r], 1.0) : 0.0;
    u = a.uniforms[r] < 0.0f ? 0.0 : (double)a.uniforms[r];       // NaN stays: no sum passes it
    by_k = k > 0 && k < a.n;
    by_p = top_p < 1.0f;
  }
};

// A sum of weights as integers: hi * 2^31 + lo, in units of 2^-62.
struct Sum {
  uint64_t count, hi, lo;
  __device__ __forceinline__ double value() const {          // rounded once: a larger sum is never a smaller value
    const uint64_t h = hi + (lo >> 31), l = lo & 0x7fffffffu;
    return h < (1ull << 53) ? ((double)h * 0x1p31 + (double)l) * 0x1p-62 : (double)h * 0x1p-31;
  }
  __device__ __forceinline__ bool same_weight(const Sum& b) const {
    return hi + (lo >> 31) == b.hi + (b.lo >> 31) && ((lo ^ b.lo) & 0x7fffffffu) == 0;
  }
};
__device__ __forceinline__ Sum operator+(const Sum& a, const Sum& b) { return Sum{a.count + b.count, a.hi + b.hi, a.lo + b.lo}; }
__device__ __forceinline__ Sum operator-(const Sum& a, const Sum& b) { return Sum{a.count - b.count, a.hi - b.hi, a.lo - b.lo}; }
struct Units {
  uint32_t hi, lo;
};
__device__ __forceinline__ Units units_of(double weight) {            // 1 at most; every step is exact
  const double t = weight * 0x1p31;
  const uint32_t hi = (uint32_t)t;
  return Units{hi, (uint32_t)((t - (double)hi) * 0x1p31)};
}

struct Histogram {
  uint32_t count[kBins];
  unsigned long long hi[kBins], lo[kBins];
};
__device__ __forceinline__ void add_to(Histogram& h, int b, bool weights, double weight) {
  atomicAdd(&h.count[b], 1u);
  if (!weights) return;
  const Units w = units_of(weight);
  if ((w.hi | w.lo) == 0) return;
  atomicAdd(&h.hi[b], (unsigned long long)w.hi);
  atomicAdd(&h.lo[b], (unsigned long long)w.lo);
}

// a sum of weights, none if it is 0; counts the additions
__device__ __forceinline__ void add_units(Histogram& h, int b, uint64_t hi, uint64_t lo) {
  if ((hi | lo) == 0) return;
  atomicAdd(&h.count[b], 1u);
  atomicAdd(&h.hi[b], (unsigned long long)hi);
  atomicAdd(&h.lo[b], (unsigned long long)lo);
}

// 2048 equal steps between the row's least and greatest finite score.  fp32: every operation is monotone, which is all that a
// cut needs (this file is compiled without contraction: each pass has to find a score in the same step).  Halves, so that the
// distance of two floats is one.
struct Steps {
  float least, inverse;
  static __device__ __forceinline__ float half_of(float s) { return fminf(s, 3.4028234663852886e38f) * 0.5f; }
  __device__ __forceinline__ Steps(uint32_t kmin, uint32_t kmax) {
    least = half_of(score_of(kmin));
    const float range = half_of(score_of(kmax)) - least;
    inverse = range > 0.0f ? fminf((float)(kBins - 1) / range, 3.4028234663852886e38f) : 0.0f;
  }
  __device__ __forceinline__ int operator()(float s) const {
    return (int)fminf((half_of(s) - least) * inverse, (float)(kBins - 1));
  }
};
// The first of the keys [lo, hi] for which `yes` holds, once it holds for hi and for every key after such a one: 64 keys at a time.
template <typename Yes>
__device__ __forceinline__ uint32_t first_key(uint32_t lo, uint32_t hi, Yes yes) {
  const uint32_t lane = threadIdx.x & 63;
  while (lo < hi) {
    const uint32_t part = (hi - lo) / 64 + 1;
    const uint64_t at = (uint64_t)lo + (uint64_t)part * lane;      // lane 0: lo itself
    const uint64_t no = __ballot(at <= hi && !yes((uint32_t)min(at, (uint64_t)hi)));
    if (no == 0) return lo;
    const uint32_t last = 63 - __clzll((long long)no);             // the last key asked for that it does not hold for
    hi = (uint32_t)min((uint64_t)hi, (uint64_t)lo + (uint64_t)part * (last + 1));
    lo = lo + part * last + 1;
  }
  return lo;
}
// the keys of steps from .. to, among [kmin, kmax]; both steps hold a key
__device__ __forceinline__ void keys_of_steps(const Steps& steps, int from, int to, uint32_t kmin, uint32_t kmax, uint32_t& lo, uint32_t& hi) {
  lo = first_key(kmin, kmax, [=](uint32_t key) { return steps(score_of(key)) >= from; });
  hi = steps(score_of(kmax)) <= to ? kmax : first_key(lo, kmax, [=](uint32_t key) { return steps(score_of(key)) > to; }) - 1;
}

struct ListShared {
  uint32_t list_count, list_base;
  uint64_t list[kListMost];                    // ~key in the high half, index in the low one: sorts by the order of the nodes
};
struct Shared : ListShared {
  double powers[kPowers];
  Histogram hist;
  Sum wave_sum[kWaves];
  Sum found_above, found_in;
  int found_bin;
};

// A row in 16-byte pieces: position = index + skew, so that pieces lie on 16-byte boundaries wherever the row begins.  The first
// and the last piece are read element by element where they reach beyond the row.
template <typename V>
struct Row {
  typedef typename V::elem elem;
  static constexpr uint32_t kPer = 16 / sizeof(elem);
  const elem* base;                            // 16-byte aligned, skew elements in front of the row
  uint32_t skew, n;
  __device__ __forceinline__ Row(const void* scores, int64_t r, int64_t n_) {
    const elem* row = static_cast<const elem*>(scores) + r * n_;
    skew = (uint32_t)(((uintptr_t)row & 15) / sizeof(elem));
    base = row - skew;
    n = (uint32_t)n_;
  }
  __device__ __forceinline__ uint32_t pieces() const { return (n + skew + kPer - 1) / kPer; }
  __device__ __forceinline__ bool inside(uint32_t piece) const { return (piece > 0 || skew == 0) && piece < (n + skew) / kPer; }
  __device__ __forceinline__ void unpack(const uint4& w, float* s) const {
    elem e[kPer];
    __builtin_memcpy(e, &w, 16);
#pragma unroll
    for (uint32_t k = 0; k < kPer; ++k) s[k] = V::get(e[k]);
  }
  __device__ __forceinline__ void load(uint32_t piece, bool wanted, float* s) const {     // -infinity if it is not wanted
    if (wanted && inside(piece)) {
      unpack(reinterpret_cast<const uint4*>(base)[piece], s);
    } else if (wanted) {
      load_edge(piece, s);
    } else {
#pragma unroll
      for (uint32_t k = 0; k < kPer; ++k) s[k] = -INFINITY;
    }
  }
  __device__ __forceinline__ void load_edge(uint32_t piece, float* s) const {        // -infinity beyond the row
    const uint32_t at = piece * kPer;
#pragma unroll
    for (uint32_t k = 0; k < kPer; ++k) s[k] = at + k >= skew && at + k < n + skew ? V::get(base[at + k]) : -INFINITY;
  }
};
// visit(index of the first, scores) for the pieces from .. to, left-out elements too, by `threads` lanes of which this is number
// `lane`.  Pieces at the row's ends are a lane's of their own: a branch to them inside the loop would make every load wait for
// the one before.  What a visit computes for all elements before it branches for one runs side by side.
template <int AHEAD, typename V, typename Visit>
__device__ __forceinline__ void for_pieces(const Row<V>& row, uint32_t from, uint32_t to, uint32_t lane, uint32_t threads, Visit visit) {
  constexpr uint32_t per = Row<V>::kPer;
  const uint32_t first = max(from, row.skew ? 1u : 0u), last = min(to, (row.n + row.skew) / per);
  const uint4* pieces = reinterpret_cast<const uint4*>(row.base);
  for (uint32_t p0 = first + lane; p0 < last; p0 += AHEAD * threads) {
    uint4 w[AHEAD];
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) w[e] = pieces[min(p0 + e * threads, last - 1)];
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) {
      if (e > 0 && p0 + e * threads >= last) break;
      float s[per];
      row.unpack(w[e], s);
      visit((p0 + e * threads) * per - row.skew, s);
    }
  }
  const uint32_t edge = lane == 0 ? 0 : row.pieces() - 1;
  if (lane < 2 && (lane == 0 || edge > 0) && edge >= from && edge < to && !row.inside(edge)) {
    float s[per];
    row.load_edge(edge, s);
    visit(edge * per - row.skew, s);
  }
}
// visit(index, score) for those that are not left out
template <int AHEAD, typename V, typename Visit>
__device__ __forceinline__ void for_row(const Row<V>& row, uint32_t from, uint32_t to, uint32_t lane, uint32_t threads, Visit visit) {
  for_pieces<AHEAD>(row, from, to, lane, threads, [&](uint32_t at, const float* s) {
#pragma unroll
    for (uint32_t k = 0; k < Row<V>::kPer; ++k)
      if (s[k] > -INFINITY) visit(at + k, s[k]);
  });
}

// Inclusive sums over the lanes of a wave, by moves inside and between the rows of 16 lanes (an add each, where a shuffle goes
// through LDS: half the time of a histogram's search was shuffles).
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t moved(uint64_t v) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, false);
  return ((uint64_t)hi << 32) | lo;
}
__device__ __forceinline__ uint64_t wave_sums(uint64_t v) {
  v += moved<0x111, 0xf>(v);                   // row_shr:1, 2, 4, 8
  v += moved<0x112, 0xf>(v);
  v += moved<0x114, 0xf>(v);
  v += moved<0x118, 0xf>(v);
  v += moved<0x142, 0xa>(v);                   // row_bcast:15 into rows 1 and 3, row_bcast:31 into rows 2 and 3
  v += moved<0x143, 0xc>(v);
  return v;
}

// Sums of `own` over the workgroup: before this lane, and of all lanes.
__device__ __forceinline__ void block_sums(Shared& sh, const Sum& own, bool weights, Sum& before, Sum& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Sum upto{wave_sums(own.count), 0, 0};
  if (weights) {
    upto.hi = wave_sums(own.hi);
    upto.lo = wave_sums(own.lo);
  }
  if (lane == 63) sh.wave_sum[wave] = upto;
  if (threadIdx.x == 0) sh.found_bin = -1;
  __syncthreads();
  before = upto - own;
  all = Sum{0, 0, 0};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const Sum s = sh.wave_sum[w];
    if (w < wave) before = before + s;
    all = all + s;
  }
}

// The first bin from above at which `reached(sum of everything above and the bin)` holds, into sh.found_*; found_bin -1 if none
// does.  `make_reached` gets the sum of all bins, which is returned.
template <typename MakeReached>
__device__ __forceinline__ Sum find_bin_of(Shared& sh, const Sum& above, bool weights, MakeReached make_reached) {
  constexpr int per = kBins / kThreads;
  const int tid = threadIdx.x;
  Sum own[per], total{0, 0, 0};
#pragma unroll
  for (int k = 0; k < per; ++k) {
    const int b = kBins - 1 - (tid * per + k);
    own[k] = Sum{sh.hist.count[b], weights ? sh.hist.hi[b] : 0, weights ? sh.hist.lo[b] : 0};
    total = total + own[k];
  }
  Sum before, all;
  block_sums(sh, total, weights, before, all);
  before = before + above;
  const auto reached = make_reached(all);
  if (total.count != 0 && reached(before + total) && !reached(before)) {           // one lane
    bool found = false;
#pragma unroll
    for (int k = 0; k < per; ++k) {
      const Sum with = before + own[k];
      if (!found && own[k].count != 0 && reached(with)) {
        found = true;
        sh.found_bin = kBins - 1 - (tid * per + k);
        sh.found_above = before;
        sh.found_in = own[k];
      }
      before = with;
    }
  }
  __syncthreads();
  return all;
}
template <typename Reached>
__device__ __forceinline__ Sum find_bin(Shared& sh, const Sum& above, bool weights, Reached reached) {
  return find_bin_of(sh, above, weights, [=](const Sum&) { return reached; });
}

__device__ __forceinline__ void clear_histogram(Shared& sh, bool weights) {
  for (int b = threadIdx.x; b < kBins; b += kThreads) {
    sh.hist.count[b] = 0;
    if (weights) {
      sh.hist.hi[b] = 0;
      sh.hist.lo[b] = 0;
    }
  }
  __syncthreads();
}

__device__ __forceinline__ Sum sum_of_bins(Shared& sh) {
  const Sum total = find_bin(sh, Sum{0, 0, 0}, true, [](const Sum&) { return false; });
  __syncthreads();
  return total;
}

// ---- the long way: histograms over the whole row down to the cut
template <typename V, typename Bin>
__device__ __forceinline__ void fill_by_key(Shared& sh, const Row<V>& row, uint32_t lo, uint32_t hi, bool weights, const Weigh& weigh, Bin bin) {
  clear_histogram(sh, weights);
  for_row<1>(row, 0, row.pieces(), threadIdx.x, kThreads, [&](uint32_t, float s) {
    const uint32_t key = key_of(s);
    if (key >= lo && key <= hi) add_to(sh.hist, bin(key, s), weights, weights ? weigh(s) : 0.0);
  });
  __syncthreads();
}

// From the bin that find_bin left (of the histogram over `steps`) down to a single key.  false: no cut, everything is kept.
template <typename V, typename Reached>
__device__ __forceinline__ bool narrow(Shared& sh, const Row<V>& row, const Steps& steps, uint32_t kmin, uint32_t kmax, bool weights,
                       const Weigh& weigh, Reached reached, uint32_t& cut, Sum& above, Sum& in) {
  if (sh.found_bin < 0) return false;
  uint32_t lo, hi;
  keys_of_steps(steps, sh.found_bin, sh.found_bin, kmin, kmax, lo, hi);
  above = sh.found_above;
  in = sh.found_in;
  __syncthreads();
  while (lo < hi) {
    const int bits = 32 - __clz(hi - lo);
    const int shift = bits > 11 ? bits - 11 : 0;
    const uint32_t from = lo;
    fill_by_key(sh, row, lo, hi, weights, weigh, [=](uint32_t key, float) { return (int)((key - from) >> shift); });
    find_bin(sh, above, weights, reached);
    const int b = sh.found_bin;                // the bins' sums add up to the interval's: one of them reaches what it did
    above = sh.found_above;
    in = sh.found_in;
    lo = from + ((uint32_t)b << shift);
    hi = min(hi, lo + ((1u << shift) - 1u));
    __syncthreads();
  }
  cut = lo;
  return true;
}

struct Cut {                                   // kept: keys above, and equal ones up to the index last_tie
  uint32_t key, last_tie;
};

// ties i = 0, 1, .. of weight e stay while  above + i * e < target, at least one and at most `most` of them
__device__ __forceinline__ uint64_t ties_below(double above, double e, double target, uint64_t most) {
  uint64_t stay = e > 0.0 ? (uint64_t)fmin(fmax(ceil((target - above) / e), 1.0), (double)most) : most;
  while (stay > 1 && above + (double)(stay - 1) * e >= target) --stay;
  while (stay < most && above + (double)stay * e < target) ++stay;
  return stay;
}

// WAVES: of the kernel that calls it, per SIMD.  One body for two kernels would take the registers of the one that may have more,
// and the other one with it.
template <int WAVES, typename V>
__device__ __noinline__ void cut_the_long_way(Shared& sh, const Row<V>& row, uint32_t kmin, uint32_t kmax, const Weigh& weigh, const RowLimits& limits, Cut& cut) {
  const Steps steps(kmin, kmax);
  uint64_t ties = 0;
  bool all_ties = true;
  double whole = 0.0;
  for (int by_p = limits.by_k ? 0 : 1; by_p <= (limits.by_p ? 1 : 0); ++by_p) {
    fill_by_key(sh, row, kmin, kmax, limits.by_p, weigh, [=](uint32_t, float s) { return steps(s); });
    if (by_p && (!limits.by_k || cut.key == 0)) whole = sum_of_bins(sh).value();     // top-k, if any, keeps everything
    const double target = (double)limits.top_p * whole;
    const uint64_t k = (uint64_t)limits.k;
    const bool first_alone = by_p && !(limits.top_p > 0.0f);
    auto reached = [=](const Sum& s) { return first_alone ? s.count >= 1 : by_p ? s.value() >= target : s.count >= k; };
    find_bin(sh, Sum{0, 0, 0}, limits.by_p, reached);
    uint32_t key;
    Sum above, in;
    if (!narrow(sh, row, steps, kmin, kmax, limits.by_p, weigh, reached, key, above, in) || key < cut.key) continue;
    if (by_p) {
      const uint64_t most = key == cut.key && !all_ties ? ties : in.count;
      ties = first_alone ? 1 : ties_below(above.value(), weigh(score_of(key)), target, most);
    } else {
      ties = k - above.count;
      whole = above.value() + (double)ties * weigh(score_of(key));
    }
    cut.key = key;
    all_ties = ties == in.count;
  }
  if (all_ties) return;
  // equal keys stay from the lowest index on: which index is the last of them?
  auto reached = [=](const Sum& s) { return s.count >= ties; };
  uint32_t lo = 0, hi = row.n - 1;             // bins go down with the index: find_bin begins above
  Sum above{0, 0, 0};
  while (lo < hi) {
    const int bits = 32 - __clz(hi - lo);
    const int shift = bits > 11 ? bits - 11 : 0;
    clear_histogram(sh, false);
    for_row<1>(row, 0, row.pieces(), threadIdx.x, kThreads, [&](uint32_t at, float s) {
      if (key_of(s) == cut.key && at >= lo && at <= hi) atomicAdd(&sh.hist.count[kBins - 1 - ((at - lo) >> shift)], 1u);
    });
    __syncthreads();
    find_bin(sh, above, false, reached);
    const int b = kBins - 1 - sh.found_bin;
    above = sh.found_above;
    lo = lo + ((uint32_t)b << shift);
    hi = min(hi, lo + ((1u << shift) - 1u));
    __syncthreads();
  }
  cut.last_tie = lo;
}

__device__ __forceinline__ double kept_weight(uint32_t key, uint32_t at, const Cut& cut, double min_p, const Weigh& weigh) {
  if (key < cut.key || (key == cut.key && at > cut.last_tie)) return 0.0;
  const double e = weigh(score_of(key));
  return min_p > 0.0 && !(e >= min_p) ? 0.0 : e;
}

// The bin (of a histogram whose bins go down with the index) that the random number falls into; `total`, of all weights, is what
// the bins add up to if it is not known yet.  Past every weight there is: the last that has any.
__device__ __forceinline__ uint32_t find_answer(Shared& sh, const Sum& above, Sum& total, double u) {
  const bool known = total.count != 0;
  const Sum given = total;
  const Sum bins = find_bin_of(sh, above, true, [=](const Sum& sum) {
    const Sum all = known ? given : sum;
    const double target = u * all.value();
    return [=](const Sum& s) { return s.value() > target || s.same_weight(all); };
  });
  if (!known) total = bins;
  return kBins - 1 - sh.found_bin;
}
__device__ __forceinline__ void answer(const SampleArgs& a, int64_t r, uint32_t at, const Sum& in, const Sum& total) {
  if (threadIdx.x != 0) return;
  a.ids[r] = (int32_t)at;
  if (a.probs) a.probs[r] = (float)(in.value() / total.value());
}

// The answer among the indices [lo, hi] of the row, of which `above` lies in front, of `total` in all (none: to be found).
template <typename V>
__device__ __forceinline__ void choose_index(Shared& sh, const Row<V>& row, uint32_t lo, uint32_t hi, Sum above, Sum total, const Cut& cut,
                             const Weigh& weigh, const RowLimits& limits, const SampleArgs& a, int64_t r) {
  while (true) {
    const int bits = lo < hi ? 32 - __clz(hi - lo) : 0;
    const int shift = bits > 11 ? bits - 11 : 0;
    clear_histogram(sh, true);
    const uint32_t from = (lo + row.skew) / Row<V>::kPer, to = (hi + row.skew) / Row<V>::kPer + 1;
    for_pieces<1>(row, from, to, threadIdx.x, kThreads, [&](uint32_t at, const float* s) {
      constexpr uint32_t per = Row<V>::kPer;
      Units w[per];
#pragma unroll
      for (uint32_t k = 0; k < per; ++k) {
        const uint32_t key = key_of(s[k]);
        const double e = weigh(s[k]);
        const bool kept = s[k] > -INFINITY && at + k >= lo && at + k <= hi && (key > cut.key || (key == cut.key && at + k <= cut.last_tie)) &&
                          !(limits.min_p > 0.0 && !(e >= limits.min_p));
        w[k] = units_of(kept ? e : 0.0);
      }
      if ((1u << shift) < per) {
#pragma unroll
        for (uint32_t k = 0; k < per; ++k) add_units(sh.hist, kBins - 1 - (int)((at + k - lo) >> shift), w[k].hi, w[k].lo);
      } else {                                 // a piece reaches into two bins at most: neighbouring lanes would add to them one by one
        const uint32_t b0 = (uint32_t)max((int32_t)at - (int32_t)lo, 0) >> shift;
        uint64_t hi2[2] = {0, 0}, lo2[2] = {0, 0};
#pragma unroll
        for (uint32_t k = 0; k < per; ++k) {
          const bool next = (at + k - lo) >> shift != b0;
          hi2[0] += next ? 0 : w[k].hi;
          lo2[0] += next ? 0 : w[k].lo;
          hi2[1] += next ? w[k].hi : 0;
          lo2[1] += next ? w[k].lo : 0;
        }
        add_units(sh.hist, kBins - 1 - (int)b0, hi2[0], lo2[0]);
        add_units(sh.hist, kBins - 2 - (int)b0, hi2[1], lo2[1]);
      }
    });
    __syncthreads();
    const uint32_t b = find_answer(sh, above, total, limits.u);
    above = sh.found_above;
    const Sum in = sh.found_in;
    lo = lo + (b << shift);
    hi = min(hi, lo + ((1u << shift) - 1u));
    __syncthreads();
    if (shift == 0) {
      answer(a, r, lo, in, total);
      return;
    }
  }
}

// ---- the list
__device__ __forceinline__ uint64_t entry_of(uint32_t key, uint32_t at) { return ((uint64_t)~key << 32) | at; }
__device__ __forceinline__ uint32_t entry_key(uint64_t e) { return ~(uint32_t)(e >> 32); }

__device__ __forceinline__ void put_entry(ListShared& sh, uint32_t key, uint32_t at) {
  const uint32_t p = atomicAdd(&sh.list_count, 1u);
  if (p < (uint32_t)kListMost) sh.list[p] = entry_of(key, at);     // always: the histogram has counted them
}

// Bitonic sort of sh.list[0 .. size), ascending; size a power of two and at least 4.  A pass takes two strides: four entries per
// lane, once through LDS.  Passes over blocks of at most 256 entries stay in a wave.
__device__ __forceinline__ void order(uint64_t& x, uint64_t& y, bool up) {
  const bool turn = (x > y) == up;
  const uint64_t a = turn ? y : x, b = turn ? x : y;
  x = a;
  y = b;
}
__device__ __forceinline__ void sort_list(ListShared& sh, uint32_t size) {
  __syncthreads();
  for (uint32_t block = 2; block <= size; block <<= 1) {
    uint32_t stride = block >> 1;
    if (__popc(block - 1) & 1) {               // an odd number of strides: the first alone
      for (uint32_t t = threadIdx.x; t < size / 2; t += kThreads) {
        const uint32_t i = ((t & ~(stride - 1)) << 1) | (t & (stride - 1));
        uint64_t x = sh.list[i], y = sh.list[i + stride];
        order(x, y, (i & block) == 0);
        sh.list[i] = x;
        sh.list[i + stride] = y;
      }
      __syncthreads();                         // the next pass deals the entries to other lanes
      stride >>= 1;
    }
    for (; stride >= 2; stride >>= 2) {
      const uint32_t h = stride >> 1;
      for (uint32_t t = threadIdx.x; t < size / 4; t += kThreads) {
        const uint32_t i = ((t & ~(h - 1)) << 2) | (t & (h - 1));
        const bool up = (i & block) == 0;
        uint64_t x0 = sh.list[i], x1 = sh.list[i + h], x2 = sh.list[i + stride], x3 = sh.list[i + stride + h];
        order(x0, x2, up);
        order(x1, x3, up);
        order(x0, x1, up);
        order(x2, x3, up);
        sh.list[i] = x0;
        sh.list[i + h] = x1;
        sh.list[i + stride] = x2;
        sh.list[i + stride + h] = x3;
      }
      if (stride > 128 || stride <= 3) __syncthreads();
      else wave_fence();
    }
  }
  __syncthreads();
}
// pads to a power of two (entries that sort last) and sorts
__device__ __forceinline__ void sort_entries(ListShared& sh, uint32_t length) {
  uint32_t size = 4;
  while (size < length) size <<= 1;
  __syncthreads();
  for (uint32_t j = length + threadIdx.x; j < size; j += kThreads) sh.list[j] = ~0ull;
  sort_list(sh, size);
}

// What the first histogram says about a row.
struct Plan {
  bool listed;                                 // there is a cut, and it falls on an entry of the list
  bool long_way;                               // .. which would be too long
  bool pieces;                                 // the weights above the list are added by pieces of the index
  uint32_t lo, hi, length;                     // keys and number of the list's entries
  Sum above;                                   // of the cut's bin
  double whole;                                // sum of all weights, where they were added
};
// The first histogram is in sh.hist (weights only for top-p without top-k).
__device__ __forceinline__ Plan make_plan(Shared& sh, uint32_t kmin, uint32_t kmax, const RowLimits& limits) {
  Plan plan{false, false, true, 1, 0, 0, Sum{0, 0, 0}, 0.0};
  if (!limits.by_k && !limits.by_p) return plan;
  const bool weights = !limits.by_k;
  const double top_p = (double)limits.top_p;
  // top_p <= 0 keeps the first node alone: the bin of the greatest
  const bool by_sum = weights && limits.top_p > 0.0f;
  const uint64_t k = weights ? 1 : (uint64_t)limits.k;
  plan.whole = find_bin_of(sh, Sum{0, 0, 0}, weights, [=](const Sum& all) {
    const double target = top_p * all.value();
    return [=](const Sum& s) { return by_sum ? s.value() >= target : s.count >= k; };
  }).value();
  plan.listed = sh.found_bin >= 0;
  if (plan.listed) {
    plan.above = sh.found_above;
    plan.length = (uint32_t)(sh.found_in.count + (limits.by_k ? sh.found_above.count : 0));
    plan.long_way = plan.length > (uint32_t)kListMost;
    const int bin = sh.found_bin;
    if (!plan.long_way) keys_of_steps(Steps(kmin, kmax), bin, limits.by_k ? kBins - 1 : bin, kmin, kmax, plan.lo, plan.hi);
  } else {
    plan.long_way = limits.by_p;               // fewer nodes than k: by top-p alone, for which no weights were added
  }
  plan.pieces = !plan.long_way && !(plan.listed && limits.by_k);
  __syncthreads();
  return plan;
}

// The first of the sorted entries 0 .. to - 1 at which `reached` holds for the sum of the weights up to it; to - 1 if there is
// none.  make_reached gets the sum of all of them.  `chosen`: that entry's weight, `total`: the sum of all.
template <typename Weight, typename MakeReached>
__device__ __forceinline__ uint32_t place_in_list(Shared& sh, uint32_t to, const Sum& above, Weight weight, MakeReached make_reached,
                                                  Sum& chosen, Sum& total) {
  const uint32_t per = (to + kThreads - 1) / kThreads, from = threadIdx.x * per, end = min(from + per, to);
  Sum own{0, 0, 0};
  for (uint32_t p = from; p < end; ++p) {
    const Units w = units_of(weight(sh.list[p]));
    own = own + Sum{1, w.hi, w.lo};
  }
  Sum before;
  block_sums(sh, own, true, before, total);
  before = before + above;
  const auto reached = make_reached(total);
  if (own.count != 0 && reached(before + own) && !reached(before)) {               // one lane
    for (uint32_t p = from; p < end; ++p) {
      const Units w = units_of(weight(sh.list[p]));
      const Sum in{1, w.hi, w.lo};
      before = before + in;
      if (reached(before)) {
        sh.found_bin = (int)p;
        sh.found_in = in;
        break;
      }
    }
  }
  __syncthreads();
  chosen = sh.found_in;
  return sh.found_bin < 0 ? to - 1 : (uint32_t)sh.found_bin;
}

// The list, sorted, to the cut.
__device__ __forceinline__ void cut_from_list(Shared& sh, const Plan& plan, const RowLimits& limits, const Weigh& weigh, Cut& cut) {
  sort_entries(sh, plan.length);
  uint32_t last = limits.by_k ? min((uint32_t)limits.k, plan.length) - 1 : plan.length - 1;
  if (limits.by_p && !(limits.top_p > 0.0f)) {
    last = 0;
  } else if (limits.by_p) {
    const double top_p = (double)limits.top_p, whole = plan.whole;
    const bool by_k = limits.by_k;
    Sum chosen, total;
    last = place_in_list(sh, last + 1, by_k ? Sum{0, 0, 0} : plan.above, [&](uint64_t x) { return weigh(score_of(entry_key(x))); },
                         [=](const Sum& all) {
                           const double target = top_p * (by_k ? all.value() : whole);
                           return [=](const Sum& s) { return s.value() >= target; };
                         }, chosen, total);
  }
  cut.key = entry_key(sh.list[last]);
  cut.last_tie = (uint32_t)sh.list[last];
}

// With top-k the list holds every node that may be chosen: by index now.
__device__ __forceinline__ void choose_from_list(Shared& sh, const Plan& plan, const Cut& cut, const RowLimits& limits, const Weigh& weigh, const SampleArgs& a, int64_t r) {
  __syncthreads();
  for (uint32_t p = threadIdx.x; p < plan.length; p += kThreads) {
    const uint64_t x = sh.list[p];
    sh.list[p] = (x << 32) | (x >> 32);        // index first
  }
  sort_entries(sh, plan.length);
  const double u = limits.u;
  Sum chosen, total;
  const uint32_t p = place_in_list(sh, plan.length, Sum{0, 0, 0},
                                   [&](uint64_t x) { return kept_weight(~(uint32_t)x, (uint32_t)(x >> 32), cut, limits.min_p, weigh); },
                                   [=](const Sum& all) {
                                     const double target = u * all.value();
                                     return [=](const Sum& s) { return s.value() > target || s.same_weight(all); };
                                   }, chosen, total);
  answer(a, r, (uint32_t)(sh.list[p] >> 32), chosen, total);
}

__device__ __forceinline__ bool answer_without_weights(uint32_t kmax, uint32_t first, const RowLimits& limits, const SampleArgs& a, int64_t r) {
  const bool none = kmax == 0 || !(limits.temperature >= 0.0f);    // nothing may be chosen, or not by this temperature
  if (!none && limits.temperature != 0.0f) return false;
  if (threadIdx.x == 0) {
    a.ids[r] = none ? -1 : (int32_t)first;
    if (a.probs) a.probs[r] = kmax == 0 ? 0.0f : none ? NAN : 1.0f;
  }
  return true;
}

// ---- least and greatest key, and the first index of the greatest (temperature 0)
struct Extreme {
  uint32_t kmin, kmax, first, unused;
  __device__ __forceinline__ void with(uint32_t lo, uint32_t hi, uint32_t at) {
    kmin = min(kmin, lo);
    if (hi > kmax || (hi == kmax && at < first)) {
      kmax = hi;
      first = at;
    }
  }
  __device__ __forceinline__ void over_wave() {
#pragma unroll
    for (int d = 32; d; d >>= 1) with(__shfl_xor(kmin, d, 64), __shfl_xor(kmax, d, 64), __shfl_xor(first, d, 64));
  }
};
// of the pieces from .. to, the same in every lane; the index only where it is asked for, by a second pass
template <typename V>
__device__ __forceinline__ Extreme extreme_of(const Row<V>& row, uint32_t from, uint32_t to, bool want_first) {
  __shared__ Extreme wave_x[2][kWaves];
  float least = INFINITY, most = -INFINITY;
  for_pieces<kAhead>(row, from, to, threadIdx.x, kThreads, [&](uint32_t, const float* s) {
#pragma unroll
    for (uint32_t k = 0; k < Row<V>::kPer; ++k) {
      most = fmaxf(most, s[k]);                // a NaN is neither
      least = fminf(least, s[k] > -INFINITY ? s[k] : INFINITY);
    }
  });
  Extreme x{key_of(least), key_of(most), 0xffffffffu, 0};
  auto over_group = [&](int which) {
    x.over_wave();
    if ((threadIdx.x & 63) == 0) wave_x[which][threadIdx.x >> 6] = x;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) x.with(wave_x[which][w].kmin, wave_x[which][w].kmax, wave_x[which][w].first);
  };
  over_group(0);
  if (want_first) {
    for_row<kAhead>(row, from, to, threadIdx.x, kThreads, [&](uint32_t at, float s) {
      if (key_of(s) == x.kmax) x.first = min(x.first, at);
    });
    over_group(1);
  }
  return x;
}

// The first histogram of the pieces from .. to.
template <typename V>
__device__ __forceinline__ void first_histogram(Histogram& hist, const Row<V>& row, uint32_t from, uint32_t to, const Steps& steps, bool weights, const Weigh& weigh) {
  if (weights)
    for_pieces<1>(row, from, to, threadIdx.x, kThreads, [&](uint32_t, const float* s) {
      int bin[Row<V>::kPer];
      Units w[Row<V>::kPer];
#pragma unroll
      for (uint32_t k = 0; k < Row<V>::kPer; ++k) {
        bin[k] = steps(s[k]);
        w[k] = units_of(weigh(s[k]));
      }
#pragma unroll
      for (uint32_t k = 0; k < Row<V>::kPer; ++k)
        if (s[k] > -INFINITY) {
          atomicAdd(&hist.count[bin[k]], 1u);
          atomicAdd(&hist.hi[bin[k]], (unsigned long long)w[k].hi);
          atomicAdd(&hist.lo[bin[k]], (unsigned long long)w[k].lo);
        }
    });
  else
    for_row<kAhead>(row, from, to, threadIdx.x, kThreads, [&](uint32_t, float s) { atomicAdd(&hist.count[steps(s)], 1u); });
}

// ---- row by row --------------------------------------------------------------------------------------------------------
// Two workgroups per compute unit, as their LDS allows: held to 128 registers the seldom used ways spill, but 4096 rows of 10,000
// take 253 instead of 387 us (every filter) and 255 instead of 284 (none), one row as long as before.  finish_rows_kernel has 256 rows
// or fewer in most calls and would lose 3 us.
template <typename V>
__global__ __launch_bounds__(kThreads, 4) void sample_rows_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const int64_t r = blockIdx.x;
  const Row<V> row(a.scores, r, a.n);
  const RowLimits limits(a, r);
  fill_powers(sh.powers);
  const Extreme x = extreme_of(row, 0, row.pieces(), limits.temperature == 0.0f);
  if (answer_without_weights(x.kmax, x.first, limits, a, r)) return;
  const Weigh weigh(score_of(x.kmax), limits.temperature, sh.powers);
  Cut cut{0, row.n};                           // every valid key lies above 0
  if (limits.by_k || limits.by_p) {
    clear_histogram(sh, true);
    first_histogram(sh.hist, row, 0, row.pieces(), Steps(x.kmin, x.kmax), !limits.by_k, weigh);
    if (threadIdx.x == 0) sh.list_count = 0;
    __syncthreads();
    const Plan plan = make_plan(sh, x.kmin, x.kmax, limits);
    if (plan.long_way) {
      cut_the_long_way<4>(sh, row, x.kmin, x.kmax, weigh, limits, cut);
    } else if (plan.listed) {
      const float lo = score_of(plan.lo), hi = score_of(plan.hi);
      for_row<kAhead>(row, 0, row.pieces(), threadIdx.x, kThreads, [&](uint32_t at, float s) {
        if (s >= lo && s <= hi) put_entry(sh, key_of(s), at);
      });
      cut_from_list(sh, plan, limits, weigh, cut);
      if (limits.by_k) {
        choose_from_list(sh, plan, cut, limits, weigh, a, r);
        return;
      }
    }
  }
  choose_index(sh, row, 0, row.n - 1, Sum{0, 0, 0}, Sum{0, 0, 0}, cut, weigh, limits, a, r);
}

// ---- split ---------------------------------------------------------------------------------------------------------------
struct SplitArgs {
  SampleArgs s;
  int32_t groups;                              // workgroups per row
  uint32_t parts;                              // of the positions of a row, `width` each, at most kBins
  uint32_t width, parts_per_group;
  Extreme* extremes;                           // [rows][groups]
  Histogram* first_hist;                       // [rows]
  unsigned long long* part_hi;                 // [rows][kBins]
  unsigned long long* part_lo;
  Plan* plans;                                 // [rows]
  uint32_t* list_count;                        // [rows]
  uint64_t* lists;                             // [rows][kListMost]
};

__device__ __forceinline__ Extreme row_extreme(const SplitArgs& a, int64_t r) {
  Extreme x{0xffffffffu, 0, 0xffffffffu, 0};
  for (int g = threadIdx.x & 63; g < a.groups; g += 64) {
    const Extreme y = a.extremes[r * a.groups + g];
    x.with(y.kmin, y.kmax, y.first);
  }
  x.over_wave();
  return x;
}
// this workgroup's 16-byte pieces of its row
template <typename V>
__device__ __forceinline__ void group_pieces(const SplitArgs& a, const Row<V>& row, int g, uint32_t& from, uint32_t& to) {
  const uint64_t span = (uint64_t)a.parts_per_group * a.width / Row<V>::kPer;
  from = (uint32_t)min(g * span, (uint64_t)row.pieces());
  to = (uint32_t)min((g + 1) * span, (uint64_t)row.pieces());
}

// first pass; also clears what the next ones add to
template <typename V>
__global__ __launch_bounds__(kThreads) void extremes_kernel(SplitArgs a) {
  const int64_t r = blockIdx.x / a.groups;
  const int g = (int)(blockIdx.x % a.groups);
  uint32_t* words = reinterpret_cast<uint32_t*>(&a.first_hist[r]);
  for (uint32_t w = g * kThreads + threadIdx.x; w < sizeof(Histogram) / 4; w += a.groups * kThreads) words[w] = 0;
  if (g == 0 && threadIdx.x == 0) a.list_count[r] = 0;
  const Row<V> row(a.s.scores, r, a.s.n);
  uint32_t from, to;
  group_pieces(a, row, g, from, to);
  const Extreme x = extreme_of(row, from, to, RowLimits(a.s, r).temperature == 0.0f);
  if (threadIdx.x == 0) a.extremes[blockIdx.x] = x;
}

// second pass: the first histogram.  Weights only for top-p without top-k: with it, the list holds all that top-p may keep.
template <typename V>
__global__ __launch_bounds__(kThreads) void first_histogram_kernel(SplitArgs a) {
  __shared__ Histogram hist;
  __shared__ double powers[kPowers];
  const int64_t r = blockIdx.x / a.groups;
  const int g = (int)(blockIdx.x % a.groups);
  const RowLimits limits(a.s, r);
  const Extreme x = row_extreme(a, r);
  if (x.kmax == 0 || !(limits.temperature > 0.0f) || !(limits.by_k || limits.by_p)) return;
  const bool weights = !limits.by_k;
  fill_powers(powers);
  for (int b = threadIdx.x; b < kBins; b += kThreads) {
    hist.count[b] = 0;
    hist.hi[b] = 0;
    hist.lo[b] = 0;
  }
  __syncthreads();
  const Row<V> row(a.s.scores, r, a.s.n);
  uint32_t from, to;
  group_pieces(a, row, g, from, to);
  first_histogram(hist, row, from, to, Steps(x.kmin, x.kmax), weights, Weigh(score_of(x.kmax), limits.temperature, powers));
  __syncthreads();
  Histogram& sum = a.first_hist[r];
  for (int b = threadIdx.x; b < kBins; b += kThreads) {
    if (hist.count[b] == 0) continue;
    atomicAdd(&sum.count[b], hist.count[b]);
    if (hist.hi[b] != 0) atomicAdd(&sum.hi[b], hist.hi[b]);
    if (hist.lo[b] != 0) atomicAdd(&sum.lo[b], hist.lo[b]);
  }
}

// what it says about each row
__global__ __launch_bounds__(kThreads) void plan_kernel(SplitArgs a) {
  __shared__ Shared sh;
  const int64_t r = blockIdx.x;
  const RowLimits limits(a.s, r);
  const Extreme x = row_extreme(a, r);
  if (x.kmax == 0 || !(limits.temperature > 0.0f)) return;
  if (limits.by_k || limits.by_p) {
    const Histogram& from = a.first_hist[r];
    for (int b = threadIdx.x; b < kBins; b += kThreads) {
      sh.hist.count[b] = from.count[b];
      sh.hist.hi[b] = from.hi[b];
      sh.hist.lo[b] = from.lo[b];
    }
  }
  __syncthreads();
  const Plan plan = make_plan(sh, x.kmin, x.kmax, limits);
  if (threadIdx.x == 0) a.plans[r] = plan;
}

// third pass: the list, gathered in LDS and handed over with one atomic per workgroup, and the weights above it by parts of the
// row, one wave a part.  Few scores lie above a cut (one in six of normal ones at temperature 1, top_p 0.85): a wave gathers them
// in LDS and weighs 64 at a time.
template <typename V>
__global__ __launch_bounds__(kThreads) void collect_kernel(SplitArgs a) {
  __shared__ ListShared sh;
  __shared__ double powers[kPowers];
  __shared__ float sh_above[kWaves][64 * (1 + Row<V>::kPer)];
  const int64_t r = blockIdx.x / a.groups;
  const int g = (int)(blockIdx.x % a.groups);
  const RowLimits limits(a.s, r);
  const Extreme x = row_extreme(a, r);
  if (x.kmax == 0 || !(limits.temperature > 0.0f)) return;
  const Plan& plan = a.plans[r];
  if (plan.long_way) return;
  fill_powers(powers);
  if (threadIdx.x == 0) sh.list_count = 0;
  __syncthreads();
  const float list_lo = score_of(plan.lo), list_hi = score_of(plan.hi);
  const Row<V> row(a.s.scores, r, a.s.n);
  auto to_list = [&](uint32_t at, float s) {
    if (s >= list_lo && s <= list_hi) put_entry(sh, key_of(s), at);
  };
  if (!plan.pieces) {
    uint32_t from, to;
    group_pieces(a, row, g, from, to);
    for_row<kAhead>(row, from, to, threadIdx.x, kThreads, to_list);
  } else {
    const Weigh weigh(score_of(x.kmax), limits.temperature, powers);
    const float floor = plan.listed ? list_hi : -INFINITY;
    const uint32_t last = min(a.parts, (g + 1) * a.parts_per_group);
    const uint32_t span = a.width / Row<V>::kPer;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float* above = sh_above[wave];
    for (uint32_t part = g * a.parts_per_group + wave; part < last; part += kWaves) {
      uint64_t hi = 0, lo = 0;
      auto weigh_one = [&](float s, bool valid) {
        const double w = weigh(s);
        const Units units = units_of(w);
        const bool kept = valid && !(limits.min_p > 0.0 && w < limits.min_p);
        hi += kept ? units.hi : 0;
        lo += kept ? units.lo : 0;
      };
      const uint32_t from = min(part * span, row.pieces()), to = min((part + 1) * span, row.pieces());
      uint32_t waiting = 0;                    // the same in every lane
      for (uint32_t p0 = from; p0 < to; p0 += 64) {
        float s[Row<V>::kPer];
        row.load(p0 + lane, p0 + lane < to, s);
#pragma unroll
        for (uint32_t k = 0; k < Row<V>::kPer; ++k) {
          const uint64_t lanes = __ballot(s[k] > floor);
          if (s[k] > floor) above[waiting + __builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0))] = s[k];
          waiting += (uint32_t)__popcll(lanes);
        }
#pragma unroll
        for (uint32_t k = 0; k < Row<V>::kPer; ++k) to_list((p0 + lane) * Row<V>::kPer + k - row.skew, s[k]);
        wave_fence();
        while (waiting >= 64) {
          waiting -= 64;
          weigh_one(above[waiting + lane], true);
        }
        wave_fence();
      }
      if (waiting > 0) weigh_one(above[min(lane, waiting - 1)], lane < waiting);
      wave_fence();
      hi = wave_sums(hi);
      lo = wave_sums(lo);
      if (lane == 63) {
        a.part_hi[r * kBins + part] = hi;
        a.part_lo[r * kBins + part] = lo;
      }
    }
  }
  __syncthreads();
  const uint32_t count = sh.list_count;
  if (count == 0) return;
  if (threadIdx.x == 0) sh.list_base = atomicAdd(&a.list_count[r], count);
  __syncthreads();
  for (uint32_t j = threadIdx.x; j < count; j += kThreads) a.lists[r * kListMost + sh.list_base + j] = sh.list[j];
}

// one workgroup a row finishes
template <typename V>
__global__ __launch_bounds__(kThreads) void finish_rows_kernel(SplitArgs a) {
  __shared__ Shared sh;
  const int64_t r = blockIdx.x;
  const RowLimits limits(a.s, r);
  const Extreme x = row_extreme(a, r);
  if (answer_without_weights(x.kmax, x.first, limits, a.s, r)) return;
  fill_powers(sh.powers);
  __syncthreads();
  const Weigh weigh(score_of(x.kmax), limits.temperature, sh.powers);
  const Row<V> row(a.s.scores, r, a.s.n);
  const Plan plan = a.plans[r];
  Cut cut{0, row.n};
  uint32_t lo = 0, hi = row.n - 1;
  Sum above{0, 0, 0}, total{0, 0, 0};
  if (plan.long_way) {
    cut_the_long_way<2>(sh, row, x.kmin, x.kmax, weigh, limits, cut);
  } else {
    if (plan.listed) {
      for (uint32_t j = threadIdx.x; j < plan.length; j += kThreads) sh.list[j] = a.lists[r * kListMost + j];
      cut_from_list(sh, plan, limits, weigh, cut);
      if (!plan.pieces) {
        choose_from_list(sh, plan, cut, limits, weigh, a.s, r);
        return;
      }
    }
    // the parts' weights, with what stays of the list, are a histogram along the index
    clear_histogram(sh, true);
    for (uint32_t p = threadIdx.x; p < a.parts; p += kThreads) {
      const uint64_t p_hi = a.part_hi[r * kBins + p], p_lo = a.part_lo[r * kBins + p];
      sh.hist.count[kBins - 1 - p] = (p_hi | p_lo) != 0;
      sh.hist.hi[kBins - 1 - p] = p_hi;
      sh.hist.lo[kBins - 1 - p] = p_lo;
    }
    __syncthreads();
    for (uint32_t j = threadIdx.x; j < plan.length; j += kThreads) {
      const uint32_t at = (uint32_t)sh.list[j];
      const double e = kept_weight(entry_key(sh.list[j]), at, cut, limits.min_p, weigh);
      if (e > 0.0) add_to(sh.hist, kBins - 1 - (int)((at + row.skew) / a.width), true, e);
    }
    __syncthreads();
    const uint32_t part = find_answer(sh, above, total, limits.u);
    above = sh.found_above;
    __syncthreads();
    lo = (uint32_t)max((int64_t)part * a.width - row.skew, (int64_t)0);
    hi = (uint32_t)min((int64_t)(part + 1) * a.width - row.skew, (int64_t)row.n) - 1;
  }
  choose_index(sh, row, lo, hi, above, total, cut, weigh, limits, a.s, r);
}

// ---- host ----------------------------------------------------------------------------------------------------------------
// Split where a workgroup per row would leave compute units idle and rows are long enough for several.
int32_t split_groups(int64_t rows, int64_t n) {
  if (rows >= 512 || n < 2 * kSplitLeast) return 1;
  const int64_t many = std::min<int64_t>(kSplitGroups / rows, ceil_div(n, kSplitMany));
  const int64_t few = std::min<int64_t>(kSplitGroups / 2 / rows, ceil_div(n, kSplitLeast));
  return (int32_t)std::max<int64_t>(1, std::max(many, few));
}

SplitArgs plan_split(void* ws, int64_t rows, int64_t n, size_t& bytes) {
  SplitArgs p{};
  p.groups = split_groups(rows, n);
  Carver c(ws);
  if (p.groups > 1) {
    p.width = (uint32_t)(ceil_div(ceil_div(n + 7, kBins), kPartLeast) * kPartLeast);    // 7: the farthest a row begins behind a boundary
    p.parts = (uint32_t)ceil_div(n + 7, p.width);
    p.parts_per_group = (uint32_t)ceil_div(p.parts, p.groups);
    p.extremes = c.take<Extreme>((size_t)rows * p.groups);
    p.first_hist = c.take<Histogram>(rows);
    p.part_hi = c.take<unsigned long long>((size_t)rows * kBins);
    p.part_lo = c.take<unsigned long long>((size_t)rows * kBins);
    p.plans = c.take<Plan>(rows);
    p.list_count = c.take<uint32_t>(rows);
    p.lists = c.take<uint64_t>((size_t)rows * kListMost);
  }
  bytes = std::max<size_t>(c.used, 256);
  return p;
}

template <typename V>
int32_t run_sample(const SampleArgs& a, SplitArgs& p, hipStream_t stream) {
  if (p.groups == 1) {
    sample_rows_kernel<V><<<(unsigned)a.rows, kThreads, 0, stream>>>(a);
    GS_LAUNCH_CHECK();
    return GS_OK;
  }
  p.s = a;
  const unsigned groups = (unsigned)(a.rows * p.groups);
  extremes_kernel<V><<<groups, kThreads, 0, stream>>>(p);
  GS_LAUNCH_CHECK();
  if (a.top_k || a.top_p) {
    first_histogram_kernel<V><<<groups, kThreads, 0, stream>>>(p);
    GS_LAUNCH_CHECK();
  }
  plan_kernel<<<(unsigned)a.rows, kThreads, 0, stream>>>(p);
  GS_LAUNCH_CHECK();
  collect_kernel<V><<<groups, kThreads, 0, stream>>>(p);
  GS_LAUNCH_CHECK();
  finish_rows_kernel<V><<<(unsigned)a.rows, kThreads, 0, stream>>>(p);
  GS_LAUNCH_CHECK();
  return GS_OK;
}

}  // namespace
}  // namespace gs

using namespace gs;

extern "C" size_t gs_sample_scores_workspace_bytes(int64_t rows, int64_t n, int32_t dtype) {
  if (rows < 0 || n < 1 || n > (int64_t)INT32_MAX || (dtype != GS_F32 && dtype != GS_BF16 && dtype != GS_F16)) return 0;
  size_t bytes = 0, most = 0;
  plan_split(nullptr, rows, n, bytes);
  if (rows > 511) plan_split(nullptr, 511, n, most);             // what serves many rows serves fewer
  return std::max(bytes, most);
}

extern "C" int32_t gs_sample_scores(const void* scores, int64_t rows, int64_t n, int32_t dtype, const float* uniforms,
                                    const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                                    int32_t* ids_out, float* probs_out, void* ws, size_t ws_bytes, void* stream_) {
  hipStream_t stream = (hipStream_t)stream_;
  if (rows < 0 || n < 1 || n > (int64_t)INT32_MAX || (dtype != GS_F32 && dtype != GS_BF16 && dtype != GS_F16)) return GS_EINVAL;
  if (rows > 0 && (!scores || !uniforms || !ids_out)) return GS_EINVAL;
  if (!aligned(scores, dtype == GS_F32 ? 4 : 2)) return GS_EINVAL;
  if (!ws || !aligned(ws, 256)) return GS_EINVAL;
  size_t need = 0;
  SplitArgs p = plan_split(ws, rows, n, need);
  if (ws_bytes < need) return GS_EWORKSPACE;
  if (rows >= ((int64_t)1 << 22)) return GS_EOVERFLOW;           // 2^31 lanes, half of what one launch takes
  if (rows == 0) return GS_OK;
  const SampleArgs a{scores, rows, n, uniforms, temperature, top_k, top_p, min_p, ids_out, probs_out};
  if (dtype == GS_F32) return run_sample<ScoreF32>(a, p, stream);
  if (dtype == GS_BF16) return run_sample<ScoreHalf<bf16_t>>(a, p, stream);
  return run_sample<ScoreHalf<f16_t>>(a, p, stream);
}
