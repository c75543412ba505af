// gs_sample_scores: one node per row of scores, by temperature, top-k, top-p and min-p, from given random numbers.
//
//   order: score descending, index ascending among equal scores;  e_j = exp((s_j - max) / temperature) in fp64
//   top-k: the first k;  top-p: those of them with sum of e before < top_p * sum of e;  min-p: e_j >= min_p
//   answer: the smallest index j with  sum_{i <= j, kept} e_i > u * sum_{kept} e
//
// Nothing is sorted.  A score becomes a 32-bit key of the same order; what the first two filters keep is then "keys above a
// cut, and the first `ties` of those equal to it", and a cut is found by histograms: the first over 2048 equal steps of the
// score between the row's least and greatest (scores spread over them; over the bits of a float they would not), the next
// ones over 2048 steps of the key inside the bin that holds the cut, until a bin is a single key.  At most four histograms
// for any 32-bit keys, two for usual scores.  Weights are added as integers (multiples of 2^-62, in two halves of 31 bits), so
// neither the order of the atomics nor the shape of the launch changes a sum; the choice itself adds fp64 weights in a fixed
// order.  Comparisons near a border are why nothing here is fp32: an error of 1e-7 of the sum would move the answer to a
// neighbour for one row in ten at a million nodes.

#include "common.h"

namespace gs {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 2048;
constexpr int kLdsKeys = 24 * 1024;            // keys of a row that fits LDS next to the histogram

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

struct ScoreF32 {
  typedef float elem;
  static __device__ __forceinline__ float get(float x) { return x; }
};
template <typename H>
struct ScoreHalf {
  typedef uint16_t elem;
  static __device__ __forceinline__ float get(uint16_t x) { return H::lo(x); }
};

// 0: left out (-infinity or NaN); otherwise larger keys for larger scores, one key for both zeros
__device__ __forceinline__ uint32_t key_of(float s) {
  if (!(s > -INFINITY)) return 0;
  const uint32_t b = __float_as_uint(s == 0.0f ? 0.0f : s);
  return (b >> 31) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float score_of(uint32_t key) {
  return __uint_as_float((key >> 31) ? (key & 0x7fffffffu) : ~key);
}

struct Weigh {
  float top;
  double inverse;                              // of the temperature
  __device__ __forceinline__ double operator()(uint32_t key) const {
    const float s = score_of(key);
    if (s == top) return 1.0;
    const double d = (double)s - (double)top;
    return d == -INFINITY ? 0.0 : exp(d * inverse);
  }
};

// A sum of weights as integers: hi * 2^31 + lo, in units of 2^-62.
struct Sum {
  uint64_t count, hi, lo;
  __device__ __forceinline__ double value() const {          // rounded once: a larger sum is never a smaller value
    const uint64_t h = hi + (lo >> 31), l = lo & 0x7fffffffu;
    return h < (1ull << 53) ? ((double)h * 0x1p31 + (double)l) * 0x1p-62 : (double)h * 0x1p-31;
  }
};
__device__ __forceinline__ Sum operator+(const Sum& a, const Sum& b) { return Sum{a.count + b.count, a.hi + b.hi, a.lo + b.lo}; }
__device__ __forceinline__ Sum operator-(const Sum& a, const Sum& b) { return Sum{a.count - b.count, a.hi - b.hi, a.lo - b.lo}; }

struct Histogram {
  uint32_t count[kBins];
  unsigned long long hi[kBins], lo[kBins];
};

// 2048 equal steps between the row's least and greatest finite score
struct Steps {
  double least, inverse;
  __device__ __forceinline__ Steps(uint32_t kmin, uint32_t kmax) {
    const double greatest = fmin((double)score_of(kmax), 3.4028234663852886e38);
    least = fmin((double)score_of(kmin), 3.4028234663852886e38);
    inverse = greatest > least ? (kBins - 1) / (greatest - least) : 0.0;
  }
  __device__ __forceinline__ int operator()(uint32_t key) const {
    const double d = fmin((double)score_of(key), 3.4028234663852886e38) - least;
    return (int)fmin(d * inverse, (double)(kBins - 1));
  }
};

struct Cut {                                   // kept: keys above, and the first `ties` of those equal to it
  uint32_t key;
  uint64_t ties;
  bool all_ties;
  Sum above;
};

struct Shared {
  Histogram hist;
  Sum wave_sum[kWaves];
  double wave_weight[kWaves];
  uint64_t wave_index[kWaves];
  Sum found_above, found_in;
  int found_bin;
  uint32_t kmin, kmax;
};

template <typename V>
struct RowSource {
  const typename V::elem* row;
  const uint32_t* keys;                        // LDS copy, or null
  int64_t n;
  __device__ __forceinline__ uint32_t operator()(int64_t j) const { return keys ? keys[j] : key_of(V::get(row[j])); }
};

__device__ __forceinline__ Sum shfl_up_sum(const Sum& s, int d) {
  return Sum{(uint64_t)__shfl_up((unsigned long long)s.count, d, 64), (uint64_t)__shfl_up((unsigned long long)s.hi, d, 64),
             (uint64_t)__shfl_up((unsigned long long)s.lo, d, 64)};
}

// The first bin from above at which `reached(sum of everything above and the bin)` holds; found_bin -1 if none does.
template <typename Reached>
__device__ void find_bin(Shared& sh, const Sum& above, bool weights, Reached reached) {
  constexpr int per = kBins / kThreads;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  Sum own[per], total{0, 0, 0};
#pragma unroll
  for (int k = 0; k < per; ++k) {
    const int b = kBins - 1 - (tid * per + k);
    own[k] = Sum{sh.hist.count[b], weights ? sh.hist.hi[b] : 0, weights ? sh.hist.lo[b] : 0};
    total = total + own[k];
  }
  Sum upto = total;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Sum up = shfl_up_sum(upto, d);
    if (lane >= d) upto = upto + up;
  }
  if (lane == 63) sh.wave_sum[wave] = upto;
  if (tid == 0) sh.found_bin = -1;
  __syncthreads();
  Sum before = above;
  for (int w = 0; w < wave; ++w) before = before + sh.wave_sum[w];
  before = before + (upto - total);
#pragma unroll
  for (int k = 0; k < per; ++k) {
    const Sum with = before + own[k];
    if (own[k].count != 0 && reached(with) && !reached(before)) {
      sh.found_bin = kBins - 1 - (tid * per + k);
      sh.found_above = before;
      sh.found_in = own[k];
    }
    before = with;
  }
  __syncthreads();
}

template <typename Source, typename Bin>
__device__ void fill_histogram(Shared& sh, const Source& source, uint32_t lo, uint32_t hi, bool weights, const Weigh& weigh, Bin bin) {
  for (int b = threadIdx.x; b < kBins; b += kThreads) {
    sh.hist.count[b] = 0;
    if (weights) {
      sh.hist.hi[b] = 0;
      sh.hist.lo[b] = 0;
    }
  }
  __syncthreads();
  for (int64_t j = threadIdx.x; j < source.n; j += kThreads) {
    const uint32_t key = source(j);
    if (key == 0 || key < lo || key > hi) continue;
    const int b = bin(key);
    atomicAdd(&sh.hist.count[b], 1u);
    if (weights) {
      const uint64_t w = (uint64_t)(weigh(key) * 0x1p62);
      if (w) {
        atomicAdd(&sh.hist.hi[b], (unsigned long long)(w >> 31));
        atomicAdd(&sh.hist.lo[b], (unsigned long long)(w & 0x7fffffffu));
      }
    }
  }
  __syncthreads();
}

// From the bin that find_bin left (of the histogram over `steps`) down to a single key.  false: no cut, everything is kept.
template <typename Source, typename Reached>
__device__ bool narrow(Shared& sh, const Source& source, const Steps& steps, uint32_t kmin, uint32_t kmax, bool weights,
                       const Weigh& weigh, Reached reached, uint32_t& cut, Sum& above, Sum& in) {
  if (sh.found_bin < 0) return false;
  const int bin = sh.found_bin;
  uint32_t lo = kmin, hi = kmax;
  {                                            // the keys of that bin: [first with steps >= bin, last with steps <= bin]
    uint32_t a = kmin, b = kmax;
    while (a < b) {
      const uint32_t mid = a + ((b - a) >> 1);
      if (steps(mid) >= bin) b = mid; else a = mid + 1;
    }
    lo = a;
    b = kmax;
    while (a < b) {
      const uint32_t mid = b - ((b - a) >> 1);
      if (steps(mid) <= bin) a = mid; else b = mid - 1;
    }
    hi = a;
  }
  above = sh.found_above;
  in = sh.found_in;
  __syncthreads();
  while (lo < hi) {
    const int bits = 32 - __clz(hi - lo);
    const int shift = bits > 11 ? bits - 11 : 0;
    const uint32_t from = lo;
    fill_histogram(sh, source, lo, hi, weights, weigh, [=](uint32_t key) { return (int)((key - from) >> shift); });
    find_bin(sh, above, weights, reached);
    const int b = sh.found_bin;                // the bin's sums are the interval's: one of them reaches what the interval did
    above = sh.found_above;
    in = sh.found_in;
    lo = from + ((uint32_t)b << shift);
    hi = min(hi, lo + ((1u << shift) - 1u));
    __syncthreads();
  }
  cut = lo;
  return true;
}

__device__ double block_sum(Shared& sh, double v, double* before) {        // total; *before: of the waves in front of this one
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.wave_weight[threadIdx.x >> 6] = v;
  __syncthreads();
  double total = 0.0;
  for (int w = 0; w < kWaves; ++w) {
    if (w == (int)(threadIdx.x >> 6)) *before = total;
    total += sh.wave_weight[w];
  }
  return total;
}

__device__ uint64_t block_min(Shared& sh, uint64_t v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v = min(v, (uint64_t)__shfl_xor((unsigned long long)v, d, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.wave_index[threadIdx.x >> 6] = v;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) v = min(v, sh.wave_index[w]);
  return v;
}

// One row by one workgroup.
template <typename V>
__global__ __launch_bounds__(kThreads) void sample_rows_kernel(SampleArgs a) {
  extern __shared__ uint32_t lds_keys[];
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t r = blockIdx.x;
  const bool copied = a.n <= kLdsKeys;
  RowSource<V> source{static_cast<const typename V::elem*>(a.scores) + r * a.n, nullptr, a.n};
  const float temperature = a.temperature ? a.temperature[r] : 1.0f;
  const int64_t k = a.top_k ? a.top_k[r] : 0;
  const float top_p = a.top_p ? a.top_p[r] : 1.0f;
  const double min_p = a.min_p && a.min_p[r] > 0.0f ? fmin((double)a.min_p[r], 1.0) : 0.0;

  // ---- least and greatest key, and how many nodes may be chosen
  if (tid == 0) {
    sh.kmin = 0xffffffffu;
    sh.kmax = 0;
  }
  __syncthreads();
  uint32_t kmin = 0xffffffffu, kmax = 0;
  for (int64_t j = tid; j < a.n; j += kThreads) {
    const uint32_t key = source(j);
    if (copied) lds_keys[j] = key;
    if (key != 0) {
      kmin = min(kmin, key);
      kmax = max(kmax, key);
    }
  }
  atomicMin(&sh.kmin, kmin);
  atomicMax(&sh.kmax, kmax);
  __syncthreads();
  kmin = sh.kmin;
  kmax = sh.kmax;
  if (copied) source.keys = lds_keys;
  if (kmax == 0 || !(temperature >= 0.0f)) {   // nothing may be chosen, or not by this temperature
    if (tid == 0) {
      a.ids[r] = -1;
      if (a.probs) a.probs[r] = kmax == 0 ? 0.0f : NAN;
    }
    return;
  }
  if (temperature == 0.0f) {
    uint64_t first = ~0ull;
    for (int64_t j = tid; j < a.n; j += kThreads)
      if (source(j) == kmax) {
        first = (uint64_t)j;
        break;
      }
    first = block_min(sh, first);
    if (tid == 0) {
      a.ids[r] = (int32_t)first;
      if (a.probs) a.probs[r] = 1.0f;
    }
    return;
  }
  const Weigh weigh{score_of(kmax), 1.0 / (double)temperature};

  // ---- the cut of top-k and top-p
  const bool by_k = k > 0 && k < a.n, by_p = top_p < 1.0f;
  uint32_t cut = 0;                            // every valid key lies above
  uint64_t ties = 0;
  bool all_ties = true;
  if (by_k || by_p) {
    const Steps steps(kmin, kmax);
    fill_histogram(sh, source, kmin, kmax, by_p, weigh, steps);
    Sum above, in, everything{0, 0, 0};
    double whole = 0.0;
    if (by_p) {
      find_bin(sh, Sum{0, 0, 0}, true, [](const Sum&) { return false; });     // for the sums of the waves alone
      for (int w = 0; w < kWaves; ++w) everything = everything + sh.wave_sum[w];
      whole = everything.value();
      __syncthreads();
    }
    bool narrowed = false;
    if (by_k) {
      auto reached = [=](const Sum& s) { return s.count >= (uint64_t)k; };
      find_bin(sh, Sum{0, 0, 0}, by_p, reached);
      if (narrow(sh, source, steps, kmin, kmax, by_p, weigh, reached, cut, above, in)) {
        ties = (uint64_t)k - above.count;
        all_ties = ties == in.count;
        whole = above.value() + (double)ties * weigh(cut);
        narrowed = true;
      }
    }
    if (by_p && !(top_p > 0.0f)) {
      cut = kmax;
      ties = 1;
      all_ties = false;
    } else if (by_p) {
      const double target = (double)top_p * whole;
      auto reached = [=](const Sum& s) { return s.value() >= target; };
      if (narrowed) fill_histogram(sh, source, kmin, kmax, true, weigh, steps);
      find_bin(sh, Sum{0, 0, 0}, true, reached);
      uint32_t cut_p;
      if (narrow(sh, source, steps, kmin, kmax, true, weigh, reached, cut_p, above, in) && cut_p >= cut) {
        // ties i = 0, 1, .. stay while  above + i * e < target
        const double w = above.value(), e = weigh(cut_p);
        const uint64_t most = cut_p == cut ? min(ties, in.count) : in.count;
        uint64_t stay = e > 0.0 ? (uint64_t)fmin(fmax(ceil((target - w) / e), 1.0), (double)most) : most;
        while (stay > 1 && w + (double)(stay - 1) * e >= target) --stay;
        while (stay < most && w + (double)stay * e < target) ++stay;
        cut = cut_p;
        ties = stay;
        all_ties = stay == in.count;
      }
    }
  }
  // ---- among equal keys the lowest indices stay: where the last of them lies
  int64_t last_tie = a.n;
  if (!all_ties) {
    uint64_t seen = 0;
    for (int64_t j0 = 0; j0 < a.n; j0 += kThreads) {
      const int64_t j = j0 + tid;
      const bool tie = j < a.n && source(j) == cut;
      const uint64_t mask = __ballot(tie);
      __syncthreads();
      if (lane == 0) sh.wave_index[wave] = __popcll(mask);
      __syncthreads();
      uint64_t before = seen, all = seen;
      for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += sh.wave_index[w];
        all += sh.wave_index[w];
      }
      const uint64_t rank = before + __popcll(mask & ((1ull << lane) - 1ull));
      const uint64_t mine = tie && rank + 1 == ties ? (uint64_t)j : ~0ull;
      if (all >= ties) {
        last_tie = (int64_t)block_min(sh, mine);
        break;
      }
      seen = all;
    }
  }
  auto weight_at = [&](int64_t j) {
    const uint32_t key = source(j);
    if (key == 0 || key < cut || (key == cut && j > last_tie)) return 0.0;
    const double e = weigh(key);
    return min_p > 0.0 && !(e >= min_p) ? 0.0 : e;
  };

  // ---- the choice: sixteenths of the range, until it is one element per lane
  int64_t from = 0, to = a.n;
  double base = 0.0, whole = -1.0, target = 0.0;
  while (to - from > kThreads || whole < 0.0) {
    const int64_t part = ((to - from + kWaves - 1) / kWaves + 63) / 64 * 64;
    const int64_t lo = from + wave * part, hi = min(lo + part, to);
    double s = 0.0;
    for (int64_t j = lo + lane; j < hi; j += 64) s += weight_at(j);
    double unused;
    const double total = block_sum(sh, s, &unused);
    if (whole < 0.0) {
      whole = total;
      target = (double)a.uniforms[r] * whole;
    }
    int chosen = -1;
    double before = base, chosen_base = base;
    for (int w = 0; w < kWaves; ++w) {
      const double own = sh.wave_weight[w];
      if (own > 0.0 && (chosen < 0 || !(chosen_base + sh.wave_weight[chosen] > target))) {
        chosen = w;                            // the first that passes the target, or the last that has any weight
        chosen_base = before;
      }
      before += own;
    }
    __syncthreads();
    from = from + (int64_t)max(chosen, 0) * part;
    to = min(from + part, to);
    base = chosen_base;
  }
  const int64_t j = from + tid;
  const double e = j < to ? weight_at(j) : 0.0;
  double upto = e;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double up = __shfl_up(upto, d, 64);
    if (lane >= d) upto += up;
  }
  if (lane == 63) sh.wave_weight[wave] = upto;
  __syncthreads();
  double before = base;
  for (int w = 0; w < wave; ++w) before += sh.wave_weight[w];
  const uint64_t first = block_min(sh, e > 0.0 && before + upto > target ? (uint64_t)j : ~0ull);
  const uint64_t last = ~block_min(sh, e > 0.0 ? ~(uint64_t)j : ~0ull);
  const uint64_t at = first != ~0ull ? first : last;
  if ((uint64_t)j == at && j < to) {
    a.ids[r] = (int32_t)j;
    if (a.probs) a.probs[r] = (float)(e / whole);
  }
}

}  // namespace
}  // namespace gs

using namespace gs;

extern "C" size_t gs_sample_scores_workspace_bytes(int64_t rows, int64_t n, int32_t dtype) {
  if (rows < 0 || n < 1 || n > (int64_t)INT32_MAX || (dtype != GS_F32 && dtype != GS_BF16 && dtype != GS_F16)) return 0;
  return 256;
}

extern "C" int32_t gs_sample_scores(const void* scores, int64_t rows, int64_t n, int32_t dtype, const float* uniforms,
                                    const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                                    int32_t* ids_out, float* probs_out, void* ws, size_t ws_bytes, void* stream_) {
  hipStream_t stream = (hipStream_t)stream_;
  if (rows < 0 || n < 1 || n > (int64_t)INT32_MAX || (dtype != GS_F32 && dtype != GS_BF16 && dtype != GS_F16)) return GS_EINVAL;
  if (rows > 0 && (!scores || !uniforms || !ids_out)) return GS_EINVAL;
  if (!aligned(scores, dtype == GS_F32 ? 4 : 2)) return GS_EINVAL;
  if (!ws || !aligned(ws, 256)) return GS_EINVAL;
  if (ws_bytes < gs_sample_scores_workspace_bytes(rows, n, dtype)) return GS_EWORKSPACE;
  if (rows >= ((int64_t)1 << 22)) return GS_EOVERFLOW;           // 2^32 lanes: more than one launch takes
  if (rows == 0) return GS_OK;
  const SampleArgs a{scores, rows, n, uniforms, temperature, top_k, top_p, min_p, ids_out, probs_out};
  const size_t lds = n <= kLdsKeys ? sizeof(uint32_t) * (size_t)n : 0;
  if (dtype == GS_F32) sample_rows_kernel<ScoreF32><<<(unsigned)rows, kThreads, lds, stream>>>(a);
  else if (dtype == GS_BF16) sample_rows_kernel<ScoreHalf<bf16_t>><<<(unsigned)rows, kThreads, lds, stream>>>(a);
  else sample_rows_kernel<ScoreHalf<f16_t>><<<(unsigned)rows, kThreads, lds, stream>>>(a);
  GS_LAUNCH_CHECK();
  return GS_OK;
}
