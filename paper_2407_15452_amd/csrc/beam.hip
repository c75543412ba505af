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
// many reach it (equal scores), the best is taken out `width` times instead, step after step: four walks on 10,000 nodes of equal scores,
// width 4, take 63 us where random ones take 15, 32 walks on 100,000, width 64, 0.9 ms instead of 47 us, and 256 walks on 5000, width 256, 9.8 ms.
//
// Bound: the weights' arithmetic.  A score costs 26 vector instructions, 18 of them the fp64 weight (a sum in fp32 would be off by more
// than neighbours of different walks are apart): 64 rows of 1,000,000 fp32 scores take 64 us, 4.0 TB/s, 49 of them instructions; reading
// alone takes 42.  256 rows of 100,003 bf16 scores 35 us.  The join is a chain of small steps in one workgroup a group, 6 us for one
// group of four walks on 10,000 nodes (the parts before it 6), 9 to 20 us for many lists.  Rows of up to 4096 scores take a wave each
// where there are 256 rows and more: no barriers in between (4096 rows of 64 fp32 scores 25 us, with a workgroup a row 81; of 1000 scores
// 18 and 72).
//
// gs_beam_reorder: memory.  64 groups of 8 walks with six rows of 32,768 fp32 values each: 131 us, 6.1 TB/s counted as every row read and
// written once (parents repeat, and such rows come from the caches).  A lane moves four pieces of sixteen bytes one after the other (the
// compiler keeps them in LDS between reading and writing, and waits for each); one launch for all states that fit one.  In place a workgroup
// holds a stripe of all rows of a group in LDS between reading and writing: the same case 334 us.

#include "weigh.h"

namespace gs {
namespace {

constexpr int kMostWidth = 256;
constexpr int kPartThreads = 256;
constexpr int kPartList = 2048;                // scores that may reach the bound
constexpr int kJoinList = 2048;
constexpr int kBins = 1024;
constexpr int kCounted = 128;                  // of a list at most, where places are counted; longer ones are sorted
static_assert(kPartThreads >= kMostWidth, "a lane each for the bound");

struct SelectArgs {
  const void* scores;
  int64_t groups, rows, n;
  int32_t beams, width;
  const float* logp;
  const uint8_t* ended;                        // or null
  int32_t parts;                               // of a row
  int64_t part_len;
  uint64_t* keys;                              // [rows][parts][width]: a part's best, in order, and zeros
  float* tops;                                 // [rows][parts]: largest score
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

// The width-th largest of a value of each lane of a wave; 0 if there are fewer than `width` above 0.  Bit by bit: the largest value that
// `width` lanes reach; one vector instruction each.
template <typename K>
__device__ __forceinline__ K wave_bound(K mine, int width) {
  K found = 0;
#pragma unroll
  for (int bit = 8 * (int)sizeof(K) - 1; bit >= 0; --bit) {
    const bool reached = (int)__popcll(__ballot(mine >= (found | (K)1 << bit))) >= width;
    found |= (K)reached << bit;
  }
  return found;
}
// The same of a workgroup, or of 64 of its values, the largest of the lanes alike; `all`: a value for each lane.  Where each value is
// one of many, a lower bound of the width-th largest of all.
template <int THREADS, typename K>
__device__ __forceinline__ K bound_of(K own, int width, K* all) {
  static_assert(THREADS >= kMostWidth, "the width-th of them");
  const int lane = threadIdx.x & 63;
  all[threadIdx.x] = own;
  __syncthreads();
  if (width <= 32) {                           // every wave for itself
    K mine = all[lane];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) mine = max(mine, all[w * 64 + lane]);
    return wave_bound(mine, width);
  }
  // of 256 values; a lane's own one is the largest of the lanes alike
  __shared__ K bound;
  if (threadIdx.x == 0) bound = 0;
  K mine = 0;
  if (threadIdx.x < 256)
#pragma unroll
    for (int w = 0; w < THREADS / 256; ++w) mine = max(mine, all[w * 256 + threadIdx.x]);
  __syncthreads();
  if (threadIdx.x < 256) all[threadIdx.x] = mine;
  __syncthreads();
  int before = 0;
  if (threadIdx.x < 256)
#pragma unroll 16
    for (int t = 0; t < 256; ++t) before += all[t] > mine || (all[t] == mine && t < (int)threadIdx.x);
  if (threadIdx.x < 256 && before == width - 1) bound = mine;
  __syncthreads();
  return bound;
}

// Puts n values (more than 1, room for the next power of two) in falling order, by THREADS lanes: bitonic.  `key` gives a place for an index, `swap`
// exchanges two; a barrier precedes.
template <int THREADS, typename Before, typename Swap>
__device__ __forceinline__ void sort_list(int n, Before before, Swap swap) {
  for (int size = 2; size <= n; size <<= 1)
    for (int step = size >> 1; step > 0; step >>= 1) {
      for (int i = threadIdx.x; i < n / 2; i += THREADS) {
        const int lo = 2 * i - (i & (step - 1)), hi = lo + step;
        const bool falling = (lo & size) == 0;
        if (falling ? before(hi, lo) : before(lo, hi)) swap(lo, hi);
      }
      __syncthreads();
    }
}
__device__ __forceinline__ int power_of_two(int n) { return n <= 1 ? 1 : 1 << (32 - __clz(n - 1)); }

// exp(s - top) as 2^(n / 64) 2^r, r within 1/128: a table of 64 powers, and the series of 2^r to r^4 (the next term is below 4e-14 of
// it).  A copy of the table for each lane of a half wave, so that no two lanes of a read meet in a bank.
// 2^(j / 64), each to the nearest
__device__ const double power_table[kPowers] = {
    0x1.0000000000000p+0, 0x1.02c9a3e778061p+0, 0x1.059b0d3158574p+0, 0x1.0874518759bc8p+0,
    0x1.0b5586cf9890fp+0, 0x1.0e3ec32d3d1a2p+0, 0x1.11301d0125b51p+0, 0x1.1429aaea92de0p+0,
    0x1.172b83c7d517bp+0, 0x1.1a35beb6fcb75p+0, 0x1.1d4873168b9aap+0, 0x1.2063b88628cd6p+0,
    0x1.2387a6e756238p+0, 0x1.26b4565e27cddp+0, 0x1.29e9df51fdee1p+0, 0x1.2d285a6e4030bp+0,
    0x1.306fe0a31b715p+0, 0x1.33c08b26416ffp+0, 0x1.371a7373aa9cbp+0, 0x1.3a7db34e59ff7p+0,
    0x1.3dea64c123422p+0, 0x1.4160a21f72e2ap+0, 0x1.44e086061892dp+0, 0x1.486a2b5c13cd0p+0,
    0x1.4bfdad5362a27p+0, 0x1.4f9b2769d2ca7p+0, 0x1.5342b569d4f82p+0, 0x1.56f4736b527dap+0,
    0x1.5ab07dd485429p+0, 0x1.5e76f15ad2148p+0, 0x1.6247eb03a5585p+0, 0x1.6623882552225p+0,
    0x1.6a09e667f3bcdp+0, 0x1.6dfb23c651a2fp+0, 0x1.71f75e8ec5f74p+0, 0x1.75feb564267c9p+0,
    0x1.7a11473eb0187p+0, 0x1.7e2f336cf4e62p+0, 0x1.82589994cce13p+0, 0x1.868d99b4492edp+0,
    0x1.8ace5422aa0dbp+0, 0x1.8f1ae99157736p+0, 0x1.93737b0cdc5e5p+0, 0x1.97d829fde4e50p+0,
    0x1.9c49182a3f090p+0, 0x1.a0c667b5de565p+0, 0x1.a5503b23e255dp+0, 0x1.a9e6b5579fdbfp+0,
    0x1.ae89f995ad3adp+0, 0x1.b33a2b84f15fbp+0, 0x1.b7f76f2fb5e47p+0, 0x1.bcc1e904bc1d2p+0,
    0x1.c199bdd85529cp+0, 0x1.c67f12e57d14bp+0, 0x1.cb720dcef9069p+0, 0x1.d072d4a07897cp+0,
    0x1.d5818dcfba487p+0, 0x1.da9e603db3285p+0, 0x1.dfc97337b9b5fp+0, 0x1.e502ee78b3ff6p+0,
    0x1.ea4afa2a490dap+0, 0x1.efa1bee615a27p+0, 0x1.f50765b6e4540p+0, 0x1.fa7c1819e90d8p+0,
};
constexpr int kCopies = 32;
struct Powers {
  double of[kPowers][kCopies];
  // by kPartThreads lanes, a quarter of a power's copies each; a barrier follows before the first use
  static __device__ __forceinline__ double mine() { return power_table[threadIdx.x / 4]; }
  __device__ __forceinline__ void fill(double p) {
    static_assert(kPartThreads == 4 * kPowers && kCopies % 8 == 0, "a quarter each");
#pragma unroll
    for (int c = 0; c < kCopies / 4; ++c) of[threadIdx.x / 4][threadIdx.x % 4 * (kCopies / 4) + c] = p;
  }
};
struct WeighBelow {
  double top;
  const double* powers;
  __device__ __forceinline__ WeighBelow(float top_, const Powers& p) : top((double)top_), powers(&p.of[0][threadIdx.x % kCopies]) {}
  // a score left out (-infinity or NaN) weighs 2^-1000, which no sum of weights up to 1 notices
  __device__ __forceinline__ double operator()(float s) const {
    const double y = fmax(((double)s - top) * (kPowers * 1.4426950408889634074), -1000.0 * kPowers);      // in steps of the table
    const double t = y + 0x1.8p52;             // its last bits: the nearest whole number
    const double r = y - (t - 0x1.8p52);
    const int n = __double2loint(t);
    const double power = powers[(n & (kPowers - 1)) * kCopies];
    constexpr double l = 0.69314718055994530942 / kPowers, l2 = l * l, l3 = l2 * l, l4 = l2 * l2;
    double q = fma(r, l4 / 24, l3 / 6);
    q = fma(r, q, l2 / 2);
    q = fma(r, q, l) * r;
    q = fma(power, q, power);                  // 2^-1000 times it is no subnormal: the exponent alone changes
    return __hiloint2double(__double2hiint(q) + (int)((unsigned)(n & -kPowers) << 14), __double2loint(q));
  }
};
static_assert(kPowers == 64, "n / 64 into the exponent: six places down, twenty up");

// 16 bytes of scores as they lie in memory, rows that begin at any element
template <typename V>
struct Raw {
  typedef typename V::elem elem;
  static constexpr int kPer = 16 / (int)sizeof(elem);
  typedef uint32_t loose __attribute__((ext_vector_type(4), aligned(2)));
  loose w;
  __device__ __forceinline__ float operator[](int k) const {
    if constexpr (kPer == 4) return __uint_as_float(w[k]);
    else return V::get_of(w[k / 2], k % 2);
  }
  __device__ __forceinline__ void none() {     // -infinity
    w = (loose){V::kNone, V::kNone, V::kNone, V::kNone};
  }
};

constexpr int kDumped = 32;                    // lanes whose scores are looked through together
template <int LOADS, int TEAM>
struct PartShared {
  Powers powers;
  uint4 dump[TEAM == 64 ? 64 : kDumped][LOADS];      // of a wave: a quarter
  uint8_t dumper[TEAM == 64 ? 64 : kDumped];
  uint32_t dumped[kPartThreads / 64];
  float wave_top[kPartThreads / 64];
  double wave_sum[kPartThreads / 64];
  uint32_t lane_top[kPartThreads];
  uint32_t listed[kPartThreads / 64];
  uint64_t list[kPartList];
  uint64_t wave_best[2][kPartThreads / 64];
};

// Parts of rows, TEAM lanes each: a workgroup, or a wave, which then needs no barrier but the table's.
template <int SCORES, int TEAM>
constexpr int kWavesOf = SCORES >= 64 ? (TEAM == 64 ? 2 : 3) : SCORES >= 32 ? 3 : 4;      // on a SIMD
template <typename V, int LOADS, int TEAM>
__global__ __launch_bounds__(kPartThreads, (kWavesOf<LOADS * Raw<V>::kPer, TEAM>)) void part_kernel(SelectArgs a, int64_t slots) {
  typedef typename V::elem elem;
  constexpr int kPer = Raw<V>::kPer, kWaves = kPartThreads / 64, kList = TEAM == 64 ? kPartList / kWaves : kPartList;
  __shared__ PartShared<LOADS, TEAM> sh;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tid = TEAM == 64 ? lane : (int)threadIdx.x;
  const int64_t slot = TEAM == 64 ? (int64_t)blockIdx.x * kWaves + wave : (int64_t)blockIdx.x;
  auto meet = [&]() {                          // of the team
    if (TEAM == 64) wave_fence();
    else __syncthreads();
  };
  const bool last_few = TEAM == 64 && slot >= slots;      // waves without a part
  const uint32_t row = last_few ? 0 : (uint32_t)slot / (uint32_t)a.parts, part = (uint32_t)slot - row * (uint32_t)a.parts;
  const bool looked_at = !last_few && a.logp[row] > -INFINITY && !(a.ended && a.ended[row]);
  uint64_t* const keys = a.keys + slot * a.width;
  auto none = [&]() {
    if (last_few) return;
    if (tid == 0) a.tops[slot] = -INFINITY, a.sums[slot] = 0.0;
    for (int c = tid; c < a.width; c += TEAM) keys[c] = 0;
  };
  if (TEAM != 64 && !looked_at) return none();
  uint32_t* const listed_at = &sh.listed[TEAM == 64 ? wave : 0];
  uint64_t* const list = sh.list + (TEAM == 64 ? wave * kList : 0);

  const int64_t from = (int64_t)part * a.part_len;
  const int len = looked_at ? (int)min(a.n - from, a.part_len) : 0, whole = len / kPer;      // of 16 bytes
  const elem* base = static_cast<const elem*>(a.scores) + (int64_t)row * a.n + from;
  Raw<V> s[LOADS];
  const double power = Powers::mine();
#pragma unroll
  for (int e = 0; e < LOADS; ++e) {
    if (whole > 0) s[e].w = *reinterpret_cast<const typename Raw<V>::loose*>(base + (int64_t)min(e * TEAM + tid, whole - 1) * kPer);
    else s[e].none();
  }
  uint32_t* const dumped_at = &sh.dumped[TEAM == 64 ? wave : 0];
  if (tid == 0) *listed_at = 0, *dumped_at = 0;
  sh.powers.fill(power);                       // while the scores are under way
  if (len < LOADS * TEAM * kPer)               // a part that ends before
#pragma unroll
    for (int e = 0; e < LOADS; ++e) {
      const int p = e * TEAM + tid;
      if (p >= whole) s[e].none();
      if (p == whole && p * kPer < len) {      // the last few
        elem x[kPer];
        __builtin_memcpy(x, &s[e].w, 16);
#pragma unroll
        for (int k = 0; k < kPer; ++k)
          if (p * kPer + k < len) x[k] = base[(int64_t)p * kPer + k];
        __builtin_memcpy(&s[e].w, x, 16);
      }
    }
  float own = -INFINITY;
#pragma unroll
  for (int e = 0; e < LOADS; ++e)
#pragma unroll
    for (int k = 0; k < kPer; ++k) own = s[e][k] > own ? s[e][k] : own;
  float top = own;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  uint32_t bound;
  if constexpr (TEAM == 64) {
    bound = wave_bound(key_of(own), a.width);
    __syncthreads();                           // the table's
    if (!looked_at) return none();
  } else {
    if (lane == 0) sh.wave_top[wave] = top;
    bound = bound_of<kPartThreads>(key_of(own), a.width, sh.lane_top);      // the barrier inside is also that of tops, table and count
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sh.wave_top[w]);
  }
  if (!(top > -INFINITY)) return none();       // nothing there

  double sum = 0.0;
  if (top < INFINITY) {
    const WeighBelow weigh(top, sh.powers);
#pragma unroll
    for (int e = 0; e < LOADS; ++e)
#pragma unroll
      for (int k = 0; k < kPer; ++k) sum += weigh(s[e][k]);
  } else {                                     // those that share the row's probability
#pragma unroll
    for (int e = 0; e < LOADS; ++e)
#pragma unroll
      for (int k = 0; k < kPer; ++k) sum += s[e][k] == INFINITY ? 1.0 : 0.0;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
  if (TEAM != 64 && lane == 0) sh.wave_sum[wave] = sum;

  const float least = bound ? score_of(bound) : -3.4028234663852886e38f;      // neither -infinity nor NaN reaches it
  auto place_at = [&](int e, int k) { return place_of(key_of(s[e][k]), (uint32_t)(from + (e * TEAM + tid) * kPer + k)); };
  auto take = [&](uint64_t place) {
    const uint32_t to = atomicAdd(listed_at, 1u);
    if (to < (uint32_t)kList) list[to] = place;
  };
  // About `width` lanes have a score that reaches the bound.  These put all of theirs into LDS, and the team looks through them: a
  // branch for each score of each lane would take as long as the weights.
  constexpr int kMost = TEAM == 64 ? 64 / kWaves : kDumped;
  uint4 (*const dump)[LOADS] = sh.dump + (TEAM == 64 ? wave * kMost : 0);
  uint8_t* const dumper = sh.dumper + (TEAM == 64 ? wave * kMost : 0);
  if (own >= least) {
    const uint32_t to = atomicAdd(dumped_at, 1u);
    if (to < (uint32_t)kMost) {
#pragma unroll
      for (int e = 0; e < LOADS; ++e) dump[to][e] = make_uint4(s[e].w.x, s[e].w.y, s[e].w.z, s[e].w.w);
      dumper[to] = (uint8_t)tid;
    }
  }
  meet();
  const int dumped = (int)*dumped_at;
  if (dumped <= kMost) {
    for (int i = tid; i < dumped * LOADS; i += TEAM) {
      const int d = i / LOADS, e = i % LOADS;
      const uint4 w = dump[d][e];
      Raw<V> x;
      x.w = (typename Raw<V>::loose){w.x, w.y, w.z, w.w};
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if (x[k] >= least) take(place_of(key_of(x[k]), (uint32_t)(from + (e * TEAM + dumper[d]) * kPer + k)));
    }
  } else {
#pragma unroll
    for (int e = 0; e < LOADS; ++e)
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if (s[e][k] >= least) take(place_at(e, k));
  }
  meet();
  const int listed = (int)*listed_at;
  for (int c = listed + tid; c < a.width; c += TEAM) keys[c] = 0;
  if (listed <= (TEAM == 64 ? kList : kCounted)) {
    for (int c = tid; c < listed; c += TEAM) {
      const uint64_t place = list[c];
      int before = 0;
#pragma unroll 4
      for (int o = 0; o < listed; ++o) before += list[o] > place;
      if (before < a.width) keys[before] = place;
    }
  } else if (TEAM != 64 && listed <= kList) {
    const int n = power_of_two(listed);
    for (int c = listed + tid; c < n; c += TEAM) list[c] = 0;
    __syncthreads();
    sort_list<TEAM>(n, [&](int i, int j) { return list[i] > list[j]; },
                    [&](int i, int j) {
                      const uint64_t x = list[i];
                      list[i] = list[j], list[j] = x;
                    });
    if (tid < a.width) keys[tid] = list[tid];  // listed > width
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
              const uint64_t place = place_at(e, k);
              if (place < last) best = max(best, place);
            }
      }
      last = wave_most(best);
      if constexpr (TEAM != 64) {
        if (lane == 0) sh.wave_best[taken & 1][wave] = last;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) last = max(last, sh.wave_best[taken & 1][w]);
      }
      if (tid == 0) keys[taken] = last;
    }
  }
  if (tid == 0) {
    if constexpr (TEAM != 64) {
      sum = 0.0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) sum += sh.wave_sum[w];
    }
    a.tops[slot] = top;
    a.sums[slot] = sum;
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

template <int THREADS>
struct JoinShared {
  float top[kMostWidth];                       // by walk of the group
  float logp[kMostWidth];
  double log_sum[kMostWidth];                  // log sum exp(s - top)
  uint8_t state[kMostWidth];                   // 0: no walk, 1: one, 2: one that has ended
  uint64_t lane_top[THREADS];
  uint32_t bins[kBins];
  uint32_t listed;
  int cut;
  uint64_t p[kJoinList], in_row[kJoinList];
  uint32_t row[kJoinList];
  Place wave_best[2][THREADS / 64];
};

// A workgroup a group, of 256 lanes for up to kJoinList candidates and of 1024 beyond: the parts' sums, then the first of all lists.  Of
// many candidates, first those above the width-th largest of the lists' heads, then those from the step up, of a thousand equal ones
// between that and the largest, where the width-th lies.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void join_kernel(SelectArgs a) {
  constexpr bool kMany = THREADS > 256;        // more than kJoinList candidates
  __shared__ JoinShared<THREADS> sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t group = blockIdx.x, first_row = group * a.beams;
  if (tid == 0) sh.listed = 0, sh.cut = 0;
  for (int b = wave; b < a.beams; b += THREADS / 64) {            // a wave adds a row's parts, in a fixed order
    const int64_t slot = (first_row + b) * a.parts;
    const float own = lane < a.parts ? a.tops[slot + lane] : -INFINITY;      // both at once: most rows have no more parts
    const double own_sum = lane < a.parts ? a.sums[slot + lane] : 0.0;
    float top = own;
    for (int part = 64 + lane; part < a.parts; part += 64) top = fmaxf(top, a.tops[slot + part]);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    auto share = [&](double sum, float t) { return t > -INFINITY ? sum * (t == top ? 1.0 : exp((double)t - (double)top)) : 0.0; };
    double sum = share(own_sum, own);
    for (int part = 64 + lane; part < a.parts; part += 64) sum += share(a.sums[slot + part], a.tops[slot + part]);
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

  const int64_t lists = (int64_t)a.beams * a.parts, candidates = lists * a.width;
  const uint64_t* const keys = a.keys + first_row * a.parts * a.width;      // of the group: a candidate each, 0 where there is none
  auto place_of_key = [&](int b, uint64_t key, bool first_of_row) {
    Place c{0, key, (uint32_t)b};
    if (sh.state[b] == 1 && key != 0) {
      const float s = score_of((uint32_t)(key >> 32));
      c.p = key64_of((double)sh.logp[b] + ((s == sh.top[b] ? 0.0 : (double)s - (double)sh.top[b]) - sh.log_sum[b]));
    } else if (sh.state[b] == 2 && first_of_row) {
      c.p = key64_of((double)sh.logp[b]), c.in_row = 0;
    }
    return c;
  };
  auto place_at = [&](int b, int part, int t) {
    return place_of_key(b, keys[((int64_t)b * a.parts + part) * a.width + t], part == 0 && t == 0);
  };
  // visit(candidate) for those of p >= least: a candidate each, or, of many, a list each, most of which end at once (4 groups of 16 walks on
  // 1,000,000 nodes, bf16 scores, width 32: 120 -> 94 us; one of 32 walks on 100,000, width 64: 87 -> 46; from 4 candidates a lane on
  // instead of 8, 8 groups of 8 walks on 100,000 nodes, width 64: 49 -> 77, where most of a list is visited)
  auto for_all = [&](uint64_t least, auto visit) {
    if (!kMany || candidates <= 8 * THREADS) {
      const int per_row = a.parts * a.width;
#pragma unroll 4
      for (int c = tid; c < (int)candidates; c += THREADS) {
        const int b = c / per_row;
        const Place place = place_of_key(b, keys[c], c == b * per_row);
        if (place.p >= least) visit(place);
      }
    } else if constexpr (kMany) {
      for (int64_t l = tid; l < lists; l += THREADS) {
        const int b = (int)(l / a.parts), part = (int)(l - (int64_t)b * a.parts);
        for (int t = 0; t < a.width; ++t) {
          const Place place = place_at(b, part, t);
          if (place.p < least) break;
          visit(place);
        }
      }
    }
  };
  auto take = [&](const Place& c) {
    const uint32_t to = atomicAdd(&sh.listed, 1u);
    if (to < (uint32_t)kJoinList) sh.p[to] = c.p, sh.in_row[to] = c.in_row, sh.row[to] = c.row;
  };
  if (!kMany && candidates <= kCounted) {
    for_all(1, take);
  } else {
    uint64_t own = 0;
    for (int64_t l = tid; l < lists; l += THREADS) {
      const int b = (int)(l / a.parts), part = (int)(l - (int64_t)b * a.parts);
      own = max(own, place_at(b, part, 0).p);
    }
    for (int i = tid; i < kBins; i += THREADS) sh.bins[i] = 0;
    const uint64_t most = wave_most(own);
    if (lane == 0) sh.wave_best[0][wave].p = most;
    const uint64_t least = max(bound_of<THREADS>(own, a.width, sh.lane_top), (uint64_t)1);
    uint64_t largest = 0;
    for (int w = 0; w < THREADS / 64; ++w) largest = max(largest, sh.wave_best[0][w].p);
    // steps between least and largest: every operation is monotone, which is all that a cut needs
    const double low = least > 1 ? value_of(least) : largest ? value_of(largest) - 100.0 : 0.0, range = (largest ? value_of(largest) : 0.0) - low;
    const double per_step = range > 0.0 && range < 1e300 ? (double)(kBins - 1) / range : 0.0;
    auto bin_of = [&](const Place& c) { return (int)fmax(0.0, fmin((value_of(c.p) - low) * per_step, (double)(kBins - 1))); };
    for_all(least, [&](const Place& c) { atomicAdd(&sh.bins[bin_of(c)], 1u); });
    __syncthreads();
    if (wave == 0) {                           // the last bin from which on there are `width`, or the first
      constexpr int kEach = kBins / 64;
      uint32_t mine = 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) mine += sh.bins[(63 - lane) * kEach + i];      // lane 0: the highest bins
      const uint32_t upto = wave_inclusive(mine, lane);
      const uint64_t enough = __ballot(upto >= (uint32_t)a.width);
      if (enough != 0 && lane == (int)__builtin_ctzll(enough)) {
        uint32_t count = upto - mine;
        int bin = (63 - lane) * kEach + kEach;
        while (count < (uint32_t)a.width) count += sh.bins[--bin];
        sh.cut = bin;
      }
    }
    __syncthreads();
    const int cut = sh.cut;
    for_all(least, [&](const Place& c) {
      if (bin_of(c) >= cut) take(c);
    });
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
  auto at = [&](int i) { return Place{sh.p[i], sh.in_row[i], sh.row[i]}; };
  if (listed <= kCounted) {
    for (int c = tid; c < listed; c += THREADS) {
      const Place own = at(c);
      int before = 0;
#pragma unroll 4
      for (int o = 0; o < listed; ++o) {       // without branches: equal ones are common among 16-bit scores
        const uint64_t p = sh.p[o], in_row = sh.in_row[o];
        const uint32_t row = sh.row[o];
        before += (p > own.p) | ((p == own.p) & ((row < own.row) | ((row == own.row) & (in_row > own.in_row))));
      }
      if (before < a.width) write(before, own);
    }
    for (int c = listed + tid; c < a.width; c += THREADS) write(c, Place{0, 0, 0});
    return;
  }
  if (!kMany || listed <= kJoinList) {
    const int n = power_of_two(listed);
    for (int c = listed + tid; c < n; c += THREADS) sh.p[c] = 0, sh.in_row[c] = 0, sh.row[c] = 0;
    __syncthreads();
    sort_list<THREADS>(n, [&](int i, int j) { return sh.p[i] > sh.p[j] || (sh.p[i] == sh.p[j] && at(i).before(at(j))); },
                       [&](int i, int j) {
                         const Place x = at(i);
                         sh.p[i] = sh.p[j], sh.in_row[i] = sh.in_row[j], sh.row[i] = sh.row[j];
                         sh.p[j] = x.p, sh.in_row[j] = x.in_row, sh.row[j] = x.row;
                       });
    for (int c = tid; c < a.width; c += THREADS) write(c, c < listed ? at(c) : Place{0, 0, 0});
    return;
  }
  if constexpr (kMany) {
    // The best is taken out `width` times; a lane looks again through its own lists only where it was its own.
    Place last{~0ull, ~0ull, 0}, best = last;
    for (int taken = 0; taken < a.width; ++taken) {
      if (!last.before(best)) {
        best = Place{0, 0, 0};
        for (int64_t l = tid; l < lists; l += THREADS) {
          const int b = (int)(l / a.parts), part = (int)(l - (int64_t)b * a.parts);
          for (int t = 0; t < a.width; ++t) {
            const Place c = place_at(b, part, t);
            if (c.p == 0) break;
            if (!last.before(c)) continue;
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
      for (int w = 1; w < THREADS / 64; ++w)
        if (sh.wave_best[taken & 1][w].before(last)) last = sh.wave_best[taken & 1][w];
      if (tid == 0) write(taken, last);
    }
  }
}

struct SelectPlan {
  int loads, team;
  int32_t parts;
  int64_t part_len;
  uint64_t* keys;
  float* tops;
  double* sums;
  size_t bytes;
};

SelectPlan plan_select(void* ws, int64_t groups, int32_t beams, int64_t n, int32_t width, int32_t dtype) {
  SelectPlan p{};
  const int64_t per = dtype == GS_F32 ? 4 : 8, rows = groups * beams;
  // Few rows: parts small enough that every compute unit has one.
  const int most = dtype == GS_F32 ? 16 : 8;                      // 64 scores a lane
  p.team = n <= 64 * per * most && width <= 32 && rows >= 256 ? 64 : kPartThreads;      // short rows: a wave each
  p.loads = most;
  if (p.team == 64) {
    while (p.loads > 2 && n <= 64 * per * p.loads / 2) p.loads /= 2;
  } else {
    while (p.loads > 2 && rows * ceil_div(n, per * kPartThreads * p.loads) < 512) p.loads /= 2;
  }
  p.part_len = per * p.team * p.loads;
  p.parts = (int32_t)ceil_div(n, p.part_len);
  Carver carve(ws);
  p.keys = carve.take<uint64_t>((size_t)rows * p.parts * width);
  p.tops = carve.take<float>((size_t)rows * p.parts);
  p.sums = carve.take<double>((size_t)rows * p.parts);
  p.bytes = carve.used;
  return p;
}

bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a_bytes > 0 && b_bytes > 0 && x < y + (uintptr_t)b_bytes && y < x + (uintptr_t)a_bytes;
}
bool dtype_known(int32_t dtype) { return dtype == GS_F32 || dtype == GS_BF16 || dtype == GS_F16; }
constexpr int64_t kMostRows = ((int64_t)1 << 22) - 1;
// before the products that they bound
bool select_shape_ok(int64_t groups, int32_t beams, int64_t n, int32_t width, int32_t dtype) {
  return groups >= 0 && groups <= (int64_t)INT32_MAX && beams >= 1 && beams <= kMostWidth && width >= 1 && width <= kMostWidth && n >= 1 &&
         n <= (int64_t)INT32_MAX && dtype_known(dtype);
}

template <typename V, int TEAM>
void launch_parts(const SelectArgs& a, int loads, int64_t slots, hipStream_t s) {
  const dim3 grid((unsigned)ceil_div(slots, kPartThreads / TEAM));
  if (sizeof(typename V::elem) == 4 && loads == 16) part_kernel<V, sizeof(typename V::elem) == 4 ? 16 : 8, TEAM><<<grid, kPartThreads, 0, s>>>(a, slots);
  if (loads == 8) part_kernel<V, 8, TEAM><<<grid, kPartThreads, 0, s>>>(a, slots);
  if (loads == 4) part_kernel<V, 4, TEAM><<<grid, kPartThreads, 0, s>>>(a, slots);
  if (loads == 2) part_kernel<V, 2, TEAM><<<grid, kPartThreads, 0, s>>>(a, slots);
}
template <typename V>
void launch_parts(const SelectArgs& a, const SelectPlan& p, int64_t slots, hipStream_t s) {
  if (p.team == 64) launch_parts<V, 64>(a, p.loads, slots, s);
  else launch_parts<V, kPartThreads>(a, p.loads, slots, s);
}

}  // namespace

// ---- gs_beam_reorder ----------------------------------------------------------
namespace {

constexpr int kCopyThreads = 256;
constexpr int kStates = 64;                    // of one launch
constexpr int64_t kMostBlocks = (((int64_t)1 << 32) - 1) / kCopyThreads;       // of one launch: fewer than 2^32 lanes
constexpr int kAhead = 4;                      // pieces of a lane in flight
constexpr int kStripe = 4096;                  // pieces of a group that a workgroup holds, in place

struct ReorderArgs {
  struct State {
    const char* data;
    char* out;
    int64_t row_bytes, append_at;
    int32_t piece;                             // bytes: 16, 4 or 1
    int32_t first;                             // workgroup of the launch
    int64_t before;                            // workgroups of the state in earlier launches
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
  const int64_t at = (int64_t)blockIdx.x - st.first + st.before;
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
  const int64_t slots = groups * beams * p.parts;
  if (ceil_div(slots, kPartThreads / p.team) * kPartThreads >= (int64_t)1 << 32) return GS_EOVERFLOW;      // a launch takes fewer lanes
  // a group's workgroup reads its walks before it writes: those alone where both begin alike
  if (!(logp_out == logp && width == beams) && overlap(logp_out, groups * width * 4, logp, groups * beams * 4)) return GS_EINVAL;
  const SelectArgs a{scores, groups, groups * beams, n, beams, width, logp, ended, p.parts, p.part_len, p.keys, p.tops, p.sums, parents_out,
                     nodes_out, logp_out};
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == GS_F32) launch_parts<ScoreF32>(a, p, slots, s);
  if (dtype == GS_BF16) launch_parts<ScoreHalf<bf16_t>>(a, p, slots, s);
  if (dtype == GS_F16) launch_parts<ScoreHalf<f16_t>>(a, p, slots, s);
  GS_LAUNCH_CHECK();
  // of many candidates a group's lists take a large workgroup less time (8 groups of 8 walks on 1,000,000 nodes, width 8: 85 -> 80 us)
  if ((int64_t)beams * p.parts * width > kJoinList) join_kernel<1024><<<dim3((unsigned)groups), 1024, 0, s>>>(a);
  else join_kernel<256><<<dim3((unsigned)groups), 256, 0, s>>>(a);
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
    if (x.row_bytes < 0 || x.row_bytes >= ((int64_t)1 << 40) || (in_place && beams != width && x.row_bytes > 0 && groups > 0))
      return GS_EINVAL;
    if (x.row_bytes > 0 && groups > 0 && !x.data) return GS_EINVAL;
    if (x.append_at < -1 || (x.append_at >= 0 && (x.append_at % 4 != 0 || x.append_at + 4 > x.row_bytes || x.row_bytes % 4 != 0 || (groups > 0 && !nodes) ||
                                                  !aligned(x.data, 4) || !aligned(x.out, 4))))
      return GS_EINVAL;
  }
  for (int i = 0; i < num_states; ++i)         // what is written overlaps nothing else
    for (int j = 0; j < num_states; ++j) {
      const gs_state &x = list[i], &y = list[j];
      const bool in_place = !x.out || x.out == x.data, other_in_place = !y.out || y.out == y.data;
      const void* out = in_place ? x.data : x.out;
      if (j == 0 && (overlap(out, rows_out * x.row_bytes, parents, rows_out * 4) || overlap(out, rows_out * x.row_bytes, nodes, nodes ? rows_out * 4 : 0)))
        return GS_EINVAL;
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
      const int64_t pieces = x.row_bytes / piece, all = in_place ? move_blocks(pieces, groups, beams) : copy_blocks(pieces, rows_out);
      for (int64_t done = 0; done < all;) {    // what a launch has no room for goes to the next: workgroups share nothing
        if (a.num_states == kStates || blocks == kMostBlocks) {
          const int32_t rc = launch();
          if (rc != GS_OK) return rc;
        }
        const int64_t now = std::min(all - done, kMostBlocks - blocks);
        a.state[a.num_states++] =
            ReorderArgs::State{static_cast<const char*>(x.data), static_cast<char*>(out), x.row_bytes, x.append_at, piece, (int32_t)blocks, done};
        blocks += now, done += now;
      }
    }
    const int32_t rc = launch();
    if (rc != GS_OK) return rc;
  }
  return GS_OK;
}
