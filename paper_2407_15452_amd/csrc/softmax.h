// gs_softmax_loss, gs_scores: skip-gram's softmax over every node.
//
//   z_ij = scale * <h_i, c_j> + bias_j,   h_i = w_in[centers[i]],  c_j = w_out[j]
//   loss_i = log sum_j exp(z_ij) - z_it,  t = contexts[i]
//   g_in[i]  = grad_scale * scale * (sum_j p_ij c_j - c_t),      p_ij = exp(z_ij) / sum_j exp(z_ij)
//   g_out[j] = grad_scale * scale * sum_i (p_ij - [t_i = j]) h_i
//
// The pairs x nodes matrices z and p are never stored.  One kernel shape does both directions.  A wave keeps 32 or 64 rows of
// one operand in registers, as the right operand of the matrix instructions; the four waves of a workgroup stream the rows of
// the other one through LDS.  A 32 x 32 block of products comes out with the kept rows across the lanes and the streamed rows
// in the registers of a lane, so that a kept row's softmax statistics belong to its lane, and the block, once it is
// probabilities, is the right operand of the second product without leaving the registers: the matrix instruction sums over
// any numbering of its inner dimension, as long as both operands use the same one.  The left operand of the second product is
// the streamed tile again, transposed on its way out of LDS (16-bit tables: ds_read_b64_tr_b16; fp32: one column per lane).
//   forward: pairs kept, nodes streamed, running maximum and sum over the nodes but the context; gives the loss, 1 - p_it and
//     sum_{j != t} p_ij c_j in one pass (16-bit tables: also the sum of the probabilities as they are rounded).
//   table gradient: nodes kept, pairs streamed, p from the forward pass's log-sum; no atomics, each row of g_out has one owner.
// Where the kept rows alone do not fill the chip the streamed ones are split, and a small kernel joins the parts in order.
//
// Precision: the second products of 16-bit tables take the probabilities rounded to the tables' format, as the matrix instructions
// do; sums are fp32.  Probabilities in two parts of the format would cost a half more of these products.  The results are rounded
// to the same format, which hides most of it: relative error of g_in 1.01 to 1.04 times that of fp32 probabilities, of g_out 1.02 to
// 1.18 times (128 columns, 8 to 2000 pairs on 64 to 1000 nodes; g_out of 2000 pairs on 1000: bf16 1.78e-3 instead of 1.67e-3, fp16
// 2.38e-4 instead of 2.08e-4), at most sqrt(2) times, of a single term; of 777 pairs on 20,000 nodes 1.00 and 1.03 times.
//
// Bound: the matrix instructions, from some hundred pairs on.  4096 pairs on 1 M bf16 nodes of 128 columns: forward 1.83 ms, table
// gradient 1.76 ms, 1.15 and 1.19 PFLOP/s (library products of 8192^3 and 16384^3 on that card: 1.16 and 1.38); 65,536 pairs on
// 10,000 fp32 nodes of 64 columns: 1.27 and 1.42 ms, 132 and 119 TFLOP/s (library: 153).  Few pairs, a tile of 64 computed whole: the
// loss alone of 16 pairs on 1 M nodes of 128 columns reads bf16 tables at 5.4 TB/s (a large copy: 4.8) and fp32 ones at 2.0; with the
// gradients 0.22 and 0.81 ms, a half and a quarter of the rate at which tables and gradients could be read and written.  Scores of
// many centres: writing them, 4.8 TB/s of 16-bit tables; fp32 rows of 256 columns the products, 115 TFLOP/s.
//
// LDS tiles are written by the loads themselves (16 bytes per lane, one tile ahead).  Such a load puts lane
// l's piece at base + 16 l, so rows cannot be padded; pieces are swapped inside a row instead, by a function of the row that
// the source address undoes.  Rows beyond the table, pieces beyond `dim` and rows of masked nodes (bias -inf) are read as zeros,
// from outside of a buffer load's range or from a piece of zeros: whatever a masked row holds, infinities and NaN included, it
// takes no part.

#pragma once

#include <type_traits>

#include "common.h"

namespace gs {

// One call, checked: what the format's own file launches.
struct SoftmaxCall {
  const void *w_in, *w_out;
  int64_t num_in, num_nodes, num_pairs;
  int32_t dim;
  const int32_t *centers, *contexts;
  const float* bias;
  float scale, grad_scale;
  float* loss;               // null: scores
  void *g_in, *g_out;
  float* scores;
};
enum { kLossOnly = 0, kForward = 1, kTableGrad = 2, kScores = 3 };

// Sizes and places in the workspace (base null: sizes alone).
struct SoftmaxPlan {
  int padded;                // columns of a copied row: dim up to a multiple of 32
  int64_t padded_pairs, pair_tiles, node_tiles;      // workgroups along the kept rows, either way
  int splits, node_splits;                           // parts of the streamed rows
  int64_t tiles_per_split, tiles_per_node_split;
  void* rows;
  int32_t* target;
  float *lse2, *miss, *part_max, *part_rounded, *part_acc;
  double* part_sum;
  size_t bytes;
};
template <typename E>
SoftmaxPlan plan_softmax(void* ws, int64_t num_pairs, int64_t num_nodes, int32_t dim, bool loss, bool grad);
template <typename E>
int32_t run_softmax(const SoftmaxCall& call, const SoftmaxPlan& plan, hipStream_t stream);

struct F32;
struct BF16;
struct F16;

#if defined(GS_SOFTMAX_KERNELS)
namespace {

typedef float acc16 __attribute__((ext_vector_type(16)));
typedef float vec4 __attribute__((ext_vector_type(4)));
typedef float vec2 __attribute__((ext_vector_type(2)));
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef short short8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 hf2 __attribute__((ext_vector_type(2)));
typedef _Float16 hf8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) short4_t lds_short4;

constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.69314718055994530942;
constexpr int kThreads = 256;

// never written: what rows that are masked, or no rows, are read as
__device__ uint4 zero_piece[1];
template <typename E>
__device__ uint4 nan_piece[1] = {{E::kNan, E::kNan, E::kNan, E::kNan}};

__device__ __forceinline__ int64_t tiles_of(int64_t rows, int tile) { return (rows + tile - 1) / tile; }

}  // namespace

// Storage formats.  kShift: the powers of two by which probabilities are scaled before they are rounded to the format (undone
// in fp32 afterwards): binary16 would lose those below 2^-24 otherwise; the scaled ones stay below 2^15.  kForwardShift: the
// same in the forward pass, where they may be 2^kSlack times larger.
struct F32 {
  typedef float elem;
  static constexpr bool kWide = true;
  static constexpr int kShift = 0;
  static constexpr int kForwardShift = 0;
  static constexpr float kSlack = 8.0f;
  static constexpr uint32_t kNan = 0x7fc00000u;
  // zero + 0 w, which is NaN if w holds infinity or NaN
  static __device__ __forceinline__ float add_none(float w, float zero) { return fmaf(w, 0.0f, zero); }
  static __device__ __forceinline__ float load(const float* p) { return *p; }
  static __device__ __forceinline__ void store4(float* p, vec4 v) { *reinterpret_cast<vec4*>(p) = v; }
};
struct BF16 {
  typedef uint16_t elem;
  static constexpr bool kWide = false;
  static constexpr int kShift = 0;
  static constexpr int kForwardShift = 0;
  static constexpr float kSlack = 8.0f;
  static constexpr uint32_t kNan = 0x7fc07fc0u;
  static __device__ __forceinline__ float load(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((vec2){lo, hi}, bf2));
  }
  static __device__ __forceinline__ float add_pair(uint32_t w, float sum) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf2, w), (bf2){(__bf16)1.0f, (__bf16)1.0f}, sum, false);
  }
  static __device__ __forceinline__ float add_none(float w, float zero) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf2, w), (bf2){(__bf16)0.0f, (__bf16)0.0f}, zero, false);
  }
  static __device__ __forceinline__ acc16 mfma(vec4 a, vec4 b, acc16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ void store4(uint16_t* p, vec4 v) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack(v[0], v[1]), pack(v[2], v[3]));
  }
};
struct F16 {
  typedef uint16_t elem;
  static constexpr bool kWide = false;
  static constexpr int kShift = 14;
  static constexpr int kForwardShift = 11;
  static constexpr float kSlack = 4.0f;
  static constexpr uint32_t kNan = 0x7e007e00u;
  static __device__ __forceinline__ float load(const uint16_t* p) { return __half2float(__ushort_as_half(*p)); }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((vec2){lo, hi}, hf2));
  }
  static __device__ __forceinline__ float add_pair(uint32_t w, float sum) {
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(hf2, w), (hf2){(_Float16)1.0f, (_Float16)1.0f}, sum, false);
  }
  static __device__ __forceinline__ float add_none(float w, float zero) {
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(hf2, w), (hf2){(_Float16)0.0f, (_Float16)0.0f}, zero, false);
  }
  static __device__ __forceinline__ acc16 mfma(vec4 a, vec4 b, acc16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(hf8, a), __builtin_bit_cast(hf8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ void store4(uint16_t* p, vec4 v) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack(v[0], v[1]), pack(v[2], v[3]));
  }
};

namespace {

// Tile shapes: kept rows per wave 32 * kNB, streamed rows per tile kTile, rows padded to DP columns, a multiple of 32.
template <typename E, int DP, int MODE>
struct Shape {
  static constexpr int kRowBytes = DP * (int)sizeof(typename E::elem);
  static constexpr int kPieces = kRowBytes / 16;                   // 16-byte pieces of a row: a multiple of 4 (fp32: of 8)
  static constexpr int kPerPiece = 16 / (int)sizeof(typename E::elem);
  static constexpr int kSteps = kPieces / 2;                       // pieces a half wave takes in the first product
  static constexpr int kBlocks = DP / 32;                          // 32-column blocks of the second product
  // Registers: DP / 2 for the sums, DP / 4 (fp32: DP / 2) for the kept rows, 16 for each 32 streamed rows.  Two waves per SIMD, so
  // that one's exponentials run beside the other's matrix instructions, where 256 registers hold that.
  static constexpr int kWaves = MODE != kScores && E::kWide && DP > 192 ? 1 : 2;
  static constexpr int kTile = MODE == kScores || DP > (E::kWide ? 128 : 192) ? 32 : 64;
  static constexpr int kNB = MODE == kScores && !E::kWide && DP <= 128 ? 2 : 1;
  // Scores take their kept rows through LDS in whole tiles where these are longer than 256 bytes, instead of 32 bytes of each of 32
  // rows per load: 16 centres on 1 M nodes, 256 fp32 columns 385 -> 327 us, 256 bf16 columns 131 -> 118, but 64 bf16 columns 33 -> 40.
  static constexpr bool kStaged = MODE == kScores && kRowBytes > 256;
  static constexpr int kKept = 32 * kNB * 4;                       // kept rows per workgroup
  static constexpr int kChunks = kTile * kPieces / 64;             // loads of a wave (1 KB) that make a tile
  static constexpr int kLoads = (kChunks + 3) / 4;                 // per wave
  // pieces that are swapped among each other: as many as keep rows apart that begin at the same banks (64 of 4 bytes)
  static constexpr int kSwapped = kPieces % 16 == 0 ? 16 : kPieces % 8 == 0 ? 8 : 4;
};

// Where a piece lies inside its row.  Reads of the first product take one piece of 32 consecutive rows, those of the second
// four neighbouring pieces of four consecutive rows; both spread over all banks.
template <int SWAPPED>
__device__ __forceinline__ constexpr int swap_of(int row) {
  return SWAPPED == 16 ? (((row & 3) << 2) | ((row >> 2) & 3)) : SWAPPED == 8 ? ((((row >> 1) & 1) << 2) | ((row >> 2) & 3)) : ((row >> 2) & 3);
}

// 16 bytes of a lane into LDS at dst + 16 lane: from its own address, or from a place in a range that is the wave's (pieces
// outside of the range are zeros).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t range_of(const void* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00027000);
}
__device__ __forceinline__ void load_piece_to_lds(__amdgpu_buffer_rsrc_t range, int offset, void* dst) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(range, (__attribute__((address_space(3))) void*)dst, 16, offset, 0, 0, 0);
}
__device__ __forceinline__ void load_piece_to_lds(const void* src, void* dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}
__device__ __forceinline__ void wait_loads_and_barrier() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// what was asked of LDS is there; loads and stores may be under way
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// in a branch that few tiles take: keeps the compiler from doing its work for all of them and selecting
__device__ __forceinline__ void rare() { asm volatile(""); }

// one step of the first product: 16 bytes of a streamed and of a kept row per lane
template <typename E>
__device__ __forceinline__ acc16 step(vec4 a, vec4 b, acc16 c) {
  if constexpr (E::kWide) {
#pragma unroll
    for (int t = 0; t < 4; ++t) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[t], b[t], c, 0, 0, 0);
    return c;
  } else {
    return E::mfma(a, b, c);
  }
}

// ---- the pairs' rows, copied for the table gradient --------------------------------------------------------------------
// 5 to 6 us: the table gradient streams them once per workgroup, which has no room for a centre's id in front of every load.
// rows[i] = w_in[centers[i]], zero-padded to DP columns and to whole tiles; zeros for pairs without gradient (target -1).
template <typename E>
__global__ __launch_bounds__(kThreads) void gather_pairs_kernel(const typename E::elem* w_in, int dim, int padded,
                                                                const int32_t* centers, const int32_t* target,
                                                                int64_t padded_pairs, typename E::elem* rows) {
  constexpr int per = 16 / (int)sizeof(typename E::elem);
  const int pieces = padded / per;
  const int64_t total = padded_pairs * pieces;
  for (int64_t s = (int64_t)blockIdx.x * kThreads + threadIdx.x; s < total; s += (int64_t)gridDim.x * kThreads) {
    const int64_t i = s / pieces;
    const int p = (int)(s - i * pieces);
    uint4 v = make_uint4(0, 0, 0, 0);
    if (target[i] >= 0 && p * per < dim) v = reinterpret_cast<const uint4*>(w_in)[((int64_t)centers[i] * dim + p * per) / per];
    reinterpret_cast<uint4*>(rows)[s] = v;
  }
}

struct StreamArgs {
  const void* kept;          // forward: w_in, through centers; table gradient and scores: w_out
  const void* streamed;      // forward: w_out; table gradient: copies of the pairs' rows; scores: w_in, through centers
  const int32_t* centers;
  int64_t num_in;
  int64_t kept_rows;         // pairs or nodes
  int64_t streamed_rows;
  int32_t dim;
  float scale2;              // scale * log2(e); scores: scale
  float out_scale;
  const float* bias;         // [nodes] or null
  const float* lse2;         // table gradient: [pairs, whole tiles] base-2 log-sums
  const float* miss;         // .. 1 - p of the pair's context
  const int32_t* target;     // .. that context, or -1; forward: contexts [pairs]
  int64_t kept_tiles;        // workgroups along the kept rows
  int32_t splits;
  int64_t tiles_per_split;
  float* part_max;           // forward: [splits][pairs]
  double* part_sum;          // forward: [splits][pairs]
  float* part_rounded;       // .. of the probabilities as they are rounded to 16 bits
  float* part_acc;           // [splits][kept_rows][DP], or null (table gradient without splits)
  void* out;                 // table gradient without splits: g_out; scores: the scores
};

template <typename E, int DP, int MODE, bool BIAS>
__global__ __launch_bounds__(kThreads, (Shape<E, DP, MODE>::kWaves)) void stream_kernel(StreamArgs a) {
  using S = Shape<E, DP, MODE>;
  using elem = typename E::elem;
  constexpr int NB = S::kNB, TILE = S::kTile, ROWB = S::kRowBytes, PIECES = S::kPieces, KS = S::kSteps, DB = S::kBlocks, SWAPPED = S::kSwapped;
  constexpr bool NODES_STREAMED = MODE == kLossOnly || MODE == kForward;
  constexpr bool SECOND = MODE == kForward || MODE == kTableGrad;
  // g_in is the sum of p_j (c_j - c_t).  Rows that share a large part leave little of it: the context's share, which the join takes
  // off, has to be that of the same rounded probabilities: an instruction per two of them.  64 bf16 nodes whose columns are 24 +- 0.5:
  // relative error of g_in 1.68e-3; 1.04e-2 with the unrounded probabilities' share; 1.66e-3 with fp32 probabilities.
  constexpr bool ROUNDED = MODE == kForward && !E::kWide;
  __shared__ __attribute__((aligned(1024))) char tile[2][TILE * ROWB];
  __shared__ __attribute__((aligned(16))) float side[2][TILE];              // nodes streamed: bias * log2(e); pairs streamed: base-2 log-sums
  __shared__ __attribute__((aligned(16))) float side_miss[2][TILE];         // pairs streamed
  __shared__ __attribute__((aligned(16))) int32_t side_target[2][TILE];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, l32 = lane & 31;
  // workgroups of one split stream the same rows: they share an XCD (consecutive workgroups go round the eight of them)
  int64_t kept_tile;
  int split;
  if (a.splits % 8 == 0) {
    const int64_t q = blockIdx.x / 8;
    split = (int)(blockIdx.x % 8 + 8 * (q / a.kept_tiles));
    kept_tile = q % a.kept_tiles;
  } else {
    split = (int)(blockIdx.x / a.kept_tiles);
    kept_tile = blockIdx.x % a.kept_tiles;
  }
  const int64_t all_tiles = tiles_of(a.streamed_rows, TILE);
  const int64_t first = split * a.tiles_per_split;
  const int64_t last = min(first + a.tiles_per_split, all_tiles);
  const int64_t kept_row0 = kept_tile * S::kKept + wave * 32 * NB + l32;      // + 32 nb

  // ---- kept rows into registers
  vec4 kept[NB][KS];
  float kept_bias[NB];
  int32_t kept_target[NB];                     // pairs kept: their contexts
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    int64_t row = kept_row0 + 32 * nb;
    bool live = row < a.kept_rows;
    kept_bias[nb] = 0.0f;
    kept_target[nb] = -1;
    if constexpr (NODES_STREAMED) {
      if (live) kept_target[nb] = a.target[row];
      row = live ? a.centers[row] : -1;
      live = row >= 0 && row < a.num_in;
    } else if constexpr (BIAS) {
      kept_bias[nb] = live ? a.bias[row] * (MODE == kScores ? 1.0f : kLog2e) : -INFINITY;
      live = kept_bias[nb] != -INFINITY;
    }
    if constexpr (S::kStaged) continue;        // below
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int at = (2 * ks + half) * S::kPerPiece;
      const void* src = live && at < a.dim ? static_cast<const void*>(static_cast<const elem*>(a.kept) + row * a.dim + at) : zero_piece;
      kept[nb][ks] = *static_cast<const vec4*>(src);
    }
  }

  // ---- staging: a wave's load number n fills the 64 pieces of chunk 4 n + wave of a tile
  float row_bias[S::kLoads];                   // nodes streamed, with bias: of the rows of the next tile to ask for
  float side_value = 0.0f, miss_value = 0.0f;
  int32_t side_id = -1;
  auto slot_row = [&](int n) { return ((4 * n + wave) * 64 + lane) / PIECES; };
  auto has_chunk = [&](int n) { return S::kChunks % 4 == 0 || 4 * n + wave < S::kChunks; };
  auto fetch_bias = [&](int64_t t) {
    if constexpr (NODES_STREAMED && BIAS) {
#pragma unroll
      for (int n = 0; n < S::kLoads; ++n) {
        const int64_t row = t * TILE + slot_row(n);
        row_bias[n] = has_chunk(n) && row < a.streamed_rows ? a.bias[row] : -INFINITY;
      }
    }
  };
  int32_t row_center[S::kLoads];               // scores: the centres of those rows
  auto fetch_centers = [&](int64_t t) {
    if constexpr (MODE == kScores) {
#pragma unroll
      for (int n = 0; n < S::kLoads; ++n) {
        const int64_t row = t * TILE + slot_row(n);
        row_center[n] = has_chunk(n) && row < a.streamed_rows ? a.centers[row] : -1;
      }
    }
  };
  constexpr int OUTSIDE = 1 << 30, FEW = 8;
  const int streamed_bytes = (MODE == kTableGrad ? DP : a.dim) * (int)sizeof(elem);
  int place[S::kLoads];                        // in the tile's range
#pragma unroll
  for (int n = 0; n < S::kLoads; ++n) {
    const int r = slot_row(n);
    const int piece = (((4 * n + wave) * 64 + lane) % PIECES) ^ swap_of<SWAPPED>(r);
    place[n] = piece * 16 < streamed_bytes ? r * streamed_bytes + piece * 16 : OUTSIDE;
    if (MODE == kScores) place[n] = piece;
  }
  auto issue = [&](int64_t t, int buf) {
    if constexpr (MODE == kScores) {
#pragma unroll
      for (int n = 0; n < S::kLoads; ++n) {
        if (!has_chunk(n)) continue;
        const int64_t c = row_center[n];
        const bool known = c >= 0 && c < a.num_in;
        const elem* src = known && place[n] * S::kPerPiece < a.dim ? static_cast<const elem*>(a.streamed) + c * a.dim + place[n] * S::kPerPiece
                                                                 : reinterpret_cast<const elem*>(known ? zero_piece : nan_piece<E>);
        load_piece_to_lds(src, &tile[buf][(4 * n + wave) * 1024]);
      }
    } else {
      const int64_t rows = min((int64_t)TILE, (MODE == kTableGrad ? all_tiles * TILE : a.streamed_rows) - t * TILE);
      const __amdgpu_buffer_rsrc_t range = range_of(static_cast<const char*>(a.streamed) + t * TILE * streamed_bytes, (int)rows * streamed_bytes);
#pragma unroll
      for (int n = 0; n < S::kLoads; ++n) {
        if (!has_chunk(n)) continue;
        int at = place[n];
        if constexpr (NODES_STREAMED && BIAS) at = row_bias[n] != -INFINITY ? at : OUTSIDE;
        load_piece_to_lds(range, at, &tile[buf][(4 * n + wave) * 1024]);
      }
    }
    if (tid < TILE) {
      const int64_t row = t * TILE + tid;
      if constexpr (MODE == kTableGrad) {
        side_value = a.lse2[row];
        miss_value = a.miss[row];
        side_id = a.target[row];
      } else if constexpr (NODES_STREAMED && BIAS) {
        side_value = row < a.streamed_rows ? a.bias[row] * kLog2e : -INFINITY;
      }
    }
  };
  auto put_side = [&](int buf) {
    if constexpr (MODE == kTableGrad || (NODES_STREAMED && BIAS)) {
      if (tid < TILE) {
        side[buf][tid] = side_value;
        if constexpr (MODE == kTableGrad) {
          side_miss[buf][tid] = miss_value;
          side_target[buf][tid] = side_id;
        }
      }
    }
  };

  acc16 out[SECOND ? DB : 1][NB];
  if constexpr (SECOND) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) out[db][nb] = (acc16)0.0f;
  }
  float run_max[NB];
  double run_sum[NB];                          // this half wave's streamed rows
  float run_rounded[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    run_max[nb] = -INFINITY;
    run_sum[nb] = 0.0;
    run_rounded[nb] = 0.0f;
  }

  // lane's parts of the LDS addresses; the swap turns bits of them that a row's place leaves zero, what lies above is added
  constexpr int SWAP_KS = SWAPPED / 2 - 1;     // steps of the first product inside the swapped pieces
  const int read1 = l32 * ROWB + ((half ^ swap_of<SWAPPED>(l32)) << 4);
  int read2;
  if constexpr (E::kWide) {
    read2 = (((l32 >> 2) ^ half) << 4) + (l32 & 3) * 4 + half * 4 * ROWB;
  } else {
    const int li = lane & 15, r = li >> 2;
    const int turn = SWAPPED == 16 ? r << 2 : SWAPPED == 8 ? ((r >> 1) & 1) << 2 : 0;
    const int piece = (((lane >> 4) & 1) * 2 + ((li & 3) >> 1)) ^ turn ^ half;
    read2 = (piece << 4) + (li & 1) * 8 + (4 * half + r) * ROWB;
  }

  if constexpr (S::kStaged) {
    // the kept rows, 32 at a time, each into the registers of the wave that keeps them
    constexpr int STEPS = 4 * NB;
    const int64_t row0 = kept_tile * S::kKept;
    float step_bias[S::kLoads];
    auto fetch_step = [&](int i) {
      if constexpr (BIAS) {
#pragma unroll
        for (int n = 0; n < S::kLoads; ++n) {
          const int64_t row = row0 + 32 * i + slot_row(n);
          step_bias[n] = has_chunk(n) && row < a.kept_rows ? a.bias[row] : -INFINITY;
        }
      }
    };
    auto issue_step = [&](int i, int buf) {
      const int64_t rows = min((int64_t)32, a.kept_rows - row0 - 32 * i);
      const __amdgpu_buffer_rsrc_t range =
          range_of(static_cast<const char*>(a.kept) + (row0 + 32 * i) * streamed_bytes, rows > 0 ? (int)rows * streamed_bytes : 0);
#pragma unroll
      for (int n = 0; n < S::kLoads; ++n) {
        if (!has_chunk(n)) continue;
        int at = place[n] * 16 < streamed_bytes ? slot_row(n) * streamed_bytes + place[n] * 16 : OUTSIDE;
        if constexpr (BIAS) at = step_bias[n] != -INFINITY ? at : OUTSIDE;
        load_piece_to_lds(range, at, &tile[buf][(4 * n + wave) * 1024]);
      }
    };
    fetch_step(0);
    issue_step(0, 0);
    fetch_step(1);
    if (first < last) fetch_centers(first);
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      wait_loads_and_barrier();
      if (i + 1 < STEPS) {
        issue_step(i + 1, (i + 1) & 1);
        if (i + 2 < STEPS) fetch_step(i + 2);
      } else if (first < last) {               // STEPS is even: buffer 0 was read a step ago
        issue(first, 0);
        if (first + 1 < last) fetch_centers(first + 1);
      }
      if (wave == i / NB) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          kept[i % NB][ks] = *reinterpret_cast<const vec4*>(tile[i & 1] + (read1 ^ ((ks & SWAP_KS) << 5)) + (ks & ~SWAP_KS) * 32);
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  } else if constexpr (MODE == kScores) {
    if (first < last) {
      fetch_centers(first);
      issue(first, 0);
      if (first + 1 < last) fetch_centers(first + 1);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  } else if (first < last) {
    fetch_bias(first);
    issue(first, 0);
    put_side(0);
    if (first + 1 < last) fetch_bias(first + 1);
  }
  // Pairs without gradient are rows of zeros, whose probability is 0 by a log-sum of infinity: but not where a node's row holds
  // infinities or NaN, which turn it into NaN.  A wave that keeps such a row sets those pairs' to 0 by name (what the others pay to
  // know that they keep none: 1 % of a batch at most).
  bool no_numbers = false;
  if constexpr (MODE == kTableGrad) {
    vec4 zero = (vec4)0.0f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int e = 0; e < 4; ++e) zero[e] = E::add_none(kept[nb][ks][e], zero[e]);
    const float sum = (zero[0] + zero[1]) + (zero[2] + zero[3]);
    no_numbers = __any(sum != sum);
  }

  // One tile.  The buffer is a constant of the code: its place is part of the LDS instructions then, and the lane's addresses
  // do not change over the loop.
  auto take_tile = [&](auto which, int64_t t) {
    constexpr int BUF = decltype(which)::value;
    constexpr int JB = TILE / 32;
    // scores: each wave has waited for its loads in front of its stores, which need not be waited for
    if constexpr (MODE == kScores) lds_barrier();
    else wait_loads_and_barrier();
    if (t + 1 < last) {
      issue(t + 1, BUF ^ 1);
      if (t + 2 < last) {
        fetch_bias(t + 2);
        fetch_centers(t + 2);
      }
    }
    const char* base = tile[BUF];
    acc16 z[JB][NB];
    if constexpr (MODE == kScores && E::kWide) {
      // a few centres alone: their sums by ordinary arithmetic, each 1/16 of what the tile's matrix instructions take (one centre
      // on 1 M nodes of 256 columns 311 -> 168 us; eight take half a tile's time)
      const int64_t left = a.streamed_rows - t * TILE;
      if (left <= FEW) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        for (int row = 0; row < (int)left; ++row) {
          float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const vec4 v = *reinterpret_cast<const vec4*>(base + row * ROWB + ((((2 * ks) | half) ^ swap_of<SWAPPED>(row)) << 4));
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] = fmaf(v[e], kept[0][ks][e], sum[e]);
          }
          float z1 = (sum[0] + sum[1]) + (sum[2] + sum[3]);
          z1 += __shfl_xor(z1, 32, 64);
          if (half == 0 && kept_row0 < a.kept_rows)
            static_cast<float*>(a.out)[(t * TILE + row) * a.kept_rows + kept_row0] =
                !BIAS ? z1 * a.scale2 : kept_bias[0] == -INFINITY ? -INFINITY : fmaf(z1, a.scale2, kept_bias[0]);
        }
        return;
      }
    }
    if constexpr (S::kWaves > 1) __builtin_amdgcn_s_setprio(1);         // of two waves the one with matrix work to issue goes first: 1 %
#pragma unroll
    for (int jb = 0; jb < JB; ++jb) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) z[jb][nb] = (acc16)0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const vec4 v = *reinterpret_cast<const vec4*>(base + (read1 ^ ((ks & SWAP_KS) << 5)) + (ks & ~SWAP_KS) * 32 + jb * 32 * ROWB);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) z[jb][nb] = step<E>(v, kept[nb][ks], z[jb][nb]);
      }
    }
    if constexpr (S::kWaves > 1) __builtin_amdgcn_s_setprio(0);
    // ---- products to probabilities: register r of block jb holds streamed row 32 jb + 8 (r / 4) + 4 half + r % 4
    if constexpr (NODES_STREAMED) {
      if constexpr (BIAS) {
#pragma unroll
        for (int jb = 0; jb < JB; ++jb)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const vec4 b = *reinterpret_cast<const vec4*>(&side[BUF][jb * 32 + 8 * q + 4 * half]);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int e = 0; e < 4; ++e) z[jb][nb][4 * q + e] = fmaf(z[jb][nb][4 * q + e], a.scale2, b[e]);
          }
      } else if ((t + 1) * TILE > a.streamed_rows) {
        rare();
        const int left = (int)(a.streamed_rows - t * TILE) - 4 * half;
#pragma unroll
        for (int jb = 0; jb < JB; ++jb)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (32 * jb + 8 * (r / 4) + r % 4 >= left) z[jb][nb][r] = -INFINITY;
      }
      // The context takes no part here: its weight is 1 minus the others' sum, and joins at the end.  Where it has nearly all
      // the weight, 1 - p would be lost in p's own rounding otherwise.
      const uint32_t tile_row0 = (uint32_t)(t * TILE);
      bool here = false;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) here = here || (uint32_t)kept_target[nb] - tile_row0 < (uint32_t)TILE;
      if (__any(here)) {
        rare();
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const uint32_t at = (uint32_t)kept_target[nb] - tile_row0 - 4 * half;
#pragma unroll
          for (int jb = 0; jb < JB; ++jb)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (at == (uint32_t)(32 * jb + 8 * (r / 4) + r % 4)) z[jb][nb][r] = -INFINITY;
        }
      }
      bool moved = false;
      float keep[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float m = z[0][nb][0];
#pragma unroll
        for (int jb = 0; jb < JB; ++jb)
#pragma unroll
          for (int r = 0; r < 16; ++r) m = fmaxf(m, z[jb][nb][r]);
        m = fmaxf(m, __shfl_xor(m, 32, 64));
        if constexpr (!BIAS) m *= a.scale2;
        // the maximum follows only by more than kSlack: until then probabilities grow to 2^kSlack, which costs nothing, and
        // the sums need no rescaling (a row's maximum moves some ten times, but one of a wave's rows' does in every third tile)
        const float next = m > run_max[nb] + E::kSlack ? m : run_max[nb];
        moved = moved || next > run_max[nb];
        const float from = next == -INFINITY ? 0.0f : next;       // nothing but masked nodes so far
        keep[nb] = __builtin_amdgcn_exp2f(run_max[nb] - from);
        run_max[nb] = next;
        float sum = 0.0f;
        const float add = (float)E::kForwardShift - from;
#pragma unroll
        for (int jb = 0; jb < JB; ++jb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float x = BIAS ? z[jb][nb][r] + add : fmaf(z[jb][nb][r], a.scale2, add);
            z[jb][nb][r] = __builtin_amdgcn_exp2f(x);
            sum += z[jb][nb][r];
          }
        run_sum[nb] = run_sum[nb] * (double)keep[nb] + (double)sum;
        if constexpr (ROUNDED) run_rounded[nb] *= keep[nb];
      }
      if constexpr (SECOND) {
        if (__any(moved)) {
          rare();
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int db = 0; db < DB; ++db) out[db][nb] *= keep[nb];
        }
      }
    } else if constexpr (MODE == kScores) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) asm volatile("s_waitcnt vmcnt(0)" : "+v"(z[0][nb]) : : "memory");      // behind the products
#pragma unroll
      for (int jb = 0; jb < JB; ++jb) {
        const int64_t pair0 = t * TILE + jb * 32 + 4 * half;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const int64_t node = kept_row0 + 32 * nb;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int64_t pair = pair0 + 8 * (r / 4) + r % 4;
            if (node < a.kept_rows && pair < a.streamed_rows)
              static_cast<float*>(a.out)[pair * a.kept_rows + node] =
                  !BIAS ? z[jb][nb][r] * a.scale2 : kept_bias[nb] == -INFINITY ? -INFINITY : fmaf(z[jb][nb][r], a.scale2, kept_bias[nb]);
          }
        }
      }
    } else {
#pragma unroll
      for (int jb = 0; jb < JB; ++jb)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const vec4 l = *reinterpret_cast<const vec4*>(&side[BUF][jb * 32 + 8 * q + 4 * half]);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float add = BIAS ? kept_bias[nb] - l[e] : -l[e];
              z[jb][nb][4 * q + e] = __builtin_amdgcn_exp2f(fmaf(z[jb][nb][4 * q + e], a.scale2, add));
            }
        }
      if (__builtin_expect(no_numbers, 0)) {
        rare();
#pragma unroll
        for (int jb = 0; jb < JB; ++jb)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int4 ids = *reinterpret_cast<const int4*>(&side_target[BUF][jb * 32 + 8 * q + 4 * half]);
            const int32_t id[4] = {ids.x, ids.y, ids.z, ids.w};
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (id[e] < 0) z[jb][nb][4 * q + e] = 0.0f;
          }
      }
      // does any pair of this tile have its context among this wave's nodes?
      const int32_t wave_node0 = (int32_t)(kept_row0 - l32), t_of_lane = side_target[BUF][lane % TILE];
      if (__any(t_of_lane >= wave_node0 && t_of_lane - wave_node0 < 32 * NB)) {
        rare();
        constexpr float one = (float)(1 << E::kShift);
#pragma unroll
        for (int jb = 0; jb < JB; ++jb)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int pair = jb * 32 + 8 * q + 4 * half;
            const int4 ids = *reinterpret_cast<const int4*>(&side_target[BUF][pair]);
            const int32_t id[4] = {ids.x, ids.y, ids.z, ids.w};
            bool hit = false;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int e = 0; e < 4; ++e) hit = hit || id[e] == (int32_t)(kept_row0 + 32 * nb);
            if (!__any(hit)) continue;
            rare();
            const vec4 p = *reinterpret_cast<const vec4*>(&side_miss[BUF][pair]) * -one;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (id[e] == (int32_t)(kept_row0 + 32 * nb)) z[jb][nb][4 * q + e] = p[e];
          }
      }
    }
    // ---- second product
    if constexpr (S::kWaves > 1) __builtin_amdgcn_s_setprio(1);
    if constexpr (SECOND) {
#pragma unroll
      for (int jb = 0; jb < JB; ++jb) {
        if constexpr (E::kWide) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
#pragma unroll
            for (int db = 0; db < DB; ++db) {
              constexpr int swap_db = SWAPPED == 16 ? 1 : 0;         // blocks of eight pieces
              const int turn = ((db & swap_db) * 8) ^ (SWAPPED == 16 ? (r % 4) << 2 : ((r % 4) >> 1) << 2) ^ (2 * ((r / 4) & 1));
              const float v = *reinterpret_cast<const float*>(base + (read2 ^ (turn << 4)) + (db & ~swap_db) * 128 +
                                                              (jb * 32 + 8 * (r / 4) + r % 4) * ROWB);
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) out[db][nb] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, z[jb][nb][r], out[db][nb], 0, 0, 0);
            }
          }
        } else {
#pragma unroll
          for (int q2 = 0; q2 < 2; ++q2) {
            vec4 p[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t w = E::pack(z[jb][nb][8 * q2 + 2 * e], z[jb][nb][8 * q2 + 2 * e + 1]);
                if constexpr (ROUNDED) run_rounded[nb] = E::add_pair(w, run_rounded[nb]);
                p[nb][e] = __uint_as_float(w);
              }
#pragma unroll
            for (int db = 0; db < DB; ++db) {
              short4_t part[2];
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int q = 2 * q2 + e;
                constexpr int swap_db = SWAPPED / 4 - 1;             // blocks of four pieces
                const int turn = ((db & swap_db) * 4) ^ (2 * (q & 1));
                part[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_short4*)(base + (read2 ^ (turn << 4)) + (db & ~swap_db) * 64 + (jb * 32 + 8 * q) * ROWB));
              }
              const vec4 v = __builtin_bit_cast(vec4, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) out[db][nb] = E::mfma(v, p[nb], out[db][nb]);
            }
          }
        }
      }
    }
    if (t + 1 < last) put_side(BUF ^ 1);
  };
  for (int64_t t = first; t < last; t += 2) {
    take_tile(std::integral_constant<int, 0>{}, t);
    if (t + 1 < last) take_tile(std::integral_constant<int, 1>{}, t + 1);
  }

  // ---- results: lane's kept row, register r of block db is column 32 db + 8 (r / 4) + 4 half + r % 4
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int64_t row = kept_row0 + 32 * nb;
    if constexpr (NODES_STREAMED) {
      const double sum = run_sum[nb] + __shfl_xor(run_sum[nb], 32, 64);
      if (row < a.kept_rows && half == 0) {
        a.part_max[split * a.kept_rows + row] = run_max[nb];
        a.part_sum[split * a.kept_rows + row] = sum;
      }
    }
    if constexpr (ROUNDED) {
      const float rounded = run_rounded[nb] + __shfl_xor(run_rounded[nb], 32, 64);
      if (row < a.kept_rows && half == 0) a.part_rounded[split * a.kept_rows + row] = rounded;
    }
    if constexpr (SECOND) {
      if (row < a.kept_rows) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int col = 32 * db + 8 * q + 4 * half;
            vec4 v = {out[db][nb][4 * q], out[db][nb][4 * q + 1], out[db][nb][4 * q + 2], out[db][nb][4 * q + 3]};
            // a masked node has no gradient, whatever the pairs' rows hold
            if (MODE == kTableGrad && BIAS && kept_bias[nb] == -INFINITY) v = (vec4)0.0f;
            if (MODE == kTableGrad && a.part_acc == nullptr) {
              if (col < a.dim) E::store4(static_cast<elem*>(a.out) + row * a.dim + col, v * a.out_scale);
            } else {
              *reinterpret_cast<vec4*>(a.part_acc + (split * a.kept_rows + row) * DP + col) = v;
            }
          }
      }
    }
  }
}

// ---- joining the parts of the forward pass ------------------------------------------------------------------------------
// Bound by reading the parts: 20 us for 65,536 pairs in one part, 22 us for 4096 in 16, 19 us for 777 in 72 (50 MB); one pair's 152
// parts 4 us of latency.
struct JoinArgs {
  const void *w_in, *w_out;
  int64_t num_in, num_nodes, num_pairs, padded_pairs;
  int32_t dim, padded, splits;
  const int32_t *centers, *contexts;
  const float* bias;
  float scale, out_scale;
  const float* part_max;
  const double* part_sum;
  const float* part_rounded;
  const float* part_acc;
  float* loss;
  float* lse2;               // for the table gradient, to whole tiles: +infinity for a pair without gradient; or null
  float* miss;               // .. 1 - p of its context
  int32_t* target;           // .. its context, or -1
  void* g_in;                // or null
};
// QUADS lanes for a row (four columns each) and SLOTS of them for a pair, which share its splits: one for the few splits of many
// pairs, the whole workgroup for the many splits of few.
template <typename E, int QUADS, int SLOTS>
__global__ __launch_bounds__(kThreads) void join_pairs_kernel(JoinArgs a) {
  constexpr int GROUP = QUADS * SLOTS, PAIRS = kThreads / GROUP;
  typedef typename E::elem elem;
  __shared__ vec4 part_g[SLOTS > 1 ? kThreads : 1];
  __shared__ double part_s[SLOTS > 1 ? kThreads / 64 : 1];
  __shared__ float part_m[SLOTS > 1 ? kThreads / 64 : 1];
  const int member = threadIdx.x % GROUP, quad = member % QUADS, slot = member / QUADS;
  const int64_t i = (int64_t)blockIdx.x * PAIRS + threadIdx.x / GROUP;
  if (i >= a.padded_pairs) return;             // whole workgroups where SLOTS > 1
  const bool exists = i < a.num_pairs;
  const int64_t c = exists ? a.centers[i] : -1;
  int32_t t = exists ? a.contexts[i] : -1;
  // what keeps a pair from having a gradient: -1 left out, -2 an id that is no row, -3 its context is masked
  if (exists && (c < 0 || c >= a.num_in || t < -1 || t >= a.num_nodes)) t = -2;
  else if (t >= 0 && a.bias && a.bias[t] == -INFINITY) t = -3;
  const bool live = t >= 0;
  // the context's row and score
  const bool column = 4 * quad < a.dim;        // the lanes beyond read nothing
  vec4 to = (vec4)0.0f;
  double dot = 0.0;
  if (live && column) {
    const elem* h = static_cast<const elem*>(a.w_in) + c * a.dim + 4 * quad;
    const elem* v = static_cast<const elem*>(a.w_out) + (int64_t)t * a.dim + 4 * quad;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      to[e] = E::load(v + e);
      dot += (double)E::load(h + e) * (double)to[e];
    }
  }
#pragma unroll
  for (int d = QUADS / 2; d; d >>= 1) dot += __shfl_xor(dot, d, 64);
  const double z2 = live ? ((double)a.scale * dot + (a.bias ? (double)a.bias[t] : 0.0)) * (1.0 / kLn2) : -INFINITY;    // base 2
  // the splits' maxima and sums, of all nodes but the context; m: the largest of them and of z2
  float m_others = -INFINITY;
  double m = z2, others = 0.0;
  if (exists) {
    for (int s = SLOTS > 1 ? member : 0; s < a.splits; s += SLOTS > 1 ? GROUP : 1) m_others = fmaxf(m_others, a.part_max[s * a.num_pairs + i]);
    if constexpr (SLOTS > 1) {
#pragma unroll
      for (int d = 32; d; d >>= 1) m_others = fmaxf(m_others, __shfl_xor(m_others, d, 64));
      if ((threadIdx.x & 63) == 0) part_m[threadIdx.x >> 6] = m_others;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kThreads / 64; ++w) m_others = fmaxf(m_others, part_m[w]);
    }
    m = fmax(z2, (double)m_others);
    for (int s = SLOTS > 1 ? member : 0; s < a.splits; s += SLOTS > 1 ? GROUP : 1) {
      const float pm = a.part_max[s * a.num_pairs + i];
      const double ps = a.part_sum[s * a.num_pairs + i];
      // a split of masked nodes alone has sum 0, whatever its maximum
      others += pm == -INFINITY && ps == 0.0 ? 0.0 : ps * exp2((double)pm - m);
    }
    if constexpr (SLOTS > 1) {
#pragma unroll
      for (int d = 32; d; d >>= 1) others += __shfl_xor(others, d, 64);
      if ((threadIdx.x & 63) == 0) part_s[threadIdx.x >> 6] = others;
      __syncthreads();
      others = 0.0;
#pragma unroll
      for (int w = 0; w < kThreads / 64; ++w) others += part_s[w];
    }
  }
  const double own = live ? exp2(z2 - m) * (double)(1 << E::kForwardShift) : 0.0;
  const double sum = others + own;
  const double total2 = m + log2(sum) - (double)E::kForwardShift;          // base-2 log-sum
  const float miss = live ? (float)(others / sum) : 0.0f;
  if (a.lse2 != nullptr && member == 0) {
    a.lse2[i] = live ? (float)(total2 - (double)E::kShift) : INFINITY;
    a.miss[i] = miss;
    a.target[i] = live ? t : -1;
  }
  if (!exists) return;
  if (member == 0) {
    // a context that leads by far: its loss is of the others' size, not of the log-sum's rounding
    double value = z2 >= (double)m_others ? log1p(others / own) : (total2 - z2) * kLn2;
    if (t == -1) value = 0.0;
    if (t == -2) value = NAN;
    if (t == -3) value = INFINITY;
    a.loss[i] = (float)value;
  }
  if (a.g_in == nullptr) return;
  vec4 g = (vec4)0.0f;
  if (live && column) {
    const double inverse = 1.0 / sum;
#pragma unroll 4
    for (int s = slot; s < a.splits; s += SLOTS) {
      const float pm = a.part_max[s * a.num_pairs + i];
      const bool empty = pm == -INFINITY && a.part_sum[s * a.num_pairs + i] == 0.0;           // masked nodes alone
      const float w = empty ? 0.0f : (float)(exp2((double)pm - m) * inverse);
      vec4 part = *reinterpret_cast<const vec4*>(a.part_acc + (s * a.num_pairs + i) * a.padded + 4 * quad);
      if constexpr (!E::kWide) part -= a.part_rounded[s * a.num_pairs + i] * to;
      g += w * part;
    }
  }
  if constexpr (SLOTS > 1) {
    part_g[threadIdx.x] = g;
    __syncthreads();
    if (slot != 0) return;
#pragma unroll
    for (int k = 1; k < SLOTS; ++k) g += part_g[k * QUADS + quad];
  }
  if (!column) return;
  if (live) {
    if constexpr (E::kWide) g -= miss * to;
    g *= a.out_scale;
  }
  E::store4(static_cast<elem*>(a.g_in) + i * a.dim + 4 * quad, g);
}

// g_out from the parts of a split table gradient, in order
template <typename E>
__global__ __launch_bounds__(kThreads) void join_nodes_kernel(const float* part_acc, int64_t num_nodes, int dim, int padded,
                                                              int splits, float out_scale, typename E::elem* g_out) {
  const int quads = dim / 4;
  const int64_t total = num_nodes * quads;
  for (int64_t s = (int64_t)blockIdx.x * kThreads + threadIdx.x; s < total; s += (int64_t)gridDim.x * kThreads) {
    const int64_t row = s / quads;
    const int d0 = 4 * (int)(s - row * quads);
    vec4 g = (vec4)0.0f;
    for (int k = 0; k < splits; ++k) g += *reinterpret_cast<const vec4*>(part_acc + (k * num_nodes + row) * padded + d0);
    E::store4(g_out + row * dim + d0, g * out_scale);
  }
}

// The same from many parts of few nodes: a workgroup a row, its lanes share the parts (512 parts of 100 nodes one lane after the
// other took 150 us).
template <typename E>
__global__ __launch_bounds__(kThreads) void join_many_kernel(const float* part_acc, int64_t num_nodes, int dim, int padded,
                                                             int splits, float out_scale, typename E::elem* g_out) {
  __shared__ vec4 part[kThreads];
  const int quads = padded / 4, slots = kThreads / quads;
  const int quad = threadIdx.x % quads, slot = threadIdx.x / quads;
  const int64_t row = blockIdx.x;
  vec4 g = (vec4)0.0f;
  if (slot < slots) {
#pragma unroll 4
    for (int k = slot; k < splits; k += slots) g += *reinterpret_cast<const vec4*>(part_acc + (k * num_nodes + row) * padded + 4 * quad);
  }
  part[threadIdx.x] = g;
  __syncthreads();
  if (slot != 0 || 4 * quad >= dim) return;
  for (int k = 1; k < slots; ++k) g += part[k * quads + quad];
  E::store4(g_out + row * dim + 4 * quad, g * out_scale);
}

// no pairs: every gradient is zero
__global__ __launch_bounds__(kThreads) void zero_pieces_kernel(uint4* to, int64_t pieces) {
  for (int64_t s = (int64_t)blockIdx.x * kThreads + threadIdx.x; s < pieces; s += (int64_t)gridDim.x * kThreads)
    to[s] = make_uint4(0, 0, 0, 0);
}

}  // namespace

// ---- host ----------------------------------------------------------------------------------------------------------------
// f with the padded number of columns as a constant
template <typename R, typename F>
static R with_padded(int dim, F f) {
  switch ((dim + 31) / 32) {
    case 1: return f(std::integral_constant<int, 32>{});
    case 2: return f(std::integral_constant<int, 64>{});
    case 3: return f(std::integral_constant<int, 96>{});
    case 4: return f(std::integral_constant<int, 128>{});
    case 5: return f(std::integral_constant<int, 160>{});
    case 6: return f(std::integral_constant<int, 192>{});
    case 7: return f(std::integral_constant<int, 224>{});
    default: return f(std::integral_constant<int, 256>{});
  }
}

template <typename E, int DP>
static void plan_tiles(SoftmaxPlan& p, int64_t num_pairs, int64_t num_nodes, bool loss, bool grad, size_t& acc_rows, size_t& part_rows) {
  using L = Shape<E, DP, kForward>;
  using Z = Shape<E, DP, kScores>;
  constexpr int64_t want = 256 * L::kWaves;    // workgroups that fill the chip
  auto split = [&](int64_t kept, int64_t streamed) {
    int64_t n = std::max<int64_t>(1, std::min(streamed, want / std::max<int64_t>(1, kept)));
    return (int)(n >= 8 ? n / 8 * 8 : n);
  };
  p.padded = DP;
  p.node_tiles = ceil_div(num_nodes, loss ? L::kKept : Z::kKept);
  const int64_t pair_parts = ceil_div(num_pairs, loss ? L::kTile : Z::kTile);
  p.node_splits = split(p.node_tiles, pair_parts);
  p.tiles_per_node_split = ceil_div(std::max<int64_t>(1, pair_parts), p.node_splits);
  if (!loss) return;
  p.padded_pairs = ceil_div(num_pairs, 256) * 256;
  p.pair_tiles = ceil_div(num_pairs, L::kKept);
  const int64_t tiles = ceil_div(num_nodes, L::kTile);
  p.splits = split(p.pair_tiles, tiles);
  p.tiles_per_split = ceil_div(tiles, p.splits);
  // every size below only grows with the number of pairs, although the number of splits falls
  part_rows = (size_t)std::max(num_pairs, std::min(std::min(tiles, want) * num_pairs, want * L::kKept));
  acc_rows = grad ? part_rows : 0;
  if (grad && p.node_splits > 1) acc_rows = std::max(acc_rows, (size_t)p.node_splits * (size_t)num_nodes);
}

template <typename E>
SoftmaxPlan plan_softmax(void* ws, int64_t num_pairs, int64_t num_nodes, int32_t dim, bool loss, bool grad) {
  SoftmaxPlan p{};
  size_t acc_rows = 0, part_rows = 0;
  with_padded<int>(dim, [&](auto padded) {
    plan_tiles<E, decltype(padded)::value>(p, num_pairs, num_nodes, loss, grad, acc_rows, part_rows);
    return 0;
  });
  Carver c(ws);
  if (loss) {
    if (grad) p.rows = c.take<typename E::elem>((size_t)p.padded_pairs * p.padded);
    p.target = c.take<int32_t>(p.padded_pairs);
    p.lse2 = c.take<float>(p.padded_pairs);
    p.miss = c.take<float>(p.padded_pairs);
    p.part_max = c.take<float>(part_rows);
    p.part_sum = c.take<double>(part_rows);
    if (grad && !E::kWide) p.part_rounded = c.take<float>(part_rows);
    p.part_acc = c.take<float>(acc_rows * p.padded);
  }
  p.bytes = std::max<size_t>(c.used, 256);
  return p;
}

template <typename E, int DP, int MODE>
static int32_t launch_stream(const StreamArgs& a, hipStream_t stream) {
  const int64_t groups = a.kept_tiles * a.splits;
  if (a.bias) stream_kernel<E, DP, MODE, true><<<(unsigned)groups, kThreads, 0, stream>>>(a);
  else stream_kernel<E, DP, MODE, false><<<(unsigned)groups, kThreads, 0, stream>>>(a);
  GS_LAUNCH_CHECK();
  return GS_OK;
}

template <typename E, int DP>
static int32_t run_padded(const SoftmaxCall& q, const SoftmaxPlan& p, hipStream_t stream) {
  using elem = typename E::elem;
  constexpr int64_t most = ((int64_t)1 << 32) / kThreads;        // a launch takes fewer than 2^32 lanes
  if ((!q.loss || q.g_out) && p.node_tiles * p.node_splits >= most) return GS_EOVERFLOW;
  // the join: four pairs a workgroup at least, but for few pairs in many parts
  if (q.loss && (p.pair_tiles * p.splits >= most || p.padded_pairs / 4 >= most)) return GS_EOVERFLOW;
  auto blocks_for = [](int64_t items) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(ceil_div(items, kThreads), 256 * 16)); };
  StreamArgs a{};
  a.dim = q.dim;
  a.bias = q.bias;
  a.centers = q.centers;
  a.num_in = q.num_in;
  if (!q.loss) {
    a.kept = q.w_out;
    a.streamed = q.w_in;
    a.kept_rows = q.num_nodes;
    a.streamed_rows = q.num_pairs;
    a.scale2 = q.scale;
    a.kept_tiles = p.node_tiles;
    a.splits = p.node_splits;
    a.tiles_per_split = p.tiles_per_node_split;
    a.out = q.scores;
    return launch_stream<E, DP, kScores>(a, stream);
  }
  a.kept = q.w_in;
  a.streamed = q.w_out;
  a.kept_rows = q.num_pairs;
  a.streamed_rows = q.num_nodes;
  a.scale2 = q.scale * kLog2e;
  a.kept_tiles = p.pair_tiles;
  a.splits = p.splits;
  a.tiles_per_split = p.tiles_per_split;
  a.part_max = p.part_max;
  a.part_sum = p.part_sum;
  a.part_rounded = p.part_rounded;
  a.part_acc = p.part_acc;
  a.target = q.contexts;
  int32_t rc = q.g_in ? launch_stream<E, DP, kForward>(a, stream) : launch_stream<E, DP, kLossOnly>(a, stream);
  if (rc != GS_OK) return rc;
  const float out_scale = q.scale * q.grad_scale;
  JoinArgs j{};
  j.w_in = q.w_in;
  j.w_out = q.w_out;
  j.num_in = q.num_in;
  j.num_nodes = q.num_nodes;
  j.num_pairs = q.num_pairs;
  j.padded_pairs = q.g_out ? p.padded_pairs : q.num_pairs;
  j.dim = q.dim;
  j.padded = DP;
  j.splits = p.splits;
  j.centers = q.centers;
  j.contexts = q.contexts;
  j.bias = q.bias;
  j.scale = q.scale;
  j.out_scale = out_scale;
  j.part_max = p.part_max;
  j.part_sum = p.part_sum;
  j.part_rounded = p.part_rounded;
  j.part_acc = p.part_acc;
  j.loss = q.loss;
  j.lse2 = q.g_out ? p.lse2 : nullptr;
  j.miss = p.miss;
  j.target = p.target;
  j.g_in = q.g_in;
  constexpr int quads = DP <= 64 ? 16 : DP <= 128 ? 32 : 64;
  if (p.splits > 8) join_pairs_kernel<E, quads, kThreads / quads><<<(unsigned)j.padded_pairs, kThreads, 0, stream>>>(j);
  else join_pairs_kernel<E, quads, 1><<<(unsigned)ceil_div(j.padded_pairs, kThreads / quads), kThreads, 0, stream>>>(j);
  GS_LAUNCH_CHECK();
  if (!q.g_out) return GS_OK;
  elem* rows = static_cast<elem*>(p.rows);
  gather_pairs_kernel<E><<<blocks_for(p.padded_pairs * (DP / (16 / (int)sizeof(elem)))), kThreads, 0, stream>>>(
      static_cast<const elem*>(q.w_in), q.dim, DP, q.centers, p.target, p.padded_pairs, rows);
  GS_LAUNCH_CHECK();
  a.kept = q.w_out;
  a.streamed = rows;
  a.kept_rows = q.num_nodes;
  a.streamed_rows = q.num_pairs;
  a.lse2 = p.lse2;
  a.miss = p.miss;
  a.target = p.target;
  a.kept_tiles = p.node_tiles;
  a.splits = p.node_splits;
  a.tiles_per_split = p.tiles_per_node_split;
  a.out_scale = out_scale / (float)(1 << E::kShift);
  a.part_acc = p.node_splits > 1 ? p.part_acc : nullptr;
  a.out = q.g_out;
  rc = launch_stream<E, DP, kTableGrad>(a, stream);
  if (rc != GS_OK || p.node_splits == 1) return rc;
  if (p.node_splits > 8) {                     // 64 tiles of nodes at most
    join_many_kernel<E><<<(unsigned)q.num_nodes, kThreads, 0, stream>>>(p.part_acc, q.num_nodes, q.dim, DP, p.node_splits, a.out_scale,
                                                                       static_cast<elem*>(q.g_out));
    GS_LAUNCH_CHECK();
    return GS_OK;
  }
  join_nodes_kernel<E><<<blocks_for(q.num_nodes * (q.dim / 4)), kThreads, 0, stream>>>(
      p.part_acc, q.num_nodes, q.dim, DP, p.node_splits, a.out_scale, static_cast<elem*>(q.g_out));
  GS_LAUNCH_CHECK();
  return GS_OK;
}

template <typename E>
int32_t run_softmax(const SoftmaxCall& q, const SoftmaxPlan& p, hipStream_t stream) {
  if (q.num_pairs == 0) {
    if (!q.g_out) return GS_OK;
    const int64_t pieces = q.num_nodes * q.dim * (int64_t)sizeof(typename E::elem) / 16;
    zero_pieces_kernel<<<(unsigned)std::min<int64_t>(ceil_div(pieces, kThreads), 256 * 16), kThreads, 0, stream>>>(static_cast<uint4*>(q.g_out), pieces);
    GS_LAUNCH_CHECK();
    return GS_OK;
  }
  return with_padded<int32_t>(q.dim, [&](auto padded) { return run_padded<E, decltype(padded)::value>(q, p, stream); });
}

#endif  // GS_SOFTMAX_KERNELS

}  // namespace gs
