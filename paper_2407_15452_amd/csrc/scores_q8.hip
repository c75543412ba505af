// gs_scores_q8: scores of centres against every node, from 8-bit rows.
//
//   z_ij = scale * sum_b 2^(e_ib + f_jb) sum_{k in block b} a_ik c_jk + bias_j
//
// a, c: e4m3 values; e, f: the powers of two of their blocks of 128 columns.  Two kinds of products:
//   fp32 scores: the values go through v_cvt_scalef32_pk_bf16_fp8 into the bf16 matrix instruction, whose products of them are exact
//     and whose sums are fp32.  The conversion multiplies by powers of two as well, by the block's own; those that bf16 has no room
//     for are looked for, and multiply sums of the block alone.
//   16-bit scores: v_mfma_scale_f32_32x32x64 on the bytes themselves, which multiplies by the powers of the blocks and runs at twice
//     the rate.  Of eight neighbouring products it drops what lies 2^13 below the largest of them (measured, and so do the 8-bit
//     instructions without scales): at most 7 * 2^-13 of the sum of the products' sizes, some 2^-16 of it for Gaussian rows; fp32
//     scores would keep 16 bits, while fp16 keeps 11 and bf16 8 of any.
// Both instructions sum over any numbering of a block's columns, as long as both operands use the same one: a lane takes 64
// neighbouring bytes of a row's 128.  Nodes are the left operand: a lane then holds four neighbouring nodes' scores of one centre,
// which lie together in memory.

#include "common.h"

#include <cmath>
#include <type_traits>

namespace gs {
namespace {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef float acc16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = 128;

struct ScoresArgs {
  const uint8_t *q_in, *scales_in;
  int64_t num_in;
  const uint8_t *q_out, *scales_out;
  int64_t num_nodes;
  int32_t pitch, blocks, scale_pitch;
  const int32_t* centers;
  int64_t num_centers;
  const float* bias;
  float scale;
  void* out;
};

// Pieces of rows of scores, which begin at any element.  One store each: types of their own, not copies of bytes, which the compiler
// takes apart where parts of them are stored elsewhere too.
typedef uint32_t of_words __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t of_halves __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t of_two_halves __attribute__((ext_vector_type(2), aligned(2)));
struct OutF32 {
  typedef float elem;
  static constexpr bool kExact = true;         // bf16 products of converted values
  static __device__ __forceinline__ void store4(float* p, const float* v) {
    *reinterpret_cast<of_words*>(p) = (of_words){__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  }
  static __device__ __forceinline__ void store(float* p, float v) { *p = v; }
  static __device__ __forceinline__ void put4(float* p, const float* v) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
};
template <typename H>
struct OutHalf {
  typedef uint16_t elem;
  static constexpr bool kExact = false;
  static __device__ __forceinline__ uint32_t round(float v) { return H::round_any(v); }
  static __device__ __forceinline__ void store4(uint16_t* p, const float* v) {
    *reinterpret_cast<of_two_halves*>(p) = (of_two_halves){round(v[0]) | round(v[1]) << 16, round(v[2]) | round(v[3]) << 16};
  }
  static __device__ __forceinline__ void store(uint16_t* p, float v) { *p = (uint16_t)round(v); }
  static __device__ __forceinline__ void put4(uint16_t* p, const float* v) {
    *reinterpret_cast<uint2*>(p) = make_uint2(round(v[0]) | round(v[1]) << 16, round(v[2]) | round(v[3]) << 16);
  }
};
struct ToBf16 {
  static __device__ __forceinline__ uint32_t round_any(float v) { return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v); }
};
struct ToF16 {
  static __device__ __forceinline__ uint32_t round_any(float v) { return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)v); }
};

typedef uint32_t word4 __attribute__((ext_vector_type(4)));
__device__ word4 zero_piece[1];                // never written: what pieces that are none are read as

// 32 bytes of a row from `col` on, zeros from `pitch` on, or all of them; the address is chosen, not the value, which would be loaded
// in words
__device__ __forceinline__ int8v load32(const uint8_t* row, int col, int pitch, bool there = true) {
  const word4 a = *(there && col < pitch ? reinterpret_cast<const word4*>(row + col) : zero_piece);
  const word4 b = *(there && col + 16 < pitch ? reinterpret_cast<const word4*>(row + col + 16) : zero_piece);
  return int8v{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t range_of(const void* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00027000);
}
constexpr int kOutside = 1 << 30;              // of every range: read as zeros
__device__ __forceinline__ int8v load32(__amdgpu_buffer_rsrc_t range, int row, int col, int pitch) {
  const word4 a = __builtin_bit_cast(word4, __builtin_amdgcn_raw_buffer_load_b128(range, col < pitch ? row + col : kOutside, 0, 0));
  const word4 b = __builtin_bit_cast(word4, __builtin_amdgcn_raw_buffer_load_b128(range, col + 16 < pitch ? row + col + 16 : kOutside, 0, 0));
  return int8v{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

// 1 for the conversion, which looks at the exponent alone, or NaN
__device__ __forceinline__ float plain_or_nan(int byte) { return __uint_as_float((uint32_t)(byte == 255 ? 255 : 127) << 23); }
// With its power a block's values are multiples of 2^-9 times that, up to 448 times, and bf16 holds multiples of 2^-133 (conversion and
// matrix instruction keep subnormal numbers) up to 2^128.  Nodes' are taken 8 times as large and centres' an eighth, so that blocks of
// zeros, which have the least power, 2^-127, need no look at their values: exact for nodes' powers up to 2^116, and for centres' from 2^-121
// to 2^122.  Beyond are blocks of values above 4e37 and centres' blocks that lie below 1e-34, but for zeros.
constexpr int kLift = 3, kMostNode = 246 - kLift, kLeastCenter = 3 + kLift, kMostCenter = 246 + kLift;      // powers, as their bytes
__device__ __forceinline__ float node_factor(int byte) { return __uint_as_float((uint32_t)(byte == 255 ? 255 : min(byte + kLift, 254)) << 23); }
__device__ __forceinline__ float center_factor(int byte) { return __uint_as_float((uint32_t)(byte == 255 ? 255 : max(byte - kLift, 1)) << 23); }
// eight values of two words
__device__ __forceinline__ bf8 widen(int lo, int hi, float scale) {
  union {
    bf2 two[4];
    bf8 all;
  } x;
  x.two[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)lo, scale, false);
  x.two[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)lo, scale, true);
  x.two[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)hi, scale, false);
  x.two[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)hi, scale, true);
  return x.all;
}

template <int LOADS>
__device__ __forceinline__ void wait_loads() {
  static_assert(LOADS < 64, "the counter's range");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LOADS) : "memory");
}
__device__ __forceinline__ void meet() {
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// ---- few centres: rows of nodes straight into registers -----------------------
// Up to 32 centres: reading the nodes' rows is the work.  A wave takes 32 nodes and a block at a time, and asks for the next one's bytes
// before it multiplies; SPLIT waves share the blocks of a tile, and add up through LDS.  Workgroups take tiles in turn.  One centre on
// 1,000,000 nodes of 128 columns: 22 us, 5.9 TB/s (a sum of 1 GiB reads 6.0).
// fp32 scores: values go into the bf16 instruction times their powers of two, which is exact while these are of 2^-117 to 2^119; other
// powers (and blocks of zeros, which have the least) multiply the block's sums instead.

template <typename O, int SPLIT>
__global__ __launch_bounds__(256, 4) void few_kernel(ScoresArgs a, int64_t turns) {
  constexpr int kTiles = 4 / SPLIT;            // of a workgroup at once
  __shared__ float others[2][SPLIT > 1 ? kTiles * (SPLIT - 1) : 1][16][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), at = lane & 31, half = lane >> 5;
  const int part = wave % SPLIT, sub = wave / SPLIT;
  const bool asked = at < a.num_centers;
  const int64_t id = asked ? (int64_t)a.centers[at] : -1;
  const bool there = id >= 0 && id < a.num_in;
  const uint8_t *h = a.q_in + (there ? id : 0) * a.pitch, *hs = a.scales_in + (there ? id : 0) * a.scale_pitch;
  const int steps = (a.blocks + SPLIT - 1) / SPLIT;                      // of a tile
  const bool keep = steps == 1;                                          // the centres' block is the same for every tile

  struct Stage {
    int8v x[2], y[2];
    int node_power, center_power;
  } st[2];
  auto load_centers = [&](Stage& to, int block) {
    const int col = block * kBlock + half * 64;
    to.center_power = !asked ? 127 : !there ? 255 : block < a.blocks ? (int)hs[block] : 127;
#pragma unroll
    for (int s = 0; s < 2; ++s) to.y[s] = load32(h, col + 32 * s, a.pitch, there);
  };
  auto load = [&](Stage& to, int64_t turn, int k) {
    const int block = part + SPLIT * k, col = block * kBlock + half * 64;
    const int64_t first = (turn * kTiles + sub) * 32;
    const int nodes = (int)max((int64_t)0, min((int64_t)32, a.num_nodes - first));
    const int64_t from = nodes > 0 ? first : 0;
    const __amdgpu_buffer_rsrc_t rows = range_of(a.q_out + from * a.pitch, nodes * a.pitch);
    const __amdgpu_buffer_rsrc_t powers = range_of(a.scales_out + from * a.scale_pitch, nodes * a.scale_pitch);
    to.node_power = __builtin_amdgcn_raw_buffer_load_b8(powers, block < a.blocks ? at * a.scale_pitch + block : kOutside, 0, 0);
#pragma unroll
    for (int s = 0; s < 2; ++s) to.x[s] = load32(rows, at * a.pitch, col + 32 * s, a.pitch);
    if (!keep) load_centers(to, block);
  };
  acc16 acc = {};
  int64_t turn = blockIdx.x;
  int k = 0, flip = 0;
  if (keep) {
    load_centers(st[0], part);
    st[1].y[0] = st[0].y[0], st[1].y[1] = st[0].y[1], st[1].center_power = st[0].center_power;
  }
  auto finish = [&]() {
    if (SPLIT > 1) {
      if (part > 0)
#pragma unroll
        for (int t = 0; t < 16; ++t) others[flip][sub * (SPLIT - 1) + part - 1][t][lane] = acc[t];
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      meet();
      if (part == 0)
#pragma unroll
        for (int o = 0; o < SPLIT - 1; ++o)
#pragma unroll
          for (int t = 0; t < 16; ++t) acc[t] += others[flip][sub * (SPLIT - 1) + o][t][lane];
      flip ^= 1;                               // the other half is free: part 0 was done with it before it came here
    }
    const int64_t first = (turn * kTiles + sub) * 32;
    if (part == 0 && asked) {
      typename O::elem* out = static_cast<typename O::elem*>(a.out) + at * a.num_nodes + first + 4 * half;
      const float* biases = a.bias ? a.bias + first + 4 * half : nullptr;
      if (first + 32 <= a.num_nodes) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = a.scale * acc[4 * g + e];
          if (a.bias) {
            const of_words w = *reinterpret_cast<const of_words*>(biases + 8 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(w[e]) == -INFINITY ? -INFINITY : v[e] + __uint_as_float(w[e]);
          }
          O::store4(out + 8 * g, v);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int j = 8 * (e / 4) + e % 4;
          if (first + 4 * half + j >= a.num_nodes) continue;
          const float z = a.scale * acc[e], bias = a.bias ? biases[j] : 0.0f;
          O::store(out + j, bias == -INFINITY ? -INFINITY : z + bias);
        }
      }
    }
    acc = acc16{};
  };
  // one step: asks for the next, multiplies this one's; false after the last
  auto step = [&](Stage& now, Stage& next) {
    int64_t next_turn = turn;
    int next_k = k + 1;
    if (next_k == steps) next_k = 0, next_turn += gridDim.x;
    if (next_turn < turns) load(next, next_turn, next_k);
    if (O::kExact) {
      auto easy = [](int byte) { return byte == 255 || (unsigned)(byte - 10) <= 236u; };
      const bool by_values = __ballot(easy(now.node_power) && easy(now.center_power)) == ~0ull;
      const float fx = by_values ? __uint_as_float((uint32_t)now.node_power << 23) : plain_or_nan(now.node_power);
      const float fy = by_values ? __uint_as_float((uint32_t)now.center_power << 23) : plain_or_nan(now.center_power);
      acc16 sum = {};
      if (by_values) sum = acc;
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int w = 0; w < 8; w += 2)
          sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(now.x[s][w], now.x[s][w + 1], fx), widen(now.y[s][w], now.y[s][w + 1], fy), sum, 0, 0, 0);
      if (by_values) {
        acc = sum;
      } else {
#pragma unroll
        for (int t = 0; t < 16; ++t)
          acc[t] += ldexpf(sum[t], now.center_power - 254 + __shfl(now.node_power, 8 * (t / 4) + 4 * half + t % 4, 64));
      }
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s)
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(now.x[s], now.y[s], acc, 0, 0, 0, now.node_power, 0, now.center_power);
    }
    if (k + 1 == steps) finish();
    turn = next_turn, k = next_k;
    return turn < turns;
  };
  if (turn >= turns) return;
  load(st[0], turn, 0);
  while (step(st[0], st[1]) && step(st[1], st[0])) {
  }
}

// ---- many centres: tiles of both through LDS ---------------------------------
// A workgroup computes 128 x TC scores in steps of 64 columns, half a block: the loads write rows' 64 bytes to LDS themselves, two
// steps ahead, one barrier a step.  Such a load puts lane l's 16 bytes at base + 16 l, so rows cannot be padded: the four pieces of a
// row are exchanged among each other by a quarter of the row's number instead, so that 16 rows' pieces of a read lie in different
// banks (four rows make 256 bytes, all 64 banks).  Centres are copied first, in the order in which a tile reads them: its rows' 64
// bytes of a step side by side, whole lines (loads of 64 bytes each of rows reach 31 to 39 bytes a clock and compute unit, whole
// lines 54 to 60), zeros behind the rows, so that no load looks at an id; a centre that is no row has the scale NaN.
// Two workgroups of four waves share a compute unit: where one waits at its barrier, begins or writes its scores, the other multiplies.
// One of 256 x 256 with eight waves reads a third fewer bytes, but everything in it stops together: 8192 centres on 32,768 nodes of
// 2048 columns (bf16 scores) 595 us, here 582; 4096 on 50,000 of 1024 columns 301, here 270; fp32 scores of the first 1040, here 995.
// What bounds it: products and loads together.  2048 columns more cost the first case 490 us (2.24 PFLOP/s).  With one workgroup (495)
// products alone took 333 of that, with their LDS reads 390, loads alone 279, and loads and products that wait for no data 501: a load's
// way into LDS and the matrix instructions hinder each other.  Reads a step ahead, loads between products, halves of a workgroup in
// opposite phases and centres straight into registers gave 479 to 611.  Beginnings and ends of tiles are the other 90 us.
// The scores go out through LDS as well, as pieces of 16 bytes of whole rows.
// fp32 scores: both sides' values go in with their powers, nodes' lifted.  Scores of rows with a block beyond what that is exact for
// are computed once more at the end, block by block, which few tables need: 4096 centres on
// 50,000 nodes of 1024 columns take 0.45 ms, with ten such nodes 0.61 and where all are 1.7.

struct Copied {                                // of the centres, in the workspace
  uint8_t* q;                                  // [tiles][steps][centres of a tile][64]
  uint8_t* scales;                             // [padded centres][scale pitch]: blocks up to a multiple of 4
  int32_t* beyond;                             // [padded centres]: whether a block's power is
  int32_t pitch, scale_pitch;                  // pitch: 128 * blocks
  int32_t tile;                                // centres
};
constexpr int kStep = 64;                      // columns

// A workgroup of 64 lanes a row.
__global__ __launch_bounds__(64) void copy_centers_kernel(ScoresArgs a, Copied to) {
  const int64_t i = blockIdx.x;
  const int lane = threadIdx.x;
  const int64_t id = i < a.num_centers ? (int64_t)a.centers[i] : -1;
  const bool there = id >= 0 && id < a.num_in;
  bool zeros = true;                           // block `lane`
  for (int first = 0; first < to.pitch; first += 64 * 16) {
    const int col = first + lane * 16;
    uint4 w = make_uint4(0, 0, 0, 0);
    if (there && col < a.pitch) w = *reinterpret_cast<const uint4*>(a.q_in + id * a.pitch + col);
    if (col < to.pitch)
      *reinterpret_cast<uint4*>(to.q + i / to.tile * to.tile * to.pitch + (col / kStep * to.tile + i % to.tile) * kStep + col % kStep) = w;
    const uint64_t some = __ballot(((w.x | w.y | w.z | w.w) & 0x7f7f7f7fu) != 0);      // eight lanes a block
    if (lane / 8 == first / (64 * 16)) zeros = (some >> (lane % 8 * 8) & 255u) == 0;
  }
  bool beyond = false;
  if (lane < to.scale_pitch) {                 // 64 at most
    const int byte = !there ? 255 : lane < a.blocks ? (int)a.scales_in[id * a.scale_pitch + lane] : 0;
    to.scales[i * to.scale_pitch + lane] = (uint8_t)byte;
    beyond = !zeros && byte != 255 && (byte < kLeastCenter || byte > kMostCenter);
  }
  const bool any = __ballot(beyond) != 0;
  if (lane == 0) to.beyond[i] = any;
}

__device__ __forceinline__ void put_piece(float* to, const uint4& w) { *reinterpret_cast<of_words*>(to) = (of_words){w.x, w.y, w.z, w.w}; }
__device__ __forceinline__ void put_piece(uint16_t* to, const uint4& w) { *reinterpret_cast<of_halves*>(to) = (of_halves){w.x, w.y, w.z, w.w}; }
// 16 bytes of LDS from any element on
__device__ __forceinline__ uint4 read_loose(const uint8_t* from) {
  const of_halves w = *reinterpret_cast<const of_halves*>(from);
  return make_uint4(w.x, w.y, w.z, w.w);
}
constexpr int kStages = 3;                     // steps in LDS

template <typename O, int NA, int NC, int WA, int WC>
__global__ __launch_bounds__(64 * WA * WC, 2) void tile_kernel(ScoresArgs a, Copied in, int64_t tiles_c, int64_t tiles_n) {
  typedef typename O::elem elem;
  constexpr int S = kStages, TN = 32 * NA * WA, TC = 32 * NC * WC, kWaves = WA * WC;
  constexpr int kLoadsN = TN / 16 / kWaves, kLoadsC = TC / 16 / kWaves, kLoads = kLoadsN + kLoadsC;       // of 1 KB: sixteen rows
  constexpr int kPer = 16 / (int)sizeof(elem), kRowBytes = TN * (int)sizeof(elem) + 16, kRound = 32 * WC;   // of scores in LDS
  constexpr int kStageBytes = S * (TN + TC) * kStep, kBytes = kStageBytes > kRound * kRowBytes ? kStageBytes : kRound * kRowBytes;
  static_assert(kLoads * 16 * kWaves == TN + TC, "whole loads");
  __shared__ __attribute__((aligned(16))) uint8_t lds[kBytes];
  __shared__ uint8_t beyond_n[TN];             // whether a block's power is
  __shared__ bool any_beyond[kWaves];
  __shared__ __attribute__((aligned(16))) float side_bias[TN];
  uint8_t* const lds_c = lds + S * TN * kStep;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), at = lane & 31, half = lane >> 5;
  const int wa = wave % WA, wc = wave / WA;

  // Consecutive workgroups go round the eight XCDs: each of them gets neighbouring tiles, 2048 nodes at a time, so that what 32 compute
  // units read at once is in their L2 (1024 nodes: 4096 centres on 50,000 of 1024 columns 283 us instead of 270; 4096: 8192 on 32,768
  // of 2048 columns 620 instead of 582).
  const int64_t tiles = tiles_c * tiles_n, per = (tiles + 7) / 8;
  const int64_t t = (int64_t)(blockIdx.x % 8) * per + blockIdx.x / 8;
  if (blockIdx.x / 8 >= per || t >= tiles) return;
  constexpr int kGroup = 2048 / TN;
  const int64_t group = t / (kGroup * tiles_c), left = min((int64_t)kGroup, tiles_n - kGroup * group), in_group = t - group * kGroup * tiles_c;
  const int64_t c0 = in_group / left * TC, n0 = (kGroup * group + in_group % left) * TN;
  const int nodes = (int)min((int64_t)TN, a.num_nodes - n0);

  const int row_n = wave * kLoadsN * 16, row_c = wave * kLoadsC * 16;
  const __amdgpu_buffer_rsrc_t range_n = range_of(a.q_out + n0 * a.pitch, nodes * a.pitch), range_c = range_of(in.q + c0 * in.pitch, TC * in.pitch);
  // as a number: where the compiler sees that loads and reads are of one array, it lets every read wait for all loads
  const uint32_t to = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds);
  const int piece = ((lane & 3) ^ (lane >> 4)) * 16;
  const int at_row = (row_n + (lane >> 2)) * a.pitch + piece, at_piece = (row_c + (lane >> 2)) * kStep + piece;
  auto load = [&](const __amdgpu_buffer_rsrc_t& range, uint32_t place, int from) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(range, (__attribute__((address_space(3))) void*)(uintptr_t)(to + place), 16, from, 0, 0, 0);
  };
  auto issue = [&](int step, int buf) {
#pragma unroll
    for (int n = 0; n < kLoadsN; ++n)
      load(range_n, (buf * TN + row_n + n * 16) * kStep, step * kStep + piece < a.pitch ? at_row + step * kStep + n * 16 * a.pitch : kOutside);
#pragma unroll
    for (int n = 0; n < kLoadsC; ++n)
      load(range_c, (S * TN + buf * TC + row_c + n * 16) * kStep, step < 2 * a.blocks ? at_piece + (step * TC + n * 16) * kStep : kOutside);
  };
#pragma unroll
  for (int s = 0; s < S - 1; ++s) issue(s, s);

  // ---- scales: of a lane's rows, four blocks at a time
  const uint8_t *scales_c = in.scales + c0 * in.scale_pitch, *scales_n = a.scales_out + n0 * a.scale_pitch;
  int scale_n[NA];
  const int scale_c = (wc * NC * 32 + at) * in.scale_pitch;
#pragma unroll
  for (int m = 0; m < NA; ++m) scale_n[m] = min((wa * NA + m) * 32 + at, nodes - 1) * a.scale_pitch;
  auto four = [&](int m, int block) { return *reinterpret_cast<const uint32_t*>(scales_n + scale_n[m] + block); };      // three blocks and more
  if (O::kExact) {
    bool any = false;
#pragma unroll
    for (int n = 0; n < NC; ++n) any |= in.beyond[c0 + (wc * NC + n) * 32 + at] != 0;
#pragma unroll
    for (int m = 0; m < NA; ++m) {
      int top = 0;
      for (int b = 0; b < a.blocks; b += 4) {
        const uint32_t w = four(m, b);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int byte = (int)((w >> (8 * k)) & 255u);
          top = max(top, byte == 255 ? 0 : byte);
        }
      }
      any |= top > kMostNode;
      if (wc == 0 && half == 0) beyond_n[(wa * NA + m) * 32 + at] = top > kMostNode;
    }
    any = __ballot(any) != 0;
    if (lane == 0) any_beyond[wave] = any;
  }
  if (a.bias)
    for (int i = tid; i < nodes; i += 64 * kWaves) side_bias[i] = a.bias[n0 + i];
  uint32_t sn[NA], sc[NC], next_n[NA], next_c[NC];
  auto fetch_scales = [&](int block) {
#pragma unroll
    for (int n = 0; n < NC; ++n) next_c[n] = *reinterpret_cast<const uint32_t*>(scales_c + scale_c + n * 32 * in.scale_pitch + block);
#pragma unroll
    for (int m = 0; m < NA; ++m) next_n[m] = four(m, block);
  };
  fetch_scales(0);

  // ---- products: pieces 2 half and 2 half + 1 of a row
  const int in_row = ((2 * half) ^ ((at >> 2) & 3)) * 16;
  const int at_n[2] = {(wa * NA * 32 + at) * kStep + in_row, (wa * NA * 32 + at) * kStep + (in_row ^ 16)};
  const int at_c[2] = {(wc * NC * 32 + at) * kStep + in_row, (wc * NC * 32 + at) * kStep + (in_row ^ 16)};
  acc16 acc[NA][NC];
#pragma unroll
  for (int m = 0; m < NA; ++m)
#pragma unroll
    for (int n = 0; n < NC; ++n) acc[m][n] = acc16{};
  auto pair = [&](const uint8_t* base, const int* place, int more) {
    const uint4 p = *reinterpret_cast<const uint4*>(base + place[0] + more), q = *reinterpret_cast<const uint4*>(base + place[1] + more);
    return int8v{(int)p.x, (int)p.y, (int)p.z, (int)p.w, (int)q.x, (int)q.y, (int)q.z, (int)q.w};
  };
  int buf = 0;
  auto step = [&](int k) {
    wait_loads<(S - 2) * kLoads>();            // this step's rows; those of later ones may be under way
    meet();
    issue(k + S - 1, buf == 0 ? S - 1 : buf - 1);      // where the step before was read
    int8v x[NA], y[NC];
#pragma unroll
    for (int n = 0; n < NC; ++n) y[n] = pair(lds_c + buf * TC * kStep, at_c, n * 32 * kStep);
#pragma unroll
    for (int m = 0; m < NA; ++m) x[m] = pair(lds + buf * TN * kStep, at_n, m * 32 * kStep);
    buf = buf == S - 1 ? 0 : buf + 1;
    if (O::kExact) {
      float fx[NA], fy[NC];
#pragma unroll
      for (int m = 0; m < NA; ++m) fx[m] = node_factor((int)(sn[m] & 255u));
#pragma unroll
      for (int n = 0; n < NC; ++n) fy[n] = center_factor((int)(sc[n] & 255u));
#pragma unroll
      for (int w = 0; w < 8; w += 2) {
        bf8 u[NA], v[NC];
#pragma unroll
        for (int n = 0; n < NC; ++n) v[n] = widen(y[n][w], y[n][w + 1], fy[n]);
#pragma unroll
        for (int m = 0; m < NA; ++m) {
          u[m] = widen(x[m][w], x[m][w + 1], fx[m]);
#pragma unroll
          for (int n = 0; n < NC; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(u[m], v[n], acc[m][n], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int m = 0; m < NA; ++m)
#pragma unroll
        for (int n = 0; n < NC; ++n)
          acc[m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x[m], y[n], acc[m][n], 0, 0, 0, (int)sn[m], 0, (int)sc[n]);
    }
  };
  static_assert(kBlock == 2 * kStep, "two steps a block");
  for (int block = 0; block < a.blocks; ++block) {
    if ((block & 3) == 0) {
#pragma unroll
      for (int m = 0; m < NA; ++m) sn[m] = next_n[m];
#pragma unroll
      for (int n = 0; n < NC; ++n) sc[n] = next_c[n];
      if (block + 4 < a.blocks) fetch_scales(block + 4);
    }
    step(2 * block);
    step(2 * block + 1);
#pragma unroll
    for (int m = 0; m < NA; ++m) sn[m] >>= 8;
#pragma unroll
    for (int n = 0; n < NC; ++n) sc[n] >>= 8;
  }

  // ---- scores: register 4 g + k of a block is node 8 g + 4 half + k, a lane's centre is ... + at
  elem* out = static_cast<elem*>(a.out);
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    wait_loads<0>();                           // also what was asked for beyond the last step: it lands where the scores go
    meet();
#pragma unroll
    for (int m = 0; m < NA; ++m)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int j = (wa * NA + m) * 32 + 8 * g + 4 * half;
        float v[4], bias[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (a.bias) __builtin_memcpy(bias, &side_bias[j], 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float z = a.scale * acc[m][n][4 * g + k] + bias[k];
          v[k] = bias[k] == -INFINITY ? -INFINITY : z;
        }
        O::put4(reinterpret_cast<elem*>(lds + (wc * 32 + at) * kRowBytes) + j, v);
      }
    wait_loads<0>();
    meet();
    constexpr int kLanes = TN / kPer;          // of a row
    if (nodes == TN) {
      for (int p = tid; p < kRound * kLanes; p += 64 * kWaves) {
        const int r = p / kLanes, j = (p - r * kLanes) * kPer;
        const int64_t i = c0 + (r / 32 * NC + n) * 32 + r % 32;
        const uint4 w = *reinterpret_cast<const uint4*>(lds + r * kRowBytes + j * (int)sizeof(elem));
        if (i < a.num_centers) put_piece(out + i * a.num_nodes + n0 + j, w);
      }
    } else {
      for (int p = tid; p < kRound * TN; p += 64 * kWaves) {
        const int r = p / TN, j = p - r * TN;
        const int64_t i = c0 + (r / 32 * NC + n) * 32 + r % 32;
        if (i < a.num_centers && j < nodes) out[i * a.num_nodes + n0 + j] = reinterpret_cast<const elem*>(lds + r * kRowBytes)[j];
      }
    }
  }
  if constexpr (O::kExact) {
    bool any = false;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) any |= any_beyond[w];
    if (!any) return;
    wait_loads<0>();                           // the stores of all waves: some of them are replaced
    meet();
    for (int sub = wave; sub < TN / 32 * (TC / 32); sub += kWaves) {         // 32 x 32 scores
      const int j0 = sub % (TN / 32) * 32, r = sub / (TN / 32) * 32 + at;
      const int64_t i = c0 + r;
      const bool beyond_c = in.beyond[i] != 0;
      if (__ballot(beyond_c || beyond_n[j0 + at]) == 0) continue;
      const uint8_t* row_c = in.q + c0 * in.pitch + r * kStep;
      acc16 z = {};
      for (int block = 0; block < a.blocks; ++block) {
        const int power = scales_n[min(j0 + at, nodes - 1) * a.scale_pitch + block], power_c = in.scales[i * in.scale_pitch + block];
        acc16 sum = {};
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int col = block * kBlock + half * kStep + s * 32;
          const int8v x = load32(range_n, (j0 + at) * a.pitch, col, a.pitch), y = load32(row_c + (2 * block + half) * TC * kStep, s * 32, kStep);
#pragma unroll
          for (int w = 0; w < 8; w += 2)
            sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(x[w], x[w + 1], plain_or_nan(power)), widen(y[w], y[w + 1], plain_or_nan(power_c)), sum, 0, 0, 0);
        }
#pragma unroll
        for (int t = 0; t < 16; ++t) z[t] += ldexpf(sum[t], power_c - 254 + __shfl(power, 8 * (t / 4) + 4 * half + t % 4, 64));
      }
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        const int j = j0 + 8 * (t / 4) + 4 * half + t % 4;
        if (i >= a.num_centers || j >= nodes || !(beyond_c || beyond_n[j])) continue;
        const float bias = a.bias ? side_bias[j] : 0.0f;
        out[i * a.num_nodes + n0 + j] = bias == -INFINITY ? -INFINITY : a.scale * z[t] + bias;
      }
    }
  }
}

// ---- narrow rows: centres kept in registers, nodes streamed ---------------------
// One or two blocks (256 columns): the scores are more bytes than the rows, and writing them is the work.  Four waves keep 32 * KC
// centres each, as the right operand; a fifth asks for the nodes' rows, 64 at a time and three tiles ahead, with their scales and
// biases, into LDS, and is the only one that waits for memory: the others' stores are never waited for.  One barrier a tile.  A
// workgroup has a range of neighbouring nodes: what it writes of a row grows along the row, so that lines that two tiles share
// meet in L2.  A wave turns 16 or 32 centres' scores in LDS of its own and writes them as pieces of 16 bytes of whole rows.  256
// centres on 1,000,000 nodes of 128 columns, fp32 scores: 245 us, 4.7 TB/s read and written (a copy 5.1, a fill 6.9).

template <typename O, int BL, bool CARRY>
struct Strip {
  static constexpr int kWaves = 4, kThreads = 64 * (kWaves + 1);                    // and the one that loads
  static constexpr int kSize = (int)sizeof(typename O::elem);
  static constexpr int kNodes = 64, kSlots = BL == 1 && !CARRY ? 4 : 3, kAhead = kSlots - 1;
  static constexpr int kRows = kNodes * kBlock * BL, kSlotBytes = kRows + 512;      // rows, scales, biases
  static constexpr int kLoads = kRows / 1024 + 2;
  static constexpr int kPer = 16 / kSize, kLanes = kNodes / kPer;                   // of a row of scores
  static constexpr int kRowBytes = kNodes * kSize + (CARRY ? 128 : 0) + 16;
  static constexpr int kTurn = BL == 1 || CARRY ? 32 : 16;                          // rows that a wave turns at once
};

template <typename O, int BL, int KC, bool CARRY>
__global__ __launch_bounds__(320, 2) void strip_kernel(ScoresArgs a, int64_t groups_c, int64_t ranges, int64_t tiles_per_range) {
  typedef Strip<O, BL, CARRY> S;
  static_assert(!CARRY || KC == 1, "a wave keeps what is left of each of its rows");
  typedef typename O::elem elem;
  __shared__ __attribute__((aligned(16))) uint8_t slots[S::kSlots][S::kSlotBytes];
  __shared__ __attribute__((aligned(16))) uint8_t turn[S::kWaves][S::kTurn * S::kRowBytes];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), at = lane & 31, half = lane >> 5;
  // XCD x has an eighth of the nodes.  Its workgroups take tiles in turn; with CARRY each has a range of neighbouring ones.
  const int64_t all_tiles = (a.num_nodes + S::kNodes - 1) / S::kNodes, xcd = blockIdx.x % 8, u = blockIdx.x / 8, group = u % groups_c;
  const int64_t of_xcd = min((xcd + 1) * tiles_per_range, all_tiles);      // the end of its tiles
  const int64_t chunk = (tiles_per_range + ranges - 1) / ranges, every = CARRY ? 1 : ranges;
  const int64_t first = xcd * tiles_per_range + u / groups_c * (CARRY ? chunk : 1), last = CARRY ? min(first + chunk, of_xcd) : of_xcd;
  if (first >= last) return;

  if (wave == S::kWaves) {                     // the wave that loads
    const int row = (lane >> 3) * a.pitch, piece = ((lane & 7) ^ (lane >> 4)) * 16;
    int next = 0;                              // slot
    auto issue = [&](int64_t t) {
      uint8_t* slot = slots[next];
      next = next + 1 == S::kSlots ? 0 : next + 1;
      const int64_t n0 = t * S::kNodes;
      const int nodes = (int)max((int64_t)0, min((int64_t)S::kNodes, a.num_nodes - n0));
      const int64_t from = t < last ? n0 : 0;  // beyond the range: nothing, but as many loads
      const int rows = t < last ? nodes : 0;
      const __amdgpu_buffer_rsrc_t q = range_of(a.q_out + from * a.pitch, rows * a.pitch);
#pragma unroll
      for (int b = 0; b < BL; ++b)
#pragma unroll
        for (int c = 0; c < S::kNodes / 8; ++c) {
          const int col = b * kBlock + (piece ^ (c & 1 ? 64 : 0));
          __builtin_amdgcn_raw_ptr_buffer_load_lds(q, (__attribute__((address_space(3))) void*)(slot + b * S::kNodes * kBlock + c * 1024), 16,
                                                   col < a.pitch ? row + c * 8 * a.pitch + col : kOutside, 0, 0, 0);
        }
      // whole words of scales: the last one's bytes beyond the table lie in a word that the table has a part of
      const __amdgpu_buffer_rsrc_t e = range_of(a.scales_out + from * BL, (rows * BL + 3) / 4 * 4);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(e, (__attribute__((address_space(3))) void*)(slot + S::kRows), 4, lane * 4, 0, 0, 0);
      const __amdgpu_buffer_rsrc_t f = range_of(a.bias ? static_cast<const void*>(a.bias + from) : a.q_out, a.bias ? rows * 4 : 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(f, (__attribute__((address_space(3))) void*)(slot + S::kRows + 256), 4, lane * 4, 0, 0, 0);
    };
    for (int s = 0; s < S::kAhead; ++s) issue(first + s * every);
    for (int64_t t = first; t < last; t += every) {
      wait_loads<(S::kAhead - 1) * S::kLoads>();
      meet();
      issue(t + S::kAhead * every);                    // where the tile before was read
    }
    wait_loads<0>();                           // nothing may land in LDS after the workgroup
    return;
  }

  // ---- centres: pieces 4 s + 2 half, + 1 of a block's eight
  const int64_t c0 = (group * S::kWaves + wave) * 32 * KC;
  int8v kept[O::kExact ? 1 : KC][BL * 2];
  bf8 wide[O::kExact ? KC : 1][BL * 8];
  int scale_c[KC][BL];
  bool zeros[KC][BL];                          // what the lane holds of a block
#pragma unroll
  for (int n = 0; n < KC; ++n) {
    const int64_t i = c0 + n * 32 + at, id = i < a.num_centers ? (int64_t)a.centers[i] : -1;
    const bool there = id >= 0 && id < a.num_in;
    const uint8_t *h = a.q_in + (there ? id : 0) * a.pitch, *e = a.scales_in + (there ? id : 0) * BL;
#pragma unroll
    for (int b = 0; b < BL; ++b) scale_c[n][b] = there ? e[b] : 255, zeros[n][b] = there;
#pragma unroll
    for (int k = 0; k < BL * 2; ++k) {
      const int8v x = load32(h, (k >> 1) * kBlock + (k & 1) * 64 + half * 32, a.pitch);
      if (O::kExact) {
#pragma unroll
        for (int w = 0; w < 8; ++w) zeros[n][k >> 1] = zeros[n][k >> 1] && (x[w] & 0x7f7f7f7f) == 0;
#pragma unroll
        for (int w = 0; w < 8; w += 2) wide[n][k * 4 + w / 2] = widen(x[w], x[w + 1], plain_or_nan(scale_c[n][k >> 1]));
      } else {
        kept[n][k] = x;
      }
    }
  }

  float factor_c[KC][BL];
  bool near_c = true;
#pragma unroll
  for (int n = 0; n < KC; ++n)
#pragma unroll
    for (int b = 0; b < BL; ++b) {
      factor_c[n][b] = center_factor(scale_c[n][b]) * a.scale;
      const bool fits = scale_c[n][b] - 27u <= 173u && factor_c[n][b] >= 0x1p-126f && factor_c[n][b] <= 0x1p126f;
      if (!fits) factor_c[n][b] = 0.0f;        // of zeros, where it is used
      near_c = near_c && (fits || zeros[n][b]);
    }
  near_c = __ballot(near_c) == ~0ull;
  uint8_t* const mine = turn[wave];
  const int rows = (int)min((int64_t)32 * KC, a.num_centers - c0);      // may be none, or fewer
  elem* const out = static_cast<elem*>(a.out);
  // pieces of the nodes: by half the row's number
  int at_n[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) at_n[c] = at * kBlock + (((4 * (c >> 1) + 2 * half + (c & 1)) ^ ((at >> 1) & 7)) * 16);
  int at_slot = 0;
  for (int64_t t = first; t < last; t += every) {
    meet();
    const uint8_t* slot = slots[at_slot];
    at_slot = at_slot + 1 == S::kSlots ? 0 : at_slot + 1;
    const uint8_t* side = slot + S::kRows;
    const int64_t n0 = t * S::kNodes;
    const int nodes = (int)min((int64_t)S::kNodes, a.num_nodes - n0);
    // fp32 scores: a sum for each block, times the centre's power, so that no block's size matters to another's.  The node's power goes in
    // with its values, which is exact and leaves sums below 2^121, but for blocks of values above 4e30 and of NaN; and the centre's is a
    // factor, but for blocks of NaN, and those below 3e-28 or above 4e24 that are no zeros.  Otherwise both multiply the sums of the
    // plain values.
    constexpr int kSums = O::kExact ? BL : 1;
    acc16 acc[kSums][2][KC];
    int byte[2][BL];
    bool near = true;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
#pragma unroll
      for (int b = 0; b < kSums; ++b)
#pragma unroll
        for (int n = 0; n < KC; ++n) acc[b][m][n] = acc16{};
#pragma unroll
      for (int b = 0; b < BL; ++b) {
        byte[m][b] = side[(m * 32 + at) * BL + b];
        near = near && byte[m][b] <= 220;
      }
    }
    const bool factors = !O::kExact || (__ballot(near) == ~0ull && near_c);
    float factor_n[2][BL];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int b = 0; b < BL; ++b) factor_n[m][b] = factors ? node_factor(byte[m][b]) : plain_or_nan(byte[m][b]);
#pragma unroll
    for (int k = 0; k < BL * 2; ++k) {
      int8v x[2];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const uint8_t* from = slot + (k >> 1) * S::kNodes * kBlock + m * 32 * kBlock;
        const uint4 p = *reinterpret_cast<const uint4*>(from + at_n[(k & 1) * 2]), q = *reinterpret_cast<const uint4*>(from + at_n[(k & 1) * 2 + 1]);
        x[m] = int8v{(int)p.x, (int)p.y, (int)p.z, (int)p.w, (int)q.x, (int)q.y, (int)q.z, (int)q.w};
      }
      if (O::kExact) {
#pragma unroll
        for (int w = 0; w < 8; w += 2)
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            const bf8 u = widen(x[m][w], x[m][w + 1], factor_n[m][k >> 1]);
#pragma unroll
            for (int n = 0; n < KC; ++n)
              acc[O::kExact ? k >> 1 : 0][m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(u, wide[n][k * 4 + w / 2], acc[O::kExact ? k >> 1 : 0][m][n], 0, 0, 0);
          }
      } else {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int n = 0; n < KC; ++n)
            acc[0][m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x[m], kept[n][k], acc[0][m][n], 0, 0, 0, byte[m][k >> 1], 0, scale_c[n][k >> 1]);
      }
    }
    // Register 4 g + k of a block is node 8 g + 4 half + k, a lane's centre is ... + at.
    auto finish = [&](auto by_factors, auto with_bias) {
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int j = m * 32 + 8 * g + 4 * half;
          float bias[4] = {0.0f, 0.0f, 0.0f, 0.0f};
          uint32_t power[4][BL];
          if constexpr (decltype(with_bias)::value) __builtin_memcpy(bias, side + 256 + 4 * j, 16);
          if constexpr (O::kExact && !decltype(by_factors)::value) {
            uint32_t w[BL];
            __builtin_memcpy(w, side + j * BL, 4 * BL);
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int b = 0; b < BL; ++b) power[k][b] = (w[(k * BL + b) / 4] >> (8 * ((k * BL + b) % 4))) & 255u;
          }
#pragma unroll
          for (int n = 0; n < KC; ++n)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              float z = 0.0f;
              if constexpr (!O::kExact) {
                z = fmaf(acc[0][m][n][4 * g + k], a.scale, bias[k]);
              } else if constexpr (decltype(by_factors)::value) {
                z = bias[k];
#pragma unroll
                for (int b = 0; b < BL; ++b) z = fmaf(acc[b][m][n][4 * g + k], factor_c[n][b], z);
              } else {
#pragma unroll
                for (int b = 0; b < BL; ++b) z += ldexpf(acc[b][m][n][4 * g + k], (int)power[k][b] + scale_c[n][b] - 254);
                z = fmaf(z, a.scale, bias[k]);
              }
              if constexpr (decltype(with_bias)::value) z = bias[k] == -INFINITY ? -INFINITY : z;
              acc[0][m][n][4 * g + k] = z;
            }
        }
    };
    if (factors) {
      if (a.bias) finish(std::true_type{}, std::true_type{});
      else finish(std::true_type{}, std::false_type{});
    } else {
      if (a.bias) finish(std::false_type{}, std::true_type{});
      else finish(std::false_type{}, std::false_type{});
    }
#pragma unroll
    for (int n = 0; n < KC; ++n)
#pragma unroll
      for (int r = 0; r < 32 / S::kTurn; ++r) {
        wave_fence();
        if (S::kTurn == 32 || at / S::kTurn == r) {
          elem* to = reinterpret_cast<elem*>(mine + at % S::kTurn * S::kRowBytes + (CARRY ? 128 : 0));
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const float v[4] = {acc[0][m][n][4 * g], acc[0][m][n][4 * g + 1], acc[0][m][n][4 * g + 2], acc[0][m][n][4 * g + 3]};
              O::put4(to + m * 32 + 8 * g + 4 * half, v);
            }
        }
        wave_fence();
        if constexpr (CARRY) {
          // A row's buffer: the last line's worth of the tile before, then this tile.  From the line on that holds the tile's first
          // node, 64 scores go out as whole lines; what lies behind goes with the next tile.
          const int row = lane / S::kLanes, piece = lane % S::kLanes * 16;
          const uint8_t* from = mine + row * S::kRowBytes + 128 + piece;
          elem* node = out + (c0 + row) * a.num_nodes + n0;
          constexpr int kStep = 64 / S::kLanes;        // rows of a store
          if (t > first && t + 1 < last) {
#pragma unroll
            for (int p = 0; p < 32 / kStep; ++p) {
              const int back = (int)(reinterpret_cast<uintptr_t>(node) & 127);
              if (row < rows - p * kStep)
                *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(node) - back + piece) = read_loose(from + p * kStep * S::kRowBytes - back);
              node += kStep * a.num_nodes;
              asm("" : "+v"(node));
            }
          } else {
#pragma unroll 1
            for (int p = 0; p < 32 / kStep; ++p, node += kStep * a.num_nodes) {
              const int back = (int)(reinterpret_cast<uintptr_t>(node) & 127);
              for (int more = 0; more < (t + 1 < last ? 1 : 2); ++more) {       // the last tile: to its end
                const int at0 = (piece + more * 64 * S::kSize - back) / S::kSize;      // of the piece, among the tile's nodes
                if (row >= rows - p * kStep || at0 >= nodes) continue;
                const uint4 w = read_loose(from + p * kStep * S::kRowBytes + more * 64 * S::kSize - back);
                elem e[S::kPer];
                __builtin_memcpy(e, &w, 16);
#pragma unroll
                for (int k = 0; k < S::kPer; ++k)
                  if ((t > first || at0 + k >= 0) && at0 + k < (t + 1 < last ? S::kNodes : nodes)) node[at0 + k] = e[k];
              }
            }
          }
          wave_fence();
          uint4 kept_back[4];
#pragma unroll
          for (int p = 0; p < 4; ++p) kept_back[p] = *reinterpret_cast<const uint4*>(mine + (p * 8 + lane / 8) * S::kRowBytes + S::kNodes * S::kSize + lane % 8 * 16);
#pragma unroll
          for (int p = 0; p < 4; ++p) *reinterpret_cast<uint4*>(mine + (p * 8 + lane / 8) * S::kRowBytes + lane % 8 * 16) = kept_back[p];
          continue;
        }
        const int row0 = n * 32 + r * S::kTurn;
        if (nodes == S::kNodes) {
          const int row = lane / S::kLanes;
          elem* to = out + (c0 + row0 + row) * a.num_nodes + n0 + lane % S::kLanes * S::kPer;
          const uint8_t* from = mine + row * S::kRowBytes + lane % S::kLanes * 16;
#pragma unroll
          for (int p = 0; p < S::kTurn * S::kLanes / 64; ++p) {
            constexpr int kStep = 64 / S::kLanes;      // rows of a store
            if (row < rows - row0 - p * kStep) put_piece(to, *reinterpret_cast<const uint4*>(from + p * kStep * S::kRowBytes));
            to += kStep * a.num_nodes;
            asm("" : "+v"(to));                // one address at a time: kept for all of them they would not fit the registers
          }
        } else if (lane < nodes) {
          elem* to = out + (c0 + row0) * a.num_nodes + n0 + lane;
#pragma unroll 1
          for (int row = 0; row < min(S::kTurn, rows - row0); ++row, to += a.num_nodes)
            *to = reinterpret_cast<const elem*>(mine + row * S::kRowBytes)[lane];
        }
      }
  }
}

bool dtype_known(int32_t dtype) { return dtype == GS_F32 || dtype == GS_BF16 || dtype == GS_F16; }

bool shape_ok(int64_t num_centers, int64_t num_nodes, int32_t dim) {
  return num_centers >= 0 && num_centers <= (int64_t)INT32_MAX && num_nodes >= 1 && num_nodes <= (int64_t)INT32_MAX && dim >= 1 && dim <= GS_Q8_MAX_DIM;
}

}  // namespace
}  // namespace gs

using namespace gs;

namespace gs {
namespace {

constexpr int kFew = 32;                       // centres at most that take no tiles
constexpr int kNarrow = 128;                   // that take tiles of 128
struct ScoresPlan {
  bool few;
  int64_t padded;
  Copied in;
  size_t bytes;
};
ScoresPlan plan_scores(void* ws, int64_t num_centers, int32_t dim) {
  ScoresPlan p{};
  p.few = num_centers <= kFew;
  p.bytes = 256;
  if (p.few || dim <= 2 * kBlock) return p;
  p.padded = ceil_div(num_centers, 256) * 256;
  const int blocks = (int)ceil_div(dim, kBlock);
  p.in.pitch = blocks * kBlock, p.in.scale_pitch = (blocks + 3) / 4 * 4, p.in.tile = num_centers <= kNarrow ? 128 : 256;
  Carver carve(ws);
  p.in.q = carve.take<uint8_t>((size_t)p.padded * p.in.pitch);
  p.in.scales = carve.take<uint8_t>((size_t)p.padded * p.in.scale_pitch);
  p.in.beyond = carve.take<int32_t>((size_t)p.padded);
  p.bytes = carve.used;
  return p;
}

template <typename O, int NA, int NC, int WA, int WC>
int32_t run_tiles(const ScoresArgs& a, const ScoresPlan& p, hipStream_t s) {
  const int64_t c = ceil_div(a.num_centers, 32 * NC * WC), n = ceil_div(a.num_nodes, 32 * NA * WA);
  if (ceil_div(c * n, 8) * 8 * (64 * WA * WC) >= (int64_t)1 << 32) return GS_EOVERFLOW;      // a launch takes fewer lanes
  copy_centers_kernel<<<dim3((unsigned)p.padded), 64, 0, s>>>(a, p.in);
  GS_LAUNCH_CHECK();
  tile_kernel<O, NA, NC, WA, WC><<<dim3((unsigned)(ceil_div(c * n, 8) * 8)), 64 * WA * WC, 0, s>>>(a, p.in, c, n);
  GS_LAUNCH_CHECK();
  return GS_OK;
}

template <typename O, int BL, int KC, bool CARRY>
int32_t run_strip(const ScoresArgs& a, int64_t per_xcd, int64_t groups, int64_t ranges, hipStream_t s) {
  if (groups * ranges * 8 > (int64_t)INT32_MAX) return GS_EOVERFLOW;
  strip_kernel<O, BL, KC, CARRY><<<dim3((unsigned)(groups * ranges * 8)), Strip<O, BL, CARRY>::kThreads, 0, s>>>(a, groups, ranges, per_xcd);
  GS_LAUNCH_CHECK();
  return GS_OK;
}

// Rows of one or two blocks.
template <typename O>
int32_t run_strips(const ScoresArgs& a, hipStream_t s) {
  const bool two = a.blocks == 2, wide = a.num_centers > 128 && !(two && O::kExact);      // 64 centres a wave, where registers hold them
  const int64_t per_xcd = ceil_div(ceil_div(a.num_nodes, 64), 8);
  auto ranges = [&](int64_t groups, int64_t workgroups, int64_t least) {   // of an XCD, of so many tiles at least
    return std::max<int64_t>(1, std::min(ceil_div(workgroups, groups * 8), per_xcd / least));
  };
  const int64_t groups = ceil_div(a.num_centers, wide ? 256 : 128), rows = ceil_div(a.num_centers, 128);
  // Rows of scores that begin inside lines: long ranges keep the ends of their lines for the next tile.  256 centres on 1,000,003 nodes
  // of 128 columns: 335 -> 275 us (fp32 scores), 190 -> 161 (bf16); shorter ranges lose more at their own ends (40 on 300,001: 17 -> 27).
  const bool lines = a.num_nodes * (int64_t)sizeof(typename O::elem) % 128 == 0 && aligned(a.out, 128);
  const int64_t few = ranges(rows, 256, 1);
  if (!two && !lines && per_xcd / few >= 48) return run_strip<O, 1, 1, true>(a, per_xcd, rows, few, s);
  const int64_t r = ranges(groups, wide ? 256 : 512, 8);      // one workgroup of 64 centres a wave fits a compute unit's registers
  if (two) {
    if constexpr (!O::kExact)
      if (wide) return run_strip<O, 2, 2, false>(a, per_xcd, groups, r, s);
    return run_strip<O, 2, 1, false>(a, per_xcd, groups, r, s);
  }
  return wide ? run_strip<O, 1, 2, false>(a, per_xcd, groups, r, s) : run_strip<O, 1, 1, false>(a, per_xcd, groups, r, s);
}

template <typename O>
int32_t run_scores(const ScoresArgs& a, const ScoresPlan& p, hipStream_t s) {
  if (p.few) {
    const int split = a.blocks >= 3 ? 4 : a.blocks;
    const int64_t turns = ceil_div(a.num_nodes, 32 * (4 / split));
    const dim3 grid((unsigned)std::min<int64_t>(turns, 1024));
    if (split == 1) few_kernel<O, 1><<<grid, 256, 0, s>>>(a, turns);
    if (split == 2) few_kernel<O, 2><<<grid, 256, 0, s>>>(a, turns);
    if (split == 4) few_kernel<O, 4><<<grid, 256, 0, s>>>(a, turns);
    GS_LAUNCH_CHECK();
    return GS_OK;
  }
  if (a.blocks <= 2) return run_strips<O>(a, s);
  if (a.num_centers <= kNarrow) return run_tiles<O, 2, 2, 2, 2>(a, p, s);
  return run_tiles<O, 4, 2, 1, 4>(a, p, s);
}

}  // namespace
}  // namespace gs

extern "C" size_t gs_scores_q8_workspace_bytes(int64_t num_centers, int64_t num_nodes, int32_t dim) {
  if (!shape_ok(num_centers, num_nodes, dim)) return 0;
  return plan_scores(nullptr, num_centers, dim).bytes;
}

extern "C" int32_t gs_scores_q8(const void* q_in, const void* scales_in, int64_t num_in, const void* q_out, const void* scales_out,
                                int64_t num_nodes, int32_t dim, const int32_t* centers, int64_t num_centers, const float* bias, float scale,
                                void* scores_out, int32_t dtype, void* ws, size_t ws_bytes, void* stream) {
  if (!shape_ok(num_centers, num_nodes, dim) || !dtype_known(dtype) || num_in < 1 || num_in > (int64_t)INT32_MAX) return GS_EINVAL;
  if (!q_in || !q_out || !scales_in || !scales_out || !aligned(q_in, 16) || !aligned(q_out, 16) || !aligned(scales_in, 4) || !aligned(scales_out, 4))
    return GS_EINVAL;
  if (!(scale > 0.0f) || !std::isfinite(scale) || !ws || !aligned(ws, 256)) return GS_EINVAL;
  if (num_centers > 0 && (!centers || !scores_out)) return GS_EINVAL;
  if (!aligned(scores_out, dtype == GS_F32 ? 4 : 2) || !aligned(bias, 4) || !aligned(centers, 4)) return GS_EINVAL;
  const ScoresPlan p = plan_scores(ws, num_centers, dim);
  if (ws_bytes < p.bytes) return GS_EWORKSPACE;
  if (num_centers >= (int64_t)1 << 21) return GS_EOVERFLOW;
  if (num_centers == 0) return GS_OK;
  const ScoresArgs a{static_cast<const uint8_t*>(q_in), static_cast<const uint8_t*>(scales_in), num_in, static_cast<const uint8_t*>(q_out),
                     static_cast<const uint8_t*>(scales_out), num_nodes, gs_q8_pitch(dim), (int32_t)ceil_div(dim, kBlock), gs_q8_scale_pitch(dim),
                     centers, num_centers, bias, scale, scores_out};
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == GS_F32) return run_scores<OutF32>(a, p, s);
  if (dtype == GS_BF16) return run_scores<OutHalf<ToBf16>>(a, p, s);
  return run_scores<OutHalf<ToF16>>(a, p, s);
}
