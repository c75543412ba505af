// gs_scores_q8: scores of centres against every node, from 8-bit rows.
//
//   z_ij = scale * sum_b 2^(e_ib + f_jb) sum_{k in block b} a_ik c_jk + bias_j
//
// a, c: e4m3 values; e, f: the powers of two of their blocks of 128 columns.  Two kinds of products:
//   fp32 scores: the values go through v_cvt_scalef32_pk_bf16_fp8 into the bf16 matrix instruction, whose products of them are exact
//     and whose sums are fp32.  The conversion multiplies by powers of two as well: by a block's relative to its row's largest, so
//     that nothing leaves bf16's range; the rows' largest ones multiply the sum.
//   16-bit scores: v_mfma_scale_f32_32x32x64 on the bytes themselves, which multiplies by the powers of the blocks and runs at twice
//     the rate.  Of eight neighbouring products it drops what lies 2^13 below the largest of them (measured, and so do the 8-bit
//     instructions without scales): at most 7 * 2^-13 of the sum of the products' sizes, some 2^-16 of it for Gaussian rows; fp32
//     scores would keep 16 bits, while fp16 keeps 11 and bf16 8 of any.
// Both instructions sum over any numbering of a block's columns, as long as both operands use the same one: a lane takes 64
// neighbouring bytes of a row's 128.  Nodes are the left operand: a lane then holds four neighbouring nodes' scores of one centre,
// which lie together in memory.

#include "common.h"

#include <cmath>

namespace gs {
namespace {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef float acc16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
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

struct OutF32 {
  typedef float elem;
  static constexpr bool kExact = true;         // bf16 products of converted values
  static __device__ __forceinline__ void store4(float* p, const float* v) { __builtin_memcpy(p, v, 16); }
  static __device__ __forceinline__ void store(float* p, float v) { *p = v; }
  static __device__ __forceinline__ void put4(float* p, const float* v) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
};
template <typename H>
struct OutHalf {
  typedef uint16_t elem;
  static constexpr bool kExact = false;
  static __device__ __forceinline__ uint32_t round(float v) { return H::round_any(v); }
  static __device__ __forceinline__ void store4(uint16_t* p, const float* v) {
    const uint32_t w[2] = {round(v[0]) | round(v[1]) << 16, round(v[2]) | round(v[3]) << 16};
    __builtin_memcpy(p, w, 8);
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

// 32 bytes of a row from `col` on, zeros from `pitch` on
__device__ __forceinline__ int8v load32(const uint8_t* row, int col, int pitch) {
  const uint4 none = make_uint4(0, 0, 0, 0);
  const uint4 a = col < pitch ? *reinterpret_cast<const uint4*>(row + col) : none;
  const uint4 b = col + 16 < pitch ? *reinterpret_cast<const uint4*>(row + col + 16) : none;
  return int8v{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

// The largest power of a row's blocks, as its byte; blocks of NaN aside.
__device__ __forceinline__ int top_scale(const uint8_t* scales, int blocks) {
  int top = 0;
  for (int b = 0; b < blocks; ++b) top = max(top, scales[b] == 255 ? 0 : (int)scales[b]);
  return top;
}
// 2^(byte - top) for the conversion, which looks at the exponent alone; NaN stays
__device__ __forceinline__ float relative(int byte, int top) {
  return __uint_as_float((uint32_t)(byte == 255 ? 255 : max(byte - top + 127, 1)) << 23);
}
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

// A wave: 32 nodes and 32 centres.
template <typename O>
__global__ __launch_bounds__(kThreads) void scores_kernel(ScoresArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = lane & 31, half = lane >> 5;
  const int64_t first = ((int64_t)blockIdx.x * 4 + wave) * 32;
  if (first >= a.num_nodes) return;
  const int64_t i = (int64_t)blockIdx.y * 32 + at;
  const int64_t id = i < a.num_centers ? (int64_t)a.centers[i] : -1;
  const bool there = id >= 0 && id < a.num_in;
  const int64_t row_in = there ? id : 0, row_out = min(first + at, a.num_nodes - 1);
  const uint8_t *h = a.q_in + row_in * a.pitch, *c = a.q_out + row_out * a.pitch;
  const uint8_t *hs = a.scales_in + row_in * a.scale_pitch, *cs = a.scales_out + row_out * a.scale_pitch;
  acc16 acc = {};
  const int top_in = O::kExact ? top_scale(hs, a.blocks) : 0, top_out = O::kExact ? top_scale(cs, a.blocks) : 0;
  for (int b = 0; b < a.blocks; ++b) {
    const int col = b * kBlock + half * 64;
    const int se = hs[b], sf = cs[b];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int8v x = load32(c, col + 32 * s, a.pitch), y = load32(h, col + 32 * s, a.pitch);
      if (O::kExact) {
        const float fx = relative(sf, top_out), fy = relative(se, top_in);
#pragma unroll
        for (int k = 0; k < 8; k += 2)
          acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(x[k], x[k + 1], fx), widen(y[k], y[k + 1], fy), acc, 0, 0, 0);
      } else {
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, acc, 0, 0, 0, sf, 0, se);
      }
    }
  }
  if (O::kExact)
#pragma unroll
    for (int t = 0; t < 16; ++t)
      acc[t] = ldexpf(acc[t], top_in - 254 + __shfl(top_out, 8 * (t / 4) + 4 * half + t % 4, 64));
  if (i >= a.num_centers) return;
  typename O::elem* out = static_cast<typename O::elem*>(a.out) + i * a.num_nodes;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int64_t j = first + 8 * t + 4 * half;
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[k] = there ? a.scale * acc[4 * t + k] : NAN;
      if (a.bias && j + k < a.num_nodes) {
        const float bias = a.bias[j + k];
        v[k] = bias == -INFINITY ? -INFINITY : v[k] + bias;
      }
    }
    if (j + 4 <= a.num_nodes) {
      O::store4(out + j, v);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (j + k < a.num_nodes) O::store(out + j + k, v[k]);
    }
  }
}


// ---- many centres: tiles of both through LDS ---------------------------------
// Centres are copied first: rows of whole blocks, zeros behind, so that no load looks at an id; a centre that is no row has the scale
// NaN.  A workgroup computes TN x TC scores in steps of 64 columns, half a block: the loads write rows' 64 bytes to LDS themselves,
// three steps ahead.  Such a load puts lane l's 16 bytes at base + 16 l, so rows cannot be padded: the four pieces of a row are exchanged
// among each other by a quarter of the row's number instead, so that 16 rows' pieces of a read lie in different banks (four rows
// make 256 bytes, all 64 banks).  One barrier a step.
// The scores go out through LDS as well, as pieces of 16 bytes of whole rows.

struct Copied {                                // of the centres, in the workspace
  uint8_t* q;                                  // [padded centres][128 * blocks]
  uint8_t* scales;                             // [padded centres][scale pitch]: blocks up to a multiple of 4
  int32_t* top;                                // [padded centres]: largest power, as its byte
  int32_t pitch, scale_pitch;
};

// A workgroup of 64 lanes a row.
__global__ __launch_bounds__(64) void copy_centers_kernel(ScoresArgs a, Copied to) {
  const int64_t i = blockIdx.x;
  const int lane = threadIdx.x;
  const int64_t id = i < a.num_centers ? (int64_t)a.centers[i] : -1;
  const bool there = id >= 0 && id < a.num_in;
  for (int col = lane * 16; col < to.pitch; col += 64 * 16) {
    uint4 w = make_uint4(0, 0, 0, 0);
    if (there && col < a.pitch) w = *reinterpret_cast<const uint4*>(a.q_in + id * a.pitch + col);
    *reinterpret_cast<uint4*>(to.q + i * to.pitch + col) = w;
  }
  int top = 0;
  if (lane < to.scale_pitch) {                 // 64 at most
    const int byte = !there ? 255 : lane < a.blocks ? (int)a.scales_in[id * a.scale_pitch + lane] : 0;
    to.scales[i * to.scale_pitch + lane] = (uint8_t)byte;
    if (byte != 255) top = byte;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = max(top, __shfl_xor(top, d, 64));
  if (lane == 0) to.top[i] = top;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t range_of(const void* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00027000);
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
constexpr int kOutside = 1 << 30;              // of every range: read as zeros
constexpr int kStep = 64;                      // columns
constexpr int kStages = 4;                     // steps in LDS

template <typename O, int NA, int NC, int WA, int WC>
__global__ __launch_bounds__(64 * WA * WC, 2) void tile_kernel(ScoresArgs a, Copied in, int64_t tiles_c, int64_t tiles_n) {
  typedef typename O::elem elem;
  constexpr int S = kStages, TN = 32 * NA * WA, TC = 32 * NC * WC, kWaves = WA * WC;
  constexpr int kLoads = (TN + TC) / 16 / kWaves;                        // of 1 KB: sixteen rows
  constexpr int kPer = 16 / (int)sizeof(elem), kRowBytes = TN * (int)sizeof(elem) + 16, kRound = 32 * WC;   // of scores in LDS
  constexpr int kStageBytes = S * (TN + TC) * kStep, kBytes = kStageBytes > kRound * kRowBytes ? kStageBytes : kRound * kRowBytes;
  static_assert((TN / 16) % kLoads == 0 && kLoads * 16 * kWaves == TN + TC, "a wave's loads are of one operand");
  __shared__ __attribute__((aligned(16))) uint8_t lds[kBytes];
  __shared__ __attribute__((aligned(16))) int32_t side_top[TN];
  __shared__ __attribute__((aligned(16))) float side_bias[TN];
  uint8_t* const lds_c = lds + S * TN * kStep;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), at = lane & 31, half = lane >> 5;
  const int wa = wave % WA, wc = wave / WA;

  // Consecutive workgroups go round the eight XCDs: each of them gets neighbouring tiles, eight of nodes at a time, so that what 32
  // compute units read at once is in their L2.
  const int64_t tiles = tiles_c * tiles_n, per = (tiles + 7) / 8;
  const int64_t t = (int64_t)(blockIdx.x % 8) * per + blockIdx.x / 8;
  if (blockIdx.x / 8 >= per || t >= tiles) return;
  const int64_t group = t / (8 * tiles_c), left = min((int64_t)8, tiles_n - 8 * group), in_group = t - group * 8 * tiles_c;
  const int64_t c0 = in_group / left * TC, n0 = (8 * group + in_group % left) * TN;
  const int nodes = (int)min((int64_t)TN, a.num_nodes - n0);

  const bool of_nodes = wave * kLoads < TN / 16;
  const int first_row = wave * kLoads * 16 - (of_nodes ? 0 : TN), pitch = of_nodes ? a.pitch : in.pitch;
  const __amdgpu_buffer_rsrc_t range = range_of(of_nodes ? a.q_out + n0 * a.pitch : in.q + c0 * in.pitch, (of_nodes ? nodes : TC) * pitch);
  uint8_t* const to = (of_nodes ? lds : lds_c) + first_row * kStep;
  const int to_next = (of_nodes ? TN : TC) * kStep;
  const int piece = ((lane & 3) ^ (lane >> 4)) * 16, row_at = (first_row + (lane >> 2)) * pitch;
  auto issue = [&](int step, int buf, int n) {
    const int col = step * kStep + piece;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(range, (__attribute__((address_space(3))) void*)(to + buf * to_next + n * 1024), 16,
                                             col < pitch ? row_at + col + n * 16 * pitch : kOutside, 0, 0, 0);
  };
#pragma unroll
  for (int s = 0; s < S - 1; ++s)
#pragma unroll
    for (int n = 0; n < kLoads; ++n) issue(s, s, n);

  // ---- scales: of a lane's rows, four blocks at a time
  const uint8_t *scales_c = in.scales + c0 * in.scale_pitch, *scales_n = a.scales_out + n0 * a.scale_pitch;
  int scale_n[NA];
  const int scale_c = (wc * NC * 32 + at) * in.scale_pitch;
#pragma unroll
  for (int m = 0; m < NA; ++m) scale_n[m] = min((wa * NA + m) * 32 + at, nodes - 1) * a.scale_pitch;
  auto four = [&](int m, int block) {
    const uint8_t* p = scales_n + scale_n[m];
    if (a.scale_pitch >= 4) return *reinterpret_cast<const uint32_t*>(p + block);
    return (uint32_t)p[0] | (a.scale_pitch == 2 ? (uint32_t)p[1] << 8 : 0u);
  };
  int top_n[NA], top_c[NC];
  if (O::kExact) {
#pragma unroll
    for (int n = 0; n < NC; ++n) top_c[n] = in.top[c0 + (wc * NC + n) * 32 + at];
#pragma unroll
    for (int m = 0; m < NA; ++m) {
      top_n[m] = 0;
      for (int b = 0; b < a.blocks; b += 4) {
        const uint32_t w = four(m, b);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int byte = (int)((w >> (8 * k)) & 255u);
          top_n[m] = max(top_n[m], byte == 255 ? 0 : byte);
        }
      }
      if (wc == 0 && half == 0) side_top[(wa * NA + m) * 32 + at] = top_n[m];
    }
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
  auto step = [&](int k) {
    const int buf = k % S;
    wait_loads<(S - 2) * kLoads>();            // this step's rows; those of later ones may be under way
    meet();
#pragma unroll
    for (int n = 0; n < kLoads; ++n) issue(k + S - 1, (k + S - 1) % S, n);      // where the step before was read
    int8v x[NA], y[NC];
#pragma unroll
    for (int n = 0; n < NC; ++n) y[n] = pair(lds_c + buf * TC * kStep, at_c, n * 32 * kStep);
#pragma unroll
    for (int m = 0; m < NA; ++m) x[m] = pair(lds + buf * TN * kStep, at_n, m * 32 * kStep);
    if (O::kExact) {
      float fx[NA], fy[NC];
#pragma unroll
      for (int m = 0; m < NA; ++m) fx[m] = relative((int)(sn[m] & 255u), top_n[m]);
#pragma unroll
      for (int n = 0; n < NC; ++n) fy[n] = relative((int)(sc[n] & 255u), top_c[n]);
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
        int top[4] = {0, 0, 0, 0};
        if (O::kExact) __builtin_memcpy(top, &side_top[j], 16);
        if (a.bias) __builtin_memcpy(bias, &side_bias[j], 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float z = acc[m][n][4 * g + k];
          if (O::kExact) z = ldexpf(z, top[k] + top_c[n] - 254);
          z = a.scale * z + bias[k];
          v[k] = bias[k] == -INFINITY ? -INFINITY : z;
        }
        O::put4(reinterpret_cast<elem*>(lds + (wc * 32 + at) * kRowBytes) + j, v);
      }
    wait_loads<0>();
    meet();
    constexpr int kLanes = TN / kPer;          // of a row
    for (int p = tid; p < kRound * kLanes; p += 64 * kWaves) {
      const int r = p / kLanes, j = (p - r * kLanes) * kPer;
      const int64_t i = c0 + (r / 32 * NC + n) * 32 + r % 32;
      const uint4 w = *reinterpret_cast<const uint4*>(lds + r * kRowBytes + j * (int)sizeof(elem));
      if (i >= a.num_centers || j >= nodes) continue;
      elem* row = out + i * a.num_nodes + n0 + j;
      if (j + kPer <= nodes) {
        __builtin_memcpy(row, &w, 16);
      } else {
        elem e[kPer];
        __builtin_memcpy(e, &w, 16);
#pragma unroll
        for (int k = 0; k < kPer; ++k)
          if (j + k < nodes) row[k] = e[k];
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
  if (p.few) return p;
  p.padded = ceil_div(num_centers, 256) * 256;
  const int blocks = (int)ceil_div(dim, kBlock);
  p.in.pitch = blocks * kBlock, p.in.scale_pitch = (blocks + 3) / 4 * 4;
  Carver carve(ws);
  p.in.q = carve.take<uint8_t>((size_t)p.padded * p.in.pitch);
  p.in.scales = carve.take<uint8_t>((size_t)p.padded * p.in.scale_pitch);
  p.in.top = carve.take<int32_t>((size_t)p.padded);
  p.bytes = carve.used;
  return p;
}

template <typename O, int NA, int NC, int WA, int WC>
int32_t run_tiles(const ScoresArgs& a, const Copied& in, hipStream_t s) {
  const int64_t c = ceil_div(a.num_centers, 32 * NC * WC), n = ceil_div(a.num_nodes, 32 * NA * WA);
  if (ceil_div(c * n, 8) * 8 > (int64_t)INT32_MAX) return GS_EOVERFLOW;
  tile_kernel<O, NA, NC, WA, WC><<<dim3((unsigned)(ceil_div(c * n, 8) * 8)), 64 * WA * WC, 0, s>>>(a, in, c, n);
  GS_LAUNCH_CHECK();
  return GS_OK;
}

template <typename O>
int32_t run_scores(const ScoresArgs& a, const ScoresPlan& p, hipStream_t s) {
  if (p.few) {
    scores_kernel<O><<<dim3((unsigned)ceil_div(a.num_nodes, 128), (unsigned)ceil_div(a.num_centers, 32)), kThreads, 0, s>>>(a);
    GS_LAUNCH_CHECK();
    return GS_OK;
  }
  copy_centers_kernel<<<dim3((unsigned)p.padded), 64, 0, s>>>(a, p.in);
  GS_LAUNCH_CHECK();
  if (a.num_centers <= 128) return run_tiles<O, 2, 2, 2, 2>(a, p.in, s);
  return run_tiles<O, 4, 2, 2, 4>(a, p.in, s);
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
