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
  // a lane's node j of rows i .. i + 3
  static __device__ __forceinline__ void store_rows(float* out, int64_t i, int64_t j, const float* v, int64_t rows, int64_t n, int) {
    if (j >= n) return;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < rows) out[(i + k) * n + j] = v[k];
  }
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
  // Neighbouring lanes exchange: of two rows, the even lane writes both nodes of the first, the odd one of the second.
  static __device__ __forceinline__ void store_rows(uint16_t* out, int64_t i, int64_t j, const float* v, int64_t rows, int64_t n, int lane) {
    const bool odd = lane & 1;
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
      const float mine = odd ? v[k + 1] : v[k], give = odd ? v[k] : v[k + 1];
      const float got = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, give), 0xb1, 0xf, 0xf, true));   // lane ^ 1
      const int64_t row = i + k + (odd ? 1 : 0), first = j - (odd ? 1 : 0);
      const uint32_t w = odd ? round(got) | round(mine) << 16 : round(mine) | round(got) << 16;
      if (row >= rows) continue;
      uint16_t* p = out + row * n + first;
      if (first + 1 < n) __builtin_memcpy(p, &w, 4);
      else if (first < n) *p = (uint16_t)w;
    }
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
// NaN.  A workgroup computes TM x TN scores; a step is a block of 128 columns of TM + TN rows, which the loads write to LDS
// themselves, a step ahead.  Such a load puts lane l's 16 bytes at base + 16 l, so rows cannot be padded: the eight pieces of a
// row's 128 bytes are exchanged among each other by the row's number instead, which keeps reads of a piece of 32 rows off each
// other's banks.  Here centres are the left operand: a lane holds one node's scores of 16 centres, neighbouring lanes
// neighbouring nodes, and 32 lanes write 128 bytes of an fp32 row or 64 of a 16-bit one.

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
constexpr int kOutside = 1 << 30;              // of every range: read as zeros

template <typename O, int MB, int NB, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 2) void tile_kernel(ScoresArgs a, Copied in, int64_t tiles_m, int64_t tiles_n) {
  constexpr int TM = 32 * MB * WM, TN = 32 * NB * WN, kWaves = WM * WN;
  constexpr int kChunks = (TM + TN) / 8, kLoads = kChunks / kWaves;      // of 1 KB: eight rows
  static_assert(kChunks % kWaves == 0 && (TM / 8) % kLoads == 0, "a wave's chunks are of one operand");
  __shared__ __attribute__((aligned(16))) uint8_t stage_m[2][TM * kBlock], stage_n[2][TN * kBlock];
  __shared__ __attribute__((aligned(16))) int32_t tops[TM];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), at = lane & 31, half = lane >> 5;
  const int wm = wave / WN, wn = wave % WN;

  // Consecutive workgroups go round the eight XCDs: each of them gets neighbouring tiles, eight of nodes at a time, so that what 32
  // compute units read at once is in their L2.
  const int64_t tiles = tiles_m * tiles_n, per = (tiles + 7) / 8;
  const int64_t t = (int64_t)(blockIdx.x % 8) * per + blockIdx.x / 8;
  if (blockIdx.x / 8 >= per || t >= tiles) return;
  const int64_t group = t / (8 * tiles_m), left = min((int64_t)8, tiles_n - 8 * group), in_group = t - group * 8 * tiles_m;
  const int64_t m0 = in_group / left * TM, n0 = (8 * group + in_group % left) * TN;

  const bool of_centers = wave * kLoads < TM / 8;
  const int64_t rows = of_centers ? (int64_t)TM : min((int64_t)TN, a.num_nodes - n0);
  const int pitch = of_centers ? in.pitch : a.pitch;
  const __amdgpu_buffer_rsrc_t range = range_of(of_centers ? in.q + m0 * in.pitch : a.q_out + n0 * a.pitch, (int)rows * pitch);
  // the rows of a wave's loads are eight apart: one place in the row, and one exchange
  const int piece = ((lane & 7) ^ (lane >> 3)) * 16, first_row = wave * kLoads * 8 - (of_centers ? 0 : TM);
  const int place = (first_row + (lane >> 3)) * pitch + piece;
  auto issue = [&](int block, int buf) {
    const int from = block * kBlock + piece < pitch ? place + block * kBlock : kOutside;
#pragma unroll
    for (int n = 0; n < kLoads; ++n)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(range, (__attribute__((address_space(3))) void*)((of_centers ? stage_m[buf] : stage_n[buf]) + first_row * kBlock + n * 1024), 16,
                                               from + n * 8 * pitch, 0, 0, 0);
  };
  issue(0, 0);

  const uint8_t *scales_m = in.scales + m0 * in.scale_pitch, *scales_n = a.scales_out + n0 * a.scale_pitch;
  int scale_n[NB];
  const int scale_m = (wm * MB * 32 + at) * in.scale_pitch;
#pragma unroll
  for (int n = 0; n < NB; ++n) scale_n[n] = min((wn * NB + n) * 32 + at, (int)min(a.num_nodes - n0, (int64_t)TN) - 1) * a.scale_pitch;
  auto of_nodes = [&](int n, int block) {      // the scales of four blocks from `block` on
    const uint8_t* p = scales_n + scale_n[n];
    if (a.scale_pitch >= 4) return *reinterpret_cast<const uint32_t*>(p + block);
    return (uint32_t)p[0] | (a.scale_pitch == 2 ? (uint32_t)p[1] << 8 : 0u);
  };
  int top_m[MB], top_n[NB];
  if (O::kExact) {
#pragma unroll
    for (int m = 0; m < MB; ++m) top_m[m] = in.top[m0 + (wm * MB + m) * 32 + at];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      top_n[n] = 0;
      for (int b = 0; b < a.blocks; b += 4) {
        const uint32_t w = of_nodes(n, b);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int byte = (int)((w >> (8 * k)) & 255u);
          top_n[n] = max(top_n[n], byte == 255 ? 0 : byte);
        }
      }
    }
    for (int i = tid; i < TM; i += 64 * kWaves) tops[i] = in.top[m0 + i];
  }

  // reads: piece 4 s + 2 half + j of a row
  int at_m[2][2], at_n[2][2];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int in_row = ((4 * (c >> 1) + 2 * half + (c & 1)) ^ (at & 7)) * 16;
    at_m[c >> 1][c & 1] = (wm * MB * 32 + at) * kBlock + in_row;
    at_n[c >> 1][c & 1] = (wn * NB * 32 + at) * kBlock + in_row;
  }
  acc16 acc[MB][NB];
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int n = 0; n < NB; ++n) acc[m][n] = acc16{};
  uint32_t sm[MB], sn[NB], next_m[MB], next_n[NB];      // the scales of four blocks, and of the next four
  auto fetch_scales = [&](int block) {
#pragma unroll
    for (int m = 0; m < MB; ++m) next_m[m] = *reinterpret_cast<const uint32_t*>(scales_m + scale_m + m * 32 * in.scale_pitch + block);
#pragma unroll
    for (int n = 0; n < NB; ++n) next_n[n] = of_nodes(n, block);
  };
  fetch_scales(0);

  auto step = [&](int block, int buf) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if ((block & 3) == 0) {
#pragma unroll
      for (int m = 0; m < MB; ++m) sm[m] = next_m[m];
#pragma unroll
      for (int n = 0; n < NB; ++n) sn[n] = next_n[n];
      if (block + 4 < a.blocks) fetch_scales(block + 4);
    }
    if (block + 1 < a.blocks) issue(block + 1, buf ^ 1);
    __builtin_amdgcn_sched_barrier(0);
    auto read = [&](const uint8_t* p) {
      const uint4 w = *reinterpret_cast<const uint4*>(p);
      return w;
    };
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (s > 0) __builtin_amdgcn_sched_barrier(0);
      int8v x[MB], y[NB];
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        const uint4 p = read(stage_m[buf] + at_m[s][0] + m * 32 * kBlock), q = read(stage_m[buf] + at_m[s][1] + m * 32 * kBlock);
        x[m] = int8v{(int)p.x, (int)p.y, (int)p.z, (int)p.w, (int)q.x, (int)q.y, (int)q.z, (int)q.w};
      }
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const uint4 p = read(stage_n[buf] + at_n[s][0] + n * 32 * kBlock), q = read(stage_n[buf] + at_n[s][1] + n * 32 * kBlock);
        y[n] = int8v{(int)p.x, (int)p.y, (int)p.z, (int)p.w, (int)q.x, (int)q.y, (int)q.z, (int)q.w};
      }
      if (O::kExact) {
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
          bf8 u[MB], v[NB];
#pragma unroll
          for (int m = 0; m < MB; ++m) u[m] = widen(x[m][k], x[m][k + 1], relative((int)(sm[m] & 255u), top_m[m]));
#pragma unroll
          for (int n = 0; n < NB; ++n) v[n] = widen(y[n][k], y[n][k + 1], relative((int)(sn[n] & 255u), top_n[n]));
#pragma unroll
          for (int m = 0; m < MB; ++m)
#pragma unroll
            for (int n = 0; n < NB; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(u[m], v[n], acc[m][n], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int m = 0; m < MB; ++m)
#pragma unroll
          for (int n = 0; n < NB; ++n)
            acc[m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x[m], y[n], acc[m][n], 0, 0, 0, (int)sm[m], 0, (int)sn[n]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int m = 0; m < MB; ++m) sm[m] >>= 8;
#pragma unroll
    for (int n = 0; n < NB; ++n) sn[n] >>= 8;
  };
  int block = 0;
  for (; block + 2 <= a.blocks; block += 2) {
    step(block, 0);
    step(block + 1, 1);
  }
  if (block < a.blocks) step(block, 0);

  // ---- scores: register 4 g + k of a block is centre 8 g + 4 half + k, a lane's node is n0 + ... + at
  typedef typename O::elem elem;
  elem* out = static_cast<elem*>(a.out);
  const int64_t row0 = m0 + wm * MB * 32 + 4 * half;
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int64_t j = n0 + (wn * NB + n) * 32 + at;
    const float bias = a.bias && j < a.num_nodes ? a.bias[j] : 0.0f;
    const bool masked = bias == -INFINITY;
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        float v[4];
        int top[4] = {0, 0, 0, 0};
        if (O::kExact) __builtin_memcpy(top, &tops[(wm * MB + m) * 32 + 8 * g + 4 * half], 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float z = acc[m][n][4 * g + k];
          if (O::kExact) z = ldexpf(z, top[k] + top_n[n] - 254);
          z = a.scale * z + bias;
          v[k] = masked ? -INFINITY : z;
        }
        const int64_t i = row0 + m * 32 + 8 * g;
        O::store_rows(out, i, j, v, a.num_centers, a.num_nodes, lane);
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

template <typename O, int MB, int NB, int WM, int WN>
int32_t run_tiles(const ScoresArgs& a, const Copied& in, hipStream_t s) {
  const int64_t m = ceil_div(a.num_centers, 32 * MB * WM), n = ceil_div(a.num_nodes, 32 * NB * WN);
  if (ceil_div(m * n, 8) * 8 > (int64_t)INT32_MAX) return GS_EOVERFLOW;
  tile_kernel<O, MB, NB, WM, WN><<<dim3((unsigned)(ceil_div(m * n, 8) * 8)), 64 * WM * WN, 0, s>>>(a, in, m, n);
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
  return run_tiles<O, 2, 2, 2, 2>(a, p.in, s);
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
