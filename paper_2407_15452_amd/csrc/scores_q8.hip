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

bool dtype_known(int32_t dtype) { return dtype == GS_F32 || dtype == GS_BF16 || dtype == GS_F16; }

bool shape_ok(int64_t num_centers, int64_t num_nodes, int32_t dim) {
  return num_centers >= 0 && num_centers <= (int64_t)INT32_MAX && num_nodes >= 1 && num_nodes <= (int64_t)INT32_MAX && dim >= 1 && dim <= GS_Q8_MAX_DIM;
}

}  // namespace
}  // namespace gs

using namespace gs;

extern "C" size_t gs_scores_q8_workspace_bytes(int64_t num_centers, int64_t num_nodes, int32_t dim) {
  if (!shape_ok(num_centers, num_nodes, dim)) return 0;
  return 256;
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
  if (ws_bytes < gs_scores_q8_workspace_bytes(num_centers, num_nodes, dim)) return GS_EWORKSPACE;
  if (num_centers == 0) return GS_OK;
  const ScoresArgs a{static_cast<const uint8_t*>(q_in), static_cast<const uint8_t*>(scales_in), num_in, static_cast<const uint8_t*>(q_out),
                     static_cast<const uint8_t*>(scales_out), num_nodes, gs_q8_pitch(dim), (int32_t)ceil_div(dim, kBlock), gs_q8_scale_pitch(dim),
                     centers, num_centers, bias, scale, scores_out};
  if (ceil_div(num_centers, 32) > 65535) return GS_EOVERFLOW;
  const dim3 grid((unsigned)ceil_div(num_nodes, 128), (unsigned)ceil_div(num_centers, 32));
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == GS_F32) scores_kernel<OutF32><<<grid, kThreads, 0, s>>>(a);
  if (dtype == GS_BF16) scores_kernel<OutHalf<ToBf16>><<<grid, kThreads, 0, s>>>(a);
  if (dtype == GS_F16) scores_kernel<OutHalf<ToF16>><<<grid, kThreads, 0, s>>>(a);
  GS_LAUNCH_CHECK();
  return GS_OK;
}
