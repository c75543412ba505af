// gs_quantize_rows: rows of a table as e4m3 values with a power of two for each block of 128 columns.
//
//   a = max |x| of the block;  2^e the least power of two with a <= 448 * 2^e, e >= -127;  q = e4m3(x * 2^-e), nearest even
//
// 448 is the format's largest value, so nothing saturates.  a = m * 2^x with 1 <= m < 2 gives e = x - 8, or x - 7 for m > 1.75: the
// bits of a alone.  The product with 2^-e is exact (what falls below fp32's range is far below the format's least value), so a value
// is rounded once.  Maxima are taken of the bits without the sign, as whole numbers: infinity and NaN are larger than every finite one.
//
// Bound: memory; every element is read once and written once.  Sixteen lanes take a block, eight columns each: a whole line of the copy
// and 16 or 32 bytes a lane of the table.  1,000,000 rows of 128 bf16 columns take 77 us, 5.0 TB/s read and written (a copy of 1 GiB
// 5.1); 256 fp32 rows by their ids 3.9 us, the latency of a launch and three dependent reads.

#include "common.h"

namespace gs {
namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 128;
constexpr int kLanes = 16;                     // of a block: 8 columns each

struct QuantizeArgs {
  const void* table;
  int64_t num_nodes;
  int32_t dim, pitch, blocks, scale_pitch;
  const int32_t* ids;                          // or null: every row
  int64_t n;
  const int64_t* count;                        // or null
  uint8_t* q;
  uint8_t* scales;
};

struct InF32 {
  static constexpr int kSize = 4;
  // eight columns from `col` on, zeros from `dim` on (a multiple of 4)
  static __device__ __forceinline__ void load(const void* row, int col, int dim, float* x) {
    const float4 none = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(row) + col);
    const float4 a = col < dim ? p[0] : none, b = col + 4 < dim ? p[1] : none;
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  }
};
template <typename H>
struct InHalf {
  static constexpr int kSize = 2;
  static __device__ __forceinline__ void load(const void* row, int col, int dim, float* x) {
    const uint4 w = col < dim ? *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(row) + col) : make_uint4(0, 0, 0, 0);
    x[0] = H::lo(w.x), x[1] = H::hi(w.x), x[2] = H::lo(w.y), x[3] = H::hi(w.y);
    x[4] = H::lo(w.z), x[5] = H::hi(w.z), x[6] = H::lo(w.w), x[7] = H::hi(w.w);
  }
};

template <typename In>
__global__ __launch_bounds__(kThreads) void quantize_kernel(QuantizeArgs a) {
  const int lane = threadIdx.x % kLanes;
  const int64_t n = a.count ? min(a.n, max((int64_t)0, *a.count)) : a.n;
  const int64_t items = n * a.blocks, step = (int64_t)gridDim.x * (kThreads / kLanes);
  for (int64_t item = (int64_t)blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes; item < items; item += step) {
    const int64_t i = item / a.blocks;
    const int block = (int)(item - i * a.blocks);
    const int64_t row = a.ids ? (int64_t)a.ids[i] : i;
    if (row < 0 || row >= a.num_nodes) continue;
    const int col = block * kBlock + lane * 8;
    float x[8];
    In::load(static_cast<const char*>(a.table) + row * a.dim * In::kSize, col, a.dim, x);
    uint32_t most = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) most = max(most, __float_as_uint(x[k]) & 0x7fffffffu);
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d, kLanes));
    const bool fine = most < 0x7f800000u;
    const int power = max((int)(most >> 23) - 127 - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0), -127);
    const float inverse = fine ? __uint_as_float((uint32_t)(127 - power) << 23) : 0.0f;
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float y[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = fine ? x[4 * h + k] * inverse : 0.0f;
      int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
      w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], v, true);
    }
    if (col < a.pitch) *reinterpret_cast<uint2*>(a.q + row * a.pitch + col) = make_uint2(w[0], w[1]);
    uint8_t* scales = a.scales + row * a.scale_pitch;
    if (lane == 0) scales[block] = (uint8_t)(fine ? power + 127 : 255);
    if (block == a.blocks - 1 && lane > 0 && block + lane < a.scale_pitch) scales[block + lane] = 0;
  }
}

}  // namespace
}  // namespace gs

using namespace gs;

extern "C" int32_t gs_quantize_rows(const void* table, int64_t num_nodes, int32_t dim, int32_t dtype, const int32_t* ids, int64_t n,
                                    const int64_t* count_dev, void* q_out, void* scales_out, void* stream) {
  if (dtype != GS_F32 && dtype != GS_BF16 && dtype != GS_F16) return GS_EINVAL;
  if (num_nodes < 1 || num_nodes > (int64_t)INT32_MAX || n < 0 || n > (int64_t)INT32_MAX) return GS_EINVAL;
  if (dim < 1 || dim > GS_Q8_MAX_DIM || dim % (dtype == GS_F32 ? 4 : 8) != 0) return GS_EINVAL;
  if (!table || !q_out || !scales_out || !aligned(table, 16) || !aligned(q_out, 16) || !aligned(scales_out, 4)) return GS_EINVAL;
  if (!aligned(ids, 4) || !aligned(count_dev, 8) || (!ids && (n != num_nodes || count_dev))) return GS_EINVAL;
  if (n == 0) return GS_OK;
  const int blocks = (int)ceil_div(dim, kBlock);
  const QuantizeArgs a{table, num_nodes, dim, gs_q8_pitch(dim), blocks, gs_q8_scale_pitch(dim), ids, n, count_dev, static_cast<uint8_t*>(q_out),
                       static_cast<uint8_t*>(scales_out)};
  const int64_t groups = std::min<int64_t>(ceil_div(n * blocks, kThreads / kLanes), 256 * 8);
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == GS_F32) quantize_kernel<InF32><<<dim3((unsigned)groups), kThreads, 0, s>>>(a);
  if (dtype == GS_BF16) quantize_kernel<InHalf<bf16_t>><<<dim3((unsigned)groups), kThreads, 0, s>>>(a);
  if (dtype == GS_F16) quantize_kernel<InHalf<f16_t>><<<dim3((unsigned)groups), kThreads, 0, s>>>(a);
  GS_LAUNCH_CHECK();
  return GS_OK;
}

extern "C" int32_t gs_q8_pitch(int32_t dim) { return dim < 1 || dim > GS_Q8_MAX_DIM ? 0 : (dim + 15) / 16 * 16; }
extern "C" int32_t gs_q8_scale_pitch(int32_t dim) {
  if (dim < 1 || dim > GS_Q8_MAX_DIM) return 0;
  const int32_t blocks = (dim + kBlock - 1) / kBlock;
  return blocks <= 2 ? blocks : (blocks + 3) / 4 * 4;
}
