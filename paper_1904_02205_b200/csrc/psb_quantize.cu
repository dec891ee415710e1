// Codes in 8-bit floating point with an fp32 scale for each block of 1 x 128 or 128 x 128 values.
//
//   scale = max(max |x| / top, 2^-126),  code = round(x * (1 / scale))
//
// The floor of the scale keeps both it and its reciprocal normal numbers (blocks of zeros and of denormal numbers
// need no case of their own), and one reciprocal per block leaves a multiplication per value.  Inf and NaN take
// no part in the maximum and become NaN codes, so that whatever is computed from them is NaN too.
// Bound by memory: in bytes per value 4 or 2 read, 1 written.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "psb_common.cuh"

namespace psb {

namespace {

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u; }

struct Scale {
  float scale, inverse;
};
__device__ __forceinline__ Scale scale_of(float amax, float top) {
  Scale s;
  s.scale = fmaxf(__fdiv_rn(amax, top), 1.17549435e-38f);
  s.inverse = __frcp_rn(s.scale);
  return s;
}

template <bool E5M2>
__device__ __forceinline__ uint32_t codes2(float a, float b) {
  // (infinities as NaN: inf - inf)
  const float2 v = {finite(a) ? a : a - a, finite(b) ? b : b - b};
  return (uint32_t)__nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, E5M2 ? __NV_E5M2 : __NV_E4M3);
}

// 16 consecutive values of a row, from column c on; zeros behind the row's end.
template <typename T>
__device__ __forceinline__ void load16(const T* row, uint32_t c, uint32_t cols, bool wide, float (&v)[16]) {
  constexpr int kPer = 16 / sizeof(T);
  if (wide && c + 16u <= cols) {
#pragma unroll
    for (int i = 0; i < 16 / kPer; ++i) {
      const uint4 w = *reinterpret_cast<const uint4*>(row + c + i * kPer);
      const T* t = reinterpret_cast<const T*>(&w);
#pragma unroll
      for (int j = 0; j < kPer; ++j) v[i * kPer + j] = to_f32<T>(t[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = c + j < cols ? to_f32<T>(row[c + j]) : 0.0f;
  }
}

template <bool E5M2>
__device__ __forceinline__ void store16(uint8_t* row, uint32_t c, uint32_t cols, bool wide, const float (&v)[16], float inverse) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = codes2<E5M2>(v[4 * i] * inverse, v[4 * i + 1] * inverse) | codes2<E5M2>(v[4 * i + 2] * inverse, v[4 * i + 3] * inverse) << 16;
  if (wide && c + 16u <= cols) {
    *reinterpret_cast<uint4*>(row + c) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (c + j < cols) row[c + j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
  }
}

__device__ __forceinline__ float max16(const float (&v)[16]) {
  float m = 0.0f;
#pragma unroll
  for (int j = 0; j < 16; ++j) m = fmaxf(m, finite(v[j]) ? fabsf(v[j]) : 0.0f);
  return m;
}

struct QuantArgs {
  const void* x;
  uint8_t* codes;
  float* scales;
  uint32_t rows, cols, blocks;       // blocks along a row
  uint64_t x_stride, code_stride, scale_stride;
  uint32_t wide_in, wide_out;        // every row starts at a multiple of 16 bytes
  float top;
};

// 1 x 128: eight lanes a block, 16 values each.
template <typename T, bool E5M2>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const QuantArgs a) {
  pdl_prologue();
  const uint32_t sub = threadIdx.x & 7u;
  // (a division a thread, not one a block of values: in 64 bits they took a third of the time)
  const uint32_t i0 = (blockIdx.x * 256u + threadIdx.x) >> 3, step_r = gridDim.x * 32u / a.blocks, step_b = gridDim.x * 32u - step_r * a.blocks;
  uint32_t r = i0 / a.blocks, b = i0 - r * a.blocks;
  for (; r < a.rows; r += step_r) {
    float v[16];
    const uint32_t c = b * 128u + sub * 16u;
    load16<T>((const T*)a.x + r * a.x_stride, c, a.cols, a.wide_in, v);
    float m = max16(v);
    const uint32_t peers = 0xFFu << (threadIdx.x & 24u);
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(peers, m, d));
    const Scale s = scale_of(m, a.top);
    if (sub == 0u) a.scales[r * a.scale_stride + b] = s.scale;
    store16<E5M2>(a.codes + r * a.code_stride, c, a.cols, a.wide_out, v, s.inverse);
    b += step_b;
    if (b >= a.blocks) { b -= a.blocks; ++r; }
  }
}

// 128 x 128: one block of threads each, 64 values a thread kept in registers between the maximum and the codes.
template <typename T, bool E5M2>
__global__ void __launch_bounds__(256) quantize_tile_kernel(const QuantArgs a) {
  pdl_prologue();
  __shared__ float part[8];
  const uint32_t b = blockIdx.x % a.blocks, rb = blockIdx.x / a.blocks;
  const uint32_t c = b * 128u + (threadIdx.x & 7u) * 16u, r0 = rb * 128u + (threadIdx.x >> 3);
  float v[4][16];
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t r = r0 + 32u * i;
    load16<T>((const T*)a.x + r * a.x_stride, c, r < a.rows ? a.cols : 0u, a.wide_in, v[i]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) m = fmaxf(m, max16(v[i]));
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
  if ((threadIdx.x & 31u) == 0u) part[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, part[i]);
  const Scale s = scale_of(m, a.top);
  if (threadIdx.x == 0u) a.scales[rb * a.scale_stride + b] = s.scale;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t r = r0 + 32u * i;
    if (r < a.rows) store16<E5M2>(a.codes + r * a.code_stride, c, a.cols, a.wide_out, v[i], s.inverse);
  }
}

template <typename T, bool E5M2>
void launch(const QuantArgs& a, uint32_t block_rows, cudaStream_t s) {
  if (block_rows == 1u) {
    const uint64_t want = ((uint64_t)a.rows * a.blocks + 31u) / 32u;
    launch_pdl(quantize_rows_kernel<T, E5M2>, (uint32_t)(want < kSms * 8u ? want : kSms * 8u), 256, 0, s, a);
  } else {
    launch_pdl(quantize_tile_kernel<T, E5M2>, (a.rows + 127u) / 128u * a.blocks, 256, 0, s, a);
  }
  note_launch();
}

}  // namespace

cudaError_t launch_quantize_fp8(const void* x, const psb_quantize_desc& d, uint8_t* codes, float* scales, cudaStream_t s) {
  QuantArgs a;
  a.x = x;
  a.codes = codes;
  a.scales = scales;
  a.rows = d.rows;
  a.cols = d.cols;
  a.blocks = (d.cols + 127u) / 128u;
  a.x_stride = d.x_stride;
  a.code_stride = d.code_stride;
  a.scale_stride = d.scale_stride;
  const uint64_t size = d.in_dtype == PSB_DT_F32 ? 4u : 2u;
  a.wide_in = (((uintptr_t)x | d.x_stride * size) & 15u) == 0u;
  a.wide_out = (((uintptr_t)codes | d.code_stride) & 15u) == 0u;
  const bool e5 = d.code_dtype == PSB_DT_E5M2;
  a.top = e5 ? 57344.0f : 448.0f;
  if (d.in_dtype == PSB_DT_F32) e5 ? launch<float, true>(a, d.block_rows, s) : launch<float, false>(a, d.block_rows, s);
  else if (d.in_dtype == PSB_DT_BF16) e5 ? launch<__nv_bfloat16, true>(a, d.block_rows, s) : launch<__nv_bfloat16, false>(a, d.block_rows, s);
  else e5 ? launch<__half, true>(a, d.block_rows, s) : launch<__half, false>(a, d.block_rows, s);
  return cudaGetLastError();
}

}  // namespace psb
