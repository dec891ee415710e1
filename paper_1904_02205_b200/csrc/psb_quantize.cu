// Codes in 8-bit floating point with an fp32 scale for each block of 1 x 128 or 128 x 128 values.
//
//   scale = max(max |x| / top, 2^-126),  code = round(x * (1 / scale))
//
// The floor of the scale keeps both it and its reciprocal normal numbers (blocks of zeros and of denormal numbers
// need no case of their own), and one reciprocal per block leaves a multiplication per value.  Scale, reciprocal and product each
// round to fp32, 2^-24 of the value: one that lies within 1.8e-7 of the middle between two codes, relatively, may become either (8 in 10000 hidden
// states in bf16, many of which lie on a middle; a few in two million fp32 weights).  Inf and NaN take
// no part in the maximum and become NaN codes, so that whatever is computed from them is NaN too.
// Bound by memory: in bytes per value 4 or 2 read, 1 written.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "psb_common.cuh"

namespace psb {

namespace {

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
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, E5M2 ? __NV_E5M2 : __NV_E4M3);
}

// Values as they come, 4 / sizeof(T) in a word.  Without their signs they are ordered as whole numbers, infinities and NaN
// behind the finite ones: the largest of a block tells whether there are any, and only then is each value asked.
template <typename T> struct Words;
template <> struct Words<float> {
  static constexpr uint32_t kInf = 0x7F800000u;
  static __device__ __forceinline__ uint32_t max_of(uint32_t m, uint32_t w) { return max(m, w & 0x7FFFFFFFu); }
  static __device__ __forceinline__ uint32_t whole(uint32_t m) { return m; }
  static __device__ __forceinline__ float value(uint32_t bits) { return __uint_as_float(bits); }
  template <int N> static __device__ __forceinline__ float get(const uint32_t (&w)[N], int j) { return __uint_as_float(w[j]); }
};
struct HalfWords {
  static __device__ __forceinline__ uint32_t max_of(uint32_t m, uint32_t w) { return __vmaxu2(m, w & 0x7FFF7FFFu); }
  static __device__ __forceinline__ uint32_t whole(uint32_t m) { return max(m & 0xFFFFu, m >> 16); }
};
template <> struct Words<__nv_bfloat16> : HalfWords {
  static constexpr uint32_t kInf = 0x7F80u;
  static __device__ __forceinline__ float value(uint32_t bits) { return __uint_as_float(bits << 16); }
  template <int N> static __device__ __forceinline__ float get(const uint32_t (&w)[N], int j) {
    return __uint_as_float(j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
  }
};
template <> struct Words<__half> : HalfWords {
  static constexpr uint32_t kInf = 0x7C00u;
  static __device__ __forceinline__ float value(uint32_t bits) { return __half2float(__ushort_as_half((uint16_t)bits)); }
  template <int N> static __device__ __forceinline__ float get(const uint32_t (&w)[N], int j) { return value(w[j / 2] >> (j & 1 ? 16 : 0) & 0xFFFFu); }
};
template <typename T> constexpr int kWords = 4 * (int)sizeof(T);      // of 16 values

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u; }

// 16 consecutive values of a row, from column c on; zeros behind the row's end.
template <typename T>
__device__ __forceinline__ void load16(const T* row, uint32_t c, uint32_t cols, bool wide, uint32_t (&w)[kWords<T>]) {
  if (wide && c + 16u <= cols) {
#pragma unroll
    for (int i = 0; i < kWords<T> / 4; ++i) {
      const uint4 q = *reinterpret_cast<const uint4*>(row + c + i * (16 / (int)sizeof(T)));
      w[4 * i] = q.x;
      w[4 * i + 1] = q.y;
      w[4 * i + 2] = q.z;
      w[4 * i + 3] = q.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kWords<T>; ++i) w[i] = 0u;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      if (c + j >= cols) continue;
      if (sizeof(T) == 4) w[j] = reinterpret_cast<const uint32_t*>(row)[c + j];
      else w[j / 2 % kWords<T>] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[c + j] << (j & 1 ? 16 : 0);
    }
  }
}

template <typename T, bool E5M2>
__device__ __forceinline__ void store16(uint8_t* row, uint32_t c, uint32_t cols, bool wide, const uint32_t (&w)[kWords<T>], float inverse, bool all_finite) {
  uint32_t q[4];
  float v[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) v[j] = Words<T>::get(w, j) * inverse;
  if (!all_finite) {
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = finite(v[j]) ? v[j] : NAN;      // (a finite value times the reciprocal is finite)
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = codes2<E5M2>(v[4 * i], v[4 * i + 1]) | codes2<E5M2>(v[4 * i + 2], v[4 * i + 3]) << 16;
  if (wide && c + 16u <= cols) {
    *reinterpret_cast<uint4*>(row + c) = make_uint4(q[0], q[1], q[2], q[3]);
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (c + j < cols) row[c + j] = (uint8_t)(q[j >> 2] >> (8 * (j & 3)));
  }
}

template <typename T>
__device__ __forceinline__ uint32_t max16(uint32_t m, const uint32_t (&w)[kWords<T>]) {
#pragma unroll
  for (int i = 0; i < kWords<T>; ++i) m = Words<T>::max_of(m, w[i]);
  return m;
}
// Of the finite values alone (the rare case).
template <typename T>
__device__ __forceinline__ float finite16(float m, const uint32_t (&w)[kWords<T>]) {
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const float v = fabsf(Words<T>::get(w, j));
    m = finite(v) ? fmaxf(m, v) : m;
  }
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
    const uint32_t c = b * 128u + sub * 16u;
    uint32_t w[kWords<T>];
    load16<T>((const T*)a.x + r * a.x_stride, c, a.cols, a.wide_in, w);
    uint32_t m = Words<T>::whole(max16<T>(0u, w));
    const uint32_t peers = 0xFFu << (threadIdx.x & 24u);
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) m = max(m, __shfl_xor_sync(peers, m, d));
    float amax = Words<T>::value(m);
    const bool all_finite = m < Words<T>::kInf;
    if (!all_finite) {
      amax = finite16<T>(0.0f, w);
#pragma unroll
      for (int d = 4; d > 0; d >>= 1) amax = fmaxf(amax, __shfl_xor_sync(peers, amax, d));
    }
    const Scale s = scale_of(amax, a.top);
    if (sub == 0u) a.scales[r * a.scale_stride + b] = s.scale;
    store16<T, E5M2>(a.codes + r * a.code_stride, c, a.cols, a.wide_out, w, s.inverse, all_finite);
    b += step_b;
    if (b >= a.blocks) { b -= a.blocks; ++r; }
  }
}

// 128 x 128: one block of threads each, 64 values a thread kept in registers between the maximum and the codes.
template <typename T, bool E5M2>
__global__ void __launch_bounds__(256) quantize_tile_kernel(const QuantArgs a) {
  pdl_prologue();
  __shared__ uint32_t part[8];
  const uint32_t b = blockIdx.x % a.blocks, rb = blockIdx.x / a.blocks;
  const uint32_t c = b * 128u + (threadIdx.x & 7u) * 16u, r0 = rb * 128u + (threadIdx.x >> 3);
  uint32_t w[4][kWords<T>];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t r = r0 + 32u * i;
    load16<T>((const T*)a.x + r * a.x_stride, c, r < a.rows ? a.cols : 0u, a.wide_in, w[i]);
  }
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max16<T>(m, w[i]);
  m = __reduce_max_sync(0xFFFFFFFFu, Words<T>::whole(m));
  if ((threadIdx.x & 31u) == 0u) part[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, part[i]);
  float amax = Words<T>::value(m);
  const bool all_finite = m < Words<T>::kInf;        // (the same for the whole block of threads)
  if (!all_finite) {
    amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) amax = finite16<T>(amax, w[i]);
    // (numbers that are not negative are ordered as their bits)
    const uint32_t bits = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(amax));
    __syncthreads();
    if ((threadIdx.x & 31u) == 0u) part[threadIdx.x >> 5] = bits;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, __uint_as_float(part[i]));
  }
  const Scale s = scale_of(amax, a.top);
  if (threadIdx.x == 0u) a.scales[rb * a.scale_stride + b] = s.scale;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t r = r0 + 32u * i;
    if (r < a.rows) store16<T, E5M2>(a.codes + r * a.code_stride, c, a.cols, a.wide_out, w[i], s.inverse, all_finite);
  }
}

template <typename T, bool E5M2>
cudaError_t launch(const QuantArgs& a, uint32_t block_rows, cudaStream_t s) {
  if (block_rows != 1u) return launched(launch_pdl(quantize_tile_kernel<T, E5M2>, (a.rows + 127u) / 128u * a.blocks, 256, 0, s, a));
  const uint64_t want = ((uint64_t)a.rows * a.blocks + 31u) / 32u;
  return launched(launch_pdl(quantize_rows_kernel<T, E5M2>, (uint32_t)(want < kSms * 8u ? want : kSms * 8u), 256, 0, s, a));
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
  if (d.in_dtype == PSB_DT_F32) return e5 ? launch<float, true>(a, d.block_rows, s) : launch<float, false>(a, d.block_rows, s);
  if (d.in_dtype == PSB_DT_BF16) return e5 ? launch<__nv_bfloat16, true>(a, d.block_rows, s) : launch<__nv_bfloat16, false>(a, d.block_rows, s);
  return e5 ? launch<__half, true>(a, d.block_rows, s) : launch<__half, false>(a, d.block_rows, s);
}

}  // namespace psb
