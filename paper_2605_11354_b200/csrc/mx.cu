// Microscaled formats: blocks of 32 values along a row share a scale 2^E (one byte, E + 127), elements are e2m1 (MXFP4) or
// e4m3 (MXFP8).  Their quantiser and its inverse.
//   E = the smallest integer, at least -127, with max|x| <= top * 2^E (top = 6 or 448): no element saturates, so every
//   element is off by at most half a step.  code = round to nearest even (x * 2^-E); the product with a power of two is exact.
//   A block that holds an infinity or a NaN gets the scale 0xFF, which stands for NaN.
// E comes from the bits of the largest magnitude: exponent - log2 of the power of two in top, plus one where the mantissa is
// beyond top's; one integer addition whose carry does that.
// The scales lie in tiles of 128 rows x 4 blocks (512 bytes), row r at (r % 32) * 16 + (r / 32) * 4: the layout from which the
// tensor cores take them, so a product copies a tile as it is.  A CTA makes one such tile, 128 rows x 128 values: its 512
// scale bytes meet in shared memory and leave in one piece, and each of its threads has eight independent loads under way.
// Bound by HBM: 43968 x 4096 bf16 values are 360 MB read and 180 MB of codes.
#include <algorithm>

#include <cuda_fp4.h>

#include "common.cuh"
#include "sm100.cuh"

namespace lite3r {

namespace {

using namespace sm100;

constexpr int kMxThreads = 256;
constexpr int kMxRows = 128, kMxCols = 128;  // of a tile
constexpr int kMxIters = kMxRows / (kMxThreads / 16);

// What is added to the bits of the largest magnitude so that a carry into the exponent says that the mantissa is beyond top's
// (1.5 or 1.75), and the exponent of top.
template <int kFormat>
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
  constexpr uint32_t kCarry = kFormat == LITE3R_MXFP4 ? 0x3FFFFFu : 0x1FFFFFu;
  constexpr int kTopExp = kFormat == LITE3R_MXFP4 ? 2 : 8;
  if (amax_bits >= 0x7F800000u) return 0xFFu;
  return static_cast<uint32_t>(max(static_cast<int>((amax_bits + kCarry) >> 23) - kTopExp, 0));
}
__device__ __forceinline__ float byte_to_scale(uint32_t byte) {  // 2^(byte - 127); 0xFF: NaN
  return byte == 0xFFu ? __uint_as_float(0x7FFFFFFFu) : __uint_as_float(byte == 0u ? 0x00400000u : byte << 23);
}

// Eight values as they lie in memory and the largest of their magnitudes as fp32 bits (NaN above infinity above all else).
template <typename T>
struct Octet;
template <>
struct Octet<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = __ldg(reinterpret_cast<const float4*>(p));
    b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void values(float v[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  __device__ __forceinline__ uint32_t top() const {
    float v[8];
    values(v);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return m;
  }
};
template <typename T>
struct Octet16 {
  uint4 w;
  __device__ __forceinline__ void load(const T* p) { w = __ldg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void clear() { w = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ uint32_t top16() const {  // the largest magnitude's 16 bits
    constexpr uint32_t kAbs = 0x7FFF7FFFu;
    const uint32_t m = __vmaxu2(__vmaxu2(w.x & kAbs, w.y & kAbs), __vmaxu2(w.z & kAbs, w.w & kAbs));
    return max(m & 0xFFFFu, m >> 16);
  }
};
template <>
struct Octet<__nv_bfloat16> : Octet16<__nv_bfloat16> {
  __device__ __forceinline__ void values(float v[8]) const {
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(x[i] << 16);
      v[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
    }
  }
  __device__ __forceinline__ uint32_t top() const { return top16() << 16; }
};
template <>
struct Octet<__half> : Octet16<__half> {
  __device__ __forceinline__ void values(float v[8]) const {
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x[i]));
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  }
  __device__ __forceinline__ uint32_t top() const { return __float_as_uint(__half2float(__ushort_as_half(static_cast<unsigned short>(top16())))); }
};

// Row pitch of the codes in bytes.
template <int kFormat>
__device__ __forceinline__ size_t code_pitch(int cols) { return kFormat == LITE3R_MXFP4 ? cols / 2 : cols; }

template <typename T, int kFormat>
__global__ void __launch_bounds__(kMxThreads) mx_quantise_kernel(const T* __restrict__ x, long long row_stride, int rows, int cols,
                                                                int col_tiles, uint8_t* __restrict__ codes,
                                                                uint32_t* __restrict__ scales) {
  __shared__ __align__(16) uint8_t s_scales[512];
  const int row_tile = blockIdx.x / col_tiles, col_tile = blockIdx.x - row_tile * col_tiles;
  const int lane16 = threadIdx.x & 15, col = col_tile * kMxCols + lane16 * 8;
  const int row_in = threadIdx.x >> 4;  // of the sixteen rows of a step
  const long long row0 = static_cast<long long>(row_tile) * kMxRows;
  wait_for_prior_grid();
  launch_dependents();
  Octet<T> in[kMxIters];
#pragma unroll
  for (int i = 0; i < kMxIters; ++i) {
    const long long row = row0 + row_in + 16 * i;
    if (row < rows && col < cols) in[i].load(x + row * row_stride + col);
    else in[i].clear();
  }
#pragma unroll
  for (int i = 0; i < kMxIters; ++i) {
    const int r = row_in + 16 * i;
    uint32_t top = in[i].top();
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
    const uint32_t byte = scale_byte<kFormat>(top);
    if ((lane16 & 3) == 0) s_scales[(r & 31) * 16 + (r >> 5) * 4 + (lane16 >> 2)] = static_cast<uint8_t>(byte);
    if (row0 + r < rows && col < cols) {
      const float inverse = __uint_as_float((254u - min(byte, 253u)) << 23);
      float v[8];
      in[i].values(v);
      uint8_t* dst = codes + static_cast<size_t>(row0 + r) * code_pitch<kFormat>(cols);
      if constexpr (kFormat == LITE3R_MXFP8) {
        uint32_t w[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * q] * inverse, v[4 * q + 1] * inverse), __NV_SATFINITE, __NV_E4M3);
          const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * q + 2] * inverse, v[4 * q + 3] * inverse), __NV_SATFINITE, __NV_E4M3);
          w[q] = byte == 0xFFu ? 0x7F7F7F7Fu : lo | hi << 16;
        }
        *reinterpret_cast<uint2*>(dst + col) = make_uint2(w[0], w[1]);
      } else {
        uint32_t w = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q)
          w |= static_cast<uint32_t>(__nv_cvt_float2_to_fp4x2(make_float2(v[2 * q] * inverse, v[2 * q + 1] * inverse), __NV_E2M1, cudaRoundNearest)) << (8 * q);
        *reinterpret_cast<uint32_t*>(dst + col / 2) = byte == 0xFFu ? 0x22222222u : w;
      }
    }
  }
  __syncthreads();
  if (threadIdx.x < 128) scales[static_cast<size_t>(blockIdx.x) * 128 + threadIdx.x] = reinterpret_cast<const uint32_t*>(s_scales)[threadIdx.x];
}

__device__ __forceinline__ void store8(float* p, const float v[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *(reinterpret_cast<float4*>(p) + 1) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float v[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(__half* p, const float v[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T, int kFormat>
__global__ void __launch_bounds__(kMxThreads) mx_dequantise_kernel(const uint8_t* __restrict__ codes, const uint32_t* __restrict__ scales,
                                                                  int rows, int cols, int col_tiles, T* __restrict__ out,
                                                                  long long row_stride) {
  __shared__ __align__(16) uint8_t s_scales[512];
  const int row_tile = blockIdx.x / col_tiles, col_tile = blockIdx.x - row_tile * col_tiles;
  const int lane16 = threadIdx.x & 15, col = col_tile * kMxCols + lane16 * 8;
  const int row_in = threadIdx.x >> 4;
  const long long row0 = static_cast<long long>(row_tile) * kMxRows;
  wait_for_prior_grid();
  launch_dependents();
  uint2 w[kMxIters];
#pragma unroll
  for (int i = 0; i < kMxIters; ++i) {
    const long long row = row0 + row_in + 16 * i;
    w[i] = make_uint2(0u, 0u);
    if (row < rows && col < cols) {
      const uint8_t* src = codes + static_cast<size_t>(row) * code_pitch<kFormat>(cols);
      if constexpr (kFormat == LITE3R_MXFP8) w[i] = __ldg(reinterpret_cast<const uint2*>(src + col));
      else w[i].x = __ldg(reinterpret_cast<const uint32_t*>(src + col / 2));
    }
  }
  if (threadIdx.x < 128) reinterpret_cast<uint32_t*>(s_scales)[threadIdx.x] = __ldg(scales + static_cast<size_t>(blockIdx.x) * 128 + threadIdx.x);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kMxIters; ++i) {
    const int r = row_in + 16 * i;
    if (row0 + r >= rows || col >= cols) continue;
    const float scale = byte_to_scale(s_scales[(r & 31) * 16 + (r >> 5) * 4 + (lane16 >> 2)]);
    float v[8];
    if constexpr (kFormat == LITE3R_MXFP8) {
      e4m3x4_to_float(w[i].x, v);
      e4m3x4_to_float(w[i].y, v + 4);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2(static_cast<__nv_fp4x2_storage_t>((w[i].x >> (8 * q)) & 0xFFu), __NV_E2M1);
        const float2 f = __half22float2(__half2(h));
        v[2 * q] = f.x;
        v[2 * q + 1] = f.y;
      }
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] *= scale;
    store8(out + (row0 + r) * row_stride + col, v);
  }
}

// Calls fn with a value of the element type and the format as template arguments.
template <typename T, typename Fn>
lite3r_status by_format(int format, const Fn& fn) {
  return format == LITE3R_MXFP4 ? fn(T{}, std::integral_constant<int, LITE3R_MXFP4>()) : fn(T{}, std::integral_constant<int, LITE3R_MXFP8>());
}
template <typename Fn>
lite3r_status by_type(int dtype, int format, const Fn& fn) {
  switch (dtype) {
    case LITE3R_F32: return by_format<float>(format, fn);
    case LITE3R_BF16: return by_format<__nv_bfloat16>(format, fn);
    case LITE3R_F16: return by_format<__half>(format, fn);
  }
  return LITE3R_ERR_UNSUPPORTED;
}

}  // namespace

lite3r_status launch_mx_quantise(const void* x, int dtype, long long row_stride, int rows, int cols, int format, uint8_t* codes,
                                 uint8_t* scales, cudaStream_t stream) {
  const int col_tiles = ceil_div(cols, kMxCols);
  const long long tiles = static_cast<long long>(ceil_div(rows, kMxRows)) * col_tiles;
  if (tiles > 0x7FFFFFFFLL) return LITE3R_ERR_UNSUPPORTED;
  return by_type(dtype, format, [&](auto type, auto fmt) {
    using T = decltype(type);
    return launch_dependent(mx_quantise_kernel<T, decltype(fmt)::value>, dim3(static_cast<unsigned>(tiles)), kMxThreads, 0, stream,
                            static_cast<const T*>(x), row_stride, rows, cols, col_tiles, codes, reinterpret_cast<uint32_t*>(scales));
  });
}

lite3r_status launch_mx_dequantise(const uint8_t* codes, const uint8_t* scales, int rows, int cols, int format, void* out,
                                   int dtype, long long row_stride, cudaStream_t stream) {
  const int col_tiles = ceil_div(cols, kMxCols);
  const long long tiles = static_cast<long long>(ceil_div(rows, kMxRows)) * col_tiles;
  if (tiles > 0x7FFFFFFFLL) return LITE3R_ERR_UNSUPPORTED;
  return by_type(dtype, format, [&](auto type, auto fmt) {
    using T = decltype(type);
    return launch_dependent(mx_dequantise_kernel<T, decltype(fmt)::value>, dim3(static_cast<unsigned>(tiles)), kMxThreads, 0, stream,
                            codes, reinterpret_cast<const uint32_t*>(scales), rows, cols, col_tiles, static_cast<T*>(out), row_stride);
  });
}

}  // namespace lite3r
