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
// Bound by HBM: 43968 x 4096 bf16 values to 4 bits in 67 us (456 MB, 6.8 TB/s), to 8 bits in 81 (546 MB), back in 72 and 86, 6.3 TB/s
// (in a run of a second at the power limit 74, 86, 75 and 89).  With scalar maxima, products and conversions it was bound by its
// 100 instructions per 256 values (now 59): 99 us.
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

__device__ __forceinline__ float max_nan(float a, float b) {
  float m;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
  return m;
}

// Eight values as they lie in memory, and the largest magnitude of them and of the three neighbouring lanes (a block) as fp32
// bits: NaN above infinity above all else.
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
  __device__ __forceinline__ void pairs(uint64_t v[4]) const {
    v[0] = pack_f32x2(a.x, a.y); v[1] = pack_f32x2(a.z, a.w);
    v[2] = pack_f32x2(b.x, b.y); v[3] = pack_f32x2(b.z, b.w);
  }
  __device__ __forceinline__ uint32_t block_top() const {
    float m = max_nan(max_nan(max_nan(fabsf(a.x), fabsf(a.y)), max_nan(fabsf(a.z), fabsf(a.w))),
                      max_nan(max_nan(fabsf(b.x), fabsf(b.y)), max_nan(fabsf(b.z), fabsf(b.w))));
    m = max_nan(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
    m = max_nan(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
    return __float_as_uint(m) & 0x7FFFFFFFu;
  }
};
// The 16-bit types, two values at a time (H2: __nv_bfloat162 or __half2).
template <typename T, typename H2>
struct Octet16 {
  uint4 w;
  __device__ __forceinline__ void load(const T* p) { w = __ldg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void clear() { w = make_uint4(0u, 0u, 0u, 0u); }
  static __device__ __forceinline__ H2 two(uint32_t x) { return *reinterpret_cast<const H2*>(&x); }
  static __device__ __forceinline__ uint32_t bits(H2 x) { return *reinterpret_cast<const uint32_t*>(&x); }
  __device__ __forceinline__ uint32_t block_top16() const {
    H2 m = __hmax2_nan(__hmax2_nan(__habs2(two(w.x)), __habs2(two(w.y))), __hmax2_nan(__habs2(two(w.z)), __habs2(two(w.w))));
    m = __hmax2_nan(m, two(__shfl_xor_sync(0xFFFFFFFFu, bits(m), 1)));
    m = __hmax2_nan(m, two(__shfl_xor_sync(0xFFFFFFFFu, bits(m), 2)));
    return bits(__hmax2_nan(m, __lowhigh2highlow(m))) & 0x7FFFu;
  }
};
template <>
struct Octet<__nv_bfloat16> : Octet16<__nv_bfloat16, __nv_bfloat162> {
  __device__ __forceinline__ void pairs(uint64_t v[4]) const {
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack_f32x2(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xFFFF0000u));
  }
  __device__ __forceinline__ uint32_t block_top() const { return block_top16() << 16; }
};
template <>
struct Octet<__half> : Octet16<__half, __half2> {
  __device__ __forceinline__ void pairs(uint64_t v[4]) const {
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(two(x[i]));
      v[i] = pack_f32x2(f.x, f.y);
    }
  }
  __device__ __forceinline__ uint32_t block_top() const {
    return __float_as_uint(__half2float(__ushort_as_half(static_cast<unsigned short>(block_top16()))));
  }
};

// Four pairs of values to codes.
__device__ __forceinline__ uint32_t e2m1x8(const uint64_t v[4]) {
  float a[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) unpack_f32x2(v[i], a[2 * i], a[2 * i + 1]);
  uint32_t r;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
      "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
      : "=r"(r)
      : "f"(a[0]), "f"(a[1]), "f"(a[2]), "f"(a[3]), "f"(a[4]), "f"(a[5]), "f"(a[6]), "f"(a[7]));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x4(uint64_t x, uint64_t y) {
  float a, b, c, d;
  unpack_f32x2(x, a, b);
  unpack_f32x2(y, c, d);
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
      "mov.b32 %0, {lo, hi};\n\t}"
      : "=r"(r)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}

// Row pitch of the codes in bytes.
template <int kFormat>
__device__ __forceinline__ size_t code_pitch(int cols) { return kFormat == LITE3R_MXFP4 ? cols / 2 : cols; }

// A thread's eight values of every sixteenth row of a tile; rows and cols are those of the tile inside the matrix, kFull: all.
template <typename T, int kFormat, bool kFull>
__device__ __forceinline__ void quantise_tile(const T* __restrict__ x, long long row_stride, int rows, int cols, uint8_t* __restrict__ codes,
                                              size_t pitch, uint32_t scales_at, int r0, int lane16) {
  Octet<T> in[kMxIters];
#pragma unroll
  for (int i = 0; i < kMxIters; ++i) {
    if (kFull || (r0 + 16 * i < rows && lane16 * 8 < cols)) in[i].load(x + 16 * i * row_stride);
    else in[i].clear();
  }
#pragma unroll
  for (int i = 0; i < kMxIters; ++i) {
    const uint32_t byte = scale_byte<kFormat>(in[i].block_top());
    // row r0 + 16 i of the tile, r0 < 16
    if ((lane16 & 3) == 0)
      asm volatile("st.shared.u8 [%0], %1;" ::"r"(scales_at + (i & 1) * 256 + (i >> 1) * 4), "r"(byte) : "memory");
    if (kFull || (r0 + 16 * i < rows && lane16 * 8 < cols)) {
      const float inverse = __uint_as_float((254u << 23) - (byte << 23));  // (a block of NaN: whatever it is)
      const uint64_t factor = pack_f32x2(inverse, inverse);
      uint64_t v[4];
      in[i].pairs(v);
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = mul_f32x2(v[q], factor);
      uint8_t* const dst = codes + 16 * i * pitch;
      if constexpr (kFormat == LITE3R_MXFP8) {
        uint2 w = make_uint2(e4m3x4(v[0], v[1]), e4m3x4(v[2], v[3]));
        if (byte == 0xFFu) w = make_uint2(0x7F7F7F7Fu, 0x7F7F7F7Fu);
        *reinterpret_cast<uint2*>(dst) = w;
      } else {
        const uint32_t w = e2m1x8(v);
        *reinterpret_cast<uint32_t*>(dst) = byte == 0xFFu ? 0x22222222u : w;
      }
    }
  }
}

template <typename T, int kFormat>
__global__ void __launch_bounds__(kMxThreads) mx_quantise_kernel(const T* __restrict__ x, long long row_stride, int rows, int cols,
                                                                int col_tiles, uint8_t* __restrict__ codes,
                                                                uint32_t* __restrict__ scales) {
  __shared__ __align__(16) uint8_t s_scales[512];
  const int row_tile = blockIdx.x / col_tiles, col_tile = blockIdx.x - row_tile * col_tiles;
  const int lane16 = threadIdx.x & 15, col0 = col_tile * kMxCols;
  const int r0 = threadIdx.x >> 4;  // of the sixteen rows of a step
  const long long row0 = static_cast<long long>(row_tile) * kMxRows;
  wait_for_prior_grid();
  launch_dependents();
  // byte of row r, block j at (r % 32) * 16 + (r / 32) * 4 + j
  const uint32_t scales_at = smem_u32(s_scales) + r0 * 16 + (lane16 >> 2);
  const T* const src = x + (row0 + r0) * row_stride + col0 + lane16 * 8;
  uint8_t* const dst = codes + static_cast<size_t>(row0 + r0) * code_pitch<kFormat>(cols) + (col0 + lane16 * 8) / (kFormat == LITE3R_MXFP4 ? 2 : 1);
  const int rows_left = static_cast<int>(min(static_cast<long long>(kMxRows), rows - row0)), cols_left = min(kMxCols, cols - col0);
  const size_t pitch = code_pitch<kFormat>(cols);
  if (rows_left == kMxRows && cols_left == kMxCols) quantise_tile<T, kFormat, true>(src, row_stride, rows_left, cols_left, dst, pitch, scales_at, r0, lane16);
  else quantise_tile<T, kFormat, false>(src, row_stride, rows_left, cols_left, dst, pitch, scales_at, r0, lane16);
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
