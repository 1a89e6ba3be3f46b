// Backward pass of a linear layer whose weight and whose kept input are microscaled codes:
//   dgrad   dx = dy . Q(W)        [rows, d_in] = [rows, d_out] x [d_out, d_in]
//   wgrad   dW = dy^T . C(x)      [d_out, d_in] = [d_out, rows] x [rows, d_in],   db = sum of dy over the rows
// Both are products C[m][n] = sum_r A(m, r) B[r][n] of bf16 values with codes whose blocks of 32 run along n.  A block's scale
// is not constant along the contraction, so block-scaled products cannot take it; the codes become bf16 on their way to the
// tensor cores instead, which is exact (e4m3 and e2m1 have at most four significant bits and the scales are powers of two).
// Persistent CTAs over tiles of 128 x 256 (wgrad: times a part of the rows).  Warp 0 loads codes and scales, warp 2 the tiles
// of dy (for wgrad as they lie, the contraction along the rows: M-major), eight warps turn codes into the bf16 operand in
// shared memory (N-major, 128B swizzle), warp 1 issues the products into one of two accumulators, four warps are the epilogue.
// The tensor cores' running sum is cut off, not rounded, at fp32: it drifts towards zero by about 4e-9 of the result per
// product of 16 steps (10992 rows in one sum: dW off by 2.6e-6).  Results in fp32 are therefore summed over 2048 steps at a time
// and the sums added with rounding by the store engine, in order, as each is finished.  The parts of the rows that wgrad gives
// to different CTAs are added in a fixed order by a second kernel: no floating-point atomics between CTAs.
// Every mbarrier wait is bounded; on expiry the CTA sets *device_status and its roles leave their loops.
#include <algorithm>

#include <cuda_fp4.h>

#include "common.cuh"
#include "sm100.cuh"

namespace lite3r {

namespace {

using namespace sm100;

constexpr int kTileM = 128, kTileN = 256, kTileR = 64;
constexpr int kScaleTile = 512;
constexpr int kConvWarps = 8;
constexpr int kThreads = 128 + 32 * kConvWarps + 128;
constexpr uint32_t kTmemCols = 512;

template <int kFormat>
struct Layout {
  static constexpr int kRaw = 3, kOps = 3;                       // stages of codes, stages of operands
  static constexpr int kRowBytes = kFormat == LITE3R_MXFP8 ? kTileN : kTileN / 2;
  static constexpr uint32_t kOffB = kTileM * kTileR * 2;         // A, then B as four boxes of 64 columns x 64 rows
  static constexpr uint32_t kOpBytes = kOffB + kTileN * kTileR * 2;
  static constexpr uint32_t kOffRaw = kOps * kOpBytes;
  static constexpr uint32_t kOffScales = kTileR * kRowBytes;     // of a raw stage: two scale tiles
  static constexpr uint32_t kRawBytes = kOffScales + 2 * kScaleTile;
  static constexpr uint32_t kOffOut = kOffRaw + kRaw * kRawBytes;  // 4 KB per epilogue warp
  static constexpr uint32_t kOffBar = kOffOut + 4 * 4096;
  static constexpr uint32_t kSmemBytes = kOffBar + 256;
  static_assert(kOffOut % 1024 == 0 && kSmemBytes <= 232448, "fits");
};

struct Bars {
  uint64_t raw_full[3], raw_empty[3], a_full[3], b_full[3], op_empty[3];
  uint64_t acc_full[2], acc_empty[2];
  uint32_t tmem_base;
  int abort;
};

struct BackParams {
  const uint8_t* scales;
  int n_total;               // d_in
  int scale_tiles;           // along n
  int steps, steps_per_part; // of 64 along the contraction, in all and of one part of it
  int steps_per_sum;         // of one running sum in tensor memory
  int col_tiles, tiles, units;
  int out_dtype;
  int* status;
};

// bf16 pairs of four codes (eight bits each) or eight (four bits each) without their block's scale: values times 2^-120
// (e4m3) or as they are (e2m1).
template <int kFormat>
struct Codes;
template <>
struct Codes<LITE3R_MXFP8> {
  static constexpr int kBias = 120;
  uint2 w;
  __device__ __forceinline__ void load(const uint8_t* raw, int chunk) { w = *(reinterpret_cast<const uint2*>(raw) + chunk); }
  // sign to bit 15, the four exponent bits behind bf16's bias, three mantissa bits on top of seven
  static __device__ __forceinline__ uint32_t spread(uint32_t pair) { return ((pair >> 4) & 0x07F007F0u) | (pair & 0x80008000u); }
  __device__ __forceinline__ void pairs(uint32_t out[4]) const {
    out[0] = spread(__byte_perm(w.x, 0u, 0x1404));
    out[1] = spread(__byte_perm(w.x, 0u, 0x3424));
    out[2] = spread(__byte_perm(w.y, 0u, 0x1404));
    out[3] = spread(__byte_perm(w.y, 0u, 0x3424));
  }
};
template <>
struct Codes<LITE3R_MXFP4> {
  static constexpr int kBias = 0;
  uint32_t w;
  __device__ __forceinline__ void load(const uint8_t* raw, int chunk) { w = *(reinterpret_cast<const uint32_t*>(raw) + chunk); }
  // the high and low bytes of the eight magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6 as bf16, by table
  __device__ __forceinline__ void pairs(uint32_t out[4]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t four = w >> (16 * i), sel = four & 0x7777u;
      const uint32_t hi = __byte_perm(0x3F3F3F00u, 0x40404040u, sel), lo = __byte_perm(0xC0800000u, 0xC0804000u, sel);
      out[2 * i] = __byte_perm(lo, hi, 0x5140) | ((four << 12) & 0x8000u) | ((four << 24) & 0x80000000u);
      out[2 * i + 1] = __byte_perm(lo, hi, 0x7362) | ((four << 4) & 0x8000u) | ((four << 16) & 0x80000000u);
    }
  }
};

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// 2^(byte - 127 + kBias) as a pair of bf16; the byte 0xFF stands for NaN.  Where that is beyond bf16's largest power the
// factor is made of two.
template <int kBias>
__device__ __forceinline__ void scale_pairs(uint32_t v[4], uint32_t byte) {
  uint32_t e = byte + kBias;
  if (e > 254u) {
    constexpr uint32_t kFirst = (static_cast<uint32_t>(kBias) + 127u) << 7;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = mul_bf16x2(v[i], kFirst | kFirst << 16);
    e = byte;
  }
  uint32_t f = e == 0u ? 0x0040u : e << 7;
  if (byte == 0xFFu) f = 0x7FC0u;
  f |= f << 16;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = mul_bf16x2(v[i], f);
}

template <int kFormat, bool kWgrad>
__global__ void __launch_bounds__(kThreads, 1)
mx_back_kernel(const __grid_constant__ CUtensorMap map_dy, const __grid_constant__ CUtensorMap map_codes,
               const __grid_constant__ CUtensorMap map_out, const BackParams p) {
  using L = Layout<kFormat>;
  constexpr int kRaw = L::kRaw, kOps = L::kOps;
  extern __shared__ __align__(1024) uint8_t smem[];
  Bars* bars = reinterpret_cast<Bars*>(smem + L::kOffBar);
  volatile int* abort_flag = &bars->abort;
  if ((smem_u32(smem) & 1023u) != 0) {
    if (threadIdx.x == 0 && p.status != nullptr) atomicCAS(p.status, 0, 900);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kRaw; ++s) {
      mbar_init(&bars->raw_full[s], 1);
      mbar_init(&bars->raw_empty[s], kConvWarps);
    }
    for (int s = 0; s < kOps; ++s) {
      mbar_init(&bars->a_full[s], 1);
      mbar_init(&bars->b_full[s], kConvWarps);
      mbar_init(&bars->op_empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&bars->acc_full[b], 1);
      mbar_init(&bars->acc_empty[b], 4);
    }
    bars->abort = 0;
    mbar_fence_init();
  }
  if (warp == 1) {
    tmem_alloc(&bars->tmem_base, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars->tmem_base;
  wait_for_prior_grid();
  launch_dependents();
  if (blockIdx.x == 0 && threadIdx.x == 0 && p.status != nullptr) *p.status = 0;

  struct UnitAt {
    int m0, n0, part, first, last;  // steps [first, last) of the contraction
  };
  auto unit_at = [&](int unit) {
    UnitAt u;
    u.part = kWgrad ? unit / p.tiles : 0;
    const int tile = unit - u.part * p.tiles, row_tile = tile / p.col_tiles;
    u.m0 = row_tile * kTileM;
    u.n0 = (tile - row_tile * p.col_tiles) * kTileN;
    u.first = u.part * p.steps_per_part;
    u.last = min(u.first + p.steps_per_part, p.steps);
    return u;
  };

  if (warp == 0) {
    if (lane == 0) {
      tma_prefetch_desc(&map_codes);
      bool ok = true;
      int kc = 0;
      for (int unit = blockIdx.x; ok && unit < p.units; unit += gridDim.x) {
        const UnitAt u = unit_at(unit);
        const int scale_tiles = min(2, p.scale_tiles - u.n0 / 128);
        for (int k = u.first; ok && k < u.last; ++k, ++kc) {
          const int st = kc % kRaw;
          if (kc >= kRaw) ok = mbar_wait_clearing(&bars->raw_empty[st], ((kc - kRaw) / kRaw) & 1, abort_flag, p.status, 811, 32);
          if (!ok) break;
          uint8_t* const dst = smem + L::kOffRaw + st * L::kRawBytes;
          mbar_arrive_expect_tx(&bars->raw_full[st], kTileR * L::kRowBytes + scale_tiles * kScaleTile);
          tma_load_2d(dst, &map_codes, &bars->raw_full[st], kFormat == LITE3R_MXFP8 ? u.n0 : u.n0 / 2, k * kTileR);
          bulk_load(dst + L::kOffScales, p.scales + (static_cast<size_t>(k / 2) * p.scale_tiles + u.n0 / 128) * kScaleTile,
                    scale_tiles * kScaleTile, &bars->raw_full[st]);
        }
      }
    }
  } else if (warp == 2) {
    if (lane == 0) {
      tma_prefetch_desc(&map_dy);
      bool ok = true;
      int kc = 0;
      for (int unit = blockIdx.x; ok && unit < p.units; unit += gridDim.x) {
        const UnitAt u = unit_at(unit);
        for (int k = u.first; ok && k < u.last; ++k, ++kc) {
          const int st = kc % kOps;
          if (kc >= kOps) ok = mbar_wait_clearing(&bars->op_empty[st], ((kc - kOps) / kOps) & 1, abort_flag, p.status, 812, 32);
          if (!ok) break;
          uint8_t* const dst = smem + st * L::kOpBytes;
          mbar_arrive_expect_tx(&bars->a_full[st], kTileM * kTileR * 2);
          if constexpr (kWgrad) {  // two boxes of 64 columns x 64 rows of dy
            tma_load_2d(dst, &map_dy, &bars->a_full[st], u.m0, k * kTileR);
            tma_load_2d(dst + 8192, &map_dy, &bars->a_full[st], u.m0 + 64, k * kTileR);
          } else {
            tma_load_2d(dst, &map_dy, &bars->a_full[st], k * kTileR, u.m0);
          }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr uint32_t idesc = instr_desc(1, kTileM, kTileN, kWgrad ? 1 : 0, 1);
      const uint32_t base = smem_u32(smem);
      bool ok = true;
      int kc = 0, it = 0;
      for (int unit = blockIdx.x; ok && unit < p.units; unit += gridDim.x) {
        const UnitAt u = unit_at(unit);
        for (int k0 = u.first; ok && k0 < u.last; k0 += p.steps_per_sum, ++it) {
        const int ab = it & 1, k1 = min(k0 + p.steps_per_sum, u.last);
        if (it >= 2) ok = mbar_wait_clearing(&bars->acc_empty[ab], ((it - 2) >> 1) & 1, abort_flag, p.status, 814);
        tc_fence_after();
        for (int k = k0; ok && k < k1; ++k, ++kc) {
          const int st = kc % kOps;
          ok = mbar_wait_clearing(&bars->a_full[st], (kc / kOps) & 1, abort_flag, p.status, 815) &&
               mbar_wait_clearing(&bars->b_full[st], (kc / kOps) & 1, abort_flag, p.status, 816);
          if (!ok) break;
          tc_fence_after();
          const uint32_t a = base + st * L::kOpBytes, b = a + L::kOffB;
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {  // 16 steps of the contraction each
            const uint64_t a_desc = kWgrad ? smem_desc(a + kk * 2048, 8192, 1024, kSwizzle128) : smem_desc(a + kk * 32, 16, 1024, kSwizzle128);
            mma_f16(tmem + ab * kTileN, a_desc, smem_desc(b + kk * 2048, 8192, 1024, kSwizzle128), idesc, (k > k0 || kk > 0) ? 1u : 0u);
          }
          mma_commit(&bars->op_empty[st]);
        }
        if (ok) mma_commit(&bars->acc_full[ab]);
        }
      }
    }
  } else if (warp >= 4 && warp < 4 + kConvWarps) {
    // ------------------------------------------------------------------------------------------ codes to bf16
    constexpr int kPerRow = kTileN / 8;                            // chunks of eight columns
    constexpr int kChunks = kTileR * kPerRow / (32 * kConvWarps);  // of a thread
    const int first = (warp - 4) * 32 + lane;
    bool ok = true;
    int kc = 0;
    for (int unit = blockIdx.x; ok && unit < p.units; unit += gridDim.x) {
      const UnitAt u = unit_at(unit);
      for (int k = u.first; ok && k < u.last; ++k, ++kc) {
        const int rs = kc % kRaw, st = kc % kOps;
        ok = mbar_wait_clearing(&bars->raw_full[rs], (kc / kRaw) & 1, abort_flag, p.status, 817);
        if (ok && kc >= kOps) ok = mbar_wait_clearing(&bars->op_empty[st], ((kc - kOps) / kOps) & 1, abort_flag, p.status, 818);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        const uint8_t* const raw = smem + L::kOffRaw + rs * L::kRawBytes;
        const uint8_t* const scales = raw + L::kOffScales;
        const uint32_t dst = smem_u32(smem) + st * L::kOpBytes + L::kOffB;
        Codes<kFormat> c[kChunks];
        uint32_t byte[kChunks];
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
          const int id = first + i * 32 * kConvWarps, row = id / kPerRow, chunk = id % kPerRow;
          const int r = (k & 1) * 64 + row;  // of the scale tile's 128 rows
          c[i].load(raw, id);
          byte[i] = scales[(chunk >> 4) * kScaleTile + (r & 31) * 16 + (r >> 5) * 4 + ((chunk >> 2) & 3)];
        }
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
          const int id = first + i * 32 * kConvWarps, row = id / kPerRow, chunk = id % kPerRow;
          uint32_t v[4];
          c[i].pairs(v);
          scale_pairs<Codes<kFormat>::kBias>(v, byte[i]);
          sts128(dst + (chunk >> 3) * 8192 + row * 128 + (((chunk & 7) ^ (row & 7)) << 4), v[0], v[1], v[2], v[3]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&bars->b_full[st]);
          mbar_arrive(&bars->raw_empty[rs]);
        }
      }
    }
  } else if (warp >= 4 + kConvWarps) {
    // ------------------------------------------------------------------------------------------ epilogue
    const int quarter = warp & 3;
    uint8_t* const warp_tile = smem + L::kOffOut + quarter * 4096;
    const uint32_t my_row = smem_u32(warp_tile) + lane * 128;
    const int swz = lane & 7;
    const bool wide = kWgrad || p.out_dtype == LITE3R_F32;
    bool ok = true;
    int it = 0;
    for (int unit = blockIdx.x; ok && unit < p.units; unit += gridDim.x) {
      const UnitAt u = unit_at(unit);
      for (int k0 = u.first; ok && k0 < u.last; k0 += p.steps_per_sum, ++it) {
      const int ab = it & 1;
      const bool add = k0 > u.first;  // to the sum before, which this warp has stored
      const uint32_t acc_addr = tmem + ((static_cast<uint32_t>(quarter) * 32u) << 16) + ab * kTileN;
      ok = mbar_wait_clearing(&bars->acc_full[ab], (it >> 1) & 1, abort_flag, p.status, 813);
      tc_fence_after();
      ok = __all_sync(0xFFFFFFFFu, ok);
      if (!ok) break;
      if (add && lane == 0) bulk_wait_group0();  // it is in place
      const int cols = min(kTileN, p.n_total - u.n0);  // a multiple of 32
#pragma unroll 1
      for (int cb = 0; cb < cols; cb += 32) {
        uint32_t v[32];
        tmem_ld32(acc_addr + cb, v);
        if (wide || (cb & 32) == 0) {  // what was staged here before has been read by the store engine
          if (lane == 0) bulk_wait_group_read0();
          __syncwarp();
        }
        tmem_wait_ld();
        if (wide) {
#pragma unroll
          for (int c = 0; c < 8; ++c) sts128(my_row + ((c ^ swz) << 4), v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const float y0 = __uint_as_float(v[8 * c + 2 * q]), y1 = __uint_as_float(v[8 * c + 2 * q + 1]);
              if (p.out_dtype == LITE3R_BF16) {
                __nv_bfloat162 h = __floats2bfloat162_rn(y0, y1);
                w[q] = *reinterpret_cast<uint32_t*>(&h);
              } else {
                __half2 h = __floats2half2_rn(y0, y1);
                w[q] = *reinterpret_cast<uint32_t*>(&h);
              }
            }
            sts128(my_row + ((((cb & 32) / 8 + c) ^ swz) << 4), w[0], w[1], w[2], w[3]);
          }
        }
        if (wide || (cb & 32) != 0 || cb + 32 >= cols) {  // (the engine clips columns past the output)
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            const int x = u.n0 + (wide ? cb : cb & ~63);
            const int y = u.m0 + quarter * 32;
            if constexpr (kWgrad) {
              if (add) tma_add_3d(&map_out, warp_tile, x, y, u.part);
              else tma_store_3d(&map_out, warp_tile, x, y, u.part);
            } else {
              if (add) tma_add_2d(&map_out, warp_tile, x, y);
              else tma_store_2d(&map_out, warp_tile, x, y);
            }
            bulk_commit_group();
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->acc_empty[ab]);
      }
    }
    bulk_wait_group_read0();  // what is staged stays in place until it has been read
  }

  tc_fence_before();
  __syncthreads();
  linger_after_abort(abort_flag);
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

// ------------------------------------------------------------------------------------------------ sums
constexpr int kBiasParts = 64;  // parts of the rows whose column sums are added by the second kernel

// Column sums of dy over one part of the rows: eight columns per thread, eight row groups per CTA.
__global__ void __launch_bounds__(256) bias_parts_kernel(const __nv_bfloat16* __restrict__ dy, long long stride, int rows, int d_out,
                                                         int rows_per_part, float* __restrict__ parts) {
  __shared__ float s_sum[8][256];
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
  const int col = blockIdx.x * 256 + lane * 8;
  const int r0 = blockIdx.y * rows_per_part, r1 = min(r0 + rows_per_part, rows);
  float acc[8] = {};
  wait_for_prior_grid();
  launch_dependents();
  if (col < d_out) {
#pragma unroll 4
    for (int r = r0 + group; r < r1; r += 8) {
      const __nv_bfloat16* src = dy + static_cast<long long>(r) * stride + col;
      if (col + 8 <= d_out) {
        const uint4 w = __ldg(reinterpret_cast<const uint4*>(src));
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc[2 * i] += __uint_as_float(x[i] << 16);
          acc[2 * i + 1] += __uint_as_float(x[i] & 0xFFFF0000u);
        }
      } else {
        for (int i = 0; i < d_out - col; ++i) acc[i] += __bfloat162float(src[i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) s_sum[group][lane * 8 + i] = acc[i];
  __syncthreads();
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c < d_out) {
    float sum = 0.f;
#pragma unroll
    for (int g = 0; g < 8; ++g) sum += s_sum[g][threadIdx.x];
    parts[static_cast<size_t>(blockIdx.y) * d_out + c] = sum;
  }
}

// out[i] = sum over the parts, in order (four values per thread where that is possible).
template <int kVec>
__global__ void __launch_bounds__(256) add_parts_kernel(const float* parts, int count, size_t values, float* __restrict__ out) {
  wait_for_prior_grid();
  launch_dependents();
  const size_t i = (static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x) * kVec;
  if (i >= values) return;
  float acc[kVec] = {};
#pragma unroll 4
  for (int s = 0; s < count; ++s) {
    const float* src = parts + static_cast<size_t>(s) * values + i;
    if constexpr (kVec == 4) {
      const float4 v = *reinterpret_cast<const float4*>(src);
      acc[0] += v.x; acc[1] += v.y; acc[2] += v.z; acc[3] += v.w;
    } else {
      acc[0] += src[0];
    }
  }
  if constexpr (kVec == 4) *reinterpret_cast<float4*>(out + i) = make_float4(acc[0], acc[1], acc[2], acc[3]);
  else out[i] = acc[0];
}

// Parts of the rows: as many as give every SM a tile, none shorter than sixteen steps.
int parts_of(int steps, int tiles, int sms) {
  return std::max(1, std::min(ceil_div(sms, tiles), steps / 16));
}
constexpr int kMostSms = 256;  // of any device, for the size of the workspace

template <int kFormat, bool kWgrad>
lite3r_status launch_back(const void* dy, long long dy_stride, const uint8_t* codes, const uint8_t* scales, int rows, int d_in,
                          int d_out, const CUtensorMap& map_out, int out_dtype, int parts, int* status, int sms, cudaStream_t stream) {
  using L = Layout<kFormat>;
  CUtensorMap map_dy, map_codes;
  lite3r_status st;
  if ((st = make_tensor_map_2d(&map_dy, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, dy, d_out, rows, 64, kWgrad ? 64 : kTileM,
                               CU_TENSOR_MAP_SWIZZLE_128B, static_cast<uint64_t>(dy_stride) * 2)) != LITE3R_OK) return st;
  const int code_rows = kWgrad ? rows : d_out;
  if ((st = make_tensor_map_2d(&map_codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, codes, kFormat == LITE3R_MXFP8 ? d_in : d_in / 2, code_rows,
                               L::kRowBytes, kTileR, CU_TENSOR_MAP_SWIZZLE_NONE)) != LITE3R_OK) return st;
  auto* kernel = mx_back_kernel<kFormat, kWgrad>;
  if ((st = ensure_dynamic_smem(kernel, static_cast<int>(L::kSmemBytes))) != LITE3R_OK) return st;
  BackParams p = {};
  p.scales = scales;
  p.n_total = d_in;
  p.scale_tiles = ceil_div(d_in, 128);
  p.steps = ceil_div(code_rows, kTileR);
  p.steps_per_part = ceil_div(p.steps, parts);
  p.steps_per_sum = out_dtype == LITE3R_F32 ? 2048 / kTileR : p.steps;
  p.col_tiles = ceil_div(d_in, kTileN);
  const long long tiles = static_cast<long long>(p.col_tiles) * ceil_div(kWgrad ? d_out : rows, kTileM);
  if (tiles * parts > 0x7FFFFFFFLL - 1024) return LITE3R_ERR_UNSUPPORTED;
  p.tiles = static_cast<int>(tiles);
  p.units = p.tiles * parts;
  p.out_dtype = out_dtype;
  p.status = status;
  return launch_dependent(kernel, dim3(static_cast<unsigned>(std::min(p.units, sms))), kThreads, static_cast<int>(L::kSmemBytes), stream,
                          map_dy, map_codes, map_out, p);
}

long long wgrad_tiles(int d_in, int d_out) { return static_cast<long long>(ceil_div(d_in, kTileN)) * ceil_div(d_out, kTileM); }

// Parts after rounding their length up to whole steps: none is empty.
int wgrad_parts(int rows, int d_in, int d_out, int sms) {
  const int steps = ceil_div(rows, kTileR);
  const int parts = parts_of(steps, static_cast<int>(std::min<long long>(wgrad_tiles(d_in, d_out), 1 << 20)), sms);
  return ceil_div(steps, ceil_div(steps, parts));
}

}  // namespace

size_t linear_mx_workspace_bytes(int rows, int d_in, int d_out) {
  const int steps = ceil_div(rows, kTileR);
  const int parts = parts_of(steps, static_cast<int>(std::min<long long>(wgrad_tiles(d_in, d_out), 1 << 20)), kMostSms);
  const size_t products = parts > 1 ? static_cast<size_t>(parts) * d_in * d_out : 0;
  return (products + static_cast<size_t>(kBiasParts) * d_out) * sizeof(float) + 256;
}

lite3r_status launch_mx_dgrad(const void* dy, long long dy_stride, const uint8_t* w_codes, const uint8_t* w_scales, int format,
                              int rows, int d_in, int d_out, void* dx, int dx_dtype, long long dx_stride, int* device_status,
                              cudaStream_t stream) {
  int sms = 0;
  lite3r_status st = sm_count(&sms);
  if (st != LITE3R_OK) return st;
  const int elem = dx_dtype == LITE3R_F32 ? 4 : 2;
  CUtensorMap map;
  st = make_tensor_map_2d(&map,
                          dx_dtype == LITE3R_F32    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                          : dx_dtype == LITE3R_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                    : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                          elem, dx, d_in, rows, 128 / elem, 32, CU_TENSOR_MAP_SWIZZLE_128B, static_cast<uint64_t>(dx_stride) * elem);
  if (st != LITE3R_OK) return st;
  return format == LITE3R_MXFP8 ? launch_back<LITE3R_MXFP8, false>(dy, dy_stride, w_codes, w_scales, rows, d_in, d_out, map, dx_dtype, 1, device_status, sms, stream)
                                : launch_back<LITE3R_MXFP4, false>(dy, dy_stride, w_codes, w_scales, rows, d_in, d_out, map, dx_dtype, 1, device_status, sms, stream);
}

lite3r_status launch_mx_wgrad(const void* dy, long long dy_stride, const uint8_t* x_codes, const uint8_t* x_scales, int format,
                              int rows, int d_in, int d_out, float* dw, float* db, float* workspace, int* device_status,
                              cudaStream_t stream) {
  int sms = 0;
  lite3r_status st = sm_count(&sms);
  if (st != LITE3R_OK) return st;
  const int parts = wgrad_parts(rows, d_in, d_out, std::min(sms, kMostSms));
  const size_t values = static_cast<size_t>(d_in) * d_out;
  float* const products = parts > 1 ? workspace : dw;
  float* const bias_parts = workspace + (parts > 1 ? parts * values : 0);
  CUtensorMap map;
  if ((st = make_tensor_map_3d(&map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, products, d_in, d_out, parts, 32, 32, CU_TENSOR_MAP_SWIZZLE_128B)) != LITE3R_OK)
    return st;
  st = format == LITE3R_MXFP8 ? launch_back<LITE3R_MXFP8, true>(dy, dy_stride, x_codes, x_scales, rows, d_in, d_out, map, LITE3R_F32, parts, device_status, sms, stream)
                              : launch_back<LITE3R_MXFP4, true>(dy, dy_stride, x_codes, x_scales, rows, d_in, d_out, map, LITE3R_F32, parts, device_status, sms, stream);
  if (st != LITE3R_OK) return st;
  if (parts > 1) {  // (d_in is a multiple of 32)
    st = launch_dependent(add_parts_kernel<4>, dim3(static_cast<unsigned>((values / 4 + 255) / 256)), 256, 0, stream,
                          static_cast<const float*>(products), parts, values, dw);
    if (st != LITE3R_OK) return st;
  }
  if (db == nullptr) return LITE3R_OK;
  const int row_parts = std::min(kBiasParts, ceil_div(rows, 64));
  const int rows_per_part = ceil_div(rows, row_parts);
  const int used = ceil_div(rows, rows_per_part);
  st = launch_dependent(bias_parts_kernel, dim3(static_cast<unsigned>(ceil_div(d_out, 256)), static_cast<unsigned>(used)), 256, 0, stream,
                        static_cast<const __nv_bfloat16*>(dy), dy_stride, rows, d_out, rows_per_part, bias_parts);
  if (st != LITE3R_OK) return st;
  return launch_dependent(add_parts_kernel<1>, dim3(static_cast<unsigned>(ceil_div(d_out, 256))), 256, 0, stream,
                          static_cast<const float*>(bias_parts), used, static_cast<size_t>(d_out), db);
}

}  // namespace lite3r
