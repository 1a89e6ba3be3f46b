// Backward pass of a linear layer whose weight and whose kept input are microscaled codes:
//   dgrad   dx = dy . Q(W)        [rows, d_in] = [rows, d_out] x [d_out, d_in]
//   wgrad   dW = dy^T . C(x)      [d_out, d_in] = [d_out, rows] x [rows, d_in],   db = sum of dy over the rows
// Both are products C[m][n] = sum_r A(m, r) B[r][n] of bf16 values with codes whose blocks of 32 run along n.  A block's scale
// is not constant along the contraction, so block-scaled products cannot take it; the codes become bf16 on their way to the
// tensor cores instead, which is exact (e4m3 and e2m1 have at most four significant bits and the scales are powers of two).
//
// Pairs of CTAs (cta_group::2) walk tiles of 256 x 256 or 256 x 128 (wgrad: times a part of the rows): each CTA has 128 rows of A
// and half of B's columns.  Per CTA: warp 0 loads codes and scales, warp 2 the tiles of dy (for wgrad as they lie, the contraction
// along the rows: M-major), sixteen warps turn codes into the bf16 operand in shared memory (N-major, 128B swizzle), warp 1 of
// the pair's first CTA issues the products into one of two accumulators, four warps are the epilogue.
// The sixteen warps work in four groups, each on every fourth step: a step's chain of load, arithmetic, store and proxy fence
// takes longer than its products (1900 cycles of a step with all warps on the same one, 512 of products), four chains side by
// side do not.  Each CTA converts half of B for the pair.  10992 x 1024 x 4096 (92 GFLOP each): dgrad 75 us, wgrad 81, or 90 with
// db, the tensor pipe busy for 62 to 65 %; in a run of a second, at the 1.5 GHz that the power limit leaves, 88, 95 and 102.
// (76 us with the conversion left out: shared memory carries the products' operands, dy, the codes and what is made of them.  A
// group also holds one of the five stages of operands through its arithmetic; and wgrad's 64 tiles leave 10 of 74 pairs idle.)
// For db the groups also add up the columns of dy while its tile lies in shared memory, the first four column tiles by turns.
//
// The second CTA's warps tell the first one that their half is there by 16 bytes of it, copied to a place there that nothing
// reads, which the first one's barrier counts.
//
// The tensor cores' running sum is cut off, not rounded, at fp32: it drifts towards zero by about 4e-9 of the result per
// product of 16 steps (10992 rows in one sum: dW off by 2.6e-6).  Results in fp32 are therefore summed over 2048 steps at a time
// and the sums added with rounding by the store engine, in order, as each is finished.  The parts of the rows that wgrad gives
// to different CTAs are added in a fixed order by a second kernel: no floating-point atomics between CTAs.
// Every mbarrier wait is bounded; on expiry the CTA sets *device_status and its roles leave their loops.
#include <algorithm>

#include "common.cuh"
#include "sm100.cuh"

namespace lite3r {

namespace {

using namespace sm100;

constexpr int kTileM = 256, kTileN = 256, kTileR = 64;  // of a pair; a tile may have half the columns
constexpr int kScaleTile = 512;
constexpr int kGroups = 4, kGroupThreads = 128;          // converting groups
constexpr int kThreads = 128 + kGroups * kGroupThreads + 128;
constexpr uint32_t kTmemCols = 512;

template <int kFormat>
struct Layout {
  // Stages of codes, one to a group: a group that waits for its next step's codes has read the stage's last ones itself.  (With a
  // stage more the stages pass from group to group, and a group could wait on a barrier whose phase before was still open,
  // which a parity test takes for done.)
  static constexpr int kRaw = kGroups;
  static constexpr int kOps = 5;                                // stages of operands
  static constexpr int kBoxBytes = kFormat == LITE3R_MXFP8 ? 64 : 32;  // of 64 columns of codes
  static constexpr uint32_t kOffB = 128 * kTileR * 2;           // A, then B as two boxes of 64 columns x 64 rows
  static constexpr uint32_t kOpBytes = kOffB + 128 * kTileR * 2;
  static constexpr uint32_t kOffRaw = kOps * kOpBytes;
  static constexpr uint32_t kOffScales = 2 * kTileR * kBoxBytes;  // of a raw stage: two boxes of codes, one scale tile
  static constexpr uint32_t kRawBytes = kOffScales + kScaleTile;
  static constexpr uint32_t kOffOut = (kOffRaw + kRaw * kRawBytes + 1023) / 1024 * 1024;  // 4 KB per epilogue warp
  static constexpr uint32_t kOffBar = kOffOut + 4 * 4096;
  static constexpr uint32_t kOffWords = kOffBar + 256;          // of the first CTA: 16 bytes of each converting warp of the second
  static constexpr uint32_t kSmemBytes = kOffWords + 256;
  static_assert(kSmemBytes <= 232448, "fits");
};

struct Bars {
  uint64_t raw_full[kGroups], raw_empty[kGroups], a_full[5], op_empty[5];
  uint64_t b_full[5];                   // of the first CTA: both CTAs' operands are there
  uint64_t acc_full[2], acc_empty[2];   // acc_empty: of the first CTA
  uint32_t tmem_base;
  int abort;
};
static_assert(sizeof(Bars) <= 256, "below the words");

struct BackParams {
  const uint8_t* scales;
  float* bias_parts;          // wgrad: [parts x groups][bias_cols][4 warps][m_total], or null
  int m_total, n_total;       // rows and columns of the result
  int scale_tiles;            // along n
  int steps, steps_per_part;  // of 64 along the contraction, in all and of one part of it
  int steps_per_sum;          // of one running sum in tensor memory
  int wide_tiles, half_tiles; // columns of a row of tiles: those of 256 first, then those of 128
  int bias_cols;              // column tiles that share the sums of dy
  int row_tiles, parts, units;
  int out_dtype;
  int* status;
};

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}

// Sixteen codes of a row to bf16 pairs.  A code's sign goes to bit 15, its exponent behind bf16's bias and its mantissa on top
// of seven bits: that is the value times 2^-kBias (denormals included), which the block's factor 2^(byte - 127 + kBias) undoes.
template <int kFormat>
struct Codes;
template <>
struct Codes<LITE3R_MXFP8> {
  static constexpr int kBias = 120, kBytes = 16;
  uint4 w;
  __device__ __forceinline__ void load(uint32_t at) { w = lds128(at); }
  static __device__ __forceinline__ uint32_t spread(uint32_t pair) { return ((pair >> 4) & 0x07F007F0u) | (pair & 0x80008000u); }
  __device__ __forceinline__ void pairs(int half, uint32_t out[4]) const {
    const uint32_t x = half == 0 ? w.x : w.z, y = half == 0 ? w.y : w.w;
    out[0] = spread(__byte_perm(x, 0u, 0x1404));
    out[1] = spread(__byte_perm(x, 0u, 0x3424));
    out[2] = spread(__byte_perm(y, 0u, 0x1404));
    out[3] = spread(__byte_perm(y, 0u, 0x3424));
  }
};
template <>
struct Codes<LITE3R_MXFP4> {
  static constexpr int kBias = 126, kBytes = 8;
  uint32_t w[2];
  __device__ __forceinline__ void load(uint32_t at) {
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
  }
  static __device__ __forceinline__ uint32_t spread(uint32_t pair) { return ((pair >> 6) & 0x01C001C0u) | (pair & 0x80008000u); }
  __device__ __forceinline__ void pairs(int half, uint32_t out[4]) const {
    const uint32_t odd = w[half], even = odd << 4;  // the even columns' codes in the bytes' upper halves, as the odd ones' are
    out[0] = spread(__byte_perm(even, odd, 0x4004));  // (what else is in these bytes the masks take away)
    out[1] = spread(__byte_perm(even, odd, 0x5111));
    out[2] = spread(__byte_perm(even, odd, 0x6222));
    out[3] = spread(__byte_perm(even, odd, 0x7333));
  }
};

// kFar: some factor of the warp's blocks is beyond bf16's largest power (or NaN) and is made of two.
template <int kBias, bool kFar>
__device__ __forceinline__ void scale_pairs(uint32_t v[4], uint32_t byte) {
  uint32_t f = (byte + kBias) << 7;
  if constexpr (kFar) {
    constexpr uint32_t kFirst = (static_cast<uint32_t>(kBias) + 127u) << 7;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = mul_bf16x2(v[i], kFirst | kFirst << 16);
    f = byte == 0xFFu ? 0x7FC0u : byte == 0u ? 0x0040u : byte << 7;
  }
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
  if ((smem_u32(smem) & 1023u) != 0) {  // the same in both CTAs of a pair
    if (threadIdx.x == 0 && p.status != nullptr) atomicCAS(p.status, 0, 900);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = static_cast<int>(cluster_rank());

  if (threadIdx.x == 0) {
    for (int s = 0; s < kRaw; ++s) {
      mbar_init(&bars->raw_full[s], 1);
      mbar_init(&bars->raw_empty[s], kGroupThreads / 32);
    }
    for (int s = 0; s < kOps; ++s) {
      mbar_init(&bars->a_full[s], 1);
      mbar_init(&bars->op_empty[s], 1);
      mbar_init(&bars->b_full[s], kGroupThreads / 32);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&bars->acc_full[b], 1);
      mbar_init(&bars->acc_empty[b], 8);
    }
    bars->abort = 0;
    mbar_fence_init();
  }
  if (warp == 1) {
    tmem_alloc_pair(&bars->tmem_base, kTmemCols);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  cluster_sync();  // barriers and tensor memory of both CTAs are there
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars->tmem_base;
  wait_for_prior_grid();
  launch_dependents();
  if (blockIdx.x == 0 && threadIdx.x == 0 && p.status != nullptr) *p.status = 0;

  // Units: the wide tiles of all parts, then the halves.
  const int wide_units = p.wide_tiles * p.row_tiles * p.parts;
  struct UnitAt {
    int m0, n0, part, first, last;  // this CTA's rows, the pair's columns, steps [first, last) of the contraction
    int col;                        // column tile
    bool half;
  };
  auto unit_at = [&](int unit) {
    UnitAt u;
    u.half = unit >= wide_units;
    if (u.half) unit -= wide_units;
    const int cols = u.half ? p.half_tiles : p.wide_tiles;
    const int per_part = cols * p.row_tiles;
    u.part = kWgrad ? unit / per_part : 0;
    const int tile = unit - u.part * per_part, row_tile = tile / cols, col = tile - row_tile * cols;
    u.m0 = row_tile * kTileM + rank * 128;
    u.col = u.half ? p.wide_tiles + col : col;
    u.n0 = u.half ? p.wide_tiles * kTileN + col * (kTileN / 2) : col * kTileN;
    u.first = u.part * p.steps_per_part;
    u.last = min(u.first + p.steps_per_part, p.steps);
    return u;
  };
  const int first_unit = blockIdx.x >> 1, unit_step = gridDim.x >> 1;

  // The loops of the loading and issuing warps run in all lanes and one of them issues: addresses and descriptors then stay in
  // uniform registers (in a loop of one lane a load took 200 cycles to issue, and 40 idle cycles lay between two products of 128).
  if (warp == 0) {
    const bool issuer = elect_one();
    if (issuer) tma_prefetch_desc(&map_codes);
    bool ok = true;
    int kc = 0, st = 0;
    uint32_t parity = 1;  // of the stage's use before, from the second round on
    for (int unit = first_unit; ok && unit < p.units; unit += unit_step) {
      const UnitAt u = unit_at(unit);
      const int n = u.n0 + rank * (u.half ? 64 : 128);  // this CTA's columns; n / 128 is a scale tile (cut_tiles makes no tile past them)
      const uint32_t bytes = (u.half ? 1 : 2) * kTileR * L::kBoxBytes + kScaleTile;
      const int x = kFormat == LITE3R_MXFP8 ? n : n / 2;
      for (int k = u.first; ok && k < u.last; ++k, ++kc) {
        if (kc >= kRaw) ok = mbar_wait_clearing(&bars->raw_empty[st], parity, abort_flag, p.status, 811);
        ok = __all_sync(0xFFFFFFFFu, ok);  // no lane falls behind by a phase
        if (!ok) break;
        if (issuer) {
          uint8_t* const dst = smem + L::kOffRaw + st * L::kRawBytes;
          mbar_arrive_expect_tx(&bars->raw_full[st], bytes);
          tma_load_2d(dst, &map_codes, &bars->raw_full[st], x, k * kTileR);
          if (!u.half) tma_load_2d(dst + kTileR * L::kBoxBytes, &map_codes, &bars->raw_full[st], x + L::kBoxBytes, k * kTileR);
          bulk_load(dst + L::kOffScales, p.scales + (static_cast<size_t>(k / 2) * p.scale_tiles + n / 128) * kScaleTile, kScaleTile,
                    &bars->raw_full[st]);
        }
        if (++st == kRaw) {
          st = 0;
          parity ^= 1u;
        }
      }
    }
  } else if (warp == 2) {
    const bool issuer = elect_one();
    if (issuer) tma_prefetch_desc(&map_dy);
    bool ok = true;
    int kc = 0, st = 0;
    uint32_t parity = 1;
    for (int unit = first_unit; ok && unit < p.units; unit += unit_step) {
      const UnitAt u = unit_at(unit);
      for (int k = u.first; ok && k < u.last; ++k, ++kc) {
        if (kc >= kOps) ok = mbar_wait_clearing(&bars->op_empty[st], parity, abort_flag, p.status, 812);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        if (issuer) {
          uint8_t* const dst = smem + st * L::kOpBytes;
          mbar_arrive_expect_tx(&bars->a_full[st], 128 * kTileR * 2);
          if constexpr (kWgrad) {  // two boxes of 64 columns x 64 rows of dy
            tma_load_2d(dst, &map_dy, &bars->a_full[st], u.m0, k * kTileR);
            tma_load_2d(dst + 8192, &map_dy, &bars->a_full[st], u.m0 + 64, k * kTileR);
          } else {
            tma_load_2d(dst, &map_dy, &bars->a_full[st], k * kTileR, u.m0);
          }
        }
        if (++st == kOps) {
          st = 0;
          parity ^= 1u;
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      const bool issuer = elect_one();
      constexpr uint32_t idesc_wide = instr_desc(1, kTileM, kTileN, kWgrad ? 1 : 0, 1);
      constexpr uint32_t idesc_half = instr_desc(1, kTileM, kTileN / 2, kWgrad ? 1 : 0, 1);
      const uint64_t a_desc0 = kWgrad ? smem_desc(smem_u32(smem), 8192, 1024, kSwizzle128) : smem_desc(smem_u32(smem), 16, 1024, kSwizzle128);
      const uint64_t b_desc0 = smem_desc(smem_u32(smem) + L::kOffB, 8192, 1024, kSwizzle128);
      bool ok = true;
      int st = 0, it = 0;
      uint32_t parity = 0;
      for (int unit = first_unit; ok && unit < p.units; unit += unit_step) {
        const UnitAt u = unit_at(unit);
        const uint32_t idesc = u.half ? idesc_half : idesc_wide;
        for (int k0 = u.first; ok && k0 < u.last; k0 += p.steps_per_sum, ++it) {
          const int ab = it & 1, k1 = min(k0 + p.steps_per_sum, u.last);
          if (it >= 2) ok = mbar_wait_cluster_clearing<true>(&bars->acc_empty[ab], ((it - 2) >> 1) & 1, abort_flag, p.status, 814);
          ok = __all_sync(0xFFFFFFFFu, ok);
          tc_fence_after();
          for (int k = k0; ok && k < k1; ++k) {
            ok = mbar_wait_cluster_clearing(&bars->b_full[st], parity, abort_flag, p.status, 816);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            tc_fence_after();
            if (issuer) {
              const uint64_t off = static_cast<uint64_t>((st * L::kOpBytes) >> 4);
#pragma unroll
              for (int kk = 0; kk < 4; ++kk)  // 16 steps of the contraction each
                mma_f16_pair(tmem + ab * kTileN, a_desc0 + off + kk * ((kWgrad ? 2048 : 32) >> 4), b_desc0 + off + kk * (2048 >> 4), idesc,
                             (k > k0 || kk > 0) ? 1u : 0u);
              mma_commit_pair(&bars->op_empty[st]);
            }
            if (++st == kOps) {
              st = 0;
              parity ^= 1u;
            }
          }
          if (ok && issuer) mma_commit_pair(&bars->acc_full[ab]);
        }
      }
    }
  } else if (warp >= 4 && warp < 4 + kGroups * 4) {
    // ------------------------------------------------------------------------------------------ codes to bf16
    const int group = (warp - 4) >> 2, t = threadIdx.x & (kGroupThreads - 1);
    const int row = t >> 2, chunk = t & 3;  // of 32 rows and four chunks of sixteen columns at a time
    const uint32_t my_raw = smem_u32(smem) + L::kOffRaw + row * L::kBoxBytes + chunk * Codes<kFormat>::kBytes;
    const uint32_t word = cluster_u32(smem + L::kOffWords + (warp - 4) * 16, 0);
    const uint32_t my_scales = smem_u32(smem) + L::kOffRaw + L::kOffScales + row * 16;
    const uint32_t my_b = smem_u32(smem) + L::kOffB + row * 128 + (((2 * chunk) ^ (row & 7)) << 4);  // and the next chunk's 16 bytes: ^ 16
    bool ok = true;
    int kc = 0;
    for (int unit = first_unit; ok && unit < p.units; unit += unit_step) {
      const UnitAt u = unit_at(unit);
      const int shift = 8 * ((u.half ? 2 * rank : 0) + (chunk >> 1));  // of the scale tile's four blocks, for the first box
      const bool sums = kWgrad && p.bias_parts != nullptr && u.col < p.bias_cols && u.m0 < p.m_total;
      float acc[4] = {};  // columns 2 lane, 2 lane + 1 of the two boxes of dy, over this warp's rows
      const int steps = u.last - u.first;
      const int mine = (group - kc % kGroups + kGroups) % kGroups;  // the first step of the unit that is this group's
      for (int i = mine; ok && i < steps; i += kGroups) {
        const int at = kc + i, k = u.first + i;
        const int rs = group, st = at % kOps;
        ok = mbar_wait_clearing(&bars->raw_full[rs], (at / kRaw) & 1, abort_flag, p.status, 817);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        const uint32_t raw = my_raw + rs * L::kRawBytes, dst = my_b + st * L::kOpBytes;
        Codes<kFormat> c[4];  // [box][32 rows]
        uint32_t byte[4], top = 0;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t word;  // of row (k & 1) * 64 + row + 32 q of the scale tile
          asm volatile("ld.shared.u32 %0, [%1];" : "=r"(word) : "r"(my_scales + rs * L::kRawBytes + ((k & 1) * 2 + q) * 4) : "memory");
          byte[q] = (word >> shift) & 0xFFu;
          byte[2 + q] = u.half ? byte[q] : (word >> (shift + 16)) & 0xFFu;
          top = max(top, max(byte[q], byte[2 + q]));
          c[q].load(raw + q * (32 * L::kBoxBytes));
          if (!u.half) c[2 + q].load(raw + (kTileR + 32 * q) * L::kBoxBytes);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->raw_empty[rs]);  // codes and scales are in registers
        if (at >= kOps) ok = mbar_wait_clearing(&bars->op_empty[st], ((at - kOps) / kOps) & 1, abort_flag, p.status, 818);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        auto convert = [&](auto far) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if (q >= 2 && u.half) break;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint32_t v[4];
              c[q].pairs(h, v);
              scale_pairs<Codes<kFormat>::kBias, decltype(far)::value>(v, byte[q]);
              sts128((dst ^ (h << 4)) + (q >> 1) * 8192 + (q & 1) * 4096, v[0], v[1], v[2], v[3]);
            }
          }
        };
        if (__any_sync(0xFFFFFFFFu, top + Codes<kFormat>::kBias > 254u)) convert(std::true_type());
        else convert(std::false_type());
        fence_proxy_async_smem();
        ok = mbar_wait_clearing(&bars->a_full[st], (at / kOps) & 1, abort_flag, p.status, 815);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        if (sums && k % p.bias_cols == u.col) {
          const uint8_t* const dy = smem + st * L::kOpBytes;
#pragma unroll
          for (int q = 0; q < 16; ++q) {
            const int r = (t >> 5) * 16 + q;
            const int off = r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              const uint32_t w = *reinterpret_cast<const uint32_t*>(dy + b * 8192 + off);
              acc[2 * b] += __uint_as_float(w << 16);
              acc[2 * b + 1] += __uint_as_float(w & 0xFFFF0000u);
            }
          }
        }
        __syncwarp();
        if (lane == 0) {  // each warp of the first CTA expects the word of one of the second: 16 bytes of what it has converted
          if (rank == 0) mbar_arrive_expect_tx(&bars->b_full[st], 16);
          else bulk_copy_cluster(word, dst, 16, cluster_u32(&bars->b_full[st], 0));
        }
      }
      kc += steps;
      if (sums && ok && mine < steps) {
        float* const dst = p.bias_parts + (static_cast<size_t>((u.part * kGroups + mine) * p.bias_cols + u.col) * 4 + (t >> 5)) * p.m_total;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int m = u.m0 + (e >> 1) * 64 + 2 * lane + (e & 1);
          if (m < p.m_total) dst[m] = acc[e];
        }
      }
    }
  } else if (warp >= 4 + kGroups * 4) {
    // ------------------------------------------------------------------------------------------ epilogue
    const int quarter = warp & 3;
    uint8_t* const warp_tile = smem + L::kOffOut + quarter * 4096;
    const uint32_t my_row = smem_u32(warp_tile) + lane * 128;
    const int swz = lane & 7;
    const bool wide = kWgrad || p.out_dtype == LITE3R_F32;
    bool ok = true;
    int it = 0;
    for (int unit = first_unit; ok && unit < p.units; unit += unit_step) {
      const UnitAt u = unit_at(unit);
      // (nothing is stored of a CTA's rows or a tile's columns that are all past the end)
      const int cols = u.m0 + quarter * 32 < p.m_total ? min(u.half ? kTileN / 2 : kTileN, p.n_total - u.n0) : 0;
      for (int k0 = u.first; ok && k0 < u.last; k0 += p.steps_per_sum, ++it) {
        const int ab = it & 1;
        const bool add = k0 > u.first;  // to the sum before, which this warp has stored
        const uint32_t acc_addr = tmem + ((static_cast<uint32_t>(quarter) * 32u) << 16) + ab * kTileN;
        ok = mbar_wait_clearing(&bars->acc_full[ab], (it >> 1) & 1, abort_flag, p.status, 813, 0, sum_limit_ns(p.steps_per_sum));
        tc_fence_after();
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        if (add && lane == 0) bulk_wait_group0();  // it is in place
#pragma unroll 1
        for (int cb = 0; cb < cols; cb += 32) {  // a multiple of 32
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
              const int x = u.n0 + (wide ? cb : cb & ~63), y = u.m0 + quarter * 32;
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
        if (lane == 0) mbar_arrive_cluster_read(cluster_u32(&bars->acc_empty[ab], 0));
      }
    }
    bulk_wait_group_read0();  // what is staged stays in place until it has been read
  }

  tc_fence_before();
  __syncthreads();
  linger_after_abort(abort_flag);
  cluster_sync();  // neither CTA leaves while the other one's products or arrivals may reach it
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, kTmemCols);
  }
}

// ------------------------------------------------------------------------------------------------ sums
struct Sums {
  const float* parts;  // [count][values]
  float* out;
  size_t values;
  int count;
};

// out[i] = sum over the parts in a fixed order: dw four values to a thread (blocks below dw_blocks), then db.
__global__ void __launch_bounds__(256) add_parts_kernel(const Sums dw, int dw_blocks, const Sums db) {
  __shared__ float s_sum[8][8];
  wait_for_prior_grid();
  launch_dependents();
  if (static_cast<int>(blockIdx.x) < dw_blocks) {
    const size_t i = (static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
    if (i >= dw.values) return;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int s = 0; s < dw.count; ++s) {
      const float4 v = *reinterpret_cast<const float4*>(dw.parts + static_cast<size_t>(s) * dw.values + i);
      acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
    }
    *reinterpret_cast<float4*>(dw.out + i) = acc;
    return;
  }
  // eight columns, 32 threads to each with every 32nd part, eight requested at a time
  const int col = threadIdx.x & 7, group = threadIdx.x >> 3;
  const size_t i = static_cast<size_t>(blockIdx.x - dw_blocks) * 8 + col;
  float acc = 0.f;
  if (i < db.values) {
#pragma unroll 8
    for (int s = group; s < db.count; s += 32) acc += db.parts[static_cast<size_t>(s) * db.values + i];
  }
#pragma unroll
  for (int o = 16; o >= 8; o >>= 1) acc += __shfl_xor_sync(0xFFFFFFFFu, acc, o);
  if ((threadIdx.x & 31) < 8) s_sum[threadIdx.x >> 5][col] = acc;
  __syncthreads();
  if (threadIdx.x < 8 && i < db.values) {
    acc = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) acc += s_sum[w][col];
    db.out[i] = acc;
  }
}

constexpr int kBiasCols = 4;

// How the tiles are cut.  Columns: all of 256, or the last 256 in two halves, which run last and fill the gaps that whole tiles
// leave, or halves throughout (few tiles).  A step of a half tile takes three quarters of a whole one's time (0.34 and 0.45 us:
// its conversion chain and its loads of A are as long).  dgrad of 10992 rows, 1024 x 1024: 22.4 us with 129 whole tiles and 86
// halves, 24.3 with 172 whole ones, 31.1 with halves; 777 rows: 11.7 with whole tiles, 9.4 with halves.
struct Cut {
  int wide, half, row_tiles, parts;
};
// Time in quarters of a whole tile's: a pair takes units p, p + pairs, ..., whole tiles first, so pair 0 has most of both.
long long most_columns(const Cut& c, int pairs) {
  const long long wide = static_cast<long long>(c.wide) * c.row_tiles * c.parts, all = wide + static_cast<long long>(c.half) * c.row_tiles * c.parts;
  const long long whole = (wide + pairs - 1) / pairs, rounds = (all + pairs - 1) / pairs;
  return 4 * whole + 3 * (rounds - whole);
}
Cut cut_tiles(int m_total, int n_total, int parts, int pairs) {
  const int n = ceil_div(n_total, kTileN / 2), rows = ceil_div(m_total, kTileM);  // halves per row of tiles
  Cut best = {n / 2, n % 2, rows, parts};
  long long least = most_columns(best, pairs);
  for (int half : {n % 2 + 2, n}) {
    if (half > n) continue;
    const Cut c = {(n - half) / 2, half, rows, parts};
    const long long time = most_columns(c, pairs);
    if (time < least) {
      best = c;
      least = time;
    }
  }
  return best;
}

// Parts of the contraction of wgrad: the number with the least time, of the products (0.113 us for a quarter of a whole tile's
// step; four steps to fill and drain the pipeline) and of the partial results (1.5 us for the kernel that adds them; they are
// written and read at about 10 TB/s, mostly in L2).  10992 rows, 1024 x 1024: 60 us in one part, 36 in two, 28 in four.
int wgrad_parts(int rows, int d_in, int d_out, int pairs) {
  const int steps = ceil_div(rows, kTileR);
  const double megabytes = static_cast<double>(d_in) * d_out * 4e-6;
  int best = 1;
  double least = 1e300;
  for (int parts = 1; parts <= std::max(1, std::min(16, steps / 8)); ++parts) {
    const int per_part = ceil_div(steps, parts);
    if (ceil_div(steps, per_part) != parts) continue;  // none is empty
    const double time = 0.113 * static_cast<double>(most_columns(cut_tiles(d_out, d_in, parts, pairs), pairs)) * (per_part + 4) +
                        (parts > 1 ? 1.5 + 0.1 * megabytes * (2 * parts + 1) : 0.0);
    if (time < least) {
      best = parts;
      least = time;
    }
  }
  return best;
}

// Numbers of pairs (of devices with 132 to 160 SMs) for whose rule the workspace has room.
constexpr int kSizedPairs[] = {66, 70, 72, 74, 76, 80};

int most_parts(int rows, int d_in, int d_out) {
  int parts = 1;
  for (int pairs : kSizedPairs) parts = std::max(parts, wgrad_parts(rows, d_in, d_out, pairs));
  return parts;
}

// The rule's parts, on any other device at most those that the workspace has room for.
int parts_of_device(int rows, int d_in, int d_out, int pairs) {
  const int parts = wgrad_parts(rows, d_in, d_out, pairs);
  for (int sized : kSizedPairs)
    if (sized == pairs) return parts;
  return std::min(parts, most_parts(rows, d_in, d_out));
}

size_t parts_bytes(int parts, int d_in, int d_out) {
  return ((parts > 1 ? static_cast<size_t>(parts) * d_in * d_out : 0) + static_cast<size_t>(parts) * kGroups * kBiasCols * 4 * d_out) * sizeof(float);
}

int pairs_of(int sms) { return std::max(1, sms / 2); }

template <int kFormat, bool kWgrad>
lite3r_status launch_back(const void* dy, long long dy_stride, const uint8_t* codes, const uint8_t* scales, int rows, int d_in,
                          int d_out, const CUtensorMap& map_out, int out_dtype, int parts, float* bias_parts, int* status, int pairs,
                          cudaStream_t stream) {
  using L = Layout<kFormat>;
  CUtensorMap map_dy, map_codes;
  lite3r_status st;
  if ((st = make_tensor_map_2d(&map_dy, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, dy, d_out, rows, 64, kWgrad ? 64 : 128,
                               CU_TENSOR_MAP_SWIZZLE_128B, static_cast<uint64_t>(dy_stride) * 2)) != LITE3R_OK) return st;
  const int code_rows = kWgrad ? rows : d_out;
  if ((st = make_tensor_map_2d(&map_codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, codes, kFormat == LITE3R_MXFP8 ? d_in : d_in / 2, code_rows,
                               L::kBoxBytes, kTileR, CU_TENSOR_MAP_SWIZZLE_NONE)) != LITE3R_OK) return st;
  auto* kernel = mx_back_kernel<kFormat, kWgrad>;
  if ((st = ensure_dynamic_smem(kernel, static_cast<int>(L::kSmemBytes))) != LITE3R_OK) return st;
  BackParams p = {};
  p.scales = scales;
  p.bias_parts = bias_parts;
  p.m_total = kWgrad ? d_out : rows;
  p.n_total = d_in;
  p.scale_tiles = ceil_div(d_in, 128);
  p.steps = ceil_div(code_rows, kTileR);
  p.steps_per_part = ceil_div(p.steps, parts);
  p.steps_per_sum = out_dtype == LITE3R_F32 ? 2048 / kTileR : p.steps;
  const Cut c = cut_tiles(p.m_total, d_in, parts, pairs);
  p.wide_tiles = c.wide;
  p.half_tiles = c.half;
  p.bias_cols = std::min(kBiasCols, c.wide + c.half);
  p.row_tiles = c.row_tiles;
  p.parts = parts;
  const long long units = static_cast<long long>(c.wide + c.half) * c.row_tiles * parts;
  if (units > 0x7FFFFFFFLL - 1024) return LITE3R_ERR_UNSUPPORTED;
  p.units = static_cast<int>(units);
  p.out_dtype = out_dtype;
  p.status = status;
  return launch_dependent_cluster(kernel, dim3(static_cast<unsigned>(2 * std::min(p.units, pairs))), kThreads,
                                  static_cast<int>(L::kSmemBytes), 2, stream, map_dy, map_codes, map_out, p);
}

lite3r_status pairs_of_device(int* pairs) {
  int sms = 0;
  const lite3r_status st = sm_count(&sms);
  *pairs = pairs_of(sms);
  return st;
}

}  // namespace

size_t linear_mx_workspace_bytes(int rows, int d_in, int d_out) {
  return parts_bytes(most_parts(rows, d_in, d_out), d_in, d_out) + 256;
}

void linear_mx_parts(int rows, int d_in, int d_out, int sms, int* parts, size_t* bytes) {
  *parts = parts_of_device(rows, d_in, d_out, pairs_of(sms));
  *bytes = parts_bytes(*parts, d_in, d_out);
}

lite3r_status launch_mx_dgrad(const void* dy, long long dy_stride, const uint8_t* w_codes, const uint8_t* w_scales, int format,
                              int rows, int d_in, int d_out, void* dx, int dx_dtype, long long dx_stride, int* device_status,
                              cudaStream_t stream) {
  int pairs = 0;
  lite3r_status st = pairs_of_device(&pairs);
  if (st != LITE3R_OK) return st;
  const int elem = dx_dtype == LITE3R_F32 ? 4 : 2;
  CUtensorMap map;
  st = make_tensor_map_2d(&map,
                          dx_dtype == LITE3R_F32    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                          : dx_dtype == LITE3R_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                    : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                          elem, dx, d_in, rows, 128 / elem, 32, CU_TENSOR_MAP_SWIZZLE_128B, static_cast<uint64_t>(dx_stride) * elem);
  if (st != LITE3R_OK) return st;
  auto* launch = format == LITE3R_MXFP8 ? launch_back<LITE3R_MXFP8, false> : launch_back<LITE3R_MXFP4, false>;
  return launch(dy, dy_stride, w_codes, w_scales, rows, d_in, d_out, map, dx_dtype, 1, nullptr, device_status, pairs, stream);
}

lite3r_status launch_mx_wgrad(const void* dy, long long dy_stride, const uint8_t* x_codes, const uint8_t* x_scales, int format,
                              int rows, int d_in, int d_out, float* dw, float* db, float* workspace, size_t workspace_bytes,
                              int* device_status, cudaStream_t stream) {
  int pairs = 0;
  lite3r_status st = pairs_of_device(&pairs);
  if (st != LITE3R_OK) return st;
  const int parts = parts_of_device(rows, d_in, d_out, pairs);
  const size_t values = static_cast<size_t>(d_in) * d_out;
  if (parts_bytes(parts, d_in, d_out) > workspace_bytes) return LITE3R_ERR_WORKSPACE;
  float* const products = parts > 1 ? workspace : dw;
  float* const bias_parts = workspace + (parts > 1 ? parts * values : 0);
  CUtensorMap map;
  if ((st = make_tensor_map_3d(&map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, products, d_in, d_out, parts, 32, 32, CU_TENSOR_MAP_SWIZZLE_128B)) != LITE3R_OK)
    return st;
  auto* launch = format == LITE3R_MXFP8 ? launch_back<LITE3R_MXFP8, true> : launch_back<LITE3R_MXFP4, true>;
  st = launch(dy, dy_stride, x_codes, x_scales, rows, d_in, d_out, map, LITE3R_F32, parts, db != nullptr ? bias_parts : nullptr, device_status,
              pairs, stream);
  if (st != LITE3R_OK || (parts == 1 && db == nullptr)) return st;
  // a part of fewer than four steps (the last, or the only one) has no sums of the groups without a step
  const int steps = ceil_div(rows, kTileR), last = steps - (parts - 1) * ceil_div(steps, parts);
  const Cut c = cut_tiles(d_out, d_in, parts, pairs);
  const int bias_count = ((parts - 1) * kGroups + std::min(kGroups, last)) * std::min(kBiasCols, c.wide + c.half) * 4;
  const Sums dw_sums = {products, dw, values, parts}, db_sums = {bias_parts, db, static_cast<size_t>(d_out), bias_count};
  const long long dw_blocks = parts > 1 ? static_cast<long long>((values / 4 + 255) / 256) : 0, db_blocks = db != nullptr ? ceil_div(d_out, 8) : 0;
  if (dw_blocks + db_blocks > 0x7FFFFFFFLL) return LITE3R_ERR_UNSUPPORTED;
  return launch_dependent(add_parts_kernel, dim3(static_cast<unsigned>(dw_blocks + db_blocks)), 256, 0, stream, dw_sums,
                          static_cast<int>(dw_blocks), db_sums);
}

}  // namespace lite3r
