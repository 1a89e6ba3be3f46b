// The linear layer on microscaled 4-bit operands: y = Q(x) Q(W)^T + b with block-scaled tcgen05 products (e2m1 x e2m1, one
// scale per 32 elements of K, fp32 accumulation in TMEM).
// A product of two e2m1 values is a multiple of 1/4 of at most 36 (8 bits) and the scales are powers of two, so a sum of K of them
// in fp32 is exact while the scales' spread along it (of both operands together) is below 2^(24 - 8 - log2 K): 2^4 for 4096
// elements.  Beyond that the running sum is cut off, not rounded: low by 0.07 to 0.11 x 2^-24 of the result for every product of
// 64 elements where all terms are positive and the blocks' scales lie within 2^6 (4096 elements: 4e-7).  One sum over all of d_in.
// Persistent CTAs over tiles of 128 rows x 64 or 128 columns, or pairs of CTAs (cta_group::2, half of A's and of B's rows
// each) over tiles of 256 x 256.  Warp 0 loads A and B as bytes (rows of 128 = 256 elements of K, 128B swizzle), warp 2 the scale
// tiles of both as they lie in memory, warp 1 copies the scales to tensor memory and issues the products into one of two
// accumulators, warps 4 on are epilogue warpgroups, one per 64 columns, which add the bias, round once and store through
// shared memory.  The products of the next tile run under the epilogue of this one.
// Tensor memory: two accumulators of 256 columns leave no room for the scales, so they share 32 columns: the warpgroup that
// has these reads them first, and the next tile's products wait for that (a few hundred cycles) and not for the epilogue.
// 43968 x 4096 x 1024 in 69 to 76 us (the first at 1.97 GHz: 5.3 PFLOP/s), the tensor pipe busy for 70 % of it, and 88 us in a run of
// a second, where the power limit leaves 1.43 GHz (by single CTAs on 128 x 128: 162 us).  A stage of 256 elements of K takes 720
// cycles: 560 of products and 100 of scale copies, which run in order with them, and at the end of a tile the wait for the shared
// columns.  10992 x 1024 x 4096 in 26 to 28 us.
// Every mbarrier wait is bounded; on expiry the CTA sets *device_status and its roles leave their loops.
#include <algorithm>

#include "common.cuh"
#include "sm100.cuh"

namespace lite3r {

namespace {

using namespace sm100;

constexpr int kTileM = 128;
constexpr int kRowBytes = 128;            // of an operand row in a stage
constexpr int kStageK = 2 * kRowBytes;    // elements of K in a stage
constexpr int kScaleTile = 512;           // scales of 128 rows x 128 elements of K
constexpr int kMaxStages = 5;

template <int kN>
struct Layout {
  static constexpr bool kPair = kN == 256;
  static constexpr int kCtas = kPair ? 2 : 1;
  static constexpr int kGroups = kN / 64;                      // epilogue warpgroups
  static constexpr int kThreads = 128 + 128 * kGroups;
  static constexpr int kStages = 5;
  static constexpr int kLoadN = kN / kCtas;                    // rows of B that this CTA loads
  static constexpr int kTilesB = (kN + 127) / 128;             // scale tiles of B per 128 elements of K: of all columns in both CTAs
  static constexpr uint32_t kOffB = kTileM * kRowBytes;
  static constexpr uint32_t kOffSfa = kOffB + kLoadN * kRowBytes;  // two scale tiles of A, two for each 128 columns of B
  static constexpr uint32_t kOffSfb = kOffSfa + 2 * kScaleTile;
  static constexpr uint32_t kScaleBytes = (2 + 2 * kTilesB) * kScaleTile;
  static constexpr uint32_t kStageBytes = kOffSfa + kScaleBytes;
  static constexpr uint32_t kOffOut = kStages * kStageBytes;   // staged output, 2 KB per epilogue warp
  static constexpr uint32_t kOffBias = kOffOut + kGroups * 8192;  // two sets by turns
  static constexpr uint32_t kOffBar = kOffBias + 2 * kN * 4;
  static constexpr uint32_t kSmemBytes = kOffBar + 256;
  // tensor memory: two accumulators, then the scales of a stage: four columns per scale tile
  static constexpr uint32_t kShared = kPair ? 32 : 0;          // columns that the accumulators share
  static constexpr uint32_t kAcc1 = kN - kShared;
  static constexpr uint32_t kSfaCol = kAcc1 + kN, kSfbCol = kSfaCol + 8;
  static constexpr uint32_t kTmemCols = kN == 64 ? 256 : 512;
  static_assert(kSfbCol + 8 * kTilesB <= kTmemCols && kStageBytes % 1024 == 0 && kSmemBytes <= 232448, "fits");
};

struct Bars {
  uint64_t full[kMaxStages], empty[kMaxStages];
  uint64_t acc_full[2], acc_empty[2];  // accumulator written (issuer -> epilogue) / read out (epilogue -> issuer)
  uint64_t shared_read;                // the columns that both accumulators have are read out of this tile's
  uint32_t tmem_base;
  int abort;
};

struct MxParams {
  const float* bias;  // [d_out] or null
  int rows, d_in, d_out;
  int k_tiles;        // scale tiles along K
  int col_tiles, tiles;
  int y_dtype;
  int ragged;         // rows of y end inside 16 bytes
  void* y;
  long long y_stride;
  int* status;
};

__device__ __forceinline__ void named_barrier_sync(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

template <int kN>
__global__ void __launch_bounds__(Layout<kN>::kThreads, 1)
linear_mxf4_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                   const __grid_constant__ CUtensorMap map_xs, const __grid_constant__ CUtensorMap map_ws,
                   const __grid_constant__ CUtensorMap map_y, const MxParams p) {
  using L = Layout<kN>;
  constexpr int kStages = L::kStages, kCtas = L::kCtas;
  constexpr bool kPair = L::kPair;
  extern __shared__ __align__(1024) uint8_t smem[];
  Bars* bars = reinterpret_cast<Bars*>(smem + L::kOffBar);
  volatile int* abort_flag = &bars->abort;
  if ((smem_u32(smem) & 1023u) != 0) {  // the same in both CTAs of a pair
    if (threadIdx.x == 0 && p.status != nullptr) atomicCAS(p.status, 0, 900);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int stages_k = (p.d_in + kStageK - 1) / kStageK;
  const int rank = kPair ? static_cast<int>(cluster_rank()) : 0;
  const int first_tile = blockIdx.x / kCtas, tile_step = gridDim.x / kCtas;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&bars->full[s], 2);  // operands, scales
      mbar_init(&bars->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&bars->acc_full[b], 1);
      mbar_init(&bars->acc_empty[b], kCtas * L::kGroups * 4);
    }
    mbar_init(&bars->shared_read, kCtas * 4);
    bars->abort = 0;
    mbar_fence_init();
  }
  if (warp == 1) {
    if constexpr (kPair) {
      tmem_alloc_pair(&bars->tmem_base, L::kTmemCols);
      tmem_relinquish_pair();
    } else {
      tmem_alloc(&bars->tmem_base, L::kTmemCols);
      tmem_relinquish();
    }
  }
  tc_fence_before();
  if constexpr (kPair) cluster_sync();  // barriers and tensor memory of both CTAs are there
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars->tmem_base;
  wait_for_prior_grid();
  launch_dependents();
  if (blockIdx.x == 0 && threadIdx.x == 0 && p.status != nullptr) *p.status = 0;

  // The loops of the loading and issuing warps run in all lanes and one of them issues: addresses and descriptors then stay in
  // uniform registers (in a loop of one lane a load took 200 cycles to issue, and 40 idle cycles lay between two products of 128).
  if (warp == 0 || warp == 2) {
    const bool operands = warp == 0, issuer = elect_one();
    if (issuer) {
      tma_prefetch_desc(operands ? &map_x : &map_xs);
      tma_prefetch_desc(operands ? &map_w : &map_ws);
    }
    constexpr uint32_t kOperandBytes = L::kOffSfa;
    const uint32_t full0 = kPair ? cluster_u32(&bars->full[0], 0) : 0u;  // both CTAs' loads count on the first one's barrier
    bool ok = true;
    int kc = 0, st = 0;
    uint32_t parity = 1;  // of the stage's use before, from the second round on
    for (int tile = first_tile; ok && tile < p.tiles; tile += tile_step) {
      const int row_tile = tile / p.col_tiles, col0 = (tile - row_tile * p.col_tiles) * kN;
      const int row0 = (row_tile * kCtas + rank) * kTileM;
      for (int k = 0; ok && k < stages_k; ++k, ++kc) {
        if (kc >= kStages) ok = mbar_wait_clearing(&bars->empty[st], parity, abort_flag, p.status, 801);
        ok = __all_sync(0xFFFFFFFFu, ok);  // no lane falls behind by a phase
        if (!ok) break;
        if (issuer) {
          uint8_t* const dst = smem + st * L::kStageBytes;
          if (rank == 0) mbar_arrive_expect_tx(&bars->full[st], kCtas * (operands ? kOperandBytes : L::kScaleBytes));
          auto load = [&](uint32_t off, const CUtensorMap* map, int x, int y) {
            if constexpr (kPair) tma_load_2d_pair(dst + off, map, full0 + st * 8, x, y);
            else tma_load_2d(dst + off, map, &bars->full[st], x, y);
          };
          if (operands) {
            load(0, &map_x, k * kRowBytes, row0);
            load(L::kOffB, &map_w, k * kRowBytes, col0 + rank * L::kLoadN);
          } else {  // two neighbouring scale tiles (the second unused at the end of an odd number of them)
            load(L::kOffSfa, &map_xs, 0, (row_tile * kCtas + rank) * p.k_tiles + 2 * k);
#pragma unroll
            for (int b = 0; b < L::kTilesB; ++b)
              load(L::kOffSfb + b * 2 * kScaleTile, &map_ws, 0, (col0 / 128 + b) * p.k_tiles + 2 * k);
          }
        }
        if (++st == kStages) {
          st = 0;
          parity ^= 1u;
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      const bool issuer = elect_one();
      constexpr uint32_t idesc0 = instr_desc_mxf4(kCtas * kTileM, kN, 0), idesc2 = instr_desc_mxf4(kCtas * kTileM, kN, 2);
      const uint64_t a_desc0 = smem_desc(smem_u32(smem), 16, 1024, kSwizzle128);
      const uint64_t b_desc0 = smem_desc(smem_u32(smem) + L::kOffB, 16, 1024, kSwizzle128);
      const uint64_t s_desc0 = smem_desc(smem_u32(smem) + L::kOffSfa, 16, 128, 0);
      const int products = (p.d_in + 63) / 64;
      bool ok = true;
      int st = 0, it = 0;
      uint32_t parity = 0;
      for (int tile = first_tile; ok && tile < p.tiles; tile += tile_step, ++it) {
        const int ab = it & 1;
        const uint32_t acc = tmem + (ab ? L::kAcc1 : 0u);
        // with tiles of 64 columns the weight's scale tile serves two of them: columns 0 and 1, or 2 and 3
        const uint32_t sfb_shift = kN == 64 ? 2u * ((tile % p.col_tiles) & 1) : 0u;
        auto wait_read = [&](uint64_t* bar, uint32_t phase, int code) {  // for the epilogues (of both CTAs)
          if constexpr (kPair) return mbar_wait_cluster_clearing<true>(bar, phase, abort_flag, p.status, code);
          else return mbar_wait_clearing(bar, phase, abort_flag, p.status, code);
        };
        if (it >= 2) ok = wait_read(&bars->acc_empty[ab], ((it - 2) >> 1) & 1, 804);
        if (L::kShared != 0 && ok && it >= 1) ok = wait_read(&bars->shared_read, (it - 1) & 1, 805);
        ok = __all_sync(0xFFFFFFFFu, ok);
        tc_fence_after();
        for (int k = 0; ok && k < stages_k; ++k) {
          ok = mbar_wait_clearing(&bars->full[st], parity, abort_flag, p.status, 802);
          ok = __all_sync(0xFFFFFFFFu, ok);
          if (!ok) break;
          tc_fence_after();
          const uint64_t off = static_cast<uint64_t>((st * L::kStageBytes) >> 4);
          const int todo = min(4, products - 4 * k);
          if (issuer) {
            auto copy = [&](uint32_t col, uint32_t smem_off) {
              if constexpr (kPair) tmem_copy_scales_pair(tmem + col, s_desc0 + off + (smem_off >> 4));
              else tmem_copy_scales(tmem + col, s_desc0 + off + (smem_off >> 4));
            };
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              if (2 * t >= todo) break;
              copy(L::kSfaCol + 4 * t, t * kScaleTile);
#pragma unroll
              for (int b = 0; b < L::kTilesB; ++b)
                copy(L::kSfbCol + 4 * (t * L::kTilesB + b), (2 + 2 * b + t) * kScaleTile);
            }
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
              if (kk >= todo) break;
              const uint64_t a_desc = a_desc0 + off + ((kk * 32) >> 4), b_desc = b_desc0 + off + ((kk * 32) >> 4);
              const uint32_t sfa = tmem + L::kSfaCol + 4 * (kk >> 1), sfb = tmem + L::kSfbCol + 4 * L::kTilesB * (kk >> 1) + sfb_shift;
              const uint32_t accumulate = (k > 0 || kk > 0) ? 1u : 0u;
              if constexpr (kPair) mma_mxf4_pair(acc, a_desc, b_desc, (kk & 1) ? idesc2 : idesc0, sfa, sfb, accumulate);
              else mma_mxf4(acc, a_desc, b_desc, (kk & 1) ? idesc2 : idesc0, sfa, sfb, accumulate);
            }
            if constexpr (kPair) mma_commit_pair(&bars->empty[st]);
            else mma_commit(&bars->empty[st]);
          }
          if (++st == kStages) {
            st = 0;
            parity ^= 1u;
          }
        }
        if (ok && issuer) {
          if constexpr (kPair) mma_commit_pair(&bars->acc_full[ab]);
          else mma_commit(&bars->acc_full[ab]);
        }
      }
    }
  } else if (warp >= 4) {
    const int quarter = warp & 3;
    const int hh = (warp - 4) >> 2;  // which 64 columns of the tile this warpgroup owns
    const int tid = threadIdx.x - (4 + hh * 4) * 32;
    uint8_t* const warp_tile = smem + L::kOffOut + hh * 8192 + quarter * 2048;
    const uint32_t my_row = smem_u32(warp_tile) + lane * 64;
    const int swz = (lane >> 1) & 3;
    const bool wide = p.y_dtype == LITE3R_F32;
    bool ok = true;
    int it = 0;
    for (int tile = first_tile; ok && tile < p.tiles; tile += tile_step, ++it) {
      const int ab = it & 1;
      const int row_tile = tile / p.col_tiles;
      const int row0 = (row_tile * kCtas + rank) * kTileM, col = (tile - row_tile * p.col_tiles) * kN + hh * 64;
      const uint32_t acc_addr = tmem + ((static_cast<uint32_t>(quarter) * 32u) << 16) + (ab ? L::kAcc1 : 0u) + hh * 64;
      float* const bia = reinterpret_cast<float*>(smem + L::kOffBias) + ab * kN + hh * 64;
      if (tid < 64) bia[tid] = (p.bias != nullptr && col + tid < p.d_out) ? __ldg(p.bias + col + tid) : 0.f;
      named_barrier_sync(1 + hh, 128);
      ok = mbar_wait_clearing(&bars->acc_full[ab], (it >> 1) & 1, abort_flag, p.status, 803, 0, sum_limit_ns(stages_k));
      tc_fence_after();
      ok = __all_sync(0xFFFFFFFFu, ok);
      if (!ok) break;
      auto read_out = [&](uint64_t* bar) {  // the issuer waits in the first CTA
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if constexpr (kPair) mbar_arrive_cluster_read(cluster_u32(bar, 0));
          else mbar_arrive(bar);
        }
      };
      // the shared columns are the first accumulator's last and the second one's first: this warpgroup reads them first
      const bool shares = L::kShared != 0 && hh == (ab ? 0 : L::kGroups - 1);
      if (col >= p.d_out) {
        if (shares) read_out(&bars->shared_read);
        read_out(&bars->acc_empty[ab]);
        continue;
      }
      // The warp stages its 32 rows, 64 bytes at a time (which leaves room for a fifth stage of operands), in the layout the
      // store engine reads (64B swizzle); rows and columns past the output are clipped by the engine, columns at 16 bytes: a
      // ragged end is stored value by value.
      const bool ragged = p.ragged && col + 64 > p.d_out;
      const int first_cb = shares && ab == 0 ? 32 : 0;
#pragma unroll 1
      for (int j = 0; j < 2; ++j) {
        const int cb = j == 0 ? first_cb : 32 - first_cb;
        uint32_t v[32];
        tmem_ld32(acc_addr + cb, v);
        tmem_wait_ld();
        if (shares && j == 0) read_out(&bars->shared_read);
        if (j == 1) read_out(&bars->acc_empty[ab]);
#pragma unroll
        for (int c = 0; c < 32; c += 4) {
          const float4 b4 = *reinterpret_cast<const float4*>(bia + cb + c);
          v[c] = __float_as_uint(__uint_as_float(v[c]) + b4.x);
          v[c + 1] = __float_as_uint(__uint_as_float(v[c + 1]) + b4.y);
          v[c + 2] = __float_as_uint(__uint_as_float(v[c + 2]) + b4.z);
          v[c + 3] = __float_as_uint(__uint_as_float(v[c + 3]) + b4.w);
        }
        if (ragged) {
          if (row0 + quarter * 32 + lane < p.rows) {
            uint8_t* const dst = static_cast<uint8_t*>(p.y) + ((row0 + quarter * 32 + lane) * p.y_stride + col + cb) * (wide ? 4 : 2);
#pragma unroll
            for (int c = 0; c < 32; ++c) {
              if (col + cb + c >= p.d_out) continue;
              const float f = __uint_as_float(v[c]);
              if (wide) reinterpret_cast<float*>(dst)[c] = f;
              else if (p.y_dtype == LITE3R_BF16) reinterpret_cast<__nv_bfloat16*>(dst)[c] = __float2bfloat16_rn(f);
              else reinterpret_cast<__half*>(dst)[c] = __float2half_rn(f);
            }
          }
          continue;
        }
        auto store = [&](int first, const uint32_t (&w)[16]) {  // 64 bytes of the row, from this column on
          if (lane == 0) bulk_wait_group_read0();  // what was staged here before has been read by the store engine
          __syncwarp();
#pragma unroll
          for (int c = 0; c < 4; ++c) sts128(my_row + ((c ^ swz) << 4), w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            if (col + first < p.d_out) tma_store_2d(&map_y, warp_tile, col + first, row0 + quarter * 32);
            bulk_commit_group();
          }
        };
        uint32_t w[16];
        if (wide) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int c = 0; c < 16; ++c) w[c] = v[16 * h + c];
            store(cb + 16 * h, w);
          }
        } else {
#pragma unroll
          for (int q = 0; q < 16; ++q) {
            const float y0 = __uint_as_float(v[2 * q]), y1 = __uint_as_float(v[2 * q + 1]);
            if (p.y_dtype == LITE3R_BF16) {
              __nv_bfloat162 h = __floats2bfloat162_rn(y0, y1);
              w[q] = *reinterpret_cast<uint32_t*>(&h);
            } else {
              __half2 h = __floats2half2_rn(y0, y1);
              w[q] = *reinterpret_cast<uint32_t*>(&h);
            }
          }
          store(cb, w);
        }
      }
    }
    bulk_wait_group_read0();  // what is staged stays in place until it has been read
  }

  tc_fence_before();
  __syncthreads();
  linger_after_abort(abort_flag);
  if constexpr (kPair) cluster_sync();  // neither CTA leaves while the other one's loads, products or arrivals may reach it
  if (warp == 1) {
    tc_fence_after();
    if constexpr (kPair) tmem_dealloc_pair(tmem, L::kTmemCols);
    else tmem_dealloc(tmem, L::kTmemCols);
  }
}

struct Operands {
  const uint8_t *x_codes, *x_scales, *w_codes, *w_scales;
};

// Scale tiles as rows of 128 words, two of them to a box.
lite3r_status scale_map(CUtensorMap* map, const uint8_t* scales, int rows, int k_tiles) {
  return make_tensor_map_2d(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 4, scales, 128, static_cast<uint64_t>(ceil_div(rows, 128)) * k_tiles, 128, 2,
                            CU_TENSOR_MAP_SWIZZLE_NONE);
}

template <int kN>
lite3r_status launch_tiles(const Operands& o, const CUtensorMap& map_y, const MxParams& p, int sms, cudaStream_t stream) {
  using L = Layout<kN>;
  CUtensorMap map_x, map_w, map_xs, map_ws;
  lite3r_status st;
  const uint64_t pitch = static_cast<uint64_t>(p.d_in) / 2;
  if ((st = make_tensor_map_2d(&map_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, o.x_codes, pitch, p.rows, kRowBytes, kTileM,
                               CU_TENSOR_MAP_SWIZZLE_128B)) != LITE3R_OK) return st;
  if ((st = make_tensor_map_2d(&map_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, o.w_codes, pitch, p.d_out, kRowBytes, L::kLoadN,
                               CU_TENSOR_MAP_SWIZZLE_128B)) != LITE3R_OK) return st;
  if ((st = scale_map(&map_xs, o.x_scales, p.rows, p.k_tiles)) != LITE3R_OK) return st;
  if ((st = scale_map(&map_ws, o.w_scales, p.d_out, p.k_tiles)) != LITE3R_OK) return st;
  if ((st = ensure_dynamic_smem(linear_mxf4_kernel<kN>, static_cast<int>(L::kSmemBytes))) != LITE3R_OK) return st;
  MxParams q = p;
  q.col_tiles = ceil_div(p.d_out, kN);
  const long long tiles = static_cast<long long>(q.col_tiles) * ceil_div(p.rows, L::kCtas * kTileM);
  // (coordinates of scale tiles and tile numbers are 32-bit)
  if (tiles > 0x7FFFFFFFLL - 1024 || static_cast<long long>(ceil_div(std::max(p.rows, p.d_out), 128) + 2) * p.k_tiles > 0x7FFFFFFFLL)
    return LITE3R_ERR_UNSUPPORTED;
  q.tiles = static_cast<int>(tiles);
  return launch_dependent_cluster(linear_mxf4_kernel<kN>, dim3(static_cast<unsigned>(L::kCtas * std::min(q.tiles, sms / L::kCtas))), L::kThreads,
                                  static_cast<int>(L::kSmemBytes), L::kCtas, stream, map_x, map_w, map_xs, map_ws, map_y, q);
}

}  // namespace

lite3r_status launch_linear_mxf4(const uint8_t* x_codes, const uint8_t* x_scales, const uint8_t* w_codes, const uint8_t* w_scales,
                                 const float* bias, int rows, int d_in, int d_out, void* y, int y_dtype, long long y_stride,
                                 int* device_status, cudaStream_t stream) {
  int sms = 0;
  lite3r_status st = sm_count(&sms);
  if (st != LITE3R_OK) return st;
  const Operands o = {x_codes, x_scales, w_codes, w_scales};
  MxParams p = {};
  p.bias = bias;
  p.rows = rows;
  p.d_in = d_in;
  p.d_out = d_out;
  p.k_tiles = ceil_div(d_in, 128);
  p.y_dtype = y_dtype;
  p.status = device_status;
  const int elem = y_dtype == LITE3R_F32 ? 4 : 2;
  p.ragged = (d_out * static_cast<long long>(elem)) % 16 != 0;
  p.y = y;
  p.y_stride = y_stride;
  CUtensorMap map_y;
  st = make_tensor_map_2d(&map_y,
                          y_dtype == LITE3R_F32    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                          : y_dtype == LITE3R_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                   : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                          elem, y, d_out, rows, 64 / elem, 32, CU_TENSOR_MAP_SWIZZLE_64B, static_cast<uint64_t>(y_stride) * elem);
  if (st != LITE3R_OK) return st;
  // Tiles of 64 columns while they are at most one to an SM, then of 128 until there are more tiles of 256 x 256 than pairs, or
  // half as many where the contraction is long.  us with tiles of 64 / 128 / 256 columns (rows x d_in x d_out):
  //   777 x 1024 x 1024  4.0 / 4.5 / 5.7    1374 x 4096 x 1024  10.3 / 7.5 / 9.3    2748 x 1024 x 1024   6.4 /  5.9 /  6.4
  //   2748 x 4096 x 1024  14.4 / 10.9 / 10.0    10992 x 1024 x 4096  48.1 / 31.6 / 26.2
  const long long row_tiles = ceil_div(rows, kTileM);
  const long long large = static_cast<long long>(ceil_div(d_out, 256)) * ceil_div(rows, 256);
  if (large * (d_in >= 2048 ? 2 : 1) > sms / 2) return launch_tiles<256>(o, map_y, p, sms, stream);
  return ceil_div(d_out, 64) * row_tiles <= sms ? launch_tiles<64>(o, map_y, p, sms, stream) : launch_tiles<128>(o, map_y, p, sms, stream);
}

}  // namespace lite3r
