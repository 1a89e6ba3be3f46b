// Norms of queries and keys for each head, with the position rotation in the same pass, and their gradient:
//   qk_norm_rope           z = norm(x) * w + b over the D values of a (batch, head, token) row, then the rotation of the pairs
//                          (i, i + S/2) of every axis section of S = D / axes values by position * base^(-2 i / S)
//   qk_norm_rope_backward  g = R^T dy;  dw = sum g xh, db = sum g over all rows;  gh = g w;
//                          dx = r (gh - mean(gh) - xh mean(gh xh))   (layer norm; no mean(gh) for the root mean square norm)
// Both are one pass over the tensors and bound by HBM.  D / 16 lanes work on a row, each on eight pairs: the eight values at i
// and the eight at i + S/2 (16-byte loads of 16-bit types), so that a rotation needs no other lane and the sums of a row of
// 64 values take two shuffles.  A group of lanes stays with one token and walks its heads
// while the next ones' loads are under way; sine, cosine, weight and bias meet in six coefficients per pair, made once per
// token.  Arithmetic on packed pairs of fp32.
// 32 frames of 1374 tokens, 16 heads of 64 bf16 queries and keys: 66 us, 5.5 TB/s (172 us with four pairs to a lane and scalar
// arithmetic, 159 instructions per 256 values); a hundred frames 184 us, 6.1 TB/s; the gradient of 32 frames 115 us, 4.7 TB/s.
// In fp32: 32 frames 136 us, 5.3 TB/s; the gradient of 16 frames 106 us, 5.1 TB/s.  (Single calls at full clocks; in a run of a
// second at the power limit 2 to 5 % longer.)
// Angles: position * base^(-2i/S) / 2 pi in 64-bit fixed point (an fp32 product of a position of a million is off by a tenth of
// a radian), whose overflow leaves the fraction of a turn; that in fp32.  Sums and norms are fp32; results are rounded once.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.cuh"
#include "sm100.cuh"

namespace lite3r {

namespace {

using namespace sm100;

constexpr int kRopeThreads = 128;
constexpr int kMaxRopeDim = 256;
constexpr int kRopeCtas = 4;  // CTAs per SM (128 registers per thread)
constexpr int back_ctas(size_t value_bytes) { return value_bytes == 4 ? 3 : 4; }  // rows of fp32 on their way need the registers
constexpr int kMaxRopePartials = 1024;  // CTAs of the backward pass per tensor; each leaves one partial sum of dw and db

using F2 = uint64_t;  // two fp32
__device__ __forceinline__ F2 both(float v) { return pack_f32x2(v, v); }
__device__ __forceinline__ F2 neg2(F2 v) { return v ^ 0x8000000080000000ull; }

// A lane's sixteen values of a row as they lie in memory: eight from `lo`, eight from `hi`.
template <typename T>
struct Row16 {  // 16-bit types
  uint4 w[2];
  __device__ __forceinline__ void load(const T* p, int lo, int hi) {
    w[0] = *reinterpret_cast<const uint4*>(p + lo);
    w[1] = *reinterpret_cast<const uint4*>(p + hi);
  }
  __device__ __forceinline__ void clear() { w[0] = w[1] = make_uint4(0u, 0u, 0u, 0u); }
  static __device__ __forceinline__ F2 two(uint32_t x) {
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
      return pack_f32x2(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x));
      return pack_f32x2(f.x, f.y);
    }
  }
  static __device__ __forceinline__ uint32_t one(F2 v) {
    float x, y;
    unpack_f32x2(v, x, y);
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
      return *reinterpret_cast<const uint32_t*>(&h);
    } else {
      const __half2 h = __floats2half2_rn(x, y);
      return *reinterpret_cast<const uint32_t*>(&h);
    }
  }
  __device__ __forceinline__ void values(F2 a[4], F2 b[4]) const {
    a[0] = two(w[0].x); a[1] = two(w[0].y); a[2] = two(w[0].z); a[3] = two(w[0].w);
    b[0] = two(w[1].x); b[1] = two(w[1].y); b[2] = two(w[1].z); b[3] = two(w[1].w);
  }
  static __device__ __forceinline__ void store(T* p, int lo, int hi, const F2 a[4], const F2 b[4]) {
    *reinterpret_cast<uint4*>(p + lo) = make_uint4(one(a[0]), one(a[1]), one(a[2]), one(a[3]));
    *reinterpret_cast<uint4*>(p + hi) = make_uint4(one(b[0]), one(b[1]), one(b[2]), one(b[3]));
  }
};
struct Row32 {
  ulonglong2 w[4];
  __device__ __forceinline__ void load(const float* p, int lo, int hi) {
    w[0] = *reinterpret_cast<const ulonglong2*>(p + lo);
    w[1] = *reinterpret_cast<const ulonglong2*>(p + lo + 4);
    w[2] = *reinterpret_cast<const ulonglong2*>(p + hi);
    w[3] = *reinterpret_cast<const ulonglong2*>(p + hi + 4);
  }
  __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = make_ulonglong2(0ull, 0ull); }
  __device__ __forceinline__ void values(F2 a[4], F2 b[4]) const {
    a[0] = w[0].x; a[1] = w[0].y; a[2] = w[1].x; a[3] = w[1].y;
    b[0] = w[2].x; b[1] = w[2].y; b[2] = w[3].x; b[3] = w[3].y;
  }
  static __device__ __forceinline__ void store(float* p, int lo, int hi, const F2 a[4], const F2 b[4]) {
    *reinterpret_cast<ulonglong2*>(p + lo) = make_ulonglong2(a[0], a[1]);
    *reinterpret_cast<ulonglong2*>(p + lo + 4) = make_ulonglong2(a[2], a[3]);
    *reinterpret_cast<ulonglong2*>(p + hi) = make_ulonglong2(b[0], b[1]);
    *reinterpret_cast<ulonglong2*>(p + hi + 4) = make_ulonglong2(b[2], b[3]);
  }
};
template <typename T>
using Row = typename std::conditional<std::is_same<T, float>::value, Row32, Row16<T>>::type;

struct RopeTensor {
  const void* x;     // [B, heads, N, D]
  const void* grad;  // backward: gradient of the result
  void* out;         // the result, or backward: the gradient of x
  long long x_b, x_h, x_n, g_b, g_h, g_n, o_b, o_h, o_n;  // strides in elements
  const float* weight;
  const float* bias;
  int heads;
  int chunk, chunks;  // heads that a group of lanes walks for its token, and such parts
};

struct RopeParams {
  RopeTensor t[2];  // queries, keys
  const int* positions;
  long long pos_b, pos_n;
  long long tokens_all;  // batch * tokens
  int tokens, axes, norm;

  float eps;
  float* partials;              // backward: [2][kMaxRopePartials][2 D]
  unsigned long long turns[kMaxRopeDim / 2];  // turns per position, base^(-2 i / S) / 2 pi, of a section's pairs in units of
                                              // 2^-64: whole turns fall out of the product with a position
};

// Batch entry and place in it of a token of all.
__device__ __forceinline__ void place(const RopeParams& p, long long token, long long& b, long long& n) {
  if (p.tokens_all <= 0x7FFFFFFF) {
    const int q = static_cast<int>(token) / p.tokens;
    b = q;
    n = static_cast<int>(token) - q * p.tokens;
  } else {
    b = token / p.tokens;
    n = token - b * p.tokens;
  }
}

template <int kLanes>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}
template <int kLanes>
__device__ __forceinline__ float group_sum(F2 v) {
  float x, y;
  unpack_f32x2(v, x, y);
  return group_sum<kLanes>(x + y);
}

// Where a lane's eight pairs lie in a row, and the sines and cosines of a token.
template <int kDim>
struct Pairs {
  int lo, hi, axis, index;  // first elements; axis of the section; number of the first pair in it
  __device__ __forceinline__ Pairs(int lane_in_group, int axes) {
    const int half = kDim / (2 * max(axes, 1));
    const int first = 8 * lane_in_group;
    axis = first / half;
    index = first - axis * half;
    lo = axis * 2 * half + index;
    hi = lo + half;
  }
  __device__ __forceinline__ int position(const RopeParams& p, long long b, long long n) const {
    return p.axes == 0 ? 0 : __ldg(p.positions + b * p.pos_b + n * p.pos_n + axis);
  }
  // kFast: by the special function unit, off by at most 2^-20.5, a thousandth of the rounding of a 16-bit result: for results
  // that are all in 16 bits (the gradient's sums are in fp32: exact ones cost it 1 us of 19, 1.3 of 112).
  template <bool kFast>
  __device__ __forceinline__ void turn(const RopeParams& p, int pos, F2 c[4], F2 s[4]) const {
    if (p.axes == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        c[i] = both(1.f);
        s[i] = both(0.f);
      }
      return;
    }
    float sv[8], cv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // the fraction of a turn, in units of 2^-32 between -1/2 and 1/2
      const int f = static_cast<int>((static_cast<unsigned long long>(static_cast<long long>(pos)) * p.turns[index + i]) >> 32);
      if constexpr (kFast) __sincosf(static_cast<float>(f) * static_cast<float>(6.283185307179586 / 4294967296.0), &sv[i], &cv[i]);
      else sincospif(static_cast<float>(f) * (1.f / 2147483648.f), &sv[i], &cv[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      c[i] = pack_f32x2(cv[2 * i], cv[2 * i + 1]);
      s[i] = pack_f32x2(sv[2 * i], sv[2 * i + 1]);
    }
  }
};
__device__ __forceinline__ void load8(const float* p, F2 v[4], float otherwise) {
  if (p == nullptr) {
    v[0] = v[1] = v[2] = v[3] = both(otherwise);
  } else {
    const ulonglong2 x = __ldg(reinterpret_cast<const ulonglong2*>(p)), y = __ldg(reinterpret_cast<const ulonglong2*>(p) + 1);
    v[0] = x.x; v[1] = x.y; v[2] = y.x; v[3] = y.y;
  }
}

// x less its mean in place of x (layer norm); returns the reciprocal of the deviation.
template <int kDim>
__device__ __forceinline__ float centre(F2 a[4], F2 b[4], int norm, float eps) {
  constexpr int kLanes = kDim / 16;
  if (norm == LITE3R_NORM_NONE) return 1.f;
  if (norm == LITE3R_NORM_LAYER) {
    F2 sum = add_f32x2(add_f32x2(add_f32x2(a[0], a[1]), add_f32x2(a[2], a[3])), add_f32x2(add_f32x2(b[0], b[1]), add_f32x2(b[2], b[3])));
    const F2 less = both(group_sum<kLanes>(sum) * (-1.f / kDim));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = add_f32x2(a[i], less);
      b[i] = add_f32x2(b[i], less);
    }
  }
  F2 sq = mul_f32x2(a[0], a[0]), sq2 = mul_f32x2(b[0], b[0]);
#pragma unroll
  for (int i = 1; i < 4; ++i) {
    sq = fma_f32x2(a[i], a[i], sq);
    sq2 = fma_f32x2(b[i], b[i], sq2);
  }
  return rsqrtf(fmaf(group_sum<kLanes>(add_f32x2(sq, sq2)), 1.f / kDim, eps));
}

// One token and a part of its heads per group of lanes (blockIdx.y: which part, of the queries first, then of the keys).  The
// rows' loop has the same length for all groups; groups past the last token load nothing and store nothing.
// With x the row less its mean and r the reciprocal of its deviation:
//   y[lo] = r (x[lo] w[lo] cos - x[hi] w[hi] sin) + (b[lo] cos - b[hi] sin),   y[hi] = r (x[hi] w[hi] cos + x[lo] w[lo] sin) + ...
template <typename T, int kDim>
__global__ void __launch_bounds__(kRopeThreads, kRopeCtas) rope_kernel(const __grid_constant__ RopeParams p) {
  constexpr int kLanes = kDim / 16;
  constexpr int kRows = sizeof(T) == 4 ? 1 : 2;  // of a step; the next step's are requested ahead of its arithmetic
  const int sub = threadIdx.x % kLanes;
  const long long token = (static_cast<long long>(blockIdx.x) * kRopeThreads + threadIdx.x) / kLanes;
  const int which = static_cast<int>(blockIdx.y) < p.t[0].chunks ? 0 : 1;
  const RopeTensor& t = p.t[which];
  const int h0 = (static_cast<int>(blockIdx.y) - (which == 0 ? 0 : p.t[0].chunks)) * t.chunk;
  const int count = min(t.chunk, t.heads - h0);
  const bool live = token < p.tokens_all;
  const Pairs<kDim> pair(sub, p.axes);
  wait_for_prior_grid();
  launch_dependents();
  long long b, n;
  place(p, live ? token : 0, b, n);
  const T* x = static_cast<const T*>(t.x) + b * t.x_b + n * t.x_n + h0 * t.x_h;
  T* out = static_cast<T*>(t.out) + b * t.o_b + n * t.o_n + h0 * t.o_h;
  Row<T> next[kRows];
  auto fetch = [&](int i) {
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      if (live && i + j < count) next[j].load(x + j * t.x_h, pair.lo, pair.hi);
      else next[j].clear();
    }
    x += kRows * t.x_h;
  };
  const int pos = pair.position(p, b, n);
  fetch(0);
  F2 alo[4], blo[4], ahi[4], bhi[4], clo[4], chi[4];
  {
    F2 c[4], s[4], wl[4], wh[4], dl[4], dh[4];
    load8(t.weight == nullptr ? nullptr : t.weight + pair.lo, wl, 1.f);
    load8(t.weight == nullptr ? nullptr : t.weight + pair.hi, wh, 1.f);
    load8(t.bias == nullptr ? nullptr : t.bias + pair.lo, dl, 0.f);
    load8(t.bias == nullptr ? nullptr : t.bias + pair.hi, dh, 0.f);
    pair.template turn<sizeof(T) == 2>(p, pos, c, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      alo[i] = mul_f32x2(wl[i], c[i]);
      blo[i] = neg2(mul_f32x2(wh[i], s[i]));
      ahi[i] = mul_f32x2(wh[i], c[i]);
      bhi[i] = mul_f32x2(wl[i], s[i]);
      clo[i] = fma_f32x2(dl[i], c[i], neg2(mul_f32x2(dh[i], s[i])));
      chi[i] = fma_f32x2(dh[i], c[i], mul_f32x2(dl[i], s[i]));
    }
  }
  for (int i = 0; i < count; i += kRows) {
    Row<T> cur[kRows];
#pragma unroll
    for (int j = 0; j < kRows; ++j) cur[j] = next[j];
    if (i + kRows < count) fetch(i + kRows);
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      F2 a[4], c[4], ya[4], yc[4];
      cur[j].values(a, c);
      const F2 r = both(centre<kDim>(a, c, p.norm, p.eps));
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        a[q] = mul_f32x2(a[q], r);
        c[q] = mul_f32x2(c[q], r);
        ya[q] = fma_f32x2(a[q], alo[q], clo[q]);
        yc[q] = fma_f32x2(c[q], ahi[q], chi[q]);
      }
      if (p.axes != 0) {  // (without a rotation the other value stays out, be it infinite)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          ya[q] = fma_f32x2(c[q], blo[q], ya[q]);
          yc[q] = fma_f32x2(a[q], bhi[q], yc[q]);
        }
      }
      if (live && i + j < count) Row<T>::store(out + j * t.o_h, pair.lo, pair.hi, ya, yc);
    }
    out += kRows * t.o_h;
  }
}

// Gradient of one tensor (blockIdx.y: queries or keys).  Groups of lanes walk tokens (and parts of their heads) in steps of
// the grid and keep dw and db of their sixteen elements in registers; a CTA adds its groups in order and leaves one partial.
// The weight lies in shared memory: registers hold the sums, the angles' sines and cosines and the next row on its way.
// Two bounds lie close together.  Instructions: four warps to a scheduler take 60 % of its issue slots, and of the time in which a
// warp is stalled 32 % goes to results of fixed latency, 20 % to busy pipes, 19 % to shuffles and shared memory, 26 % to loads.
// Loads: with the arithmetic left out one row ahead still takes 110 us of 115 (and a plain addition over the same three
// streams 88).  Rows through a ring in shared memory, three ahead and across tokens, mend the second at the cost of the first: 125.
template <typename T, int kDim>
__global__ void __launch_bounds__(kRopeThreads, back_ctas(sizeof(T))) rope_back_kernel(const __grid_constant__ RopeParams p) {
  constexpr int kLanes = kDim / 16;
  constexpr int kGroups = kRopeThreads / kLanes;
  __shared__ __align__(16) float s_sum[kGroups][2 * kDim];
  __shared__ __align__(16) float s_weight[kDim];
  const RopeTensor& t = p.t[blockIdx.y];
  const int sub = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  const long long units = p.tokens_all * t.chunks;
  const Pairs<kDim> pair(sub, p.axes);
  wait_for_prior_grid();
  launch_dependents();
  for (int i = threadIdx.x; i < kDim; i += kRopeThreads) s_weight[i] = t.weight == nullptr ? 1.f : __ldg(t.weight + i);
  __syncthreads();
  F2 dwa[4], dwb[4], dba[4], dbb[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) dwa[i] = dwb[i] = dba[i] = dbb[i] = 0ull;
  for (long long base = static_cast<long long>(blockIdx.x) * kGroups; base < units; base += static_cast<long long>(gridDim.x) * kGroups) {
    const long long unit = base + group;
    const bool live = unit < units;
    const long long token = !live ? 0 : t.chunks == 1 ? unit : unit / t.chunks;
    const int h0 = live ? static_cast<int>(unit - token * t.chunks) * t.chunk : 0;
    const int count = live ? min(t.chunk, t.heads - h0) : 0;
    long long b, n;
    place(p, token, b, n);
    const T* x = static_cast<const T*>(t.x) + b * t.x_b + n * t.x_n + h0 * t.x_h;
    const T* grad = static_cast<const T*>(t.grad) + b * t.g_b + n * t.g_n + h0 * t.g_h;
    T* out = static_cast<T*>(t.out) + b * t.o_b + n * t.o_n + h0 * t.o_h;
    Row<T> next_x, next_g;
    auto fetch = [&](int i) {
      if (i < count) {
        next_x.load(x, pair.lo, pair.hi);
        next_g.load(grad, pair.lo, pair.hi);
      } else {
        next_x.clear();
        next_g.clear();
      }
      x += t.x_h;
      grad += t.g_h;
    };
    const int pos = pair.position(p, b, n);
    fetch(0);
    F2 c[4], s[4];
    pair.template turn<false>(p, pos, c, s);
    for (int i = 0; i < t.chunk; ++i) {
      F2 xa[4], xb[4], ga[4], gb[4];
      next_x.values(xa, xb);
      next_g.values(ga, gb);
      if (i + 1 < t.chunk) fetch(i + 1);
      const float root = centre<kDim>(xa, xb, p.norm, p.eps);
      const float r1 = i < count ? root : 0.f;  // (rows past the end are zeros; without an epsilon their root is infinite)
      const F2 r = both(r1);
      const ulonglong2* const w = reinterpret_cast<const ulonglong2*>(s_weight);
      F2 m1 = 0ull, m2 = 0ull;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (p.axes != 0) {
          const F2 u = ga[q], v = gb[q];
          ga[q] = fma_f32x2(u, c[q], mul_f32x2(v, s[q]));
          gb[q] = fma_f32x2(v, c[q], neg2(mul_f32x2(u, s[q])));
        }
        xa[q] = mul_f32x2(xa[q], r);
        xb[q] = mul_f32x2(xb[q], r);
        dwa[q] = fma_f32x2(ga[q], xa[q], dwa[q]);
        dwb[q] = fma_f32x2(gb[q], xb[q], dwb[q]);
        dba[q] = add_f32x2(dba[q], ga[q]);
        dbb[q] = add_f32x2(dbb[q], gb[q]);
        const ulonglong2 wl = w[(pair.lo >> 2) + (q >> 1)], wh = w[(pair.hi >> 2) + (q >> 1)];
        ga[q] = mul_f32x2(ga[q], (q & 1) ? wl.y : wl.x);
        gb[q] = mul_f32x2(gb[q], (q & 1) ? wh.y : wh.x);
        m1 = add_f32x2(m1, add_f32x2(ga[q], gb[q]));
        m2 = fma_f32x2(ga[q], xa[q], fma_f32x2(gb[q], xb[q], m2));
      }
      if (p.norm != LITE3R_NORM_NONE) {
        // r (gh - m1 - xh m2)
        const F2 k2 = both(group_sum<kLanes>(m2) * (-r1 / kDim));
        const F2 k1 = both(p.norm == LITE3R_NORM_LAYER ? group_sum<kLanes>(m1) * (-r1 / kDim) : 0.f);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          ga[q] = fma_f32x2(ga[q], r, fma_f32x2(xa[q], k2, k1));
          gb[q] = fma_f32x2(gb[q], r, fma_f32x2(xb[q], k2, k1));
        }
      }
      if (i < count) Row<T>::store(out, pair.lo, pair.hi, ga, gb);
      out += t.o_h;
    }
  }
  Row32::store(s_sum[group], pair.lo, pair.hi, dwa, dwb);
  Row32::store(s_sum[group] + kDim, pair.lo, pair.hi, dba, dbb);
  __syncthreads();
  for (int e = threadIdx.x; e < 2 * kDim; e += kRopeThreads) {
    float sum = 0.f;
#pragma unroll 8
    for (int g = 0; g < kGroups; ++g) sum += s_sum[g][e];
    p.partials[(static_cast<size_t>(blockIdx.y) * kMaxRopePartials + blockIdx.x) * 2 * kDim + e] = sum;
  }
}

struct RopeSums {
  float* d[2][2];  // [queries, keys][weight, bias] or null
};

// Adds the partials in a fixed order: a CTA has 8 elements of a tensor's dw and db, thread (i, e) every 128th partial of
// element e, all requested at once (a chain of batches of loads took 6 us, as long as a tenth of the gradient itself).
constexpr int kSumThreads = 1024, kSumElements = 8, kSumGroups = kSumThreads / kSumElements;
__global__ void __launch_bounds__(kSumThreads) rope_sums_kernel(const float* partials, int count, int dim, const __grid_constant__ RopeSums sums) {
  __shared__ float s_sum[kSumThreads / 32][kSumElements];
  constexpr int kMost = kMaxRopePartials / kSumGroups;
  const int which = blockIdx.y, e = threadIdx.x % kSumElements, group = threadIdx.x / kSumElements;
  const int element = blockIdx.x * kSumElements + e;  // of 2 dim: dw, db
  const float* src = partials + static_cast<size_t>(which) * kMaxRopePartials * 2 * dim + element;
  wait_for_prior_grid();
  launch_dependents();
  float v[kMost], acc = 0.f;
#pragma unroll
  for (int i = 0; i < kMost; ++i) v[i] = group + i * kSumGroups < count ? src[static_cast<size_t>(group + i * kSumGroups) * 2 * dim] : 0.f;
#pragma unroll
  for (int i = 0; i < kMost; ++i) acc += v[i];
  // the groups' sums: those of a warp by shuffles, then the warps'
#pragma unroll
  for (int o = 16; o >= kSumElements; o >>= 1) acc += __shfl_xor_sync(0xFFFFFFFFu, acc, o);
  const int warp = threadIdx.x >> 5;
  if ((threadIdx.x & 31) < kSumElements) s_sum[warp][e] = acc;
  __syncthreads();
  if (threadIdx.x < kSumElements) {
    acc = 0.f;
#pragma unroll
    for (int w = 0; w < kSumThreads / 32; ++w) acc += s_sum[w][e];
    float* dst = sums.d[which][element >= dim];
    if (dst != nullptr) dst[element >= dim ? element - dim : element] = acc;
  }
}

RopeTensor tensor_of(const lite3r_tensor* x, const lite3r_tensor* grad, const lite3r_tensor* out, const float* weight,
                     const float* bias, int heads) {
  RopeTensor t = {};
  t.heads = heads;
  if (heads == 0) return t;
  t.x = x->ptr;
  t.x_b = x->stride_b; t.x_h = x->stride_h; t.x_n = x->stride_n;
  if (grad != nullptr) {
    t.grad = grad->ptr;
    t.g_b = grad->stride_b; t.g_h = grad->stride_h; t.g_n = grad->stride_n;
  }
  t.out = const_cast<void*>(out->ptr);
  t.o_b = out->stride_b; t.o_h = out->stride_h; t.o_n = out->stride_n;
  t.weight = weight;
  t.bias = bias;
  return t;
}

RopeParams params_of(const lite3r_rope& how) {
  RopeParams p = {};
  p.positions = how.positions;
  p.pos_b = how.position_stride_b;
  p.pos_n = how.position_stride_n;
  p.tokens_all = static_cast<long long>(how.batch) * how.tokens;
  p.tokens = how.tokens;
  p.axes = how.axes;
  p.norm = static_cast<int>(how.norm);
  p.eps = how.eps;
  if (how.axes > 0) {
    // the factors of this thread's last base and section (64 powers take a microsecond, as much as the launch)
    thread_local double base = 0.0;
    thread_local int half = 0;
    thread_local unsigned long long turns[kMaxRopeDim / 2];
    if (base != how.base || half != how.head_dim / (2 * how.axes)) {
      base = how.base;
      half = how.head_dim / (2 * how.axes);
      const double step = std::log2(base) / half;
      for (int i = 0; i < half; ++i) {
        const double per_position = std::exp2(-step * i) * 0.15915494309189533577;
        turns[i] = static_cast<unsigned long long>(std::ldexp(per_position - std::floor(per_position), 64));
      }
    }
    std::copy(turns, turns + half, p.turns);
  }
  return p;
}

// Parts of a token's heads: as many heads to a part as leave every SM its `ctas` resident CTAs, so that a token's coefficients
// serve many heads; one head at the fewest tokens.  (Counted for a CTA more than reside, the forward of two frames took 11.9 us
// instead of 7.5, of eight 17.4 instead of 16.8.)
void set_chunks(RopeTensor& t, long long tokens_all, int dim, int most, int sms, int ctas) {
  if (t.heads == 0) return;
  const long long groups = static_cast<long long>(sms) * ctas * (kRopeThreads / (dim / 16));
  int chunk = static_cast<int>(std::min<long long>(std::min(most, t.heads), std::max<long long>(1, tokens_all * t.heads / groups)));
  chunk = std::max(chunk, ceil_div(t.heads, 32767));  // (parts are the grid's second dimension)
  t.chunks = ceil_div(t.heads, chunk);
  t.chunk = ceil_div(t.heads, t.chunks);
}

// Calls fn with a value of the element type and the head dimension as template arguments.
template <typename T, typename Fn>
lite3r_status by_dim(int dim, const Fn& fn) {
  switch (dim) {
    case 32: return fn(T{}, std::integral_constant<int, 32>());
    case 64: return fn(T{}, std::integral_constant<int, 64>());
    case 128: return fn(T{}, std::integral_constant<int, 128>());
    case 256: return fn(T{}, std::integral_constant<int, 256>());
  }
  return LITE3R_ERR_UNSUPPORTED;
}
template <typename Fn>
lite3r_status by_type(int dtype, int dim, const Fn& fn) {
  switch (dtype) {
    case LITE3R_F32: return by_dim<float>(dim, fn);
    case LITE3R_BF16: return by_dim<__nv_bfloat16>(dim, fn);
    case LITE3R_F16: return by_dim<__half>(dim, fn);
  }
  return LITE3R_ERR_UNSUPPORTED;
}

}  // namespace

size_t rope_workspace_bytes(int head_dim) { return static_cast<size_t>(2) * kMaxRopePartials * 2 * head_dim * sizeof(float); }

lite3r_status launch_rope(const lite3r_tensor* q, const lite3r_tensor* k, const lite3r_rope& how, const lite3r_tensor* q_out,
                          const lite3r_tensor* k_out, cudaStream_t stream) {
  int sms = 0;
  const lite3r_status st = sm_count(&sms);
  if (st != LITE3R_OK) return st;
  RopeParams p = params_of(how);
  p.t[0] = tensor_of(q, nullptr, q_out, how.q_weight, how.q_bias, how.q_heads);
  p.t[1] = tensor_of(k, nullptr, k_out, how.k_weight, how.k_bias, how.k_heads);
  for (RopeTensor& x : p.t) set_chunks(x, p.tokens_all, how.head_dim, 16, sms, kRopeCtas);
  const int groups = kRopeThreads / (how.head_dim / 16);
  const long long blocks = (p.tokens_all + groups - 1) / groups;
  const int parts = p.t[0].chunks + p.t[1].chunks;
  if (blocks > 0x7FFFFFFFLL || parts > 65535) return LITE3R_ERR_UNSUPPORTED;
  return by_type(q->dtype, how.head_dim, [&](auto type, auto dim) {
    return launch_dependent(rope_kernel<decltype(type), decltype(dim)::value>, dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(parts)), kRopeThreads, 0, stream, p);
  });
}

lite3r_status launch_rope_backward(const lite3r_tensor* q, const lite3r_tensor* k, const lite3r_tensor* dq_out,
                                   const lite3r_tensor* dk_out, const lite3r_rope& how, const lite3r_tensor* dq,
                                   const lite3r_tensor* dk, const lite3r_rope_grads& grads, float* partials, cudaStream_t stream) {
  int sms = 0;
  lite3r_status st = sm_count(&sms);
  if (st != LITE3R_OK) return st;
  RopeParams p = params_of(how);
  p.t[0] = tensor_of(q, dq_out, dq, how.q_weight, how.q_bias, how.q_heads);
  p.t[1] = tensor_of(k, dk_out, dk, how.k_weight, how.k_bias, how.k_heads);
  p.partials = partials;
  const int tensors = how.k_heads > 0 ? 2 : 1, resident = back_ctas(q->dtype == LITE3R_F32 ? 4 : 2);
  long long units = 0;
  for (RopeTensor& x : p.t) {
    set_chunks(x, p.tokens_all, how.head_dim, 4, sms, resident);
    units = std::max(units, p.tokens_all * x.chunks);
  }
  const int groups = kRopeThreads / (how.head_dim / 16);
  const int blocks = static_cast<int>(std::min<long long>({kMaxRopePartials, static_cast<long long>(resident) * sms, (units + groups - 1) / groups}));
  st = by_type(q->dtype, how.head_dim, [&](auto type, auto dim) {
    return launch_dependent(rope_back_kernel<decltype(type), decltype(dim)::value>, dim3(static_cast<unsigned>(blocks), tensors),
                            kRopeThreads, 0, stream, p);
  });
  if (st != LITE3R_OK) return st;
  RopeSums sums = {{{grads.q_weight, grads.q_bias}, {grads.k_weight, grads.k_bias}}};
  if (grads.q_weight == nullptr && grads.q_bias == nullptr && grads.k_weight == nullptr && grads.k_bias == nullptr) return LITE3R_OK;
  return launch_dependent(rope_sums_kernel, dim3(static_cast<unsigned>(2 * how.head_dim / kSumElements), tensors), kSumThreads, 0, stream,
                          static_cast<const float*>(partials), blocks, how.head_dim, sums);
}

}  // namespace lite3r
