// Norms of queries and keys for each head, with the position rotation in the same pass, and their gradient:
//   qk_norm_rope           z = norm(x) * w + b over the D values of a (batch, head, token) row, then the rotation of the pairs
//                          (i, i + S/2) of every axis section of S = D / axes values by position * base^(-2 i / S)
//   qk_norm_rope_backward  g = R^T dy;  dw = sum g xh, db = sum g over all rows;  gh = g w;
//                          dx = r (gh - mean(gh) - xh mean(gh xh))   (layer norm; no mean(gh) for the root mean square norm)
// Both are one pass over the tensors and bound by HBM.  D / 8 lanes work on a row, each on four pairs: the four values at i
// and the four at i + S/2, so that a rotation needs no other lane and a row's two loads fill whole 32-byte sectors.  A
// group of lanes stays with one token and walks its heads: sine and cosine of the token's angles are made once, in
// registers, for all heads of queries and keys.
// Angles: position * base^(-2i/S) / 2 pi in fp64 (an fp32 product of a position of a million is off by a tenth of a
// radian), its fraction of a turn in fp32 by sincospif.  Sums and norms are fp32; results are rounded once.
#include <algorithm>
#include <cmath>

#include "common.cuh"
#include "sm100.cuh"

namespace lite3r {

namespace {

using namespace sm100;

constexpr int kRopeThreads = 256;
constexpr int kMaxRopeDim = 256;
constexpr int kMaxRopePartials = 1024;  // CTAs of the backward pass per tensor; each leaves one partial sum of dw and db

// Four consecutive values.
__device__ __forceinline__ void load4(const float* p, float v[4]) {
  const float4 a = *reinterpret_cast<const float4*>(p);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
}
__device__ __forceinline__ void load4(const __nv_bfloat16* p, float v[4]) {
  const uint2 a = *reinterpret_cast<const uint2*>(p);
  v[0] = __uint_as_float(a.x << 16); v[1] = __uint_as_float(a.x & 0xFFFF0000u);
  v[2] = __uint_as_float(a.y << 16); v[3] = __uint_as_float(a.y & 0xFFFF0000u);
}
__device__ __forceinline__ void load4(const __half* p, float v[4]) {
  const uint2 a = *reinterpret_cast<const uint2*>(p);
  const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&a.x)), y = __half22float2(*reinterpret_cast<const __half2*>(&a.y));
  v[0] = x.x; v[1] = x.y; v[2] = y.x; v[3] = y.y;
}
__device__ __forceinline__ void store4(float* p, const float v[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float v[4]) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ void store4(__half* p, const float v[4]) {
  const __half2 a = __floats2half2_rn(v[0], v[1]), b = __floats2half2_rn(v[2], v[3]);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

struct RopeTensor {
  const void* x;     // [B, heads, N, D]
  const void* grad;  // backward: gradient of the result
  void* out;         // the result, or backward: the gradient of x
  long long x_b, x_h, x_n, g_b, g_h, g_n, o_b, o_h, o_n;  // strides in elements
  const float* weight;
  const float* bias;
  int heads;
};

struct RopeParams {
  RopeTensor t[2];  // queries, keys
  const int* positions;
  long long pos_b, pos_n;
  long long tokens_all;  // batch * tokens
  int tokens, axes, norm;
  int heads_per_group, chunks;  // heads a group of lanes walks for its token; groups per token
  float eps;
  float* partials;              // backward: [2][kMaxRopePartials][2 D]
  double turns[kMaxRopeDim / 2];  // base^(-2 i / S) / 2 pi of the pairs of a section
};

template <int kLanes>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

// Where a lane's four pairs lie in a row, and the sines and cosines of a token.
template <int kDim>
struct Pairs {
  int lo, hi, axis, index;  // first elements; axis of the section; number of the first pair in it
  float c[4], s[4];
  __device__ __forceinline__ Pairs(int lane_in_group, int axes) {
    const int half = kDim / (2 * max(axes, 1));
    const int first = 4 * lane_in_group;
    axis = first / half;
    index = first - axis * half;
    lo = axis * 2 * half + index;
    hi = lo + half;
  }
  __device__ __forceinline__ void at(const RopeParams& p, long long token) {
    if (p.axes == 0) return;
    const long long b = token / p.tokens;
    const int pos = __ldg(p.positions + b * p.pos_b + (token - b * p.tokens) * p.pos_n + axis);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double t = static_cast<double>(pos) * p.turns[index + i];
      sincospif(2.f * static_cast<float>(t - rint(t)), &s[i], &c[i]);
    }
  }
};

// xh in place of x; returns the reciprocal of the deviation.
template <int kDim>
__device__ __forceinline__ float normalise(float a[4], float b[4], int norm, float eps) {
  constexpr int kLanes = kDim / 8;
  if (norm == LITE3R_NORM_NONE) return 1.f;
  if (norm == LITE3R_NORM_LAYER) {
    const float mean = group_sum<kLanes>(((a[0] + a[1]) + (a[2] + a[3])) + ((b[0] + b[1]) + (b[2] + b[3]))) * (1.f / kDim);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] -= mean;
      b[i] -= mean;
    }
  }
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) sq = fmaf(a[i], a[i], fmaf(b[i], b[i], sq));
  const float r = rsqrtf(fmaf(group_sum<kLanes>(sq), 1.f / kDim, eps));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i] *= r;
    b[i] *= r;
  }
  return r;
}

// One token and a part of its heads (queries first, then keys) per group of lanes.  Every lane of a warp runs the same
// number of rows (groups past the last token and heads past the last load nothing and store nothing), so that the shuffles
// of the norms have all lanes.
template <typename T, int kDim>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeParams p) {
  constexpr int kLanes = kDim / 8;
  constexpr int kAhead = 4;  // rows requested before the first is used
  const int sub = threadIdx.x % kLanes;
  const long long unit = (static_cast<long long>(blockIdx.x) * kRopeThreads + threadIdx.x) / kLanes;
  const long long token = unit / p.chunks;
  const int chunk = static_cast<int>(unit - token * p.chunks);
  const bool live = token < p.tokens_all;
  Pairs<kDim> pair(sub, p.axes);
  wait_for_prior_grid();
  launch_dependents();
  const long long b = live ? token / p.tokens : 0, n = live ? token - b * p.tokens : 0;
  if (live) pair.at(p, token);
  const int begin = chunk * p.heads_per_group;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const RopeTensor& t = p.t[which];
    const int first = which == 0 ? 0 : p.t[0].heads;
    const int h0 = max(begin - first, 0), h1 = live ? min(begin + p.heads_per_group - first, t.heads) : 0;
    int most = h1 - h0;  // of any group of the warp
#pragma unroll
    for (int o = 16; o >= kLanes; o >>= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
    if (most <= 0) continue;
    float wa[4], wb[4], ba[4], bb[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      wa[i] = wb[i] = 1.f;
      ba[i] = bb[i] = 0.f;
    }
    if (t.weight != nullptr) {
      load4(t.weight + pair.lo, wa);
      load4(t.weight + pair.hi, wb);
    }
    if (t.bias != nullptr) {
      load4(t.bias + pair.lo, ba);
      load4(t.bias + pair.hi, bb);
    }
    const T* x = static_cast<const T*>(t.x) + b * t.x_b + n * t.x_n;
    T* out = static_cast<T*>(t.out) + b * t.o_b + n * t.o_n;
    for (int i0 = 0; i0 < most; i0 += kAhead) {
      float a[kAhead][4], c[kAhead][4];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int h = h0 + i0 + j;
        if (h < h1) {
          load4(x + h * t.x_h + pair.lo, a[j]);
          load4(x + h * t.x_h + pair.hi, c[j]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) a[j][i] = c[j][i] = 0.f;
        }
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int h = h0 + i0 + j;
        normalise<kDim>(a[j], c[j], p.norm, p.eps);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float u = fmaf(a[j][i], wa[i], ba[i]), v = fmaf(c[j][i], wb[i], bb[i]);
          a[j][i] = p.axes == 0 ? u : fmaf(u, pair.c[i], -(v * pair.s[i]));
          c[j][i] = p.axes == 0 ? v : fmaf(v, pair.c[i], u * pair.s[i]);
        }
        if (h < h1) {
          store4(out + h * t.o_h + pair.lo, a[j]);
          store4(out + h * t.o_h + pair.hi, c[j]);
        }
      }
    }
  }
}

// Gradient of one tensor (blockIdx.y: queries or keys).  Groups of lanes walk tokens (and parts of their heads) in steps of
// the grid and keep dw and db of their eight elements in registers; a CTA adds its groups in order and leaves one partial.
template <typename T, int kDim>
__global__ void __launch_bounds__(kRopeThreads) rope_back_kernel(const __grid_constant__ RopeParams p) {
  constexpr int kLanes = kDim / 8;
  constexpr int kGroups = kRopeThreads / kLanes;
  constexpr int kAhead = 2;
  __shared__ float s_sum[kGroups][2 * kDim];
  const RopeTensor& t = p.t[blockIdx.y];
  const int sub = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  const int chunks = (t.heads + p.heads_per_group - 1) / p.heads_per_group;
  const long long units = p.tokens_all * chunks;
  Pairs<kDim> pair(sub, p.axes);
  wait_for_prior_grid();
  launch_dependents();
  float wa[4], wb[4], dwa[4], dwb[4], dba[4], dbb[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    wa[i] = wb[i] = 1.f;
    dwa[i] = dwb[i] = dba[i] = dbb[i] = 0.f;
  }
  if (t.weight != nullptr) {
    load4(t.weight + pair.lo, wa);
    load4(t.weight + pair.hi, wb);
  }
  for (long long base = static_cast<long long>(blockIdx.x) * kGroups; base < units; base += static_cast<long long>(gridDim.x) * kGroups) {
    const long long unit = base + group;
    const bool live = unit < units;
    const long long token = live ? unit / chunks : 0;
    const int h0 = live ? static_cast<int>(unit - token * chunks) * p.heads_per_group : 0;
    const int h1 = live ? min(h0 + p.heads_per_group, t.heads) : 0;
    const long long b = token / p.tokens, n = token - b * p.tokens;
    pair.at(p, token);
    const T* x = static_cast<const T*>(t.x) + b * t.x_b + n * t.x_n;
    const T* grad = static_cast<const T*>(t.grad) + b * t.g_b + n * t.g_n;
    T* out = static_cast<T*>(t.out) + b * t.o_b + n * t.o_n;
    for (int i0 = 0; i0 < p.heads_per_group; i0 += kAhead) {
      float xa[kAhead][4], xb[kAhead][4], ga[kAhead][4], gb[kAhead][4];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int h = h0 + i0 + j;
        if (h < h1) {
          load4(x + h * t.x_h + pair.lo, xa[j]);
          load4(x + h * t.x_h + pair.hi, xb[j]);
          load4(grad + h * t.g_h + pair.lo, ga[j]);
          load4(grad + h * t.g_h + pair.hi, gb[j]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) xa[j][i] = xb[j][i] = ga[j][i] = gb[j][i] = 0.f;
        }
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int h = h0 + i0 + j;
        const float r = normalise<kDim>(xa[j], xb[j], p.norm, p.eps);
        float m1 = 0.f, m2 = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (p.axes != 0) {
            const float u = ga[j][i], v = gb[j][i];
            ga[j][i] = fmaf(u, pair.c[i], v * pair.s[i]);
            gb[j][i] = fmaf(v, pair.c[i], -(u * pair.s[i]));
          }
          dwa[i] = fmaf(ga[j][i], xa[j][i], dwa[i]);
          dwb[i] = fmaf(gb[j][i], xb[j][i], dwb[i]);
          dba[i] += ga[j][i];
          dbb[i] += gb[j][i];
          ga[j][i] *= wa[i];
          gb[j][i] *= wb[i];
          m1 += ga[j][i] + gb[j][i];
          m2 = fmaf(ga[j][i], xa[j][i], fmaf(gb[j][i], xb[j][i], m2));
        }
        if (p.norm != LITE3R_NORM_NONE) {
          m2 = group_sum<kLanes>(m2) * (1.f / kDim);
          m1 = p.norm == LITE3R_NORM_LAYER ? group_sum<kLanes>(m1) * (1.f / kDim) : 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            ga[j][i] = r * (ga[j][i] - fmaf(xa[j][i], m2, m1));
            gb[j][i] = r * (gb[j][i] - fmaf(xb[j][i], m2, m1));
          }
        }
        if (h < h1) {
          store4(out + h * t.o_h + pair.lo, ga[j]);
          store4(out + h * t.o_h + pair.hi, gb[j]);
        }
      }
    }
  }
  store4(&s_sum[group][pair.lo], dwa);
  store4(&s_sum[group][pair.hi], dwb);
  store4(&s_sum[group][kDim + pair.lo], dba);
  store4(&s_sum[group][kDim + pair.hi], dbb);
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

// Adds the partials in a fixed order: a CTA has 32 elements of a tensor's dw and db, its 32 warps every 32nd partial each.
__global__ void __launch_bounds__(1024) rope_sums_kernel(const float* partials, int count, int dim, const RopeSums sums) {
  __shared__ float s_sum[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int which = blockIdx.y, e = blockIdx.x * 32 + lane;  // 2 dim elements: dw, db
  const float* src = partials + static_cast<size_t>(which) * kMaxRopePartials * 2 * dim + e;
  float acc = 0.f;
  wait_for_prior_grid();
  launch_dependents();
#pragma unroll 8
  for (int i = warp; i < count; i += 32) acc += src[static_cast<size_t>(i) * 2 * dim];
  s_sum[warp][lane] = acc;
  __syncthreads();
  if (warp == 0) {
    acc = 0.f;
#pragma unroll
    for (int w = 0; w < 32; ++w) acc += s_sum[w][lane];
    float* dst = sums.d[which][e >= dim];
    if (dst != nullptr) dst[e >= dim ? e - dim : e] = acc;
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
    const int half = how.head_dim / (2 * how.axes);
    const double step = std::log2(how.base) / half;
    for (int i = 0; i < half; ++i) p.turns[i] = std::exp2(-step * i) * 0.15915494309189533577;
  }
  return p;
}

// Heads a group walks for its token: as many as leave every SM four CTAs, so that a token's sines and cosines serve them all;
// one at the fewest tokens.
int heads_per_group(long long tokens_all, int heads, int dim, int sms) {
  const long long groups = static_cast<long long>(sms) * 4 * (kRopeThreads / (dim / 8));
  return static_cast<int>(std::min<long long>(heads, std::max<long long>(1, tokens_all * heads / groups)));
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
  const int heads = how.q_heads + how.k_heads;
  p.heads_per_group = heads_per_group(p.tokens_all, heads, how.head_dim, sms);
  p.chunks = ceil_div(heads, p.heads_per_group);
  const int groups = kRopeThreads / (how.head_dim / 8);
  const long long blocks = (p.tokens_all * p.chunks + groups - 1) / groups;
  if (blocks > 0x7FFFFFFFLL) return LITE3R_ERR_UNSUPPORTED;
  return by_type(q->dtype, how.head_dim, [&](auto type, auto dim) {
    return launch_dependent(rope_kernel<decltype(type), decltype(dim)::value>, dim3(static_cast<unsigned>(blocks)), kRopeThreads, 0, stream, p);
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
  const int heads = std::max(how.q_heads, how.k_heads);
  p.heads_per_group = heads_per_group(p.tokens_all, heads, how.head_dim, sms);
  const int groups = kRopeThreads / (how.head_dim / 8);
  const long long units = p.tokens_all * ceil_div(heads, p.heads_per_group);
  const int tensors = how.k_heads > 0 ? 2 : 1;
  const int blocks = static_cast<int>(std::min<long long>({kMaxRopePartials, 6LL * sms / tensors, (units + groups - 1) / groups}));
  st = by_type(q->dtype, how.head_dim, [&](auto type, auto dim) {
    return launch_dependent(rope_back_kernel<decltype(type), decltype(dim)::value>, dim3(static_cast<unsigned>(blocks), tensors),
                            kRopeThreads, 0, stream, p);
  });
  if (st != LITE3R_OK) return st;
  RopeSums sums = {{{grads.q_weight, grads.q_bias}, {grads.k_weight, grads.k_bias}}};
  if (grads.q_weight == nullptr && grads.q_bias == nullptr && grads.k_weight == nullptr && grads.k_bias == nullptr) return LITE3R_OK;
  return launch_dependent(rope_sums_kernel, dim3(static_cast<unsigned>(how.head_dim / 16), tensors), 1024, 0, stream,
                          static_cast<const float*>(partials), blocks, how.head_dim, sums);
}

}  // namespace lite3r
