// Cross attention and its gradient for rows of any alignment and stride: a warp a row,
// dims lane, lane + 32, .. of it in every lane, one element a load.  Bound by its
// instructions (a dot product takes five shuffles), some hundred times slower than the
// kernels for aligned rows, and the plainest form of the definitions.
#include "cross.cuh"

namespace reskv {
namespace {

constexpr int kWarps = 8;

template <bool kF16>
__device__ __forceinline__ float element(const void* p, int64_t at) {
  if constexpr (kF16) return __half2float(static_cast<const __half*>(p)[at]);
  else return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at]);
}

template <bool kF16, int E>
__device__ __forceinline__ void load_row(float (&x)[E], const CrossRows& r, int64_t row, int head, int lane) {
  const int64_t at = row * r.token + head * r.head + lane;
#pragma unroll
  for (int j = 0; j < E; ++j) x[j] = element<kF16>(r.data, at + 32 * j);
}
template <bool kF16, int E>
__device__ __forceinline__ void store_row(const CrossRows& r, int64_t row, int head, int lane, const float (&x)[E], float f) {
  const int64_t at = row * r.token + head * r.head + lane;
#pragma unroll
  for (int j = 0; j < E; ++j) {
    if constexpr (kF16) static_cast<__half*>(r.data)[at + 32 * j] = __float2half_rn(x[j] * f);
    else static_cast<__nv_bfloat16*>(r.data)[at + 32 * j] = __float2bfloat16_rn(x[j] * f);
  }
}
template <int E>
__device__ __forceinline__ float dot(const float (&a)[E], const float (&b)[E]) {
  float x = 0.f;
#pragma unroll
  for (int j = 0; j < E; ++j) x = fmaf(a[j], b[j], x);
#pragma unroll
  for (int o = 16; o; o /= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// The sequence that holds token or row t: sequences are in order.  -1: none.
__device__ __forceinline__ int owner(const int32_t* begin, int batch, int64_t total, int64_t t) {
  if (!begin) {
    const int64_t each = total / batch;
    return each == 0 || t / each >= batch ? -1 : int(t / each);
  }
  int lo = 0, hi = batch;         // the last sequence that begins at t or before
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (begin[mid] <= t) lo = mid;
    else hi = mid;
  }
  return begin[lo] <= t && t < begin[lo + 1] ? lo : -1;
}

template <int D, bool kF16>
__global__ void __launch_bounds__(kWarps * 32) k_cross(const __grid_constant__ CrossParams p) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31;
  const int64_t unit = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int64_t tok = unit / p.heads;
  const int h = int(unit - tok * p.heads);
  wait_for_previous();
  if (tok >= p.n_tokens) return;
  const int b = owner(p.q_begin, p.batch, p.n_tokens, tok);
  if (b < 0) return;
  const CrossSequence s = cross_sequence(p, b);
  float q[E], o[E] = {}, top = -INFINITY, l = 0.f;
  load_row<kF16>(q, p.q, tok, h, lane);
#pragma unroll 1
  for (int j = 0; j < s.seen; ++j) {
    float k[E], v[E];
    load_row<kF16>(k, p.k, s.k0 + j, h / p.group, lane);
    load_row<kF16>(v, p.v, s.k0 + j, h / p.group, lane);
    const float x = dot(q, k) * p.scale2;
    if (x > top) {
      const float keep = exp2f(top - x);
      l *= keep;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] *= keep;
      top = x;
    }
    const float w = x == -INFINITY ? 0.f : exp2f(x - top);
    l += w;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(w, v[e], o[e]);
  }
  store_row<kF16>(p.o, tok, h, lane, o, l != 0.f ? 1.f / l : 0.f);
  if (p.lse && lane == 0) p.lse[tok * p.heads + h] = l != 0.f ? (top + log2f(l)) * 0.693147180559945f : -INFINITY;
}


template <int D, bool kF16>
__global__ void __launch_bounds__(kWarps * 32) k_cross_grad_q(const __grid_constant__ CrossParams p) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31;
  const int64_t unit = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int64_t tok = unit / p.heads;
  const int h = int(unit - tok * p.heads);
  wait_for_previous();
  if (tok >= p.n_tokens) return;
  const int b = owner(p.q_begin, p.batch, p.n_tokens, tok);
  if (b < 0) return;
  const CrossSequence s = cross_sequence(p, b);
  float q[E], o[E], g[E], dq[E] = {}, mean[E] = {}, lacks = 0.f;        // sums of T k, P k and T
  load_row<kF16>(q, p.q, tok, h, lane);
  load_row<kF16>(o, p.o, tok, h, lane);
  load_row<kF16>(g, p.d_o, tok, h, lane);
  const float delta = dot(o, g), lse = p.lse[tok * p.heads + h];
  RowShift shift{log2_sum(lse), 0.f, 0.f};
  if (far_sum(lse)) {
    FarSum sum;
#pragma unroll 1
    for (int j = 0; j < s.seen; ++j) {
      float k[E];
      load_row<kF16>(k, p.k, s.k0 + j, h / p.group, lane);
      const float x = dot(q, k);
      sum.move(p.scale2 < 0.f ? -x : x, p.scale2);
      sum.l += sum.weight(x, p.scale2);
    }
    shift = RowShift{sum.hi, sum.lo, log2f(sum.l)};
  }
#pragma unroll 1
  for (int j = 0; j < s.seen; ++j) {
    float k[E], v[E];
    load_row<kF16>(k, p.k, s.k0 + j, h / p.group, lane);
    load_row<kF16>(v, p.v, s.k0 + j, h / p.group, lane);
    const float w = exp2f(shift.exponent(dot(q, k), p.scale2)), t = w * (dot(g, v) - delta);
    lacks += t;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      dq[e] = fmaf(t, k[e], dq[e]);
      mean[e] = fmaf(w, k[e], mean[e]);
    }
  }
  // P sums up to 1, so the sum of T is what D of the rounded o lacks
#pragma unroll
  for (int e = 0; e < E; ++e) dq[e] = fmaf(-lacks, mean[e], dq[e]);
  store_row<kF16>(p.d_q, tok, h, lane, dq, p.scale);
  if (lane == 0) p.stats[tok * p.heads + h] = make_float4(shift.hi, shift.lo, shift.less, delta + lacks);
}

template <int D, bool kF16>
__global__ void __launch_bounds__(kWarps * 32) k_cross_grad_kv(const __grid_constant__ CrossParams p) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31;
  const int64_t unit = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int64_t row = unit / p.kv_heads;
  const int h = int(unit - row * p.kv_heads);
  wait_for_previous();
  if (row >= p.n_rows) return;
  const int b = owner(p.kv_begin, p.batch, p.n_rows, row);
  if (b < 0) return;
  const CrossSequence s = cross_sequence(p, b);
  float k[E], v[E], dk[E] = {}, dv[E] = {};
  if (row - s.k0 < s.seen) {
    load_row<kF16>(k, p.k, row, h, lane);
    load_row<kF16>(v, p.v, row, h, lane);
#pragma unroll 1
    for (int64_t i = 0; i < int64_t(s.count) * p.group; ++i) {
      const int64_t tok = s.q0 + i / p.group;
      const int hq = h * p.group + int(i % p.group);
      float q[E], g[E];
      load_row<kF16>(q, p.q, tok, hq, lane);
      load_row<kF16>(g, p.d_o, tok, hq, lane);
      const float4 stat = p.stats[tok * p.heads + hq];
      const float w = exp2f(RowShift{stat.x, stat.y, stat.z}.exponent(dot(q, k), p.scale2)), t = w * (dot(g, v) - stat.w);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        dv[e] = fmaf(w, g[e], dv[e]);
        dk[e] = fmaf(t, q[e], dk[e]);
      }
    }
  }
  store_row<kF16>(p.d_k, row, h, lane, dk, p.scale);
  store_row<kF16>(p.d_v, row, h, lane, dv, 1.f);
}

template <typename F>
cudaError_t over(F kernel, const CrossParams& p, int64_t units, cudaStream_t s) {
  if (units == 0) return cudaSuccess;
  return launch_early(kernel, unsigned((units + kWarps - 1) / kWarps), kWarps * 32, 0, s, p);
}
template <int D, bool kF16>
cudaError_t grad(const CrossParams& p, cudaStream_t s) {
  const cudaError_t err = over(k_cross_grad_q<D, kF16>, p, p.n_tokens * p.heads, s);
  return err != cudaSuccess ? err : over(k_cross_grad_kv<D, kF16>, p, p.n_rows * p.kv_heads, s);
}

}  // namespace

cudaError_t launch_cross_general(const CrossParams& p, int d, cudaStream_t s) {
  const int64_t units = p.n_tokens * p.heads;
  if (d == 128) return p.f16 ? over(k_cross<128, true>, p, units, s) : over(k_cross<128, false>, p, units, s);
  return p.f16 ? over(k_cross<64, true>, p, units, s) : over(k_cross<64, false>, p, units, s);
}
cudaError_t launch_cross_grad_general(const CrossParams& p, int d, cudaStream_t s) {
  if (d == 128) return p.f16 ? grad<128, true>(p, s) : grad<128, false>(p, s);
  return p.f16 ? grad<64, true>(p, s) : grad<64, false>(p, s);
}

}  // namespace reskv
