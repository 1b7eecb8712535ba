// Attention of every sequence's newest tokens over its paged 4-bit cache
// (reskv_paged_attn).
#include <cmath>

#include "paged.cuh"

namespace reskv {
namespace {

struct AttnParams {
  const void* q;
  void* o;
  float* lse;
  int64_t q_token, q_head, o_token, o_head;
  const int32_t* q_begin;
  const int32_t* lens;
  const int32_t* page_table;
  const uint8_t* pages;
  uint32_t* status;
  int64_t n_pages, n_tokens;
  int32_t batch, table_pages, page_tokens, kv_heads, heads;
  int32_t window, o_f32;
  float scale2;                   // scale * log2 e
};

// One warp per (query token, query head), one position at a time, lane l
// holding dims 4l .. 4l+3 (two halves of the warp on neighbouring positions for
// d = 64): the running maximum m, sum l and weighted sum of the softmax.
template <typename T, int D, int kGroup>
__global__ void __launch_bounds__(128) k_paged_attn(const __grid_constant__ AttnParams p) {
  constexpr int L = D / 4, NG = D / kGroup, S = 32 / L;
  constexpr TileShape ts{D, NG};
  const int lane = threadIdx.x % 32, u = lane % L, sub = lane / L;
  const int64_t row = int64_t(blockIdx.x) * 4 + threadIdx.x / 32;
  if (row >= p.n_tokens * p.heads) return;
  const int64_t tok = row / p.heads;
  const int head = int(row - tok * p.heads), h = head / (p.heads / p.kv_heads);
  int b;
  int64_t first, count;
  if (p.q_begin) {
    int lo = 0, hi = p.batch;                         // last b with q_begin[b] <= tok
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (p.q_begin[mid] <= tok) lo = mid;
      else hi = mid;
    }
    b = lo;
    first = p.q_begin[b];
    count = p.q_begin[b + 1] - first;
    if (tok < first || tok >= first + count) return;
  } else {
    count = p.n_tokens / p.batch;
    b = int(tok / count);
    first = b * count;
  }
  const int64_t room = int64_t(p.table_pages) * p.page_tokens;
  int64_t len = p.lens[b];
  if (len < 0 || len > room) {
    if (lane == 0) report_status(p.status, kStatusBadIndex);
    len = len < 0 ? 0 : room;
  }
  const int64_t pos = len - count + (tok - first);
  const int64_t from = p.window > 0 && pos - p.window + 1 > 0 ? pos - p.window + 1 : 0;
  const T* q = static_cast<const T*>(p.q) + tok * p.q_token + head * p.q_head + 4 * u;
  float qx[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) qx[i] = to_f32(q[i]) * p.scale2;
  float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int64_t t0 = from; t0 <= pos; t0 += S) {
    const int64_t t = t0 + sub;
    bool see = t <= pos;
    const int64_t pg = t / p.page_tokens;
    int page = 0;
    if (see) {
      page = p.page_table[int64_t(b) * p.table_pages + pg];
      if (page < 0 || page >= p.n_pages) {
        if (u == 0) report_status(p.status, kStatusBadIndex);
        see = false;
      }
    }
    float x = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
    if (see) {
      const int slot = int(t - pg * p.page_tokens), r = slot % kTile;
      const uint8_t* tile =
          p.pages + ((int64_t(page) * p.kv_heads + h) * (p.page_tokens / kTile) + slot / kTile) * ts.bytes();
      const uint32_t kc = *reinterpret_cast<const uint16_t*>(tile + ts.k_unit(r, u));
      const uint32_t vc = *reinterpret_cast<const uint16_t*>(tile + ts.v_codes() + ts.v_unit(r, u));
      const uint16_t* km = reinterpret_cast<const uint16_t*>(tile + ts.k_meta()) + r * 2 * NG + 4 * u / kGroup;
      const uint16_t* vm = reinterpret_cast<const uint16_t*>(tile + ts.v_meta()) + r * 2 * NG + 4 * u / kGroup;
      const float ks = __uint_as_float(uint32_t(km[0]) << 16), kmin = __uint_as_float(uint32_t(km[NG]) << 16);
      const float vs = __uint_as_float(uint32_t(vm[0]) << 16), vmin = __uint_as_float(uint32_t(vm[NG]) << 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x = fmaf(qx[i], fmaf(ks, float((kc >> (4 * i)) & 15u), kmin), x);
        v[i] = fmaf(vs, float((vc >> (4 * i)) & 15u), vmin);
      }
    }
#pragma unroll
    for (int o = 1; o < L; o *= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (see) {
      const float top = x > m || x != x ? x : m;
      const float keep = m == -INFINITY ? 0.f : exp2f(m - top), w = top == -INFINITY ? 0.f : exp2f(x - top);
      l = l * keep + w;
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = acc[i] * keep + w * v[i];
      m = top;
    }
  }
  if (S == 2) {                                       // join the two halves
    const float m2 = __shfl_xor_sync(0xffffffffu, m, 16), l2 = __shfl_xor_sync(0xffffffffu, l, 16);
    const float top = m > m2 ? m : m2;
    const float a = m == -INFINITY ? 0.f : exp2f(m - top), c = m2 == -INFINITY ? 0.f : exp2f(m2 - top);
    l = l * a + l2 * c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float y = __shfl_xor_sync(0xffffffffu, acc[i], 16);
      acc[i] = acc[i] * a + y * c;
    }
    m = top;
  }
  const float inv = l != 0.f ? 1.f / l : 0.f;
  if (sub == 0) {
    const int64_t at = tok * p.o_token + head * p.o_head + 4 * u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (p.o_f32) static_cast<float*>(p.o)[at + i] = acc[i] * inv;
      else static_cast<T*>(p.o)[at + i] = from_f32<T>(acc[i] * inv);
    }
  }
  if (lane == 0 && p.lse) p.lse[tok * p.heads + head] = l != 0.f ? (m + log2f(l)) * 0.69314718056f : -INFINITY;
}

template <typename T>
void dispatch_attn(const AttnParams& p, int d, int group, cudaStream_t s) {
  const unsigned blocks = unsigned((p.n_tokens * p.heads + 3) / 4);
  if (d == 128 && group == 32) k_paged_attn<T, 128, 32><<<blocks, 128, 0, s>>>(p);
  else if (d == 128 && group == 64) k_paged_attn<T, 128, 64><<<blocks, 128, 0, s>>>(p);
  else if (d == 128) k_paged_attn<T, 128, 128><<<blocks, 128, 0, s>>>(p);
  else if (group == 32) k_paged_attn<T, 64, 32><<<blocks, 128, 0, s>>>(p);
  else k_paged_attn<T, 64, 64><<<blocks, 128, 0, s>>>(p);
}

std::string check_attn(const reskv_paged_kv* kv, const reskv_paged_attn_args* a) {
  std::string bad = check_paged(kv);
  if (!bad.empty()) return bad;
  if (!a) return "args is NULL";
  bad = check_heads(&a->q, "q");
  if (bad.empty()) bad = check_heads(&a->o, "o");
  if (!bad.empty()) return bad;
  if (a->q.dtype != RESKV_BF16 && a->q.dtype != RESKV_F16) return "q must be bf16 or fp16";
  if (a->o.dtype != a->q.dtype && a->o.dtype != RESKV_F32) return "o must have q's dtype or fp32";
  if (a->o.n_heads != a->q.n_heads) return "q and o must have the same heads";
  if (a->q.n_heads % kv->n_kv_heads || a->q.n_heads / kv->n_kv_heads > 64)
    return "q's heads must be a multiple of n_kv_heads, at most 64 per KV head";
  if (!a->lens) return "lens is NULL";
  if (a->n_tokens < 0 || double(a->n_tokens) * a->q.n_heads >= double(int64_t(1) << 31))
    return "n_tokens must not be negative, n_tokens * heads below 2^31";
  if (!a->q_begin && a->n_tokens % kv->batch) return "n_tokens must be a multiple of batch without q_begin";
  if (a->lse && !aligned_to(a->lse, 4)) return "lse must be 4-byte aligned";
  if (!a->workspace || !aligned_to(a->workspace, 256) || a->workspace_bytes < reskv_paged_attn_workspace(kv, a))
    return "workspace must be 256-byte aligned and hold reskv_paged_attn_workspace() bytes";
  if (!std::isfinite(a->scale) || a->window < 0) return "scale must be finite and window not negative";
  return "";
}

}  // namespace
}  // namespace reskv

using namespace reskv;

extern "C" size_t reskv_paged_attn_workspace(const reskv_paged_kv* kv, const reskv_paged_attn_args* a) {
  (void)kv;
  (void)a;
  return 256;
}

extern "C" reskv_status reskv_paged_attn(const reskv_paged_kv* kv, const reskv_paged_attn_args* a, void* stream) {
  if (a && a->n_tokens == 0) return RESKV_OK;
  const std::string bad = check_attn(kv, a);
  if (!bad.empty()) return paged_fail(RESKV_ERR_INVALID_ARG, bad);
  AttnParams p{};
  p.q = a->q.data;
  p.o = a->o.data;
  p.lse = a->lse;
  p.q_token = a->q.token_stride;
  p.q_head = a->q.head_stride;
  p.o_token = a->o.token_stride;
  p.o_head = a->o.head_stride;
  p.q_begin = a->q_begin;
  p.lens = a->lens;
  p.page_table = kv->page_table;
  p.pages = static_cast<const uint8_t*>(kv->pages);
  p.status = kv->status;
  p.n_pages = kv->n_pages;
  p.n_tokens = a->n_tokens;
  p.batch = kv->batch;
  p.table_pages = kv->table_pages;
  p.page_tokens = kv->page_tokens;
  p.kv_heads = kv->n_kv_heads;
  p.heads = a->q.n_heads;
  p.window = a->window;
  p.o_f32 = a->o.dtype == RESKV_F32;
  p.scale2 = (a->scale != 0.f ? a->scale : 1.f / std::sqrt(float(kv->head_dim))) * kLog2e;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a->q.dtype == RESKV_F16) dispatch_attn<__half>(p, kv->head_dim, kv->quant_group, s);
  else dispatch_attn<__nv_bfloat16>(p, kv->head_dim, kv->quant_group, s);
  return launch_status("paged attention");
}
