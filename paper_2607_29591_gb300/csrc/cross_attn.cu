// Attention to states of another length: the entry points (reskv_cross_attn,
// reskv_cross_attn_backward), what they refuse and which kernels they take.
#include <cmath>
#include <initializer_list>

#include "cross.cuh"

namespace reskv {
namespace {

constexpr size_t kLeftAlone = 1024;               // of a workspace: tickets of reskv_paged_attn

std::string check_cross(const reskv_cross_attn_args* a) {
  if (!a) return "args is NULL";
  std::string bad;
  if (a->n_tokens != 0) bad = check_heads(&a->q, "q");
  if (bad.empty() && a->n_tokens != 0) bad = check_heads(&a->o, "o");
  if (bad.empty() && a->n_rows != 0) bad = check_heads(&a->k, "k");
  if (bad.empty() && a->n_rows != 0) bad = check_heads(&a->v, "v");
  if (!bad.empty()) return bad;
  if (a->head_dim != 64 && a->head_dim != 128) return "head_dim must be 64 or 128";
  if (a->q.dtype != RESKV_BF16 && a->q.dtype != RESKV_F16) return "q must be bf16 or fp16";
  if (a->k.dtype != a->q.dtype || a->v.dtype != a->q.dtype || a->o.dtype != a->q.dtype) return "q, k, v and o must have one dtype";
  if (a->q.n_heads < 1 || a->o.n_heads != a->q.n_heads) return "q and o must have the same heads";
  if (a->k.n_heads < 1 || a->v.n_heads != a->k.n_heads) return "k and v must have the same heads";
  if (a->q.n_heads % a->k.n_heads || a->q.n_heads / a->k.n_heads > 64)
    return "q's heads must be a multiple of k's, at most 64 per KV head";
  if (a->batch < 1 || a->batch > (1 << 24) || int64_t(a->batch) * a->k.n_heads > (1 << 28))
    return "batch must be in [1, 2^24], batch * n_kv_heads at most 2^28";
  if (a->n_tokens < 0 || double(a->n_tokens) * a->q.n_heads >= double(int64_t(1) << 31))
    return "n_tokens must not be negative, n_tokens * heads below 2^31";
  if (a->n_rows < 0 || double(a->n_rows) * a->k.n_heads >= double(int64_t(1) << 31))
    return "n_rows must not be negative, n_rows * n_kv_heads below 2^31";
  if (!a->q_begin && a->n_tokens % a->batch) return "n_tokens must be a multiple of batch without q_begin";
  if (!a->kv_begin && a->n_rows % a->batch) return "n_rows must be a multiple of batch without kv_begin";
  if (a->lse && !aligned_to(a->lse, 4)) return "lse must be 4-byte aligned";
  if ((a->q_begin && !aligned_to(a->q_begin, 4)) || (a->kv_begin && !aligned_to(a->kv_begin, 4)) ||
      (a->kv_lens && !aligned_to(a->kv_lens, 4)) || (a->status && !aligned_to(a->status, 4)))
    return "q_begin, kv_begin, kv_lens and status must be 4-byte aligned";
  if (!std::isfinite(a->scale)) return "scale must be finite";
  return "";
}

CrossRows rows_of(const reskv_heads& t) { return {t.data, t.token_stride, t.head_stride}; }

CrossParams params_of(const reskv_cross_attn_args* a) {
  CrossParams p{};
  p.q = rows_of(a->q);
  p.k = rows_of(a->k);
  p.v = rows_of(a->v);
  p.o = rows_of(a->o);
  p.lse = a->lse;
  p.q_begin = a->q_begin;
  p.kv_begin = a->kv_begin;
  p.kv_lens = a->kv_lens;
  p.status = a->status;
  p.n_tokens = a->n_tokens;
  p.n_rows = a->n_rows;
  p.q_each = int32_t(a->n_tokens / a->batch);
  p.kv_each = int32_t(a->n_rows / a->batch);
  p.batch = a->batch;
  p.heads = a->q.n_heads;
  p.kv_heads = a->k.n_heads;
  p.group = p.heads / p.kv_heads;
  p.f16 = a->q.dtype == RESKV_F16;
  p.scale = a->scale != 0.f ? a->scale : 1.f / std::sqrt(float(a->head_dim));
  p.scale2 = p.scale * kLog2e;
  return p;
}

cudaError_t device_sms(int* dev, int* sms) {
  const cudaError_t err = cudaGetDevice(dev);
  return err != cudaSuccess ? err : cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, *dev);
}

// false: rows that copies cannot address
bool encode_maps(CrossMaps* maps, const reskv_cross_attn_args* a, const CrossParams& p, int box_states) {
  return a->n_rows > 0 && a->n_tokens > 0 &&
         encode_heads(&maps->q, a->q, a->n_tokens, a->head_dim, p.group, cross_tile_tokens(p.group)) &&
         encode_heads(&maps->k, a->k, a->n_rows, a->head_dim, 1, box_states) &&
         encode_heads(&maps->v, a->v, a->n_rows, a->head_dim, 1, box_states);
}

// Whether a gradient begins where another tensor does that blocks beside its own still read or write (no full look for
// overlaps; over o, and d_k and d_v over k or v, each block has read its rows before it writes them).
bool in_the_way(const reskv_cross_attn_args* a, const reskv_heads* d_o, const reskv_heads* d_q, const reskv_heads* d_k,
                const reskv_heads* d_v, bool tokens, bool rows) {
  if (tokens && (d_q->data == a->q.data || d_q->data == d_o->data)) return true;
  if (rows && d_k->data == d_v->data) return true;
  if (!tokens || !rows) return false;
  for (const void* x : {d_k->data, d_v->data})
    if (x == a->q.data || x == d_o->data || x == d_q->data) return true;
  return d_q->data == a->k.data || d_q->data == a->v.data;
}

// The kernel of few rows where a sequence and KV head have kFewRows of them on average.
constexpr int kFewRows = 16;

}  // namespace
}  // namespace reskv

using namespace reskv;

extern "C" reskv_status reskv_cross_attn(const reskv_cross_attn_args* a, void* stream) {
  return no_throw([&]() -> reskv_status {
    const std::string bad = check_cross(a);
    if (!bad.empty()) return paged_fail(RESKV_ERR_INVALID_ARG, bad);
    if (a->n_tokens == 0) return RESKV_OK;
    const CrossParams p = params_of(a);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int dev = 0, sms = 0;
    const cudaError_t err = device_sms(&dev, &sms);
    if (err != cudaSuccess) return launch_result(err, "reading the device");
    CrossMaps maps;
    const bool few = a->n_tokens * p.group <= kFewRows * int64_t(a->batch);
    const bool fast = rows_aligned(a->q, 16) && rows_aligned(a->o, 16) && encode_maps(&maps, a, p, few ? kRowStates : 128);
    return launch_result(!fast ? launch_cross_general(p, a->head_dim, s)
                         : few ? launch_cross_rows(p, maps, a->head_dim, dev, sms, s)
                               : launch_cross_blocks(p, maps, a->head_dim, dev, s),
                         "cross attention");
  });
}

extern "C" size_t reskv_cross_attn_workspace(const reskv_cross_attn_args* a) {
  if (!a || a->n_tokens < 0 || a->q.n_heads < 1) return 0;
  return kLeftAlone + (size_t(a->n_tokens) * size_t(a->q.n_heads) * sizeof(float4) + 255) / 256 * 256;
}

extern "C" reskv_status reskv_cross_attn_backward(const reskv_cross_attn_args* a, const reskv_heads* d_o, const reskv_heads* d_q,
                                                  const reskv_heads* d_k, const reskv_heads* d_v, void* stream) {
  return no_throw([&]() -> reskv_status {
    std::string bad = check_cross(a);
    const bool tokens = bad.empty() && a->n_tokens != 0, rows = bad.empty() && a->n_rows != 0;
    if (bad.empty() && tokens) bad = check_heads(d_o, "d_o");
    if (bad.empty() && tokens) bad = check_heads(d_q, "d_q");
    if (bad.empty() && rows) bad = check_heads(d_k, "d_k");
    if (bad.empty() && rows) bad = check_heads(d_v, "d_v");
    if (bad.empty() && tokens && (d_o->n_heads != a->q.n_heads || d_q->n_heads != a->q.n_heads ||
                                  d_o->dtype != a->q.dtype || d_q->dtype != a->q.dtype))
      bad = "d_o and d_q must have q's heads and dtype";
    if (bad.empty() && rows && (d_k->n_heads != a->k.n_heads || d_v->n_heads != a->k.n_heads ||
                                d_k->dtype != a->q.dtype || d_v->dtype != a->q.dtype))
      bad = "d_k and d_v must have k's heads and dtype";
    if (bad.empty() && tokens && !a->lse) bad = "the gradient needs the lse of reskv_cross_attn";
    if (bad.empty() && tokens &&
        (!a->workspace || !aligned_to(a->workspace, 256) || a->workspace_bytes < reskv_cross_attn_workspace(a)))
      bad = "workspace must be 256-byte aligned and hold reskv_cross_attn_workspace() bytes";
    if (bad.empty() && in_the_way(a, d_o, d_q, d_k, d_v, tokens, rows))
      bad = "d_q must not lie over q, d_o, k or v, d_k and d_v not over q or d_o, and none over another";
    if (!bad.empty()) return paged_fail(RESKV_ERR_INVALID_ARG, bad);
    if (!tokens && !rows) return RESKV_OK;
    CrossParams p = params_of(a);
    if (tokens) {
      p.d_o = rows_of(*d_o);
      p.d_q = rows_of(*d_q);
      p.stats = reinterpret_cast<float4*>(static_cast<char*>(a->workspace) + kLeftAlone);
    }
    if (rows) {
      p.d_k = rows_of(*d_k);
      p.d_v = rows_of(*d_v);
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int dev = 0, sms = 0;
    const cudaError_t err = device_sms(&dev, &sms);
    if (err != cudaSuccess) return launch_result(err, "reading the device");
    CrossMaps maps;
    const bool fast = tokens && rows && rows_aligned(a->o, 16) && rows_aligned(*d_o, 16) && rows_aligned(*d_q, 16) &&
                      rows_aligned(*d_k, 16) && rows_aligned(*d_v, 16) && encode_maps(&maps, a, p, 128) &&
                      encode_heads(&maps.d_o, *d_o, a->n_tokens, a->head_dim, p.group, cross_tile_tokens(p.group));
    return launch_result(fast ? launch_cross_grad(p, maps, a->head_dim, dev, s) : launch_cross_grad_general(p, a->head_dim, s),
                         "the gradient of cross attention");
  });
}
