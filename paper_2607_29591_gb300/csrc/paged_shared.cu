// Attention with a shared prefix (reskv_paged_attn_shared): the join of its two passes.
//
// The passes leave, for every query row, the softmax's output over what they saw and the log
// of the sum of its weights: the own tokens' in one row, the prefix's in one row or, where
// it was taken in blocks of rows, in one record for each part of its positions, not yet
// divided by its sum.  With references s_k, sums l_k and outputs l_k o_k (1 and o_k of a whole
// row) the output is sum 2^(s_k - S) l_k o_k, S = log2 sum 2^s_k l_k.
// A warp a row; bound by latencies: the places are looked up before the passes have ended, and the rows are
// read together with the sums that weigh them, four records at a time (4 sequences behind 2000 positions
// 23.8 -> 22.1 us, 64 query tokens behind 4096 36.8 -> 33.9; eight at a time 22.6 and 34.5).
#include "paged_attn.cuh"

namespace reskv {
namespace {

constexpr int kWarps = 8;

// Index i with begin[i] <= x < begin[i + 1], or -1.
__device__ __forceinline__ int range_of(const int32_t* begin, int n, int64_t x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (begin[mid] <= x) lo = mid;
    else hi = mid;
  }
  return begin[lo] <= x && x < begin[lo + 1] ? lo : -1;
}

template <int D>
__global__ void __launch_bounds__(kWarps * 32) k_shared_join(const __grid_constant__ SharedJoin j) {
  const SharedParams& p = j.a;
  const int lane = threadIdx.x & 31;
  const int64_t row = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int64_t tok = row / p.heads;
  const int head = int(row - tok * p.heads);
  // the sequence, then the group: what no launch of this call writes, and what came before the call is done
  // (the pass before this waited for it before it let this begin)
  int seq = -1, group = -1;
  if (tok < p.n_tokens) {
    seq = p.q_begin ? range_of(p.q_begin, p.sequences, tok) : int(tok / (p.n_tokens / p.sequences));
    if (seq >= 0) group = p.seq_begin ? range_of(p.seq_begin, j.groups, seq) : seq / (p.sequences / j.groups);
  }
  int parts = 0;
  int64_t first = 0, stride = 0;                  // rows of the prefix's records
  if (group >= 0 && !j.plans) {
    const Sequence s = group_of(p, group, j.groups);
    parts = tok >= s.q0 && tok < s.q0 + s.count ? 1 : 0;
    first = row;
  }
  wait_for_previous();
  if (seq < 0) return;                            // a query of no sequence
  const int u = lane < D / 4 ? lane : 0;
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
  // rows are asked for before it is known whether they count: what does not may hold anything
  const float own = j.own_lse[row] * j.own_unit;  // (-inf, NaN: as they are)
  float4 a = reinterpret_cast<const float4*>(j.own + row * D)[u];
  if (group >= 0 && j.plans) {
    const GroupPlan g = j.plans[group];
    const int64_t r = (tok - g.q0) * p.group + head % p.group;
    // (of a seq_begin out of order there may be more items than CTAs and records)
    if (tok >= g.q0 && tok < g.q0 + g.count && g.first + int64_t(g.parts) * g.row_blocks * p.kv_heads <= j.items) {
      // item i has records i, or (streams) 2 i and 2 i + 1
      const int streams = j.block_rows == 128 ? 2 : 1;
      const int64_t block = r / j.block_rows;
      parts = g.parts * streams;
      stride = int64_t(g.row_blocks) * j.block_rows;
      first = (g.first + int64_t(head / p.group) * g.parts * g.row_blocks + block) * streams * j.block_rows + r % j.block_rows;
    }
  }
  // Record k of a row: of part k, or (streams) of part k / 2.
  auto at = [&](int k) {
    return j.plans && j.block_rows == 128 ? first + (k >> 1) * 2 * stride + (k & 1) * 128 : first + k * stride;
  };
  // 32 records at a time, their references and sums in the lanes; one of weight 0 still counts: a NaN in it is seen
  float top = -INFINITY, sum = 0.f;
#pragma unroll 1
  for (int k0 = 0; k0 < parts; k0 += 32) {
    const int n = min(32, parts - k0);
    float ref = -INFINITY, l = 1.f;
    if (lane < n) {
      if (j.plans) {
        const float2 s = reinterpret_cast<const float2*>(j.prefix_ref)[at(k0 + lane)];
        ref = s.x;
        l = s.y;
      } else {
        ref = j.prefix_ref[first];
      }
    }
    constexpr int kAtOnce = 4;
    float4 v[kAtOnce];
    auto ask = [&](int k) {
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        v[i] = k + i < n ? reinterpret_cast<const float4*>(j.prefix + at(k0 + k + i) * D)[u] : zero;
    };
    ask(0);
    if (k0 == 0) {
      top = own;
      sum = own != -INFINITY ? 1.f : 0.f;
      a = own != -INFINITY ? a : zero;
    }
    float now = ref;
#pragma unroll
    for (int o = 16; o; o /= 2) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, o));
    now = fmaxf(now, top);
    const uint32_t present = __ballot_sync(0xffffffffu, ref != -INFINITY);
    if (!present) continue;
    const float keep = top == -INFINITY ? 0.f : exp2f(top - now), f = ref == -INFINITY ? 0.f : exp2f(ref - now);
    float more = ref == -INFINITY ? 0.f : f * l;
#pragma unroll
    for (int o = 16; o; o /= 2) more += __shfl_xor_sync(0xffffffffu, more, o);
    sum = top == -INFINITY ? more : fmaf(sum, keep, more);
    a = top == -INFINITY ? zero : make_float4(a.x * keep, a.y * keep, a.z * keep, a.w * keep);
    top = now;
#pragma unroll 1
    for (int k = 0;;) {
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        add_scaled(a, __shfl_sync(0xffffffffu, f, (k + i) & 31), (present >> ((k + i) & 31)) & 1 ? v[i] : zero);
      if ((k += kAtOnce) >= n) break;
      ask(k);
    }
  }
  if (parts == 0) {
    top = own;
    sum = own != -INFINITY ? 1.f : 0.f;
    a = own != -INFINITY ? a : zero;
  }
  const bool seen = sum != 0.f;
  const float inv = seen ? 1.f / sum : 0.f;
  Sequence self{};
  self.q0 = int(tok);
  self.count = 1;
  const int h = head / p.group, r = head % p.group;
  if (lane < D / 4) store_out(p, self, h, r, lane, make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv));
  if (lane == 0) store_lse(p, self, h, r, seen ? top + log2f(sum) : -INFINITY);
}

}  // namespace

cudaError_t launch_shared_join(const SharedJoin& j, cudaStream_t s) {
  const int64_t rows = j.a.n_tokens * j.a.heads;
  const unsigned blocks = unsigned((rows + kWarps - 1) / kWarps);
  return j.dim == 128 ? launch_early(k_shared_join<128>, blocks, kWarps * 32, 0, s, j)
                      : launch_early(k_shared_join<64>, blocks, kWarps * 32, 0, s, j);
}

}  // namespace reskv
