// Attention to states of another length (include/reskv.h, reskv_cross_attn) and its
// gradient: what the kernels of cross*.cu share.
#pragma once
#include <cuda.h>

#include <atomic>

#include "paged.cuh"
#include "warp_mma.cuh"

namespace reskv {

struct CrossRows {
  void* data;
  int64_t token, head;            // strides in elements
};

struct CrossParams {
  CrossRows q, k, v, o, d_o, d_q, d_k, d_v;
  float* lse;
  float4* stats;                  // [n_tokens, heads] (backward): a row's RowShift, and <d_o, o>
  const int32_t* q_begin;
  const int32_t* kv_begin;
  const int32_t* kv_lens;
  uint32_t* status;
  int64_t n_tokens, n_rows;
  int32_t q_each, kv_each;        // tokens and rows of a sequence without q_begin, kv_begin
  int32_t batch, heads, kv_heads, group;
  int32_t f16;
  float scale, scale2;            // of the logits; times log2 e
};

// Weights are 2^(s f - ref) of a sum of products s, f = scale log2 e, with a reference near the row's largest s f, as
// fp32 holds it.  One rounding of s f - ref keeps most of a weight's digits, but from 2^26 on s f may lie past the reference
// by more than the weights' types reach.  So from kFarLogits on, where fp32 sums of products are some 2^-6 off anyway,
// weights come from s f rounded, as the reference does.  Either way equal sums have equal weights, in whichever tile.
constexpr float kFarLogits = 65536.f;
// log2 of a row's sum, less `up`, of its ln: -inf (all logits are) as what leaves every weight 0.
__device__ __forceinline__ float log2_sum(float lse, float up = 0.f) { return lse == -INFINITY ? 3.0e38f : fmaf(lse, kLog2e, -up); }

// The weights of a row in the gradient: 2^((s f - hi) - lo - less), s f - hi rounded once.  The log-sum-exp that
// the gradient is given will do for hi (with lo = less = 0) up to kFarSum, as log2: it is then off by 2^-15 of a weight.  Past
// it fp32 has ever fewer of its digits for a weight (at 1e7 none), so the gradient finds the row's largest s f itself:
// hi and lo are its product in full, less the log2 of the weights' sum beside it.
constexpr float kFarSum = 512.f;
__device__ __forceinline__ bool far_sum(float lse) { return fabsf(lse) * kLog2e > kFarSum && fabsf(lse) <= 3.0e38f; }
struct RowShift {
  float hi, lo, less;
  __device__ __forceinline__ float exponent(float s, float f) const { return (fmaf(s, f, -hi) - lo) - less; }
};
struct FarSum {
  float top = -INFINITY;          // the largest s so far, or -s where f < 0
  float hi = 0.f, lo = 0.f, l = 0.f;          // top f in two parts; sum of the weights beside it
  bool ok = true;
  __device__ __forceinline__ float weight(float s, float f) const { return exp2_fast(fmaf(s, f, -hi) - lo); }
  __device__ __forceinline__ void move(float to, float f) {
    if (!(to > top)) return;
    const float before = f < 0.f ? -top : top, now = f < 0.f ? -to : to;
    hi = __fmul_rn(now, f);
    lo = fmaf(now, f, -hi);
    l = top == -INFINITY ? l : l * weight(before, f);
    top = to;
  }
};

// A sequence's query tokens and rows; `seen` of the rows take part.
struct CrossSequence {
  int q0, count;
  int k0, rows, seen;
};

// Range b of `total` things: begin[b] .. begin[b + 1], or `each`.
__device__ __forceinline__ void cross_range(const int32_t* begin, int b, int each, int64_t total, uint32_t* status, int& first,
                                            int& count) {
  if (begin) {
    const int b0 = begin[b], b1 = begin[b + 1], n = int(total);
    if (b0 < 0 || b0 > n || b1 < b0 || b1 > n) report_status(status, kStatusBadIndex);
    first = min(max(b0, 0), n);
    count = min(max(b1, first), n) - first;
  } else {
    count = each;
    first = b * each;
  }
}
__device__ __forceinline__ CrossSequence cross_sequence(const CrossParams& p, int b) {
  CrossSequence s;
  cross_range(p.q_begin, b, p.q_each, p.n_tokens, p.status, s.q0, s.count);
  cross_range(p.kv_begin, b, p.kv_each, p.n_rows, p.status, s.k0, s.rows);
  s.seen = s.rows;
  if (p.kv_lens) {
    const int n = p.kv_lens[b];
    if (n < 0 || n > s.rows) report_status(p.status, kStatusBadIndex);
    s.seen = min(max(n, 0), s.rows);
  }
  return s;
}

// Whether the lengths are the call's own: then a block is found before the kernel before has ended.
__device__ __forceinline__ bool cross_fixed(const CrossParams& p) { return !p.q_begin && !p.kv_begin && !p.kv_lens; }

// The block that a CTA takes: of the tokens (or rows) of every sequence, begin[b] .. begin[b + 1] of `total` or
// `each`, `times` things each, `per` of those a block, for each KV head; blocks of a KV head lie side
// by side.  One warp; false: no such block.
//
// With begins, items are numbered so that no sequence need know those before it: sequence b's begin at
// first(b) times / per + b, rounded down, for each KV head, which leaves it as many as it has blocks at least
// (those beyond are none).  It is found by 32 looks at a time: one batch of loads up to 32 sequences, two up to
// 1024, five at most.  (A scan from the first sequence on: 16384 single tokens of 64 states 73 ms for 2.1.)
struct CrossBlock {
  int b, h, first;                // sequence, KV head, first of its things
};
__device__ __forceinline__ bool cross_block(const CrossParams& p, const int32_t* begin, int each, int64_t total, int per, int item,
                                            int lane, CrossBlock& out, int times = 1) {
  int blocks;
  if (begin) {
    int lo = 0, hi = p.batch;
#pragma unroll 1
    for (;;) {
      const int step = (hi - lo + 31) / 32, at = lo + lane * step;
      int first = 0, count = 0, start = 0;
      if (at < hi) {
        cross_range(begin, at, each, total, p.status, first, count);
        start = int(uint32_t(first) * uint32_t(times) / uint32_t(per)) + at;
      }
      const uint32_t after = ~__ballot_sync(0xffffffffu, at < hi && int64_t(start) * p.kv_heads <= item);
      if (after & 1) return false;                // before the first sequence
      const int l = after ? __ffs(after) - 2 : 31;
      if (step == 1) {
        out.b = lo + l;
        blocks = ceil_div(__shfl_sync(0xffffffffu, count, l) * times, per);
        item -= __shfl_sync(0xffffffffu, start, l) * p.kv_heads;
        break;
      }
      lo += l * step;
      hi = min(lo + step, hi);
    }
    // (each sequence's begins are looked at by one CTA at least)
    if (p.batch > 32 && threadIdx.x < 32 && blockIdx.x < unsigned(p.batch + 31) / 32 && int(blockIdx.x) * 32 + lane < p.batch) {
      int first, count;
      cross_range(begin, int(blockIdx.x) * 32 + lane, each, total, p.status, first, count);
    }
    if (item >= blocks * p.kv_heads) return false;
  } else {
    blocks = ceil_div(each * times, per);
    out.b = item / (blocks * p.kv_heads);
    item -= out.b * blocks * p.kv_heads;
  }
  out.h = item / blocks;
  out.first = (item - out.h * blocks) * per;
  return true;
}
// Tiles before rank r's, of `all` (below 2^24) that a cluster of 1, 2, 4 or 8 shares.
__device__ __forceinline__ int tiles_before(int all, int r, int cluster) {
  return int(uint32_t(all) * uint32_t(r) >> (cluster >> 1) - (cluster >> 3));
}
// Blocks that a call may have.
inline int64_t cross_blocks(const CrossParams& p, const int32_t* begin, int64_t total, int per, int times = 1) {
  return begin ? (total * times / per + p.batch) * p.kv_heads : (total / p.batch * times + per - 1) / per * p.batch * p.kv_heads;
}

// --- clusters ---
__device__ __forceinline__ uint32_t rank_in_cluster() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void sync_cluster() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The same, or of the block alone: for warps whose code has parted.
__device__ __forceinline__ void meet(int cluster) {
  if (cluster > 1) sync_cluster();
  else asm volatile("barrier.cta.sync 0;" ::: "memory");
}
__device__ __forceinline__ uint32_t of_rank(uint32_t local, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local), "r"(rank));
  return r;
}
__device__ __forceinline__ float read_cluster(uint32_t at) {
  float x;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ float4 read_cluster4(uint32_t at) {
  float4 x;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(at) : "memory");
  return x;
}
// One launch with programmatic dependence, in clusters where `cluster` > 1.
template <typename K, typename P>
cudaError_t launch_clusters(K kernel, int64_t blocks, int cluster, int threads, size_t shared, cudaStream_t s, const P& params) {
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = unsigned(cluster);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(unsigned(blocks * cluster));
  cfg.blockDim = dim3(unsigned(threads));
  cfg.dynamicSmemBytes = shared;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, params);
}
// M sums over sources i < n in order, those without a bit in `present` left out: out[m] = sum weight(m, i) * what
// lies at at(m, i), four elements a lane.  4 M are asked for at a time: one after the other each
// takes the cluster's latency (some 0.6 us).
template <int M, typename A, typename W>
__device__ __forceinline__ void add_sources(float4 (&out)[M], int n, uint32_t present, A at, W weight) {
#pragma unroll
  for (int m = 0; m < M; ++m) out[m] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += 4) {
    float4 v[M][4];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v[m][j] = i0 + j < n && ((present >> (i0 + j)) & 1) ? read_cluster4(at(m, i0 + j)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const float w = i0 + j < n && ((present >> (i0 + j)) & 1) ? weight(m, i0 + j) : 0.f;
        out[m].x = fmaf(w, v[m][j].x, out[m].x);
        out[m].y = fmaf(w, v[m][j].y, out[m].y);
        out[m].z = fmaf(w, v[m][j].z, out[m].z);
        out[m].w = fmaf(w, v[m][j].w, out[m].w);
      }
  }
}

// Clusters of `size` (2, 4, 8) CTAs of a kernel that run side by side; asked once a device.
struct SideBySide {
  std::atomic<int> known[64][4];
};
template <typename K>
int side_by_side(K kernel, SideBySide& kept, int size, int threads, size_t shared, int dev) {
  const int at = size == 2 ? 1 : size == 4 ? 2 : size == 8 ? 3 : 0;
  std::atomic<int>* k = dev >= 0 && dev < 64 ? &kept.known[dev][at] : nullptr;
  int n = k ? k->load(std::memory_order_relaxed) : 0;
  if (n == 0) {
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = unsigned(size);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(unsigned(size));
    cfg.blockDim = dim3(unsigned(threads));
    cfg.dynamicSmemBytes = shared;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, reinterpret_cast<const void*>(kernel), &cfg) != cudaSuccess) {
      cudaGetLastError();
      return 0;
    }
    if (k && n > 0) k->store(n, std::memory_order_relaxed);
  }
  return n;
}
// The cluster that shares a block's `tiles`: as large as all `blocks` (about) run side by side, of two tiles a CTA
// at least.
template <typename K>
int cluster_for(K kernel, SideBySide& kept, int64_t blocks, int64_t tiles, int threads, size_t shared, int dev) {
  int size = 1;
  while (size < 8 && size * 4 <= tiles && blocks <= side_by_side(kernel, kept, 2 * size, threads, shared, dev)) size *= 2;
  return size;
}
// A kernel's shared memory limit, raised once a device.
template <typename K>
cudaError_t raise_shared(K kernel, std::atomic<uint64_t>& raised, int bytes, int dev) {
  const uint64_t bit = dev >= 0 && dev < 64 ? uint64_t(1) << dev : 0;
  if (bit && (raised.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
  const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (err == cudaSuccess) raised.fetch_or(bit, std::memory_order_relaxed);
  return err;
}

// Many query rows, on the fifth-generation tensor cores; cross_blocks.cu.  Copies take whole tokens:
// a tile of 128 rows has cross_tile_tokens of them.
struct CrossMaps {
  CUtensorMap q, k, v, d_o;
};
inline int cross_tile_tokens(int group) { return 128 / group; }
// Few query rows: cross_rows.cu.  Copies of kRowStates states.
constexpr int kRowStates = 64;
cudaError_t launch_cross_rows(const CrossParams& p, const CrossMaps& maps, int d, int dev, int sms, cudaStream_t s);
cudaError_t launch_cross_grad(const CrossParams& p, const CrossMaps& maps, int d, int dev, cudaStream_t s);      // cross_grad.cu
cudaError_t launch_cross_blocks(const CrossParams& p, const CrossMaps& maps, int d, int dev, cudaStream_t s);

// Rows of any alignment; cross_general.cu.
cudaError_t launch_cross_general(const CrossParams& p, int d, cudaStream_t s);
cudaError_t launch_cross_grad_general(const CrossParams& p, int d, cudaStream_t s);

}  // namespace reskv
