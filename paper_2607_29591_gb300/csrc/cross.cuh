// Attention to states of another length (include/reskv.h, reskv_cross_attn) and its
// gradient: what the kernels of cross*.cu share.
#pragma once
#include <cuda.h>

#include "paged.cuh"

namespace reskv {

struct CrossRows {
  void* data;
  int64_t token, head;            // strides in elements
};

struct CrossParams {
  CrossRows q, k, v, o, d_o, d_q, d_k, d_v;
  float* lse;
  float* delta;                   // [n_tokens, heads]: <d_o, o> of every row (backward)
  const int32_t* q_begin;
  const int32_t* kv_begin;
  const int32_t* kv_lens;
  uint32_t* status;
  int64_t n_tokens, n_rows;
  int32_t batch, heads, kv_heads, group;
  int32_t f16;
  float scale, scale2;            // of the logits; times log2 e
};

// A sequence's query tokens and rows; `seen` of the rows take part.
struct CrossSequence {
  int q0, count;
  int k0, rows, seen;
};

// Range b of `total` things: begin[b] .. begin[b + 1], or equal shares.
__device__ __forceinline__ void cross_range(const int32_t* begin, int b, int batch, int64_t total, uint32_t* status,
                                            int& first, int& count) {
  if (begin) {
    const int b0 = begin[b], b1 = begin[b + 1], n = int(total);
    if (b0 < 0 || b0 > n || b1 < b0 || b1 > n) report_status(status, kStatusBadIndex);
    first = min(max(b0, 0), n);
    count = min(max(b1, first), n) - first;
  } else {
    count = int(total / batch);
    first = b * count;
  }
}
__device__ __forceinline__ CrossSequence cross_sequence(const CrossParams& p, int b) {
  CrossSequence s;
  cross_range(p.q_begin, b, p.batch, p.n_tokens, p.status, s.q0, s.count);
  cross_range(p.kv_begin, b, p.batch, p.n_rows, p.status, s.k0, s.rows);
  s.seen = s.rows;
  if (p.kv_lens) {
    const int n = p.kv_lens[b];
    if (n < 0 || n > s.rows) report_status(p.status, kStatusBadIndex);
    s.seen = min(max(n, 0), s.rows);
  }
  return s;
}

// Many query rows, on the fifth-generation tensor cores; cross_blocks.cu.  Copies take whole tokens:
// a tile of 128 rows has cross_tile_tokens of them.
struct CrossMaps {
  CUtensorMap q, k, v;
};
inline int cross_tile_tokens(int group) { return 128 / group; }
cudaError_t launch_cross_blocks(const CrossParams& p, const CrossMaps& maps, int d, int dev, int sms, cudaStream_t s);

// Rows of any alignment; cross_general.cu.
cudaError_t launch_cross_general(const CrossParams& p, int d, cudaStream_t s);
cudaError_t launch_cross_grad_general(const CrossParams& p, int d, cudaStream_t s);

}  // namespace reskv
