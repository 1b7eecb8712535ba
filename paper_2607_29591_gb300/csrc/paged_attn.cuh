// Attention over the paged 4-bit cache: parameters, the split of a call's work
// and the matrix step of one 16-token tile, shared by the kernels of
// paged_attn*.cu.
#pragma once
#include "paged.cuh"

namespace reskv {

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
  float* partials;                // [CTAs][2][record]
  int32_t* tickets;               // [CTAs], zero between calls
  int64_t n_pages, n_tokens;
  int32_t batch, table_pages, page_tokens, kv_heads, heads, group;
  int32_t window, q_f16, o_f32, q_wide, o_wide;
  float scale2;                   // scale * log2 e
};

// One block of query rows of one sequence: row r of the sequence is query token
// r / group, head r % group of the KV head.  Its tiles are those any of its rows
// sees (none: all of them stand before position 0).
struct RowBlock {
  int first, tiles;               // first tile of the sequence's positions; count
};

struct Sequence {
  int len, count, q0;             // held tokens, query tokens, first query token
};

__device__ __forceinline__ Sequence sequence_of(const AttnParams& p, int b) {
  Sequence s;
  if (p.q_begin) {
    const int64_t lo = min(max(int64_t(p.q_begin[b]), int64_t(0)), p.n_tokens);
    const int64_t hi = min(max(int64_t(p.q_begin[b + 1]), lo), p.n_tokens);
    s.q0 = int(lo);
    s.count = int(hi - lo);
  } else {
    s.count = int(p.n_tokens / p.batch);
    s.q0 = b * s.count;
  }
  const int room = p.table_pages * p.page_tokens;      // below 2^31
  const int len = p.lens[b];
  if (len < 0 || len > room) report_status(p.status, kStatusBadIndex);
  s.len = min(max(len, 0), room);
  return s;
}

// First position that a query at `pos` sees (pos may lie far below 0, a window be any).
__device__ __forceinline__ int first_seen(const AttnParams& p, int pos) {
  return p.window > 0 && pos >= p.window ? pos - p.window + 1 : 0;
}

// Rows [r0, r1) of a sequence.
__device__ __forceinline__ RowBlock row_block(const AttnParams& p, const Sequence& s, int r0, int r1) {
  // (one block of a sequence's rows, the usual case, divides nothing)
  const int lo = s.len - s.count + (r0 == 0 ? 0 : r0 / p.group);
  const int hi = s.len - s.count + (r1 == s.count * p.group ? s.count - 1 : (r1 - 1) / p.group);
  RowBlock b;
  b.first = first_seen(p, lo) / kTile;
  b.tiles = hi < 0 ? 0 : hi / kTile - b.first + 1;
  return b;
}

// --- matrix instructions -----------------------------------------------------

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                        uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

// what pack_f16 left over
__device__ __forceinline__ uint32_t rest_f16(float lo, float hi, uint32_t packed) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&packed));
  return pack_f16(lo - f.x, hi - f.y);
}

__device__ __forceinline__ float exp2_fast(float x) {          // 2^-inf = 0
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float min_nan(float a, float b) {     // a NaN kept
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// --- outputs -----------------------------------------------------------------

// Output row r of a sequence, dims 4u .. 4u + 3.
__device__ __forceinline__ void store_out(const AttnParams& p, const Sequence& s, int h, int r, int u, float4 v) {
  const int64_t tok = s.q0 + r / p.group;
  const int64_t at = tok * p.o_token + int64_t(h * p.group + r % p.group) * p.o_head + 4 * u;
  const float f[4] = {v.x, v.y, v.z, v.w};
  if (p.o_f32) {
    float* y = static_cast<float*>(p.o) + at;
    if (p.o_wide) {
      *reinterpret_cast<float4*>(y) = v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = f[i];
    }
    return;
  }
  uint16_t* y = static_cast<uint16_t*>(p.o) + at;
  uint16_t e[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    e[i] = p.q_f16 ? __half_as_ushort(__float2half_rn(f[i])) : __bfloat16_as_ushort(__float2bfloat16_rn(f[i]));
  if (p.o_wide) {
    *reinterpret_cast<uint2*>(y) = make_uint2(e[0] | uint32_t(e[1]) << 16, e[2] | uint32_t(e[3]) << 16);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = e[i];
  }
}

__device__ __forceinline__ void store_lse(const AttnParams& p, const Sequence& s, int h, int r, float ref) {
  if (p.lse) p.lse[(s.q0 + r / p.group) * int64_t(p.heads) + h * p.group + r % p.group] = ref * 0.693147180559945f;
}
// The softmaxes of up to 32 records joined: each lane's weight for its record's
// output, from their log2 sums (-inf: an empty or no record), the records that are none
// of these, and the joint sum.  A record of weight 0 still counts: a NaN in it is seen.
struct Joined {
  float weight, ref;
  uint32_t present;
};
__device__ __forceinline__ Joined join_weights(float ref) {
  float top = ref;
#pragma unroll
  for (int o = 16; o; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  const float f = ref == -INFINITY ? 0.f : exp2f(ref - top);
  float sum = f;
#pragma unroll
  for (int o = 16; o; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  const uint32_t present = __ballot_sync(0xffffffffu, ref != -INFINITY);
  return sum != 0.f ? Joined{f / sum, top + log2f(sum), present} : Joined{0.f, -INFINITY, 0u};
}
__device__ __forceinline__ void add_scaled(float4& a, float f, float4 v) {
  a.x = fmaf(f, v.x, a.x);
  a.y = fmaf(f, v.y, a.y);
  a.z = fmaf(f, v.z, a.z);
  a.w = fmaf(f, v.w, a.w);
}

// --- the tile step -----------------------------------------------------------

// R (8 or 4) query rows of one warp against tiles of 16 tokens.  In units of log2,
// with lane = 4 g + t:
//
//   logits  S^T[16 tokens x 8] = sum over groups  scale * (codes Q^T) + minimum * sum Q
//   output  O^T[dims x 8]     += codes^T (scale * P)^T,  and minima * P apart in fp32
//
// The codes enter the products as they lie: a masked word holds two 4-bit codes
// n as the fp16 subnormals n 2^-24 (n 2^-20 from the odd places), which the
// tensor cores multiply exactly, so that unpacking eight codes takes five
// integer instructions and no conversion.  A group's scale is applied to the
// fp32 products of the logits, and to the weights P before they are rounded to
// fp16 (two planes, 22 bits, unless the output is bf16).  Queries are scaled by a
// power of two to fp16's top, weights by the running reference: it follows the
// largest logit + log2 of the token's largest value scale, so that P * scale
// stays in fp16's range for value scales between 2^-96 and 2^96.  A token whose values
// are constant within every group has no scale and counts as one of 2^-48: its weight
// stays below 2^62, and times a minimum of up to 2^48 a sum within fp32.
//
// The reference moves only when it is passed by more than 8 (2^14 of fp16's
// range, where 2^6 stands for a weight of one).
//
// Eight rows fill the eight columns of a product.  Four rows take the columns
// twice: 0..3 for the first half of a row's groups, 4..7 for the second (zeros in
// the query operand keep the halves apart; one shuffle adds their logits), and in
// the output's product dims of the first half are its rows 0..7, of the second
// rows 8..15.  A lane then scales and rounds the weights of half the groups:
// 20 % fewer instructions a tile, and those bound the kernel.
constexpr float kNoRef = -3.0e38f;
constexpr float kLeastScale = 1.2621774483536189e-29f, kNoScale = 3.552713678800501e-15f;      // 2^-96, 2^-48

template <int D, int NG, bool kTwoPlanes, int R>
struct TileStep {
  static constexpr int kRows = R;
  static constexpr bool kHalves = R == 4;
  static constexpr int C = D / 32;               // 32-dim blocks
  static constexpr int H = kHalves ? C / 2 : C;  // of them per lane
  static constexpr int K = kHalves && NG > 1 ? NG / 2 : NG;         // groups per lane
  static constexpr int PG = H / K;               // blocks of one group

  // this lane's share of the query operand, column g: block c, code place 0..3
  uint32_t qb[kHalves ? 2 * H : H][4];
  uint32_t qs[2];                                // sums over groups, three bf16 planes
  float cq[2];                                   // logit scale of this lane's rows
  // running state of rows row(j)
  float ref[2], l[2];
  float o[2 * C][4];
  float om[K][2];
  int t, g, half;

  __device__ __forceinline__ void init(int lane) {
    g = lane >> 2;
    t = lane & 3;
    half = kHalves ? t >> 1 : 0;
  }
  __device__ __forceinline__ int row(int j) const { return (kHalves ? 2 * (t & 1) : 2 * t) + j; }
  // the 32-dim block that out(c, ., .) is of
  __device__ __forceinline__ int block(int c) const { return c + half * H; }

  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      ref[i] = kNoRef;
      l[i] = 0.f;
#pragma unroll
      for (int k = 0; k < K; ++k) om[k][i] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < 2 * C; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[j][i] = 0.f;
  }

  // Query row of column g (g & 3 of four; NULL: no such row).  Lane t takes dims 8 (4c + t) .. + 7 of blocks c.
  __device__ __forceinline__ void load_q(const AttnParams& p, const void* qrow) {
    const int second = kHalves ? g >> 2 : 0;
    float x[H][8];
    float top = 0.f;
#pragma unroll
    for (int c = 0; c < H; ++c) {
      const int at = 8 * (4 * (c + second * H) + t);
      if (!qrow) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[c][i] = 0.f;
      } else if (p.q_wide) {
        const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(qrow) + at);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 f = p.q_f16 ? __half22float2(*reinterpret_cast<const __half2*>(&w[i])) : bf16x2_to_float2(w[i]);
          x[c][2 * i] = f.x;
          x[c][2 * i + 1] = f.y;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          x[c][i] = p.q_f16 ? to_f32(static_cast<const __half*>(qrow)[at + i])
                            : to_f32(static_cast<const __nv_bfloat16*>(qrow)[at + i]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[c][i]));
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    if constexpr (kHalves) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
    // 2^e |x| < 2^15; two factors, as 2^e may pass fp32's range
    const int e = 141 - min(max(__float_as_int(top) >> 23, 1), 254), e1 = e >> 1, e2 = e - e1;
    const float f1 = __int_as_float((127 + e1) << 23), f2 = __int_as_float((127 + e2) << 23);
    float gs[NG];                                // group sums in units of the products, n 2^-24
#pragma unroll
    for (int k = 0; k < NG; ++k) gs[k] = 0.f;
#pragma unroll
    for (int c = 0; c < H; ++c) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[c][i] = x[c][i] * f1 * f2;
        sum += x[c][i];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float f = j & 1 ? 0.0625f : 1.f;
        const uint32_t w = pack_f16(x[c][j] * f, x[c][4 + j] * f);
        if constexpr (kHalves) {
          qb[c][j] = second ? 0u : w;
          qb[H + c][j] = second ? w : 0u;
        } else {
          qb[c][j] = w;
        }
      }
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      sum *= 5.9604644775390625e-8f;
      if constexpr (kHalves) {
        const float other = __shfl_xor_sync(0xffffffffu, sum, 16);
        gs[c / PG] += second ? other : sum;
        gs[NG == 1 ? 0 : K + c / PG] += second ? sum : other;
      } else {
        gs[c / PG] += sum;
      }
    }
    float plane[NG][3];
#pragma unroll
    for (int k = 0; k < NG; ++k) {
      float r = second ? 0.f : gs[k];            // counted once
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        plane[k][i] = __bfloat162float(__float2bfloat16_rn(r));
        r -= plane[k][i];
      }
    }
    auto two = [](float lo, float hi) {            // both exact bf16
      return (__float_as_uint(lo) >> 16) | (__float_as_uint(hi) & 0xffff0000u);
    };
    // k columns of the minima's product: lane t supplies columns 2t, 2t+1 and 2t+8, 2t+9
    if constexpr (NG == 4) {
      const int k = 2 * (t & 1), i = t >> 1;       // hi (t 0, 1), mid (t 2, 3); lo (t 0, 1)
      qs[0] = k == 0 ? (i == 0 ? two(plane[0][0], plane[1][0]) : two(plane[0][1], plane[1][1]))
                     : (i == 0 ? two(plane[2][0], plane[3][0]) : two(plane[2][1], plane[3][1]));
      qs[1] = i != 0 ? 0u : k == 0 ? two(plane[0][2], plane[1][2]) : two(plane[2][2], plane[3][2]);
    } else if constexpr (NG == 2) {
      qs[0] = t == 0 ? two(plane[0][0], plane[1][0]) : t == 1 ? two(plane[0][1], plane[1][1])
              : t == 2 ? two(plane[0][2], plane[1][2]) : 0u;
      qs[1] = 0u;
    } else {                                       // pairs (scale, minimum): zero against the scale
      qs[0] = t == 0 ? two(0.f, plane[0][0]) : t == 1 ? two(0.f, plane[0][1]) : t == 2 ? two(0.f, plane[0][2]) : 0u;
      qs[1] = 0u;
    }
    const float c = p.scale2 * 16777216.f * __int_as_float((127 - e1) << 23) * __int_as_float((127 - e2) << 23);
    cq[0] = __shfl_sync(0xffffffffu, c, 4 * row(0));
    cq[1] = __shfl_sync(0xffffffffu, c, 4 * row(1));
  }

  // This lane's scales (first) or minima of one row, from the row's 4 NG bytes.
  template <bool kMinima>
  __device__ __forceinline__ void lane_meta(float (&s)[K], const uint8_t* meta) const {
    if constexpr (NG == 4 && kHalves) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(meta + 4 * half + (kMinima ? 8 : 0));
      s[0] = low_bf16(w);
      s[1] = high_bf16(w);
    } else if constexpr (NG == 4) {
      const uint2 w = *reinterpret_cast<const uint2*>(meta + (kMinima ? 8 : 0));
      s[0] = low_bf16(w.x);
      s[1] = high_bf16(w.x);
      s[2] = low_bf16(w.y);
      s[3] = high_bf16(w.y);
    } else if constexpr (NG == 2) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(meta + (kMinima ? 4 : 0));
      if constexpr (kHalves) {
        s[0] = half ? high_bf16(w) : low_bf16(w);
      } else {
        s[0] = low_bf16(w);
        s[1] = high_bf16(w);
      }
    } else {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(meta);
      s[0] = kMinima ? high_bf16(w) : low_bf16(w);
    }
  }

  // One tile in shared memory.  With kMask, token g + 8 i takes part in row(j) only where see[i][j].
  template <bool kMask>
  __device__ __forceinline__ void step(const uint8_t* tile, const bool (&see)[2][2]) {
    constexpr TileShape ts{D, NG};
    uint32_t kw[2][C];
    load_words<C>(kw[0], tile + g * (D / 2) + t * (D / 8));
    load_words<C>(kw[1], tile + (g + 8) * (D / 2) + t * (D / 8));
    const uint8_t* kmeta = tile + ts.k_meta() + g * 4 * NG;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    {
      // minima against the sums of the query
      const int at = NG == 4 ? 8 + 4 * (t & 1) : NG == 2 ? 4 : 0;
      const uint32_t m0 = *reinterpret_cast<const uint32_t*>(kmeta + at);
      const uint32_t m1 = *reinterpret_cast<const uint32_t*>(kmeta + 8 * 4 * NG + at);
      if constexpr (NG == 4) mma_bf16(acc, m0, m1, m0, m1, qs[0], qs[1]);
      else mma_bf16(acc, m0, m1, 0u, 0u, qs[0], 0u);
    }
    float ks[2][K];
    lane_meta<false>(ks[0], kmeta);
    lane_meta<false>(ks[1], kmeta + 8 * 4 * NG);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = k * PG; c < (k + 1) * PG; ++c) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t w0 = j ? kw[0][c] >> 8 : kw[0][c], w1 = j ? kw[1][c] >> 8 : kw[1][c];
          if constexpr (kHalves) {
            const uint32_t u0 = j ? kw[0][c + H] >> 8 : kw[0][c + H], u1 = j ? kw[1][c + H] >> 8 : kw[1][c + H];
            mma_f16(a, w0 & 0x000f000fu, w1 & 0x000f000fu, u0 & 0x000f000fu, u1 & 0x000f000fu, qb[c][2 * j], qb[H + c][2 * j]);
            mma_f16(a, w0 & 0x00f000f0u, w1 & 0x00f000f0u, u0 & 0x00f000f0u, u1 & 0x00f000f0u, qb[c][2 * j + 1],
                    qb[H + c][2 * j + 1]);
          } else {
            mma_f16(a, w0 & 0x000f000fu, w1 & 0x000f000fu, w0 & 0x00f000f0u, w1 & 0x00f000f0u, qb[c][2 * j], qb[c][2 * j + 1]);
          }
        }
      }
      acc[0] = fmaf(ks[0][k], a[0], acc[0]);
      acc[1] = fmaf(ks[0][k], a[1], acc[1]);
      acc[2] = fmaf(ks[1][k], a[2], acc[2]);
      acc[3] = fmaf(ks[1][k], a[3], acc[3]);
    }
    if constexpr (kHalves) {
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], 2);
    }
    float vs[2][K], vm[2][K], top_s[2];
    const uint8_t* vmeta = tile + ts.v_meta() + g * 4 * NG;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      lane_meta<false>(vs[i], vmeta + i * 8 * 4 * NG);
      lane_meta<true>(vm[i], vmeta + i * 8 * 4 * NG);
      top_s[i] = kNoScale;                       // at least; fmaxf passes over NaN, whose rows decide nothing
#pragma unroll
      for (int k = 0; k < K; ++k) top_s[i] = fmaxf(top_s[i], vs[i][k]);
    }
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = exp2_fast(fmaf(acc[i], cq[i & 1], -ref[i & 1]));
      if (kMask && !see[i >> 1][i & 1]) w[i] = 0.f;
    }
    const float over = fmaxf(fmaxf(w[0], w[1]) * top_s[0], fmaxf(w[2], w[3]) * top_s[1]);
    if (__any_sync(0xffffffffu, over > 16384.f)) {
      // a row's reference: 6 below its largest logit + log2 scale
      float sg[2], x[4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) s = fmaxf(s, vs[i][k]);
        if constexpr (kHalves && NG > 1) s = fmaxf(s, __shfl_xor_sync(0xffffffffu, s, 2));
        sg[i] = fminf(log2f(s == 0.f ? kNoScale : fmaxf(s, kLeastScale)), 96.f);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float top = kNoRef;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          x[2 * i + j] = __fmul_rn(acc[2 * i + j], cq[j]);
          if (!kMask || see[i][j]) top = fmaxf(top, x[2 * i + j] + sg[i]);
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
        const float now = fmaxf(ref[j], top - 6.f);
        const float keep = exp2f(ref[j] - now);
        ref[j] = now;
        l[j] *= keep;
#pragma unroll
        for (int k = 0; k < K; ++k) om[k][j] *= keep;
#pragma unroll
        for (int m = 0; m < 2 * C; ++m) {
          o[m][j] *= keep;
          o[m][2 + j] *= keep;
        }
      }
      // From the rounded logits that the reference was taken from: past 2^26 it may lie many
      // units off the unrounded ones, and 6 and sg may be lost in it.
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = exp2_fast(min_nan(x[i] - ref[i & 1], 6.5f - sg[i >> 1]));
        if (kMask && !see[i >> 1][i & 1]) w[i] = 0.f;
      }
    }
    l[0] += w[0] + w[2];
    l[1] += w[1] + w[3];
    uint32_t b[K][2], b2[K][2];
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float x0 = w[2 * i] * vs[i][k], x1 = w[2 * i + 1] * vs[i][k];
        if constexpr (kMask) {                   // what is not seen may be NaN
          if (!see[i][0]) x0 = 0.f;
          if (!see[i][1]) x1 = 0.f;
          if (see[i][0]) om[k][0] = fmaf(w[2 * i], vm[i][k], om[k][0]);
          if (see[i][1]) om[k][1] = fmaf(w[2 * i + 1], vm[i][k], om[k][1]);
        } else {
          om[k][0] = fmaf(w[2 * i], vm[i][k], om[k][0]);
          om[k][1] = fmaf(w[2 * i + 1], vm[i][k], om[k][1]);
        }
        const uint32_t h = pack_f16(x0, x1);
        b[k][i] = transpose8x8(h);
        if constexpr (kTwoPlanes) b2[k][i] = transpose8x8(rest_f16(x0, x1, h));
      }
    }
    uint32_t v0[C], v1[C];
    const uint8_t* codes = tile + ts.v_codes();
    load_words<C>(v0, codes + t * D + ts.v_place(t, g) * (D / 8));
    load_words<C>(v1, codes + (t + 4) * D + ts.v_place(t + 4, g) * (D / 8));
#pragma unroll
    for (int c = 0; c < H; ++c) {
      const int k = c / PG;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t w0 = j ? v0[c] >> 8 : v0[c], w1 = j ? v1[c] >> 8 : v1[c];
        if constexpr (kHalves) {
          const uint32_t u0 = j ? v0[c + H] >> 8 : v0[c + H], u1 = j ? v1[c + H] >> 8 : v1[c + H];
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const uint32_t mask = n ? 0x00f000f0u : 0x000f000fu;
            float(&d)[4] = o[4 * c + 2 * j + n];
            mma_f16(d, w0 & mask, u0 & mask, w1 & mask, u1 & mask, b[k][0], b[k][1]);
            if constexpr (kTwoPlanes) mma_f16(d, w0 & mask, u0 & mask, w1 & mask, u1 & mask, b2[k][0], b2[k][1]);
          }
        } else {
          const uint32_t a0 = w0 & 0x000f000fu, a1 = w0 & 0x00f000f0u, a2 = w1 & 0x000f000fu, a3 = w1 & 0x00f000f0u;
          mma_f16(o[2 * c + j], a0, a1, a2, a3, b[k][0], b[k][1]);
          if constexpr (kTwoPlanes) mma_f16(o[2 * c + j], a0, a1, a2, a3, b2[k][0], b2[k][1]);
        }
      }
    }
  }

  // What a group's dims have in common goes from the accumulators to the minima's sum.
  // Codes are not negative, so that the sums grow with every tile and only the minima
  // take them back; the matrix unit cuts its sums off, by up to 2^-23 of them a product.
  // What a row's first dim of the group holds is about what all hold.  Every 16 tiles:
  // fp32 outputs over 8K positions in one piece are off by 5.4e-5 of themselves (without
  // 9.6e-4; every 32: 1e-4), 8 sequences of 32K take 63.4 us (63.0).
  __device__ __forceinline__ void settle() {
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float d;
        if constexpr (kHalves) d = half ? o[4 * k * PG][2 + j] : o[4 * k * PG][j];
        else d = o[2 * k * PG][j];
        d = __shfl_sync(0xffffffffu, d, t);
        if (g == 0) om[k][j] = fmaf(d, 16777216.f, om[k][j]);
#pragma unroll
        for (int c = k * PG; c < (k + 1) * PG; ++c) {
          if constexpr (kHalves) {                 // (the other half's elements are no one's)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              o[4 * c + i][j] = fmaf(i & 1 ? -16.f : -1.f, d, o[4 * c + i][j]);
              o[4 * c + i][2 + j] = fmaf(i & 1 ? -16.f : -1.f, d, o[4 * c + i][2 + j]);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              o[2 * c + i][j] -= d;
              o[2 * c + i][2 + j] = fmaf(-16.f, d, o[2 * c + i][2 + j]);
            }
          }
        }
      }
    }
  }

  // Sums over the lanes of a row; then out(c, i, j) is the softmax's output at dim
  // 32 block(c) + 4g + i of row(j), ref its log2 of the sum of 2^logit (-inf: nothing seen).
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
      for (int s = 4; s < 32; s *= 2) {
        l[j] += __shfl_xor_sync(0xffffffffu, l[j], s);
#pragma unroll
        for (int k = 0; k < K; ++k) om[k][j] += __shfl_xor_sync(0xffffffffu, om[k][j], s);
      }
      const bool seen = ref[j] != kNoRef || l[j] != 0.f;
      const float inv = seen ? 1.f / l[j] : 0.f;
      ref[j] = seen ? ref[j] + log2f(l[j]) : -INFINITY;
      l[j] = inv;
    }
  }
  __device__ __forceinline__ float out(int c, int i, int j) const {
    const float f = (i & 1) ? 1048576.f : 16777216.f;
    float v;
    if constexpr (kHalves) v = half ? o[4 * c + i][2 + j] : o[4 * c + i][j];
    else v = o[2 * c + i / 2][2 * (i & 1) + j];
    return (v * f + om[c / PG][j]) * l[j];
  }
};

// --- many rows: paged_attn_blocks.cu ---
// Units are blocks of 128 mt rows of a KV head and sequence.  The first `whole` are
// one CTA's work each.  The positions of the others are cut into `even` parts of
// share / 2^16 of a unit's steps and, where `tail`, a shorter last one.
struct BlockPlan {
  int mt, row_blocks;
  int units, whole;
  int even, tail, share;
  int items;                      // CTAs: whole units, even parts, last parts
  __host__ __device__ int parts() const { return even + tail; }
  __host__ __device__ int64_t slots() const { return parts() > 1 ? int64_t(units - whole) * parts() : 0; }      // records
};
BlockPlan plan_attn_blocks(int64_t rows, int batch, int kv_heads, int64_t capacity, int sms);
size_t attn_blocks_bytes(const BlockPlan& plan, int d);              // of records, where parts are joined
cudaError_t launch_attn_blocks(const AttnParams& p, const BlockPlan& plan, int d, int quant_group, int dev, float* records,
                               cudaStream_t s);

}  // namespace reskv
