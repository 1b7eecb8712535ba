// Cross attention of few query rows (a decode step's tokens, or beams, against an encoder's
// states): every state is read once for eight or sixteen rows (query tokens x heads of a KV head), so
// the kernel is bound by reading them.
//
// A cluster of CTAs shares the states of one KV head of a sequence.  Copies of 64 states land in a CTA's
// ring; each of its four warps takes 16 of them:
//
//   S^T [16 states x 8 rows] = K Q^T        mma.sync: eight rows would leave the fifth generation's
//   O^T [dims x 8 rows] += V^T P^T          128 idle; K and V come as fragments by ldmatrix
//
// The weights go into the second product in two planes (bf16: 16 bits, fp16: 22).  Warps leave
// their rows in shared memory, where the cluster's warps join them, a row each, in order.
//
// Three stages of 32 KB (d = 128; two CTAs an SM) keep some 190 KB of an SM's under way: 32 tokens over up
// to 6400 states of 8 KV heads (534 MB) 90 us, 5.9 TB/s, what is left being the sequences' unequal lengths (64
// of 2000: 80 us, 6.6 TB/s).  One token over 1500 states 6.4 us, a chain of launch, copies, two products and
// the join.
#include "cross.cuh"
#include "tensor_core.cuh"
#include "warp_mma.cuh"

namespace reskv {
namespace {

using namespace tc;

constexpr int kWarps = 4;                         // computing; one more copies
constexpr int kThreads = (kWarps + 1) * 32;
constexpr float kNoReference = -3.0e38f;

struct RowsParams {
  CrossParams a;
  CUtensorMap k, v;
  int32_t cluster;
};

template <int D, int NB>
struct RowsSmem {
  static constexpr int half = kRowStates * 128;   // 64 dims of a tile
  static constexpr int tile = D / 64 * half;
  static constexpr int stages = D == 128 ? 3 : 4;
  static constexpr int at_ref = kWarps * 8 * NB * D * 4;              // behind the rows to be joined, over the drained ring
  static constexpr int bytes = stages * 2 * tile + 1024;
  static_assert(at_ref + 2 * kWarps * 8 * NB * 4 <= stages * 2 * tile, "rows to be joined");
};
template <int kStages>
struct RowsShared {
  uint64_t full[kStages], vacant[kStages];
  uint32_t abort;
};

template <bool kTrans>
__device__ __forceinline__ void fragment(uint32_t (&a)[4], uint32_t at) {
  if constexpr (kTrans)
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]) : "r"(at) : "memory");
  else
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]) : "r"(at) : "memory");
}
template <bool kF16>
__device__ __forceinline__ void multiply_add(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (kF16) mma_f16(d, a[0], a[1], a[2], a[3], b0, b1);
  else mma_bf16(d, a[0], a[1], a[2], a[3], b0, b1);
}
// what pack_two left over
template <bool kF16>
__device__ __forceinline__ uint32_t rest_two(float lo, float hi, uint32_t packed) {
  if constexpr (kF16) return rest_f16(lo, hi, packed);
  const float2 f = bf16x2_to_float2(packed);
  return pack_bf16(lo - f.x, hi - f.y);
}

template <int D, bool kF16, int NB>
__global__ void __launch_bounds__(kThreads) k_cross_rows(const __grid_constant__ RowsParams rp) {
  using S = RowsSmem<D, NB>;
  constexpr int kRows = 8 * NB;
  const CrossParams& p = rp.a;
  extern __shared__ uint8_t dynamic[];
  uint8_t* smem = dynamic + ((1024u - (smem_u32(dynamic) & 1023u)) & 1023u);
  __shared__ __align__(16) RowsShared<S::stages> sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int cs = rp.cluster, rank = cs > 1 ? int(rank_in_cluster()) : 0;
  if (tid == 0) {
    for (int i = 0; i < S::stages; ++i) {
      mbar_init(&sh.full[i], 1);
      mbar_init(&sh.vacant[i], kWarps);
    }
    sh.abort = 0;
    fence_mbar_init();
  }
  if (warp == kWarps && elected()) {
    fetch_map(&rp.k);
    fetch_map(&rp.v);
  }
  __syncthreads();
  const bool fixed = cross_fixed(p);
  if (!fixed) wait_for_previous();
  CrossBlock block;
  if (!cross_block(p, p.q_begin, p.q_each, p.n_tokens, kRows, int(blockIdx.x) / cs, lane, block, p.group)) return;      // the whole cluster
  const int h = block.h, r0 = block.first;
  const CrossSequence sq = cross_sequence(p, block.b);
  const int rows = min(sq.count * p.group - r0, kRows);               // of this block
  const int all = ceil_div(sq.seen, kRowStates);
  const int first = tiles_before(all, rank, cs), n = tiles_before(all, rank + 1, cs) - first;
  const uint32_t ring = smem_u32(smem);
  if (fixed) wait_for_previous();

  if (warp == kWarps) {
    // --- copies ---
    int copied = 0;
    bool ok = true;
#pragma unroll 1
    for (int i = 0; i < n && ok; ++i) {
      const int st = i % S::stages;
      if (i >= S::stages) ok = role_wait(&sh.vacant[st], (i / S::stages - 1) & 1, &sh.abort, p.status);
      if (!ok) break;
      if (elected()) {
        mbar_arrive_expect_tx(&sh.full[st], 2 * S::tile);
        const int row = sq.k0 + (first + i) * kRowStates;
#pragma unroll
        for (int x = 0; x < D / 64; ++x) {
          copy_box(ring + st * 2 * S::tile + x * S::half, &rp.k, 64 * x, h, row, &sh.full[st]);
          copy_box(ring + st * 2 * S::tile + S::tile + x * S::half, &rp.v, 64 * x, h, row, &sh.full[st]);
        }
      }
      __syncwarp();
      copied = i + 1;
    }
    if (!ok && lane == 0)                         // a wait gave up: let what is in flight land
      for (int i = copied > S::stages ? copied - S::stages : 0; i < copied; ++i)
        mbar_wait_bounded(&sh.full[i % S::stages], (i / S::stages) & 1);
    __syncwarp();
  }
  const int g = lane >> 2, t = lane & 3;
  float o[NB][D / 16][4], ref[NB][2], l[NB][2];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      ref[b][j] = kNoReference;
      l[b][j] = 0.f;
    }
#pragma unroll
    for (int m = 0; m < D / 16; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[b][m][i] = 0.f;
  }
  bool ok = true;
  if (warp < kWarps) {
    // the query operand: column g (row r0 + 8 b + g), terms 2t, 2t + 1 and those + 8 of each 16 dims
    uint32_t q[NB][D / 16][2];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int r = r0 + 8 * b + g;
      const bool here = 8 * b + g < rows;
      const uint16_t* src = static_cast<const uint16_t*>(p.q.data) +
                            (here ? (sq.q0 + r / p.group) * p.q.token + int64_t(h * p.group + r % p.group) * p.q.head : 0);
#pragma unroll
      for (int m = 0; m < D / 16; ++m)
#pragma unroll
        for (int i = 0; i < 2; ++i) q[b][m][i] = here ? *reinterpret_cast<const uint32_t*>(src + 16 * m + 8 * i + 2 * t) : 0u;
    }
    const float f = p.scale2;
    // this lane's rows of a warp's 16 states: of K by lane & 15, of V by its place among 4 x 8
    const int k_row = warp * 16 + (lane & 15), k_word = lane >> 4;
    const int v_row = warp * 16 + (lane & 7) + (lane >> 4) * 8, v_word = (lane >> 3) & 1;
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      const int st = i % S::stages;
      ok = role_wait(&sh.full[st], (i / S::stages) & 1, &sh.abort, p.status);
      if (!ok) break;
      const uint32_t kt = ring + st * 2 * S::tile + k_row * 128, vt = ring + st * 2 * S::tile + S::tile + v_row * 128;
      const int left = sq.seen - (first + i) * kRowStates - warp * 16;      // of the warp's states, those that count
      if (left > 0) {
        float s[NB][4];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int j = 0; j < 4; ++j) s[b][j] = 0.f;
#pragma unroll
        for (int m = 0; m < D / 16; ++m) {
          uint32_t a[4];
          fragment<false>(a, kt + (m >> 2) * S::half + (((2 * (m & 3) + k_word) ^ (k_row & 7)) << 4));
#pragma unroll
          for (int b = 0; b < NB; ++b) multiply_add<kF16>(s[b], a, q[b][m][0], q[b][m][1]);
        }
        uint32_t w[NB][2], w2[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          float x[4];
          auto weights = [&]() {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float r = ref[b][j & 1];
              x[j] = exp2_fast(fabsf(r) > kFarLogits ? __fsub_rn(__fmul_rn(s[b][j], f), r) : fmaf(s[b][j], f, -r));
              if (left < 16 && g + (j >> 1) * 8 >= left) x[j] = 0.f;
            }
          };
          weights();
          if (__any_sync(0xffffffffu, !(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) <= 16384.f))) {
            // the reference 6 below the largest logit
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float top = -INFINITY;
#pragma unroll
              for (int k = 0; k < 2; ++k)
                if (g + k * 8 < left) top = fmaxf(top, __fmul_rn(s[b][2 * k + j], f));
#pragma unroll
              for (int e = 4; e < 32; e *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, e));
              const float now = fmaxf(ref[b][j], top - 6.f), keep = exp2f(ref[b][j] - now);
              ref[b][j] = now;
              l[b][j] *= keep;
#pragma unroll
              for (int m = 0; m < D / 16; ++m) {
                o[b][m][j] *= keep;
                o[b][m][2 + j] *= keep;
              }
            }
            weights();
          }
          l[b][0] += x[0] + x[2];
          l[b][1] += x[1] + x[3];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t hi = pack_two<kF16>(x[2 * k], x[2 * k + 1]);
            w[b][k] = transpose8x8(hi);
            w2[b][k] = transpose8x8(rest_two<kF16>(x[2 * k], x[2 * k + 1], hi));
          }
        }
#pragma unroll
        for (int m = 0; m < D / 16; ++m) {
          uint32_t a[4];
          fragment<true>(a, vt + (m >> 2) * S::half + (((2 * (m & 3) + v_word) ^ (v_row & 7)) << 4));
          if (left < 16) {                        // values that nobody sees may be anything
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int s0 = 2 * t + 8 * k;
              const uint32_t mask = s0 + 1 < left ? 0xffffffffu : s0 < left ? 0xffffu : 0u;
              a[2 * k] &= mask;
              a[2 * k + 1] &= mask;
            }
          }
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            multiply_add<kF16>(o[b][m], a, w[b][0], w[b][1]);
            multiply_add<kF16>(o[b][m], a, w2[b][0], w2[b][1]);
          }
        }
      }
      role_arrive(&sh.vacant[st]);
    }
  }
  __syncthreads();                                // the ring is drained
  float* const refs = reinterpret_cast<float*>(smem + S::at_ref);
  if (warp < kWarps) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int e = 4; e < 32; e *= 2) l[b][j] += __shfl_xor_sync(0xffffffffu, l[b][j], e);
        const int r = 8 * b + 2 * t + j;
        float* row = reinterpret_cast<float*>(smem) + (warp * kRows + r) * D;
#pragma unroll
        for (int m = 0; m < D / 16; ++m) {        // (turned by 8 r, so that rows lie on banks of their own)
          row[(16 * m + g + 8 * r) & (D - 1)] = o[b][m][j];
          row[(16 * m + 8 + g + 8 * r) & (D - 1)] = o[b][m][2 + j];
        }
        if (g == 0) {
          const bool seen = ok && (ref[b][j] != kNoReference || l[b][j] != 0.f);
          refs[warp * kRows + r] = seen ? ref[b][j] : -INFINITY;
          refs[(kWarps + warp) * kRows + r] = l[b][j];
        }
      }
  }
  __syncthreads();
  if (cs > 1) sync_cluster();
  // --- the join: a row a warp, lane i the records of source i: warp i % 4 of rank i / 4 ---
  if (warp < kWarps) {
#pragma unroll 1
    for (int r = rank * kWarps + warp; r < rows; r += cs * kWarps) {
      const int sources = cs * kWarps;
      float rf = -INFINITY, sum = 0.f;
      if (lane < sources) {
        const uint32_t at = ring + S::at_ref + uint32_t((lane % kWarps) * kRows + r) * 4, from = uint32_t(lane / kWarps);
        rf = read_cluster(of_rank(at, from));
        sum = read_cluster(of_rank(at + kWarps * kRows * 4, from));
      }
      float top = rf;
#pragma unroll
      for (int e = 16; e; e /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, e));
      const float wt = rf == -INFINITY ? 0.f : exp2f(rf - top);
      float total = rf == -INFINITY ? 0.f : wt * sum;
#pragma unroll
      for (int e = 16; e; e /= 2) total += __shfl_xor_sync(0xffffffffu, total, e);
      const uint32_t present = __ballot_sync(0xffffffffu, rf != -INFINITY);
      const int u = lane < D / 4 ? lane : 0;
      float4 sums[1];
      add_sources(
          sums, sources, present,
          [&](int, int i) {
            return of_rank(ring + uint32_t(((i % kWarps) * kRows + r) * D + ((4 * u + 8 * r) & (D - 1))) * 4, uint32_t(i / kWarps));
          },
          [&](int, int i) { return __shfl_sync(0xffffffffu, wt, i); });
      const float4 a = sums[0];
      const float inv = present ? 1.f / total : 0.f;
      const int64_t tok = sq.q0 + (r0 + r) / p.group;
      const int hd = h * p.group + (r0 + r) % p.group;
      if (lane < D / 4)
        reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.o.data) + tok * p.o.token + hd * p.o.head)[u] =
            make_uint2(pack_two<kF16>(a.x * inv, a.y * inv), pack_two<kF16>(a.z * inv, a.w * inv));
      const float lse = present ? (top + log2f(total)) * 0.693147180559945f : -INFINITY;
      if (lane == 0 && p.lse) p.lse[tok * p.heads + hd] = lse;
      __syncwarp();
    }
  }
  __syncthreads();
  if (cs > 1) sync_cluster();                     // nobody leaves while its rows are read
}

template <int D, bool kF16, int NB>
cudaError_t launch(const RowsParams& rp, int dev, int sms, cudaStream_t s) {
  static std::atomic<uint64_t> raised{0};
  const cudaError_t err = raise_shared(k_cross_rows<D, kF16, NB>, raised, RowsSmem<D, NB>::bytes, dev);
  if (err != cudaSuccess) return err;
  const CrossParams& p = rp.a;
  const int64_t items = cross_blocks(p, p.q_begin, p.n_tokens, 8 * NB, p.group);
  // about as many as there are: with q_begin there may be one more a sequence
  const int64_t rows = p.n_tokens / p.batch * p.group, sure = ((rows + 8 * NB - 1) / (8 * NB) + (rows == 0)) * p.batch * p.kv_heads;
  const int64_t tiles = (p.n_rows / p.batch + kRowStates - 1) / kRowStates;
  // As many CTAs as SMs at least; what a CTA takes beside its states (some 6 us) makes more of them
  // slower: 16 x 16 heads of 64, 5 beams over 1500 states 19 us by one CTA a head, 25 by 4, 42 by 8; 64 heads
  // over 3000 states, 16 rows each, 26 by 2, 24 by 4, 33 by 8; 32 heads over 8192 28 by 8.
  RowsParams l = rp;
  l.cluster = 1;
  while (l.cluster < 8 && sure * l.cluster < sms && l.cluster * 2 <= tiles) l.cluster *= 2;
  return launch_clusters(k_cross_rows<D, kF16, NB>, items, l.cluster, kThreads, RowsSmem<D, NB>::bytes, s, l);
}

template <int D, bool kF16>
cudaError_t dispatch(const RowsParams& rp, int dev, int sms, cudaStream_t s) {
  return rp.a.n_tokens * rp.a.group <= 8 * int64_t(rp.a.batch) ? launch<D, kF16, 1>(rp, dev, sms, s)
                                                               : launch<D, kF16, 2>(rp, dev, sms, s);
}

}  // namespace

cudaError_t launch_cross_rows(const CrossParams& p, const CrossMaps& maps, int d, int dev, int sms, cudaStream_t s) {
  RowsParams rp{};
  rp.a = p;
  rp.k = maps.k;
  rp.v = maps.v;
  if (d == 128) return p.f16 ? dispatch<128, true>(rp, dev, sms, s) : dispatch<128, false>(rp, dev, sms, s);
  return p.f16 ? dispatch<64, true>(rp, dev, sms, s) : dispatch<64, false>(rp, dev, sms, s);
}

}  // namespace reskv
