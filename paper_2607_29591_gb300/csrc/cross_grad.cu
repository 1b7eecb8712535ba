// The gradient of cross attention on the fifth-generation tensor cores, in two kernels
// that each form the weights again; every sum has one owner and one order, so there are no
// atomics:
//
//   queries   a CTA has 128 rows (query tokens x heads of a KV head) and walks the states 128 at a time:
//             S = Q K^T, G = dO V^T (TMEM);  P = 2^(S - lse) over S, T = P (G - D) over G, in q's type;
//             B += P K, dQ += T K
//   states    a CTA has 128 states and walks the rows 128 at a time:
//             S^T = K Q^T, G^T = V dO^T;  P^T over S^T, T^T over G^T;  dV += P^T dO, dK += T^T Q
//
// D = <dO, O> with the O that was rounded to 16 bits is off by up to half a step of it, which
// in rows whose attention has a peak is much of G - D (a batch of 512 tokens over 577 states:
// dQ off by 8e-3 of itself, of which 2.3e-3 are the roundings of T and dQ).  As the P of a row sum up to
// 1, the row's sum of T is what D lacks: D + sum T goes to the second kernel, and dQ is corrected
// to T K - e P K.  There e sums T as rounded, so that the weights of the K sum up to 0 as those of the
// formula do: what all keys of a row have in common (they are akin to its query) stays out of
// dQ, and with it T's roundings (dQ 3.3e-3 off otherwise).  So a tile costs eight products; seven without that, five if dQ
// were summed with atomics.  Heads of a KV head are rows of one sum.  P and T are rounded to q's
// type (half a step of themselves; P times 2^12 in fp16, whose range ends at 2^-24), sums are fp32.
//
// Bound by the products: 4 x 2048 tokens of 32 heads over up to 4097 states (1.5 TFLOP in the eight products)
// 1.10 ms, 1.4 PFLOP/s; without exponentials, sums and roundings 1.0.  A tile's two pairs of products run while
// the weights of the other pair are formed; tensor memory (S, G and two sums) is full at d = 128.
//
// Weights are formed from the log-sum-exp that the forward pass left up to kFarSum.  A block of queries with a row
// past it first walks the sequence's states for the rows' own sums (S alone, every rank of a cluster all of
// them), and leaves them for the states' kernel: with queries 100 times as large 4 x 2048 tokens with their forward
// pass take 2.47 ms for 1.46, 8 x 512 over 577 states 192 us for 125.
//
// Where there are too few blocks for the SMs, a cluster of CTAs shares a block's tiles: each leaves its two
// sums in shared memory, where the cluster adds them up in order.
//
// Roles: warps 0-7 turn S and G into P and T, a row of TMEM a thread, half of its columns each; 8
// copies; 9 issues products; 10 puts zeros where a last tile's rows are no one's (a product sums
// over them, times 0, and they may be NaN); 11 (states) the rows' lse and D.
#include "cross.cuh"
#include "tensor_core.cuh"
#include "warp_mma.cuh"

namespace reskv {
namespace {

using namespace tc;

constexpr int kTile = 128;                        // rows and states of a tile
constexpr int kThreads = 384;
constexpr int kCopyWarp = 8, kIssueWarp = 9, kTailWarp = 10;
constexpr int kRegsSoftmax = 224, kRegsIssue = 56;
static_assert((2 * kRegsSoftmax + kRegsIssue) * 128 <= 168 * kThreads, "registers");
constexpr int kHalf = kTile * 128;                // bytes of 128 rows of 64 elements

struct GradParams {
  CrossParams a;
  CUtensorMap q, k, v, g;
  int32_t tile_tokens, cluster;
};

// 64 values in q's type over the first 32 of the 64 columns that they came from; `sum`: and their sum, as rounded
template <bool kF16>
__device__ __forceinline__ void store64(uint32_t at, const float (&x)[64], float2* sum = nullptr) {
  uint32_t w[32];
#pragma unroll
  for (int k = 0; k < 32; ++k) w[k] = pack_two<kF16>(x[2 * k], x[2 * k + 1]);
  store32(at, w);
  if (sum) {
#pragma unroll
    for (int k = 0; k < 32; ++k)
      *sum = fadd2(*sum, kF16 ? __half22float2(*reinterpret_cast<const __half2*>(&w[k])) : bf16x2_to_float2(w[k]));
  }
  stored();
}
// Columns [c0, c0 + n) of a thread's TMEM row, times f, to y in 16 bits.
template <bool kF16, int N>
__device__ __forceinline__ void store_columns(uint32_t at, float f, uint16_t* y, bool real) {
#pragma unroll 1
  for (int c = 0; c < N / 16; ++c) {
    float o[16];
    load16(at + 16 * c, o);
    landed();
    defined16(o);
    if (real) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack_two<kF16>(o[8 * k + 2 * e] * f, o[8 * k + 2 * e + 1] * f);
        reinterpret_cast<uint4*>(y)[2 * c + k] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
}
template <int N>
__device__ __forceinline__ void store_zeros(uint16_t* y) {
#pragma unroll 1
  for (int k = 0; k < N / 8; ++k) reinterpret_cast<uint4*>(y)[k] = make_uint4(0, 0, 0, 0);
}

// N columns from `at` of a thread's TMEM row into its row of fp32 in shared memory, from dim c0 on (word u of row r
// at u ^ r: rows on banks of their own).
template <int D, int N>
__device__ __forceinline__ void leave_columns(uint32_t at, float4* rows, int r, int c0) {
#pragma unroll 1
  for (int k0 = 0; k0 < N / 16; ++k0) {
    float o[16];
    load16(at + 16 * k0, o);
    landed();
    defined16(o);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      rows[r * (D / 4) + ((c0 / 4 + 4 * k0 + k) ^ (r & (D / 4 - 1)))] = make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
  }
}
// The ranks that have tiles, of `all`.
__device__ __forceinline__ uint32_t ranks_with_tiles(int cs, int all) {
  uint32_t present = 0;
  for (int k = 0; k < cs; ++k) present |= uint32_t(tiles_before(all, k + 1, cs) != tiles_before(all, k, cs)) << k;
  return present;
}
// Where rank k has dims 4u .. of row r.
template <int D>
__device__ __forceinline__ uint32_t row_of_rank(uint32_t rows, int r, int u, int k) {
  return of_rank(rows + uint32_t(r * (D / 4) + (u ^ (r & (D / 4 - 1)))) * 16, uint32_t(k));
}
template <bool kF16>
__device__ __forceinline__ uint2 pack_four(float4 a, float f) {
  return make_uint2(pack_two<kF16>(a.x * f, a.y * f), pack_two<kF16>(a.z * f, a.w * f));
}

// Zeros into rows [r0, r1) of a tile in shared memory (one warp).
template <int D>
__device__ __forceinline__ void clear_rows(uint8_t* tile, int r0, int r1, int lane) {
  const int words = (r1 - r0) * 8;
  for (int i = lane; i < words * (D / 64); i += 32) {
    const int x = i / words;
    *reinterpret_cast<uint4*>(tile + x * kHalf + r0 * 128 + (i - x * words) * 16) = make_uint4(0, 0, 0, 0);
  }
}

template <bool kF16>
__device__ __forceinline__ float dot8(uint4 a, uint4 b) {
  const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float2 u, v;
    if constexpr (kF16) {
      u = __half22float2(*reinterpret_cast<const __half2*>(&x[i]));
      v = __half22float2(*reinterpret_cast<const __half2*>(&y[i]));
    } else {
      u = bf16x2_to_float2(x[i]);
      v = bf16x2_to_float2(y[i]);
    }
    s = fmaf(u.x, v.x, fmaf(u.y, v.y, s));
  }
  return s;
}

// --- rows whose logits are large (RowShift) ---
// Few calls have any.  What they alone need is in functions of its own: within the kernels' loops, though
// not run, it cost the others 4 to 6 of 46 us (8 x 512 tokens over 577 states).

// Products s of a thread's row in TMEM, 64 columns, into what f makes their weights' exponents of.
__noinline__ __device__ void shift_row(uint32_t at, RowShift shift, float f) {
  const float inv = 1.f / f;
#pragma unroll 1
  for (int k0 = 0; k0 < 64; k0 += 16) {
    float x[16];
    load16(at + k0, x);
    landed();
    defined16(x);
#pragma unroll
    for (int k = 0; k < 16; ++k) x[k] = shift.exponent(x[k], f) * inv;
    store16(at + k0, x);
  }
  stored();
}
// The same where columns are the rows, with a shift each; a weight is 2^up at most, whatever the last
// digits of s are in the other order of its factors.
__noinline__ __device__ void shift_columns(uint32_t at, const float* hi, const float* lo, const float* less, float f, float up) {
  const float inv = 1.f / f;
#pragma unroll 1
  for (int k0 = 0; k0 < 64; k0 += 16) {
    float x[16];
    load16(at + k0, x);
    landed();
    defined16(x);
#pragma unroll
    for (int k = 0; k < 16; ++k) x[k] = min_nan(RowShift{hi[k0 + k], lo[k0 + k], less[k0 + k]}.exponent(x[k], f), up) * inv;
    store16(at + k0, x);
  }
  stored();
}

// --- queries -------------------------------------------------------------------

template <int D>
struct QuerySmem {
  static constexpr int tile = D / 64 * kHalf;
  static constexpr int slots = (224 * 1024 - 2 * tile) / tile > 8 ? 8 : (224 * 1024 - 2 * tile) / tile;
  static constexpr int at_g = tile, at_ring = 2 * tile;
  static constexpr int bytes = at_ring + slots * tile + 1024;
};
struct QueryShared {
  uint64_t q, full[8], empty[8], s, g, p, t, done, tail, mode;
  uint32_t tmem, abort, far;      // far: of any row; known once `mode` is complete
  float sums[2][kTile];           // D at the beginning, sums of T at the end
};

// The sums of a row's weights over its half of all tiles' columns, from tile `first` on: states left .. of them from
// tile 0 on.
__noinline__ __device__ FarSum far_sums(QueryShared& sh, uint32_t at, int first, int all, int left, float f, uint32_t* status) {
  FarSum sum;
#pragma unroll 1
  for (int i = 0; i < all; ++i) {
    const int tile = first + i < all ? first + i : first + i - all, upto = left - tile * kTile;
    sum.ok = role_wait(&sh.s, i & 1, &sh.abort, status);
    // (the G that came with the first S; its next comes after the last arrival below)
    if (sum.ok && i == 0) sum.ok = role_wait(&sh.g, 0, &sh.abort, status);
    if (!sum.ok) break;
    fence_after();
    float x[16], top = -INFINITY;
    auto sixteen = [&](int k0) {
      load16(at + k0, x);
      landed();
      defined16(x);
    };
#pragma unroll 1
    for (int k0 = 0; k0 < 64; k0 += 16) {
      sixteen(k0);
#pragma unroll
      for (int k = 0; k < 16; ++k)
        if (k0 + k < upto) top = fmaxf(top, f < 0.f ? -x[k] : x[k]);
    }
    sum.move(top, f);
#pragma unroll 1
    for (int k0 = 0; k0 < 64; k0 += 16) {
      sixteen(k0);
#pragma unroll
      for (int k = 0; k < 16; ++k)
        if (k0 + k < upto) sum.l += sum.weight(x[k], f);
    }
    fence_before();
    role_arrive(&sh.p);
  }
  return sum;
}

template <int D, bool kF16>
__global__ void __launch_bounds__(kThreads, 1) k_cross_grad_q(const __grid_constant__ GradParams gp) {
  using S = QuerySmem<D>;
  constexpr uint32_t kType = kF16 ? 0u : kBf16;
  constexpr uint32_t kLogits = shape_of(kTile) | kType, kSums = shape_of(D) | kType | kAcross;
  constexpr float kUp = kF16 ? 12.f : 0.f, kDown = kF16 ? 0x1p-12f : 1.f;          // of P
  const CrossParams& p = gp.a;
  extern __shared__ uint8_t dynamic[];
  uint8_t* smem = dynamic + ((1024u - (smem_u32(dynamic) & 1023u)) & 1023u);
  __shared__ __align__(16) QueryShared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    mbar_init(&sh.q, 1);
    for (int i = 0; i < S::slots; ++i) {
      mbar_init(&sh.full[i], 1);
      mbar_init(&sh.empty[i], 1);
    }
    mbar_init(&sh.s, 1);
    mbar_init(&sh.g, 1);
    mbar_init(&sh.p, 8);
    mbar_init(&sh.t, 8);
    mbar_init(&sh.done, 1);
    mbar_init(&sh.tail, 1);
    mbar_init(&sh.mode, 8);
    sh.abort = sh.far = 0;
    fence_mbar_init();
  }
  if (warp == kCopyWarp && elected()) {
    fetch_map(&gp.q);
    fetch_map(&gp.g);
    fetch_map(&gp.k);
    fetch_map(&gp.v);
  }
  const bool fixed = cross_fixed(p);
  if (!fixed) wait_for_previous();

  const int tt = gp.tile_tokens, cs = gp.cluster, rank = cs > 1 ? int(rank_in_cluster()) : 0;
  CrossBlock block;
  if (!cross_block(p, p.q_begin, p.q_each, p.n_tokens, tt, int(blockIdx.x) / cs, lane, block)) return;      // the whole cluster
  const int h = block.h, t0 = block.first, used_rows = tt * p.group;
  const CrossSequence sq = cross_sequence(p, block.b);
  const int all = ceil_div(sq.seen, kTile);
  const int first = tiles_before(all, rank, cs), n = tiles_before(all, rank + 1, cs) - first;      // tiles of states
  const int left = sq.seen - (first + n - 1) * kTile;                 // states of the last
  const bool cut = n > 0 && left < kTile;
  // a softmax thread's row, and its half of the columns
  const int c = warp >> 2, rt = (warp & 3) * 32 + lane, row_token = rt / p.group, token = t0 + row_token;
  const bool real = warp < 8 && row_token < tt && token < sq.count;
  const int head = h * p.group + rt - row_token * p.group;
  const int64_t at_token = sq.q0 + token;
  uint16_t* const dq = static_cast<uint16_t*>(p.d_q.data) + (real ? at_token * p.d_q.token + head * p.d_q.head + c * (D / 2) : 0);
  if (all == 0) {                                 // the same for the whole cluster
    if (fixed) wait_for_previous();
    if (real && rank == 0) store_zeros<D / 2>(dq);
    return;
  }
  if (warp == kIssueWarp) take_columns(smem_u32(&sh.tmem));
  if (fixed) wait_for_previous();
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = sh.tmem, smem_q = smem_u32(smem), smem_g = smem_q + S::at_g, ring = smem_q + S::at_ring;
  const uint32_t s_cols = tmem, g_cols = tmem + kTile, b_cols = tmem + 2 * kTile, o_cols = tmem + 3 * kTile;

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
    if (warp == kCopyWarp) {
      // --- copies: K0 V0 K1 V1 .. ---
      if (elected() && n > 0) {
        mbar_arrive_expect_tx(&sh.q, uint32_t(2 * (D / 64) * tt * p.group * 128));
        for (int x = 0; x < D / 64; ++x) {
          copy_box(smem_q + x * kHalf, &gp.q, 64 * x, h * p.group, sq.q0 + t0, &sh.q);
          copy_box(smem_g + x * kHalf, &gp.g, 64 * x, h * p.group, sq.q0 + t0, &sh.q);
        }
      }
      __syncwarp();
      int copied = 0;
      bool ok = true;
      auto copy = [&](int op, int tile, bool last) {
        const int slot = op % S::slots, turn = op / S::slots;
        if (turn > 0) ok = role_wait(&sh.empty[slot], (turn - 1) & 1, &sh.abort, p.status);
        if (!ok) return;
        if (elected()) {
          uint64_t* bar = last ? &sh.tail : &sh.full[slot];
          mbar_arrive_expect_tx(bar, S::tile);
#pragma unroll
          for (int x = 0; x < D / 64; ++x)
            copy_box(ring + slot * S::tile + x * kHalf, op & 1 ? &gp.v : &gp.k, 64 * x, h, sq.k0 + tile * kTile, bar);
        }
        __syncwarp();
        copied = op + 1;
      };
#pragma unroll 1
      for (int op = 0; op < 2 * n && ok; ++op) copy(op, first + op / 2, cut && op == 2 * n - 2);
      if (ok && n > 0) ok = role_wait(&sh.mode, 0, &sh.abort, p.status);
      if (ok && sh.far) {                         // the other ranks' tiles, then the own ones again
#pragma unroll 1
        for (int op = 2 * n; op < 2 * (all + n) && ok; ++op)
          copy(op, op < 2 * all ? (first + op / 2) % all : first + op / 2 - all, cut && op == 2 * (all + n) - 2);
      }
      if (!ok && lane == 0) {                     // a wait gave up: let what is in flight land
        mbar_wait_bounded(&sh.q, 0);
        for (int op = copied > S::slots ? copied - S::slots : 0; op < copied; ++op) {
          const bool again = op == 2 * (all + n) - 2, last = cut && (op == 2 * n - 2 || again);
          mbar_wait_bounded(last ? &sh.tail : &sh.full[op % S::slots], last ? again : (op / S::slots) & 1);
        }
      }
      __syncwarp();
    } else if (warp == kIssueWarp) {
      // --- products ---
      auto wait_tile = [&](int op) { return role_wait(&sh.full[op % S::slots], (op / S::slots) & 1, &sh.abort, p.status); };
      auto tile_of = [&](int op) { return ring + op % S::slots * S::tile; };
      auto outer = [&](uint32_t d, uint32_t a, uint32_t b, uint64_t* bar) {      // [128 x 128] = A B^T over D dims
        fence_after();
        if (elected()) {
          const uint32_t a0 = cluster_operand(a), b0 = cluster_operand(b);
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            multiply<kRows128, kLogits>(d, a0 + (((k / 4) * kHalf + (k & 3) * 32) >> 4), b0 + (((k / 4) * kHalf + (k & 3) * 32) >> 4),
                                        k > 0);
          commit(bar);
        }
        __syncwarp();
      };
      auto release = [&](int op) {
        if (elected()) commit(&sh.empty[op % S::slots]);
        __syncwarp();
      };
      auto add_to = [&](uint32_t d, uint32_t a, uint32_t b, bool add) {          // [128 x D] += A B over 128 states
        fence_after();
        if (elected()) {
          const uint32_t b0 = operand_across(b, kHalf);
#pragma unroll
          for (int k = 0; k < kTile / 16; ++k)
            multiply_from<kRows128, kSums>(d, step_of(a, k), b0 + ((k * 16 * 128) >> 4), add || k > 0);
        }
        __syncwarp();
      };
      bool ok = n > 0 && role_wait(&sh.q, 0, &sh.abort, p.status) && wait_tile(0);
      if (ok) {
        outer(s_cols, smem_q, tile_of(0), &sh.s);
        ok = wait_tile(1);
      }
      if (ok) {
        outer(g_cols, smem_g, tile_of(1), &sh.g);
        release(1);
        ok = role_wait(&sh.mode, 0, &sh.abort, p.status);
      }
      int s0 = 0;                                 // tiles whose logits went to the rows' sums
      if (ok && sh.far) {
        s0 = all;
        // S of every tile, then the own tiles' first products again
#pragma unroll 1
        for (int i = 0; i < all && ok; ++i) {
          ok = role_wait(&sh.p, i & 1, &sh.abort, p.status);       // the tile is read
          if (!ok) break;
          release(2 * i);
          ok = wait_tile(2 * i + 2);
          if (!ok) break;
          outer(s_cols, smem_q, tile_of(2 * i + 2), &sh.s);
          ok = wait_tile(2 * i + 3);
          if (!ok) break;
          if (i + 1 == all) outer(g_cols, smem_g, tile_of(2 * i + 3), &sh.g);
          release(2 * i + 3);
        }
      }
#pragma unroll 1
      for (int i = 0; i < n && ok; ++i) {
        const int op = 2 * (s0 + i);
        ok = role_wait(&sh.p, (s0 + i) & 1, &sh.abort, p.status);
        if (!ok) break;
        add_to(b_cols, s_cols, tile_of(op), i > 0);
        if (i + 1 < n) {
          ok = wait_tile(op + 2);
          if (!ok) break;
          outer(s_cols, smem_q, tile_of(op + 2), &sh.s);
        }
        ok = role_wait(&sh.t, i & 1, &sh.abort, p.status);
        if (!ok) break;
        add_to(o_cols, g_cols, tile_of(op), i > 0);
        release(op);
        if (i + 1 < n) {
          ok = wait_tile(op + 3);
          if (!ok) break;
          outer(g_cols, smem_g, tile_of(op + 3), &sh.g);
          release(op + 3);
        }
      }
      if (elected()) commit(&sh.done);
      __syncwarp();
      if (!ok) mbar_wait_bounded(&sh.done, 0);
    } else if (warp == kTailWarp && cut) {
      // --- behind the last state: P and T are zero there, keys may be anything ---
      auto clear = [&](int op, uint32_t parity) {
        const int slot = op % S::slots;
        if (!role_wait(&sh.tail, parity, &sh.abort, p.status)) return false;
        clear_rows<D>(smem + S::at_ring + slot * S::tile, left, kTile, lane);
        fence_proxy_async_smem();
        role_arrive(&sh.full[slot]);
        return true;
      };
      if (clear(2 * n - 2, 0) && role_wait(&sh.mode, 0, &sh.abort, p.status) && sh.far) clear(2 * (all + n) - 2, 1);
    }
    __syncwarp();
    meet(cs);                                     // the others have read what they read of tensor memory
    if (warp == kIssueWarp) {
      fence_after();
      give_columns(tmem);
    }
    if (cs > 1) meet(cs);
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    // --- weights ---
    const uint32_t lanes = uint32_t((warp & 3) * 32) << 16;
    // D: half of the row's dims each
    float delta = 0.f;
    const int64_t stat = at_token * p.heads + head;
    const float lse = real ? p.lse[stat] : 0.f;
    if (real) {
      const uint4* g = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.d_o.data) + at_token * p.d_o.token +
                                                      head * p.d_o.head + c * (D / 2));
      const uint4* o = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.o.data) + at_token * p.o.token +
                                                      head * p.o.head + c * (D / 2));
#pragma unroll
      for (int k = 0; k < D / 16; ++k) delta += dot8<kF16>(g[k], o[k]);
    }
    const bool far_row = far_sum(lse);
    if (__any_sync(0xffffffffu, far_row) && lane == 0) *static_cast<volatile uint32_t*>(&sh.far) = 1u;
    role_arrive(&sh.mode);
    sh.sums[c][rt] = delta;
    asm volatile("bar.sync 1, 256;" ::: "memory");
    delta = sh.sums[0][rt] + sh.sums[1][rt];
    const bool far = sh.far != 0;
    asm volatile("bar.sync 1, 256;" ::: "memory");      // (a rank without tiles comes to its next sums at once)
    auto both_halves = [&](float x) {
      sh.sums[c][rt] = x;
      asm volatile("bar.sync 1, 256;" ::: "memory");
      x = sh.sums[0][rt] + sh.sums[1][rt];
      asm volatile("bar.sync 1, 256;" ::: "memory");
      return x;
    };
    const float f = p.scale2, down = -delta * kDown;
    RowShift shift{log2_sum(lse, kUp), 0.f, 0.f};
    float2 more = make_float2(0.f, 0.f), rounded = more;      // sums of T
    bool ok = true;
    if (far && n > 0) {
      // the rows' sums, over all tiles of the sequence (each rank for itself)
      FarSum sum = far_sums(sh, s_cols + lanes + 64 * c, first, all, sq.seen - 64 * c, f, p.status);
      ok = sum.ok;
      // both halves of the row
      sh.sums[c][rt] = sum.top;
      asm volatile("bar.sync 1, 256;" ::: "memory");
      const float top = fmaxf(sh.sums[0][rt], sh.sums[1][rt]);
      asm volatile("bar.sync 1, 256;" ::: "memory");
      sum.move(top, f);
      const float l = both_halves(sum.l);
      if (far_row) shift = RowShift{sum.hi, sum.lo, log2f(l) - kUp};
    }
    const int s0 = far ? all : 0, g0 = far ? 1 : 0;       // phases that are over
    const float lse2 = far ? 0.f : shift.hi;
#pragma unroll 1
    for (int i = 0; i < n && ok; ++i) {
      const int upto = (i == n - 1 ? left : kTile) - 64 * c;
      ok = role_wait(&sh.s, (s0 + i) & 1, &sh.abort, p.status);
      if (!ok) break;
      fence_after();
      if (far) shift_row(s_cols + lanes + 64 * c, shift, f);
      float x[64];
      load64(s_cols + lanes + 64 * c, x);
      landed64(x);
#pragma unroll
      for (int k = 0; k < 64; k += 2) {
        const float2 e = ffma2(make_float2(x[k], x[k + 1]), make_float2(f, f), make_float2(-lse2, -lse2));
        x[k] = exp2_fast(e.x);
        x[k + 1] = exp2_fast(e.y);
      }
      if (upto < 64) {
#pragma unroll
        for (int k = 0; k < 64; ++k)
          if (k >= upto) x[k] = 0.f;
      }
      store64<kF16>(s_cols + lanes + 64 * c, x);
      fence_before();
      role_arrive(&sh.p);
      ok = role_wait(&sh.g, (g0 + i) & 1, &sh.abort, p.status);
      if (!ok) break;
      fence_after();
      float y[64];
      load64(g_cols + lanes + 64 * c, y);
      landed64(y);
#pragma unroll
      for (int k = 0; k < 64; k += 2) {
        const float2 t = fmul2(make_float2(x[k], x[k + 1]),
                               ffma2(make_float2(y[k], y[k + 1]), make_float2(kDown, kDown), make_float2(down, down)));
        y[k] = t.x;
        y[k + 1] = t.y;
      }
      if (upto < 64) {
#pragma unroll
        for (int k = 0; k < 64; ++k)
          if (k >= upto) y[k] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < 64; k += 2) more = fadd2(more, make_float2(y[k], y[k + 1]));
      store64<kF16>(g_cols + lanes + 64 * c, y, &rounded);
      fence_before();
      role_arrive(&sh.t);
    }
    if (ok && n > 0) ok = role_wait(&sh.done, 0, &sh.abort, p.status);
    const float lacks = both_halves(more.x + more.y), e = both_halves(rounded.x + rounded.y);
    if (rank == cs - 1 && real && c == 0) p.stats[stat] = make_float4(shift.hi, shift.lo, shift.less, delta + lacks);
    if (cs > 1) {
      // for the join: all products are done, operands' memory is free
      fence_after();
      float4* rows = reinterpret_cast<float4*>(smem);
      if (n > 0) {
        leave_columns<D, D / 2>(o_cols + lanes + c * (D / 2), rows, rt, c * (D / 2));
        leave_columns<D, D / 2>(b_cols + lanes + c * (D / 2), rows + kTile * (D / 4), rt, c * (D / 2));
      }
      if (c == 0) reinterpret_cast<float4*>(smem + 2 * kTile * D * 4)[rt] = make_float4(rank == cs - 1 ? delta : 0.f, lacks, e, 0.f);
    } else if (ok) {
      fence_after();
      const float back = -e * kDown;
#pragma unroll 1
      for (int m = 0; m < D / 32; ++m) {
        float a[16], b[16];
        load16(o_cols + lanes + c * (D / 2) + 16 * m, a);
        load16(b_cols + lanes + c * (D / 2) + 16 * m, b);
        landed();
        defined16(a);
        defined16(b);
#pragma unroll
        for (int k = 0; k < 16; ++k) a[k] = fmaf(back, b[k], a[k]) * p.scale;
        if (real) {
#pragma unroll
          for (int k = 0; k < 2; ++k)
            reinterpret_cast<uint4*>(dq)[2 * m + k] =
                make_uint4(pack_two<kF16>(a[8 * k], a[8 * k + 1]), pack_two<kF16>(a[8 * k + 2], a[8 * k + 3]),
                           pack_two<kF16>(a[8 * k + 4], a[8 * k + 5]), pack_two<kF16>(a[8 * k + 6], a[8 * k + 7]));
        }
      }
    }
    __syncwarp();
    fence_before();
    meet(cs);
    if (cs == 1) return;
    // --- the join: rows dealt to the cluster's warps ---
    const uint32_t present = ranks_with_tiles(cs, all);
    auto one = [](int, int) { return 1.f; };
#pragma unroll 1
    for (int r = 2 * (rank * 8 + warp); r < used_rows; r += 2 * cs * 8) {       // two rows at a time
      if (t0 + r / p.group >= sq.count) break;
      const int u = lane < D / 4 ? lane : 0;
      // D, sum T and sum T as rounded: of all ranks the last two
      float4 s[2], a[4];
      add_sources(s, cs, (1u << cs) - 1u, [&](int m, int k) { return of_rank(smem_q + 2 * kTile * D * 4 + uint32_t(r + m) * 16, uint32_t(k)); }, one);
      add_sources(a, cs, present, [&](int m, int k) { return row_of_rank<D>(smem_q + (m & 1) * kTile * D * 4, r + m / 2, u, k); }, one);
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const int tk = t0 + (r + m) / p.group, hd = h * p.group + (r + m) % p.group;
        if (r + m >= used_rows || tk >= sq.count) continue;
        const float back = -s[m].z * kDown;
        const float4 x = a[2 * m], y = a[2 * m + 1];
        const int64_t tok = sq.q0 + tk;
        if (lane < D / 4)
          reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.d_q.data) + tok * p.d_q.token + hd * p.d_q.head)[u] = pack_four<kF16>(
              make_float4(fmaf(back, y.x, x.x), fmaf(back, y.y, x.y), fmaf(back, y.z, x.z), fmaf(back, y.w, x.w)), p.scale);
        if (lane == 0) p.stats[tok * p.heads + hd].w = s[m].x + s[m].y;
      }
      __syncwarp();
    }
    __syncwarp();
    meet(cs);                                     // nobody leaves while its sums are read
  }
}

// --- states --------------------------------------------------------------------

constexpr int kStages = 2;
template <int D>
struct StateSmem {
  static constexpr int tile = D / 64 * kHalf;
  static constexpr int at_v = tile, at_ring = 2 * tile;               // a stage: Q, then dO
  static constexpr int bytes = at_ring + kStages * 2 * tile + 1024;
};
struct StateShared {
  uint64_t kv, full[kStages], empty[kStages], s, g, p, t, done, tail;
  uint32_t tmem, abort;
  uint32_t far[kStages];          // of any row of the tile
  alignas(16) float lse2[kStages][kTile], hi[kStages][kTile], lo[kStages][kTile], less[kStages][kTile], delta[kStages][kTile];
};

template <int D, bool kF16>
__global__ void __launch_bounds__(kThreads, 1) k_cross_grad_kv(const __grid_constant__ GradParams gp) {
  using S = StateSmem<D>;
  constexpr uint32_t kType = kF16 ? 0u : kBf16;
  constexpr uint32_t kLogits = shape_of(kTile) | kType, kSums = shape_of(D) | kType | kAcross;
  constexpr float kUp = kF16 ? 12.f : 0.f, kDown = kF16 ? 0x1p-12f : 1.f;          // of P
  const CrossParams& p = gp.a;
  extern __shared__ uint8_t dynamic[];
  uint8_t* smem = dynamic + ((1024u - (smem_u32(dynamic) & 1023u)) & 1023u);
  __shared__ __align__(16) StateShared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    mbar_init(&sh.kv, 1);
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&sh.full[i], 2);
      mbar_init(&sh.empty[i], 1);
    }
    mbar_init(&sh.s, 1);
    mbar_init(&sh.g, 1);
    mbar_init(&sh.p, 8);
    mbar_init(&sh.t, 8);
    mbar_init(&sh.done, 1);
    mbar_init(&sh.tail, 1);
    sh.abort = 0;
    fence_mbar_init();
  }
  if (warp == kCopyWarp && elected()) {
    fetch_map(&gp.q);
    fetch_map(&gp.g);
    fetch_map(&gp.k);
    fetch_map(&gp.v);
  }
  const bool fixed = cross_fixed(p);
  if (!fixed) wait_for_previous();

  const int cs = gp.cluster, rank = cs > 1 ? int(rank_in_cluster()) : 0;
  CrossBlock block;
  if (!cross_block(p, p.kv_begin, p.kv_each, p.n_rows, kTile, int(blockIdx.x) / cs, lane, block)) return;    // the whole cluster
  const int h = block.h, j0 = block.first;
  const CrossSequence sq = cross_sequence(p, block.b);
  const int tt = gp.tile_tokens, used = tt * p.group;                 // rows of a full tile
  const int all = j0 < sq.seen ? ceil_div(sq.count, tt) : 0;
  const int first = tiles_before(all, rank, cs), n = tiles_before(all, rank + 1, cs) - first;      // tiles of rows
  const int left = min((sq.count - (first + n - 1) * tt) * p.group, used);      // rows of the last
  const bool cut = n > 0 && left < used;
  // a softmax thread's state; warps 0-3 write dV, 4-7 dK
  const int c = warp >> 2, rt = (warp & 3) * 32 + lane, j = j0 + rt;
  const bool owned = warp < 8 && j < sq.rows;
  const CrossRows& to = c ? p.d_k : p.d_v;
  uint16_t* const out = static_cast<uint16_t*>(to.data) + (owned ? (sq.k0 + j) * to.token + h * to.head : 0);
  if (all == 0) {                                 // nobody sees them: the same for the whole cluster
    if (fixed) wait_for_previous();
    if (owned && rank == 0) store_zeros<D>(out);
    return;
  }
  if (warp == kIssueWarp) take_columns(smem_u32(&sh.tmem));
  if (fixed) wait_for_previous();
  if (used < kTile && warp < 2 * kStages) {       // rows that no copy writes
    clear_rows<D>(smem + S::at_ring + warp * S::tile, used, kTile, lane);
    fence_proxy_async_smem();
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = sh.tmem, smem_k = smem_u32(smem), smem_v = smem_k + S::at_v, ring = smem_k + S::at_ring;
  const uint32_t s_cols = tmem, g_cols = tmem + kTile, v_cols = tmem + 2 * kTile, k_cols = tmem + 3 * kTile;

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
    if (warp == kCopyWarp) {
      // --- copies ---
      if (elected() && n > 0) {
        mbar_arrive_expect_tx(&sh.kv, 2 * S::tile);
        for (int x = 0; x < D / 64; ++x) {
          copy_box(smem_k + x * kHalf, &gp.k, 64 * x, h, sq.k0 + j0, &sh.kv);
          copy_box(smem_v + x * kHalf, &gp.v, 64 * x, h, sq.k0 + j0, &sh.kv);
        }
      }
      __syncwarp();
      int copied = 0;
      bool ok = true;
#pragma unroll 1
      for (int i = 0; i < n && ok; ++i) {
        const int stage = i % kStages;
        if (i >= kStages) ok = role_wait(&sh.empty[stage], (i / kStages - 1) & 1, &sh.abort, p.status);
        if (!ok) break;
        if (elected()) {
          uint64_t* bar = cut && i == n - 1 ? &sh.tail : &sh.full[stage];
          mbar_arrive_expect_tx(bar, uint32_t(2 * (D / 64) * used * 128));
          const uint32_t dst = ring + stage * 2 * S::tile;
#pragma unroll
          for (int x = 0; x < D / 64; ++x) {
            copy_box(dst + x * kHalf, &gp.q, 64 * x, h * p.group, sq.q0 + (first + i) * tt, bar);
            copy_box(dst + S::tile + x * kHalf, &gp.g, 64 * x, h * p.group, sq.q0 + (first + i) * tt, bar);
          }
        }
        __syncwarp();
        copied = i + 1;
      }
      if (!ok && lane == 0) {                     // a wait gave up: let what is in flight land
        mbar_wait_bounded(&sh.kv, 0);
        for (int i = copied > kStages ? copied - kStages : 0; i < copied; ++i) {
          const bool last = cut && i == n - 1;
          mbar_wait_bounded(last ? &sh.tail : &sh.full[i % kStages], last ? 0 : (i / kStages) & 1);
        }
      }
      __syncwarp();
    } else if (warp == kIssueWarp) {
      // --- products ---
      auto wait_tile = [&](int i) { return role_wait(&sh.full[i % kStages], (i / kStages) & 1, &sh.abort, p.status); };
      auto outer = [&](uint32_t d, uint32_t a, uint32_t b, uint64_t* bar) {      // [128 x 128] = A B^T over D dims
        fence_after();
        if (elected()) {
          const uint32_t a0 = cluster_operand(a), b0 = cluster_operand(b);
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            multiply<kRows128, kLogits>(d, a0 + (((k / 4) * kHalf + (k & 3) * 32) >> 4), b0 + (((k / 4) * kHalf + (k & 3) * 32) >> 4),
                                        k > 0);
          commit(bar);
        }
        __syncwarp();
      };
      auto add_to = [&](uint32_t d, uint32_t a, uint32_t b, bool add) {          // [128 x D] += A B over 128 rows
        fence_after();
        if (elected()) {
          const uint32_t b0 = operand_across(b, kHalf);
#pragma unroll
          for (int k = 0; k < kTile / 16; ++k)
            multiply_from<kRows128, kSums>(d, step_of(a, k), b0 + ((k * 16 * 128) >> 4), add || k > 0);
        }
        __syncwarp();
      };
      auto q_tile = [&](int i) { return ring + i % kStages * 2 * S::tile; };
      bool ok = n > 0 && role_wait(&sh.kv, 0, &sh.abort, p.status) && wait_tile(0);
      if (ok) {
        outer(s_cols, smem_k, q_tile(0), &sh.s);
        outer(g_cols, smem_v, q_tile(0) + S::tile, &sh.g);
      }
#pragma unroll 1
      for (int i = 0; i < n && ok; ++i) {
        ok = role_wait(&sh.p, i & 1, &sh.abort, p.status);
        if (!ok) break;
        add_to(v_cols, s_cols, q_tile(i) + S::tile, i > 0);
        if (i + 1 < n) {
          ok = wait_tile(i + 1);
          if (!ok) break;
          outer(s_cols, smem_k, q_tile(i + 1), &sh.s);
        }
        ok = role_wait(&sh.t, i & 1, &sh.abort, p.status);
        if (!ok) break;
        add_to(k_cols, g_cols, q_tile(i), i > 0);
        if (elected()) commit(&sh.empty[i % kStages]);
        __syncwarp();
        if (i + 1 < n) outer(g_cols, smem_v, q_tile(i + 1) + S::tile, &sh.g);
      }
      if (elected()) commit(&sh.done);
      __syncwarp();
      if (!ok) mbar_wait_bounded(&sh.done, 0);
    } else if (warp == kTailWarp) {
      // --- the last tile's rows that are another sequence's ---
      if (cut && role_wait(&sh.tail, 0, &sh.abort, p.status)) {
        const int stage = (n - 1) % kStages;
        uint8_t* tile = smem + S::at_ring + stage * 2 * S::tile;
        clear_rows<D>(tile, left, used, lane);
        clear_rows<D>(tile + S::tile, left, used, lane);
        fence_proxy_async_smem();
        role_arrive(&sh.full[stage]);
      }
    } else {
      // --- the rows' sums and D ---
      bool ok = true;
#pragma unroll 1
      for (int i = 0; i < n && ok; ++i) {
        const int stage = i % kStages;
        float4 v[4];
        bool far = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = lane + 32 * k, tk = (first + i) * tt + r / p.group;
          const bool here = r < used && tk < sq.count;
          v[k] = here ? p.stats[int64_t(sq.q0 + tk) * p.heads + h * p.group + r % p.group] : make_float4(0.f, 0.f, 0.f, 0.f);
          far |= v[k].y != 0.f || v[k].z != 0.f;
        }
        far = __any_sync(0xffffffffu, far);
        if (i >= kStages) ok = role_wait(&sh.empty[stage], (i / kStages - 1) & 1, &sh.abort, p.status);
        if (!ok) break;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          sh.lse2[stage][lane + 32 * k] = far ? 0.f : v[k].x;
          if (far) {
            sh.hi[stage][lane + 32 * k] = v[k].x;
            sh.lo[stage][lane + 32 * k] = v[k].y;
            sh.less[stage][lane + 32 * k] = v[k].z;
          }
          sh.delta[stage][lane + 32 * k] = v[k].w * kDown;
        }
        if (lane == 0) sh.far[stage] = far;
        role_arrive(&sh.full[stage]);
      }
    }
    __syncwarp();
    meet(cs);                                     // the others have read what they read of tensor memory
    if (warp == kIssueWarp) {
      fence_after();
      give_columns(tmem);
    }
    if (cs > 1) meet(cs);
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    // --- weights: rows 64 c .. 64 c + 63 of a tile ---
    const uint32_t lanes = uint32_t((warp & 3) * 32) << 16;
    const float f = p.scale2;
    bool ok = true;
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      const int stage = i % kStages, upto = (i == n - 1 ? left : used) - 64 * c;
      // (the tile's barrier also has its sums behind it)
      ok = role_wait(&sh.full[stage], (i / kStages) & 1, &sh.abort, p.status);
      const bool far = sh.far[stage] != 0;
      ok = ok && role_wait(&sh.s, i & 1, &sh.abort, p.status);
      if (!ok) break;
      fence_after();
      if (far) shift_columns(s_cols + lanes + 64 * c, &sh.hi[stage][64 * c], &sh.lo[stage][64 * c], &sh.less[stage][64 * c], f, kUp);
      float x[64];
      load64(s_cols + lanes + 64 * c, x);
      landed64(x);
      const float4* l4 = reinterpret_cast<const float4*>(&sh.lse2[stage][64 * c]);
      const float4* e4 = reinterpret_cast<const float4*>(&sh.delta[stage][64 * c]);
#pragma unroll
      for (int k = 0; k < 64; k += 4) {
        const float4 l = l4[k / 4];
        const float2 u = ffma2(make_float2(x[k], x[k + 1]), make_float2(f, f), make_float2(-l.x, -l.y));
        const float2 v = ffma2(make_float2(x[k + 2], x[k + 3]), make_float2(f, f), make_float2(-l.z, -l.w));
        x[k] = exp2_fast(u.x);
        x[k + 1] = exp2_fast(u.y);
        x[k + 2] = exp2_fast(v.x);
        x[k + 3] = exp2_fast(v.y);
      }
      if (upto < 64) {
#pragma unroll
        for (int k = 0; k < 64; ++k)
          if (k >= upto) x[k] = 0.f;
      }
      store64<kF16>(s_cols + lanes + 64 * c, x);
      fence_before();
      role_arrive(&sh.p);
      ok = role_wait(&sh.g, i & 1, &sh.abort, p.status);
      if (!ok) break;
      fence_after();
      float y[64];
      load64(g_cols + lanes + 64 * c, y);
      landed64(y);
#pragma unroll
      for (int k = 0; k < 64; k += 4) {
        const float4 e = e4[k / 4];
        const float2 u = fmul2(make_float2(x[k], x[k + 1]),
                               ffma2(make_float2(y[k], y[k + 1]), make_float2(kDown, kDown), make_float2(-e.x, -e.y)));
        const float2 v = fmul2(make_float2(x[k + 2], x[k + 3]),
                               ffma2(make_float2(y[k + 2], y[k + 3]), make_float2(kDown, kDown), make_float2(-e.z, -e.w)));
        y[k] = u.x;
        y[k + 1] = u.y;
        y[k + 2] = v.x;
        y[k + 3] = v.y;
      }
      if (upto < 64) {
#pragma unroll
        for (int k = 0; k < 64; ++k)
          if (k >= upto) y[k] = 0.f;
      }
      store64<kF16>(g_cols + lanes + 64 * c, y);
      fence_before();
      role_arrive(&sh.t);
    }
    if (ok && n > 0) ok = role_wait(&sh.done, 0, &sh.abort, p.status);
    if (cs > 1) {
      // for the join: all products are done, operands' memory is free
      asm volatile("bar.sync 1, 256;" ::: "memory");
      fence_after();
      if (n > 0) leave_columns<D, D>((c ? k_cols : v_cols) + lanes, reinterpret_cast<float4*>(smem) + c * kTile * (D / 4), rt, 0);
    } else if (ok) {
      fence_after();
      const bool seen = owned && j < sq.seen;
      store_columns<kF16, D>((c ? k_cols : v_cols) + lanes, c ? p.scale : kDown, out, seen);
      if (owned && !seen) store_zeros<D>(out);
    }
    __syncwarp();
    fence_before();
    meet(cs);
    if (cs == 1) return;
    // --- the join ---
    const uint32_t present = ranks_with_tiles(cs, all);
#pragma unroll 1
    for (int r = 2 * (rank * 8 + warp); r < kTile; r += 2 * cs * 8) {           // two rows of both at a time
      if (j0 + r >= sq.rows) break;
      const int u = lane < D / 4 ? lane : 0;
      float4 a[4];
      add_sources(a, cs, present, [&](int m, int k) { return row_of_rank<D>(smem_k + (m & 1) * kTile * D * 4, r + m / 2, u, k); },
                  [](int, int) { return 1.f; });
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const int row = j0 + r + m / 2;
        if (row >= sq.rows || lane >= D / 4) continue;
        const CrossRows& y = m & 1 ? p.d_k : p.d_v;
        reinterpret_cast<uint2*>(static_cast<uint16_t*>(y.data) + (sq.k0 + row) * y.token + h * y.head)[u] =
            row < sq.seen ? pack_four<kF16>(a[m], m & 1 ? p.scale : kDown) : make_uint2(0u, 0u);
      }
      __syncwarp();
    }
    __syncwarp();
    meet(cs);                                     // nobody leaves while its sums are read
  }
}


template <int D, bool kF16>
cudaError_t both(const GradParams& gp, int dev, cudaStream_t s) {
  static std::atomic<uint64_t> raised_q{0}, raised_kv{0};
  const CrossParams& p = gp.a;
  cudaError_t err = raise_shared(k_cross_grad_q<D, kF16>, raised_q, QuerySmem<D>::bytes, dev);
  if (err == cudaSuccess) err = raise_shared(k_cross_grad_kv<D, kF16>, raised_kv, StateSmem<D>::bytes, dev);
  static SideBySide kept_q{}, kept_kv{};
  const int64_t rows = (p.n_tokens / p.batch + gp.tile_tokens - 1) / gp.tile_tokens, states = (p.n_rows / p.batch + kTile - 1) / kTile;
  const int64_t units = int64_t(p.batch) * p.kv_heads;                // (tiles of them: on average)
  GradParams l = gp;
  if (err == cudaSuccess) {
    l.cluster = cluster_for(k_cross_grad_q<D, kF16>, kept_q, (rows > 0 ? rows : 1) * units, states, kThreads, QuerySmem<D>::bytes, dev);
    err = launch_clusters(k_cross_grad_q<D, kF16>, cross_blocks(p, p.q_begin, p.n_tokens, gp.tile_tokens), l.cluster, kThreads,
                          QuerySmem<D>::bytes, s, l);
  }
  if (err == cudaSuccess) {
    l.cluster = cluster_for(k_cross_grad_kv<D, kF16>, kept_kv, (states > 0 ? states : 1) * units, rows, kThreads, StateSmem<D>::bytes, dev);
    err = launch_clusters(k_cross_grad_kv<D, kF16>, cross_blocks(p, p.kv_begin, p.n_rows, kTile), l.cluster, kThreads,
                          StateSmem<D>::bytes, s, l);
  }
  return err;
}

}  // namespace

cudaError_t launch_cross_grad(const CrossParams& p, const CrossMaps& maps, int d, int dev, cudaStream_t s) {
  GradParams gp{};
  gp.a = p;
  gp.q = maps.q;
  gp.k = maps.k;
  gp.v = maps.v;
  gp.g = maps.d_o;
  gp.tile_tokens = cross_tile_tokens(p.group);
  if (d == 128) return p.f16 ? both<128, true>(gp, dev, s) : both<128, false>(gp, dev, s);
  return p.f16 ? both<64, true>(gp, dev, s) : both<64, false>(gp, dev, s);
}

}  // namespace reskv
