// Cross attention of many query rows (a prompt against an encoder's states) on the
// fifth-generation tensor cores.
//
// A row is a query token and head of a KV head; a tile is 128 rows (as many whole tokens as
// fit).  A CTA takes two tiles and walks the states 128 at a time:
//
//   S = Q K^T       [128 rows x 128 states]  both operands in shared memory, into TMEM
//   P = 2^(S - ref) half a row a thread, in the type of q, over S in TMEM
//   O += P V        [128 rows x d]           P from TMEM, V as it lies (across), into TMEM
//
// Copies, products and the softmax (eight warps a tile, two threads a row) are roles of their own; while one
// tile's softmax runs, the tensor cores work for the other.  Where a sequence has one tile's rows
// only, the CTA's two streams take the even and the odd tiles of states (kSplit).  Where
// there are too few blocks for the SMs, a cluster of CTAs shares a block's states.  Streams and
// CTAs leave their rows in shared memory and are joined over the cluster, in order.
//
//   q             queries have landed
//   full[op]      a tile of K or V has landed                (copies -> products)
//   empty[op]     its products are done                      (products -> copies)
//   s[m]          S of stream m is there, and the O before   (products -> softmax)
//   p[m]          P is in place                              (softmax -> products)
//   tail          the last V has landed, behind its last state anything: a warp puts zeros there
//                 and passes it on as full[op]
//
// The reference of a row moves only when a weight passes 2^13; it then lies 6 below the largest logit.
//
// Bound by the exponentials between two products of a stream, then by the products: 8 x 1024 tokens of 32 heads
// over 4096 states, 8 KV heads of 128 (550 GFLOP) 450 us, 1.22 PFLOP/s; without any exponential, and
// without the two threads' barrier, 365, which is what the products alone take in these tiles.  (P keeps both streams from a second S: the sums of 256 rows
// and two S fill the tensor memory.)  Weights before their largest logit, 16 at a time in the shadow of the
// other half's loads, spilled: 546.
#include "cross.cuh"
#include "tensor_core.cuh"
#include "warp_mma.cuh"

namespace reskv {
namespace {

using namespace tc;

constexpr int kStates = 128;                      // of a tile
constexpr int kThreads = 640;                     // warps 0-7, 8-15 softmax, 16 copies, 17 products, 18 the tail
constexpr int kSoftmaxWarps = 16, kCopyWarp = 16, kIssueWarp = 17, kTailWarp = 18;
constexpr int kRegsSoftmax = 104, kRegsIssue = 56;
static_assert((4 * kRegsSoftmax + kRegsIssue) * 128 <= 96 * kThreads, "registers");
constexpr float kNoReference = -3.0e38f;

struct BlocksParams {
  CrossParams a;
  CUtensorMap q, k, v;
  int32_t tile_tokens;            // whole tokens of a tile
  int32_t cluster;
};

template <int D, bool kSplit>
struct BlocksSmem {
  static constexpr int half = 128 * 128;          // 128 rows of 64 elements
  static constexpr int tile = D / 64 * half;
  static constexpr int q = (kSplit ? 1 : 2) * tile;
  static constexpr int slots = (224 * 1024 - q) / tile > 8 ? 8 : (224 * 1024 - q) / tile;
  static constexpr int bytes = q + slots * tile + 1024;               // on a boundary of 1024
  static constexpr int at_ref = 2 * 128 * D * 4;  // of rows to be joined: outputs, then references and sums
  static_assert(at_ref + 3 * 256 * 4 <= q + slots * tile, "rows to be joined");
};

struct BlocksShared {
  uint64_t q, full[8], empty[8], s[2], p[2], done, tail;
  uint32_t tmem, abort;
  float half[2][128];             // of a row's second half, for the first and back
};
static_assert(BlocksSmem<64, false>::bytes + sizeof(BlocksShared) + 16 <= 227 * 1024 && BlocksSmem<64, true>::bytes + sizeof(BlocksShared) + 16 <= 227 * 1024 &&
                  BlocksSmem<128, false>::bytes + sizeof(BlocksShared) + 16 <= 227 * 1024 && BlocksSmem<128, true>::bytes + sizeof(BlocksShared) + 16 <= 227 * 1024,
              "shared memory");
// A barrier of two warps, and one's share of it where it goes no further.
__device__ __forceinline__ void pair_sync(int id) { asm volatile("barrier.cta.sync %0, 64;" ::"r"(id) : "memory"); }
__device__ __forceinline__ void pair_leave(int id) { asm volatile("barrier.cta.arrive %0, 64;" ::"r"(id) : "memory"); }


template <int D, bool kF16, bool kSplit>
__global__ void __launch_bounds__(kThreads, 1) k_cross_blocks(const __grid_constant__ BlocksParams bp) {
  using S = BlocksSmem<D, kSplit>;
  constexpr uint32_t kType = kF16 ? 0u : kBf16;
  constexpr uint32_t kLogits = shape_of(kStates) | kType, kOutputs = shape_of(D) | kType | kAcross;
  const CrossParams& p = bp.a;
  extern __shared__ uint8_t dynamic[];
  uint8_t* smem = dynamic + ((1024u - (smem_u32(dynamic) & 1023u)) & 1023u);
  __shared__ __align__(16) BlocksShared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int cs = bp.cluster, rank = cs > 1 ? int(rank_in_cluster()) : 0;

  if (tid == 0) {
    mbar_init(&sh.q, 1);
    for (int i = 0; i < S::slots; ++i) {
      mbar_init(&sh.full[i], 1);
      mbar_init(&sh.empty[i], 1);
    }
    for (int m = 0; m < 2; ++m) {
      mbar_init(&sh.s[m], 1);
      mbar_init(&sh.p[m], 8);
    }
    mbar_init(&sh.done, 1);
    mbar_init(&sh.tail, 1);
    sh.abort = 0;
    fence_mbar_init();
  }
  if (warp == kCopyWarp && elected()) {
    fetch_map(&bp.q);
    fetch_map(&bp.k);
    fetch_map(&bp.v);
  }
  const bool fixed = cross_fixed(p);
  if (!fixed) wait_for_previous();

  // the block: tokens t0 .. of sequence b, KV head h
  const int tt = bp.tile_tokens, block_tokens = (kSplit ? 1 : 2) * tt;
  CrossBlock block;
  if (!cross_block(p, p.q_begin, p.q_each, p.n_tokens, block_tokens, int(blockIdx.x) / cs, lane, block)) return;      // the whole cluster
  const int b = block.b, h = block.h, t0 = block.first;
  const CrossSequence sq = cross_sequence(p, b);
  const bool two = !kSplit && t0 + tt < sq.count, joins = kSplit || cs > 1;
  const int all = ceil_div(sq.seen, kStates);
  const int first = tiles_before(all, rank, cs), n = tiles_before(all, rank + 1, cs) - first;      // tiles of states
  const int steps[2] = {kSplit ? (n + 1) / 2 : n, kSplit ? n / 2 : two ? n : 0};
  const int left = sq.seen - (first + n - 1) * kStates;               // states of the last tile
  const bool cut = n > 0 && left < kStates;

  // a softmax thread's row and half
  const int m = (warp >> 3) & 1, c = (warp >> 2) & 1, rt = (warp & 3) * 32 + lane;
  const int row_token = rt / p.group, token = t0 + (kSplit ? 0 : m * tt) + row_token;
  const bool real = warp < kSoftmaxWarps && row_token < tt && token < sq.count;
  const int head = h * p.group + rt - row_token * p.group;
  if (sq.seen == 0) {                             // the same for the whole cluster
    if (fixed) wait_for_previous();
    if (real && rank == 0 && (m == 0 || !kSplit)) {
      uint16_t* y = static_cast<uint16_t*>(p.o.data) + (sq.q0 + token) * p.o.token + head * p.o.head + c * (D / 2);
#pragma unroll 1
      for (int i = 0; i < D / 16; ++i) reinterpret_cast<uint4*>(y)[i] = make_uint4(0, 0, 0, 0);
      if (p.lse && c == 0) p.lse[int64_t(sq.q0 + token) * p.heads + head] = -INFINITY;
    }
    return;
  }
  if (warp == kIssueWarp) take_columns(smem_u32(&sh.tmem));
  if (fixed) wait_for_previous();
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = sh.tmem, smem_q = smem_u32(smem), ring = smem_q + S::q;
  auto s_cols = [&](int s) { return tmem + uint32_t(s * kStates); };
  auto o_cols = [&](int s) { return tmem + uint32_t(2 * kStates + s * D); };
  // Tiles come in the order of their first use: K0 V0 K1 V1 .., or split K0 K1 V0 K2 V1 ..
  auto k_op = [&](int t) { return kSplit ? (t == 0 ? 0 : 2 * t - 1) : 2 * t; };
  auto v_op = [&](int t) { return kSplit ? (t + 1 < n ? 2 * t + 2 : 2 * t + 1) : 2 * t + 1; };

  if (warp >= kSoftmaxWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
    if (warp == kCopyWarp) {
      // --- copies ---
      int copied = 0;
      bool ok = true;
      if (elected() && n > 0) {
        const int halves = D / 64, tiles = kSplit || !two ? 1 : 2;
        mbar_arrive_expect_tx(&sh.q, uint32_t(tiles * halves * tt * p.group * 128));
        for (int i = 0; i < tiles; ++i)
          for (int x = 0; x < halves; ++x)
            copy_box(smem_q + i * S::tile + x * S::half, &bp.q, 64 * x, h * p.group, sq.q0 + t0 + i * tt, &sh.q);
      }
      __syncwarp();
#pragma unroll 1
      for (int op = 0; op < 2 * n && ok; ++op) {
        const int slot = op % S::slots, turn = op / S::slots;
        if (turn > 0) ok = role_wait(&sh.empty[slot], (turn - 1) & 1, &sh.abort, p.status);
        if (!ok) break;
        const bool values = kSplit ? (op > 0 && (op == 2 * n - 1 || (op & 1) == 0)) : (op & 1);
        const int t = !kSplit ? op / 2 : op == 0 ? 0 : op == 2 * n - 1 ? n - 1 : values ? op / 2 - 1 : (op + 1) / 2;
        if (elected()) {
          uint64_t* bar = cut && values && t == n - 1 ? &sh.tail : &sh.full[slot];
          mbar_arrive_expect_tx(bar, S::tile);
#pragma unroll
          for (int x = 0; x < D / 64; ++x)
            copy_box(ring + slot * S::tile + x * S::half, values ? &bp.v : &bp.k, 64 * x, h, sq.k0 + (first + t) * kStates, bar);
        }
        __syncwarp();
        copied = op + 1;
      }
      if (!ok && lane == 0) {                     // a wait gave up: let what is in flight land
        mbar_wait_bounded(&sh.q, 0);
        for (int op = copied > S::slots ? copied - S::slots : 0; op < copied; ++op)
          mbar_wait_bounded(cut && op == v_op(n - 1) ? &sh.tail : &sh.full[op % S::slots],
                            cut && op == v_op(n - 1) ? 0 : (op / S::slots) & 1);
      }
      __syncwarp();
    } else if (warp == kIssueWarp) {
      // --- products ---
      auto wait_tile = [&](int op) { return role_wait(&sh.full[op % S::slots], (op / S::slots) & 1, &sh.abort, p.status); };
      auto release = [&](int op) {
        if (elected()) commit(&sh.empty[op % S::slots]);
        __syncwarp();
      };
      const uint32_t logits = kLogits | (p.scale2 < 0.f ? kNegative : 0u);
      auto issue_s = [&](int s, int op) {
        fence_after();
        if (elected()) {
          const uint32_t q0 = cluster_operand(smem_q + (kSplit ? 0 : s) * S::tile), k0 = cluster_operand(ring + op % S::slots * S::tile);
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            multiply<kRows128>(s_cols(s), q0 + (((k / 4) * S::half + (k & 3) * 32) >> 4),
                               k0 + (((k / 4) * S::half + (k & 3) * 32) >> 4), logits, k > 0);
          commit(&sh.s[s]);
        }
        __syncwarp();
      };
      auto issue_o = [&](int s, int op, bool add) {
        fence_after();
        if (elected()) {
          const uint32_t v0 = operand_across(ring + op % S::slots * S::tile, S::half);
#pragma unroll
          for (int k = 0; k < kStates / 16; ++k)
            multiply_from<kRows128, kOutputs>(o_cols(s), step_of(s_cols(s), k), v0 + ((k * 16 * 128) >> 4), add || k > 0);
        }
        __syncwarp();
      };
      bool ok = n == 0 || role_wait(&sh.q, 0, &sh.abort, p.status);
      // the first logits of both streams
      for (int s = 0; s < 2 && ok; ++s) {
        if (steps[s] == 0) continue;
        const int op = k_op(kSplit ? s : 0);
        if (kSplit || s == 0) ok = wait_tile(op);
        if (!ok) break;
        issue_s(s, op);
        if (kSplit || s == 1 || !two) release(op);
      }
#pragma unroll 1
      for (int i = 0; i < steps[0] && ok; ++i) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          if (i >= steps[s] || !ok) continue;
          const int t = kSplit ? 2 * i + s : i, next = kSplit ? t + 2 : t + 1;
          const bool last_use = kSplit || s == 1 || !two;
          if (kSplit || s == 0) ok = wait_tile(v_op(t));
          if (ok) ok = role_wait(&sh.p[s], i & 1, &sh.abort, p.status);
          if (!ok) break;
          issue_o(s, v_op(t), i > 0);
          if (last_use) release(v_op(t));
          if (next < n) {
            if (kSplit || s == 0) ok = wait_tile(k_op(next));
            if (!ok) break;
            issue_s(s, k_op(next));
            if (last_use) release(k_op(next));
          }
        }
      }
      // all products: also where a wait gave up, which the softmax does not see then
      if (elected()) commit(&sh.done);
      __syncwarp();
      if (!ok) mbar_wait_bounded(&sh.done, 0);
    } else if (warp == kTailWarp && cut) {
      // --- what lies behind the last state: weights are zero there, values may be anything ---
      const int slot = v_op(n - 1) % S::slots;
      if (role_wait(&sh.tail, 0, &sh.abort, p.status)) {
        for (int i = lane; i < (kStates - left) * 8 * (D / 64); i += 32) {
          const int x = i / ((kStates - left) * 8), r = i - x * (kStates - left) * 8;
          *reinterpret_cast<uint4*>(smem + S::q + slot * S::tile + x * S::half + left * 128 + r * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
        role_arrive(&sh.full[slot]);
      }
    }
    __syncwarp();
    meet(cs);                                     // the softmax has read what it reads of tensor memory
    if (warp == kIssueWarp) {
      fence_after();
      give_columns(tmem);
    }
    if (joins) meet(cs);
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    // --- the softmax, half a row a thread: states 64 c .. 64 c + 63 of a tile.  Both threads of a row look
    // for its largest logit in all of it and so agree on it; they meet before P goes over S, which both
    // have looked through.  8 x 1024 tokens over 4096 states, us: with one thread a row, whose 128
    // exponentials a tile waits for, 523 (without any exponential 365); with half a row each that exchange
    // their largest logits at a barrier 478; so 450 (465 with an mbarrier for each warp's reading) ---
    const uint32_t lanes = uint32_t((warp & 3) * 32) << 16;
    const int mine = steps[m], pair = 1 + 4 * m + (warp & 3);
    const float f = fabsf(p.scale2);              // (a negative scale is the product's: S = -Q K^T)
    float ref = kNoReference, l = 0.f;
    bool ok = true, far = false;                  // far: logits of any row of the warp
#pragma unroll 1
    for (int i = 0; i < mine; ++i) {
      ok = role_wait(&sh.s[m], i & 1, &sh.abort, p.status);
      if (!ok) break;
      fence_after();
      const int t = kSplit ? 2 * i + m : i;
      const int states = t == n - 1 ? left : kStates, upto = states - 64 * c;
      float x[64], top = -INFINITY;
      {
        // the other half, for its largest logit alone
        const uint32_t at = s_cols(m) + lanes + 64 * (1 - c);
        const int other = states - 64 * (1 - c);
        load64(at, x);
        landed64(x);
        if (other < 64) {
#pragma unroll
          for (int k = 0; k < 64; ++k)
            if (k >= other) x[k] = -INFINITY;
        }
#pragma unroll
        for (int k = 0; k < 64; k += 2) asm("max.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(x[k]), "f"(x[k + 1]));
      }
      load64(s_cols(m) + lanes + 64 * c, x);
      landed64(x);
      if (upto < 64) {
#pragma unroll
        for (int k = 0; k < 64; ++k)
          if (k >= upto) x[k] = -INFINITY;
      }
#pragma unroll
      for (int k = 0; k < 64; k += 2) asm("max.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(x[k]), "f"(x[k + 1]));
      if (!real) top = -INFINITY;                   // a row of another sequence, or of nothing, moves no reference
      float keep = 1.f;
      float2 s2[4] = {};
      if (__any_sync(0xffffffffu, (far ? __fsub_rn(__fmul_rn(top, f), ref) : fmaf(top, f, -ref)) > 13.f)) {
        // the reference 6 below the row's largest (the same rows, and what becomes of them, in both warps)
        const float now = fmaxf(ref, __fmul_rn(top, f) - 6.f);
        keep = exp2f(ref - now);
        ref = now;
        far = __any_sync(0xffffffffu, fabsf(ref) > kFarLogits && ref != kNoReference);
      }
      if (far) {
#pragma unroll
        for (int k = 0; k < 64; ++k) x[k] = __fsub_rn(__fmul_rn(x[k], f), ref);
      } else {
#pragma unroll
        for (int k = 0; k < 64; k += 2) {
          const float2 y = ffma2(make_float2(x[k], x[k + 1]), make_float2(f, f), make_float2(-ref, -ref));
          x[k] = y.x;
          x[k + 1] = y.y;
        }
      }
#pragma unroll
      for (int k = 0; k < 64; k += 2) {
        x[k] = exp2_fast(x[k]);
        x[k + 1] = exp2_fast(x[k + 1]);
        s2[(k / 2) & 3] = fadd2(s2[(k / 2) & 3], make_float2(x[k], x[k + 1]));
      }
      s2[0] = fadd2(fadd2(s2[0], s2[1]), fadd2(s2[2], s2[3]));
      const float sum = s2[0].x + s2[0].y;
      l = l * keep + sum;
      if (i > 0 && __any_sync(0xffffffffu, keep != 1.f)) {       // (S's barrier has the products before it behind it)
#pragma unroll 1
        for (int k0 = 0; k0 < D / 32; ++k0) {
          float v[16];
          load16(o_cols(m) + lanes + c * (D / 2) + 16 * k0, v);
          landed();
          defined16(v);
#pragma unroll
          for (int k = 0; k < 16; ++k) v[k] *= keep;
          store16(o_cols(m) + lanes + c * (D / 2) + 16 * k0, v);
        }
      }
      uint32_t w[32];
#pragma unroll
      for (int k = 0; k < 32; ++k) w[k] = pack_two<kF16>(x[2 * k], x[2 * k + 1]);
      // (both warps of the rows have read S: what one puts P over was the other's to look through, too)
      fence_before();
      pair_sync(pair);
      fence_after();
      store32(s_cols(m) + lanes + 64 * c, w);
      stored();
      fence_before();
      role_arrive(&sh.p[m]);
    }
    if (!ok) pair_leave(pair);                    // a wait gave up: the other warp may be at the barrier of a tile
    if (ok && mine > 0) ok = role_wait(&sh.done, 0, &sh.abort, p.status);
    fence_after();
    const bool seen = mine > 0 && ok;
    // the row's sum, of both halves
    if (c == 1) sh.half[m][rt] = l;
    asm volatile("bar.sync 9, 512;" ::: "memory");
    if (c == 0) {
      l += sh.half[m][rt];
      sh.half[m][rt] = l;
    }
    asm volatile("bar.sync 9, 512;" ::: "memory");
    l = sh.half[m][rt];
    if (cs == 1 && !kSplit) {
      const float inv = l != 0.f ? 1.f / l : 0.f;         // (0: every logit is -inf)
      if (seen) {
        uint16_t* y = static_cast<uint16_t*>(p.o.data) + (sq.q0 + token) * p.o.token + head * p.o.head + c * (D / 2);
#pragma unroll 1
        for (int k0 = 0; k0 < D / 32; ++k0) {
          float o[16];
          load16(o_cols(m) + lanes + c * (D / 2) + 16 * k0, o);
          landed();
          defined16(o);
          if (real) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              uint32_t w[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) w[e] = pack_two<kF16>(o[8 * k + 2 * e] * inv, o[8 * k + 2 * e + 1] * inv);
              reinterpret_cast<uint4*>(y)[2 * k0 + k] = make_uint4(w[0], w[1], w[2], w[3]);
            }
          }
        }
        if (real && p.lse && c == 0)
          p.lse[int64_t(sq.q0 + token) * p.heads + head] = l != 0.f ? (ref + log2f(l)) * 0.693147180559945f : -INFINITY;
      }
    } else {
      // for the join: all products are done, operands' memory is free (word u of row r at u ^ r)
      asm volatile("bar.sync 9, 512;" ::: "memory");
      float4* rows = reinterpret_cast<float4*>(smem) + (m * 128 + rt) * (D / 4);
      if (seen) {
#pragma unroll 1
        for (int k0 = 0; k0 < D / 32; ++k0) {
          float o[16];
          load16(o_cols(m) + lanes + c * (D / 2) + 16 * k0, o);
          landed();
          defined16(o);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            rows[(c * (D / 8) + 4 * k0 + k) ^ (rt & (D / 4 - 1))] = make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
        }
      }
      float* refs = reinterpret_cast<float*>(smem + S::at_ref);
      if (c == 0) {
        refs[m * 128 + rt] = seen ? ref : -INFINITY;
        refs[256 + m * 128 + rt] = seen ? l : 0.f;
      }
    }
    __syncwarp();
    fence_before();
    meet(cs);
    if (!joins) return;
    // --- the join: rows dealt to the ranks in runs, sources (streams of all ranks) in order ---
    constexpr int kSources = kSplit ? 2 : 1;
    const int rows = kSplit || !two ? 128 : 256, sources = cs * kSources, share = rows / cs, row0 = rank * share;
    const uint32_t at_ref = smem_q + S::at_ref;
    float* const weight = reinterpret_cast<float*>(smem + S::at_ref + 2 * 256 * 4);      // [share][sources], < 0: no states
    auto place = [&](int i, int r) { return uint32_t((kSplit ? i & 1 : r >> 7) * 128 + (r & 127)); };      // of source i's row r
    auto token_of = [&](int r) { return (r & 127) / p.group < tt ? t0 + (r >> 7) * tt + (r & 127) / p.group : sq.count; };
    // each source of each row a thread: at most 256; a row's side by side
    if (tid < share * sources) {
      const int q = tid / sources, i = tid - q * sources, r = row0 + q;
      const uint32_t at = place(i, r) * 4, from = uint32_t(i / kSources);
      const float ref = read_cluster(of_rank(at_ref + at, from)), sum = read_cluster(of_rank(at_ref + 256 * 4 + at, from));
      const uint32_t group = __activemask();        // whole warps
      float top = ref;
      for (int o = 1; o < sources; o *= 2) top = fmaxf(top, __shfl_xor_sync(group, top, o));
      const float w = ref == -INFINITY ? 0.f : exp2f(ref - top);
      float total = ref == -INFINITY ? 0.f : w * sum;
      for (int o = 1; o < sources; o *= 2) total += __shfl_xor_sync(group, total, o);
      weight[tid] = ref == -INFINITY ? -1.f : total != 0.f ? w / total : 0.f;
      const int tok = token_of(r);
      if (i == 0 && p.lse && tok < sq.count)
        p.lse[int64_t(sq.q0 + tok) * p.heads + h * p.group + (r & 127) % p.group] = total != 0.f ? (top + log2f(total)) * 0.693147180559945f : -INFINITY;
    }
    asm volatile("bar.sync 9, 512;" ::: "memory");
    // then a row a warp, four rows at a time
#pragma unroll 1
    for (int q = warp * 4; q < share; q += kSoftmaxWarps * 4) {
      const int u = lane < D / 4 ? lane : 0;
      auto w_of = [&](int m, int i) { return weight[(q + m) * sources + i]; };
      float4 a[4];
      uint32_t present = 0;                         // (of all rows alike)
      for (int i = 0; i < sources; ++i) present |= uint32_t(!(w_of(0, i) < 0.f)) << i;
      add_sources(
          a, sources, present,
          [&](int m, int i) {
            const int r = row0 + q + m;
            return of_rank(smem_q + (place(i, r) * (D / 4) + uint32_t(u ^ (r & (D / 4 - 1)))) * 16, uint32_t(i / kSources));
          },
          w_of);
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const int r = row0 + q + m, tok = token_of(r), hd = h * p.group + (r & 127) % p.group;
        if (tok < sq.count && lane < D / 4)
          reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.o.data) + (sq.q0 + tok) * p.o.token + hd * p.o.head)[u] =
              make_uint2(pack_two<kF16>(a[m].x, a[m].y), pack_two<kF16>(a[m].z, a[m].w));
      }
    }
    __syncwarp();
    meet(cs);                                     // nobody leaves while its rows are read
  }
}

template <int D, bool kF16, bool kSplit>
cudaError_t launch(const BlocksParams& bp, int64_t items, int64_t sure, int64_t tiles, int dev, cudaStream_t s) {
  static std::atomic<uint64_t> raised{0};
  const cudaError_t err = raise_shared(k_cross_blocks<D, kF16, kSplit>, raised, BlocksSmem<D, kSplit>::bytes, dev);
  if (err != cudaSuccess) return err;
  // (16 blocks of 32 tiles: 28 us by clusters of 4, 41 of 8, of which 16 do not run side by side, 63 alone)
  static SideBySide kept{};
  BlocksParams l = bp;
  l.cluster = cluster_for(k_cross_blocks<D, kF16, kSplit>, kept, sure, tiles, kThreads, BlocksSmem<D, kSplit>::bytes, dev);
  return launch_clusters(k_cross_blocks<D, kF16, kSplit>, items, l.cluster, kThreads, BlocksSmem<D, kSplit>::bytes, s, l);
}

}  // namespace

cudaError_t launch_cross_blocks(const CrossParams& p, const CrossMaps& maps, int d, int dev, cudaStream_t s) {
  BlocksParams bp{};
  bp.a = p;
  bp.q = maps.q;
  bp.k = maps.k;
  bp.v = maps.v;
  bp.tile_tokens = cross_tile_tokens(p.group);
  // one tile a CTA where sequences have no more on average
  const bool split = p.n_tokens <= int64_t(bp.tile_tokens) * p.batch;
  const int64_t block_tokens = int64_t(split ? 1 : 2) * bp.tile_tokens;
  const int64_t blocks = (p.n_tokens / p.batch + block_tokens - 1) / block_tokens;
  const int64_t sure = (blocks > 0 ? blocks : 1) * p.batch * p.kv_heads;           // about as many blocks as there are
  const int64_t items = cross_blocks(p, p.q_begin, p.n_tokens, int(block_tokens));
  const int64_t tiles = (p.n_rows / p.batch + kStates - 1) / kStates;
  if (d == 128)
    return p.f16 ? (split ? launch<128, true, true>(bp, items, sure, tiles, dev, s) : launch<128, true, false>(bp, items, sure, tiles, dev, s))
                 : (split ? launch<128, false, true>(bp, items, sure, tiles, dev, s) : launch<128, false, false>(bp, items, sure, tiles, dev, s));
  return p.f16 ? (split ? launch<64, true, true>(bp, items, sure, tiles, dev, s) : launch<64, true, false>(bp, items, sure, tiles, dev, s))
               : (split ? launch<64, false, true>(bp, items, sure, tiles, dev, s) : launch<64, false, false>(bp, items, sure, tiles, dev, s));
}

}  // namespace reskv
