// Attention of many query rows (a chunk of a prompt) over the paged 4-bit cache,
// on the fifth-generation tensor cores.
//
// A CTA takes one block of 128 or 256 query rows of one KV head and walks its
// positions 64 at a time.  With few rows (paged_attn.cu) a code is unpacked for
// every eight of them; here each tile is unpacked once for the block, into fp16
// operands in shared memory:
//
//   S = Q K^T       [128 rows x 64 positions]   tcgen05.mma, per 128 rows, into TMEM
//   P = 2^(S - ref) one row a thread, fp16 into TMEM (256 rows: shared memory)
//   O += P V        [128 rows x d]              tcgen05.mma, accumulated in TMEM
//
// Four or eight warps take the softmax, a row a thread, eight others unpack up to
// two steps ahead, one issues the products and one the copies.  Steps pass between them
// through mbarriers:
//
//   q             the queries' operands are in shared memory (softmax -> products)
//   raw[i % 3]    step i's packed tiles have landed        (copy -> unpack)
//   looked[i & 3] its largest exponents are known           (two warps of their own -> unpack)
//   ready[i & 3]  its operands are in shared memory         (unpack -> products, softmax)
//   s[i & 1]      S is in TMEM, K's buffer is free          (products -> softmax, unpack)
//   p             P is in place, S's buffer is free         (softmax -> products)
//   pv[i % 3]     O holds it, P's and V's buffers are free   (products -> softmax, unpack)
//
// No barrier completes a phase again before all that wait for the last one have
// seen it: each next completion needs a step of the one that waits.
//
// Roundings.  Keys and values are divided by a power of two that only grows along
// the block (the largest exponent met so far), queries by one per row, so that any
// magnitude fits fp16.  Logits are formed from exact products: s (n - 8) has 11
// bits, and m + 8 s, in two fp16 planes, meets the query's sums over the groups, in
// two planes too, in one more step of the same product.  Values s n + m and weights
// are rounded to fp16's 11 bits, no coarser than the 16-bit types the output is rounded
// to; fp32 outputs take the kernel of few rows.  Sums, statistics and accumulators are
// fp32.  A row whose logits or output come out small beside what the block's largest key
// or value leaves of fp16's digits (a token that other rows see, far larger than all it
// sees) is computed again in fp32, by plain_rows().
//
// Bound by the warps' instructions (the schedulers issue in 57 % of the cycles, the
// tensor cores work in 29 %): 512 tokens behind 8K (2 sequences, 8 KV heads, 32 query
// heads, 133 GFLOP) take 219 us, 608 TFLOP/s.  With eight warps that unpacked and took
// the softmax in turn, between two barriers of the whole block, it was 357 us; with
// the roles apart 280; with exponents in warps of their own, and weights formed
// before a largest logit is looked for, 218.
#include <atomic>

#include "paged_attn.cuh"
#include "tensor_core.cuh"

namespace reskv {
namespace {

using namespace tc;

constexpr int kPos = 64;                          // positions of a step
constexpr int kSub = kPos / kTile;                // cache tiles of a step
constexpr int kThreads = 640;                     // warps 0-7 softmax, 8-15 unpack, 16 products, 17 copies, 18-19 exponents
constexpr int kUnpackWarp = 8, kIssueWarp = 16, kCopyWarp = 17, kLookWarp = 18;
constexpr int kRaw = 3;                           // steps of packed tiles in flight
// What a row makes of operands that were held for the whole block is checked at its end.
// The block's keys leave logits off by 2^-10 of their unit at most, which is below 2^-14 up
// to kFarLogits (rows whose query times the largest key is some 2^17); past that logits
// may also be too large for weights formed from unrounded ones.  Values are off by 2^-25,
// 2^-12 of an output of kFarValues.
constexpr float kFarLogits = 0.03125f, kFarValues = 1.220703125e-4f;          // 2^-5, 2^-13
// Registers a thread of each part: (2 x 128 + 2 x 88 + 40) x 128 of the launch's 96 x 640.
constexpr int kRegsSoftmax = 128, kRegsUnpack = 88, kRegsIssue = 40;
static_assert((2 * kRegsSoftmax + 2 * kRegsUnpack + kRegsIssue) * 128 <= 96 * kThreads, "registers");

// 2^(14 - (e - 127)) and its inverse, of a biased exponent 15 <= e <= 254
__device__ __forceinline__ float down(int e) { return __int_as_float((268 - e) << 23); }
__device__ __forceinline__ float up(int e) { return __int_as_float((e - 14) << 23); }

// --- shared memory ---

template <int D, int NG, int MT>
struct BlockSmem {
  static constexpr int half = 128 * 128;          // 128 rows of 64 fp16
  static constexpr int q = MT * (D / 64) * half;
  static constexpr int kbuf = kPos * D * 2, vbuf = kPos * D * 2;
  static constexpr int raw1 = kSub * TileShape{D, NG}.bytes();
  static constexpr int q_more = 128 * 32, k_more = kPos * 32;         // the step of minima
  static constexpr int p = MT == 2 ? MT * half : 0;
  static constexpr int at_k = q, at_v = at_k + 2 * kbuf, at_p = at_v + 3 * vbuf, at_qm = at_p + p, at_km = at_qm + MT * q_more,
                       at_raw = at_km + 2 * k_more;
  static constexpr int bytes = at_raw + kRaw * raw1 + 1024;           // operands on 1024 bytes
};

struct BlockShared {
  uint64_t q, raw[kRaw], looked[4], ready[4], s[2], p, pv[3];
  uint32_t tmem, abort;
  // of step i at i & 7
  uint32_t valid[8];                              // which of its cache tiles exist
  int top[8][2];                                  // largest biased exponent of its K and V
  int held[8][2];                                 // the exponents they are held at
  uint32_t odd[8];                                // it has V groups that are NaN
  uint8_t odd_groups[8][kPos];                    // which, per position
};

// Wait for phase `parity`; false once a wait of any warp has given up.
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, BlockShared& sh, uint32_t* status) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  volatile uint32_t* abort = &sh.abort;
  while (!mbar_try_wait(bar, parity)) {
    if (*abort) return false;
    if (clock64() - t0 > kWaitLimitCycles) {
      *abort = 1u;
      report_status(status, kStatusWaitTimeout);
      return false;
    }
  }
  return true;
}
// The same for a whole warp.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, BlockShared& sh, uint32_t* status) {
  return __all_sync(0xffffffffu, wait_for(bar, parity, sh, status));
}
__device__ __forceinline__ void warp_arrive(uint64_t* bar, int lane) {
  __syncwarp();
  if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

struct BlockParams {
  AttnParams a;
  BlockPlan plan;
  float* records;                                 // [slot][rows][D], then [slot][rows] log2 sums
};

// A softmax warp's rows without tensor cores, one after the other, in fp32, whatever the
// magnitudes: a lane has four dims, four positions are taken at a time.  Far slower (a
// chunk all of whose rows go this way, 512 tokens behind 8K of two sequences: 54 ms) and
// for inputs past what a model makes; out of line, so that the loops of the roles do not
// move in the instruction caches for it.
template <int D, int NG>
__device__ __noinline__ void plain_rows(const BlockParams& bp, const Sequence& sq, int b, int h, int r0, int first, int tiles,
                                        float* record, float* record_ref) {
  const AttnParams& p = bp.a;
  constexpr TileShape ts{D, NG};
  constexpr int TB = ts.bytes();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rows = sq.count * p.group, base = sq.len - sq.count;
  __syncwarp();
  const int tpp = p.page_tokens / kTile, u = lane < D / 4 ? lane : 0, group = 4 * u * NG / D;
#pragma unroll 1
  for (int i = 0; i < 32; ++i) {
    const int local = warp * 32 + i, row = r0 + local;
    if (row >= rows) break;
    const uint16_t* src = static_cast<const uint16_t*>(p.q) + (sq.q0 + row / p.group) * p.q_token +
                          int64_t(h * p.group + row % p.group) * p.q_head + 4 * u;
    float qv[4], o[4] = {0.f, 0.f, 0.f, 0.f}, top = -INFINITY, l = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float x = p.q_f16 ? __half2float(__ushort_as_half(src[j])) : __bfloat162float(__ushort_as_bfloat16(src[j]));
      qv[j] = lane < D / 4 ? x : 0.f;
    }
    const int hi = base + row / p.group, lo = first_seen(p, hi);
    const int stop = hi < 0 ? 0 : min(hi / kTile + 1, first + tiles);
#pragma unroll 1
    for (int t = max(lo / kTile, first); t < stop; ++t) {
      const int page = p.page_table[int64_t(b) * p.table_pages + t / tpp];
      if (page < 0 || page >= p.n_pages) continue;
      const uint8_t* tile = p.pages + ((int64_t(page) * p.kv_heads + h) * tpp + t % tpp) * int64_t(TB);
#pragma unroll 1
      for (int k0 = 0; k0 < kTile; k0 += 4) {
        auto value = [&](int k, int codes, int meta, int j) {
          const uint16_t* sm = reinterpret_cast<const uint16_t*>(tile + meta) + 2 * NG * k + group;
          const float s = __bfloat162float(__ushort_as_bfloat16(sm[0])), m = __bfloat162float(__ushort_as_bfloat16(sm[NG]));
          return fmaf(s, float(*reinterpret_cast<const uint16_t*>(tile + codes) >> (4 * j) & 15), m);
        };
        float x[4], v[4][4], now = top;
        bool any = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[k] = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            x[k] = fmaf(qv[j], value(k0 + k, ts.k_unit(k0 + k, u), ts.k_meta(), j), x[k]);
            v[k][j] = value(k0 + k, ts.v_codes() + ts.v_unit(k0 + k, u), ts.v_meta(), j);
          }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
#pragma unroll
          for (int d = 16; d; d /= 2) x[k] += __shfl_xor_sync(0xffffffffu, x[k], d);
          const int pos = t * kTile + k0 + k;
          x[k] = pos >= lo && pos <= hi ? x[k] * p.scale2 : -INFINITY;
          now = fmaxf(now, x[k]);
          any |= x[k] != -INFINITY;
        }
        if (!any) continue;
        const float keep = exp2f(top - now);
        top = now;
        l *= keep;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] *= keep;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (x[k] == -INFINITY) continue;
          const float w = exp2f(x[k] - now);
          l += w;
#pragma unroll
          for (int j = 0; j < 4; ++j) o[j] = fmaf(w, v[k][j], o[j]);
        }
      }
    }
    const bool seen = l != 0.f;
    const float inv = seen ? 1.f / l : 0.f;
    const float4 v = make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    if (lane < D / 4) {
      if (record) reinterpret_cast<float4*>(record + int64_t(local) * D)[lane] = v;
      else store_out(p, sq, h, row, lane, v);
    }
    if (lane == 0) {
      const float sum = seen ? top + log2f(l) : -INFINITY;
      if (record) record_ref[local] = sum;
      else store_lse(p, sq, h, row, sum);
    }
  }
}

template <int D, int NG, int MT>
__global__ void __launch_bounds__(kThreads, 1) k_attn_blocks(const __grid_constant__ BlockParams bp) {
  using S = BlockSmem<D, NG, MT>;
  constexpr int kRows = 128 * MT, C = D / 32, PG = C / NG, TB = TileShape{D, NG}.bytes();
  constexpr TileShape ts{D, NG};
  constexpr uint32_t kColumns = 512;
  constexpr bool kPTensor = MT == 1;              // P in tensor memory, where two blocks leave it no room
  const AttnParams& p = bp.a;
  extern __shared__ uint8_t dynamic[];
  uint8_t* smem = dynamic + ((1024u - (smem_u32(dynamic) & 1023u)) & 1023u);
  __shared__ __align__(16) BlockShared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    mbar_init(&sh.q, 4 * MT);
    for (int i = 0; i < kRaw; ++i) mbar_init(&sh.raw[i], 1);
    for (int i = 0; i < 4; ++i) {
      mbar_init(&sh.ready[i], 8);
      mbar_init(&sh.looked[i], 2);
    }
    mbar_init(&sh.s[0], 1);
    mbar_init(&sh.s[1], 1);
    mbar_init(&sh.p, 4 * MT);
    for (int i = 0; i < 3; ++i) mbar_init(&sh.pv[i], 1);
    sh.abort = 0;
    fence_mbar_init();
  }
  wait_for_previous();

  // the item: part of the positions of one block of rows
  const BlockPlan& plan = bp.plan;
  const int cut = plan.units - plan.whole, item = int(blockIdx.x) - plan.whole;
  const bool apart = item >= 0 && plan.parts() > 1;
  int part = 0, unit = blockIdx.x;
  if (apart) {
    const bool last = item >= cut * plan.even;
    unit = last ? item - cut * plan.even : item / plan.even;
    part = last ? plan.even : item - unit * plan.even;
    unit += plan.whole;
  }
  const int blk = unit % plan.row_blocks, bh = unit / plan.row_blocks;
  const int b = bh / p.kv_heads, h = bh - b * p.kv_heads;
  const Sequence sq = sequence_of(p, b);
  const int rows = sq.count * p.group, r0 = blk * kRows;
  const RowBlock rb = row_block(p, sq, r0, min(r0 + kRows, rows));
  const int steps_all = (rb.tiles + kSub - 1) / kSub;
  const int step0 = apart ? int((int64_t(steps_all) * part * plan.share) >> 16) : 0;
  const int n = (apart && part + 1 < plan.parts() ? int((int64_t(steps_all) * (part + 1) * plan.share) >> 16) : steps_all) - step0;
  const int first = rb.first + step0 * kSub;      // first cache tile
  const int tiles = min(rb.tiles - step0 * kSub, n * kSub);
  // what the block's rows see
  const int base = sq.len - sq.count;
  const int hi_first = base + r0 / p.group, hi_last = base + (min(r0 + kRows, rows) - 1) / p.group;
  const int from = first_seen(p, hi_first);
  const int lo_last = first_seen(p, hi_last);

  // a softmax thread's row (rows that do not exist see what the last one does)
  const int mt = warp >> 2;
  const int rt = (warp & 3) * 32 + lane;          // row within its 128
  const int r = r0 + mt * 128 + rt;
  const bool real = warp < 4 * MT && r < rows;
  const int64_t slot = apart ? int64_t(unit - plan.whole) * plan.parts() + part : 0;
  float* const record = bp.records + slot * kRows * D;
  float* const record_ref = bp.records + plan.slots() * kRows * D + slot * kRows;
  auto finish_row = [&](int c, const float (&v)[32]) {       // dims 32c .. 32c + 31 of this thread's row
    if (!real) return;
    if (apart) {
      float* y = record + int64_t(mt * 128 + rt) * D + 32 * c;
#pragma unroll
      for (int i = 0; i < 8; ++i) reinterpret_cast<float4*>(y)[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) store_out(p, sq, h, r, 8 * c + i, make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]));
    }
  };
  auto finish_sum = [&](float sum) {
    if (!real) return;
    if (apart) record_ref[mt * 128 + rt] = sum;
    else store_lse(p, sq, h, r, sum);
  };
  if (n == 0) {                                   // nothing to see: the same for the whole CTA
    const float zero[32] = {};
#pragma unroll 1
    for (int c = 0; c < C; ++c) finish_row(c, zero);
    finish_sum(-INFINITY);
    return;
  }

  if (warp == kIssueWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = sh.tmem;
  const uint32_t smem_q = smem_u32(smem), smem_k = smem_q + S::at_k, smem_v = smem_q + S::at_v;
  auto s_cols = [&](int buf, int m) { return tmem + uint32_t((buf * MT + m) * kPos); };
  auto o_cols = [&](int m) { return tmem + uint32_t(2 * MT * kPos + m * 128); };
  const uint32_t p_cols = tmem + uint32_t(2 * MT * kPos + MT * 128);

  auto in_block = [&](int pos) { return pos >= from && pos <= hi_last; };
  if (warp >= kIssueWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
    if (warp == kIssueWarp) {
      // --- products ---
      int s_issued = 0, o_issued = 0;
      // Every product is one instruction of one thread, so the operands' words are
      // worked out here and the loops below have only additions.
      const uint32_t q0 = operand(smem_q), qm0 = operand(smem_q + S::at_qm), p0 = operand(smem_q + S::at_p);
      auto issue_s = [&](int i) {                 // S of step i
        s_issued = i + 1;
        fence_after();
        if (elected()) {
          const uint32_t k0 = operand(smem_k + (i & 1) * S::kbuf), km0 = operand(smem_q + S::at_km + (i & 1) * S::k_more);
          const uint32_t d0 = s_cols(i & 1, 0);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
              multiply<kRows128, shape_of(kPos)>(d0 + m * kPos, q0 + (((m * (D / 64) + k / 4) * S::half + (k & 3) * 32) >> 4),
                                                 k0 + (((k / 4) * (kPos * 128) + (k & 3) * 32) >> 4), k > 0);
            multiply<kRows32, shape_of(kPos)>(d0 + m * kPos, qm0 + ((m * S::q_more) >> 4), km0, true);
          }
          commit(&sh.s[i & 1]);
        }
        __syncwarp();
      };
      auto issue_o = [&](int i) {
        o_issued = i + 1;
        fence_after();
        if (elected()) {
          const uint32_t v0 = operand(smem_v + (i % 3) * S::vbuf), d0 = o_cols(0);
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int k = 0; k < kPos / 16; ++k)
              if constexpr (kPTensor)
                multiply_from<kRows128, shape_of(D)>(d0, p_cols + k * 8, v0 + ((k * 32) >> 4), i > 0 || k > 0);
              else
                multiply<kRows128, shape_of(D)>(d0 + m * 128, p0 + ((m * S::half + k * 32) >> 4), v0 + ((k * 32) >> 4), i > 0 || k > 0);
          commit(&sh.pv[i % 3]);
        }
        __syncwarp();
      };
      bool ok = warp_wait(&sh.q, 0, sh, p.status);
      // S of step i + 1 goes out before O of step i, whose weights take longer
#pragma unroll 1
      for (int i = -1; i < n && ok; ++i) {
        if (i + 1 < n) {
          ok = warp_wait(&sh.ready[(i + 1) & 3], ((i + 1) >> 2) & 1, sh, p.status);
          if (!ok) break;
          issue_s(i + 1);
        }
        if (i >= 0) {
          ok = warp_wait(&sh.p, i & 1, sh, p.status);
          if (!ok) break;
          issue_o(i);
        }
      }
      if (!ok && lane == 0) {
        // a wait gave up: let what is in flight land (each wait with the same bound); the output is incomplete
        for (int i = s_issued > 2 ? s_issued - 2 : 0; i < s_issued; ++i) mbar_wait_bounded(&sh.s[i & 1], (i >> 1) & 1);
        for (int i = o_issued > 3 ? o_issued - 3 : 0; i < o_issued; ++i) mbar_wait_bounded(&sh.pv[i % 3], (i / 3) & 1);
      }
      __syncwarp();
    } else if (warp == kCopyWarp) {
      // --- copies ---
      const int tpp = p.page_tokens / kTile;
      int copied = 0;
      auto copy_step = [&](int i) {               // lanes 0..3: one cache tile each
        copied = i + 1;
        const int stage = i % kRaw, t = i * kSub + lane;
        int page = -1, at = 0;
        const bool asked = lane < kSub && t < tiles;
        if (asked) {
          const int tile = first + t, pg = tile / tpp;
          at = tile - pg * tpp;
          page = p.page_table[int64_t(b) * p.table_pages + pg];
        }
        const bool ok = asked && page >= 0 && page < p.n_pages;
        if (asked && !ok) report_status(p.status, kStatusBadIndex);
        const uint32_t mask = __ballot_sync(0xffffffffu, ok);
        if (lane == 0) {
          sh.valid[i & 7] = mask;
          if (mask) mbar_arrive_expect_tx(&sh.raw[stage], __popc(mask) * TB);
          else asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(&sh.raw[stage])) : "memory");
        }
        __syncwarp();
        if (ok)
          bulk_g2s(smem + S::at_raw + stage * S::raw1 + lane * TB,
                   p.pages + ((int64_t(page) * p.kv_heads + h) * tpp + at) * int64_t(TB), TB, &sh.raw[stage]);
      };
      bool ok = true;
#pragma unroll 1
      for (int i = 0; i < n && ok; ++i) {
        if (i >= kRaw) ok = warp_wait(&sh.ready[(i - kRaw) & 3], ((i - kRaw) >> 2) & 1, sh, p.status);
        if (ok) copy_step(i);
      }
      if (!ok && lane == 0)
        for (int i = copied > kRaw ? copied - kRaw : 0; i < copied; ++i) mbar_wait_bounded(&sh.raw[i % kRaw], (i / kRaw) & 1);
      __syncwarp();
    } else {
      // --- a step's largest exponents: two positions' keys (warp 18) or values (19) a lane ---
      const int which = warp - kLookWarp;
      bool ok = true;
#pragma unroll 1
      for (int i = 0; i < n && ok; ++i) {
        ok = warp_wait(&sh.raw[i % kRaw], (i / kRaw) & 1, sh, p.status);
        // its slots were step i - 8's, whose weights are long in P
        float top = 0.f;
        uint32_t any_odd = 0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int tk = lane + 32 * j;
          uint32_t odd = 0;
          if (((sh.valid[i & 7] >> (tk / kTile)) & 1) && in_block((first + i * kSub) * kTile + tk)) {
            const uint8_t* tile = smem + S::at_raw + (i % kRaw) * S::raw1 + (tk / kTile) * TB;
            uint32_t meta[NG];
            load_words<NG>(meta, tile + (which ? ts.v_meta() : ts.k_meta()) + (tk % kTile) * 4 * NG);
#pragma unroll
            for (int k = 0; k < NG; ++k) {
              float s, m;
              group_meta<NG>(meta, k, s, m);
              if (s != s || m != m) odd |= 1u << k;
              else top = fmaxf(top, fminf(fmaxf(fabsf(m), fabsf(fmaf(15.f, s, m))), 3.0e38f));
            }
          }
          if (which) sh.odd_groups[i & 7][tk] = uint8_t(odd);
          any_odd |= odd;
        }
        const int e = __reduce_max_sync(0xffffffffu, __float_as_int(top) >> 23);
        const bool some = __any_sync(0xffffffffu, any_odd != 0);
        if (lane == 0) {
          sh.top[i & 7][which] = e;
          if (which) sh.odd[i & 7] = some;
        }
        warp_arrive(&sh.looked[i & 3], lane);
        // three steps ahead of the unpacking at most, as the copies are
      }
    }
  } else if (warp >= kUnpackWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsUnpack));
    // --- unpacking: warp w takes K (even) or V (odd) of cache tile w / 2 of a step ---
    const int uw = warp - kUnpackWarp, ut = tid - kUnpackWarp * 32;
    // Exponents that steps are held at: they only grow.
    int ek = 15, ev = 15;
    auto unpack = [&](int i) {
      const int stage = i % kRaw, sub = uw >> 1;
      const int g = lane >> 2, t = lane & 3;
      const uint8_t* tile = smem + S::at_raw + stage * S::raw1 + sub * TB;
      const int pos = (first + i * kSub + sub) * kTile;
      const bool exists = (sh.valid[i & 7] >> sub) & 1, odd = sh.odd[i & 7] != 0;
      // codes n, less `less`, of the even and the odd places as fp16 numbers
      auto whole = [](uint32_t v, float less) {
        const uint32_t w = (v & 0x000f000fu) | 0x64006400u;              // 1024 + n
        return __hsub2(*reinterpret_cast<const __half2*>(&w), __float2half2_rn(1024.f + less));
      };
      auto odd_place = [](uint32_t v, float less) {
        const uint32_t w = (v & 0x00f000f0u) | 0x64006400u;              // 1024 + 16 n
        return __hfma2(*reinterpret_cast<const __half2*>(&w), __float2half2_rn(0.0625f), __float2half2_rn(-64.f - less));
      };
      auto bits = [](__half2 x) { return *reinterpret_cast<const uint32_t*>(&x); };
      if ((uw & 1) == 0) {
        const float f = down(ek);
        uint32_t words[2][C] = {}, metas[2][NG] = {};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int row = g + 8 * j;
          if (exists && in_block(pos + row)) {
            load_words<C>(words[j], tile + row * (D / 2) + t * (D / 8));
            load_words<NG>(metas[j], tile + ts.k_meta() + row * 4 * NG);
          }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int tk = sub * kTile + g + 8 * j;
          const uint32_t(&w)[C] = words[j];
          const uint32_t(&meta)[NG] = metas[j];
#pragma unroll
          for (int c = 0; c < C; ++c) {
            float s, m;
            group_meta<NG>(meta, c / PG, s, m);
            const __half2 s2 = __float2half2_rn(s * f);
            // dims 0, 4, 1, 5, 2, 6, 3, 7 of the word's eight
            const uint4 v = make_uint4(bits(__hmul2(whole(w[c], 8.f), s2)), bits(__hmul2(odd_place(w[c], 8.f), s2)),
                                       bits(__hmul2(whole(w[c] >> 8, 8.f), s2)), bits(__hmul2(odd_place(w[c] >> 8, 8.f), s2)));
            const int word = 4 * c + t;
            *reinterpret_cast<uint4*>(smem + S::at_k + (i & 1) * S::kbuf + (word >> 3) * (kPos * 128) + tk * 128 +
                                      (((word & 7) ^ (tk & 7)) << 4)) = v;
          }
          // the groups' m + 8 s: first planes (t = 0), second planes (1), first again (2), nothing (3)
          float plane[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < NG; ++k) {
            float s, m;
            group_meta<NG>(meta, k, s, m);
            const float x = fmaf(8.f, s, m) * f, first_plane = __half2float(__float2half_rn(x));
            plane[k] = t == 3 ? 0.f : t == 1 ? x - first_plane : first_plane;
          }
          *reinterpret_cast<uint2*>(smem + S::at_km + (i & 1) * S::k_more + tk * 32 + (((t >> 1) ^ ((tk >> 2) & 1)) << 4) + (t & 1) * 8) =
              make_uint2(pack_f16(plane[0], plane[1]), pack_f16(plane[2], plane[3]));
        }
      } else {
        const float f = down(ev);
        uint32_t words[2][C] = {}, metas[4][NG] = {};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int pair = t + 4 * j;
          const bool held0 = exists && in_block(pos + 2 * pair), held1 = exists && in_block(pos + 2 * pair + 1);
          if (held0 || held1) load_words<C>(words[j], tile + ts.v_codes() + pair * D + ts.v_place(pair, g) * (D / 8));
          if (held0) load_words<NG>(metas[2 * j], tile + ts.v_meta() + 2 * pair * 4 * NG);
          if (held1) load_words<NG>(metas[2 * j + 1], tile + ts.v_meta() + (2 * pair + 1) * 4 * NG);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int tk = sub * kTile + 2 * (t + 4 * j);
          const uint32_t(&w)[C] = words[j];
          const uint32_t(&meta0)[NG] = metas[2 * j];
          const uint32_t(&meta1)[NG] = metas[2 * j + 1];
#pragma unroll
          for (int c = 0; c < C; ++c) {
            float sa, ma, sb, mb;
            group_meta<NG>(meta0, c / PG, sa, ma);
            group_meta<NG>(meta1, c / PG, sb, mb);
              if (odd) {                            // NaN is put into the rows that see it at the end
              if (sa != sa || ma != ma) sa = ma = 0.f;
              if (sb != sb || mb != mb) sb = mb = 0.f;
            }
            const __half2 s2 = __floats2half2_rn(sa * f, sb * f), m2 = __floats2half2_rn(ma * f, mb * f);
            const __half2 v[4] = {__hfma2(whole(w[c], 0.f), s2, m2), __hfma2(odd_place(w[c], 0.f), s2, m2),
                                  __hfma2(whole(w[c] >> 8, 0.f), s2, m2), __hfma2(odd_place(w[c] >> 8, 0.f), s2, m2)};
            // dim 32c + 4g + e in row 32c + 8e + g: lanes of one store in eight rows, as many 16-byte words
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int row = 32 * c + 8 * e + g;
              *reinterpret_cast<uint32_t*>(smem + S::at_v + (i % 3) * S::vbuf + row * 128 + (((tk >> 3) ^ (row & 7)) << 4) +
                                           (tk & 7) * 2) = bits(v[e]);
            }
          }
        }
      }
    };
    bool ok = true;
#pragma unroll 1
    for (int i = 0; i < n && ok; ++i) {
      ok = warp_wait(&sh.raw[i % kRaw], (i / kRaw) & 1, sh, p.status) && warp_wait(&sh.looked[i & 3], (i >> 2) & 1, sh, p.status);
      if (ok && i >= 2) ok = warp_wait(&sh.s[i & 1], ((i - 2) >> 1) & 1, sh, p.status);
      if (ok && i >= 3) ok = warp_wait(&sh.pv[i % 3], ((i - 3) / 3) & 1, sh, p.status);
      if (!ok) break;
      ek = min(max(ek, sh.top[i & 7][0]), 254);
      ev = min(max(ev, sh.top[i & 7][1]), 254);
      if (ut == 0) {
        sh.held[i & 7][0] = ek;
        sh.held[i & 7][1] = ev;
      }
      unpack(i);
      fence_proxy_async_smem();
      warp_arrive(&sh.ready[i & 3], lane);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    if (warp < 4 * MT) {
      // --- the softmax, a row a thread ---
      const uint32_t lanes = uint32_t((warp & 3) * 32) << 16;
      const int hi = base + min(r, rows - 1) / p.group;
      const int lo = first_seen(p, hi);
      float ref = kNoRef, l = 0.f;
      uint32_t nan_groups = 0;
      // the row's query, scaled below 2^8 (128 of them sum up within fp16), in the order of the keys' dims
      uint32_t w[D / 2];                          // two neighbouring dims a word
#pragma unroll
      for (int k = 0; k < D / 2; ++k) w[k] = 0u;
      if (real) {
        const uint16_t* src = static_cast<const uint16_t*>(p.q) + (sq.q0 + r / p.group) * p.q_token +
                              int64_t(h * p.group + r % p.group) * p.q_head;
        if (p.q_wide) {
#pragma unroll
          for (int k = 0; k < D / 8; ++k) {
            const uint4 v = reinterpret_cast<const uint4*>(src)[k];
            w[4 * k] = v.x;
            w[4 * k + 1] = v.y;
            w[4 * k + 2] = v.z;
            w[4 * k + 3] = v.w;
          }
        } else {
#pragma unroll
          for (int k = 0; k < D / 2; ++k) w[k] = src[2 * k] | uint32_t(src[2 * k + 1]) << 16;
        }
      }
      auto two = [&](int k) { return p.q_f16 ? __half22float2(*reinterpret_cast<const __half2*>(&w[k])) : bf16x2_to_float2(w[k]); };
      float top = 0.f;
#pragma unroll
      for (int k = 0; k < D / 2; ++k) top = fmaxf(top, fmaxf(fabsf(two(k).x), fabsf(two(k).y)));
      const int e = 134 - min(max(__float_as_int(top) >> 23, 1), 254), e1 = e >> 1, e2 = e - e1;
      const float f1 = __int_as_float((127 + e1) << 23), f2 = __int_as_float((127 + e2) << 23);
      float sums[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < D / 8; ++k) {
        const float2 v0 = two(4 * k), v1 = two(4 * k + 1), v2 = two(4 * k + 2), v3 = two(4 * k + 3);
        // dims 0, 4, 1, 5, 2, 6, 3, 7 of eight
        const uint4 v = make_uint4(pack_f16(v0.x * f1 * f2, v2.x * f1 * f2), pack_f16(v0.y * f1 * f2, v2.y * f1 * f2),
                                   pack_f16(v1.x * f1 * f2, v3.x * f1 * f2), pack_f16(v1.y * f1 * f2, v3.y * f1 * f2));
        const uint32_t held[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&held[j]));
          sums[k / (D / 8 / NG)] += x.x + x.y;
        }
        *reinterpret_cast<uint4*>(smem + (mt * (D / 64) + (k >> 3)) * S::half + rt * 128 + (((k & 7) ^ (rt & 7)) << 4)) = v;
      }
      // against the keys' planes: first planes twice, then what they left over
      float left[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        left[k] = sums[k];
        sums[k] = __half2float(__float2half_rn(sums[k]));
        left[k] -= sums[k];
      }
      const uint2 top_planes = make_uint2(pack_f16(sums[0], sums[1]), pack_f16(sums[2], sums[3]));
      const uint2 low_planes = make_uint2(pack_f16(left[0], left[1]), pack_f16(left[2], left[3]));
      uint8_t* more = smem + S::at_qm + mt * S::q_more + rt * 32;
      const int turn_word = ((rt >> 2) & 1) << 4;
      *reinterpret_cast<uint4*>(more + turn_word) = make_uint4(top_planes.x, top_planes.y, top_planes.x, top_planes.y);
      *reinterpret_cast<uint4*>(more + (16 ^ turn_word)) = make_uint4(low_planes.x, low_planes.y, 0u, 0u);
      const float cq = p.scale2 * __int_as_float((127 - e1) << 23) * __int_as_float((127 - e2) << 23);
      fence_proxy_async_smem();
      warp_arrive(&sh.q, lane);
      int ev_was = 15;
      bool ok = true;
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        ok = warp_wait(&sh.ready[i & 3], (i >> 2) & 1, sh, p.status) && warp_wait(&sh.s[i & 1], (i >> 1) & 1, sh, p.status);
        if (!ok) break;
        fence_after();
        const int ek0 = sh.held[i & 7][0], ev0 = sh.held[i & 7][1];
        float x[kPos];
#pragma unroll
        for (int k = 0; k < 4; ++k) load16(s_cols(i & 1, mt) + lanes + 16 * k, x + 16 * k);
        landed();
#pragma unroll
        for (int k = 0; k < 4; ++k) defined16(x + 16 * k);
        const float f = fmaxf(cq * up(ek0), 1.17549435e-38f);      // positive: -inf stays -inf
        const int pos = (first + i * kSub) * kTile;
        const uint32_t valid = sh.valid[i & 7];
        const bool all = pos >= lo_last && pos + kPos - 1 <= hi_first;
        // the row sees positions pos + a .. pos + z - 1 of the step
        const int a = min(max(lo - pos, 0), kPos), z = min(max(hi + 1 - pos, 0), kPos);
        uint64_t see = ~0ull;
        if (!all || valid != (1u << kSub) - 1u) {
          see = z <= a ? 0ull : ((z == 64 ? ~0ull : (1ull << z) - 1ull) & ~((a == 64 ? 0ull : 1ull << a) - 1ull));
#pragma unroll
          for (int k = 0; k < kSub; ++k)
            if (!((valid >> k) & 1)) see &= ~(0xffffull << (16 * k));
        }
        const bool masked = __any_sync(0xffffffffu, see != ~0ull);
        auto mask = [&]() {
          if (!masked) return;
#pragma unroll
          for (int k = 0; k < kPos; ++k)
            if (!((see >> k) & 1)) x[k] = -INFINITY;
        };
        auto weights = [&]() {                    // x: logits -> weights, in place; returns their sum
          float2 s2[4] = {};
#pragma unroll
          for (int k = 0; k < kPos; k += 2) {
            const float2 y = ffma2(make_float2(x[k], x[k + 1]), make_float2(f, f), make_float2(-ref, -ref));
            const float2 v = make_float2(exp2_fast(y.x), exp2_fast(y.y));
            s2[(k / 2) & 3] = fadd2(s2[(k / 2) & 3], v);
            x[k] = v.x;
            x[k + 1] = v.y;
          }
          const float2 t = fadd2(fadd2(s2[0], s2[1]), fadd2(s2[2], s2[3]));
          return t.x + t.y;
        };
        mask();
        float sum = weights(), keep = 1.f;
        // A sum within 2^14 has every weight within fp16.  Otherwise the logits, still in
        // TMEM, are taken again and the reference goes 6 below the largest.
        if (__any_sync(0xffffffffu, !(sum <= 16384.f))) {
#pragma unroll
          for (int k = 0; k < 4; ++k) load16(s_cols(i & 1, mt) + lanes + 16 * k, x + 16 * k);
          landed();
#pragma unroll
          for (int k = 0; k < 4; ++k) defined16(x + 16 * k);
          mask();
          float top = -INFINITY;
#pragma unroll
          for (int k = 0; k < kPos; k += 2) asm("max.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(x[k]), "f"(x[k + 1]));
          const float now = sum <= 16384.f ? ref : fmaxf(ref, top * f - 6.f);
          keep = exp2f(ref - now);
          ref = now;
          sum = weights();
        }
        l = l * keep + sum;
        if (sh.odd[i & 7]) {                        // NaN values: which groups this row sees
#pragma unroll 1
          for (int k = 0; k < kPos; ++k)
            if ((see >> k) & 1) nan_groups |= sh.odd_groups[i & 7][k];
        }
        // P and O once the products before have been added
        if (i > 0) {
          ok = warp_wait(&sh.pv[(i - 1) % 3], ((i - 1) / 3) & 1, sh, p.status);
          if (!ok) break;
          fence_after();
          if (ev0 != ev_was) keep *= __int_as_float((127 + max(ev_was - ev0, -126)) << 23);
          if (__any_sync(0xffffffffu, keep != 1.f)) {
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
              float v[16];
              load16(o_cols(mt) + lanes + 16 * c, v);
              landed();
              defined16(v);
#pragma unroll
              for (int k = 0; k < 16; ++k) v[k] *= keep;
              store16(o_cols(mt) + lanes + 16 * c, v);
            }
            stored();
          }
        }
        ev_was = ev0;
        if constexpr (kPTensor) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float pair[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) pair[j] = __uint_as_float(pack_f16(x[32 * k + 2 * j], x[32 * k + 2 * j + 1]));
            store16(p_cols + lanes + 16 * k, pair);
          }
          stored();
        } else {
#pragma unroll
          for (int w = 0; w < 8; ++w)
            *reinterpret_cast<uint4*>(smem + S::at_p + mt * S::half + rt * 128 + ((w ^ (rt & 7)) << 4)) =
                make_uint4(pack_f16(x[8 * w], x[8 * w + 1]), pack_f16(x[8 * w + 2], x[8 * w + 3]),
                           pack_f16(x[8 * w + 4], x[8 * w + 5]), pack_f16(x[8 * w + 6], x[8 * w + 7]));
          fence_proxy_async_smem();
        }
        fence_before();
        warp_arrive(&sh.p, lane);
      }
      if (ok) ok = warp_wait(&sh.pv[(n - 1) % 3], ((n - 1) / 3) & 1, sh, p.status);
      if (ok) {
        fence_after();
        const bool seen = ref != kNoRef || l != 0.f;
        const float inv = seen ? up(ev_was) / l : 0.f;
        float top_o = 0.f;
#pragma unroll 1
        for (int c = 0; c < C; ++c) {
          float o[32], v[32];
          load16(o_cols(mt) + lanes + 32 * c, o);
          load16(o_cols(mt) + lanes + 32 * c + 16, o + 16);
          landed();
          defined16(o);
          defined16(o + 16);
          const bool bad = (nan_groups >> (c / PG)) & 1;
#pragma unroll
          for (int k = 0; k < 32; ++k) top_o = fmaxf(top_o, fabsf(o[k]));
#pragma unroll
          for (int k = 0; k < 32; ++k) v[4 * (k & 7) + (k >> 3)] = bad ? __int_as_float(0x7fc00000) : o[k] * inv;
          finish_row(c, v);
        }
        finish_sum(seen ? ref + log2f(l) : -INFINITY);
        // a row that lost digits to keys or values far larger than its own: the warp's rows again
        const bool lost = cq * up(sh.held[(n - 1) & 7][0]) > kFarLogits || (ev_was > 15 && top_o < l * kFarValues);
        if (__any_sync(0xffffffffu, real && seen && lost))
          plain_rows<D, NG>(bp, sq, b, h, r0, first, tiles, apart ? record : nullptr, record_ref);
      }
    }
  }
  fence_before();
  __syncthreads();
  fence_after();
  if (warp == kIssueWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kColumns));
}

// The parts of a block's positions joined: one row per warp.
template <int D, int MT>
__global__ void __launch_bounds__(256) k_attn_join(const __grid_constant__ BlockParams bp) {
  constexpr int kRows = 128 * MT;
  const AttnParams& p = bp.a;
  wait_for_previous();
  const int64_t w = int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  const int cut = int(w / kRows), row = int(w - int64_t(cut) * kRows);
  const int parts = bp.plan.parts(), unit = bp.plan.whole + cut;
  const int blk = unit % bp.plan.row_blocks, bh = unit / bp.plan.row_blocks;
  const int b = bh / p.kv_heads, h = bh - b * p.kv_heads;
  if (b >= p.batch) return;
  const Sequence sq = sequence_of(p, b);
  const int r = blk * kRows + row;
  if (r >= sq.count * p.group) return;
  const int64_t slot = int64_t(cut) * parts;
  const float* refs = bp.records + bp.plan.slots() * kRows * D;
  const float ref = lane < parts ? refs[(slot + lane) * kRows + row] : -INFINITY;
  const Joined j = join_weights(ref);
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int k = 0; k < parts; ++k) {
    const float f = __shfl_sync(0xffffffffu, j.weight, k);
    const float4 v = lane < D / 4 ? reinterpret_cast<const float4*>(bp.records + ((slot + k) * kRows + row) * D)[lane]
                                  : make_float4(0.f, 0.f, 0.f, 0.f);
    add_scaled(a, f, (j.present >> k) & 1 ? v : make_float4(0.f, 0.f, 0.f, 0.f));
  }
  if (lane < D / 4) store_out(p, sq, h, r, lane, a);
  if (lane == 0) store_lse(p, sq, h, r, j.ref);
}

template <int D, int NG, int MT>
cudaError_t launch(const BlockParams& bp, int dev, cudaStream_t s) {
  // the kernel's shared memory limit, raised once a device
  static std::atomic<uint64_t> raised{0};
  const uint64_t bit = dev >= 0 && dev < 64 ? uint64_t(1) << dev : 0;
  if (!(raised.load(std::memory_order_relaxed) & bit) || !bit) {
    const cudaError_t err = cudaFuncSetAttribute(k_attn_blocks<D, NG, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 BlockSmem<D, NG, MT>::bytes);
    if (err != cudaSuccess) return err;
    raised.fetch_or(bit, std::memory_order_relaxed);
  }
  cudaError_t err = launch_early(k_attn_blocks<D, NG, MT>, bp.plan.items, kThreads, BlockSmem<D, NG, MT>::bytes, s, bp);
  if (err == cudaSuccess && bp.plan.slots() > 0) {
    const int64_t rows = int64_t(bp.plan.units - bp.plan.whole) * 128 * MT;
    err = launch_early(k_attn_join<D, MT>, unsigned((rows + 7) / 8), 256, 0, s, bp);
  }
  return err;
}

template <int MT>
cudaError_t dispatch(const BlockParams& bp, int d, int group, int dev, cudaStream_t s) {
  if (d == 128 && group == 32) return launch<128, 4, MT>(bp, dev, s);
  if (d == 128 && group == 64) return launch<128, 2, MT>(bp, dev, s);
  if (d == 128) return launch<128, 1, MT>(bp, dev, s);
  if (group == 32) return launch<64, 2, MT>(bp, dev, s);
  return launch<64, 1, MT>(bp, dev, s);
}

}  // namespace

BlockPlan plan_attn_blocks(int64_t rows, int batch, int kv_heads, int64_t capacity, int sms) {
  BlockPlan plan{};
  plan.mt = rows > 128 ? 2 : 1;
  const int64_t block = 128 * plan.mt;
  plan.row_blocks = int((rows + block - 1) / block);
  plan.units = batch * kv_heads * plan.row_blocks;             // below 2^24
  // An SM takes one CTA at a time, in the order of their numbers.  Units that do not
  // fill the SMs once more are cut into parts that do, of 512 positions at least.
  // SMs still left over then take one short part of each, `turns` of those in the time
  // of a longer one; what a CTA does before its first step and after its last takes as
  // long as twelve (18 us).  Against cutting only what leaves SMs idle from the start,
  // into equal parts: 16 tokens behind 8K of 20 sequences (160 units) 312 -> 196 us,
  // 512 behind 128K of one (64 units) 1614 -> 1410.
  const int cut = plan.units % sms;
  plan.whole = plan.units - cut;
  const int64_t most = capacity / 512 < 32 ? capacity / 512 : 32;
  int64_t even = cut ? sms / cut : 1;
  if (even > most) even = most;
  plan.even = int(even < 1 ? 1 : even);
  plan.share = 65536 / plan.even;
  const int left = cut ? sms - cut * plan.even : 0;
  if (left > 0 && plan.even < 32) {
    const int turns = (cut + left - 1) / left;
    const double fixed = 12.0 * kPos / double(capacity);
    const double tail = (1.0 - plan.even * (turns - 1) * fixed) / (1.0 + turns * plan.even);
    // below 1024 positions records and their joining cost what is gained (512 tokens
    // behind 8K of two sequences, 128 units: 226 us cut, 216 whole)
    if (tail * double(capacity) >= 1024.0) {
      plan.tail = 1;
      plan.share = int(65536.0 * (1.0 - tail) / plan.even);
    }
  }
  if (plan.parts() == 1) plan.whole = plan.units;
  plan.items = plan.whole + (plan.units - plan.whole) * plan.parts();
  return plan;
}

size_t attn_blocks_bytes(const BlockPlan& plan, int d) {
  return size_t(plan.slots()) * 128 * plan.mt * (d + 1) * 4;
}

cudaError_t launch_attn_blocks(const AttnParams& p, const BlockPlan& plan, int d, int quant_group, int dev, float* records,
                               cudaStream_t s) {
  BlockParams bp{};
  bp.a = p;
  bp.plan = plan;
  bp.records = records;
  return plan.mt == 2 ? dispatch<2>(bp, d, quant_group, dev, s) : dispatch<1>(bp, d, quant_group, dev, s);
}

}  // namespace reskv
