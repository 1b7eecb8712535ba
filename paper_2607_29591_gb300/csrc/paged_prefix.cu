// Attention of a group's query rows over the prefix that its sequences share (the
// first pass of reskv_paged_attn_shared where groups have many rows), on the
// fifth-generation tensor cores.
//
// Every row sees every position, so a tile needs no masks: it is 64 positions, unpacked once for two
// blocks of 128 rows, or, where a group has no more than 128 rows (kSplit), for one while the CTA's other
// stream has the next tile:
//
//   S = Q K^T       [128 rows x 64 positions]  fp16 operands in shared memory, into TMEM, two deep
//   P = 2^(S f + c - ref)                      a row a thread, fp16 over S
//   O += P V        [128 rows x d]             P from TMEM, V^T [dims x positions] in shared memory
//
// Eight warps unpack, each from packed rows that it copies itself, four tiles ahead; eight take the
// softmax, one issues the products.
//
//   ready[t % n]  tile t's operands are in shared memory, in one of n slots      (unpack -> products)
//   free[t % n]   its products are done                        (products -> unpack)
//   s[m][i & 1]   S of stream m's tile i is in TMEM            (products -> softmax)
//   p[m][i & 1]   P is in place (a warp may be a tile ahead)   (softmax -> products)
//   pv[m]         O holds it                                   (products -> softmax)
//
// Any magnitude fits fp16, whatever stands beside it: each position's key and each position's value is divided
// by a power of two of its own, each query row by one (its elements are exact down to 2^-21 of the largest, and to
// 2^-32 of it below).  Keys enter as s (n - 8), exact in 11
// bits, and m + 8 s in two planes against the sums of the query over its groups, so that logits are
// sums of exact products; f is the power of two that the logit of a row and position takes.  Values
// s n + m are rounded to 11 bits, no coarser than the 16-bit types of the output.  Their
// power of two goes into the weight's exponent (c), and the reference follows the largest
// logit + c; the sum of the weights takes 2^-c back.  Positions that do not exist have c = -inf.
//
// A tile takes 1.4 us with one block of rows or two (some 1700 instructions a scheduler, unpacking and softmax
// about half each; the products alone 0.75), a CTA some 12 beside its tiles: the plan, the queries, the first
// tile, and 128 KB of records.  32 sequences of 4 rows behind 131072 positions 175 us, 64 behind 8192 42 with
// their own tokens beside them.  What runs once is kept in short loops: unrolled, all of a CTA's beginning and
// end took 23 us, for the instructions' sake.
#include <atomic>

#include "paged_attn.cuh"
#include "tensor_core.cuh"

namespace reskv {
namespace {

using namespace tc;

constexpr int kPos = kBlockPos;                   // positions of a tile
constexpr int kSub = kPos / kTile;                // cache tiles of it
constexpr int kAhead = 4;                          // tiles whose packed rows a warp has under way
constexpr int kThreads = 640;                     // warps 0-7 softmax, 8-15 unpack, 16 products, 17 the plans
constexpr int kUnpackWarp = 8, kIssueWarp = 16, kPlanWarp = 17;
constexpr int kRegsSoftmax = 128, kRegsUnpack = 88, kRegsIssue = 40;
static_assert((2 * kRegsSoftmax + 2 * kRegsUnpack + kRegsIssue) * 128 <= 96 * kThreads, "registers");
constexpr int kHalf = 128 * 128;                  // bytes of 128 rows of 64 fp16
// The power of two that a value is held at: no lower than 2^-60 of the largest that its warp has met, or 2^-100.
constexpr int kLeastBelow = 60, kLeastExponent = 41;

struct PrefixParams {
  SharedParams a;
  GroupPlan* plans;
  float* records;                                 // [record][rows][D]: outputs times their sum; kSplit: two an item
  float2* sums;                                   // [record][rows]: reference (log2) and sum; -inf: nothing seen
  int32_t ctas;
};

constexpr int kMostPacked = TileShape{128, 4}.bytes() / 2;            // of K or V of a cache tile
template <int D, bool kSplit>
struct PrefixSmem {
  static constexpr int tiles = kSplit ? 1 : 2, slots = kSplit ? 4 : 3;
  static constexpr int q = D / 64 * kHalf, q_more = 128 * 32;         // of 128 rows
  static constexpr int k = D / 64 * kPos * 128, k_more = kPos * 32, v = D * 128;
  static constexpr int at_q_more = tiles * q, at_slots = at_q_more + tiles * q_more;
  static constexpr int slot = k + v + k_more;                         // K, V^T, the keys' minima
  static constexpr int raw = 8 * kMostPacked;                         // packed rows of a tile
  static constexpr int at_raw = at_slots + slots * slot, all = at_raw + kAhead * raw;
  static constexpr int bytes = all + 1024;
  static_assert(2 * 128 * D * 4 <= all && slot % 1024 == 0 && at_slots % 1024 == 0, "shared memory");
};
struct PrefixShared {
  uint64_t q, ready[4], free[4], s[2][2], p[2][2], pv[2], done;
  uint32_t tmem, abort;
  GroupPlan plan;
  // per position of a slot: 2^e of its key; log2 of its value's scale (-inf: no such position), and 2^- of that
  alignas(16) float up[4][kPos], c[4][kPos], inv[4][kPos];
  float cq[128];                                  // of a row: its logits' factor
};

// 2^(14 - (e - 127)) and its inverse, of a biased exponent 15 <= e <= 254
__device__ __forceinline__ float down(int e) { return __int_as_float((268 - e) << 23); }
__device__ __forceinline__ float up(int e) { return __int_as_float((e - 14) << 23); }
__device__ __forceinline__ uint32_t bits(__half2 x) { return *reinterpret_cast<const uint32_t*>(&x); }
// codes n, less `less`, of the even and the odd places as fp16 numbers
__device__ __forceinline__ __half2 even_codes(uint32_t v, float less) {
  const uint32_t w = (v & 0x000f000fu) | 0x64006400u;                // 1024 + n
  return __hsub2(*reinterpret_cast<const __half2*>(&w), __float2half2_rn(1024.f + less));
}
__device__ __forceinline__ __half2 odd_codes(uint32_t v, float less) {
  const uint32_t w = (v & 0x00f000f0u) | 0x64006400u;                // 1024 + 16 n
  return __hfma2(*reinterpret_cast<const __half2*>(&w), __float2half2_rn(0.0625f), __float2half2_rn(-64.f - less));
}
// The biased exponent of a row's largest value or minimum, NaN passed over.
template <int NG>
__device__ __forceinline__ int top_exponent(const uint32_t (&meta)[NG]) {
  float top = 0.f;
#pragma unroll
  for (int k = 0; k < NG; ++k) {
    float s, m;
    group_meta<NG>(meta, k, s, m);
    top = fmaxf(top, fminf(fmaxf(fabsf(m), fabsf(fmaf(15.f, s, m))), 3.0e38f));
  }
  return min(max(__float_as_int(top) >> 23, 15), 254);
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

template <int D, int NG, bool kSplit>
__global__ void __launch_bounds__(kThreads, 1) k_attn_prefix(const __grid_constant__ PrefixParams pp) {
  using S = PrefixSmem<D, kSplit>;
  constexpr int kRows = 128 * S::tiles, C = D / 32, PG = C / NG, TB = TileShape{D, NG}.bytes();
  constexpr TileShape ts{D, NG};
  const SharedParams& p = pp.a;
  extern __shared__ uint8_t dynamic[];
  uint8_t* smem = dynamic + ((1024u - (smem_u32(dynamic) & 1023u)) & 1023u);
  __shared__ __align__(16) PrefixShared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    mbar_init(&sh.q, 8);
    for (int i = 0; i < S::slots; ++i) {
      mbar_init(&sh.ready[i], 8);
      mbar_init(&sh.free[i], 1);
    }
    for (int m = 0; m < 2; ++m) {
      mbar_init(&sh.s[m][0], 1);
      mbar_init(&sh.s[m][1], 1);
      mbar_init(&sh.p[m][0], 4);
      mbar_init(&sh.p[m][1], 4);
      mbar_init(&sh.pv[m], 1);
    }
    mbar_init(&sh.done, 1);
    sh.abort = 0;
    fence_mbar_init();
  }
  // This launch reads nothing that the one before it, over the own tokens, writes, and that one lets it
  // begin only once all before are done; it ends after it, for the join behind both.
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (warp == kPlanWarp) {
    const GroupPlan g = group_plan(p, kRows, pp.ctas, int(blockIdx.x), lane);
    if (lane == 0) sh.plan = g;
  }
  if (warp == kIssueWarp) take_columns(smem_u32(&sh.tmem));
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = sh.tmem;
  const GroupPlan plan = sh.plan;
  if (plan.group < 0) {                           // no item: the same for the whole CTA
    if (blockIdx.x == 0 && warp == kPlanWarp) group_plan(p, kRows, pp.ctas, 0, lane, pp.plans);
    if (warp == kIssueWarp) give_columns(tmem);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    return;
  }
  const int local = int(blockIdx.x) - plan.first, hp = local / plan.row_blocks, part = hp % plan.parts, h = hp / plan.parts;
  const int r0 = (local - hp * plan.row_blocks) * kRows, rows = min(plan.count * p.group - r0, kRows);
  const int all = ceil_div(plan.len, kPos);
  const int first = int(int64_t(all) * part / plan.parts), n = int(int64_t(all) * (part + 1) / plan.parts) - first;      // tiles, > 0
  const int steps[2] = {kSplit ? (n + 1) / 2 : n, kSplit ? n / 2 : rows > 128 ? n : 0};
  const uint32_t smem_q = smem_u32(smem);
  auto s_cols = [&](int m, int i) { return tmem + uint32_t((2 * m + (i & 1)) * kPos); };
  auto o_cols = [&](int m) { return tmem + uint32_t(4 * kPos + m * 128); };

  if (warp >= kIssueWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
    if (warp == kIssueWarp) {
      // --- products ---
      const uint32_t q0 = operand(smem_q), qm0 = operand(smem_q + S::at_q_more);
      auto slot_of = [&](int t) { return smem_q + S::at_slots + t % S::slots * S::slot; };
      auto wait_tile = [&](int t) { return role_wait(&sh.ready[t % S::slots], (t / S::slots) & 1, &sh.abort, p.status); };
      auto issue_s = [&](int m, int i, int t) {
        fence_after();
        if (elected()) {
          const uint32_t k0 = operand(slot_of(t)), km0 = operand(slot_of(t) + S::k + S::v), d = s_cols(m, i);
          const uint32_t a0 = q0 + (kSplit ? 0 : m * (S::q >> 4)), am0 = qm0 + (kSplit ? 0 : m * (S::q_more >> 4));
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            multiply<kRows128, shape_of(kPos)>(d, a0 + (((k / 4) * kHalf + (k & 3) * 32) >> 4),
                                               k0 + (((k / 4) * (kPos * 128) + (k & 3) * 32) >> 4), k > 0);
          multiply<kRows32, shape_of(kPos)>(d, am0, km0, true);
          commit(&sh.s[m][i & 1]);
        }
        __syncwarp();
      };
      auto issue_o = [&](int m, int i, int t) {
        fence_after();
        if (elected()) {
          const uint32_t v0 = operand(slot_of(t) + S::k);
#pragma unroll
          for (int k = 0; k < kPos / 16; ++k)
            multiply_from<kRows128, shape_of(D)>(o_cols(m), s_cols(m, i) + k * 8, v0 + ((k * 32) >> 4), i > 0 || k > 0);
          commit(&sh.pv[m]);
        }
        __syncwarp();
      };
      auto tile_of = [&](int m, int i) { return kSplit ? 2 * i + m : i; };
      bool ok = role_wait(&sh.q, 0, &sh.abort, p.status);
      for (int m = 0; m < 2 && ok; ++m) {
        if (steps[m] == 0) continue;
        ok = wait_tile(tile_of(m, 0));
        if (ok) issue_s(m, 0, tile_of(m, 0));
      }
      // S of a stream's next tile goes out before O of the last, whose weights take longer
#pragma unroll 1
      for (int i = 0; i < steps[0] && ok; ++i) {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          if (i >= steps[m] || !ok) continue;
          const int t = tile_of(m, i);
          if (i + 1 < steps[m]) {
            ok = wait_tile(tile_of(m, i + 1));
            if (!ok) break;
            issue_s(m, i + 1, tile_of(m, i + 1));
          }
          ok = role_wait(&sh.p[m][i & 1], (i >> 1) & 1, &sh.abort, p.status);
          if (!ok) break;
          issue_o(m, i, t);
          if (kSplit || m == 1 || steps[1] == 0) {
            if (elected()) commit(&sh.free[t % S::slots]);
            __syncwarp();
          }
        }
      }
      if (elected()) commit(&sh.done);
      __syncwarp();
      if (!ok) mbar_wait_bounded(&sh.done, 0);
    } else if (warp == kPlanWarp && blockIdx.x == 0) {
      group_plan(p, kRows, pp.ctas, 0, lane, pp.plans);
    }
  } else if (warp >= kUnpackWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsUnpack));
    // --- unpacking: warp w takes K (even) or V (odd) of cache tile w / 2 ---
    const int uw = warp - kUnpackWarp, sub = uw >> 1, g = lane >> 2, t4 = lane & 3;
    const bool values = uw & 1;
    const int tpp = p.page_tokens / kTile;
    const int32_t* table = p.page_table + int64_t(plan.group) * p.table_pages;
    const int tiles = ceil_div(plan.len, kTile);                   // cache tiles held
    auto page_of = [&](int i) {                   // of this warp's cache tile of tile i
      const int tile = (first + i) * kSub + sub;
      return i < n && tile < tiles ? __ldg(table + tile / tpp) : -1;
    };
    uint32_t there = 0;                           // bit i & 7: the cache tile of tile i exists
    // The warp's packed rows of tile i, 16 bytes a lane and copy; a group of copies whether there are any or not
    auto fetch = [&](int i, int page) {
      const int tile = (first + i) * kSub + sub;
      bool ok = i < n && tile < tiles;
      if (ok && (page < 0 || page >= p.n_pages)) {
        if (lane == 0) report_status(p.status, kStatusBadIndex);
        ok = false;
      }
      there = (there & ~(1u << (i & 7))) | uint32_t(ok) << (i & 7);
      if (ok) {
        const uint8_t* src = p.pages + ((int64_t(page) * p.kv_heads + h) * tpp + tile % tpp) * int64_t(TB) + (values ? TB / 2 : 0);
        const uint32_t dst = smem_q + S::at_raw + (i % kAhead) * S::raw + uw * kMostPacked;
#pragma unroll
        for (int k = 0; k < (TB / 32 + 31) / 32; ++k)
          if (32 * k + lane < TB / 32) copy16(dst + (32 * k + lane) * 16, src + (32 * k + lane) * 16);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int most = 0;                                 // the largest exponent of a value that the warp has met
    auto unpack = [&](int i, int slot) {
      const uint8_t* src = smem + S::at_raw + (i % kAhead) * S::raw + uw * kMostPacked;
      const int left = (there >> (i & 7)) & 1 ? plan.len - ((first + i) * kSub + sub) * kTile : 0;       // rows that exist
      uint8_t* at = smem + S::at_slots + slot * S::slot;
      // the row's exponent, found by lane row, and what the softmax takes of it
      int mine = 15;
      if (lane < kTile && lane < left) {
        uint32_t meta[NG];
        load_words<NG>(meta, src + ts.codes() + lane * 4 * NG);
        mine = top_exponent<NG>(meta);
      }
      if (!values) {
        if (lane < kTile) sh.up[slot][sub * kTile + lane] = up(mine);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int row = g + 8 * j, tk = sub * kTile + row;
          uint32_t words[C] = {}, meta[NG] = {};
          if (row < left) {
            load_words<C>(words, src + row * (D / 2) + t4 * (D / 8));
            load_words<NG>(meta, src + ts.codes() + row * 4 * NG);
          }
          const float f = down(__shfl_sync(0xffffffffu, mine, row));
#pragma unroll
          for (int k = 0; k < NG; ++k) {
            float s, m;
            group_meta<NG>(meta, k, s, m);
            const __half2 s2 = __float2half2_rn(s * f);
#pragma unroll
            for (int c = k * PG; c < (k + 1) * PG; ++c) {
              const uint32_t w = words[c];
              // dims 0, 4, 1, 5, 2, 6, 3, 7 of the word's eight
              const uint4 v = make_uint4(bits(__hmul2(even_codes(w, 8.f), s2)), bits(__hmul2(odd_codes(w, 8.f), s2)),
                                         bits(__hmul2(even_codes(w >> 8, 8.f), s2)), bits(__hmul2(odd_codes(w >> 8, 8.f), s2)));
              const int word = 4 * c + t4;
              *reinterpret_cast<uint4*>(at + (word >> 3) * (kPos * 128) + tk * 128 + (((word & 7) ^ (tk & 7)) << 4)) = v;
            }
          }
          // the groups' m + 8 s: first planes (t4 = 0), second planes (1), first again (2), nothing (3)
          float plane[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < NG; ++k) {
            float s, m;
            group_meta<NG>(meta, k, s, m);
            const float x = fmaf(8.f, s, m) * f, top = __half2float(__float2half_rn(x));
            plane[k] = t4 == 3 ? 0.f : t4 == 1 ? x - top : top;
          }
          *reinterpret_cast<uint2*>(at + S::k + S::v + tk * 32 + (((t4 >> 1) ^ ((tk >> 2) & 1)) << 4) + (t4 & 1) * 8) =
              make_uint2(pack_f16(plane[0], plane[1]), pack_f16(plane[2], plane[3]));
        }
      } else {
        most = max(most, int(__reduce_max_sync(0xffffffffu, uint32_t(mine))));
        mine = max(mine, max(most - kLeastBelow, kLeastExponent));
        if (lane < kTile) {
          sh.c[slot][sub * kTile + lane] = lane < left ? float(mine - 141) : -INFINITY;
          sh.inv[slot][sub * kTile + lane] = down(mine);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int pair = t4 + 4 * j, tk = sub * kTile + 2 * pair;
          uint32_t words[C] = {}, meta0[NG] = {}, meta1[NG] = {};
          if (2 * pair < left) {
            load_words<C>(words, src + pair * D + ts.v_place(pair, g) * (D / 8));
            load_words<NG>(meta0, src + ts.codes() + 2 * pair * 4 * NG);
          }
          if (2 * pair + 1 < left) load_words<NG>(meta1, src + ts.codes() + (2 * pair + 1) * 4 * NG);
          const float fa = down(__shfl_sync(0xffffffffu, mine, 2 * pair)), fb = down(__shfl_sync(0xffffffffu, mine, 2 * pair + 1));
#pragma unroll
          for (int k = 0; k < NG; ++k) {
            float sa, ma, sb, mb;
            group_meta<NG>(meta0, k, sa, ma);
            group_meta<NG>(meta1, k, sb, mb);
            const __half2 s2 = __floats2half2_rn(sa * fa, sb * fb), m2 = __floats2half2_rn(ma * fa, mb * fb);
#pragma unroll
            for (int c = k * PG; c < (k + 1) * PG; ++c) {
              const uint32_t w = words[c];
              const __half2 v[4] = {__hfma2(even_codes(w, 0.f), s2, m2), __hfma2(odd_codes(w, 0.f), s2, m2),
                                    __hfma2(even_codes(w >> 8, 0.f), s2, m2), __hfma2(odd_codes(w >> 8, 0.f), s2, m2)};
              // dim 32c + 4g + i in row 32c + 8i + g: lanes of one store in eight rows, as many 16-byte words
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int row = 32 * c + 8 * i + g;
                *reinterpret_cast<uint32_t*>(at + S::k + row * 128 + (((tk >> 3) ^ (row & 7)) << 4) + (tk & 7) * 2) = bits(v[i]);
              }
            }
          }
        }
      }
    };
    bool ok = true;
#pragma unroll 1
    for (int i = 0; i < kAhead - 1; ++i) fetch(i, page_of(i));
    int page = page_of(kAhead - 1);               // of the next to fetch, asked for a tile ahead
#pragma unroll 1
    for (int i = 0; i < n && ok; ++i) {
      const int slot = i % S::slots;
      __syncwarp();                               // (all lanes have read what lay there)
      fetch(i + kAhead - 1, page);
      page = page_of(i + kAhead);
      if (i >= S::slots) ok = role_wait(&sh.free[slot], (i / S::slots - 1) & 1, &sh.abort, p.status);
      if (!ok) break;
      asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
      __syncwarp();
      unpack(i, slot);
      fence_proxy_async_smem();
      role_arrive(&sh.ready[slot]);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");        // (a wait that gave up leaves some)
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    // --- the softmax, a row a thread ---
    const int m = warp >> 2, rt = (warp & 3) * 32 + lane;
    const uint32_t lanes = uint32_t((warp & 3) * 32) << 16;
    float cq = 0.f;
    {
      // The block's queries, to where they will lie: lanes along the rows, 16 bytes each, all under way at once.
      // (A row a thread, 32 lines a load: 32 sequences behind 131072 positions 180 us for 175.)  Two streams have one block of rows: a half of it each.
      constexpr int kWords = D / 8, kEach = kSplit ? 16 : 32;
      auto place = [&](int row, int k) {          // word k (dims 8k .. 8k + 7) of a row of this warp's block
        return (kSplit ? 0 : m * S::q) + row * 128 + (k >> 3) * kHalf + (((k & 7) ^ (row & 7)) << 4);
      };
#pragma unroll 1
      for (int i = lane / kWords; i < kEach; i += 32 / kWords) {
        const int own = (warp & 3) * 32 + (kSplit ? m * 16 : 0) + i, k = lane % kWords, at = (kSplit ? 0 : m * 128) + own;
        uint8_t* const to = smem + place(own, k);
        const uint16_t* e = static_cast<const uint16_t*>(p.q);
        if (at < rows) e += (plan.q0 + (r0 + at) / p.group) * p.q_token + int64_t(h * p.group + (r0 + at) % p.group) * p.q_head + 8 * k;
        if (at < rows && p.q_wide)
          copy16(smem_u32(to), e);
        else if (at < rows)
          *reinterpret_cast<uint4*>(to) = make_uint4(e[0] | uint32_t(e[1]) << 16, e[2] | uint32_t(e[3]) << 16,
                                                     e[4] | uint32_t(e[5]) << 16, e[6] | uint32_t(e[7]) << 16);
        else
          *reinterpret_cast<uint4*>(to) = make_uint4(0u, 0u, 0u, 0u);
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      if (kSplit) asm volatile("bar.sync 1, 256;" ::: "memory");
      else __syncwarp();
    }
    if (!kSplit || m == 0) {
      // The row's query in place, scaled below 2^8 (128 of them sum up within fp16), in the order of the keys' dims.
      // In short loops, as all code that runs once here is: straight on, every 128 bytes of it are waited for.
      uint8_t* const row = smem + m * S::q + rt * 128;
      auto word = [&](int k) { return reinterpret_cast<uint4*>(row + (k >> 3) * kHalf + (((k & 7) ^ (rt & 7)) << 4)); };
      auto eight = [&](int k, float (&x)[8]) {    // dims 8k .. 8k + 7
        const uint4 v = *word(k);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 f = p.q_f16 ? __half22float2(*reinterpret_cast<const __half2*>(&w[j])) : bf16x2_to_float2(w[j]);
          x[2 * j] = f.x;
          x[2 * j + 1] = f.y;
        }
      };
      float top = 0.f;
#pragma unroll 2
      for (int k = 0; k < D / 8; ++k) {
        float x[8];
        eight(k, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[j]));
      }
      const int e = 134 - min(max(__float_as_int(top) >> 23, 1), 254), e1 = e >> 1, e2 = e - e1;
      const float f1 = __int_as_float((127 + e1) << 23), f2 = __int_as_float((127 + e2) << 23);
      uint8_t* const more = smem + S::at_q_more + m * S::q_more + rt * 32;
      const int turn_word = ((rt >> 2) & 1) << 4;
      *reinterpret_cast<uint4*>(more) = make_uint4(0u, 0u, 0u, 0u);
      *reinterpret_cast<uint4*>(more + 16) = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 1
      for (int n0 = 0; n0 < NG; ++n0) {
        float sum = 0.f;
#pragma unroll 2
        for (int k = n0 * (D / 8 / NG); k < (n0 + 1) * (D / 8 / NG); ++k) {
          float x[8];
          eight(k, x);
          uint32_t held[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {           // dims 0, 4, 1, 5, 2, 6, 3, 7 of eight
            held[j] = pack_f16(x[j] * f1 * f2, x[4 + j] * f1 * f2);
            const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&held[j]));
            sum += y.x + y.y;
          }
          *word(k) = make_uint4(held[0], held[1], held[2], held[3]);
        }
        // against the keys' planes: first planes twice, then what they left over
        const __half first_plane = __float2half_rn(sum), rest = __float2half_rn(sum - __half2float(first_plane));
        __half* at = reinterpret_cast<__half*>(more);
        at[turn_word / 2 + n0] = first_plane;
        at[turn_word / 2 + 4 + n0] = first_plane;
        at[(16 ^ turn_word) / 2 + n0] = rest;
      }
      cq = p.scale2 * __int_as_float((127 - e1) << 23) * __int_as_float((127 - e2) << 23);
      if (kSplit) sh.cq[rt] = cq;
      fence_proxy_async_smem();
    }
    if (kSplit) {
      asm volatile("bar.sync 1, 256;" ::: "memory");
      cq = sh.cq[rt];
    }
    role_arrive(&sh.q);
    const int mine = steps[m];
    float ref = kNoRef, l = 0.f;
    bool ok = true;
#pragma unroll 1
    for (int i = 0; i < mine; ++i) {
      ok = role_wait(&sh.s[m][i & 1], (i >> 1) & 1, &sh.abort, p.status);
      if (!ok) break;
      fence_after();
      const int slot = (kSplit ? 2 * i + m : i) % S::slots;
      float x[kPos];
      load64(s_cols(m, i) + lanes, x);
      landed64(x);
      const float4* up4 = reinterpret_cast<const float4*>(sh.up[slot]);
      const float4* c4 = reinterpret_cast<const float4*>(sh.c[slot]);
      const float4* inv4 = reinterpret_cast<const float4*>(sh.inv[slot]);
      // logits with the values' scale, the largest, then weights in place and the sum of the weights alone
      float top = -INFINITY;
#pragma unroll
      for (int k = 0; k < kPos; k += 4) {
        const float4 u = up4[k / 4], c = c4[k / 4];
        const float2 a = ffma2(make_float2(x[k], x[k + 1]), fmul2(make_float2(u.x, u.y), make_float2(cq, cq)), make_float2(c.x, c.y));
        const float2 b = ffma2(make_float2(x[k + 2], x[k + 3]), fmul2(make_float2(u.z, u.w), make_float2(cq, cq)), make_float2(c.z, c.w));
        x[k] = a.x;
        x[k + 1] = a.y;
        x[k + 2] = b.x;
        x[k + 3] = b.y;
        asm("max.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(a.x), "f"(a.y));
        asm("max.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(b.x), "f"(b.y));
      }
      float keep = 1.f;
      if (__any_sync(0xffffffffu, top - ref > 13.f)) {
        const float now = fmaxf(ref, top - 6.f);
        keep = exp2f(ref - now);
        ref = now;
      }
      float2 l2 = make_float2(0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kPos; k += 4) {
        const float4 v = inv4[k / 4];
        const float2 a = fadd2(make_float2(x[k], x[k + 1]), make_float2(-ref, -ref));
        const float2 b = fadd2(make_float2(x[k + 2], x[k + 3]), make_float2(-ref, -ref));
        x[k] = exp2_fast(a.x);
        x[k + 1] = exp2_fast(a.y);
        x[k + 2] = exp2_fast(b.x);
        x[k + 3] = exp2_fast(b.y);
        l2 = ffma2(make_float2(x[k], x[k + 1]), make_float2(v.x, v.y), l2);
        l2 = ffma2(make_float2(x[k + 2], x[k + 3]), make_float2(v.z, v.w), l2);
      }
      l = l * keep + (l2.x + l2.y);
      if (i > 0 && __any_sync(0xffffffffu, keep != 1.f)) {
        ok = role_wait(&sh.pv[m], (i - 1) & 1, &sh.abort, p.status);
        if (!ok) break;
        fence_after();
#pragma unroll 1
        for (int c = 0; c < D / 16; ++c) {
          float v[16];
          load16(o_cols(m) + lanes + 16 * c, v);
          landed();
          defined16(v);
#pragma unroll
          for (int k = 0; k < 16; ++k) v[k] *= keep;
          store16(o_cols(m) + lanes + 16 * c, v);
        }
      }
      uint32_t w[32];
#pragma unroll
      for (int k = 0; k < 32; ++k) w[k] = pack_f16(x[2 * k], x[2 * k + 1]);
      store32(s_cols(m, i) + lanes, w);
      stored();
      fence_before();
      role_arrive(&sh.p[m][i & 1]);
    }
    if (ok) ok = role_wait(&sh.done, 0, &sh.abort, p.status);
    fence_after();
    asm volatile("bar.sync 1, 256;" ::: "memory");        // all products are done: their operands' memory is free
    // --- the records: outputs as they are, each row's reference and sum.  Through shared memory (word u of row
    // r at u ^ r, on banks of their own), so that a warp writes whole rows ---
    const bool seen = mine > 0 && ok && (ref != kNoRef || l != 0.f);
    const int64_t slot = (kSplit ? 2 * int64_t(blockIdx.x) : int64_t(blockIdx.x)) * kRows;       // (a record a stream)
    if ((kSplit ? rt : m * 128 + rt) < rows) pp.sums[slot + m * 128 + rt] = make_float2(seen ? ref : -INFINITY, l);
    float4* held = reinterpret_cast<float4*>(smem) + (m * 128 + (warp & 3) * 32) * (D / 4);      // the warp's 32 rows
    const int there = min(max((kSplit ? rows : rows - m * 128) - (warp & 3) * 32, 0), 32);
    if (mine > 0 && ok) {
#pragma unroll 1
      for (int c = 0; c < C; ++c) {
        float o[32];
        load16(o_cols(m) + lanes + 32 * c, o);
        load16(o_cols(m) + lanes + 32 * c + 16, o + 16);
        landed();
        defined16(o);
        defined16(o + 16);
        // dims 4k .. 4k + 3 of the 32 came as columns k, 8 + k, ..
#pragma unroll
        for (int k = 0; k < 8; ++k)
          held[lane * (D / 4) + ((8 * c + k) ^ (lane & (D / 4 - 1)))] = make_float4(o[k], o[8 + k], o[16 + k], o[24 + k]);
      }
      __syncwarp();
      float4* out = reinterpret_cast<float4*>(pp.records + (slot + m * 128 + (warp & 3) * 32) * D);
#pragma unroll 4
      for (int i = lane; i < there * (D / 4); i += 32) {
        const int r1 = i / (D / 4), u = i % (D / 4);
        out[i] = held[r1 * (D / 4) + (u ^ (r1 & (D / 4 - 1)))];
      }
    }
  }
  fence_before();
  __syncthreads();
  fence_after();
  if (warp == kIssueWarp) give_columns(tmem);
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

template <int D, int NG, bool kSplit>
cudaError_t launch(const PrefixParams& pp, int items, int dev, cudaStream_t s) {
  // the kernel's shared memory limit, raised once a device
  static std::atomic<uint64_t> raised{0};
  const uint64_t bit = dev >= 0 && dev < 64 ? uint64_t(1) << dev : 0;
  if (!(raised.load(std::memory_order_relaxed) & bit) || !bit) {
    const cudaError_t err = cudaFuncSetAttribute(k_attn_prefix<D, NG, kSplit>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 PrefixSmem<D, kSplit>::bytes);
    if (err != cudaSuccess) return err;
    raised.fetch_or(bit, std::memory_order_relaxed);
  }
  return launch_early(k_attn_prefix<D, NG, kSplit>, unsigned(items), kThreads, PrefixSmem<D, kSplit>::bytes, s, pp);
}

template <bool kSplit>
cudaError_t dispatch(const PrefixParams& pp, int items, int d, int group, int dev, cudaStream_t s) {
  if (d == 128 && group == 32) return launch<128, 4, kSplit>(pp, items, dev, s);
  if (d == 128 && group == 64) return launch<128, 2, kSplit>(pp, items, dev, s);
  if (d == 128) return launch<128, 1, kSplit>(pp, items, dev, s);
  if (group == 32) return launch<64, 2, kSplit>(pp, items, dev, s);
  return launch<64, 1, kSplit>(pp, items, dev, s);
}

}  // namespace

cudaError_t launch_attn_groups(const SharedParams& p, int mt, int items, int ctas, int d, int quant_group, int dev, float* records,
                               GroupPlan* plans, cudaStream_t s) {
  PrefixParams pp{};
  pp.a = p;
  pp.a.page_table = p.prefix_table;               // the kernel has groups for sequences
  pp.a.pages = p.prefix_data;
  pp.a.status = p.prefix_status;
  pp.a.n_pages = p.prefix_n_pages;
  pp.a.table_pages = p.prefix_pages;
  pp.plans = plans;
  pp.records = records;
  pp.sums = reinterpret_cast<float2*>(p.prefix_ref);
  pp.ctas = ctas;
  return mt == 1 ? dispatch<true>(pp, items, d, quant_group, dev, s) : dispatch<false>(pp, items, d, quant_group, dev, s);
}

}  // namespace reskv
