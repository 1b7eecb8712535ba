// Attention of every sequence's newest tokens over its paged 4-bit cache
// (reskv_paged_attn).
#include <atomic>
#include <cmath>

#include "paged_attn.cuh"

namespace reskv {
namespace {

// --- few query rows: one warp, one block of rows ---------------------------
//
// A call's work is a list of units, one per (sequence, block of 8 query rows, KV
// head), each a run of 16-token tiles.  The tiles of all units, laid end to end,
// are cut into equal pieces, one per warp, whatever the sequences' lengths: a
// warp finishes the units that lie in its piece, a unit cut between warps of a
// CTA is joined in shared memory, one cut between CTAs by the last of them to
// arrive (records in order, so the result does not depend on the arrival).  Every CTA
// works the cut out for itself from the lengths, which only the device knows.
//
// One more warp feeds all the others: its lane w keeps warp w's ring of tiles
// full, one bulk copy per tile, so that page lookups and copies cost the tile
// step nothing.
constexpr int kAttnWarps = 15;                      // computing; with the feeding warp 16, of 128 registers
constexpr int kAttnStages = 2;                    // of a warp's ring
constexpr int kStageTiles = 2;                    // neighbours within a page, one copy
constexpr int kSettleStages = 8;                  // taken between two settle()s
constexpr int kMinTiles = 2;                      // of a piece, before more CTAs are used
constexpr int kWholeTiles = 135;                  // 9 a warp

struct RecordInfo {
  int64_t start;                                  // first tile of the record's unit
  Sequence s;
  int tiles, r0, h;
  int present;
};

__host__ __device__ constexpr int record_stride(int d) { return d + 4; }          // floats of a row: spreads rows over banks
__host__ __device__ constexpr int record_floats(int d, int rows) { return rows * record_stride(d); }

template <int D, int NG, int R>
struct AttnSmem {
  static constexpr int ring = kAttnWarps * kAttnStages * kStageTiles * TileShape{D, NG}.bytes();
  static constexpr int heads = kAttnWarps * record_floats(D, R) * 4;
  static constexpr int refs = 2 * kAttnWarps * R * 4;
  static constexpr int info = 2 * kAttnWarps * int(sizeof(RecordInfo));
  static constexpr int bars = 2 * kAttnWarps * kAttnStages * 8;
  static constexpr int counts = kAttnWarps * kAttnStages * 4;
  static constexpr int fixed = (ring + heads + refs + info + bars + counts + 16 + 15) / 16 * 16;
  static_assert((ring + heads + refs) % 8 == 0 && (ring + heads + refs + info) % 8 == 0 && ring % 16 == 0, "alignment");
  static_assert(kAttnStages * kStageTiles * TileShape{D, NG}.bytes() >= record_floats(D, R) * 4, "a drained ring holds a record");
  static int bytes(int batch) { return fixed + (batch + 1) * 8; }
};

// floor(i * n / parts), in 32 bits where they hold (an issue of instructions: every
// CTA works this out before its first copy).
__device__ __forceinline__ int64_t part_begin(int64_t i, int64_t n, int parts) {
  if (n < (1 << 22)) return int64_t(uint32_t(i) * uint32_t(n) / uint32_t(parts));
  return i * n / parts;
}
// The part that holds x.
__device__ __forceinline__ int part_of(int64_t x, int64_t n, int parts) {
  if (n < (1 << 22)) return int((uint32_t(x + 1) * uint32_t(parts) - 1) / uint32_t(n));
  return int(((x + 1) * parts - 1) / n);
}

// Tiles and units of all sequences before one, in one word.
constexpr int kUnitBits = 24;
__device__ __forceinline__ int64_t tiles_of(int64_t x) { return x >> kUnitBits; }
__device__ __forceinline__ int64_t units_of(int64_t x) { return x & ((int64_t(1) << kUnitBits) - 1); }

template <int R, bool kShared>
struct RowCursor {
  int b, r0, h, tile;                             // tile: within the unit
  Sequence s;
  RowBlock k;
  int64_t start;                                  // the unit's first tile among all

  __device__ __forceinline__ void block(const Params<kShared>& p) {
    const int rows = s.count * p.group;
    k = row_block(p, s, r0, min(r0 + R, rows));
  }
  __device__ void locate(const Params<kShared>& p, const int64_t* prefix, int64_t x) {
    int lo = 0, hi = p.batch;                     // tiles before lo <= x < tiles before hi
#pragma unroll 1
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (tiles_of(prefix[mid]) <= x) lo = mid;
      else hi = mid;
    }
    b = lo;
    s = sequence_of<kShared>(p, b);
    int64_t left = x - tiles_of(prefix[b]);
#pragma unroll 1
    for (r0 = 0;; r0 += R) {
      block(p);
      const int64_t n = int64_t(k.tiles) * p.kv_heads;
      if (left < n || r0 + R >= s.count * p.group) break;
      left -= n;
    }
    h = min(left < (int64_t(1) << 32) ? int(uint32_t(left) / uint32_t(k.tiles)) : int(left / k.tiles), p.kv_heads - 1);
    tile = int(left - int64_t(h) * k.tiles);
    start = x - tile;
  }
  // To the beginning of unit i, which exists.
  __device__ void locate_unit(const Params<kShared>& p, const int64_t* prefix, int64_t i) {
    int lo = 0, hi = p.batch;
#pragma unroll 1
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (units_of(prefix[mid]) <= i) lo = mid;
      else hi = mid;
    }
    b = lo;
    s = sequence_of<kShared>(p, lo);
    tile = 0;
    int left = int(i - units_of(prefix[lo]));
    start = tiles_of(prefix[lo]);
#pragma unroll 1
    for (r0 = 0;; r0 += R) {
      block(p);
      if (k.tiles == 0) continue;                 // no unit; the last block is one
      if (left < p.kv_heads) break;
      left -= p.kv_heads;
      start += int64_t(k.tiles) * p.kv_heads;
    }
    h = left;
    start += int64_t(h) * k.tiles;
  }
  __device__ void next(const Params<kShared>& p, const int64_t* prefix) {
    start += k.tiles;
    tile = 0;
    if (++h < p.kv_heads) return;
    h = 0;
    r0 += R;
    if (r0 >= s.count * p.group) {
#pragma unroll 1
      do ++b; while (b < p.batch && prefix[b + 1] == prefix[b]);        // nothing to do
      if (b >= p.batch) return;
      s = sequence_of<kShared>(p, b);
      r0 = 0;
    }
    block(p);
#pragma unroll 1
    while (k.tiles == 0 && r0 + R < s.count * p.group) {                  // rows before position 0
      r0 += R;
      block(p);
    }
  }
};


__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
  return ok != 0;
}

__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// one tile, read once: first out of L2
__device__ __forceinline__ void copy_tile(void* dst, const void* src, uint32_t bytes, uint64_t* bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::
          "r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)), "l"(policy)
      : "memory");
}

template <int D, int NG, bool kTwoPlanes, int R, bool kShared>
__global__ void __launch_bounds__((kAttnWarps + 1) * 32, 1) k_attn_rows(const __grid_constant__ Params<kShared> p) {
  using S = AttnSmem<D, NG, R>;
  using Cursor = RowCursor<R, kShared>;
  constexpr int kRows = R;
  constexpr TileShape ts{D, NG};
  constexpr int TB = ts.bytes(), SB = kStageTiles * TB, RS = record_stride(D), RF = record_floats(D, R);
  extern __shared__ __align__(128) uint8_t smem[];
  uint8_t* ring = smem;
  float* heads = reinterpret_cast<float*>(smem + S::ring);
  float* refs = reinterpret_cast<float*>(smem + S::ring + S::heads);
  RecordInfo* info = reinterpret_cast<RecordInfo*>(smem + S::ring + S::heads + S::refs);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::ring + S::heads + S::refs + S::info);
  uint64_t* vacant = full + kAttnWarps * kAttnStages;
  int* counts = reinterpret_cast<int*>(vacant + kAttnWarps * kAttnStages);
  int* shared_int = counts + kAttnWarps * kAttnStages;                 // [4]
  int64_t* prefix = reinterpret_cast<int64_t*>(smem + S::fixed);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) shared_int[2] = 0;
  if (threadIdx.x < 2 * kAttnWarps) info[threadIdx.x].present = 0;
  if (threadIdx.x < kAttnWarps * kAttnStages) {
    mbar_init(&full[threadIdx.x], 1);
    mbar_init(&vacant[threadIdx.x], 1);
  }
  fence_mbar_init();
  if (p.batch > 1) __syncthreads();
  wait_for_previous();

  // the tiles of every sequence, and what they sum up to
#pragma unroll 1
  for (int b = threadIdx.x; b < p.batch; b += blockDim.x) {
    const Sequence s = sequence_of<kShared>(p, b);
    const int rows = s.count * p.group;
    int64_t n = 0;
    int longest = 0, blocks = 0;
#pragma unroll 1
    for (int r0 = 0; r0 < rows; r0 += kRows) {
      const int k = row_block(p, s, r0, min(r0 + kRows, rows)).tiles;
      n += k;
      blocks += k > 0;
      longest = max(longest, k);
    }
    prefix[b + 1] = (n * p.kv_heads << kUnitBits) + int64_t(blocks) * p.kv_heads;
    if (p.batch == 1) shared_int[2] = longest;
    else atomicMax(&shared_int[2], longest);
  }
  __syncthreads();
  if (warp == 0) {
    int64_t sum = 0;
    if (lane == 0) prefix[0] = 0;
#pragma unroll 1
    for (int b = 0; b < p.batch; b += 32) {
      int64_t v = b + lane < p.batch ? prefix[b + lane + 1] : 0;
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const int64_t u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
      }
      if (b + lane < p.batch) prefix[b + lane + 1] = sum + v;
      sum += __shfl_sync(0xffffffffu, v, 31);
    }
  }
  __syncthreads();
  const int64_t N = tiles_of(prefix[p.batch]);
  int ctas = gridDim.x;
  if (N < int64_t(ctas) * kAttnWarps * kMinTiles) ctas = max(1, (int(N) + kAttnWarps * kMinTiles - 1) / (kAttnWarps * kMinTiles));
  const int cta = blockIdx.x;
  // Whole units to every CTA where that costs it few tiles more than equal pieces:
  // joining records across CTAs takes about the time of kWholeTiles tiles.
  const int units = int(units_of(prefix[p.batch]));
  const int whole_ctas = min(units, int(gridDim.x));
  const int64_t most = units ? int64_t((units + whole_ctas - 1) / whole_ctas) * shared_int[2] : 0;
  const bool whole = most <= part_begin(1, N, ctas) + kWholeTiles;
  if (whole) ctas = whole_ctas;
  const bool active = cta < ctas;
  if (!active && warp != kAttnWarps) return;      // a CTA without tiles only has rows without any to write
  int64_t c0, c1;                                 // this CTA's tiles
  Cursor unit{};                                  // its first unit, or (no tiles) not known
  if (!active) {
    c0 = c1 = 0;
  } else if (whole) {
    const int u0 = int(part_begin(cta, units, ctas)), u1 = int(part_begin(cta + 1, units, ctas));
    if (u1 > u0 + 1 && u1 < units) {
      unit.locate_unit(p, prefix, u1);
      c1 = unit.start;
    } else {
      c1 = N;
    }
    unit.locate_unit(p, prefix, u0);
    c0 = unit.start;
    if (u1 == u0 + 1) c1 = c0 + unit.k.tiles;
  } else {
    c0 = part_begin(cta, N, ctas);
    c1 = part_begin(cta + 1, N, ctas);
  }
  auto to_tile = [&](Cursor& c, int64_t x) {      // within the first unit without another search
    if (x - unit.start < unit.k.tiles && unit.k.tiles > 0) {
      c = unit;
      c.tile = int(x - unit.start);
    } else {
      c.locate(p, prefix, x);
    }
  };
  auto piece = [&](int w) { return c0 + part_begin(w, c1 - c0, kAttnWarps); };

  if (warp == kAttnWarps) {
    // --- the feeding warp: lane w for warp w ---
    // One turn of its loop serves every lane whose ring has a free stage; its length is
    // what a stage waits for, so a turn does little: sizes come in bytes, pages are
    // asked for one ahead.
    const int w = lane;
    int left = 0;                                 // tiles to feed
    Cursor c{};
    if (active && w < kAttnWarps) {
      const int64_t x = piece(w);
      left = int(piece(w + 1) - x);
      if (left > 0) to_tile(c, x);
    }
    uint64_t policy;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    const int tpp = p.page_tokens / kTile;        // tiles of a page
    const int64_t page_bytes = int64_t(p.kv_heads) * tpp * TB;
    const uint8_t* head = p.pages;                // the unit's head in page 0
    int64_t n_pages = p.n_pages;
    uint32_t* status = p.status;
    const uint8_t* src = head;                    // the next tile
    int in_unit = 0, in_page = 0;                 // tiles left of the unit and of the page, the next one included
    bool ok = false;                              // the page exists
    int page = 0;                                 // the page after this one, asked for a page ahead
    const int32_t* ask = p.page_table;
    auto turn_page = [&]() {                      // to `page`
      ok = uint32_t(page) < uint32_t(n_pages);
      if (!ok) report_status(status, kStatusBadIndex);
      src = head + (ok ? page : 0) * page_bytes;
      in_page = tpp;
      ++ask;
      if (in_unit > tpp) page = *ask;
    };
    auto begin_unit = [&]() {
      in_unit = c.k.tiles - c.tile;
      const int tile = c.k.first + c.tile, at = tile / tpp, first = tile - at * tpp;
      head = p.pages + int64_t(c.h) * tpp * TB;
      if constexpr (kShared) {
        n_pages = c.s.all ? p.prefix_n_pages : p.n_pages;
        status = c.s.all ? p.prefix_status : p.status;
        if (c.s.all) head = p.prefix_data + int64_t(c.h) * tpp * TB;
        ask = c.s.all ? p.prefix_table + int64_t(c.b - p.own) * p.prefix_pages + at : p.page_table + int64_t(c.b) * p.table_pages + at;
      } else {
        ask = p.page_table + int64_t(c.b) * p.table_pages + at;
      }
      page = *ask;
      in_unit += first;                           // as from the page's first tile
      turn_page();
      in_unit -= first;
      in_page -= first;
      src += first * TB;
    };
    if (left > 0) begin_unit();
    int st = 0;                                   // next stage
    uint32_t parity = 1;                          // of the vacancy to wait for: a fresh barrier passes
    int k = 0;                                    // stages fed
    long long t0 = clock64();
    uint32_t busy = __ballot_sync(0xffffffffu, left > 0);
#pragma unroll 1
    while (busy) {
      bool fed = false;
      const int at = w * kAttnStages + st;
      if (left > 0 && mbar_test(&vacant[at], parity)) {
        const int n = min(min(kStageTiles, left), min(in_page, in_unit));
        counts[at] = ok ? n : -n;
        if (ok) {
          mbar_arrive_expect_tx(&full[at], n * TB);
          copy_tile(ring + at * SB, src, n * TB, &full[at], policy);
        } else {
          mbar_arrive(&full[at]);
        }
        src += n * TB;
        ++k;
        left -= n;
        in_unit -= n;
        in_page -= n;
        if (++st == kAttnStages) {
          st = 0;
          parity ^= 1;
        }
        if (left > 0) {
          if (in_unit == 0) {
            c.next(p, prefix);
            begin_unit();
          } else if (in_page == 0) {
            turn_page();
          }
        }
        fed = true;
      }
      if (__any_sync(0xffffffffu, fed)) {
        t0 = clock64();
        busy = __ballot_sync(0xffffffffu, left > 0);
        continue;
      }
      __nanosleep(32);
      if (clock64() - t0 > kWaitLimitCycles) {
        // a warp stopped taking tiles: let the copies in flight land, feed no more
        if (lane == 0) report_status(p.status, kStatusWaitTimeout);
        if (w < kAttnWarps)
          for (int i = k > kAttnStages ? k - kAttnStages : 0; i < k; ++i)
            mbar_wait_bounded(&full[w * kAttnStages + i % kAttnStages], (i / kAttnStages) & 1);
        break;
      }
    }
    // The feeding done, zeros where rows see nothing: the blocks of rows that are no unit.
#pragma unroll 1
    for (int b = blockIdx.x; b < p.batch; b += gridDim.x) {
      const Sequence s = sequence_of<kShared>(p, b);
      if (position_of(s, 0) >= 0) continue;
      const int64_t rows = int64_t(s.count - s.len) * p.group;       // (of a group: it has no positions)
      const int r1 = s.len == 0 ? int(rows) : int(rows / kRows) * kRows;
#pragma unroll 1
      for (int64_t i = lane; i < int64_t(r1) * p.kv_heads * (D / 4); i += 32) {
        const int u = int(i % (D / 4));
        const int64_t hr = i / (D / 4);
        const int h = int(hr / r1), r = int(hr - int64_t(h) * r1);
        store_out<kShared>(p, s, h, r, u, make_float4(0.f, 0.f, 0.f, 0.f));
        if (u == 0) store_sum<kShared>(p, s, h, r, -INFINITY);
      }
    }
    if (!active) return;
  } else {
    // --- a computing warp ---
    int64_t x = piece(warp);
    const int64_t end = piece(warp + 1);
    Cursor c{};
    if (x < end) to_tile(c, x);
    TileStep<D, NG, kTwoPlanes, R> st;
    st.init(lane);
    int k = 0;
    bool failed = false;
#pragma unroll 1
    while (x < end && !failed) {
      const int n = int(min(int64_t(c.k.tiles - c.tile), end - x));
      const int rows = c.s.count * p.group;
      {
        const int r = c.r0 + (st.g & (R - 1));
        const void* row = nullptr;
        if (r < rows)
          row = static_cast<const uint16_t*>(p.q) + (c.s.q0 + r / p.group) * p.q_token +
                int64_t(c.h * p.group + r % p.group) * p.q_head;
        st.load_q(p, row);
      }
      // positions the lane's columns see; rows that do not exist see what the last one does
      int lo[2], hi[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        hi[j] = position_of(c.s, min(c.r0 + st.row(j), rows - 1) / p.group);
        lo[j] = first_seen(p, hi[j]);
      }
      const int all_hi = position_of(c.s, c.r0 / p.group);
      const int last = position_of(c.s, min(c.r0 + kRows - 1, rows - 1) / p.group);
      const int all_lo = first_seen(p, last);
      st.reset();
#pragma unroll 1
      for (int i = 0; i < n; ++k) {
        const int stage = warp * kAttnStages + k % kAttnStages;
        if (!__all_sync(0xffffffffu, mbar_wait_bounded(&full[stage], (k / kAttnStages) & 1))) {
          failed = true;
          break;
        }
        const int count = counts[stage];          // negative: a page that does not exist
        const uint8_t* tile = ring + stage * SB;
        int pos = (c.k.first + c.tile + i) * kTile;
#pragma unroll 1
        for (int j = 0; j < count; ++j, pos += kTile, tile += TB) {
          bool see[2][2] = {{true, true}, {true, true}};
          if (pos >= all_lo && pos + kTile - 1 <= all_hi) {
            st.template step<false>(tile, see);
          } else {
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
              for (int q = 0; q < 2; ++q) see[r][q] = pos + st.g + 8 * r >= lo[q] && pos + st.g + 8 * r <= hi[q];
            st.template step<true>(tile, see);
          }
        }
        i += abs(count);
        if (k % kSettleStages == kSettleStages - 1) st.settle();
        __syncwarp();
        if (lane == 0) mbar_arrive(&vacant[stage]);
      }
      if (failed) {
        if (lane == 0) report_status(p.status, kStatusWaitTimeout);
        break;
      }
      st.finish();
      const bool unit = c.tile == 0 && n == c.k.tiles;
      // else a record: begun before this piece, or cut off at its end
      const int slot = c.tile > 0 ? 0 : 1;
      float* rec = slot == 0 ? heads + warp * RF : reinterpret_cast<float*>(ring + warp * kAttnStages * SB);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = st.row(j);
#pragma unroll
        for (int b = 0; b < st.H; ++b) {
          const float4 v = make_float4(st.out(b, 0, j), st.out(b, 1, j), st.out(b, 2, j), st.out(b, 3, j));
          const int u = 8 * st.block(b) + st.g;
          if (!unit) *reinterpret_cast<float4*>(rec + r * RS + 4 * u) = v;
          else if (c.r0 + r < rows) store_out<kShared>(p, c.s, c.h, c.r0 + r, u, v);
        }
        if (st.g == 0 && st.half == 0) {
          if (!unit) refs[(2 * warp + slot) * kRows + r] = st.ref[j];
          else if (c.r0 + r < rows) store_sum<kShared>(p, c.s, c.h, c.r0 + r, st.ref[j]);
        }
      }
      if (!unit && lane == 0) info[2 * warp + slot] = RecordInfo{c.start, c.s, c.k.tiles, c.r0, c.h, 1};
      x += n;
      if (x < end) c.next(p, prefix);
    }
  }
  __syncthreads();

  // --- join the records: runs of one unit, in order; its rows to as many warps ---
  const bool present = lane < 2 * kAttnWarps && info[lane].present;
  const int64_t start = present ? info[lane].start : -1;
  const uint32_t have = __ballot_sync(0xffffffffu, present);
  const uint32_t below = have & ((1u << lane) - 1);
  const int64_t before = __shfl_sync(0xffffffffu, start, below ? 31 - __clz(below) : lane);
  const uint32_t begins = __ballot_sync(0xffffffffu, present && (!below || before != start));
  if (!begins) return;                            // the same in every warp
  auto cut = [&](const RecordInfo& r) { return r.start < c0 || r.start + r.tiles > c1; };
  // One run: each of its rows to `across` warps, which share its dims.  More: each row
  // to one warp, runs in turn.  Lane = lanes e + i takes dims 4i .. 4i + 3 of a
  // warp's share, of every `apart`-th record from e on.
  constexpr int kAcross = 16 / kRows;
  const int across = (begins & (begins - 1)) == 0 ? kAcross : 1;
  const int lanes = D / 4 / across, apart = 32 / lanes, every = lane / lanes;
  const int row = across == 1 ? warp % kRows : warp / kAcross;
  const int u = (across == 1 ? 0 : warp % kAcross * lanes) + lane % lanes;               // dims 4u .. 4u + 3
  auto all_lanes = [&](float4 a, int from) {
#pragma unroll 1
    for (int o = from; o < 32; o *= 2) {
      a.x += __shfl_xor_sync(0xffffffffu, a.x, o);
      a.y += __shfl_xor_sync(0xffffffffu, a.y, o);
      a.z += __shfl_xor_sync(0xffffffffu, a.z, o);
      a.w += __shfl_xor_sync(0xffffffffu, a.w, o);
    }
    return a;
  };
  int turn_of = 0;
#pragma unroll 1
  for (uint32_t m = begins; m; m &= m - 1, ++turn_of) {
    if (across == 1 && turn_of % kAcross != warp / kRows) continue;
    const int first = __ffs(m) - 1;
    const uint32_t after = m & (m - 1);
    const int stop = after ? __ffs(after) - 1 : 32;
    const RecordInfo& ri = info[first];
    if (ri.r0 + row >= ri.s.count * p.group) continue;
    const bool mine = lane >= first && lane < stop && ((have >> lane) & 1);
    const Joined j = join_weights(mine ? refs[lane * kRows + row] : -INFINITY);
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int e0 = first; e0 < stop; e0 += apart) {
      const int i = e0 + every;
      const float f = __shfl_sync(0xffffffffu, j.weight, i & 31);
      const float* rec = (i & 1) ? reinterpret_cast<const float*>(ring + (i >> 1) * kAttnStages * SB) : heads + (i >> 1) * RF;
      if (i < stop && ((j.present >> i) & 1)) add_scaled(a, f, *reinterpret_cast<const float4*>(rec + row * RS + 4 * u));
    }
    a = all_lanes(a, lanes);
    if (!cut(ri)) {
      if (every == 0) store_out<kShared>(p, ri.s, ri.h, ri.r0 + row, u, a);
      if (lane == 0 && u == 0) store_sum<kShared>(p, ri.s, ri.h, ri.r0 + row, j.ref);
    } else {
      float* rec = p.partials + (cta * 2 + (ri.start >= c0 ? 1 : 0)) * (RF + kRows);
      if (every == 0) *reinterpret_cast<float4*>(rec + row * RS + 4 * u) = a;
      if (lane == 0 && u == 0) rec[RF + row] = j.ref;
    }
  }
  // units cut between CTAs: at most the first and the last run
  const int run_a = __ffs(begins) - 1, run_b = 31 - __clz(begins);
  const bool cut_a = cut(info[run_a]), cut_b = run_b != run_a && cut(info[run_b]);
  if (!cut_a && !cut_b) return;
  __syncthreads();
  if (threadIdx.x < 2) {
    const RecordInfo& ri = info[threadIdx.x ? run_b : run_a];
    int last = 0;
    if (threadIdx.x ? cut_b : cut_a) {
      const int a0 = part_of(ri.start, N, ctas), a1 = part_of(ri.start + ri.tiles - 1, N, ctas);
      __threadfence();                            // the CTA's records, ordered by the barrier
      last = atomicAdd(&p.tickets[a0], 1) == a1 - a0;
      if (last) p.tickets[a0] = 0;
      __threadfence();
    }
    shared_int[threadIdx.x] = last;
  }
  __syncthreads();
  constexpr int kLanes = D / 4 / kAcross, kEvery = 32 / kLanes;         // a row to kAcross warps
  const int row2 = warp / kAcross, every2 = lane / kLanes, u2 = warp % kAcross * kLanes + lane % kLanes;
#pragma unroll 1
  for (int which = 0; which < 2; ++which) {
    if (!shared_int[which]) continue;
    const RecordInfo& ri = info[which ? run_b : run_a];
    if (ri.r0 + row2 >= ri.s.count * p.group) continue;
    const int a0 = part_of(ri.start, N, ctas), n = part_of(ri.start + ri.tiles - 1, N, ctas) - a0 + 1;
    // record i of the unit: the CTA it begins in keeps it second, the others first
    auto record = [&](int i) { return p.partials + ((a0 + i) * 2 + (i == 0 ? 1 : 0)) * (RF + kRows); };
    Joined all{0.f, -INFINITY, 0u};
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += 32) {
      const float ref = i0 + lane < n ? __ldcg(record(i0 + lane) + RF + row2) : -INFINITY;
      const Joined j = join_weights(ref);
      float4 b = make_float4(0.f, 0.f, 0.f, 0.f);
      const int stop = min(32, n - i0);
#pragma unroll 2
      for (int e0 = 0; e0 < stop; e0 += kEvery) {
        const int i = e0 + every2;
        const float f = __shfl_sync(0xffffffffu, j.weight, i & 31);
        const float4 v = i < stop ? __ldcg(reinterpret_cast<const float4*>(record(i0 + i) + row2 * RS + 4 * u2))
                                  : make_float4(0.f, 0.f, 0.f, 0.f);
        add_scaled(b, f, i < stop && ((j.present >> i) & 1) ? v : make_float4(0.f, 0.f, 0.f, 0.f));
      }
      b = all_lanes(b, kLanes);
      if (n <= 32) {
        a = b;
        all = j;
      } else {                                    // join the 32 with those before
        const float two = lane == 0 ? all.ref : lane == 1 ? j.ref : -INFINITY;
        const Joined k = join_weights(two);
        const float fa = __shfl_sync(0xffffffffu, k.weight, 0), fb = __shfl_sync(0xffffffffu, k.weight, 1);
        a = make_float4(a.x * fa, a.y * fa, a.z * fa, a.w * fa);
        add_scaled(a, fb, b);
        all = k;
      }
    }
    if (every2 == 0) store_out<kShared>(p, ri.s, ri.h, ri.r0 + row2, u2, a);
    if (lane == 0 && u2 == 0) store_sum<kShared>(p, ri.s, ri.h, ri.r0 + row2, all.ref);
  }
}

// SMs of a device; asked once a device (a decode step makes this call per layer)
int sm_count(int dev) {
  static std::atomic<int> known[64];
  std::atomic<int>* k = dev >= 0 && dev < 64 ? &known[dev] : nullptr;
  int n = k ? k->load(std::memory_order_relaxed) : 0;
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (k) k->store(n, std::memory_order_relaxed);
  }
  return n;
}

constexpr int kMaxCtas = 256;                     // of a launch; the workspace holds as many records
constexpr int kMaxBatch = 1024;                   // of a launch: the cut is worked out in shared memory
constexpr size_t kTicketBytes = kMaxCtas * 4;

template <int D, int NG, bool kTwoPlanes, int R, bool kShared>
cudaError_t launch_rows(const Params<kShared>& p, int dev, int ctas, cudaStream_t s) {
  // the kernel's shared memory limit, raised once a device
  static std::atomic<uint64_t> raised{0};
  const uint64_t bit = dev >= 0 && dev < 64 ? uint64_t(1) << dev : 0;
  if (!(raised.load(std::memory_order_relaxed) & bit) || !bit) {
    const cudaError_t err = cudaFuncSetAttribute(k_attn_rows<D, NG, kTwoPlanes, R, kShared>,
                                                 cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 AttnSmem<D, NG, R>::bytes(kMaxBatch));
    if (err != cudaSuccess) return err;
    raised.fetch_or(bit, std::memory_order_relaxed);
  }
  return launch_early(k_attn_rows<D, NG, kTwoPlanes, R, kShared>, ctas, (kAttnWarps + 1) * 32, AttnSmem<D, NG, R>::bytes(p.batch), s, p);
}

template <bool kTwoPlanes, int R, bool kShared>
cudaError_t dispatch_rows(const Params<kShared>& p, int d, int group, int dev, int ctas, cudaStream_t s) {
  if (d == 128 && group == 32) return launch_rows<128, 4, kTwoPlanes, R, kShared>(p, dev, ctas, s);
  if (d == 128 && group == 64) return launch_rows<128, 2, kTwoPlanes, R, kShared>(p, dev, ctas, s);
  if (d == 128) return launch_rows<128, 1, kTwoPlanes, R, kShared>(p, dev, ctas, s);
  if (group == 32) return launch_rows<64, 2, kTwoPlanes, R, kShared>(p, dev, ctas, s);
  return launch_rows<64, 1, kTwoPlanes, R, kShared>(p, dev, ctas, s);
}

// Whole blocks of rows (paged_attn_blocks.cu) from kBlockRows rows a sequence on: a
// block costs the same up to 128, eight rows after eight cost more and more.  At 32,
// 48 and 64 rows, us: one sequence of 32K 46, 61, 73 against 53, 53, 55; 8 of 8K 73, 99,
// 125 against 97 at all three; one of 1000 17, 19, 20 against 22.  So it is for bf16
// outputs; fp16 ones take the other kernel's two planes: 69, 114 and 20 at 48 rows against
// 53, 96 and 22.  fp32 outputs and sequences of different query counts keep to the other
// kernel, whose cut is made on the device.
constexpr int kBlockRows = 48;
bool takes_blocks(const reskv_paged_kv* kv, const reskv_paged_attn_args* a) {
  if (a->q_begin || a->o.dtype == RESKV_F32 || a->scale < 0.f || kv->batch < 1 || kv->n_kv_heads < 1) return false;
  return a->n_tokens / kv->batch * (a->q.n_heads / kv->n_kv_heads) >= kBlockRows;
}
BlockPlan block_plan(const reskv_paged_kv* kv, const reskv_paged_attn_args* a, int sms) {
  return plan_attn_blocks(a->n_tokens / kv->batch * (a->q.n_heads / kv->n_kv_heads), kv->batch, kv->n_kv_heads,
                          int64_t(kv->table_pages) * kv->page_tokens, sms);
}

cudaError_t device_sms(int* dev, int* sms) {
  const cudaError_t err = cudaGetDevice(dev);
  if (err != cudaSuccess) return err;
  *sms = sm_count(*dev);
  return *sms < 1 ? cudaErrorInvalidDevice : cudaSuccess;
}

std::string check_attn(const reskv_paged_kv* kv, const reskv_paged_attn_args* a) {
  std::string bad = check_paged(kv);
  if (!bad.empty()) return bad;
  if (!a) return "args is NULL";
  bad = check_heads(&a->q, "q");
  if (bad.empty()) bad = check_heads(&a->o, "o");
  if (!bad.empty()) return bad;
  if (a->q.dtype != RESKV_BF16 && a->q.dtype != RESKV_F16) return "q must be bf16 or fp16";
  if (a->o.dtype != a->q.dtype && a->o.dtype != RESKV_F32) return "o must have q's dtype or fp32";
  if (a->o.n_heads != a->q.n_heads) return "q and o must have the same heads";
  if (a->q.n_heads % kv->n_kv_heads || a->q.n_heads / kv->n_kv_heads > 64)
    return "q's heads must be a multiple of n_kv_heads, at most 64 per KV head";
  if (!a->lens) return "lens is NULL";
  if (a->n_tokens < 0 || double(a->n_tokens) * a->q.n_heads >= double(int64_t(1) << 31))
    return "n_tokens must not be negative, n_tokens * heads below 2^31";
  // units: at most one more per sequence than full blocks of rows
  if ((double(a->n_tokens) * (a->q.n_heads / kv->n_kv_heads) / 4 + kv->batch) * kv->n_kv_heads >= double(1 << kUnitBits))
    return "n_tokens * heads / 4 + batch * n_kv_heads must be below 2^24";
  if (!a->q_begin && a->n_tokens % kv->batch) return "n_tokens must be a multiple of batch without q_begin";
  if (a->lse && !aligned_to(a->lse, 4)) return "lse must be 4-byte aligned";
  if (!std::isfinite(a->scale) || a->window < 0) return "scale must be finite and window not negative";
  return "";
}

// Once the rest is fine: `need` goes by it.
std::string check_workspace(const reskv_paged_attn_args* a, size_t need, const char* name) {
  if (a->workspace && aligned_to(a->workspace, 256) && a->workspace_bytes >= need) return "";
  return std::string("workspace must be 256-byte aligned and hold ") + name + "() bytes";
}

AttnParams attn_params(const reskv_paged_kv* kv, const reskv_paged_attn_args* a) {
  AttnParams p{};
  p.q = a->q.data;
  p.o = a->o.data;
  p.lse = a->lse;
  p.q_token = a->q.token_stride;
  p.q_head = a->q.head_stride;
  p.o_token = a->o.token_stride;
  p.o_head = a->o.head_stride;
  p.q_begin = a->q_begin;
  p.lens = a->lens;
  p.page_table = kv->page_table;
  p.pages = static_cast<const uint8_t*>(kv->pages);
  p.status = kv->status;
  p.n_pages = kv->n_pages;
  p.n_tokens = a->n_tokens;
  p.batch = kv->batch;
  p.table_pages = kv->table_pages;
  p.page_tokens = kv->page_tokens;
  p.kv_heads = kv->n_kv_heads;
  p.heads = a->q.n_heads;
  p.window = a->window;
  p.o_f32 = a->o.dtype == RESKV_F32;
  p.scale2 = (a->scale != 0.f ? a->scale : 1.f / std::sqrt(float(kv->head_dim))) * kLog2e;
  p.group = p.heads / p.kv_heads;
  p.q_f16 = a->q.dtype == RESKV_F16;
  p.q_wide = rows_aligned(a->q, 16);
  p.o_wide = rows_aligned(a->o, size_t(4 * dtype_size(a->o.dtype)));
  p.tickets = static_cast<int32_t*>(a->workspace);
  p.partials = reinterpret_cast<float*>(static_cast<char*>(a->workspace) + kTicketBytes);
  return p;
}

// The kernel of few rows, in launches of kMaxBatch sequences (or groups).  `one`: weights in
// one fp16 plane (2^-11), finer than bf16's 2^-8.  Four rows a unit where a sequence has no more on average.
cudaError_t attn_rows(const AttnParams& p, const reskv_paged_kv* kv, bool one, int dev, int ctas, cudaStream_t s) {
  if (ctas > kMaxCtas) ctas = kMaxCtas;
  const bool few = p.n_tokens * p.group <= 4 * int64_t(p.batch);
  const int64_t each = p.n_tokens / p.batch;       // query tokens a sequence without q_begin
  cudaError_t err = cudaSuccess;
  for (int b0 = 0; b0 < p.batch && err == cudaSuccess; b0 += kMaxBatch) {
    AttnParams l = p;
    l.batch = p.batch - b0 < kMaxBatch ? p.batch - b0 : kMaxBatch;
    l.lens += b0;
    l.page_table += int64_t(b0) * p.table_pages;
    if (p.q_begin) {
      l.q_begin += b0;
    } else {
      const int64_t t0 = b0 * each;
      l.n_tokens = l.batch * each;
      l.q = static_cast<const char*>(p.q) + t0 * p.q_token * 2;
      l.o = static_cast<char*>(p.o) + t0 * p.o_token * (p.o_f32 ? 4 : 2);
      if (p.lse) l.lse = p.lse + t0 * p.heads;
    }
    err = one ? (few ? dispatch_rows<false, 4, false>(l, kv->head_dim, kv->quant_group, dev, ctas, s)
                     : dispatch_rows<false, 8, false>(l, kv->head_dim, kv->quant_group, dev, ctas, s))
              : (few ? dispatch_rows<true, 4, false>(l, kv->head_dim, kv->quant_group, dev, ctas, s)
                     : dispatch_rows<true, 8, false>(l, kv->head_dim, kv->quant_group, dev, ctas, s));
  }
  return err;
}

}  // namespace
}  // namespace reskv

using namespace reskv;

extern "C" size_t reskv_paged_attn_workspace(const reskv_paged_kv* kv, const reskv_paged_attn_args* a) {
  if (!kv || !a || (kv->head_dim != 64 && kv->head_dim != 128)) return 0;
  size_t bytes = size_t(kMaxCtas) * 2 * (record_floats(kv->head_dim, 8) + 8) * 4;
  int dev = 0, sms = 0;
  if (takes_blocks(kv, a) && cudaGetDevice(&dev) == cudaSuccess && (sms = sm_count(dev)) > 0) {
    const size_t more = attn_blocks_bytes(block_plan(kv, a, sms), kv->head_dim);
    if (more > bytes) bytes = more;
  }
  cudaGetLastError();
  return kTicketBytes + bytes;
}

extern "C" reskv_status reskv_paged_attn(const reskv_paged_kv* kv, const reskv_paged_attn_args* a, void* stream) {
  return no_throw([&]() -> reskv_status {
    if (a && a->n_tokens == 0) return RESKV_OK;
    std::string bad = check_attn(kv, a);
    if (bad.empty()) bad = check_workspace(a, reskv_paged_attn_workspace(kv, a), "reskv_paged_attn_workspace");
    if (!bad.empty()) return paged_fail(RESKV_ERR_INVALID_ARG, bad);
    const AttnParams p = attn_params(kv, a);
    int dev = 0, sms = 0;
    const cudaError_t err = device_sms(&dev, &sms);
    if (err != cudaSuccess) return launch_result(err, "reading the device");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (takes_blocks(kv, a))
      return launch_result(launch_attn_blocks(p, block_plan(kv, a, sms), kv->head_dim, kv->quant_group, dev, p.partials, s),
                           "paged attention");
    return launch_result(attn_rows(p, kv, a->o.dtype == RESKV_BF16, dev, sms, s), "paged attention");
  });
}

// --- a shared prefix ---
// Over the own tokens and over the prefix into fp32 rows and sums, and a join.  Where groups have
// few rows both are units of one launch of the kernel of few rows (units of eight rows: a group has
// more).  Otherwise the prefix goes by blocks of rows, in a launch that begins while the own tokens' runs.
namespace reskv {
namespace {

// Units of 8 query rows of all sequences (or groups) of a cache, and their tiles by the tables' room.
struct FewRows {
  double units, tiles;
};
FewRows few_rows(const reskv_paged_kv* c, const reskv_paged_attn_args* a) {
  const double rows = double(a->n_tokens) * (a->q.n_heads / c->n_kv_heads);
  const double units = double(c->batch) * c->n_kv_heads * std::ceil(rows / c->batch / 8.0);
  return {units, units * (double(c->table_pages) * c->page_tokens / kTile)};
}

// The prefix in blocks of rows, by the mean rows of a group: as in takes_blocks, but from 32 rows on, us:
// four groups of 32 rows to 16384 positions 65 against 82, 32 rows of 32768 64 against 70, of 4096 34 against 32;
// 24 rows of 1000 26 against 21, 16 of 32768 63 against 48.
// Below 128 rows that is not so where each SM has a unit and a dozen tiles at most, of both passes: one launch
// ends before two then.  8 KV heads, 4 query heads each, us: 8 sequences of 100 behind 512 23.0 against 18.5,
// 12 of 60 behind 256 22.5 against 18.0; 8 of 60 behind 1000 (15 tiles) 22.0 against 21.3, behind 4096 27 against
// 31; 16 of 60 behind 256 (1.3 units) 25 against 27; with one KV head 128 rows of 1000 23.8 against 24.7.
constexpr int kPrefixRows = 32, kFewTiles = 12;
bool prefix_in_blocks(const reskv_paged_kv* kv, const reskv_paged_kv* prefix, const reskv_paged_attn_args* a, int sms) {
  const double rows = double(a->n_tokens) * (a->q.n_heads / prefix->n_kv_heads) / prefix->batch;       // of a group
  if (a->o.dtype == RESKV_F32 || !(a->scale >= 0.f) || rows < kPrefixRows) return false;
  const FewRows own = few_rows(kv, a), shared = few_rows(prefix, a);
  return rows >= 128 || takes_blocks(kv, a) || own.units + shared.units > sms || own.tiles + shared.tiles > double(kFewTiles) * sms;
}
// Sequences and groups that one launch of the kernel of few rows holds.
bool one_launch(const reskv_paged_kv* kv, const reskv_paged_kv* prefix, const reskv_paged_attn_args* a) {
  return int64_t(kv->batch) + prefix->batch <= kMaxBatch && !takes_blocks(kv, a);
}
// Blocks of 128 rows a CTA takes.
int prefix_mt(const reskv_paged_kv* prefix, const reskv_paged_attn_args* a) {
  return a->n_tokens * (a->q.n_heads / prefix->n_kv_heads) > 128 * int64_t(prefix->batch) ? 2 : 1;
}

// SMs of the pass over the own tokens while the prefix has the others; 0: one after the other, with all.  By
// the times of both (us) with n SMs, as measured, for the tables' room; what is fixed of them is most of it
// where a prefix has some thousand positions: 64 sequences of 512 behind 8192 68 -> 43 us.
int own_sms(const reskv_paged_kv* kv, const reskv_paged_kv* prefix, const reskv_paged_attn_args* a, int sms) {
  const double rows = double(a->n_tokens) * (a->q.n_heads / kv->n_kv_heads);
  const double tiles = few_rows(kv, a).tiles;
  const double block = 128.0 * prefix_mt(prefix, a);
  const double steps = double(prefix->table_pages) * prefix->page_tokens / kBlockPos * kv->n_kv_heads * prefix->batch *
                       std::ceil(rows / prefix->batch / block);
  const double tile = rows <= 4.0 * kv->batch ? 0.07 : 0.1;
  auto own = [&](int n) { return 9.0 + tile * tiles / n; };
  auto other = [&](int n) { return 18.0 + 1.5 * steps / n; };
  double best = own(sms) + other(sms) - 3.0;
  int best_n = 0;
  for (int n = 8; n + 8 <= sms; n += 8) {
    const double t = own(n) > other(sms - n) ? own(n) : other(sms - n);
    if (t < best) {
      best = t;
      best_n = n;
    }
  }
  return best_n;
}

struct SharedLayout {             // of the workspace, in bytes from its start
  size_t own, own_lse, prefix, prefix_ref, plans, bytes;
};
size_t padded(size_t n) { return (n + 255) / 256 * 256; }
SharedLayout shared_layout(const reskv_paged_kv* kv, const reskv_paged_kv* prefix, const reskv_paged_attn_args* a, int sms) {
  const size_t rows = size_t(a->n_tokens) * a->q.n_heads;
  size_t records = size_t(kMaxCtas) * 2 * (record_floats(kv->head_dim, 8) + 8) * 4;
  if (takes_blocks(kv, a)) {
    const size_t more = attn_blocks_bytes(block_plan(kv, a, sms), kv->head_dim);
    if (more > records) records = more;
  }
  SharedLayout l{};
  l.own = padded(kTicketBytes + records);
  l.own_lse = l.own + padded(rows * kv->head_dim * 4);
  l.prefix = l.own_lse + padded(rows * 4);
  size_t held = rows;
  if (prefix_in_blocks(kv, prefix, a, sms)) {
    const int block = 128 * prefix_mt(prefix, a);
    // rows of records: 128 or 256 of two streams or blocks an item
    held = size_t(group_items(a->n_tokens * (a->q.n_heads / kv->n_kv_heads), prefix->batch, kv->n_kv_heads, block, sms)) * 256;
  }
  l.prefix_ref = l.prefix + padded(held * kv->head_dim * 4);
  l.plans = l.prefix_ref + padded(held * 8);
  l.bytes = l.plans + padded(size_t(prefix->batch) * sizeof(GroupPlan));
  return l;
}

std::string check_shared(const reskv_paged_kv* kv, const reskv_paged_kv* prefix, const int32_t* seq_begin,
                         const int32_t* prefix_lens, const reskv_paged_attn_args* a) {
  std::string bad = check_paged(prefix);
  if (!bad.empty()) return "the prefix: " + bad;
  bad = check_attn(kv, a);
  if (!bad.empty()) return bad;
  if (prefix->head_dim != kv->head_dim || prefix->n_kv_heads != kv->n_kv_heads || prefix->quant_group != kv->quant_group ||
      prefix->page_tokens != kv->page_tokens)
    return "the prefix must have the cache's head_dim, n_kv_heads, quant_group and page_tokens";
  if (!prefix_lens) return "prefix_lens is NULL";
  if (!seq_begin && kv->batch % prefix->batch) return "batch must be a multiple of the prefixes without seq_begin";
  if (a->window != 0) return "window must be 0";
  if (prefix->batch >= kMaxBatch) return "fewer than 1024 prefixes a call";
  if ((double(a->n_tokens) * (a->q.n_heads / kv->n_kv_heads) / 2 + kv->batch + prefix->batch) * kv->n_kv_heads >= double(1 << kUnitBits))
    return "n_tokens * heads / 2 + (batch + prefixes) * n_kv_heads must be below 2^24";
  return check_workspace(a, reskv_paged_attn_shared_workspace(kv, prefix, a), "reskv_paged_attn_shared_workspace");
}

}  // namespace
}  // namespace reskv

extern "C" size_t reskv_paged_attn_shared_workspace(const reskv_paged_kv* kv, const reskv_paged_kv* prefix,
                                                    const reskv_paged_attn_args* a) {
  if (!kv || !prefix || !a || (kv->head_dim != 64 && kv->head_dim != 128) || kv->batch < 1 || kv->n_kv_heads < 1 ||
      prefix->batch < 1 || prefix->n_kv_heads != kv->n_kv_heads || a->n_tokens < 0 || a->q.n_heads < 1)
    return 0;
  int dev = 0, sms = 0;
  if (device_sms(&dev, &sms) != cudaSuccess) {
    cudaGetLastError();
    sms = 1;                                      // (no call without a device comes to use it)
  }
  return shared_layout(kv, prefix, a, sms).bytes;
}

extern "C" reskv_status reskv_paged_attn_shared(const reskv_paged_kv* kv, const reskv_paged_kv* prefix, const int32_t* seq_begin,
                                                const int32_t* prefix_lens, const reskv_paged_attn_args* a, void* stream) {
  return no_throw([&]() -> reskv_status {
    if (a && a->n_tokens == 0) return RESKV_OK;
    const std::string bad = check_shared(kv, prefix, seq_begin, prefix_lens, a);
    if (!bad.empty()) return paged_fail(RESKV_ERR_INVALID_ARG, bad);
    int dev = 0, sms = 0;
    cudaError_t err = device_sms(&dev, &sms);
    if (err != cudaSuccess) return launch_result(err, "reading the device");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const SharedLayout l = shared_layout(kv, prefix, a, sms);
    char* ws = static_cast<char*>(a->workspace);
    const bool one = a->o.dtype == RESKV_BF16;
    // the own tokens into fp32 rows [token][head][dim]
    const AttnParams call = attn_params(kv, a);
    AttnParams p = call;
    p.o = ws + l.own;
    p.lse = reinterpret_cast<float*>(ws + l.own_lse);
    p.o_f32 = p.o_wide = 1;
    p.o_head = kv->head_dim;
    p.o_token = int64_t(p.heads) * kv->head_dim;
    // the prefix: a group's query tokens are one sequence's that all see all
    SharedParams g{};
    static_cast<AttnParams&>(g) = p;
    g.sequences = kv->batch;
    g.seq_begin = seq_begin;
    g.prefix_lens = prefix_lens;
    g.prefix_table = prefix->page_table;
    g.prefix_data = static_cast<const uint8_t*>(prefix->pages);
    g.prefix_status = prefix->status;
    g.prefix_n_pages = prefix->n_pages;
    g.prefix_pages = prefix->table_pages;
    g.prefix_o = reinterpret_cast<float*>(ws + l.prefix);
    g.prefix_ref = reinterpret_cast<float*>(ws + l.prefix_ref);
    const bool blocks = prefix_in_blocks(kv, prefix, a, sms), fused = !blocks && one_launch(kv, prefix, a);
    const int mt = prefix_mt(prefix, a);
    const int apart = blocks && !takes_blocks(kv, a) ? own_sms(kv, prefix, a, sms) : 0;
    const int items = blocks ? int(group_items(p.n_tokens * p.group, prefix->batch, p.kv_heads, 128 * mt, sms - apart)) : 0;
    GroupPlan* plans = reinterpret_cast<GroupPlan*>(ws + l.plans);
    if (fused) {
      g.batch = kv->batch + prefix->batch;
      g.own = kv->batch;
      const int ctas = sms < kMaxCtas ? sms : kMaxCtas;
      err = one ? dispatch_rows<false, 8, true>(g, kv->head_dim, kv->quant_group, dev, ctas, s)
                : dispatch_rows<true, 8, true>(g, kv->head_dim, kv->quant_group, dev, ctas, s);
    } else {
      err = takes_blocks(kv, a) ? launch_attn_blocks(p, block_plan(kv, a, sms), kv->head_dim, kv->quant_group, dev, p.partials, s)
                                : attn_rows(p, kv, one, dev, apart ? apart : sms, s);
    }
    g.batch = prefix->batch;
    g.own = 0;
    if (err == cudaSuccess && blocks)
      err = launch_attn_groups(g, mt, items, sms - apart, kv->head_dim, kv->quant_group, dev, g.prefix_o, plans, s);
    if (err == cudaSuccess && !blocks && !fused) {
      const int ctas = sms < kMaxCtas ? sms : kMaxCtas;
      err = one ? dispatch_rows<false, 8, true>(g, kv->head_dim, kv->quant_group, dev, ctas, s)
                : dispatch_rows<true, 8, true>(g, kv->head_dim, kv->quant_group, dev, ctas, s);
    }
    SharedJoin j{};
    j.a = g;
    j.a.o = call.o;
    j.a.lse = call.lse;
    j.a.o_token = call.o_token;
    j.a.o_head = call.o_head;
    j.a.o_f32 = call.o_f32;
    j.a.o_wide = call.o_wide;
    j.own = static_cast<const float*>(p.o);
    j.own_lse = p.lse;
    j.own_unit = fused ? 1.f : kLog2e;
    j.prefix = g.prefix_o;
    j.prefix_ref = g.prefix_ref;
    j.plans = blocks ? plans : nullptr;
    j.block_rows = 128 * mt;
    j.items = items;
    j.groups = prefix->batch;
    j.dim = kv->head_dim;
    if (err == cudaSuccess) err = launch_shared_join(j, s);
    return launch_result(err, "attention with a shared prefix");
  });
}

extern "C" int32_t reskv_stream_capturing(void* stream) {
  cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(static_cast<cudaStream_t>(stream), &st) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  return st != cudaStreamCaptureStatusNone;
}
