// Writing a paged 4-bit cache (reskv_paged_append) and reading its values back
// (reskv_paged_gather).  The format is in include/reskv.h.
#include <cmath>

#include "paged.cuh"

namespace reskv {

std::string check_paged(const reskv_paged_kv* kv) {
  if (!kv || !kv->pages || !kv->page_table) return "a paged cache with pages and a page_table is needed";
  if (reskv_paged_head_bytes(kv->page_tokens, kv->head_dim, kv->quant_group) == 0)
    return "page_tokens must be a multiple of 16 in [16, 1024], head_dim 64 or 128, quant_group 32, 64 or 128 "
           "and a divisor of head_dim";
  if (!aligned_to(kv->pages, 16)) return "pages must be 16-byte aligned";
  if (kv->n_pages < 1 || kv->n_pages > 0x7fffffff) return "n_pages must be in [1, 2^31)";
  if (kv->n_kv_heads < 1 || kv->n_kv_heads > 1024) return "n_kv_heads must be in [1, 1024]";
  if (kv->batch < 1 || kv->table_pages < 1) return "batch and table_pages must be >= 1";
  if (int64_t(kv->table_pages) * kv->page_tokens > 0x7fffffff)
    return "table_pages * page_tokens must be below 2^31";
  return "";
}

namespace {

struct AppendParams {
  const int32_t* seqs;
  const int32_t* positions;
  const int32_t* page_table;
  uint8_t* pages;
  uint32_t* status;
  const float2* table;            // NULL: keys as they are
  const void *k, *v;
  int64_t k_token, k_head, v_token, v_head;
  int64_t n_pages, n_positions, n_tokens;
  int32_t batch, table_pages, page_tokens, kv_heads;
  int32_t rot, interleaved;
  int32_t head_groups, heads_each;  // of a token; KV heads a thread takes, at most kHeads
  uint32_t blocks;                // of the launch that hold rows; the others turn queries
};

// least and largest of three, a NaN kept
__device__ __forceinline__ float min3_nan(float a, float b, float c) {
  float r;
  asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float mul_01(float a, float b) {        // within [0, 1]
  float r;
  asm("mul.rn.sat.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Eight neighbouring dims per lane, kGroup / 8 lanes a group: the codes of the
// lane's dims and its group's scale (low half) and minimum (high half).
//
// A code is rint((x - m) / s), within 0..15, of the correctly rounded quotient.  It is
// found as rint(15 u), u = (x - m) r within [0, 1], r = 1 / 15 s: 15 u is off by less
// than 2^-17, so that a value whose fraction lies further than that from one half
// has its code.  Where one of the lane's values is nearer (of 16-bit inputs many are
// halfway), the lane compares them with t s, t the half next to 15 u: one fma has the
// sign of x - m - t s.  The quotient itself would say the same: t s has 13 bits, so
// that x - m, unless it is t s, is further from it than the quotient's rounding
// reaches.  Both passes end in 0..15: a minimum that bf16 rounds down leaves the largest
// values of a group far from zero more than 15.5 scales above it.
template <int kGroup>
__device__ __forceinline__ void hold(const float2 (&x)[4], uint32_t& codes, uint32_t& sm) {
  float lo = min3_nan(min3_nan(x[0].x, x[0].y, x[1].x), min3_nan(x[1].y, x[2].x, x[2].y), min3_nan(x[3].x, x[3].y, x[3].y));
  float hi = max3_nan(max3_nan(x[0].x, x[0].y, x[1].x), max3_nan(x[1].y, x[2].x, x[2].y), max3_nan(x[3].x, x[3].y, x[3].y));
#pragma unroll
  for (int o = 1; o < kGroup / 8; o *= 2) {
    const float l = __shfl_xor_sync(0xffffffffu, lo, o), h = __shfl_xor_sync(0xffffffffu, hi, o);
    lo = min3_nan(lo, l, l);
    hi = max3_nan(hi, h, h);
  }
  uint32_t s16 = __bfloat16_as_ushort(__float2bfloat16_rn(__fdiv_rn(__fsub_rn(hi, lo), 15.f)));
  uint32_t m16 = __bfloat16_as_ushort(__float2bfloat16_rn(lo));
  const float s = __uint_as_float(s16 << 16), m = __uint_as_float(m16 << 16);
  codes = 0;
  if (!(isfinite(s) && isfinite(m))) {
    s16 = m16 = 0x7fc0;
  } else if (s < 1.17549435e-38f) {
    s16 = 0;
  } else {
    constexpr float kRound = 12582912.f;          // 1.5 2^23: adding it rounds to whole numbers
    const float r = __frcp_rn(s) * 0.06666667f;
    // codes 0..3 and 4..7 as 16-bit numbers, negated; scales past 2^120 leave r few digits
    float2 sum = make_float2(0.f, 0.f);
    float worst = s > 1.3e36f ? 1.f : 0.f;
    const float2 mm = make_float2(m, m), k15 = make_float2(15.f, 15.f), up = make_float2(kRound, kRound);
    const float2 k16 = make_float2(16.f, 16.f);
    auto pair = [&](int i) {                      // values i and 4 + i
      return i & 1 ? make_float2(x[i / 2].y, x[2 + i / 2].y) : make_float2(x[i / 2].x, x[2 + i / 2].x);
    };
#pragma unroll
    for (int i = 3; i >= 0; --i) {
      const float2 a = fsub2(pair(i), mm);
      const float2 u = make_float2(mul_01(a.x, r), mul_01(a.y, r));
      const float2 n = fsub2(up, ffma2(u, k15, up));               // -n
      const float2 d = ffma2(u, k15, n);
      worst = fmaxf(worst, fmaxf(fabsf(d.x), fabsf(d.y)));
      sum = ffma2(sum, k16, n);
    }
    if (worst > 0.5f - 7.62939453125e-6f) {
      sum = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 3; i >= 0; --i) {
        const float2 a = fsub2(pair(i), mm);
        const float u[2] = {mul_01(a.x, r), mul_01(a.y, r)};
        float n[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float near = __fsub_rn(fmaf(u[k], 15.f, kRound), kRound);
          const float t = near + copysignf(0.5f, fmaf(u[k], 15.f, -near));
          const float over = fmaf(-t, s, k ? a.y : a.x);
          // (u ends at one: what lies past the top code comes out as 16 here, from t = 15.5)
          n[k] = fminf(over == 0.f ? rintf(t) : t + copysignf(0.5f, over), 15.f);
        }
        sum = ffma2(sum, k16, make_float2(-n[0], -n[1]));
      }
    }
    codes = uint32_t(-sum.x) | uint32_t(-sum.y) << 16;
  }
  sm = s16 | (m16 << 16);
}

// Up to kHeads KV heads of one token per D / 8 lanes: K row, then V row.  The rows' cos and
// sin are read once.  What a row costs is instructions: the rows of 32768 tokens of 8 KV heads
// of 128 by themselves take 65 us (176 MB, 2.7 TB/s; schedulers 72 % busy).  With their
// 32 query heads turned beside them (713 MB) it is 146 us, 4.9 TB/s; turns and rows
// mixed block by block were slower (168 us), as fewer loads were in flight.
template <typename T, int D, int kGroup, bool kWide, int kHeads>
__device__ __forceinline__ void append_rows(const AppendParams& p, int64_t r, int lane) {
  constexpr int NG = D / kGroup;
  constexpr TileShape ts{D, NG};
  const int groups = p.head_groups, each = kHeads == 1 ? 1 : p.heads_each;
  const bool in = r < p.n_tokens * groups;
  if (!in) r = 0;                                   // stays for the shuffles, writes nothing
  const int64_t tok = uint32_t(r) / uint32_t(groups);
  const int h0 = (int(r) - int(tok) * groups) * each;
  const int pos = p.positions[tok], seq = p.seqs[tok];
  bool live = in && pos >= 0;
  uint8_t* tile = nullptr;                          // of head 0
  int row = 0;
  const int64_t head_bytes = int64_t(p.page_tokens / kTile) * ts.bytes();
  if (live) {
    const int pg = pos / p.page_tokens;
    bool fault = seq < 0 || seq >= p.batch || pg >= p.table_pages || (p.table && pos >= p.n_positions);
    if (!fault) {
      const int page = p.page_table[int64_t(seq) * p.table_pages + pg];
      fault = page < 0 || page >= p.n_pages;
      const int slot = pos - pg * p.page_tokens;
      row = slot % kTile;
      tile = p.pages + int64_t(page) * p.kv_heads * head_bytes + slot / kTile * ts.bytes();
    }
    if (fault && lane == 0) report_status(p.status, kStatusBadIndex);
    live = !fault;
  }
  union Eight {
    uint4 w[sizeof(T) * 8 / 16];
    T v[8];
    __device__ Eight() {}
  };
  auto load = [&](const T* at, Eight& u) {
    if constexpr (kWide) {
#pragma unroll
      for (int i = 0; i < int(sizeof(u) / 16); ++i) u.w[i] = reinterpret_cast<const uint4*>(at)[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) u.v[i] = at[i];
    }
  };
  auto floats = [](const Eight& u, float2 (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = make_float2(to_f32(u.v[2 * i]), to_f32(u.v[2 * i + 1]));
  };
  // The lane's pairs: its eight dims against the eight rot / 2 away, or neighbours.
  // Rotations that cut a lane's dims take them one by one.
  const bool turns = p.table && live && 8 * lane < p.rot;
  const int half = p.rot / 2;
  const bool whole = p.interleaved ? p.rot % 8 == 0 : p.rot % 16 == 0;
  const bool lower = 8 * lane < half;
  // a dim x with partner o becomes x c + o s, s negated for the lower of a pair
  float2 co[4], si[4];
  if (turns && whole) {
    const float2* c = p.table + int64_t(pos) * half + (p.interleaved ? 4 * lane : 8 * lane - (lower ? 0 : half));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (p.interleaved) {
        const float2 w = c[i];
        co[i] = make_float2(w.x, w.x);
        si[i] = make_float2(-w.y, w.y);
      } else {
        const float2 w0 = c[2 * i], w1 = c[2 * i + 1];
        co[i] = make_float2(w0.x, w1.x);
        si[i] = lower ? make_float2(-w0.y, -w1.y) : make_float2(w0.y, w1.y);
      }
    }
  }
  // A head's words are asked for before those of the one before are held.
  Eight kw, vw, ow;
  auto ask = [&](int h) {
    const T* k = static_cast<const T*>(p.k) + tok * p.k_token + h * p.k_head + 8 * lane;
    load(k, kw);
    load(static_cast<const T*>(p.v) + tok * p.v_token + h * p.v_head + 8 * lane, vw);
    if (turns && whole && !p.interleaved) load(k + (lower ? half : -half), ow);
  };
  ask(h0);
#pragma unroll 1
  for (int i = 0; i < each; ++i) {
    const int h = min(h0 + i, p.kv_heads - 1);      // the last head again: the same bytes
    const T* k = static_cast<const T*>(p.k) + tok * p.k_token + h * p.k_head;
    uint8_t* at = tile + h * head_bytes;
    float2 x[4], y[4], o[4];
    floats(kw, x);
    floats(vw, y);
    if (turns && whole) {
      if (p.interleaved) {
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = make_float2(x[j].y, x[j].x);
      } else {
        floats(ow, o);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[j].x = __fadd_rn(__fmul_rn(x[j].x, co[j].x), __fmul_rn(o[j].x, si[j].x));
        x[j].y = __fadd_rn(__fmul_rn(x[j].y, co[j].y), __fmul_rn(o[j].y, si[j].y));
      }
    } else if (turns) {
#pragma unroll 1
      for (int j = 0; j < 8; ++j) {
        const int dim = 8 * lane + j;
        if (dim >= p.rot) break;
        const bool low = p.interleaved ? dim % 2 == 0 : dim < half;
        const int pair = p.interleaved ? dim / 2 : (low ? dim : dim - half);
        const int other = p.interleaved ? dim ^ 1 : (low ? dim + half : dim - half);
        float a = to_f32(k[low ? dim : other]), b = to_f32(k[low ? other : dim]);
        const float2 c = p.table[int64_t(pos) * half + pair];
        turn(a, b, c.x, c.y);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (2 * q == j) x[q].x = low ? a : b;
          if (2 * q + 1 == j) x[q].y = low ? a : b;
        }
      }
    }
    if (kHeads > 1 && i + 1 < each) ask(min(h + 1, p.kv_heads - 1));
    uint32_t codes, sm;
    hold<kGroup>(x, codes, sm);
    const bool first = lane % (kGroup / 8) == 0;
    if (live) {
      *reinterpret_cast<uint32_t*>(at + ts.k_unit(row, 2 * lane)) = codes;
      if (first) {
        uint16_t* meta = reinterpret_cast<uint16_t*>(at + ts.k_meta()) + row * 2 * NG + lane / (kGroup / 8);
        meta[0] = uint16_t(sm);
        meta[NG] = uint16_t(sm >> 16);
      }
    }
    hold<kGroup>(y, codes, sm);
    if (live) {
      uint8_t* c = at + ts.v_codes();
      *reinterpret_cast<uint16_t*>(c + ts.v_unit(row, 2 * lane)) = uint16_t(codes);
      *reinterpret_cast<uint16_t*>(c + ts.v_unit(row, 2 * lane + 1)) = uint16_t(codes >> 16);
      if (first) {
        uint16_t* meta = reinterpret_cast<uint16_t*>(at + ts.v_meta()) + row * 2 * NG + lane / (kGroup / 8);
        meta[0] = uint16_t(sm);
        meta[NG] = uint16_t(sm >> 16);
      }
    }
  }
}

// The tokens' rows in the first blocks, their queries' rotation in the others (blocks of
// 128 threads, against 256: 4 x 1024 tokens 24.3 and 26.6 us, 8 x 4096 146 and 150).
constexpr int kAppendThreads = 128;
template <typename T, int D, int kGroup, bool kWide, int kHeads>
__global__ void __launch_bounds__(kAppendThreads, 1024 / kAppendThreads) k_paged_append(const __grid_constant__ AppendParams p,
                                                      const __grid_constant__ RopeParams q) {
  constexpr int L = D / 8;
  wait_for_previous();
  if (blockIdx.x < p.blocks) {
    append_rows<T, D, kGroup, kWide, kHeads>(p, int64_t(blockIdx.x) * (kAppendThreads / L) + threadIdx.x / L, threadIdx.x % L);
  } else if constexpr (kWide) {
    constexpr int V = 16 / int(sizeof(T));
    const int lane = threadIdx.x % q.lanes, row = threadIdx.x / q.lanes;
    const int64_t r = int64_t(blockIdx.x - p.blocks) * q.rows_per_block + row;
    if (row >= q.rows_per_block) return;
    constexpr int kQ = kHeads == 1 ? 1 : kManyHeads<T>;
    if (q.interleaved) rope_rows<T, V, true, kQ>(q, r, lane);
    else rope_rows<T, V, false, kQ>(q, r, lane);
  }
}

template <typename T, int D, int kGroup, bool kWide, int kHeads>
cudaError_t launch_append_rows(AppendParams p, RopeParams q, cudaStream_t s) {
  constexpr int rows = kAppendThreads / (D / 8), V = 16 / int(sizeof(T));
  // all threads take the same number of heads (9 as 5 and 4, so that one of ten is the last again)
  p.head_groups = (p.kv_heads + kHeads - 1) / kHeads;
  p.heads_each = (p.kv_heads + p.head_groups - 1) / p.head_groups;
  p.blocks = unsigned((p.n_tokens * p.head_groups + rows - 1) / rows);
  unsigned blocks = p.blocks;
  if (q.heads) {
    q.lanes = rope_lanes(q.dim, q.rot, V);
    q.rows_per_block = kAppendThreads / q.lanes;
    constexpr int kQ = kHeads == 1 ? 1 : kManyHeads<T>;
    q.head_groups = (q.heads + kQ - 1) / kQ;
    blocks += unsigned((q.n_tokens * q.head_groups + q.rows_per_block - 1) / q.rows_per_block);
  }
  return launch_early(k_paged_append<T, D, kGroup, kWide, kHeads>, blocks, kAppendThreads, 0, s, p, q);
}

// Up to eight heads a thread where that leaves every SM a thousand threads (32K tokens of
// 8 KV and 32 query heads: 146 us; four heads took 5 % more); one where there are fewer
// rows.  2^18 rows of 1, 2, 4, 8 and 9 KV heads: 101, 76, 67, 64 and 72 us (one head a
// thread: 88 to 90).
template <typename T, int D, int kGroup>
cudaError_t dispatch_heads(const AppendParams& p, const RopeParams& q, bool wide, cudaStream_t s) {
  if (!wide) return launch_append_rows<T, D, kGroup, false, 1>(p, q, s);
  if (p.n_tokens * p.kv_heads * (D / 8) >= int64_t(152) * 8192) return launch_append_rows<T, D, kGroup, true, 8>(p, q, s);
  return launch_append_rows<T, D, kGroup, true, 1>(p, q, s);
}

template <typename T>
cudaError_t dispatch_append(const AppendParams& p, const RopeParams& q, int d, int group, bool wide, cudaStream_t s) {
  if (d == 128 && group == 32) return dispatch_heads<T, 128, 32>(p, q, wide, s);
  if (d == 128 && group == 64) return dispatch_heads<T, 128, 64>(p, q, wide, s);
  if (d == 128) return dispatch_heads<T, 128, 128>(p, q, wide, s);
  if (group == 32) return dispatch_heads<T, 64, 32>(p, q, wide, s);
  return dispatch_heads<T, 64, 64>(p, q, wide, s);
}

// --- reading back ----------------------------------------------------------

struct GatherParams {
  const int32_t* starts;
  const int32_t* lens;
  const int32_t* page_table;
  const uint8_t* pages;
  uint32_t* status;
  void* out[2];                   // K, V; NULL: not wanted
  int64_t b_stride[2], h_stride[2], t_stride[2];
  int64_t n, n_pages;
  int32_t table_pages, page_tokens, kv_heads, batch;
};

template <typename T, int N, bool kWide>
__device__ __forceinline__ void store_values(T* y, const float (&x)[N]) {
  Pack<T, N> o;
#pragma unroll
  for (int i = 0; i < N; ++i) o.v[i] = from_f32<T>(x[i]);
  if constexpr (!kWide) {
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = o.v[i];
  } else if constexpr (sizeof(o) == 32) {
    reinterpret_cast<uint4*>(y)[0] = reinterpret_cast<const uint4*>(&o)[0];
    reinterpret_cast<uint4*>(y)[1] = reinterpret_cast<const uint4*>(&o)[1];
  } else {
    *reinterpret_cast<Pack<T, N>*>(y) = o;
  }
}

// n codes of a masked word as fp32 (exact): two from the halves' low 4 bits.
__device__ __forceinline__ float2 two_codes(uint32_t w) {
  const uint32_t h = (w & 0x000f000fu) | 0x64006400u;               // 1024 + n in fp16
  const __half2 n = __hsub2(*reinterpret_cast<const __half2*>(&h), __float2half2_rn(1024.f));
  return __half22float2(n);
}

// One tile per warp, read as its attention reads it (whole 16-byte words), eight
// dims of K and four of V a lane and word.  s n is exact in fp32, so a value is one
// fma, rounded once more to the output's type.  Bound by DRAM: 8 prompts of up to
// 32K positions (1.31 GB read and written) in 194 us, 0.99 of the measured copy
// rate; one row's eight dims a thread, with seven loads of 2 or 4 bytes, took 338.
template <typename T, int D, int kGroup, bool kWide>
__global__ void __launch_bounds__(256) k_paged_gather(const __grid_constant__ GatherParams p) {
  constexpr int NG = D / kGroup, C = D / 32;
  constexpr TileShape ts{D, NG};
  wait_for_previous();
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int h = blockIdx.y % p.kv_heads;
  for (int b = blockIdx.y / p.kv_heads; b < p.batch; b += gridDim.y / p.kv_heads) {
    const int64_t start = p.starts ? p.starts[b] : 0, len = p.lens[b];
    // tiles of the sequence, the first one that of position `start`
    const int64_t first = start >= 0 ? start / kTile : -((-start + kTile - 1) / kTile);
    const int64_t pos0 = (first + int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5)) * kTile;
    if (pos0 >= start + p.n) continue;
    const uint8_t* tile = nullptr;
    if (pos0 >= 0 && pos0 < len) {
      const int64_t pg = pos0 / p.page_tokens;
      const int page = pg < p.table_pages ? p.page_table[int64_t(b) * p.table_pages + pg] : -1;
      if (page >= 0 && page < p.n_pages)
        tile = p.pages + ((int64_t(page) * p.kv_heads + h) * (p.page_tokens / kTile) + (pos0 - pg * p.page_tokens) / kTile) *
                             int64_t(ts.bytes());
      else if (lane == 0)
        report_status(p.status, kStatusBadIndex);
    }
    // output row of the tile's token r; NULL: not asked for
    auto out = [&](int kv, int r) -> T* {
      const int64_t i = pos0 + r - start;
      if (i < 0 || i >= p.n) return nullptr;
      return static_cast<T*>(p.out[kv]) + b * p.b_stride[kv] + h * p.h_stride[kv] + i * p.t_stride[kv];
    };
    if (p.out[0]) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = g + 8 * i;
        uint32_t w[C] = {}, meta[NG] = {};
        if (tile && pos0 + r < len) {
          load_words<C>(w, tile + r * (D / 2) + t * (D / 8));
          load_words<NG>(meta, tile + ts.k_meta() + r * 4 * NG);
        }
        T* y = out(0, r);
        if (!y) continue;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          float s, m, x[8];
          group_meta<NG>(meta, 32 * c / kGroup, s, m);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 n = two_codes(w[c] >> (4 * j));
            x[j] = fmaf(s, n.x, m);
            x[4 + j] = fmaf(s, n.y, m);
          }
          store_values<T, 8, kWide>(y + 8 * (4 * c + t), x);
        }
      }
    }
    if (p.out[1]) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int pair = t + 4 * i, r = 2 * pair;
        uint32_t w[C] = {}, meta[2][NG] = {};
        if (tile) load_words<C>(w, tile + ts.v_codes() + pair * D + ts.v_place(pair, g) * (D / 8));
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const bool held = tile && pos0 + r + k < len;
          if (held) load_words<NG>(meta[k], tile + ts.v_meta() + (r + k) * 4 * NG);
          T* y = out(1, r + k);
          if (!y) continue;
#pragma unroll
          for (int c = 0; c < C; ++c) {
            float s, m, x[4];
            group_meta<NG>(meta[k], 32 * c / kGroup, s, m);
            const uint32_t u = held ? (k ? w[c] >> 16 : w[c] & 0xffffu) : 0u;
            const float2 n0 = two_codes(u | u << 12), n1 = two_codes(u >> 8 | u << 4);      // codes 0, 1 and 2, 3
            x[0] = fmaf(s, n0.x, m);
            x[1] = fmaf(s, n0.y, m);
            x[2] = fmaf(s, n1.x, m);
            x[3] = fmaf(s, n1.y, m);
            store_values<T, 4, kWide>(y + 32 * c + 4 * g, x);
          }
        }
      }
    }
  }
}

template <typename T, int D, int kGroup>
cudaError_t launch_gather_rows(const GatherParams& p, bool wide, cudaStream_t s) {
  // one tile more than n holds, for a start inside a tile
  const int64_t tiles = (p.n + kTile - 1) / kTile + (p.starts ? 1 : 0);
  const int seqs = p.batch < 65535 / p.kv_heads ? p.batch : 65535 / p.kv_heads;
  const dim3 grid(unsigned((tiles + 7) / 8), unsigned(seqs * p.kv_heads));
  return wide ? launch_early(k_paged_gather<T, D, kGroup, true>, grid, 256, 0, s, p)
              : launch_early(k_paged_gather<T, D, kGroup, false>, grid, 256, 0, s, p);
}

template <typename T>
cudaError_t dispatch_gather(const GatherParams& p, int d, int group, bool wide, cudaStream_t s) {
  if (d == 128 && group == 32) return launch_gather_rows<T, 128, 32>(p, wide, s);
  if (d == 128 && group == 64) return launch_gather_rows<T, 128, 64>(p, wide, s);
  if (d == 128) return launch_gather_rows<T, 128, 128>(p, wide, s);
  if (group == 32) return launch_gather_rows<T, 64, 32>(p, wide, s);
  return launch_gather_rows<T, 64, 64>(p, wide, s);
}

}  // namespace
}  // namespace reskv

using namespace reskv;

extern "C" int64_t reskv_paged_head_bytes(int32_t page_tokens, int32_t head_dim, int32_t quant_group) {
  if (page_tokens < kTile || page_tokens > 1024 || page_tokens % kTile) return 0;
  if (head_dim != 64 && head_dim != 128) return 0;
  if ((quant_group != 32 && quant_group != 64 && quant_group != 128) || head_dim % quant_group) return 0;
  return int64_t(page_tokens / kTile) * TileShape{head_dim, head_dim / quant_group}.bytes();
}

extern "C" reskv_status reskv_paged_append(const reskv_paged_kv* kv, int64_t n_tokens, const int32_t* seqs,
                                           const int32_t* positions, const reskv_rotation* rot,
                                           const reskv_heads* k, const reskv_heads* v, const reskv_heads* q,
                                           const reskv_heads* q_out, void* stream) {
  return no_throw([&]() -> reskv_status {
    if (n_tokens == 0) return RESKV_OK;
    std::string bad = check_paged(kv);
    if (bad.empty()) bad = check_heads(k, "k");
    if (bad.empty()) bad = check_heads(v, "v");
    if (bad.empty() && rot) bad = check_rotation(rot, kv->head_dim);
    if (bad.empty() && (!seqs || !positions)) bad = "seqs or positions is NULL";
    if (bad.empty() && (k->n_heads != kv->n_kv_heads || v->n_heads != kv->n_kv_heads))
      bad = "k and v must have the cache's n_kv_heads";
    if (bad.empty() && k->dtype != v->dtype) bad = "k and v must have one dtype";
    if (bad.empty() && (q != nullptr) != (q_out != nullptr)) bad = "q and q_out go together";
    if (bad.empty() && q && !rot) bad = "q needs a rotation";
    if (bad.empty() && q) bad = check_heads(q, "q");
    if (bad.empty() && q) bad = check_heads(q_out, "q_out");
    if (bad.empty() && q && (q->n_heads != q_out->n_heads || q->dtype != q_out->dtype))
      bad = "q and q_out must have the same heads and one dtype";
    if (bad.empty() && (n_tokens < 0 || double(n_tokens) * kv->n_kv_heads >= double(int64_t(1) << 31)))
      bad = "n_tokens must not be negative, n_tokens * n_kv_heads below 2^31";
    if (bad.empty() && q && double(n_tokens) * q->n_heads >= double(int64_t(1) << 31)) bad = "n_tokens * heads must be below 2^31";
    if (!bad.empty()) return paged_fail(RESKV_ERR_INVALID_ARG, bad);
    AppendParams p{};
    p.seqs = seqs;
    p.positions = positions;
    p.page_table = kv->page_table;
    p.pages = static_cast<uint8_t*>(kv->pages);
    p.status = kv->status;
    p.k = k->data;
    p.v = v->data;
    p.k_token = k->token_stride;
    p.k_head = k->head_stride;
    p.v_token = v->token_stride;
    p.v_head = v->head_stride;
    p.n_pages = kv->n_pages;
    p.n_tokens = n_tokens;
    p.batch = kv->batch;
    p.table_pages = kv->table_pages;
    p.page_tokens = kv->page_tokens;
    p.kv_heads = kv->n_kv_heads;
    if (rot) {
      p.table = reinterpret_cast<const float2*>(rot->table);
      p.n_positions = rot->n_positions;
      p.rot = rot->rot_dim;
      p.interleaved = rot->interleaved;
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool wide = rows_aligned(*k, 16) && rows_aligned(*v, 16);
    RopeParams r{};
    if (q) {
      // in the same launch where its rows are moved in whole words like the keys', else in one of its own
      const int v16 = 16 / dtype_size(q->dtype);
      if (wide && q->dtype == k->dtype && rows_aligned(*q, 16) && rows_aligned(*q_out, 16) && aligned_to(rot->table, 16) &&
          rot->rot_dim % (2 * v16) == 0) {
        r.t[0] = RopeTensor{q->data, q_out->data, q->token_stride, q->head_stride, q_out->token_stride,
                            q_out->head_stride, q->n_heads};
        r.heads = q->n_heads;
        r.table = p.table;
        r.positions = positions;
        r.n_positions = rot->n_positions;
        r.n_tokens = n_tokens;
        r.status = kv->status;
        r.dim = kv->head_dim;
        r.rot = rot->rot_dim;
        r.interleaved = rot->interleaved;
      } else {
        const reskv_status st = reskv_rope(rot, positions, n_tokens, kv->head_dim, 1, q, q_out, 0, kv->status, stream);
        if (st != RESKV_OK) return st;
      }
    }
    const cudaError_t err =
        k->dtype == RESKV_F32   ? dispatch_append<float>(p, r, kv->head_dim, kv->quant_group, wide, s)
        : k->dtype == RESKV_F16 ? dispatch_append<__half>(p, r, kv->head_dim, kv->quant_group, wide, s)
                                : dispatch_append<__nv_bfloat16>(p, r, kv->head_dim, kv->quant_group, wide, s);
    return launch_result(err, "paged append");
  });
}

extern "C" reskv_status reskv_paged_gather(const reskv_paged_kv* kv, const int32_t* starts, const int32_t* lens,
                                           int64_t n, const reskv_rows* k, const reskv_rows* v, void* stream) {
  return no_throw([&]() -> reskv_status {
    if (n == 0) return RESKV_OK;
    std::string bad = check_paged(kv);
    if (bad.empty() && !lens) bad = "lens is NULL";
    if (bad.empty() && !k && !v) bad = "k and v are both NULL";
    if (bad.empty() && k && v && k->dtype != v->dtype) bad = "k and v must have one dtype";
    GatherParams p{};
    bool wide = true;
    const reskv_rows* rows[2] = {k, v};
    for (int i = 0; i < 2 && bad.empty(); ++i) {
      const reskv_rows* r = rows[i];
      if (!r) continue;
      if (!r->data || !dtype_known(r->dtype)) { bad = "an output is NULL or of an unknown dtype"; break; }
      const int64_t size = dtype_size(r->dtype);
      if (!aligned_to(r->data, size)) bad = "outputs must be aligned to their element size";
      if (r->batch_stride < 0 || r->head_stride < 0 || r->token_stride < 0) bad = "strides must not be negative";
      wide = wide && aligned_to(r->data, 16) && r->batch_stride * size % 16 == 0 && r->head_stride * size % 16 == 0 &&
             r->token_stride * size % 16 == 0;
      p.out[i] = r->data;
      p.b_stride[i] = r->batch_stride;
      p.h_stride[i] = r->head_stride;
      p.t_stride[i] = r->token_stride;
    }
    if (bad.empty() && (n < 0 || n >= (int64_t(1) << 31))) bad = "n must be in [0, 2^31)";
    if (!bad.empty()) return paged_fail(RESKV_ERR_INVALID_ARG, bad);
    p.starts = starts;
    p.lens = lens;
    p.page_table = kv->page_table;
    p.pages = static_cast<const uint8_t*>(kv->pages);
    p.status = kv->status;
    p.n = n;
    p.n_pages = kv->n_pages;
    p.table_pages = kv->table_pages;
    p.page_tokens = kv->page_tokens;
    p.kv_heads = kv->n_kv_heads;
    p.batch = kv->batch;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int32_t dt = k ? k->dtype : v->dtype;
    const cudaError_t err = dt == RESKV_F32   ? dispatch_gather<float>(p, kv->head_dim, kv->quant_group, wide, s)
                            : dt == RESKV_F16 ? dispatch_gather<__half>(p, kv->head_dim, kv->quant_group, wide, s)
                                              : dispatch_gather<__nv_bfloat16>(p, kv->head_dim, kv->quant_group, wide, s);
    return launch_result(err, "paged gather");
  });
}
