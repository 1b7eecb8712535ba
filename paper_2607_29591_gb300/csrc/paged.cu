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
};

// min and max that keep a NaN
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Four neighbouring dims per lane, D / 4 lanes a row: the codes of the lane's
// dims (16 bits) and its group's scale (low half) and minimum (high half).
template <int kGroup>
__device__ __forceinline__ void hold(const float (&x)[4], uint32_t& codes, uint32_t& sm) {
  float lo = min_nan(min_nan(x[0], x[1]), min_nan(x[2], x[3]));
  float hi = max_nan(max_nan(x[0], x[1]), max_nan(x[2], x[3]));
#pragma unroll
  for (int o = 1; o < kGroup / 4; o *= 2) {
    lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
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
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float n = fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(x[i], m), s)), 0.f), 15.f);
      codes |= uint32_t(int(n)) << (4 * i);
    }
  }
  sm = s16 | (m16 << 16);
}

// One (token, KV head) per D / 4 lanes: K row, then V row.
template <typename T, int D, int kGroup, bool kWide>
__global__ void __launch_bounds__(256) k_paged_append(const __grid_constant__ AppendParams p) {
  constexpr int L = D / 4, NG = D / kGroup;
  constexpr TileShape ts{D, NG};
  using P = Pack<T, 4>;
  const int lane = threadIdx.x % L;
  int64_t r = int64_t(blockIdx.x) * (256 / L) + threadIdx.x / L;
  const bool in = r < p.n_tokens * p.kv_heads;
  if (!in) r = 0;                                   // stays for the shuffles, writes nothing
  const int64_t tok = r / p.kv_heads;
  const int h = int(r - tok * p.kv_heads);
  const int pos = p.positions[tok], seq = p.seqs[tok];
  bool live = in && pos >= 0, fault = false;
  uint8_t* tile = nullptr;
  int row = 0;
  if (live) {
    const int pg = pos / p.page_tokens;
    fault = seq < 0 || seq >= p.batch || pg >= p.table_pages || (p.table && pos >= p.n_positions);
    if (!fault) {
      const int page = p.page_table[int64_t(seq) * p.table_pages + pg];
      fault = page < 0 || page >= p.n_pages;
      const int slot = pos - pg * p.page_tokens;
      row = slot % kTile;
      tile = p.pages + ((int64_t(page) * p.kv_heads + h) * (p.page_tokens / kTile) + slot / kTile) * ts.bytes();
    }
    if (fault && lane == 0) report_status(p.status, kStatusBadIndex);
    live = !fault;
  }
  const T* k = static_cast<const T*>(p.k) + tok * p.k_token + h * p.k_head;
  const T* v = static_cast<const T*>(p.v) + tok * p.v_token + h * p.v_head;
  float x[4];
  auto load = [&](const T* at) {
    if constexpr (kWide) {
      const P a = *reinterpret_cast<const P*>(at);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = to_f32(a.v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = to_f32(at[i]);
    }
  };
  uint32_t codes, sm;
  load(k + 4 * lane);
  if (p.table && live) {
    const float2* cs = p.table + int64_t(pos) * (p.rot / 2);
    const int half = p.rot / 2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int dim = 4 * lane + i;
      if (dim >= p.rot) continue;
      const bool lower = p.interleaved ? dim % 2 == 0 : dim < half;
      const int pair = p.interleaved ? dim / 2 : (lower ? dim : dim - half);
      const int other = p.interleaved ? dim ^ 1 : (lower ? dim + half : dim - half);
      float a = to_f32(k[lower ? dim : other]), b = to_f32(k[lower ? other : dim]);
      const float2 c = cs[pair];
      turn(a, b, c.x, c.y);
      x[i] = lower ? a : b;
    }
  }
  hold<kGroup>(x, codes, sm);
  if (live) {
    *reinterpret_cast<uint16_t*>(tile + ts.k_unit(row, lane)) = uint16_t(codes);
    if (lane % (kGroup / 4) == 0) {
      uint16_t* meta = reinterpret_cast<uint16_t*>(tile + ts.k_meta()) + row * 2 * NG + lane / (kGroup / 4);
      meta[0] = uint16_t(sm);
      meta[NG] = uint16_t(sm >> 16);
    }
  }
  load(v + 4 * lane);
  hold<kGroup>(x, codes, sm);
  if (live) {
    *reinterpret_cast<uint16_t*>(tile + ts.v_codes() + ts.v_unit(row, lane)) = uint16_t(codes);
    if (lane % (kGroup / 4) == 0) {
      uint16_t* meta = reinterpret_cast<uint16_t*>(tile + ts.v_meta()) + row * 2 * NG + lane / (kGroup / 4);
      meta[0] = uint16_t(sm);
      meta[NG] = uint16_t(sm >> 16);
    }
  }
}

template <typename T, int D, int kGroup>
void launch_append_rows(const AppendParams& p, bool wide, cudaStream_t s) {
  constexpr int rows = 256 / (D / 4);
  const unsigned blocks = unsigned((p.n_tokens * p.kv_heads + rows - 1) / rows);
  if (wide) k_paged_append<T, D, kGroup, true><<<blocks, 256, 0, s>>>(p);
  else k_paged_append<T, D, kGroup, false><<<blocks, 256, 0, s>>>(p);
}

template <typename T>
void dispatch_append(const AppendParams& p, int d, int group, bool wide, cudaStream_t s) {
  if (d == 128 && group == 32) launch_append_rows<T, 128, 32>(p, wide, s);
  else if (d == 128 && group == 64) launch_append_rows<T, 128, 64>(p, wide, s);
  else if (d == 128) launch_append_rows<T, 128, 128>(p, wide, s);
  else if (group == 32) launch_append_rows<T, 64, 32>(p, wide, s);
  else launch_append_rows<T, 64, 64>(p, wide, s);
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

// Eight dims per thread, D / 8 threads a row; blockIdx.y: sequence and head.
template <typename T, int D, int kGroup, bool kWide>
__global__ void __launch_bounds__(256) k_paged_gather(const __grid_constant__ GatherParams p) {
  constexpr int L = D / 8, NG = D / kGroup;
  constexpr TileShape ts{D, NG};
  const int w = threadIdx.x % L;
  const int64_t i = int64_t(blockIdx.x) * (256 / L) + threadIdx.x / L;
  if (i >= p.n) return;
  for (int bh = blockIdx.y; bh < p.batch * p.kv_heads; bh += gridDim.y) {
    const int b = bh / p.kv_heads, h = bh - b * p.kv_heads;
    const int64_t pos = (p.starts ? int64_t(p.starts[b]) : 0) + i;
    const uint8_t* tile = nullptr;
    int row = 0;
    if (pos >= 0 && pos < p.lens[b]) {
      const int64_t pg = pos / p.page_tokens;
      const int page = pg < p.table_pages ? p.page_table[int64_t(b) * p.table_pages + pg] : -1;
      if (page >= 0 && page < p.n_pages) {
        const int slot = int(pos - pg * p.page_tokens);
        row = slot % kTile;
        tile = p.pages + ((int64_t(page) * p.kv_heads + h) * (p.page_tokens / kTile) + slot / kTile) * ts.bytes();
      } else if (w == 0) {
        report_status(p.status, kStatusBadIndex);
      }
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      if (!p.out[kv]) continue;
      float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (tile) {
        uint32_t word;
        if (kv == 0) {
          word = *reinterpret_cast<const uint32_t*>(tile + ts.k_unit(row, 2 * w));
        } else {
          const uint8_t* codes = tile + ts.v_codes();
          word = *reinterpret_cast<const uint16_t*>(codes + ts.v_unit(row, 2 * w)) |
                 uint32_t(*reinterpret_cast<const uint16_t*>(codes + ts.v_unit(row, 2 * w + 1))) << 16;
        }
        const uint16_t* meta =
            reinterpret_cast<const uint16_t*>(tile + (kv ? ts.v_meta() : ts.k_meta())) + row * 2 * NG + 8 * w / kGroup;
        const float s = __uint_as_float(uint32_t(meta[0]) << 16), m = __uint_as_float(uint32_t(meta[NG]) << 16);
        // s n is exact in fp32, so this is one rounding like s * n + m
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = fmaf(s, float((word >> (4 * j)) & 15u), m);
      }
      T* y = static_cast<T*>(p.out[kv]) + b * p.b_stride[kv] + h * p.h_stride[kv] + i * p.t_stride[kv] + 8 * w;
      if constexpr (kWide) {
        Pack<T, 8> o;                               // 16 bytes, 32 for fp32
#pragma unroll
        for (int j = 0; j < 8; ++j) o.v[j] = from_f32<T>(x[j]);
        constexpr int words = sizeof(T) * 8 / 16;
        const uint4* from = reinterpret_cast<const uint4*>(&o);
#pragma unroll
        for (int j = 0; j < words; ++j) reinterpret_cast<uint4*>(y)[j] = from[j];
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = from_f32<T>(x[j]);
      }
    }
  }
}

template <typename T, int D, int kGroup>
void launch_gather_rows(const GatherParams& p, bool wide, cudaStream_t s) {
  constexpr int rows = 256 / (D / 8);
  const int64_t bh = int64_t(p.batch) * p.kv_heads;
  const dim3 grid(unsigned((p.n + rows - 1) / rows), unsigned(bh < 65535 ? bh : 65535));
  if (wide) k_paged_gather<T, D, kGroup, true><<<grid, 256, 0, s>>>(p);
  else k_paged_gather<T, D, kGroup, false><<<grid, 256, 0, s>>>(p);
}

template <typename T>
void dispatch_gather(const GatherParams& p, int d, int group, bool wide, cudaStream_t s) {
  if (d == 128 && group == 32) launch_gather_rows<T, 128, 32>(p, wide, s);
  else if (d == 128 && group == 64) launch_gather_rows<T, 128, 64>(p, wide, s);
  else if (d == 128) launch_gather_rows<T, 128, 128>(p, wide, s);
  else if (group == 32) launch_gather_rows<T, 64, 32>(p, wide, s);
  else launch_gather_rows<T, 64, 64>(p, wide, s);
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
  if (bad.empty() && (n_tokens < 0 || double(n_tokens) * kv->n_kv_heads >= double(int64_t(1) << 31)))
    bad = "n_tokens must not be negative, n_tokens * n_kv_heads below 2^31";
  if (!bad.empty()) return paged_fail(RESKV_ERR_INVALID_ARG, bad);
  if (q) {
    const reskv_status st = reskv_rope(rot, positions, n_tokens, kv->head_dim, 1, q, q_out, 0, kv->status, stream);
    if (st != RESKV_OK) return st;
  }
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
  const size_t word = 4 * dtype_size(k->dtype);
  const bool wide = rows_aligned(*k, word) && rows_aligned(*v, word);
  if (k->dtype == RESKV_F32) dispatch_append<float>(p, kv->head_dim, kv->quant_group, wide, s);
  else if (k->dtype == RESKV_F16) dispatch_append<__half>(p, kv->head_dim, kv->quant_group, wide, s);
  else dispatch_append<__nv_bfloat16>(p, kv->head_dim, kv->quant_group, wide, s);
  return launch_status("paged append");
}

extern "C" reskv_status reskv_paged_gather(const reskv_paged_kv* kv, const int32_t* starts, const int32_t* lens,
                                           int64_t n, const reskv_rows* k, const reskv_rows* v, void* stream) {
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
  if (dt == RESKV_F32) dispatch_gather<float>(p, kv->head_dim, kv->quant_group, wide, s);
  else if (dt == RESKV_F16) dispatch_gather<__half>(p, kv->head_dim, kv->quant_group, wide, s);
  else dispatch_gather<__nv_bfloat16>(p, kv->head_dim, kv->quant_group, wide, s);
  return launch_status("paged gather");
}
