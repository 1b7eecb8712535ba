// Rotary positions: the table of cos and sin (reskv_rope_table) and the
// rotation of rows by it (reskv_rope).
#include <cmath>

#include "paged.cuh"

namespace reskv {

reskv_status paged_fail(reskv_status st, const std::string& msg) {
  set_error(msg);
  return st;
}

reskv_status launch_result(cudaError_t err, const char* what) {
  if (err == cudaSuccess) return RESKV_OK;
  cudaGetLastError();
  return paged_fail(RESKV_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(err));
}

std::string check_heads(const reskv_heads* t, const char* name) {
  const std::string n(name);
  if (!t || !t->data) return n + " is NULL";
  if (!dtype_known(t->dtype)) return n + ": unknown dtype";
  if (t->n_heads < 1 || t->n_heads > 65536) return n + ": n_heads must be in [1, 65536]";
  if (t->token_stride < 0 || t->head_stride < 0) return n + ": strides must not be negative";
  if (!aligned_to(t->data, dtype_size(t->dtype))) return n + " must be aligned to its element size";
  return "";
}

std::string check_rotation(const reskv_rotation* r, int32_t head_dim) {
  if (!r || !r->table) return "the rotation's table is NULL";
  if (!aligned_to(r->table, 8)) return "the rotation's table must be 8-byte aligned";
  if (r->rot_dim < 2 || r->rot_dim % 2 || r->rot_dim > head_dim)
    return "rot_dim must be even and in [2, head_dim]";
  if (r->n_positions < 1 || r->n_positions > (int64_t(1) << 31)) return "n_positions must be in [1, 2^31]";
  if (r->interleaved != 0 && r->interleaved != 1) return "interleaved must be 0 or 1";
  return "";
}

namespace {

// --- the table -------------------------------------------------------------

constexpr int kMaxPairs = 256;
struct Frequencies {
  double f[kMaxPairs];
};

// One thread per (position, pair).  Written once per model, so fp64: at position
// 2^17 an fp32 angle is off by up to 2^-7.
__global__ void k_rope_table(const __grid_constant__ Frequencies fr, float2* table, int64_t n, int pairs,
                             double magnitude) {
  const int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  if (i >= n * pairs) return;
  const int64_t p = i / pairs;
  double s, c;
  sincos(double(p) * fr.f[i - p * pairs], &s, &c);
  table[i] = make_float2(float(magnitude * c), float(magnitude * s));
}

// --- the rotation ----------------------------------------------------------

// a' = a c - b s, b' = b c + a s, every product and sum rounded once (s negated: the
// gradient).  A row's bytes pass once, its cos and sin once for kHeads heads.
// Blocks of 128 threads end more evenly than ones of 256 (8191 tokens of 40 heads 32.5
// against 33.9 us); single elements may take 256 for a row.
template <int V> constexpr int kRopeThreads = V == 1 ? 256 : 128;
template <typename T, int V, bool kInter, int kHeads>
__global__ void __launch_bounds__(kRopeThreads<V>, (kHeads == 1 ? 1536 : 1024) / kRopeThreads<V>) k_rope(const __grid_constant__ RopeParams p) {
  wait_for_previous();
  rope_rows<T, V, kInter, kHeads>(p, int64_t(blockIdx.x) * p.rows_per_block + threadIdx.y, threadIdx.x);
}

// Two heads (fp32: four) a thread where the rows of one leave every SM four times
// 2048 threads, one where there are fewer (a single token's launch is all latency).
// Bound by its bytes: 8191 tokens of 40 heads of 128, 172 MB of bf16 read and written
// in 32 us, 5.3 TB/s (the rows, of half the L2's size, are partly written back
// after the call); of fp32 back, 98 us at 6.9 TB/s.
template <typename T, int V, int kHeads>
cudaError_t launch_rope(RopeParams p, cudaStream_t s) {
  p.lanes = rope_lanes(p.dim, p.rot, V);
  p.rows_per_block = kRopeThreads<V> / p.lanes;
  p.head_groups = (p.heads + kHeads - 1) / kHeads;
  const int64_t rows = p.n_tokens * p.head_groups;
  const unsigned blocks = unsigned((rows + p.rows_per_block - 1) / p.rows_per_block);
  const dim3 block(p.lanes, p.rows_per_block);
  return p.interleaved ? launch_early(k_rope<T, V, true, kHeads>, blocks, block, 0, s, p)
                       : launch_early(k_rope<T, V, false, kHeads>, blocks, block, 0, s, p);
}

template <typename T>
cudaError_t dispatch_rope(const RopeParams& p, bool wide, cudaStream_t s) {
  constexpr int V = 16 / int(sizeof(T));
  if (!wide || p.rot % (2 * V) || p.dim % V) return launch_rope<T, 1, 1>(p, s);
  if (p.n_tokens * p.heads * rope_lanes(p.dim, p.rot, V) >= int64_t(152) * 8192) return launch_rope<T, V, kManyHeads<T>>(p, s);
  return launch_rope<T, V, 1>(p, s);
}

}  // namespace
}  // namespace reskv

using namespace reskv;

extern "C" void reskv_rope_config_default(reskv_rope_config* cfg) {
  if (!cfg) return;
  *cfg = reskv_rope_config{};
  cfg->rot_dim = kHeadDim;
  cfg->scaling = RESKV_ROPE_NONE;
  cfg->base = 500000.0;
  cfg->factor = 1.0;
  cfg->original_positions = 8192.0;
  cfg->low_freq = 1.0;
  cfg->high_freq = 4.0;
  cfg->beta_fast = 32.0;
  cfg->beta_slow = 1.0;
  cfg->magnitude = 0.0;
}

extern "C" reskv_status reskv_rope_table(const reskv_rope_config* c, int64_t n_positions, float* table,
                                         void* stream) {
  return no_throw([&]() -> reskv_status {
    if (!c || !table) return paged_fail(RESKV_ERR_INVALID_ARG, "NULL argument");
    if (!aligned_to(table, 8)) return paged_fail(RESKV_ERR_INVALID_ARG, "table must be 8-byte aligned");
    const int R = c->rot_dim, pairs = R / 2;
    if (R < 2 || R % 2 || pairs > kMaxPairs)
      return paged_fail(RESKV_ERR_INVALID_ARG, "rot_dim must be even and in [2, 512]");
    if (n_positions < 1 || n_positions > (int64_t(1) << 31))
      return paged_fail(RESKV_ERR_INVALID_ARG, "n_positions must be in [1, 2^31]");
    if (!(c->base > 1.0) || !std::isfinite(c->base) || !(c->factor >= 1.0) || !std::isfinite(c->factor))
      return paged_fail(RESKV_ERR_INVALID_ARG, "need base > 1 and factor >= 1");
    if (!(c->magnitude >= 0.0) || !std::isfinite(c->magnitude))
      return paged_fail(RESKV_ERR_INVALID_ARG, "magnitude must not be negative");
    const double two_pi = 6.283185307179586476925;
    const bool by_turns = c->scaling == RESKV_ROPE_WAVELENGTH, yarn = c->scaling == RESKV_ROPE_YARN;
    if ((by_turns || yarn) && (!(c->original_positions >= 1.0) || !std::isfinite(c->original_positions)))
      return paged_fail(RESKV_ERR_INVALID_ARG, "original_positions must be >= 1");
    if (by_turns && !(c->low_freq > 0.0 && c->high_freq > c->low_freq && std::isfinite(c->high_freq)))
      return paged_fail(RESKV_ERR_INVALID_ARG, "need 0 < low_freq < high_freq");
    if (yarn && !(c->beta_slow > 0.0 && c->beta_fast > c->beta_slow && std::isfinite(c->beta_fast)))
      return paged_fail(RESKV_ERR_INVALID_ARG, "need 0 < beta_slow < beta_fast");
    if (c->scaling < RESKV_ROPE_NONE || c->scaling > RESKV_ROPE_YARN)
      return paged_fail(RESKV_ERR_INVALID_ARG, "unknown scaling");
    if (c->scaling == RESKV_ROPE_BASE && R < 4)
      return paged_fail(RESKV_ERR_INVALID_ARG, "RESKV_ROPE_BASE needs rot_dim >= 4");

    Frequencies fr{};
    const double base = c->scaling == RESKV_ROPE_BASE ? c->base * std::pow(c->factor, double(R) / (R - 2)) : c->base;
    // YARN: the (fractional) pair that makes b turns within the original positions
    auto pair_of = [&](double b) {
      return R * std::log(c->original_positions / (b * two_pi)) / (2.0 * std::log(base));
    };
    const double first = std::fmax(0.0, std::floor(pair_of(c->beta_fast)));
    const double last = std::fmax(first + 1e-3, std::fmin(R - 1.0, std::ceil(pair_of(c->beta_slow))));
    for (int i = 0; i < pairs; ++i) {
      const double f = std::pow(base, -2.0 * i / R);
      double w = 0.0;                       // share of the interpolated frequency
      if (c->scaling == RESKV_ROPE_LINEAR) w = 1.0;
      if (by_turns)
        w = (c->high_freq - c->original_positions * f / two_pi) / (c->high_freq - c->low_freq);
      if (yarn) w = (i - first) / (last - first);
      w = std::fmin(1.0, std::fmax(0.0, w));
      fr.f[i] = f * (1.0 - w) + f / c->factor * w;
    }
    double m = c->magnitude;
    if (m == 0.0) m = yarn ? 0.1 * std::log(c->factor) + 1.0 : 1.0;
    const int64_t n = n_positions * pairs, blocks = (n + 255) / 256;
    if (blocks > 0x7fffffff) return paged_fail(RESKV_ERR_UNSUPPORTED, "table too large");
    k_rope_table<<<unsigned(blocks), 256, 0, static_cast<cudaStream_t>(stream)>>>(
        fr, reinterpret_cast<float2*>(table), n_positions, pairs, m);
    return launch_result(cudaGetLastError(), "rope table");
  });
}

extern "C" reskv_status reskv_rope(const reskv_rotation* rot, const int32_t* positions, int64_t n_tokens,
                                   int32_t head_dim, int32_t n_tensors, const reskv_heads* x,
                                   const reskv_heads* y, int32_t backward, uint32_t* status, void* stream) {
  return no_throw([&]() -> reskv_status {
    if (n_tokens == 0) return RESKV_OK;
    if (!x || !y || !positions) return paged_fail(RESKV_ERR_INVALID_ARG, "NULL argument");
    if (n_tensors != 1 && n_tensors != 2) return paged_fail(RESKV_ERR_INVALID_ARG, "n_tensors must be 1 or 2");
    if (head_dim < 2 || head_dim % 2 || head_dim > 512)
      return paged_fail(RESKV_ERR_INVALID_ARG, "head_dim must be even and in [2, 512]");
    std::string bad = check_rotation(rot, head_dim);
    if (!bad.empty()) return paged_fail(RESKV_ERR_INVALID_ARG, bad);
    RopeParams p{};
    bool wide = true;
    for (int i = 0; i < n_tensors; ++i) {
      bad = check_heads(&x[i], "x");
      if (bad.empty()) bad = check_heads(&y[i], "y");
      if (!bad.empty()) return paged_fail(RESKV_ERR_INVALID_ARG, bad);
      if (x[i].n_heads != y[i].n_heads || x[i].dtype != y[i].dtype || x[i].dtype != x[0].dtype)
        return paged_fail(RESKV_ERR_INVALID_ARG, "x and y must have the same heads and one dtype");
      wide = wide && rows_aligned(x[i], 16) && rows_aligned(y[i], 16) && aligned_to(rot->table, 16);
      p.t[i] = RopeTensor{x[i].data, y[i].data, x[i].token_stride, x[i].head_stride, y[i].token_stride,
                          y[i].head_stride, x[i].n_heads};
      p.heads += x[i].n_heads;
    }
    if (n_tokens < 0 || double(n_tokens) * p.heads >= double(int64_t(1) << 31))
      return paged_fail(RESKV_ERR_INVALID_ARG, "n_tokens must not be negative, n_tokens * heads below 2^31");
    p.table = reinterpret_cast<const float2*>(rot->table);
    p.positions = positions;
    p.n_positions = rot->n_positions;
    p.n_tokens = n_tokens;
    p.status = status;
    p.dim = head_dim;
    p.rot = rot->rot_dim;
    p.interleaved = rot->interleaved;
    p.backward = backward != 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t err = x[0].dtype == RESKV_F32   ? dispatch_rope<float>(p, wide, s)
                            : x[0].dtype == RESKV_F16 ? dispatch_rope<__half>(p, wide, s)
                                                      : dispatch_rope<__nv_bfloat16>(p, wide, s);
    return launch_result(err, "rope");
  });
}
