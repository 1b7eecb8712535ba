// The paged 4-bit cache (include/reskv.h, reskv_paged_kv): where a tile keeps
// its codes, scales and minima, element types of the rows around it, and the
// rotation of a pair.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <string>

#include "device_utils.cuh"
#include "internal.h"
#include "reskv.h"

namespace reskv {

constexpr int kTile = 16;             // tokens of a tile

// Offsets within a tile of d dims and ng groups a row.
struct TileShape {
  int d, ng;
  __host__ __device__ constexpr int codes() const { return kTile * d / 2; }
  __host__ __device__ constexpr int meta() const { return kTile * ng * 4; }
  __host__ __device__ constexpr int k_meta() const { return codes(); }
  __host__ __device__ constexpr int v_codes() const { return codes() + meta(); }
  __host__ __device__ constexpr int v_meta() const { return 2 * codes() + meta(); }
  __host__ __device__ constexpr int bytes() const { return 2 * (codes() + meta()); }
  // byte of the 16-bit unit of dims 4u .. 4u+3 of row r of the K codes
  __host__ __device__ constexpr int k_unit(int r, int u) const {
    return r * (d / 2) + ((u / 2 % 4) * (d / 32) + u / 8) * 4 + (u & 1) * 2;
  }
  // place of chunk g in pair row r of the V codes
  __host__ __device__ constexpr int v_place(int r, int g) const {
    return g ^ (d == 128 ? 2 * (r & 3) : 4 * ((r >> 1) & 1));
  }
  // byte (from v_codes()) of the 16-bit unit of dims 4u .. 4u+3 of row r
  __host__ __device__ constexpr int v_unit(int r, int u) const {
    return (r >> 1) * d + v_place(r >> 1, u & 7) * (d / 8) + (u >> 3) * 4 + (r & 1) * 2;
  }
};

// One element of a row of any dtype, as fp32 and back (round to nearest even).
template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32(float x) { return x; }
template <> __device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32(float x) { return x; }
template <> __device__ __forceinline__ __half from_f32(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float x) { return __float2bfloat16_rn(x); }

// N neighbouring elements, moved as one word (aligned to their size).
template <typename T, int N>
struct alignas(sizeof(T) * N) Pack {
  T v[N];
};

__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// One, two or four neighbouring 32-bit words.
template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const void* p) {
  if constexpr (N == 4) {
    const uint4 v = *static_cast<const uint4*>(p);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  } else if constexpr (N == 2) {
    const uint2 v = *static_cast<const uint2*>(p);
    w[0] = v.x; w[1] = v.y;
  } else {
    w[0] = *static_cast<const uint32_t*>(p);
  }
}

// Scale and minimum of one group from a row's words.
template <int NG>
__device__ __forceinline__ void group_meta(const uint32_t (&w)[NG], int k, float& s, float& m) {
  if constexpr (NG == 1) {
    s = low_bf16(w[0]);
    m = high_bf16(w[0]);
  } else {
    s = k & 1 ? high_bf16(w[k / 2]) : low_bf16(w[k / 2]);
    m = k & 1 ? high_bf16(w[NG / 2 + k / 2]) : low_bf16(w[NG / 2 + k / 2]);
  }
}

// (a, b) turned by (cos, sin): products and sums rounded one by one, so that a
// key is held with the same codes whatever path rotated it.  (Packed mul.rn and
// add.rn pairs came out fused.)
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
  const float x = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
  const float y = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
  a = x;
  b = y;
}

// The kernels of a decode step follow one another within microseconds: each is
// launched while the one before it on the stream still runs, and waits for its
// end before it touches memory (wait_for_previous, the first thing they do).
template <typename... P, typename... A>
cudaError_t launch_early(void (*kernel)(P...), dim3 grid, dim3 block, size_t shared, cudaStream_t s, A... args) {
  cudaLaunchAttribute early{};
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = shared;
  cfg.stream = s;
  cfg.attrs = &early;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
__device__ __forceinline__ void wait_for_previous() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

inline int dtype_size(int32_t dtype) { return dtype == RESKV_F32 ? 4 : 2; }
inline bool dtype_known(int32_t dtype) { return dtype >= RESKV_BF16 && dtype <= RESKV_F32; }
inline bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Whether every row of the tensor starts on a `bytes` boundary.
inline bool rows_aligned(const reskv_heads& t, size_t bytes) {
  const int64_t size = dtype_size(t.dtype);
  return aligned_to(t.data, bytes) && t.token_stride * size % int64_t(bytes) == 0 &&
         t.head_stride * size % int64_t(bytes) == 0;
}

// An entry point's body: nothing is thrown across the C boundary (what can throw
// is the text of an error).
template <typename F>
reskv_status no_throw(F body) noexcept {
  try {
    return body();
  } catch (...) {
    return RESKV_ERR_OOM;
  }
}

// Host checks shared by the entry points; "" when fine.
std::string check_heads(const reskv_heads* t, const char* name);
std::string check_rotation(const reskv_rotation* r, int32_t head_dim);
std::string check_paged(const reskv_paged_kv* kv);
reskv_status paged_fail(reskv_status st, const std::string& msg);
reskv_status launch_result(cudaError_t err, const char* what);

// One or two tensors of rows turned in one launch; rope.cu.
struct RopeTensor {
  const void* x;
  void* y;
  int64_t x_token, x_head, y_token, y_head;
  int32_t heads;
};
struct RopeParams {
  RopeTensor t[2];
  const float2* table;
  const int32_t* positions;
  int64_t n_positions;
  int64_t n_tokens;
  uint32_t* status;
  int32_t heads;          // of both tensors
  int32_t dim, rot;
  int32_t lanes;          // threads of a row
  int32_t rows_per_block; // rows (of kHeads heads) a block takes
  int32_t head_groups;    // ceil(heads / heads a thread takes)
  int32_t interleaved, backward;
};

// Threads of a row for V elements a word: rot / 2V of them turn V pairs each, the
// others copy 2V of the remaining dims.
inline int rope_lanes(int dim, int rot, int v) { return rot / (2 * v) + ((dim - rot) / v + 1) / 2; }

// Heads a thread takes where a call has rows enough: 16-bit words come out of more
// registers, so that four heads would leave fewer threads to an SM.
template <typename T> constexpr int kManyHeads = sizeof(T) == 2 ? 2 : 4;

// Thread `lane` of row group r: the lane's pairs of kHeads neighbouring heads of one
// token, whose cos and sin are read once.  All rows are asked for before the first
// is turned.
template <typename T, int V, bool kInter, int kHeads>
__device__ __forceinline__ void rope_rows(const RopeParams& p, int64_t r, int lane) {
  using P = Pack<T, V>;
  const int64_t tok = uint32_t(r) / uint32_t(p.head_groups);        // r is below 2^31
  if (tok >= p.n_tokens) return;
  const int h0 = (int(r) - int(tok) * p.head_groups) * kHeads;
  const int turners = p.rot / (2 * V);
  const int64_t pos = p.positions[tok];
  const bool live = pos >= 0 && pos < p.n_positions;
  if (pos >= p.n_positions && h0 == 0 && lane == 0) report_status(p.status, kStatusBadIndex);
  // the lane's two words of a row
  const bool turns = lane < turners;
  const int ia = turns ? (kInter ? 2 * V * lane : V * lane) : p.rot + 2 * V * (lane - turners);
  const int ib = turns && !kInter ? ia + p.rot / 2 : ia + V;
  const bool two = ib < p.dim;
  P a[kHeads], b[kHeads];
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int h = min(h0 + i, p.heads - 1);
    const bool second = h >= p.t[0].heads;
    const RopeTensor& t = p.t[second];
    const T* x = static_cast<const T*>(t.x) + tok * t.x_token + (second ? h - p.t[0].heads : h) * t.x_head;
    a[i] = *reinterpret_cast<const P*>(x + ia);
    if (two) b[i] = *reinterpret_cast<const P*>(x + ib);
  }
  if (turns && live) {
    const float2* cs = p.table + pos * (p.rot / 2) + V * lane;
    if constexpr (V == 1) {
      const float2 c = cs[0];
#pragma unroll
      for (int i = 0; i < kHeads; ++i) {
        float fa = to_f32(a[i].v[0]), fb = to_f32(b[i].v[0]);
        turn(fa, fb, c.x, p.backward ? -c.y : c.y);
        a[i].v[0] = from_f32<T>(fa);
        b[i].v[0] = from_f32<T>(fb);
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; j += 2) {
        const float4 w = *reinterpret_cast<const float4*>(cs + j);
        const float2 c = make_float2(w.x, w.z);
        const float2 s = p.backward ? make_float2(-w.y, -w.w) : make_float2(w.y, w.w);
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
          // pairs j, j + 1 of this lane: (a[j], b[j]), or neighbours of the 2V elements
          P& half = 2 * j < V ? a[i] : b[i];
          T& a0 = kInter ? half.v[(2 * j) % V] : a[i].v[j];
          T& b0 = kInter ? half.v[(2 * j + 1) % V] : b[i].v[j];
          T& a1 = kInter ? half.v[(2 * j + 2) % V] : a[i].v[j + 1];
          T& b1 = kInter ? half.v[(2 * j + 3) % V] : b[i].v[j + 1];
          float fa0 = to_f32(a0), fb0 = to_f32(b0), fa1 = to_f32(a1), fb1 = to_f32(b1);
          turn(fa0, fb0, c.x, s.x);
          turn(fa1, fb1, c.y, s.y);
          a0 = from_f32<T>(fa0);
          b0 = from_f32<T>(fb0);
          a1 = from_f32<T>(fa1);
          b1 = from_f32<T>(fb1);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int h = h0 + i;
    if (h >= p.heads) break;
    const bool second = h >= p.t[0].heads;
    const RopeTensor& t = p.t[second];
    T* y = static_cast<T*>(t.y) + tok * t.y_token + (second ? h - p.t[0].heads : h) * t.y_head;
    *reinterpret_cast<P*>(y + ia) = a[i];
    if (two) *reinterpret_cast<P*>(y + ib) = b[i];
  }
}

}  // namespace reskv
