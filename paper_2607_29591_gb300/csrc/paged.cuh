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

// (a, b) turned by (cos, sin): products and sums rounded one by one, so that a
// key is held with the same codes whatever path rotated it.
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

// Host checks shared by the entry points; "" when fine.
std::string check_heads(const reskv_heads* t, const char* name);
std::string check_rotation(const reskv_rotation* r, int32_t head_dim);
std::string check_paged(const reskv_paged_kv* kv);
reskv_status paged_fail(reskv_status st, const std::string& msg);
reskv_status launch_status(const char* what);

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
  int32_t rows_per_block;
  int32_t head_groups;    // ceil(heads / heads a thread)
  int32_t interleaved, backward;
};

}  // namespace reskv
