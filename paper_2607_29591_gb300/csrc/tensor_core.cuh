// Instructions of the fifth-generation tensor cores (tcgen05) that the attention
// kernels share: operand descriptors, products, commits, tensor memory to registers.
#pragma once
#include <cuda.h>

#include <cstdint>

#include "device_utils.cuh"

namespace reskv {
namespace tc {

// Descriptors of K-major operands in shared memory: the address / 16 in the low
// word, beside a constant; in the high word the distance of groups of eight rows
// / 16, version 1 and the swizzle.  Rows of 128 bytes (64 fp16) have the 128-byte
// swizzle (16-byte word w of row r at w ^ (r & 7)); rows of 32 bytes (one step) the
// 32-byte swizzle (w at w ^ ((r >> 2) & 1)).
__device__ __forceinline__ uint32_t operand(uint32_t saddr) { return (saddr >> 4) | (1u << 16); }
// The same in a cluster, where a shared address has the CTA's rank above its 18 bits and a descriptor other
// fields there (an operand that lies across took its distances from the rank).
__device__ __forceinline__ uint32_t cluster_operand(uint32_t saddr) { return operand(saddr & 0x3ffffu); }
constexpr uint32_t kRows128 = (1024 >> 4) | (1u << 14) | (2u << 29);
// An operand that lies the other way round (a row holds 64 neighbours of the product's rows or
// columns, for one term of its sums): groups of eight such rows follow each other as above, `next64`
// bytes lead to the next 64 rows or columns.
__device__ __forceinline__ uint32_t operand_across(uint32_t saddr, uint32_t next64) { return ((saddr & 0x3ffffu) >> 4) | (next64 >> 4) << 16; }
constexpr uint32_t kRows32 = (256 >> 4) | (1u << 14) | (6u << 29);

// kind::f16, fp16 operands, fp32 accumulators, 128 rows, n columns
__host__ __device__ constexpr uint32_t shape_of(int n) { return (1u << 4) | (uint32_t(n >> 3) << 17) | (uint32_t(128 >> 4) << 24); }
// Of a shape: bf16 operands; the second operand lies across
constexpr uint32_t kBf16 = 1u << 7 | 1u << 10, kAcross = 1u << 16;
constexpr uint32_t kNegative = 1u << 13;          // the first operand's sign turned
template <uint32_t kHigh>
__device__ __forceinline__ void multiply(uint32_t d, uint32_t a, uint32_t b, uint32_t shape, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(kHigh), "r"(shape),
      "r"(add ? 1 : 0));
}
template <uint32_t kHigh, uint32_t kShape>
__device__ __forceinline__ void multiply(uint32_t d, uint32_t a, uint32_t b, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(kHigh), "r"(kShape),
      "r"(add ? 1 : 0));
}
// The same with the first operand in tensor memory: a row a lane, two fp16 a column.
template <uint32_t kHigh, uint32_t kShape>
__device__ __forceinline__ void multiply_from(uint32_t d, uint32_t a, uint32_t b, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 db, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(kHigh), "r"(kShape),
      "r"(add ? 1 : 0));
}
// True in one thread of a converged warp.
__device__ __forceinline__ bool elected() {
  uint32_t e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e != 0;
}
__device__ __forceinline__ void commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 16 columns of this thread's row; defined after landed()
__device__ __forceinline__ void load16(uint32_t at, float* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
        "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
      : "r"(at));
}
__device__ __forceinline__ void landed() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void defined16(float* r) {
  asm volatile("" : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]), "+f"(r[8]),
               "+f"(r[9]), "+f"(r[10]), "+f"(r[11]), "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15]));
}
__device__ __forceinline__ void store16(uint32_t at, const float* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::
          "r"(at), "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]), "f"(r[8]),
      "f"(r[9]), "f"(r[10]), "f"(r[11]), "f"(r[12]), "f"(r[13]), "f"(r[14]), "f"(r[15])
      : "memory");
}
// 32 columns at once: words of a row
__device__ __forceinline__ void store32(uint32_t at, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(at),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
      "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
      "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// All columns of tensor memory for a CTA (one warp; the address lands at `at` in shared memory), and back.
__device__ __forceinline__ void take_columns(uint32_t at) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(at) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void give_columns(uint32_t tmem) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

__device__ __forceinline__ void fetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}
// Copy of a box of a tensor [tokens, heads, dims] from element (x, head, token), landing on `bar`.
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* map, int x, int head, int token, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(head), "r"(token), "r"(smem_u32(bar))
      : "memory");
}

// Half of a 128-column row in TMEM: columns at .. at + 63.
__device__ __forceinline__ void load64(uint32_t at, float (&x)[64]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) load16(at + 16 * k, x + 16 * k);
}
__device__ __forceinline__ void landed64(float (&x)[64]) {
  landed();
#pragma unroll
  for (int k = 0; k < 4; ++k) defined16(x + 16 * k);
}
// Two halves of a row, 64 values of 16 bits in the first 32 of 64 columns each: where step k (16 values) of a
// product over them finds its own.
__device__ __forceinline__ uint32_t step_of(uint32_t at, int k) { return at + uint32_t((k >> 2) * 64 + (k & 3) * 8); }

// Waits of kernels whose warps have roles: bounded, and over for all once one gave up.
__device__ __forceinline__ bool role_wait(uint64_t* bar, uint32_t parity, uint32_t* abort, uint32_t* status) {
  bool ok = mbar_try_wait(bar, parity);
  if (!ok) {
    const long long t0 = clock64();
    while (!(ok = mbar_try_wait(bar, parity))) {
      if (*static_cast<volatile uint32_t*>(abort)) break;
      if (clock64() - t0 > kWaitLimitCycles) {
        *static_cast<volatile uint32_t*>(abort) = 1u;
        report_status(status, kStatusWaitTimeout);
        break;
      }
    }
  }
  return __all_sync(0xffffffffu, ok);
}
__device__ __forceinline__ void role_arrive(uint64_t* bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

}  // namespace tc
}  // namespace reskv
