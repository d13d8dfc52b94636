// bf_blackwell.cuh -- the instructions that the tiled kernels are made of: barriers
// in shared memory, tensor copies (TMA), tensor-core products with accumulators in
// tensor memory.
#pragma once

#include <stdint.h>

namespace bfk {

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// ---- barriers ---------------------------------------------------------------

__device__ __forceinline__ void barrier_init(uint64_t* b, uint32_t arrivals) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(shared_address(b)), "r"(arrivals) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(shared_address(b)) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(shared_address(b)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint64_t* b, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(shared_address(b)), "r"(parity)
      : "memory");
  return done;
}
// A whole warp waits for the phase of that parity; false (and *gave_up set) where it
// does not come within far more time than any of it takes, or another warp gave up.
__device__ __forceinline__ bool barrier_wait(uint64_t* b, uint32_t parity, volatile uint32_t* gave_up) {
  bool done = barrier_try(b, parity);
  for (uint32_t i = 0; !done && i < 1u << 22; ++i) {
    done = barrier_try(b, parity);
    if (i % 256 == 255 && *gave_up) break;
  }
  if (__all_sync(~0u, done)) return true;
  *gave_up = 1;
  return false;
}
__device__ __forceinline__ void fence_barriers() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
// What this thread wrote to shared memory is seen by copies and products behind.
__device__ __forceinline__ void fence_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- tensor copies ----------------------------------------------------------

struct alignas(64) TensorMap {
  uint64_t words[16];
};
__device__ __forceinline__ void copy_box(void* to, const TensorMap* map, int32_t x, int32_t y, int32_t z, int32_t w,
                                         uint64_t* barrier) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
          shared_address(to)),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(shared_address(barrier))
      : "memory");
}
__device__ __forceinline__ void prefetch_map(const TensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// Runs of bytes (multiples of 16, at multiples of 16) to and from shared memory.
__device__ __forceinline__ void copy_run(void* to, const void* from, uint32_t bytes, uint64_t* barrier) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(shared_address(to)),
               "l"(__cvta_generic_to_global(from)), "r"(bytes), "r"(shared_address(barrier))
               : "memory");
}
__device__ __forceinline__ void put_run(void* to, const void* from, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(__cvta_generic_to_global(to)),
               "r"(shared_address(from)), "r"(bytes)
               : "memory");
}
// This thread's runs out of shared memory are on their way: it may be written over, or end.
__device__ __forceinline__ void put_runs_end() {
  asm volatile("cp.async.bulk.commit_group;\n\tcp.async.bulk.wait_group.read 0;" ::: "memory");
}

// ---- tensor memory and products ---------------------------------------------

// Columns of tensor memory, by a whole warp; the address comes in *to (shared memory).
__device__ __forceinline__ void tensor_alloc(uint32_t* to, uint32_t columns) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_address(to)), "r"(columns)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tensor_free(uint32_t at, uint32_t columns) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
__device__ __forceinline__ void tensor_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// What the warp's loads brought may be used: `r` are their registers, which nothing uses before this.
template <int N>
__device__ __forceinline__ void tensor_wait_load(uint32_t (&r)[N]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]));
}
__device__ __forceinline__ void tensor_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Products and their ends are issued by one thread of a whole warp, always the same.
// The warp stays together: where only that thread ran, its operands would have to be
// moved to the uniform registers one by one (an instruction took 125 cycles, twice
// what the product does).
//
// The barrier's phase ends when all products issued so far are done.
__device__ __forceinline__ void tensor_commit(uint64_t* barrier) {
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(shared_address(barrier))
      : "memory");
}
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(~0u, v, 0); }

// A matrix in shared memory in rows of 128 bytes whose 16-byte pieces are at their
// place exclusive-or the row's number modulo 8, 8 rows to a kilobyte; `lead`: bytes
// between columns of 64 elements (of operands whose rows are the summed dimension).
__device__ __forceinline__ uint64_t matrix_at(uint32_t address, uint32_t lead) {
  return (uint64_t)(address >> 4 & 0x3FFF) | (uint64_t)(lead >> 4 & 0x3FFF) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 |
         2ull << 61;
}
// Products of 16-bit types summed in 32 bits: 128 x columns.  `b_rows`: b's rows are the summed dimension.
__device__ __forceinline__ constexpr uint32_t product_of(bool bf16, uint32_t columns, bool b_rows) {
  return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (b_rows ? 1u << 16 : 0u) | columns / 8 << 17 | 128u / 16 << 24;
}
__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\tsetp.ne.u32 p, %4, 0;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(what), "r"((uint32_t)add)
      : "memory");
}
// The same with the first operand in tensor memory.
__device__ __forceinline__ void multiply_held(uint32_t d, uint32_t a, uint64_t b, uint32_t what, bool add) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\tsetp.ne.u32 p, %4, 0;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(what), "r"((uint32_t)add)
      : "memory");
}

// Four products one after the other, `step` apart in both operands (16 bytes each, or columns of the held one):
// together, because each one's choice of a thread and its branch took longer than its product.
__device__ __forceinline__ void multiply4(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add, uint64_t step) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "add.u64 a1, %1, %5;\n\tadd.u64 a2, a1, %5;\n\tadd.u64 a3, a2, %5;\n\t"
      "add.u64 b1, %2, %5;\n\tadd.u64 b2, b1, %5;\n\tadd.u64 b3, b2, %5;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a1, b1, %3, 1;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a2, b2, %3, 1;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a3, b3, %3, 1;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(what), "r"((uint32_t)add), "l"(step)
      : "memory");
}
__device__ __forceinline__ void multiply4_held(uint32_t d, uint32_t a, uint64_t b, uint32_t what, bool add, uint32_t a_step,
                                               uint64_t b_step) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t.reg .b32 a1, a2, a3;\n\t.reg .b64 b1, b2, b3;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "add.u32 a1, %1, %5;\n\tadd.u32 a2, a1, %5;\n\tadd.u32 a3, a2, %5;\n\t"
      "add.u64 b1, %2, %6;\n\tadd.u64 b2, b1, %6;\n\tadd.u64 b3, b2, %6;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a1], b1, %3, 1;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a2], b2, %3, 1;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a3], b3, %3, 1;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(what), "r"((uint32_t)add), "r"(a_step), "l"(b_step)
      : "memory");
}

#define BF_R4(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3])
#define BF_I4(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3])
// 32 columns of the warp's 32 lanes, a lane to a thread.
__device__ __forceinline__ void tensor_load32(uint32_t at, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
      "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : BF_R4(r, 0), BF_R4(r, 4), BF_R4(r, 8), BF_R4(r, 12), BF_R4(r, 16), BF_R4(r, 20), BF_R4(r, 24), BF_R4(r, 28)
      : "r"(at));
}
__device__ __forceinline__ void tensor_load8(uint32_t at, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : BF_R4(r, 0), BF_R4(r, 4)
               : "r"(at));
}
__device__ __forceinline__ void tensor_store32(uint32_t at, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
      "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(at),
      BF_I4(r, 0), BF_I4(r, 4), BF_I4(r, 8), BF_I4(r, 12), BF_I4(r, 16), BF_I4(r, 20), BF_I4(r, 24), BF_I4(r, 28)
      : "memory");
}
__device__ __forceinline__ void tensor_store8(uint32_t at, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(at), BF_I4(r, 0), BF_I4(r, 4)
               : "memory");
}
#undef BF_R4
#undef BF_I4


// 16 bytes to shared memory, zeros where they are not there.
__device__ __forceinline__ void copy_piece(uint32_t to, const void* from, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(__cvta_generic_to_global(from)), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {  // all but the last N groups have arrived
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void copies_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// Four values added to what is in global memory.
__device__ __forceinline__ void add4(float* to, const float4& x) {
  asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(__cvta_generic_to_global(to)), "f"(x.x), "f"(x.y), "f"(x.z), "f"(x.w) : "memory");
}

}  // namespace bfk
