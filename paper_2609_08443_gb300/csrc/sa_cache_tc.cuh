// Pieces of the cache's tcgen05 kernels: bounded waits, copies and products issued from
// uniform control flow.
#pragma once
#include "sa_cache.cuh"
#include "sa_cache_walk.cuh"
#include "sa_tc_common.cuh"

namespace sa {
namespace cache {

// Instruction descriptor of kind::f16 with float16 A and B, fp32 D.
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, int a_mn, int b_mn) {
  return (1u << 4) | (uint32_t(a_mn) << 15) | (uint32_t(b_mn) << 16) | (uint32_t(N >> 3) << 17) | (uint32_t(M >> 4) << 24);
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool valid) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

__device__ __forceinline__ void l2_prefetch(const void* src, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(bytes) : "memory");
}

// One lane's bulk operations, in uniform control flow (issued by several lanes at once
// they take turns, at about a hundred cycles each).
__device__ __forceinline__ void bulk_copy_if(uint32_t e, uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %4, 0;\n\t"
      "@q cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n\t}" ::"r"(dst),
      "l"(src), "r"(bytes), "r"(bar), "r"(e)
      : "memory");
}

__device__ __forceinline__ void l2_prefetch_if(uint32_t e, const void* src, uint32_t bytes) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t"
      "@q cp.async.bulk.prefetch.L2.global [%0], %1;\n\t}" ::"l"(src), "r"(bytes), "r"(e)
      : "memory");
}

// The roles share one instruction cache, whose first level is small; a role that runs
// straight through cold code takes about ten cycles an instruction, and with the waits'
// slow paths inlined the issuing warp alone was slower than its products.  So the loops
// below are kept short and not unrolled.

// Control words of a CTA in shared memory.
struct Ctl {
  uint32_t abort;  // somebody gave up: everybody leaves
  uint32_t site;   // where
};

// Limit of a wait in ns: never below two seconds, whatever sa_set_wait_limit_ns asks for its
// tests of the sketch's kernels.  A correct pipeline waits microseconds.
__device__ __forceinline__ uint32_t wait_limit(const AttnArgs& a) {
  const uint64_t ns = a.wait_limit_ns < 2000000000ull ? 2000000000ull : a.wait_limit_ns;
  return ns > 0xFFFFFFFFull ? 0xFFFFFFFFu : uint32_t(ns);
}

// Polls until the phase is complete, the limit (ns) is over or the CTA aborts.  (A try-wait may
// sleep until its phase completes: it is no way to ask whether one has.)  A few
// instructions and no call: a dozen of these sit in the roles' loops.
__device__ __forceinline__ bool poll(uint32_t bar, uint32_t parity, uint32_t abort_addr, uint32_t limit_ns) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .u32 t0, t1, f;\n\t"
      "mov.u32 %0, 1;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "@p bra DONE;\n\t"
      "mov.u32 t0, %%globaltimer_lo;\n"
      "MORE:\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "@p bra DONE;\n\t"
      "ld.volatile.shared::cta.u32 f, [%3];\n\t"
      "mov.u32 t1, %%globaltimer_lo;\n\t"
      "sub.u32 t1, t1, t0;\n\t"
      "setp.gt.u32 q, t1, %4;\n\t"
      "setp.ne.or.u32 q, f, 0, q;\n\t"
      "@!q bra MORE;\n\t"
      "mov.u32 %0, 0;\n"
      "DONE:\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity), "r"(abort_addr), "r"(limit_ns)
      : "memory");
  return ok != 0;
}

__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, Ctl* ctl, uint32_t limit_ns, uint32_t site) {
  if (__all_sync(0xffffffffu, poll(bar, parity & 1u, smem_u32(&ctl->abort), limit_ns))) return true;
  ctl->site = site;
  *static_cast<volatile uint32_t*>(&ctl->abort) = 1u;
  return false;
}

// The forms below run on a whole warp in uniform control flow, with `e` true in one
// lane: operands then stay in uniform registers and a product costs a few instructions
// to issue instead of twenty, which the issuing warp cannot hide.
__device__ __forceinline__ uint32_t elect_one() {
  uint32_t e;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(e));
  return e;
}
// Low word of sdesc(); the high words are constants of the operand's layout.
__device__ __forceinline__ uint32_t desc_lo(uint32_t saddr, uint32_t lbo_bytes) {
  return ((saddr & 0x3FFFFu) >> 4) | ((lbo_bytes >> 4) << 16);
}
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);  // 1024 bytes between 8-row groups
__device__ __forceinline__ void mma_ss(uint32_t e, uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "mov.b64 da, {%1, %6};\n\tmov.b64 db, {%2, %6};\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}" ::"r"(d),
      "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(e), "r"(kDescHi));
}
__device__ __forceinline__ void mma_ts(uint32_t e, uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 db;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "mov.b64 db, {%2, %6};\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(e), "r"(kDescHi));
}
__device__ __forceinline__ void commit_if(uint32_t e, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
      "r"(e)
      : "memory");
}
// 128 rows of D bf16 values into the swizzled layout [D / 64][128][128 bytes], by one
// warp: each lane works out four rows' places (offset(row), in elements; negative: zeros),
// and the copies take them from it.
template <int D, class F>
__device__ __forceinline__ void load_rows(const void* src, uint32_t dst, int lane, F&& offset) {
  constexpr int CH = D / 8;  // 16-byte pieces of a row
  const int c = lane % CH, sub = lane / CH;
  const char* base = static_cast<const char*>(src) + 16 * c;
  const uint32_t to = dst + (c >> 3) * 16384;
#pragma unroll 1
  for (int j = 0; j < 4; ++j) {
    const int64_t mine = offset(32 * j + lane);
#pragma unroll 4
    for (int r = sub; r < 32; r += 32 / CH) {
      const int64_t o = __shfl_sync(0xffffffffu, mine, r);
      const int row = 32 * j + r;
      cp_async16(to + row * 128 + (((c & 7) ^ (row & 7)) << 4), base + 2 * (o < 0 ? 0 : o), o >= 0);
    }
  }
  cp_async_wait_all();
  fence_proxy_async_smem();
  __syncwarp();
}

}  // namespace cache
}  // namespace sa
