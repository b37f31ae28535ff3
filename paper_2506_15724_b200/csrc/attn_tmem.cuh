// What the tensor-core kernels of prompt and tree attention share: waits, tensor memory, row stores.
#pragma once

#include <type_traits>

#include "attn_common.cuh"
#include "tc_common.cuh"

namespace madakv {
namespace {

// What a role waits with: bounded; once a wait has run out, here or in another role, everything that follows returns at once. A
// single thread calls it; warps call all(), which all lanes leave together and with the same answer (instructions that take a whole
// warp follow).
struct Waiter {
  volatile int* abort;
  int32_t* status;
  long long limit;
  bool dead = false;
  __device__ __forceinline__ bool operator()(uint64_t* bar, uint32_t parity, int site) {
    if (dead) return false;
    if (mbar_try(bar, parity)) return true;
    const long long t0 = clock64();
    int spins = 0;
    while (!mbar_try(bar, parity)) {
      if ((++spins & 15) == 0) {
        if (*abort) return dead = true, false;
        if (clock64() - t0 > limit) {
          give_up(abort, status, site);
          return dead = true, false;
        }
      }
    }
    return true;
  }
  __device__ __forceinline__ bool all(uint64_t* bar, uint32_t parity, int site) {
    if (!__all_sync(0xffffffffu, (*this)(bar, parity, site))) dead = true;
    return !dead;
  }
};

__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// A from tensor memory, B from shared memory.
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_desc_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p;\n.reg .b64 db;\nsetp.ne.b32 p, %4, 0;\nmov.b64 db, {%2, %5};\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n}" ::"r"(d_tmem),
      "r"(a_tmem), "r"(b_desc_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi)
      : "memory");
}
#define R8(r, o) "=r"(r[o]), "=r"(r[o + 1]), "=r"(r[o + 2]), "=r"(r[o + 3]), "=r"(r[o + 4]), "=r"(r[o + 5]), "=r"(r[o + 6]), "=r"(r[o + 7])
#define T8(r, o) "+r"(r[o]), "+r"(r[o + 1]), "+r"(r[o + 2]), "+r"(r[o + 3]), "+r"(r[o + 4]), "+r"(r[o + 5]), "+r"(r[o + 6]), "+r"(r[o + 7])
#define I8(r, o) "r"(r[o]), "r"(r[o + 1]), "r"(r[o + 2]), "r"(r[o + 3]), "r"(r[o + 4]), "r"(r[o + 5]), "r"(r[o + 6]), "r"(r[o + 7])
// 32 columns of a warp's lanes; valid behind tmem_wait and tie.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, "
      "%19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : R8(r, 0), R8(r, 8), R8(r, 16), R8(r, 24)
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : R8(r, 0), R8(r, 8)
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::I8(r, 0),
      I8(r, 8), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tie16(uint32_t* r) { asm volatile("" : T8(r, 0), T8(r, 8) : : "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tie32(uint32_t* r) { asm volatile("" : T8(r, 0), T8(r, 8), T8(r, 16), T8(r, 24) : : "memory"); }
#undef R8
#undef T8
#undef I8
// 32 bytes to or from global memory at once, or as two halves. (A thread has a row: what a warp's access takes is its lines, 32 each time,
// so it goes by the number of accesses.)
__device__ __forceinline__ void store32(void* to, const uint32_t* r, bool wide) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]),
                 "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(to)[0] = make_uint4(r[0], r[1], r[2], r[3]);
    reinterpret_cast<uint4*>(to)[1] = make_uint4(r[4], r[5], r[6], r[7]);
  }
}
__device__ __forceinline__ void load32(const void* from, uint32_t* r, bool wide) {
  if (wide) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "l"(from)
                 : "memory");
  } else {
    const uint4 a = reinterpret_cast<const uint4*>(from)[0], b = reinterpret_cast<const uint4*>(from)[1];
    r[0] = a.x, r[1] = a.y, r[2] = a.z, r[3] = a.w, r[4] = b.x, r[5] = b.y, r[6] = b.z, r[7] = b.w;
  }
}
// Weights are 2^(z * scale - round(m * scale)): all of a row's share the factor that the rounding leaves, 2^-24 of the logit in the exponent. True: that
// is so much that weights or their sum leave fp32's range; the row's logits are then taken less m before they are scaled.
__device__ __forceinline__ bool beyond_rounding(float m, float scale2) { return fabsf(fmaf(m, scale2, -__fmul_rn(m, scale2))) > 8.f; }  // (of infinities: false)
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}


// Bounds of the waits. Failure-path test (no GPU fault involved), as in decode attention: the copies are withheld, waits last that many clocks.
inline void attn_waits(AttnParams& p) {
  p.wait_clocks = kWaitCycles;
  if (const char* e = getenv("MADAKV_TEST_HOLD_COPIES")) {
    const long long v = atoll(e);
    if (v >= 100000 && v < kWaitCycles) p.hold_copies = 1, p.wait_clocks = v;
  }
}

}  // namespace
}  // namespace madakv
