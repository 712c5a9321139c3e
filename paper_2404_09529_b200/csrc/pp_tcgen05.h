// What the attention kernels on tcgen05 share: PTX wrappers (barriers with a time limit, TMEM, tcgen05.mma, packed
// fp32 arithmetic), and on the host the tensor map encoder and the limit of the waits.
#ifndef PREPACK_B200_PP_TCGEN05_H_
#define PREPACK_B200_PP_TCGEN05_H_

#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <cstdlib>

#include "pp_internal.h"

namespace pp {
namespace {

// ------------------------------------------------------------------------------------------
// PTX wrappers
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_u32(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
__device__ __forceinline__ unsigned long long global_ns() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes, uint32_t issue) {
  asm volatile("{\n.reg .pred q;\nsetp.ne.b32 q, %2, 0;\n@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n}"
               ::"r"(bar), "r"(bytes), "r"(issue) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// A value that is the same in all lanes, said so to the compiler (all 32 lanes call).
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }

// Every wait in the kernel goes through here or through the two forms for a warp below: it gives up after `limit`, leaving
// why in the CTA-wide abort word, so that all roles leave their loops; the code goes to the device status word at the end
// of the kernel at the latest. A kernel of this file has some forty waits, inlined, and the warps of a scheduler run three
// to five roles: what they execute has to fit its instruction cache (a straight line of code takes 1.0 cycles an
// instruction up to 32 KB, 3.1 to 128 KB, 6 beyond, one scheduler at work). In the independent mode, with a 64-bit clock,
// a global atomic and a poll counter in each wait 1.1 of the 6 warps of a scheduler stood without an instruction at any
// time; in this form, and with each load of the producer loop at one place, 0.18 (64 prompts on a 7B layer: attention
// 194 -> 158 us under ncu with the changes around them, whole steps 285 -> 258). (As calls of one function the waits do not
// fit the softmax threads' registers.)
struct WaitCtx {
  uint32_t abort;               // address in shared memory, 0: go on
  uint32_t limit;               // in units of 1024 ns
  int32_t* status;              // global, may be null
};
// (A poll parks the thread for about 20 us, so the clock, which starts at the first failed one, is read seldom.)
template <int kCode>
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, const WaitCtx& w) {
  uint32_t ok;
  asm volatile(
      "{\n.reg .pred p;\n.reg .b32 t0, t1, x;\n.reg .b64 g;\n"
      "mov.b32 t0, 0;\n"
      "AGAIN_%=:\n"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
      "selp.u32 %0, 1, 0, p;\n"
      "@p bra DONE_%=;\n"
      "ld.volatile.shared.b32 x, [%3];\n"
      "setp.ne.b32 p, x, 0;\n"
      "@p bra DONE_%=;\n"
      "mov.u64 g, %%globaltimer;\n"
      "shr.u64 g, g, 10;\n"
      "cvt.u32.u64 t1, g;\n"
      "or.b32 t1, t1, 1;\n"
      "setp.eq.b32 p, t0, 0;\n"
      "selp.b32 t0, t1, t0, p;\n"
      "sub.u32 t1, t1, t0;\n"
      "setp.le.u32 p, t1, %4;\n"
      "@p bra AGAIN_%=;\n"
      "st.volatile.shared.b32 [%3], %5;\n"
      "DONE_%=:\n}"
      : "=r"(ok) : "r"(bar), "r"(parity), "r"(w.abort), "r"(w.limit), "n"(kCode) : "memory");
  return ok != 0;
}
// The same for a whole warp in uniform control flow: every lane polls, the vote decides.
template <int kCode>
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity, const WaitCtx& w) {
  return __all_sync(0xffffffffu, mbar_wait<kCode>(bar, parity, w));
}

// For the warps of the shared-stream mode that load and issue: one loop of the whole warp, which reads the clock at every
// eighth failed poll and writes the code to the status word itself. There the instruction cache is not the limit, and the
// form above made the issuing warp slower: one prompt of 16 000 tokens on 8 / 4 heads of 64 367 us a step with it, 353 in
// this form; six of 9000 on 32 / 8 heads of 64 2790 -> 2690; 16 prompts of up to 22 861 tokens on 32 heads of 128 12.18 ->
// 12.01 ms. (The softmax threads' waits take the same time in either form.)
template <int kCode>
__device__ __forceinline__ bool mbar_wait_issuer(uint32_t bar, uint32_t parity, const WaitCtx& w) {
  uint32_t t0 = 0, polls = 0;
  while (true) {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    if (__all_sync(0xffffffffu, ok != 0)) return true;
    if ((++polls & 7u) == 0) {
      uint32_t gone;
      asm volatile("ld.volatile.shared.b32 %0, [%1];" : "=r"(gone) : "r"(w.abort) : "memory");
      const uint32_t now = (uint32_t)(global_ns() >> 10) | 1u;
      if (t0 == 0) t0 = now;
      if (gone == 0 && now - t0 > w.limit) {
        asm volatile("st.volatile.shared.b32 [%0], %1;" ::"r"(w.abort), "n"(kCode) : "memory");
        if (w.status) atomicCAS(w.status, 0, kCode);
        gone = 1;
      }
      if (__any_sync(0xffffffffu, gone != 0)) return false;
    }
  }
}

// The warps that issue TMA loads and MMAs run in uniform control flow: all 32 lanes execute the loop, the waits
// and the address arithmetic, and a predicate (`issue`, set on one lane by elect.sync) picks the lane that
// issues. With a branch on the lane index instead, every tcgen05.mma takes ~50 cycles to issue whatever its size
// (a group of 8: 400 cycles against 101-136 in this form, one CTA per SM, with or without 16 busy warps
// beside it), which held the tensor pipe below its rate of one 128 x 128 x 16 product per 64 cycles. A TMA
// load with its expect_tx and the wait for an earlier one takes a warp 307 ns with the branch and 259 ns in this
// form, for any box from 2 to 32 KB, so a tile is one load: whole steps 3.5 % faster for 256 prompts of up to
// 3991 tokens on 32 / 8 heads, 2.7 % for 2048 short ones, 1 to 2 % for the others.
__device__ __forceinline__ uint32_t elect_one() {
  uint32_t r;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(r));
  return r;
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar, uint32_t issue) {
  asm volatile(
      "{\n.reg .pred q;\nsetp.ne.b32 q, %1, 0;\n"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar), "r"(issue) : "memory");
}
__device__ __forceinline__ void tc_wait_ld() { __syncwarp(); asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { __syncwarp(); asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory matrix descriptors (tcgen05), 128-byte swizzle, rows of 128 bytes, 8-row groups
// 1024 bytes apart. Low word: start address >> 4 and (MN-major operands only) the distance between
// 64-element spans of the MN dimension >> 4. High word: constant (8-row group stride, descriptor
// version, swizzle mode). Stepping along a tile only ever adds a small constant to the low word.
__device__ __forceinline__ uint32_t desc_lo(uint32_t saddr, uint32_t lbo_bytes) {
  return ((saddr & 0x3FFFFu) >> 4) | ((lbo_bytes >> 4) << 16);
}
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);

// D[tmem] (+)= A[smem] * B[smem]
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc,
                                       uint32_t accumulate, uint32_t issue) {
  asm volatile(
      "{\n.reg .pred p, q;\n.reg .b64 da, db;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 q, %6, 0;\n"
      "mov.b64 da, {%1, %5};\nmov.b64 db, {%2, %5};\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n}"
      ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi), "r"(issue) : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc,
                                       uint32_t accumulate, uint32_t issue) {
  asm volatile(
      "{\n.reg .pred p, q;\n.reg .b64 db;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 q, %6, 0;\n"
      "mov.b64 db, {%2, %5};\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n}"
      ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi), "r"(issue) : "memory");
}

// 32 consecutive fp32 columns of this thread's TMEM lane.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
  __syncwarp();
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr) : "memory");
}
// tcgen05.wait::ld with the loaded registers passed through it, so that nothing can be moved between
// the load and the wait (used where other work stands between the two).
__device__ __forceinline__ void tc_wait_ld32(uint32_t (&r)[32]) {
  __syncwarp();
  asm volatile("tcgen05.wait::ld.sync.aligned;"
      : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
        "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
        "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
        "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
      :: "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  __syncwarp();
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  __syncwarp();
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(taddr) : "memory");
}

__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float fmax3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// Packed pairs of fp32 (sm_100 f32x2 arithmetic): halves the FMA-pipe instruction count of the
// softmax inner loop.
__device__ __forceinline__ uint64_t pack_f2(uint32_t lo, uint32_t hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(hi));
  return d;
}
__device__ __forceinline__ void unpack_f2(uint64_t x, float& lo, float& hi) {
  uint32_t a, b;
  asm("mov.b64 {%0, %1}, %2;" : "=r"(a), "=r"(b) : "l"(x));
  lo = __uint_as_float(a);
  hi = __uint_as_float(b);
}
__device__ __forceinline__ uint64_t fma_f2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add_f2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t mul_f2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float sum_f2x2(uint64_t a, uint64_t b) {
  float x, y, z, w;
  unpack_f2(a, x, y);
  unpack_f2(b, z, w);
  return (x + z) + (y + w);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);     // .x (low 16 bits) = lo
  return *reinterpret_cast<uint32_t*>(&h);
}

// Probabilities of 32 scores: p = exp2(s * c - m), added up in sum_a / sum_b (two packed accumulators)
// and packed to bf16.
__device__ __forceinline__ void exp_chunk(const uint32_t* v, uint64_t c2, uint64_t negm2, uint64_t& sum_a, uint64_t& sum_b,
                                          uint32_t (&pk)[16]) {
#pragma unroll
  for (int i = 0; i < 32; i += 4) {
    float p0, p1, p2, p3;
    unpack_f2(fma_f2(pack_f2(v[i], v[i + 1]), c2, negm2), p0, p1);
    unpack_f2(fma_f2(pack_f2(v[i + 2], v[i + 3]), c2, negm2), p2, p3);
    p0 = fast_exp2(p0); p1 = fast_exp2(p1); p2 = fast_exp2(p2); p3 = fast_exp2(p3);
    sum_a = add_f2(sum_a, pack_f2(__float_as_uint(p0), __float_as_uint(p1)));
    sum_b = add_f2(sum_b, pack_f2(__float_as_uint(p2), __float_as_uint(p3)));
    pk[i >> 1] = pack_bf16(p0, p1);
    pk[(i >> 1) + 1] = pack_bf16(p2, p3);
  }
}

// Largest of 64 scores.
__device__ __forceinline__ float max64(const uint32_t (&v)[64]) {
  float m0 = fmax3(__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]));
  float m1 = fmax3(__uint_as_float(v[3]), __uint_as_float(v[4]), __uint_as_float(v[5]));
  float m2 = fmax3(__uint_as_float(v[6]), __uint_as_float(v[7]), __uint_as_float(v[8]));
  float m3 = fmax3(__uint_as_float(v[9]), __uint_as_float(v[10]), __uint_as_float(v[11]));
#pragma unroll
  for (int i = 12; i + 7 < 64; i += 8) {
    m0 = fmax3(m0, __uint_as_float(v[i]), __uint_as_float(v[i + 1]));
    m1 = fmax3(m1, __uint_as_float(v[i + 2]), __uint_as_float(v[i + 3]));
    m2 = fmax3(m2, __uint_as_float(v[i + 4]), __uint_as_float(v[i + 5]));
    m3 = fmax3(m3, __uint_as_float(v[i + 6]), __uint_as_float(v[i + 7]));
  }
  m0 = fmax3(m0, __uint_as_float(v[60]), __uint_as_float(v[61]));      // 12 + 8 * 6 = 60
  m1 = fmax3(m1, __uint_as_float(v[62]), __uint_as_float(v[63]));
  return fmaxf(fmax3(m0, m1, m2), m3);
}

// Instruction descriptor: fp32 accumulate, bf16 A and B, A K-major, M = 128.
__host__ __device__ constexpr uint32_t instr_desc(uint32_t n, bool b_mn_major) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn_major ? 1u : 0u) << 16) | ((n >> 3) << 17) |
         ((128u >> 4) << 24);
}

// ------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------
using EncodeFn = PFN_cuTensorMapEncodeTiled_v12000;

inline EncodeFn get_encode_fn() {
  static EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeFn>(p);
  }();
  return fn;
}

inline unsigned long long wait_limit_ns() {
  // Debug overrides of the device-side wait limit, in milliseconds or microseconds.
  if (const char* e = std::getenv("PP_WAIT_LIMIT_MS")) {
    const long ms = std::atol(e);
    if (ms > 0) return (unsigned long long)ms * 1000000ull;
  }
  if (const char* e = std::getenv("PP_WAIT_LIMIT_US")) {
    const long us = std::atol(e);
    if (us > 0) return (unsigned long long)us * 1000ull;
  }
  return 2000000000ull;   // 2 s
}

inline int sm_count() {
  static thread_local int cached_dev = -1, cached = 0;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  if (dev != cached_dev) {
    if (cudaDeviceGetAttribute(&cached, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    cached_dev = dev;
  }
  return cached;
}

}  // namespace
}  // namespace pp

#endif  // PREPACK_B200_PP_TCGEN05_H_
