// What the tensor-core kernels of caller-held caches share: tcgen05 operands in TMEM and with the outer dimension contiguous, and
// exponentials that do not wait for the special-function unit.
#pragma once

#include "attn_rows.cuh"
#include "tcgen05.cuh"
#include "tma_mma.cuh"

namespace bkv {
namespace tc {

constexpr int kTcRows = 128, kTcKeys = 128;      // a tile of logits

// A product's second operand B[k][n] with n contiguous: 64 columns x 8 rows of k are an atom of 1024 bytes (128-byte swizzle), the next
// 8 rows 1024 bytes on (the stride byte offset, as in kDescHi), the next 64 columns kLead bytes (the leading byte offset).
__device__ inline uint32_t umma_desc_lo_outer(uint32_t smem_addr, uint32_t lead) { return ((smem_addr & 0x3FFFFu) >> 4) | ((lead >> 4) << 16); }
constexpr uint32_t kOuterB = 1u << 16;           // instruction descriptor: B is laid out so

// D[128][N] (+)= A[128][16] B[N][16], both from shared memory, N by the instruction descriptor.
__device__ inline void umma_n(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t instr, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "mov.b64 da, {%1, %3};\n\t"
      "mov.b64 db, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p;\n\t}"
      ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(kDescHi), "r"((uint32_t)accumulate), "r"(instr) : "memory");
}
// D[128][N] (+)= A[128][16] B[16][N] with A in TMEM, two bf16 to a column.
template <uint32_t kInstr>
__device__ inline void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "mov.b64 db, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %5, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(kDescHi), "r"((uint32_t)accumulate), "r"(kInstr) : "memory");
}

// 16 columns of this warp's 32 TMEM lanes.
__device__ inline void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// 8 fp32 columns of this warp's 32 TMEM lanes.
__device__ inline void tmem_ld8(uint32_t taddr, float (&v)[8]) {
  uint32_t r[8];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ inline void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ inline float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
template <int N>
__device__ inline float max_of(const float (&x)[N]) {
  float a = x[0], b = x[1];
#pragma unroll
  for (int i = 2; i < N; i += 4) {
    a = max3(a, x[i], x[i + 1]);
    if (i + 3 < N) b = max3(b, x[i + 2], x[i + 3]);
  }
  return fmaxf(a, b);
}
__device__ inline float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 2^x on the FMA pipe for x <= 126: x = n + f with n the nearest integer (it falls out of the low bits of x + 1.5 2^23), 2^f by the polynomial
// of degree 5 of least relative error on [-1/2, 1/2] (Remez exchange: 7.5e-8; 2.1e-7 with its evaluation in fp32), n added to the
// exponent.  Below -126 (and for -inf) 2^-126.
__device__ inline float2 exp2_fma(float2 x) {
  constexpr float kMagic = 12582912.f;
  x = make_float2(fmaxf(x.x, -126.f), fmaxf(x.y, -126.f));
  const float2 t = __fadd2_rn(x, make_float2(kMagic, kMagic));
  const float2 n = __fadd2_rn(t, make_float2(-kMagic, -kMagic));
  const float2 f = __ffma2_rn(n, make_float2(-1.f, -1.f), x);
  auto both = [](float c) { return make_float2(c, c); };
  float2 p = __ffma2_rn(both(0.0013276471979050046f), f, both(0.00967554133420403f));
  p = __ffma2_rn(p, f, both(0.055507132735436365f));
  p = __ffma2_rn(p, f, both(0.24022119723848773f));
  p = __ffma2_rn(p, f, both(0.693146967064733f));
  p = __ffma2_rn(p, f, both(1.0000000716546822f));
  return make_float2(__uint_as_float(__float_as_uint(p.x) + (__float_as_uint(t.x) << 23)), __uint_as_float(__float_as_uint(p.y) + (__float_as_uint(t.y) << 23)));
}

// What a warp asked for or issued is over before its CTA uses the memory for something else or ends, whichever warp gave up and when: the last warp
// to leave waits for it, within limits.  (Without a wait that gave up, another warp has seen the same phases before.)  The copies of a ring, of which
// `asked` entries have been asked for:
template <int kRing>
__device__ inline void copies_landed(uint64_t (&full)[kRing], int asked) {
  const long long t0 = clock64();
  for (int i = max(0, asked - kRing); i < asked; ++i)
    while (!mbar_try_wait(full + i % kRing, (uint32_t)(i / kRing) & 1u) && clock64() - t0 < kWaitCycles) {}
}
// a copy by itself:
__device__ inline void copy_landed(uint64_t* full) {
  const long long t0 = clock64();
  while (!mbar_try_wait(full, 0) && clock64() - t0 < kWaitCycles) {}
}
// and the products that this warp issued:
__device__ inline void products_done(uint64_t* drained) {
  if (elect_one()) umma_commit(drained);
  __syncwarp();
  copy_landed(drained);
}

template <int kRegs>
__device__ inline void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs)); }
template <int kRegs>
__device__ inline void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs)); }

}  // namespace tc
}  // namespace bkv
