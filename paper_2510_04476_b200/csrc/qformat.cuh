// The 4-bit format shared by the quantised cache and the quantised weights, and the warp-level tensor-core helpers that read it.
//
// Groups of 32 channels share a bf16 scale s; a channel is c * s with a whole number c in -7 .. 7.  Two codes lie in a byte in
// sign and magnitude: e0 = sign in bit 7, magnitude in bits 0-2; e1 = sign in bit 6, magnitude in bits 3-5.  With the byte
// copied into both bytes of a 16-bit lane, (lane & 0x8007) IS the bf16 number e0 * 2^-133 and ((lane << 1) & 0x8070) IS
// e1 * 2^-129: bf16 subnormals, which mma.sync multiplies exactly.  So a code needs no conversion and leaves no offset to take
// off; the other operand carries 2^64 (for e0) and 2^60 (for e1), and sums come out times 2^-69.
//
// A row is cut into blocks of min(d, 128) channels with NG = block / 32 groups; in a block, byte g * 2 NG + grp * 2 + j
// (g = 0..7, j = 0, 1) holds channels grp * 32 + 4 g + j (e0) and grp * 32 + 4 g + 2 + j (e1).  That order serves both ways a
// contraction reads the row with one contiguous load per lane: over the channels (lane t of a quad takes the bytes of g = 2t,
// 2t + 1, whichever group each pair is in) and over the rows (lane group g takes its own 2 NG bytes, byte i being one 16-channel
// output tile).
#pragma once
#include "common.cuh"

namespace q4 {

constexpr int GROUP = 32;
constexpr uint32_t MUL_E0 = 0x5f805f80u;   // bf16x2 {2^64, 2^64}
constexpr uint32_t MUL_E1 = 0x5d805d80u;   // bf16x2 {2^60, 2^60}
constexpr float TWO_69 = 590295810358705651712.f;
constexpr float TWO_65 = 36893488147419103232.f;
constexpr float TWO_64 = 18446744073709551616.f;
constexpr float TWO_M64 = 5.42101086242752217e-20f;

CCA_DEVINL void mma_16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
CCA_DEVINL void mma_16816_zero(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {   // d = a b
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
// The 8 x 8 tile of 16-bit elements held as {row lane / 4, columns 2 (lane % 4), + 1}, transposed.
CCA_DEVINL uint32_t transpose_8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
CCA_DEVINL uint32_t pack_bf16x2(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
CCA_DEVINL uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
CCA_DEVINL float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
CCA_DEVINL float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Lanes of e0 and e1 from a register whose two 16-bit halves each hold one code byte twice.
CCA_DEVINL uint32_t code_e0(uint32_t p) { return p & 0x80078007u; }
CCA_DEVINL uint32_t code_e1(uint32_t p) { return (p << 1) & 0x80708070u; }

// Two 32-bit values of a scale row as floats: scale `i` of a packed array of bf16.
template <int NW>
CCA_DEVINL float scale_at(const uint32_t (&w)[NW], int i) {
  return (i & 1) ? bf_hi(w[i >> 1]) : bf_lo(w[i >> 1]);
}

// NW consecutive 32-bit words (NW = 1, 2, 4, 8; the address is a multiple of min(16, 4 NW) bytes), read once: streamed.
template <int NW>
CCA_DEVINL void load_words(uint32_t (&w)[NW], const void* p) {
  if constexpr (NW == 1) {
    w[0] = __ldcs(reinterpret_cast<const uint32_t*>(p));
  } else if constexpr (NW == 2) {
    const uint2 u = __ldcs(reinterpret_cast<const uint2*>(p));
    w[0] = u.x; w[1] = u.y;
  } else {
#pragma unroll
    for (int i = 0; i < NW / 4; ++i) {
      const uint4 u = __ldcs(reinterpret_cast<const uint4*>(p) + i);
      w[4 * i] = u.x; w[4 * i + 1] = u.y; w[4 * i + 2] = u.z; w[4 * i + 3] = u.w;
    }
  }
}
template <int NW>
CCA_DEVINL void zero_words(uint32_t (&w)[NW]) {
#pragma unroll
  for (int i = 0; i < NW; ++i) w[i] = 0u;
}

// The scale of a group from the largest magnitude in it, and a channel's code.  IEEE division, so that the result does not
// depend on the build's fast-math setting; an infinity or NaN in the group makes the scale NaN (and every code 0), a scale
// below the smallest normal number counts as zero.
CCA_DEVINL bf16 group_scale(float amax) {
  if (!(amax <= 3.3895313892515355e38f)) return __ushort_as_bfloat16((unsigned short)0x7fc0);
  const bf16 s = __float2bfloat16_rn(__fdiv_rn(amax, 7.f));
  return __bfloat162float(s) < 1.17549435e-38f ? __ushort_as_bfloat16((unsigned short)0) : s;
}
// x / s correctly rounded from r = 1 / s (correctly rounded): one Newton step on the quotient.  It holds while nothing over- or
// underflows on the way; a scale below 2^-96 takes the division itself.
CCA_DEVINL int code_of(float x, float s, float r) {
  if (!(s > 0.f)) return 0;
  float q = x * r;
  q = s < 1.2621774e-29f ? __fdiv_rn(x, s) : fmaf(fmaf(-s, q, x), r, q);
  return (int)fminf(fmaxf(rintf(q), -7.f), 7.f);
}
CCA_DEVINL uint32_t code_byte(int c0, int c1) {
  return (c0 < 0 ? 0x80u : 0u) | (uint32_t)(c0 < 0 ? -c0 : c0) | (c1 < 0 ? 0x40u : 0u) | ((uint32_t)(c1 < 0 ? -c1 : c1) << 3);
}
CCA_DEVINL int value_e0(uint32_t byte) { const int m = (int)(byte & 7u); return (byte & 0x80u) ? -m : m; }
CCA_DEVINL int value_e1(uint32_t byte) { const int m = (int)((byte >> 3) & 7u); return (byte & 0x40u) ? -m : m; }

// One thread's share of quantising a block: 4 channels 4 g .. 4 g + 3 of each of its NG groups, the eight threads g of a block
// being eight neighbouring lanes.  `x(grp)` returns the 4 channels as bf16x2 pairs; out: 2 NG code bytes and the NG scales
// (the same in all eight lanes).  All 32 lanes call it.
template <int NG, typename F>
CCA_DEVINL void quantise_block(F x, uint8_t (&code)[2 * NG], bf16 (&scale)[NG]) {
#pragma unroll
  for (int grp = 0; grp < NG; ++grp) {
    const uint2 u = x(grp);
    const float v[4] = {bf_lo(u.x), bf_hi(u.x), bf_lo(u.y), bf_hi(u.y)};
    // a NaN must win the maximum: compare the magnitudes' bit patterns
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
#pragma unroll
    for (int s = 1; s < 8; s <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, s));
    scale[grp] = group_scale(__uint_as_float(m));
    const float sf = __bfloat162float(scale[grp]), r = __frcp_rn(sf);
    code[2 * grp] = (uint8_t)code_byte(code_of(v[0], sf, r), code_of(v[2], sf, r));
    code[2 * grp + 1] = (uint8_t)code_byte(code_of(v[1], sf, r), code_of(v[3], sf, r));
  }
}

}  // namespace q4
