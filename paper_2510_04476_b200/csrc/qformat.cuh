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
constexpr uint32_t MUL_69 = 0x62006200u;   // bf16x2 {2^69, 2^69}
constexpr float TWO_69 = 590295810358705651712.f;

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
// Two numbers as two bf16 pairs that add up to them: the first 8 significant bits, cut off (returned), and the rest, rounded.
CCA_DEVINL uint32_t split_bf16x2(float lo, float hi, uint32_t& rest) {
  const uint32_t l = __float_as_uint(lo), h = __float_as_uint(hi);
  rest = pack_bf16x2(lo - __uint_as_float(l & 0xffff0000u), hi - __uint_as_float(h & 0xffff0000u));
  return __byte_perm(l, h, 0x7632);
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

// NW = 2 or 4 consecutive 32-bit words (the address is a multiple of their size), read once: streamed.
template <int NW>
CCA_DEVINL void load_words(uint32_t (&w)[NW], const void* p) {
  if constexpr (NW == 2) {
    const uint2 u = __ldcs(reinterpret_cast<const uint2*>(p));
    w[0] = u.x; w[1] = u.y;
  } else {
    const uint4 u = __ldcs(reinterpret_cast<const uint4*>(p));
    w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
  }
}

CCA_DEVINL float divide(float a, float b) {                // to nearest, subnormal numbers as they are whatever the build's setting
  float r;
  asm("div.rn.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// The whole number nearest to q (ties to even), |q| < 2^21: what adding 1.5 * 2^23 leaves in the low bits.  No clamp to -7 .. 7 is
// needed: a scale rounded down by its 2^-9 still leaves the largest quotient below 7.02.
CCA_DEVINL int nearest(float q) { return __float_as_int(__fadd_rn(q, 12582912.f)) - 0x4b400000; }
// Codes as a byte, in sign and magnitude; no negative zero.
CCA_DEVINL uint32_t code_byte(int c0, int c1) {
  return (uint32_t)abs(c0) | ((uint32_t)abs(c1) << 3) | (((uint32_t)c0 >> 24) & 0x80u) | (((uint32_t)c1 >> 25) & 0x40u);
}

// One thread's share of quantising a block: 4 channels 4 g .. 4 g + 3 of each of its NG groups, the eight threads g of a block
// being eight neighbouring lanes.  `x(grp)` returns the 4 channels as bf16x2 pairs; out, two groups to a word: the code bytes in
// order and the scales (the same in all eight lanes).  All 32 lanes call it.  What bounds it is instructions: two groups go
// through the maximum and the scale as halves of one register, the eight lanes share the groups out while they find their maxima,
// and magnitude and sign of a code are put in place for four bytes at a time.
template <int NG, typename F>
CCA_DEVINL void quantise_block(F x, uint32_t (&code)[(NG + 1) / 2], uint32_t (&scale)[(NG + 1) / 2]) {
  constexpr int NP = (NG + 1) / 2;                         // pairs of groups
  const bool odd = threadIdx.x & 1;
  uint2 u[2 * NP];
#pragma unroll
  for (int grp = 0; grp < 2 * NP; ++grp) u[grp] = grp < NG ? x(grp) : make_uint2(0, 0);
  // magnitudes compared as 16-bit patterns: their order is the numbers', and a NaN wins
  uint32_t m[NP];
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const uint32_t a = __vmaxu2(u[2 * p].x & 0x7fff7fffu, u[2 * p].y & 0x7fff7fffu);
    const uint32_t b = __vmaxu2(u[2 * p + 1].x & 0x7fff7fffu, u[2 * p + 1].y & 0x7fff7fffu);
    m[p] = __vmaxu2(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));
  }
  // even lanes go on with the first pair, odd ones with the second (of one pair: all with it)
  uint32_t top = __vmaxu2(NP == 2 && odd ? m[NP - 1] : m[0], __shfl_xor_sync(0xffffffffu, NP == 2 && !odd ? m[NP - 1] : m[0], 1));
  top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 2));
  top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 4));
  auto both = [&](uint32_t mine, uint32_t (&w)[NP]) {      // this lane's pair and its neighbour's
    if constexpr (NP == 2) {
      const uint32_t other = __shfl_xor_sync(0xffffffffu, mine, 1);
      w[0] = odd ? other : mine; w[1] = odd ? mine : other;
    } else {
      w[0] = mine;
    }
  };
  auto plain = [](uint32_t t) { return t == 0u || t - 0x1100u <= 0x7f7fu - 0x1100u; };      // zero, or 2^-93 and more, and finite
  if (__any_sync(0xffffffffu, !plain(top & 0xffffu) || !plain(top >> 16))) {
    // Below 2^-93 (in any of the warp's groups) the steps of the other branch would underflow.  A scale below the smallest
    // normal number counts as zero; an infinity or a NaN makes the scale a NaN.
    uint32_t all[NP];
    both(top, all);
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      code[p] = scale[p] = 0u;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint2 w = u[2 * p + h];
        const uint32_t t = h ? all[p] >> 16 : all[p] & 0xffffu;
        float sf = __bfloat162float(__float2bfloat16_rn(divide(__uint_as_float(t << 16), 7.f)));
        if (sf < 1.17549435e-38f) sf = 0.f;
        if (t > 0x7f7fu) sf = __uint_as_float(0x7fc00000u);
        const float v[4] = {bf_lo(w.x), bf_hi(w.x), bf_lo(w.y), bf_hi(w.y)};
        int c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = nearest(divide(v[i], sf));
        const uint32_t two = sf > 0.f ? code_byte(c[0], c[2]) | (code_byte(c[1], c[3]) << 8) : 0u;
        code[p] |= two << (16 * h);
        scale[p] |= (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(sf)) << (16 * h);
      }
    }
    return;
  }
  // Quotients by one Newton step, so that nothing depends on the build's fast-math setting.  A maximum / 7 comes out correctly
  // rounded (the reciprocal of 7 is).  |x| / s comes out exact where it is half way between two whole numbers: then the
  // residual is exact and the correction off by less than a last place; elsewhere it is at least 2^-12 of itself away from
  // half way (x and s have 8 significant bits each), a thousand times what is left of the error.
  constexpr float R7 = 1.f / 7.f;
  auto seventh = [&](uint32_t t) {
    const float a = __uint_as_float(t), q = a * R7;
    return fmaf(fmaf(-7.f, q, a), R7, q);
  };
  both(pack_bf16x2(seventh(top << 16), seventh(top & 0xffff0000u)), scale);
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    uint32_t c[2][4];                                      // |code| in the low bits of each
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint2 w = u[2 * p + h];
      const float v[4] = {bf_lo(w.x), bf_hi(w.x), bf_lo(w.y), bf_hi(w.y)};
      const float s = h ? bf_hi(scale[p]) : bf_lo(scale[p]);
      float r;
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
      r = fminf(r, 3.402823466e38f);                       // a group of zeros: 0 r must be 0
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = fabsf(v[i]), q = a * r;
        c[h][i] = __float_as_uint(__fadd_rn(fmaf(fmaf(-s, q, a), r, q), 12582912.f));
      }
    }
    // four bytes at a time; a sign counts where the magnitude is not 0, that is where adding 127 carries into bit 7
    const uint32_t e0 = __byte_perm(__byte_perm(c[0][0], c[0][1], 0x0040), __byte_perm(c[1][0], c[1][1], 0x0040), 0x5410);
    const uint32_t e1 = __byte_perm(__byte_perm(c[0][2], c[0][3], 0x0040), __byte_perm(c[1][2], c[1][3], 0x0040), 0x5410);
    const uint32_t s0 = __byte_perm(u[2 * p].x, u[2 * p + 1].x, 0x7531) & (e0 + 0x7f7f7f7fu) & 0x80808080u;
    const uint32_t s1 = __byte_perm(u[2 * p].y, u[2 * p + 1].y, 0x7531) & (e1 + 0x7f7f7f7fu) & 0x80808080u;
    code[p] = e0 | s0 | (e1 << 3) | (s1 >> 1);
  }
}

}  // namespace q4
