// The latent cache in 4 bits: rows put in (quantised), read back, attended to by one new token per sequence, and evicted by the
// attention weight that they have gathered.  The format is that of qformat.cuh.
//
// All of it is bound by memory traffic.  Per (sequence, kv head) the cache is one contiguous run of rows, so that a head's rows
// stream as whole lines and a row moves without touching its neighbours' heads.
#include <cstring>

#include "cluster.cuh"
#include "pdl.cuh"
#include "qrow.cuh"

namespace {

using namespace q4;
constexpr float LOG2E = 1.4426950408889634f;

// ------------------------------------------------------------------------------------------------ rows in and out
struct IoArgs {
  const bf16 *k, *v;             // [B, n, hk, dh]
  float *k_out, *v_out;          // the same, fp32
  const int *position, *count, *first;
  QCache c;
  long long n, limit;            // n * hk * blocks * 2 <= 2^31; limit: rows a sequence may hold
  int hk;
  uint32_t hk_inv;               // 2^32 / hk rounded down, 2^32 - 1 for one head
  int* status;
};

// Eight neighbouring lanes take one block of one row (quantise_block); units run over (sequence, new row, head, block, key | value)
// with the last fastest, so that a warp reads whole token rows.  1 x 16384 rows of 2 heads x 128 and their reading back take 13.9 us
// (8.6 us of traffic, the rest two launches; 16.9 with the groups quantised one by one: 503 instructions a warp instead of 362), one row
// of each of 32 sequences and its reading back 3.0.
struct IoUnit { int kv, blk, i, h; };
template <int DH>
CCA_DEVINL IoUnit io_unit(const IoArgs& a, uint32_t u) {
  constexpr int NB = Row<DH>::NB;
  IoUnit w;
  w.kv = (int)(u & 1); w.blk = (int)((u >> 1) % NB);
  const uint32_t ih = (u >> 1) / NB;                       // (new row, head)
  w.i = (int)__umulhi(ih, a.hk_inv); w.h = (int)ih - w.i * a.hk;       // the quotient, or one less
  if (w.h >= a.hk) { w.h -= a.hk; ++w.i; }
  return w;
}

template <int DH>
__global__ void __launch_bounds__(256) qcache_append_kernel(IoArgs a) {
  pdl_enter();
  using R = Row<DH>;
  constexpr int NG = R::NG;
  const int lane8 = threadIdx.x & 7, b = blockIdx.y;
  const uint32_t units = (uint32_t)a.n * a.hk * R::NB * 2;
  uint2 x[NG];
  IoUnit w;
  auto fetch = [&](uint32_t u) {
    w = io_unit<DH>(a, u);
    const bf16* src = (w.kv ? a.v : a.k) + (((size_t)b * a.n + w.i) * a.hk + w.h) * DH + w.blk * R::BLK + lane8 * 4;
#pragma unroll
    for (int grp = 0; grp < NG; ++grp) x[grp] = u < units ? __ldcs(reinterpret_cast<const uint2*>(src + grp * GROUP)) : make_uint2(0, 0);
  };
  uint32_t u0 = blockIdx.x * 32 + (threadIdx.x >> 5) * 4;
  const uint32_t mine = (threadIdx.x & 31) >> 3;
  fetch(u0 + mine);                                        // on its way while the length is asked for
  const int len = a.c.len[b], first_pos = a.position ? a.position[b] : 0;
  const int cnt = a.count ? max(0, min(a.count[b], (int)a.n)) : (int)a.n;
  if (len < 0 || (long long)len + cnt > a.limit || first_pos < 0 || (long long)first_pos + cnt > 0x80000000ll) {
    // a sequence whose rows do not fit, or whose positions are none: nothing of it is written
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicCAS(a.status, 0, ST_QCACHE_BAD_LEN);
    return;
  }
  // whole warps stay in the loop: the shuffles need every lane
  while (u0 < units) {
    const IoUnit o = w;
    const bool ok = u0 + mine < units && o.i < cnt;
    uint32_t code[(NG + 1) / 2], scale[(NG + 1) / 2];
    // rows behind `count` may hold anything: as zeros they leave their neighbours in the warp on the short way
    quantise_block<NG>([&](int grp) { return ok ? x[grp] : make_uint2(0, 0); }, code, scale);
    u0 += gridDim.x * 32;
    if (u0 < units) fetch(u0 + mine);
    if (!ok) continue;
    const size_t row = ((size_t)b * a.hk + o.h) * a.c.S_max + len + o.i;
    store_block<DH>(a.c, row, o.kv, o.blk, lane8, (a.position ? first_pos : len) + o.i, code, scale);
  }
}

// The same units.  A code becomes a number exactly: the bf16 subnormal that its bits are, times powers of two.
template <int DH>
__global__ void __launch_bounds__(256) qcache_read_kernel(IoArgs a) {
  pdl_enter();
  using R = Row<DH>;
  constexpr int NG = R::NG, NP = (NG + 1) / 2;
  constexpr uint32_t UP_E0 = 0x7b807b80u, UP_E1 = 0x79807980u, UP = 0x46004600u;      // bf16x2 2^120, 2^116, 2^13
  const int lane8 = threadIdx.x & 7, b = blockIdx.y;
  const uint32_t units = (uint32_t)a.n * a.hk * R::NB * 2;
  const long long first = a.first ? a.first[b] : a.c.len[b];
  for (uint32_t u = blockIdx.x * 32 + (threadIdx.x >> 3); u < units; u += gridDim.x * 32) {
    const IoUnit o = io_unit<DH>(a, u);
    const long long r = first + o.i;
    const bool there = r >= 0 && r < a.c.S_max;
    const size_t row = ((size_t)b * a.hk + o.h) * a.c.S_max + (there ? r : 0);
    const uint8_t* src = (o.kv ? a.c.v_codes : a.c.k_codes) + row * R::CODES + o.blk * (R::BLK / 2) + lane8 * 2 * NG;
    const bf16* sc = (o.kv ? a.c.v_scales : a.c.k_scales) + row * R::SCALES + o.blk * NG;
    float* dst = (o.kv ? a.v_out : a.k_out) + (((size_t)b * a.n + o.i) * a.hk + o.h) * DH + o.blk * R::BLK + lane8 * 4;
    uint32_t code[NP], scale[NP];
    if constexpr (NG == 1) {
      code[0] = *reinterpret_cast<const uint16_t*>(src);
      scale[0] = *reinterpret_cast<const uint16_t*>(sc);
    } else {
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        code[p] = reinterpret_cast<const uint32_t*>(src)[p];
        scale[p] = reinterpret_cast<const uint32_t*>(sc)[p];
      }
    }
#pragma unroll
    for (int grp = 0; grp < NG; ++grp) {
      const uint32_t pr = __byte_perm(code[grp / 2], 0, (grp & 1) ? 0x3322u : 0x1100u);
      const uint32_t lo = mul_bf16x2(mul_bf16x2(code_e0(pr), UP_E0), UP), hi = mul_bf16x2(mul_bf16x2(code_e1(pr), UP_E1), UP);
      const float s = scale_at(scale, grp);
      const float4 v = make_float4(s * bf_lo(lo), s * bf_hi(lo), s * bf_lo(hi), s * bf_hi(hi));
      __stcs(reinterpret_cast<float4*>(dst + grp * GROUP), there ? v : make_float4(0.f, 0.f, 0.f, 0.f));
    }
  }
}

// ------------------------------------------------------------------------------------------------ attention
struct QaArgs {
  CcaDims d;
  const bf16* q;             // [B, Lq], one of the two
  const float* q32;
  QCache c;
  const int* pos;            // decode step: a sequence whose position is negative is skipped; else null
  int extra, max_len, chunk, splits;
  float* part_o;             // [B, hq, splits, DH]
  float* part_ml;            // [B, hq, splits, 2]
  int gather;                // add what each row is given to its weight
  float* scores;             // [B, hk, max_len, g]: logits times log2(e), where the weights are gathered by the second kernel
  bf16* o;
  int* status;
};

CCA_DEVINL int rows_of(const QaArgs& a, int b) {          // -1: does not fit
  const int len = a.c.len[b];
  const long long n = (long long)len + a.extra;
  return (len < 0 || n > a.max_len || n > a.c.S_max || (a.pos && a.pos[b] < 0)) ? -1 : (int)n;
}

// The row of a 16-row tile that operand row r (of 8) stands for.  With this order the key rows of lane groups 2i, 2i + 1 and the
// four value rows of a quad are spread evenly over the two halves of a 128-byte line of shared memory.
CCA_DEVINL int tile_row(int r) { return r ^ ((r >> 1) & 1); }

template <int BYTES>
CCA_DEVINL void cp_async(uint32_t dst, const void* src) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
template <int BYTES>
CCA_DEVINL void cp_async_or_zero(uint32_t dst, const void* src, bool ok) {       // not ok: zeros, nothing is read
  const int n = ok ? BYTES : 0;
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(n) : "memory");
}
CCA_DEVINL void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
CCA_DEVINL void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int V>
struct Int { static constexpr int value = V; };

// A warp's stage of the cache: SR rows' codes and scales as they lie in global memory.  Each warp copies its own (asynchronously,
// 16 bytes a lane, whole lines) and reads it alone, so no barrier but the warp's own stands between them.
template <int DH>
struct Stage {
  using R = Row<DH>;
  static constexpr int SR = DH == 256 ? 16 : 32;           // rows
  static constexpr int SB = R::SCALES * 2;                 // bytes of scales of a row
  static constexpr int K = 0, V = SR * R::CODES, KS = 2 * SR * R::CODES, VS = KS + SR * SB, BYTES = VS + SR * SB;
  static constexpr int N = 2;                              // stages of a warp: one in flight while the other is worked on
  static constexpr int KW = R::NB * R::NG;                 // words of codes of a key row per lane: 2 channel octets of every group
  static constexpr int VB = 2 * R::NG;                     // bytes of codes of a value row per lane and block
  static constexpr int VW = (VB + 3) / 4;

  static constexpr int PER_ROW = R::CODES / 16, PIECES = SR * PER_ROW / 32;

  // Copies rows r0 .. r0 + SR - 1; the pointers are this lane's places in them: byte 16 lane of the codes, row `lane` of the scales.
  CCA_DEVINL static void fill(uint32_t dst, const uint8_t* kp, const uint8_t* vp, const bf16* ksp, const bf16* vsp, int lane) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      cp_async<16>(dst + K + i * 512 + lane * 16, kp + i * 512);
      cp_async<16>(dst + V + i * 512 + lane * 16, vp + i * 512);
    }
    if constexpr (SB >= 4) {                               // d_h = 32: 2 bytes a row are too few for a copy (see Rows)
      if (SR == 32 || lane < SR) {
        cp_async<SB>(dst + KS + lane * SB, ksp);
        cp_async<SB>(dst + VS + lane * SB, vsp);
      }
    }
  }
  // The same for the first `rows` < SR rows alone; the others' places are filled with zeros.
  CCA_DEVINL static void fill_part(uint32_t dst, const uint8_t* kp, const uint8_t* vp, const bf16* ksp, const bf16* vsp, int lane, int rows) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const bool ok = lane / PER_ROW + i * (32 / PER_ROW) < rows;
      cp_async_or_zero<16>(dst + K + i * 512 + lane * 16, ok ? kp + i * 512 : kp - lane * 16, ok);
      cp_async_or_zero<16>(dst + V + i * 512 + lane * 16, ok ? vp + i * 512 : vp - lane * 16, ok);
    }
    if constexpr (SB >= 4) {
      if (lane < SR) {
        const bool ok = lane < rows;
        cp_async_or_zero<SB>(dst + KS + lane * SB, ok ? ksp : ksp - lane * R::SCALES, ok);
        cp_async_or_zero<SB>(dst + VS + lane * SB, ok ? vsp : vsp - lane * R::SCALES, ok);
      }
    }
  }
};

// What a lane takes of 16 rows of a stage: key rows tile_row(g) and 8 more, value rows tile_row(2t), tile_row(2t + 1) and 8 more of each.
template <int DH>
struct Rows {
  using R = Row<DH>;
  using S = Stage<DH>;
  uint32_t k[2][S::KW], v[4][R::NB * S::VW], ks[2][R::SW], vs[2][R::SW];

  // This lane's places in a stage, relative to its start: key row tile_row(g), value rows tile_row(2t) and tile_row(2t + 1), scale
  // row tile_row(g).  Everything else lies at constant distances.
  struct Places {
    uint32_t k, v0, v1, s;
    CCA_DEVINL Places(uint32_t stage, int g, int t)
        : k(stage + S::K + tile_row(g) * R::CODES + t * 4 * R::NG), v0(stage + S::V + tile_row(2 * t) * R::CODES + g * S::VB),
          v1(stage + S::V + tile_row(2 * t + 1) * R::CODES + g * S::VB), s(stage + S::KS + tile_row(g) * S::SB) {}
  };
  template <int NW, int OFF>
  CCA_DEVINL static void take(uint32_t* w, uint32_t at) {
    if constexpr (NW == 1) asm volatile("ld.shared.u32 %0, [%1+%2];" : "=r"(w[0]) : "r"(at), "n"(OFF));
    else if constexpr (NW == 2) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2+%3];" : "=r"(w[0]), "=r"(w[1]) : "r"(at), "n"(OFF));
    else
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4+%5];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at), "n"(OFF));
  }
  // ROW: the 16 rows' number in the stage; r0: the first one's number in the sequence
  template <int ROW>
  CCA_DEVINL void read_keys(const Places& p, int r0, int last, const bf16* ksc, int g) {
    take<R::NG, ROW * R::CODES>(k[0], p.k);
    take<R::NG, (ROW + 8) * R::CODES>(k[1], p.k);
    if constexpr (R::NB == 2) {
      take<R::NG, ROW * R::CODES + R::BLK / 2>(k[0] + R::NG, p.k);
      take<R::NG, (ROW + 8) * R::CODES + R::BLK / 2>(k[1] + R::NG, p.k);
    }
    if constexpr (DH == 32) single_scales(ks, r0, last, ksc, g);
    else { take<R::SW, ROW * S::SB>(ks[0], p.s); take<R::SW, (ROW + 8) * S::SB>(ks[1], p.s); }
  }
  template <int OFF>
  CCA_DEVINL static void take_v(uint32_t* w, uint32_t at) {
    if constexpr (S::VB == 2) {
      unsigned short h;
      asm volatile("ld.shared.u16 %0, [%1+%2];" : "=h"(h) : "r"(at), "n"(OFF));
      w[0] = h;
    } else {
      take<S::VW, OFF>(w, at);
      if constexpr (R::NB == 2) take<S::VW, OFF + R::BLK / 2>(w + S::VW, at);
    }
  }
  template <int ROW>
  CCA_DEVINL void read_values(const Places& p) {
    take_v<ROW * R::CODES>(v[0], p.v0);                    // operand rows 2t, 2t + 1, 2t + 8, 2t + 9
    take_v<ROW * R::CODES>(v[1], p.v1);
    take_v<(ROW + 8) * R::CODES>(v[2], p.v0);
    take_v<(ROW + 8) * R::CODES>(v[3], p.v1);
  }
  template <int ROW>
  CCA_DEVINL void read_value_scales(const Places& p, int r0, int last, const bf16* vsc, int g) {
    if constexpr (DH == 32) single_scales(vs, r0, last, vsc, g);
    else { take<R::SW, S::VS - S::KS + ROW * S::SB>(vs[0], p.s); take<R::SW, S::VS - S::KS + (ROW + 8) * S::SB>(vs[1], p.s); }
  }
  CCA_DEVINL static void single_scales(uint32_t (&w)[2][R::SW], int r0, int last, const bf16* sc, int g) {
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) w[hi][0] = *reinterpret_cast<const unsigned short*>(sc + min(r0 + 8 * hi + tile_row(g), last));
  }
};

constexpr int QA_WARPS = 4, QA_MAX_SPLITS = 128, QA_FIXED = 192;
constexpr int QA_FUSED_SPLITS = 8, QA_FUSED_ROWS = 256, QA_FUSED_LOGITS = 32 * 1024;    // chunks, rows of one, bytes of its logits

template <int DH, int H>
struct FusedShare {                                        // what the CTAs of a cluster read of each other, and what they make of it
  float o[H * DH];
  float2 ml[H];
  float fac[H][8];
  float2 norm[H];                                          // maximum, reciprocal of the sum
};
// CTAs of the attention kernel that an SM holds; registers are given out accordingly.
__host__ __device__ constexpr int qa_resident(int dh, int nht) {
  return nht == 1 ? (dh == 32 ? 7 : dh == 64 ? 6 : dh == 128 ? 4 : 3) : (dh == 32 ? 5 : dh == 64 ? 4 : 3);
}

// One CTA: rows [split * chunk, ...) of sequence b, kv head j, up to 8 NHT of its query heads; its four warps take 16 rows each in
// turn.  S^T = K Q^T has the rows as the 16 and the heads as the 8 of m16n8k16, so that up to 8 heads cost one instruction per
// 256 codes; O^T = V^T P^T has the channels as the 16.  Both read the codes from the registers that they were loaded into.  A
// group's scale multiplies the group's partial logit in fp32; a value row's scale is multiplied into the probability, once
// per group, and goes to the tensor cores as two bf16 numbers: its first 8 significant bits, cut off, and the rest, rounded to 8 (the
// only rounding of the probabilities, 2^-15 at most; the sums are taken before it).  A single bf16 operand adds to the error of the
// output (0.0023 to 0.0026 relative to 64 bits instead of the output's own 0.0017), and a single fp16 one has too few exponents for
// values of different sizes side by side.  32 x 16384 rows: 47.2 us; with a single operand 41.1 to 42.6.
//
// FUSED: a cluster is all of a (sequence, kv head)'s chunks (8 at most); its CTAs join their results through each other's shared
// memory, keep their logits in their own, and finish the whole call: one launch instead of two.
template <int DH, int NHT, bool FUSED>
__global__ void __launch_bounds__(QA_WARPS * 32, qa_resident(DH, NHT)) qcache_attn_kernel(QaArgs a) {
  pdl_enter();
  using R = Row<DH>;
  using S = Stage<DH>;
  constexpr int MT = DH / 16;                              // 16-channel tiles of O^T
  const CcaDims& d = a.d;
  const int split = blockIdx.x, b = blockIdx.z;
  const int n_grp = (d.g + 8 * NHT - 1) / (8 * NHT);
  const int j = blockIdx.y / n_grp, h0 = (blockIdx.y % n_grp) * 8 * NHT;
  const int nh = min(8 * NHT, d.g - h0);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;
  const int n_rows = rows_of(a, b);
  if (n_rows < 0) {
    if (threadIdx.x == 0 && split == 0 && blockIdx.y == 0) atomicCAS(a.status, 0, ST_QCACHE_BAD_LEN);
    return;
  }
  const int r_begin = split * a.chunk, r_end = min(n_rows, r_begin + a.chunk);

  // query operand: head h0 + g (+ 8), channels grp * 32 + 8 t .. + 7 of every group, times 2^64 (e0 lanes) or 2^60 (e1 lanes)
  __shared__ uint4 qs[NHT][R::NB * R::NG][32];
#pragma unroll
  for (int x = warp; x < NHT * R::NB * R::NG; x += QA_WARPS) {
    const int ht = x / (R::NB * R::NG), gi = x % (R::NB * R::NG);
    uint4 w = make_uint4(0, 0, 0, 0);
    if (g + 8 * ht < nh) {
      const size_t off = (size_t)b * d.Lq + (size_t)(j * d.g + h0 + g + 8 * ht) * DH + gi * GROUP + t * 8;
      if (a.q32) {
        const float4 x = *reinterpret_cast<const float4*>(a.q32 + off), y = *reinterpret_cast<const float4*>(a.q32 + off + 4);
        w = make_uint4(pack_bf16x2(x.x, x.y), pack_bf16x2(x.z, x.w), pack_bf16x2(y.x, y.y), pack_bf16x2(y.z, y.w));
      } else {
        w = *reinterpret_cast<const uint4*>(a.q + off);
      }
    }
    qs[ht][gi][lane] = make_uint4(mul_bf16x2(w.x, MUL_E0), mul_bf16x2(w.y, MUL_E1), mul_bf16x2(w.z, MUL_E0), mul_bf16x2(w.w, MUL_E1));
  }
  const float c_scale = rsqrtf((float)DH) * LOG2E * TWO_69;

  // softmax state of heads 2t, 2t + 1 (+ 8 ht): a reference that no logit passes by more than SLACK (the maximum of when it was last
  // moved), the same in all lanes of a column, and sums per lane.  Nothing is ever added to a logit but another logit, so that large ones
  // keep their differences.  The values' scales carry 2^70, which the bf16 subnormals of their codes need: scales of up to 2^48 stay
  // in range, and so do products of probability and scale down to 2^-63.
  constexpr float SLACK = 8.f;
  constexpr uint32_t TWO_70 = 0x62806280u;                 // bf16x2
  float ref[NHT][2], sum[NHT][2];
  float o[NHT][MT][4];
#pragma unroll
  for (int ht = 0; ht < NHT; ++ht) {
#pragma unroll
    for (int c = 0; c < 2; ++c) { ref[ht][c] = -INFINITY; sum[ht][c] = 0.f; }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int c = 0; c < 4; ++c) o[ht][mt][c] = 0.f;
  }

  const size_t base = ((size_t)b * d.hk + j) * a.c.S_max;
  const uint8_t *kc = a.c.k_codes + base * R::CODES, *vc = a.c.v_codes + base * R::CODES;
  const bf16 *ksc = a.c.k_scales + base * R::SCALES, *vsc = a.c.v_scales + base * R::SCALES;
  extern __shared__ __align__(128) unsigned char ring[];
  float* sco = nullptr;                                    // logits of this CTA's rows, from the sequence's row 0 on
  if (FUSED) {
    if (a.gather) sco = reinterpret_cast<float*>(ring + QA_WARPS * S::N * S::BYTES) - r_begin * d.g;
  } else if (a.gather) {
    sco = a.scores + ((size_t)b * d.hk + j) * a.max_len * d.g + h0;
  }

  const int last = r_end - 1, g8 = 8 * d.g;
  const bool even_heads = d.g % 2 == 0;
  const bool put = sco != nullptr && 2 * t < nh;
  auto tile = [&](const typename Rows<DH>::Places& at, int r0, float* sp, auto row_t, auto masked_t) {
    constexpr int ROW = decltype(row_t)::value;
    constexpr bool masked = decltype(masked_t)::value != 0;
    Rows<DH> cur;
    cur.template read_keys<ROW>(at, r0, last, ksc, g);
    // ---- logits (times log2 e) of rows tile_row(g), 8 + tile_row(g), heads 2t, 2t + 1
    float s[NHT][4];
#pragma unroll
    for (int ht = 0; ht < NHT; ++ht)
#pragma unroll
      for (int c = 0; c < 4; ++c) s[ht][c] = 0.f;
#pragma unroll
    for (int gi = 0; gi < R::NB * R::NG; ++gi) {
      const float s_lo = scale_at(cur.ks[0], gi), s_hi = scale_at(cur.ks[1], gi);
      float part[NHT][4];
      uint4 qb[NHT];
#pragma unroll
      for (int ht = 0; ht < NHT; ++ht) qb[ht] = qs[ht][gi][lane];
#pragma unroll
      for (int c = 0; c < 2; ++c) {                        // channel octets of lanes 2t and 2t + 1
        const int blk = gi / R::NG, byte = c * 2 * R::NG + (gi % R::NG) * 2;
        const uint32_t sel = (byte & 2) ? 0x3322u : 0x1100u;
        const uint32_t p0 = __byte_perm(cur.k[0][blk * R::NG + byte / 4], 0, sel), p1 = __byte_perm(cur.k[1][blk * R::NG + byte / 4], 0, sel);
        const uint32_t ka[4] = {code_e0(p0), code_e0(p1), code_e1(p0), code_e1(p1)};
#pragma unroll
        for (int ht = 0; ht < NHT; ++ht) {
          if (c == 0) mma_16816_zero(part[ht], ka, qb[ht].x, qb[ht].y);
          else mma_16816(part[ht], ka, qb[ht].z, qb[ht].w);
        }
      }
#pragma unroll
      for (int ht = 0; ht < NHT; ++ht) {
        s[ht][0] = fmaf(s_lo, part[ht][0], s[ht][0]); s[ht][1] = fmaf(s_lo, part[ht][1], s[ht][1]);
        s[ht][2] = fmaf(s_hi, part[ht][2], s[ht][2]); s[ht][3] = fmaf(s_hi, part[ht][3], s[ht][3]);
      }
    }
    const int r_lo = r0 + tile_row(g), r_hi = r_lo + 8;
#pragma unroll
    for (int ht = 0; ht < NHT; ++ht)
#pragma unroll
      for (int c = 0; c < 4; ++c) s[ht][c] *= c_scale;
    if (put) {
#pragma unroll
      for (int ht = 0; ht < NHT; ++ht) {
        const bool ok_lo = (ht == 0 || 8 * ht + 2 * t < nh) && (!masked || r_lo <= last), ok_hi = ok_lo && (!masked || r_hi <= last);
        if (even_heads) {
          if (ok_lo) *reinterpret_cast<float2*>(sp + 8 * ht) = make_float2(s[ht][0], s[ht][1]);
          if (ok_hi) *reinterpret_cast<float2*>(sp + 8 * ht + g8) = make_float2(s[ht][2], s[ht][3]);
        } else {
          const bool two = 8 * ht + 2 * t + 1 < nh;
          if (ok_lo) { sp[8 * ht] = s[ht][0]; if (two) sp[8 * ht + 1] = s[ht][1]; }
          if (ok_hi) { sp[8 * ht + g8] = s[ht][2]; if (two) sp[8 * ht + g8 + 1] = s[ht][3]; }
        }
      }
    }
    if constexpr (masked) {
#pragma unroll
      for (int ht = 0; ht < NHT; ++ht)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if ((c < 2 ? r_lo : r_hi) > last) s[ht][c] = -INFINITY;
    }
    bool grow = false;
#pragma unroll
    for (int ht = 0; ht < NHT; ++ht)
#pragma unroll
      for (int c = 0; c < 2; ++c) grow = grow || fmaxf(s[ht][c], s[ht][2 + c]) - ref[ht][c] > SLACK;
    if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
      for (int ht = 0; ht < NHT; ++ht)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float m = fmaxf(s[ht][c], s[ht][2 + c]);
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
          if (m > ref[ht][c]) {
            const float al = exp2f(ref[ht][c] - m);        // 0 while nothing has been seen
            ref[ht][c] = m;
            sum[ht][c] *= al;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) { o[ht][mt][c] *= al; o[ht][mt][2 + c] *= al; }
          }
        }
    }
#pragma unroll
    for (int ht = 0; ht < NHT; ++ht)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        s[ht][c] = exp2f(s[ht][c] - ref[ht][c & 1]);
        sum[ht][c & 1] += s[ht][c];
      }
    cur.template read_value_scales<ROW>(at, r0, last, vsc, g);
#pragma unroll
    for (int x = 0; x < R::SW; ++x) { cur.vs[0][x] = mul_bf16x2(cur.vs[0][x], TWO_70); cur.vs[1][x] = mul_bf16x2(cur.vs[1][x], TWO_70); }
    // ---- O^T += V^T P^T
    cur.template read_values<ROW>(at);
#pragma unroll
    for (int gi = 0; gi < R::NB * R::NG; ++gi) {
      const float s_lo = scale_at(cur.vs[0], gi), s_hi = scale_at(cur.vs[1], gi);
      uint32_t pb[NHT][4];                                 // first parts of both rows, second parts
#pragma unroll
      for (int ht = 0; ht < NHT; ++ht) {
        uint32_t rest[2];
        pb[ht][0] = transpose_8x8(split_bf16x2(s[ht][0] * s_lo, s[ht][1] * s_lo, rest[0]));
        pb[ht][1] = transpose_8x8(split_bf16x2(s[ht][2] * s_hi, s[ht][3] * s_hi, rest[1]));
        pb[ht][2] = transpose_8x8(rest[0]);
        pb[ht][3] = transpose_8x8(rest[1]);
      }
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) {
        const int blk = gi / R::NG, byte = (gi % R::NG) * 2 + jj, w = blk * S::VW + byte / 4;
        const uint32_t sel = (byte & 3) * 0x11u + ((byte & 3) + 4) * 0x1100u;
        const uint32_t p0 = __byte_perm(cur.v[0][w], cur.v[1][w], sel), p1 = __byte_perm(cur.v[2][w], cur.v[3][w], sel);
        const uint32_t va[4] = {code_e0(p0), code_e1(p0), code_e0(p1), code_e1(p1)};
#pragma unroll
        for (int ht = 0; ht < NHT; ++ht) {
          mma_16816(o[ht][2 * gi + jj], va, pb[ht][0], pb[ht][1]);
          mma_16816(o[ht][2 * gi + jj], va, pb[ht][2], pb[ht][3]);
        }
      }
    }
  };
  // warp w takes stages w, w + 4, ... of the chunk
  constexpr int STEP = QA_WARPS * S::SR;
  unsigned char* mine = ring + warp * (S::N * S::BYTES);
  const uint32_t mine_u32 = (uint32_t)__cvta_generic_to_shared(mine);
  int r0 = r_begin + warp * S::SR, slot = 0;
  int ahead = r0;                                          // first row of the next stage to be filled
  auto fill_next = [&](int into) {
    const uint32_t dst = mine_u32 + into;
    const uint32_t at = (uint32_t)ahead * R::CODES + lane * 16, sat = (uint32_t)(ahead + lane) * R::SCALES;   // 2^31 bytes at most
    if (ahead + S::SR <= r_end) S::fill(dst, kc + at, vc + at, ksc + sat, vsc + sat, lane);
    else if (ahead < r_end) S::fill_part(dst, kc + at, vc + at, ksc + sat, vsc + sat, lane, r_end - ahead);
    cp_async_commit();
    ahead += STEP;
  };
#pragma unroll
  for (int i = 0; i < S::N; ++i) fill_next(i * S::BYTES);
  static_assert(S::N == 2, "the stages' places alternate");
  __syncthreads();                                         // the query operand
  float* sp = sco + (r0 + tile_row(g)) * d.g + 2 * t;
  const int g16 = 16 * d.g;
  for (; r0 < r_end; r0 += STEP) {
    cp_async_wait<S::N - 1>();
    __syncwarp();
    const typename Rows<DH>::Places at(mine_u32 + slot, g, t);
    if (r0 + S::SR <= r_end) {
      tile(at, r0, sp, Int<0>{}, Int<0>{});
      if constexpr (S::SR == 32) tile(at, r0 + 16, sp + g16, Int<16>{}, Int<0>{});
    } else {
      tile(at, r0, sp, Int<0>{}, Int<1>{});
      if constexpr (S::SR == 32)
        if (r0 + 16 < r_end) tile(at, r0 + 16, sp + g16, Int<16>{}, Int<1>{});
    }
    __syncwarp();
    fill_next(slot);
    slot ^= S::BYTES;
    sp += STEP * d.g;
  }
  cp_async_wait<0>();
#pragma unroll
  for (int ht = 0; ht < NHT; ++ht)
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) sum[ht][c] += __shfl_xor_sync(0xffffffffu, sum[ht][c], x);
  // merge the warps through shared memory
  static_assert(8 * NHT * (DH + 1) * 4 <= S::N * S::BYTES, "a warp's partial result takes the place of its stages");
  __shared__ float sm_ml[QA_WARPS][8 * NHT][2];
  __shared__ FusedShare<FUSED ? DH : 1, FUSED ? 8 * NHT : 1> fz;
  float* my_o = reinterpret_cast<float*>(mine);
  __syncwarp();
#pragma unroll
  for (int ht = 0; ht < NHT; ++ht)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        my_o[(8 * ht + 2 * t + (c & 1)) * (DH + 1) + (mt >> 1) * GROUP + 4 * g + (mt & 1) + 2 * (c >> 1)] =
            o[ht][mt][c] * (c < 2 ? 9.223372036854775808e18f : 5.76460752303423488e17f);    // 2^63, 2^59: 2^133 or 2^129 for the codes, 2^-70
  if (g == 0) {
#pragma unroll
    for (int ht = 0; ht < NHT; ++ht)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        sm_ml[warp][8 * ht + 2 * t + c][0] = ref[ht][c];
        sm_ml[warp][8 * ht + 2 * t + c][1] = sum[ht][c];
      }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < nh * DH; i += QA_WARPS * 32) {
    const int h = i / DH, c = i % DH;
    float mn = -INFINITY;
#pragma unroll
    for (int w = 0; w < QA_WARPS; ++w) mn = fmaxf(mn, sm_ml[w][h][0]);
    float lo = 0.f, oo = 0.f;
#pragma unroll
    for (int w = 0; w < QA_WARPS; ++w) {
      const float al = (sm_ml[w][h][0] == -INFINITY) ? 0.f : exp2f(sm_ml[w][h][0] - mn);
      lo += sm_ml[w][h][1] * al;
      oo += reinterpret_cast<const float*>(ring + w * (S::N * S::BYTES))[h * (DH + 1) + c] * al;
    }
    if constexpr (FUSED) {
      fz.o[h * DH + c] = oo;
      if (c == 0) fz.ml[h] = make_float2(mn, lo);
    } else {
      const size_t pidx = ((size_t)b * d.hq + j * d.g + h0 + h) * a.splits + split;
      a.part_o[pidx * DH + c] = oo;
      if (c == 0) { a.part_ml[pidx * 2] = mn; a.part_ml[pidx * 2 + 1] = lo; }
    }
  }
  if constexpr (FUSED) {
    const int ranks = gridDim.x;
    cluster_barrier();
    for (int h = warp; h < nh; h += QA_WARPS) {            // lane = chunk
      float2 ml = make_float2(-INFINITY, 0.f);
      if (lane < ranks) ml = cluster_float2(&fz.ml[h], lane);
      float m = ml.x;
#pragma unroll
      for (int x = 4; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
      const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - m);
      float l = ml.y * f;
#pragma unroll
      for (int x = 4; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
      const float inv = n_rows > 0 ? 1.f / l : 0.f;
      if (lane < 8) fz.fac[h][lane] = f * inv;
      if (lane == 0) fz.norm[h] = make_float2(m, inv);
    }
    __syncthreads();
    // the output's channels are shared out among the CTAs
    for (int i = split * (QA_WARPS * 32) + threadIdx.x; i < nh * DH; i += ranks * (QA_WARPS * 32)) {
      float part[8], acc = 0.f;
#pragma unroll
      for (int x = 0; x < 8; ++x) part[x] = x < ranks ? cluster_float(&fz.o[i], x) : 0.f;
#pragma unroll
      for (int x = 0; x < 8; ++x) acc = fmaf(part[x], x < ranks ? fz.fac[i / DH][x] : 0.f, acc);
      a.o[(size_t)b * d.Lq + (size_t)(j * d.g) * DH + i] = __float2bfloat16(acc);
    }
    cluster_arrive();                                      // this CTA reads no other's memory any more
    if (sco) {
      float* w = a.c.weight + ((size_t)b * d.hk + j) * a.c.S_max;
      for (int r = r_begin + threadIdx.x; r < r_end; r += QA_WARPS * 32) {
        float acc = 0.f;
        for (int h = 0; h < d.g; ++h) acc = fmaf(exp2f(sco[r * d.g + h] - fz.norm[h].x), fz.norm[h].y, acc);
        atomicAdd(w + r, acc);                             // the row's only one: no order to depend on, and nothing to wait for
      }
    }
    cluster_wait();                                        // nobody leaves while its memory may be read
  }
}

// Joins the chunks' partial results of one (sequence, kv head) and, where the weights are gathered, adds to every row what its
// heads gave it: 2^(logit - maximum) / sum, from the logits that the first kernel left.  Maximum and sum stay apart: a large maximum would
// swallow the logarithm of the sum.  Its time is latency: the logits and weights of its rows are asked for before the sums that they wait for are formed, and a head's
// channels are shared out so that no thread adds up more than four chunks (1 x 16384 rows, both kernels: 7.4 us, 0.9 more with a CTA a head).
constexpr int QJ_ROWS = 4;                                 // rows of a thread, where the weights are gathered
template <int DH>
__global__ void __launch_bounds__(256) qcache_join_kernel(QaArgs a) {
  pdl_enter();
  __shared__ float sm_max[64], sm_inv[64], fac[QA_MAX_SPLITS];
  __shared__ float4 red[64];
  constexpr int PIECES = DH / 32;                          // CTAs that share a head's channels
  const CcaDims& d = a.d;
  const int j = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_rows = rows_of(a, b);
  if (n_rows < 0) return;
  const size_t p0 = ((size_t)b * d.hq + j * d.g) * a.splits;
  const int used = (n_rows + a.chunk - 1) / a.chunk;       // chunks that hold rows
  const float* sc = a.scores + ((size_t)b * d.hk + j) * a.max_len * d.g;
  float* w = a.c.weight + ((size_t)b * d.hk + j) * a.c.S_max;
  const int r_first = blockIdx.x * (256 * QJ_ROWS) + tid;
  float4 s4[QJ_ROWS];
  float wr[QJ_ROWS];
  if (a.gather) {
#pragma unroll
    for (int i = 0; i < QJ_ROWS; ++i) {
      const int r = r_first + i * 256;
      wr[i] = 0.f; s4[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < n_rows) {
        wr[i] = w[r];
        if (d.g % 4 == 0) s4[i] = *reinterpret_cast<const float4*>(sc + (size_t)r * d.g);
      }
    }
  }
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
  for (int h = warp; h < d.g; h += 8) {
    float2 v[QA_MAX_SPLITS / 32];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < QA_MAX_SPLITS / 32; ++i) {
      v[i] = make_float2(-INFINITY, 0.f);
      if (lane + 32 * i < used) v[i] = ml[p0 + (size_t)h * a.splits + lane + 32 * i];
    }
#pragma unroll
    for (int i = 0; i < QA_MAX_SPLITS / 32; ++i) m = fmaxf(m, v[i].x);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
#pragma unroll
    for (int i = 0; i < QA_MAX_SPLITS / 32; ++i) {
      const float f = v[i].x == -INFINITY ? 0.f : exp2f(v[i].x - m);
      if (h == (int)blockIdx.x / PIECES && lane + 32 * i < used) fac[lane + 32 * i] = f;
      l += v[i].y * f;
    }
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
    if (lane == 0) { sm_max[h] = m; sm_inv[h] = n_rows > 0 ? 1.f / l : 0.f; }
  }
  __syncthreads();
  if ((int)blockIdx.x < d.g * PIECES) {                    // a CTA joins 32 channels of a head: 32 threads share 4 of them
    const int h = blockIdx.x / PIECES, c = blockIdx.x % PIECES * 8 + (tid & 7);
    const float4* po = reinterpret_cast<const float4*>(a.part_o + (p0 + (size_t)h * a.splits) * DH) + c;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int s = tid >> 3; s < used; s += 32) {
      const float4 v = po[(size_t)s * (DH / 4)];
      const float f = fac[s];
      acc.x = fmaf(v.x, f, acc.x); acc.y = fmaf(v.y, f, acc.y); acc.z = fmaf(v.z, f, acc.z); acc.w = fmaf(v.w, f, acc.w);
    }
#pragma unroll
    for (int x = 8; x < 32; x <<= 1) {
      acc.x += __shfl_xor_sync(0xffffffffu, acc.x, x); acc.y += __shfl_xor_sync(0xffffffffu, acc.y, x);
      acc.z += __shfl_xor_sync(0xffffffffu, acc.z, x); acc.w += __shfl_xor_sync(0xffffffffu, acc.w, x);
    }
    if (lane < 8) red[warp * 8 + lane] = acc;
    __syncthreads();
    if (tid < 8) {
      for (int x = 1; x < 8; ++x) {
        const float4 v = red[x * 8 + tid];
        acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
      }
      const float inv = sm_inv[h];
      const uint2 u = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
      reinterpret_cast<uint2*>(a.o + (size_t)b * d.Lq + (size_t)(j * d.g + h) * DH)[c] = u;
    }
  }
  if (!a.gather) return;
  auto given = [&](float logit, int h) { return exp2f(logit - sm_max[h]) * sm_inv[h]; };
#pragma unroll
  for (int i = 0; i < QJ_ROWS; ++i) {
    const int r = r_first + i * 256;
    if (r >= n_rows) break;
    float acc = 0.f;
    if (d.g % 4 == 0) {
      acc = given(s4[i].x, 0) + given(s4[i].y, 1) + given(s4[i].z, 2) + given(s4[i].w, 3);
      for (int h = 4; h < d.g; h += 4) {
        const float4 v = *reinterpret_cast<const float4*>(sc + (size_t)r * d.g + h);
        acc += given(v.x, h) + given(v.y, h + 1) + given(v.z, h + 2) + given(v.w, h + 3);
      }
    } else {
      for (int h = 0; h < d.g; ++h) acc += given(sc[(size_t)r * d.g + h], h);
    }
    w[r] = wr[i] + acc;
  }
}

int heads_per_cta(const CcaDims& d) { return d.g <= 8 || d.dh == 256 ? 8 : 16; }

// Rows per CTA and number of chunks for sequences of up to max_len rows.  A chunk costs its rows plus what a CTA costs whatever its
// rows (the way to its first loads, the merge of its warps, its share of the join: about as long as QA_FIXED rows take); of one to four
// full waves of resident CTAs the one with the least is taken.
void attn_plan(const CcaDims& d, int max_len, int sm_count, int* chunk, int* splits) {
  const int n_grp = (d.g + heads_per_cta(d) - 1) / heads_per_cta(d);
  const long long base = (long long)d.B * d.hk * n_grp;
  const int resident = sm_count * qa_resident(d.dh, heads_per_cta(d) / 8);
  long long best = -1;
  for (int waves = 1; waves <= 4; ++waves) {
    long long n = (long long)resident * waves / base;
    if (n < 1) n = 1;
    if (n > QA_MAX_SPLITS) n = QA_MAX_SPLITS;
    long long ch = (max_len + n - 1) / n;
    ch = (ch + 63) / 64 * 64;                              // the four warps of a CTA take 16 rows each per round
    const long long used = (max_len + ch - 1) / ch;
    const long long cost = (base * used + resident - 1) / resident * (ch + QA_FIXED);
    if (best < 0 || cost < best) { best = cost; *chunk = (int)ch; *splits = (int)used; }
  }
}

// Chunks that the plan above makes at most, over all sequences, for any number of rows up to max_len and any batch up to d.B: what a
// workspace holds, so that one made for the longest caches serves shorter ones, which the plan may cut into more chunks.
size_t attn_parts(const CcaDims& d, int max_len, int sm_count) {
  const int n_grp = (d.g + heads_per_cta(d) - 1) / heads_per_cta(d);
  const long long most = 4LL * sm_count * qa_resident(d.dh, heads_per_cta(d) / 8) / (d.hk * n_grp);      // four waves of CTAs
  const long long by_rows = (max_len + 63) / 64 < QA_MAX_SPLITS ? (max_len + 63) / 64 : QA_MAX_SPLITS;
  const long long all = by_rows * d.B;
  return (size_t)(all < most ? all : most > d.B ? most : d.B);
}

// One launch does where 8 chunks hold the sequence that have no more rows than 256 or than the plan above gives a chunk (d_h 128, h_q 8,
// h_k 2, in a graph: 1 x 1024 rows 5.1 us against 6.0 in two launches, 1 x 2048 6.3 against 6.2, 1 x 4096 8.6 against 6.3, 32 x 4096
// 17.7 against 20.8; called one by one, 5.7 against 8.5 us of host time), one CTA has all of a kv head's query heads, and a chunk's logits
// find room.  Chunks of 128 rows: a stage for each warp.
bool attn_fused(const CcaDims& d, int max_len, int sm_count, int gather, int plan_chunk, int* chunk, int* splits) {
  if (d.g > heads_per_cta(d)) return false;
  const long long base = (long long)d.B * d.hk, resident = (long long)sm_count * qa_resident(d.dh, heads_per_cta(d) / 8);
  long long best = -1;
  for (int n = 1; n <= QA_FUSED_SPLITS; n *= 2) {
    const int ch = ((max_len + n - 1) / n + 127) / 128 * 128;
    if ((ch > QA_FUSED_ROWS && ch > plan_chunk) || (gather && ch * d.g * 4 > QA_FUSED_LOGITS)) continue;
    const long long cost = (base * n + resident - 1) / resident * (ch + QA_FIXED);
    if (best < 0 || cost < best) { best = cost; *chunk = ch; *splits = n; }
  }
  return best >= 0;
}

template <int DH, int NHT>
cudaError_t attn_run(const QaArgs& a, dim3 grid, bool fused, cudaStream_t st) {
  constexpr int smem = QA_WARPS * Stage<DH>::N * Stage<DH>::BYTES;
  static_assert(smem <= 48 * 1024, "no opt-in needed");
  if (!fused) return launch_pdl_smem(qcache_attn_kernel<DH, NHT, false>, grid, dim3(QA_WARPS * 32), smem, st, a);
  static bool done[MAX_DEVICES];
  const cudaError_t e = opt_in(qcache_attn_kernel<DH, NHT, true>, smem + QA_FUSED_LOGITS, done);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(QA_WARPS * 32);
  cfg.dynamicSmemBytes = (size_t)(smem + (a.gather ? a.chunk * a.d.g * 4 : 0));
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = grid.x; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, qcache_attn_kernel<DH, NHT, true>, a);
}
template <int DH>
cudaError_t attn_dh(const QaArgs& a, bool fused, cudaStream_t st) {
  const CcaDims& d = a.d;
  const int per = heads_per_cta(d);
  dim3 grid((unsigned)a.splits, (unsigned)(d.hk * ((d.g + per - 1) / per)), (unsigned)d.B);
  if constexpr (DH <= 128)
    if (per == 16) return attn_run<DH, 2>(a, grid, fused, st);
  return attn_run<DH, 1>(a, grid, fused, st);
}

// ------------------------------------------------------------------------------------------------ eviction
struct EvArgs {
  QCache c;
  int hk, keep, recent, max_len;
  int per_cta;                   // rows of a CTA, a multiple of 32
  int move_here;                 // the selecting CTAs move the rows too; else the next kernel does
  int* count;                    // [B * hk] rows to move, for the next kernel
  const int* next;               // [B] position of the next token
  unsigned long long* arrived;   // [B] heads that are done with a sequence
  unsigned long long tag;        // of this call, 48 bits, not 0
  int* list;                     // [B * hk][2][cap]: destinations (rows that go, ascending), sources (rows that come, ascending)
  long long cap;
  int* status;
};

constexpr int EV_SMEM_ROWS = 49152;                        // 192 KB of keys in shared memory
constexpr int EV_THREADS = 1024, EV_BINS = 2048, EV_RANK = 16384;

// The order of eviction as an unsigned number, larger = kept: 0xffffffff for the newest, else the weight's order (a NaN is lowest).
CCA_DEVINL uint32_t keep_key(float w, int pos, long long first_recent) {
  if ((long long)pos >= first_recent) return 0xffffffffu;
  uint32_t u = __float_as_uint(w);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;
  if ((u << 1) == 0u) u = 0u;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Exclusive sum over the 32 warps of a value that is the same in a warp's lanes; `total`: over all of them.
CCA_DEVINL int warp_offsets(int v, int* sm, int warp, int lane, int& total) {
  __syncthreads();
  if (lane == 0) sm[warp] = v;
  __syncthreads();
  const int x = sm[lane];
  int inc = x;
#pragma unroll
  for (int s = 1; s < 32; s <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, inc, s);
    if (lane >= s) inc += y;
  }
  total = __shfl_sync(0xffffffffu, inc, 31);
  return __shfl_sync(0xffffffffu, inc - x, warp);
}

// Moves the listed rows of one head: DH / 16 lanes take the 16-byte pieces of a row's codes (and as many scales); the
// next row's numbers are asked for meanwhile.  A destination is below `keep` and a source is not, so the moves
// need no order.  Bound by scattered reads and writes of rows and
// of their few bytes of scales, weight and position, each of which moves a 32-byte sector (one to four rows a thread, 6 to 48 CTAs per
// SM: all within 5 %).
template <int DH, int THREADS>
CCA_DEVINL void move_rows(const EvArgs& a, size_t base, const int* src, const int* dst, int moves, int part, int parts) {
  using R = Row<DH>;
  constexpr int PIECES = R::CODES / 16, LANES = 2 * PIECES, ROWS = THREADS / LANES;
  const int l = threadIdx.x % LANES, piece = l % PIECES;
  uint4* codes = reinterpret_cast<uint4*>((l < PIECES ? a.c.k_codes : a.c.v_codes) + base * R::CODES) + piece;
  bf16* scales = (l < PIECES ? a.c.k_scales : a.c.v_scales) + base * R::SCALES + piece;
  // lane 0 of a row also moves its weight, lane PIECES its position
  int* extra = l == 0 ? reinterpret_cast<int*>(a.c.weight + base) : l == PIECES ? a.c.position + base : nullptr;
  const int step = parts * ROWS;
  int i = part * ROWS + threadIdx.x / LANES;
  uint32_t from = 0, to = 0;
  if (i < moves) { from = (uint32_t)src[i]; to = (uint32_t)dst[i]; }
  for (; i < moves; i += step) {
    const uint4 u = __ldcs(codes + from * (uint32_t)PIECES);           // a head's rows: 2^27 pieces at most
    const bf16 s = scales[from * (uint32_t)R::SCALES];
    int e = 0;
    if (extra) e = extra[from];
    const uint32_t here = to;
    if (i + step < moves) { from = (uint32_t)src[i + step]; to = (uint32_t)dst[i + step]; }
    codes[here * (uint32_t)PIECES] = u;
    scales[here * (uint32_t)R::SCALES] = s;
    if (extra) extra[here] = e;
  }
}
template <int DH>
__global__ void __launch_bounds__(256, 8) qcache_move_kernel(EvArgs a) {
  pdl_enter();
  const int bj = blockIdx.z * a.hk + blockIdx.y;
  const int* dst = a.list + (size_t)bj * 2 * a.cap;
  move_rows<DH, 256>(a, (size_t)bj * a.c.S_max, dst + a.cap, dst, a.count[bj], blockIdx.x, gridDim.x);
}

// One cluster of 1 to 8 CTAs per (sequence, head), each with a contiguous run of rows: the keep-th largest key by three counting
// passes over its digits (11, 11, 10 bits; the CTAs read each other's counts), then, in ascending order of rows, the rows below `keep` that go and
// the rows behind it that stay, and their moves.  A warp takes a contiguous run of rows, 32 at a time, so ranks come
// from ballots and sums over warps and CTAs.  IN_SMEM: the keys are kept in shared memory after the first reading; longer caches
// read weight and position again (from L2).  A destination is below `keep` and a source is not, so the moves need no order.
// Its time is latency (barriers, one pass after the other) where little moves, else the rows' traffic.
template <int DH, bool IN_SMEM>
__global__ void __launch_bounds__(EV_THREADS, 1) qcache_evict_kernel(EvArgs a) {
  pdl_enter();
  using R = Row<DH>;
  extern __shared__ uint32_t keys[];
  __shared__ __align__(8) int hist[3][EV_BINS];
  __shared__ int sm[32];
  __shared__ int found[3];
  __shared__ int mine[4];                                  // this CTA's counts, read by the others: equal keys, rows that go, that come
  const int rank = blockIdx.x, ranks = gridDim.x, j = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int bj = b * a.hk + j;
  const int n = *reinterpret_cast<volatile int*>(a.c.len + b);
  if (n < 0 || n > a.max_len || n > a.c.S_max) {
    if (tid == 0 && j == 0 && rank == 0) atomicCAS(a.status, 0, ST_QCACHE_BAD_LEN);
    if (tid == 0 && rank == 0) a.count[bj] = 0;
    return;
  }
  if (n <= a.keep) {
    if (tid == 0 && rank == 0) a.count[bj] = 0;
    return;
  }
  const size_t base = (size_t)bj * a.c.S_max;
  int moves = 0;
  int* dst = a.list + (size_t)bj * 2 * a.cap;
  int* src = dst + a.cap;
  const float* w = a.c.weight + base;
  const int* pos = a.c.position + base;
  const long long first_recent = (long long)a.next[b] - a.recent;
  if (a.keep > 0 && n == a.keep + 1 && ranks == 1) {
    // One row goes, as at every step of a cache at its bound: the lowest key's, of equal ones the last row's.  A single minimum
    // instead of three counting passes and two lists (32 x 4097 rows,
    // 2 heads: 8.1 us instead of 14.9, both with the copy that restores the lengths).
    unsigned long long least = ~0ull;
#pragma unroll 4
    for (int r = tid; r < n; r += EV_THREADS) {
      const unsigned long long k = (unsigned long long)keep_key(w[r], pos[r], first_recent) << 32 | (uint32_t)~r;
      least = k < least ? k : least;
    }
    unsigned long long* part = reinterpret_cast<unsigned long long*>(hist[0]);
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) {
      const unsigned long long o = __shfl_xor_sync(0xffffffffu, least, s);
      least = o < least ? o : least;
    }
    if (lane == 0) part[warp] = least;
    __syncthreads();
    least = part[lane];
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) {
      const unsigned long long o = __shfl_xor_sync(0xffffffffu, least, s);
      least = o < least ? o : least;
    }
    const int gone = (int)~(uint32_t)least;
    moves = gone < a.keep ? 1 : 0;
    if (tid == 0) { dst[0] = gone; src[0] = a.keep; }
    __syncthreads();
  } else if (a.keep > 0) {
    const int row0 = min(n, rank * a.per_cta), row1 = min(n, row0 + a.per_cta);
    auto key_of = [&](int r) { return IN_SMEM ? keys[r - row0] : keep_key(w[r], pos[r], first_recent); };
    for (int i = tid; i < EV_BINS; i += EV_THREADS) hist[0][i] = hist[1][i] = hist[2][i] = 0;
    __syncthreads();
    uint32_t prefix = 0;
    int left = a.keep, equal = 0;                          // how many of the rows that share the prefix are kept, and there are
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
      if (IN_SMEM && pass == 0) {                          // eight rows of a thread on their way at a time
        for (int r0 = row0 + tid; r0 < row1; r0 += 8 * EV_THREADS) {
          float wr[8];
          int pr[8];
#pragma unroll
          for (int x = 0; x < 8; ++x)
            if (r0 + x * EV_THREADS < row1) { wr[x] = w[r0 + x * EV_THREADS]; pr[x] = pos[r0 + x * EV_THREADS]; }
#pragma unroll
          for (int x = 0; x < 8; ++x)
            if (r0 + x * EV_THREADS < row1) {
              const uint32_t k = keep_key(wr[x], pr[x], first_recent);
              keys[r0 + x * EV_THREADS - row0] = k;
              atomicAdd(&hist[0][k >> shift], 1);
            }
        }
      } else
#pragma unroll 4
      for (int r = row0 + tid; r < row1; r += EV_THREADS) {
        const uint32_t k = key_of(r);
        if (pass == 0 || (k >> (shift + bits)) == prefix) atomicAdd(&hist[pass][(k >> shift) & ((1u << bits) - 1u)], 1);
      }
      all_sync(ranks);
      // bins from the top: thread i has bins BINS - 1 - 2i and BINS - 2 - 2i
      const int* mybins = &hist[pass][EV_BINS - 2 - 2 * tid];
      int c0 = 0, c1 = 0;
      if (ranks == 1) { c0 = mybins[1]; c1 = mybins[0]; }
      else
        for (int x = 0; x < ranks; ++x) {
          const int2 v = cluster_load2(mybins, x);
          c0 += v.y; c1 += v.x;
        }
      int inc = c0 + c1;
#pragma unroll
      for (int s = 1; s < 32; s <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, s);
        if (lane >= s) inc += y;
      }
      int all;
      const int before = warp_offsets(__shfl_sync(0xffffffffu, inc, 31), sm, warp, lane, all) + inc - c0 - c1;
      if (before < left && left <= before + c0) { found[0] = EV_BINS - 1 - 2 * tid; found[1] = left - before; found[2] = c0; }
      if (before + c0 < left && left <= before + c0 + c1) { found[0] = EV_BINS - 2 - 2 * tid; found[1] = left - before - c0; found[2] = c1; }
      __syncthreads();
      prefix = (prefix << bits) | (uint32_t)found[0];
      left = found[1];
      equal = found[2];
    }
    const uint32_t lowest = prefix;                        // keys above it stay, and the first `left` rows that equal it
    const int run = (a.per_cta + EV_THREADS - 1) / EV_THREADS * 32;    // rows of a warp
    const int r_begin = min(row1, row0 + warp * run), r_end = min(row1, r_begin + run);
    // what this CTA's and the lower CTAs' warps before this one have counted
    auto place = [&](int v, int slot) {
      int total;
      int at = warp_offsets(v, sm, warp, lane, total);
      if (ranks > 1) {
        if (tid == 0) mine[slot] = total;
        all_sync(ranks);
        for (int x = 0; x < rank; ++x) at += cluster_load(&mine[slot], x);
      }
      return at;
    };
    int eq0 = 0;
    if (equal > left) {                                    // the same in every CTA of the cluster
      int eq = 0;
      for (int r0 = r_begin; r0 < r_end; r0 += 32) {
        const int r = r0 + lane;
        eq += __popc(__ballot_sync(0xffffffffu, r < r_end && key_of(r) == lowest));
      }
      eq0 = place(eq, 0);
    }
    const unsigned below = (1u << lane) - 1u;
    int e = eq0;
    auto stays_of = [&](int r0) {                          // of rows r0 .. r0 + 31, as a mask; called for a warp's rows in order
      const int r = r0 + lane;
      const uint32_t k = r < r_end ? key_of(r) : 0u;
      bool stays = k > lowest;
      if (equal <= left) return __ballot_sync(0xffffffffu, r < r_end && (stays || k == lowest));
      const unsigned beq = __ballot_sync(0xffffffffu, r < r_end && k == lowest);
      stays = stays || (k == lowest && e + __popc(beq & below) < left);
      e += __popc(beq);
      return __ballot_sync(0xffffffffu, r < r_end && stays);
    };
    // 32 times 32 rows at a time: lane i keeps the mask of the i-th 32, and from it the masks of those that go and that come
    unsigned mgo, mco;
    auto masks = [&](int s0) {
      unsigned st = 0;
      const int chunks = min(32, (r_end - s0 + 31) >> 5);
#pragma unroll 4
      for (int i = 0; i < chunks; ++i) {
        const unsigned m = stays_of(s0 + 32 * i);
        if (lane == i) st = m;
      }
      const int r0 = s0 + 32 * lane, head = a.keep - r0, there = r_end - r0;
      const unsigned below_keep = head >= 32 ? 0xffffffffu : head <= 0 ? 0u : (1u << head) - 1u;
      const unsigned rows = there >= 32 ? 0xffffffffu : there <= 0 ? 0u : (1u << there) - 1u;
      mgo = rows & below_keep & ~st;
      mco = ~below_keep & st;
    };
    int go = 0, come = 0;
    for (int s0 = r_begin; s0 < r_end; s0 += 1024) {
      masks(s0);
      go += __popc(mgo); come += __popc(mco);
    }
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) {
      go += __shfl_xor_sync(0xffffffffu, go, s);
      come += __shfl_xor_sync(0xffffffffu, come, s);
    }
    int tg, tc;
    int go0 = warp_offsets(go, sm, warp, lane, tg), come0 = warp_offsets(come, sm, warp, lane, tc);
    moves = tg;
    if (ranks > 1) {
      if (tid == 0) { mine[1] = tg; mine[2] = tc; }
      all_sync(ranks);
      moves = 0;
      for (int x = 0; x < ranks; ++x) {
        const int xg = cluster_load(&mine[1], x), xc = cluster_load(&mine[2], x);
        moves += xg;
        if (x < rank) { go0 += xg; come0 += xc; }
      }
    }
    e = eq0;
    for (int s0 = r_begin; s0 < r_end; s0 += 1024) {
      if (s0 > r_begin || r_end - r_begin > 1024) masks(s0);           // else they are still there
      const int both = __popc(mgo) | (__popc(mco) << 16);
      int inc = both;
#pragma unroll
      for (int s = 1; s < 32; s <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, s);
        if (lane >= s) inc += y;
      }
      const int at = inc - both;
      const int chunks = min(32, (r_end - s0 + 31) >> 5);
#pragma unroll 4
      for (int i = 0; i < chunks; ++i) {
        const unsigned g = __shfl_sync(0xffffffffu, mgo, i), c = __shfl_sync(0xffffffffu, mco, i);
        const int p = __shfl_sync(0xffffffffu, at, i), r = s0 + 32 * i + lane;
        if (g >> lane & 1u) dst[go0 + (p & 0xffff) + __popc(g & below)] = r;
        if (c >> lane & 1u) src[come0 + (p >> 16) + __popc(c & below)] = r;
      }
      const int all = __shfl_sync(0xffffffffu, inc, 31);
      go0 += all & 0xffff; come0 += all >> 16;
    }
    all_sync(ranks);                                       // the lists are whole, and nobody reads weights or positions any more
  }
  if (a.move_here) move_rows<DH, EV_THREADS>(a, base, src, dst, moves, rank, ranks);
  else if (tid == 0 && rank == 0) a.count[bj] = moves;
  // The length is written by the last head to be done with it, so that every CTA, early or late, reads the length from before.  The
  // workspace comes as it is: a count is one only under this call's tag (48 bits), and the last head leaves a zero, so that a
  // replayed call finds none of its own.
  if (a.keep == 0) all_sync(ranks);                        // (else: every CTA of the cluster has read it before the lists were whole)
  if (rank == 0 && tid == 0) {
    unsigned long long seen = a.arrived[b], now;
    bool last;
    do {
      now = seen;
      const int heads = (now >> 16) == a.tag ? (int)(now & 0xffffu) + 1 : 1;
      last = heads == a.hk;
      seen = atomicCAS(a.arrived + b, now, last ? 0ull : (a.tag << 16 | (unsigned long long)heads));
    } while (seen != now);
    if (last) a.c.len[b] = a.keep;
  }
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }


}  // namespace

#define QC_BY_HEAD(call)           \
  switch (d.dh) {                  \
    case 32: { constexpr int DH = 32; e = call; break; }    \
    case 64: { constexpr int DH = 64; e = call; break; }    \
    case 128: { constexpr int DH = 128; e = call; break; }  \
    case 256: { constexpr int DH = 256; e = call; break; }  \
    default: return 1;             \
  }

namespace {
uint32_t head_inverse(int hk) { return hk == 1 ? 0xffffffffu : (uint32_t)((1ull << 32) / (unsigned)hk); }
long long io_units(const CcaDims& d, long long n) { return n * d.hk * (d.dh > 128 ? d.dh / 128 : 1) * 2; }
// 32 units a CTA and the sequences side by side; at most about 32 CTAs for each of 148 SMs, then around again
dim3 io_grid(const CcaDims& d, long long n) {
  long long x = (io_units(d, n) + 31) / 32, most = 4736 / d.B;
  if (most < 1) most = 1;
  return dim3((unsigned)(x < most ? x : most), (unsigned)d.B);
}
}  // namespace

int launch_qcache_append(const CcaDims& d, const bf16* k, const bf16* v, const int* position, const int* count, const QCache& c,
                         long long n, long long limit, int* status, long long* launches, cudaStream_t st) {
  IoArgs a;
  memset(&a, 0, sizeof(a));
  a.k = k; a.v = v; a.position = position; a.count = count; a.c = c; a.n = n; a.limit = limit; a.hk = d.hk;
  a.hk_inv = head_inverse(d.hk);
  a.status = status;
  if (io_units(d, n) > 1LL << 31) return 1;
  const dim3 grid = io_grid(d, n);
  cudaError_t e;
  QC_BY_HEAD((launch_pdl(qcache_append_kernel<DH>, grid, dim3(256), st, a)))
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  return 0;
}

int launch_qcache_read(const CcaDims& d, const QCache& c, const int* first, float* k, float* v, long long n, long long* launches,
                       cudaStream_t st) {
  IoArgs a;
  memset(&a, 0, sizeof(a));
  a.k_out = k; a.v_out = v; a.first = first; a.c = c; a.n = n; a.hk = d.hk; a.hk_inv = head_inverse(d.hk);
  if (io_units(d, n) > 1LL << 31) return 1;
  const dim3 grid = io_grid(d, n);
  cudaError_t e;
  QC_BY_HEAD((launch_pdl(qcache_read_kernel<DH>, grid, dim3(256), st, a)))
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  return 0;
}

size_t qcache_workspace_bytes(const CcaDims& d, int max_len, int sm_count) {
  const size_t parts = d.hq * attn_parts(d, max_len, sm_count);
  const size_t attn = up256(parts * d.dh * 4) + up256(parts * 2 * 4) +
                      up256((size_t)d.B * d.hq * max_len * 4);
  const size_t ev = up256((size_t)d.B * 8) + up256((size_t)d.B * d.hk * 4) + up256((size_t)d.B * d.hk * 2 * (max_len / 2 + 1) * 4);
  return attn > ev ? attn : ev;
}

int launch_qcache_attention(const CcaDims& d, const bf16* q, const float* q32, bf16* o, const QCache& c, const int* pos, int extra,
                            int max_len, int accumulate, void* workspace, int sm_count, int* status, long long* launches,
                            cudaEvent_t ev_begin, cudaEvent_t ev_end, cudaStream_t st) {
  QaArgs a;
  memset(&a, 0, sizeof(a));
  a.d = d; a.q = q; a.q32 = q32; a.c = c; a.pos = pos; a.extra = extra; a.max_len = max_len; a.o = o; a.status = status;
  attn_plan(d, max_len, sm_count, &a.chunk, &a.splits);
  unsigned char* p = static_cast<unsigned char*>(workspace);
  a.part_o = reinterpret_cast<float*>(p); p += up256((size_t)d.B * d.hq * a.splits * d.dh * 4);
  a.part_ml = reinterpret_cast<float*>(p); p += up256((size_t)d.B * d.hq * a.splits * 2 * 4);
  a.scores = reinterpret_cast<float*>(p);
  a.gather = accumulate != 0;
  const bool fused = attn_fused(d, max_len, sm_count, a.gather, a.chunk, &a.chunk, &a.splits);
  cudaError_t e;
  if (ev_begin && (e = cudaEventRecord(ev_begin, st)) != cudaSuccess) return -(int)e;
  QC_BY_HEAD(attn_dh<DH>(a, fused, st))
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  if (ev_end && (e = cudaEventRecord(ev_end, st)) != cudaSuccess) return -(int)e;
  if (fused) return 0;
  int nx = d.g * (d.dh / 32);                              // a CTA per 32 channels of a head at least
  const int by_rows = (max_len + 256 * QJ_ROWS - 1) / (256 * QJ_ROWS);
  if (accumulate && by_rows > nx) nx = by_rows;
  QC_BY_HEAD((launch_pdl(qcache_join_kernel<DH>, dim3((unsigned)nx, (unsigned)d.hk, (unsigned)d.B), dim3(256), st, a)))
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  return 0;
}

namespace {
template <int DH, bool IN_SMEM>
cudaError_t evict_run(const EvArgs& a, int ranks, int B, int smem, cudaStream_t st) {
  static bool done[MAX_DEVICES];
  if (IN_SMEM) {
    const cudaError_t e = opt_in(qcache_evict_kernel<DH, IN_SMEM>, EV_SMEM_ROWS * 4, done);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ranks, (unsigned)a.hk, (unsigned)B);
  cfg.blockDim = dim3(EV_THREADS);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)ranks; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, qcache_evict_kernel<DH, IN_SMEM>, a);
}
}  // namespace

int launch_qcache_evict(const CcaDims& d, const QCache& c, int keep, int recent, const int* next_position, int max_len,
                        void* workspace, unsigned long long tag, int sm_count, int* status, long long* launches, cudaStream_t st) {
  EvArgs a;
  memset(&a, 0, sizeof(a));
  a.c = c; a.hk = d.hk; a.keep = keep; a.recent = recent; a.max_len = max_len; a.next = next_position; a.status = status;
  a.cap = max_len / 2 + 1;                                 // as many rows go below `keep` as come from behind it
  a.arrived = static_cast<unsigned long long*>(workspace);
  a.tag = tag;
  a.count = reinterpret_cast<int*>(static_cast<unsigned char*>(workspace) + up256((size_t)d.B * 8));
  a.list = reinterpret_cast<int*>(reinterpret_cast<unsigned char*>(a.count) + up256((size_t)d.B * d.hk * 4));
  // more CTAs a head while there are SMs for them and each keeps EV_RANK rows or more (fewer cost more in barriers than they save)
  int ranks = 1;
  while (ranks < 8 && (long long)d.B * d.hk * ranks * 2 <= sm_count && max_len >= ranks * 2 * EV_RANK) ranks *= 2;
  const int most = keep < max_len - keep ? keep : max_len - keep;      // rows of a head that can move
  a.move_here = most <= 512 * ranks;                                   // more are moved by a kernel over all SMs
  a.per_cta = ((max_len + ranks - 1) / ranks + 31) / 32 * 32;
  const bool in_smem = a.per_cta <= EV_SMEM_ROWS;
  cudaError_t e;
  if (in_smem) QC_BY_HEAD((evict_run<DH, true>(a, ranks, d.B, a.per_cta * 4, st)))
  else QC_BY_HEAD((evict_run<DH, false>(a, ranks, d.B, 0, st)))
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  if (a.move_here) return 0;
  // up to four full waves of CTAs over all heads (fewer rows a CTA hide less of what each waits for), none without a turn of its loop
  const int rows = 256 / (d.dh / 16);
  int nx = (most + rows - 1) / rows;
  const int per_head = (int)((32LL * sm_count + (long long)d.B * d.hk - 1) / ((long long)d.B * d.hk));
  if (nx > per_head) nx = per_head;
  QC_BY_HEAD((launch_pdl(qcache_move_kernel<DH>, dim3((unsigned)nx, (unsigned)d.hk, (unsigned)d.B), dim3(256), st, a)))
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  return 0;
}
