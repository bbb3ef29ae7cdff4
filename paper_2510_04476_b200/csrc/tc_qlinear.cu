// y = x W^T for up to 64 tokens at a time on the tensor cores of this architecture, W in the 4-bit format of qformat.cuh.
//
//   warp 0       : TMA producer (one lane)            -- x tiles, up to 64 tokens x 128 channels, 6 stages
//   warp 1       : TMEM owner + MMA issuer (one lane) -- 128 weight rows x tokens x 16 channels per instruction
//   warps 2..13  : three groups of four, a thread per weight row: a block of 128 channels from its 64 bytes of codes into tensor
//                  memory, as the MMA's A operand; the groups take the blocks in turn
//
// A weight c * s has up to 11 significant bits, which one bf16 operand cannot hold.  It becomes two, c * s' and c * (s - s'), with
// s' the scale's first four significant bits: both products are exact (3 + 4 bits), so that the only roundings are those
// of adds.  One operand alone would add an error of up to 2^-8 of each weight to a result that is rounded once.
// 64 x 8192 x 8192 takes 22.9 us (floor: 6.2 us to read the codes, 7.7 us of matrix instructions).  Timed with parts left out, a third of
// it is a CTA's way to its first block and from its last, 8.4 us the matrix unit, which the dequantisation (2 instructions a code,
// 3.4 us by itself, 3.4 more for its loads) does not overlap well: three groups of warps are what tensor memory has room for.
// The inner dimension is split over the CTAs of a cluster where there are fewer row blocks than SMs; each rank adds up its share of the
// tokens, in rank order, from parts that the others write into its shared memory (four tokens a store: 1.8 us less than one).
#include "pdl.cuh"
#include "qformat.cuh"
#include "qlinear.cuh"
#include "tc_ptx.cuh"
#include "tc_state.cuh"

using namespace tc;
using namespace q4;

namespace {

constexpr int TQ_GROUPS = 3, TQ_WARPS = 2 + 4 * TQ_GROUPS, TQ_THREADS = 32 * TQ_WARPS;
constexpr int TQ_STAGES = 2 * TQ_GROUPS, TQ_TOKENS = 64;
constexpr int TQ_STAGE_BYTES = TQ_TOKENS * 256;
constexpr int TQ_PART_BYTES = 8 * 128 * 12 * 4;                       // a cluster's sums: [rank][128 rows][this rank's tokens + 4] fp32
constexpr int TQ_SUM_BYTES = 128 * TQ_TOKENS * 4;                     // sums of the chunks so far: [16 quads of tokens][128 rows] float4
constexpr int TQ_SMEM = TQ_STAGES * TQ_STAGE_BYTES + TQ_PART_BYTES + TQ_SUM_BYTES + 256 + 1024;      // barriers, 1024-byte alignment
constexpr int TQ_CHUNK = 4;                                           // blocks of a chain of adds; each group has one of them at least
static_assert(TQ_CHUNK >= TQ_GROUPS, "a group takes a chunk over behind its first block of the next");
constexpr int TQ_A_COL = 64;                                          // accumulator columns, then the groups' operands,
constexpr int TQ_ACC1 = TQ_A_COL + TQ_GROUPS * 128;                   // then the other accumulator's
constexpr uint32_t MUL_104 = 0x73807380u, MUL_100 = 0x71807180u;      // bf16x2 2^104, 2^100: operands become c s 2^-29
constexpr float TWO_29 = 536870912.f;                                 // exact for scales from 2^-90 to 2^22

struct TqSeg {
  const uint8_t* codes;
  const bf16* scales;
  int N, out_off;
};
struct TqParams {
  TqSeg seg0, seg1;
  int blocks0;               // row blocks of the first segment
  int K128, M, n_tok;        // n_tok: tokens of a pass, a multiple of 16
  int per_cta;               // channel blocks of a CTA
  int mine;                  // tokens that a rank adds up: the ranks' shares, rounded up to a multiple of 4
  float* out_f32;
  bf16* out_bf16;
  int ldo;
  int* status;
};

TC_DEVINL void fail(volatile int* abort_flag, int* status, int code) {
  *abort_flag = 1;
  atomicCAS(status, 0, code);
}
CCA_DEVINL uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
CCA_DEVINL uint32_t cluster_addr(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
CCA_DEVINL void st_cluster_v4(uint32_t addr, float a, float b, float c, float d) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(a), "f"(b), "f"(c), "f"(d) : "memory");
}
CCA_DEVINL void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
CCA_DEVINL void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

__global__ void __launch_bounds__(TQ_THREADS, 1)
tc_qlinear_kernel(const __grid_constant__ CUtensorMap tm0, const __grid_constant__ CUtensorMap tm1, TqParams p) {
  pdl_enter();
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* smem = smem_align1024(smem_dyn);
  float* part = reinterpret_cast<float*>(smem + TQ_STAGES * TQ_STAGE_BYTES);
  float4* sums = reinterpret_cast<float4*>(smem + TQ_STAGES * TQ_STAGE_BYTES + TQ_PART_BYTES);
  uint64_t* b_full = reinterpret_cast<uint64_t*>(smem + TQ_STAGES * TQ_STAGE_BYTES + TQ_PART_BYTES + TQ_SUM_BYTES);
  uint64_t* b_empty = b_full + TQ_STAGES;
  uint64_t* a_full = b_empty + TQ_STAGES;
  uint64_t* a_empty = a_full + TQ_GROUPS;
  uint64_t* acc_full = a_empty + TQ_GROUPS;
  uint64_t* acc_empty = acc_full + 2;
  uint64_t* done_bar = acc_empty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done_bar + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x, ranks = gridDim.x;
  const bool second = (int)blockIdx.y >= p.blocks0;
  const TqSeg sg = second ? p.seg1 : p.seg0;
  const CUtensorMap* map = second ? &tm1 : &tm0;
  const int row0 = ((int)blockIdx.y - (second ? p.blocks0 : 0)) * 128, tok0 = (int)blockIdx.z * TQ_TOKENS;
  const int kb_begin = rank * p.per_cta, n_kb = max(0, min(p.K128, kb_begin + p.per_cta) - kb_begin);

  const int sub = p.n_tok * 128;                           // bytes of a 64-channel half of an x tile
  auto load_x = [&](int i, int st) {
    unsigned char* dst = smem + st * TQ_STAGE_BYTES;
    mbar_expect_tx(&b_full[st], 2 * sub);
    tma_load_2d(dst, map, (kb_begin + i) * 128, tok0, &b_full[st]);
    tma_load_2d(dst + sub, map, (kb_begin + i) * 128 + 64, tok0, &b_full[st]);
  };
  // a dequantising thread's row and its first two blocks, on their way while the barriers and the tensor memory are set up
  const int gr = (warp - 2) >> 2, q = warp & 3;
  const int row = row0 + q * 32 + lane;
  const bool there = warp >= 2 && row < (sg.N + 15) / 16 * 16;      // rows that the tiles hold
  const size_t tile = (size_t)(row >> 4) * p.K128 + kb_begin;
  const uint4* codes = reinterpret_cast<const uint4*>(sg.codes + (tile * 16 + (row & 15)) * 64);
  const uint2* scales = reinterpret_cast<const uint2*>(sg.scales + (tile * 16 + (row & 15)) * 4);
  struct Block { uint4 c[4]; uint2 s; };
  Block w0, w1, w2;
#pragma unroll
  for (int x = 0; x < 4; ++x) w0.c[x] = w1.c[x] = w2.c[x] = make_uint4(0, 0, 0, 0);
  w0.s = w1.s = w2.s = make_uint2(0, 0);
  auto load = [&](Block& w, int i) {
    if (i < n_kb && there) {
#pragma unroll
      for (int x = 0; x < 4; ++x) w.c[x] = __ldg(codes + (size_t)i * 64 + x);
      w.s = __ldg(scales + (size_t)i * 16);
    }
  };
  load(w0, gr); load(w1, gr + TQ_GROUPS);

  if (threadIdx.x == 0) {
    for (int s = 0; s < TQ_STAGES; ++s) { mbar_init(&b_full[s], 1); mbar_init(&b_empty[s], 1); }
    for (int s = 0; s < TQ_GROUPS; ++s) { mbar_init(&a_full[s], 4); mbar_init(&a_empty[s], 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(&acc_full[s], 1); mbar_init(&acc_empty[s], 4 * min(TQ_GROUPS, p.n_tok / 16)); }
    mbar_init(done_bar, 1);
    fence_barrier_init();
    for (int i = 0; i < min(n_kb, TQ_STAGES); ++i) load_x(i, i);
  }
  if (threadIdx.x == 64) wait_ctl_init(abort_flag, p.status);
  if (warp == 1) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (ranks > 1) cluster_arrive();                         // from here on the others may be written to (see the sums)
  const uint32_t tmem = *tmem_slot;

  if (warp == 0) {
    if (lane == 0) {
      for (int i = TQ_STAGES; i < n_kb; ++i) {
        const int st = i % TQ_STAGES;
        if (!mbar_wait(&b_empty[st], ((i / TQ_STAGES) & 1) ^ 1, abort_flag)) { fail(abort_flag, p.status, ST_TIMEOUT_TMA); break; }
        load_x(i, st);
      }
    }
  } else if (warp == 1) {
    const bool leader = elect_one();
    const uint32_t idesc = idesc_bf16(p.n_tok, 0, 0);
    const uint32_t desc_hi = (uint32_t)(smem_desc_sw128(0, 0, 1024) >> 32);
    const uint32_t smem_lo = smem_u32(smem) >> 4;
    bool ok = true;
    uint32_t sph = 0;
    for (int i0 = 0; ok && i0 < n_kb; i0 += TQ_STAGES, sph ^= 1) {
#pragma unroll
      for (int st = 0; st < TQ_STAGES; ++st) {             // stage and group are constants here, and so are the operands' places
        const int i = i0 + st, gr = st % TQ_GROUPS;
        if (i >= n_kb) break;
        ok = __all_sync(0xffffffffu, mbar_wait(&b_full[st], sph, abort_flag)) &&
             __all_sync(0xffffffffu, mbar_wait(&a_full[gr], (st / TQ_GROUPS) & 1, abort_flag));
        const int chunk = i / TQ_CHUNK, in_chunk = i - chunk * TQ_CHUNK;
        if (ok && in_chunk == 0)
          ok = __all_sync(0xffffffffu, mbar_wait(&acc_empty[chunk & 1], ((chunk >> 1) & 1) ^ 1, abort_flag));
        if (!ok) { fail(abort_flag, p.status, ST_TIMEOUT_MMA); break; }
        tc_fence_after();
        const uint32_t a = tmem + TQ_A_COL + gr * 128;
        const uint32_t b = (smem_lo + st * (TQ_STAGE_BYTES >> 4)) | (1u << 16);
        if (leader) {
#pragma unroll
          for (int part = 0; part < 2; ++part)
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
              mma_ts_w(tmem + (chunk & 1) * TQ_ACC1, a + part * 64 + ks * 8, b + (ks >> 2) * (sub >> 4) + (ks & 3) * 2, desc_hi, idesc,
                       (in_chunk | part | ks) != 0);
          mma_commit(&a_empty[gr]);
          mma_commit(&b_empty[st]);
          if (in_chunk == TQ_CHUNK - 1) mma_commit(&acc_full[chunk & 1]);
          if (i == n_kb - 1) mma_commit(done_bar);
        }
      }
    }
  } else {
    const uint32_t a = tmem + ((uint32_t)(q * 32) << 16) + TQ_A_COL + gr * 128;
    // two blocks of the group ahead are on their way while one is worked on
    uint32_t phase = 1;
    auto work = [&](const Block& w) -> bool {
      if (!__all_sync(0xffffffffu, mbar_wait(&a_empty[gr], phase, abort_flag))) { fail(abort_flag, p.status, ST_TIMEOUT_EPI); return false; }
      phase ^= 1;
      tc_fence_after();
#pragma unroll
      for (int grp = 0; grp < 4; ++grp) {
        const uint32_t s2 = __byte_perm(grp < 2 ? w.s.x : w.s.y, 0, (grp & 1) ? 0x3232u : 0x1010u);
        const uint32_t h2 = s2 & 0xfff0fff0u, l2 = sub_bf16x2(s2, h2);             // four significant bits, and the rest
        const uint32_t m0 = mul_bf16x2(h2, MUL_104), m1 = mul_bf16x2(h2, MUL_100);
        const uint32_t n0 = mul_bf16x2(l2, MUL_104), n1 = mul_bf16x2(l2, MUL_100);
        uint32_t hi[16], lo[16];
#pragma unroll
        for (int g = 0; g < 8; ++g) {
          const uint4 c = w.c[g >> 1];
          const uint32_t word = (g & 1) ? (grp < 2 ? c.z : c.w) : (grp < 2 ? c.x : c.y);
          const uint32_t pr = __byte_perm(word, 0, (grp & 1) ? 0x3322u : 0x1100u);
          const uint32_t e0 = code_e0(pr), e1 = code_e1(pr);
          hi[2 * g] = mul_bf16x2(e0, m0); hi[2 * g + 1] = mul_bf16x2(e1, m1);
          lo[2 * g] = mul_bf16x2(e0, n0); lo[2 * g + 1] = mul_bf16x2(e1, n1);
        }
        tmem_st16(a + grp * 16, hi);
        tmem_st16(a + 64 + grp * 16, lo);
      }
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&a_full[gr]);
      return true;
    };
    const int r = q * 32 + lane;
    // The tensor cores cut off what an add shifts out, always towards the same side, so that a chain's error grows with its length (64 x 8192
    // x 8192 in chains of 512 adds: 4.6e-6 relative to 64 bits, of 1024 9.7e-6).  So a chain is TQ_CHUNK blocks, 64 adds; its sum is added to
    // those before it in fp32 by the warps that have its rows, while the other accumulator takes the next chunk: 4.8e-7,
    // and for longer rows one fp32 add more for every 64; 22.9 us (one chain: 21.3; chunks of 3: 3.6e-7, 23.9; of 6: 7.0e-7, 22.5).
    int next = 0;                                          // the chunk to be taken over next
    auto take_over = [&](int end) -> bool {
      for (; next < end; ++next) {
        if (gr >= p.n_tok / 16) continue;
        const int buf = next & 1;
        if (!__all_sync(0xffffffffu, mbar_wait(&acc_full[buf], (next >> 1) & 1, abort_flag))) { fail(abort_flag, p.status, ST_TIMEOUT_EPI); return false; }
        tc_fence_after();
        for (int c = gr; c < p.n_tok / 16; c += TQ_GROUPS) {
          uint32_t v[16];
          tmem_ld16(tmem + ((uint32_t)(q * 32) << 16) + buf * TQ_ACC1 + c * 16, v);
          tmem_ld_wait();
          float4* at = sums + c * 4 * 128 + r;
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            float4 o = next ? at[x * 128] : make_float4(0.f, 0.f, 0.f, 0.f);
            o.x += __uint_as_float(v[4 * x]); o.y += __uint_as_float(v[4 * x + 1]);
            o.z += __uint_as_float(v[4 * x + 2]); o.w += __uint_as_float(v[4 * x + 3]);
            at[x * 128] = o;
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&acc_empty[buf]);
      }
      return true;
    };
    // A chunk is taken over behind the group's first block of the next one, so that the tensor cores have work meanwhile.
    for (int i = gr; i < n_kb; i += 3 * TQ_GROUPS) {
      load(w2, i + 2 * TQ_GROUPS);
      if (!work(w0) || !take_over(i / TQ_CHUNK)) break;
      if (i + TQ_GROUPS >= n_kb) break;
      load(w0, i + 3 * TQ_GROUPS);
      if (!work(w1) || !take_over((i + TQ_GROUPS) / TQ_CHUNK)) break;
      if (i + 2 * TQ_GROUPS >= n_kb) break;
      load(w1, i + 4 * TQ_GROUPS);
      if (!work(w2) || !take_over((i + 2 * TQ_GROUPS) / TQ_CHUNK)) break;
    }
    const int last_chunk = max(n_kb - 1, 0) / TQ_CHUNK;
    // ---- sums: thread = row, one column per token.  In a cluster a rank adds up `mine` neighbouring tokens: every CTA writes its part
    // of them into that rank's shared memory, four at a time (rows 16 bytes further apart than they are long, so that the lanes' pieces
    // fall into different banks).
    bool ok = take_over(last_chunk);
    if (ok && n_kb > 0) {
      ok = __all_sync(0xffffffffu, mbar_wait(done_bar, 0, abort_flag));
      if (!ok) fail(abort_flag, p.status, ST_TIMEOUT_EPI);
      tc_fence_after();
    }
    if (ranks > 1) cluster_wait();
    const uint32_t to = smem_u32(part) + (uint32_t)((rank * 128 + r) * (p.mine + 4)) * 4;
    for (int c = gr; ok && c < p.n_tok / 16; c += TQ_GROUPS) {
      uint32_t v[16];
#pragma unroll
      for (int x = 0; x < 16; ++x) v[x] = 0u;
      if (n_kb > 0) {
        tmem_ld16(tmem + ((uint32_t)(q * 32) << 16) + (last_chunk & 1) * TQ_ACC1 + c * 16, v);
        tmem_ld_wait();
        if (last_chunk > 0) {
          const float4* at = sums + c * 4 * 128 + r;
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float4 o = at[x * 128];
            v[4 * x] = __float_as_uint(__uint_as_float(v[4 * x]) + o.x); v[4 * x + 1] = __float_as_uint(__uint_as_float(v[4 * x + 1]) + o.y);
            v[4 * x + 2] = __float_as_uint(__uint_as_float(v[4 * x + 2]) + o.z); v[4 * x + 3] = __float_as_uint(__uint_as_float(v[4 * x + 3]) + o.w);
          }
        }
      }
      if (ranks > 1) {
        int owner = c * 16 / p.mine, at = c * 16 - owner * p.mine;       // of the chunk's first token; mine is a multiple of 4
#pragma unroll
        for (int x = 0; x < 16; x += 4) {
          st_cluster_v4(cluster_addr(to + (uint32_t)at * 4, owner), __uint_as_float(v[x]) * TWO_29, __uint_as_float(v[x + 1]) * TWO_29,
                        __uint_as_float(v[x + 2]) * TWO_29, __uint_as_float(v[x + 3]) * TWO_29);
          at += 4;
          if (at == p.mine) { at = 0; ++owner; }
        }
      } else {
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int tok = tok0 + c * 16 + x;
          const float y = __uint_as_float(v[x]) * TWO_29;
          if (tok < p.M && row < sg.N) {
            const size_t o = (size_t)tok * p.ldo + sg.out_off + row;
            if (p.out_f32) p.out_f32[o] = y;
            else p.out_bf16[o] = __float2bfloat16(y);
          }
        }
      }
    }
  }
  if (ranks > 1 && warp < 2) { __syncwarp(); cluster_wait(); }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {                                       // let copies and MMAs still in flight land
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000) {}
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (ranks > 1) {
    cluster_arrive();                                      // all parts are written once everybody has come here
    cluster_wait();
    const int r = threadIdx.x & 127, first = tok0 + rank * p.mine, n = min(p.mine, min(p.M, tok0 + p.n_tok) - first);
    if (threadIdx.x < 384 && row0 + r < sg.N)
      for (int k = (threadIdx.x >> 7) * 4; k < n; k += 12) {
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int x = 0; x < 8; ++x)
          if (x < ranks) {
            const float4 v = *reinterpret_cast<const float4*>(part + (x * 128 + r) * (p.mine + 4) + k);
            y.x += v.x; y.y += v.y; y.z += v.z; y.w += v.w;
          }
        const float ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (k + e < n) {
            const size_t o = (size_t)(first + k + e) * p.ldo + sg.out_off + row0 + r;
            if (p.out_f32) p.out_f32[o] = ys[e];
            else p.out_bf16[o] = __float2bfloat16(ys[e]);
          }
      }
  }
}

}  // namespace

int tc_qlinear(TcState* tc, const QLinArgs& a, int* status, cudaStream_t st) {
  TqParams p;
  const QLinSeg &s0 = a.seg[0], &s1 = a.seg[a.n_seg - 1];
  p.seg0 = TqSeg{s0.codes, s0.scales, s0.N, s0.out_off};
  p.seg1 = TqSeg{s1.codes, s1.scales, s1.N, s1.out_off};
  p.blocks0 = (s0.N + 127) / 128;
  const int blocks = p.blocks0 + (a.n_seg > 1 ? (s1.N + 127) / 128 : 0);
  if (blocks > 65535) return 1;                            // a grid dimension
  p.K128 = (a.K + 127) / 128; p.M = a.M;
  p.n_tok = a.M >= TQ_TOKENS ? TQ_TOKENS : (a.M + 15) / 16 * 16;
  p.out_f32 = a.out_f32; p.out_bf16 = a.out_bf16; p.ldo = a.ldo; p.status = status;
  const int passes = (a.M + TQ_TOKENS - 1) / TQ_TOKENS;
  // the inner dimension over a cluster while that leaves every CTA two blocks and the SMs are not all taken
  int ranks = 1;
  while (ranks < 8 && (long long)blocks * passes * ranks * 2 <= tc->sm_count && p.K128 >= ranks * 4) ranks *= 2;
  p.mine = ((p.n_tok + ranks - 1) / ranks + 3) / 4 * 4;
  p.per_cta = (p.K128 + ranks - 1) / ranks;
  CUtensorMap maps[2];
  for (int s = 0; s < a.n_seg; ++s)
    if (!tc_make_map_2d(tc, &maps[s], a.seg[s].X, (uint64_t)a.K, (uint64_t)a.M, (uint64_t)a.K, 64, (uint32_t)p.n_tok)) return 1;
  if (a.n_seg == 1) maps[1] = maps[0];
  static bool done[TC_MAX_DEVICES];
  if (!done[tc->device]) {
    const cudaError_t e = cudaFuncSetAttribute(tc_qlinear_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, TQ_SMEM);
    if (e != cudaSuccess) return -(int)e;
    done[tc->device] = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ranks, (unsigned)blocks, (unsigned)passes);
  cfg.blockDim = dim3(TQ_THREADS);
  cfg.dynamicSmemBytes = TQ_SMEM;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)ranks; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, tc_qlinear_kernel, maps[0], maps[1], p);
  return e == cudaSuccess ? 0 : -(int)e;
}
