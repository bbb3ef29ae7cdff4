// y = x W^T for up to 64 tokens at a time on the tensor cores of this architecture, W in the 4-bit format of qformat.cuh.
//
//   warp 0       : TMA producer (one lane)            -- x tiles, up to 64 tokens x 128 channels, 4 stages
//   warp 1       : TMEM owner + MMA issuer (one lane) -- 128 weight rows x tokens x 16 channels per instruction
//   warps 2..13  : three groups of four, a thread per weight row: a block of 128 channels from its 64 bytes of codes into tensor
//                  memory, as the MMA's A operand; the groups take the blocks in turn
//
// A weight c * s has up to 11 significant bits, which one bf16 operand cannot hold.  It becomes two: hi = bf16(c * s) by
// a product and lo = c * s - hi by one fused multiply-add, both exact, so that the only roundings are the accumulator's.  (One operand alone would
// add an error of 2^-9 of each weight; the matrix unit has the time for two: at 64 tokens its work is 0.6 of the dequantisation's.)
// Bound by the integer and half-precision instructions of the dequantisation, 2 a code, which come close to the time of reading the
// codes.  The inner dimension is split over the CTAs of a cluster where there are fewer row blocks than SMs; their sums
// are added in rank order through distributed shared memory.
#include "pdl.cuh"
#include "qformat.cuh"
#include "qlinear.cuh"
#include "tc_ptx.cuh"
#include "tc_state.cuh"

using namespace tc;
using namespace q4;

namespace {

constexpr int TQ_GROUPS = 3, TQ_WARPS = 2 + 4 * TQ_GROUPS, TQ_THREADS = 32 * TQ_WARPS;
constexpr int TQ_STAGES = 4, TQ_TOKENS = 64;
constexpr int TQ_STAGE_BYTES = TQ_TOKENS * 256;
constexpr int TQ_SMEM = TQ_STAGES * TQ_STAGE_BYTES + 256 + 1024;      // barriers, slack for the 1024-byte alignment
constexpr int TQ_A_COL = 64;                                          // accumulator columns, then the groups' operands
constexpr uint32_t MUL_96 = 0x6f806f80u, MUL_92 = 0x6d806d80u;        // bf16x2 2^96, 2^92: operands become c s 2^-37
constexpr float TWO_37 = 137438953472.f;

struct TqParams {
  const uint8_t* codes[2];
  const bf16* scales[2];
  int N[2], out_off[2];
  int blocks0;               // row blocks of the first segment
  int K128, M, n_tok;        // n_tok: tokens of a pass, a multiple of 16
  int per_cta;               // channel blocks of a CTA
  float* out_f32;
  bf16* out_bf16;
  int ldo;
  int* status;
};

TC_DEVINL void fail(volatile int* abort_flag, int* status, int code) {
  *abort_flag = 1;
  atomicCAS(status, 0, code);
}
CCA_DEVINL uint32_t rest_bf16x2(uint32_t a, uint32_t b, uint32_t ab) {          // a * b - ab
  uint32_t r;
  asm("{\n\t.reg .b32 t;\n\tneg.bf16x2 t, %3;\n\tfma.rn.bf16x2 %0, %1, %2, t;\n\t}" : "=r"(r) : "r"(a), "r"(b), "r"(ab));
  return r;
}
CCA_DEVINL float ld_cluster_f32(uint32_t addr, uint32_t rank) {
  uint32_t remote;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(remote) : "memory");
  return v;
}
CCA_DEVINL void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__global__ void __launch_bounds__(TQ_THREADS, 1)
tc_qlinear_kernel(const __grid_constant__ CUtensorMap tm0, const __grid_constant__ CUtensorMap tm1, TqParams p) {
  pdl_enter();
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* smem = smem_align1024(smem_dyn);
  uint64_t* b_full = reinterpret_cast<uint64_t*>(smem + TQ_STAGES * TQ_STAGE_BYTES);
  uint64_t* b_empty = b_full + TQ_STAGES;
  uint64_t* a_full = b_empty + TQ_STAGES;
  uint64_t* a_empty = a_full + TQ_GROUPS;
  uint64_t* done_bar = a_empty + TQ_GROUPS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done_bar + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x, ranks = gridDim.x;
  const int seg = (int)blockIdx.y >= p.blocks0 ? 1 : 0;
  const int row0 = ((int)blockIdx.y - (seg ? p.blocks0 : 0)) * 128, tok0 = (int)blockIdx.z * TQ_TOKENS;
  const int kb_begin = rank * p.per_cta, n_kb = max(0, min(p.K128, kb_begin + p.per_cta) - kb_begin);

  if (threadIdx.x == 0) {
    for (int s = 0; s < TQ_STAGES; ++s) { mbar_init(&b_full[s], 1); mbar_init(&b_empty[s], 1); }
    for (int s = 0; s < TQ_GROUPS; ++s) { mbar_init(&a_full[s], 4); mbar_init(&a_empty[s], 1); }
    mbar_init(done_bar, 1);
    wait_ctl_init(abort_flag, p.status);
    fence_barrier_init();
    prefetch_tmap(seg ? &tm1 : &tm0);
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int sub = p.n_tok * 128;                           // bytes of a 64-channel half of an x tile

  if (warp == 0) {
    if (lane == 0) {
      for (int i = 0; i < n_kb; ++i) {
        const int st = i % TQ_STAGES;
        if (!mbar_wait(&b_empty[st], ((i / TQ_STAGES) & 1) ^ 1, abort_flag)) { fail(abort_flag, p.status, ST_TIMEOUT_TMA); break; }
        unsigned char* dst = smem + st * TQ_STAGE_BYTES;
        mbar_expect_tx(&b_full[st], 2 * sub);
        tma_load_2d(dst, seg ? &tm1 : &tm0, (kb_begin + i) * 128, tok0, &b_full[st]);
        tma_load_2d(dst + sub, seg ? &tm1 : &tm0, (kb_begin + i) * 128 + 64, tok0, &b_full[st]);
      }
    }
  } else if (warp == 1) {
    const bool leader = elect_one();
    const uint32_t idesc = idesc_bf16(p.n_tok, 0, 0);
    const uint32_t desc_hi = (uint32_t)(smem_desc_sw128(0, 0, 1024) >> 32);
    const uint32_t smem_lo = smem_u32(smem) >> 4;
    bool ok = true;
    for (int i = 0; i < n_kb; ++i) {
      const int st = i % TQ_STAGES, gr = i % TQ_GROUPS;
      ok = __all_sync(0xffffffffu, mbar_wait(&b_full[st], (i / TQ_STAGES) & 1, abort_flag)) &&
           __all_sync(0xffffffffu, mbar_wait(&a_full[gr], (i / TQ_GROUPS) & 1, abort_flag));
      if (!ok) { fail(abort_flag, p.status, ST_TIMEOUT_MMA); break; }
      tc_fence_after();
      const uint32_t a = tmem + TQ_A_COL + gr * 128;
      const uint32_t b = (smem_lo + st * (TQ_STAGE_BYTES >> 4)) | (1u << 16);
      if (leader) {
#pragma unroll
        for (int part = 0; part < 2; ++part)               // hi, lo
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
            mma_ts_w(tmem, a + part * 64 + ks * 8, b + (ks >> 2) * (sub >> 4) + (ks & 3) * 2, desc_hi, idesc, (i | part | ks) != 0);
        mma_commit(&a_empty[gr]);
        mma_commit(&b_empty[st]);
        if (i == n_kb - 1) mma_commit(done_bar);
      }
    }
  } else {
    const int gr = (warp - 2) >> 2, q = warp & 3;
    const int row = row0 + q * 32 + lane;
    const bool there = row < (p.N[seg] + 15) / 16 * 16;    // rows that the tiles hold
    const size_t tile = (size_t)(row >> 4) * p.K128 + kb_begin;
    const uint4* codes = reinterpret_cast<const uint4*>(p.codes[seg] + (tile * 16 + (row & 15)) * 64);
    const uint2* scales = reinterpret_cast<const uint2*>(p.scales[seg] + (tile * 16 + (row & 15)) * 4);
    const uint32_t a = tmem + ((uint32_t)(q * 32) << 16) + TQ_A_COL + gr * 128;
    uint32_t w[16], nw[16];
    uint2 sc = make_uint2(0, 0), nsc = make_uint2(0, 0);
    auto load = [&](int i) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const uint4 u = there ? __ldg(codes + (size_t)i * 64 + x) : make_uint4(0, 0, 0, 0);
        nw[4 * x] = u.x; nw[4 * x + 1] = u.y; nw[4 * x + 2] = u.z; nw[4 * x + 3] = u.w;
      }
      nsc = there ? __ldg(scales + (size_t)i * 16) : make_uint2(0, 0);
    };
    if (gr < n_kb) load(gr);
    for (int i = gr, turn = 0; i < n_kb; i += TQ_GROUPS, ++turn) {
#pragma unroll
      for (int x = 0; x < 16; ++x) w[x] = nw[x];
      sc = nsc;
      if (i + TQ_GROUPS < n_kb) load(i + TQ_GROUPS);
      if (!mbar_wait(&a_empty[gr], (turn & 1) ^ 1, abort_flag)) { fail(abort_flag, p.status, ST_TIMEOUT_EPI); break; }
      tc_fence_after();
#pragma unroll
      for (int grp = 0; grp < 4; ++grp) {
        const uint32_t s2 = __byte_perm(grp < 2 ? sc.x : sc.y, 0, (grp & 1) ? 0x3232u : 0x1010u);
        const uint32_t m0 = mul_bf16x2(s2, MUL_96), m1 = mul_bf16x2(s2, MUL_92);
        uint32_t hi[16], lo[16];
#pragma unroll
        for (int g = 0; g < 8; ++g) {
          const uint32_t pr = __byte_perm(w[g * 2 + (grp >> 1)], 0, (grp & 1) ? 0x3322u : 0x1100u);
          const uint32_t e0 = code_e0(pr), e1 = code_e1(pr);
          hi[2 * g] = mul_bf16x2(e0, m0); hi[2 * g + 1] = mul_bf16x2(e1, m1);
          lo[2 * g] = rest_bf16x2(e0, m0, hi[2 * g]); lo[2 * g + 1] = rest_bf16x2(e1, m1, hi[2 * g + 1]);
        }
        tmem_st16(a + grp * 16, hi);
        tmem_st16(a + 64 + grp * 16, lo);
      }
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&a_full[gr]);
    }
    // ---- sums: thread = row, one column per token
    if (gr == 0) {
      bool ok = true;
      if (n_kb > 0) {
        ok = __all_sync(0xffffffffu, mbar_wait(done_bar, 0, abort_flag));
        if (!ok) fail(abort_flag, p.status, ST_TIMEOUT_EPI);
        tc_fence_after();
      }
      float* part = reinterpret_cast<float*>(smem);        // [tokens][128] where a cluster joins its sums; the x stages are done with
      const int r = q * 32 + lane;
      for (int c = 0; ok && c < p.n_tok / 16; ++c) {
        uint32_t v[16];
#pragma unroll
        for (int x = 0; x < 16; ++x) v[x] = 0u;
        if (n_kb > 0) {
          tmem_ld16(tmem + ((uint32_t)(q * 32) << 16) + c * 16, v);
          tmem_ld_wait();
        }
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int tok = c * 16 + x;
          const float y = __uint_as_float(v[x]) * TWO_37;
          if (ranks > 1) {
            part[tok * 128 + r] = y;
          } else if (tok0 + tok < p.M && row < p.N[seg]) {
            const size_t o = (size_t)(tok0 + tok) * p.ldo + p.out_off[seg] + row;
            if (p.out_f32) p.out_f32[o] = y;
            else p.out_bf16[o] = __float2bfloat16(y);
          }
        }
      }
    }
  }
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
    cluster_sync();
    const uint32_t part = smem_u32(smem);
    const int n = min(p.n_tok, p.M - tok0);
    for (int i = threadIdx.x; i < n * 128; i += TQ_THREADS) {
      const int tok = i >> 7, r = i & 127;
      if (tok % ranks != rank || row0 + r >= p.N[seg]) continue;
      float y = 0.f;
      for (int x = 0; x < ranks; ++x) y += ld_cluster_f32(part + (uint32_t)(tok * 128 + r) * 4, x);
      const size_t o = (size_t)(tok0 + tok) * p.ldo + p.out_off[seg] + row0 + r;
      if (p.out_f32) p.out_f32[o] = y;
      else p.out_bf16[o] = __float2bfloat16(y);
    }
    cluster_sync();                                        // nobody leaves while its sums may still be read
  }
}

}  // namespace

int tc_qlinear(TcState* tc, const QLinArgs& a, int* status, cudaStream_t st) {
  TqParams p;
  p.blocks0 = 0;
  int blocks = 0;
  for (int s = 0; s < 2; ++s) {
    const QLinSeg& sg = a.seg[s < a.n_seg ? s : 0];
    p.codes[s] = sg.codes; p.scales[s] = sg.scales; p.N[s] = sg.N; p.out_off[s] = sg.out_off;
    if (s < a.n_seg) blocks += (sg.N + 127) / 128;
    if (s == 0) p.blocks0 = blocks;
  }
  p.K128 = (a.K + 127) / 128; p.M = a.M;
  p.n_tok = a.M >= TQ_TOKENS ? TQ_TOKENS : (a.M + 15) / 16 * 16;
  p.out_f32 = a.out_f32; p.out_bf16 = a.out_bf16; p.ldo = a.ldo; p.status = status;
  const int passes = (a.M + TQ_TOKENS - 1) / TQ_TOKENS;
  // the inner dimension over a cluster while that leaves every CTA two blocks and the SMs are not all taken
  int ranks = 1;
  while (ranks < 8 && (long long)blocks * passes * ranks * 2 <= tc->sm_count && p.K128 >= ranks * 4) ranks *= 2;
  p.per_cta = (p.K128 + ranks - 1) / ranks;
  CUtensorMap maps[2];
  for (int s = 0; s < 2; ++s)
    if (!tc_make_map_2d(tc, &maps[s], a.seg[s < a.n_seg ? s : 0].X, (uint64_t)a.K, (uint64_t)a.M, (uint64_t)a.K, 64, (uint32_t)p.n_tok)) return 1;
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
