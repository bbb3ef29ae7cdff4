// y = x W^T for a few tokens, W in the 4-bit format of qformat.cuh.  Bound by reading W at few tokens.
#include "pdl.cuh"
#include "qformat.cuh"
#include "qlinear.cuh"
#include "tc_state.cuh"

namespace {

using namespace q4;
constexpr int QL_WARPS = 8;

struct PackArgs {
  const bf16* w;
  uint8_t* codes;
  bf16* scales;
  int N, K, n16, k128;
};

// Eight neighbouring lanes take one block of 128 columns of one row; four rows of a warp are neighbours in the tile.
__global__ void __launch_bounds__(256) qlinear_pack_kernel(PackArgs a) {
  const int lane8 = threadIdx.x & 7;
  const long long units = (long long)a.n16 * a.k128 * 16;          // (row tile, column tile, row)
  for (long long u0 = (long long)blockIdx.x * 32 + (threadIdx.x >> 5) * 4; u0 < units; u0 += (long long)gridDim.x * 32) {
    const long long u = u0 + ((threadIdx.x & 31) >> 3);            // units is a multiple of 16: every lane has one
    const int r = (int)(u & 15);
    const long long tile = u >> 4;
    const int kb = (int)(tile % a.k128);
    const long long row = tile / a.k128 * 16 + r;
    uint32_t code[2], scale[2];
    quantise_block<4>([&](int grp) {
      const int col = kb * 128 + grp * GROUP;
      return row < a.N && col < a.K ? __ldcs(reinterpret_cast<const uint2*>(a.w + (size_t)row * a.K + col + lane8 * 4)) : make_uint2(0, 0);
    }, code, scale);
    *reinterpret_cast<uint2*>(a.codes + (size_t)u * 64 + lane8 * 8) = make_uint2(code[0], code[1]);
    if (lane8 == 0) *reinterpret_cast<uint2*>(a.scales + (size_t)u * 4) = make_uint2(scale[0], scale[1]);
  }
}

// 16 weight rows per CTA, 8 NT tokens, the inner dimension split over the 8 warps and summed through shared memory in a fixed
// order.  A lane's 16 bytes of a weight row are 8 channels of each of 4 groups: two instructions per group, whose sum is multiplied
// by the group's scale in fp32.  The codes are exact operands, so the only roundings are fp32's.  A group's sum comes out times 2^-69, which
// its scale takes off before the groups are added: sums of small weights would fall below the smallest normal number.
// At few tokens it is bound by the 204 instructions that a block of 16 rows by 128 columns takes, and what hides their latency is
// warps: four CTAs per SM with one block of each warp on its way take 18.7 us for 5 x 16383 x 8192 (75 MB: 64 % of the measured copy
// rate), three with two or three 20.1 to 21.2, two with four 21.1; rings of asynchronous copies under CTAs that stay (16 or 32 warps, x in
// registers or in shared memory, one row tile or two) 22.6 to 24.3.
template <int NT>
__global__ void __launch_bounds__(QL_WARPS * 32, NT == 1 ? 4 : 1) qlinear_kernel(QLinArgs a) {
  pdl_enter();
  __shared__ float red[QL_WARPS][16][NT * 8 + 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int tok0 = blockIdx.y * (NT * 8);
  const int k128 = (a.K + 127) / 128;
  int tile = blockIdx.x;
  QLinSeg sg = a.seg[0];
  if (a.n_seg > 1) {
    const int t0 = (a.seg[0].N + 15) / 16;
    if (tile >= t0) { sg = a.seg[1]; tile -= t0; }
  }
  const uint8_t* codes = sg.codes + (size_t)tile * k128 * 1024 + lane * 16;
  const bf16* scales = sg.scales + (size_t)tile * k128 * 64 + g * 4;
  bool ok_tok[NT];
  const bf16* xp[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int tok = tok0 + nt * 8 + g;
    ok_tok[nt] = tok < a.M;
    xp[nt] = sg.X + (size_t)(ok_tok[nt] ? tok : 0) * a.K + t * 8;
  }
  float acc[NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[nt][c] = 0.f;
  for (int kb = warp; kb < k128; kb += QL_WARPS) {
    uint32_t wl[4], wh[4], sl[2], sh[2];
    load_words<4>(wl, codes + (size_t)kb * 1024);
    load_words<4>(wh, codes + (size_t)kb * 1024 + 512);
    load_words<2>(sl, scales + (size_t)kb * 64);
    load_words<2>(sh, scales + (size_t)kb * 64 + 32);
#pragma unroll
    for (int i = 0; i < 2; ++i) { sl[i] = mul_bf16x2(sl[i], MUL_69); sh[i] = mul_bf16x2(sh[i], MUL_69); }
#pragma unroll
    for (int gi = 0; gi < 4; ++gi) {
      const int col = kb * 128 + gi * GROUP;
      uint32_t ka[2][4];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int byte = c * 8 + gi * 2;
        const uint32_t sel = (byte & 2) ? 0x3322u : 0x1100u;
        const uint32_t p0 = __byte_perm(wl[byte / 4], 0, sel), p1 = __byte_perm(wh[byte / 4], 0, sel);
        ka[c][0] = code_e0(p0); ka[c][1] = code_e0(p1); ka[c][2] = code_e1(p0); ka[c][3] = code_e1(p1);
      }
      const float s_lo = scale_at(sl, gi), s_hi = scale_at(sh, gi);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        uint4 xv = make_uint4(0, 0, 0, 0);
        if (ok_tok[nt] && col < a.K) xv = __ldg(reinterpret_cast<const uint4*>(xp[nt] + col));
        float part[4];
        mma_16816_zero(part, ka[0], mul_bf16x2(xv.x, MUL_E0), mul_bf16x2(xv.y, MUL_E1));
        mma_16816(part, ka[1], mul_bf16x2(xv.z, MUL_E0), mul_bf16x2(xv.w, MUL_E1));
        acc[nt][0] = fmaf(s_lo, part[0], acc[nt][0]); acc[nt][1] = fmaf(s_lo, part[1], acc[nt][1]);
        acc[nt][2] = fmaf(s_hi, part[2], acc[nt][2]); acc[nt][3] = fmaf(s_hi, part[3], acc[nt][3]);
      }
    }
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int c = 0; c < 4; ++c) red[warp][g + 8 * (c >> 1)][nt * 8 + 2 * t + (c & 1)] = acc[nt][c];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * NT * 8; i += QL_WARPS * 32) {
    const int row = i % 16, tok = i / 16;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < QL_WARPS; ++w) v += red[w][row][tok];
    const int r = tile * 16 + row;
    if (r < sg.N && tok0 + tok < a.M) {
      const size_t o = (size_t)(tok0 + tok) * a.ldo + sg.out_off + r;
      if (a.out_f32) a.out_f32[o] = v;
      else a.out_bf16[o] = __float2bfloat16(v);
    }
  }
}

int row_tiles(const QLinArgs& a) {
  int tiles = 0;
  for (int s = 0; s < a.n_seg; ++s) tiles += (a.seg[s].N + 15) / 16;
  return tiles;
}
template <int NT>
cudaError_t run_nt(const QLinArgs& a, cudaStream_t st) {
  return launch_pdl(qlinear_kernel<NT>, dim3((unsigned)row_tiles(a), (unsigned)((a.M + NT * 8 - 1) / (NT * 8))), dim3(QL_WARPS * 32), st, a);
}

// Whether more than 8 tokens go to the tcgen05 kernel.  The kernel here takes 32 of them at a time, one CTA an SM, in 1 us and 1 more for
// every 1024 columns a wave of CTAs; the other one takes 4 to 9 us however small the matrix is.  They cross at two waves or 4096
// columns in all.  us, this one | tcgen05, at 9, 32 and 64 tokens:
//   1000 x 1024   2.2  2.9  2.7 |  4.9  5.5  6.3        4096 x 2048    5.9  7.4 13.2 |  6.4  7.0  9.1
//   4096 x 1024   4.1  4.9  8.7 |  5.1  5.6  7.7        8192 x 1024    6.8  8.5 15.0 |  6.2  6.8  8.0
//   2368 x 2048   3.4  4.6  7.7 |  6.1  6.7  8.7         960 x 8192    8.5 10.4      |  8.2  8.9
//   1536 x 4096   5.3  6.5 11.4 |  6.7  7.1  9.0        4096 x 4096   11.2 13.1 23.0 |  8.8  9.6 11.8
//   2368 x 4096   5.4  6.8 12.5 |  8.0  8.8 11.2       16383 x 8192   64.2 74.3  136 | 29.2 31.0 36.5
bool tcgen05_pays(const QLinArgs& a, int sm_count) {
  const long long ctas = (long long)row_tiles(a) * ((a.M + 31) / 32), waves = (ctas + sm_count - 1) / sm_count;
  return waves > 2 || waves * a.K > 4096;
}

}  // namespace

size_t qlinear_code_bytes(long long N, long long K) { return (size_t)((N + 15) / 16) * ((K + 127) / 128) * 1024; }
size_t qlinear_scale_bytes(long long N, long long K) { return (size_t)((N + 15) / 16) * ((K + 127) / 128) * 128; }

int launch_qlinear_pack(const bf16* w, uint8_t* codes, bf16* scales, int N, int K, long long* launches, cudaStream_t st) {
  PackArgs a{w, codes, scales, N, K, (N + 15) / 16, (K + 127) / 128};
  const long long ctas = ((long long)a.n16 * a.k128 * 16 + 31) / 32;
  qlinear_pack_kernel<<<(unsigned)(ctas < 4736 ? ctas : 4736), 256, 0, st>>>(a);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  return 0;
}

int launch_qlinear(const QLinArgs& a, TcState* tc, int* status, long long* launches, cudaStream_t st) {
  // 8 tokens cost here what 1 costs (on a tall matrix two passes of 8 take longer than the tcgen05 kernel: 16 x 16383 x 8192 38.0 us against
  // 29.3), unless the handle has the tensor-core kernels switched off
  if (tc && a.M > 8 && tcgen05_pays(a, tc->sm_count)) {
    const int r = tc_qlinear(tc, a, status, st);
    if (r < 0) return r;
    if (r == 0) { ++*launches; return 0; }
  }
  const cudaError_t e = a.M <= 8 ? run_nt<1>(a, st) : run_nt<4>(a, st);
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  return 0;
}
