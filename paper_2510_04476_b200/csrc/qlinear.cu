// y = x W^T for a few tokens, W in the 4-bit format of qformat.cuh.  Bound by reading W at few tokens.
#include "pdl.cuh"
#include "qformat.cuh"
#include "qlinear.cuh"

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
    uint8_t code[8];
    bf16 scale[4];
    quantise_block<4>([&](int grp) {
      const int col = kb * 128 + grp * GROUP;
      return row < a.N && col < a.K ? __ldcs(reinterpret_cast<const uint2*>(a.w + (size_t)row * a.K + col + lane8 * 4)) : make_uint2(0, 0);
    }, code, scale);
    uint2 w;
    w.x = code[0] | (code[1] << 8) | (code[2] << 16) | ((uint32_t)code[3] << 24);
    w.y = code[4] | (code[5] << 8) | (code[6] << 16) | ((uint32_t)code[7] << 24);
    *reinterpret_cast<uint2*>(a.codes + (size_t)u * 64 + lane8 * 8) = w;
#pragma unroll
    for (int grp = 0; grp < 4; ++grp)
      if (lane8 == grp) a.scales[(size_t)u * 4 + grp] = scale[grp];
  }
}

// 16 MT weight rows per CTA, 8 NT tokens, the inner dimension split over the 8 warps and summed through shared memory in a fixed
// order.  A lane's 16 bytes of a weight row are 8 channels of each of 4 groups: two instructions per group, whose sum is multiplied
// by the group's scale in fp32.  The codes are exact operands, so the only roundings are fp32's.
template <int NT, int MT>
__global__ void __launch_bounds__(QL_WARPS * 32) qlinear_kernel(QLinArgs a) {
  pdl_enter();
  constexpr int UNR = MT == 1 ? 4 : 2;                     // blocks of 128 columns on their way at a time
  __shared__ float red[QL_WARPS][16 * MT][NT * 8 + 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int tok0 = blockIdx.y * (NT * 8);
  const int k128 = (a.K + 127) / 128;
  int tile = blockIdx.x * MT;
  QLinSeg sg = a.seg[0];
  if (a.n_seg > 1) {                                       // a CTA's tiles are of one segment: their number is rounded up to MT
    const int t0 = ((a.seg[0].N + 15) / 16 + MT - 1) / MT * MT;
    if (tile >= t0) { sg = a.seg[1]; tile -= t0; }
  }
  const int n16 = (sg.N + 15) / 16;
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
  float acc[MT][NT][4];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[mt][nt][c] = 0.f;
  for (int kb0 = warp; kb0 < k128; kb0 += QL_WARPS * UNR) {
    uint32_t wl[UNR][MT][4], wh[UNR][MT][4], sl[UNR][MT][2], sh[UNR][MT][2];
#pragma unroll
    for (int u = 0; u < UNR; ++u) {
      const int kb = kb0 + u * QL_WARPS;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        zero_words(wl[u][mt]); zero_words(wh[u][mt]); zero_words(sl[u][mt]); zero_words(sh[u][mt]);
        if (kb < k128 && (MT == 1 || tile + mt < n16)) {
          const size_t at = (size_t)mt * k128 + kb;
          load_words<4>(wl[u][mt], codes + at * 1024);
          load_words<4>(wh[u][mt], codes + at * 1024 + 512);
          load_words<2>(sl[u][mt], scales + at * 64);
          load_words<2>(sh[u][mt], scales + at * 64 + 32);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < UNR; ++u) {
      const int kb = kb0 + u * QL_WARPS;
      if (kb >= k128) break;
#pragma unroll
      for (int gi = 0; gi < 4; ++gi) {
        const int col = kb * 128 + gi * GROUP;
        uint32_t ka[MT][2][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int byte = c * 8 + gi * 2;
            const uint32_t sel = (byte & 2) ? 0x3322u : 0x1100u;
            const uint32_t p0 = __byte_perm(wl[u][mt][byte / 4], 0, sel), p1 = __byte_perm(wh[u][mt][byte / 4], 0, sel);
            ka[mt][c][0] = code_e0(p0); ka[mt][c][1] = code_e0(p1); ka[mt][c][2] = code_e1(p0); ka[mt][c][3] = code_e1(p1);
          }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          uint4 xv = make_uint4(0, 0, 0, 0);
          if (ok_tok[nt] && col < a.K) xv = __ldg(reinterpret_cast<const uint4*>(xp[nt] + col));
          xv.x = mul_bf16x2(xv.x, MUL_E0); xv.y = mul_bf16x2(xv.y, MUL_E1);
          xv.z = mul_bf16x2(xv.z, MUL_E0); xv.w = mul_bf16x2(xv.w, MUL_E1);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            float part[4];
            mma_16816_zero(part, ka[mt][0], xv.x, xv.y);
            mma_16816(part, ka[mt][1], xv.z, xv.w);
            const float s_lo = scale_at(sl[u][mt], gi), s_hi = scale_at(sh[u][mt], gi);
            float (&ac)[4] = acc[mt][nt];
            ac[0] = fmaf(s_lo, part[0], ac[0]); ac[1] = fmaf(s_lo, part[1], ac[1]);
            ac[2] = fmaf(s_hi, part[2], ac[2]); ac[3] = fmaf(s_hi, part[3], ac[3]);
          }
        }
      }
    }
  }
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 4; ++c) red[warp][mt * 16 + g + 8 * (c >> 1)][nt * 8 + 2 * t + (c & 1)] = acc[mt][nt][c];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * MT * NT * 8; i += QL_WARPS * 32) {
    const int row = i % (16 * MT), tok = i / (16 * MT);
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < QL_WARPS; ++w) v += red[w][row][tok];
    v *= TWO_69;
    const int r = tile * 16 + row;
    if (r < sg.N && tok0 + tok < a.M) {
      const size_t o = (size_t)(tok0 + tok) * a.ldo + sg.out_off + r;
      if (a.out_f32) a.out_f32[o] = v;
      else a.out_bf16[o] = __float2bfloat16(v);
    }
  }
}

template <int NT, int MT>
cudaError_t run_nt(const QLinArgs& a, cudaStream_t st) {
  int ctas = 0;
  for (int s = 0; s < a.n_seg; ++s) ctas += ((a.seg[s].N + 15) / 16 + MT - 1) / MT;
  return launch_pdl(qlinear_kernel<NT, MT>, dim3((unsigned)ctas, (unsigned)((a.M + NT * 8 - 1) / (NT * 8))), dim3(QL_WARPS * 32), st, a);
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

int launch_qlinear(const QLinArgs& a, TcState* tc, int sm_count, int* status, long long* launches, cudaStream_t st) {
  if (tc && a.M > 8) {
    const int r = tc_qlinear(tc, a, status, st);
    if (r < 0) return r;
    if (r == 0) { ++*launches; return 0; }
  }
  int tiles = 0;
  for (int s = 0; s < a.n_seg; ++s) tiles += (a.seg[s].N + 15) / 16;
  cudaError_t e;
  if (a.M <= 8) e = tiles >= 4 * sm_count ? run_nt<1, 2>(a, st) : run_nt<1, 1>(a, st);
  else if (a.M <= 16) e = run_nt<2, 1>(a, st);
  else if (a.M <= 32) e = run_nt<4, 1>(a, st);
  else e = run_nt<8, 1>(a, st);
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  return 0;
}
