// Products with 4-bit weights: host-side launcher interface.  Return values as in qcache.cuh.
#pragma once
#include "tc_kernels.cuh"

// One weight matrix [N, K] in tiles of 16 rows by 128 columns, rows and columns padded with zeros: codes [N16][K128][16][64] bytes,
// scales [N16][K128][16][4] bf16, a tile's row being a block of the format.
struct QLinSeg {
  const uint8_t* codes;
  const bf16* scales;
  const bf16* X;       // [M, K]
  int N;
  int out_off;         // first output column
};
struct QLinArgs {
  QLinSeg seg[2];
  int n_seg, K, M;
  float* out_f32;      // [M, ldo], one of the two
  bf16* out_bf16;
  int ldo;
};

size_t qlinear_code_bytes(long long N, long long K);
size_t qlinear_scale_bytes(long long N, long long K);
int launch_qlinear_pack(const bf16* w, uint8_t* codes, bf16* scales, int N, int K, long long* launches, cudaStream_t st);
// tc: the handle's tensor-map state, or null (then only the warp-level kernel is used)
int launch_qlinear(const QLinArgs& a, TcState* tc, int* status, long long* launches, cudaStream_t st);
int tc_qlinear(TcState* tc, const QLinArgs& a, int* status, cudaStream_t st);     // tc_qlinear.cu
