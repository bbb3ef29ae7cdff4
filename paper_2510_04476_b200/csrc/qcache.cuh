// Cache in 4 bits: host-side launcher interface.  Return values: 0 = enqueued, 1 = shape not covered, < 0 = minus a cudaError_t;
// *launches is advanced by the kernels enqueued.
#pragma once
#include "common.cuh"

struct QCache {
  uint8_t *k_codes, *v_codes;     // [B, hk, S_max, dh / 2]
  bf16 *k_scales, *v_scales;      // [B, hk, S_max, dh / 32]
  float* weight;                  // [B, hk, S_max] or null
  int* position;                  // [B, hk, S_max] or null
  int* len;                       // [B]
  long long S_max;
};

constexpr int ST_QCACHE_BAD_LEN = 121;   // a sequence's rows do not fit its cache

// n new rows a sequence, behind its len[b] rows, up to `limit` rows in all.
int launch_qcache_append(const CcaDims& d, const bf16* k, const bf16* v, const int* position, const int* count, const QCache& c,
                         long long n, long long limit, int* status, long long* launches, cudaStream_t st);
int launch_qcache_read(const CcaDims& d, const QCache& c, const int* first, float* k, float* v, long long n, long long* launches,
                       cudaStream_t st);
// Workspace of one attention or eviction call over at most max_len rows (the larger of the two).
size_t qcache_workspace_bytes(const CcaDims& d, int max_len, int sm_count);
// Rows 0 .. len[b] + extra - 1; pos (may be null): a sequence whose entry is negative is skipped.  q: bf16 or, where q32 is set, fp32 rounded to bf16 on the way in.
int launch_qcache_attention(const CcaDims& d, const bf16* q, const float* q32, bf16* o, const QCache& c, const int* pos, int extra,
                            int max_len, int accumulate, void* workspace, int sm_count, int* status, long long* launches,
                            cudaEvent_t ev_begin, cudaEvent_t ev_end, cudaStream_t st);
// tag: a number below 2^48, not 0, that no memory is expected to hold by chance, another one for every call.
int launch_qcache_evict(const CcaDims& d, const QCache& c, int keep, int recent, const int* next_position, int max_len,
                        void* workspace, unsigned long long tag, int sm_count, int* status, long long* launches,
                        cudaStream_t st);
