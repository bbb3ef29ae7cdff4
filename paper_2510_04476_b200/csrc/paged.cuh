// Cache in pages: host-side launcher interface and what the kernels on it share.  Return values: 0 = enqueued, 1 = shape not covered,
// < 0 = minus a cudaError_t; *launches is advanced by the kernels enqueued.
#pragma once
#include "common.cuh"

struct Paged {
  bf16 *k, *v;                    // [n_pages, hk, P, dh]
  int* refs;                      // [n_pages]: sequences that hold the page
  int* table;                     // [B, max_pages]
  int* len;                       // [B]
  int n_pages, P, max_pages;
  unsigned long long inv_P;       // ceil(2^40 / P): a row below 2^24 divided by P <= 2^16 is (row * inv_P) >> 40
};

constexpr int ST_PAGE_MISSING = 122;     // a row without a page of its sequence's own, or an index outside its range
constexpr int ST_PAGES_SHORT = 123;      // more pages asked for than are free

#ifdef __CUDACC__
CCA_DEVINL int page_index(const Paged& c, int row) { return (int)(((unsigned long long)(unsigned)row * c.inv_P) >> 40); }
// Entry i of sequence b; -1 where it names no page of the pool.
CCA_DEVINL int page_at(const Paged& c, int b, int i) {
  const int e = c.table[(size_t)b * c.max_pages + i];
  return (unsigned)e < (unsigned)c.n_pages ? e : -1;
}
// Row `place` of kv head j in a page, counted over the whole pool (n_pages * hk * P < 2^31).
CCA_DEVINL int pool_row(const Paged& c, int hk, int page, int j, int place) { return (page * hk + j) * c.P + place; }
#endif

// n new rows a sequence, behind its len[b] rows.
int launch_paged_append(const CcaDims& d, const bf16* k, const bf16* v, const int* count, const Paged& c, long long n, int* status,
                        long long* launches, cudaStream_t st);
int launch_paged_read(const CcaDims& d, const Paged& c, const int* first, bf16* k, bf16* v, long long n, long long* launches,
                      cudaStream_t st);
// What a decode step needs of the tokens before it besides keys and values, from a forward's input x [B, S, E] and saved q0|k0 latent [B, S, L]: the last
// input and the last `pad` latent rows (zeros before the first), of the sequences that are in use.
int launch_paged_token_state(const CcaDims& d, const Paged& c, const bf16* x, const float* qk0, bf16* x_prev, float* hist, long long* launches,
                             cudaStream_t st);
size_t paged_workspace_bytes(const CcaDims& d, int max_len, int sm_count);
// Rows 0 .. len[b] + extra - 1.  q: bf16 or, where q32 is set, fp32 rounded to bf16 on the way in.  lse may be null.
int launch_paged_attention(const CcaDims& d, const bf16* q, const float* q32, bf16* o, float* lse, const Paged& c, int extra, int max_len,
                           void* workspace, int sm_count, int* status, long long* launches, cudaEvent_t ev_begin, cudaEvent_t ev_end,
                           cudaStream_t st);

// Workspace of a reservation, fork or compaction (the largest of them).
size_t pages_workspace_bytes(long long n_pages, long long max_pages, long long B);
int launch_pages_reserve(const CcaDims& d, const Paged& c, long long n, const int* count, const int* first, void* workspace, int sm_count,
                         int* status, long long* launches, cudaStream_t st);
int launch_pages_fork(const CcaDims& d, const Paged& c, const int* parent, const int* child, int n, void* workspace, int* status,
                      long long* launches, cudaStream_t st);
int launch_pages_free(const CcaDims& d, const Paged& c, const int* keep, int* status, long long* launches, cudaStream_t st);
int launch_pages_compact(const CcaDims& d, const Paged& c, int* used, void* workspace, int sm_count, int* status, long long* launches,
                         cudaStream_t st);
