// Pages of the latent cache: reserving (allocation, and copies of what is shared), forking, freeing, compacting.  All of it happens on
// the device, in stream order, and the results do not depend on the order in which threads run: pages are handed out by their number.
#include <cstring>

#include "cluster.cuh"
#include "common.cuh"
#include "paged.cuh"
#include "pdl.cuh"

namespace {

constexpr int PG_THREADS = 1024, PG_WARPS = PG_THREADS / 32;

// Sum of `v` over the block, and of the threads before this one (`before`).
CCA_DEVINL int block_scan(int v, int* sm, int& before) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int upto = v;
#pragma unroll
  for (int s = 1; s < 32; s <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, upto, s);
    if (lane >= s) upto += x;
  }
  __syncthreads();                                             // (sm may still be read from the call before)
  if (lane == 31) sm[warp] = upto;
  __syncthreads();
  const int w = sm[lane];                                      // 32 warps
  int wu = w;
#pragma unroll
  for (int s = 1; s < 32; s <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, wu, s);
    if (lane >= s) wu += x;
  }
  before = upto - v + (warp > 0 ? __shfl_sync(0xffffffffu, wu, warp - 1) : 0);
  return __shfl_sync(0xffffffffu, wu, 31);
}

// ------------------------------------------------------------------------------------------------ reserve
struct RsArgs {
  Paged c;
  int B;
  long long n;
  const int *count, *first;
  int *asked, *last;              // [n_pages]: of a shared page, how many of its holders ask for it, and the last of them
  int* fresh;                     // [n_pages]: the pages handed out
  int2* pairs;                    // [n_pages]: pages to copy, from and to
  int* need;                      // [B]: pages a sequence needs, then its place in `fresh`
  int* n_pairs;
  int hk, dh;
  int* status;
};

// Page indexes [i0, i1) of the rows that sequence b is to hold alone.
CCA_DEVINL void window(const RsArgs& a, int b, int& i0, int& i1) {
  i0 = i1 = 0;
  long long n = a.n;
  if (a.count) n = min(n, (long long)max(a.count[b], 0));
  const int from = a.first ? a.first[b] : a.c.len[b];
  if (n == 0) return;
  if (from < 0 || from + n > (long long)a.c.max_pages * a.c.P) {
    if ((threadIdx.x & 31) == 0) atomicCAS(a.status, 0, ST_PAGE_MISSING);
    return;
  }
  i0 = page_index(a.c, from);
  i1 = page_index(a.c, (int)(from + n - 1)) + 1;
}
// What becomes of entry e of sequence b: whether it gets a new page.
CCA_DEVINL bool wants_page(const RsArgs& a, int b, int e) {
  if (e < 0) return true;
  const int refs = __ldcg(a.c.refs + e);
  return refs > 1 && !(__ldcg(a.asked + e) == refs && __ldcg(a.last + e) == b);
}

// One cluster.  Its CTAs share out the sequences and the pool, both in contiguous runs, and learn each other's counts through shared memory.
__global__ void __launch_bounds__(PG_THREADS) pages_reserve_kernel(RsArgs a, int ranks) {
  __shared__ int sm[PG_WARPS];
  __shared__ int mine[2];                                      // pages needed and pages free in this CTA's runs
  const int rank = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int s0 = (int)((long long)a.B * rank / ranks), s1 = (int)((long long)a.B * (rank + 1) / ranks);
  const int p0 = (int)((long long)a.c.n_pages * rank / ranks), p1 = (int)((long long)a.c.n_pages * (rank + 1) / ranks);
  pdl_enter();
  if (rank == 0 && tid == 0) *a.n_pairs = 0;
  // ---- who asks for shared pages
  for (int b = s0 + warp; b < s1; b += PG_WARPS) {
    int i0, i1;
    window(a, b, i0, i1);
    for (int i = i0 + lane; i < i1; i += 32) {
      const int e = page_at(a.c, b, i);
      if (e >= 0 && a.c.refs[e] > 1) { __stcg(a.asked + e, 0); __stcg(a.last + e, -1); }
    }
  }
  all_sync(ranks);
  for (int b = s0 + warp; b < s1; b += PG_WARPS) {
    int i0, i1;
    window(a, b, i0, i1);
    for (int i = i0 + lane; i < i1; i += 32) {
      const int e = page_at(a.c, b, i);
      if (e >= 0 && a.c.refs[e] > 1) { atomicAdd(a.asked + e, 1); atomicMax(a.last + e, b); }
    }
  }
  all_sync(ranks);
  // ---- pages needed, by sequence and in all
  for (int b = s0 + warp; b < s1; b += PG_WARPS) {
    int i0, i1, n = 0;
    window(a, b, i0, i1);
    for (int i = i0; i < i1; i += 32) {
      const bool wants = i + lane < i1 && wants_page(a, b, page_at(a.c, b, i + lane));
      n += __popc(__ballot_sync(0xffffffffu, wants));
    }
    if (lane == 0) __stcg(a.need + b, n);
  }
  __syncthreads();
  int needed = 0;
  for (int b = s0; b < s1; b += PG_THREADS) {
    int before;
    const int n = b + tid < s1 ? __ldcg(a.need + b + tid) : 0;
    const int all = block_scan(n, sm, before);
    if (b + tid < s1) __stcg(a.need + b + tid, needed + before);
    needed += all;
  }
  int free_here = 0;
  for (int p = p0; p < p1; p += PG_THREADS) {
    free_here += __syncthreads_count(p + tid < p1 && a.c.refs[p + tid] <= 0);
  }
  if (tid == 0) { mine[0] = needed; mine[1] = free_here; }
  all_sync(ranks);
  int total = 0, free_all = 0, seq_base = 0, page_base = 0;
  for (int x = 0; x < ranks; ++x) {
    const int n = ranks == 1 ? mine[0] : cluster_load(&mine[0], x), f = ranks == 1 ? mine[1] : cluster_load(&mine[1], x);
    if (x < rank) { seq_base += n; page_base += f; }
    total += n;
    free_all += f;
  }
  if (total > free_all && rank == 0 && tid == 0) atomicCAS(a.status, 0, ST_PAGES_SHORT);
  const bool go = total > 0 && total <= free_all;
  // ---- the free pages, ascending, as many as are needed
  if (go)
    for (int p = p0, at = page_base; p < p1 && at < total; p += PG_THREADS) {
      int before;
      const bool is_free = p + tid < p1 && a.c.refs[p + tid] <= 0;
      const int all = block_scan(is_free, sm, before);
      if (is_free && at + before < total) __stcg(a.fresh + at + before, p + tid);
      at += all;
    }
  all_sync(ranks);                                             // (nobody leaves while its shared memory may be read)
  if (!go) return;
  // ---- handed out in the order of the sequences and their pages
  for (int b = s0 + warp; b < s1; b += PG_WARPS) {
    int i0, i1, at = seq_base + __ldcg(a.need + b);
    window(a, b, i0, i1);
    for (int i = i0; i < i1; i += 32) {
      const int e = i + lane < i1 ? page_at(a.c, b, i + lane) : -1;
      const bool wants = i + lane < i1 && wants_page(a, b, e);
      const unsigned all = __ballot_sync(0xffffffffu, wants);
      if (wants) {
        const int page = __ldcg(a.fresh + at + __popc(all & ((1u << lane) - 1)));
        a.c.table[(size_t)b * a.c.max_pages + i + lane] = page;
        a.c.refs[page] = 1;
        if (e >= 0) a.pairs[atomicAdd(a.n_pairs, 1)] = make_int2(e, page);     // refs[e] falls with the copy
      }
      at += __popc(all);
    }
  }
}

constexpr int CP_THREADS = 256, CP_PIECES = 1024;              // 16-byte pieces a block copies at once

CCA_DEVINL void copy_pieces(const Paged& c, int from, int to, long long page_pieces, int part, int tid) {
  const long long parts = (page_pieces + CP_PIECES - 1) / CP_PIECES;
  const bool v = part >= parts;
  const long long p0 = (long long)(v ? part - parts : part) * CP_PIECES;
  const uint4* src = reinterpret_cast<const uint4*>(v ? c.v : c.k) + (size_t)from * page_pieces;
  uint4* dst = reinterpret_cast<uint4*>(v ? c.v : c.k) + (size_t)to * page_pieces;
  uint4 x[CP_PIECES / CP_THREADS];
#pragma unroll
  for (int i = 0; i < CP_PIECES / CP_THREADS; ++i)
    if (p0 + i * CP_THREADS + tid < page_pieces) x[i] = __ldcs(src + p0 + i * CP_THREADS + tid);
#pragma unroll
  for (int i = 0; i < CP_PIECES / CP_THREADS; ++i)
    if (p0 + i * CP_THREADS + tid < page_pieces) dst[p0 + i * CP_THREADS + tid] = x[i];
}

__global__ void __launch_bounds__(CP_THREADS) pages_copy_kernel(RsArgs a) {
  pdl_enter();
  const long long page_pieces = (long long)a.hk * a.c.P * a.dh / 8;
  const int parts = 2 * (int)((page_pieces + CP_PIECES - 1) / CP_PIECES);
  const long long items = (long long)*a.n_pairs * parts;
  for (long long x = blockIdx.x; x < items; x += gridDim.x) {
    const int pair = (int)(x / parts), part = (int)(x - (long long)pair * parts);
    const int2 ft = a.pairs[pair];
    copy_pieces(a.c, ft.x, ft.y, page_pieces, part, threadIdx.x);
    if (part == 0 && threadIdx.x == 0) atomicSub(a.c.refs + ft.x, 1);
  }
}

// ------------------------------------------------------------------------------------------------ fork and free
struct FkArgs {
  Paged c;
  int B, n;
  const int *parent, *child;
  int* rows;                      // [n, max_pages]: the children's new rows
  int* lens;                      // [n]: their lengths, -1: nothing to do
  int* status;
};
constexpr int FK_THREADS = 256;

CCA_DEVINL void let_go(const Paged& c, int page, int* status) {
  if (atomicSub(c.refs + page, 1) <= 0) {                      // held by nobody: the table and the counts do not agree
    atomicAdd(c.refs + page, 1);
    atomicCAS(status, 0, ST_PAGE_MISSING);
  }
}

// Everything that is read of the state before the call: the parents' rows, kept aside; the counts change here, in any order.
__global__ void __launch_bounds__(FK_THREADS) pages_fork_read_kernel(FkArgs a) {
  pdl_enter();
  const int x = blockIdx.x, tid = threadIdx.x;
  const int p = a.parent[x], c = a.child[x];
  const bool inside = (unsigned)p < (unsigned)a.B && (unsigned)c < (unsigned)a.B;
  int len = inside ? a.c.len[p] : -1;
  bool later = false;                                          // another pair has the same child: the last one counts
  for (int y = x + 1 + tid; y < a.n; y += FK_THREADS)
    if (a.child[y] == c && (unsigned)a.parent[y] < (unsigned)a.B) later = true;
  later = __syncthreads_or(later);
  const long long held = len < 0 ? 0 : ((long long)len + a.c.P - 1) / a.c.P;
  if (len < 0 || held > a.c.max_pages) {
    if (tid == 0) atomicCAS(a.status, 0, ST_PAGE_MISSING);
    len = -1;
  }
  const bool go = len >= 0 && !later && p != c;
  if (tid == 0) a.lens[x] = go ? len : -1;
  if (!go) return;
  for (int i = tid; i < a.c.max_pages; i += FK_THREADS) {
    const int e = i < held ? page_at(a.c, p, i) : -1, old = page_at(a.c, c, i);
    a.rows[(size_t)x * a.c.max_pages + i] = e;
    if (e == old) continue;
    if (e >= 0) atomicAdd(a.c.refs + e, 1);
    if (old >= 0) let_go(a.c, old, a.status);
  }
}
__global__ void __launch_bounds__(FK_THREADS) pages_fork_write_kernel(FkArgs a) {
  pdl_enter();
  const int x = blockIdx.x, tid = threadIdx.x;
  const int len = a.lens[x];
  if (len < 0) return;
  const int c = a.child[x];
  for (int i = tid; i < a.c.max_pages; i += FK_THREADS)
    a.c.table[(size_t)c * a.c.max_pages + i] = a.rows[(size_t)x * a.c.max_pages + i];
  if (tid == 0) a.c.len[c] = len;
}

struct FrArgs {
  Paged c;
  const int* keep;
  int* status;
};
__global__ void __launch_bounds__(FK_THREADS) pages_free_kernel(FrArgs a) {
  pdl_enter();
  const int b = blockIdx.x, tid = threadIdx.x;
  const int keep = a.keep[b], len = a.c.len[b];
  if (keep < 0) return;
  const int left = max(min(keep, len), 0);
  __syncthreads();                                             // everybody has read the length
  if (tid == 0) a.c.len[b] = left;
  const long long held = ((long long)left + a.c.P - 1) / a.c.P;
  for (long long i = held + tid; i < a.c.max_pages; i += FK_THREADS) {
    int* at = a.c.table + (size_t)b * a.c.max_pages + i;
    const int e = *at;
    if (e == -1) continue;
    *at = -1;
    if ((unsigned)e < (unsigned)a.c.n_pages) let_go(a.c, e, a.status);
  }
}

// ------------------------------------------------------------------------------------------------ compact
struct CmArgs {
  Paged c;
  int B, hk, dh;
  int* src;                       // [n_pages]: held page of each number among the held ones (from the first that moves on)
  int* dst;                       // [n_pages]: where the moving pages go, ascending
  int* number;                    // [n_pages]: a page's number among the held ones, -1 where it is free (behind the held ones' count)
  int* counts;                    // held pages, moving pages
  int* used;                      // the caller's
};

// One cluster, as in pages_reserve_kernel: held pages are counted, then those that move and the places they go to are listed.
__global__ void __launch_bounds__(PG_THREADS) pages_compact_kernel(CmArgs a, int ranks) {
  __shared__ int sm[PG_WARPS];
  __shared__ int mine[1];
  const int rank = blockIdx.x, tid = threadIdx.x;
  const int p0 = (int)((long long)a.c.n_pages * rank / ranks), p1 = (int)((long long)a.c.n_pages * (rank + 1) / ranks);
  pdl_enter();
  if (rank == 0 && tid == 0) a.counts[1] = 0;
  int held = 0;
  for (int p = p0; p < p1; p += PG_THREADS) held += __syncthreads_count(p + tid < p1 && a.c.refs[p + tid] > 0);
  if (tid == 0) mine[0] = held;
  all_sync(ranks);
  int total = 0, at = 0;
  for (int x = 0; x < ranks; ++x) {
    const int n = ranks == 1 ? mine[0] : cluster_load(&mine[0], x);
    if (x < rank) at += n;
    total += n;
  }
  all_sync(ranks);                                             // (nobody leaves while its shared memory may be read)
  if (rank == 0 && tid == 0) { a.counts[0] = total; *a.used = total; }
  int holes = 0;
  for (int p = p0; p < p1; p += PG_THREADS) {
    const int page = p + tid;
    const bool is_held = page < p1 && a.c.refs[page] > 0;
    int before;
    const int all = block_scan(is_held, sm, before);
    const int number = at + before;
    if (page < p1) {
      if (page >= total) {
        a.number[page] = is_held ? number : -1;
        if (is_held) a.src[number] = page;
      } else if (!is_held) {
        a.dst[page - number] = page;
      }
    }
    holes += __syncthreads_count(page < p1 && page < total && !is_held);
    at += all;
  }
  if (tid == 0 && holes) atomicAdd(a.counts + 1, holes);
}
__global__ void __launch_bounds__(CP_THREADS) pages_move_kernel(CmArgs a) {
  pdl_enter();
  const int total = a.counts[0], moves = a.counts[1], stay = total - moves;      // number of the first held page that moves
  if (moves == 0) return;
  const long long page_pieces = (long long)a.hk * a.c.P * a.dh / 8;
  const int parts = 2 * (int)((page_pieces + CP_PIECES - 1) / CP_PIECES);
  const long long items = (long long)moves * parts;
  for (long long x = blockIdx.x; x < items; x += gridDim.x) {
    const int m = (int)(x / parts), part = (int)(x - (long long)m * parts);
    const int from = a.src[stay + m], to = a.dst[m];
    copy_pieces(a.c, from, to, page_pieces, part, threadIdx.x);
    if (part == 0 && threadIdx.x == 0) {
      a.c.refs[to] = a.c.refs[from];
      a.c.refs[from] = 0;
    }
  }
  const long long entries = (long long)a.B * a.c.max_pages;
  for (long long i = (long long)blockIdx.x * CP_THREADS + threadIdx.x; i < entries; i += (long long)gridDim.x * CP_THREADS) {
    const int e = a.c.table[i];
    if (e >= total && e < a.c.n_pages) {
      const int number = a.number[e];
      if (number >= 0) a.c.table[i] = a.dst[number - stay];
    }
  }
}

int cluster_ranks(long long) { return 8; }
int copy_blocks(int sm_count) { return sm_count * 8; }         // what is resident at 256 threads

struct PagesLayout { size_t asked, last, fresh, pairs, need, counts, rows, lens, end; };
PagesLayout pages_layout(long long n_pages, long long max_pages, long long B) {
  PagesLayout l;
  size_t off = 0, fork = 0;
  auto take = [](size_t& at, size_t n) { const size_t o = at; at += (n + 255) / 256 * 256; return o; };
  l.asked = take(off, (size_t)n_pages * 4);
  l.last = take(off, (size_t)n_pages * 4);
  l.fresh = take(off, (size_t)n_pages * 4);
  l.pairs = take(off, (size_t)n_pages * 8);
  l.need = take(off, (size_t)B * 4);
  l.counts = take(off, 8);
  l.rows = take(fork, (size_t)B * max_pages * 4);
  l.lens = take(fork, (size_t)B * 4);
  l.end = off > fork ? off : fork;
  return l;
}

}  // namespace

size_t pages_workspace_bytes(long long n_pages, long long max_pages, long long B) { return pages_layout(n_pages, max_pages, B).end; }

int launch_pages_reserve(const CcaDims& d, const Paged& c, long long n, const int* count, const int* first, void* workspace, int sm_count,
                         int* status, long long* launches, cudaStream_t st) {
  const PagesLayout l = pages_layout(c.n_pages, c.max_pages, d.B);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  auto at = [&](size_t o) { return reinterpret_cast<int*>(ws + o); };
  RsArgs a;
  memset(&a, 0, sizeof(a));
  a.c = c; a.B = d.B; a.n = n; a.count = count; a.first = first; a.asked = at(l.asked); a.last = at(l.last); a.fresh = at(l.fresh);
  a.pairs = reinterpret_cast<int2*>(ws + l.pairs); a.need = at(l.need); a.n_pairs = at(l.counts); a.hk = d.hk; a.dh = d.dh; a.status = status;
  const int ranks = cluster_ranks(c.n_pages);
  cudaError_t e = launch_clusters(pages_reserve_kernel, dim3((unsigned)ranks), dim3(PG_THREADS), 0, ranks, st, a, ranks);
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  e = launch_pdl(pages_copy_kernel, dim3((unsigned)copy_blocks(sm_count)), dim3(CP_THREADS), st, a);
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  return 0;
}

int launch_pages_fork(const CcaDims& d, const Paged& c, const int* parent, const int* child, int n, void* workspace, int* status,
                      long long* launches, cudaStream_t st) {
  const PagesLayout l = pages_layout(c.n_pages, c.max_pages, d.B);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  FkArgs a;
  memset(&a, 0, sizeof(a));
  a.c = c; a.B = d.B; a.n = n; a.parent = parent; a.child = child; a.rows = reinterpret_cast<int*>(ws + l.rows);
  a.lens = reinterpret_cast<int*>(ws + l.lens); a.status = status;
  cudaError_t e = launch_pdl(pages_fork_read_kernel, dim3((unsigned)n), dim3(FK_THREADS), st, a);
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  if ((e = launch_pdl(pages_fork_write_kernel, dim3((unsigned)n), dim3(FK_THREADS), st, a)) != cudaSuccess) return -(int)e;
  ++*launches;
  return 0;
}

int launch_pages_free(const CcaDims& d, const Paged& c, const int* keep, int* status, long long* launches, cudaStream_t st) {
  const cudaError_t e = launch_pdl(pages_free_kernel, dim3((unsigned)d.B), dim3(FK_THREADS), st, FrArgs{c, keep, status});
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  return 0;
}

int launch_pages_compact(const CcaDims& d, const Paged& c, int* used, void* workspace, int sm_count, long long* launches, cudaStream_t st) {
  const PagesLayout l = pages_layout(c.n_pages, c.max_pages, d.B);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  auto at = [&](size_t o) { return reinterpret_cast<int*>(ws + o); };
  CmArgs a;
  memset(&a, 0, sizeof(a));
  a.c = c; a.B = d.B; a.hk = d.hk; a.dh = d.dh; a.src = at(l.asked); a.dst = at(l.last); a.number = at(l.fresh); a.counts = at(l.counts);
  a.used = used;
  const int ranks = cluster_ranks(c.n_pages);
  cudaError_t e = launch_clusters(pages_compact_kernel, dim3((unsigned)ranks), dim3(PG_THREADS), 0, ranks, st, a, ranks);
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  if ((e = launch_pdl(pages_move_kernel, dim3((unsigned)copy_blocks(sm_count)), dim3(CP_THREADS), st, a)) != cudaSuccess) return -(int)e;
  ++*launches;
  return 0;
}
