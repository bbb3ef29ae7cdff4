// Pages of the latent cache: reserving (allocation, and copies of what is shared), forking, freeing, compacting.  All of it happens on
// the device, in stream order, and the results do not depend on the order in which threads run: pages are handed out by their number.
#include <cstring>

#include "cluster.cuh"
#include "common.cuh"
#include "paged.cuh"
#include "pdl.cuh"
#include "tc_ptx.cuh"

namespace {

constexpr int PG_THREADS = 1024, PG_WARPS = PG_THREADS / 32;
constexpr int RANKS = 8;                                       // CTAs of a cluster

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

// ------------------------------------------------------------------------------------------------ copies
// Pages are copied by the bulk copy engine, 16 KB at a time through a ring in shared memory: one warp a CTA, whose first lane starts the
// copies in and out.  A stage is filled again two steps after its copy out began, so four loads are on their way while two stages drain.
// Bound by memory: 1792 pages of 64 KB copied from 256 (the sources stay in the L2) in 27 us, 4096 moved from all over a pool of a gigabyte in
// 92 us = 5.8 TB/s in and out.  Stages of 8 or 32 KB, three CTAs an SM: the same.  By threads, 16 bytes a load, the first took 50 us.
constexpr int EN_STAGES = 6, EN_BYTES = 16384, EN_CTAS = 2;    // CTAs of an SM
constexpr size_t EN_RING = (size_t)EN_STAGES * EN_BYTES;
struct EngineShare {
  uint64_t bar[EN_STAGES];
  void* to[EN_STAGES];
  uint32_t bytes[EN_STAGES];
  int ctl[2];
};
CCA_DEVINL void bulk_load(void* to, const void* from, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(tc::smem_u32(to)), "l"(from), "r"(bytes), "r"(tc::smem_u32(bar)) : "memory");
}
CCA_DEVINL void bulk_store(void* to, const void* from, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(to), "r"(tc::smem_u32(from)), "r"(bytes) : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}

// Copies of one warp: item x of `items` (from, to, bytes: multiples of 16, at most EN_BYTES, for any lane's x) for x = first, first + step, ...
template <typename Item>
CCA_DEVINL void engine(unsigned char* ring, EngineShare& sh, long long first, long long step, long long items, Item item, int* status) {
  const int lane = threadIdx.x & 31;
  constexpr int LAG = EN_STAGES - 2;
  if (lane == 0) {
    for (int i = 0; i < EN_STAGES; ++i) tc::mbar_init(&sh.bar[i], 1);
    tc::fence_barrier_init();
    tc::wait_ctl_init(sh.ctl, status);
    asm volatile("fence.proxy.async.global;" ::: "memory");    // the pages were written by ordinary stores of earlier kernels
  }
  __syncwarp();
  const long long mine = items > first ? (items - first + step - 1) / step : 0;
  const void* from = nullptr;
  void* to = nullptr;
  uint32_t bytes = 0;
  bool ok = true;
  long long i = 0;
  for (; i < mine + LAG && ok; ++i) {
    if (i < mine) {
      if (i % 32 == 0 && i + lane < mine) item(first + (i + lane) * step, from, to, bytes);      // 32 items ahead, one a lane
      const int l = (int)(i % 32), s = (int)(i % EN_STAGES);
      const unsigned long long f = __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(from), l);
      const unsigned long long t = __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(to), l);
      const uint32_t n = __shfl_sync(0xffffffffu, bytes, l);
      if (lane == 0) {
        asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
        sh.to[s] = reinterpret_cast<void*>(t);
        sh.bytes[s] = n;
        tc::mbar_expect_tx(&sh.bar[s], n);
        bulk_load(ring + (size_t)s * EN_BYTES, reinterpret_cast<const void*>(f), n, &sh.bar[s]);
      }
    }
    if (i >= LAG) {
      const long long k = i - LAG;
      const int s = (int)(k % EN_STAGES);
      if (lane == 0) {
        ok = tc::mbar_wait(&sh.bar[s], (uint32_t)(k / EN_STAGES) & 1, sh.ctl);
        if (ok) bulk_store(sh.to[s], ring + (size_t)s * EN_BYTES, sh.bytes[s]);
      }
      ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
    }
  }
  if (lane == 0) {
    if (!ok) {                                                 // a load never came: the others are waited for before the CTA ends
      atomicCAS(status, 0, tc::ST_TIMEOUT_TMA);
      for (long long k = i - 1 - LAG; k < i && k < mine; ++k) tc::mbar_wait(&sh.bar[k % EN_STAGES], (uint32_t)(k / EN_STAGES) & 1, sh.ctl);
    }
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  __syncwarp();
}

// The CTA's share of the copies of n pairs of pages, pair(m) for m < n: keys and values in parts of EN_BYTES.
template <typename Pair>
CCA_DEVINL void copy_pages(const Paged& c, int hk, int dh, int n, unsigned char* ring, EngineShare& sh, Pair pair, int* status) {
  const long long page_bytes = (long long)hk * c.P * dh * 2;
  const int half = (int)((page_bytes + EN_BYTES - 1) / EN_BYTES), parts = 2 * half;
  engine(ring, sh, blockIdx.x, gridDim.x, (long long)n * parts, [&](long long x, const void*& from, void*& to, uint32_t& bytes) {
    const int m = (int)(x / parts), part = (int)(x - (long long)m * parts);
    const int2 ft = pair(m);
    const long long at = (long long)(part < half ? part : part - half) * EN_BYTES;
    unsigned char* base = reinterpret_cast<unsigned char*>(part < half ? c.k : c.v) + at;
    from = base + ft.x * page_bytes;
    to = base + ft.y * page_bytes;
    bytes = (uint32_t)min((long long)EN_BYTES, page_bytes - at);
  }, status);
}

// The same by the threads of a cluster, where few bytes can be meant.
template <typename Pair>
CCA_DEVINL void copy_by_threads(const Paged& c, int hk, int dh, int n, int rank, Pair pair) {
  const unsigned pieces = (unsigned)(hk * c.P * dh / 8), all = 2 * pieces * n;              // 16 bytes each
#pragma unroll 4
  for (unsigned x = rank * PG_THREADS + threadIdx.x; x < all; x += RANKS * PG_THREADS) {
    const unsigned half = x / pieces, piece = x - half * pieces;
    const int2 ft = pair(half >> 1);
    uint4* at = reinterpret_cast<uint4*>(half & 1 ? c.v : c.k) + piece;
    at[(size_t)ft.y * pieces] = __ldcg(at + (size_t)ft.x * pieces);
  }
}

// ------------------------------------------------------------------------------------------------ reserve
struct RsArgs {
  Paged c;
  int B;
  int width;                      // page indexes that n rows reach into at most
  long long n;
  const int *count, *first;
  int *asked, *last;              // [n_pages]: of a shared page, how many of its holders ask for it, and the last of them
  int* fresh;                     // [n_pages]: the pages handed out
  int2* pairs;                    // [n_pages]: pages to copy, from and to
  int* n_pairs;
  int hk, dh;
  int* status;
};

// Entry x of the list of all sequences' page indexes, `width` for each: its sequence and index; false where the sequence has fewer.
CCA_DEVINL bool entry_of(const RsArgs& a, int x, int& b, int& i) {
  b = x / a.width;
  const int k = x - b * a.width;
  if (b >= a.B) return false;
  long long n = a.n;
  const int from = a.first ? a.first[b] : a.c.len[b];
  if (a.count) n = min(n, (long long)max(a.count[b], 0));
  if (n == 0) return false;
  if (from < 0 || from + n > (long long)a.c.max_pages * a.c.P) {
    if (k == 0 && (a.first || from >= 0)) atomicCAS(a.status, 0, ST_PAGE_MISSING);         // (a negative length: not in use)
    return false;
  }
  i = page_index(a.c, from) + k;
  return i <= page_index(a.c, (int)(from + n - 1));
}

// Few entries: one cluster.  The first CTA looks at the entries, counting who asks for a shared page in a hash table in shared memory, while the
// others list the free pages of a part of the pool each; then it hands these out.  HERE: all of them copy what is to be copied, otherwise
// pages_copy_kernel does.  Bound by the latency of three loads that follow one another (length, table, count), two barriers of the cluster and
// what is copied: 32 entries without copies 5.9 us, 1024 6.3, 3000 8.5 (the other kernel 9.5, 9.6, 10.1, with 16 pages copied 14.4 against 7.5).
constexpr int RV_ENTRIES = 4096, RV_SLOTS = 2 * RV_ENTRIES, RV_ROUNDS = RV_ENTRIES / PG_THREADS;
struct ReserveShare {
  int page[RV_SLOTS], asked[RV_SLOTS], last[RV_SLOTS];         // first CTA: shared pages that are asked for
  int2 pairs[RV_ENTRIES];
  int fresh[RV_ENTRIES];                                       // others: free pages, ascending
  int n_fresh, n_pairs;
  int counts[RANKS];
  int scan[PG_WARPS];
};
template <bool HERE>
__global__ void __launch_bounds__(PG_THREADS) pages_reserve_few_kernel(RsArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  ReserveShare& sh = *reinterpret_cast<ReserveShare*>(smem);
  const int rank = blockIdx.x, tid = threadIdx.x;
  const int entries = a.B * a.width, rounds = (entries + PG_THREADS - 1) / PG_THREADS;
  int slots = 64;                                              // at least twice as many as entries
  while (slots < 2 * entries) slots *= 2;
  if (rank == 0)
    for (int x = tid; x < slots; x += PG_THREADS) { sh.page[x] = -1; sh.asked[x] = 0; sh.last[x] = -1; }
  if (tid == 0) sh.n_pairs = sh.n_fresh = 0;
  __syncthreads();
  pdl_enter();
  int seq[RV_ROUNDS], index[RV_ROUNDS], page[RV_ROUNDS], slot[RV_ROUNDS], place[RV_ROUNDS];
  bool wants[RV_ROUNDS];
  int total = 0;
  if (rank == 0) {
    int refs[RV_ROUNDS];
#pragma unroll
    for (int r = 0; r < RV_ROUNDS; ++r) {
      wants[r] = false;
      page[r] = -1;
      refs[r] = 0;
      if (r < rounds) wants[r] = entry_of(a, r * PG_THREADS + tid, seq[r], index[r]);
    }
#pragma unroll
    for (int r = 0; r < RV_ROUNDS; ++r)
      if (wants[r]) page[r] = page_at(a.c, seq[r], index[r]);
#pragma unroll
    for (int r = 0; r < RV_ROUNDS; ++r)
      if (page[r] >= 0) refs[r] = a.c.refs[page[r]];
#pragma unroll
    for (int r = 0; r < RV_ROUNDS; ++r)
      if (refs[r] > 1) {
        unsigned at = (unsigned)page[r] * 2654435761u;         // (multiplicative hashing)
        for (int tries = 0; tries < slots; ++tries, ++at) {
          slot[r] = at & (slots - 1);
          const int was = atomicCAS(&sh.page[slot[r]], -1, page[r]);
          if (was == -1 || was == page[r]) break;
        }
        atomicAdd(&sh.asked[slot[r]], 1);
        atomicMax(&sh.last[slot[r]], seq[r]);
      }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RV_ROUNDS; ++r)
      if (page[r] >= 0) wants[r] = refs[r] > 1 && !(sh.asked[slot[r]] == refs[r] && sh.last[slot[r]] == seq[r]);
#pragma unroll
    for (int r = 0; r < RV_ROUNDS; ++r)
      if (r < rounds) {
        const int all = block_scan(wants[r], sh.scan, place[r]);
        place[r] += total;
        total += all;
      }
  } else {
    const int parts = RANKS - 1;
    const int p0 = (int)((long long)a.c.n_pages * (rank - 1) / parts), p1 = (int)((long long)a.c.n_pages * rank / parts);
    constexpr int EACH = 8;                                    // neighbouring pages a thread looks at
    int n = 0;
    for (int p = p0; p < p1 && n < entries; p += EACH * PG_THREADS) {
      unsigned free = 0;
#pragma unroll
      for (int k = 0; k < EACH; ++k) {
        const int at = p + tid * EACH + k;
        if (at < p1 && a.c.refs[at] <= 0) free |= 1u << k;
      }
      int before;
      const int all = block_scan(__popc(free), sh.scan, before);
      before += n;
      for (; free; free &= free - 1, ++before)
        if (before < RV_ENTRIES) sh.fresh[before] = p + tid * EACH + __ffs(free) - 1;
      n += all;
    }
    if (tid == 0) sh.n_fresh = min(n, RV_ENTRIES);
  }
  cluster_barrier();
  if (rank == 0) {
    if (tid < RANKS) sh.counts[tid] = tid > 0 ? cluster_load(&sh.n_fresh, tid) : 0;
    __syncthreads();
    int there = 0;
#pragma unroll
    for (int x = 1; x < RANKS; ++x) there += sh.counts[x];
    if (total > there && tid == 0) atomicCAS(a.status, 0, ST_PAGES_SHORT);
    if (total <= there) {
#pragma unroll
      for (int r = 0; r < RV_ROUNDS; ++r)
        if (r < rounds && wants[r]) {
          int at = place[r], x = 1;
          while (at >= sh.counts[x]) at -= sh.counts[x++];
          const int fresh = cluster_load(&sh.fresh[at], x);
          a.c.table[(size_t)seq[r] * a.c.max_pages + index[r]] = fresh;
          a.c.refs[fresh] = 1;
          if (page[r] >= 0) {
            atomicSub(a.c.refs + page[r], 1);
            sh.pairs[atomicAdd(&sh.n_pairs, 1)] = make_int2(page[r], fresh);
          }
        }
    }
    if (!HERE) {
      __syncthreads();
      for (int x = tid; x < sh.n_pairs; x += PG_THREADS) a.pairs[x] = sh.pairs[x];
      if (tid == 0) *a.n_pairs = sh.n_pairs;
    }
  }
  cluster_barrier();                                           // (nobody leaves while its shared memory may be read)
  if (HERE) {
    const int n = cluster_load(&sh.n_pairs, 0);
    copy_by_threads(a.c, a.hk, a.dh, n, rank, [&](int x) { return cluster_load2(&sh.pairs[x].x, 0); });
    cluster_barrier();
  }
}

// Whether the entry gets a new page, by what has been counted in global memory.
CCA_DEVINL bool wants_page(const RsArgs& a, int b, int e) {
  if (e < 0) return true;
  const int refs = __ldcg(a.c.refs + e);
  return refs > 1 && !(__ldcg(a.asked + e) == refs && __ldcg(a.last + e) == b);
}

// Any number of entries: one cluster whose CTAs share out the entries and the pool, both in contiguous runs, and count in global memory.  Bound by
// the loads' latency and four barriers of 8 SMs that pass over the entries four times: 8192 entries (a pool of 9831 pages) 13.5 us, 65536 (of
// 78651) 41.
__global__ void __launch_bounds__(PG_THREADS) pages_reserve_kernel(RsArgs a) {
  __shared__ int sm[PG_WARPS];
  __shared__ int mine[2];                                      // pages needed and pages free in this CTA's runs
  const int rank = blockIdx.x, tid = threadIdx.x;
  const long long entries = (long long)a.B * a.width;
  const int x0 = (int)(entries * rank / RANKS), x1 = (int)(entries * (rank + 1) / RANKS);
  const int p0 = (int)((long long)a.c.n_pages * rank / RANKS), p1 = (int)((long long)a.c.n_pages * (rank + 1) / RANKS);
  pdl_enter();
  if (rank == 0 && tid == 0) *a.n_pairs = 0;
  auto look = [&](int x, int& b, int& i, int& e) {             // false: no entry
    if (x >= x1 || !entry_of(a, x, b, i)) return false;
    e = page_at(a.c, b, i);
    return true;
  };
  // ---- who asks for shared pages
#pragma unroll 4
  for (int x = x0 + tid; x < x1; x += PG_THREADS) {
    int b, i, e;
    if (look(x, b, i, e) && e >= 0 && a.c.refs[e] > 1) { __stcg(a.asked + e, 0); __stcg(a.last + e, -1); }
  }
  cluster_barrier();
#pragma unroll 4
  for (int x = x0 + tid; x < x1; x += PG_THREADS) {
    int b, i, e;
    if (look(x, b, i, e) && e >= 0 && a.c.refs[e] > 1) { atomicAdd(a.asked + e, 1); atomicMax(a.last + e, b); }
  }
  cluster_barrier();
  // ---- pages needed and pages free
  int n = 0, free_here = 0;
#pragma unroll 4
  for (int x = x0 + tid; x < x1; x += PG_THREADS) {
    int b, i, e;
    n += look(x, b, i, e) && wants_page(a, b, e);
  }
#pragma unroll 4
  for (int p = p0 + tid; p < p1; p += PG_THREADS) free_here += a.c.refs[p] <= 0;
  int before;
  n = block_scan(n, sm, before);
  free_here = block_scan(free_here, sm, before);
  if (tid == 0) { mine[0] = n; mine[1] = free_here; }
  cluster_barrier();
  int total = 0, free_all = 0, need_base = 0, page_base = 0;
  for (int x = 0; x < RANKS; ++x) {
    const int need = cluster_load(&mine[0], x), f = cluster_load(&mine[1], x);
    if (x < rank) { need_base += need; page_base += f; }
    total += need;
    free_all += f;
  }
  if (total > free_all && rank == 0 && tid == 0) atomicCAS(a.status, 0, ST_PAGES_SHORT);
  const bool go = total > 0 && total <= free_all;
  // ---- the free pages, ascending, as many as are needed
  if (go)
    for (int p = p0, at = page_base; p < p1 && at < total; p += PG_THREADS) {
      const bool is_free = p + tid < p1 && a.c.refs[p + tid] <= 0;
      const int all = block_scan(is_free, sm, before);
      if (is_free && at + before < total) __stcg(a.fresh + at + before, p + tid);
      at += all;
    }
  cluster_barrier();                                             // (nobody leaves while its shared memory may be read)
  if (!go) return;
  // ---- handed out in the order of the entries
  for (int x = x0, at = need_base; x < x1; x += PG_THREADS) {
    int b, i, e;
    const bool wants = look(x + tid, b, i, e) && wants_page(a, b, e);
    const int all = block_scan(wants, sm, before);
    if (wants) {
      const int page = __ldcg(a.fresh + at + before);
      a.c.table[(size_t)b * a.c.max_pages + i] = page;
      a.c.refs[page] = 1;
      if (e >= 0) a.pairs[atomicAdd(a.n_pairs, 1)] = make_int2(e, page);       // refs[e] falls with the copy: it is still read here
    }
    at += all;
  }
}

// What has been paired, copied; `let_go`: the old pages' counts fall here.
constexpr int CP_THREADS = 256;
__global__ void __launch_bounds__(CP_THREADS) pages_copy_kernel(RsArgs a, int let_go) {
  extern __shared__ __align__(128) unsigned char ring[];
  __shared__ EngineShare sh;
  pdl_enter();
  const int n = *a.n_pairs;
  if (threadIdx.x < 32) {
    copy_pages(a.c, a.hk, a.dh, n, ring, sh, [&](int x) { return a.pairs[x]; }, a.status);
  } else if (let_go) {
    for (long long x = (long long)blockIdx.x * (CP_THREADS - 32) + threadIdx.x - 32; x < n; x += (long long)gridDim.x * (CP_THREADS - 32))
      atomicSub(a.c.refs + a.pairs[x].x, 1);
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
constexpr int FK_THREADS = 512, FK_EACH = 4;                   // table entries that a thread has on their way at once

CCA_DEVINL void let_go(const Paged& c, const int* page, int* status) {     // FK_EACH pages, -1: none
  int held[FK_EACH];
#pragma unroll
  for (int k = 0; k < FK_EACH; ++k) held[k] = page[k] >= 0 ? atomicSub(c.refs + page[k], 1) : 1;
#pragma unroll
  for (int k = 0; k < FK_EACH; ++k)
    if (held[k] <= 0) {                                        // held by nobody: the table and the counts do not agree
      atomicAdd(c.refs + page[k], 1);
      atomicCAS(status, 0, ST_PAGE_MISSING);
    }
}

struct AnyOfBlock {
  static constexpr int threads = FK_THREADS;
  CCA_DEVINL bool operator()(bool v) const { return __syncthreads_or(v) != 0; }
};
struct AnyOfWarp {
  static constexpr int threads = 32;
  CCA_DEVINL bool operator()(bool v) const { return __any_sync(0xffffffffu, v) != 0; }
};
// Pair x, by `threads` threads: everything that is read of the state before the call.  The parent's row is kept aside; the counts change
// here, in any order.  Returns the child's new length, -1: nothing to do.  any(v): whether one of its
// group of threads, which look at all later pairs together, has v.
template <typename Any>
CCA_DEVINL int fork_read(const FkArgs& a, int x, int tid, int threads, Any any) {
  const int p = a.parent[x], c = a.child[x];
  auto rows = [&](int parent) {                                // -1: a pair with this parent is skipped
    const int n = (unsigned)parent < (unsigned)a.B ? __ldcg(a.c.len + parent) : -1;
    return n <= (long long)a.c.max_pages * a.c.P ? n : -1;
  };
  const int len = (unsigned)c < (unsigned)a.B ? rows(p) : -1;
  bool later = false;                                          // another pair has the same child: the last one counts
  const int group = any.threads;
  for (int y = x + 1 + tid % group; y < a.n; y += group)
    if (a.child[y] == c && rows(a.parent[y]) >= 0) later = true;
  later = any(later);
  if (len < 0 && tid == 0) atomicCAS(a.status, 0, ST_PAGE_MISSING);
  const int held = len > 0 ? (len - 1) / a.c.P + 1 : 0;
  const bool go = len >= 0 && !later && p != c;
  if (!go) return -1;
  for (int i0 = tid; i0 < a.c.max_pages; i0 += FK_EACH * threads) {
    int e[FK_EACH], old[FK_EACH];
#pragma unroll
    for (int k = 0; k < FK_EACH; ++k) {
      const int i = i0 + k * threads;
      e[k] = i < held ? page_at(a.c, p, i) : -1;
      old[k] = i < a.c.max_pages ? page_at(a.c, c, i) : -1;
    }
#pragma unroll
    for (int k = 0; k < FK_EACH; ++k) {
      const int i = i0 + k * threads;
      if (i < a.c.max_pages) __stcg(a.rows + (size_t)x * a.c.max_pages + i, e[k]);
      if (e[k] == old[k]) e[k] = old[k] = -1;
      if (e[k] >= 0) atomicAdd(a.c.refs + e[k], 1);
    }
    let_go(a.c, old, a.status);
  }
  return len;
}
CCA_DEVINL void fork_write(const FkArgs& a, int x, int len, int tid, int threads) {
  if (len < 0) return;
  const int c = a.child[x];
  for (int i0 = tid; i0 < a.c.max_pages; i0 += FK_EACH * threads) {
    int e[FK_EACH];
#pragma unroll
    for (int k = 0; k < FK_EACH; ++k) {
      const int i = i0 + k * threads;
      if (i < a.c.max_pages) e[k] = __ldcg(a.rows + (size_t)x * a.c.max_pages + i);
    }
#pragma unroll
    for (int k = 0; k < FK_EACH; ++k) {
      const int i = i0 + k * threads;
      if (i < a.c.max_pages) a.c.table[(size_t)c * a.c.max_pages + i] = e[k];
    }
  }
  if (tid == 0) a.c.len[c] = len;
}
__global__ void __launch_bounds__(FK_THREADS) pages_fork_read_kernel(FkArgs a) {
  pdl_enter();
  const int len = fork_read(a, blockIdx.x, threadIdx.x, FK_THREADS, AnyOfBlock{});
  if (threadIdx.x == 0) a.lens[blockIdx.x] = len;
}
__global__ void __launch_bounds__(FK_THREADS) pages_fork_write_kernel(FkArgs a) {
  pdl_enter();
  fork_write(a, blockIdx.x, a.lens[blockIdx.x], threadIdx.x, FK_THREADS);
}
// Both in one launch: a cluster of 8, a pair by some of its warps.
__global__ void __launch_bounds__(PG_THREADS) pages_fork_few_kernel(FkArgs a) {
  pdl_enter();
  const int each = gridDim.x * PG_WARPS / a.n;                 // warps of a pair
  const int w = blockIdx.x * PG_WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int x = w / each, t = w % each * 32 + lane, threads = each * 32;
  int len = -1;
  if (x < a.n) len = fork_read(a, x, t, threads, AnyOfWarp{});
  cluster_barrier();
  if (x < a.n) fork_write(a, x, len, t, threads);
}

struct FrArgs {
  Paged c;
  const int* keep;
  int* status;
};
// A block a sequence.  Bound by latency: length, row, counts one after the other (256 rows of 1026 pages, half of them let go: 5.5 us).
__global__ void __launch_bounds__(FK_THREADS) pages_free_kernel(FrArgs a) {
  pdl_enter();
  const int b = blockIdx.x, tid = threadIdx.x;
  const int keep = a.keep[b], len = a.c.len[b];
  if (keep < 0) return;
  const int left = min(keep, max(len, 0));
  __syncthreads();                                             // everybody has read the length
  if (tid == 0 && len >= 0) a.c.len[b] = left;
  int* row = a.c.table + (size_t)b * a.c.max_pages;
  const long long held = ((long long)left + a.c.P - 1) / a.c.P;
  for (long long i0 = held + tid; i0 < a.c.max_pages; i0 += FK_EACH * FK_THREADS) {
    int e[FK_EACH];
#pragma unroll
    for (int k = 0; k < FK_EACH; ++k) e[k] = i0 + k * FK_THREADS < a.c.max_pages ? row[i0 + k * FK_THREADS] : -1;
#pragma unroll
    for (int k = 0; k < FK_EACH; ++k) {
      if (e[k] != -1) row[i0 + k * FK_THREADS] = -1;
      if ((unsigned)e[k] >= (unsigned)a.c.n_pages) e[k] = -1;
    }
    let_go(a.c, e, a.status);
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
  int* status;
};

// One cluster: held pages are counted, then those that move and the places they go to are listed, each CTA a contiguous run of the pool.  Bound by
// latency up to 10^5 pages (5.2 us with the launch behind it where nothing moves, 9.9 at 78651 pages), then by what 8 SMs read (46 at 629153).
__global__ void __launch_bounds__(PG_THREADS) pages_compact_kernel(CmArgs a) {
  __shared__ int sm[PG_WARPS];
  __shared__ int mine;                                         // held pages of this CTA's run
  const int rank = blockIdx.x, tid = threadIdx.x;
  const int p0 = (int)((long long)a.c.n_pages * rank / RANKS), p1 = (int)((long long)a.c.n_pages * (rank + 1) / RANKS);
  constexpr int EACH = 4;                                      // neighbouring pages of a thread
  pdl_enter();
  if (rank == 0 && tid == 0) a.counts[1] = 0;
  int held = 0, before;
#pragma unroll 4
  for (int p = p0 + tid; p < p1; p += PG_THREADS) held += a.c.refs[p] > 0;
  held = block_scan(held, sm, before);
  if (tid == 0) mine = held;
  cluster_barrier();
  int total = 0, at = 0;
  for (int x = 0; x < RANKS; ++x) {
    const int n = cluster_load(&mine, x);
    if (x < rank) at += n;
    total += n;
  }
  if (rank == 0 && tid == 0) { a.counts[0] = total; *a.used = total; }
  int holes = 0;
  for (int p = p0; p < p1; p += EACH * PG_THREADS) {
    int refs[EACH], n = 0;
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int page = p + tid * EACH + k;
      refs[k] = page < p1 ? a.c.refs[page] : 0;
      n += refs[k] > 0;
    }
    const int all = block_scan(n, sm, before);
    int number = at + before;
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int page = p + tid * EACH + k;
      if (page < p1) {
        if (page >= total) {
          a.number[page] = refs[k] > 0 ? number : -1;
          if (refs[k] > 0) a.src[number] = page;
        } else if (refs[k] <= 0) {
          a.dst[page - number] = page;
          ++holes;
        }
        number += refs[k] > 0;
      }
    }
    at += all;
  }
  holes = block_scan(holes, sm, before);
  if (tid == 0 && holes) atomicAdd(a.counts + 1, holes);
  cluster_barrier();                                           // (nobody leaves while its shared memory may be read)
}
__global__ void __launch_bounds__(CP_THREADS) pages_move_kernel(CmArgs a) {
  extern __shared__ __align__(128) unsigned char ring[];
  __shared__ EngineShare sh;
  pdl_enter();
  const int total = a.counts[0], moves = a.counts[1], stay = total - moves;
  if (moves == 0) return;
  if (threadIdx.x < 32) {
    copy_pages(a.c, a.hk, a.dh, moves, ring, sh, [&](int m) { return make_int2(a.src[stay + m], a.dst[m]); }, a.status);
    return;
  }
  const long long t = (long long)blockIdx.x * (CP_THREADS - 32) + threadIdx.x - 32, threads = (long long)gridDim.x * (CP_THREADS - 32);
  for (long long m = t; m < moves; m += threads) {
    const int from = a.src[stay + m], to = a.dst[m];
    a.c.refs[to] = a.c.refs[from];
    a.c.refs[from] = 0;
  }
  const long long entries = (long long)a.B * a.c.max_pages;
#pragma unroll 4
  for (long long i = t; i < entries; i += threads) {
    const int e = a.c.table[i];
    if (e >= total && e < a.c.n_pages) {
      const int number = a.number[e];
      if (number >= 0) a.c.table[i] = a.dst[number - stay];
    }
  }
}

// One launch or two (us on the device; a launch costs the host 2.5 more).  Reserving: what could have to be copied, 16 pages of 64 KB: 4.3
// where nothing is, 7.5 where 8 pages are, against 5.9 and 7.4 with a launch for the copies; 32 pages: 4.2 and 9.3 against 5.9 and 7.5.
constexpr long long FEW_BYTES = 1 << 20;
// Forking: 32 pairs of rows of 64 pages 4.3 against 3.6, 64 of 256 5.2 against 4.0, 64 of 1024 7.1 against 4.3.
constexpr int FK_FEW = 64;
constexpr long long FK_FEW_ENTRIES = 64 * 256;

template <typename... KArgs, typename... Args>
int launch_copies(void (*kernel)(KArgs...), bool* done, int sm_count, long long* launches, cudaStream_t st, Args... args) {
  cudaError_t e = opt_in(kernel, (int)EN_RING, done);
  if (e == cudaSuccess) e = launch_pdl_smem(kernel, dim3((unsigned)(sm_count * EN_CTAS)), dim3(CP_THREADS), EN_RING, st, args...);
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  return 0;
}

struct PagesLayout { size_t asked, last, fresh, pairs, counts, rows, lens, end; };
PagesLayout pages_layout(long long n_pages, long long max_pages, long long B) {
  PagesLayout l;
  size_t off = 0, fork = 0;
  auto take = [](size_t& at, size_t n) { const size_t o = at; at += (n + 255) / 256 * 256; return o; };
  l.asked = take(off, (size_t)n_pages * 4);
  l.last = take(off, (size_t)n_pages * 4);
  l.fresh = take(off, (size_t)n_pages * 4);
  l.pairs = take(off, (size_t)n_pages * 8);
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
  a.pairs = reinterpret_cast<int2*>(ws + l.pairs); a.n_pairs = at(l.counts); a.hk = d.hk; a.dh = d.dh; a.status = status;
  const long long width = (n + c.P - 2) / c.P + 1, page_bytes = 4ll * d.hk * c.P * d.dh;
  a.width = (int)(width < c.max_pages ? width : c.max_pages);
  const long long entries = (long long)d.B * a.width;
  const bool few = entries <= RV_ENTRIES, here = few && entries * page_bytes <= FEW_BYTES;
  static bool done[3][MAX_DEVICES];
  cudaError_t e = cudaSuccess;
  if (few) {
    e = here ? opt_in(pages_reserve_few_kernel<true>, (int)sizeof(ReserveShare), done[0])
             : opt_in(pages_reserve_few_kernel<false>, (int)sizeof(ReserveShare), done[1]);
    if (e == cudaSuccess)
      e = launch_clusters(here ? pages_reserve_few_kernel<true> : pages_reserve_few_kernel<false>, dim3(RANKS), dim3(PG_THREADS),
                          sizeof(ReserveShare), RANKS, st, a);
  } else {
    e = launch_clusters(pages_reserve_kernel, dim3(RANKS), dim3(PG_THREADS), 0, RANKS, st, a);
  }
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  return here ? 0 : launch_copies(pages_copy_kernel, done[2], sm_count, launches, st, a, (int)!few);
}

int launch_pages_fork(const CcaDims& d, const Paged& c, const int* parent, const int* child, int n, void* workspace, int* status,
                      long long* launches, cudaStream_t st) {
  const PagesLayout l = pages_layout(c.n_pages, c.max_pages, d.B);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  FkArgs a;
  memset(&a, 0, sizeof(a));
  a.c = c; a.B = d.B; a.n = n; a.parent = parent; a.child = child; a.rows = reinterpret_cast<int*>(ws + l.rows);
  a.lens = reinterpret_cast<int*>(ws + l.lens); a.status = status;
  cudaError_t e;
  if (n <= FK_FEW && (long long)n * c.max_pages <= FK_FEW_ENTRIES) {
    if ((e = launch_clusters(pages_fork_few_kernel, dim3(RANKS), dim3(PG_THREADS), 0, RANKS, st, a)) != cudaSuccess) return -(int)e;
    ++*launches;
    return 0;
  }
  if ((e = launch_pdl(pages_fork_read_kernel, dim3((unsigned)n), dim3(FK_THREADS), st, a)) != cudaSuccess) return -(int)e;
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

int launch_pages_compact(const CcaDims& d, const Paged& c, int* used, void* workspace, int sm_count, int* status, long long* launches,
                         cudaStream_t st) {
  const PagesLayout l = pages_layout(c.n_pages, c.max_pages, d.B);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  auto at = [&](size_t o) { return reinterpret_cast<int*>(ws + o); };
  CmArgs a;
  memset(&a, 0, sizeof(a));
  a.c = c; a.B = d.B; a.hk = d.hk; a.dh = d.dh; a.src = at(l.asked); a.dst = at(l.last); a.number = at(l.fresh); a.counts = at(l.counts);
  a.used = used; a.status = status;
  const cudaError_t e = launch_clusters(pages_compact_kernel, dim3(RANKS), dim3(PG_THREADS), 0, RANKS, st, a);
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  static bool done[MAX_DEVICES];
  return launch_copies(pages_move_kernel, done, sm_count, launches, st, a);
}
