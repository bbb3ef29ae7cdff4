// A latent cache in pages: rows put in and read back, and attention of one new token per sequence over them.
#include <cstring>

#include "cluster.cuh"
#include "common.cuh"
#include "paged.cuh"
#include "paged_rule.h"
#include "pdl.cuh"

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

CCA_DEVINL uint32_t pack_bf16x2(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
CCA_DEVINL float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
CCA_DEVINL float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// A sum of weighted values from the weights' first parts and from what these left over: an infinite value makes the first infinite, and the second
// no number wherever nothing, or less than nothing, was left over.
CCA_DEVINL float both_parts(float first, float rest) { return fabsf(first) == INFINITY ? first : first + rest; }
CCA_DEVINL void mma_16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
CCA_DEVINL void ldmatrix_x4(uint32_t* r, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
CCA_DEVINL void ldmatrix_x4_trans(uint32_t* r, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
// 16 bytes to shared memory, zeros where !there (nothing is read then).
CCA_DEVINL void copy_async(uint32_t to, const void* from, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
CCA_DEVINL void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
CCA_DEVINL void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// ------------------------------------------------------------------------------------------------ rows in and out
constexpr int RW_TOKENS = 16, RW_THREADS = 256, RW_AHEAD = 2;   // tokens of a block; 16-byte pieces of k and of v that a thread has on their way

struct RowsArgs {
  Paged c;
  int B, hk, row_chunks;          // 16-byte pieces of a row
  const bf16 *k_in, *v_in;        // append: [B, n, hk, dh]
  bf16 *k_out, *v_out;            // read
  const int* first;               // first row of each sequence, or null: len[b]
  const int* count;               // append: rows of each sequence, or null: n
  long long n;
  int* status;
};

// A block moves 16 tokens of one sequence.  The rows of a token lie together on the dense side and hk * P rows apart in its page; both
// are whole 64-byte pieces or more, so the kernel is bound by its traffic (each byte once in and once out).  New rows are on their way while
// their places are looked up.  16384 rows of 2 x 128 from the L2: 5.1 us each way; from memory and back 13.1 for both.
template <bool APPEND>
__global__ void __launch_bounds__(RW_THREADS) paged_rows_kernel(RowsArgs a) {
  __shared__ int at[RW_TOKENS];                             // pool row of kv head 0, -1: none
  const int b = blockIdx.y, tid = threadIdx.x;
  const long long t0 = (long long)blockIdx.x * RW_TOKENS;
  const int per_token = a.hk * a.row_chunks;
  const int here = (int)min((long long)RW_TOKENS, a.n - t0) * per_token;
  const size_t dense0 = ((size_t)b * a.n + t0) * per_token;
  const uint4 *kd = reinterpret_cast<const uint4*>(a.k_in) + dense0, *vd = reinterpret_cast<const uint4*>(a.v_in) + dense0;
  uint4 *ko = reinterpret_cast<uint4*>(a.k_out) + dense0, *vo = reinterpret_cast<uint4*>(a.v_out) + dense0;
  uint4 *kp = reinterpret_cast<uint4*>(a.c.k), *vp = reinterpret_cast<uint4*>(a.c.v);
  uint4 k[RW_AHEAD], v[RW_AHEAD];
  auto fetch = [&](int x0) {
#pragma unroll
    for (int i = 0; i < RW_AHEAD; ++i)
      if (x0 + i * RW_THREADS < here) {
        k[i] = __ldcs(kd + x0 + i * RW_THREADS);
        v[i] = __ldcs(vd + x0 + i * RW_THREADS);
      }
  };
  pdl_enter();
  if (APPEND) fetch(tid);
  if (tid < RW_TOKENS) {
    int to = -1;
    const long long i = t0 + tid;
    const int held = a.first ? a.first[b] : a.c.len[b];
    long long n = a.n;
    if (APPEND && a.count) n = min(n, (long long)max(a.count[b], 0));
    if (i < n) {
      const long long row = held + i, most = (long long)a.c.max_pages * a.c.P;
      if (row >= 0 && row < most && (held >= 0 || a.first)) {      // (a negative length: not in use; a negative start is one like others)
        const int pi = page_index(a.c, (int)row), page = page_at(a.c, b, pi);
        if (page >= 0 && (!APPEND || a.c.refs[page] == 1)) to = pool_row(a.c, a.hk, page, 0, (int)row - pi * a.c.P);
      }
      if (APPEND && to < 0 && held >= 0) atomicCAS(a.status, 0, ST_PAGE_MISSING);
    }
    at[tid] = to;
  }
  __syncthreads();
  auto place = [&](int x, bool& there) {                    // of the block's x-th piece in the pool
    const int token = x / per_token, in = x - token * per_token;
    const int j = in / a.row_chunks, piece = in - j * a.row_chunks;
    there = at[token] >= 0;
    return (size_t)(at[token] + j * a.c.P) * a.row_chunks + piece;
  };
  for (int x0 = tid; x0 < here; x0 += RW_AHEAD * RW_THREADS) {
    if (APPEND && x0 != tid) fetch(x0);
#pragma unroll
    for (int i = 0; i < RW_AHEAD; ++i) {
      const int x = x0 + i * RW_THREADS;
      bool there = false;
      const size_t pool = x < here ? place(x, there) : 0;
      if (APPEND) {
        if (there) { kp[pool] = k[i]; vp[pool] = v[i]; }
      } else {
        k[i] = v[i] = make_uint4(0, 0, 0, 0);
        if (there) { k[i] = kp[pool]; v[i] = vp[pool]; }
      }
    }
    if (!APPEND) {
#pragma unroll
      for (int i = 0; i < RW_AHEAD; ++i)
        if (x0 + i * RW_THREADS < here) {
          ko[x0 + i * RW_THREADS] = k[i];
          vo[x0 + i * RW_THREADS] = v[i];
        }
    }
  }
}

// ------------------------------------------------------------------------------------------------ from a prefill to the first step
struct TsArgs {
  const int* len;
  const uint4 *x, *qk0;           // [B, S] rows of x_chunks and l_chunks 16-byte pieces
  uint4 *x_prev, *hist;           // [B] and [B, pad] rows
  int S, pad, x_chunks, l_chunks;
};
// A row a block: row r < pad of the history is token S - pad + r's latent, row pad the last token's input.  A few KB a sequence: bound by the launch.
constexpr int TS_THREADS = 256;
__global__ void __launch_bounds__(TS_THREADS) paged_token_state_kernel(TsArgs a) {
  pdl_enter();
  const int b = blockIdx.y, r = blockIdx.x;
  if (a.len[b] < 0) return;                                 // not in use
  const bool input = r == a.pad;
  const int chunks = input ? a.x_chunks : a.l_chunks, token = input ? a.S - 1 : a.S - a.pad + r;
  const uint4* from = (input ? a.x : a.qk0) + ((size_t)b * a.S + max(token, 0)) * chunks;
  uint4* to = input ? a.x_prev + (size_t)b * chunks : a.hist + ((size_t)b * a.pad + r) * chunks;
  for (int i = threadIdx.x; i < chunks; i += TS_THREADS) to[i] = token >= 0 ? from[i] : make_uint4(0, 0, 0, 0);
}

// ------------------------------------------------------------------------------------------------ attention
struct PaArgs {
  Paged c;
  const bf16* q;
  const float* q32;
  bf16* o;                // [B, hq, DH]
  float* lse;             // [B, hq] or null
  int B, hk, g, hq;
  int heads, n_grp;       // query heads per pass over a kv head's rows, passes
  int extra, max_len;
  int ctas;               // of the attention kernel that shares its units out
  float* part_o;          // [2 ctas][8][DH]
  float2* part_ml;        // [2 ctas][8]
  int* status;
};

// How a warp's rows go through shared memory: R rows of keys and values a stage.
template <int DH>
struct At {
  static constexpr int R = DH >= 128 ? 16 : DH == 64 ? 32 : 64;
  static constexpr int WARPS = 4, STAGES = 3, CTAS = DH == 256 ? 1 : 2;
  static constexpr int ROW = DH * 2, HALF = R * ROW, STAGE = 2 * HALF;
  static constexpr int CH = DH / 8;              // 16-byte pieces of a row
  static constexpr int UNIT = WARPS * R;         // rows a CTA takes at once
  static constexpr int OLD = DH + 4;             // stride of a head's sums in shared memory (no bank conflicts)
  static constexpr int RING = WARPS * STAGES * STAGE;
  static constexpr size_t smem(int hg) { return RING + (size_t)WARPS * hg * OLD * 4; }
  // Place of a 16-byte piece of a row: eight rows that an ldmatrix reads lie in different banks.
  static CCA_DEVINL int place(int row, int piece) {
    return DH == 32 ? row * ROW + ((piece ^ ((row >> 1) & 3)) << 4) : row * ROW + ((piece ^ (row & 7)) << 4);
  }
};

CCA_DEVINL int rows_of(const PaArgs& a, int b) {              // -1: does not fit, or is not in use
  const int n = __ldcg(a.c.len + b);
  return n >= 0 && n <= a.max_len - a.extra && n + a.extra <= (long long)a.c.max_pages * a.c.P ? n + a.extra : -1;
}

// The list of units: sequences in order, in each its kv heads (and passes over them), in each its units of rows.  It is cut into `used`
// parts, one for each CTA that has something to do, the first `more` of them one unit longer than the others.  (B max_len <= 2^30: less
// than 2^31 units.)
struct Plan {
  unsigned units, used, each, more, groups;
  CCA_DEVINL unsigned begin(unsigned cta) const { return cta * each + min(cta, more); }
  CCA_DEVINL int owner(unsigned unit) const {
    const unsigned longer = more * (each + 1);
    return (int)(unit < longer ? unit / (each + 1) : more + (unit - longer) / each);
  }
};

CCA_DEVINL unsigned warp_upto(unsigned v, int lane) {         // sum over the lanes up to this one
#pragma unroll
  for (int s = 1; s < 32; s <<= 1) {
    const unsigned x = __shfl_up_sync(0xffffffffu, v, s);
    if (lane >= s) v += x;
  }
  return v;
}
template <int UNIT>
CCA_DEVINL unsigned tiles_of(int rows) { return (unsigned)(max(rows, 0) + UNIT - 1) / UNIT; }

// Every warp for itself, from the lengths: the plan, and the sequence that `pick(plan)`, a tile of the sequences laid end to end (each taken
// once, not once a kv head), belongs to, with its rows and the tiles before it.  seq = -1: there is no such tile.
template <int UNIT, typename Pick>
CCA_DEVINL Plan make_plan(const PaArgs& a, int lane, Pick pick, int& seq, int& rows, unsigned& before) {
  constexpr int KEPT = 4;                                      // rows of the first 128 sequences stay in registers
  int n[KEPT];
  unsigned total = 0;
#pragma unroll
  for (int i = 0; i < KEPT; ++i) n[i] = i * 32 + lane < a.B ? rows_of(a, i * 32 + lane) : 0;
#pragma unroll
  for (int i = 0; i < KEPT; ++i) total += tiles_of<UNIT>(n[i]);
  for (int b = KEPT * 32 + lane; b < a.B; b += 32) total += tiles_of<UNIT>(rows_of(a, b));
  total = __reduce_add_sync(0xffffffffu, total);
  Plan p;
  p.groups = a.hk * a.n_grp;
  p.units = total * p.groups;
  p.used = min((unsigned)a.ctas, p.units);
  p.each = p.used > 0 ? p.units / p.used : 0;
  p.more = p.units - p.each * p.used;
  seq = -1;
  before = 0;
  const unsigned want = pick(p);
  if (want >= total) return p;
  for (int i = 0; seq < 0 && i * 32 < a.B; ++i) {
    int here = 0;
#pragma unroll
    for (int x = 0; x < KEPT; ++x)
      if (i == x) here = n[x];
    if (i >= KEPT) here = i * 32 + lane < a.B ? rows_of(a, i * 32 + lane) : 0;
    const unsigned tiles = tiles_of<UNIT>(here), upto = warp_upto(tiles, lane);
    const unsigned hit = __ballot_sync(0xffffffffu, want < before + upto);
    if (hit) {
      const int l = __ffs(hit) - 1;
      seq = i * 32 + l;
      rows = __shfl_sync(0xffffffffu, here, l);
      before += __shfl_sync(0xffffffffu, upto - tiles, l);
    } else {
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
  }
  return p;
}

template <int DH>
struct Cursor {
  int b, j, tile, tiles, rows;
  CCA_DEVINL void next(const PaArgs& a) {
    if (++tile < tiles) return;
    tile = 0;
    if (++j < a.hk * a.n_grp) return;
    j = 0;
    do {
      ++b;
      rows = b < a.B ? rows_of(a, b) : 1;                      // (behind the last: never used)
    } while (rows <= 0);
    tiles = (rows + At<DH>::UNIT - 1) / At<DH>::UNIT;
  }
};

// Softmax and both products in one pass, for the query heads that share a kv head, over rows that pages scatter.  Of a unit each warp takes R rows: lanes look their
// pages up one stage ahead and bring the rows by cp.async, 16 bytes a lane, into places from which ldmatrix reads without conflicts (a page may
// begin and end anywhere; a row is whole); S = Q K^T and O^T += V^T P^T by mma.sync, heads being 8 of its rows, then its 8 columns.  With 4
// heads or fewer the columns hold the weights' two bf16 parts, with more there are two products.  (tcgen05 would want 128 rows in its M: heads
// are 4, and what bounds the kernel is memory: 32 x 16384 rows, 8/2 heads x 128, 537 MB in 80 us = 6.7 TB/s, 1.02 of the measured copy rate,
// with issue at 22 % and the tensor pipe below that.  A CTA alone is bound by cp.async's way through the SM, 40 bytes a cycle.)
// JOINED: the CTAs of a cluster share the rows of one (sequence, kv head) and join their results through each other's shared memory.
// Otherwise every CTA takes its part of the list of units, and paged_join_kernel joins what several CTAs had part in.
template <int DH, int HG, bool JOINED>
__global__ void __launch_bounds__(At<DH>::WARPS * 32, At<DH>::CTAS) paged_attn_kernel(PaArgs a) {
  using S = At<DH>;
  constexpr int NT = S::WARPS * 32, MT = DH / 16, R = S::R, NB = R / 16, RL = R > 32 ? 2 : 1;
  constexpr int PARTS = HG == 4 ? 1 : 2;                       // accumulator tiles of the weights' two parts
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ float2 sm_ml[S::WARPS][8];
  __shared__ float2 cta_ml[8];                                 // JOINED: what the others of the cluster read
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  float* sm_o = reinterpret_cast<float*>(smem + S::RING);      // [WARPS][HG][OLD]
  pdl_enter();

  // ---- this CTA's units
  const int ranks = JOINED ? gridDim.x : 1, cta = blockIdx.x;
  Cursor<DH> cur = {0, 0, 0, 1, 0}, ld;                        // (no rows: a CTA without units)
  int to_load = 0;
  if (JOINED) {
    cur.b = blockIdx.z;
    cur.j = blockIdx.y;
    cur.rows = rows_of(a, cur.b);
    cur.tiles = tiles_of<S::UNIT>(cur.rows);
    cur.tile = cur.tiles * cta / ranks;
    to_load = cur.tiles * (cta + 1) / ranks - cur.tile;
  } else {
    unsigned before;
    int seq, rows;
    const Plan plan = make_plan<S::UNIT>(a, lane, [&](const Plan& p) { return cta < p.used ? p.begin(cta) / p.groups : 0xffffffffu; },
                                         seq, rows, before);
    if (seq >= 0) {
      cur.b = seq;
      cur.rows = rows;
      cur.tiles = tiles_of<S::UNIT>(rows);
      const unsigned u0 = plan.begin(cta), rem = u0 - before * plan.groups;
      cur.j = rem / cur.tiles;
      cur.tile = rem - cur.j * cur.tiles;
      to_load = plan.begin(cta + 1) - u0;
    }
  }
  // sequences without rows
  auto no_rows = [&](int b, int h0, int n) {
    const int rows = rows_of(a, b);
    if (rows > 0) return;
    if (rows < 0) {                                            // too long; not in use if the length is negative
      if (tid == 0 && a.c.len[b] >= 0) atomicCAS(a.status, 0, ST_PAGE_MISSING);
      return;
    }
    const size_t head = (size_t)b * a.hq + h0;
    for (int i = tid; i < n * DH; i += NT) a.o[head * DH + i] = __float2bfloat16(0.f);
    if (a.lse)
      for (int i = tid; i < n; i += NT) a.lse[head + i] = -INFINITY;
  };
  if (JOINED && cur.rows <= 0) {                               // the same in the whole cluster
    const int j = cur.j / a.n_grp, h0 = (cur.j - j * a.n_grp) * a.heads;
    if (cta == 0) no_rows(cur.b, j * a.g + h0, min(a.heads, a.g - h0));
    return;
  }

  // ---- loads: a lane knows the pool row of its row of the warp's next stage, looked up one stage ahead
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * (S::STAGES * S::STAGE);
  struct Stage {                                               // one to be loaded: its rows (below `rows` where there is one) and their pages
    int j, row, rows, entry[RL];
  };
  int ahead = to_load;                                         // units that have not been looked up
  ld = cur;
  auto look_up = [&] {
    Stage x;
    x.j = ld.j;
    x.row = ld.tile * S::UNIT + warp * R + (R < 32 ? lane % R : lane);
    x.rows = ahead > 0 ? ld.rows : 0;
#pragma unroll
    for (int i = 0; i < RL; ++i)                               // (nothing is done with an entry before its stage's turn: it is on its way)
      x.entry[i] = x.row + i * 32 < x.rows ? a.c.table[(size_t)ld.b * a.c.max_pages + page_index(a.c, x.row + i * 32)] : -1;
    if (--ahead > 0) {
      if (JOINED) ++ld.tile;
      else ld.next(a);
    }
    return x;
  };
  auto issue = [&](const Stage& x, int slot, uint32_t* mask) {
    const int j = x.j / a.n_grp;
    int at[RL];
#pragma unroll
    for (int i = 0; i < RL; ++i) {
      const int row = x.row + i * 32;
      at[i] = -1;
      if ((unsigned)x.entry[i] < (unsigned)a.c.n_pages) at[i] = pool_row(a.c, a.hk, x.entry[i], j, row - page_index(a.c, row) * a.c.P);
      else if (row < x.rows) atomicCAS(a.status, 0, ST_PAGE_MISSING);
      mask[i] = __ballot_sync(0xffffffffu, at[i] >= 0);
    }
    bool any = mask[0] != 0;
    if (RL > 1) any = any || mask[RL - 1] != 0;
    if (any) {
      const uint32_t to = ring + slot * S::STAGE;
      constexpr int PER = 32 / S::CH;                          // rows a warp copies at once
#pragma unroll
      for (int i = 0; i < R / PER; ++i) {
        const int row = i * PER + lane / S::CH, piece = lane % S::CH;
        const int from = __shfl_sync(0xffffffffu, at[i * PER / 32], row & 31);
        const size_t off = (size_t)max(from, 0) * DH + piece * 8;
        copy_async(to + S::place(row, piece), a.c.k + off, from >= 0);
        copy_async(to + S::HALF + S::place(row, piece), a.c.v + off, from >= 0);
      }
    }
  };
  uint32_t masks[S::STAGES - 1][RL];                           // rows there are, of the stages on their way
  Stage next;
  {
    Stage first[S::STAGES - 1];
#pragma unroll
    for (int s = 0; s < S::STAGES - 1; ++s) first[s] = look_up();
    next = look_up();
#pragma unroll
    for (int s = 0; s < S::STAGES - 1; ++s) {
      issue(first[s], s, masks[s]);
      copies_commit();
    }
  }
  if (!JOINED) {
    for (int b = cta; b < a.B; b += gridDim.x) no_rows(b, 0, a.hq);
    if (to_load == 0) return;
  }
  int to_do = to_load;

  // ---- queries: row r of the 16-row operand is head r (HG = 4: r % 4), rows 8 to 15 are zero
  uint32_t qa[MT][2];
  int nh = 0, h0 = 0;
  auto load_q = [&] {
    const int j = cur.j / a.n_grp;
    h0 = (cur.j - j * a.n_grp) * a.heads;
    nh = min(a.heads, a.g - h0);
    const int head = HG == 4 ? g & 3 : g;
    const size_t at = ((size_t)cur.b * a.hq + j * a.g + h0 + head) * DH + 2 * t;
#pragma unroll
    for (int ks = 0; ks < MT; ++ks) {
      qa[ks][0] = qa[ks][1] = 0;
      if (head < nh) {
        if (a.q32) {
          const float2 lo = *reinterpret_cast<const float2*>(a.q32 + at + ks * 16), hi = *reinterpret_cast<const float2*>(a.q32 + at + ks * 16 + 8);
          qa[ks][0] = pack_bf16x2(lo.x, lo.y);
          qa[ks][1] = pack_bf16x2(hi.x, hi.y);
        } else {
          qa[ks][0] = *reinterpret_cast<const uint32_t*>(a.q + at + ks * 16);
          qa[ks][1] = *reinterpret_cast<const uint32_t*>(a.q + at + ks * 16 + 8);
        }
      }
    }
  };
  // softmax state of head g (HG = 4: g % 4) in units of log2; the sum is this lane's part
  float top, sum, o[PARTS][MT][4];
  auto fresh = [&] {
    top = -INFINITY;
    sum = 0.f;
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[p][mt][c] = 0.f;
  };
  load_q();
  fresh();
  bool from_start = cur.tile == 0;
  const float scale = rsqrtf((float)DH) * LOG2E;

  // The CTA's result for channels c .. c + 3 of head h from its warps' (which lie in shared memory): sums under the maximum mx.
  auto of_warps = [&](int h, int c, float& mx, float& l) {
    float2 ml[S::WARPS];
    mx = -INFINITY;
    l = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < S::WARPS; ++w) {
      ml[w] = sm_ml[w][h];
      mx = fmaxf(mx, ml[w].x);
    }
#pragma unroll
    for (int w = 0; w < S::WARPS; ++w) {
      const float f = mx == -INFINITY ? 1.f : exp2f(ml[w].x - mx);
      const float4 x = *reinterpret_cast<const float4*>(&sm_o[(w * HG + h) * S::OLD + c]);
      l += ml[w].y * f;
      v.x += x.x * f; v.y += x.y * f; v.z += x.z * f; v.w += x.w * f;
    }
    return v;
  };
  auto put = [&](int h, int c, float4 v, float mx, float l) {
    const size_t head = (size_t)cur.b * a.hq + (cur.j / a.n_grp) * a.g + h0 + h;
    const float f = l == 0.f ? 0.f : 1.f / l;
    *reinterpret_cast<uint2*>(a.o + head * DH + c) = make_uint2(pack_bf16x2(v.x * f, v.y * f), pack_bf16x2(v.z * f, v.w * f));
    if (c == 0 && a.lse) a.lse[head] = (mx + log2f(l)) * LN2;
  };
  auto leave_warps = [&] {                                     // this warp's result into shared memory
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    float* so = sm_o + warp * HG * S::OLD;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float v = o[0][mt][c];
        const int ch = mt * 16 + g + 8 * (c >> 1);
        if (HG == 4) {
          v = both_parts(v, __shfl_xor_sync(0xffffffffu, v, 2));      // (used where t < 2, whose columns are the first parts)
          if (t < 2) so[(2 * t + (c & 1)) * S::OLD + ch] = v;
        } else {
          so[(2 * t + (c & 1)) * S::OLD + ch] = both_parts(v, o[PARTS - 1][mt][c]);
        }
      }
    if (t == 0) sm_ml[warp][g] = make_float2(top, sum);
    __syncthreads();
  };

  for (int slot = 0; to_do > 0; --to_do, slot = slot + 1 == S::STAGES ? 0 : slot + 1) {
    copies_wait<S::STAGES - 2>();
    __syncwarp();
    uint32_t mask[RL];
#pragma unroll
    for (int x = 0; x < RL; ++x) {
      mask[x] = masks[0][x];
#pragma unroll
      for (int s = 0; s + 1 < S::STAGES - 1; ++s) masks[s][x] = masks[s + 1][x];
    }
    issue(next, slot == 0 ? S::STAGES - 1 : slot - 1, masks[S::STAGES - 2]);
    copies_commit();
    next = look_up();
    bool any = mask[0] != 0, all = mask[0] == 0xffffffffu;
    if (RL > 1) { any = any || mask[RL - 1] != 0; all = all && mask[RL - 1] == 0xffffffffu; }
    if (any) {
      const uint32_t kb = ring + slot * S::STAGE, vb = kb + S::HALF;
      const int lrow = ((lane >> 4) << 3) + (lane & 7), lpiece = (lane >> 3) & 1;
      float s[2 * NB][4];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
        for (int c = 0; c < 4; ++c) s[2 * nb][c] = s[2 * nb + 1][c] = 0.f;
#pragma unroll
        for (int ks = 0; ks < MT; ++ks) {
          uint32_t kf[4];
          const uint32_t qf[4] = {qa[ks][0], 0u, qa[ks][1], 0u};
          ldmatrix_x4(kf, kb + S::place(nb * 16 + lrow, 2 * ks + lpiece));
          mma_16816(s[2 * nb], qf, kf[0], kf[1]);
          mma_16816(s[2 * nb + 1], qf, kf[2], kf[3]);
        }
      }
      float most = -INFINITY;
#pragma unroll
      for (int i = 0; i < 2 * NB; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          s[i][c] *= scale;
          if (!all && !((mask[RL > 1 ? i >> 2 : 0] >> ((i * 8 + 2 * t + c) & 31)) & 1)) s[i][c] = -INFINITY;
          most = fmaxf(most, s[i][c]);
        }
      most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
      most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
      if (__any_sync(0xffffffffu, most > top)) {
        const float now = fmaxf(top, most);
        const float alpha = now == -INFINITY ? 1.f : exp2f(top - now);
        top = now;
        sum *= alpha;
        const float a0 = __shfl_sync(0xffffffffu, alpha, 8 * t), a1 = __shfl_sync(0xffffffffu, alpha, 8 * t + 4);
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            o[p][mt][0] *= a0; o[p][mt][1] *= a1; o[p][mt][2] *= a0; o[p][mt][3] *= a1;
          }
      }
      const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        // weights as two bf16 parts that together hold 16 bits: HG = 4: heads' first parts are the columns 0 to 3 and their second
        // parts the columns 4 to 7 of one operand
        uint32_t pb[PARTS][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float p0 = exp2f(s[2 * nb + i][0] - ref), p1 = exp2f(s[2 * nb + i][1] - ref);
          sum += p0 + p1;
          const uint32_t w = pack_bf16x2(p0, p1), rest = pack_bf16x2(p0 - bf_lo(w), p1 - bf_hi(w));
          if (HG == 4) {
            pb[0][i] = g < 4 ? w : rest;
          } else {
            pb[0][i] = w;
            pb[PARTS - 1][i] = rest;
          }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          uint32_t vf[4];
          ldmatrix_x4_trans(vf, vb + S::place(nb * 16 + lrow, 2 * mt + lpiece));
#pragma unroll
          for (int p = 0; p < PARTS; ++p) mma_16816(o[p][mt], vf, pb[p][0], pb[p][1]);
        }
      }
    }
    if (JOINED) continue;
    // ---- the end of a run of units of one (sequence, kv head): the warps' results are joined
    const bool ends = cur.tile + 1 == cur.tiles;
    if (ends || to_do == 1) {
      leave_warps();
      const bool whole = from_start && ends;
      const int slot_of = cta * 2 + (from_start ? 1 : 0);      // a run that begins here and one that began before
      for (int i = tid; i < nh * DH / 4; i += NT) {
        const int h = i / (DH / 4), c = i % (DH / 4) * 4;
        float mx, l;
        const float4 v = of_warps(h, c, mx, l);
        if (whole) {
          put(h, c, v, mx, l);
        } else {
          const size_t p = (size_t)slot_of * 8 + h;
          __stcg(reinterpret_cast<float4*>(a.part_o + p * DH + c), v);
          if (c == 0) __stcg(a.part_ml + p, make_float2(mx, l));
        }
      }
      if (to_do > 1) {
        cur.next(a);
        from_start = true;
        load_q();
        fresh();
        __syncthreads();
      }
    } else {
      ++cur.tile;
    }
  }
  if (!JOINED) return;

  // ---- the cluster's results
  leave_warps();
  if (ranks == 1) {
    for (int i = tid; i < nh * DH / 4; i += NT) {
      const int h = i / (DH / 4), c = i % (DH / 4) * 4;
      float mx, l;
      const float4 v = of_warps(h, c, mx, l);
      put(h, c, v, mx, l);
    }
    return;
  }
  float* cta_o = reinterpret_cast<float*>(smem);               // [nh][DH], where the loads are over
  copies_wait<0>();
  __syncthreads();
  for (int i = tid; i < nh * DH / 4; i += NT) {
    const int h = i / (DH / 4), c = i % (DH / 4) * 4;
    float mx, l;
    *reinterpret_cast<float4*>(&cta_o[h * DH + c]) = of_warps(h, c, mx, l);
    if (c == 0) cta_ml[h] = make_float2(mx, l);
  }
  cluster_barrier();
  const int share = nh * DH / 4 / ranks;                       // (DH / 4 is a multiple of 8)
  for (int i = cta * share + tid; i < (cta + 1) * share; i += NT) {
    const int h = i / (DH / 4), c = i % (DH / 4) * 4;
    float mx = -INFINITY, l = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f), part[8];
    float2 ml[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      ml[x] = x < ranks ? cluster_float2(&cta_ml[h], x) : make_float2(-INFINITY, 0.f);
      part[x] = x < ranks ? cluster_float4(&cta_o[h * DH + c], x) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int x = 0; x < 8; ++x) mx = fmaxf(mx, ml[x].x);
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const float f = mx == -INFINITY ? 1.f : exp2f(ml[x].x - mx);
      l += ml[x].y * f;
      v.x += part[x].x * f; v.y += part[x].y * f; v.z += part[x].z * f; v.w += part[x].w * f;
    }
    put(h, c, v, mx, l);
  }
  cluster_barrier();                                           // nobody leaves while its memory may be read
}

// Joins the partial results of a run of units that several CTAs shared, 4 CL channels of one head, in a fixed order, so the same every
// time.  Which run: the x-th (sequence, kv head) or, where there are more of those than CTAs, the one that begins in CTA x of the attention
// and is not over there.  That is worked out from the lengths while the attention is still running (pdl.cuh says why they can be read).  A slice of
// CL lanes takes one part at a time, four channels a lane; a head's slices are those of a warp (ONE) or of the CTA.
constexpr int PJ_WARPS = 4, PJ_THREADS = PJ_WARPS * 32;
template <int DH, int CL, bool ONE>
__global__ void __launch_bounds__(PJ_THREADS) paged_join_kernel(PaArgs a, int by_run) {
  constexpr int UNIT = At<DH>::UNIT, SLICES = (ONE ? 32 : PJ_THREADS) / CL;
  __shared__ float4 red[PJ_WARPS][CL];
  __shared__ float2 red_ml[PJ_WARPS];
  const int x = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int h = ONE ? blockIdx.z * PJ_WARPS + warp : blockIdx.z;
  int b, rows = 0, j = 0, first = 0, last = 0;
  unsigned before;
  const Plan p = make_plan<UNIT>(a, lane, [&](const Plan& pl) {
    return by_run || x + 1 >= pl.used ? 0xffffffffu : (pl.begin(x + 1) - 1) / pl.groups;
  }, b, rows, before);
  if (by_run) {
    b = x / p.groups;
    j = x - b * p.groups;
    unsigned sum = 0;
    for (int i = lane; i < b; i += 32) sum += tiles_of<UNIT>(rows_of(a, i));
    before = __reduce_add_sync(0xffffffffu, sum);
    rows = rows_of(a, b);
  }
  const unsigned tiles = tiles_of<UNIT>(rows);
  bool work = b >= 0 && tiles > 0;
  if (work) {
    if (!by_run) j = (p.begin(x + 1) - 1 - before * p.groups) / tiles;
    const unsigned s0 = before * p.groups + j * tiles;
    first = p.owner(s0);
    last = p.owner(s0 + tiles - 1);
    work = last > first && (by_run || first == x);
  }
  pdl_enter();
  if (!work) return;
  const int parts = last - first + 1;
  const int kv = j / a.n_grp, h0 = (j - kv * a.n_grp) * a.heads;
  if (h >= min(a.heads, a.g - h0)) return;                     // (ONE: a warp alone; otherwise the whole CTA)
  float mx = -INFINITY, l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  auto factor = [](float m, float to) { return to == -INFINITY ? 1.f : exp2f(m - to); };
  auto add = [&](float4 v, float2 ml) {
    const float now = fmaxf(mx, ml.x), f0 = factor(mx, now), f1 = factor(ml.x, now);
    acc.x = acc.x * f0 + v.x * f1; acc.y = acc.y * f0 + v.y * f1;
    acc.z = acc.z * f0 + v.z * f1; acc.w = acc.w * f0 + v.w * f1;
    l = l * f0 + ml.y * f1;
    mx = now;
  };
  const int c = (blockIdx.y * CL + lane % CL) * 4;
  constexpr int AHEAD = 4;                                     // parts of a slice on their way
  for (int q0 = (ONE ? lane : tid) / CL; q0 < parts; q0 += AHEAD * SLICES) {
    float4 v[AHEAD];
    float2 ml[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int q = q0 + k * SLICES;
      v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      ml[k] = make_float2(-INFINITY, 0.f);
      if (q < parts) {
        const size_t slot = (size_t)((first + q) * 2 + (q == 0 ? 1 : 0)) * 8 + h;
        v[k] = __ldcg(reinterpret_cast<const float4*>(a.part_o + slot * DH + c));
        ml[k] = __ldcg(a.part_ml + slot);
      }
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) add(v[k], ml[k]);
  }
#pragma unroll
  for (int s = CL; s < 32; s <<= 1) {
    const float2 ml = make_float2(__shfl_xor_sync(0xffffffffu, mx, s), __shfl_xor_sync(0xffffffffu, l, s));
    add(make_float4(__shfl_xor_sync(0xffffffffu, acc.x, s), __shfl_xor_sync(0xffffffffu, acc.y, s),
                    __shfl_xor_sync(0xffffffffu, acc.z, s), __shfl_xor_sync(0xffffffffu, acc.w, s)), ml);
  }
  if (!ONE) {
    if (lane < CL) red[warp][lane] = acc;
    if (lane == 0) red_ml[warp] = make_float2(mx, l);
    __syncthreads();
    if (tid >= CL) return;
#pragma unroll
    for (int w = 1; w < PJ_WARPS; ++w) add(red[w][tid], red_ml[w]);
  }
  if (lane >= CL) return;
  const size_t head = (size_t)b * a.hq + kv * a.g + h0 + h;
  const float f = l == 0.f ? 0.f : 1.f / l;
  *reinterpret_cast<uint2*>(a.o + head * DH + c) = make_uint2(pack_bf16x2(acc.x * f, acc.y * f), pack_bf16x2(acc.z * f, acc.w * f));
  if (a.lse && blockIdx.y == 0 && lane == 0) a.lse[head] = (mx + log2f(l)) * LN2;
}

int attn_ctas(int dh, int sm_count) { return sm_count * (dh == 256 ? 1 : 2); }

template <int DH, int HG, bool JOINED>
cudaError_t launch_attn(const PaArgs& a, dim3 grid, int ranks, cudaStream_t st) {
  static bool done[MAX_DEVICES];
  const cudaError_t e = opt_in(paged_attn_kernel<DH, HG, JOINED>, (int)At<DH>::smem(HG), done);
  if (e != cudaSuccess) return e;
  if (JOINED) return launch_clusters(paged_attn_kernel<DH, HG, JOINED>, grid, dim3(At<DH>::WARPS * 32), At<DH>::smem(HG), ranks, st, a);
  return launch_pdl_smem(paged_attn_kernel<DH, HG, JOINED>, grid, dim3(At<DH>::WARPS * 32), At<DH>::smem(HG), st, a);
}

// CTAs of clusters of 1, 2, 4 and 8 that find room on the device at once (a cluster lies within a part of it), asked for once a device; -1: not even one.
template <int DH, int HG>
cudaError_t cluster_room(int* room) {
  static int known[MAX_DEVICES][PA_SIZES];                     // 0: not asked
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  static bool done[MAX_DEVICES];
  for (int i = 0; i < PA_SIZES; ++i) {
    room[i] = dev < MAX_DEVICES ? known[dev][i] : 0;
    if (room[i] != 0) continue;
    if ((e = opt_in(paged_attn_kernel<DH, HG, true>, (int)At<DH>::smem(HG), done)) != cudaSuccess) return e;
    int n = 0;
    if ((e = clusters_at_once(paged_attn_kernel<DH, HG, true>, dim3(At<DH>::WARPS * 32), At<DH>::smem(HG), 1 << i, &n)) != cudaSuccess) return e;
    room[i] = cluster_ctas(n, 1 << i);
    if (dev < MAX_DEVICES) known[dev][i] = room[i];
  }
  return cudaSuccess;
}

// Few parts a run: a warp for a head, 16 parts of 32 channels at once.  Many: a CTA for a head, 256 parts of 8 channels.
template <int DH>
cudaError_t launch_join(const PaArgs& a, long long runs, cudaStream_t st) {
  const int by_run = runs <= a.ctas;
  const unsigned x = (unsigned)(by_run ? runs : a.ctas), z = (unsigned)a.heads;
  if (a.ctas / runs <= 8) return launch_pdl(paged_join_kernel<DH, 8, true>, dim3(x, DH / 32, (z + 3) / 4), dim3(PJ_THREADS), st, a, by_run);
  return launch_pdl(paged_join_kernel<DH, 2, false>, dim3(x, DH / 8, z), dim3(PJ_THREADS), st, a, by_run);
}

template <int DH>
int launch_attention_dh(PaArgs a, int sm_count, long long* launches, cudaEvent_t ev_begin, cudaEvent_t ev_end, cudaStream_t st) {
  cudaError_t e;
  if (ev_begin && (e = cudaEventRecord(ev_begin, st)) != cudaSuccess) return -(int)e;
  const long long runs = (long long)a.B * a.hk * a.n_grp;
  int room[PA_SIZES];
  if ((e = a.heads <= 4 ? cluster_room<DH, 4>(room) : cluster_room<DH, 8>(room)) != cudaSuccess) return -(int)e;
  const long long tiles = (a.max_len + At<DH>::UNIT - 1) / At<DH>::UNIT;
  const int ranks = paged_join_ranks(DH, runs, tiles, attn_ctas(DH, sm_count), room);
  if (ranks > 0) {
    const dim3 grid((unsigned)ranks, (unsigned)(a.hk * a.n_grp), (unsigned)a.B);
    e = a.heads <= 4 ? launch_attn<DH, 4, true>(a, grid, ranks, st) : launch_attn<DH, 8, true>(a, grid, ranks, st);
  } else {
    const long long units = runs * tiles, most = attn_ctas(DH, sm_count);
    a.ctas = (int)(units < most ? units : most);
    const dim3 grid((unsigned)a.ctas);
    e = a.heads <= 4 ? launch_attn<DH, 4, false>(a, grid, 0, st) : launch_attn<DH, 8, false>(a, grid, 0, st);
  }
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  if (ev_end && (e = cudaEventRecord(ev_end, st)) != cudaSuccess) return -(int)e;
  if (ranks > 0) return 0;
  e = launch_join<DH>(a, runs, st);
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  return 0;
}

}  // namespace

int launch_paged_append(const CcaDims& d, const bf16* k, const bf16* v, const int* count, const Paged& c, long long n, int* status,
                        long long* launches, cudaStream_t st) {
  RowsArgs a;
  memset(&a, 0, sizeof(a));
  a.c = c; a.B = d.B; a.hk = d.hk; a.row_chunks = d.dh / 8; a.k_in = k; a.v_in = v; a.count = count; a.n = n; a.status = status;
  const cudaError_t e = launch_pdl(paged_rows_kernel<true>, dim3((unsigned)((n + RW_TOKENS - 1) / RW_TOKENS), (unsigned)d.B),
                                   dim3(RW_THREADS), st, a);
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  return 0;
}

int launch_paged_read(const CcaDims& d, const Paged& c, const int* first, bf16* k, bf16* v, long long n, long long* launches,
                      cudaStream_t st) {
  RowsArgs a;
  memset(&a, 0, sizeof(a));
  a.c = c; a.B = d.B; a.hk = d.hk; a.row_chunks = d.dh / 8; a.k_out = k; a.v_out = v; a.first = first; a.n = n;
  const cudaError_t e = launch_pdl(paged_rows_kernel<false>, dim3((unsigned)((n + RW_TOKENS - 1) / RW_TOKENS), (unsigned)d.B),
                                   dim3(RW_THREADS), st, a);
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  return 0;
}

int launch_paged_token_state(const CcaDims& d, const Paged& c, const bf16* x, const float* qk0, bf16* x_prev, float* hist, long long* launches,
                             cudaStream_t st) {
  const int pad = d.k_seq + d.k_ch - 2;                     // (d_model is a multiple of 8, a latent row of 4)
  const TsArgs a{c.len, reinterpret_cast<const uint4*>(x), reinterpret_cast<const uint4*>(qk0), reinterpret_cast<uint4*>(x_prev),
                 reinterpret_cast<uint4*>(hist), d.S, pad, d.E / 8, d.L / 4};
  const cudaError_t e = launch_pdl(paged_token_state_kernel, dim3((unsigned)(pad + 1), (unsigned)d.B), dim3(TS_THREADS), st, a);
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  return 0;
}

namespace {
struct PagedLayout { size_t part_o, part_ml, end; };
PagedLayout paged_layout(const CcaDims& d, int sm_count) {
  const size_t ctas = attn_ctas(d.dh, sm_count);
  PagedLayout l;
  size_t off = 0;
  auto take = [&](size_t n) { const size_t o = off; off += (n + 255) / 256 * 256; return o; };
  l.part_o = take(ctas * 2 * 8 * d.dh * 4);
  l.part_ml = take(ctas * 2 * 8 * 8);
  l.end = off;
  return l;
}
}  // namespace

size_t paged_workspace_bytes(const CcaDims& d, int max_len, int sm_count) {
  (void)max_len;                                               // partial results are counted by CTAs
  return paged_layout(d, sm_count).end;
}

int launch_paged_attention(const CcaDims& d, const bf16* q, const float* q32, bf16* o, float* lse, const Paged& c, int extra, int max_len,
                           void* workspace, int sm_count, int* status, long long* launches, cudaEvent_t ev_begin, cudaEvent_t ev_end,
                           cudaStream_t st) {
  const PagedLayout l = paged_layout(d, sm_count);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  PaArgs a;
  memset(&a, 0, sizeof(a));
  a.c = c; a.q = q; a.q32 = q32; a.o = o; a.lse = lse; a.B = d.B; a.hk = d.hk; a.g = d.g; a.hq = d.hq;
  a.n_grp = (d.g + 7) / 8;
  a.heads = (d.g + a.n_grp - 1) / a.n_grp;
  a.extra = extra; a.max_len = max_len; a.status = status;
  a.part_o = reinterpret_cast<float*>(ws + l.part_o);
  a.part_ml = reinterpret_cast<float2*>(ws + l.part_ml);
  switch (d.dh) {
    case 32: return launch_attention_dh<32>(a, sm_count, launches, ev_begin, ev_end, st);
    case 64: return launch_attention_dh<64>(a, sm_count, launches, ev_begin, ev_end, st);
    case 128: return launch_attention_dh<128>(a, sm_count, launches, ev_begin, ev_end, st);
    case 256: return launch_attention_dh<256>(a, sm_count, launches, ev_begin, ev_end, st);
    default: return 1;
  }
}
