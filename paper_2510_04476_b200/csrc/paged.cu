// A latent cache in pages: rows put in and read back, and attention of one new token per sequence over them.
#include <cstring>

#include "cluster.cuh"
#include "common.cuh"
#include "paged.cuh"
#include "pdl.cuh"

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

CCA_DEVINL uint32_t pack_bf16x2(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
CCA_DEVINL float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
CCA_DEVINL float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
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
constexpr int RW_TOKENS = 16, RW_THREADS = 256;

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
// are whole 64-byte pieces or more, so the kernel is bound by its traffic (each byte once in and once out).
template <bool APPEND>
__global__ void __launch_bounds__(RW_THREADS) paged_rows_kernel(RowsArgs a) {
  __shared__ int at[RW_TOKENS];                             // pool row of kv head 0, -1: none
  const int b = blockIdx.y, tid = threadIdx.x;
  const long long t0 = (long long)blockIdx.x * RW_TOKENS;
  pdl_enter();
  if (tid < RW_TOKENS) {
    int to = -1;
    const long long i = t0 + tid;
    const int held = a.first ? a.first[b] : a.c.len[b];
    long long n = a.n;
    if (APPEND && a.count) n = min(n, (long long)max(a.count[b], 0));
    if (i < n) {
      const long long row = held + i, most = (long long)a.c.max_pages * a.c.P;
      if (held >= 0 || !APPEND) {
        if (row >= 0 && row < most) {
          const int pi = page_index(a.c, (int)row), page = page_at(a.c, b, pi);
          if (page >= 0 && (!APPEND || a.c.refs[page] == 1)) to = pool_row(a.c, a.hk, page, 0, (int)row - pi * a.c.P);
        }
      }
      if (APPEND && to < 0) atomicCAS(a.status, 0, ST_PAGE_MISSING);
    }
    at[tid] = to;
  }
  __syncthreads();
  const int per_token = a.hk * a.row_chunks;
  const int here = (int)min((long long)RW_TOKENS, a.n - t0) * per_token;
  const uint4 *kd = reinterpret_cast<const uint4*>(a.k_in), *vd = reinterpret_cast<const uint4*>(a.v_in);
  uint4 *ko = reinterpret_cast<uint4*>(a.k_out), *vo = reinterpret_cast<uint4*>(a.v_out);
  uint4 *kp = reinterpret_cast<uint4*>(a.c.k), *vp = reinterpret_cast<uint4*>(a.c.v);
  const size_t dense0 = ((size_t)b * a.n + t0) * per_token;
#pragma unroll 2
  for (int x = tid; x < here; x += RW_THREADS) {
    const int token = x / per_token, in = x - token * per_token;
    const int j = in / a.row_chunks, piece = in - j * a.row_chunks;
    const size_t pool = (size_t)(at[token] + j * a.c.P) * a.row_chunks + piece;
    if (APPEND) {
      if (at[token] < 0) continue;
      const uint4 kx = __ldcs(kd + dense0 + x), vx = __ldcs(vd + dense0 + x);
      kp[pool] = kx;
      vp[pool] = vx;
    } else {
      uint4 kx = make_uint4(0, 0, 0, 0), vx = kx;
      if (at[token] >= 0) { kx = kp[pool]; vx = vp[pool]; }
      ko[dense0 + x] = kx;
      vo[dense0 + x] = vx;
    }
  }
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
  float* part_o;          // [2 G][8][DH]
  float2* part_ml;        // [2 G][8]
  int4* desc;             // [G]: what the join has to do: sequence, kv head and pass, last CTA
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

CCA_DEVINL int rows_of(const PaArgs& a, int b) {              // -1: does not fit
  const int n = a.c.len[b];
  return n >= 0 && n <= a.max_len - a.extra && n + a.extra <= (long long)a.c.max_pages * a.c.P ? n + a.extra : -1;
}

// Where a CTA is in the list of units: sequences in order, in each its kv heads (and passes), in each its units of rows.
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

template <int DH, int HG>
__global__ void __launch_bounds__(At<DH>::WARPS * 32, At<DH>::CTAS) paged_attn_kernel(PaArgs a) {
  using S = At<DH>;
  constexpr int NT = S::WARPS * 32, MT = DH / 16, R = S::R, NB = R / 16, RL = R > 32 ? 2 : 1;
  constexpr int PARTS = HG == 4 ? 1 : 2;                       // accumulator tiles of the weights' two parts
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ long long scan[S::WARPS];
  __shared__ long long found[2];
  __shared__ float2 sm_ml[S::WARPS][8];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int cta = blockIdx.x, n_cta = gridDim.x;
  float* sm_o = reinterpret_cast<float*>(smem + S::RING);      // [WARPS][HG][OLD]
  pdl_enter();

  // ---- this CTA's share of the units: all rows there are, in equal parts
  const int groups = a.hk * a.n_grp;
  long long total = 0, mine = 0;
  for (int b = tid; b < a.B; b += NT) mine += (max(rows_of(a, b), 0) + S::UNIT - 1) / S::UNIT;
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, s);
  if (lane == 0) scan[warp] = mine;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < S::WARPS; ++w) total += scan[w];
  const long long units = total * groups;
  const int used = (int)min((long long)n_cta, units);          // CTAs that have something to do
  // sequences without rows
  for (int b = cta; b < a.B; b += n_cta) {
    const int n = rows_of(a, b);
    if (n > 0) continue;
    if (n < 0) {
      if (tid == 0) atomicCAS(a.status, 0, ST_PAGE_MISSING);
      continue;
    }
    for (int i = tid; i < a.hq * DH; i += NT) a.o[(size_t)b * a.hq * DH + i] = __float2bfloat16(0.f);
    if (a.lse)
      for (int i = tid; i < a.hq; i += NT) a.lse[(size_t)b * a.hq + i] = -INFINITY;
  }
  if (cta >= used) {
    if (tid == 0) a.desc[cta] = make_int4(-1, 0, 0, 0);
    return;
  }
  const long long u0 = cta * units / used, u1 = (cta + 1) * units / used;
  const long long want = u0 / groups;
  {
    long long base = 0;
    for (int b0 = 0; b0 < a.B; b0 += NT) {                     // the sequence whose units hold `want`
      const int b = b0 + tid;
      const long long n = b < a.B ? (max(rows_of(a, b), 0) + S::UNIT - 1) / S::UNIT : 0;
      long long upto = n;
#pragma unroll
      for (int s = 1; s < 32; s <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, upto, s);
        if (lane >= s) upto += v;
      }
      __syncthreads();
      if (lane == 31) scan[warp] = upto;
      __syncthreads();
      long long before = base;
#pragma unroll
      for (int w = 0; w < S::WARPS; ++w) {
        if (w < warp) before += scan[w];
        base += scan[w];
      }
      if (want >= before + upto - n && want < before + upto) { found[0] = b; found[1] = before + upto - n; }
      if (want < base) break;
    }
    __syncthreads();
  }
  Cursor<DH> cur, ld;
  cur.b = (int)found[0];
  cur.rows = rows_of(a, cur.b);
  cur.tiles = (cur.rows + S::UNIT - 1) / S::UNIT;
  {
    const long long rem = u0 - found[1] * groups;
    cur.j = (int)(rem / cur.tiles);
    cur.tile = (int)(rem - (long long)cur.j * cur.tiles);
  }
  ld = cur;
  int to_load = (int)(u1 - u0), to_do = to_load;

  // ---- loads: a lane knows the pool row of its row of the warp's next stage, looked up one stage ahead
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * (S::STAGES * S::STAGE);
  int entry[RL];
  auto look_up = [&] {
#pragma unroll
    for (int x = 0; x < RL; ++x) {
      const int row = ld.tile * S::UNIT + warp * R + x * 32 + (R < 32 ? lane % R : lane);
      entry[x] = -1;
      if (to_load > 0 && row < ld.rows) {
        entry[x] = a.c.table[(size_t)ld.b * a.c.max_pages + page_index(a.c, row)];
        if ((unsigned)entry[x] >= (unsigned)a.c.n_pages) entry[x] = -2;
      }
    }
  };
  auto issue = [&](int slot, uint32_t* mask) {
    const int j = ld.j / a.n_grp;
    int at[RL];
#pragma unroll
    for (int x = 0; x < RL; ++x) {
      const int row = ld.tile * S::UNIT + warp * R + x * 32 + (R < 32 ? lane % R : lane);
      at[x] = entry[x] >= 0 ? pool_row(a.c, a.hk, entry[x], j, row - page_index(a.c, row) * a.c.P) : -1;
      if (entry[x] == -2) atomicCAS(a.status, 0, ST_PAGE_MISSING);
      mask[x] = __ballot_sync(0xffffffffu, at[x] >= 0);
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
    if (to_load > 0) {
      --to_load;
      if (to_load > 0) ld.next(a);
    }
    look_up();
  };
  uint32_t masks[S::STAGES - 1][RL];                           // rows there are, of the stages on their way
  look_up();
#pragma unroll
  for (int s = 0; s < S::STAGES - 1; ++s) {
    issue(s, masks[s]);
    copies_commit();
  }

  // ---- queries: row r of the 16-row operand is head r (HG = 4: r % 4), rows 8 to 15 are zero
  uint32_t qa[MT][4];
  int nh = 0, h0 = 0;
  auto load_q = [&] {
    const int j = cur.j / a.n_grp;
    h0 = (cur.j - j * a.n_grp) * a.heads;
    nh = min(a.heads, a.g - h0);
    const int head = HG == 4 ? g & 3 : g;
    const size_t at = ((size_t)cur.b * a.hq + j * a.g + h0 + head) * DH + 2 * t;
#pragma unroll
    for (int ks = 0; ks < MT; ++ks) {
      qa[ks][0] = qa[ks][1] = qa[ks][2] = qa[ks][3] = 0;
      if (head < nh) {
        if (a.q32) {
          const float2 lo = *reinterpret_cast<const float2*>(a.q32 + at + ks * 16), hi = *reinterpret_cast<const float2*>(a.q32 + at + ks * 16 + 8);
          qa[ks][0] = pack_bf16x2(lo.x, lo.y);
          qa[ks][2] = pack_bf16x2(hi.x, hi.y);
        } else {
          qa[ks][0] = *reinterpret_cast<const uint32_t*>(a.q + at + ks * 16);
          qa[ks][2] = *reinterpret_cast<const uint32_t*>(a.q + at + ks * 16 + 8);
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
  int which = 0;                                               // slot of this CTA's partial results: 1 for a run that begins here
  bool desc_set = false;
  const float scale = rsqrtf((float)DH) * LOG2E;

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
    issue(slot == 0 ? S::STAGES - 1 : slot - 1, masks[S::STAGES - 2]);
    copies_commit();
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
          ldmatrix_x4(kf, kb + S::place(nb * 16 + lrow, 2 * ks + lpiece));
          mma_16816(s[2 * nb], qa[ks], kf[0], kf[1]);
          mma_16816(s[2 * nb + 1], qa[ks], kf[2], kf[3]);
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
      // the maximum moves only when a logit passes it by a factor of 2^8: weights stay below 2^8 and nothing is lost in fp32
      if (__any_sync(0xffffffffu, most > top + 8.f || (top == -INFINITY && most != -INFINITY))) {
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
    // ---- the end of a run of units of one (sequence, kv head): the warps' results are joined
    const bool ends = cur.tile + 1 == cur.tiles;
    if (ends || to_do == 1) {
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
            v += __shfl_xor_sync(0xffffffffu, v, 2);
            if (t < 2) so[(2 * t + (c & 1)) * S::OLD + ch] = v;
          } else {
            so[(2 * t + (c & 1)) * S::OLD + ch] = v + o[PARTS - 1][mt][c];
          }
        }
      if (t == 0) sm_ml[warp][g] = make_float2(top, sum);
      __syncthreads();
      const bool whole = from_start && ends;
      const int j = cur.j / a.n_grp;
      which = from_start ? 1 : 0;
      for (int i = tid; i < nh * DH; i += NT) {
        const int h = i / DH, c = i % DH;
        float mx = -INFINITY;
#pragma unroll
        for (int w = 0; w < S::WARPS; ++w) mx = fmaxf(mx, sm_ml[w][h].x);
        float l = 0.f, v = 0.f;
#pragma unroll
        for (int w = 0; w < S::WARPS; ++w) {
          const float f = mx == -INFINITY ? 1.f : exp2f(sm_ml[w][h].x - mx);
          l += sm_ml[w][h].y * f;
          v += sm_o[(w * HG + h) * S::OLD + c] * f;
        }
        const size_t head = (size_t)cur.b * a.hq + j * a.g + h0 + h;
        if (whole) {
          a.o[head * DH + c] = __float2bfloat16(l == 0.f ? 0.f : v / l);
          if (c == 0 && a.lse) a.lse[head] = (mx + log2f(l)) * LN2;
        } else {
          const size_t p = ((size_t)(cta * 2 + which) * 8 + h);
          a.part_o[p * DH + c] = v;
          if (c == 0) a.part_ml[p] = make_float2(mx, l);
        }
      }
      if (from_start && !ends && tid == 0) {                   // the rest of this run is other CTAs': they join it up to the last one
        const long long end = u1 + (cur.tiles - 1 - cur.tile);  // unit behind the run's last
        a.desc[cta] = make_int4(cur.b, cur.j, (int)((end * used - 1) / units), 0);
      }
      if (from_start && !ends) desc_set = true;
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
  if (!desc_set && tid == 0) a.desc[cta] = make_int4(-1, 0, 0, 0);
}

// Joins the partial results of a run of units that several CTAs shared: CTA x is about the run that begins in CTA x of the attention
// and is not over there, 32 channels of it.  In the order of the CTAs, so the same every time.
constexpr int PJ_THREADS = 512, PJ_WARPS = PJ_THREADS / 32;
template <int DH>
__global__ void __launch_bounds__(PJ_THREADS) paged_join_kernel(PaArgs a) {
  extern __shared__ float factor[];                            // [8][parts]
  __shared__ float red[PJ_WARPS][8][32];
  __shared__ float total[8];
  pdl_enter();
  const int first = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int4 d = a.desc[first];
  if (d.x < 0) return;
  const int parts = d.z - first + 1;
  const int j = d.y / a.n_grp, h0 = (d.y - j * a.n_grp) * a.heads, nh = min(a.heads, a.g - h0);
  auto slot = [&](int p) { return (size_t)((first + p) * 2 + (p == 0 ? 1 : 0)) * 8; };
  if (warp < nh) {
    float mx = -INFINITY, l = 0.f;
    for (int p = lane; p < parts; p += 32) mx = fmaxf(mx, a.part_ml[slot(p) + warp].x);
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, s));
    for (int p = lane; p < parts; p += 32) {
      const float2 ml = a.part_ml[slot(p) + warp];
      const float f = mx == -INFINITY ? 1.f : exp2f(ml.x - mx);
      factor[warp * parts + p] = f;
      l += ml.y * f;
    }
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) l += __shfl_xor_sync(0xffffffffu, l, s);
    if (lane == 0) {
      total[warp] = l;
      if (a.lse && blockIdx.y == 0) a.lse[(size_t)d.x * a.hq + j * a.g + h0 + warp] = (mx + log2f(l)) * LN2;
    }
  }
  __syncthreads();
  float acc[8];
#pragma unroll
  for (int h = 0; h < 8; ++h) acc[h] = 0.f;
  const int c = blockIdx.y * 32 + lane;
#pragma unroll 2
  for (int p = warp; p < parts; p += PJ_WARPS) {
    const float* po = a.part_o + slot(p) * DH + c;
#pragma unroll
    for (int h = 0; h < 8; ++h)
      if (h < nh) acc[h] += po[h * DH] * factor[h * parts + p];
  }
#pragma unroll
  for (int h = 0; h < 8; ++h) red[warp][h][lane] = acc[h];
  __syncthreads();
  if (warp < nh) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < PJ_WARPS; ++w) v += red[w][warp][lane];
    const float l = total[warp];
    a.o[((size_t)d.x * a.hq + j * a.g + h0 + warp) * DH + c] = __float2bfloat16(l == 0.f ? 0.f : v / l);
  }
}

int attn_ctas(int dh, int sm_count) { return sm_count * (dh == 256 ? 1 : 2); }

template <int DH, int HG>
cudaError_t launch_attn(const PaArgs& a, int ctas, cudaStream_t st) {
  const size_t smem = At<DH>::smem(HG);
  static bool done[MAX_DEVICES];
  const cudaError_t e = opt_in(paged_attn_kernel<DH, HG>, (int)smem, done);
  if (e != cudaSuccess) return e;
  return launch_pdl_smem(paged_attn_kernel<DH, HG>, dim3((unsigned)ctas), dim3(At<DH>::WARPS * 32), smem, st, a);
}

template <int DH>
int launch_attention_dh(PaArgs a, int sm_count, long long* launches, cudaEvent_t ev_begin, cudaEvent_t ev_end, cudaStream_t st) {
  const long long units = (long long)a.B * a.hk * a.n_grp * ((a.max_len + At<DH>::UNIT - 1) / At<DH>::UNIT);
  const long long most = attn_ctas(DH, sm_count);
  const int ctas = (int)(units < most ? units : most);
  cudaError_t e;
  if (ev_begin && (e = cudaEventRecord(ev_begin, st)) != cudaSuccess) return -(int)e;
  e = a.heads <= 4 ? launch_attn<DH, 4>(a, ctas, st) : launch_attn<DH, 8>(a, ctas, st);
  if (e != cudaSuccess) return -(int)e;
  ++*launches;
  if (ev_end && (e = cudaEventRecord(ev_end, st)) != cudaSuccess) return -(int)e;
  e = launch_pdl_smem(paged_join_kernel<DH>, dim3((unsigned)ctas, DH / 32), dim3(PJ_THREADS), (size_t)8 * ctas * 4, st, a);
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

namespace {
struct PagedLayout { size_t part_o, part_ml, desc, end; };
PagedLayout paged_layout(const CcaDims& d, int sm_count) {
  const size_t ctas = attn_ctas(d.dh, sm_count);
  PagedLayout l;
  size_t off = 0;
  auto take = [&](size_t n) { const size_t o = off; off += (n + 255) / 256 * 256; return o; };
  l.part_o = take(ctas * 2 * 8 * d.dh * 4);
  l.part_ml = take(ctas * 2 * 8 * 8);
  l.desc = take(ctas * 16);
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
  a.desc = reinterpret_cast<int4*>(ws + l.desc);
  switch (d.dh) {
    case 32: return launch_attention_dh<32>(a, sm_count, launches, ev_begin, ev_end, st);
    case 64: return launch_attention_dh<64>(a, sm_count, launches, ev_begin, ev_end, st);
    case 128: return launch_attention_dh<128>(a, sm_count, launches, ev_begin, ev_end, st);
    case 256: return launch_attention_dh<256>(a, sm_count, launches, ev_begin, ev_end, st);
    default: return 1;
  }
}
