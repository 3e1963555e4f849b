// Attention over the pages that a cheap score selects for each query.
//
// Row t and kv head g score page j by an upper bound of the group's summed scores with any
// of its keys, from the channel bounds kmin, kmax of the page's keys:
//   score(j) = sum_d a_d kmax[j]_d + b_d kmin[j]_d,
//   a_d = sum_h max(q_hd, 0),  b_d = sum_h min(q_hd, 0)      over the group's query heads.
// The score decides which pages are read, so it is formed in 64 bits: products of a bf16
// value and a short sum are exact there, and two pages change places only where their
// scores are equal to about 1 in 2^50.
//
// Measured: one request of 32000 keys (500 pages) 22.7 us a call; the kernels alone: selection 12.8,
// attention 7.4, merge 4.0.  Batch 16 at 16 to 64 thousand keys 56.4: selection 22.5 (39 to 46 MB of bounds in
// 256-byte pieces, 1.9 TB/s), the chosen pages 30.0, 134 MB at 4.5 TB/s, merge 4.8.
#include "paged.h"

namespace dcut {

namespace {

struct SparseArgs {
  PagedArgs p;
  const uint16_t *kmin, *kmax;
  int n_sel, n_sink, n_local, max_pages;
  double *score;              // [rows][n_kv][max_pages]
  int32_t *list, *list_keys;  // [rows][n_kv][n_sel], [rows][n_kv]
  int32_t *blocks;            // [rows][n_kv][n_sel] or null
};

// A row's request and where it sits, found by all threads: the one that holds the request's
// bounds passes them on.  False (for all) where the row is not live or its request is refused.
// With `report` every request's faults are noted, that of one without live rows too.
struct RowAt {
  int i, pos;
};
template <int THREADS>
__device__ __forceinline__ bool find_row(const PagedArgs &a, int t, int *s_row, bool report, RowAt &row) {
  if (threadIdx.x == 0) s_row[0] = -1;
  __syncthreads();
  for (int j = threadIdx.x; j < a.B; j += THREADS) {
    const int lo = a.cu[j], hi = a.cu[j + 1], L = a.ctx_len[j];
    ReqRows r;
    if (report) paged_request(a, j, true, r);
    if (lo <= t && t < hi) {
      if (t < a.max_rows && t < a.cu[a.B] && paged_request(a, j, false, r)) {
        s_row[1] = L + t - lo;
        s_row[0] = j;
      }
    }
  }
  __syncthreads();
  row.i = uniform_int(s_row[0]);
  row.pos = uniform_int(s_row[1]);
  return row.i >= 0;
}

// The group's sums of one (row, kv head), by the first HD threads of the workgroup.  A NaN stays
// one, in both sums, and so in every score.
template <int HD>
__device__ __forceinline__ void group_sums(const PagedArgs &a, int t, int g, double *s_a, double *s_b) {
  if (threadIdx.x < HD) {
    double p = 0.0, n = 0.0;
    const uint16_t *q = a.q + (size_t)t * a.ldq + (size_t)g * a.G * HD + threadIdx.x;
#pragma unroll 4
    for (int h = 0; h < a.G; ++h) {
      const float x = bf2f(q[h * HD]);
      p += (double)(x < 0.0f ? 0.0f : x);
      n += (double)(x > 0.0f ? 0.0f : x);
    }
    s_a[threadIdx.x] = p;
    s_b[threadIdx.x] = n;
  }
}

// Scores of pages j0 .. j1-1 of one (row, kv head), eight lanes a page: lane c reads 16-byte
// chunks c, c + 8 of its page's bounds, whole lines a load, and keeps its eighth of the sums in
// registers.  The bounds of U pages a lane are asked for together: a page is 512 bytes at a
// random place.  Bound by those loads: without its arithmetic it takes as long.  A page number
// outside the pool is scored with page 0's bounds and reported, chosen or not.
template <int HD, int THREADS, int U, typename Store>
__device__ __forceinline__ void score_pages(const SparseArgs &s, const int32_t *table, int g, int j0, int j1,
                                            const double *s_a, const double *s_b, Store store) {
  constexpr int Q = HD / 8, STEP = THREADS / 8;
  const PagedArgs &a = s.p;
  const int c = threadIdx.x & 7;
  double av[Q], bv[Q];
#pragma unroll
  for (int d = 0; d < Q; ++d) {
    const int at = 8 * (c + 8 * (d / 8)) + d % 8;
    av[d] = s_a[at];
    bv[d] = s_b[at];
  }
  unsigned worst = 0;
  for (int j = j0 + (threadIdx.x >> 3); j < j1; j += U * STEP) {
    int pg[U];
#pragma unroll
    for (int u = 0; u < U; ++u) pg[u] = table[min(j + u * STEP, j1 - 1)];
    uint4 hi[U][Q / 8], lo[U][Q / 8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      worst = max(worst, (unsigned)pg[u]);
      const size_t row = ((size_t)((unsigned)pg[u] < (unsigned)a.n_pages ? pg[u] : 0) * a.n_kv + g) * HD + 8 * c;
#pragma unroll
      for (int e = 0; e < Q / 8; ++e) {
        hi[u][e] = *(const uint4 *)(s.kmax + row + 64 * e);
        lo[u][e] = *(const uint4 *)(s.kmin + row + 64 * e);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      double acc = 0.0;
#pragma unroll
      for (int e = 0; e < Q / 8; ++e) {
        const uint16_t *eh = (const uint16_t *)&hi[u][e], *el = (const uint16_t *)&lo[u][e];
#pragma unroll
        for (int w = 0; w < 8; ++w) {
          acc = fma(av[8 * e + w], (double)bf2f(eh[w]), acc);
          acc = fma(bv[8 * e + w], (double)bf2f(el[w]), acc);
        }
      }
      acc += __shfl_xor(acc, 1, 64);
      acc += __shfl_xor(acc, 2, 64);
      acc += __shfl_xor(acc, 4, 64);
      if (c == 0 && j + u * STEP < j1) store(j + u * STEP, acc);
    }
  }
  if (worst >= (unsigned)a.n_pages && a.dev_err) atomicOr(a.dev_err, DCUT_DERR_PAGE);
}

constexpr int SCORE_PAGES = 256;      // pages a workgroup of k_page_score takes

template <int HD>
__global__ void __launch_bounds__(256)
k_page_score(SparseArgs s) {
  const PagedArgs &a = s.p;
  __shared__ double s_a[HD], s_b[HD];
  __shared__ int s_row[2];
  const int t = blockIdx.x, g = blockIdx.y;
  RowAt row;
  if (!find_row<256>(a, t, s_row, false, row)) return;
  const int last = row.pos >> a.lpage;
  const int j0 = blockIdx.z * SCORE_PAGES;
  if (j0 > last || last < s.n_sel) return;                          // all of its pages are read
  group_sums<HD>(a, t, g, s_a, s_b);
  __syncthreads();
  double *score = s.score + ((size_t)t * a.n_kv + g) * s.max_pages;
  score_pages<HD, 256, 2>(s, a.table + (size_t)row.i * a.table_ld, g, j0, min(j0 + SCORE_PAGES, last + 1), s_a, s_b,
                  [&](int j, double x) { score[j] = x; });
}

// Unsigned keys in the order of the scores, NaN below every number.
__device__ __forceinline__ unsigned long long order_key(double x) {
  if (x != x) return 1;
  const unsigned long long u = (unsigned long long)__double_as_longlong(x + 0.0);
  return (u >> 63) ? ~u : u | 0x8000000000000000ull;
}

// Pages up to which one workgroup scores and selects: one launch less.  Past it the scores of one
// (row, kv head) are worth several workgroups.  Whole calls of 1, 4 and 16 requests, in one launch and
// in two: 600 pages 24, 28, 48 and 26, 30, 51 us; 1020 pages 28, 32, 57 and 26, 30, 58; 1500 pages
// 33, 37, 65 and 27, 31, 65.
constexpr int FUSED_PAGES = 1024;

// The n_sel pages of one (row, kv head): the first n_sink and the last n_local, then by score,
// ties to the lower page.  Each thread owns a run of pages.  A radix select over the scores'
// bits, from the highest that differs, finds the score of the last page taken; the pages
// above it, and the lowest ones equal to it, are listed in ascending order by one scan.
// NK: pages a thread keeps in registers, 0: any number, read again in every round.
constexpr int ST = 1024;              // threads of k_page_select

template <int HD, bool FUSED, int NK>
__global__ void __launch_bounds__(ST)
k_page_select(SparseArgs s) {
  const PagedArgs &a = s.p;
  __shared__ double s_a[FUSED ? HD : 1], s_b[FUSED ? HD : 1], s_score[FUSED ? FUSED_PAGES : 1];
  __shared__ int s_row[2], s_hist[2][256], s_pick[2], s_eq[ST / 64], s_gt[ST / 64];
  __shared__ unsigned long long s_diff[ST / 64];
  const int t = blockIdx.x, g = blockIdx.y, tid = threadIdx.x;
  const size_t tg = (size_t)t * a.n_kv + g;
  RowAt row;
  if (!find_row<ST>(a, t, s_row, t == 0 && g == 0, row)) {
    if (tid == 0) s.list_keys[tg] = 0;
    return;
  }
  const int pos = row.pos;
  const int last = pos >> a.lpage, np = last + 1;
  const int32_t *table = a.table + (size_t)row.i * a.table_ld;
  int32_t *list = s.list + tg * s.n_sel;
  int32_t *blocks = s.blocks ? s.blocks + tg * s.n_sel : nullptr;
  const int n = min(np, s.n_sel);
  if (tid == 0) s.list_keys[tg] = (n - 1) * a.page + (pos & (a.page - 1)) + 1;
  if (np <= s.n_sel) {
    for (int j = tid; j < s.n_sel; j += ST) {
      if (j < np) list[j] = table[j];
      if (blocks) blocks[j] = j < np ? j : -1;
    }
    return;
  }
  const double *score = FUSED ? s_score : s.score + tg * s.max_pages;
  if (FUSED) {
    group_sums<HD>(a, t, g, s_a, s_b);
    __syncthreads();
    score_pages<HD, ST, 2>(s, table, g, 0, np, s_a, s_b, [&](int j, double x) { s_score[j] = x; });
    __syncthreads();
  }
  const int local = np - s.n_local;         // pages from here on and those below n_sink are taken in any case
  const int per = NK ? NK : (np + ST - 1) / ST;
  const int j0 = tid * per;
  // a forced page has key 0, which no score has, and is no candidate
  auto read = [&](int j) { return j < s.n_sink || j >= local ? 0ull : order_key(score[j]); };
  unsigned long long kreg[NK ? NK : 1];
  if (NK) {
#pragma unroll
    for (int e = 0; e < NK; ++e) kreg[e] = read(j0 + e);
  }
  auto each = [&](auto f) {
    if (NK) {
#pragma unroll
      for (int e = 0; e < NK; ++e) f(e, kreg[NK ? e : 0]);
    } else {
      for (int e = 0; e < per; ++e) f(e, read(j0 + e));
    }
  };
  // the highest bit in which two candidates differ
  const unsigned long long first = read(min(s.n_sink, local - 1));          // a candidate: np > n_sel >= n_sink + n_local
  unsigned long long diff = 0;
  each([&](int, unsigned long long k) { diff |= k ? k ^ first : 0; });
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) diff |= __shfl_xor(diff, off, 64);
  if ((tid & 63) == 0) s_diff[tid >> 6] = diff;
  if (tid < 256) s_hist[0][tid] = 0;
  __syncthreads();
  diff = 0;
#pragma unroll
  for (int w = 0; w < ST / 64; ++w) diff |= s_diff[w];
  const int top = 64 - __clzll((long long)diff);                            // bits from `top` on are common
  unsigned long long mask = top >= 64 ? 0 : ~0ull << top, prefix = first & mask;
  int need = n - min(s.n_sink, np) - min(s.n_local, np);                    // np > n_sel: sinks and locals are apart
  int lo = top;                                                             // bits below lo are open
  for (int round = 0; lo > 0 && need > 0; ++round) {
    const int bits = lo < 8 ? lo : 8, shift = lo - bits;
    int *hist = s_hist[round & 1];
    each([&](int, unsigned long long k) {
      if (k && (k & mask) == prefix) atomicAdd(&hist[(int)(k >> shift) & ((1 << bits) - 1)], 1);
    });
    if (tid < 256) s_hist[(round + 1) & 1][tid] = 0;
    __syncthreads();
    if (tid < 64) {                         // digits from the largest: four a lane
      int c[4], sum = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) { c[e] = hist[255 - 4 * tid - e]; sum += c[e]; }
      int x = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o, 64);
        if (tid >= o) x += y;
      }
      int before = x - sum;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (before < need && need <= before + c[e]) {
          s_pick[0] = (255 - 4 * tid - e) | (need - before == c[e] ? 256 : 0);
          s_pick[1] = need - before;
        }
        before += c[e];
      }
    }
    __syncthreads();
    const int pick = s_pick[0];
    mask |= (unsigned long long)((1 << bits) - 1) << shift;
    prefix |= (unsigned long long)(pick & 255) << shift;
    need = s_pick[1];
    lo = shift;
    if (pick & 256) break;                  // every key of this prefix is taken
  }
  // of the keys with this prefix, `need` are taken, the lowest pages first
  int eq = 0, gt = 0;
  each([&](int e, unsigned long long k) {
    const int j = j0 + e;
    gt += j < np && (k == 0 || (k & mask) > prefix);
    eq += j < np && k && (k & mask) == prefix;
  });
  int xe = eq, xg = gt;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int ye = __shfl_up(xe, o, 64), yg = __shfl_up(xg, o, 64);
    if ((tid & 63) >= o) { xe += ye; xg += yg; }
  }
  if ((tid & 63) == 63) { s_eq[tid >> 6] = xe; s_gt[tid >> 6] = xg; }
  __syncthreads();
  xe -= eq;
  xg -= gt;
  for (int w = 0; w < (tid >> 6); ++w) { xe += s_eq[w]; xg += s_gt[w]; }
  each([&](int e, unsigned long long k) {
    const int j = j0 + e;
    if (j >= np) return;
    const bool is_gt = k == 0 || (k & mask) > prefix, is_eq = k && (k & mask) == prefix;
    if (is_gt || (is_eq && xe < need)) {
      const int at = xg + min(xe, need);
      list[at] = table[j];
      if (blocks) blocks[at] = j;
    }
    xg += is_gt;
    xe += is_eq;
  });
}

template <int HD>
int select_launch(const SparseArgs &s, dim3 grid, hipStream_t st) {
  if (s.max_pages <= s.n_sel || s.max_pages <= FUSED_PAGES)
    return launch(DCUT_KERNEL_PAGE_SELECT, k_page_select<HD, true, (FUSED_PAGES + ST - 1) / ST>, grid, dim3(ST), 0, st, s);
  const dim3 sgrid(grid.x, grid.y, (s.max_pages + SCORE_PAGES - 1) / SCORE_PAGES);
  DCUT_TRY(launch(DCUT_KERNEL_PAGE_SCORE, k_page_score<HD>, sgrid, dim3(256), 0, st, s));
  if (s.max_pages <= 4 * ST)
    return launch(DCUT_KERNEL_PAGE_SELECT, k_page_select<HD, false, 4>, grid, dim3(ST), 0, st, s);
  return launch(DCUT_KERNEL_PAGE_SELECT, k_page_select<HD, false, 0>, grid, dim3(ST), 0, st, s);
}

struct SparsePlan {
  Split split;
  int mc, max_pages;
  long long items;            // workgroups of the attention kernel
  size_t score, list, keys, part, row_nc, total;
};
SparsePlan sparse_plan(const dcut_paged_cfg *c, int n_sel) {
  SparsePlan p = {};
  const size_t rows = c->max_rows, tg = rows * c->n_kv;
  p.max_pages = (c->max_ctx + c->page - 1) / c->page;
  p.split = paged_split((long long)rows * c->n_kv, 768, false);     // one round of three workgroups a CU
  const long long most = (long long)n_sel * c->page;
  p.mc = split_max(p.split, (int)(most < c->max_ctx ? most : c->max_ctx));
  p.items = (long long)tg * p.mc;
  size_t off = 0;
  p.score = off; off = align256(off + (p.max_pages > n_sel && p.max_pages > FUSED_PAGES ? tg * p.max_pages * sizeof(double) : 0));
  p.list = off; off = align256(off + tg * n_sel * sizeof(int32_t));
  p.keys = off; off = align256(off + tg * sizeof(int32_t));
  p.part = off;
  if (p.mc > 1) off = align256(off + rows * c->n_q * p.mc * ATTN_PITCH(c->head_dim) * sizeof(float));
  p.row_nc = off; off = align256(off + (p.mc > 1 ? rows * sizeof(int32_t) : 0));
  p.total = off;
  return p;
}

}  // namespace

size_t paged_sparse_ws_bytes(const dcut_paged_cfg *c, int n_sel) {
  const SparsePlan p = sparse_plan(c, n_sel);
  return p.items > PAGED_MAX_ITEMS ? (size_t)-1 : p.total;
}

}  // namespace dcut

using namespace dcut;

extern "C" int dcut_paged_attn_sparse(const dcut_paged_cfg *cfg, const dcut_pages *pages, int B, const dcut_bf16 *q,
                                      int64_t ldq, const int32_t *cu, const int32_t *ctx_len, int n_sel, int n_sink,
                                      int n_local, int32_t *blocks, dcut_bf16 *out, float *lse, int32_t *dev_err, void *ws,
                                      size_t ws_bytes, hipStream_t stream) {
  const int st = paged_cfg_check(cfg, B);
  if (st == DCUT_EINVAL || paged_pages_check(cfg, pages) != DCUT_OK) return DCUT_EINVAL;
  if (!q || !cu || !ctx_len || !out || !pages->kmin || !pages->kmax) return DCUT_EINVAL;
  if (((uintptr_t)q | (uintptr_t)out | (uintptr_t)pages->kmin | (uintptr_t)pages->kmax) & 15) return DCUT_EINVAL;
  if (ldq % 8 || ldq < (long long)cfg->n_q * cfg->head_dim) return DCUT_EINVAL;
  if (n_sink < 0 || n_local < 1 || n_sel < 1 || n_sink > n_sel || n_local > n_sel - n_sink) return DCUT_EINVAL;
  if (st != DCUT_OK) return st;
  if (n_sel > DCUT_PAGED_MAX_SEL) return DCUT_EUNSUPPORTED;
  const SparsePlan p = sparse_plan(cfg, n_sel);
  if (p.items > PAGED_MAX_ITEMS) return DCUT_EUNSUPPORTED;
  if (!ws || ws_bytes < p.total || ((uintptr_t)ws & 255)) return DCUT_EWORKSPACE;
  SparseArgs s = {};
  s.p = paged_args(cfg, pages, B, q, ldq, cu, ctx_len, out, lse, dev_err);
  s.kmin = pages->kmin; s.kmax = pages->kmax;
  s.n_sel = n_sel; s.n_sink = n_sink; s.n_local = n_local; s.max_pages = p.max_pages;
  s.score = (double *)((char *)ws + p.score);
  s.list = (int32_t *)((char *)ws + p.list);
  s.list_keys = (int32_t *)((char *)ws + p.keys);
  s.blocks = blocks;
  s.p.list = s.list; s.p.list_keys = s.list_keys; s.p.n_sel = n_sel;
  s.p.split = p.split; s.p.MC = p.mc;
  if (p.mc > 1) {
    s.p.part = (float *)((char *)ws + p.part);
    s.p.row_nc = (int32_t *)((char *)ws + p.row_nc);
  }
  const dim3 grid(cfg->max_rows, cfg->n_kv);
  DCUT_TRY(cfg->head_dim == 128 ? select_launch<128>(s, grid, stream) : select_launch<64>(s, grid, stream));
  return paged_list_attn_launch(s.p, cfg->head_dim, stream);
}
