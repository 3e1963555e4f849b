// Attention over the pages that a cheap score selects for each query.
//
// Row t and kv head g score page j by an upper bound of the group's summed scores with any
// of its keys, from the channel bounds kmin, kmax of the page's keys:
//   score(j) = sum_d a_d kmax[j]_d + b_d kmin[j]_d,
//   a_d = sum_h max(q_hd, 0),  b_d = sum_h min(q_hd, 0)      over the group's query heads.
// The score decides which pages are read, so it is formed in 64 bits: products of a bf16
// value and a short sum are exact there, and two pages change places only where their
// scores are equal to about 1 in 2^50.
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

// A row's request and position, by counting the requests that start at or before it.
__device__ __forceinline__ int request_of(const PagedArgs &a, int t, int *s_cnt) {
  int cnt = 0;
  for (int j = threadIdx.x; j < a.B; j += 256) cnt += a.cu[j + 1] <= t;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) cnt += __shfl_xor(cnt, off, 64);
  if ((threadIdx.x & 63) == 0) s_cnt[threadIdx.x >> 6] = cnt;
  __syncthreads();
  cnt = s_cnt[0] + s_cnt[1] + s_cnt[2] + s_cnt[3];
  __syncthreads();
  return cnt;
}

// Scores of 256 pages of one (row, kv head): a page a thread, which reads its page's bounds
// 16 bytes at a time; the group's sums a and b come from LDS.
template <int HD>
__global__ void __launch_bounds__(256)
k_page_score(SparseArgs s) {
  const PagedArgs &a = s.p;
  __shared__ double s_a[HD], s_b[HD];
  __shared__ int s_cnt[4];
  const int t = blockIdx.x, g = blockIdx.y;
  if (t >= a.cu[a.B] || t >= a.max_rows) return;
  const int i = request_of(a, t, s_cnt);
  ReqRows r;
  if (i >= a.B || !paged_request(a, i, false, r)) return;
  const int pos = r.L + t - r.t0;
  const int last = pos >> a.lpage;
  const int j = blockIdx.z * 256 + threadIdx.x;
  if ((int)(blockIdx.z * 256) > last || last < s.n_sel) return;     // all of its pages are read
  if (threadIdx.x < HD) {
    double p = 0.0, n = 0.0;
    for (int h = 0; h < a.G; ++h) {
      const float q = bf2f(a.q[(size_t)t * a.ldq + (size_t)(g * a.G + h) * HD + threadIdx.x]);
      p += (double)fmaxf(q, 0.0f);
      n += (double)fminf(q, 0.0f);
    }
    s_a[threadIdx.x] = p;
    s_b[threadIdx.x] = n;
  }
  __syncthreads();
  if (j > last) return;
  const int pg = a.table[(size_t)i * a.table_ld + j];
  const size_t row = ((size_t)((unsigned)pg < (unsigned)a.n_pages ? pg : 0) * a.n_kv + g) * HD;
  double acc = 0.0;
  for (int d = 0; d < HD; d += 8) {
    const uint4 hi = *(const uint4 *)(s.kmax + row + d), lo = *(const uint4 *)(s.kmin + row + d);
    const uint16_t *eh = (const uint16_t *)&hi, *el = (const uint16_t *)&lo;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      acc = fma(s_a[d + u], (double)bf2f(eh[u]), acc);
      acc = fma(s_b[d + u], (double)bf2f(el[u]), acc);
    }
  }
  s.score[((size_t)t * a.n_kv + g) * s.max_pages + j] = acc;
}

// Unsigned keys in the order of the scores, NaN below every number.
__device__ __forceinline__ unsigned long long order_key(double x) {
  if (x != x) return 1;
  const unsigned long long u = (unsigned long long)__double_as_longlong(x + 0.0);
  return (u >> 63) ? ~u : u | 0x8000000000000000ull;
}

// The n_sel pages of one (row, kv head): the first n_sink and the last n_local, then by score,
// ties to the lower page.  A radix select finds the score of the last page taken; pages above
// it, and the lowest ones equal to it, are listed in ascending order by a scan.
__global__ void __launch_bounds__(256)
k_page_select(SparseArgs s) {
  const PagedArgs &a = s.p;
  __shared__ int s_cnt[4], s_hist[256], s_pick[2];
  const int t = blockIdx.x, g = blockIdx.y, tid = threadIdx.x;
  if (t >= a.cu[a.B] || t >= a.max_rows) return;
  const size_t tg = (size_t)t * a.n_kv + g;
  const int i = request_of(a, t, s_cnt);
  ReqRows r;
  if (i >= a.B || !paged_request(a, i, g == 0 && tid == 0, r)) {
    if (tid == 0) s.list_keys[tg] = 0;
    return;
  }
  const int pos = r.L + t - r.t0;
  const int last = pos >> a.lpage, np = last + 1;
  const int32_t *table = a.table + (size_t)i * a.table_ld;
  int32_t *list = s.list + tg * s.n_sel;
  int32_t *blocks = s.blocks ? s.blocks + tg * s.n_sel : nullptr;
  const int n = min(np, s.n_sel);
  if (tid == 0) s.list_keys[tg] = (n - 1) * a.page + (pos & (a.page - 1)) + 1;
  if (np <= s.n_sel) {
    for (int j = tid; j < s.n_sel; j += 256) {
      if (j < np) list[j] = table[j];
      if (blocks) blocks[j] = j < np ? j : -1;
    }
    return;
  }
  const double *score = s.score + tg * s.max_pages;
  auto key = [&](int j) {
    if (j < s.n_sink || j > last - s.n_local) return ~0ull;
    return order_key(score[j]);
  };
  // the n-th largest key: eight bits a round
  unsigned long long prefix = 0;
  int need = n;
  for (int shift = 56; shift >= 0; shift -= 8) {
    s_hist[tid] = 0;
    __syncthreads();
    const unsigned long long mask = shift == 56 ? 0 : ~0ull << (shift + 8);
    for (int j = tid; j < np; j += 256) {
      const unsigned long long k = key(j);
      if ((k & mask) == prefix) atomicAdd(&s_hist[(int)(k >> shift) & 255], 1);
    }
    __syncthreads();
    if (tid < 64) {                         // digits from the largest: four a lane
      int c[4], sum = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) { c[e] = s_hist[255 - 4 * tid - e]; sum += c[e]; }
      int x = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o, 64);
        if (tid >= o) x += y;
      }
      int before = x - sum;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (before < need && need <= before + c[e]) { s_pick[0] = 255 - 4 * tid - e; s_pick[1] = need - before; }
        before += c[e];
      }
    }
    __syncthreads();
    prefix |= (unsigned long long)s_pick[0] << shift;
    need = s_pick[1];
    __syncthreads();
  }
  // need: how many of the keys equal to `prefix` are taken, the lowest pages first
  int taken = 0, equal = 0;
  for (int j0 = 0; j0 < np; j0 += 256) {
    const int j = j0 + tid;
    const unsigned long long k = j < np ? key(j) : 0;
    const int eq = j < np && k == prefix, gt = j < np && k > prefix;
    // ranks of this thread among the equal and the taken ones
    int v = eq | (gt << 16);
    int x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(x, o, 64);
      if ((tid & 63) >= o) x += y;
    }
    if ((tid & 63) == 63) s_cnt[tid >> 6] = x;
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (w < (tid >> 6)) before += s_cnt[w];
      total += s_cnt[w];
    }
    x += before - v;                         // exclusive
    const int eq_rank = equal + (x & 0xffff), gt_rank = x >> 16;
    const int eq_before = min(eq_rank, need) - min(equal, need);
    if (gt || (eq && eq_rank < need)) {
      const int at = taken + gt_rank + eq_before;
      list[at] = table[j];
      if (blocks) blocks[at] = j;
    }
    const int eq_all = total & 0xffff, gt_all = total >> 16;
    taken += gt_all + min(equal + eq_all, need) - min(equal, need);
    equal += eq_all;
    __syncthreads();
  }
}

struct SparsePlan {
  Split split;
  int mc, max_pages;
  size_t score, list, keys, part, row_nc, total;
};
SparsePlan sparse_plan(const dcut_paged_cfg *c, int n_sel) {
  SparsePlan p = {};
  const size_t rows = c->max_rows, tg = rows * c->n_kv;
  p.max_pages = (c->max_ctx + c->page - 1) / c->page;
  p.split = paged_split((long long)rows * c->n_kv, 2048, false);
  const long long most = (long long)n_sel * c->page;
  p.mc = split_max(p.split, (int)(most < c->max_ctx ? most : c->max_ctx));
  size_t off = 0;
  p.score = off; off = align256(off + (p.max_pages > n_sel ? tg * p.max_pages * sizeof(double) : 0));
  p.list = off; off = align256(off + tg * n_sel * sizeof(int32_t));
  p.keys = off; off = align256(off + tg * sizeof(int32_t));
  p.part = off;
  if (p.mc > 1) off = align256(off + rows * c->n_q * p.mc * ATTN_PITCH(c->head_dim) * sizeof(float));
  p.row_nc = off; off = align256(off + (p.mc > 1 ? rows * sizeof(int32_t) : 0));
  p.total = off;
  return p;
}

}  // namespace

size_t paged_sparse_ws_bytes(const dcut_paged_cfg *c, int n_sel) { return sparse_plan(c, n_sel).total; }

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
  if (p.max_pages > n_sel) {
    const dim3 grid(cfg->max_rows, cfg->n_kv, (p.max_pages + 255) / 256);
    if (cfg->head_dim == 128)
      DCUT_TRY(launch(DCUT_KERNEL_PAGE_SCORE, k_page_score<128>, grid, dim3(256), 0, stream, s));
    else
      DCUT_TRY(launch(DCUT_KERNEL_PAGE_SCORE, k_page_score<64>, grid, dim3(256), 0, stream, s));
  }
  DCUT_TRY(launch(DCUT_KERNEL_PAGE_SELECT, k_page_select, dim3(cfg->max_rows, cfg->n_kv), dim3(256), 0, stream, s));
  return paged_list_attn_launch(s.p, cfg->head_dim, stream);
}
