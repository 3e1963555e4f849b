// Attention over the paged key/value cache: a request's new rows over its pages, rows of
// requests that share a prefix over its pages, rows over pages chosen for each of them.
//
// Work item = (tile of query rows, kv head, key chunk).  A tile's rows are (packed row,
// query head of the group) pairs, packed row slowest, so all query heads of a kv head and
// all kept rows of a request share each 32-key tile of its pages.  For row r of a tile and
// keys j, with S = q_r . k_j / sqrt(hd),
//   m = max_j S_rj,   l = sum_j exp(S_rj - m),   o = sum_j exp(S_rj - m) v_j,
// kept in one pass (m, l, o rescaled when m grows), out = o / l, lse = m + ln l.  Chunks give
// partial (o, m, l), which k_paged_merge joins in chunk order.
//
// paged_stream.h has the kernel body of units of up to 64 pairs, paged_wide.h that of more.
#include "paged_stream.h"
#include "paged_wide.h"

namespace dcut {

namespace {

template <int HD, int MODE>
__global__ void __launch_bounds__(STREAM_WAVES * 64) __attribute__((amdgpu_waves_per_eu(3)))
k_paged_stream(PagedArgs a, int units) {
  extern __shared__ __align__(1024) unsigned char ring[];
  __shared__ int s_cnt[STREAM_WAVES];
  Item it;
  if (!make_item<MODE, false, 16 * STREAM_WAVES, 64 * STREAM_WAVES>(a, blockIdx.x, units, s_cnt, it)) return;
  stream_body<HD, MODE>(a, it, ring);
}

template <int HD>
__global__ void __launch_bounds__(WIDE_WAVES * 64) __attribute__((amdgpu_waves_per_eu(2)))
k_paged_wide(PagedArgs a, int units) {
  extern __shared__ __align__(1024) unsigned char ring[];
  __shared__ int s_cnt[WIDE_WAVES];
  Item it;
  if (!make_item<OWN, false, WIDE_ROWS, 64 * WIDE_WAVES>(a, blockIdx.x, units, s_cnt, it)) return;
  wide_body<HD, OWN>(a, it, ring);
}

// A shared call's items in one launch, so that the requests' own keys are read beside the
// prefixes: the first pre_items workgroups take prefix items in tiles of 128 pairs, the
// others the requests' own, wide or streamed.
template <int HD, bool WIDE>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
k_paged_shared(PagedArgs a, int pre_units, int pre_items, int units) {
  extern __shared__ __align__(1024) unsigned char ring[];
  __shared__ int s_cnt[4];
  Item it;
  if ((int)blockIdx.x < pre_items) {
    if (!make_item<PREFIX, true, WIDE_ROWS, 256>(a, blockIdx.x, pre_units, s_cnt, it)) return;
    wide_body<HD, PREFIX>(a, it, ring);
    return;
  }
  const int idx = blockIdx.x - pre_items;
  if (WIDE) {
    if (!make_item<OWN, true, WIDE_ROWS, 256>(a, idx, units, s_cnt, it)) return;
    wide_body<HD, OWN>(a, it, ring);
  } else {
    if (!make_item<OWN, true, 64, 256>(a, idx, units, s_cnt, it)) return;
    stream_body<HD, OWN>(a, it, ring);
  }
}

// Merge of a (row, head)'s partials by one wave, whose halves take every second one: lane i of a
// half reads its i-th partial's (max, sum), so the weights of up to 64 partials cost one memory
// round trip, taken together with the first eight partials' values.  The order of the sums is fixed.
// Bound by its round trips and the launch: 3.5 to 5 us for a few partials a row, 7 for 32 partials of
// 1024 (row, head) pairs (by half a wave each 9.2), 8 to 10 for the largest calls (16 values at once there: 10 to 14).
template <int HD>
__global__ void __launch_bounds__(256)
k_paged_merge(PagedArgs a) {
  constexpr int PER = HD / 32, CG = 4;
  const int lane = threadIdx.x & 31, odd = (threadIdx.x >> 5) & 1;
  const int pair = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int t = pair / a.n_q;
  const int nc0 = a.row_nc[min(t, a.max_rows - 1)];
  const int M0 = a.cu[0], M = a.cu[a.B];
  if (t < M0 || t >= M || t >= a.max_rows) return;          // no request's row
  const int nc = min(nc0, a.MC);
  if (nc <= 1) return;
  const float *pp = a.part + ((size_t)pair * a.MC + odd) * ATTN_PITCH(HD);
  float acc[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) acc[e] = 0.0f;
  float mx = -__builtin_inff(), lsum = 0.0f;
  for (int c0 = 0; c0 < nc; c0 += 64) {
    const int both = min(64, nc - c0), cnt = (both + 1 - odd) >> 1;          // partials c0 + odd + 2 i
    const float *p0 = pp + (size_t)c0 * ATTN_PITCH(HD);
    float xv[CG][PER];
    auto load = [&](int cc) {
#pragma unroll
      for (int u = 0; u < CG; ++u)
#pragma unroll
        for (int e = 0; e < PER; ++e) xv[u][e] = cc + u < cnt ? p0[(cc + u) * 2 * ATTN_PITCH(HD) + lane * PER + e] : 0.0f;
    };
    load(0);
    const float mv = lane < cnt ? p0[lane * 2 * ATTN_PITCH(HD) + HD] : -__builtin_inff();
    const float lv = lane < cnt ? p0[lane * 2 * ATTN_PITCH(HD) + HD + 1] : 0.0f;
    float gm = mv;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) gm = fmaxf(gm, __shfl_xor(gm, off, 32));
    const float mn = fmaxf(mx, half_max(gm)), sub = mn == -__builtin_inff() ? 0.0f : mn;
    const float w = __builtin_amdgcn_exp2f(mv - sub);         // 0 for an empty partial
    float ls = lane < cnt ? lv * w : 0.0f;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) ls += __shfl_xor(ls, off, 32);
    const float old = __builtin_amdgcn_exp2f(mx - sub);
    lsum = lsum * old + ls;
    mx = mn;
#pragma unroll
    for (int e = 0; e < PER; ++e) acc[e] *= old;
    for (int cc = 0;; cc += CG) {
#pragma unroll
      for (int u = 0; u < CG; ++u) {
        const float wc = __shfl(w, cc + u, 32);
#pragma unroll
        for (int e = 0; e < PER; ++e) acc[e] += cc + u < cnt ? xv[u][e] * wc : 0.0f;
      }
      if (2 * (cc + CG) >= both) break;
      load(cc + CG);
    }
  }
  lsum = half_sum(lsum);
#pragma unroll
  for (int e = 0; e < PER; ++e) acc[e] = half_sum(acc[e]);
  if (odd) return;
  const float inv = lsum > 0.0f ? 1.0f / lsum : lsum == 0.0f ? 0.0f : lsum;
  uint16_t *op = a.out + (size_t)pair * HD + lane * PER;
#pragma unroll
  for (int e = 0; e < PER; e += 2) *(uint32_t *)(op + e) = cvt_bf2(acc[e] * inv, acc[e + 1] * inv);
  if (a.lse && lane == 0) a.lse[pair] = 0.6931471805599453f * (mx + __builtin_amdgcn_logf(lsum));
}

// The work order of the requests' own items, {request, first pair of the tile, chunk} by
// descending number of keys (to an eighth of an octave), built by one workgroup: a count of
// the items of each length, their places, the items.  4.7 us; the whole call of 64 decoding
// requests of up to 4096 keys takes 96 us with it, 116 without.
__global__ void __launch_bounds__(1024)
k_paged_plan(PagedArgs a, int units, int TM) {
  extern __shared__ int s_first[];          // first tile of each request
  __shared__ int s_at[256], s_sum[4];
  const int tid = threadIdx.x;
  const bool tiles = a.G * a.max_block > TM;
  if (tiles)
    for (int j = tid; j < a.B; j += 1024) {
      ReqRows r;
      paged_request(a, j, true, r);         // a refused request need not be any tile's
      s_first[j] = run_tile(a.cu[j], a.G, TM, j);
    }
  if (tid < 256) s_at[tid] = 0;
  __syncthreads();
  auto items = [&](bool report, auto emit) {
    for (int u = tid; u < units; u += 1024) {
      int i = u;
      long long r0 = 0;
      if (tiles) {
        int lo = 0, hi = a.B;               // requests before lo start at or before u
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (s_first[mid] <= u) lo = mid + 1;
          else hi = mid;
        }
        if (lo == 0) continue;
        i = lo - 1;
        r0 = ((long long)u - s_first[i]) * TM;
      }
      ReqRows r;
      if (!paged_request(a, i, report, r) || r0 < 0 || r0 >= (long long)r.d * a.G) continue;
      const int nc = split_count(a.split, r.L), ch = split_chunk(a.split, r.L);
      const int rows = (int)((min(r0 + TM, (long long)r.d * a.G) - 1) / a.G) + 1;
      for (int c = 0; c < nc; ++c) {
        const int keys = c == nc - 1 ? r.L - c * ch + rows : ch;
        // the top three bits below the leading one and the exponent: 8 classes an octave
        const int cls = 255 - min((int)((__float_as_uint((float)keys) - 0x3f800000u) >> 20), 255);
        emit(cls, i, (int)r0, c);
      }
    }
  };
  items(!tiles, [&](int cls, int, int, int) { atomicAdd(&s_at[cls], 1); });
  __syncthreads();
  int n = 0, x = 0;
  if (tid < 256) {                          // places: exclusive sum of the counts
    n = x = s_at[tid];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(x, o, 64);
      if ((tid & 63) >= o) x += y;
    }
    if ((tid & 63) == 63) s_sum[tid >> 6] = x;
  }
  __syncthreads();
  if (tid < 256) {
    for (int w = 0; w < (tid >> 6); ++w) x += s_sum[w];
    s_at[tid] = x - n;
    if (tid == 255) a.plan[0] = x;
  }
  __syncthreads();
  int4 *list = (int4 *)((char *)a.plan + PLAN_HEAD);
  items(false, [&](int cls, int i, int r0, int c) { list[atomicAdd(&s_at[cls], 1)] = make_int4(i, r0, c, 0); });
}

// Tiles of TM pairs that consecutive runs of at most `rows` rows in all can have (find_run).
long long tile_bound(long long rows, int G, int TM, int runs) { return rows * G / TM + runs; }

// How the (row, query head) pairs of a unit are tiled: 64 where a unit has no more (streamed),
// else 128 (wide).  Whole calls of 64 requests on contexts of 2048 to 4096, streamed and wide: 32
// pairs (8 kv heads) 146 and 169 us, 64 pairs 155 and 180, 64 pairs (4 kv heads) 91 and 95; 80 pairs
// 110 and 97, 128 pairs 133 and 102, 132 pairs (8 kv heads) 206 and 183.  Tiles of 256 pairs,
// 8 waves: equal to 128.
int tile_rows(long long pairs) { return pairs <= 64 ? 64 : WIDE_ROWS; }

long long items(long long units, int n_kv, int mc) { return units * n_kv * mc; }

template <int HD, int MODE>
int launch_stream(const PagedArgs &a, int units, int mc, hipStream_t s) {
  const long long n = items(units, a.n_kv, mc);
  return launch(DCUT_KERNEL_PAGED_ATTN, k_paged_stream<HD, MODE>, dim3((unsigned)n), dim3(256), stream_lds(HD), s, a, units);
}
template <int HD>
int launch_own(const PagedArgs &a, int rows, int units, int mc, hipStream_t s) {
  if (rows == 64) return launch_stream<HD, OWN>(a, units, mc, s);
  const long long n = items(units, a.n_kv, mc);
  return launch(DCUT_KERNEL_PAGED_ATTN, k_paged_wide<HD>, dim3((unsigned)n), dim3(256), wide_lds(HD), s, a, units);
}
template <int HD>
int launch_shared(const PagedArgs &a, int rows, int pre_units, int mc_pre, int units, int mc, hipStream_t s) {
  const long long pre = items(pre_units, a.n_kv, mc_pre), n = pre + items(units, a.n_kv, mc);
  const size_t lds = wide_lds(HD) > stream_lds(HD) ? wide_lds(HD) : stream_lds(HD);
  if (rows == 64)
    return launch(DCUT_KERNEL_PAGED_ATTN, k_paged_shared<HD, false>, dim3((unsigned)n), dim3(256), lds, s, a, pre_units, (int)pre, units);
  return launch(DCUT_KERNEL_PAGED_ATTN, k_paged_shared<HD, true>, dim3((unsigned)n), dim3(256), lds, s, a, pre_units, (int)pre, units);
}
int merge(const PagedArgs &a, int hd, hipStream_t s) {
  if (a.MC == 1) return DCUT_OK;
  const dim3 grid((unsigned)(((long long)a.max_rows * a.n_q + 3) / 4));
  if (hd == 128) return launch(DCUT_KERNEL_PAGED_MERGE, k_paged_merge<128>, grid, dim3(256), 0, s, a);
  return launch(DCUT_KERNEL_PAGED_MERGE, k_paged_merge<64>, grid, dim3(256), 0, s, a);
}

// Work items aimed at: the requests' own rows in 64-pair tiles 1536, twice the workgroup slots,
// since their lengths differ; beside prefixes, which fill the slots first, 768; wide tiles 256.
// Verification under three prompts of 2000 to 6000 keys, the mean of five batches: 83.0 us; own
// items for 1536 and prefix pieces uncapped (two of up to 3000 keys: the longest of few long
// items ends last), 87.0; pieces of 1024 keys 87.6.  One of the batches takes 71.2 us, own
// items dispatched before the prefixes 88.7, in turns with them 80.2.
struct AttnPlan {
  Split own, pre;
  int rows, mc_own, mc_pre, units;
  long long items;          // workgroups of the attention kernel (shared: at most)
  size_t part, row_nc, plan, plan_bytes, total;
};
// Items a launch may have before they are listed longest first: what fits about one round of
// the workgroup slots gains nothing, and the list costs a launch.  Decoding on ragged contexts,
// listed and not: 512 items 16 to 17 and 12 us, 1024 items 18 and 16; 1536 items of up to 192 keys 26
// and 24, of up to 1024 keys 37 and 37, 2048 keys 56 and 63, 4096 keys 96 and 116.  Not for shared
// calls, whose own items are short beside the prefix.
constexpr long long PLAN_MIN = 1024;

AttnPlan attn_plan(const dcut_paged_cfg *c, int B, bool shared) {
  AttnPlan p = {};
  const int G = c->n_q / c->n_kv;
  const long long pairs = (long long)G * c->max_block;
  p.rows = tile_rows(pairs);
  p.units = pairs <= p.rows ? B : (int)tile_bound(c->max_rows, G, p.rows, B);
  p.own = paged_split((long long)p.units * c->n_kv, p.rows > 64 ? 256 : shared ? 768 : 1536, pairs <= p.rows);
  p.mc_own = split_max(p.own, c->max_ctx);
  if (shared) {
    p.pre = paged_split((((long long)c->max_rows * G + WIDE_ROWS - 1) / WIDE_ROWS) * c->n_kv, 256, false);
    // Prefixes differ in length and the launch's bounds do not tell: pieces of 1536 keys even
    // their items out, up to 8 of them for the partials' sake.
    const int eighth = ((c->max_ctx + 7) / 8 + 63) & ~63;
    p.pre.cmax = eighth > 1536 ? eighth : 1536;
    p.mc_pre = split_max(p.pre, c->max_ctx);
  }
  p.items = items(p.units, c->n_kv, p.mc_own) + items(shared ? tile_bound(c->max_rows, G, WIDE_ROWS, B) : 0, c->n_kv, p.mc_pre);
  const int mc = p.mc_own + p.mc_pre;
  size_t off = 0;
  p.part = off;
  if (mc > 1) off = align256(off + (size_t)c->max_rows * c->n_q * mc * ATTN_PITCH(c->head_dim) * sizeof(float));
  p.row_nc = off;
  if (mc > 1) off = align256(off + (size_t)c->max_rows * sizeof(int32_t));
  p.plan = off;
  const long long listed = (long long)p.units * p.mc_own;
  if (!shared && listed * c->n_kv > PLAN_MIN) p.plan_bytes = PLAN_HEAD + (size_t)listed * sizeof(int4);
  p.total = align256(off + p.plan_bytes);
  return p;
}

}  // namespace

// Pieces for a launch of about `items` work items.  Pieces under 128 keys cost more in partials
// than they win.
Split paged_split(long long units, int items, bool capped) {
  long long S = (items + units - 1) / (units > 0 ? units : 1);
  if (S < 1) S = 1;
  if (S > 64) S = 64;
  return Split{(int)S, 128, capped ? 2048 : 1 << 30};
}
int split_max(const Split &s, int max_keys) {
  const int by_cap = (max_keys + s.cmax - 1) / s.cmax, by_min = (max_keys + s.cmin - 1) / s.cmin;
  int m = s.S > by_cap ? s.S : by_cap;
  m = m < by_min ? m : by_min;
  return m > 1 ? m : 1;
}

int paged_cfg_check(const dcut_paged_cfg *c, int B) {
  if (!c || B < 1 || B > DCUT_MAX_BATCH) return DCUT_EINVAL;
  if (c->n_q <= 0 || c->n_kv <= 0 || c->n_q % c->n_kv || c->head_dim <= 0) return DCUT_EINVAL;
  if (c->page <= 0 || c->max_ctx < 1 || c->max_block < 1 || c->max_rows < 1 || c->max_block > c->max_ctx) return DCUT_EINVAL;
  if (c->head_dim != 64 && c->head_dim != 128) return DCUT_EUNSUPPORTED;
  if ((c->page & (c->page - 1)) || c->page < 16 || c->page > 256) return DCUT_EUNSUPPORTED;
  if (c->n_q / c->n_kv > PAGED_MAX_GROUP || c->n_q > 1024) return DCUT_EUNSUPPORTED;
  if (c->max_rows > PAGED_MAX_ROWS || c->max_ctx > PAGED_MAX_CTX) return DCUT_EUNSUPPORTED;
  if ((long long)c->max_rows * c->n_q > PAGED_MAX_PAIRS) return DCUT_EUNSUPPORTED;
  return DCUT_OK;
}
int paged_pages_check(const dcut_paged_cfg *c, const dcut_pages *p) {
  if (!p || !p->k || !p->v || !p->table || p->n_pages < 1 || p->table_ld < 1) return DCUT_EINVAL;
  if (((uintptr_t)p->k | (uintptr_t)p->v) & 15) return DCUT_EINVAL;
  return DCUT_OK;
}

PagedArgs paged_args(const dcut_paged_cfg *c, const dcut_pages *p, int B, const dcut_bf16 *q, long long ldq,
                     const int32_t *cu, const int32_t *ctx_len, dcut_bf16 *out, float *lse, int32_t *dev_err) {
  PagedArgs a = {};
  a.q = q; a.ldq = ldq; a.k = p->k; a.v = p->v; a.table = p->table;
  a.n_pages = p->n_pages; a.table_ld = p->table_ld; a.page = c->page; a.lpage = __builtin_ctz(c->page);
  a.cu = cu; a.ctx_len = ctx_len;
  a.B = B; a.n_q = c->n_q; a.n_kv = c->n_kv; a.G = c->n_q / c->n_kv;
  a.max_rows = c->max_rows; a.max_block = c->max_block; a.max_ctx = c->max_ctx;
  a.out = out; a.lse = lse; a.dev_err = dev_err; a.MC = 1;
  return a;
}

size_t paged_attn_ws_bytes(const dcut_paged_cfg *c, int B, bool shared) {
  const AttnPlan p = attn_plan(c, B, shared);
  return p.items > PAGED_MAX_ITEMS ? (size_t)-1 : p.total;
}

// Rows over their listed pages (a.list set, a.split, a.MC, a.part and a.row_nc too).
int paged_list_attn_launch(const PagedArgs &a, int hd, hipStream_t s) {
  const int st = hd == 128 ? launch_stream<128, LIST>(a, a.max_rows, a.MC, s) : launch_stream<64, LIST>(a, a.max_rows, a.MC, s);
  DCUT_TRY(st);
  return merge(a, hd, s);
}

}  // namespace dcut

using namespace dcut;

static int paged_attn_check(const dcut_paged_cfg *cfg, const dcut_pages *pg, int B, const dcut_bf16 *q, long long ldq,
                            const int32_t *cu, const int32_t *ctx_len, const dcut_bf16 *out) {
  const int st = paged_cfg_check(cfg, B);
  if (st == DCUT_EINVAL) return st;
  if (paged_pages_check(cfg, pg) != DCUT_OK) return DCUT_EINVAL;
  if (!q || !cu || !ctx_len || !out) return DCUT_EINVAL;
  if (((uintptr_t)q & 15) || ((uintptr_t)out & 15) || ldq % 8 || ldq < (long long)cfg->n_q * cfg->head_dim) return DCUT_EINVAL;
  return st;
}

extern "C" int dcut_paged_attn(const dcut_paged_cfg *cfg, const dcut_pages *pages, int B, const dcut_bf16 *q, int64_t ldq,
                               const int32_t *cu, const int32_t *ctx_len, dcut_bf16 *out, float *lse,
                               int32_t *dev_err, void *ws, size_t ws_bytes, hipStream_t stream) {
  DCUT_TRY(paged_attn_check(cfg, pages, B, q, ldq, cu, ctx_len, out));
  const AttnPlan p = attn_plan(cfg, B, false);
  if (p.items > PAGED_MAX_ITEMS) return DCUT_EUNSUPPORTED;
  if (p.total && (!ws || ws_bytes < p.total || ((uintptr_t)ws & 255))) return DCUT_EWORKSPACE;
  PagedArgs a = paged_args(cfg, pages, B, q, ldq, cu, ctx_len, out, lse, dev_err);
  a.split = p.own;
  a.MC = p.mc_own;
  if (a.MC > 1) {
    a.part = (float *)((char *)ws + p.part);
    a.row_nc = (int32_t *)((char *)ws + p.row_nc);
  }
  if (p.plan_bytes) {
    a.plan = (int32_t *)((char *)ws + p.plan);
    const size_t lds = a.G * a.max_block > p.rows ? (size_t)B * sizeof(int) : 0;
    DCUT_TRY(launch(DCUT_KERNEL_PAGED_PLAN, k_paged_plan, dim3(1), dim3(1024), lds, stream, a, p.units, p.rows));
  }
  const int st = cfg->head_dim == 128 ? launch_own<128>(a, p.rows, p.units, p.mc_own, stream)
                                      : launch_own<64>(a, p.rows, p.units, p.mc_own, stream);
  DCUT_TRY(st);
  return merge(a, cfg->head_dim, stream);
}

extern "C" int dcut_paged_attn_shared(const dcut_paged_cfg *cfg, const dcut_pages *pages, int B, const dcut_bf16 *q,
                                      int64_t ldq, const int32_t *cu, const int32_t *ctx_len, int n_groups,
                                      const int32_t *group_cu, const int32_t *prefix_len, dcut_bf16 *out, float *lse,
                                      int32_t *dev_err, void *ws, size_t ws_bytes, hipStream_t stream) {
  const int st = paged_attn_check(cfg, pages, B, q, ldq, cu, ctx_len, out);
  if (st == DCUT_EINVAL) return st;
  if (n_groups < 1 || n_groups > B || !group_cu || !prefix_len) return DCUT_EINVAL;
  if (st != DCUT_OK) return st;
  const AttnPlan p = attn_plan(cfg, B, true);
  if (p.items > PAGED_MAX_ITEMS) return DCUT_EUNSUPPORTED;
  if (!ws || ws_bytes < p.total || ((uintptr_t)ws & 255)) return DCUT_EWORKSPACE;
  PagedArgs a = paged_args(cfg, pages, B, q, ldq, cu, ctx_len, out, lse, dev_err);
  a.split = p.own;
  a.psplit = p.pre;
  a.MC = p.mc_own + p.mc_pre;
  a.part = (float *)((char *)ws + p.part);
  a.row_nc = (int32_t *)((char *)ws + p.row_nc);
  a.n_groups = n_groups;
  a.group_cu = group_cu;
  a.prefix_len = prefix_len;
  const int pre_units = (int)tile_bound(cfg->max_rows, a.G, WIDE_ROWS, n_groups);
  const int ls = cfg->head_dim == 128 ? launch_shared<128>(a, p.rows, pre_units, p.mc_pre, p.units, p.mc_own, stream)
                                      : launch_shared<64>(a, p.rows, pre_units, p.mc_pre, p.units, p.mc_own, stream);
  DCUT_TRY(ls);
  return merge(a, cfg->head_dim, stream);
}
