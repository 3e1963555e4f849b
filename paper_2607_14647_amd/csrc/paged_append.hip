// Appending keys and values to the paged cache, with the position rotation on the way.
//
// Row t of request i at position p: q and k are rotated (RoPE, pairs (j, j + hd/2), angle
// p * theta^(-2j/hd)), q is written to q_out, k and v to slot p % page of page
// table[i][p / page].  Angles, sines and cosines are formed in 64 bits (a far position
// turns its fastest pair many times), the rotation in 32, one rounding to bf16 at the end.
//
// Bound by HBM: every element is read and written once.  A workgroup takes one row; its
// threads first form the row's sines and cosines in LDS, then walk the row's 16-byte pieces.
// 8 prompts of about 1000 rows (178 MB) 37 us, and 10 for the bounds, 3.9 TB/s in all where a
// large copy reaches 4.8; two and four rows a workgroup took 41 and 42.
// 64 single rows 4.4 us: a launch, two dependent loads and the sines.
#include "paged.h"

namespace dcut {

namespace {

struct AppendArgs {
  const void *q, *k, *v;
  long long ldq, ldk, ldv;
  uint16_t *q_out, *pk, *pv;
  const int32_t *table, *cu, *pos, *req;
  int B, n_pages, table_ld, lpage, n_q, n_kv, max_rows, max_ctx;
  double log2_theta;
  int32_t *dev_err;
};

// Eight consecutive elements as floats.
__device__ __forceinline__ void load8(const uint16_t *p, float (&x)[8]) {
  const uint4 u = *(const uint4 *)p;
  const uint16_t *e = (const uint16_t *)&u;
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = bf2f(e[j]);
}
__device__ __forceinline__ void load8(const float *p, float (&x)[8]) {
  const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void store8(uint16_t *p, const float (&x)[8]) {
  *(uint4 *)p = make_uint4(pack_bf2(x[0], x[1]), pack_bf2(x[2], x[3]), pack_bf2(x[4], x[5]), pack_bf2(x[6], x[7]));
}

template <int HD, typename T>
__global__ void __launch_bounds__(256)
k_paged_append(AppendArgs a) {
  constexpr int HALF = HD / 2, PP = HALF / 8, VP = HD / 8;   // 16-byte pairs of a head, 16-byte pieces of a value
  __shared__ float2 s_cs[HALF];
  __shared__ long long s_slot;              // element offset of (the row's page, kv head 0, slot), or -1
  const int tid = threadIdx.x, t = blockIdx.x;
  const int end = a.cu[a.B];
  if (t >= min(end, a.max_rows)) {
    if (end < 0 && tid == 0 && a.dev_err) atomicOr(a.dev_err, DCUT_DERR_CAPACITY);
    return;
  }
  const int page = 1 << a.lpage;
  if (tid < HALF) {
    const double ang = (double)a.pos[t] * exp2(-(2.0 * tid / HD) * a.log2_theta);
    double sn, cs;
    sincos(ang, &sn, &cs);
    s_cs[tid] = make_float2((float)cs, (float)sn);
  }
  if (tid == 0) {
    long long slot = -1;
    const int i = a.req[t], p = a.pos[t];
    if (end > a.max_rows && a.dev_err) atomicOr(a.dev_err, DCUT_DERR_CAPACITY);
    if (i < 0 || i >= a.B || p < 0 || p >= a.max_ctx || (p >> a.lpage) >= a.table_ld) {
      if (a.dev_err) atomicOr(a.dev_err, DCUT_DERR_CAPACITY);
    } else {
      const int pg = a.table[(size_t)i * a.table_ld + (p >> a.lpage)];
      if ((unsigned)pg >= (unsigned)a.n_pages) {
        if (a.dev_err) atomicOr(a.dev_err, DCUT_DERR_PAGE);
      } else {
        slot = (((long long)pg * a.n_kv) * page + (p & (page - 1))) * HD;
      }
    }
    s_slot = slot;
  }
  __syncthreads();
  const long long slot = s_slot;
  const int nq = a.q ? a.n_q : 0;
  const int pairs = (nq + a.n_kv) * PP, per = pairs + a.n_kv * VP;
  const long long head_step = (long long)page * HD;
  for (int w = tid; w < per; w += 256) {
    if (w >= pairs) {
      const int u = w - pairs, g = u / VP, j = 8 * (u - g * VP);
      if (slot < 0) continue;
      float x[8];
      load8((const T *)a.v + (size_t)t * a.ldv + g * HD + j, x);
      store8(a.pv + slot + g * head_step + j, x);
      continue;
    }
    const int h = w / PP, j = 8 * (w - h * PP);
    const bool key = h >= nq;
    if (key && slot < 0) continue;
    const T *src = key ? (const T *)a.k + (size_t)t * a.ldk + (h - nq) * HD : (const T *)a.q + (size_t)t * a.ldq + h * HD;
    float x1[8], x2[8];
    load8(src + j, x1);
    load8(src + j + HALF, x2);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float2 y = rope_pair(x1[u], x2[u], s_cs[j + u]);
      x1[u] = y.x;
      x2[u] = y.y;
    }
    uint16_t *dst = key ? a.pk + slot + (h - nq) * head_step : a.q_out + ((size_t)t * a.n_q + h) * HD;
    store8(dst + j, x1);
    store8(dst + j + HALF, x2);
  }
}

// Channel bounds of the pages that the appended rows filled.  A workgroup looks through 16 rows
// (no page is smaller) for one kv head; for each that took its page's last slot it reads the
// page's keys, 8 channels and every (256 / (HD / 8))-th key a thread, and joins the threads of
// a channel in LDS.  The keys come out of the caches that the append left them in.
constexpr int BOUND_ROWS = 16;

template <int HD>
__global__ void __launch_bounds__(256)
k_page_bounds(AppendArgs a, uint16_t *kmin, uint16_t *kmax) {
  constexpr int CH = HD / 8, KS = 256 / CH;
  __shared__ float s_lo[KS][HD], s_hi[KS][HD];
  __shared__ int s_page[BOUND_ROWS];        // pool page that the row filled, or -1
  const int g = blockIdx.y, t0 = blockIdx.x * BOUND_ROWS;
  const int M = min(a.cu[a.B], a.max_rows);
  const int page = 1 << a.lpage;
  if (t0 >= M) return;
  if (threadIdx.x < BOUND_ROWS) {
    const int t = t0 + threadIdx.x;
    int pg = -1;
    if (t < M) {
      const int p = a.pos[t], i = a.req[t];
      if ((p & (page - 1)) == page - 1 && i >= 0 && i < a.B && p >= 0 && p < a.max_ctx && (p >> a.lpage) < a.table_ld) {
        pg = a.table[(size_t)i * a.table_ld + (p >> a.lpage)];
        if ((unsigned)pg >= (unsigned)a.n_pages) pg = -1;
      }
    }
    s_page[threadIdx.x] = pg;
  }
  __syncthreads();
  const int c = threadIdx.x % CH, k0 = threadIdx.x / CH;
  for (int e = 0; e < BOUND_ROWS; ++e) {
    const int pg = s_page[e];
    if (pg < 0) continue;                   // uniform
    const uint16_t *src = a.pk + ((size_t)pg * a.n_kv + g) * (size_t)page * HD + 8 * c;
    float lo[8], hi[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) { lo[j] = __builtin_inff(); hi[j] = -__builtin_inff(); }
    for (int k = k0; k < page; k += KS) {
      float x[8];
      load8(src + (size_t)k * HD, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) { lo[j] = fminf(lo[j], x[j]); hi[j] = fmaxf(hi[j], x[j]); }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) { s_lo[k0][8 * c + j] = lo[j]; s_hi[k0][8 * c + j] = hi[j]; }
    __syncthreads();
    if (threadIdx.x < HD) {
      float l = s_lo[0][threadIdx.x], h = s_hi[0][threadIdx.x];
      for (int k = 1; k < KS; ++k) { l = fminf(l, s_lo[k][threadIdx.x]); h = fmaxf(h, s_hi[k][threadIdx.x]); }
      const size_t o = ((size_t)pg * a.n_kv + g) * HD + threadIdx.x;
      kmin[o] = f2bf(l);
      kmax[o] = f2bf(h);
    }
    __syncthreads();
  }
}

template <int HD, typename T>
int append_launch(const AppendArgs &a, const dcut_pages *pg, hipStream_t s) {
  DCUT_TRY(launch(DCUT_KERNEL_PAGED_APPEND, k_paged_append<HD, T>, dim3(a.max_rows), dim3(256), 0, s, a));
  if (!pg->kmin) return DCUT_OK;
  return launch(DCUT_KERNEL_PAGED_BOUNDS, k_page_bounds<HD>, dim3((a.max_rows + BOUND_ROWS - 1) / BOUND_ROWS, a.n_kv), dim3(256), 0, s, a, pg->kmin, pg->kmax);
}

}  // namespace

}  // namespace dcut

using namespace dcut;

extern "C" int dcut_paged_append(const dcut_paged_cfg *cfg, const dcut_pages *pages, int B, const int32_t *cu,
                                 const int32_t *packed_pos, const int32_t *packed_req, int type, const void *q, int64_t ldq,
                                 const void *k, int64_t ldk, const void *v, int64_t ldv, float rope_theta,
                                 dcut_bf16 *q_out, int32_t *dev_err, hipStream_t stream) {
  const int st = paged_cfg_check(cfg, B);
  if (st == DCUT_EINVAL || paged_pages_check(cfg, pages) != DCUT_OK) return DCUT_EINVAL;
  if (!cu || !packed_pos || !packed_req || !k || !v || (q != nullptr) != (q_out != nullptr)) return DCUT_EINVAL;
  if ((pages->kmin != nullptr) != (pages->kmax != nullptr)) return DCUT_EINVAL;
  if (type != DCUT_BF16 && type != DCUT_F32) return DCUT_EINVAL;
  if (!(rope_theta > 0.0f) || !(rope_theta < __builtin_inff())) return DCUT_EINVAL;
  const int unit = type == DCUT_BF16 ? 8 : 4;                // elements of 16 bytes
  const long long kvw = (long long)cfg->n_kv * cfg->head_dim;
  if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_out) & 15) return DCUT_EINVAL;
  if (ldk < kvw || ldv < kvw || ldk % unit || ldv % unit) return DCUT_EINVAL;
  if (q && (ldq < (long long)cfg->n_q * cfg->head_dim || ldq % unit)) return DCUT_EINVAL;
  if (st != DCUT_OK) return st;
  AppendArgs a = {};
  a.q = q; a.k = k; a.v = v; a.ldq = ldq; a.ldk = ldk; a.ldv = ldv;
  a.q_out = q_out; a.pk = pages->k; a.pv = pages->v;
  a.table = pages->table; a.cu = cu; a.pos = packed_pos; a.req = packed_req;
  a.B = B; a.n_pages = pages->n_pages; a.table_ld = pages->table_ld; a.lpage = __builtin_ctz(cfg->page);
  a.n_q = cfg->n_q; a.n_kv = cfg->n_kv; a.max_rows = cfg->max_rows; a.max_ctx = cfg->max_ctx;
  a.log2_theta = log2((double)rope_theta);
  a.dev_err = dev_err;
  if (cfg->head_dim == 128)
    return type == DCUT_BF16 ? append_launch<128, uint16_t>(a, pages, stream) : append_launch<128, float>(a, pages, stream);
  return type == DCUT_BF16 ? append_launch<64, uint16_t>(a, pages, stream) : append_launch<64, float>(a, pages, stream);
}
