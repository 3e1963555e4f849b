// The paged key/value cache: arguments and device helpers shared by its kernels.
//
// Keys and values lie in pages, [n_pages][n_kv][page][head_dim]; request i's key j is slot
// j % page of page table[i][j / page].  The page size is a power of two from 16 on, so the
// 4 or 8 consecutive keys of one wave load always lie in one page.
#pragma once
#include "dcut_internal.h"

namespace dcut {

constexpr int PAGED_MAX_ROWS = 1 << 17;
constexpr int PAGED_MAX_CTX = 1 << 24;
constexpr int PAGED_MAX_GROUP = 64;       // query heads of a kv head
constexpr int PAGED_MAX_PAIRS = 1 << 25;  // (row, query head) pairs: four a workgroup of the merge, a grid has fewer than 2^32 threads
constexpr long long PAGED_MAX_ITEMS = 0xffffff;  // work items of a launch, 256 threads each, likewise
constexpr int PLAN_HEAD = 256;

// Key chunks of a row: a run of L keys is cut into pieces of chunk(L) keys, a multiple of 64,
// at most S pieces unless they would pass cmax keys.  A function of L and of the launch's
// shapes only, so a row's partial sums depend neither on the rows kept beside it nor on
// what other requests hold.
struct Split {
  int S, cmin, cmax;
};
__host__ __device__ inline int split_chunk(const Split &s, int L) {
  const int even = ((L + s.S - 1) / s.S + 63) & ~63;
  const int c = even > s.cmin ? even : s.cmin;
  return c < s.cmax ? c : s.cmax;
}
__host__ __device__ inline int split_count(const Split &s, int L) {
  const int c = split_chunk(s, L);
  return L > 0 ? (L + c - 1) / c : 1;
}

struct PagedArgs {
  const uint16_t *q;          // [rows][n_q][hd], row stride ldq
  long long ldq;
  const uint16_t *k, *v;      // pages
  const int32_t *table;       // [B][table_ld]
  int n_pages, table_ld, page, lpage;
  const int32_t *cu, *ctx_len;
  int B, n_q, n_kv, G, max_rows, max_block, max_ctx;
  uint16_t *out;              // [rows][n_q][hd]
  float *lse;                 // [rows][n_q] or null
  int32_t *dev_err;
  Split split;                // of a request's own keys (sparse: of a row's listed keys)
  int MC;                     // partials a (row, head) may have
  float *part;                // [rows][n_q][MC][ATTN_PITCH(hd)]
  int32_t *row_nc;            // [rows] partials of the row's heads, 1: finished in place
  int32_t *plan;              // work order of the requests' own items (PLAN_HEAD: count, items), or null
  // requests that share a prefix
  int n_groups;
  const int32_t *group_cu, *prefix_len;
  Split psplit;
  // pages chosen for each (row, kv head)
  const int32_t *list;        // [rows][n_kv][n_sel] pool pages, ascending by position
  const int32_t *list_keys;   // [rows][n_kv] keys they hold for the row
  int n_sel;
};

// A request's rows and context, all clamped so that bad device data stays in bounds; false
// where the request has no rows or its arguments contradict the launch bounds.
struct ReqRows {
  int t0, d, L;
};
__device__ __forceinline__ bool paged_request(const PagedArgs &a, int i, bool report, ReqRows &r) {
  r.t0 = a.cu[i];
  r.d = a.cu[i + 1] - r.t0;
  r.L = a.ctx_len[i];
  if (r.d == 0) return false;
  const long long cap = (long long)a.table_ld << a.lpage;
  const bool ok = r.d > 0 && r.d <= a.max_block && r.t0 >= 0 && r.t0 <= a.max_rows - r.d && r.L >= 0 &&
                  (long long)r.L + r.d <= a.max_ctx && (long long)r.L + r.d <= cap;
  if (!ok && report && a.dev_err) atomicOr(a.dev_err, DCUT_DERR_CAPACITY);
  return ok;
}

// A value, a condition, that every lane finds alike, in a scalar register.
__device__ __forceinline__ int uniform_int(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ bool uniform_if(bool x) { return uniform_int(x) != 0; }

// Uniform loads from arrays that the running kernel does not write: one scalar load instead of
// a vector load, whose wait would drain the operand stream in flight.
typedef __attribute__((address_space(4))) const int32_t const_i32;
__device__ __forceinline__ int uniform_load(const int32_t *p, int idx) {
  const uintptr_t b = (uintptr_t)(p + idx);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)b);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
  return *(const_i32 *)(((uintptr_t)hi << 32) | lo);
}

// Host side: argument checks and the split rule (paged_attn.hip).
int paged_cfg_check(const dcut_paged_cfg *c, int B);
int paged_pages_check(const dcut_paged_cfg *c, const dcut_pages *p);
Split paged_split(long long units, int items, bool capped);
int split_max(const Split &s, int max_keys);
PagedArgs paged_args(const dcut_paged_cfg *c, const dcut_pages *p, int B, const dcut_bf16 *q, long long ldq,
                     const int32_t *cu, const int32_t *ctx_len, dcut_bf16 *out, float *lse, int32_t *dev_err);
int paged_list_attn_launch(const PagedArgs &a, int head_dim, hipStream_t s);
size_t paged_attn_ws_bytes(const dcut_paged_cfg *c, int B, bool shared);
size_t paged_sparse_ws_bytes(const dcut_paged_cfg *c, int n_sel);

}  // namespace dcut
