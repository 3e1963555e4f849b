// Work items of the paged attention kernels (device side): which rows, kv head and keys a
// workgroup takes, and the operand loads they share.
//
// The work order (k_paged_plan, paged_attn.hip): workgroups are dispatched in the order of their
// index as slots free up, so items listed longest first end together, the short ones filling
// the gaps.  Results do not depend on the order.
//
// A work item is (tile of query rows, kv head, key chunk).  A tile's rows are (packed row,
// query head of the group) pairs, packed row slowest.
#pragma once
#include "paged.h"

namespace dcut {
namespace {

typedef short short4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) const bf16x8 lds_frag;

// Barrier of the LDS ring: each wave has waited (s_waitcnt vmcnt) for its own loads of the
// stage it reads next, so only the hardware barrier is needed; a memory fence here would
// drain every stage still in flight.
__device__ __forceinline__ void ring_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t uniform_rsrc(const void *base, int bytes) {
  const uintptr_t b = (uintptr_t)base;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)b);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
  return __builtin_amdgcn_make_buffer_rsrc((void *)(((uintptr_t)hi << 32) | lo), (short)0, bytes, 0x00020000);
}

enum Mode { OWN = 0, PREFIX = 1, LIST = 2 };    // a request's own keys, a group's prefix, chosen pages

// What a work item reads and computes; uniform over the workgroup.
struct Item {
  int g;               // kv head
  int t0, rows, r0;    // first packed row of the unit, its (row, head) pairs, first of this tile
  const int32_t *tab;  // page of keys j*page.. of the unit
  int klo, kend;       // keys of the chunk; below klo and from kend on: none
  int kstart;          // first key of the first key tile, in klo's page, a multiple of 16
  int diag;            // packed row t0 + r sees keys up to diag + r
  int nc, slot;        // partials of the rows, and which this one is
  bool first;          // this item notes the rows' count of partials
};

// Units are tiles of TM pairs of consecutive runs of rows: run i's are numbered from
// floor(start_i G / TM) + i on, which no two runs share.
__device__ __forceinline__ int run_tile(int start, int G, int TM, int i) { return (int)((long long)start * G / TM) + i; }

// The run that unit u belongs to.
template <int THREADS, typename Start>
__device__ __forceinline__ int find_run(int n, int u, int *s_cnt, Start first_tile) {
  int cnt = 0;
  for (int j = threadIdx.x; j < n; j += THREADS) cnt += first_tile(j) <= u;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) cnt += __shfl_xor(cnt, off, 64);
  if ((threadIdx.x & 63) == 0) s_cnt[threadIdx.x >> 6] = cnt;
  __syncthreads();
  cnt = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) cnt += s_cnt[w];
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(cnt) - 1;
}

// The groups of requests that share a prefix, looked through by a wave: group j's first request
// and prefix, for up to 63 groups kept in lane j, so that one round trip to memory finds a
// request's group (a search of its own for each work item took longer than short items' work).
struct Groups {
  int n, cu, prefix;
  bool few;
  __device__ __forceinline__ Groups(const PagedArgs &a) : n(a.n_groups), few(a.n_groups < 64) {
    const int lane = threadIdx.x & 63;
    cu = n > 0 ? a.group_cu[min(lane, n)] : 0;
    prefix = n > 0 ? a.prefix_len[min(lane, n - 1)] : 0;
  }
  __device__ __forceinline__ int first(const PagedArgs &a, int j) const {
    return few ? __builtin_amdgcn_readlane(cu, j) : uniform_load(a.group_cu, j);
  }
  // Groups whose number `below(first request, group)` calls below; they are the first ones.
  template <typename Below>
  __device__ __forceinline__ int count(const PagedArgs &a, Below below) const {
    const int lane = threadIdx.x & 63;
    int c = __popcll(__ballot(lane < n && below(cu, lane)));
    for (int j0 = 64; j0 < n; j0 += 64) {
      const int j = j0 + lane, f = a.group_cu[min(j, n)];
      c += __popcll(__ballot(j < n && below(f, j)));
    }
    return c;
  }
  // Keys of group j's prefix (0: none).
  __device__ __forceinline__ int keys(const PagedArgs &a, int j) const {
    const int lo = first(a, j), hi = first(a, j + 1);
    const int P = few ? __builtin_amdgcn_readlane(prefix, j) : uniform_load(a.prefix_len, j);
    if (lo < 0 || hi > a.B || lo >= hi || P <= 0) return 0;
    return P;
  }
};
// Keys that request i (context L) reads through its group: those of the last group that starts
// at or before i, if it holds i.
__device__ __forceinline__ int request_prefix(const PagedArgs &a, const Groups &gr, int i, int L, bool report) {
  const int lo = gr.count(a, [&](int f, int) { return f <= i; });
  if (lo == 0 || i >= gr.first(a, lo)) return 0;
  const int P = gr.keys(a, lo - 1);
  if (P > L) {
    if (report && a.dev_err) atomicOr(a.dev_err, DCUT_DERR_GROUP);
    return 0;
  }
  return P;
}

// SHARED: in a call with groups.
template <int MODE, bool SHARED, int TM, int THREADS>
__device__ __forceinline__ bool find_item(const PagedArgs &a, int idx, int units, int *s_cnt, Item &it) {
  it.g = idx % a.n_kv;
  const int rest = idx / a.n_kv;
  const int u = rest % units;
  int c = rest / units;
  if (MODE == LIST) {
    const int t = u;
    if (t >= a.cu[a.B] || t >= a.max_rows) return false;
    const int n = a.list_keys[t * a.n_kv + it.g];
    it.t0 = t; it.rows = a.G; it.r0 = 0;
    it.tab = a.list + ((size_t)t * a.n_kv + it.g) * a.n_sel;
    it.nc = split_count(a.split, n);
    if (n <= 0 || c >= it.nc) return false;
    const int ch = split_chunk(a.split, n);
    it.kstart = it.klo = c * ch;
    it.kend = min(n, it.klo + ch);
    it.diag = n - 1;
    it.slot = c;
    it.first = c == 0 && it.g == 0;
    return true;
  }
  if (MODE == PREFIX) {
    const Groups gr(a);
    auto start = [&](int f) { return a.cu[min(max(f, 0), a.B)]; };
    const int grp = gr.count(a, [&](int f, int j) { return run_tile(start(f), a.G, TM, j) <= u; }) - 1;
    if (grp < 0) return false;
    const int P = gr.keys(a, grp);
    if (P == 0) return false;
    const int lo = gr.first(a, grp);
    it.t0 = uniform_load(a.cu, lo);
    const int d = uniform_load(a.cu, gr.first(a, grp + 1)) - it.t0;
    if (it.t0 < 0 || d <= 0 || it.t0 > a.max_rows - d) return false;
    it.rows = d * a.G;
    const long long r0 = ((long long)u - run_tile(it.t0, a.G, TM, grp)) * TM;
    if (r0 < 0 || r0 >= it.rows) return false;
    it.r0 = (int)r0;
    if ((long long)P > (long long)a.table_ld << a.lpage || P > a.max_ctx) return false;
    it.tab = a.table + (size_t)lo * a.table_ld;
    const int ncp = split_count(a.psplit, P);
    if (c >= ncp) return false;
    const int ch = split_chunk(a.psplit, P);
    it.kstart = it.klo = c * ch;
    it.kend = min(P, it.klo + ch);
    it.diag = 1 << 30;
    it.nc = 2;
    it.slot = c;
    it.first = false;
    return true;
  }
  int i = u;
  long long r0 = 0;
  if (!SHARED && a.plan) {
    const int e = idx / a.n_kv;
    const int4 item = ((const int4 *)((const char *)a.plan + PLAN_HEAD))[e];
    if (e >= a.plan[0]) return false;
    i = item.x;
    r0 = item.y;
    c = item.z;
  } else if (a.G * a.max_block > TM) {
    auto first_tile = [&](int j) { return run_tile(a.cu[j], a.G, TM, j); };
    // a refused request need not be any tile's: the first workgroup looks at all of them
    if (idx == 0)
      for (int j = threadIdx.x; j < a.B; j += THREADS) {
        ReqRows r;
        paged_request(a, j, true, r);
      }
    i = find_run<THREADS>(a.B, u, s_cnt, first_tile);
    if (i < 0) return false;
    r0 = ((long long)u - first_tile(i)) * TM;
  }
  const bool report = (SHARED || !a.plan) && c == 0 && it.g == 0 && threadIdx.x == 0;      // the plan has reported
  ReqRows r;
  if (!paged_request(a, i, report, r)) return false;
  it.t0 = r.t0;
  it.rows = r.d * a.G;
  if (r0 < 0 || r0 >= it.rows) return false;
  it.r0 = (int)r0;
  it.tab = a.table + (size_t)i * a.table_ld;
  const int P = SHARED ? request_prefix(a, Groups(a), i, r.L, report) : 0;
  const int ncp = P > 0 ? split_count(a.psplit, P) : 0;
  const int nc = split_count(a.split, r.L - P);
  if (c >= nc) return false;
  const int ch = split_chunk(a.split, r.L - P);
  const int last_row = (min(it.r0 + TM, it.rows) - 1) / a.G;
  it.klo = P + c * ch;
  it.kend = c == nc - 1 ? r.L + last_row + 1 : P + (c + 1) * ch;
  it.kstart = it.klo & ~15;                 // within klo's page: the table's entries before it may be unset
  it.diag = r.L;
  it.nc = ncp + nc;
  it.slot = ncp + c;
  it.first = c == 0 && it.g == 0;
  return true;
}

// The same in scalar registers: every thread found the same item, which the compiler cannot
// see through its searches (branches of the key loop would become divergent ones: a prompt's
// attention with 64-wide heads took 234 us instead of 178).
template <int MODE, bool SHARED, int TM, int THREADS>
__device__ __forceinline__ bool make_item(const PagedArgs &a, int idx, int units, int *s_cnt, Item &it) {
  Item x;
  if (!find_item<MODE, SHARED, TM, THREADS>(a, idx, units, s_cnt, x)) return false;
  it.g = uniform_int(x.g);
  it.t0 = uniform_int(x.t0);
  it.rows = uniform_int(x.rows);
  it.r0 = uniform_int(x.r0);
  it.klo = uniform_int(x.klo);
  it.kend = uniform_int(x.kend);
  it.kstart = uniform_int(x.kstart);
  it.diag = uniform_int(x.diag);
  it.nc = uniform_int(x.nc);
  it.slot = uniform_int(x.slot);
  it.first = uniform_int(x.first) != 0;
  const uintptr_t t = (uintptr_t)x.tab;
  it.tab = (const int32_t *)(((uintptr_t)(uint32_t)uniform_int((int)(t >> 32)) << 32) | (uint32_t)uniform_int((int)t));
  return true;
}

// Two floats rounded to bf16 (nearest even) in one instruction.
__device__ __forceinline__ uint32_t cvt_bf2(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef float float2v __attribute__((ext_vector_type(2)));
  const bf16x2 r = __builtin_convertvector((float2v){a, b}, bf16x2);
  return __builtin_bit_cast(uint32_t, r);
}

// Value and partner's in the other half of the wave, in the lane 16 on or back: joined.
__device__ __forceinline__ float half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float row_max(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float row_sum(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The reference m of a row's weights exp2(s - m) is only raised when a score passes it by this:
// the weights stay below 2^8, well within float32 and with bf16's full precision, and most
// tiles leave the accumulators alone.  Each row decides for itself (others multiply by 1).
constexpr float RAISE = 8.0f;

// log2(e) / sqrt(hd): scores in the exp2 domain.  Large scores are scaled first and the
// reference subtracted then (no fused multiply-add): however large they are, the largest weight
// is exact; scaled inside the subtraction's fma, a score past 2^34 keeps a rounding error of 2^7
// and more, whose exp2 overflows.
template <int HD>
constexpr float SCORE_SCALE = 1.4426950408889634f / (HD == 128 ? 11.313708498984761f : 8.0f);

// LDS layout of a tile: key r at r * ROWB, its 16-byte chunk c at place c ^ swizzle(r), linear in
// r's bits.  The 16-byte places of a 256-byte line are then met once by each of
//   - the 16 lanes that a 16-byte read serves together (0-3, 12-15 and 20-27; the others likewise),
//     reading keys 0-15 at one chunk (32 x 32 tiles) or, in lanes 16-31, at its neighbour
//     (16 x 16), so keys at neighbouring places are 12 apart;
//   - the 32 lanes of a transposing read: four chunks of four keys, or two chunks of eight.
// The conflict counter reads 0; keys at place c ^ 2 r + (r >> 3) cost a third of the LDS's cycles.
template <int HD>
__device__ __forceinline__ constexpr int swizzle(int r) {
  return (HD == 128 ? 4 * (r & 3) : 2 * (r & 2)) | (((r >> 1) & 2) ^ (3 * ((r >> 3) & 1)));
}

// Loads of one stage of KEYS keys (a K tile and a V tile) from the pages of a work item by NW
// waves, straight into LDS, 1 KB a wave load. 
// Every wave load lies in one page, whose number is a scalar load asked for
// one stage ahead; keys outside the item's chunk read as zeros, whatever stale slots hold.
template <int HD, int KEYS, int NW, int POLICY>
struct StageLoader {
  static constexpr int ROWB = HD * 2, CPR = ROWB / 16, TILEB = KEYS * ROWB, RPI = 1024 / ROWB;
  static constexpr int LPK = TILEB / 1024 / NW;        // wave loads for K (and for V)
  static_assert(TILEB / 1024 % NW == 0 && LPK >= 1, "every wave loads the same number of blocks");
  int pid[LPK];                             // pages of the stage asked for last
  unsigned worst = 0;                       // largest page number met: all are of keys of the item
  const char *k, *v;                        // the kv head's part of page 0
  uint32_t stride;                          // bytes from a page to the next
  int wave, lrow, lchk, page_bytes, last_page;

  __device__ __forceinline__ StageLoader(const PagedArgs &a, const Item &it, int lane, int w)
      : wave(w), lrow(lane / CPR), lchk(lane % CPR), page_bytes(a.page * ROWB), last_page((it.kend - 1) >> a.lpage) {
    k = (const char *)a.k + (size_t)it.g * page_bytes;
    v = (const char *)a.v + (size_t)it.g * page_bytes;
    stride = (uint32_t)(a.n_kv * page_bytes);
  }

  __device__ __forceinline__ void ask(const PagedArgs &a, const Item &it, int stage) {
#pragma unroll
    for (int j = 0; j < LPK; ++j) {
      const int p = it.kstart + stage * KEYS + (wave + NW * j) * RPI;
      pid[j] = uniform_load(it.tab, min(p >> a.lpage, last_page));
    }
  }
  __device__ __forceinline__ uint64_t page_at(const PagedArgs &a, int id) {
    const unsigned pg = (unsigned)id;
    worst = worst > pg ? worst : pg;
    return (uint64_t)(pg < (unsigned)a.n_pages ? pg : 0u) * stride;
  }
  // Byte of block j's page that this lane loads; 0x80000000 (past every page) for keys outside the chunk.
  __device__ __forceinline__ unsigned lane_byte(const PagedArgs &a, const Item &it, int stage, int j) const {
    const int blk = wave + NW * j;                   // 1 KB block of the tile
    const int r = blk * RPI + lrow, pb = it.kstart + stage * KEYS + blk * RPI, p = pb + lrow;
    const unsigned in = ((pb & (a.page - 1)) + lrow) * ROWB + 16 * (lchk ^ swizzle<HD>(r));
    return p >= it.klo && p < it.kend ? in : 0x80000000u;
  }
  __device__ __forceinline__ void block(const char *page, unsigned vo, int j, unsigned char *to) const {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(uniform_rsrc(page, page_bytes), (lds_void *)(to + (wave + NW * j) * 1024), 16, vo, 0, 0, POLICY);
  }
  // Both tiles of a stage.
  __device__ __forceinline__ void load(const PagedArgs &a, const Item &it, int stage, unsigned char *to_k, unsigned char *to_v) {
#pragma unroll
    for (int j = 0; j < LPK; ++j) {
      const uint64_t off = page_at(a, pid[j]);
      const unsigned vo = lane_byte(a, it, stage, j);
      block(k + off, vo, j, to_k);
      block(v + off, vo, j, to_v);
    }
  }
  // The K tile of a stage, whose pages and lane bytes are kept for its V tile.
  uint64_t v_off[LPK];
  unsigned v_vo[LPK];
  __device__ __forceinline__ void load_k(const PagedArgs &a, const Item &it, int stage, unsigned char *to) {
#pragma unroll
    for (int j = 0; j < LPK; ++j) {
      v_off[j] = page_at(a, pid[j]);
      v_vo[j] = lane_byte(a, it, stage, j);
      block(k + v_off[j], v_vo[j], j, to);
    }
  }
  __device__ __forceinline__ void load_v(unsigned char *to) const {
#pragma unroll
    for (int j = 0; j < LPK; ++j) block(v + v_off[j], v_vo[j], j, to);
  }
  __device__ __forceinline__ void report(const PagedArgs &a, int lane) const {
    if (worst >= (unsigned)a.n_pages && lane == 0 && a.dev_err) atomicOr(a.dev_err, DCUT_DERR_PAGE);
  }
};

// A value that is infinite or NaN at a key that some row does not see would reach that row
// through its weight 0.  Stages with such keys are searched: the values become zeros in LDS,
// and after the loop go to the rows that see them (special_value).  The whole workgroup calls
// this between its barrier and the use of the stage; returns whether there was one.
template <int TILEB, int THREADS>
__device__ __forceinline__ bool clear_specials(unsigned char *v) {
  bool odd = false;
#pragma unroll
  for (int i = 0; i < TILEB / 16 / THREADS; ++i) {
    uint4 *at = (uint4 *)(v + 16 * (threadIdx.x + THREADS * i));
    uint4 x = *at;
    uint32_t *w = (uint32_t *)&x;
    bool here = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool lo = (w[e] & 0x7f80u) == 0x7f80u, hi = (w[e] & 0x7f800000u) == 0x7f800000u;
      here |= lo | hi;
      w[e] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0x0000ffffu : ~0u);
    }
    if (here) *at = x;
    odd |= here;
  }
  return __syncthreads_or(odd);
}
__device__ __forceinline__ float special_value(uint16_t x, bool seen) { return (x & 0x7f80) == 0x7f80 && seen ? bf2f(x) : 0.0f; }

}  // namespace
}  // namespace dcut
