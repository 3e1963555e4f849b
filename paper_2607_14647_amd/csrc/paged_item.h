// Work items of the paged attention kernels (device side): which rows, kv head and keys a
// workgroup takes, and the operand loads they share.
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

enum Mode { OWN = 0, PREFIX = 1, LIST = 2 };

// What a work item reads and computes; uniform over the workgroup.
struct Item {
  int g;               // kv head
  int t0, rows, r0;    // first packed row of the unit, its (row, head) pairs, first of this tile
  const int32_t *tab;  // page of keys j*page.. of the unit
  int klo, kend;       // keys of the chunk; below klo and from kend on: none
  int kstart;          // first key tile
  int diag;            // packed row t0 + r sees keys up to diag + r
  int nc, slot;        // partials of the rows, and which this one is
  bool first;          // this item notes the rows' count of partials
};

// The unit a launch index names, where units are tiles of TM pairs of consecutive runs:
// run i's tiles are numbered from floor(start_i G / TM) + i on, which no two runs share.
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

// Keys of the group's prefix that request i reads through it (0: none), and its chunks.
__device__ __forceinline__ int shared_prefix(const PagedArgs &a, int grp) {
  const int lo = a.group_cu[grp], hi = a.group_cu[grp + 1], P = a.prefix_len[grp];
  if (lo < 0 || hi > a.B || lo >= hi || P <= 0) return 0;
  return P;
}

// ALIGN: key tiles start at multiples of it.
template <int MODE, int TM, int THREADS, int ALIGN>
__device__ __forceinline__ bool make_item(const PagedArgs &a, int idx, int units, int *s_cnt, Item &it) {
  it.g = idx % a.n_kv;
  const int rest = idx / a.n_kv;
  const int u = rest % units;
  const int c = rest / units;
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
    auto first_tile = [&](int j) {
      const int lo = min(max(a.group_cu[j], 0), a.B);
      return (int)((long long)a.cu[lo] * a.G / TM) + j;
    };
    const int grp = find_run<THREADS>(a.n_groups, u, s_cnt, first_tile);
    if (grp < 0) return false;
    const int P = shared_prefix(a, grp);
    if (P == 0) return false;
    const int lo = a.group_cu[grp], hi = a.group_cu[grp + 1];
    it.t0 = a.cu[lo];
    const int d = a.cu[hi] - it.t0;
    if (it.t0 < 0 || d <= 0 || it.t0 > a.max_rows - d) return false;
    it.rows = d * a.G;
    const long long r0 = ((long long)u - first_tile(grp)) * TM;
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
  if (a.G * a.max_block > TM) {
    auto first_tile = [&](int j) { return (int)((long long)a.cu[j] * a.G / TM) + j; };
    i = find_run<THREADS>(a.B, u, s_cnt, first_tile);
    if (i < 0) return false;
    r0 = ((long long)u - first_tile(i)) * TM;
  }
  ReqRows r;
  if (!paged_request(a, i, c == 0 && it.g == 0 && threadIdx.x == 0, r)) return false;
  it.t0 = r.t0;
  it.rows = r.d * a.G;
  if (r0 < 0 || r0 >= it.rows) return false;
  it.r0 = (int)r0;
  it.tab = a.table + (size_t)i * a.table_ld;
  int P = 0, ncp = 0;
  if (a.n_groups > 0) {
    // the last group that starts at or before i, if it holds i
    const int grp = find_run<THREADS>(a.n_groups, i, s_cnt, [&](int j) { return a.group_cu[j]; });
    if (grp >= 0 && i < a.group_cu[grp + 1]) {
      P = shared_prefix(a, grp);
      if (P > r.L) {
        if (c == 0 && it.g == 0 && threadIdx.x == 0 && a.dev_err) atomicOr(a.dev_err, DCUT_DERR_GROUP);
        P = 0;
      } else if (P > 0) {
        ncp = split_count(a.psplit, P);
      }
    }
  }
  const int nc = split_count(a.split, r.L - P);
  if (c >= nc) return false;
  const int ch = split_chunk(a.split, r.L - P);
  const int last_row = (min(it.r0 + TM, it.rows) - 1) / a.G;
  it.klo = P + c * ch;
  it.kend = c == nc - 1 ? r.L + last_row + 1 : P + (c + 1) * ch;
  it.kstart = it.klo & ~(ALIGN - 1);
  it.diag = r.L;
  it.nc = ncp + nc;
  it.slot = ncp + c;
  it.first = c == 0 && it.g == 0;
  return true;
}

// Two floats rounded to bf16 (nearest even) in one instruction.
__device__ __forceinline__ uint32_t cvt_bf2(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef float float2v __attribute__((ext_vector_type(2)));
  const bf16x2 r = __builtin_convertvector((float2v){a, b}, bf16x2);
  return __builtin_bit_cast(uint32_t, r);
}

}  // namespace
}  // namespace dcut
