// Attention over the paged cache for units of many rows: prompts, and the prefix of a group.
//
// The same sums as paged_attn.hip in tiles of 32 keys x 32 rows a wave
// (v_mfma_f32_32x32x16_bf16), which halves the LDS reads a product takes against 16 x 16:
//   S^T[key][row] = K[key][:] . Q[row][:]   -> lane (row = lane%32, h = lane/32) owns keys
//                                              8 i + 4 h + j (i, j < 4) of the tile
//   O^T[d][row]  += V^T[d][key] . P^T[key][row], P straight from the S^T accumulators, V with
//                   the same order of keys from transposing LDS reads.
// The reference m of a row's weights exp2(s - m) is only raised when a score passes it by 8:
// the weights stay below 2^8, well within float32 and with bf16's full precision, and most
// tiles leave the accumulators alone.  Each row decides for itself (others multiply by 1).
#include <type_traits>

#include "paged_item.h"

namespace dcut {

namespace {

#ifndef TILE_NW
#define TILE_NW 8
#define TILE_NST 2
#define TILE_RB 1
#define TILE_KS 64
#define TILE_WPE 2
#endif
constexpr int KS = TILE_KS;     // keys per LDS stage
constexpr float RAISE = 8.0f;

// Transposing LDS reads of the V^T fragments of 32 keys, OFF bytes into the stage's tile, issued
// and awaited in one statement: fragment (16-key step u, column tile n) from its 8-key halves
// e = 0, 1, at r[(u NT + n) 2 + e].  The 8 keys of e = 1 flip chunk bit 3 of 256-byte keys, that
// is, they are read at the base of column tile n ^ 2.
template <int OFF>
__device__ __forceinline__ void read_values(short4v (&r)[16], const uint32_t (&b)[4]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %16 offset:%20\n\t"
      "ds_read_b64_tr_b16 %1, %18 offset:%21\n\t"
      "ds_read_b64_tr_b16 %2, %17 offset:%20\n\t"
      "ds_read_b64_tr_b16 %3, %19 offset:%21\n\t"
      "ds_read_b64_tr_b16 %4, %18 offset:%20\n\t"
      "ds_read_b64_tr_b16 %5, %16 offset:%21\n\t"
      "ds_read_b64_tr_b16 %6, %19 offset:%20\n\t"
      "ds_read_b64_tr_b16 %7, %17 offset:%21\n\t"
      "ds_read_b64_tr_b16 %8, %16 offset:%22\n\t"
      "ds_read_b64_tr_b16 %9, %18 offset:%23\n\t"
      "ds_read_b64_tr_b16 %10, %17 offset:%22\n\t"
      "ds_read_b64_tr_b16 %11, %19 offset:%23\n\t"
      "ds_read_b64_tr_b16 %12, %18 offset:%22\n\t"
      "ds_read_b64_tr_b16 %13, %16 offset:%23\n\t"
      "ds_read_b64_tr_b16 %14, %19 offset:%22\n\t"
      "ds_read_b64_tr_b16 %15, %17 offset:%23\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7]), "=&v"(r[8]), "=&v"(r[9]), "=&v"(r[10]), "=&v"(r[11]), "=&v"(r[12]), "=&v"(r[13]), "=&v"(r[14]), "=&v"(r[15])
      : "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "n"(OFF + 0), "n"(OFF + 2048), "n"(OFF + 4096), "n"(OFF + 6144)
      : "memory");
}
template <int OFF>
__device__ __forceinline__ void read_values(short4v (&r)[8], const uint32_t (&b)[2]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8 offset:%10\n\t"
      "ds_read_b64_tr_b16 %1, %8 offset:%11\n\t"
      "ds_read_b64_tr_b16 %2, %9 offset:%10\n\t"
      "ds_read_b64_tr_b16 %3, %9 offset:%11\n\t"
      "ds_read_b64_tr_b16 %4, %8 offset:%12\n\t"
      "ds_read_b64_tr_b16 %5, %8 offset:%13\n\t"
      "ds_read_b64_tr_b16 %6, %9 offset:%12\n\t"
      "ds_read_b64_tr_b16 %7, %9 offset:%13\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
      : "v"(b[0]), "v"(b[1]), "n"(OFF + 0), "n"(OFF + 1024), "n"(OFF + 2048), "n"(OFF + 3072)
      : "memory");
}

// The larger of a value and its partner's in the other half of the wave.
__device__ __forceinline__ float half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A wave owns RB blocks of 32 rows, 32 * NW rows apart.
template <int HD, int NW, int NSTAGE, int RB, int MODE>
__global__ void __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(TILE_WPE)))
k_paged_tile(PagedArgs a, int units) {
  constexpr int ROWB = HD * 2;
  constexpr int CPR = ROWB / 16;
  constexpr int TILEB = KS * ROWB;
  constexpr int STAGEB = 2 * TILEB;         // K tile then V tile
  constexpr int RPI = 1024 / ROWB;          // keys per 1 KB wave load
  constexpr int LPK = TILEB / 1024 / NW;
  constexpr int LPW = 2 * LPK;
  constexpr int NS = HD / 16;               // k-steps of the score product
  constexpr int NT = HD / 32;               // 32-row tiles of O^T
  constexpr int TM = RB * NW * 32;
  static_assert(TILEB / 1024 % NW == 0 && LPK >= 1, "every wave loads the same number of blocks");
  extern __shared__ __align__(1024) unsigned char ring[];
  __shared__ int s_cnt[NW];

  Item it;
  if (!make_item<MODE, TM, NW * 64, KS>(a, blockIdx.x, units, s_cnt, it)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5, l16 = lane & 15, g1 = (lane >> 4) & 1;
  const int R = it.rows - it.r0;

  bool row_ok[RB];
  int trow[RB], head[RB], kmax[RB];
  int kfirst[RB], klast[RB];                // last keys seen by the block's first and last rows: uniform
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int b0 = (rb * NW + wave) * 32, rr = b0 + l32;
    row_ok[rb] = rr < R;
    const int pair = row_ok[rb] ? it.r0 + rr : it.r0;
    const int krow = pair / a.G;
    head[rb] = it.g * a.G + pair - krow * a.G;
    trow[rb] = it.t0 + krow;
    kmax[rb] = MODE == OWN ? it.diag + krow : it.diag;
    kfirst[rb] = __builtin_amdgcn_readfirstlane(kmax[rb]);
    const int last = min(b0 + 31, R - 1);
    klast[rb] = b0 >= R ? -1 : MODE == OWN ? it.diag + (it.r0 + last) / a.G : it.diag;
  }

  bf16x8 qf[RB][NS];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const uint16_t *qp = a.q + (size_t)trow[rb] * a.ldq + (size_t)head[rb] * HD + 8 * h;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      uint4 z = make_uint4(0, 0, 0, 0);
      qf[rb][s] = row_ok[rb] ? *(const bf16x8 *)(qp + 16 * s) : *(bf16x8 *)&z;
    }
  }

  floatx16 o[RB][NT];
  float m_run[RB], l_run[RB];               // l: this lane's keys only, joined at the end
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[rb][n][r] = 0.0f;
    m_run[rb] = -__builtin_inff();
    l_run[rb] = 0.0f;
  }
  constexpr float sl2 = 1.4426950408889634f / (HD == 128 ? 11.313708498984761f : 8.0f);   // log2(e) / sqrt(hd)
  static_assert(HD == 64 || HD == 128, "sqrt of the head dimension");

  const int lrow = lane / CPR, lchk = lane % CPR;
  const int page_bytes = a.page * ROWB;
  const int last_page = (it.kend - 1) >> a.lpage;
  auto page_of = [&](int tile, int j) {
    const int p = it.kstart + tile * KS + (wave + NW * j) * RPI;
    return uniform_load(it.tab, min(p >> a.lpage, last_page));
  };
  int pid[LPK];
  bool bad_page = false;
  auto issue = [&](int tile, int slot) {
    const int p0 = it.kstart + tile * KS;
    unsigned char *st = ring + slot * STAGEB;
#pragma unroll
    for (int j = 0; j < LPK; ++j) {
      const int blk = wave + NW * j;
      const int r = blk * RPI + lrow;
      const int pb = p0 + blk * RPI;
      int pg = pid[j];
      if ((unsigned)pg >= (unsigned)a.n_pages) {     // uniform
        if (pb < it.kend) bad_page = true;
        pg = 0;
      }
      const size_t off = ((size_t)pg * a.n_kv + it.g) * (size_t)page_bytes;
      const __amdgpu_buffer_rsrc_t rK = uniform_rsrc((const char *)a.k + off, page_bytes);
      const __amdgpu_buffer_rsrc_t rV = uniform_rsrc((const char *)a.v + off, page_bytes);
      const int p = p0 + r;
      const unsigned in = ((pb & (a.page - 1)) + lrow) * ROWB + 16 * (lchk ^ (r % CPR));
      const unsigned vo = p >= it.klo && p < it.kend ? in : 0x80000000u;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rK, (lds_void *)(st + blk * 1024), 16, vo, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rV, (lds_void *)(st + TILEB + blk * 1024), 16, vo, 0, 0, 0);
    }
  };

  // Fragment addresses within a step of 32 keys.  K: key l32, chunk (2 s + h) ^ (key % CPR).
  // V: keys 16 u + 8 e + 4 h + (l16 >> 2), columns 32 n + 16 g1 + 4 (l16 & 3)..+3; the column
  // tile n flips chunk bits 2-3.
  const uint32_t ring0 = (uint32_t)(uintptr_t)(lds_void *)ring;
  const uint32_t kfrag = ring0 + l32 * ROWB + 16 * (h ^ (l32 % CPR));
  const int vkey = 4 * h + (l16 >> 2);
  const uint32_t vfrag = ring0 + TILEB + vkey * ROWB + 16 * ((2 * g1 + ((l16 & 3) >> 1)) ^ vkey) + 8 * (l16 & 1);

  // keys up to seen_last are seen by some row of the wave, those below full_end by all
  const int seen_last = max(klast[0], klast[RB - 1]);
  const int full_end = min(it.kend, min(kfirst[0], kfirst[RB - 1]) + 1);
  constexpr int KB = KS / 32;
  auto step = [&](const int p0, const uint32_t ks, const uint32_t vs) __attribute__((always_inline)) {
#pragma clang fp contract(off)     // the scaled scores' subtraction stays one, as in paged_attn.hip
    floatx16 s[RB][KB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[rb][kb][r] = 0.0f;
#pragma unroll
    for (int st = 0; st < NS; ++st)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const bf16x8 kf = *(lds_frag *)(uintptr_t)((ks ^ (32 * st)) + kb * 32 * ROWB);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) s[rb][kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[rb][st], s[rb][kb], 0, 0, 0);
      }
    // some key of the step is hidden from some row of the wave
    if (p0 < it.klo || p0 + KS > full_end) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const uint32_t n = (uint32_t)max(min(it.kend, kmax[rb] + 1) - it.klo, 0);    // keys from klo on that the row sees
        const int first = p0 + 4 * h - it.klo;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            s[rb][kb][r] = (uint32_t)(first + 32 * kb + 8 * (r >> 2) + (r & 3)) < n ? s[rb][kb][r] : -__builtin_inff();
      }
    }
    bf16x8 pf[RB][2 * KB];
    bool raise = false;
    float alpha[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[rb][kb] *= sl2;
      float tmax = s[rb][0][0];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) tmax = fmaxf(tmax, s[rb][kb][r]);
      tmax = half_max(tmax);
      const float m_new = tmax > m_run[rb] + RAISE ? tmax : m_run[rb];
      // a row that has seen no key yet keeps m = -inf; subtracting 0 then keeps its weights at 0
      const float sub = m_new == -__builtin_inff() ? 0.0f : m_new;
      alpha[rb] = __builtin_amdgcn_exp2f(m_run[rb] - sub);
      raise |= m_new != m_run[rb];
      m_run[rb] = m_new;
      float psum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float pv = __builtin_amdgcn_exp2f(s[rb][kb][r] - sub);
          s[rb][kb][r] = pv;
          psum[r & 3] += pv;
        }
      l_run[rb] = __builtin_fmaf(l_run[rb], alpha[rb], (psum[0] + psum[1]) + (psum[2] + psum[3]));
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        uint32_t *pw = (uint32_t *)&pf[rb][2 * kb];
#pragma unroll
        for (int e = 0; e < 8; ++e) pw[e] = cvt_bf2(s[rb][kb][2 * e], s[rb][kb][2 * e + 1]);
      }
    }
    if (__any(raise)) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int n = 0; n < NT; ++n) o[rb][n] *= alpha[rb];
    }
    uint32_t vb[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) vb[n] = vs ^ (64 * n);
    auto values = [&](auto off, int kb) __attribute__((always_inline)) {
      short4v vr[4 * NT];
      read_values<decltype(off)::value>(vr, vb);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          bf16x8 vf;
          short4v *vw = (short4v *)&vf;
          vw[0] = vr[(u * NT + n) * 2];
          vw[1] = vr[(u * NT + n) * 2 + 1];
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
            o[rb][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[rb][2 * kb + u], o[rb][n], 0, 0, 0);
        }
    };
    values(std::integral_constant<int, 0>{}, 0);
    if (KB == 2) values(std::integral_constant<int, 32 * ROWB>{}, KB - 1);
  };
  // A value that is infinite or NaN at a key that some row does not see would reach that row
  // through its weight 0.  Stages with such keys are searched for them: they become zeros in
  // LDS, and after the loop (add_specials) go to the rows that see them.
  const int mixed_from = MODE == OWN ? it.diag + it.r0 / a.G + 1 : it.kend;     // first key hidden from the tile's first row
  int special_from = it.kend;                                    // first stage that had one
  auto clear_specials = [&](int p0, unsigned char *v) {
    bool odd = false;
#pragma unroll
    for (int i = 0; i < TILEB / 16 / (NW * 64); ++i) {
      uint4 *at = (uint4 *)(v + 16 * (tid + NW * 64 * i));
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
    if (__syncthreads_or(odd)) special_from = min(special_from, p0);
  };

  const int ntiles = (it.kend - it.kstart + KS - 1) / KS;
#pragma unroll
  for (int s = 0; s < NSTAGE; ++s) {
#pragma unroll
    for (int j = 0; j < LPK; ++j) pid[j] = page_of(s, j);
    if (s < NSTAGE - 1 && s < ntiles) issue(s, s);
  }
  constexpr int W0 = 0 | (7 << 4) | (15 << 8);
  constexpr int W1 = (LPW & 15) | ((LPW >> 4) << 14) | (7 << 4) | (15 << 8);
  static_assert(NSTAGE == 2 || NSTAGE == 3, "waits for at most one stage in flight");
  int slot = 0;
  for (int tile = 0; tile < ntiles; ++tile) {
    if (NSTAGE == 3 && tile + 1 < ntiles) __builtin_amdgcn_s_waitcnt(W1);
    else __builtin_amdgcn_s_waitcnt(W0);
    ring_barrier();
    int next = slot + NSTAGE - 1;
    if (next >= NSTAGE) next -= NSTAGE;
    if (tile + NSTAGE - 1 < ntiles) issue(tile + NSTAGE - 1, next);
#pragma unroll
    for (int j = 0; j < LPK; ++j) pid[j] = page_of(tile + NSTAGE, j);
    const int p0 = it.kstart + tile * KS;
    if (p0 + KS > mixed_from) clear_specials(p0, ring + slot * STAGEB + TILEB);     // uniform over the workgroup
    if (p0 <= seen_last) step(p0, kfrag + slot * STAGEB, vfrag + slot * STAGEB);
    if (++slot == NSTAGE) slot = 0;
  }
  if (special_from < it.kend) {
    for (int p = max(special_from, it.klo); p < it.kend; ++p) {
      const int pg = uniform_load(it.tab, p >> a.lpage);
      if ((unsigned)pg >= (unsigned)a.n_pages) continue;
      const uint16_t *v = a.v + (((size_t)pg * a.n_kv + it.g) * a.page + (p & (a.page - 1))) * HD + 4 * h;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const uint16_t x = v[32 * n + 8 * (r >> 2) + (r & 3)];
            if ((x & 0x7f80) == 0x7f80 && p <= kmax[rb]) o[rb][n][r] += bf2f(x);
            if ((r & 3) == 3) __builtin_amdgcn_sched_barrier(0);     // rare: keep its loads from taking registers of the loop
          }
    }
  }
  if (bad_page && lane == 0 && a.dev_err) atomicOr(a.dev_err, DCUT_DERR_PAGE);
  // lane holds O^T[32n + 8 i + 4 h + j][row]
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const float l = half_sum(l_run[rb]);
    if (!row_ok[rb]) continue;
    const size_t pair = (size_t)trow[rb] * a.n_q + head[rb];
    if (it.nc == 1) {
      const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
      uint16_t *op = a.out + pair * HD + 4 * h;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *(uint2 *)(op + 32 * n + 8 * i) = make_uint2(cvt_bf2(o[rb][n][4 * i] * inv, o[rb][n][4 * i + 1] * inv),
                                                       cvt_bf2(o[rb][n][4 * i + 2] * inv, o[rb][n][4 * i + 3] * inv));
      if (a.lse && h == 0) a.lse[pair] = 0.6931471805599453f * (m_run[rb] + __builtin_amdgcn_logf(l));
    } else {
      float *pp = a.part + (pair * a.MC + it.slot) * ATTN_PITCH(HD);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *(float4 *)(pp + 32 * n + 8 * i + 4 * h) = make_float4(o[rb][n][4 * i], o[rb][n][4 * i + 1], o[rb][n][4 * i + 2], o[rb][n][4 * i + 3]);
      if (h == 0) {
        pp[HD] = m_run[rb];
        pp[HD + 1] = l;
      }
    }
    if (it.first && h == 0 && a.row_nc) a.row_nc[trow[rb]] = it.nc;
  }
}

template <int HD, int NW, int NSTAGE, int RB, int MODE>
int launch_tile(const PagedArgs &a, int units, int mc, hipStream_t s) {
  const long long grid = (long long)units * a.n_kv * mc;
  if (grid > 0x7fffffffLL) return DCUT_EUNSUPPORTED;
  const size_t lds = (size_t)NSTAGE * 2 * KS * HD * 2;
  return launch(MODE == PREFIX ? DCUT_KERNEL_PAGED_PREFIX : DCUT_KERNEL_PAGED_ATTN, k_paged_tile<HD, NW, NSTAGE, RB, MODE>,
                dim3((unsigned)grid), dim3(NW * 64), lds, s, a, units);
}


}  // namespace

int paged_tile_rows() { return TILE_NW * TILE_RB * 32; }

int paged_tile_launch(const PagedArgs &a, int head_dim, bool prefix, int units, int mc, hipStream_t s) {
  if (head_dim == 128)
    return prefix ? launch_tile<128, TILE_NW, TILE_NST, TILE_RB, PREFIX>(a, units, mc, s)
                  : launch_tile<128, TILE_NW, TILE_NST, TILE_RB, OWN>(a, units, mc, s);
  return prefix ? launch_tile<64, TILE_NW, TILE_NST, TILE_RB, PREFIX>(a, units, mc, s)
                : launch_tile<64, TILE_NW, TILE_NST, TILE_RB, OWN>(a, units, mc, s);
}

}  // namespace dcut
