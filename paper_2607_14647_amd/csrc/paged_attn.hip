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
// Per key tile and wave (v_mfma_f32_16x16x32_bf16):
//   S^T[key][row] = K[key][:] . Q[row][:]   -> lane (row = lane%16) owns keys 4*(lane/16)+j
//   O^T[d][row]  += V^T[d][key] . P^T[key][row], P straight from the S^T accumulators (rounded
//                   to bf16, the width of the matrix operand), V transposed by the LDS reads.
// Keys and values arrive through a ring of LDS stages (buffer loads with the LDS destination);
// every wave load of 1 KB lies in one page, whose number is one scalar load, asked for a tile
// ahead.  Keys outside the chunk read as zeros, whatever stale slots hold.
#include "paged_item.h"

namespace dcut {

namespace {

constexpr int KT = 32;     // keys per tile

// Transposing LDS reads of four column tiles x two key halves, the second half HALF bytes
// after the first, issued and awaited in one statement.
template <int HALF>
__device__ __forceinline__ void lds_read_tr16_x8(short4v (&r)[8], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\t"
      "ds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
      "ds_read_b64_tr_b16 %2, %9\n\t"
      "ds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
      "ds_read_b64_tr_b16 %4, %10\n\t"
      "ds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
      "ds_read_b64_tr_b16 %6, %11\n\t"
      "ds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
      : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "n"(HALF)
      : "memory");
}

// A wave owns RB blocks of 16 rows, 16 * NW rows apart.
template <int HD, int NW, int NSTAGE, int RB, int MODE>
__global__ void __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(3)))
k_paged_attn(PagedArgs a, int units) {
  constexpr int ROWB = HD * 2;              // bytes per key
  constexpr int CPR = ROWB / 16;            // 16-byte chunks per key
  constexpr int TILEB = KT * ROWB;
  constexpr int STAGEB = 2 * TILEB;         // K tile then V tile
  constexpr int RPI = 1024 / ROWB;          // keys per 1 KB wave load
  constexpr int LPK = (TILEB / 1024 + NW - 1) / NW;
  constexpr int LPW = 2 * LPK;
  constexpr int NS = HD / 32;
  constexpr int NT = HD / 16;
  constexpr int TM = RB * NW * 16;
  static_assert(TILEB / 1024 % NW == 0, "every wave loads the same number of blocks");
  __shared__ __align__(1024) unsigned char ring[NSTAGE * STAGEB];
  __shared__ int s_cnt[NW];

  Item it;
  if (!make_item<MODE, TM, NW * 64, KT>(a, blockIdx.x, units, s_cnt, it)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, grp4 = lane >> 4;
  const int R = it.rows - it.r0;            // pairs of this tile, if fewer than TM

  bool row_ok[RB];
  int trow[RB], head[RB], kmax[RB];         // packed row, query head, last visible key
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int rr = (rb * NW + wave) * 16 + l16;
    row_ok[rb] = rr < R;
    const int pair = row_ok[rb] ? it.r0 + rr : it.r0;
    const int krow = pair / a.G;
    head[rb] = it.g * a.G + pair - krow * a.G;
    trow[rb] = it.t0 + krow;
    kmax[rb] = MODE == LIST ? it.diag : it.diag + krow;
  }

  bf16x8 qf[RB][NS];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const uint16_t *qp = a.q + (size_t)trow[rb] * a.ldq + (size_t)head[rb] * HD + 8 * grp4;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      uint4 z = make_uint4(0, 0, 0, 0);
      qf[rb][s] = row_ok[rb] ? *(const bf16x8 *)(qp + 32 * s) : *(bf16x8 *)&z;
    }
  }

  floatx4 o[RB][NT];
  float m_run[RB], l_run[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
    for (int n = 0; n < NT; ++n) o[rb][n] = {0.f, 0.f, 0.f, 0.f};
    m_run[rb] = -__builtin_inff();
    l_run[rb] = 0.0f;
  }
  constexpr float sl2 = 1.4426950408889634f / (HD == 128 ? 11.313708498984761f : 8.0f);   // log2(e) / sqrt(hd)
  static_assert(HD == 64 || HD == 128, "sqrt of the head dimension");

  // Tile layout in LDS: key r at r * ROWB; its 16-byte chunk c holds the key's chunk
  // c ^ (r % CPR), so 16 consecutive keys read at one column land in different banks.
  const int lrow = lane / CPR, lchk = lane % CPR;
  const int page_bytes = a.page * ROWB;
  const int last_page = (it.kend - 1) >> a.lpage;
  auto page_of = [&](int tile, int j) {
    const int p = it.kstart + tile * KT + (wave + NW * j) * RPI;
    return uniform_load(it.tab, min(p >> a.lpage, last_page));
  };
  int pid[LPK];
  bool bad_page = false;
  auto issue = [&](int tile, int slot) {
    const int p0 = it.kstart + tile * KT;
    unsigned char *st = ring + slot * STAGEB;
#pragma unroll
    for (int j = 0; j < LPK; ++j) {
      const int blk = wave + NW * j;                 // 1 KB block of the K (and V) tile
      const int r = blk * RPI + lrow;                // key within the tile
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
      // a request's keys are read once: non-temporal; a prefix is read by every row tile
      constexpr int POL = MODE == OWN && RB == 1 ? CPOL_NT : 0;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rK, (lds_void *)(st + blk * 1024), 16, vo, 0, 0, POL);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rV, (lds_void *)(st + TILEB + blk * 1024), 16, vo, 0, 0, POL);
    }
  };

  // Fragment addresses within a tile.  K: key l16 (16-key blocks 16 keys apart), chunk
  // grp4 ^ (key % CPR), k-step s flips chunk bits 2-3.  V: source lane s of a 16-lane group
  // reads key k0 + s/4, columns 16n + 4(s%4)..+3, and lane d receives keys k0..k0+3 of column
  // 16n + d; the column tile n flips chunk bits 1-3, the second 16 keys lie 16 keys on.
  const int vrow = 4 * grp4 + (l16 >> 2);
  const uint32_t ring0 = (uint32_t)(uintptr_t)(lds_void *)ring;
  const uint32_t kfrag = ring0 + l16 * ROWB + 16 * (grp4 ^ (l16 % CPR));
  const uint32_t vfrag = ring0 + TILEB + vrow * ROWB + 16 * (((l16 & 3) >> 1) ^ (vrow % CPR)) + 8 * (l16 & 1);

  const int ntiles = (it.kend - it.kstart + KT - 1) / KT;
#pragma unroll
  for (int s = 0; s < NSTAGE; ++s) {
#pragma unroll
    for (int j = 0; j < LPK; ++j) pid[j] = page_of(s, j);
    if (s < NSTAGE - 1 && s < ntiles) issue(s, s);
  }
  constexpr int W0 = 0 | (7 << 4) | (15 << 8);
  constexpr int W1 = (LPW & 15) | ((LPW >> 4) << 14) | (7 << 4) | (15 << 8);
  constexpr int W2 = ((2 * LPW) & 15) | (((2 * LPW) >> 4) << 14) | (7 << 4) | (15 << 8);
  static_assert(NSTAGE <= 4, "waits for at most two tiles in flight");
  for (int tile = 0; tile < ntiles; ++tile) {
    const int pending = min(NSTAGE - 2, ntiles - 1 - tile);
    if (pending >= 2) __builtin_amdgcn_s_waitcnt(W2);
    else if (pending == 1) __builtin_amdgcn_s_waitcnt(W1);
    else __builtin_amdgcn_s_waitcnt(W0);
    ring_barrier();
    if (tile + NSTAGE - 1 < ntiles) issue(tile + NSTAGE - 1, (tile + NSTAGE - 1) % NSTAGE);
#pragma unroll
    for (int j = 0; j < LPK; ++j) pid[j] = page_of(tile + NSTAGE, j);
    const int p0 = it.kstart + tile * KT;
    const uint32_t ks = kfrag + (tile % NSTAGE) * STAGEB, vs = vfrag + (tile % NSTAGE) * STAGEB;
    // every key of the tile is visible to every row: no masks
    const bool full = p0 >= it.klo && p0 + KT <= min(it.kend, it.diag + 1);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
#pragma clang fp contract(off)     // the scaled scores' subtraction stays one (see below)
      if ((rb * NW + wave) * 16 >= R) break;   // uniform: no rows in this block or any later one
      floatx4 s4[KT / 16];
#pragma unroll
      for (int kb = 0; kb < KT / 16; ++kb) {
        s4[kb] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          const bf16x8 kf = *(lds_frag *)(uintptr_t)((ks ^ (64 * s)) + kb * 16 * ROWB);
          s4[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[rb][s], s4[kb], 0, 0, 0);
        }
      }
      uint32_t seen = 0xffu;                    // bit 4 kb + j: this lane's keys its row sees
      if (!full) {
        seen = 0;
#pragma unroll
        for (int kb = 0; kb < KT / 16; ++kb)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int p = p0 + kb * 16 + 4 * grp4 + j;
            const bool see = p >= it.klo && p < it.kend && p <= kmax[rb];
            seen |= (uint32_t)see << (4 * kb + j);
            if (!see) s4[kb][j] = -__builtin_inff();
          }
      }
      // Weights in the exp2 domain.  A score is scaled first and the maximum of the scaled
      // scores subtracted, so the largest weight is exactly 1 however large the scores are.
#pragma unroll
      for (int kb = 0; kb < KT / 16; ++kb) s4[kb] *= sl2;
      float tmax = fmaxf(fmaxf(s4[0][0], s4[0][1]), fmaxf(s4[0][2], s4[0][3]));
      tmax = fmaxf(tmax, fmaxf(fmaxf(s4[1][0], s4[1][1]), fmaxf(s4[1][2], s4[1][3])));
      tmax = fmaxf(tmax, __shfl_xor(tmax, 16, 64));
      tmax = fmaxf(tmax, __shfl_xor(tmax, 32, 64));
      const float m_new = fmaxf(m_run[rb], tmax);
      // a row that has seen no key yet keeps m = -inf; subtracting 0 then keeps its weights at 0
      const float sub = m_new == -__builtin_inff() ? 0.0f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m_run[rb] - sub);
      float psum = 0.0f;
#pragma unroll
      for (int kb = 0; kb < KT / 16; ++kb)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float pv = __builtin_amdgcn_exp2f(s4[kb][j] - sub);
          s4[kb][j] = pv;
          psum += pv;
        }
      psum += __shfl_xor(psum, 16, 64);
      psum += __shfl_xor(psum, 32, 64);
      l_run[rb] = __builtin_fmaf(l_run[rb], alpha, psum);
      m_run[rb] = m_new;
#pragma unroll
      for (int n = 0; n < NT; ++n) o[rb][n] *= alpha;

      // O^T += V^T P^T.  P^T slots of this lane: keys 4*grp4+j of the two 16-key blocks; the
      // V^T fragment with the same keys comes from two transposing reads.
      bf16x8 pf;
      uint32_t *pw = (uint32_t *)&pf;
      pw[0] = cvt_bf2(s4[0][0], s4[0][1]);
      pw[1] = cvt_bf2(s4[0][2], s4[0][3]);
      pw[2] = cvt_bf2(s4[1][0], s4[1][1]);
      pw[3] = cvt_bf2(s4[1][2], s4[1][3]);
      static_assert(NT % 4 == 0 && KT == 32, "transposing reads come in groups of four columns, one 32-key step");
#pragma unroll
      for (int n0 = 0; n0 < NT; n0 += 4) {
        short4v vr[8];
        lds_read_tr16_x8<16 * ROWB>(vr, vs ^ (32 * n0), vs ^ (32 * (n0 + 1)), vs ^ (32 * (n0 + 2)), vs ^ (32 * (n0 + 3)));
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          bf16x8 vf;
          short4v *vw = (short4v *)&vf;
          vw[0] = vr[2 * u];
          vw[1] = vr[2 * u + 1];
          if (!full) {
            // A key that a row does not see has weight 0, but 0 times an infinity or a NaN of
            // its value would reach the row.  Such values leave the product and are added to
            // the rows that see them, counted by kind.  Rare: one test a fragment of a masked tile.
            const uint16_t *vb = (const uint16_t *)&vf;
            bool odd = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) odd |= (vb[e] & 0x7f80) == 0x7f80;
            if (__any(odd)) {
              bf16x8 nanv, posv, negv, one;
              uint16_t *nb = (uint16_t *)&nanv, *pb = (uint16_t *)&posv, *gb = (uint16_t *)&negv, *ob = (uint16_t *)&one;
              uint16_t *cb = (uint16_t *)&vf;
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const uint16_t x = vb[e];
                const bool special = (x & 0x7f80) == 0x7f80, nan = special && (x & 0x7f);
                nb[e] = nan ? 0x3f80 : 0;
                pb[e] = special && !nan && !(x & 0x8000) ? 0x3f80 : 0;
                gb[e] = special && !nan && (x & 0x8000) ? 0x3f80 : 0;
                ob[e] = (seen >> e) & 1 ? 0x3f80 : 0;
                if (special) cb[e] = 0;
              }
              const floatx4 z = {0.f, 0.f, 0.f, 0.f};
              const floatx4 cn = __builtin_amdgcn_mfma_f32_16x16x32_bf16(nanv, one, z, 0, 0, 0);
              const floatx4 cp = __builtin_amdgcn_mfma_f32_16x16x32_bf16(posv, one, z, 0, 0, 0);
              const floatx4 cm = __builtin_amdgcn_mfma_f32_16x16x32_bf16(negv, one, z, 0, 0, 0);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                if (cp[j] > 0.0f) o[rb][n0 + u][j] += __builtin_inff();
                if (cm[j] > 0.0f) o[rb][n0 + u][j] -= __builtin_inff();
                if (cn[j] > 0.0f) o[rb][n0 + u][j] = __builtin_nanf("");
              }
            }
          }
          o[rb][n0 + u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf, o[rb][n0 + u], 0, 0, 0);
        }
      }
    }
  }
  if (bad_page && lane == 0 && a.dev_err) atomicOr(a.dev_err, DCUT_DERR_PAGE);
  // lane holds O^T[16n + 4*grp4 + j][row]
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    if (!row_ok[rb]) continue;
    const size_t pair = (size_t)trow[rb] * a.n_q + head[rb];
    if (it.nc == 1) {
      const float inv = l_run[rb] > 0.0f ? 1.0f / l_run[rb] : l_run[rb] == 0.0f ? 0.0f : l_run[rb];
      uint16_t *op = a.out + pair * HD;
#pragma unroll
      for (int n = 0; n < NT; ++n)
        *(uint2 *)(op + 16 * n + 4 * grp4) = make_uint2(cvt_bf2(o[rb][n][0] * inv, o[rb][n][1] * inv),
                                                        cvt_bf2(o[rb][n][2] * inv, o[rb][n][3] * inv));
      if (a.lse && grp4 == 0) a.lse[pair] = 0.6931471805599453f * (m_run[rb] + __builtin_amdgcn_logf(l_run[rb]));
    } else {
      float *pp = a.part + (pair * a.MC + it.slot) * ATTN_PITCH(HD);
#pragma unroll
      for (int n = 0; n < NT; ++n)
        *(float4 *)(pp + 16 * n + 4 * grp4) = make_float4(o[rb][n][0], o[rb][n][1], o[rb][n][2], o[rb][n][3]);
      if (grp4 == 0) {
        pp[HD] = m_run[rb];
        pp[HD + 1] = l_run[rb];
      }
    }
    if (it.first && grp4 == 0 && a.row_nc) a.row_nc[trow[rb]] = it.nc;
  }
}

// Merge of a (row, head)'s partials, one half wave each, in chunk order: lane c reads partial
// c's (max, sum), so the weights of up to 32 partials cost one memory round trip, taken
// together with the first eight partials' values.
template <int HD>
__global__ void __launch_bounds__(256)
k_paged_merge(PagedArgs a) {
  constexpr int PER = HD / 32, CG = 8;
  const int lane = threadIdx.x & 31;
  const int pair = blockIdx.x * 8 + (threadIdx.x >> 5);
  const int t = pair / a.n_q;
  const int nc0 = a.row_nc[min(t, a.max_rows - 1)];
  const int M = a.cu[a.B];
  if (t >= M || t >= a.max_rows) return;
  const int nc = min(nc0, a.MC);
  if (nc <= 1) return;
  const float *pp = a.part + (size_t)pair * a.MC * ATTN_PITCH(HD);
  float acc[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) acc[e] = 0.0f;
  float mx = -__builtin_inff(), lsum = 0.0f;
  for (int c0 = 0; c0 < nc; c0 += 32) {
    const int cnt = min(32, nc - c0);
    const float *p0 = pp + (size_t)c0 * ATTN_PITCH(HD);
    float xv[CG][PER];
    auto load = [&](int cc) {
#pragma unroll
      for (int u = 0; u < CG; ++u)
#pragma unroll
        for (int e = 0; e < PER; ++e) xv[u][e] = cc + u < cnt ? p0[(cc + u) * ATTN_PITCH(HD) + lane * PER + e] : 0.0f;
    };
    load(0);
    const float mv = lane < cnt ? p0[lane * ATTN_PITCH(HD) + HD] : -__builtin_inff();
    const float lv = lane < cnt ? p0[lane * ATTN_PITCH(HD) + HD + 1] : 0.0f;
    float gm = mv;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) gm = fmaxf(gm, __shfl_xor(gm, off, 32));
    const float mn = fmaxf(mx, gm), sub = mn == -__builtin_inff() ? 0.0f : mn;
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
      if (cc + CG >= cnt) break;
      load(cc + CG);
    }
  }
  const float inv = lsum > 0.0f ? 1.0f / lsum : lsum == 0.0f ? 0.0f : lsum;
  uint16_t *op = a.out + (size_t)pair * HD + lane * PER;
#pragma unroll
  for (int e = 0; e < PER; e += 2) *(uint32_t *)(op + e) = cvt_bf2(acc[e] * inv, acc[e + 1] * inv);
  if (a.lse && lane == 0) a.lse[pair] = 0.6931471805599453f * (mx + __builtin_amdgcn_logf(lsum));
}

// Tiles of TM pairs that consecutive runs of at most `rows` rows in all can have (find_run).
long long tile_bound(long long rows, int G, int TM, int runs) { return rows * G / TM + runs; }

template <int HD, int NW, int NSTAGE, int RB, int MODE>
int launch_items(const PagedArgs &a, int units, int mc, hipStream_t s) {
  const long long grid = (long long)units * a.n_kv * mc;
  if (grid > 0x7fffffffLL) return DCUT_EUNSUPPORTED;
  return launch(MODE == PREFIX ? DCUT_KERNEL_PAGED_PREFIX : DCUT_KERNEL_PAGED_ATTN, k_paged_attn<HD, NW, NSTAGE, RB, MODE>,
                dim3((unsigned)grid), dim3(NW * 64), 0, s, a, units);
}

// How the (row, query head) pairs of a unit are tiled: 64 (a block of 16 a wave) where a unit
// has no more, 128, or the wide kernel's tiles.
struct Tiling {
  int rows;
  bool wide;
};
Tiling tiling(long long pairs) {
  if (pairs <= 64) return {64, false};
  if (pairs <= 128) return {128, false};
  return {paged_tile_rows(), true};
}

template <int HD, int MODE>
int launch_mode(const PagedArgs &a, int units, int mc, int rows, hipStream_t s) {
  if (rows == 64) return launch_items<HD, 4, 3, 1, MODE>(a, units, mc, s);
  return launch_items<HD, 4, 3, 2, MODE>(a, units, mc, s);
}
template <int MODE>
int launch_hd(const PagedArgs &a, int hd, int units, int mc, Tiling t, hipStream_t s) {
  if (t.wide) return paged_tile_launch(a, hd, MODE == PREFIX, units, mc, s);
  return hd == 128 ? launch_mode<128, MODE>(a, units, mc, t.rows, s) : launch_mode<64, MODE>(a, units, mc, t.rows, s);
}
int merge(const PagedArgs &a, int hd, hipStream_t s) {
  if (a.MC == 1) return DCUT_OK;
  const dim3 grid((unsigned)(((long long)a.max_rows * a.n_q + 7) / 8));
  if (hd == 128) return launch(DCUT_KERNEL_PAGED_MERGE, k_paged_merge<128>, grid, dim3(256), 0, s, a);
  return launch(DCUT_KERNEL_PAGED_MERGE, k_paged_merge<64>, grid, dim3(256), 0, s, a);
}

struct AttnPlan {
  Split own, pre;
  Tiling tile, ptile;
  int mc_own, mc_pre, units;
  size_t part, row_nc, total;
};
AttnPlan attn_plan(const dcut_paged_cfg *c, int B, bool shared) {
  AttnPlan p = {};
  const int G = c->n_q / c->n_kv;
  const long long pairs = (long long)G * c->max_block;
  p.tile = tiling(pairs);
  p.units = pairs <= p.tile.rows ? B : (int)tile_bound(c->max_rows, G, p.tile.rows, B);
  p.own = paged_split((long long)p.units * c->n_kv, p.tile.wide ? 512 : 2048, pairs <= p.tile.rows);
  p.mc_own = split_max(p.own, c->max_ctx);
  if (shared) {
    p.ptile = tiling((long long)G * c->max_rows);
    p.pre = paged_split(((long long)c->max_rows * G / p.ptile.rows + 1) * c->n_kv, p.ptile.wide ? 512 : 256, false);
    p.mc_pre = split_max(p.pre, c->max_ctx);
  }
  const int mc = p.mc_own + p.mc_pre;
  size_t off = 0;
  p.part = off;
  if (mc > 1) off = align256(off + (size_t)c->max_rows * c->n_q * mc * ATTN_PITCH(c->head_dim) * sizeof(float));
  p.row_nc = off;
  if (mc > 1) off = align256(off + (size_t)c->max_rows * sizeof(int32_t));
  p.total = off;
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

size_t paged_attn_ws_bytes(const dcut_paged_cfg *c, int B, bool shared) { return attn_plan(c, B, shared).total; }

// Rows over their listed pages (a.list set, a.split, a.MC, a.part and a.row_nc too).
int paged_list_attn_launch(const PagedArgs &a, int hd, hipStream_t s) {
  DCUT_TRY(launch_hd<LIST>(a, hd, a.max_rows, a.MC, Tiling{64, false}, s));
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
  if (p.total && (!ws || ws_bytes < p.total || ((uintptr_t)ws & 255))) return DCUT_EWORKSPACE;
  PagedArgs a = paged_args(cfg, pages, B, q, ldq, cu, ctx_len, out, lse, dev_err);
  a.split = p.own;
  a.MC = p.mc_own;
  if (a.MC > 1) {
    a.part = (float *)((char *)ws + p.part);
    a.row_nc = (int32_t *)((char *)ws + p.row_nc);
  }
  DCUT_TRY(launch_hd<OWN>(a, cfg->head_dim, p.units, p.mc_own, p.tile, stream));
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
  const int punits = (int)tile_bound(cfg->max_rows, a.G, p.ptile.rows, n_groups);
  DCUT_TRY(launch_hd<PREFIX>(a, cfg->head_dim, punits, p.mc_pre, p.ptile, stream));
  DCUT_TRY(launch_hd<OWN>(a, cfg->head_dim, p.units, p.mc_own, p.tile, stream));
  return merge(a, cfg->head_dim, stream);
}
