// Attention of few rows a request (decoding, verified blocks, rows over chosen pages): the
// cache is streamed past up to 64 rows.
//
// Tiles of 32 keys, 16 rows a wave (v_mfma_f32_16x16x32_bf16), four waves:
//   S^T[key][row] = K[key][:] . Q[row][:]   -> lane (row = lane%16) owns keys 4*(lane/16)+j of
//                                              each 16-key block
//   O^T[d][row]  += V^T[d][key] . P^T[key][row], P straight from the S^T accumulators, V
//                   transposed by the LDS reads.
// P is rounded to bf16, the width of the matrix operand; the weights' sum keeps float32 (the
// error this makes: paged_wide.h).
// A ring of three stages keeps two tiles in flight; three workgroups a CU.
//
// What bounds it: the cache stream.  Decoding batch 128 at contexts 512-8191 (1.45 GB) 234 us,
// 6.2 TB/s of the 6.9 that a plain read of one range reaches here; verification of batch 64 at
// contexts 2048-4096 (0.81 GB, up to 32 rows a tile) 136 us, 6.0 TB/s (this kernel alone; the
// calls, with work order and merge, 242 and 146).
#pragma once
#include "paged_item.h"

namespace dcut {

namespace {

constexpr int STREAM_KEYS = 32, STREAM_STAGES = 3, STREAM_WAVES = 4;
constexpr size_t stream_lds(int hd) { return (size_t)STREAM_STAGES * 2 * STREAM_KEYS * hd * 2; }

// Transposing LDS reads of all column tiles x two key halves, the second half HALF bytes after
// the first, issued and awaited in one statement.
template <int HALF>
__device__ __forceinline__ void read_columns(short4v (&r)[16], const uint32_t (&b)[8]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %16\n\t"
      "ds_read_b64_tr_b16 %1, %16 offset:%24\n\t"
      "ds_read_b64_tr_b16 %2, %17\n\t"
      "ds_read_b64_tr_b16 %3, %17 offset:%24\n\t"
      "ds_read_b64_tr_b16 %4, %18\n\t"
      "ds_read_b64_tr_b16 %5, %18 offset:%24\n\t"
      "ds_read_b64_tr_b16 %6, %19\n\t"
      "ds_read_b64_tr_b16 %7, %19 offset:%24\n\t"
      "ds_read_b64_tr_b16 %8, %20\n\t"
      "ds_read_b64_tr_b16 %9, %20 offset:%24\n\t"
      "ds_read_b64_tr_b16 %10, %21\n\t"
      "ds_read_b64_tr_b16 %11, %21 offset:%24\n\t"
      "ds_read_b64_tr_b16 %12, %22\n\t"
      "ds_read_b64_tr_b16 %13, %22 offset:%24\n\t"
      "ds_read_b64_tr_b16 %14, %23\n\t"
      "ds_read_b64_tr_b16 %15, %23 offset:%24\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7]), "=&v"(r[8]), "=&v"(r[9]), "=&v"(r[10]), "=&v"(r[11]), "=&v"(r[12]), "=&v"(r[13]), "=&v"(r[14]), "=&v"(r[15])
      : "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "v"(b[4]), "v"(b[5]), "v"(b[6]), "v"(b[7]), "n"(HALF)
      : "memory");
}
template <int HALF>
__device__ __forceinline__ void read_columns(short4v (&r)[8], const uint32_t (&b)[4]) {
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
      : "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "n"(HALF)
      : "memory");
}

// Rows 16 wave .. + 15 of the tile are the wave's.
template <int HD, int MODE>
__device__ __forceinline__ void stream_body(const PagedArgs &a, const Item &it, unsigned char *ring) {
  constexpr int NW = STREAM_WAVES, NSTAGE = STREAM_STAGES, KT = STREAM_KEYS;
  // a request's keys are read once: non-temporal; chosen pages are shared by a block's rows
  typedef StageLoader<HD, KT, NW, MODE == OWN ? CPOL_NT : 0> Loader;
  constexpr int ROWB = HD * 2, TILEB = KT * ROWB, STAGEB = 2 * TILEB;
  constexpr int NS = HD / 32, NT = HD / 16;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, grp4 = lane >> 4;
  const int R = it.rows - it.r0;

  const int rr = wave * 16 + l16;
  const bool row_ok = rr < R;
  const int pair = row_ok ? it.r0 + rr : it.r0;
  const int krow = pair / a.G;
  const int head = it.g * a.G + pair - krow * a.G;
  const int trow = it.t0 + krow;
  const int kmax = MODE == LIST ? it.diag : it.diag + krow;          // last key the lane's row sees

  bf16x8 qf[NS];
  const uint16_t *qp = a.q + (size_t)trow * a.ldq + (size_t)head * HD + 8 * grp4;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    uint4 z = make_uint4(0, 0, 0, 0);
    qf[s] = row_ok ? *(const bf16x8 *)(qp + 32 * s) : *(bf16x8 *)&z;
  }
  floatx4 o[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) o[n] = {0.f, 0.f, 0.f, 0.f};
  float m_run = -__builtin_inff(), l_run = 0.0f;                     // l: this lane's keys only, joined at the end

  // Fragment addresses within a tile.  K: key l16 (16-key blocks 16 keys apart), chunk
  // grp4 ^ swizzle(key), k-step s flips chunk bits 2-3.  V: source lane s of a 16-lane group
  // reads key k0 + s/4, columns 16n + 4(s%4)..+3, and lane d receives keys k0..k0+3 of column
  // 16n + d; the column tile n flips chunk bits 1-3, the second 16 keys lie 16 keys on.
  const int vrow = 4 * grp4 + (l16 >> 2);
  const uint32_t ring0 = (uint32_t)(uintptr_t)(lds_void *)ring;
  const uint32_t kfrag = ring0 + l16 * ROWB + 16 * (grp4 ^ swizzle<HD>(l16));
  const uint32_t vfrag = ring0 + TILEB + vrow * ROWB + 16 * (((l16 & 3) >> 1) ^ swizzle<HD>(vrow)) + 8 * (l16 & 1);

  const int mixed_from = MODE == OWN ? it.diag + it.r0 / a.G + 1 : it.kend;     // first key hidden from the tile's first row
  const int full_end = min(it.kend, it.diag + 1);                    // keys below it are seen by every row
  int special_from = it.kend;                                        // first tile with an infinite or NaN value among hidden keys

  const int ntiles = (it.kend - it.kstart + KT - 1) / KT;
  Loader ld(a, it, lane, wave);
#pragma unroll
  for (int s = 0; s < NSTAGE; ++s) {
    ld.ask(a, it, s);
    if (s < NSTAGE - 1 && s < ntiles) ld.load(a, it, s, ring + s * STAGEB, ring + s * STAGEB + TILEB);
  }
  constexpr int LPW = 2 * Loader::LPK;
  constexpr int W0 = 0 | (7 << 4) | (15 << 8);
  constexpr int W1 = (LPW & 15) | ((LPW >> 4) << 14) | (7 << 4) | (15 << 8);
  static_assert(NSTAGE == 3, "waits for at most one tile in flight");
  int slot = 0;
  for (int tile = 0; tile < ntiles; ++tile) {
#pragma clang fp contract(off)
    if (tile + 1 < ntiles) __builtin_amdgcn_s_waitcnt(W1);
    else __builtin_amdgcn_s_waitcnt(W0);
    ring_barrier();
    const int next = slot == 0 ? NSTAGE - 1 : slot - 1;
    if (tile + NSTAGE - 1 < ntiles) ld.load(a, it, tile + NSTAGE - 1, ring + next * STAGEB, ring + next * STAGEB + TILEB);
    ld.ask(a, it, tile + NSTAGE);
    const int p0 = it.kstart + tile * KT;
    const uint32_t at = slot * STAGEB;
    if (++slot == NSTAGE) slot = 0;
    if (uniform_if(p0 + KT > mixed_from))                            // over the workgroup
      if (clear_specials<TILEB, NW * 64>(ring + at + TILEB)) special_from = min(special_from, p0);
    if (uniform_if(wave * 16 >= R)) continue;                        // no rows
    floatx4 s4[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      s4[kb] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const bf16x8 kf = *(lds_frag *)(uintptr_t)(((kfrag + at) ^ (64 * s)) + kb * 16 * ROWB);
        s4[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[s], s4[kb], 0, 0, 0);
      }
    }
    if (uniform_if(p0 < it.klo || p0 + KT > full_end)) {
      const uint32_t n = (uint32_t)max(min(it.kend, kmax + 1) - it.klo, 0);      // keys from klo on that the row sees
      const int first = p0 + 4 * grp4 - it.klo;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int j = 0; j < 4; ++j) s4[kb][j] = (uint32_t)(first + 16 * kb + j) < n ? s4[kb][j] : -__builtin_inff();
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) s4[kb] *= SCORE_SCALE<HD>;
    float tmax = fmaxf(fmaxf(s4[0][0], s4[0][1]), fmaxf(s4[0][2], s4[0][3]));
    tmax = fmaxf(tmax, fmaxf(fmaxf(s4[1][0], s4[1][1]), fmaxf(s4[1][2], s4[1][3])));
    tmax = half_max(row_max(tmax));
    const float m_new = tmax > m_run + RAISE ? tmax : m_run;
    // a row that has seen no key yet keeps m = -inf; subtracting 0 then keeps its weights at 0
    const float sub = m_new == -__builtin_inff() ? 0.0f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m_run - sub);
    const bool raise = m_new != m_run;
    m_run = m_new;
    float psum = 0.0f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float pv = __builtin_amdgcn_exp2f(s4[kb][j] - sub);
        s4[kb][j] = pv;
        psum += pv;
      }
    l_run = __builtin_fmaf(l_run, alpha, psum);
    if (__any(raise)) {
#pragma unroll
      for (int n = 0; n < NT; ++n) o[n] *= alpha;
    }
    // O^T += V^T P^T.  P^T slots of this lane: keys 4*grp4+j of the two 16-key blocks; the V^T
    // fragment with the same keys comes from two transposing reads.
    bf16x8 pf;
    uint32_t *pw = (uint32_t *)&pf;
    pw[0] = cvt_bf2(s4[0][0], s4[0][1]);
    pw[1] = cvt_bf2(s4[0][2], s4[0][3]);
    pw[2] = cvt_bf2(s4[1][0], s4[1][1]);
    pw[3] = cvt_bf2(s4[1][2], s4[1][3]);
    uint32_t vb[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) vb[n] = (vfrag + at) ^ (32 * n);
    short4v vr[2 * NT];
    read_columns<16 * ROWB>(vr, vb);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      bf16x8 vf;
      short4v *vw = (short4v *)&vf;
      vw[0] = vr[2 * n];
      vw[1] = vr[2 * n + 1];
      o[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf, o[n], 0, 0, 0);
    }
  }
  if (special_from < it.kend) {
    for (int p = max(special_from, it.klo); p < it.kend; ++p) {
      const int pg = uniform_load(it.tab, p >> a.lpage);
      if ((unsigned)pg >= (unsigned)a.n_pages) continue;
      const uint16_t *v = a.v + (((size_t)pg * a.n_kv + it.g) * a.page + (p & (a.page - 1))) * HD + 4 * grp4;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[n][j] += special_value(v[16 * n + j], p <= kmax);
    }
  }
  ld.report(a, lane);
  const float l = half_sum(row_sum(l_run));
  if (!row_ok) return;
  const size_t at = (size_t)trow * a.n_q + head;
  if (it.first && grp4 == 0 && a.row_nc) a.row_nc[trow] = it.nc;
  // lane holds O^T[16n + 4*grp4 + j][row]
  if (it.nc == 1) {
    const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
    uint16_t *op = a.out + at * HD;
#pragma unroll
    for (int n = 0; n < NT; ++n)
      *(uint2 *)(op + 16 * n + 4 * grp4) = make_uint2(cvt_bf2(o[n][0] * inv, o[n][1] * inv), cvt_bf2(o[n][2] * inv, o[n][3] * inv));
    if (a.lse && grp4 == 0) a.lse[at] = 0.6931471805599453f * (m_run + __builtin_amdgcn_logf(l));
  } else {
    float *pp = a.part + (at * a.MC + it.slot) * ATTN_PITCH(HD);
#pragma unroll
    for (int n = 0; n < NT; ++n) *(float4 *)(pp + 16 * n + 4 * grp4) = make_float4(o[n][0], o[n][1], o[n][2], o[n][3]);
    if (grp4 == 0) {
      pp[HD] = m_run;
      pp[HD + 1] = l;
    }
  }
}

}  // namespace

}  // namespace dcut
