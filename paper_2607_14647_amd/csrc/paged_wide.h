// Attention of many rows at once (prompts, the prefix of a group): 32 x 32 tiles.
//
// 32 keys x 32 rows a wave (v_mfma_f32_32x32x16_bf16), which halves the LDS reads a product
// takes against 16 x 16:
//   S^T[key][row] = K[key][:] . Q[row][:]   -> lane (row = lane%32, h = lane/32) owns keys
//                                              8 i + 4 h + j (i, j < 4) of a 32-key block
//   O^T[d][row]  += V^T[d][key] . P^T[key][row], P straight from the S^T accumulators, V with
//                   the same order of keys from transposing LDS reads.
// Steps of 64 keys.  A step's products run with the next step's scores, so that matrix work
// and exponentials of one wave overlap; two stages of K and of V tiles, the V tile one step
// behind.  128 rows a workgroup of four waves, two workgroups a CU.
//
// Weights meet the values in bf16, the width of the matrix operand, as in the slab's attention;
// their sum keeps float32.  Each weight is off by at most 2^-8 of itself: outputs differ from the
// 64-bit definition by 0.0023 (norm of the difference over the norm), by 0.0017 with float32
// weights, where only the outputs' own rounding to bf16 is left.
//
// What bounds it: the serial chain of a step (fragments, scores, maximum, exponentials,
// rounding, products), two waves a SIMD filling each other's gaps: the matrix units are busy
// 39% of the time, the LDS 20%.  Prompt of 4 x 2000 rows on contexts up to 2000 (262 GFLOP): the
// clock gives way under the matrix work, so the kernel alone takes 281 us at least and 346 in the
// mean of 54 runs in a row, 930 and 760 TFLOP/s; the whole call 280 to 330.
// Tried: three waves a SIMD with 32-key steps (equal), 256 rows in 8 waves (equal), half of the waves
// a phase behind (3% slower), partials written in whole rows through the LDS (equal), scores and
// products of one step in turn (equal here, 93 us for 84 where batch 64 reads 350 MB in blocks of
// up to 16).  Two 32-row blocks a wave, one wave a SIMD, were tried only before the products ran
// with the next scores (525 us for 387).
#pragma once
#include <type_traits>

#include "paged_item.h"

namespace dcut {

namespace {

constexpr int WIDE_KEYS = 64;         // keys per LDS stage
constexpr int WIDE_WAVES = 4, WIDE_ROWS = 32 * WIDE_WAVES;
constexpr size_t wide_lds(int hd) { return (size_t)2 * 2 * WIDE_KEYS * hd * 2; }

// Transposing LDS reads of the V^T fragments of 32 keys, OFF bytes into the stage's tile, issued
// and awaited in one statement: fragment (16-key step u, column tile n) from its 8-key halves
// e = 0, 1, at r[(u NT + n) 2 + e], read at b[n + NT e].
template <int OFF>
__device__ __forceinline__ void read_values(short4v (&r)[16], const uint32_t (&b)[8]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %16 offset:%24\n\t"
      "ds_read_b64_tr_b16 %1, %20 offset:%25\n\t"
      "ds_read_b64_tr_b16 %2, %17 offset:%24\n\t"
      "ds_read_b64_tr_b16 %3, %21 offset:%25\n\t"
      "ds_read_b64_tr_b16 %4, %18 offset:%24\n\t"
      "ds_read_b64_tr_b16 %5, %22 offset:%25\n\t"
      "ds_read_b64_tr_b16 %6, %19 offset:%24\n\t"
      "ds_read_b64_tr_b16 %7, %23 offset:%25\n\t"
      "ds_read_b64_tr_b16 %8, %16 offset:%26\n\t"
      "ds_read_b64_tr_b16 %9, %20 offset:%27\n\t"
      "ds_read_b64_tr_b16 %10, %17 offset:%26\n\t"
      "ds_read_b64_tr_b16 %11, %21 offset:%27\n\t"
      "ds_read_b64_tr_b16 %12, %18 offset:%26\n\t"
      "ds_read_b64_tr_b16 %13, %22 offset:%27\n\t"
      "ds_read_b64_tr_b16 %14, %19 offset:%26\n\t"
      "ds_read_b64_tr_b16 %15, %23 offset:%27\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7]), "=&v"(r[8]), "=&v"(r[9]), "=&v"(r[10]), "=&v"(r[11]), "=&v"(r[12]), "=&v"(r[13]), "=&v"(r[14]), "=&v"(r[15])
      : "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "v"(b[4]), "v"(b[5]), "v"(b[6]), "v"(b[7]), "n"(OFF), "n"(OFF + 2048), "n"(OFF + 2 * 2048), "n"(OFF + 3 * 2048)
      : "memory");
}
template <int OFF>
__device__ __forceinline__ void read_values(short4v (&r)[8], const uint32_t (&b)[4]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8 offset:%12\n\t"
      "ds_read_b64_tr_b16 %1, %10 offset:%13\n\t"
      "ds_read_b64_tr_b16 %2, %9 offset:%12\n\t"
      "ds_read_b64_tr_b16 %3, %11 offset:%13\n\t"
      "ds_read_b64_tr_b16 %4, %8 offset:%14\n\t"
      "ds_read_b64_tr_b16 %5, %10 offset:%15\n\t"
      "ds_read_b64_tr_b16 %6, %9 offset:%14\n\t"
      "ds_read_b64_tr_b16 %7, %11 offset:%15\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
      : "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "n"(OFF), "n"(OFF + 1024), "n"(OFF + 2 * 1024), "n"(OFF + 3 * 1024)
      : "memory");
}

// Rows 32 wave .. + 31 of the tile are the wave's.
template <int HD, int MODE>
__device__ __forceinline__ void wide_body(const PagedArgs &a, const Item &it, unsigned char *ring) {
#pragma clang fp contract(off)
  constexpr int NW = WIDE_WAVES;
  typedef StageLoader<HD, WIDE_KEYS, NW, 0> Loader;
  constexpr int KS = WIDE_KEYS, KB = KS / 32;
  constexpr int ROWB = HD * 2, TILEB = KS * ROWB;
  constexpr int NS = HD / 16;               // k-steps of the score product
  constexpr int NT = HD / 32;               // 32-row tiles of O^T
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5, l16 = lane & 15, g1 = (lane >> 4) & 1;
  const int R = it.rows - it.r0;

  const int b0 = wave * 32, rr = b0 + l32;
  const bool row_ok = rr < R;
  const int pair = row_ok ? it.r0 + rr : it.r0;
  const int krow = pair / a.G;
  const int head = it.g * a.G + pair - krow * a.G;
  const int trow = it.t0 + krow;
  const int kmax = MODE == OWN ? it.diag + krow : it.diag;          // last key the lane's row sees
  // keys up to seen_last are seen by some row of the wave, those below full_end by all
  const int seen_last = b0 >= R ? -1 : MODE == OWN ? it.diag + (it.r0 + min(b0 + 31, R - 1)) / a.G : it.diag;
  const int full_end = min(it.kend, __builtin_amdgcn_readfirstlane(kmax) + 1);

  bf16x8 qf[NS];
  const uint16_t *qp = a.q + (size_t)trow * a.ldq + (size_t)head * HD + 8 * h;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    uint4 z = make_uint4(0, 0, 0, 0);
    qf[s] = row_ok ? *(const bf16x8 *)(qp + 16 * s) : *(bf16x8 *)&z;
  }
  floatx16 o[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[n][r] = 0.0f;
  float m_run = -__builtin_inff(), l_run = 0.0f;                    // l: this lane's keys only, joined at the end

  // Fragment addresses within a stage.  K: key l32, chunk (2 s + h) ^ swizzle(key).  V: keys
  // 16 u + 8 e + 4 h + (l16 >> 2), columns 32 n + 16 g1 + 4 (l16 & 3)..+3; the column tile n
  // flips chunk bits 2-3, e chunk bits 0-1.
  const uint32_t ring0 = (uint32_t)(uintptr_t)(lds_void *)ring;
  const uint32_t kfrag = ring0 + l32 * ROWB + 16 * (h ^ swizzle<HD>(l32));
  const int vkey = 4 * h + (l16 >> 2);
  const uint32_t vfrag = ring0 + 2 * TILEB + vkey * ROWB + 16 * ((2 * g1 + ((l16 & 3) >> 1)) ^ swizzle<HD>(vkey)) + 8 * (l16 & 1);

  bf16x8 pf[2 * KB];                        // P^T of the step scored last
  auto k_at = [&](int st) { return kfrag + (st & 1) * TILEB; };
  auto v_at = [&](int st) { return vfrag + (st & 1) * TILEB; };

  // Half a step's products, with the weights kept of 32 keys: O^T += V^T P^T.
  auto products = [&](auto off, const uint32_t vs, const bf16x8 &p0, const bf16x8 &p1) __attribute__((always_inline)) {
    uint32_t vb[2 * NT];
#pragma unroll
    for (int n = 0; n < 2 * NT; ++n) vb[n] = vs ^ (64 * (n % NT)) ^ (n >= NT ? 48 : 0);
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
        o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, u ? p1 : p0, o[n], 0, 0, 0);
      }
  };
  typedef std::integral_constant<int, 0> FirstHalf;
  typedef std::integral_constant<int, 32 * ROWB> SecondHalf;

  Loader ld(a, it, lane, wave);

  // Scores of step st and their weights; with BEHIND, the products of the step before, whose
  // weights were kept: matrix work beside the exponentials.
  auto step = [&](auto behind, const int st) __attribute__((always_inline)) {
    constexpr bool BEHIND = decltype(behind)::value;
    const int p0 = it.kstart + st * KS;
    const uint32_t ks = k_at(st), vs = v_at(st - 1);
    floatx16 s[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] = 0.0f;
#pragma unroll
    for (int f = 0; f < NS; ++f)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const bf16x8 kf = *(lds_frag *)(uintptr_t)((ks ^ (32 * f)) + kb * 32 * ROWB);
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[f], s[kb], 0, 0, 0);
      }
    // K fragments are asked for four products ahead
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int i = 0; i < NS * KB - 4; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    if (uniform_if(p0 < it.klo || p0 + KS > full_end)) {    // some key of the step is hidden from some row of the wave
      const uint32_t n = (uint32_t)max(min(it.kend, kmax + 1) - it.klo, 0);      // keys from klo on that the row sees
      const int first = p0 + 4 * h - it.klo;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          s[kb][r] = (uint32_t)(first + 32 * kb + 8 * (r >> 2) + (r & 3)) < n ? s[kb][r] : -__builtin_inff();
    }
    float tm[4] = {s[0][0], s[0][1], s[0][2], s[0][3]};
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) tm[r & 3] = fmaxf(tm[r & 3], s[kb][r]);
    const float smax = half_max(fmaxf(fmaxf(tm[0], tm[1]), fmaxf(tm[2], tm[3])));
    const float tmax = smax * SCORE_SCALE<HD>;
    // Scaling goes into the subtraction's multiply-add (a prompt takes 2% longer otherwise)
    // except for a row whose score passes 2^31 (SCORE_SCALE); up to there it adds at most 2^4 to
    // RAISE.  Each row decides from its own scores: the others multiply by 1.
    const bool big = fabsf(smax) > 0x1p31f && smax != -__builtin_inff();
    float scale = SCORE_SCALE<HD>;
    if (__any(big)) {
      const float first = big ? SCORE_SCALE<HD> : 1.0f;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[kb] *= first;
      scale = big ? 1.0f : SCORE_SCALE<HD>;
    }
    const float m_new = tmax > m_run + RAISE ? tmax : m_run;
    // a row that has seen no key yet keeps m = -inf; subtracting 0 then keeps its weights at 0
    const float sub = m_new == -__builtin_inff() ? 0.0f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m_run - sub);
    const bool raise = m_new != m_run;
    m_run = m_new;
    float psum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    bf16x8 pn[2 * KB];
    auto weights = [&](int kb) __attribute__((always_inline)) {
      uint32_t *pw = (uint32_t *)&pn[2 * kb];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float pv = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][r], scale, -sub));
        s[kb][r] = pv;
        psum[r & 3] += pv;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) pw[e] = cvt_bf2(s[kb][2 * e], s[kb][2 * e + 1]);
    };
    if (BEHIND) products(FirstHalf{}, vs, pf[0], pf[1]);
    weights(0);
    if (BEHIND) products(SecondHalf{}, vs, pf[2], pf[3]);
    if (BEHIND) ld.ask(a, it, st + 2);      // here no LDS read waits for it
    weights(1);
#pragma unroll
    for (int u = 0; u < 2 * KB; ++u) pf[u] = pn[u];
    l_run = __builtin_fmaf(l_run, alpha, (psum[0] + psum[1]) + (psum[2] + psum[3]));
    if (__any(raise)) {
#pragma unroll
      for (int n = 0; n < NT; ++n) o[n] *= alpha;
    }
    static_assert(KB == 2, "two blocks of 32 keys");
  };
  const int mixed_from = MODE == OWN ? it.diag + it.r0 / a.G + 1 : it.kend;     // first key hidden from the tile's first row
  int special_from = it.kend;                                       // first stage with an infinite or NaN value there

  const int nst = (it.kend - it.kstart + KS - 1) / KS;
  // K tiles 0 and 1 and V tile 0 are asked for at once; then interval st finds K tile st and V
  // tile st-1 there and asks for V tile st and K tile st+1.
  ld.ask(a, it, 0);
  ld.load_k(a, it, 0, ring);
  ld.load_v(ring + 2 * TILEB);
  ld.ask(a, it, 1);
  if (nst > 1) ld.load_k(a, it, 1, ring + TILEB);
  ld.ask(a, it, 2);
  constexpr int LPK = Loader::LPK;
  static_assert(2 * LPK < 16, "low bits of the wait count");
  constexpr int WAIT_ALL = 0 | (7 << 4) | (15 << 8), WAIT_K0 = (2 * LPK) | (7 << 4) | (15 << 8), WAIT_K0_ONLY = LPK | (7 << 4) | (15 << 8);
  auto interval = [&](int st) __attribute__((always_inline)) {
    if (st == 0 && nst > 1) __builtin_amdgcn_s_waitcnt(WAIT_K0);
    else if (st == 0) __builtin_amdgcn_s_waitcnt(WAIT_K0_ONLY);
    else __builtin_amdgcn_s_waitcnt(WAIT_ALL);
    ring_barrier();
    if (st > 0) {
      if (st < nst) ld.load_v(ring + (2 + (st & 1)) * TILEB);
      if (st + 1 < nst) ld.load_k(a, it, st + 1, ring + ((st + 1) & 1) * TILEB);
    }
    const int p0 = it.kstart + (st - 1) * KS;
    if (uniform_if(st > 0 && p0 + KS > mixed_from))                  // over the workgroup
      if (clear_specials<TILEB, NW * 64>(ring + (2 + ((st - 1) & 1)) * TILEB)) special_from = min(special_from, p0);
  };
  // Steps this wave's rows see something of: the first ones.  Every wave passes the same intervals.
  const int mine = uniform_int(seen_last < it.kstart ? 0 : min(nst, (seen_last - it.kstart) / KS + 1));
  int st = 0;
  if (mine > 0) {
    interval(0);
    step(std::false_type{}, 0);
    for (st = 1; st < mine; ++st) {
      interval(st);
      step(std::true_type{}, st);
    }
    interval(st);
    products(FirstHalf{}, v_at(st - 1), pf[0], pf[1]);
    products(SecondHalf{}, v_at(st - 1), pf[2], pf[3]);
    ld.ask(a, it, st + 2);
    ++st;
  }
  for (; st <= nst; ++st) {
    interval(st);
    if (st > 0) ld.ask(a, it, st + 2);
  }
  if (special_from < it.kend) {
    for (int p = max(special_from, it.klo); p < it.kend; ++p) {
      const int pg = uniform_load(it.tab, p >> a.lpage);
      if ((unsigned)pg >= (unsigned)a.n_pages) continue;
      const uint16_t *v = a.v + (((size_t)pg * a.n_kv + it.g) * a.page + (p & (a.page - 1))) * HD + 4 * h;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          o[n][r] += special_value(v[32 * n + 8 * (r >> 2) + (r & 3)], p <= kmax);
          if ((r & 3) == 3) __builtin_amdgcn_sched_barrier(0);      // rare: keep its loads from taking the loop's registers
        }
    }
  }
  ld.report(a, lane);
  const float l = half_sum(l_run);
  if (!row_ok) return;
  const size_t at = (size_t)trow * a.n_q + head;
  if (it.first && h == 0 && a.row_nc) a.row_nc[trow] = it.nc;
  // lane holds O^T[32n + 8 i + 4 h + j][row]
  if (it.nc == 1) {
    const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
    uint16_t *op = a.out + at * HD + 4 * h;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(uint2 *)(op + 32 * n + 8 * i) = make_uint2(cvt_bf2(o[n][4 * i] * inv, o[n][4 * i + 1] * inv),
                                                     cvt_bf2(o[n][4 * i + 2] * inv, o[n][4 * i + 3] * inv));
    if (a.lse && h == 0) a.lse[at] = 0.6931471805599453f * (m_run + __builtin_amdgcn_logf(l));
  } else {
    float *pp = a.part + (at * a.MC + it.slot) * ATTN_PITCH(HD);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(float4 *)(pp + 32 * n + 8 * i + 4 * h) = make_float4(o[n][4 * i], o[n][4 * i + 1], o[n][4 * i + 2], o[n][4 * i + 3]);
    if (h == 0) {
      pp[HD] = m_run;
      pp[HD + 1] = l;
    }
  }
}

}  // namespace

}  // namespace dcut
