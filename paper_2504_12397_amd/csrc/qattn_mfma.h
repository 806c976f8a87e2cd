// Attention over rows of 4 bits on the matrix units (Eq.1 with the causal mask, Eq.4): for head sizes that are multiples of 8.
//
// A wave takes 16 * NC columns -- (row, query head) pairs that read one kv head -- and walks a range of keys, 32 a step:
//   * Codes of K go, as they are, into the A operand of v_mfma_f32_16x16x32_bf16: lane (j, kg) has the HT / 4 channels from kg * HT / 4 on of
//     key j of 16, a dword (8 channels) per product; the queries, laid out alike, are the B operand: S[key][column].  v_cvt_scalef32_pk_bf16_fp4
//     turns two codes into two numbers, scale included, in one instruction: bf16 holds every code times every power of two exactly, where
//     fp16 would overflow or lose bits for exponents far from 127.
//   * Accumulator register v of lane (j, kg) is key 4 kg + v of column j: a lane owns one column, the softmax needs no other lane but
//     for a new maximum, and the probabilities of two blocks of 16 keys are, as they sit, the B operand (32 keys) of O += V P.
//   * V: lane (j, kg) has CPL = HT / 16 channels from CPL j on of those 8 keys; after conversion a byte permute of two keys' words puts
//     one channel of two keys side by side, which is the transposition: product c is channel CPL i + c of lane row i.
// Two kernels differ in how codes reach the lanes' registers: through LDS (heads of 64 and 128: qattn_lds_kernel), or from memory (qattn_mfma_kernel: any head size and alignment).  Where
// several waves share a head's keys (KR > 1), they join through LDS at the end, in pairs.
// Queries of bf16 are one operand, exactly; fp16 two (high and low bits as bf16; one beside keys of fp16, below), fp32 three.  Probabilities are two operands (16 bits; one of 8
// bits would add half of what the rounding of a bf16 result does), three for fp32.  Units of many columns, where the products count and not memory, take one operand
// of fp16 (11 bits) with values of fp16, as long as that holds them exactly: a workgroup looks at the smallest exponent that it met and at whether its sums
// are numbers (queries of fp16 take keys of fp16 likewise: both ends of their exponents count), and says so where fp16 was too narrow; a second launch does those items, and no others, with operands of bf16.  128 rows of 32 heads on 32896 keys
// 139 -> 117 us, the second launch (4 us) included.
// The reference exponent of a column moves only when a score exceeds it by 2^8 more than it did: almost no step rescales the sums.  It begins 8 above the largest score
// so far, so that probabilities are 1 at most and 2^-8 at a new maximum (sums of values near fp32's largest have that much room: about 300 keys of equal weight); in fp16 7 below it, for the sake
// of that type's small numbers: 2^15 at most.
#pragma once
#include "lds_dma.h"
#include "qcache.h"

namespace alora {

typedef __bf16 qa_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 qa_bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t qa_u32x4 __attribute__((ext_vector_type(4)));
typedef float qa_f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 qa_f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 qa_f16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t QA_F16_FIRST = 114, QA_F16_LAST = 140;      // the exponent bytes whose smallest value, 0.5 * 2^(E - 127), and largest, 6 * 2^(E - 127), are normal numbers of fp16

// byte b of w: two codes, as a pair of bf16
__device__ __forceinline__ uint32_t qa_pair(uint32_t w, float scale, int b) {
  qa_bf16x2 r;
  switch (b) {
    case 0: r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0); break;
    case 1: r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1); break;
    case 2: r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2); break;
    default: r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  }
  return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ uint32_t qa_pair16(uint32_t w, float scale, int b) {      // as a pair of fp16
  qa_f16x2 r;
  switch (b) {
    case 0: r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0); break;
    case 1: r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1); break;
    case 2: r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2); break;
    default: r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3);
  }
  return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ uint32_t qa_pack(float a, float b) {
  qa_bf16x2 r;
  r.x = (__bf16)a;
  r.y = (__bf16)b;
  return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ float qa_lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float qa_hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
__device__ __forceinline__ float qa_scale(uint32_t e) { return __builtin_bit_cast(float, e << 23); }

// two numbers as N pairs of bf16 whose sums they are, to 8 N bits
template <int N> __device__ __forceinline__ void qa_split(float a, float b, uint32_t *to, int stride) {
#pragma unroll
  for (int p = 0; p < N; ++p) {
    const uint32_t w = qa_pack(a, b);
    to[p * stride] = w;
    if (p + 1 < N) { a -= qa_lo(w); b -= qa_hi(w); }
  }
}

// over the four lanes (j, 0..3)
__device__ __forceinline__ float qa_max4(float x) {
  x = fmaxf(x, __shfl_xor(x, 16, 64));
  return fmaxf(x, __shfl_xor(x, 32, 64));
}
__device__ __forceinline__ float qa_sum4(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}

// What a wave is to do, from its item and its place in the workgroup.
struct QaWork {
  int g, sub, cg, kr;            // kv head; share of the keys, group of columns
  bool active, shared;
  int col0, n_cols;              // its columns
  int kbeg, kend, see_all;       // its keys; keys below see_all are seen by every column
  int steps;                     // of 32 keys that a wave of the workgroup takes at most
  int64_t key_row0;
  int first_row, pos0, part;
};
template <int NC> __device__ __forceinline__ QaWork qa_work(const QAttnArgs &a, const QAttnItem &it, int wave) {
  QaWork w;
  const int G = a.n_q_heads / a.n_kv_heads, hw = wave % a.hw, rest = wave / a.hw;
  w.sub = rest % a.kr; w.cg = rest / a.kr; w.kr = a.kr;
  const int c_first = w.cg * 16 * NC;
  w.n_cols = min(it.n_cols - c_first, 16 * NC);
  w.active = it.g0 + hw < a.n_kv_heads && w.n_cols > 0;
  w.g = min(it.g0 + hw, a.n_kv_heads - 1);
  w.col0 = it.col0 + c_first;
  w.shared = it.shared;
  w.key_row0 = it.key_row0; w.first_row = it.first_row; w.pos0 = it.pos0; w.part = it.part;
  const int last_tok = (w.col0 + max(w.n_cols, 1) - 1) / G, first_tok = w.col0 / G;
  int per = (it.kend - it.kbeg + a.kr - 1) / a.kr;
  per = (per + 31) & ~31;
  w.steps = per >> 5;
  w.kbeg = it.kbeg + w.sub * per;
  w.kend = min(it.kend, w.kbeg + per);
  if (!it.shared) w.kend = min(w.kend, it.pos0 + last_tok + 1);
  if (!w.active) w.kend = w.kbeg;
  w.see_all = it.shared ? w.kend : min(w.kend, it.pos0 + first_tok + 1);
  return w;
}

// Codes and exponents of 32 keys, as the lanes hold them
template <int HT> struct QaTile {
  static constexpr int KS = HT / 32;                  // products per block of 16 keys, dwords of K per lane
  static constexpr int CPL = HT / 16;                 // channels of V per lane ...
  static constexpr int VB = CPL / 2;                  // ... and their bytes
  static constexpr int VW = (VB + 3) / 4;
  static constexpr int KSC = HT == 256 ? 2 : 1;       // exponents of K per lane
  uint32_t k[2][KS];
  uint32_t ks[2][KSC];
  uint32_t v[2][4][VW];                               // [u][n]: key 16 u + 4 kg + n
  uint32_t vs[2][4];
};

// The columns of a wave: queries, running sums, and what is done with 32 keys.
// HALF: probabilities and values as fp16; K16: keys too, beside queries of fp16 (one operand instead of two).
template <int HT, int NQ, int NP, int NC, bool HALF, typename TQ, typename T> struct QaColumns {
  typedef QaTile<HT> Tile;
  static constexpr float ABOVE = HALF ? -7.f : 8.f, LAZY = HALF ? 15.f : 0.f;      // log2 units: where a new reference lies, how far a score may exceed it
  static constexpr int KS = Tile::KS, CPL = Tile::CPL, VW = Tile::VW, KSC = Tile::KSC;
  static constexpr bool K16 = HALF && NQ == 1 && __is_same(TQ, _Float16);
  uint32_t qf[NC][NQ][KS][4];
  int lim[NC];                            // last key that the column sees
  qa_f32x4 o[NC][CPL];                    // o[c][v] of lane (j, kg): channel CPL * (4 kg + v) + c of column j
  float m_ref[NC], neg_m[NC], l[NC];      // reference exponent (log2), its negative or 0 where there is none, this lane's part of the sum
  uint32_t nan_blocks[NC];                // blocks of 32 channels in which the column has met a value that is not a number
  uint32_t e_min;                         // HALF: the smallest exponent of a value so far
  uint32_t k_far;                         // K16: how far above QA_F16_FIRST a key's exponent was (below: wrapped)
  int j, kg;
  float c_scale;

  __device__ __forceinline__ int row_of(const QAttnArgs &a, const QaWork &w, int tok) const { return w.shared ? a.rows[w.first_row + tok] : w.first_row + tok; }

  __device__ __forceinline__ void begin(const QAttnArgs &a, const QaWork &w, int lane) {
    j = lane & 15; kg = lane >> 4;
    c_scale = a.sm_scale * 1.4426950408889634f;
    const int G = a.n_q_heads / a.n_kv_heads, h = a.head_dim;
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
      const int c = 16 * nc + j, tok = (w.col0 + c) / G, hj = w.col0 + c - tok * G;
      const bool there = w.active && c < w.n_cols;
      lim[nc] = w.shared || !there ? 0x7fffffff : w.pos0 + tok;
      const int row = there ? row_of(a, w, tok) : 0;
      const TQ *q = (const TQ *)a.Q + ((int64_t)row * a.n_q_heads + w.g * G + (there ? hj : 0)) * h;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int ch = kg * (HT / 4) + 8 * s;
        const bool in = there && ch < h;
        if constexpr (sizeof(TQ) == 2 && NQ == 1) {
          const qa_u32x4 x = in ? *reinterpret_cast<const qa_u32x4 *>(q + ch) : qa_u32x4{0, 0, 0, 0};
#pragma unroll
          for (int i = 0; i < 4; ++i) qf[nc][0][s][i] = x[i];
        } else {
          float x[8];
          if constexpr (sizeof(TQ) == 2) {
            typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
            f16x8_t y = {};
            if (in) y = *reinterpret_cast<const f16x8_t *>(q + ch);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (float)y[i];
          } else {
            qa_f32x4 y0 = {}, y1 = {};
            if (in) { y0 = *reinterpret_cast<const qa_f32x4 *>(q + ch); y1 = *reinterpret_cast<const qa_f32x4 *>(q + ch + 4); }
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = y0[i]; x[4 + i] = y1[i]; }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) qa_split<NQ>(x[2 * i], x[2 * i + 1], &qf[nc][0][s][i], KS * 4);
        }
      }
#pragma unroll
      for (int c2 = 0; c2 < CPL; ++c2) o[nc][c2] = qa_f32x4{0.f, 0.f, 0.f, 0.f};
      m_ref[nc] = -INFINITY;
      neg_m[nc] = l[nc] = 0.f;
      nan_blocks[nc] = 0;
    }
    e_min = 255;
    k_far = 0;
  }

  // Some value was too small for fp16, or too large (the sums are infinite or no numbers; or they would be so anyway).
  __device__ __forceinline__ bool too_narrow() const {
    float z = 0.f;
#pragma unroll
    for (int nc = 0; nc < NC; ++nc)
#pragma unroll
      for (int c = 0; c < CPL; ++c)
#pragma unroll
        for (int v = 0; v < 4; ++v) z += o[nc][c][v] - o[nc][c][v];
    return e_min < QA_F16_FIRST || k_far > QA_F16_LAST - QA_F16_FIRST || !(z == 0.f);
  }

  // 32 keys from k0 on.  k_used() is called once t.k has been read, need_v() before t.v is, v_used() after.
  template <typename KU, typename NV, typename VU>
  __device__ __forceinline__ void step(const QAttnArgs &a, const QaWork &w, Tile &t, int k0, KU k_used, NV need_v, VU v_used) {
    qa_f32x4 sc[NC][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int nc = 0; nc < NC; ++nc) sc[nc][u] = qa_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const float e = qa_scale(t.ks[u][KSC == 2 ? s / 4 : 0]);
        const uint32_t c = t.k[u][s];
        const qa_u32x4 kf = K16 ? qa_u32x4{qa_pair16(c, e, 0), qa_pair16(c, e, 1), qa_pair16(c, e, 2), qa_pair16(c, e, 3)}
                                : qa_u32x4{qa_pair(c, e, 0), qa_pair(c, e, 1), qa_pair(c, e, 2), qa_pair(c, e, 3)};
#pragma unroll
        for (int nc = 0; nc < NC; ++nc)
#pragma unroll
          for (int p = 0; p < NQ; ++p) {
            const qa_u32x4 qv = {qf[nc][p][s][0], qf[nc][p][s][1], qf[nc][p][s][2], qf[nc][p][s][3]};
            if constexpr (K16) sc[nc][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(qa_f16x8, kf), __builtin_bit_cast(qa_f16x8, qv), sc[nc][u], 0, 0, 0);
            else sc[nc][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(qa_bf16x8, kf), __builtin_bit_cast(qa_bf16x8, qv), sc[nc][u], 0, 0, 0);
          }
      }
    }
    k_used();
    need_v();
    if (k0 + 32 > w.see_all) {      // a step that some column sees in part
      int first = k0 + 4 * kg;
      asm volatile("" : "+v"(first));      // (the comparisons stay here: made ahead of the branch they cost every step 17 instructions and as many pairs of registers)
      bool bad = false;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (K16 && first - 4 * kg + 16 * u + j >= w.kend) t.ks[u][0] = 127;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int key = first + 16 * u + v;
          bad |= t.vs[u][v] == (uint32_t)Q_E_NAN;
          if (HALF && key >= w.kend) t.vs[u][v] = 127;      // (rows that are not there read as zeros, whose exponent is no concern)
#pragma unroll
          for (int nc = 0; nc < NC; ++nc)
            if (key >= w.kend || key > lim[nc]) sc[nc][u][v] = -INFINITY;
        }
      }
      if (__any(bad)) {
        // 0 times NaN would reach the columns that do not see the key: its values count as 0, and the columns that do see it remember the block
        const int nb = q_blocks(a.head_dim);
        const uint8_t *scales = a.c.v_scale + (w.key_row0 * a.n_kv_heads + w.g) * nb;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const int key = first + 16 * u + v;
            const uint8_t *sp = scales + (int64_t)min(key, w.kend - 1) * a.n_kv_heads * nb;
            uint32_t blocks = 0;
            for (int b = 0; b < nb; ++b) blocks |= (sp[b] == Q_E_NAN ? 1u : 0u) << b;
#pragma unroll
            for (int nc = 0; nc < NC; ++nc)
              if (key < w.kend && key <= lim[nc]) nan_blocks[nc] |= blocks;
            if (t.vs[u][v] == (uint32_t)Q_E_NAN) {
              t.vs[u][v] = 127;
#pragma unroll
              for (int i = 0; i < VW; ++i) t.v[u][v][i] = 0;
            }
          }
      }
    }
    if constexpr (K16) k_far = max(k_far, max(t.ks[0][0] - QA_F16_FIRST, t.ks[1][0] - QA_F16_FIRST));
    constexpr int PP = HALF ? 1 : NP;
    uint32_t pf[NC][PP][4];
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
      float mx = sc[nc][0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) mx = fmaxf(mx, sc[nc][i >> 2][i & 3]);
      mx *= c_scale;
      if (__any(mx > m_ref[nc] + LAZY)) {
        const float m_new = fmaxf(m_ref[nc], qa_max4(mx) + ABOVE), neg_new = m_new == -INFINITY ? 0.f : -m_new;
        const float alpha = __builtin_amdgcn_exp2f(m_ref[nc] + neg_new);
        m_ref[nc] = m_new;
        neg_m[nc] = neg_new;
        l[nc] *= alpha;
#pragma unroll
        for (int c = 0; c < CPL; ++c)
#pragma unroll
          for (int v = 0; v < 4; ++v) o[nc][c][v] *= alpha;
      }
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(sc[nc][i >> 2][i & 3], c_scale, neg_m[nc]));
      if constexpr (HALF) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {      // (the sum is of the rounded probabilities: numerator and denominator carry the same rounding)
          const qa_f16x2 w = {(_Float16)p[2 * i], (_Float16)p[2 * i + 1]};
          pf[nc][0][i] = __builtin_bit_cast(uint32_t, w);
          l[nc] = __builtin_amdgcn_fdot2(w, qa_f16x2{(_Float16)1.f, (_Float16)1.f}, l[nc], false);
        }
      } else {
        l[nc] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
#pragma unroll
        for (int i = 0; i < 4; ++i) qa_split<NP>(p[2 * i], p[2 * i + 1], &pf[nc][0][i], 4);
      }
    }
    if constexpr (HALF) {
#pragma unroll
      for (int i = 0; i < 8; ++i) e_min = min(e_min, t.vs[i >> 2][i & 3]);
    }
    float ev[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int n = 0; n < 4; ++n) ev[u][n] = qa_scale(t.vs[u][n]);
#pragma unroll
    for (int c2 = 0; c2 < CPL / 2; ++c2) {
      uint32_t e[8];      // channels 2 c2 and 2 c2 + 1 of the lane's eight keys
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t c = t.v[i >> 2][i & 3][c2 / 4];
        e[i] = HALF ? qa_pair16(c, ev[i >> 2][i & 3], c2 & 3) : qa_pair(c, ev[i >> 2][i & 3], c2 & 3);
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t sel = half ? 0x07060302u : 0x05040100u;
        qa_u32x4 vf;
#pragma unroll
        for (int i = 0; i < 4; ++i) vf[i] = __builtin_amdgcn_perm(e[2 * i + 1], e[2 * i], sel);
#pragma unroll
        for (int nc = 0; nc < NC; ++nc)
#pragma unroll
          for (int p = 0; p < PP; ++p) {
            const qa_u32x4 pv = {pf[nc][p][0], pf[nc][p][1], pf[nc][p][2], pf[nc][p][3]};
            qa_f32x4 &to = o[nc][2 * c2 + half];
            if constexpr (HALF) to = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(qa_f16x8, vf), __builtin_bit_cast(qa_f16x8, pv), to, 0, 0, 0);
            else to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(qa_bf16x8, vf), __builtin_bit_cast(qa_bf16x8, pv), to, 0, 0, 0);
          }
      }
    }
    v_used();
  }

  // joins the waves that share a head's keys, in pairs: the upper half of those left hands its sums to the lower half.  All waves of the workgroup call this.
  static constexpr int REGS = NC * (CPL * 4 + 3);
  __device__ __forceinline__ void join(const QAttnArgs &a, const QaWork &w, int hw, int lane, float *s_join) {
    for (int left = a.kr; left > 1; left >>= 1) {
      const int to = left >> 1;
      float *slot = s_join + (size_t)((w.cg * to + (w.sub & (to - 1))) * a.hw + hw) * REGS * 64 + lane;
      if (w.sub >= to && w.sub < left) {
        int r = 0;
#pragma unroll
        for (int nc = 0; nc < NC; ++nc) {
#pragma unroll
          for (int c = 0; c < CPL; ++c)
#pragma unroll
            for (int v = 0; v < 4; ++v) slot[64 * r++] = o[nc][c][v];
          slot[64 * r++] = m_ref[nc];
          slot[64 * r++] = l[nc];
          slot[64 * r++] = __builtin_bit_cast(float, nan_blocks[nc]);
        }
      }
      __syncthreads();
      if (w.sub < to) {
#pragma unroll
        for (int nc = 0; nc < NC; ++nc) {
          const float *from = slot + 64 * nc * (CPL * 4 + 3);
          const float m2 = from[64 * CPL * 4], m_new = fmaxf(m_ref[nc], m2), neg_new = m_new == -INFINITY ? 0.f : -m_new;
          const float w1 = __builtin_amdgcn_exp2f(m_ref[nc] + neg_new), w2 = __builtin_amdgcn_exp2f(m2 + neg_new);
          // (a sum without a maximum is 0, or of scores that are not numbers)
          auto add = [&](float x, float y) { return (m_ref[nc] == -INFINITY ? x : w1 * x) + (m2 == -INFINITY ? y : w2 * y); };
          l[nc] = add(l[nc], from[64 * (CPL * 4 + 1)]);
#pragma unroll
          for (int c = 0; c < CPL; ++c)
#pragma unroll
            for (int v = 0; v < 4; ++v) o[nc][c][v] = add(o[nc][c][v], from[64 * (c * 4 + v)]);
          nan_blocks[nc] |= __builtin_bit_cast(uint32_t, from[64 * (CPL * 4 + 2)]);
          m_ref[nc] = m_new;
        }
      }
      __syncthreads();
    }
  }

  // the result, or the partial record
  __device__ __forceinline__ void finish(const QAttnArgs &a, const QaWork &w) {
    const int G = a.n_q_heads / a.n_kv_heads, h = a.head_dim;
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
      const float l_tot = qa_sum4(l[nc]);
      uint32_t bad = nan_blocks[nc];
      bad |= __shfl_xor(bad, 16, 64);
      bad |= __shfl_xor(bad, 32, 64);
      const int c = 16 * nc + j;
      if (!w.active || c >= w.n_cols) continue;
      const int tok = (w.col0 + c) / G, hj = w.col0 + c - tok * G;
      const int64_t rh = (int64_t)row_of(a, w, tok) * a.n_q_heads + w.g * G + hj;
      const bool direct = a.out != nullptr;
      const float inv = direct ? 1.0f / l_tot : 1.0f;
      float *rec = direct ? nullptr : a.partials + (rh * a.n_parts + w.part) * (h + 2);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        constexpr int PIECE = CPL < 8 ? CPL : 8;
#pragma unroll
        for (int c0 = 0; c0 < CPL; c0 += PIECE) {
          const int ch = CPL * (4 * kg + v) + c0;
          if (ch >= h) continue;
          const float nan = (bad >> (ch / QBLOCK)) & 1 ? __builtin_nanf("") : 0.f;
          float x[PIECE];
#pragma unroll
          for (int i = 0; i < PIECE; ++i) x[i] = o[nc][c0 + i][v] * inv + nan;
          if (!direct) {
#pragma unroll
            for (int i = 0; i < PIECE; i += 2) *reinterpret_cast<float2 *>(rec + ch + i) = make_float2(x[i], x[i + 1]);
          } else if constexpr (sizeof(T) == 2) {
            uint32_t y[PIECE / 2];
#pragma unroll
            for (int i = 0; i < PIECE / 2; ++i) y[i] = qa_pack(x[2 * i], x[2 * i + 1]);
            T *out = (T *)a.out + rh * h + ch;
            if constexpr (PIECE == 8) *reinterpret_cast<uint4 *>(out) = uint4{y[0], y[1], y[2], y[3]};
            else *reinterpret_cast<uint2 *>(out) = uint2{y[0], y[1]};
          } else {
            T *out = (T *)a.out + rh * h + ch;
#pragma unroll
            for (int i = 0; i < PIECE; i += 4) *reinterpret_cast<float4 *>(out + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
          }
        }
      }
      if (!direct && kg == 0) {
        rec[h] = m_ref[nc] == -INFINITY ? (l_tot == 0.f ? -INFINITY : 0.f) : m_ref[nc] * 0.6931471805599453f;      // (NaN scores have no maximum, and have to count)
        rec[h + 1] = l_tot;
      }
    }
  }
};

// Any head size h <= HT that is a multiple of 8; codes wait in registers.  Channels from h on: the queries have zeros there and nothing is stored for
// them; what the lanes read in their place (the next head's codes with this head's exponents) is a number where the head's own are.
// DEPTH steps' codes are on the way at a time.
template <int HT, int NQ, int NP, int NC, int DEPTH, typename TQ, typename T>
__global__ __launch_bounds__(64 * qattn_waves(HT), HT == 256 ? 1 : 2) void qattn_mfma_kernel(QAttnArgs a) {
  typedef QaTile<HT> Tile;
  extern __shared__ float s_join[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = lane & 15, kg = lane >> 4;
  const QaWork w = qa_work<NC>(a, a.items[blockIdx.x], wave);
  const int hb = a.head_dim / 2, nb = q_blocks(a.head_dim), g = w.g;
  const int pitch = a.n_kv_heads * hb, spitch = a.n_kv_heads * nb;
  const uint8_t *Kp = a.c.k + w.key_row0 * pitch + g * hb, *Vp = a.c.v + w.key_row0 * pitch + g * hb;
  const uint8_t *Ksp = a.c.k_scale + w.key_row0 * spitch + g * nb, *Vsp = a.c.v_scale + w.key_row0 * spitch + g * nb;
  const int ks_blk = min(kg * (HT / 4) / QBLOCK, nb - 1), vs_blk = min(Tile::CPL * j / QBLOCK, nb - 1);
  const int k_off = j * pitch + kg * (HT / 8), v_off = 4 * kg * pitch + j * Tile::VB;
  const int ks_off = j * spitch + ks_blk, vs_off = 4 * kg * spitch + vs_blk;

  // Through a resource that ends with the wave's last key: keys beyond it read as zeros, without a branch.
  auto rsrc = [&](const uint8_t *p, int k0, int row, int head) {
    const int left = max(0, min(w.kend - k0, 32)) * row;
    return __builtin_amdgcn_make_buffer_rsrc((void *)(p + (int64_t)k0 * row), (short)0, left > head ? left - head : 0, 0x00020000);
  };
  auto load_k = [&](Tile &t, int k0) {
    const auto r = rsrc(Kp, k0, pitch, g * hb), rs = rsrc(Ksp, k0, spitch, g * nb);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if constexpr (Tile::KS == 2) {
        const auto x = __builtin_amdgcn_raw_buffer_load_b64(r, k_off, 16 * u * pitch, 0);
        t.k[u][0] = x[0]; t.k[u][1] = x[1];
      } else {
#pragma unroll
        for (int d = 0; d < Tile::KS; d += 4) {
          const auto x = __builtin_amdgcn_raw_buffer_load_b128(r, k_off + 4 * d, 16 * u * pitch, 0);
          t.k[u][d] = x[0]; t.k[u][d + 1] = x[1]; t.k[u][d + 2] = x[2]; t.k[u][d + 3] = x[3];
        }
      }
      t.ks[u][0] = __builtin_amdgcn_raw_buffer_load_b8(rs, ks_off, 16 * u * spitch, 0);
      if constexpr (Tile::KSC == 2) t.ks[u][1] = __builtin_amdgcn_raw_buffer_load_b8(rs, ks_off + (ks_blk + 1 < nb ? 1 : 0), 16 * u * spitch, 0);
    }
  };
  auto load_v = [&](Tile &t, int k0) {
    const auto r = rsrc(Vp, k0, pitch, g * hb), rs = rsrc(Vsp, k0, spitch, g * nb);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        if constexpr (Tile::VB == 2) {
          t.v[u][n][0] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, v_off, (16 * u + n) * pitch, 0);
        } else if constexpr (Tile::VB == 4) {
          t.v[u][n][0] = __builtin_amdgcn_raw_buffer_load_b32(r, v_off, (16 * u + n) * pitch, 0);
        } else {
          const auto x = __builtin_amdgcn_raw_buffer_load_b64(r, v_off, (16 * u + n) * pitch, 0);
          t.v[u][n][0] = x[0]; t.v[u][n][1] = x[1];
        }
        t.vs[u][n] = __builtin_amdgcn_raw_buffer_load_b8(rs, vs_off, (16 * u + n) * spitch, 0);
      }
  };

  Tile ring[DEPTH];
#pragma unroll
  for (int d = 0; d < DEPTH; ++d) { load_k(ring[d], w.kbeg + 32 * d); load_v(ring[d], w.kbeg + 32 * d); }
  QaColumns<HT, NQ, NP, NC, false, TQ, T> q;
  q.begin(a, w, lane);
  for (int k0 = w.kbeg; k0 < w.kend; k0 += 32 * DEPTH) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {      // each half of a tile is asked for again as soon as it has been used
      const int at = k0 + 32 * d;
      if (at < w.kend) q.step(a, w, ring[d], at, [&] { load_k(ring[d], at + 32 * DEPTH); }, [] {}, [&] { load_v(ring[d], at + 32 * DEPTH); });
    }
  }
  if (a.kr > 1) {
    q.join(a, w, wave % a.hw, lane, s_join);
    if (w.sub != 0) return;
  }
  q.finish(a, w);
}

// Head sizes 64 and 128 whose codes begin at multiples of 16 bytes: codes and exponents go from memory into LDS, in whole 16-byte pieces of
// a head's row, each wave into a ring of its own (no barriers), and from there into registers.  A request of 64 lanes keeps the vector memory unit busy for
// about 16 clocks whatever its lanes ask for: six of them a step instead of twenty.  Rows of V lie in LDS in the order that gives the four lanes
// (j, 0..3) of a read different banks; pieces of K are turned by a place every four rows for the same reason.
template <int HT, int DEPTH> struct QaRing {
  static constexpr int RB = HT / 2, ROWS = 32 * RB, STAGE = 2 * ROWS + 512, WAVE = DEPTH * STAGE;      // bytes: a row, 32 of them, a step, a wave's ring
  static constexpr int REQ = RB / 32, PER_STEP = 2 * REQ + 2;                                         // requests of an array and of a step
};
__device__ __forceinline__ void qa_dword_to_lds(i32x4 rsrc, int voff, int lds) {
  lds = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(rsrc) : "memory");
}
// OCC: waves on a SIMD.
template <int HT, int NQ, int NP, int NC, int DEPTH, int OCC, bool HALF, typename TQ, typename T>
__global__ __launch_bounds__(512, OCC) void qattn_lds_kernel(QAttnArgs a) {
  if (!HALF && a.narrow != nullptr && a.narrow[blockIdx.x] == 0) return;      // (done in fp16)
  typedef QaTile<HT> Tile;
  typedef QaRing<HT, DEPTH> R;
  extern __shared__ __align__(16) char s_ring[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = lane & 15, kg = lane >> 4;
  const QaWork w = qa_work<NC>(a, a.items[blockIdx.x], wave);
  constexpr int hb = HT / 2, nb = HT / QBLOCK;
  const int pitch = a.n_kv_heads * hb, spitch = a.n_kv_heads * nb, g = w.g;
  const uint8_t *Kp = a.c.k + w.key_row0 * pitch + g * hb, *Vp = a.c.v + w.key_row0 * pitch + g * hb;
  // exponents come as the dword that holds a head's (two heads share one at HT = 64)
  const int e_at = g * nb & ~3, e_in = g * nb & 3;
  const uint8_t *Ksp = a.c.k_scale + w.key_row0 * spitch + e_at, *Vsp = a.c.v_scale + w.key_row0 * spitch + e_at;

  // lane i of a request: place i of 64 pieces of 16 bytes
  constexpr int PIECES = hb / 16, RPR = 64 / PIECES;      // pieces of a row, rows of a request
  const int slot_row = lane / PIECES, piece = lane % PIECES;
  int k_voff, v_voff;
  if constexpr (HT == 128) {
    k_voff = slot_row * pitch + ((piece - (slot_row >> 2)) & 3) * 16;
    v_voff = (4 * (slot_row & 3) + (slot_row >> 2)) * pitch + piece * 16;
  } else {
    k_voff = slot_row * pitch + ((piece - (slot_row >> 3)) & 1) * 16;
    v_voff = ((slot_row & 16) + 4 * (slot_row & 3) + ((slot_row & 15) >> 2)) * pitch + piece * 16;
  }
  const int e_voff = lane < 32 ? lane * spitch : (int)0x80000000;      // (the upper lanes ask for nothing)
  char *ring = s_ring + wave * R::WAVE;
  const int lds0 = (int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)ring;
  auto ask = [&](int k0, int slot) {
    const int left = max(0, min(w.kend - k0, 32)), rows = left * pitch - g * hb, exps = left * spitch - e_at;
    const i32x4 rk = make_rsrc(Kp + (int64_t)k0 * pitch, left > 0 ? rows : 0), rv = make_rsrc(Vp + (int64_t)k0 * pitch, left > 0 ? rows : 0);
    const i32x4 ek = make_rsrc(Ksp + (int64_t)k0 * spitch, left > 0 ? exps : 0), ev = make_rsrc(Vsp + (int64_t)k0 * spitch, left > 0 ? exps : 0);
    const int to = lds0 + slot * R::STAGE;
#pragma unroll
    for (int i = 0; i < R::REQ; ++i) load_to_lds(rk, k_voff, i * RPR * pitch, to + i * 1024);
    qa_dword_to_lds(ek, e_voff, to + 2 * R::ROWS);
#pragma unroll
    for (int i = 0; i < R::REQ; ++i) load_to_lds(rv, v_voff, i * RPR * pitch, to + R::ROWS + i * 1024);
    qa_dword_to_lds(ev, e_voff, to + 2 * R::ROWS + 256);
  };
#pragma unroll
  for (int d = 0; d < DEPTH; ++d) ask(w.kbeg + 32 * d, d);
  QaColumns<HT, NQ, NP, NC, HALF, TQ, T> q;
  q.begin(a, w, lane);
  // the queries are here before the first step (a wait for them inside the loop would be one for everything on the way)
#pragma unroll
  for (int nc = 0; nc < NC; ++nc)
#pragma unroll
    for (int p = 0; p < NQ; ++p)
#pragma unroll
      for (int s = 0; s < Tile::KS; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(q.qf[nc][p][s][i]));

  const int k_at = HT == 128 ? j * hb + ((kg + (j >> 2)) & 3) * 16 : j * hb + (((kg >> 1) + (j >> 3)) & 1) * 16 + (kg & 1) * 8;
  const int ks_at = 2 * R::ROWS + 4 * j + e_in + kg * (HT / 4) / QBLOCK;
  const int v_at = R::ROWS + kg * hb + j * Tile::VB;      // slot of row 16 u + 4 kg + n: 16 u + 4 n + kg
  const int vs_at = 2 * R::ROWS + 256 + 16 * kg + e_in + Tile::CPL * j / QBLOCK;
  int slot = 0;
  // HALF: products and conversions count, not memory.  No wave waits for another, and of the two on a SIMD one goes first, so that its products run beside the
  // other's conversions (in step and alike: 300 rows each of 4 sequences on 3000 keys 154 us, so 148; 2500 rows 124, so 121).
  if (HALF && wave >= 4) __builtin_amdgcn_s_setprio(2);
  for (int i = 0; i < w.steps; ++i) {
    // The heads of a token share lines of memory: waves that drift apart fetch them twice (64 x 16449 keys: 1.29 GB instead of 1.15, 248 us; so 206).
    // Every wave of the workgroup comes by here as often as the others.
    if (!HALF) __builtin_amdgcn_s_barrier();
    const int k0 = w.kbeg + 32 * i;
    if (k0 >= w.kend) continue;
    wait_vm<(DEPTH - 1) * R::PER_STEP>();
    const char *st = ring + slot * R::STAGE;
    Tile t;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if constexpr (HT == 128) {
        const qa_u32x4 x = *reinterpret_cast<const qa_u32x4 *>(st + k_at + u * 16 * hb);
        t.k[u][0] = x[0]; t.k[u][1] = x[1]; t.k[u][2] = x[2]; t.k[u][3] = x[3];
      } else {
        const uint2 x = *reinterpret_cast<const uint2 *>(st + k_at + u * 16 * hb);
        t.k[u][0] = x.x; t.k[u][1] = x.y;
      }
      t.ks[u][0] = (uint8_t)st[ks_at + 64 * u];
    }
    auto need_v = [&] {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          if constexpr (HT == 128) t.v[u][n][0] = *reinterpret_cast<const uint32_t *>(st + v_at + (16 * u + 4 * n) * hb);
          else t.v[u][n][0] = *reinterpret_cast<const uint16_t *>(st + v_at + (16 * u + 4 * n) * hb);
          t.vs[u][n] = (uint8_t)st[vs_at + 64 * u + 4 * n];
        }
      wait_lds();      // the step has left its place in the ring
      ask(k0 + 32 * DEPTH, slot);
    };
    q.step(a, w, t, k0, [] {}, need_v, [] {});
    slot = slot + 1 == DEPTH ? 0 : slot + 1;
  }
  wait_vm<0>();      // (nothing of this wave may land in LDS that is another's by then)
  if constexpr (HALF) {
    __syncthreads();      // (every wave is through with its ring)
    int *said = reinterpret_cast<int *>(s_ring);
    const bool narrow = __any(q.too_narrow());
    if (lane == 0) said[wave] = narrow;
    __syncthreads();
    if (threadIdx.x == 0) {
      int any = 0;
      for (int i = 0; i < 8; ++i) any |= said[i];
      a.narrow[blockIdx.x] = (uint32_t)any;
    }
  }
  if (a.kr > 1) {
    __syncthreads();
    q.join(a, w, wave % a.hw, lane, reinterpret_cast<float *>(s_ring));
    if (w.sub != 0) return;
  }
  q.finish(a, w);
}

template <int HT, int NQ, int NP, int NC, int DEPTH, typename TQ, typename T>
void qattn_mfma_start(const QAttnArgs &a, int n_items, hipStream_t s) {
  auto kern = qattn_mfma_kernel<HT, NQ, NP, NC, DEPTH, TQ, T>;
  constexpr int W = qattn_waves(HT);
  const size_t smem = a.kr == 1 ? 0 : (size_t)(W / 2) * NC * (HT / 4 + 3) * 64 * sizeof(float);      // half of the waves hand over at most
  if (smem > 48 * 1024) (void)hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  hipLaunchKernelGGL(kern, dim3(n_items), dim3(64 * W), smem, s, a);
}
template <int HT, int NQ, int NP, int NC, int DEPTH, int OCC, bool HALF, typename TQ, typename T>
void qattn_lds_start(const QAttnArgs &a, int n_items, hipStream_t s) {
  auto kern = qattn_lds_kernel<HT, NQ, NP, NC, DEPTH, OCC, HALF, TQ, T>;
  const size_t join = a.kr == 1 ? 0 : (size_t)4 * NC * (HT / 4 + 3) * 64 * sizeof(float), ring = (size_t)8 * QaRing<HT, DEPTH>::WAVE;
  const size_t smem = join > ring ? join : ring;
  static_assert(8 * QaRing<HT, DEPTH>::WAVE <= 160 * 1024 && 4 * NC * (HT / 4 + 3) * 256 <= 160 * 1024, "");
  if (smem > 48 * 1024) (void)hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  hipLaunchKernelGGL(kern, dim3(n_items), dim3(512), smem, s, a);
}

}  // namespace alora
