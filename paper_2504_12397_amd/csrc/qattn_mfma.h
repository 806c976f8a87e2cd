// Attention over rows of 4 bits on the matrix units (Eq.1 with the causal mask, Eq.4): for head sizes that are multiples of 8.
//
// A wave takes 16 * NC columns -- (row, query head) pairs that read one kv head -- and walks a range of keys, 32 a step:
//   * Codes of K go from memory straight into the A operand of v_mfma_f32_16x16x32_bf16: lane (j, kg) has the HT / 4 channels from kg * HT / 4 on of
//     key j of 16, a dword (8 channels) per product; the queries, laid out alike, are the B operand: S[key][column].  v_cvt_scalef32_pk_bf16_fp4
//     turns two codes into two numbers, scale included, in one instruction: bf16 holds every code times every power of two exactly, where
//     fp16 would overflow or lose bits for exponents far from 127.
//   * Accumulator register v of lane (j, kg) is key 4 kg + v of column j: a lane owns one column, the softmax needs no other lane but
//     for a new maximum, and the probabilities of two blocks of 16 keys are, as they sit, the B operand (32 keys) of O += V P.
//   * V: lane (j, kg) has CPL = HT / 16 channels from CPL j on of those 8 keys; after conversion a byte permute of two keys' words puts
//     one channel of two keys side by side, which is the transposition: product c is channel CPL i + c of lane row i.
// No LDS and no barrier but where several waves share a head's keys (KR > 1): they join at the end, in pairs.
// Queries of bf16 are one operand, exactly; fp16 two (high and low bits as bf16), fp32 three.  Probabilities are two operands (16 bits; one of 8
// bits would add half of what the rounding of a bf16 result does), three for fp32.
// The reference exponent of a column moves only when a score exceeds it by 2^8: almost no step rescales the sums.
#pragma once
#include "qcache.h"

namespace alora {

typedef __bf16 qa_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 qa_bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t qa_u32x4 __attribute__((ext_vector_type(4)));
typedef float qa_f32x4 __attribute__((ext_vector_type(4)));

constexpr float QA_LAZY = 8.0f;      // log2 units

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

// Any head size h <= HT that is a multiple of 8.  Channels from h on: the queries have zeros there and nothing is stored for them; what the lanes
// read in their place (the next head's codes with this head's exponents) is a number where the head's own are.
// DEPTH steps' codes are on the way at a time.
template <int HT, int NQ, int NP, int NC, int DEPTH, typename TQ, typename T>
__global__ __launch_bounds__(512, 2) void qattn_mfma_kernel(QAttnArgs a) {
  constexpr int KS = HT / 32;       // products per block of 16 keys, dwords of K per lane
  constexpr int CPL = HT / 16;      // channels of V per lane
  constexpr int VB = CPL / 2;       // bytes of them
  constexpr int VW = (VB + 3) / 4;
  constexpr int KSC = HT == 256 ? 2 : 1;      // exponents of K per lane
  extern __shared__ float s_join[];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = lane & 15, kg = lane >> 4;
  const QAttnItem it = a.items[blockIdx.x];
  const int h = a.head_dim, hb = h / 2, nb = q_blocks(h);
  const int G = a.n_q_heads / a.n_kv_heads;
  const int hw = wave % a.hw, rest = wave / a.hw, sub = rest % a.kr, cg = rest / a.kr;
  const int c_first = cg * 16 * NC, n_cols = min(it.n_cols - c_first, 16 * NC);      // columns of this wave, counted from c_first
  const bool active = it.g0 + hw < a.n_kv_heads && n_cols > 0;
  const int g = min(it.g0 + hw, a.n_kv_heads - 1);
  const int col0 = it.col0 + c_first;

  // keys of this wave: its share of those that its last column sees
  const int last_tok = (col0 + max(n_cols, 1) - 1) / G, first_tok = col0 / G;
  int per = (it.kend - it.kbeg + a.kr - 1) / a.kr;
  per = (per + 31) & ~31;
  const int kbeg = it.kbeg + sub * per;
  int kend = min(it.kend, kbeg + per);
  if (!it.shared) kend = min(kend, it.pos0 + last_tok + 1);
  if (!active) kend = kbeg;
  const int see_all = it.shared ? kend : min(kend, it.pos0 + first_tok + 1);      // keys below are seen by every column

  const int pitch = a.n_kv_heads * hb, spitch = a.n_kv_heads * nb;
  const uint8_t *Kp = a.c.k + it.key_row0 * pitch + g * hb, *Vp = a.c.v + it.key_row0 * pitch + g * hb;
  const uint8_t *Ksp = a.c.k_scale + it.key_row0 * spitch + g * nb, *Vsp = a.c.v_scale + it.key_row0 * spitch + g * nb;
  const int ks_blk = min(kg * (HT / 4) / QBLOCK, nb - 1), vs_blk = min(CPL * j / QBLOCK, nb - 1);
  const int k_off = j * pitch + kg * (HT / 8), v_off = 4 * kg * pitch + j * VB;
  const int ks_off = j * spitch + ks_blk, vs_off = 4 * kg * spitch + vs_blk;

  // A step of 32 keys from k0 on, through a resource that ends with the wave's last key: keys beyond it read as zeros, without a branch.
  struct Tile {
    uint32_t k[2][KS];
    uint32_t ks[2][KSC];
    uint32_t v[2][4][VW];      // [u][n]: key 16 u + 4 kg + n
    uint32_t vs[2][4];
  };
  auto rsrc = [&](const uint8_t *p, int k0, int row, int head) {
    const int left = max(0, min(kend - k0, 32)) * row;
    return __builtin_amdgcn_make_buffer_rsrc((void *)(p + (int64_t)k0 * row), (short)0, left > head ? left - head : 0, 0x00020000);
  };
  auto load_k = [&](Tile &t, int k0) {
    const auto r = rsrc(Kp, k0, pitch, g * hb), rs = rsrc(Ksp, k0, spitch, g * nb);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if constexpr (KS == 2) {
        const auto w = __builtin_amdgcn_raw_buffer_load_b64(r, k_off, 16 * u * pitch, 0);
        t.k[u][0] = w[0]; t.k[u][1] = w[1];
      } else {
#pragma unroll
        for (int d = 0; d < KS; d += 4) {
          const auto w = __builtin_amdgcn_raw_buffer_load_b128(r, k_off + 4 * d, 16 * u * pitch, 0);
          t.k[u][d] = w[0]; t.k[u][d + 1] = w[1]; t.k[u][d + 2] = w[2]; t.k[u][d + 3] = w[3];
        }
      }
      t.ks[u][0] = __builtin_amdgcn_raw_buffer_load_b8(rs, ks_off, 16 * u * spitch, 0);
      if constexpr (KSC == 2) t.ks[u][1] = __builtin_amdgcn_raw_buffer_load_b8(rs, ks_off + (ks_blk + 1 < nb ? 1 : 0), 16 * u * spitch, 0);
    }
  };
  auto load_v = [&](Tile &t, int k0) {
    const auto r = rsrc(Vp, k0, pitch, g * hb), rs = rsrc(Vsp, k0, spitch, g * nb);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        if constexpr (VB == 2) {
          t.v[u][n][0] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, v_off, (16 * u + n) * pitch, 0);
        } else if constexpr (VB == 4) {
          t.v[u][n][0] = __builtin_amdgcn_raw_buffer_load_b32(r, v_off, (16 * u + n) * pitch, 0);
        } else {
          const auto w = __builtin_amdgcn_raw_buffer_load_b64(r, v_off, (16 * u + n) * pitch, 0);
          t.v[u][n][0] = w[0]; t.v[u][n][1] = w[1];
        }
        t.vs[u][n] = __builtin_amdgcn_raw_buffer_load_b8(rs, vs_off, (16 * u + n) * spitch, 0);
      }
  };

  Tile ring[DEPTH];
#pragma unroll
  for (int d = 0; d < DEPTH; ++d) { load_k(ring[d], kbeg + 32 * d); load_v(ring[d], kbeg + 32 * d); }

  // queries
  uint32_t qf[NC][NQ][KS][4];
  int lim[NC];      // last key that the column sees
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) {
    const int c = 16 * nc + j, tok = (col0 + c) / G, hj = col0 + c - tok * G;
    const bool there = active && c < n_cols;
    lim[nc] = it.shared || !there ? 0x7fffffff : it.pos0 + tok;
    const int row = !there ? 0 : it.shared ? a.rows[it.first_row + tok] : it.first_row + tok;
    const TQ *q = (const TQ *)a.Q + ((int64_t)row * a.n_q_heads + g * G + (there ? hj : 0)) * h;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int ch = kg * (HT / 4) + 8 * s;
      const bool in = there && ch < h;
      if constexpr (sizeof(TQ) == 2 && NQ == 1) {
        const qa_u32x4 w = in ? *reinterpret_cast<const qa_u32x4 *>(q + ch) : qa_u32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) qf[nc][0][s][i] = w[i];
      } else {
        float x[8];
        if constexpr (sizeof(TQ) == 2) {
          typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
          f16x8_t w = {};
          if (in) w = *reinterpret_cast<const f16x8_t *>(q + ch);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = (float)w[i];
        } else {
          qa_f32x4 w0 = {}, w1 = {};
          if (in) { w0 = *reinterpret_cast<const qa_f32x4 *>(q + ch); w1 = *reinterpret_cast<const qa_f32x4 *>(q + ch + 4); }
#pragma unroll
          for (int i = 0; i < 4; ++i) { x[i] = w0[i]; x[4 + i] = w1[i]; }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) qa_split<NQ>(x[2 * i], x[2 * i + 1], &qf[nc][0][s][i], KS * 4);
      }
    }
  }

  qa_f32x4 o[NC][CPL];
  float m_ref[NC], neg_m[NC], l[NC];      // reference exponent (log2), its negative or 0 where there is none, this lane's part of the sum
  uint32_t nan_blocks[NC];                // blocks of 32 channels in which the column has met a value that is not a number
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) {
#pragma unroll
    for (int c = 0; c < CPL; ++c) o[nc][c] = qa_f32x4{0.f, 0.f, 0.f, 0.f};
    m_ref[nc] = -INFINITY;
    neg_m[nc] = l[nc] = 0.f;
    nan_blocks[nc] = 0;
  }
  const float c_scale = a.sm_scale * 1.4426950408889634f;

  auto step = [&](Tile &t, int k0) {
    qa_f32x4 sc[NC][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int nc = 0; nc < NC; ++nc) sc[nc][u] = qa_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const float e = qa_scale(t.ks[u][KSC == 2 ? s / 4 : 0]);
        const uint32_t w = t.k[u][s];
        const qa_u32x4 kf = {qa_pair(w, e, 0), qa_pair(w, e, 1), qa_pair(w, e, 2), qa_pair(w, e, 3)};
#pragma unroll
        for (int nc = 0; nc < NC; ++nc)
#pragma unroll
          for (int p = 0; p < NQ; ++p) {
            const qa_u32x4 qv = {qf[nc][p][s][0], qf[nc][p][s][1], qf[nc][p][s][2], qf[nc][p][s][3]};
            sc[nc][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(qa_bf16x8, kf), __builtin_bit_cast(qa_bf16x8, qv), sc[nc][u], 0, 0, 0);
          }
      }
    }
    load_k(t, k0 + 32 * DEPTH);      // (each half of the tile is asked for again as soon as it has been used)
    if (k0 + 32 > see_all) {      // a step that some column sees in part
      bool bad = false;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int key = k0 + 16 * u + 4 * kg + v;
          bad |= t.vs[u][v] == (uint32_t)Q_E_NAN;
#pragma unroll
          for (int nc = 0; nc < NC; ++nc)
            if (key >= kend || key > lim[nc]) sc[nc][u][v] = -INFINITY;
        }
      if (__any(bad)) {
        // 0 times NaN would reach the columns that do not see the key: its values count as 0, and the columns that do see it remember the block
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const int key = k0 + 16 * u + 4 * kg + v;
            const uint8_t *sp = Vsp + (int64_t)min(key, kend - 1) * spitch;
            uint32_t blocks = 0;
            for (int b = 0; b < nb; ++b) blocks |= (sp[b] == Q_E_NAN ? 1u : 0u) << b;
#pragma unroll
            for (int nc = 0; nc < NC; ++nc)
              if (key < kend && key <= lim[nc]) nan_blocks[nc] |= blocks;
            if (t.vs[u][v] == (uint32_t)Q_E_NAN) {
              t.vs[u][v] = 127;
#pragma unroll
              for (int i = 0; i < VW; ++i) t.v[u][v][i] = 0;
            }
          }
      }
    }
    uint32_t pf[NC][NP][4];
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
      float mx = sc[nc][0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) mx = fmaxf(mx, sc[nc][i >> 2][i & 3]);
      mx *= c_scale;
      if (__any(mx > m_ref[nc] + QA_LAZY)) {
        const float m_new = fmaxf(m_ref[nc], qa_max4(mx)), neg_new = m_new == -INFINITY ? 0.f : -m_new;
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
      l[nc] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
#pragma unroll
      for (int i = 0; i < 4; ++i) qa_split<NP>(p[2 * i], p[2 * i + 1], &pf[nc][0][i], 4);
    }
    float ev[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int n = 0; n < 4; ++n) ev[u][n] = qa_scale(t.vs[u][n]);
#pragma unroll
    for (int w = 0; w < CPL / 2; ++w) {
      uint32_t e[8];      // channels 2 w and 2 w + 1 of the lane's eight keys
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = qa_pair(t.v[i >> 2][i & 3][w / 4], ev[i >> 2][i & 3], w & 3);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t sel = half ? 0x07060302u : 0x05040100u;
        qa_u32x4 vf;
#pragma unroll
        for (int i = 0; i < 4; ++i) vf[i] = __builtin_amdgcn_perm(e[2 * i + 1], e[2 * i], sel);
#pragma unroll
        for (int nc = 0; nc < NC; ++nc)
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            const qa_u32x4 pv = {pf[nc][p][0], pf[nc][p][1], pf[nc][p][2], pf[nc][p][3]};
            o[nc][2 * w + half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(qa_bf16x8, vf), __builtin_bit_cast(qa_bf16x8, pv), o[nc][2 * w + half], 0, 0, 0);
          }
      }
    }
    load_v(t, k0 + 32 * DEPTH);
  };
  for (int k0 = kbeg; k0 < kend; k0 += 32 * DEPTH) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
      if (k0 + 32 * d < kend) step(ring[d], k0 + 32 * d);
  }

  // ---- join the waves that share a head's keys, in pairs: the upper half of those left hands its sums to the lower half
  if (a.kr > 1) {
    constexpr int REGS = NC * (CPL * 4 + 3);
    for (int left = a.kr; left > 1; left >>= 1) {
      const int to = left >> 1;
      float *slot = s_join + (size_t)((cg * to + (sub & (to - 1))) * a.hw + hw) * REGS * 64 + lane;
      if (sub >= to && sub < left) {
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
      if (sub < to) {
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
    if (sub != 0) return;
  }

  // ---- o[c][v] of lane (j, kg) is channel CPL * (4 kg + v) + c of column j
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) {
    const float l_tot = qa_sum4(l[nc]);
    uint32_t bad = nan_blocks[nc];
    bad |= __shfl_xor(bad, 16, 64);
    bad |= __shfl_xor(bad, 32, 64);
    const int c = 16 * nc + j;
    if (!active || c >= n_cols) continue;
    const int tok = (col0 + c) / G, hj = col0 + c - tok * G;
    const int row = it.shared ? a.rows[it.first_row + tok] : it.first_row + tok;
    const int64_t rh = (int64_t)row * a.n_q_heads + g * G + hj;
    const bool direct = a.out != nullptr;
    const float inv = direct ? 1.0f / l_tot : 1.0f;
    float *rec = direct ? nullptr : a.partials + (rh * a.n_parts + it.part) * (h + 2);
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
          uint32_t w[PIECE / 2];
#pragma unroll
          for (int i = 0; i < PIECE / 2; ++i) w[i] = qa_pack(x[2 * i], x[2 * i + 1]);
          T *out = (T *)a.out + rh * h + ch;
          if constexpr (PIECE == 8) *reinterpret_cast<uint4 *>(out) = uint4{w[0], w[1], w[2], w[3]};
          else *reinterpret_cast<uint2 *>(out) = uint2{w[0], w[1]};
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

template <int HT, int NQ, int NP, int NC, int DEPTH, typename TQ, typename T>
void qattn_mfma_start(const QAttnArgs &a, int n_items, hipStream_t s) {
  auto kern = qattn_mfma_kernel<HT, NQ, NP, NC, DEPTH, TQ, T>;
  const size_t smem = a.kr == 1 ? 0 : (size_t)4 * NC * (HT / 4 + 3) * 64 * sizeof(float);      // four waves hand over at most
  if (smem > 48 * 1024) (void)hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  hipLaunchKernelGGL(kern, dim3(n_items), dim3(512), smem, s, a);
}

}  // namespace alora
