// Attention over rows of 4 bits (Eq.1 with the causal mask, Eq.4), the keys and values turned into numbers on their way into the products.
#include "qcache.h"

namespace alora {

constexpr float QA_LOG2E = 1.4426950408889634f;
constexpr float QA_LN2 = 0.6931471805599453f;

__device__ __forceinline__ float q_value(uint32_t code, int e) {
  // e2m1: exponent 0 is 0 or 0.5, the others 1.m * 2^(exponent - 1)
  const int ex = (code >> 1) & 3, m = code & 1;
  const float mag = ex == 0 ? 0.5f * m : (1.0f + 0.5f * m) * (float)(1 << (ex - 1));
  const float sc = e == Q_E_NAN ? __builtin_nanf("") : __builtin_bit_cast(float, (uint32_t)e << 23);
  return (code & 8 ? -mag : mag) * sc;
}

// Any even head size.  One wave per (row, query head, part of the row's keys): 64 keys a step, a key per lane for the scores, two channels
// per lane for the sum; running maximum and sum as everywhere.  Keys that the row does not see are never read.
template <typename T>
__global__ __launch_bounds__(64) void qattn_plain_kernel(const void *__restrict__ Q, QueryType qt, QRows c, const SeqMeta *__restrict__ seqs,
                                                         const int32_t *__restrict__ row_seq, LayerDims L, int n_splits,
                                                         float *__restrict__ partials, T *__restrict__ out) {
  __shared__ float s_q[256], s_p[64];
  __shared__ int64_t s_row[64];
  const int lane = threadIdx.x, h = L.head_dim, half = h / 2, nb = q_blocks(h);
  const int row = blockIdx.x / L.n_q_heads, hq = blockIdx.x % L.n_q_heads, part = blockIdx.y;
  const int g = hq / (L.n_q_heads / L.n_kv_heads);
  const SeqMeta sm = seqs[row_seq[row]];
  const int n_vis = sm.P + (row - sm.row_start) + 1;      // keys that the row sees
  const int per = ((n_vis + n_splits - 1) / n_splits + 63) & ~63;
  const int kbeg = min(n_vis, part * per), kend = min(n_vis, kbeg + per);
  for (int i = lane; i < h; i += 64) {
    const int64_t at = (int64_t)row * L.n_q + hq * h + i;
    s_q[i] = qt == Q_F32 ? ((const float *)Q)[at] : qt == Q_BF16 ? (float)((const bf16 *)Q)[at] : (float)((const _Float16 *)Q)[at];
  }
  __syncthreads();
  const float sc = QA_LOG2E / sqrtf((float)h);
  float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = kbeg; k0 < kend; k0 += 64) {
    const int n = min(64, kend - k0);
    float s = -INFINITY;
    if (lane < n) {
      const int64_t at = seq_pool_row(sm, k0 + lane) * L.n_kv_heads + g;
      s_row[lane] = at;
      s = 0.f;
      for (int i = 0; i < half; ++i) {
        const uint32_t b = c.k[at * half + i];
        const int e = c.k_scale[at * nb + 2 * i / QBLOCK];
        s += s_q[2 * i] * q_value(b & 15, e) + s_q[2 * i + 1] * q_value(b >> 4, e);
      }
      s *= sc;
    }
    const float m_new = fmaxf(m, wave_max(s)), ref = m_new == -INFINITY ? 0.f : m_new;
    const float p = lane < n ? exp2f(s - ref) : 0.f, alpha = exp2f(m - ref);
    s_p[lane] = p;
    __syncthreads();
    l = l * alpha + wave_sum(p);
    m = m_new;
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] *= alpha;
    for (int k = 0; k < n; ++k)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (lane + 64 * j < half) {
          const uint32_t b = c.v[s_row[k] * half + lane + 64 * j];
          const int e = c.v_scale[s_row[k] * nb + 2 * (lane + 64 * j) / QBLOCK];
          acc[2 * j] += s_p[k] * q_value(b & 15, e);
          acc[2 * j + 1] += s_p[k] * q_value(b >> 4, e);
        }
    __syncthreads();
  }
  if (out != nullptr) {
    const float inv = 1.0f / l;
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (lane + 64 * j < half) {
        T *o = out + (int64_t)row * L.n_q + hq * h + 2 * (lane + 64 * j);
        o[0] = from_f32<T>(acc[2 * j] * inv);
        o[1] = from_f32<T>(acc[2 * j + 1] * inv);
      }
    return;
  }
  float *pp = partials + (((int64_t)row * L.n_q_heads + hq) * n_splits + part) * (h + 2);
#pragma unroll
  for (int j = 0; j < 2; ++j)
    if (lane + 64 * j < half) { pp[2 * (lane + 64 * j)] = acc[2 * j]; pp[2 * (lane + 64 * j) + 1] = acc[2 * j + 1]; }
  if (lane == 0) {
    pp[h] = m == -INFINITY ? (l == 0.f ? -INFINITY : 0.f) : m * QA_LN2;      // (NaN scores have no maximum, and have to count)
    pp[h + 1] = l;
  }
}

template <typename T>
void launch_qattn_plain(const void *Q, QueryType qt, const QRows &c, const SeqMeta *seqs, const int32_t *row_seq, const LayerDims &L, int T_rows,
                        int n_splits, float *partials, T *out, hipStream_t s) {
  if (T_rows == 0) return;
  hipLaunchKernelGGL(qattn_plain_kernel<T>, dim3((unsigned)(T_rows * L.n_q_heads), n_splits), dim3(64), 0, s, Q, qt, c, seqs, row_seq, L, n_splits,
                     partials, out);
}
template void launch_qattn_plain<float>(const void *, QueryType, const QRows &, const SeqMeta *, const int32_t *, const LayerDims &, int, int, float *, float *, hipStream_t);
template void launch_qattn_plain<bf16>(const void *, QueryType, const QRows &, const SeqMeta *, const int32_t *, const LayerDims &, int, int, float *, bf16 *, hipStream_t);

}  // namespace alora
