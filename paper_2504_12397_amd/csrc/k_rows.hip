// Moving cached rows: copies between pools and inside one (forking, compacting), and the two directions between rows of the storage
// type and rows of 4 bits.  All of it is bound by memory; a call is one launch over (pieces of ranges) x (arrays of all layers).
#include "qcache.h"

namespace alora {

// The piece of a range that workgroup x of the launch moves (binary search over the ranges' first pieces, uniform, unless every range is one), and the
// array that workgroup y does.
struct RowPiece { int64_t src, dst; int rows; };
template <bool FEW> __device__ __forceinline__ RowPiece row_piece(const RowsArgs &a, const RowsFew &few) {
  const RowRange *ranges = FEW ? reinterpret_cast<const RowRange *>(few.data) : a.ranges;
  const uint32_t chunk = blockIdx.x;
  int lo = 0, hi = a.n_ranges - 1;
  if (a.n_chunks == a.n_ranges) lo = hi = (int)chunk;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (ranges[mid].first_chunk <= chunk) lo = mid; else hi = mid - 1;
  }
  const RowRange r = ranges[lo];
  const int64_t at = (int64_t)(chunk - r.first_chunk) * a.chunk_rows, left = r.n - at;
  return RowPiece{r.src + at, r.dst + at, (int)(left < a.chunk_rows ? left : a.chunk_rows)};
}
template <bool FEW> __device__ __forceinline__ RowPlane row_plane(const RowsArgs &a, const RowsFew &few) {
  return FEW ? reinterpret_cast<const RowPlane *>(few.data + a.planes_at)[blockIdx.y] : a.planes[blockIdx.y];
}

template <typename U>
__device__ __forceinline__ void copy_piece(const RowPlane &pl, const RowPiece &p) {
  const U *src = reinterpret_cast<const U *>((const char *)pl.src + p.src * pl.row_bytes);
  U *dst = reinterpret_cast<U *>((char *)pl.dst + p.dst * pl.row_bytes);
  const int64_t n = p.rows * (int64_t)pl.row_bytes / (int64_t)sizeof(U);
  for (int64_t i0 = threadIdx.x; i0 < n; i0 += 4 * 256) {      // four pieces on the way
    U v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i0 + j * 256 < n) v[j] = src[i0 + j * 256];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i0 + j * 256 < n) dst[i0 + j * 256] = v[j];
  }
}

template <bool FEW>
__global__ __launch_bounds__(256) void rows_copy_kernel(RowsArgs a, RowsFew few) {
  const RowPlane pl = row_plane<FEW>(a, few);
  const RowPiece p = row_piece<FEW>(a, few);
  if (pl.unit == 16) copy_piece<uint4>(pl, p);
  else if (pl.unit == 4) copy_piece<uint32_t>(pl, p);
  else copy_piece<uint8_t>(pl, p);
}

void launch_rows_copy(const RowsArgs &a, const RowsFew &few, hipStream_t s) {
  if (a.n_chunks == 0 || a.n_planes == 0) return;
  const dim3 grid((unsigned)a.n_chunks, (unsigned)a.n_planes);
  auto kern = a.planes == nullptr ? rows_copy_kernel<true> : rows_copy_kernel<false>;
  hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, a, few);
}

// Workgroups take the pieces of their array by tickets, so that one only ever waits for pieces that running workgroups have taken, and those for earlier ones: every
// wait ends.  One pass over memory, where staging takes two (a workspace written and read).
// (U: what is moved at a time; R: the register it waits in)
template <typename U, typename R>
__device__ __forceinline__ void ordered_piece(const RowsOrderedArgs &a, const RowPlane &pl, const RowStep &st, int step, int plane) {
  const U *src = reinterpret_cast<const U *>((const char *)pl.src + st.src * pl.row_bytes);
  U *dst = reinterpret_cast<U *>((char *)pl.dst + st.dst * pl.row_bytes);
  const int n = (int)((int64_t)st.rows * pl.row_bytes / (int)sizeof(U)), tid = threadIdx.x;      // <= ROWS_ORDERED_UNITS
  R v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = tid + j * 256 < n ? (R)src[tid + j * 256] : R{};
  // The piece is in registers before anyone is told so.  (No data passes between workgroups, only that: relaxed flags; acquiring and releasing would write the
  // caches back and empty them at every piece: 75000 rows of 1088 bytes in four layers 1470 us, so 205; through a workspace 385.)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) __hip_atomic_store(a.read + (int64_t)step * a.n_planes + plane, a.epoch, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  for (int d = st.dep0 + tid; d < st.dep1; d += 256)
    if (d != step)
      while (__hip_atomic_load(a.read + (int64_t)d * a.n_planes + plane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != a.epoch) __builtin_amdgcn_s_sleep(1);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (tid + j * 256 < n) dst[tid + j * 256] = (U)v[j];
}
template <bool FEW>
__global__ __launch_bounds__(256) void rows_copy_ordered_kernel(RowsOrderedArgs a, RowsFew few) {
  __shared__ uint32_t s_step;
  const int plane = (int)(blockIdx.x % (uint32_t)a.n_planes);
  if (threadIdx.x == 0) {
    uint32_t *ticket = a.ticket + plane * ROWS_TICKET_STRIDE;
    s_step = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (s_step == (uint32_t)a.n_steps - 1) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // (the last one: nobody else takes any)
  }
  __syncthreads();
  const int step = __builtin_amdgcn_readfirstlane((int)s_step);
  if (step >= a.n_steps) return;
  const RowPlane pl = FEW ? reinterpret_cast<const RowPlane *>(few.data + a.planes_at)[plane] : a.planes[plane];
  const RowStep st = FEW ? reinterpret_cast<const RowStep *>(few.data)[step] : a.steps[step];
  if (pl.unit == 16) ordered_piece<uint4, uint4>(a, pl, st, step, plane);
  else if (pl.unit == 4) ordered_piece<uint32_t, uint32_t>(a, pl, st, step, plane);
  else ordered_piece<uint8_t, uint32_t>(a, pl, st, step, plane);
}
void launch_rows_copy_ordered(const RowsOrderedArgs &a, const RowsFew &few, hipStream_t s) {
  auto kern = a.steps == nullptr ? rows_copy_ordered_kernel<true> : rows_copy_ordered_kernel<false>;
  hipLaunchKernelGGL(kern, dim3((unsigned)a.n_steps * (unsigned)a.n_planes), dim3(256), 0, s, a, few);
}

// ---- rows of the storage type <-> rows of 4 bits -------------------------------------------------------------
// The exponent byte of a block with this largest magnitude (as bits): that of the magnitude less 2, so that it lands in [4, 8) of the
// codes' [0, 6]; less 1 where its mantissa is over 1.75, so that at most a seventh of the magnitude is cut off (7 -> 6; at Q_E_MAX, over 1.75 * 2^127, 8 -> 6).  Blocks of zeros have 127.
__device__ __forceinline__ int q_exponent(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return Q_E_NAN;
  const int e = (int)((amax_bits + 0x1fffffu) >> 23) - 2;
  return amax_bits == 0 ? 127 : min(max(e, Q_E_MIN), Q_E_MAX);
}
__device__ __forceinline__ float q_scale(int e) { return __builtin_bit_cast(float, (uint32_t)e << 23); }
__device__ __forceinline__ uint32_t abs_bits(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

// One thread per block of 32 channels, any head size and alignment.
template <typename T, bool FEW>
__global__ __launch_bounds__(256) void rows_store_any_kernel(RowsArgs a, RowsFew few, int n_kv_heads, int head_dim) {
  const RowPlane pl = row_plane<FEW>(a, few);
  const RowPiece p = row_piece<FEW>(a, few);
  const int nb = q_blocks(head_dim), per_row = n_kv_heads * nb;
  for (int i = threadIdx.x; i < p.rows * per_row; i += 256) {
    const int r = i / per_row, hb = i - r * per_row, g = hb / nb, blk = hb - g * nb;
    const int c0 = blk * QBLOCK, n = min(QBLOCK, head_dim - c0);
    const int64_t hs = (p.src + r) * n_kv_heads + g, hd = (p.dst + r) * n_kv_heads + g;
    const T *x = (const T *)pl.src + hs * head_dim + c0;
    uint32_t top = 0;
    for (int c = 0; c < n; ++c) top = max(top, abs_bits(to_f32<T>(x[c])));
    const int e = q_exponent(top);
    const float sc = q_scale(e);
    uint8_t *q = (uint8_t *)pl.dst + hd * (head_dim / 2) + c0 / 2;
    for (int c = 0; c < n; c += 2)
      q[c / 2] = e == Q_E_NAN ? 0 : (uint8_t)__builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, to_f32<T>(x[c]), to_f32<T>(x[c + 1]), sc, 0);
    ((uint8_t *)pl.scale)[hd * nb + blk] = (uint8_t)e;
  }
}

template <typename T, bool FEW>
__global__ __launch_bounds__(256) void rows_load_any_kernel(RowsArgs a, RowsFew few, int n_kv_heads, int head_dim) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  const RowPlane pl = row_plane<FEW>(a, few);
  const RowPiece p = row_piece<FEW>(a, few);
  const int nb = q_blocks(head_dim), half = head_dim / 2, per_row = n_kv_heads * half;
  for (int i = threadIdx.x; i < p.rows * per_row; i += 256) {
    const int r = i / per_row, hb = i - r * per_row, g = hb / half, c2 = hb - g * half;
    const int64_t hs = (p.src + r) * n_kv_heads + g, hd = (p.dst + r) * n_kv_heads + g;
    const uint32_t code = ((const uint8_t *)pl.src)[hs * half + c2];
    const int e = ((const uint8_t *)pl.scale)[hs * nb + 2 * c2 / QBLOCK];
    const f32x2_t v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, q_scale(e), 0);
    T *x = (T *)pl.dst + hd * head_dim + 2 * c2;
    x[0] = from_f32<T>(e == Q_E_NAN ? __builtin_nanf("") : v.x);
    x[1] = from_f32<T>(e == Q_E_NAN ? __builtin_nanf("") : v.y);
  }
}

// Head sizes that are multiples of 8: four lanes share a block, a lane has 8 channels -- 16 bytes of bf16, 4 of codes -- so that both sides of a piece are one run of
// memory (lanes past a head's last channels, where they are no whole block, have nothing to do: PAD).  WIDE_AHEAD such loads are on the way per lane.  16384
// rows of eight layers (8 heads of 128, bf16): 107 us in, 97 back, 6.3 and 7.0 TB/s of both sides, part of it from the last-level cache.
constexpr int WIDE_AHEAD = 4;
typedef uint32_t rows_u32x4 __attribute__((ext_vector_type(4)));
template <typename T> struct Wide8;
template <> struct Wide8<bf16> {
  rows_u32x4 w;
  __device__ __forceinline__ void load(const bf16 *p) { w = __builtin_nontemporal_load(reinterpret_cast<const rows_u32x4 *>(p)); }
  __device__ __forceinline__ float at(int i) const { return __builtin_bit_cast(float, i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
  __device__ __forceinline__ uint32_t top() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, max(w[i] & 0x7fff0000u, w[i] << 16 & 0x7fff0000u));
    return m;
  }
};
template <> struct Wide8<float> {
  rows_u32x4 w[2];
  __device__ __forceinline__ void load(const float *p) {
    w[0] = __builtin_nontemporal_load(reinterpret_cast<const rows_u32x4 *>(p));
    w[1] = __builtin_nontemporal_load(reinterpret_cast<const rows_u32x4 *>(p) + 1);
  }
  __device__ __forceinline__ float at(int i) const {
    const uint32_t u = w[i >> 2][i & 3];      // (a bit cast of the element itself would take the vector's first)
    return __builtin_bit_cast(float, u);
  }
  __device__ __forceinline__ uint32_t top() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, w[i >> 2][i & 3] & 0x7fffffffu);
    return m;
  }
};
// Lane i's place: head (counted from the piece's first), its 8 channels of it; there: some are
struct WideAt { int head, eight; bool there; };
template <bool PAD> __device__ __forceinline__ WideAt wide_at(int i, int n, int eights, int lanes) {
  if (!PAD) return WideAt{0, i, i < n};      // (one run over all heads)
  const int head = i / lanes, e = i - head * lanes;
  return WideAt{head, e, i < n && e < eights};
}
// the largest of a block's four lanes
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));      // lanes 1 0 3 2
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));   // lanes 2 3 0 1
}

template <typename T, bool FEW, bool PAD>
__global__ __launch_bounds__(256) void rows_store_wide_kernel(RowsArgs a, RowsFew few, int n_kv_heads, int head_dim) {
  const RowPlane pl = row_plane<FEW>(a, few);
  const RowPiece p = row_piece<FEW>(a, few);
  const int eights = head_dim / 8, blocks = q_blocks(head_dim), lanes = 4 * blocks, n = p.rows * n_kv_heads * lanes;
  const T *src = (const T *)pl.src + p.src * n_kv_heads * head_dim;
  uint32_t *dst = (uint32_t *)pl.dst + p.dst * n_kv_heads * eights;
  uint8_t *scale = (uint8_t *)pl.scale + p.dst * n_kv_heads * blocks;
  for (int i0 = threadIdx.x; i0 < n; i0 += WIDE_AHEAD * 256) {
    Wide8<T> x[WIDE_AHEAD];
    WideAt at[WIDE_AHEAD];
#pragma unroll
    for (int u = 0; u < WIDE_AHEAD; ++u) {
      at[u] = wide_at<PAD>(i0 + u * 256, n, eights, lanes);
      if (at[u].there) x[u].load(src + ((int64_t)at[u].head * eights + at[u].eight) * 8);
      else x[u] = Wide8<T>{};
    }
#pragma unroll
    for (int u = 0; u < WIDE_AHEAD; ++u) {
      const int e = q_exponent(quad_max(x[u].top()));
      const float sc = q_scale(e);
      uint32_t w = 0;
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[u].at(0), x[u].at(1), sc, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[u].at(2), x[u].at(3), sc, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[u].at(4), x[u].at(5), sc, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[u].at(6), x[u].at(7), sc, 3);
      if (!at[u].there) continue;
      dst[at[u].head * eights + at[u].eight] = e == Q_E_NAN ? 0u : w;
      if ((at[u].eight & 3) == 0) scale[at[u].head * blocks + (at[u].eight >> 2)] = (uint8_t)e;
    }
  }
}

template <typename T, bool FEW, bool PAD>
__global__ __launch_bounds__(256) void rows_load_wide_kernel(RowsArgs a, RowsFew few, int n_kv_heads, int head_dim) {
  const RowPlane pl = row_plane<FEW>(a, few);
  const RowPiece p = row_piece<FEW>(a, few);
  const int eights = head_dim / 8, blocks = q_blocks(head_dim), lanes = PAD ? eights : 4 * blocks, n = p.rows * n_kv_heads * lanes;
  const uint32_t *src = (const uint32_t *)pl.src + p.src * n_kv_heads * eights;
  const uint8_t *scale = (const uint8_t *)pl.scale + p.src * n_kv_heads * blocks;
  T *dst = (T *)pl.dst + p.dst * n_kv_heads * head_dim;
  for (int i0 = threadIdx.x; i0 < n; i0 += WIDE_AHEAD * 256) {
    uint32_t w[WIDE_AHEAD], e[WIDE_AHEAD];
#pragma unroll
    for (int u = 0; u < WIDE_AHEAD; ++u) {
      const int i = i0 + u * 256;
      w[u] = e[u] = 0;
      if (i >= n) continue;
      const WideAt at = wide_at<PAD>(i, n, eights, lanes);
      w[u] = src[i];
      e[u] = scale[at.head * blocks + (at.eight >> 2)];
    }
#pragma unroll
    for (int u = 0; u < WIDE_AHEAD; ++u) {
      const int i = i0 + u * 256;
      if (i >= n) continue;
      const float sc = q_scale((int)e[u]);      // (an exponent of 255 makes every code NaN)
      if constexpr (sizeof(T) == 2) {
        rows_u32x4 y;
        y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[u], sc, 0));
        y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[u], sc, 1));
        y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[u], sc, 2));
        y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[u], sc, 3));
        __builtin_nontemporal_store(y, reinterpret_cast<rows_u32x4 *>(dst) + i);
      } else {
        rows_u32x4 y[2];
        auto put = [&](int at, auto v) {
          const float x0 = v[0], x1 = v[1];
          y[at >> 2][at & 3] = __builtin_bit_cast(uint32_t, x0);
          y[at >> 2][(at & 3) + 1] = __builtin_bit_cast(uint32_t, x1);
        };
        put(0, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], sc, 0));
        put(2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], sc, 1));
        put(4, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], sc, 2));
        put(6, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], sc, 3));
        __builtin_nontemporal_store(y[0], reinterpret_cast<rows_u32x4 *>(dst) + 2 * i);
        __builtin_nontemporal_store(y[1], reinterpret_cast<rows_u32x4 *>(dst) + 2 * i + 1);
      }
    }
  }
}

template <typename T> void launch_rows_store(const RowsArgs &a, const RowsFew &few, int n_kv_heads, int head_dim, bool wide, hipStream_t s) {
  if (a.n_chunks == 0 || a.n_planes == 0) return;
  const dim3 grid((unsigned)a.n_chunks, (unsigned)a.n_planes);
  const bool f = a.planes == nullptr;
  auto any = f ? rows_store_any_kernel<T, true> : rows_store_any_kernel<T, false>;
  auto fast = head_dim % QBLOCK == 0 ? (f ? rows_store_wide_kernel<T, true, false> : rows_store_wide_kernel<T, false, false>)
                                     : (f ? rows_store_wide_kernel<T, true, true> : rows_store_wide_kernel<T, false, true>);
  if (wide) hipLaunchKernelGGL(fast, grid, dim3(256), 0, s, a, few, n_kv_heads, head_dim);
  else hipLaunchKernelGGL(any, grid, dim3(256), 0, s, a, few, n_kv_heads, head_dim);
}
template <typename T> void launch_rows_load(const RowsArgs &a, const RowsFew &few, int n_kv_heads, int head_dim, bool wide, hipStream_t s) {
  if (a.n_chunks == 0 || a.n_planes == 0) return;
  const dim3 grid((unsigned)a.n_chunks, (unsigned)a.n_planes);
  const bool f = a.planes == nullptr;
  auto any = f ? rows_load_any_kernel<T, true> : rows_load_any_kernel<T, false>;
  auto fast = head_dim % QBLOCK == 0 ? (f ? rows_load_wide_kernel<T, true, false> : rows_load_wide_kernel<T, false, false>)
                                     : (f ? rows_load_wide_kernel<T, true, true> : rows_load_wide_kernel<T, false, true>);
  if (wide) hipLaunchKernelGGL(fast, grid, dim3(256), 0, s, a, few, n_kv_heads, head_dim);
  else hipLaunchKernelGGL(any, grid, dim3(256), 0, s, a, few, n_kv_heads, head_dim);
}
template void launch_rows_store<float>(const RowsArgs &, const RowsFew &, int, int, bool, hipStream_t);
template void launch_rows_store<bf16>(const RowsArgs &, const RowsFew &, int, int, bool, hipStream_t);
template void launch_rows_load<float>(const RowsArgs &, const RowsFew &, int, int, bool, hipStream_t);
template void launch_rows_load<bf16>(const RowsArgs &, const RowsFew &, int, int, bool, hipStream_t);

}  // namespace alora
