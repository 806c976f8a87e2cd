// Moving cached rows: copies between pools and inside one (forking, compacting), and the two directions between rows of the storage
// type and rows of 4 bits.  All of it is bound by memory; a call is one launch over (pieces of ranges) x (arrays of all layers).
#include "qcache.h"

namespace alora {

// The piece of a range that workgroup x of the launch moves: binary search over the ranges' first pieces (uniform, scalar loads).
struct RowPiece { int64_t src, dst; int rows; };
__device__ __forceinline__ RowPiece row_piece(const RowRange *ranges, int n_ranges, int64_t chunk, int chunk_rows) {
  int lo = 0, hi = n_ranges - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (ranges[mid].first_chunk <= chunk) lo = mid; else hi = mid - 1;
  }
  const RowRange r = ranges[lo];
  const int64_t at = (chunk - r.first_chunk) * chunk_rows, left = r.n - at;
  return RowPiece{r.src + at, r.dst + at, (int)(left < chunk_rows ? left : chunk_rows)};
}

template <typename U>
__device__ __forceinline__ void copy_piece(const RowPlane &pl, const RowPiece &p) {
  const U *src = reinterpret_cast<const U *>((const char *)pl.src + p.src * pl.row_bytes);
  U *dst = reinterpret_cast<U *>((char *)pl.dst + p.dst * pl.row_bytes);
  const int64_t n = p.rows * pl.row_bytes / (int64_t)sizeof(U);
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
  const RowPlane pl = FEW ? few.planes[blockIdx.y] : a.planes[blockIdx.y];
  const RowPiece p = row_piece(FEW ? few.ranges : a.ranges, a.n_ranges, blockIdx.x, a.chunk_rows);
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

// ---- rows of the storage type <-> rows of 4 bits -------------------------------------------------------------
// The exponent byte of a block with this largest magnitude (as bits): that of the magnitude less 2, so that it lands in [4, 8) of the
// codes' [0, 6]; less 1 where its mantissa is over 1.75, so that at most a seventh of the magnitude is cut off (7 -> 6).
__device__ __forceinline__ int q_exponent(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return Q_E_NAN;
  const int e = (int)((amax_bits + 0x1fffffu) >> 23) - 2;
  return min(max(e, Q_E_MIN), Q_E_MAX);
}
__device__ __forceinline__ float q_scale(int e) { return __builtin_bit_cast(float, (uint32_t)e << 23); }
__device__ __forceinline__ uint32_t abs_bits(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

// One thread per block of 32 channels, any head size and alignment.
template <typename T, bool FEW>
__global__ __launch_bounds__(256) void rows_store_any_kernel(RowsArgs a, RowsFew few, int n_kv_heads, int head_dim) {
  const RowPlane pl = FEW ? few.planes[blockIdx.y] : a.planes[blockIdx.y];
  const RowPiece p = row_piece(FEW ? few.ranges : a.ranges, a.n_ranges, blockIdx.x, a.chunk_rows);
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
  const RowPlane pl = FEW ? few.planes[blockIdx.y] : a.planes[blockIdx.y];
  const RowPiece p = row_piece(FEW ? few.ranges : a.ranges, a.n_ranges, blockIdx.x, a.chunk_rows);
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

template <typename T> void launch_rows_store(const RowsArgs &a, const RowsFew &few, int n_kv_heads, int head_dim, bool wide, hipStream_t s) {
  if (a.n_chunks == 0 || a.n_planes == 0) return;
  (void)wide;
  const dim3 grid((unsigned)a.n_chunks, (unsigned)a.n_planes);
  auto kern = a.planes == nullptr ? rows_store_any_kernel<T, true> : rows_store_any_kernel<T, false>;
  hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, a, few, n_kv_heads, head_dim);
}
template <typename T> void launch_rows_load(const RowsArgs &a, const RowsFew &few, int n_kv_heads, int head_dim, bool wide, hipStream_t s) {
  if (a.n_chunks == 0 || a.n_planes == 0) return;
  (void)wide;
  const dim3 grid((unsigned)a.n_chunks, (unsigned)a.n_planes);
  auto kern = a.planes == nullptr ? rows_load_any_kernel<T, true> : rows_load_any_kernel<T, false>;
  hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, a, few, n_kv_heads, head_dim);
}
template void launch_rows_store<float>(const RowsArgs &, const RowsFew &, int, int, bool, hipStream_t);
template void launch_rows_store<bf16>(const RowsArgs &, const RowsFew &, int, int, bool, hipStream_t);
template void launch_rows_load<float>(const RowsArgs &, const RowsFew &, int, int, bool, hipStream_t);
template void launch_rows_load<bf16>(const RowsArgs &, const RowsFew &, int, int, bool, hipStream_t);

}  // namespace alora
