// Launchers of the kernels on cached rows: copying them, storing them in 4 bits and loading them again, attention over them.
#pragma once
#include "common.h"

namespace alora {

// ---- rows of 4 bits -------------------------------------------------------------------------------------
// A row holds head_dim codes of 4 bits per kv head (sign and e2m1 magnitude: 0, 0.5, 1, 1.5, 2, 3, 4, 6; element 2i in the low half of
// byte i) and one exponent byte E for each QBLOCK channels (the last block of a head may be shorter): value = code * 2^(E - 127).
constexpr int QBLOCK = 32;
constexpr int Q_E_MIN = 2, Q_E_MAX = 252, Q_E_NAN = 255;      // (every value and half of the smallest one are normal fp32 and bf16 numbers)
__host__ __device__ inline int q_blocks(int head_dim) { return (head_dim + QBLOCK - 1) / QBLOCK; }

// ---- moving rows (alora_cache_copy, alora_qcache_copy / store / load) ------------------------------------
// One array per layer and kind of data (keys, values; codes and exponents): row r begins at base + r * row_bytes.  Storing and
// loading use dst and src for the rows of 4 bits and of the storage type, `scale` for the exponents.
struct RowPlane {
  const void *src;
  void *dst;
  void *scale;             // store: written; load: read
  uint32_t row_bytes;      // copy ...
  uint32_t unit;           // ... in pieces of 16, 4 or 1 bytes, which both bases and the rows are multiples of
};
// n rows from src on go to dst on; first_chunk: how many pieces of chunk_rows rows the ranges before it are cut in
struct RowRange { int64_t src, dst; uint32_t n, first_chunk; };
// Few of both travel as kernel arguments (no staging kernel before the copy, and a captured call keeps them): ranges, then planes.  More of them
// lie in device memory.
constexpr int ROWS_FEW_BYTES = 3584;
struct RowsFew { alignas(16) char data[ROWS_FEW_BYTES]; };
inline size_t rows_few_planes_at(size_t n_ranges) { return (n_ranges * sizeof(RowRange) + 15) & ~(size_t)15; }
inline bool rows_are_few(size_t n_ranges, size_t n_planes) { return rows_few_planes_at(n_ranges) + n_planes * sizeof(RowPlane) <= ROWS_FEW_BYTES; }
struct RowsArgs {
  const RowRange *ranges;        // both nullptr: in `few`
  const RowPlane *planes;
  int n_ranges, n_planes;
  int64_t n_chunks;              // of all ranges
  int chunk_rows;
  int planes_at;                 // in `few`
};
void launch_rows_copy(const RowsArgs &a, const RowsFew &few, hipStream_t s);
// Rows that move over each other, all of them towards the front (or all towards the back) of one pool: pieces in the order of their destinations, from
// the end that they move to.  A piece is read, says so, and is written once the pieces dep0 .. dep1 - 1 -- those whose sources its destination
// covers, all of them before it -- have been read.
struct RowStep { int64_t src, dst; int32_t rows, dep0, dep1, pad_; };
struct RowsOrderedArgs {
  const RowStep *steps;          // both nullptr: in `few`, steps first
  const RowPlane *planes;
  int n_steps, n_planes, planes_at;
  uint32_t *ticket;              // [n_planes], ROWS_TICKET_STRIDE apart (a line of memory each: one counter for all was 290 us of 19000 workgroups); 0 before and after a call
  uint32_t *read;                // [n_steps, n_planes]: `epoch` once the piece has been read
  uint32_t epoch;                // another one for every call on these flags
};
constexpr int ROWS_TICKET_STRIDE = 32, ROWS_ORDERED_PLANES = 1024;
constexpr int ROWS_ORDERED_UNITS = 256 * 8;      // most units that a piece of any plane has
constexpr int ROWS_ORDERED_STEPS = 32768;        // most pieces of a launch (a table of 1.3 MB)
void launch_rows_copy_ordered(const RowsOrderedArgs &a, const RowsFew &few, hipStream_t s);
// T rows of n_kv heads of head_dim <-> rows of 4 bits; wide: head_dim is a multiple of 8, rows begin at multiples of 16 bytes, codes of 4
template <typename T> void launch_rows_store(const RowsArgs &a, const RowsFew &few, int n_kv_heads, int head_dim, bool wide, hipStream_t s);
template <typename T> void launch_rows_load(const RowsArgs &a, const RowsFew &few, int n_kv_heads, int head_dim, bool wide, hipStream_t s);

// ---- attention over rows of 4 bits ---------------------------------------------------------------------------
struct QRows { const uint8_t *k, *v, *k_scale, *v_scale; };      // pool arrays of one layer
enum QueryType { Q_F32 = 0, Q_BF16 = 1, Q_F16 = 2 };

// any even head size: a wave per (row, query head, part); row_seq[T]: the row's sequence.  out: the result itself, with n_splits == 1 only
template <typename T>
void launch_qattn_plain(const void *Q, QueryType qt, const QRows &c, const SeqMeta *seqs, const int32_t *row_seq, const LayerDims &L, int T_rows,
                        int n_splits, float *partials, T *out, hipStream_t s);

// Head sizes that are multiples of 8, on the matrix units.  A workgroup of eight waves (four for heads of more than 128 channels, whose sums and
// queries take more registers than a wave of eight may have) is hw kv heads x kr shares of the item's keys x cw
// groups of 16 * nc columns; a column is a (row, query head) pair: column c of a unit is head c % G of its row c / G.
__host__ __device__ constexpr int qattn_waves(int ht) { return ht == 256 ? 4 : 8; }
struct QAttnItem {
  int64_t key_row0;         // pool row of key 0
  int32_t kbeg, kend;       // keys, counted from key_row0; none beyond kend is read
  int32_t first_row;        // own keys: packed row of the unit's row 0; shared: where the unit's rows begin in QAttnArgs::rows
  int32_t col0, n_cols;     // columns of the unit that this item takes
  int32_t pos0;             // own keys: the last key that row 0 sees (row i: pos0 + i); shared: every row sees all
  int32_t g0, part;         // first kv head; which of the n_parts partial records of a (row, head) it writes
  int32_t shared, pad_;
};
static_assert(sizeof(QAttnItem) == 48, "");
struct QAttnArgs {
  const void *Q;            // [T, n_q_heads, head_dim]
  QRows c;
  const QAttnItem *items;
  const int32_t *rows;      // packed rows of the shared units
  int n_q_heads, n_kv_heads, head_dim;
  int hw, kr, cw;
  int n_parts;
  float sm_scale;
  float *partials;          // [T, n_q_heads, n_parts, head_dim + 2] (sums, maximum, sum of probabilities), used when out == nullptr
  void *out;                // [T, n_q_heads, head_dim], with n_parts == 1 only
  uint32_t *narrow;         // [items] or nullptr: written by a launch in fp16, 1 where that was too narrow; the launch after it does those items
};
// ht: 64, 128 or 256, the smallest that holds head_dim.  Codes begin at multiples of 4 bytes, queries and results of 16.
// lds: head_dim is 64 (with an even number of kv heads) or 128, codes begin at multiples of 16 bytes and exponents at multiples of 4.
// half: fp16 (lds and nc > 1 only); otherwise, with args.narrow, only items that are marked there.
void launch_qattn_mfma_bf16(const QAttnArgs &a, int n_items, int ht, int nc, bool lds, bool half, hipStream_t s);      // queries of bf16; nc 1, 2 or 4 (ht 128: 1, 2; 256: 1)
void launch_qattn_mfma_f16(const QAttnArgs &a, int n_items, int ht, int nc, bool lds, bool half, hipStream_t s);       // of fp16; nc 1 or 2 (ht 256: 1)
void launch_qattn_mfma_f32(const QAttnArgs &a, int n_items, int ht, int nc, bool lds, hipStream_t s);                  // of fp32; nc 1

}  // namespace alora
