// Attention over rows of 4 bits on the matrix units: queries of fp16, results of bf16.
#include "qattn_mfma.h"

namespace alora {

void launch_qattn_mfma_f16(const QAttnArgs &a, int n_items, int ht, int nc, bool lds, bool half, hipStream_t s) {
  if (lds && half && ht == 64 && nc == 2) return qattn_lds_start<64, 1, 2, 2, 5, 2, true, _Float16, bf16>(a, n_items, s);
  if (lds && ht == 64 && nc == 2) return qattn_lds_start<64, 2, 2, 2, 5, 2, false, _Float16, bf16>(a, n_items, s);
  if (lds && ht == 64 && nc == 1) return qattn_lds_start<64, 2, 2, 1, 6, 2, false, _Float16, bf16>(a, n_items, s);
  if (lds && half && ht == 128 && nc == 2) return qattn_lds_start<128, 1, 2, 2, 4, 2, true, _Float16, bf16>(a, n_items, s);
  if (lds && ht == 128 && nc == 2) return qattn_lds_start<128, 2, 2, 2, 4, 2, false, _Float16, bf16>(a, n_items, s);
  if (lds && ht == 128 && nc == 1) return qattn_lds_start<128, 2, 2, 1, 4, 2, false, _Float16, bf16>(a, n_items, s);
  if (!lds && ht == 64 && nc == 2) return qattn_mfma_start<64, 2, 2, 2, 2, _Float16, bf16>(a, n_items, s);
  if (!lds && ht == 64 && nc == 1) return qattn_mfma_start<64, 2, 2, 1, 4, _Float16, bf16>(a, n_items, s);
  if (!lds && ht == 128 && nc == 2) return qattn_mfma_start<128, 2, 2, 2, 1, _Float16, bf16>(a, n_items, s);
  if (!lds && ht == 128 && nc == 1) return qattn_mfma_start<128, 2, 2, 1, 3, _Float16, bf16>(a, n_items, s);
  if (!lds && ht == 256 && nc == 1) return qattn_mfma_start<256, 2, 2, 1, 1, _Float16, bf16>(a, n_items, s);
}

}  // namespace alora
