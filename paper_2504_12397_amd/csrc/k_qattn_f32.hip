// Attention over rows of 4 bits on the matrix units: queries and results of fp32.
#include "qattn_mfma.h"

namespace alora {

void launch_qattn_mfma_f32(const QAttnArgs &a, int n_items, int ht, int nc, bool lds, hipStream_t s) {
  if (lds && ht == 64 && nc == 1) return qattn_lds_start<64, 3, 3, 1, 6, 2, false, float, float>(a, n_items, s);
  if (lds && ht == 128 && nc == 1) return qattn_lds_start<128, 3, 3, 1, 4, 2, false, float, float>(a, n_items, s);
  if (!lds && ht == 64 && nc == 1) return qattn_mfma_start<64, 3, 3, 1, 3, float, float>(a, n_items, s);
  if (!lds && ht == 128 && nc == 1) return qattn_mfma_start<128, 3, 3, 1, 2, float, float>(a, n_items, s);
  if (!lds && ht == 256 && nc == 1) return qattn_mfma_start<256, 3, 3, 1, 1, float, float>(a, n_items, s);
}

}  // namespace alora
