// Attention over a paged cache, bf16, where a KV head has at most 64 rows: the builds of the kernel in tree_attn_bf16.h that
// read pages.
#include "tree_attn_bf16.h"

namespace dreams {
namespace {

template <int D, int NST>
hipError_t launch_for_rows(const AttnArgs& a, hipStream_t stream) {
  switch (a.rows_per_wg) {
    case 16: return launch_streaming<D, 1, 4, 4, NST, 1, false, true>(a, stream);
    case 32: return launch_streaming<D, 1, 4, 8, NST, 1, false, true>(a, stream);
    case 64: return launch_streaming<D, 2, 2, 4, NST / 2, 2, false, true>(a, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_paged_attn_bf16(const AttnArgs& a, hipStream_t stream) {
  if (a.unit_parts < 1 || a.units * a.unit_parts % 8 != 0) return hipErrorInvalidValue;
  if (a.D == 128) return launch_for_rows<128, 8>(a, stream);
  if (a.D == 64) return launch_for_rows<64, 16>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace dreams
