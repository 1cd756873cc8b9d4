// Attention over a paged cache in 8 bits, up to 64 rows a workgroup: the builds of the kernel in tree_attn_bf16.h that read
// e4m3 pages and their scales.
//
// Tokens of long contexts are bound by the memory (8 sequences x 8 KV heads behind 16384 to 32768 slots, 403 MB, 74.8 us with
// the launch that merges: 5.4 TB/s; 8 x 32 heads behind 6000 each 62 us in one piece, 6.3 TB/s), those of short ones by the chain of
// lengths, table, first copies and merge (4 sequences with 1028 keys in sight 13.7).  64 rows of contexts like 32 heads x 60 nodes
// behind 3136 slots, 22.3 us (bf16 pages, twice the bytes: 23.2), are bound by that chain too: 12 until the first step and from
// the last one on (11.7 behind 40 slots), 4 to 5 for the pieces' exchange and merge, 5.8 for the keys, 1.8 for each 1000.  So over the
// whole call waves wait for counts and barriers 58 % of the time, for issue 11 %, and matrix cores work 4 %.  In the loop over
// steps instructions are about half of the time (a wave's 32 rows and 32 keys: 32 products, 64 conversions, 16 exponentials, 110
// other vector and 120 scalar instructions), a third waits for barriers and counts.
// Tried there: two steps' operands in registers (24.7), reads ahead of the copies' addresses and look-ups behind the score
// product (registers spill at 128 columns, 20.3 instead of 19.5 us at 64).
#include "tree_attn_bf16.h"

namespace dreams {
namespace {

// (16 rows: two workgroups of half a ring each to a compute unit: 8 x 8 KV heads of 16384 to 32768 tokens, one row of 4 heads
// each, 85.5 us with one of a whole ring, 73.9 with two.  64 rows: 8 waves in 4 key groups, one workgroup to a unit, would be
// 22.6 us instead of 22.0 for 32 heads x 60 nodes behind 3136.)
// (32 rows: 8 waves on a whole ring, or 4 on half of one; 64 rows of 64 columns are on the 128-row kernel.)
template <int D, bool WIDE>
hipError_t launch_for_rows(const AttnArgs8& a, hipStream_t stream) {
  switch (a.rows_per_wg) {
    case 16: return launch_streaming<D, 1, 4, 4, 1024 / D, 2, false, true, true, WIDE>(a, stream);
    case 32:
      if (a.half_ring) return launch_streaming<D, 2, 4, 4, 1024 / D, 2, false, true, true, WIDE>(a, stream);
      return launch_streaming<D, 1, 4, 8, 16, 1, false, true, true, WIDE>(a, stream);
    case 64:
      if constexpr (D == 128) return launch_streaming<D, 2, 2, 4, 1024 / D, 2, false, true, true, WIDE>(a, stream);
  }
  return hipErrorInvalidValue;
}
template <int D>
hipError_t launch_for_pages(const AttnArgs8& a, hipStream_t stream) {
  return 1 << a.page_shift >= kStep ? launch_for_rows<D, true>(a, stream) : launch_for_rows<D, false>(a, stream);
}

}  // namespace

hipError_t launch_paged_attn_e4m3(const AttnArgs8& a, hipStream_t stream) {
  if (a.unit_parts < 1) return hipErrorInvalidValue;
  if (a.D == 128) return launch_for_pages<128>(a, stream);
  if (a.D == 64) return launch_for_pages<64>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace dreams
