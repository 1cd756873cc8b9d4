// Attention over a paged cache, bf16, where a KV head has more than 64 rows: the builds of the kernel in paged_rows_bf16.h
// that read bf16 pages.
#include "paged_rows_bf16.h"

namespace dreams {

hipError_t launch_paged_rows_bf16(const AttnArgs& a, hipStream_t stream) { return launch_rows<false>(a, stream); }

}  // namespace dreams
