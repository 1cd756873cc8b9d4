// Attention over a paged cache in 8 bits where a KV head has more than 64 rows: the builds of the kernel in paged_rows_bf16.h
// that read e4m3 pages and their scales.
#include "paged_rows_bf16.h"

namespace dreams {

hipError_t launch_paged_rows_e4m3(const AttnArgs8& a, hipStream_t stream) { return launch_rows<true>(a, stream); }

}  // namespace dreams
