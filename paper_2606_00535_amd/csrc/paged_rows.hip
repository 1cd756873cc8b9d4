// Rows of a paged cache: new rows written into their slots (append), and the accepted path's rows moved to the slots
// behind the committed prefix (commit).  Both are copies of 16-byte words, bit for bit; a row costs one read and one
// write of K and of V.
#include "kernels.h"

namespace dreams {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Byte offset of a slot's row within a layer, or -1: past the table, or a page outside the pool.
__device__ __forceinline__ int64_t slot_offset(const PagedRowsArgs& a, const int32_t* table, int g, long long slot) {
  if (slot < 0 || (slot >> a.page_shift) >= a.width) return -1;
  const int id = table[slot >> a.page_shift];
  if (id < 0 || id >= a.num_pages) return -1;
  const int row = (int)slot & ((1 << a.page_shift) - 1);
  return (int64_t)id * a.page_stride + (((int64_t)g << a.page_shift) + row) * a.row_bytes;
}

constexpr int kAppendThreads = 256;

// A thread per 16 bytes of a new row (K and V).  Memory bounds it: 32 layers x 4 x 60 rows of 32 heads, D = 128 (252 MB read and
// written) take 47-51 us from HBM, 5.0-5.4 TB/s, a large copy's rate; a few rows 2.5 us.
__global__ __launch_bounds__(kAppendThreads) void paged_append_kernel(PagedRowsArgs a) {
  const int b = blockIdx.y, layer = blockIdx.z;
  const int words = a.row_bytes / 16;
  const long long item = (long long)blockIdx.x * kAppendThreads + threadIdx.x;
  const long long rows = item / words;
  const int w = (int)(item - rows * words);
  const int g = (int)(rows % a.Hkv);
  const long long i = rows / a.Hkv;
  int n = a.N;
  if (a.row_len) n = min(a.row_len[b], n);
  if (i >= n) return;
  const int L = a.kv_len[b];
  if (L < 0) return;
  const int64_t to = slot_offset(a, a.table + (size_t)b * a.width, g, (long long)L + i);
  if (to < 0) return;
  const int64_t from = layer * a.new_layer + b * a.new_batch + g * a.new_head + i * a.new_row + w * 16;
  const u32x4 k = *(const u32x4*)(a.k_new + from), v = *(const u32x4*)(a.v_new + from);
  *(u32x4*)(a.k + layer * a.layer_stride + to + w * 16) = k;
  *(u32x4*)(a.v + layer * a.layer_stride + to + w * 16) = v;
}

// A node at depth k has k ancestors with smaller indices, so path[k] >= k: sources lie at or behind their
// destinations, and a destination can be a later row's source.  Passes over k run in increasing order, each with all of its
// rows in registers before it writes one.  Rows with path[k] == k stay.  A wave per (layer, sequence, KV head), a lane per 16
// bytes of a row; a pass has kCommitLoads times as many rows as a wave holds at once.  Latency bounds it (the lengths and
// the path, the table, the rows, one after another): waves that need no LDS and no barrier, four to a workgroup (32 layers
// x 4 sequences x 32 heads, up to 6 rows each: 7.5 us; through LDS, a workgroup a head, 12.6; one sequence's 4 heads 3.6).
constexpr int kCommitLoads = 4;

__global__ __launch_bounds__(kCommitThreads) void paged_commit_kernel(PagedRowsArgs a) {
  const int lane = threadIdx.x & 63;
  const long long n = (long long)blockIdx.x * (kCommitThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (n >= (long long)a.NL * a.B * a.Hkv) return;       // (layer * B + b) * Hkv + g
  const int g = (int)(n % a.Hkv), lb = (int)(n / a.Hkv);
  const int b = lb % a.B, layer = lb / a.B;
  const int words = a.row_bytes / 16, at_once = 64 / words;   // rows of a wave
  const int r = lane / words, w = lane - r * words;
  const int32_t* path = a.path + (size_t)b * a.path_stride;
  const int L = a.kv_len[b];
  int A = a.accept_len[b];
  A = A < 0 ? 0 : (A > a.path_stride - 1 ? a.path_stride - 1 : A);
  if (layer == 0 && g == 0 && lane == 0) a.kv_len_out[b] = L + A + 1;
  if (L < 0) return;
  char* kc = a.k + layer * a.layer_stride + w * 16;
  char* vc = a.v + layer * a.layer_stride + w * 16;
  const int32_t* table = a.table + (size_t)b * a.width;
  for (int k0 = 0; k0 <= A; k0 += kCommitLoads * at_once) {
    u32x4 kr[kCommitLoads], vr[kCommitLoads];
    int64_t to[kCommitLoads];
#pragma unroll
    for (int t = 0; t < kCommitLoads; ++t) {
      const int k = k0 + t * at_once + r;
      const int src = r < at_once && k <= A ? path[k] : 0;
      const int64_t from = src > k ? slot_offset(a, table, g, (long long)L + src) : -1;
      to[t] = from >= 0 ? slot_offset(a, table, g, (long long)L + k) : -1;
      if (to[t] >= 0) {
        kr[t] = *(const u32x4*)(kc + from);
        vr[t] = *(const u32x4*)(vc + from);
      }
    }
    wait_vector_memory();   // (every lane's rows are in registers)
#pragma unroll
    for (int t = 0; t < kCommitLoads; ++t)
      if (to[t] >= 0) {
        *(u32x4*)(kc + to[t]) = kr[t];
        *(u32x4*)(vc + to[t]) = vr[t];
      }
  }
}

}  // namespace

hipError_t launch_paged_append(const PagedRowsArgs& a, hipStream_t stream) {
  const long long items = (long long)a.N * a.Hkv * (a.row_bytes / 16);
  if (items == 0 || a.B == 0) return hipSuccess;
  const dim3 grid((unsigned)((items + kAppendThreads - 1) / kAppendThreads), (unsigned)a.B, (unsigned)a.NL);
  hipLaunchKernelGGL(paged_append_kernel, grid, dim3(kAppendThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_paged_commit(const PagedRowsArgs& a, hipStream_t stream) {
  const long long waves = (long long)a.NL * a.B * a.Hkv, grid = (waves + kCommitThreads / 64 - 1) / (kCommitThreads / 64);
  if (grid <= 0) return hipSuccess;
  hipLaunchKernelGGL(paged_commit_kernel, dim3((unsigned)grid), dim3(kCommitThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace dreams
