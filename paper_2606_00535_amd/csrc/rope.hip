// Rotary positions: queries or keys rotated by themselves, and rows rotated on their way into the pages of a cache (their
// queries in the same launch, their values copied).
//
// (x, y) -> (x cos - y sin, y cos + x sin) for the R / 2 pairs of a row, the angle position * frequency.  Every value is read and
// written once, so large calls are bound by the memory: a thread takes a unit (two 16-byte runs) of a row of a head, the heads
// of a row after one another, so that a wave's loads and stores are whole lines.  A row's angles are those of all its heads:
// a workgroup computes its rows' cosines and sines once, in LDS, while its rows are on their way (each thread for its own
// pairs: 28 heads x 8192 rows of 128 columns 27.9 us instead of 19.9).  That is 117 MB at 5.9 TB/s, where a large copy makes 5.2;
// 4 x 300 to 2049 rows of 28 query heads and 2 x 4 heads into pages 20.5 us (112 MB, 5.4 TB/s).  Small calls
// are a chain of a launch, the positions, the turns and a store: 4 sequences' tokens of 32 heads 3.0 us, 4 x 60 nodes of 3 x 32
// heads 4.9.
#include "rope.h"

namespace dreams {
namespace {

// Cosines and sines of the rows that a workgroup's items are of: k >= R / (2 W) items a row, so at most 254 / k + 2 rows of
// R / 2 <= W k.
constexpr int kTurns = 8 * kRopeThreads + kRopeMaxDim;

// What a workgroup's items are of: item = (row * heads + head) * units + unit.
struct Item {
  int row, head, unit;
  int first, rows;      // of the workgroup
};
__device__ __forceinline__ Item item_of(int units, int heads, int N) {
  const uint32_t per_row = (uint32_t)units * (uint32_t)heads, base = blockIdx.x * kRopeThreads, item = base + threadIdx.x;
  Item x;
  x.row = (int)(item / per_row);
  const uint32_t rest = item - x.row * per_row;
  x.head = (int)(rest / units);
  x.unit = (int)(rest - x.head * (uint32_t)units);
  x.first = (int)(base / per_row);
  x.rows = min((int)((base + kRopeThreads - 1) / per_row), N - 1) - x.first + 1;
  return x;
}

template <typename T, int W, bool PAST>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeCallArgs a, int units) {
  __shared__ TurnScratch scratch;
  __shared__ __attribute__((aligned(16))) float2 turns[kTurns];
  const int b = blockIdx.y;
  const Item it = item_of(units, a.H, a.N);
  const Unit u = unit_of<W>(it.unit, a.rope.R, a.D);
  const bool mine = it.row < a.N && !(a.in_place && !u.rotated);
  Run<T, W> x, y;
  if (mine) {      // (on their way while the turns are computed)
    const char* row = a.x + b * a.x_batch + it.head * a.x_head + it.row * a.x_row;
    x.load(row, u.first);
    if (u.second >= 0) y.load(row, u.second);
  }
  fill_turns<kRopeThreads>(a.rope, scratch, b, it.first, it.rows, a.N, turns);
  if (!mine) return;
  if (u.rotated) {
    float c[W], s[W];
    take_turns(turns + (it.row - it.first) * (a.rope.R / 2), it.unit, a.rope.R, a.rope.interleaved != 0, c, s);
    rotate(x, y, c, s, a.rope.interleaved != 0);
  }
  char* to = a.out + b * a.out_batch + it.head * a.out_head + it.row * a.out_row;
  x.template store<PAST>(to, u.first);
  if (u.second >= 0) y.template store<PAST>(to, u.second);
}

// Heads 0 .. Hq - 1 are the queries', then Hkv of keys, then Hkv of values.
template <typename T, int W, bool PAST>
__global__ __launch_bounds__(kRopeThreads) void paged_append_rope_kernel(PagedRowsArgs a, RopeArgs r, RopeQueryArgs q, int D,
                                                                        int units) {
  __shared__ TurnScratch scratch;
  __shared__ __attribute__((aligned(16))) float2 turns[kTurns];
  const int b = blockIdx.y, layer = blockIdx.z;
  const Item it = item_of(units, q.Hq + 2 * a.Hkv, a.N);
  const int i = it.row, h = it.head;
  int n = a.N;
  if (a.row_len) n = min(a.row_len[b], n);
  const bool mine = i < a.N, live = i < n;
  const bool query = h < q.Hq, value = h >= q.Hq + a.Hkv;
  const int g = query ? h : h - q.Hq - (value ? a.Hkv : 0);
  const Unit u = unit_of<W>(it.unit, r.R, D);
  Run<T, W> x, y;
  x.zero();
  y.zero();
  if (mine && live) {      // (on their way while the turns are computed)
    const char* from = query ? q.q + b * q.batch + g * q.head + i * q.row
                             : (value ? a.v_new : a.k_new) + layer * a.new_layer + b * a.new_batch + g * a.new_head +
                                   i * a.new_row;
    x.load(from, u.first);
    if (u.second >= 0) y.load(from, u.second);
  }
  fill_turns<kRopeThreads>(r, scratch, b, it.first, min(it.rows, n - it.first), a.N, turns);
  if (!mine) return;
  char* to;
  if (query) {
    to = q.out + (((size_t)b * q.Hq + g) * a.N + i) * a.row_bytes;
  } else {
    const long long slot = (long long)a.kv_len[b] + i;
    if (!live || slot < i || (slot >> a.page_shift) >= a.width) return;     // (a negative length: none)
    const int id = a.table[(size_t)b * a.width + (slot >> a.page_shift)];
    if (id < 0 || id >= a.num_pages) return;
    to = (value ? a.v : a.k) + layer * a.layer_stride + (int64_t)id * a.page_stride +
         (((int64_t)g << a.page_shift) + ((int)slot & ((1 << a.page_shift) - 1))) * a.row_bytes;
  }
  if (u.rotated && !value && live) {
    float c[W], s[W];
    take_turns(turns + (i - it.first) * (r.R / 2), it.unit, r.R, r.interleaved != 0, c, s);
    rotate(x, y, c, s, r.interleaved != 0);
  }
  x.template store<PAST>(to, u.first);
  if (u.second >= 0) y.template store<PAST>(to, u.second);
}

}  // namespace

hipError_t launch_rope(const RopeCallArgs& a, hipStream_t stream) {
  const int units = a.elem == 2 ? rope_units<8>(a.rope.R, a.D) : rope_units<4>(a.rope.R, a.D);
  const long long items = (long long)a.N * units * a.H;
  if (items == 0 || a.B == 0) return hipSuccess;
  const dim3 grid((unsigned)((items + kRopeThreads - 1) / kRopeThreads), (unsigned)a.B);
  const bool past = stored_past((long long)a.B * a.H * a.N * a.D * a.elem, a.rope.R, a.D, a.elem);
  auto kern = a.elem == 2 ? (past ? rope_kernel<__bf16, 8, true> : rope_kernel<__bf16, 8, false>)
                          : (past ? rope_kernel<float, 4, true> : rope_kernel<float, 4, false>);
  hipLaunchKernelGGL(kern, grid, dim3(kRopeThreads), 0, stream, a, units);
  return hipGetLastError();
}

hipError_t launch_paged_append_rope(const PagedRowsArgs& a, const RopeArgs& rope, const RopeQueryArgs& q, int elem, int D,
                                    hipStream_t stream) {
  const int units = elem == 2 ? rope_units<8>(rope.R, D) : rope_units<4>(rope.R, D);
  const long long heads = q.Hq + 2LL * a.Hkv, items = (long long)a.N * units * heads;
  if (items == 0 || a.B == 0) return hipSuccess;
  const dim3 grid((unsigned)((items + kRopeThreads - 1) / kRopeThreads), (unsigned)a.B, (unsigned)a.NL);
  const bool past = stored_past(a.NL * a.B * heads * a.N * a.row_bytes, rope.R, D, elem);
  auto kern = elem == 2 ? (past ? paged_append_rope_kernel<__bf16, 8, true> : paged_append_rope_kernel<__bf16, 8, false>)
                        : (past ? paged_append_rope_kernel<float, 4, true> : paged_append_rope_kernel<float, 4, false>);
  hipLaunchKernelGGL(kern, grid, dim3(kRopeThreads), 0, stream, a, rope, q, D, units);
  return hipGetLastError();
}

}  // namespace dreams
