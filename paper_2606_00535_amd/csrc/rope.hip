// Rotary positions: queries or keys rotated by themselves, and rows rotated on their way into the pages of a cache (their
// queries in the same launch, their values copied).
//
// A thread takes a unit of 8 pairs (16 columns) of a row for `per_thread` heads, whose cosines and sines are the same: it
// computes them once.
#include "rope.h"

namespace dreams {
namespace {

// A row's position, by a table, by a tree (parents in LDS) or in order.
__device__ __forceinline__ double position_of(const RopeArgs& r, const int* parents, int b, int i, int N) {
  if (r.positions) return (double)r.positions[(size_t)b * N + i];
  const int base = r.kv_len ? r.kv_len[b] : 0;
  return (double)base + (double)(r.parent ? depth_of(parents, i) : i);
}
__device__ __forceinline__ void load_parents(const RopeArgs& r, int* parents, int b, int N) {
  if (!r.parent || r.positions) return;
  for (int i = threadIdx.x; i < N; i += kRopeThreads) parents[i] = r.parent[(size_t)b * N + i];
  __syncthreads();
}
__device__ __forceinline__ void cos_sin(const RopeArgs& r, double position, int p, float (&c)[8], float (&s)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) turn(position, r.freq[8 * p + i], r.gain, &c[i], &s[i]);
}

template <typename T>
__device__ __forceinline__ void rotate(Run<T>& x, Run<T>& y, const float (&c)[8], const float (&s)[8], bool interleaved) {
  float a[8], b[8];
  x.get(a);
  y.get(b);
  rotate(a, b, c, s, interleaved);
  x.set(a);
  y.set(b);
}

template <typename T>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeCallArgs a, int units, int groups) {
  __shared__ int parents[kMaxNodes];
  const int b = blockIdx.y;
  load_parents(a.rope, parents, b, a.N);
  const uint32_t item = blockIdx.x * kRopeThreads + threadIdx.x, rest = item / units;
  const int p = (int)(item - rest * units), i = (int)(rest / groups), group = (int)(rest - i * (uint32_t)groups);
  if (i >= a.N) return;
  const Unit u = unit_of(p, a.rope.R, a.D, a.rope.interleaved != 0);
  if (!u.rotated && a.in_place) return;
  float c[8], s[8];
  if (u.rotated) cos_sin(a.rope, position_of(a.rope, parents, b, i, a.N), p, c, s);
  for (int h = group; h < a.H; h += groups) {
    const char* row = a.x + b * a.x_batch + h * a.x_head + i * a.x_row;
    char* to = a.out + b * a.out_batch + h * a.out_head + i * a.out_row;
    Run<T> x, y;
    x.load(row, u.first);
    if (u.second >= 0) y.load(row, u.second);
    if (u.rotated) rotate(x, y, c, s, a.rope.interleaved != 0);
    x.store(to, u.first);
    if (u.second >= 0) y.store(to, u.second);
  }
}

// Heads 0 .. Hq - 1 are the queries', then Hkv of keys, then Hkv of values.
template <typename T>
__global__ __launch_bounds__(kRopeThreads) void paged_append_rope_kernel(PagedRowsArgs a, RopeArgs r, RopeQueryArgs q, int D,
                                                                        int units, int groups) {
  __shared__ int parents[kMaxNodes];
  const int b = blockIdx.y, layer = blockIdx.z;
  load_parents(r, parents, b, a.N);
  const uint32_t item = blockIdx.x * kRopeThreads + threadIdx.x, rest = item / units;
  const int p = (int)(item - rest * units), i = (int)(rest / groups), group = (int)(rest - i * (uint32_t)groups);
  if (i >= a.N) return;
  int n = a.N;
  if (a.row_len) n = min(a.row_len[b], n);
  const bool live = i < n;
  const int L = a.kv_len[b];
  // the row's slot
  int64_t to = -1;
  const long long slot = (long long)L + i;
  if (live && L >= 0 && (slot >> a.page_shift) < a.width) {
    const int id = a.table[(size_t)b * a.width + (slot >> a.page_shift)];
    if (id >= 0 && id < a.num_pages)
      to = layer * a.layer_stride + (int64_t)id * a.page_stride +
           (int64_t)((int)slot & ((1 << a.page_shift) - 1)) * a.row_bytes;
  }
  const Unit u = unit_of(p, r.R, D, r.interleaved != 0);
  float c[8], s[8];
  if (u.rotated && live) cos_sin(r, position_of(r, parents, b, i, a.N), p, c, s);
  const int heads = q.Hq + 2 * a.Hkv;
  for (int h = group; h < heads; h += groups) {
    const bool query = h < q.Hq, value = h >= q.Hq + a.Hkv;
    const int g = query ? h : (h - q.Hq) % a.Hkv;
    Run<T> x, y;
    if (!live) {
      x.zero();
      y.zero();
    } else {
      const char* from = query ? q.q + b * q.batch + g * q.head + i * q.row
                               : (value ? a.v_new : a.k_new) + layer * a.new_layer + b * a.new_batch + g * a.new_head +
                                     i * a.new_row;
      x.load(from, u.first);
      if (u.second >= 0) y.load(from, u.second);
      if (u.rotated && !value) rotate(x, y, c, s, r.interleaved != 0);
    }
    char* row;
    if (query) {
      row = q.out + (((size_t)b * q.Hq + g) * a.N + i) * a.row_bytes;
    } else {
      if (to < 0) continue;
      row = (value ? a.v : a.k) + to + ((int64_t)g << a.page_shift) * a.row_bytes;
    }
    x.store(row, u.first);
    if (u.second >= 0) y.store(row, u.second);
  }
}

}  // namespace

hipError_t launch_rope(const RopeCallArgs& a, hipStream_t stream) {
  const int units = rope_units(a.rope.R, a.D), per_thread = 1;
  const int groups = (a.H + per_thread - 1) / per_thread;
  const long long items = (long long)a.N * units * groups;
  if (items == 0 || a.B == 0) return hipSuccess;
  const dim3 grid((unsigned)((items + kRopeThreads - 1) / kRopeThreads), (unsigned)a.B);
  if (a.elem == 2) hipLaunchKernelGGL(rope_kernel<__bf16>, grid, dim3(kRopeThreads), 0, stream, a, units, groups);
  else hipLaunchKernelGGL(rope_kernel<float>, grid, dim3(kRopeThreads), 0, stream, a, units, groups);
  return hipGetLastError();
}

hipError_t launch_paged_append_rope(const PagedRowsArgs& a, const RopeArgs& rope, const RopeQueryArgs& q, int elem, int D,
                                    hipStream_t stream) {
  const int units = rope_units(rope.R, D), per_thread = 1, heads = q.Hq + 2 * a.Hkv;
  const int groups = (heads + per_thread - 1) / per_thread;
  const long long items = (long long)a.N * units * groups;
  if (items == 0 || a.B == 0) return hipSuccess;
  const dim3 grid((unsigned)((items + kRopeThreads - 1) / kRopeThreads), (unsigned)a.B, (unsigned)a.NL);
  if (elem == 2)
    hipLaunchKernelGGL(paged_append_rope_kernel<__bf16>, grid, dim3(kRopeThreads), 0, stream, a, rope, q, D, units, groups);
  else
    hipLaunchKernelGGL(paged_append_rope_kernel<float>, grid, dim3(kRopeThreads), 0, stream, a, rope, q, D, units, groups);
  return hipGetLastError();
}

}  // namespace dreams
