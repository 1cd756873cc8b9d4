// Rows of a paged cache in 8 bits: codes of e4m3 and a power-of-two scale for every 16 slots of a head (PagedScaleArgs).
//
//   * append: a wave per block of 16 slots, head, and K or V.  It holds the block's new rows in fp32 (rotated, for K), takes
//     their largest magnitude across its lanes, hence the scale, and writes their codes.  Rows that the block holds
//     already move to the new scale where it is larger than theirs.
//   * commit: a wave per (layer, sequence, KV head) and K or V, which goes through the path's blocks in order: a block's rows are
//     in registers before one is written.  As in the 16-bit cache a row's source lies at or behind its slot, so that no
//     block's rows or scale are changed before they are read.
//   * read: a thread per 16 codes.
// A code times a power of two is exact in bf16, and a scale that grows moves a code's exponent: only codes that fall below
// e4m3's normal range are rounded again.
#include "rope.h"

namespace dreams {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;

// 2^(byte - 127) of bytes 1 .. 254
__device__ __forceinline__ float power(int byte) { return __builtin_bit_cast(float, (uint32_t)byte << 23); }

// The least scale byte at which magnitudes up to that of these bits (fp32, finite) are at most 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_byte(uint32_t magnitude) {
  const int at = (int)(magnitude >> 23) - 8 + ((magnitude & 0x7fffffu) > 0x600000u ? 1 : 0);
  return at < 1 ? 1 : at;
}
__device__ __forceinline__ uint32_t finite_magnitude(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
}
// 4 values (at most 448 in magnitude, or not finite) to 4 codes, to the nearest, ties to even
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
// 4 codes times 2^(by - 127) (by >= 1), as codes again
__device__ __forceinline__ uint32_t rescale4(uint32_t codes, float by) {
  const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, by, false);
  const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, by, true);
  return encode4((float)lo[0], (float)lo[1], (float)hi[0], (float)hi[1]);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t y = (uint32_t)__shfl_xor((int)x, off);
    x = x > y ? x : y;
  }
  return x;
}
// A factor that moves codes from scale byte `from` to `to` >= from: below 2^-126 every code becomes 0 with 2^-126 too.
__device__ __forceinline__ float move_by(int from, int to) {
  const int by = 127 + from - to;
  return power(by < 1 ? 1 : by);
}

// A slot's page, or -1: past the table, or outside the pool.
__device__ __forceinline__ int page_of(const PagedRowsArgs& a, const int32_t* table, long long slot) {
  if (slot < 0 || (slot >> a.page_shift) >= a.width) return -1;
  const int id = table[slot >> a.page_shift];
  return id < 0 || id >= a.num_pages ? -1 : id;
}

// A block's row r (16) and unit of 16 columns of a lane, pass by pass: 64 / units rows a pass.
template <typename T, int PASSES>
__global__ __launch_bounds__(kThreads) void paged_append_e4m3_kernel(PagedRowsArgs a, PagedScaleArgs sc, RopeArgs r,
                                                                    RopeQueryArgs q, int D, int units, int blocks,
                                                                    unsigned query_groups) {
  __shared__ int parents[kMaxNodes];
  const int b = blockIdx.y, layer = blockIdx.z, tid = threadIdx.x;
  if (r.parent && !r.positions) {
    for (int i = tid; i < a.N; i += kThreads) parents[i] = r.parent[(size_t)b * a.N + i];
    __syncthreads();
  }
  int n = a.N;
  if (a.row_len) n = min(a.row_len[b], n);
  const int L = a.kv_len[b];
  auto position = [&](int i) {
    if (r.positions) return (double)r.positions[(size_t)b * a.N + i];
    return (double)L + (double)(r.parent ? depth_of(parents, i) : i);
  };
  if (blockIdx.x < query_groups) {   // the queries: a thread per unit of a row
    const uint32_t item = blockIdx.x * kThreads + tid, rest = item / units;
    const int p = (int)(item - rest * units), i = (int)(rest / q.Hq), h = (int)(rest - i * (uint32_t)q.Hq);
    if (i >= a.N) return;
    const Unit u = unit_of(p, r.R, D, r.interleaved != 0);
    Run<T> x, y;
    x.zero();
    y.zero();
    if (i < n) {
      const char* from = q.q + b * q.batch + h * q.head + i * q.row;
      x.load(from, u.first);
      y.load(from, u.second);
      if (u.rotated) {
        float c[8], s[8], xf[8], yf[8];
        const double at = position(i);
#pragma unroll
        for (int e = 0; e < 8; ++e) turn(at, r.freq[8 * p + e], r.gain, &c[e], &s[e]);
        x.get(xf);
        y.get(yf);
        rotate(xf, yf, c, s, r.interleaved != 0);
        x.set(xf);
        y.set(yf);
      }
    }
    char* to = q.out + (((size_t)b * q.Hq + h) * a.N + i) * (size_t)(D * sizeof(T));
    x.store(to, u.first);
    y.store(to, u.second);
    return;
  }
  const int lane = tid & 63;
  const uint32_t task = (blockIdx.x - query_groups) * (kThreads / 64) + __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = (int)(task & 1), g = (int)((task >> 1) % (uint32_t)a.Hkv), m = (int)((task >> 1) / (uint32_t)a.Hkv);
  if (m >= blocks || L < 0 || n <= 0) return;
  const long long slot0 = ((long long)L / kScaleBlock + m) * kScaleBlock;    // the block's first slot
  const int i0 = (int)(slot0 - L);                                           // its row of the new ones (may be < 0)
  if (i0 >= n) return;
  const int id = page_of(a, a.table + (size_t)b * a.width, slot0);
  if (id < 0) return;
  const int in_page = (int)slot0 & ((1 << a.page_shift) - 1);
  char* codes = (half ? a.v : a.k) + layer * a.layer_stride + (int64_t)id * a.page_stride +
                (((int64_t)g << a.page_shift) + in_page) * a.row_bytes;
  uint8_t* scale = (half ? sc.v : sc.k) + layer * sc.layer_stride + (int64_t)id * sc.page_stride +
                   (((int64_t)g << a.page_shift) + in_page) / kScaleBlock;
  const char* rows = (half ? a.v_new : a.k_new) + layer * a.new_layer + b * a.new_batch + g * a.new_head;
  const int held = i0 < 0 ? *scale : 0;
  const int per_pass = 64 / units, sub = lane / units, p = lane - sub * units;
  const Unit u = unit_of(p, r.R, D, r.interleaved != 0);
  float x[PASSES][8], y[PASSES][8];
  uint32_t top = 0;
#pragma unroll
  for (int t = 0; t < PASSES; ++t) {
    const int row = t * per_pass + sub, i = i0 + row;
    if (sub < per_pass && row < kScaleBlock && i >= 0 && i < n) {
      Run<T> lo, hi;
      lo.load(rows + i * a.new_row, u.first);
      hi.load(rows + i * a.new_row, u.second);
      lo.get(x[t]);
      hi.get(y[t]);
      if (u.rotated && half == 0) {
        float c[8], s[8];
        const double at = position(i);
#pragma unroll
        for (int e = 0; e < 8; ++e) turn(at, r.freq[8 * p + e], r.gain, &c[e], &s[e]);
        rotate(x[t], y[t], c, s, r.interleaved != 0);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t ux = finite_magnitude(x[t][e]), uy = finite_magnitude(y[t][e]);
        top = top > ux ? top : ux;
        top = top > uy ? top : uy;
      }
    }
  }
  const int mine = scale_byte(wave_max(top)), byte = mine > held ? mine : held;
  const float inverse = power(254 - byte);
#pragma unroll
  for (int t = 0; t < PASSES; ++t) {
    const int row = t * per_pass + sub, i = i0 + row;
    if (sub >= per_pass || row >= kScaleBlock) continue;
    uint32_t* lo = (uint32_t*)(codes + (int64_t)row * a.row_bytes + u.first);
    uint32_t* hi = (uint32_t*)(codes + (int64_t)row * a.row_bytes + u.second);
    if (i >= 0 && i < n) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        lo[e] = encode4(x[t][4 * e] * inverse, x[t][4 * e + 1] * inverse, x[t][4 * e + 2] * inverse, x[t][4 * e + 3] * inverse);
        hi[e] = encode4(y[t][4 * e] * inverse, y[t][4 * e + 1] * inverse, y[t][4 * e + 2] * inverse, y[t][4 * e + 3] * inverse);
      }
    } else if (i < 0 && byte > held) {
      const float by = move_by(held, byte);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        lo[e] = rescale4(lo[e], by);
        hi[e] = rescale4(hi[e], by);
      }
    }
  }
  if (lane == 0) *scale = (uint8_t)byte;
}

template <int PASSES>
__global__ __launch_bounds__(kThreads) void paged_commit_e4m3_kernel(PagedRowsArgs a, PagedScaleArgs sc, int units) {
  const int lane = threadIdx.x & 63;
  const long long task = (long long)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (task >= 2LL * a.NL * a.B * a.Hkv) return;
  const int half = (int)(task & 1), g = (int)((task >> 1) % a.Hkv), lb = (int)((task >> 1) / a.Hkv);
  const int b = lb % a.B, layer = lb / a.B;
  const int32_t* path = a.path + (size_t)b * a.path_stride;
  const int32_t* table = a.table + (size_t)b * a.width;
  const int L = a.kv_len[b];
  int A = a.accept_len[b];
  A = A < 0 ? 0 : (A > a.path_stride - 1 ? a.path_stride - 1 : A);
  if (layer == 0 && g == 0 && half == 0 && lane == 0) a.kv_len_out[b] = L + A + 1;
  if (L < 0) return;
  char* codes = (half ? a.v : a.k) + layer * a.layer_stride;
  uint8_t* scales = (half ? sc.v : sc.k) + layer * sc.layer_stride;
  const int per_pass = 64 / units, sub = lane / units, p = lane - sub * units;
  auto head_slot = [&](long long slot) { return ((int64_t)g << a.page_shift) + ((int)slot & ((1 << a.page_shift) - 1)); };
  for (long long slot0 = (long long)L / kScaleBlock * kScaleBlock; slot0 <= (long long)L + A; slot0 += kScaleBlock) {
    const int id = page_of(a, table, slot0);
    if (id < 0) continue;
    uint8_t* scale = scales + (int64_t)id * sc.page_stride + head_slot(slot0) / kScaleBlock;
    const int old = *scale;
    u32x4 x[PASSES];
    int from[PASSES];      // the scale byte of a live row (-1: dead)
    uint32_t moved = 0;    // a bit a pass
    int top = 0;
#pragma unroll
    for (int t = 0; t < PASSES; ++t) {
      const int row = t * per_pass + sub;
      const long long slot = slot0 + row;
      const int k = (int)(slot - L);     // < 0: before the rows
      from[t] = -1;
      if (sub >= per_pass || row >= kScaleBlock || k > A) continue;
      int64_t at = (int64_t)id * a.page_stride + head_slot(slot) * a.row_bytes;
      from[t] = old;
      if (k >= 0 && path[k] > k) {
        const long long src = (long long)L + path[k];
        const int src_id = page_of(a, table, src);
        if (src_id >= 0) {
          at = (int64_t)src_id * a.page_stride + head_slot(src) * a.row_bytes;
          from[t] = scales[(int64_t)src_id * sc.page_stride + head_slot(src) / kScaleBlock];
          moved |= 1u << t;
        }
      }
      x[t] = *(const u32x4*)(codes + at + p * 16);
      top = top > from[t] ? top : from[t];
    }
    const int byte = (int)wave_max((uint32_t)top);
    if (!__any(moved != 0)) continue;    // (the block's rows stay where they are)
    wait_vector_memory();                // (every lane's rows are in registers)
#pragma unroll
    for (int t = 0; t < PASSES; ++t) {
      const int row = t * per_pass + sub;
      if (from[t] < 0 || !((moved >> t & 1u) || from[t] != byte)) continue;
      const float by = move_by(from[t], byte);
      u32x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = from[t] == byte ? x[t][e] : rescale4(x[t][e], by);
      *(u32x4*)(codes + (int64_t)id * a.page_stride + head_slot(slot0 + row) * a.row_bytes + p * 16) = y;
    }
    if (lane == 0) *scale = (uint8_t)byte;
    wait_vector_memory();
  }
}

__global__ __launch_bounds__(kThreads) void paged_read_e4m3_kernel(PagedRowsArgs a, PagedScaleArgs sc, int num_slots,
                                                                  char* k_out, char* v_out, int units) {
  const int layer = blockIdx.z, bg = blockIdx.y, b = bg / a.Hkv, g = bg - b * a.Hkv;
  const uint32_t item = blockIdx.x * kThreads + threadIdx.x;
  const int slot = (int)(item / units), p = (int)(item - slot * (uint32_t)units);
  if (slot >= num_slots) return;
  int id = -1;
  if (slot < a.kv_len[b]) id = page_of(a, a.table + (size_t)b * a.width, slot);
  const int64_t in_head = ((int64_t)g << a.page_shift) + (slot & ((1 << a.page_shift) - 1));
  const size_t to = (((size_t)layer * a.B * a.Hkv + bg) * num_slots + slot) * a.row_bytes * 2 + p * 32;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    u32x4 lo{0u, 0u, 0u, 0u}, hi{0u, 0u, 0u, 0u};
    if (id >= 0) {
      const u32x4 x = *(const u32x4*)((half ? a.v : a.k) + layer * a.layer_stride + (int64_t)id * a.page_stride +
                                      in_head * a.row_bytes + p * 16);
      const float by = power((half ? sc.v : sc.k)[layer * sc.layer_stride + (int64_t)id * sc.page_stride +
                                                  in_head / kScaleBlock]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t y0 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[e], by, false));
        const uint32_t y1 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[e], by, true));
        (e < 2 ? lo : hi)[2 * (e & 1)] = y0;
        (e < 2 ? lo : hi)[2 * (e & 1) + 1] = y1;
      }
    }
    char* row = (half ? v_out : k_out) + to;
    *(u32x4*)row = lo;
    *(u32x4*)(row + 16) = hi;
  }
}

template <typename T, int PASSES>
void append(const PagedRowsArgs& a, const PagedScaleArgs& sc, const RopeArgs& rope, const RopeQueryArgs& q, dim3 grid,
            int units, int blocks, unsigned query_groups, hipStream_t stream) {
  hipLaunchKernelGGL((paged_append_e4m3_kernel<T, PASSES>), grid, dim3(kThreads), 0, stream, a, sc, rope, q, a.row_bytes, units,
                     blocks, query_groups);
}
template <typename T>
void append_passes(int passes, const PagedRowsArgs& a, const PagedScaleArgs& sc, const RopeArgs& rope, const RopeQueryArgs& q,
                   dim3 grid, int units, int blocks, unsigned query_groups, hipStream_t stream) {
  if (passes <= 1) append<T, 1>(a, sc, rope, q, grid, units, blocks, query_groups, stream);
  else if (passes <= 2) append<T, 2>(a, sc, rope, q, grid, units, blocks, query_groups, stream);
  else if (passes <= 4) append<T, 4>(a, sc, rope, q, grid, units, blocks, query_groups, stream);
  else append<T, 8>(a, sc, rope, q, grid, units, blocks, query_groups, stream);
}

// passes over a block's 16 rows of `units` lanes each (units <= 32: 8 at most)
int passes_of(int units) { return (kScaleBlock + 64 / units - 1) / (64 / units); }

}  // namespace

hipError_t launch_paged_append_e4m3(const PagedRowsArgs& a, const PagedScaleArgs& sc, const RopeArgs& rope,
                                    const RopeQueryArgs& q, int elem, hipStream_t stream) {
  if (a.N == 0 || a.B == 0) return hipSuccess;
  const int units = a.row_bytes / 16, blocks = (int)(((long long)a.N + 2 * kScaleBlock - 2) / kScaleBlock);
  const long long waves = 2LL * blocks * a.Hkv, per = kThreads / 64;
  const unsigned query_groups = (unsigned)(((long long)a.N * q.Hq * units + kThreads - 1) / kThreads);
  const dim3 grid(query_groups + (unsigned)((waves + per - 1) / per), (unsigned)a.B, (unsigned)a.NL);
  const int passes = passes_of(units);
  if (elem == 2) append_passes<__bf16>(passes, a, sc, rope, q, grid, units, blocks, query_groups, stream);
  else append_passes<float>(passes, a, sc, rope, q, grid, units, blocks, query_groups, stream);
  return hipGetLastError();
}

hipError_t launch_paged_commit_e4m3(const PagedRowsArgs& a, const PagedScaleArgs& sc, hipStream_t stream) {
  const long long waves = 2LL * a.NL * a.B * a.Hkv, per = kThreads / 64;
  if (waves == 0) return hipSuccess;
  const dim3 grid((unsigned)((waves + per - 1) / per));
  const int units = a.row_bytes / 16, passes = passes_of(units);
  if (passes <= 1) hipLaunchKernelGGL(paged_commit_e4m3_kernel<1>, grid, dim3(kThreads), 0, stream, a, sc, units);
  else if (passes <= 2) hipLaunchKernelGGL(paged_commit_e4m3_kernel<2>, grid, dim3(kThreads), 0, stream, a, sc, units);
  else if (passes <= 4) hipLaunchKernelGGL(paged_commit_e4m3_kernel<4>, grid, dim3(kThreads), 0, stream, a, sc, units);
  else hipLaunchKernelGGL(paged_commit_e4m3_kernel<8>, grid, dim3(kThreads), 0, stream, a, sc, units);
  return hipGetLastError();
}

hipError_t launch_paged_read_e4m3(const PagedRowsArgs& a, const PagedScaleArgs& sc, int num_slots, char* k_out, char* v_out,
                                  hipStream_t stream) {
  const int units = a.row_bytes / 16;
  const long long items = (long long)num_slots * units;
  if (items == 0 || a.B == 0) return hipSuccess;
  const dim3 grid((unsigned)((items + kThreads - 1) / kThreads), (unsigned)(a.B * a.Hkv), (unsigned)a.NL);
  hipLaunchKernelGGL(paged_read_e4m3_kernel, grid, dim3(kThreads), 0, stream, a, sc, num_slots, k_out, v_out, units);
  return hipGetLastError();
}

}  // namespace dreams
