// Rows of a paged cache in 8 bits: codes of e4m3 and a power-of-two scale for every 16 slots of a head (PagedScaleArgs).
//
//   * append: a wave per block of 16 slots, head, and K or V.  It holds the block's new rows in fp32 (rotated, for K), takes
//     their largest magnitude across its lanes, hence the scale, and writes their codes.  Rows that the block holds
//     already move to the new scale where it is larger than theirs.
//   * commit: a wave per (layer, sequence, KV head) and K or V, which goes through the path's blocks in order, two at a time:
//     their rows are in registers before one is written.  As in the 16-bit cache a row's source lies at or behind its slot, so that no
//     block's rows or scale are changed before they are read.
//   * read: a thread per 8 codes.
// A value x becomes the code nearest to x 2^(127 - s), where s is the least byte at which the block's largest magnitude is at
// most 448 2^(s - 127); the byte follows from that magnitude's bits.  A code times a power of two is exact in bf16, and a scale
// that grows moves a code's exponent: only codes that fall below e4m3's normal range are rounded again.  A scale for 16 slots
// makes the wave's own lanes enough to find it, and a block's rows lie in one page.
// What bounds them: append, the memory and the chain of load, wave maximum and store (32 heads x 3136 rows with their queries,
// 128 MB, 29.4 us, 4.4 TB/s; without the queries 20.8, unrotated 17.5; 8 x 60 nodes of 8 heads 7.5).  Commit, the chain of path,
// table, rows (8 sequences 4.7).  Read, the memory (32 x 3136 slots, 77 MB, 13.9 us, 5.5 TB/s).
#include "rope.h"

#include <algorithm>

namespace dreams {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kMaxTurns = 4 * kScaleBlock * (kRopeMaxDim / 2);   // of the keys of 4 blocks (the queries': fewer)

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

// Workgroups: query_groups of the queries (a thread per unit of a row), then key_groups of the keys' waves and as many of the
// values', in the order (block of the sequence, head): the waves of a group are of one block, or of neighbouring ones.  The
// rows' cosines and sines are computed once a group, in LDS.  A lane holds row t * (64 / units) + lane / units of its wave's
// block in pass t.  Dynamic LDS: the turns.
template <typename T, int PASSES>
__global__ __launch_bounds__(kThreads) void paged_append_e4m3_kernel(PagedRowsArgs a, PagedScaleArgs sc, RopeArgs r,
                                                                    RopeQueryArgs q, int D, int units, int blocks,
                                                                    unsigned query_groups, unsigned key_groups, bool past) {
  extern __shared__ __attribute__((aligned(16))) float2 turns[];
  __shared__ TurnScratch scratch;
  const int b = blockIdx.y, layer = blockIdx.z, tid = threadIdx.x;
  int n = a.N;
  if (a.row_len) n = min(a.row_len[b], n);
  if (blockIdx.x < query_groups) {
    const uint32_t per_row = (uint32_t)units * (uint32_t)q.Hq, base = blockIdx.x * kThreads, item = base + tid;
    const int i = (int)(item / per_row), first = (int)(base / per_row);
    const int rows = min((int)((base + kThreads - 1) / per_row) + 1, n) - first;
    const uint32_t rest = item - i * per_row;
    const int h = (int)(rest / units), p = (int)(rest - h * (uint32_t)units);
    const Unit u = unit_of<8>(p, r.R, D);
    Run<T, 8> x, y;
    x.zero();
    y.zero();
    if (i < n) {
      const char* from = q.q + b * q.batch + h * q.head + i * q.row;
      x.load(from, u.first);
      if (u.second >= 0) y.load(from, u.second);
    }
    fill_turns<kThreads>(r, scratch, b, first, rows, a.N, turns);
    if (i >= a.N) return;
    if (u.rotated && i < n) {
      float c[8], s[8];
      take_turns(turns + (i - first) * (r.R / 2), p, r.R, r.interleaved != 0, c, s);
      rotate(x, y, c, s, r.interleaved != 0);
    }
    char* to = q.out + (((size_t)b * q.Hq + h) * a.N + i) * (size_t)(D * sizeof(T));
    if (past) {
      x.template store<true>(to, u.first);
      y.template store<true>(to, u.second);
    } else {
      x.store(to, u.first);
      y.store(to, u.second);
    }
    return;
  }
  const int lane = tid & 63;
  unsigned group = blockIdx.x - query_groups;
  const int half = group >= key_groups ? 1 : 0;
  group -= half * key_groups;
  const uint32_t task0 = group * (kThreads / 64), task = task0 + __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m = (int)(task / (uint32_t)a.Hkv), g = (int)(task - m * (uint32_t)a.Hkv), m0 = (int)(task0 / (uint32_t)a.Hkv);
  const int L = a.kv_len[b];
  if (L < 0 || n <= 0) return;
  const long long slot0 = ((long long)L / kScaleBlock + m) * kScaleBlock;    // the block's first slot
  const int i0 = (int)(slot0 - L);                                           // its row of the new ones (may be < 0)
  const bool mine = m < blocks && i0 < n;
  const int per_pass = 64 / units, sub = lane / units, p = lane - sub * units;
  Unit u = unit_of<8>(p, r.R, D);
  if (half) u = Unit{16 * p, 16 * p + 8, false};     // (a unit of values: 16 columns in a row)
  // the rows (fresh: a pass's row of this lane is a new one), on their way while the turns are computed
  Run<T, 8> lo[PASSES], hi[PASSES];
  uint32_t fresh = 0;
  if (mine) {
    const char* rows = (half ? a.v_new : a.k_new) + layer * a.new_layer + b * a.new_batch + g * a.new_head;
#pragma unroll
    for (int t = 0; t < PASSES; ++t) {
      const int row = t * per_pass + sub, i = i0 + row;
      if (sub < per_pass && row < kScaleBlock && i >= 0 && i < n) {
        // (rows of two words a run are read in halves of lines, so through the caches)
        lo[t].template load<sizeof(T) == 2>(rows + i * a.new_row, u.first);
        hi[t].template load<sizeof(T) == 2>(rows + i * a.new_row, u.second);
        fresh |= 1u << t;
      }
    }
  }
  const int id = mine ? page_of(a, a.table + (size_t)b * a.width, slot0) : -1;
  const int first = i0 - (m - m0) * kScaleBlock;     // the row that the turns start with
  if (r.freq && half == 0) {
    const int last = (int)((task0 + kThreads / 64 - 1) / (uint32_t)a.Hkv);
    fill_turns<kThreads>(r, scratch, b, first, min((last - m0 + 1) * kScaleBlock, n - first), a.N, turns);
  }
  if (id < 0) return;
  const int in_page = (int)slot0 & ((1 << a.page_shift) - 1);
  char* codes = (half ? a.v : a.k) + layer * a.layer_stride + (int64_t)id * a.page_stride +
                (((int64_t)g << a.page_shift) + in_page) * a.row_bytes;
  uint8_t* scale = (half ? sc.v : sc.k) + layer * sc.layer_stride + (int64_t)id * sc.page_stride +
                   (((int64_t)g << a.page_shift) + in_page) / kScaleBlock;
  const int held = i0 < 0 ? *scale : 0;
  float x[PASSES][8], y[PASSES][8];
  uint32_t top = 0;
#pragma unroll
  for (int t = 0; t < PASSES; ++t) {
    if (!(fresh >> t & 1u)) continue;
    lo[t].get(x[t]);
    hi[t].get(y[t]);
    if (u.rotated) {
      float c[8], s[8];
      take_turns(turns + (i0 + t * per_pass + sub - first) * (r.R / 2), p, r.R, r.interleaved != 0, c, s);
      rotate(x[t], y[t], c, s, r.interleaved != 0);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t ux = finite_magnitude(x[t][e]), uy = finite_magnitude(y[t][e]);
      top = top > ux ? top : ux;
      top = top > uy ? top : uy;
    }
  }
  const int wanted = scale_byte(wave_max(top)), byte = wanted > held ? wanted : held;
  const float inverse = power(254 - byte);
#pragma unroll
  for (int t = 0; t < PASSES; ++t) {
    const int row = t * per_pass + sub;
    if (sub >= per_pass || row >= kScaleBlock) continue;
    u32x2* to = (u32x2*)(codes + (int64_t)row * a.row_bytes + u.first);
    u32x2* to2 = (u32x2*)(codes + (int64_t)row * a.row_bytes + u.second);
    u32x2 w, w2;
    if (fresh >> t & 1u) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        w[e] = encode4(x[t][4 * e] * inverse, x[t][4 * e + 1] * inverse, x[t][4 * e + 2] * inverse, x[t][4 * e + 3] * inverse);
        w2[e] = encode4(y[t][4 * e] * inverse, y[t][4 * e + 1] * inverse, y[t][4 * e + 2] * inverse, y[t][4 * e + 3] * inverse);
      }
    } else if (i0 + row < 0 && byte > held) {
      const float by = move_by(held, byte);
      w = *to;
      w2 = *to2;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        w[e] = rescale4(w[e], by);
        w2[e] = rescale4(w2[e], by);
      }
    } else {
      continue;
    }
    if (half == 1) {
      *(u32x4*)to = u32x4{w[0], w[1], w2[0], w2[1]};
    } else {
      *to = w;
      *to2 = w2;
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
  // (two blocks at a time: a path seldom reaches into a third)
  constexpr int BLOCKS = 2;
  for (long long base = (long long)L / kScaleBlock * kScaleBlock; base <= (long long)L + A; base += BLOCKS * kScaleBlock) {
    u32x4 x[BLOCKS][PASSES];
    int from[BLOCKS][PASSES];      // the scale byte of a live row (-1: dead)
    uint32_t moved[BLOCKS] = {};   // a bit a pass
    int id[BLOCKS], top[BLOCKS] = {};
#pragma unroll
    for (int j = 0; j < BLOCKS; ++j) {
      const long long slot0 = base + j * kScaleBlock;
      id[j] = slot0 <= (long long)L + A ? page_of(a, table, slot0) : -1;
#pragma unroll
      for (int t = 0; t < PASSES; ++t) {
        const int row = t * per_pass + sub;
        const long long slot = slot0 + row;
        const int k = (int)(slot - L);     // < 0: before the rows
        from[j][t] = -1;
        if (id[j] < 0 || sub >= per_pass || row >= kScaleBlock || k > A) continue;
        int src_id = id[j];
        long long src = slot;
        if (k >= 0 && path[k] > k) {
          const int there = page_of(a, table, (long long)L + path[k]);
          if (there >= 0) {
            src_id = there;
            src = (long long)L + path[k];
            moved[j] |= 1u << t;
          }
        }
        from[j][t] = scales[(int64_t)src_id * sc.page_stride + head_slot(src) / kScaleBlock];
        x[j][t] = *(const u32x4*)(codes + (int64_t)src_id * a.page_stride + head_slot(src) * a.row_bytes + p * 16);
      }
    }
#pragma unroll
    for (int j = 0; j < BLOCKS; ++j) {
#pragma unroll
      for (int t = 0; t < PASSES; ++t) top[j] = top[j] > from[j][t] ? top[j] : from[j][t];
      top[j] = (int)wave_max((uint32_t)top[j]);
    }
    wait_vector_memory();                  // (every lane's rows are in registers)
#pragma unroll
    for (int j = 0; j < BLOCKS; ++j) {
      if (!__any(moved[j] != 0)) continue;     // (the block's rows stay where they are)
      const long long slot0 = base + j * kScaleBlock;
#pragma unroll
      for (int t = 0; t < PASSES; ++t) {
        const int row = t * per_pass + sub;
        if (from[j][t] < 0 || !((moved[j] >> t & 1u) || from[j][t] != top[j])) continue;
        const float by = move_by(from[j][t], top[j]);
        u32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = from[j][t] == top[j] ? x[j][t][e] : rescale4(x[j][t][e], by);
        *(u32x4*)(codes + (int64_t)id[j] * a.page_stride + head_slot(slot0 + row) * a.row_bytes + p * 16) = y;
      }
      if (lane == 0) scales[(int64_t)id[j] * sc.page_stride + head_slot(slot0) / kScaleBlock] = (uint8_t)top[j];
    }
    wait_vector_memory();
  }
}

template <bool PAST>
__global__ __launch_bounds__(kThreads) void paged_read_e4m3_kernel(PagedRowsArgs a, PagedScaleArgs sc, int num_slots,
                                                                  char* k_out, char* v_out, int units) {
  const int layer = blockIdx.z, bg = blockIdx.y, b = bg / a.Hkv, g = bg - b * a.Hkv;
  const uint32_t item = blockIdx.x * kThreads + threadIdx.x;
  const int slot = (int)(item / units), p = (int)(item - slot * (uint32_t)units);
  if (slot >= num_slots) return;
  int id = -1;
  if (slot < a.kv_len[b]) id = page_of(a, a.table + (size_t)b * a.width, slot);
  const int64_t in_head = ((int64_t)g << a.page_shift) + (slot & ((1 << a.page_shift) - 1));
  const size_t to = (((size_t)layer * a.B * a.Hkv + bg) * num_slots + slot) * a.row_bytes * 2 + p * 16;
  u32x2 x[2] = {};
  uint32_t byte[2] = {};
  if (id >= 0) {
    const int64_t at = layer * a.layer_stride + (int64_t)id * a.page_stride + in_head * a.row_bytes + p * 8;
    const int64_t scale_at = layer * sc.layer_stride + (int64_t)id * sc.page_stride + in_head / kScaleBlock;
    x[0] = *(const u32x2*)(a.k + at);
    x[1] = *(const u32x2*)(a.v + at);
    byte[0] = sc.k[scale_at];
    byte[1] = sc.v[scale_at];
  }
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    u32x4 y{0u, 0u, 0u, 0u};
    if (id >= 0) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t w = x[half][e];
        y[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power((int)byte[half]), false));
        y[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power((int)byte[half]), true));
      }
    }
    u32x4* out = (u32x4*)((half ? v_out : k_out) + to);
    if constexpr (PAST) __builtin_nontemporal_store(y, out);
    else *out = y;
  }
}

struct AppendGrid {
  dim3 grid;
  size_t lds;
  int units, blocks;
  unsigned query_groups, key_groups;
  bool past;       // the queries are stored past the caches
};

template <typename T, int PASSES>
hipError_t append(const PagedRowsArgs& a, const PagedScaleArgs& sc, const RopeArgs& rope, const RopeQueryArgs& q,
                  const AppendGrid& s, hipStream_t stream) {
  auto kern = paged_append_e4m3_kernel<T, PASSES>;
  static bool configured[64] = {};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  if (!configured[dev]) {
    e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kMaxTurns * 8);
    if (e != hipSuccess) return e;
    configured[dev] = true;
  }
  hipLaunchKernelGGL(kern, s.grid, dim3(kThreads), s.lds, stream, a, sc, rope, q, a.row_bytes, s.units, s.blocks,
                     s.query_groups, s.key_groups, s.past);
  return hipGetLastError();
}
template <typename T>
hipError_t append_passes(int passes, const PagedRowsArgs& a, const PagedScaleArgs& sc, const RopeArgs& rope,
                         const RopeQueryArgs& q, const AppendGrid& s, hipStream_t stream) {
  if (passes <= 1) return append<T, 1>(a, sc, rope, q, s, stream);
  if (passes <= 2) return append<T, 2>(a, sc, rope, q, s, stream);
  if (passes <= 4) return append<T, 4>(a, sc, rope, q, s, stream);
  return append<T, 8>(a, sc, rope, q, s, stream);
}

// passes over a block's 16 rows of `units` lanes each (units <= 32: 8 at most)
int passes_of(int units) { return (kScaleBlock + 64 / units - 1) / (64 / units); }

}  // namespace

hipError_t launch_paged_append_e4m3(const PagedRowsArgs& a, const PagedScaleArgs& sc, const RopeArgs& rope,
                                    const RopeQueryArgs& q, int elem, hipStream_t stream) {
  if (a.N == 0 || a.B == 0) return hipSuccess;
  const int waves = kThreads / 64, pairs = rope.R / 2;
  AppendGrid s{};
  s.units = a.row_bytes / 16;
  s.blocks = (int)(((long long)a.N + 2 * kScaleBlock - 2) / kScaleBlock);
  s.query_groups = (unsigned)(((long long)a.N * q.Hq * s.units + kThreads - 1) / kThreads);
  s.key_groups = (unsigned)(((long long)s.blocks * a.Hkv + waves - 1) / waves);
  s.grid = dim3(s.query_groups + 2 * s.key_groups, (unsigned)a.B, (unsigned)a.NL);
  // the turns of a group's rows: of the blocks that 4 waves can be of, of the rows that the queries' items can be of
  const int key_rows = (a.Hkv % waves == 0 ? 1 : std::min(waves, (waves - 2) / a.Hkv + 2)) * kScaleBlock;
  const int query_rows = q.Hq > 0 ? (kThreads - 2) / (s.units * q.Hq) + 2 : 0;
  s.lds = (size_t)std::max(key_rows, query_rows) * pairs * sizeof(float2);
  if (s.lds > (size_t)kMaxTurns * 8) return hipErrorInvalidValue;
  // (fp32: a run of 8 columns is two words, half lines a store)
  s.past = elem == 2 && stored_past((long long)a.B * a.N * q.Hq * a.row_bytes * elem, rope.R, a.row_bytes, elem);
  const int passes = passes_of(s.units);
  return elem == 2 ? append_passes<__bf16>(passes, a, sc, rope, q, s, stream)
                   : append_passes<float>(passes, a, sc, rope, q, s, stream);
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
  const int units = a.row_bytes / 8;
  const long long items = (long long)num_slots * units;
  if (items == 0 || a.B == 0) return hipSuccess;
  const dim3 grid((unsigned)((items + kThreads - 1) / kThreads), (unsigned)(a.B * a.Hkv), (unsigned)a.NL);
  const bool past = 2LL * a.NL * a.B * a.Hkv * num_slots * a.row_bytes * 2 >= kPastBytes;
  hipLaunchKernelGGL(past ? paged_read_e4m3_kernel<true> : paged_read_e4m3_kernel<false>, grid, dim3(kThreads), 0, stream, a, sc,
                     num_slots, k_out, v_out, units);
  return hipGetLastError();
}

}  // namespace dreams
