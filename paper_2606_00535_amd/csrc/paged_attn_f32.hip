// Attention over a paged cache, fp32: rows that are tree nodes (every node sees the prefix and its ancestors-or-self) or
// consecutive positions of a prompt (row i sees the slots up to its own), in either case only keys within `window`
// positions, or among the first `sinks`.  Few rows on the vector ALU, many in tiles on the matrix cores (below).
//
// A workgroup of 16 waves owns R rows (1, 2 or 4) of one KV head and every key that one of them sees: the sinks and one
// run of slots.  A key's K (or V) row is held by D/4 neighbouring lanes, so a wave reads 64 / (D/4) rows per load; its
// lanes look their key's page up in the table.  Every lane group keeps its own online softmax (running maximum, running
// sum, accumulator) in fp32; the states are merged within the wave, then across the waves in wave order through LDS,
// so results are reproducible.
//
// Latency bounds small calls: 8 heads on 2 x 16 nodes and 300 keys in sight take 7.5 us, a chain of lengths, tree, table,
// rows and merge.  Larger ones are bound by the vector ALU, which pays a reduction over D/4 lanes for each score (32
// heads on 60 nodes and 3136 keys, D = 128: 164 us, 19 TFLOP/s).  With 4 rows a workgroup's 16 waves leave 128 registers each,
// and three of the four builds spill 3 or 4 of them, with one access inside a loop.
#include "kernels.h"

#include <math.h>
#include <type_traits>

namespace dreams {
namespace {

constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kWaves = kPagedF32Threads / 64;

typedef float f32x4 __attribute__((ext_vector_type(4)));

template <int CTRL>
__device__ __forceinline__ float add_rotated(float x) {
  const int y = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true);
  return x + __builtin_bit_cast(float, y);
}
// sum over 16 or 32 neighbouring lanes; every lane gets the same bits
template <int LANES>
__device__ __forceinline__ float sum_lanes(float x) {
  x = add_rotated<0x128>(x);   // row_ror:8, 4, 2, 1
  x = add_rotated<0x124>(x);
  x = add_rotated<0x122>(x);
  x = add_rotated<0x121>(x);
  if constexpr (LANES == 32) x += __shfl_xor(x, 16);
  return x;
}

template <int D, int R, bool PROMPT>
__global__ __launch_bounds__(64 * kWaves) void paged_attn_f32_kernel(PagedAttnArgs a) {
  constexpr int NW = kWaves;
  constexpr int LPK = D / 4;          // lanes per key
  constexpr int KPI = 64 / LPK;       // keys a wave reads per load
  constexpr int U = 4;                // such groups of keys per pass
  __shared__ int par_lds[kMaxNodes];
  __shared__ int depth_lds[kMaxNodes];
  __shared__ uint64_t anc_lds[R][2];
  __shared__ float st_ml[NW][R][2];
  __shared__ float st_acc[NW][R][D];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane % LPK, kg = lane / LPK;   // this lane's piece of a row, and its key of a group
  const int T = a.T;
  const long long rows_u = (long long)a.G * T;
  const int units = a.B * a.Hkv;
  const int u = (int)(blockIdx.x % (unsigned)units);
  const long long r0 = (long long)(blockIdx.x / (unsigned)units) * R;
  const int b = u / a.Hkv, g = u - b * a.Hkv;
  int nb = T;   // the sequence's live rows
  if (PROMPT && a.row_len) {
    nb = a.row_len[b];
    nb = nb < 0 ? 0 : (nb > T ? T : nb);
  }
  int L = a.kv_len[b];
  L = L < 0 ? 0 : (L > a.capacity - nb ? a.capacity - nb : L);
  const size_t row0 = (size_t)u * rows_u;   // row 0 of this KV head's query rows
  const int32_t* table = a.table + (size_t)b * a.width;
  const int ps1 = (1 << a.page_shift) - 1;
  auto at = [&](int slot) {   // this lane's piece of a slot's row, in elements
    int id = table[slot >> a.page_shift];
    id = id < 0 ? 0 : (id >= a.num_pages ? a.num_pages - 1 : id);
    return (int64_t)id * (a.page_stride / 4) + (((int64_t)g << a.page_shift) + (slot & ps1)) * D + 4 * c;
  };
  const float* kp = (const float*)a.k;
  const float* vp = (const float*)a.v;

  // depths and ancestor sets of the tree's rows
  if constexpr (!PROMPT) {
    if (tid < T) {
      par_lds[tid] = a.parent ? a.parent[(size_t)b * T + tid] : -1;
    }
    __syncthreads();
    if (tid < T) {
      int j = tid, d = 0;
      for (int st = 0; st < T; ++st) {
        const int p = par_lds[j];
        if (p < 0 || p >= j) break;   // the root, or not a valid parent: the walk ends here
        j = p;
        ++d;
      }
      depth_lds[tid] = d;
    }
    __syncthreads();
    if (tid < R) {
      const int i = (int)(min(r0 + tid, rows_u - 1) % T);
      uint64_t anc[2] = {0, 0};
      if (a.mask) {
        const int W = (T + 63) / 64;
        const uint64_t* mr = a.mask + ((size_t)b * T + i) * W;
        anc[0] = mr[0];
        anc[1] = W > 1 ? mr[1] : 0;
      } else {
        int j = i;
        for (int st = 0; st < T; ++st) {
          anc[j >> 6] |= 1ull << (j & 63);
          const int p = par_lds[j];
          if (p < 0 || p >= j) break;
          j = p;
        }
      }
      if (a.window > 0) {
        for (int j = 0; j < T; ++j)
          if (depth_lds[i] - depth_lds[j] >= a.window && L + depth_lds[j] >= a.sinks) anc[j >> 6] &= ~(1ull << (j & 63));
      }
      anc_lds[tid][0] = anc[0];
      anc_lds[tid][1] = anc[1];
    }
    __syncthreads();
  }

  // the rows' slots: [0, min(sinks, lo)) and [lo, end)
  f32x4 q[R], acc[R];
  float m[R], l[R];
  int lo[R], end[R], lo_min = 0x7fffffff, lo_max = 0, end_min = 0x7fffffff, end_max = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const long long row = min(r0 + r, rows_u - 1);
    const int i = (int)(row % T);
    q[r] = *(const f32x4*)((const float*)a.q + (row0 + row) * D + 4 * c);
    acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
    m[r] = -INFINITY;
    l[r] = 0.f;
    const int pos = PROMPT ? L + i : L + depth_lds[i];
    const bool live = !PROMPT || i < nb;
    end[r] = live ? (PROMPT ? pos + 1 : L) : 0;
    lo[r] = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
    lo[r] = min(lo[r], end[r]);
    end_max = max(end_max, end[r]);
    end_min = min(end_min, end[r]);
    if (live) lo_min = min(lo_min, lo[r]);
    lo_max = max(lo_max, lo[r]);
  }
  if (lo_min > end_max) lo_min = end_max;
  const int first = min(a.sinks, lo_min);            // sinks before the run
  const int total = first + (end_max - lo_min);
  auto slot_of = [&](int n) { return n < first ? n : n - first + lo_min; };

  // NK groups of keys into every row's state; masked: only the keys that see(r, t), whose values alone count
  auto update = [&](auto nk, auto masked, const f32x4* kk, const f32x4* vv, auto see) {
    constexpr int NK = decltype(nk)::value;
    constexpr bool MASKED = decltype(masked)::value;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float x[NK], mx = m[r];
#pragma unroll
      for (int t = 0; t < NK; ++t) {
        float s = q[r][0] * kk[t][0];
        s = fmaf(q[r][1], kk[t][1], s);
        s = fmaf(q[r][2], kk[t][2], s);
        s = fmaf(q[r][3], kk[t][3], s);
        x[t] = sum_lanes<LPK>(s);
        if (!MASKED || see(r, t)) mx = fmaxf(mx, x[t] * a.scale_log2);
      }
      const float ref = mx == -INFINITY ? 0.f : mx;   // (nothing seen yet: every weight below is 2^-inf = 0)
      const float alpha = __builtin_amdgcn_exp2f(m[r] - ref);
      float psum = 0.f;
      f32x4 pv = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < NK; ++t) {
        const bool s = !MASKED || see(r, t);
        const float p = s ? __builtin_amdgcn_exp2f(fmaf(x[t], a.scale_log2, -ref)) : 0.f;
        psum += p;
#pragma unroll
        for (int i = 0; i < 4; ++i) pv[i] = fmaf(p, s ? vv[t][i] : 0.f, pv[i]);
      }
      l[r] = fmaf(l[r], alpha, psum);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[r][i] = fmaf(acc[r][i], alpha, pv[i]);
      m[r] = mx;
    }
  };

  for (int n0 = wave * (KPI * U); n0 < total; n0 += NW * KPI * U) {
    f32x4 kk[U], vv[U];
    int slot[U];
    int64_t e[U];
#pragma unroll
    for (int t = 0; t < U; ++t) {
      slot[t] = slot_of(min(n0 + t * KPI + kg, total - 1));
      e[t] = at(slot[t]);
    }
#pragma unroll
    for (int t = 0; t < U; ++t) kk[t] = *(const f32x4*)(kp + e[t]);
#pragma unroll
    for (int t = 0; t < U; ++t) vv[t] = *(const f32x4*)(vp + e[t]);
    const int first_slot = slot_of(n0), last_slot = slot_of(n0 + KPI * U - 1);   // (a pass in sight of every row)
    if (n0 + KPI * U <= total && last_slot < end_min && first_slot >= lo_max)
      update(std::integral_constant<int, U>{}, std::false_type{}, kk, vv, [](int, int) { return true; });
    else
      update(std::integral_constant<int, U>{}, std::true_type{}, kk, vv, [&](int r, int t) {
        return n0 + t * KPI + kg < total && slot[t] < end[r] && (slot[t] >= lo[r] || slot[t] < a.sinks);
      });
  }
  if constexpr (!PROMPT) {
    for (int j0 = wave * KPI; j0 < T; j0 += NW * KPI) {
      const int j = min(j0 + kg, T - 1);
      const int64_t e = at(L + j);
      const f32x4 kt = *(const f32x4*)(kp + e), vt = *(const f32x4*)(vp + e);
      update(std::integral_constant<int, 1>{}, std::true_type{}, &kt, &vt,
             [&](int r, int) { return j0 + kg < T && ((anc_lds[r][j >> 6] >> (j & 63)) & 1ull) != 0; });
    }
  }

  // ---- the wave's lane groups, then the waves in wave order
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int off = LPK; off < 64; off <<= 1) {
      const float mo = __shfl_xor(m[r], off), lo2 = __shfl_xor(l[r], off);
      const float M = fmaxf(m[r], mo);
      const float w = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[r] - M);
      const float wo = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mo - M);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[r][i] = acc[r][i] * w + __shfl_xor(acc[r][i], off) * wo;
      l[r] = l[r] * w + lo2 * wo;
      m[r] = M;
    }
    if (kg == 0) *(f32x4*)&st_acc[wave][r][4 * c] = acc[r];
    if (lane == 0) {
      st_ml[wave][r][0] = m[r];
      st_ml[wave][r][1] = l[r];
    }
  }
  __syncthreads();
  if (tid >= R * D) return;
  const int r = tid / D, d = tid % D;   // this thread's row and output column
  if (r0 + r >= rows_u) return;
  float M = st_ml[0][r][0];
#pragma unroll
  for (int w = 1; w < NW; ++w) M = fmaxf(M, st_ml[w][r][0]);
  float l4[4] = {}, o4[4] = {};   // four chains, then their sums in pairs
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const float wt = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st_ml[w][r][0] - M);
    l4[w % 4] = fmaf(st_ml[w][r][1], wt, l4[w % 4]);
    o4[w % 4] = fmaf(st_acc[w][r][d], wt, o4[w % 4]);
  }
  const float lt = (l4[0] + l4[1]) + (l4[2] + l4[3]), o = (o4[0] + o4[1]) + (o4[2] + o4[3]);
  const size_t row = row0 + r0 + r;
  const bool some = lt != 0.f;   // (a row that sees a NaN has a NaN sum, and is NaN)
  ((float*)a.out)[row * D + d] = some ? o / lt : 0.f;
  if (a.lse && d == 0) a.lse[row] = some ? (M + log2f(lt)) * kLn2 : -INFINITY;
}

// Many rows: the same on the matrix cores, fp32 in and out.  A workgroup of 4 waves owns 64 consecutive
// rows of a KV head's G * T, a wave 16 of them; keys go through LDS in tiles of 32, two buffers, the next tile's rows in
// registers meanwhile.  S^T = K Q^T and O^T += V^T P^T on v_mfma_f32_16x16x4_f32: lane (g, n) = (lane / 16, lane % 16) holds
// the scores of row n with keys 4 g + 0..3 of 16, just the operand that the value product takes if its step i is over keys
// 4 g + i.  Sums run over any order of a row's D, so four steps share a 16-byte read of K (columns 16 t + 4 g + 0..3) and four
// output blocks one of V (block jb: columns 64 c + 4 m + jb).  Bound by latency: with one or two waves a SIMD, a tile's loads,
// score products, exponentials and value products follow one another.  5 x 32 heads on 310 rows, D = 128, 88 us, 45 TFLOP/s of
// what the rows see, 29 % of the matrix cores' fp32 rate (157).
constexpr int kTile = 32, kTileRows = 64, kTileWaves = 4;

template <int D, bool PROMPT>
__global__ __launch_bounds__(64 * kTileWaves, 2) void paged_tiles_f32_kernel(PagedAttnArgs a) {
  constexpr int KS = D / 16, KROW = D + 4;           // a K row's padding: 16 rows' reads fall on different banks
  constexpr int C4 = D / 4, PER = kTile * C4 / 256;  // 16-byte pieces of a row, and of a tile per thread
  extern __shared__ __attribute__((aligned(16))) float kv_lds[];   // two buffers of a tile's K rows and V rows
  __shared__ int par_lds[PROMPT ? 1 : kMaxNodes], depth_lds[PROMPT ? 1 : kMaxNodes];
  __shared__ int range_lds[kTileWaves][2];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int T = a.T, rows_u = a.G * T, units = a.B * a.Hkv;
  const int u = (int)(blockIdx.x % (unsigned)units), r0 = (int)(blockIdx.x / (unsigned)units) * kTileRows;
  const int b = u / a.Hkv, head = u - b * a.Hkv;
  int nb = T;
  if (PROMPT && a.row_len) nb = min(max(a.row_len[b], 0), T);
  const int L = min(max(a.kv_len[b], 0), a.capacity - nb);
  const size_t row0 = (size_t)u * rows_u;
  const int row = r0 + wave * 16 + n, i = min(row, rows_u - 1) % T;
  const bool live = row < rows_u && (!PROMPT || i < nb);

  // the row's slots: [0, min(sinks, lo)), [lo, end), and of a tree the ancestors'
  int pos = L + i;
  uint64_t anc0 = 0, anc1 = 0;
  if constexpr (!PROMPT) {
    if (tid < T) par_lds[tid] = a.parent ? a.parent[(size_t)b * T + tid] : -1;
    __syncthreads();
    auto walk = [&](int from, auto visit) {   // from a node to the root, or to an entry that breaks the rules
      int j = from, d = 0;
      for (;; ++d) {
        visit(j);
        const int p = par_lds[j];
        if (p < 0 || p >= j) return d;
        j = p;
      }
    };
    if (tid < T) depth_lds[tid] = walk(tid, [](int) {});
    __syncthreads();
    pos = L + depth_lds[i];
    if (a.mask) {
      const int words = (T + 63) / 64;
      const uint64_t* bits = a.mask + ((size_t)b * T + i) * words;
      anc0 = bits[0];
      anc1 = words > 1 ? bits[1] : 0;
    } else {
      walk(i, [&](int j) { (j < 64 ? anc0 : anc1) |= 1ull << (j & 63); });
    }
    if (a.window > 0)
      for (int j = 0; j < T; ++j)
        if (depth_lds[i] - depth_lds[j] >= a.window && L + depth_lds[j] >= a.sinks) (j < 64 ? anc0 : anc1) &= ~(1ull << (j & 63));
  }
  const int end = live ? (PROMPT ? pos + 1 : L) : 0;
  const int lo = min(a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0, end);
  auto over_rows = [&](int x, auto op) {   // of the wave's 16 rows
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) x = op(x, __shfl_xor(x, off));
    return __builtin_amdgcn_readfirstlane(x);
  };
  auto lower = [](int x, int y) { return min(x, y); };
  auto upper = [](int x, int y) { return max(x, y); };
  const int w_lo = over_rows(live ? lo : 0x7fffffff, lower);             // some row's
  const int w_end = over_rows(live ? (PROMPT ? end : L + T) : 0, upper);
  const int plain_lo = over_rows(live ? lo : 0, upper), plain_end = over_rows(live ? end : 0x7fffffff, lower);   // every live row's
  if (lane == 0) {
    range_lds[wave][0] = w_lo;
    range_lds[wave][1] = w_end;
  }
  __syncthreads();
  int lo_all = range_lds[0][0], end_all = range_lds[0][1];
#pragma unroll
  for (int w = 1; w < kTileWaves; ++w) {
    lo_all = min(lo_all, range_lds[w][0]);
    end_all = max(end_all, range_lds[w][1]);
  }
  lo_all = min(lo_all, end_all);
  const int first = min(a.sinks, lo_all);            // sinks before the run
  const int total = first + (end_all - lo_all), tiles = (total + kTile - 1) / kTile;
  auto slot_of = [&](int key) { return key < first ? key : key - first + lo_all; };

  f32x4 q[KS], o[D / 16];
#pragma unroll
  for (int t = 0; t < KS; ++t) {
    q[t] = *(const f32x4*)((const float*)a.q + (row0 + min(row, rows_u - 1)) * D + 16 * t + 4 * g);
    if (!live) q[t] = f32x4{0.f, 0.f, 0.f, 0.f};     // (may hold anything)
  }
#pragma unroll
  for (int t = 0; t < D / 16; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  // a tile's rows: thread tid takes piece tid % C4 of rows tid / C4 + (256 / C4) x
  const int32_t* table = a.table + (size_t)b * a.width;
  const int ps1 = (1 << a.page_shift) - 1, piece = tid % C4;
  int page[PER];
  f32x4 kr[PER], vr[PER];
  auto key_of = [&](int tile, int x) { return tile * kTile + tid / C4 + (256 / C4) * x; };
  auto look_up = [&](int tile) {
#pragma unroll
    for (int x = 0; x < PER; ++x) page[x] = table[slot_of(min(key_of(tile, x), total - 1)) >> a.page_shift];
  };
  auto load = [&](int tile) {
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      const int key = key_of(tile, x), slot = slot_of(min(key, total - 1));
      const int id = min(max(page[x], 0), a.num_pages - 1);
      const int64_t at = (int64_t)id * (a.page_stride / 4) + (((int64_t)head << a.page_shift) + (slot & ps1)) * D + 4 * piece;
      kr[x] = *(const f32x4*)((const float*)a.k + at);
      vr[x] = *(const f32x4*)((const float*)a.v + at);
      if (key >= total) kr[x] = vr[x] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  if (tiles > 0) {
    look_up(0);
    load(0);
    if (tiles > 1) look_up(1);
  }
  for (int k = 0; k < tiles; ++k) {
    float* const kt = kv_lds + (k & 1) * (kTile * (KROW + D));
    float* const vt = kt + kTile * KROW;
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      const int r = tid / C4 + (256 / C4) * x;
      *(f32x4*)(kt + r * KROW + 4 * piece) = kr[x];
      *(f32x4*)(vt + r * D + 4 * piece) = vr[x];
    }
    __syncthreads();   // (the tile before last is behind every wave, so its buffer is free at the next turn)
    if (k + 1 < tiles) load(k + 1);
    if (k + 2 < tiles) look_up(k + 2);
    const int s_first = slot_of(k * kTile), s_last = slot_of(min(k * kTile + kTile, total) - 1);
    if (s_first >= w_end || (s_last < w_lo && s_first >= a.sinks)) continue;   // no row of the wave sees it
    f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      const f32x4 k0 = *(const f32x4*)(kt + n * KROW + 16 * t + 4 * g);
      const f32x4 k1 = *(const f32x4*)(kt + (16 + n) * KROW + 16 * t + 4 * g);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(k0[j], q[t][j], s[0], 0, 0, 0);
        s[1] = __builtin_amdgcn_mfma_f32_16x16x4f32(k1[j], q[t][j], s[1], 0, 0, 0);
      }
    }
    const bool plain = k * kTile + kTile <= total && s_last < plain_end && s_first >= plain_lo;
    float top = m;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x = s[kb][e] * a.scale_log2;
        if (!plain) {
          const int key = k * kTile + 16 * kb + 4 * g + e, slot = slot_of(key), j = slot - L;
          bool vis = slot < end && (slot >= lo || slot < a.sinks);
          if constexpr (!PROMPT) vis |= j >= 0 && j < T && (((j < 64 ? anc0 : anc1) >> (j & 63)) & 1ull) != 0;
          if (!vis || !live || key >= total) x = -INFINITY;
        }
        s[kb][e] = x;
        top = fmaxf(top, x);
      }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    if (__any(top > m)) {
      const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
      l *= alpha;
#pragma unroll
      for (int t = 0; t < D / 16; ++t) o[t] *= alpha;
      m = top;
    }
    const float ref = m == -INFINITY ? 0.f : m;      // (nothing seen yet: every weight below is 2^-inf = 0)
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[kb][e] = __builtin_amdgcn_exp2f(s[kb][e] - ref);
        l += s[kb][e];
      }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
          const f32x4 v = *(const f32x4*)(vt + (16 * kb + 4 * g + e) * D + 64 * c + 4 * n);
#pragma unroll
          for (int jb = 0; jb < 4; ++jb)
            o[4 * c + jb] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[jb], s[kb][e], o[4 * c + jb], 0, 0, 0);
        }
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (row >= rows_u) return;
  const bool any = live && l != 0.f;   // (a NaN sum gives a NaN)
  float* const out = (float*)a.out + (row0 + row) * D;
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f32x4 x;
#pragma unroll
      for (int jb = 0; jb < 4; ++jb) x[jb] = any ? o[4 * c + jb][e] / l : 0.f;
      *(f32x4*)(out + 64 * c + 16 * g + 4 * e) = x;
    }
  if (a.lse && g == 0) a.lse[row0 + row] = any ? (m + log2f(l)) * kLn2 : -INFINITY;
}

template <int D, bool PROMPT, int R>
hipError_t launch_rows(const PagedAttnArgs& a, hipStream_t stream) {
  const long long grid = (long long)a.B * a.Hkv * (((long long)a.G * a.T + R - 1) / R);
  hipLaunchKernelGGL((paged_attn_f32_kernel<D, R, PROMPT>), dim3((unsigned)grid), dim3(64 * kWaves), 0, stream, a);
  return hipGetLastError();
}

template <int D, bool PROMPT>
hipError_t launch_tiles(const PagedAttnArgs& a, hipStream_t stream) {
  constexpr int lds = 2 * kTile * (2 * D + 4) * (int)sizeof(float);
  static bool configured[64] = {};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  if (!configured[dev]) {
    e = hipFuncSetAttribute((const void*)paged_tiles_f32_kernel<D, PROMPT>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    configured[dev] = true;
  }
  const long long grid = (long long)a.B * a.Hkv * (((long long)a.G * a.T + kTileRows - 1) / kTileRows);
  hipLaunchKernelGGL((paged_tiles_f32_kernel<D, PROMPT>), dim3((unsigned)grid), dim3(64 * kTileWaves), lds, stream, a);
  return hipGetLastError();
}

template <int D, bool PROMPT>
hipError_t launch(const PagedAttnArgs& a, hipStream_t stream) {
  const long long rows = (long long)a.B * a.Hq * a.T;
  // The tiles want rows for every unit's matrix cores, and enough of one KV head to fill a wave's 16 by half (by rows in all:
  // 7 x 24 heads on 171 rows, D = 64: 154 us on the vector ALU, 23 in tiles; 5 x 32 on 310, D = 128: 383, 88; 4096 behind 1000
  // keys 76, 68; 3840 behind 3136 325, 334; 2048 behind 300 18, 30; 4096 rows, 8 a KV head, behind 300: 63, 42; 4 a head 72, 88).
  if (rows >= 16LL * a.cus && (long long)a.G * a.T >= 8) return launch_tiles<D, PROMPT>(a, stream);
  // (More rows a workgroup read a key for all of them; fewer leave no compute unit idle.  With 1, 2 and 4 rows: 32 rows in all,
  // 2000 keys 23, 31, 51 us; 256: 27, 32, 53; 512: 50, 33, 52; 640 x 3136 keys 113, 97, 80; 1920: 305, 198, 164.)
  if (rows <= a.cus) return launch_rows<D, PROMPT, 1>(a, stream);
  if (rows <= 2LL * a.cus) return launch_rows<D, PROMPT, 2>(a, stream);
  return launch_rows<D, PROMPT, 4>(a, stream);
}

}  // namespace

hipError_t launch_paged_attn_f32(const PagedAttnArgs& a, hipStream_t stream) {
  if (a.D == 64) return a.prompt ? launch<64, true>(a, stream) : launch<64, false>(a, stream);
  if (a.D == 128) return a.prompt ? launch<128, true>(a, stream) : launch<128, false>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace dreams
