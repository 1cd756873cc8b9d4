// Attention over a paged cache, fp32, on the vector ALU: rows that are tree nodes (every node sees the prefix and its
// ancestors-or-self) or consecutive positions of a prompt (row i sees the slots up to its own), in either case only
// keys within `window` positions, or among the first `sinks`.
//
// A workgroup of 16 waves owns R rows (1, 2 or 4) of one KV head and every key that one of them sees: the sinks and one
// run of slots.  A key's K (or V) row is held by D/4 neighbouring lanes, so a wave reads 64 / (D/4) rows per load; its
// lanes look their key's page up in the table.  Every lane group keeps its own online softmax (running maximum, running
// sum, accumulator) in fp32; the states are merged within the wave, then across the waves in wave order through LDS,
// so results are reproducible.
//
// Latency bounds small calls: 8 heads on 2 x 16 nodes and 300 keys in sight take 7.5 us, a chain of lengths, tree, table,
// rows and merge.  Large ones are bound by the vector ALU, which pays a reduction over D/4 lanes for each score (32
// heads on 60 nodes and 3136 keys, D = 128: 164 us, 19 TFLOP/s).
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
  ((float*)a.out)[row * D + d] = lt > 0.f ? o / lt : 0.f;
  if (a.lse && d == 0) a.lse[row] = lt > 0.f ? (M + log2f(lt)) * kLn2 : -INFINITY;
}

template <int D, bool PROMPT, int R>
hipError_t launch_rows(const PagedAttnArgs& a, hipStream_t stream) {
  const long long grid = (long long)a.B * a.Hkv * (((long long)a.G * a.T + R - 1) / R);
  hipLaunchKernelGGL((paged_attn_f32_kernel<D, R, PROMPT>), dim3((unsigned)grid), dim3(64 * kWaves), 0, stream, a);
  return hipGetLastError();
}

template <int D, bool PROMPT>
hipError_t launch(const PagedAttnArgs& a, hipStream_t stream) {
  // (More rows a workgroup read a key for all of them; fewer leave no compute unit idle.  With 1, 2 and 4 rows: 32 rows in all,
  // 2000 keys 23, 31, 51 us; 256: 27, 32, 53; 512: 50, 33, 52; 640 x 3136 keys 113, 97, 80; 1920: 305, 198, 164.)
  const long long rows = (long long)a.B * a.Hq * a.T;
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
