// Rotary positions: the angles of a row's pairs, and units (two runs of columns) of a row in registers.
#pragma once

#include "kernels.h"

namespace dreams {
namespace {

// cos and sin of position * freq radians, times gain.  In fp64 and rounded once, so that the rotated columns are as near as
// fp32 products can be: rows that go into 8 bits fall on another code where an error reaches its border.  The angle is reduced
// to a quarter turn (its error grows with the turns, 2^-52 of them); the rest x, |x| <= pi/4, goes through the Taylor
// polynomials of sine and cosine about 0, whose first terms left out are x^13/13! < 7e-12 and x^12/12! < 2e-10.
__device__ __forceinline__ void turn(double position, double freq, float gain, float* c, float* s) {
  const double t = position * (freq * 0.15915494309189533577);
  const double u = 4.0 * (t - rint(t)), quarter = rint(u);
  const double x = (u - quarter) * 1.57079632679489661923, y = x * x;
  const double sn = x * fma(y, fma(y, fma(y, fma(y, fma(y, -1.0 / 39916800, 1.0 / 362880), -1.0 / 5040), 1.0 / 120), -1.0 / 6), 1.0);
  const double cs = fma(y, fma(y, fma(y, fma(y, fma(y, -1.0 / 3628800, 1.0 / 40320), -1.0 / 720), 1.0 / 24), -0.5), 1.0);
  const int q = (int)quarter;
  const double a = (q & 1) ? sn : cs, b = (q & 1) ? cs : sn, g = (double)gain;
  *c = (float)(g * ((q + 1) & 2 ? -a : a));
  *s = (float)(g * (q & 2 ? -b : b));
}

// Depth of tree node i by parents in LDS (an entry that breaks the rules ends the walk).
__device__ __forceinline__ int depth_of(const int* parent, int i) {
  int d = 0;
  for (int j = i;; ++d) {
    const int p = parent[j];
    if (p < 0 || p >= j) return d;
    j = p;
  }
}

// Bytes of output from which they are stored past the caches, where a unit's runs fill 64 bytes at least (28 heads x 8192
// rows 25.1 us in the caches, 19.7 past them; 2 x 8 heads x 437 rows of 64 columns in fp32, 1.8 MB, 4.0 and 4.4).
constexpr long long kPastBytes = 4 << 20;
inline bool stored_past(long long bytes, int R, int D, int elem) {
  return bytes >= kPastBytes && R / 2 * elem >= 64 && (D == R || (D - R) / 2 * elem >= 64);
}

// W columns of a row from column `at` on, as they are in memory, and as fp32.
template <typename T, int W>
struct Run {
  static constexpr int WORDS = W * (int)sizeof(T) / 16;    // of 16 bytes
  typedef uint32_t words __attribute__((ext_vector_type(4)));
  typedef T txw __attribute__((ext_vector_type(W)));
  words w[WORDS];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (auto& x : w) x = words{0u, 0u, 0u, 0u};
  }
  // (PAST: data that is not kept in the caches)
  template <bool PAST = false>
  __device__ __forceinline__ void load(const char* row, int at) {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      const words* from = (const words*)(row + at * sizeof(T)) + i;
      if constexpr (PAST) w[i] = __builtin_nontemporal_load(from);
      else w[i] = *from;
    }
  }
  template <bool PAST = false>
  __device__ __forceinline__ void store(char* row, int at) const {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      words* to = (words*)(row + at * sizeof(T)) + i;
      if constexpr (PAST) __builtin_nontemporal_store(w[i], to);
      else *to = w[i];
    }
  }
  __device__ __forceinline__ void get(float (&x)[W]) const {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const uint32_t u = sizeof(T) == 2 ? w[0][i / 2] : w[i / 4][i % 4];   // (a bit cast of the element itself takes element 0)
      x[i] = __builtin_bit_cast(float, sizeof(T) == 4 ? u : i & 1 ? u & 0xffff0000u : u << 16);
    }
  }
  __device__ __forceinline__ void set(const float (&x)[W]) {
    txw y;
#pragma unroll
    for (int i = 0; i < W; ++i) y[i] = (T)x[i];
    __builtin_memcpy(&w, &y, sizeof(y));
  }
};

// Unit p of a row is two runs of W columns: 8 p (W = 8) and half of the rotated columns behind it, so that the lanes of a wave
// read and write whole lines, run by run.  In the half layout they are W pairs, in the interleaved one W / 2 each.  The
// columns past R are halved likewise (an odd run is the first of a unit whose second is -1).
struct Unit {
  int first, second;
  bool rotated;
};
template <int W>
__device__ __forceinline__ Unit unit_of(int p, int R, int D) {
  Unit u;
  const int turned = R / (2 * W);
  u.rotated = p < turned;
  if (u.rotated) {
    u.first = W * p;
    u.second = R / 2 + W * p;
  } else {
    const int runs = (D - R) / W, half = (runs + 1) / 2, t = p - turned;
    u.first = R + W * t;
    u.second = t + half < runs ? R + W * (t + half) : -1;
  }
  return u;
}
template <int W>
__host__ __device__ inline int rope_units(int R, int D) { return R / (2 * W) + (D - R + 2 * W - 1) / (2 * W); }

// The cosines and sines of a unit's W pairs, of a row's R / 2: half layout W in a row, interleaved W / 2 for each run.
template <int W>
__device__ __forceinline__ void take_turns(const float2* row, int p, int R, bool interleaved, float (&c)[W], float (&s)[W]) {
  typedef float f32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int i = 0; i < W / 2; ++i) {
    const int at = !interleaved ? W * p + 2 * i : i < W / 4 ? W / 2 * p + 2 * i : R / 4 + W / 2 * p + 2 * (i - W / 4);
    const f32x4 x = *(const f32x4*)(row + at);
    c[2 * i] = x[0];
    s[2 * i] = x[1];
    c[2 * i + 1] = x[2];
    s[2 * i + 1] = x[3];
  }
}
// a unit's two runs, turned
template <int W>
__device__ __forceinline__ void rotate(float (&a)[W], float (&b)[W], const float (&c)[W], const float (&s)[W],
                                       bool interleaved) {
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < W; i += 2) {
      float x = a[i], y = a[i + 1];
      a[i] = fmaf(x, c[i / 2], -(y * s[i / 2]));
      a[i + 1] = fmaf(y, c[i / 2], x * s[i / 2]);
      x = b[i];
      y = b[i + 1];
      b[i] = fmaf(x, c[W / 2 + i / 2], -(y * s[W / 2 + i / 2]));
      b[i + 1] = fmaf(y, c[W / 2 + i / 2], x * s[W / 2 + i / 2]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float x = a[i], y = b[i];
      a[i] = fmaf(x, c[i], -(y * s[i]));
      b[i] = fmaf(y, c[i], x * s[i]);
    }
  }
}
template <typename T, int W>
__device__ __forceinline__ void rotate(Run<T, W>& x, Run<T, W>& y, const float (&c)[W], const float (&s)[W],
                                       bool interleaved) {
  float a[W], b[W];
  x.get(a);
  y.get(b);
  rotate(a, b, c, s, interleaved);
  x.set(a);
  y.set(b);
}

// A row's position, by a table, by a tree (parents in LDS) or in order.
__device__ __forceinline__ double position_of(const RopeArgs& r, const int* parents, int b, int i, int N) {
  if (r.positions) return (double)r.positions[(size_t)b * N + i];
  const int base = r.kv_len ? r.kv_len[b] : 0;
  return (double)base + (double)(r.parent ? depth_of(parents, i) : i);
}
// Cosine and sine of the pairs of rows first .. first + rows - 1 (of them those in 0 .. N - 1): every head turns by the same,
// so a workgroup computes them once, a pair a thread at a time.  [rows][R / 2].  Called by all threads; `scratch` is LDS for
// the positions and, for a tree, its parents.
constexpr int kTurnRows = 256;      // rows of a workgroup, at most
struct TurnScratch {
  double position[kTurnRows];
  int parent[kMaxNodes];
};
template <int THREADS>
__device__ __forceinline__ void fill_turns(const RopeArgs& r, TurnScratch& scratch, int b, int first, int rows, int N, float2* to) {
  const int pairs = r.R / 2, tid = threadIdx.x;
  int row = tid / pairs, pair = tid - row * pairs;
  double freq = r.freq[pair];          // (on its way while the positions come)
  if (r.parent && !r.positions) {
    if (tid < N) scratch.parent[tid] = r.parent[(size_t)b * N + tid];
    __syncthreads();
  }
  if (tid < rows && first + tid >= 0 && first + tid < N) scratch.position[tid] = position_of(r, scratch.parent, b, first + tid, N);
  __syncthreads();
  const int row_step = THREADS / pairs, pair_step = THREADS - row_step * pairs;
  while (row < rows) {
    if (first + row >= 0 && first + row < N) {
      float c, s;
      turn(scratch.position[row], freq, r.gain, &c, &s);
      to[row * pairs + pair] = make_float2(c, s);
    }
    row += row_step;
    if (pair_step > 0) {
      pair += pair_step;
      if (pair >= pairs) {
        pair -= pairs;
        ++row;
      }
      freq = r.freq[pair];
    }
  }
  __syncthreads();
}

}  // namespace
}  // namespace dreams
