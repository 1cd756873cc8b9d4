// Tree-masked verification attention, bf16 inputs, fp32 accumulation on the matrix cores.
//
// What is computed (the paper's Section 3.2 attention mask applied to the target's verification pass of
// Section 2): for every tree node i of every query head, softmax(scale * q_i . k_j) v_j over the committed
// prefix slots and the slots of node i's ancestors-or-self.
//
// Work decomposition
//   * A workgroup of W waves (4 or 8) owns R query rows of one KV head (the rows of the G query heads sharing it
//     are packed: row r -> head r / T, node r % T, which is also their order in memory) and one piece of that
//     head's key axis.  Each wave owns 16*RB rows of its key group (below) for every key the group takes, and
//     every K/V byte the workgroup reads serves all of its rows.  The 64- and 128-row configurations take at
//     most half of a compute unit's LDS and registers (WPC = 2), so two workgroups share a compute unit.
//   * The pieces are cut from the host's bound on the key count (the first copies need nothing from the
//     device), or, with several sequences, from each sequence's own count.
//   * K/V stream through a ring of NST step slots in LDS (a step = 32 keys: 32 K rows then 32 V rows).  The
//     waves copy their share of every step straight from global memory into LDS (global_load_lds_dwordx4: no
//     registers in between), a whole ring ahead.  One barrier per super-step hands a landed step to all waves;
//     in the pipelined loop a second one frees the slots every wave has read, which are refilled at once.  The
//     copies are issued with inline assembly and waited for by exact count; nothing else in the kernel loads
//     through the vector memory path before the epilogue, so the compiler never inserts a wait that would
//     drain the ring.
//   * Each lane fetches the source chunk that lands where an XOR-swizzled row layout wants it, which makes
//     both operand reads below bank-conflict free:
//       S^T = K Q^T        v_mfma_f32_16x16x32_bf16, K rows as the A operand (16-byte LDS reads)
//       online softmax     per query row; each lane holds one row's scores, 4-way cross-lane reductions
//       O^T += V^T P^T     A operand read with ds_read_b64_tr_b16 (a 4 x 16 transposing LDS read); the
//                          probabilities are already in B-operand layout, so they never leave registers.
//   * Waves are arranged as KW key groups of W/KW waves: the groups take alternate steps (group k the steps
//     k, k+KW, ...), so a wave's operand reads serve as many rows as possible; the groups' (max, sum,
//     accumulator) states are merged through LDS at the end.
//   * With several pieces per (sequence, KV head, row group) -- a set -- each piece stores its rows' output
//     normalised by their softmax sum (bf16) and their (max, sum) to the workspace and arrives on the set's
//     counter.  A piece whose set has fully started waits for every arrival and merges its own slice of the
//     rows; a piece that finds its set not yet fully started leaves its slice to the piece that started last,
//     which learnt at its start which pieces had already arrived.  So a wait is only ever for a running piece.
//     The merge goes in piece order, so the result does not depend on which piece came last.  All pieces of
//     a set run on one XCD (below), so their rows are exchanged through that XCD's L2: plain stores, no
//     device-scope write-through, no second launch.  Each piece adds its XCD id (and its square) to the set's
//     counter when it starts, and a merging piece checks that they all match its own.
//   * Workgroup ids are remapped so that all workgroups of one (sequence, KV head) share blockIdx % 8:
//     consecutive ids of a dispatch are dealt round-robin over the 8 XCDs, so these run on one XCD (which one
//     takes id 0 varies between dispatches), and row groups reading the same keys share them in its L2.
//   * Over a paged cache (PAGED), the caller's blocks of 16 slots come from the pages that the sequence's table names, a
//     scalar load each, one super-step ahead.  The rows are tree nodes, or (chain) consecutive positions of a prompt.
//     With a window, the keys of a workgroup are its sinks and one run of slots; both start at multiples of 32 and are
//     numbered through, so pieces, steps and the ring do not know of the gap.
//     (32 heads on 60 nodes behind 3136 slots: 20.9 us, 18.1 from one slab, of which the pieces' rows in fp32 are 1.1; one
//     token of 32 heads on 4 sequences with 1028 keys in sight 13.0 us from HBM, nearly all of it latency: lengths, table,
//     ring, exchange, merge.  10 to 42 scalar registers spill to lanes of vector registers, with up to
//     16 accesses in the loop over steps.)
//   * Over pages of 8 bits (E8) the ring holds codes and, beside it, a step's four scale bytes; they become bf16 on the way from
//     LDS into the products, so that a ring of the same size is twice as deep.  Keys in other rows than the bf16 build's (key_row) let
//     the 8-bit transposing reads deliver values in the order of the probabilities.  The keys of a batch may also be spread
//     over all workgroups in pieces of one length, merged by a second launch (SpreadPlan).
#pragma once

#include "kernels.h"

#include <math.h>
#include <type_traits>

namespace dreams {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <bool E8>
using Args = std::conditional_t<E8, AttnArgs8, AttnArgs>;

constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kStep = 32;          // keys per step
constexpr int kSpreadMinSteps = 4; // steps of a piece of spread keys, at least
constexpr float kLazyLog2 = 8.0f;  // slack of the running maximum, log2 units

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Attention entropy from a row's softmax state.  With scores z in log2 units, a reference m, l = sum 2^(z-m)
// and e = sum 2^(z-m) (z-m), the row's probabilities are 2^(z-m)/l and its entropy (nats) is
// ln2 * (log2 l - e/l).  Re-referencing a state to M (weight w = 2^(m-M)) turns e into w (e + (m-M) l).
__device__ __forceinline__ float ent_term(float w, float e, float m, float M, float l) {
  return w == 0.f ? 0.f : w * fmaf(m - M, l, e);
}
__device__ __forceinline__ float row_entropy(float l, float e) {
  return l > 0.f ? 0.69314718055994530942f * (__log2f(l) - e / l) : 0.f;
}

// 8 codes of e4m3 as bf16, the first four times one power of two, the others times another
__device__ __forceinline__ bf16x8 decode8(uint32_t lo, uint32_t hi, float scale_lo, float scale_hi) {
  bf16x8 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16x2 y = i == 0   ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale_lo, false)
                     : i == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale_lo, true)
                     : i == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale_hi, false)
                              : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale_hi, true);
    x[2 * i] = y[0];
    x[2 * i + 1] = y[1];
  }
  return x;
}

typedef __attribute__((address_space(3))) void lds_void;
__device__ __forceinline__ uint32_t lds_addr(const void* p) { return (uint32_t)(uintptr_t)(lds_void*)p; }

// Wave-wide copies from global memory into LDS.  m0 (wave-uniform) is the LDS byte address of lane 0's
// data; lane l's data lands at m0 + 16*l (dwordx4) or m0 + 4*l (dword).  The 16-byte copies move data that
// is read exactly once (queries, keys, values) and carry the non-temporal hint.
__device__ __forceinline__ void copy16_to_lds(uint32_t m0, const void* src) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"s"(m0), "v"(src) : "memory");
}
// Same, addressed as a wave-uniform base plus a per-lane 32-bit byte offset.
__device__ __forceinline__ void copy16_to_lds(uint32_t m0, const void* sbase, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(m0), "v"(voff), "s"(sbase)
               : "memory");
}
__device__ __forceinline__ void copy4_to_lds(uint32_t m0, const void* src) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(m0), "v"(src) : "memory");
}
// N copies to consecutive KB from m0 on, from one base: the instructions' offsets count on both sides, so voff[j % 2] are those
// of rows that lie as in the first (two) KB.
template <int N>
__device__ __forceinline__ void copy_run_to_lds(uint32_t m0, const void* sbase, const uint32_t (&voff)[2]) {
  static_assert(N == 2 || N == 4);
  if constexpr (N == 2)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3 nt\n\t"
                 "global_load_lds_dwordx4 %2, %3 offset:1024 nt" ::"s"(m0), "v"(voff[0]), "v"(voff[1]), "s"(sbase) : "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3 nt\n\t"
                 "global_load_lds_dwordx4 %2, %3 offset:1024 nt\n\tglobal_load_lds_dwordx4 %1, %3 offset:2048 nt\n\t"
                 "global_load_lds_dwordx4 %2, %3 offset:3072 nt" ::"s"(m0), "v"(voff[0]), "v"(voff[1]), "s"(sbase) : "memory");
}
// At most N of this wave's vector-memory operations still outstanding (they complete in issue order).
template <int N>
__device__ __forceinline__ void wait_vm() {
  static_assert(N >= 0 && N <= 63, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// wait_vm<PER * k> for a run-time k in [0, K]
template <int PER, int K>
__device__ __forceinline__ void wait_vm_steps(int k) {
  if constexpr (K > 0) {
    if (k >= K) {
      wait_vm<PER * K>();
      return;
    }
    wait_vm_steps<PER, K - 1>(k);
  } else {
    wait_vm<0>();
  }
}
// Workgroup barrier after this wave's LDS reads and writes have completed; outstanding copies stay in
// flight (a __syncthreads() would also wait for them).  The wait is the compiler's own instruction
// (vmcnt and expcnt at their maxima, lgkmcnt 0), so its wait-count bookkeeping knows that every LDS read
// issued before the barrier has returned.
__device__ __forceinline__ void barrier_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Row layout in LDS: rows of D bf16, unpadded; the 16-byte chunk c of row r sits at position c ^ swz(r),
// which spreads the 16 rows one operand read touches over distinct banks.  The swizzle repeats every 16
// rows.  A step slot holds 32 K rows then 32 V rows; the query rows use the same layout.
template <int D>
struct Rows {
  static constexpr int ROW = D * 2;           // bytes per row
  static constexpr int CPR = D / 8;           // 16-byte chunks per row
  static constexpr int RPL = 256 / ROW;       // rows per 256-byte bank line
  static constexpr int HALF = kStep * ROW;    // bytes of the K (or V) part of a step
  static constexpr int SLOT = 2 * HALF;       // bytes of a step
  static constexpr int C16 = 16 * ROW / 1024; // wave-wide 1 KB copies per 16 rows
  // D = 128 (one row per 256-byte bank line): gfx950 serves a 16-byte read (ds_read_b128) in groups of lanes
  // and a transposing 8-byte read (ds_read_b64_tr_b16) in two halves of 32 lanes over 64 banks.  The key
  // reads touch rows (m%4)*4 + m/4 at one chunk, the value reads rows 4j+q, q in {0,1} (or {2,3}), at an
  // aligned pair of chunks; swz(r) = 4*((r/4)%4) + 2*(r%2) + 1 puts both on distinct banks (measured: 213 and
  // 165 B/clk per compute unit, against 126 and 122 with r % 16).  D = 64: two rows per bank line.
  __device__ static __forceinline__ int swz(int r) {
    if constexpr (D == 128) return ((r >> 2) & 3) * 4 + (r & 1) * 2 + 1;
    return (r / RPL) % CPR;
  }
  __device__ static __forceinline__ int off(int r, int c) { return r * ROW + ((c ^ swz(r)) << 4); }
};

// The same for keys and values in 8 bits (E8): rows of D codes, 16 to a chunk.  A key read takes one chunk of 16 rows, a
// transposing value read (ds_read_b64_tr_b8) one chunk of 8 rows a quad, in halves of two quads: 16 rows that differ modulo
// 16 (key_row).  swz is a bijection over the rows of a bank line's parity (D = 64: residue modulo 4) that also keeps rows 0..3
// and 12..15 at one chunk apart from 4..11 at its neighbour, as a 16-byte read's groups of lanes mix them.
template <int D>
struct Rows8 {
  static constexpr int ROW = D, CPR = D / 16, RPL = 256 / ROW, HALF = kStep * ROW, SLOT = 2 * HALF, C16 = 16 * ROW / 1024;
  __device__ static __forceinline__ int swz(int r) {
    if constexpr (D == 128) return (r >> 1) & 7;
    return (0x78 >> (2 * ((r >> 2) & 3))) & 3;
  }
  __device__ static __forceinline__ int off(int r, int c) { return r * ROW + ((c ^ swz(r)) << 4); }
};
// The key of a step that operand row m of its block kb holds.
__device__ __forceinline__ int key_row(int kb, int m) { return kb * 16 + (m ^ (8 * kb)); }

// Bytes into LDS (zero-extended to 32 bits), lane l's from src + voff to m0 + 4 l, by the lanes that call it.
__device__ __forceinline__ void copy_byte_to_lds(uint32_t m0, const void* src, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ubyte %1, %2" ::"s"(m0), "v"(voff), "s"(src) : "memory");
}

// Merge of a set's pieces for rows [r0, r0 + nrows) of the set, in piece order (so the result does not
// depend on which piece finished last): out = sum_s w_s l_s o_s / sum_s w_s l_s, w_s = 2^(m_s - max_s m_s).
// Every piece's rows come from this XCD's L2 (not from this compute unit's L1, which has never held them):
// non-temporal 16-byte loads, a row's pieces side by side, whole 128-byte lines.  The loads are issued
// unconditionally (addresses clamped into the set), so that all of them are in flight together (loads under a
// branch are each waited for before the branch joins); waves with no row of the slice skip it.  Rows at or
// past rows_valid are not written.  good = false writes NaN rows (a failed wait).  PT: type of the pieces' rows (paged calls
// keep them in fp32: 64 rows of 32 heads in 8 pieces are 8 MB in L2 instead of 4, and the output is rounded once less).
template <int D, int W, bool ENT, typename PT>
__device__ __forceinline__ void merge_pieces(const AttnArgs& a, size_t prow0, int R, __bf16* out_rows, float* lse_rows,
                                             float* ent_rows, int rows_valid, int r0, int nrows, bool good) {
  constexpr int CPR = D / 8;
  constexpr int PCH = 8;    // pieces per batch of loads
  typedef __bf16 bf16x8m __attribute__((ext_vector_type(8)));
  typedef PT ptx8 __attribute__((ext_vector_type(8)));
  const PT* const part_o = (const PT*)a.part_o;
  const int S = a.splits;
  const int items = nrows * CPR;
  const int wave = (int)threadIdx.x >> 6;
  for (int base = 0; base < items; base += 64 * W) {
    if (base + 64 * wave >= items) break;   // (wave-uniform) nothing left for this wave
    const int item = base + (int)threadIdx.x;
    const int ch = item % CPR;
    const bool live = item < items && r0 + item / CPR < rows_valid;
    const int rl = min(r0 + item / CPR, R - 1);   // (a dead item's loads stay inside the set)
    float M = -INFINITY, lsum = 0.f, esum = 0.f;
    float acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    for (int s0 = 0; s0 < S; s0 += PCH) {
      f32x2 ml[PCH];
      float ev[PCH];
      ptx8 x[PCH];
#pragma unroll
      for (int k = 0; k < PCH; ++k) {
        const size_t pr = prow0 + (size_t)min(s0 + k, S - 1) * R + rl;
        ml[k] = __builtin_nontemporal_load((const f32x2*)(a.part_ml + 2 * pr));
        ev[k] = ENT ? __builtin_nontemporal_load(a.part_e + pr) : 0.f;
        x[k] = __builtin_nontemporal_load((const ptx8*)(part_o + pr * D + ch * 8));
      }
      float Mn = M;
#pragma unroll
      for (int k = 0; k < PCH; ++k)
        if (s0 + k < S) Mn = fmaxf(Mn, ml[k].x);
      const float scale_old = M == -INFINITY ? 0.f : fast_exp2(M - Mn);
      if (ENT) esum = ent_term(scale_old, esum, M, Mn, lsum);
      lsum *= scale_old;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] *= scale_old;
#pragma unroll
      for (int k = 0; k < PCH; ++k) {
        const float w = (s0 + k >= S || ml[k].x == -INFINITY) ? 0.f : fast_exp2(ml[k].x - Mn);
        if (ENT) esum += ent_term(w, ev[k], ml[k].x, Mn, ml[k].y);
        const float wl = w * ml[k].y;
        lsum += wl;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = fmaf(wl, (float)x[k][e], acc[e]);
      }
      M = Mn;
    }
    if (!live) continue;
    const float inv = !good ? NAN : lsum > 0.f ? 1.0f / lsum : 0.f;
    bf16x8m res;
#pragma unroll
    for (int e = 0; e < 8; ++e) res[e] = (__bf16)(acc[e] * inv);
    *(bf16x8m*)(out_rows + (size_t)rl * D + ch * 8) = res;
    if (ch == 0) {
      const bool some = sizeof(PT) == 4 ? lsum != 0.f : lsum > 0.f;   // (paged: a NaN sum gives a NaN)
      if (lse_rows) lse_rows[rl] = !good ? NAN : some ? (M + __log2f(lsum)) * kLn2 : -INFINITY;
      if (ENT) ent_rows[rl] = !good ? NAN : row_entropy(lsum, esum);
    }
  }
}

// The set's merge, spread over its pieces.  One 64-bit counter word per set (fields at the kCtr*
// shifts): pieces started, pieces arrived, a bit per arrived piece, and the sum and the sum of squares of the
// started pieces' XCD ids.  A piece that arrives when its whole set has started waits for every arrival and
// merges its own slice of the rows: every piece it waits for is running and arrives without waiting for
// anything.  A piece that arrives earlier leaves; the piece whose start completed the set saw it among the
// arrived bits then, and merges its slice too (that piece arrives after the set is complete, so it never
// leaves).  So every wait ends, and each slice is merged once.  The last arrival puts the word back to zero
// for the next call; a waiting piece takes either the full count or that zero as the end of its wait.  The
// pieces' rows are read from this XCD's L2: all pieces of a set share blockIdx % 8, and consecutive
// workgroups of a dispatch go to consecutive XCDs (which XCD takes workgroup 0 differs, e.g. between direct
// and graph launches).  A merging piece checks that: S ids whose sum is S x and sum of squares S x^2 all
// equal x, this piece's own.
template <int D, int W, bool ENT, typename PT>
__device__ __forceinline__ void merge_set(const AttnArgs& a, size_t pset, int R, int split, unsigned long long start_old,
                                          size_t orow0, int rows_valid, uint32_t* merge_lds, uint32_t* good_lds) {
  const int S = a.splits, tid = threadIdx.x;
  const size_t prow0 = pset * S * R;   // the set's piece 0, row 0
  unsigned long long* ctr = a.set_ctr + pset * a.ctr_stride;
  wait_vector_memory();   // this piece's rows have reached the L2
  __syncthreads();
  if (tid == 0) {
    const unsigned long long old = __hip_atomic_fetch_add(
        ctr, (1ull << kCtrArrived) | (1ull << (kCtrMask + split)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const unsigned long long cnt = (1ull << kCtrCountBits) - 1;
    const bool coop = (old & cnt) == (unsigned long long)S;
    const bool last = ((old >> kCtrArrived) & cnt) == (unsigned long long)(S - 1);
    bool good = true;
    if (coop) {
      const unsigned long long x = xcd_id();
      const unsigned long long sum = (old >> kCtrXcdSum) & ((1ull << (kCtrXcdSq - kCtrXcdSum)) - 1);
      const unsigned long long sq = old >> kCtrXcdSq;
      if (sum != S * x || sq != S * x * x) {
        raise_device_error(a.err, kErrXcdSplit);
        good = false;
      }
    }
    if (last) {
      __hip_atomic_store(ctr, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    } else if (coop) {
      const uint64_t t0 = __builtin_amdgcn_s_memrealtime();
      for (;;) {
        const unsigned long long now = __hip_atomic_load(ctr, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (((now >> kCtrArrived) & cnt) == (unsigned long long)S || (now & cnt) == 0ull) break;
        if (__builtin_amdgcn_s_memrealtime() - t0 > a.wait_ticks) {
          raise_device_error(a.err, kErrWaitTimeout);
          good = false;
          break;
        }
        __builtin_amdgcn_s_sleep(1);
      }
    }
    // slices this workgroup merges: its own (when it waited), and those of the pieces that left before this
    // piece's start completed the set
    uint32_t slices = coop ? 1u << split : 0u;
    if ((start_old & cnt) == (unsigned long long)(S - 1))
      slices |= (uint32_t)(start_old >> kCtrMask) & (uint32_t)((1ull << S) - 1);
    *merge_lds = slices;
    *good_lds = good ? 1u : 0u;
  }
  __syncthreads();
  const uint32_t slices = *merge_lds;
  for (int k = 0; k < S; ++k) {
    if (!((slices >> k) & 1u)) continue;
    const int r0 = k * R / S, r1 = (k + 1) * R / S;
    merge_pieces<D, W, ENT, PT>(a, prow0, R, (__bf16*)a.out + orow0 * D, a.lse ? a.lse + orow0 : nullptr,
                            ENT ? a.entropy + orow0 : nullptr, rows_valid, r0, r1 - r0, *good_lds == 1u);
  }
}

// Pieces of one length over every sequence (spread_wgs), so that a batch's long sequences take no longer than its short
// ones and the units need not be as many as the dies: lane b holds sequence b's steps and pieces.  The length is the
// smallest of 64 candidates (from what the workgroups would need without rounding up, 1/24 of it apart) with no more pieces
// than workgroups.  Every wave that asks computes the same.
struct SpreadPlan {
  int steps, pieces;    // of the lane's sequence; pieces of one KV head
  int piece;            // steps of a piece
};
__device__ __forceinline__ int ceil_div(int x, int y, float inv) {   // x >= 1, y >= 1, inv near 1 / y
  int q = (int)((float)(x - 1) * inv);
  int r = x - 1 - q * y;
  q += r >= y ? 1 : 0;
  q -= r < 0 ? 1 : 0;
  return q + 1;
}
__device__ __forceinline__ SpreadPlan spread_plan(const AttnArgs8& a, int lane) {
  SpreadPlan sp;
  sp.steps = 0;
  if (lane < a.B) {
    int nb = a.T;
    if (a.chain && a.row_len) nb = min(max(a.row_len[lane], 0), a.T);
    const int Lp = min(max(a.kv_len[lane], 0), a.S_cap - nb);
    const int N = nb > 0 ? Lp + nb : 0;
    int gap = 0;
    if (a.window > 0 && N > 0) {
      const int low = max(Lp - a.window + 1, 0);
      gap = max(low / kStep * kStep - (min(a.sinks, low) + kStep - 1) / kStep * kStep, 0);
    }
    sp.steps = max((N - gap + kStep - 1) / kStep, 1);    // (a sequence without keys has its rows' zeros to write)
  }
  uint32_t total = (uint32_t)sp.steps;      // (64 sequences of 2^25 steps at most)
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) total += (uint32_t)__shfl_xor((int)total, off);
  const int even = (int)(((long long)total * a.Hkv + a.spread_wgs - 1) / a.spread_wgs);
  const int base = max(even, kSpreadMinSteps), mine = base + (int)((long long)base * lane / 24);
  const float inv = 1.0f / (float)mine;
  long long count = 0;
  for (int b = 0; b < a.B; ++b) count += ceil_div(__builtin_amdgcn_readlane(sp.steps, b), mine, inv);
  const uint64_t fits = __ballot(count * a.Hkv <= a.spread_wgs);
  sp.piece = __builtin_amdgcn_readlane(mine, fits ? __builtin_ctzll(fits) : 63);
  sp.pieces = sp.steps > 0 ? ceil_div(sp.steps, sp.piece, 1.0f / (float)sp.piece) : 0;
  return sp;
}

// LDS of a workgroup: the ring, the query rows when they sit beside it, the ancestor sets and the tree as
// copied (static), and a few words; WPC workgroups share a compute unit's 160 KB.
// (E8: steps of half the bytes, and a word for each of a step's four scales)
template <int D, int NST, int WPC, bool E8>
constexpr bool q_beside_ring(int R) {
  return (size_t)NST * (E8 ? Rows8<D>::SLOT + 16 : Rows<D>::SLOT) + (size_t)R * D * 2 + 4 * kMaxNodes * 8 + 64 <=
         160 * 1024 / WPC;
}
template <int D, int NST, int WPC, bool E8>
constexpr size_t dynamic_lds(int R) {
  return (size_t)NST * (E8 ? Rows8<D>::SLOT : Rows<D>::SLOT) + (q_beside_ring<D, NST, WPC, E8>(R) ? (size_t)R * D * 2 : 0);
}

// WPC: workgroups meant to share a compute unit (their waves share each SIMD, so the register budget is that
// of WPC * W / 4 waves per SIMD).
// E8 (paged): keys and values in e4m3 with a power-of-two scale for 16 slots of a head.  The ring holds their codes, and
// they become bf16, exactly, in registers (v_cvt_scalef32_pk_bf16_fp8, the scale's exponent in the same instruction): a
// step's 64 conversions a wave run beside its 16 RB products.
// WIDE (E8): pages of 32 slots or more, so that a step's keys lie in one.
template <int D, int RB, int KW, int W, int NST, bool PIPE, bool ENT, int WPC, bool PAGED, bool E8 = false, bool WIDE = false>
__global__ __launch_bounds__(64 * W, WPC * W / 4) void tree_attn_bf16_kernel(Args<E8> a) {
  constexpr int WR = W / KW;          // waves per key group; each owns a different slice of the rows
  constexpr int RW = 16 * RB;         // query rows per wave
  constexpr int R = WR * RW;          // query rows per workgroup
  constexpr int DS = D / 32;          // k-steps of S^T = K Q^T
  constexpr int DB = D / 16;          // 16-column blocks of O^T
  using L = Rows<D>;                                      // query rows
  using V = std::conditional_t<E8, Rows8<D>, Rows<D>>;    // key and value rows
  static_assert(!E8 || PAGED, "8 bits: paged");
  constexpr int C16 = V::C16;         // wave-wide copies per 16 rows
  constexpr int NSS = NST / KW;       // ring slots in super-steps (KW consecutive steps, one per key group)
  // The query rows get an LDS region of their own beside the ring where it fits (so the first copies fill the
  // whole ring); otherwise they occupy the ring's last step slots until the prologue has read them.
  constexpr bool QSEP = q_beside_ring<D, NST, WPC, E8>(R);
  constexpr int QSLOTS = QSEP ? 0 : (R * L::ROW + V::SLOT - 1) / V::SLOT;   // step slots the query rows occupy
  constexpr int QSS = (QSLOTS + KW - 1) / KW;                                // ... in super-steps
  constexpr int CPS = 4 * KW * C16 / W;   // copies per wave per super-step (4*KW blocks of 16 rows)
  constexpr int QB = R / 16;          // 16-row blocks of query rows, dealt to the waves round-robin
  static_assert(W % KW == 0 && (NST & (NST - 1)) == 0 && NSS > QSS && NSS >= 2, "ring layout");
  static_assert(CPS * W == 4 * KW * C16 && CPS >= 1 && (C16 % CPS == 0 || CPS % C16 == 0), "copy split");
  static_assert(16 * V::ROW == C16 * 1024 && (E8 || (16 / L::RPL) % L::CPR == 0), "swizzle repeats every 16 rows");
  // ... with the scales' (one for a block's codes, or (WIDE) two blocks')
  constexpr int CPT = CPS + (WIDE ? CPS / (2 * C16) : E8 ? (CPS + C16 - 1) / C16 : 0);
  static_assert(!E8 || CPS % C16 == 0, "whole blocks");
  static_assert(!WIDE || (E8 && (CPS == 2 * C16 || CPS == 4 * C16)), "a wave's copies are of one step");
  static_assert(NSS * CPT + ((QB + W - 1) / W) * L::C16 + 8 <= 63, "outstanding copies fit the counter");
  static_assert((size_t)(KW - 1) * R * D * 4 + (size_t)KW * R * 12 <= (size_t)NST * V::SLOT, "group states fit the ring");

  extern __shared__ __attribute__((aligned(1024))) unsigned char ring[];   // NST step slots (+ the query rows)
  __shared__ uint64_t anc_lds[2 * kMaxNodes];
  __shared__ uint64_t meta_lds[2 * kMaxNodes];   // the sequence's parents or tree mask rows, as copied
  __shared__ uint32_t merge_lds;                  // slices of the set's rows this workgroup merges
  __shared__ uint32_t good_lds;                   // 0: a wait gave up (the merged rows are written as NaN)
  __shared__ int par_lds[PAGED ? kMaxNodes : 1];      // paged, mask and window: the parents
  __shared__ int depth_lds[PAGED ? kMaxNodes : 1];    // paged, window: the nodes' depths
  __shared__ __attribute__((aligned(16))) uint32_t scale_lds[E8 ? NST * 4 : 1];   // a step's scale bytes: 2 K, 2 V

  // ---- work item
  const int n = blockIdx.x;
  const int xcd = n & 7, slot = n >> 3;
  int u, split, rg;
  [[maybe_unused]] int spread_pieces = 0, spread_piece = 0;   // (spread: the unit's pieces, steps of one)
  bool placed = false;
  if constexpr (E8) {
    placed = a.spread_wgs > 0;
    if (placed) {
      const SpreadPlan sp = spread_plan(a, threadIdx.x & 63);
      int first = 0, seq = 0, pieces = 0;
      for (; seq < a.B; ++seq) {
        pieces = __builtin_amdgcn_readlane(sp.pieces, seq);
        if (n < first + pieces * a.Hkv) break;
        first += pieces * a.Hkv;
      }
      if (seq == a.B) return;
      split = (n - first) / a.Hkv;      // (a piece's heads beside one another, as in the pages)
      u = seq * a.Hkv + (n - first) - split * a.Hkv;
      rg = 0;
      spread_pieces = pieces;
      spread_piece = sp.piece;
    }
  }
  if (placed) {
  } else if constexpr (PAGED) {
    // Every unit's row groups are dealt to unit_parts parts (units * unit_parts is a multiple of 8, or, E8, rounded up to
    // one), a part to an XCD.
    // An XCD takes the q-th row group of all of its parts before the next.
    const int here = (a.units * a.unit_parts + (E8 ? 7 : 0)) / 8;
    const int q = slot / (here * a.splits), rest = slot - q * (here * a.splits);
    const int vu = xcd + 8 * (rest / a.splits);
    split = rest - (rest / a.splits) * a.splits;
    u = vu / a.unit_parts;
    rg = q * a.unit_parts + (vu - u * a.unit_parts);
    if (rg >= a.row_groups || (E8 && u >= a.units)) return;
  } else {
    const int per_unit = a.splits * a.row_groups;
    u = xcd + 8 * (slot / per_unit);
    if (u >= a.units) return;
    const int within = slot - (slot / per_unit) * per_unit;
    split = within / a.row_groups;
    rg = within - split * a.row_groups;
  }
  const int b = u / a.Hkv, g = u - b * a.Hkv;
  const int tid = threadIdx.x, lane = tid & 63, quad = lane >> 4, col = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kw = wave / WR, rh = wave - kw * WR;   // key group; row slice [rh*RW, rh*RW + RW)
  const int T = a.T;
  const int rows_total = a.G * T;
  const uint32_t ring_lds = __builtin_amdgcn_readfirstlane(lds_addr(ring));
  const uint32_t scale_base = E8 ? __builtin_amdgcn_readfirstlane(lds_addr(scale_lds)) : 0;
  const int kv_len_b = a.kv_len[b];   // issued before the copies below, ahead of their traffic

  // ---- the workgroup's rows: [row_base, row_base + rows_here) of the unit's rows_total
  int row_base = rg * R, rows_here = rows_total - rg * R;
  // Paged: the slots that its rows see, as a prefix length and the sequence's end, the sinks' slots (rounded up to
  // steps) and the gap behind them.
  int Lp_paged = 0, N_paged = 0, low = 0, sink_end = 0, sink_steps = 0, gap = 0, nb = T;
  int i_first = 0, i_last = 0;   // chain: the first and last position of the workgroup's rows
  if constexpr (PAGED) {
    rows_here = min(rows_here, R);
    if (a.chain && a.row_len) nb = min(max(a.row_len[b], 0), T);
    Lp_paged = min(max(kv_len_b, 0), a.S_cap - nb);
    int first_row = 0;     // the lowest position of a row, from the prefix on
    N_paged = Lp_paged + T;
    if (a.chain) {
      const int i0 = row_base % T;
      i_first = i0 + rows_here <= T ? i0 : 0;
      i_last = min(i0 + rows_here <= T ? i0 + rows_here - 1 : T - 1, nb - 1);
      first_row = i_first;
      N_paged = i_last >= i_first ? Lp_paged + i_last + 1 : 0;
    }
    if (a.window > 0 && N_paged > 0) {
      low = max(Lp_paged + first_row - a.window + 1, 0);
      sink_end = min(a.sinks, low);
      sink_steps = (sink_end + kStep - 1) / kStep * kStep;
      gap = max(low / kStep * kStep - sink_steps, 0);
    }
  }
  // the slot of a key number (a multiple of kStep, or within its step)
  auto slot_of = [&](int key) {
    if constexpr (PAGED) return key < sink_steps ? key : key + gap;
    return key;
  };

  // ---- this workgroup's piece of the key axis, planned from the host's bound on the key count, or (several
  // sequences of different lengths) from this sequence's own count, so that a short sequence's pieces are
  // shorter rather than its last piece nearly empty; the first copies then wait for its length
  int keys = a.max_keys;
  if constexpr (PAGED) keys = N_paged - gap;
  else if (a.piece_by_len) keys = min(max(kv_len_b, 0), a.S_cap - T) + T;
  int piece = (keys + a.splits - 1) / a.splits, last = a.splits - 1;
  piece = (piece + kStep - 1) / kStep * kStep;
  if constexpr (E8) {
    if (placed) {
      piece = spread_piece * kStep;
      last = spread_pieces - 1;
    }
  }
  const int k_begin = split * piece;
  const int k_end_plan = split == last ? keys : min(keys, k_begin + piece);
  const int nplan = k_end_plan > k_begin ? (k_end_plan - k_begin + kStep - 1) / kStep : 0;
  const int nsp = (nplan + KW - 1) / KW;
  const size_t head_off = PAGED ? ((size_t)g << a.page_shift) * V::ROW : (size_t)u * a.S_cap * V::ROW;
  const unsigned char* kbase = (const unsigned char*)a.k + head_off;
  const unsigned char* vbase = (const unsigned char*)a.v + head_off;

  // Per-lane byte offsets of the copies of 16 consecutive rows: copy j, lane l brings row r = (j*1024 +
  // 16*l) / ROW, position p = l % CPR, i.e. the global chunk p ^ swz(r) of that row.
  uint32_t coff[C16];
#pragma unroll
  for (int j = 0; j < C16; ++j) {
    const int e = j * 64 + lane;
    const int r = e / V::CPR, p = e - r * V::CPR;
    coff[j] = (uint32_t)(r * V::ROW + ((p ^ V::swz(r)) << 4));
  }
  // A super-step is KW steps x (32 K rows + 32 V rows) = 4*KW blocks of 16 rows = 4*KW*C16 wave-wide 1 KB
  // copies; wave w issues copies w*CPS .. w*CPS + CPS - 1 (copy ci: block bi = ci / C16 -- step bi/4 of the
  // super-step, K or V part (bi/2)%2, rows 16*(bi%2).. -- and copy ci % C16 of that block), in groups of
  // GRP = min(CPS, C16) copies that share a block.
  constexpr int GRP = CPS < C16 ? CPS : C16;
  constexpr int NGRP = CPS / GRP;
  // Paged: the pages of this wave's next super-step to copy, looked up a super-step ahead (scalar loads: the constant
  // address space, so that no vector load and no wait for one comes between the copies).
  typedef const __attribute__((address_space(4))) int32_t* const_table;
  int next_page[PAGED && !WIDE ? NGRP : 1];
  auto group_slot = [&](int jj, int t) {
    const int bi = (wave * CPS + t * GRP) / C16;
    return slot_of(k_begin + (jj * KW + (bi >> 2)) * kStep) + 16 * (bi & 1);
  };
  auto look_up = [&](int jj) {
    if constexpr (PAGED) {
      const const_table table = (const_table)(uintptr_t)(a.table + (size_t)b * a.width);
#pragma unroll
      for (int t = 0; t < (WIDE ? 1 : NGRP); ++t) next_page[t] = table[min(group_slot(jj, t) >> a.page_shift, a.width - 1)];
    }
  };
  auto issue_group = [&](int jj, int t) {
    const uint32_t sbase = ring_lds + (jj & (NSS - 1)) * KW * V::SLOT;
    const int ci0 = wave * CPS + t * GRP;
    const int bi = ci0 / C16, j0 = ci0 - bi * C16;
    const int sis = bi >> 2, part = (bi >> 1) & 1, half = bi & 1;
    const int key0 = k_begin + (jj * KW + sis) * kStep + 16 * half;
    const unsigned char* pbase = part ? vbase : kbase;
    const uint32_t dst = sbase + sis * V::SLOT + part * V::HALF + half * C16 * 1024;
    if constexpr (PAGED) {
      // (a page outside the pool, or past the table: some page of the pool, whose rows no one sees)
      const int page = min(max(next_page[t], 0), a.num_pages - 1);
      const int row = group_slot(jj, t) & ((1 << a.page_shift) - 1);
      const unsigned char* src = pbase + (int64_t)page * a.page_stride + (int64_t)row * V::ROW;
#pragma unroll
      for (int j = 0; j < GRP; ++j) copy16_to_lds(dst + (j0 + j) * 1024, src, coff[j0 + j]);
      if constexpr (E8) {
        const uint8_t* byte = (part ? a.v_scale : a.k_scale) + (int64_t)page * a.scale_stride +
                              (int64_t)((((size_t)g << a.page_shift) + row) / kScaleBlock);
        const uint32_t at = scale_base + ((jj & (NSS - 1)) * KW + sis) * 16 + part * 8 + half * 4;
        if (lane == 0) copy_byte_to_lds(at, byte, 0u);
      }
    } else if (key0 + 16 <= a.S_cap) {
      const unsigned char* src = pbase + (size_t)key0 * L::ROW;
#pragma unroll
      for (int j = 0; j < GRP; ++j) copy16_to_lds(dst + (j0 + j) * 1024, src, coff[j0 + j]);
    } else {  // rows past the cache capacity repeat its last row
#pragma unroll
      for (int j = 0; j < GRP; ++j) {
        const int r = ((j0 + j) * 64 + lane) / L::CPR;
        const int key = min(key0 + r, a.S_cap - 1);
        copy16_to_lds(dst + (j0 + j) * 1024, pbase + (size_t)key * L::ROW + (coff[j0 + j] - r * L::ROW));
      }
    }
  };
  // WIDE: the 32 key rows or value rows (or both) of a step that are this wave's are one run of their page, and so are
  // their two scales: one look-up, one offset.  (With those for every 16 rows, 12 sequences x 28 heads of 64 columns behind 774
  // to 7740 slots 72 us instead of 59, 8 x 8 of 128 behind 16384 to 32768 76.9 instead of 74.8, 8 x 32 heads x 60 nodes behind
  // 2000 47.5 instead of 43.7.)
  auto issue_run = [&]([[maybe_unused]] int jj) {
    if constexpr (WIDE) {
      const uint32_t slot_at = (jj & (NSS - 1)) * KW;
      const int sis = wave * CPS / C16 >> 2;
      const int page = min(max(next_page[0], 0), a.num_pages - 1);
      const int row = group_slot(jj, 0) & ((1 << a.page_shift) - 1);
      const int64_t off = (int64_t)page * a.page_stride + (int64_t)row * V::ROW;
      const int64_t scale_off = (int64_t)page * a.scale_stride + (((int64_t)g << a.page_shift) + row) / kScaleBlock;
      const uint32_t voff[2] = {coff[0], C16 == 2 ? coff[C16 - 1] - 1024 : coff[0]};
#pragma unroll
      for (int t = 0; t < CPS / (2 * C16); ++t) {
        const int part = (wave * CPS / C16 >> 1 & 1) + t;
        copy_run_to_lds<2 * C16>(ring_lds + (slot_at + sis) * V::SLOT + part * V::HALF, (part ? vbase : kbase) + off, voff);
        if (lane < 2) copy_byte_to_lds(scale_base + (slot_at + sis) * 16 + part * 8, (part ? a.v_scale : a.k_scale) + scale_off, lane);
      }
    }
  };
  auto issue_super = [&](int jj) {
    if constexpr (WIDE) {
      issue_run(jj);
    } else {
#pragma unroll
      for (int t = 0; t < NGRP; ++t) issue_group(jj, t);
    }
    look_up(jj + 1);
  };

  // ---- first copies: the query rows (into the last step slots), the tree (wave 0), then the ring
  const size_t qrow0 = ((size_t)b * a.Hq + (size_t)g * a.G) * T;   // row 0 of this KV head's query rows
  const unsigned char* qslab = QSEP ? ring + NST * V::SLOT : ring + (NST - QSLOTS) * V::SLOT;
#pragma unroll
  for (int qb = wave; qb < QB; qb += W) {
#pragma unroll
    for (int j = 0; j < L::C16; ++j) {
      const int r = (j * 64 + lane) / L::CPR;
      const int row = PAGED ? row_base + min(qb * 16 + r, rows_here - 1) : min(rg * R + qb * 16 + r, rows_total - 1);
      if constexpr (E8)
        copy16_to_lds(lds_addr(qslab) + (qb * L::C16 + j) * 1024,
                      (const unsigned char*)a.q + (qrow0 + row) * L::ROW + ((((j * 64 + lane) % L::CPR) ^ L::swz(r)) << 4));
      else
        copy16_to_lds(lds_addr(qslab) + (qb * L::C16 + j) * 1024,
                      (const unsigned char*)a.q + (qrow0 + row) * L::ROW + (coff[j] - r * L::ROW));
    }
  }
  const int Wm = (T + 63) / 64;
  if (wave == 0 && !(PAGED && a.chain)) {
    const uint32_t mdst = lds_addr(meta_lds);
    if (PAGED && a.mask && a.window > 0) {   // the depths' parents, beside the mask rows
      const int32_t* src = a.parent + (size_t)b * T;
      for (int c = 0; c * 64 < T; ++c) copy4_to_lds(lds_addr(par_lds) + c * 256, src + min(c * 64 + lane, T - 1));
    }
    if (a.mask) {
      const int nd = 2 * T * Wm;   // dwords of this sequence's mask rows
      const uint32_t* src = (const uint32_t*)(a.mask + (size_t)b * T * Wm);
      for (int c = 0; c * 64 < nd; ++c) copy4_to_lds(mdst + c * 256, src + min(c * 64 + lane, nd - 1));
    } else {
      const int32_t* src = a.parent + (size_t)b * T;
      for (int c = 0; c * 64 < T; ++c) copy4_to_lds(mdst + c * 256, src + min(c * 64 + lane, T - 1));
    }
  }
  // (paged: super-steps are issued one after another, none twice, so that the look-ups stay one ahead)
  constexpr int FIRST = PAGED && !PIPE && QSS == 0 ? NSS - 1 : NSS - QSS;
  const int fa = min(FIRST, nsp);
  look_up(0);
  for (int j = 0; j < fa; ++j) issue_super(j);
  // This piece has started (the merge at the end relies on knowing that every piece of the set runs), on the
  // XCD it adds to the set's sums.  The counter's value before this start is kept (thread 0) until the
  // epilogue: the piece that starts last finds there the pieces that arrived before the whole set was running,
  // whose rows it then merges.
  unsigned long long start_old = 0;
  if (a.splits > 1 && tid == 0) {
    const unsigned long long x = xcd_id();
    start_old = __hip_atomic_fetch_add(a.set_ctr + ((size_t)u * a.row_groups + rg) * a.ctr_stride,
                                       1ull | (x << kCtrXcdSum) | ((x * x) << kCtrXcdSq), __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
  }

  // ---- prologue: prefix length, ancestor sets, queries (all overlapping the copies above)
  int Lp = kv_len_b;
  Lp = Lp < 0 ? 0 : (Lp > a.S_cap - T ? a.S_cap - T : Lp);
  if constexpr (PAGED) Lp = Lp_paged;
  const int N = PAGED ? N_paged : Lp + T;
  // the last piece runs to this sequence's true end, whatever the host's bound said
  const int k_end = split == last ? N - gap : min(N - gap, k_begin + piece);
  const int nact = k_end > k_begin ? (k_end - k_begin + kStep - 1) / kStep : 0;
  const int nsa = (nact + KW - 1) / KW;

  wait_vm_steps<CPT, NSS - QSS>(fa);   // this wave's query rows and the tree have landed
  barrier_lds();
  // Only a piece that reaches the tree slots consults ancestor sets (a step before them has key < L_b
  // everywhere, and a masked step past k_end hides its keys whatever the sets say).
  bool need_anc = k_end > Lp;
  if constexpr (PAGED) need_anc = !a.chain && (k_end + gap > Lp || a.window > 0);
  if constexpr (PAGED) {
    if (need_anc && a.window > 0) {
      if (tid < T) {
        const int* par = a.mask ? par_lds : (const int*)meta_lds;
        int j = tid, d = 0;
        for (; d < T; ++d) {
          const int p = par[j];
          if (p < 0 || p >= j) break;
          j = p;
        }
        depth_lds[tid] = d;
      }
      barrier_lds();
    }
  }
  if (need_anc && tid < T) {
    uint64_t m0 = 0, m1 = 0;
    if (a.mask) {
      const uint64_t* mr = meta_lds + tid * Wm;
      m0 = mr[0];
      m1 = Wm > 1 ? mr[1] : 0;
    } else {
      const int* par = (const int*)meta_lds;
      int j = tid;
      for (int st = 0; st <= T && j >= 0; ++st) {
        if (j < 64) m0 |= 1ull << j; else m1 |= 1ull << (j - 64);
        const int p = par[j];
        if (p >= j) break;  // not a valid parent: the walk ends here
        j = p;
      }
    }
    if constexpr (PAGED) {
      if (a.window > 0) {   // nodes out of a node's sight
        const int far = depth_lds[tid] - a.window;
        uint64_t* const words[2] = {&m0, &m1};
#pragma unroll
        for (int w = 0; w < 2; ++w)
          for (uint64_t rest = *words[w]; rest; rest &= rest - 1) {
            const int j = __builtin_ctzll(rest);
            const int d = 64 * w + j < T ? depth_lds[64 * w + j] : 0;
            if (d <= far && Lp + d >= a.sinks) *words[w] &= ~(1ull << j);
          }
      }
    }
    anc_lds[2 * tid] = m0;
    anc_lds[2 * tid + 1] = m1;
  }
  bf16x8 qf[RB][DS];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int ds = 0; ds < DS; ++ds) {
      // (E8: a lane's 16 codes of a key are 16 columns, of two products)
      const int chunk = E8 ? (ds >> 1) * 8 + quad * 2 + (ds & 1) : ds * 4 + quad;
      qf[rb][ds] = *(const bf16x8*)(qslab + L::off(rh * RW + rb * 16 + col, chunk));
    }
  // Scores are scaled by c = |scale| log2(e) > 0 inside the exponent (one fma per score); a negative scale
  // flips the sign of the queries instead (exact in bf16), a zero scale becomes the smallest normal float.
  const float c_scale = fmaxf(fabsf(a.scale_log2), 1.17549435e-38f);
  if (a.scale_log2 < 0.f) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int ds = 0; ds < DS; ++ds) qf[rb][ds] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, qf[rb][ds]) ^ 0x80008000u);
  }
  barrier_lds();   // ancestor sets written; every wave's query reads returned (their slots are reused next)
  uint64_t anc0[RB], anc1[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = PAGED ? row_base + min(rh * RW + rb * 16 + col, rows_here - 1)
                          : min(rg * R + rh * RW + rb * 16 + col, rows_total - 1);
    const int node = row % T;
    anc0[rb] = need_anc ? anc_lds[2 * node] : 0;
    anc1[rb] = need_anc ? anc_lds[2 * node + 1] : 0;
  }
  // Paged: the slots that a row sees: [0, sinks) and [see_from, ...), up to see_to (chain; -1: not a live row), or the
  // prefix and the ancestors' (tree).  plain_from, plain_to: a step inside is in sight of every row of the wave;
  // wave_to: its last row's own slot (chain).
  int see_from[RB], see_to[RB], plain_from = 0, plain_to = Lp, wave_to = N - 1;
  if constexpr (PAGED) {
    int deepest = 0;
    if (!a.chain && a.window > 0) {
      for (int j = lane; j < T; j += 64) deepest = max(deepest, depth_lds[j]);
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) deepest = max(deepest, __shfl_xor(deepest, off));
      deepest = __builtin_amdgcn_readfirstlane(deepest);
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int node = (row_base + min(rh * RW + rb * 16 + col, rows_here - 1)) % T;
      int pos = Lp;
      if (a.chain) pos += node;
      else if (a.window > 0) pos += depth_lds[node];
      see_from[rb] = a.window > 0 ? pos - a.window + 1 : 0;
      see_to[rb] = a.chain && node < nb ? pos : -1;
      if (a.chain && node >= nb) {   // (its queries may hold anything)
#pragma unroll
        for (int ds = 0; ds < DS; ++ds) qf[rb][ds] = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
      }
    }
    if (a.chain) {
      plain_to = Lp + i_first + 1;
      wave_to = Lp + i_last;
    }
    if (a.window > 0) plain_from = Lp + (a.chain ? i_last : deepest) - a.window + 1;
  }
  // Ring depth: the pipelined loop frees a super-step's slots at the barrier that follows its operand reads,
  // so every slot can hold a copy in flight; the plain loop keeps one slot for the super-step being read.
  constexpr int AHEAD = PIPE ? NSS : NSS - 1;
  const int fb = max(fa, min(AHEAD, nsa));
  for (int j = fa; j < fb; ++j) issue_super(j);
  // super-steps issued by this wave once the refill of iteration js - 1 is out
  auto issued_by = [&](int js) { return max(fa, min(js + AHEAD, nsa)); };

  f32x4 o[RB][DB];
  float m_run[RB], l_run[RB];
  float e_run[RB];   // entropy term: sum of p * (z - m) over the keys so far (ENT only)
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
    for (int d = 0; d < DB; ++d) o[rb][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run[rb] = -INFINITY;
    l_run[rb] = 0.f;
    e_run[rb] = 0.f;
  }

  const int ka_row = (col & 3) * 4 + (col >> 2);       // A row m holds key kb*16 + (m%4)*4 + m/4
  const int tr_row = (col >> 2) * 4 + quad;            // transposed read: 4 keys j*4+quad, 16 columns
  const int tr_c = (col & 3) >> 1, tr_half = (col & 1) * 8;

  // Key and value rows at or past the sequence end hold whatever the cache had there: the waves that copied
  // them zero them once their own copies have landed, so that no bit pattern (an infinity, a NaN) can reach
  // the products; their scores are then exactly the mask's -inf.
  auto zero_tail = [&](int jj) {
    unsigned char* sslot = ring + (jj & (NSS - 1)) * KW * V::SLOT;
#pragma unroll
    for (int t = 0; t < NGRP; ++t) {
      const int ci0 = wave * CPS + t * GRP;
      const int bi = ci0 / C16, j0 = ci0 - bi * C16;
      const int sis = bi >> 2, part = (bi >> 1) & 1, half = bi & 1;
      const int key0 = slot_of(k_begin + (jj * KW + sis) * kStep);
      // (paged: slots between the sinks and the run that some row sees, too)
      const bool before = PAGED && key0 < low && key0 + kStep > sink_end;
      if (key0 + kStep > N || before) {
        // the rows this wave's copies brought: 64*GRP lanes' worth of 16-byte chunks, rows j0*1024/ROW ..
        constexpr int RPG = GRP * 1024 / V::ROW;   // rows per group of copies
        constexpr int LPR = 64 / RPG;              // lanes per row
        constexpr int PER = V::CPR / LPR;          // chunks per lane
        const int r = 16 * half + j0 * 1024 / V::ROW + lane / LPR;
        if (key0 + r >= N || (before && key0 + r < low && key0 + r >= sink_end)) {
          unsigned char* vrow = sslot + sis * V::SLOT + part * V::HALF + r * V::ROW;
#pragma unroll
          for (int c = 0; c < PER; ++c) *(u32x4*)(vrow + ((lane % LPR) * PER + c) * 16) = u32x4{0u, 0u, 0u, 0u};
        }
      }
    }
  };

  // A step's operands: K fragments (A operand of S^T: A row m holds key kb*16 + (m%4)*4 + m/4) and V^T
  // fragments (A operand of O^T, transposing reads: lo = keys j*4+quad, hi = keys 16+j*4+quad, matching the
  // probabilities' slots).  All are issued together, so their LDS latencies overlap.
  struct Ops16 {
    bf16x8 kf[2][DS];
    s16x4 vlo[DB], vhi[DB];
  };
  struct Ops8 {
    u32x4 k[2][DS / 2];
    i32x2 v[DB];
    u32x4 scale;
  };
  using Ops = std::conditional_t<E8, Ops8, Ops16>;
  auto read_ops8 = [&](Ops8& op, int jj) {
    const unsigned char* tile = ring + ((jj & (NSS - 1)) * KW + kw) * V::SLOT;
    const unsigned char* vt = tile + V::HALF;
    op.scale = *(const u32x4*)(scale_lds + ((jj & (NSS - 1)) * KW + kw) * 4);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int x = 0; x < DS / 2; ++x) op.k[kb][x] = *(const u32x4*)(tile + V::off(key_row(kb, col), x * 4 + quad));
    const int vrow = key_row((col >> 3) & 1, quad * 4 + ((col >> 1) & 3));    // this lane's row of 8, 8 columns of it
#pragma unroll
    for (int d = 0; d < DB; ++d)
      op.v[d] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
          (__attribute__((address_space(3))) i32x2*)(vt + V::off(vrow, d) + (col & 1) * 8));
  };
  // 2^(byte - 127) of a scale byte (a block that no row sees may have any)
  auto scale_of = [](uint32_t byte) { return __builtin_bit_cast(float, min(byte, 254u) << 23); };
  auto read_ops = [&](Ops& op, int jj) {
    if constexpr (E8) {
      read_ops8(op, jj);
    } else {
      const unsigned char* tile = ring + (jj & (NSS - 1)) * KW * L::SLOT + kw * L::SLOT;
      const unsigned char* vt = tile + L::HALF;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int ds = 0; ds < DS; ++ds) op.kf[kb][ds] = *(const bf16x8*)(tile + L::off(kb * 16 + ka_row, ds * 4 + quad));
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        const int c = d * 2 + tr_c;
        op.vlo[d] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(vt + L::off(tr_row, c) + tr_half));
        op.vhi[d] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(vt + L::off(16 + tr_row, c) + tr_half));
      }
    }
  };
  // a key fragment of a step, and a block of its values
  auto key_of = [&](const Ops& op, int kb, int ds) {
    if constexpr (E8) {
      const float scale = scale_of(op.scale[kb]);
      return decode8(op.k[kb][ds >> 1][2 * (ds & 1)], op.k[kb][ds >> 1][2 * (ds & 1) + 1], scale, scale);
    } else {
      return op.kf[kb][ds];
    }
  };
  auto values_of = [&](const Ops& op, int d) {
    bf16x8 va;
    if constexpr (E8) {
      const uint32_t b0 = op.scale[2], b1 = op.scale[3];
      va = decode8((uint32_t)op.v[d][0], (uint32_t)op.v[d][1], scale_of(b0), scale_of(b1));
    } else {
      const bf16x4 lo_b = __builtin_bit_cast(bf16x4, op.vlo[d]), hi_b = __builtin_bit_cast(bf16x4, op.vhi[d]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        va[e] = lo_b[e];
        va[4 + e] = hi_b[e];
      }
    }
    return va;
  };

  // One step (32 keys) of this wave's rows: scores, mask, online softmax, value product.
  auto compute = [&](const Ops& op, int step) {
    const int key0 = slot_of(k_begin + step * kStep);
    if constexpr (PAGED) {
      if (key0 > wave_to) return;
    }
    // S^T blocks kb = 0, 1: element e of a lane in quad q is key kb*16 + e*4 + q, row col.  One slab: the mask enters
    // as the products' starting value (0 or -inf), so nothing rewrites the scores after the matrix cores
    // have written them.  Paged: it replaces the scores, since a key that this row does not see may hold anything where
    // another row sees it, or a mask hides it (-inf plus the product of a NaN or an infinity would be NaN).  Only steps that
    // reach the tree slots or the piece end need it.
    f32x4 s[RB][2];
    // (E8: conversions run ahead of the products that take them, here and below, while the products before are on the matrix
    // cores: 8 x 64 rows behind 8000 slots, whole, 129.5 to 122.4 us)
    auto products = [&](bool from_zero) {
      // (the products are issued at a raised wave priority, so that the SIMD's other wave -- in its softmax --
      // does not hold them back: gqa_long 355 -> 339 us)
      bf16x8 kf[2], next[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) next[kb] = key_of(op, kb, 0);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int ds = 0; ds < DS; ++ds) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          kf[kb] = next[kb];
          if (ds + 1 < DS) next[kb] = key_of(op, kb, ds + 1);
        }
        if constexpr (E8) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
            s[rb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                kf[kb], qf[rb][ds], (from_zero && ds == 0) ? f32x4{0.f, 0.f, 0.f, 0.f} : s[rb][kb], 0, 0, 0);
      }
      __builtin_amdgcn_s_setprio(0);
    };
    bool edge = key0 + kStep > Lp || key0 + kStep > k_end;
    if constexpr (PAGED) edge = key0 + kStep > plain_to || (key0 < plain_from && key0 + kStep > a.sinks);
    if (PAGED || !edge) products(true);   // (the first products start from an inline zero: no accumulator to clear)
    if (edge) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = key0 + (E8 ? key_row(kb, quad * 4 + e) : kb * 16 + e * 4 + quad);
            const int j = key - Lp;                      // tree node of a key past the prefix
            const uint64_t word = j < 64 ? anc0[rb] : anc1[rb];
            const bool anc = ((word >> (j & 63)) & 1ull) != 0;
            bool vis = (key < k_end) & ((key < Lp) | anc);
            if constexpr (PAGED) {
              const bool near = (key >= see_from[rb]) | (key < a.sinks);
              vis = a.chain ? (key <= see_to[rb]) & near : (key < N) & ((key < Lp) ? near : anc);
            }
            s[rb][kb][e] = vis ? (PAGED ? s[rb][kb][e] : 0.f) : -INFINITY;
          }
        }
      }
      if (!PAGED) products(false);
    }

    // this lane's maximum over its 8 keys of each row, in scaled log2 units (c > 0 keeps the order)
    float lmax[RB];
    bool grow = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      // (NaN-propagating maximum: three-input instructions, no canonicalising of the products' results; a
      // score is NaN only of a key that the row sees, the rows past a sequence's end being zeroed)
      // Two row blocks: a chain, so that every step is one three-input maximum (four instructions instead of six:
      // head_dim 64 with entropies 18.05 -> 17.65 us); one row block: a tree, which is shorter (18.8 against 18.9 us).
      float x;
      if constexpr (RB > 1) {
        x = vmax(vmax(s[rb][0][0], s[rb][0][1]), s[rb][0][2]);
        x = vmax(vmax(x, s[rb][0][3]), s[rb][1][0]);
        x = vmax(vmax(x, s[rb][1][1]), s[rb][1][2]);
        x = vmax(x, s[rb][1][3]);
      } else {
        x = vmax(vmax(vmax(s[rb][0][0], s[rb][0][1]), vmax(s[rb][0][2], s[rb][0][3])),
                 vmax(vmax(s[rb][1][0], s[rb][1][1]), vmax(s[rb][1][2], s[rb][1][3])));
      }
      lmax[rb] = c_scale * x;
      grow |= lmax[rb] > m_run[rb] + kLazyLog2;
    }
    // The reference maximum m only moves when some score exceeds it by more than 2^8 (the exponentials then
    // stay <= 256, and softmax does not depend on the reference), which after the first steps is rare: in
    // the common case no cross-lane reduction and no rescale happen at all, and one branch covers every
    // row block, so the exponentials and value products of all of them form one scheduling region.
    if (__any(grow)) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        float tmax = fmaxf(lmax[rb], __shfl_xor(lmax[rb], 16));
        tmax = fmaxf(tmax, __shfl_xor(tmax, 32));
        if (tmax > m_run[rb] + kLazyLog2) {
          const float alpha = m_run[rb] == -INFINITY ? 0.f : fast_exp2(m_run[rb] - tmax);
          // p * (z - m) with the new reference: each old term gains (m_old - m_new) before the rescale
          if (ENT) e_run[rb] = alpha == 0.f ? 0.f : alpha * fmaf(m_run[rb] - tmax, l_run[rb], e_run[rb]);
          m_run[rb] = tmax;
          l_run[rb] *= alpha;
#pragma unroll
          for (int d = 0; d < DB; ++d) o[rb][d] *= alpha;
        }
      }
    }
    // (probabilities are rounded to bf16 for the value product, half a step of 2^-8 of each: in fp32 the product would take a
    // second, of the remainders; their sum is of the unrounded ones.  32 heads x 60 nodes behind 3136 slots: outputs off 64-bit
    // ones by 0.0021 of their norm, 0.0017 with fp32 probabilities, which is the outputs' own rounding)
    bf16x8 pb[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const float m_use = m_run[rb] == -INFINITY ? 0.f : m_run[rb];
      float psum = 0.f, esum = 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float t = fmaf(s[rb][kb][e], c_scale, -m_use);
          const float p = fast_exp2(t);
          psum += p;
          // (a masked key has t = -inf and p = 0; the clamp keeps its term 0 rather than NaN)
          if (ENT) esum = fmaf(p, fmaxf(t, -1.0e4f), esum);
          pb[rb][kb * 4 + e] = (__bf16)p;
        }
      }
      l_run[rb] += psum;
      if (ENT) e_run[rb] += esum;
    }

    // O^T[d][row] += sum over the 32 keys of V[key][d] P[row][key]
    __builtin_amdgcn_s_setprio(1);
    bf16x8 next_values = values_of(op, 0);
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      const bf16x8 va = next_values;
      if (d + 1 < DB) next_values = values_of(op, d + 1);
      if constexpr (E8) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) o[rb][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[rb], o[rb][d], 0, 0, 0);
    }
    __builtin_amdgcn_s_setprio(0);
  };

  if constexpr (PIPE) {
    // Software-pipelined: after the barrier that hands over super-step js+1, a wave issues that super-step's
    // operand reads and then computes super-step js from registers, so the LDS reads of one step overlap the
    // products and softmax of the previous one on every wave.
    Ops op[2];
    if (nsa > 0) {
      wait_vm_steps<CPT, NSS - 1>(issued_by(0) - 1);   // this wave's copies of super-step 0 have landed
      zero_tail(0);
      barrier_lds();
      if (kw < nact) read_ops(op[0], 0);
    }
    auto half_step = [&](int js, const Ops& cur, Ops& nxt) {
      const bool more = js + 1 < nsa;
      // Every wave has computed super-step js-1, and its reads of super-step js (issued before that) have
      // returned: the slots of super-step js take the copies of super-step js+NSS at once, without waiting for
      // super-step js+1 to land.
      barrier_lds();
      if (js + NSS < nsa) issue_super(js + NSS);
      if (more) {
        // this wave's copies of super-step js+1
        if (E8 && js + 1 + NSS <= nsa) wait_vm<(NSS - 1) * CPT>();
        else wait_vm_steps<CPT, NSS - 1>(issued_by(js + 1) - 2 - js);
        zero_tail(js + 1);
      }
      // super-step js+1 complete in LDS for every wave.  (Also taken after the last super-step, so that on
      // every path the operands of super-step js are known to have landed in registers.)
      barrier_lds();
      if (more && (js + 1) * KW + kw < nact) read_ops(nxt, js + 1);
      __builtin_amdgcn_sched_barrier(0);
      if (js * KW + kw < nact) compute(cur, js * KW + kw);
    };
    for (int js = 0; js < nsa; js += 2) {
      half_step(js, op[0], op[1]);
      if (js + 1 < nsa) half_step(js + 1, op[1], op[0]);
    }
  } else {
    // One pass of the inner loop per turn of the ring: the slot is a constant in each unrolled copy, so the
    // operand reads take it as an immediate offset (no per-step address arithmetic).
    for (int js0 = 0; js0 < nsa; js0 += NSS) {
#pragma unroll
      for (int sl = 0; sl < NSS; ++sl) {
        const int js = js0 + sl;
        if (js >= nsa) break;
        // this wave's copies of super-step js have landed
        if (E8 && js + NSS - 1 <= nsa) wait_vm<(NSS - 2) * CPT>();
        else wait_vm_steps<CPT, NSS - 2>(issued_by(js) - 1 - js);
        zero_tail(js);
        barrier_lds();   // super-step js complete in LDS for every wave; the slots of super-step js-1 are free
        if (js + NSS - 1 < nsa) issue_super(js + NSS - 1);
        const int step = js * KW + kw;   // this wave's step
        if (step >= nact) continue;
        Ops op;
        read_ops(op, sl);
        __builtin_amdgcn_sched_barrier(0);
        compute(op, step);
      }
    }
  }
  wait_vm<0>();   // copies planned past a sequence's own end land before LDS is reused
  if constexpr (PAGED) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
      if (a.chain && see_to[rb] < 0) {   // rows past the sequence's own see nothing, whatever a plain step made of them
        m_run[rb] = -INFINITY;
        l_run[rb] = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[rb][d] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
  }

#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    l_run[rb] += __shfl_xor(l_run[rb], 16);
    l_run[rb] += __shfl_xor(l_run[rb], 32);
    if (ENT) {
      e_run[rb] += __shfl_xor(e_run[rb], 16);
      e_run[rb] += __shfl_xor(e_run[rb], 32);
    }
  }

  // ---- key groups: group k finalises output columns [16*DBK*k, 16*DBK*(k+1)) of its rows, from every group's
  // state for those columns (exchanged through LDS, merged in group order)
  constexpr int DBK = DB / KW;     // 16-column blocks of the output this wave finalises
  static_assert(DB % KW == 0, "column share");
  f32x4 fin[RB][DBK];
  if constexpr (KW == 1) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int dd = 0; dd < DBK; ++dd) fin[rb][dd] = o[rb][dd];
  } else {
    barrier_lds();   // every wave is done with the ring
    // [owner group][source group, own one left out][DBK*4 16-byte chunks][R rows]: the 16 lanes of a quad touch
    // 256 consecutive bytes, so neither the writes nor the reads conflict on banks
    f32x4* st_o = (f32x4*)ring;
    float2* st_ml = (float2*)(st_o + (size_t)KW * (KW - 1) * DBK * 4 * R);   // [KW][R]
    float* st_e = (float*)(st_ml + KW * R);                                   // [KW][R]
    auto chunk = [&](int owner, int source, int dd, int row) {
      return ((owner * (KW - 1) + (source < owner ? source : source - 1)) * DBK * 4 + dd * 4 + quad) * R + row;
    };
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int row = rh * RW + rb * 16 + col;
#pragma unroll
      for (int d = 0; d < DB; ++d)
        if (d / DBK != kw) st_o[chunk(d / DBK, kw, d % DBK, row)] = o[rb][d];
      if (quad == 0) {
        st_ml[kw * R + row] = make_float2(m_run[rb], l_run[rb]);
        if (ENT) st_e[kw * R + row] = e_run[rb];
      }
    }
    barrier_lds();
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int row = rh * RW + rb * 16 + col;
      float mk[KW], lk[KW], ek[KW];
#pragma unroll
      for (int k = 0; k < KW; ++k) {
        const float2 ml = st_ml[k * R + row];
        mk[k] = k == kw ? m_run[rb] : ml.x;
        lk[k] = k == kw ? l_run[rb] : ml.y;
        ek[k] = ENT ? (k == kw ? e_run[rb] : st_e[k * R + row]) : 0.f;
      }
      float M = mk[0];
#pragma unroll
      for (int k = 1; k < KW; ++k) M = fmaxf(M, mk[k]);
      float L = 0.f, E = 0.f;
#pragma unroll
      for (int dd = 0; dd < DBK; ++dd) fin[rb][dd] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KW; ++k) {
        const float w = mk[k] == -INFINITY ? 0.f : fast_exp2(mk[k] - M);
        if (ENT) E += ent_term(w, ek[k], mk[k], M, lk[k]);
        L += w * lk[k];
#pragma unroll
        for (int dd = 0; dd < DBK; ++dd) {
          f32x4 x;
          if (k == kw) {   // this wave's own state: block kw*DBK + dd of o (kw is wave-uniform)
            x = o[rb][dd];
#pragma unroll
            for (int j = 1; j < KW; ++j)
              if (j == kw) x = o[rb][j * DBK + dd];
          } else {
            x = st_o[chunk(kw, k, dd, row)];
          }
          fin[rb][dd] += w * x;
        }
      }
      m_run[rb] = M;
      l_run[rb] = L;
      e_run[rb] = E;
    }
  }
  const int c0 = kw * DBK * 16 + quad * 4;   // first output column of this lane's block dd = 0

  // ---- the workgroup's rows, normalised and rounded to bf16, go row-major into LDS (after the key groups'
  // exchange area; 16-byte pieces of a row XOR-swizzled by the row, so neither the matrix-core-layout writes
  // nor the row reads conflict on banks), with each row's (max, sum) and entropy term; they are then written
  // out as whole 16-byte pieces of rows.
  const int S = a.splits;
  const size_t pset = (size_t)u * a.row_groups + rg;
  const size_t prow0 = pset * S * R;   // the set's piece 0, row 0
  const int rows_valid = min(R, rows_here);
  if constexpr (PAGED) {
    if (S > 1 || placed) {   // (a piece's rows go to the workspace in fp32, straight from the registers)
      size_t prow = prow0 + (size_t)split * R;
      if (placed) prow = (size_t)n * R;
      float* const dst = (float*)a.part_o + prow * D;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const int rl = rh * RW + rb * 16 + col;
        if (rl >= rows_valid) continue;
        const float inv = l_run[rb] > 0.f ? 1.0f / l_run[rb] : 0.f;
#pragma unroll
        for (int dd = 0; dd < DBK; ++dd) *(f32x4*)(dst + (size_t)rl * D + c0 + dd * 16) = fin[rb][dd] * inv;
        if (kw == 0 && quad == 0)
          *(float2*)(a.part_ml + 2 * (prow + rl)) = make_float2(m_run[rb], l_run[rb]);
      }
      if (placed) return;
      merge_set<D, W, ENT, float>(a, pset, R, split, start_old, qrow0 + (size_t)row_base, rows_valid, &merge_lds,
                                &good_lds);
      return;
    }
  }
  constexpr int CPR = D / 8;                  // 16-byte pieces per row
  constexpr size_t XBYTES = KW > 1 ? ((size_t)(KW - 1) * R * D * 4 + (size_t)KW * R * 12 + 1023) / 1024 * 1024 : 0;
  static_assert(XBYTES + (size_t)R * D * 2 + (size_t)R * 12 <= (size_t)NST * V::SLOT, "row staging fits the ring");
  unsigned char* row_lds = ring + XBYTES;                               // [R][CPR] 16-byte pieces
  float2* ml_lds = (float2*)(row_lds + (size_t)R * D * 2);              // [R]
  float* e_lds = (float*)(ml_lds + R);                                  // [R]
  auto row_piece = [&](int r, int ch) { return row_lds + ((size_t)r * CPR + (ch ^ (r & (CPR - 1)))) * 16; };
  if constexpr (KW == 1) barrier_lds();   // every wave's last operand reads of the ring have returned
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int rl = rh * RW + rb * 16 + col;
    const float inv = l_run[rb] > 0.f ? 1.0f / l_run[rb] : 0.f;
#pragma unroll
    for (int dd = 0; dd < DBK; ++dd) {
      bf16x4 res;
#pragma unroll
      for (int e = 0; e < 4; ++e) res[e] = (__bf16)(fin[rb][dd][e] * inv);
      const int c = c0 + dd * 16;
      *(bf16x4*)(row_piece(rl, c / 8) + (c % 8) * 2) = res;
    }
    if (kw == 0 && quad == 0) {
      ml_lds[rl] = make_float2(m_run[rb], l_run[rb]);
      if (ENT) e_lds[rl] = e_run[rb];
    }
  }
  barrier_lds();

  // (row, 16-byte piece) items of the workgroup's rows, dealt to the threads
  constexpr int ITEMS = (R * CPR + 64 * W - 1) / (64 * W);   // items per thread
  // One piece writes the output; with several, every piece stores its rows (normalised, bf16), their (max,
  // sum) and entropy terms as piece `split` of its set.  Rows of one KV head are consecutive in memory.
  {
    __bf16* dst = S == 1 ? (__bf16*)a.out + (qrow0 + (size_t)row_base) * D : a.part_o + (prow0 + (size_t)split * R) * D;
#pragma unroll
    for (int t = 0; t < ITEMS; ++t) {
      const int item = t * 64 * W + tid;
      const int r = item / CPR, ch = item % CPR;
      if (item < R * CPR && r < rows_valid) *(u32x4*)(dst + (size_t)r * D + ch * 8) = *(const u32x4*)row_piece(r, ch);
    }
    if (tid < rows_valid) {
      const float2 ml = ml_lds[tid];
      if (S == 1) {
        const size_t orow = qrow0 + row_base + tid;
        const bool some = PAGED ? ml.y != 0.f : ml.y > 0.f;   // (paged: a NaN sum gives a NaN)
        if (a.lse) a.lse[orow] = some ? (ml.x + __log2f(ml.y)) * kLn2 : -INFINITY;
        if (ENT) a.entropy[orow] = row_entropy(ml.y, e_lds[tid]);
      } else {
        const size_t pr = prow0 + (size_t)split * R + tid;
        *(float2*)(a.part_ml + 2 * pr) = ml;
        if (ENT) a.part_e[pr] = e_lds[tid];
      }
    }
  }
  if (PAGED || S == 1) return;

  merge_set<D, W, ENT, __bf16>(a, pset, R, split, start_old, qrow0 + (size_t)row_base, rows_valid, &merge_lds, &good_lds);
}

// The rows of spread keys: a workgroup per row of a unit, its pieces dealt to groups of D / 8 threads (8 columns each), whose
// sums meet in LDS in group order.
template <int D>
__global__ __launch_bounds__(256) void spread_merge_kernel(AttnArgs8 a, int R) {
  constexpr int LANES = D / 8, GROUPS = 256 / LANES, PCH = 4;
  typedef float f32x8 __attribute__((ext_vector_type(8)));
  __shared__ f32x8 sums[GROUPS][LANES];
  __shared__ float2 mls[GROUPS];
  const int u = blockIdx.x, row = blockIdx.y, seq = u / a.Hkv, g = u - seq * a.Hkv;
  const SpreadPlan sp = spread_plan(a, threadIdx.x & 63);
  int first = g;
  for (int b = 0; b < seq; ++b) first += __builtin_amdgcn_readlane(sp.pieces, b) * a.Hkv;
  const int S = __builtin_amdgcn_readlane(sp.pieces, seq);
  const int group = threadIdx.x / LANES, ch = threadIdx.x % LANES;
  float M = -INFINITY, lsum = 0.f;
  f32x8 acc;
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  auto join = [&](float m, float l, const f32x8& x, float weight) {   // (m, l) of a state and its rows times `weight`
    const float Mn = fmaxf(M, m);
    const float wo = M == -INFINITY ? 0.f : fast_exp2(M - Mn), w = m == -INFINITY ? 0.f : fast_exp2(m - Mn);
    lsum = lsum * wo + l * w;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = acc[e] * wo + w * weight * x[e];
    M = Mn;
  };
  for (int s0 = group; s0 < S; s0 += GROUPS * PCH) {
    f32x8 x[PCH];
    float2 ml[PCH];
#pragma unroll
    for (int k = 0; k < PCH; ++k) {   // (all in flight; those past the last piece repeat it)
      const size_t at = ((size_t)first + (size_t)min(s0 + k * GROUPS, S - 1) * a.Hkv) * R + row;
      ml[k] = *(const float2*)(a.part_ml + 2 * at);
      x[k] = *(const f32x8*)((const float*)a.part_o + at * D + ch * 8);
    }
#pragma unroll
    for (int k = 0; k < PCH; ++k)
      if (s0 + k * GROUPS < S) join(ml[k].x, ml[k].y, x[k], ml[k].y);
  }
  sums[group][ch] = acc;
  if (ch == 0) mls[group] = make_float2(M, lsum);
  __syncthreads();
  if (group > 0) return;
  const int live = min(S, GROUPS);
  for (int k = 1; k < live; ++k) join(mls[k].x, mls[k].y, sums[k][ch], 1.f);
  const size_t orow = ((size_t)seq * a.Hq + (size_t)g * a.G) * a.T + row;
  const bool some = lsum != 0.f;        // (a NaN sum gives a NaN)
  const float inv = some ? 1.0f / lsum : 0.f;
  bf16x8 res;
#pragma unroll
  for (int e = 0; e < 8; ++e) res[e] = (__bf16)(acc[e] * inv);
  *(bf16x8*)((__bf16*)a.out + orow * D + ch * 8) = res;
  if (ch == 0 && a.lse) a.lse[orow] = some ? (M + __log2f(lsum)) * kLn2 : -INFINITY;
}

template <int D, int RB, int KW, int W, int NST, int WPC, bool ENT, bool PAGED, bool E8 = false, bool WIDE = false>
hipError_t launch_streaming(const Args<E8>& a, hipStream_t stream) {
  constexpr size_t lds = dynamic_lds<D, NST, WPC, E8>(16 * RB * (W / KW));
  static_assert(lds + 2 * kMaxNodes * 8 + 2 * kMaxNodes * 8 + (PAGED ? 2 * kMaxNodes * 4 : 8) + (E8 ? NST * 16 : 0) + 64 <=
                    160 * 1024 / WPC,
                "LDS budget");
  // two sets of operand registers fit beside one 16-row block's state, not beside two
  auto kern = tree_attn_bf16_kernel<D, RB, KW, W, NST, RB == 1, ENT, WPC, PAGED, E8, WIDE>;
  static bool configured[E8 ? 64 : 1] = {};
  int dev = 0;
  if constexpr (E8) {      // (on each device)
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  }
  if (!configured[dev]) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    configured[dev] = true;
  }
  if (a.rows_per_wg != 16 * RB * (W / KW)) return hipErrorInvalidValue;
  if (a.splits > 1 && (!a.part_o || !a.part_ml || !a.set_ctr || (ENT && !a.part_e))) return hipErrorInvalidValue;
  if (a.splits > 1 && a.ctr_stride < 2) return hipErrorInvalidValue;
  const unsigned units_rounded = E8 ? (a.units * a.unit_parts + 7) / 8 * 8 : PAGED ? a.units * a.unit_parts : (a.units + 7) / 8 * 8;
  const unsigned groups = PAGED ? (a.row_groups + a.unit_parts - 1) / a.unit_parts : a.row_groups;
  unsigned grid = units_rounded * (unsigned)a.splits * groups;
  if constexpr (E8) {
    if (a.spread_wgs > 0) {
      if (a.row_groups != 1 || a.splits != 1 || a.B > kSpreadSeqs || a.spread_wgs < 2 * a.units || !a.part_o || !a.part_ml)
        return hipErrorInvalidValue;
      hipLaunchKernelGGL(kern, dim3((unsigned)a.spread_wgs), dim3(64 * W), lds, stream, a);
      hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL(spread_merge_kernel<D>, dim3((unsigned)a.units, (unsigned)(a.G * a.T)), dim3(256), 0, stream, a,
                         a.rows_per_wg);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL(kern, dim3(grid), dim3(64 * W), lds, stream, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace dreams
