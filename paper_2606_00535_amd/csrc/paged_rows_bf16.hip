// Attention over a paged cache, bf16 inputs, fp32 accumulation on the matrix cores, for KV heads of more than 64 rows (heads
// x positions): the rows of a prompt, where row i (at position L_b + i) sees the slots up to its own, and large trees; with
// a window only those and the sinks in sight.
//
//   * A workgroup of 4 waves owns 128 rows, a wave 32 of them; two workgroups share a compute unit, so the waves of a SIMD
//     belong to different ones and no barrier ties their phases.  A prompt's rows are 128 consecutive ones of one query head
//     (which end at different keys) or the heads' rows one after another, as are a tree's.
//   * Keys come in tiles of 32.  S^T = K Q^T and O^T += V^T P^T on v_mfma_f32_32x32x16_bf16: a lane holds 16 scores of
//     one row (lane l and l + 32 share row l % 32), the probabilities are in the value product's operand order as they
//     come (keys numbered 16 t + 4 (l / 32) + {0..3, 8..11} in both operands), and the values are read transposed
//     (ds_read_b64_tr_b16).
//   * A wave's work is pipelined over tiles: the score product of tile k + 1 runs on the matrix cores while the vector
//     ALU takes the exponentials of tile k, whose value product follows.  So at the time that the wave needs key tile k + 1
//     it needs value tile k: a stage is two key tiles and the two value tiles one earlier, one barrier a stage (D = 128:
//     32 KB, two stages; D = 64: 16 KB, four).
//   * A stage is copied straight into LDS (global_load_lds_dwordx4), each wave a block of 16 key rows and one of 16 value
//     rows, from the pages that scalar loads of the table name a stage ahead.  Rows in LDS are XOR-swizzled: chunk c of
//     row r at position c ^ swz(r), so that neither the 32-row key reads nor the 4 x 32 value reads conflict on banks.
//   * Slots that no row sees are zeroed in LDS, so whatever they hold cannot reach the products.
//   * Few workgroups: two key groups in each (a ring each, one workgroup to a compute unit), then pieces of the key axis over
//     several, merged as the tree kernel's are, in fp32.
//
// What bounds it, at 28 heads on 4 x 8192 rows, D = 128 (440 to 490 us by the device, 980 to 1090 TFLOP/s, where a library
// product of 16384^3 makes 1360):
// power and issue.  The matrix cores work 54 % of the cycles at a clock of 1.5 to 1.6 GHz (inputs of zeros, which cost less power,
// take 15 % less time).  A wave issues in order: a tile's 16 products, 72 vector, 24 LDS and 36 scalar instructions leave it
// waiting to issue for 38 % of its time, and barriers and copies for 19 %.  Without the waits for copies the time is the
// same, without the barriers 3 % less (10 % for 1000 rows with a window of 1024), without the key or value reads 2-5 % each.
// Scalar instructions count like others: with 80 to 100 a tile it was 482 us.  Short calls are bound by their masked tiles and
// the epilogue: 24 heads on 8 x 8 x 187 rows, D = 64, 10.0 us, 3.1 of them until the first stage has landed, 1.5 behind the
// last; with a mask of several compares a score 11.0 (trees, 28 heads on 4 x 60 nodes behind 500: 19.4 and 17.1).
// Tried: 64 rows a wave (half the LDS reads, but one wave a SIMD: 640 us, 442 instead of 285 for trees of 896 x 8320), 8 waves on
// one ring of 128 KB (level at 8192 rows, 20 % slower at 6000), the next tile's keys fetched ahead of the barrier and the
// last value products put off to the next tile (2-3 % slower), the copies' addresses beside the products (level).
#include "tree_attn_bf16.h"

#include <type_traits>

namespace dreams {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kTile = 32;            // keys per tile
constexpr int kRows = 32;            // rows per wave
constexpr int kWaves = 4;
constexpr int kRowsWg = kRows * kWaves;

// wave-wide copy into LDS: lane l's 16 bytes, from a uniform base plus the lane's offset, land at m0 + 16 l.  (Without the
// streaming hint: the query heads of a KV head read the same keys.)
template <int N>
__device__ __forceinline__ void tile16_to_lds(uint32_t m0, const void* sbase, const uint32_t (&voff)[N]) {
  static_assert(N == 2 || N == 4);
  if constexpr (N == 2)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\t"
                 "global_load_lds_dwordx4 %2, %3 offset:%4" ::"s"(m0), "v"(voff[0]), "v"(voff[1]), "s"(sbase), "n"(1024)
                 : "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\t"
                 "global_load_lds_dwordx4 %2, %5 offset:%6\n\tglobal_load_lds_dwordx4 %3, %5 offset:%7\n\t"
                 "global_load_lds_dwordx4 %4, %5 offset:%8" ::"s"(m0), "v"(voff[0]), "v"(voff[1]), "v"(voff[2]),
                 "v"(voff[3]), "s"(sbase), "n"(1024), "n"(2 * 1024), "n"(3 * 1024) : "memory");
}

// Rows of D bf16 in LDS.  A 256-byte bank line holds one row (D = 128) or two (D = 64).  A key read takes one 16-byte chunk
// of 32 rows, 16 rows at a time: swz is a bijection over the 16 (8 of a parity) rows.  A value read takes 4 aligned
// chunks of 4 consecutive rows: the rows differ in swz / 4 (or in their half of the line).
template <int D>
struct TileRows {
  static constexpr int ROW = D * 2, CPR = D / 8;
  static constexpr int BLOCK = 16 * ROW;            // bytes of 16 rows
  static constexpr int COPIES = BLOCK / 1024;       // wave-wide copies of a block
  static constexpr int HALF = 2 * kTile * ROW;      // bytes of a stage's keys (or values)
  static constexpr int STAGE = 2 * HALF;
  static constexpr int STAGES = 65536 / STAGE;
  static __device__ __forceinline__ int swz(int r) {
    if constexpr (D == 128) return (r & 3) * 4 + ((r >> 2) & 3);
    return ((r >> 1) & 1) * 4 + ((r >> 2) & 3);
  }
  static __device__ __forceinline__ int off(int r, int c) { return r * ROW + ((c ^ swz(r)) << 4); }
};

// KG: key groups of 4 waves (1 or 2), each on its half of the workgroup's tiles with a ring of its own; their states meet in
// LDS at the end.  With several pieces of the key axis (workgroups), each takes its run of tiles, and the pieces merge as the
// tree kernel's do.
// TREE: tree nodes; else consecutive positions, in groups of one head's rows (groups_per_head > 0) or packed likewise.
template <int D, int KG, bool TREE>
__global__ __launch_bounds__(64 * kWaves * KG, 2) void paged_rows_bf16_kernel(AttnArgs a) {
  using L = TileRows<D>;
  constexpr int KS = D / 16;        // products of a tile's scores
  constexpr int DB = D / 32;        // 32-column blocks of the output
  constexpr int AHEAD = L::STAGES - 1;
  constexpr int CP = 2 * L::COPIES; // copies a wave issues per stage
  extern __shared__ __attribute__((aligned(1024))) unsigned char rings[];
  __shared__ float merge_lds[KG > 1 ? 2 * 64 * kWaves : 1];   // the second key group's maxima and sums
  __shared__ uint32_t pieces_lds[2];                // (merge_set)
  __shared__ int par_lds[TREE ? kMaxNodes : 1], depth_lds[TREE ? kMaxNodes : 1];

  // ---- work item: every (sequence, KV head)'s row groups are dealt to unit_parts parts, a part to an XCD, which takes the
  // q-th group of all of its parts before the next; groups of 128 rows of a head, the ones with the most keys first
  // (Two workgroups to a compute unit: the second ones take their groups in the opposite order, so that the longest run
  // beside the shortest of the first round.)
  const int n = blockIdx.x;
  const int here = a.units * a.unit_parts / 8;
  const int on_xcd = n >> 3, slots = KG > 1 ? 1 << 30 : a.cus / 4;
  const int rank = on_xcd >= slots / 2 && on_xcd < slots && (int)(gridDim.x >> 3) >= slots ? slots + slots / 2 - 1 - on_xcd
                                                                                             : on_xcd;
  const int q_group = rank / (here * a.splits), within = rank - q_group * (here * a.splits);
  const int vu = (n & 7) + 8 * (within / a.splits), split = within - (within / a.splits) * a.splits;
  const int u = vu / a.unit_parts;
  const int rg = q_group * a.unit_parts + (vu - u * a.unit_parts);
  if (rg >= a.row_groups) return;
  const int b = u / a.Hkv, g = u - b * a.Hkv;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, h = lane >> 5;
  const int wave8 = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave = wave8 % kWaves, kg = wave8 / kWaves;
  unsigned char* ring = rings + kg * 65536;
  const int T = a.T;
  // the workgroup's rows: [row_base, row_base + rows_here) of the KV head's G * T
  int row_base = rg * kRowsWg, rows_here = a.G * T - row_base;
  if (!TREE && a.groups_per_head > 0) {
    const int blk = a.groups_per_head - 1 - rg / a.G, hh = rg - (rg / a.G) * a.G;
    row_base = hh * T + blk * kRowsWg;
    rows_here = T - blk * kRowsWg;
  }
  rows_here = min(rows_here, kRowsWg);
  // the lowest position of a row, from the prefix on (of a chain's rows in one head: the first's)
  const bool one_head = !TREE && row_base % T + rows_here <= T;
  const int i0 = one_head ? row_base % T : 0;
  const size_t row0 = ((size_t)b * a.Hq + (size_t)g * a.G) * T + row_base;

  // ---- queries: B operand of the score products, row col of the wave, 8 columns from 16 ds + 8 h on.  (Loaded ahead of the
  // lengths and the table, used once the first copies are out.)
  const int row = wave * kRows + col;                // this lane's row of the workgroup
  bf16x8 qf[KS];
  {
    const unsigned char* src = (const unsigned char*)a.q + (row0 + min(row, rows_here - 1)) * L::ROW;
#pragma unroll
    for (int ds = 0; ds < KS; ++ds) qf[ds] = *(const bf16x8*)(src + (ds * 16 + 8 * h) * 2);
  }

  int nb = T;
  if (!TREE && a.row_len) nb = min(max(a.row_len[b], 0), T);
  const int Lp = min(max(a.kv_len[b], 0), a.S_cap - nb);
  const int i_last = TREE ? T - 1 : min(one_head ? i0 + rows_here : T, nb) - 1;   // the last live row's (< i0: none)
  const int N = i_last >= i0 ? Lp + i_last + 1 : 0;  // slots that some row sees: [0, sink_end) and [low, N)
  int low = 0, sink_end = 0, sink_tiles = 0, gap = 0;
  if (a.window > 0 && N > 0) {
    low = max(Lp + i0 - a.window + 1, 0);
    sink_end = min(a.sinks, low);
    sink_tiles = (sink_end + kTile - 1) / kTile * kTile;
    gap = max(low / kTile * kTile - sink_tiles, 0);
  }
  auto slot_of = [&](int key) { return key < sink_tiles ? key : key + gap; };   // (of a tile's keys)
  // the piece's tiles, and this key group's of them: [tile0, tile0 + tiles) (the first group's are never fewer: its count
  // sets the barriers)
  const int all_tiles = (N - gap + kTile - 1) / kTile, piece = (all_tiles + a.splits - 1) / a.splits;
  const int begin = min(split * piece, all_tiles), piece_tiles = min(piece, all_tiles - begin);
  const int half = (piece_tiles + KG - 1) / KG;
  const int tile0 = begin + kg * half, tiles = min(half, piece_tiles - kg * half);
  const int periods = half > 0 ? half / 2 + 1 : 0;

  // ---- copies.  Stage j: key blocks of 16 from key 64 j on, value blocks from key 64 j - 32 on.  Wave w brings key block w and
  // value block (w + 2) % 4, the same slots' values (waves 0 and 1) or those of its keys a stage earlier: one look-up and one
  // offset a stage.  (The value blocks before the first key repeat it, unread; those past the last tile are some page's.)
  typedef const __attribute__((address_space(4))) int32_t* const_table;
  const const_table table = (const_table)(uintptr_t)(a.table + (size_t)b * a.width);
  const int ps1 = (1 << a.page_shift) - 1;
  const size_t head_off = ((size_t)g << a.page_shift) * L::ROW;
  const unsigned char* kbase = (const unsigned char*)a.k + head_off;
  const unsigned char* vbase = (const unsigned char*)a.v + head_off;
  const uint32_t ring_lds = __builtin_amdgcn_readfirstlane(lds_addr(ring));
  auto key_slot = [&](int j) { return slot_of((tile0 + j * 2) * kTile + 16 * wave); };
  const int slot_before = slot_of(max((tile0 - 2) * kTile + 16 * wave, 0));   // of stage -1
  auto value_slot = [&](int j) { return wave < 2 ? key_slot(j) : j > 0 ? key_slot(j - 1) : slot_before; };
  auto look_up = [&](int slot) { return table[min((uint32_t)slot >> a.page_shift, (uint32_t)a.width - 1)]; };
  // (unsigned 32-bit parts: scalar instructions cost a wave as much as others)
  auto offset = [&](int page, int slot) {
    const uint32_t p = min(max(page, 0), a.num_pages - 1);
    return (uint64_t)p * (uint64_t)a.page_stride + (uint32_t)(slot & ps1) * (uint32_t)L::ROW;
  };
  // (lane's offset of copy 0; copy c is 1 KB on, its rows' swizzle differs by swz(first row of c))
  const uint32_t coff0 = (uint32_t)((lane / L::CPR) * L::ROW + (((lane % L::CPR) ^ L::swz(lane / L::CPR)) << 4));
  uint32_t coff[L::COPIES];
#pragma unroll
  for (int c = 0; c < L::COPIES; ++c) coff[c] = coff0 ^ (uint32_t)(L::swz(c * (64 / L::CPR)) << 4);
  const uint32_t value_at = L::HALF + ((wave + 2) & 3) * L::BLOCK;
  int page = 0;                    // of the next stage to copy
  uint64_t before = 0;             // the offset of the stage before
  auto issue = [&](int j) {
    const uint32_t dst = ring_lds + (j % L::STAGES) * L::STAGE;
    const uint64_t at = offset(page, key_slot(j));
    tile16_to_lds(dst + wave * L::BLOCK, kbase + at, coff);
    tile16_to_lds(dst + value_at, vbase + (wave < 2 ? at : before), coff);
    before = at;
    page = look_up(key_slot(j + 1));
  };
  // this wave's rows of stage j that no row of the workgroup sees become zeros (of stages [whole0, whole1) all are seen)
  const int first_seen = a.window > 0 ? max(sink_tiles, low - gap) + kTile - tile0 * kTile : 0;
  const int whole0 = max((first_seen + 63) / 64, 0), whole1 = (N - gap - tile0 * kTile) / 64;
  auto zero_unseen = [&](int j) {
    unsigned char* stage = ring + (j % L::STAGES) * L::STAGE;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      unsigned char* at = stage + (part ? value_at : wave * L::BLOCK);
      const int s0 = part ? value_slot(j) : key_slot(j);
      if (s0 + 16 > N || (s0 < low && s0 + 16 > sink_end)) {
        constexpr int LPR = 4, PER = L::CPR / LPR;     // 4 lanes a row
        const int s = s0 + lane / LPR;
        if (s >= N || (s < low && s >= sink_end)) {
#pragma unroll
          for (int c = 0; c < PER; ++c)
            *(u32x4*)(at + (lane / LPR) * L::ROW + ((lane % LPR) * PER + c) * 16) = u32x4{0u, 0u, 0u, 0u};
        }
      }
    }
  };

  // (this piece has started: see merge_set)
  unsigned long long start_old = 0;
  const size_t pset = (size_t)u * a.row_groups + rg;
  if (a.splits > 1 && tid == 0) {
    const unsigned long long x = xcd_id();
    start_old = __hip_atomic_fetch_add(a.set_ctr + pset * a.ctr_stride,
                                       1ull | (x << kCtrXcdSum) | ((x * x) << kCtrXcdSq), __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
  }
  const bool parents = TREE && (!a.mask || a.window > 0);
  if (parents && wave8 == 0)
    for (int c = 0; c * 64 < T; ++c)
      copy4_to_lds(__builtin_amdgcn_readfirstlane(lds_addr(par_lds)) + c * 256,
                   a.parent + (size_t)b * T + min(c * 64 + lane, T - 1));
  const int page_before = look_up(slot_before);
  page = look_up(key_slot(0));
  before = offset(page_before, slot_before);
  for (int j = 0; j < AHEAD; ++j)
    if (j < periods) issue(j);

  const int node = (row_base + min(row, rows_here - 1)) % T;   // the lane's tree node, or its position behind the prefix
  const bool live = row < rows_here && (TREE || node < nb);
  const float c_scale = fmaxf(fabsf(a.scale_log2), 1.17549435e-38f);
#pragma unroll
  for (int ds = 0; ds < KS; ++ds) {
    u32x4 x = __builtin_bit_cast(u32x4, qf[ds]);
    if (a.scale_log2 < 0.f) x ^= 0x80008000u;        // (a negative scale flips the queries' signs, exact)
    if (!live) x = u32x4{0u, 0u, 0u, 0u};            // (rows past the sequence's own may hold anything)
    qf[ds] = __builtin_bit_cast(bf16x8, x);
  }
  // ---- what the rows see: of a chain the slots [see_from, see_to] and the sinks; of a tree the prefix from see_from on, the
  // sinks, and the nodes in anc0, anc1
  int pos = Lp + node, deepest = 0;
  uint64_t anc0 = 0, anc1 = 0;
  if constexpr (TREE) {
    if (a.mask) {
      const int words = (T + 63) / 64;
      const uint64_t* bits = a.mask + ((size_t)b * T + node) * words;
      anc0 = bits[0];
      anc1 = words > 1 ? bits[1] : 0;
    }
    if (parents) {
      wait_vm<0>();
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
      if (a.window > 0) {
        if (tid < T) depth_lds[tid] = walk(tid, [](int) {});
        __syncthreads();
        for (int j = lane; j < T; j += 64) deepest = max(deepest, depth_lds[j]);
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) deepest = max(deepest, __shfl_xor(deepest, off));
        deepest = __builtin_amdgcn_readfirstlane(deepest);
      }
      if (!a.mask) walk(node, [&](int j) { (j < 64 ? anc0 : anc1) |= 1ull << (j & 63); });
      pos = Lp;
      if (a.window > 0) {
        const int depth = depth_lds[node], far = depth - a.window;
        pos += depth;
        auto drop_far = [&](uint64_t& word, int first) {   // nodes out of sight
          for (uint64_t rest = word; rest; rest &= rest - 1) {
            const int j = __builtin_ctzll(rest), d = first + j < T ? depth_lds[first + j] : 0;
            if (d <= far && Lp + d >= a.sinks) word &= ~(1ull << j);
          }
        };
        drop_far(anc0, 0);
        drop_far(anc1, 64);
      }
    }
  }
  const int see_from = a.window > 0 ? max(pos - a.window + 1, 0) : 0, see_to = live ? pos : -1;
  // the last slot that every row of the wave may see, and the last that one of them does
  const int wave_first = TREE ? Lp - 1 : one_head ? Lp + i0 + wave * kRows : Lp;
  const int wave_last = one_head ? min(wave_first + kRows - 1, Lp + i_last) : N - 1;
  const int plain_from = a.window > 0 ? (TREE ? Lp + deepest : wave_last) - a.window + 1 : 0;
  // tiles of this wave: those up to its last row's slot (in key numbers: the slot less the gap)
  const int wave_tiles = wave_last < wave_first ? 0 : max(min(tiles, (wave_last - gap) / kTile + 1 - tile0), 0);

  f32x16 o[DB];
  float m = -3.402823466e38f, l = 0.f;   // (finite: no score, -inf, less the reference is NaN)
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

  const int tr_row = 4 * h + ((lane & 15) >> 2);     // transposed read: this lane's row of 4 and its piece of 16 columns
  const int tr_c = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1), tr_half = (lane & 1) * 8;

  // Operand addresses within a tile: the swizzle leaves one offset per 32 (keys: 16) columns, the rest are constants.
  uint32_t koff[KS], voff[DB][2];
#pragma unroll
  for (int ds = 0; ds < KS; ++ds) {
    koff[ds] = ring_lds + L::off(col, ds * 2 + h);
    asm("" : "+v"(koff[ds]));     // (whole, not to be put together at every read)
  }
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int x = 0; x < 2; ++x) voff[d][x] = ring_lds + L::HALF + L::off(8 * x + tr_row, d * 4 + tr_c) + tr_half;
  typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  // kt, vt: byte offsets of a tile's keys (values) in the ring, constants in the unrolled loop
  auto read_keys = [&](bf16x8 (&kf)[KS], int kt) {
#pragma unroll
    for (int ds = 0; ds < KS; ++ds) kf[ds] = *(lds_bf16x8*)(uintptr_t)(koff[ds] + kt);
  };
  auto read_values = [&](bf16x8 (&va)[DB], int vt, int t) {
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      const bf16x4 lo = __builtin_bit_cast(
          bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(voff[d][0] + vt + 16 * t * L::ROW)));
      const bf16x4 hi = __builtin_bit_cast(
          bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(voff[d][1] + vt + 16 * t * L::ROW)));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        va[d][i] = lo[i];
        va[d][4 + i] = hi[i];
      }
    }
  };
  // keys out of a row's sight.  (Lane's score i is key at + c(i), c a constant: the row's limits move instead of the keys.)
  auto mask = [&](f32x16& s, int s0) {
    const int at = s0 + 4 * h;
    auto c = [](int i) { return 8 * (i >> 2) + (i & 3); };
    if constexpr (TREE) {
      // a bit a key of the tile: the prefix's in sight and the nodes in anc0, anc1
      auto range = [](int lo, int hi) {     // keys [lo, hi) of the tile
        auto below = [](int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; };
        return below(hi) & ~below(lo);
      };
      const int first = Lp - s0;            // the first node's key
      const uint32_t prefix = (range(see_from - s0, first) | range(0, a.sinks - s0)) & range(0, first);
      const uint64_t nodes = first >= 32    ? 0
                             : first >= 0   ? anc0 << first
                             : first > -64  ? anc0 >> -first | anc1 << (64 + first)
                             : first > -128 ? anc1 >> (-64 - first)
                                            : 0;
      const uint32_t bits = (prefix | ((uint32_t)nodes & range(first, N - s0))) >> (4 * h);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = bits & (1u << c(i)) ? s[i] : -INFINITY;
    } else if (s0 >= a.sinks || a.window == 0) {
      const int from = see_from - at;
      const uint32_t seen = max(see_to - see_from + 1, 0);     // (none of a dead row's)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = (uint32_t)(c(i) - from) < seen ? s[i] : -INFINITY;
    } else {
      const int from = see_from - at, to = see_to - at, sinks = a.sinks - at;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = (c(i) <= to) & ((c(i) >= from) | (c(i) < sinks)) ? s[i] : -INFINITY;
    }
  };
  auto row_max = [&](const f32x16& s) {
    float x = vmax(vmax(s[0], s[1]), s[2]);
#pragma unroll
    for (int i = 3; i < 15; i += 2) x = vmax(vmax(x, s[i]), s[i + 1]);
    return vmax(x, s[15]);
  };
  // the reference moves where a score passes it by more than 2^8 (rare after the first tiles)
  float limit = -INFINITY;     // (before scaling)
  auto move_reference = [&](float x) {
    if (__any(x > limit)) {
      const float t = c_scale * fmaxf(x, __shfl_xor(x, 32));
      if (t > m + kLazyLog2) {
        const float alpha = __builtin_amdgcn_exp2f(m - t);
        m = t;
        limit = (t + kLazyLog2) / c_scale;
        l *= alpha;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] *= alpha;
      }
    }
  };
  // One basic block in a fixed order, a matrix instruction and what the vector ALU does in its shadow at a time: the scores
  // of the next tile (NEXT) beside the exponentials of this one, then its value product beside the next tile's maximum,
  // which is returned.
  auto block = [&](auto next, f32x16& sn, const f32x16& sc, int kt, int vt) {
    constexpr bool NEXT = decltype(next)::value;
    constexpr int FIRST = 4, PER = (16 - FIRST) / (KS + DB);   // exponentials ahead of the products, and beside each
    static_assert(FIRST + PER * (KS + DB) == 16 && FIRST + PER * KS >= 8, "the first 8 keys' weights precede their product");
    bf16x8 kf[KS], va[DB], vb[DB];
    bf16x8 p[2];
    float sum[2], e[2], x = 0.f;
    auto score = [&](int ds) {
      if constexpr (NEXT) {
        f32x16 z;
        if (ds == 0) {
#pragma unroll
          for (int i = 0; i < 16; ++i) z[i] = 0.f;
        } else {
          z = sn;
        }
        sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ds], qf[ds], z, 0, 0, 0);
      }
    };
    auto weight = [&](int i) {
      e[i & 1] = __builtin_amdgcn_exp2f(fmaf(sc[i], c_scale, -m));
      sum[i & 1] = i < 2 ? e[i & 1] : sum[i & 1] + e[i & 1];
      if (i & 1) {
        p[i / 8][i % 8 - 1] = (__bf16)e[0];
        p[i / 8][i % 8] = (__bf16)e[1];
      }
    };
#define FENCE __builtin_amdgcn_sched_barrier(0)
    FENCE;
    if constexpr (NEXT) read_keys(kf, kt);
    FENCE;
#pragma unroll
    for (int i = 0; i < FIRST; ++i) weight(i);
    FENCE;
#pragma unroll
    for (int ds = 0; ds < KS; ++ds) {
      score(ds);
      if (ds == KS / 2 - 1) read_values(va, vt, 0);
      if (ds == KS - 1) read_values(vb, vt, 1);
#pragma unroll
      for (int i = 0; i < PER; ++i) weight(FIRST + ds * PER + i);
      FENCE;
    }
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[d], p[0], o[d], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < PER; ++i) weight(FIRST + (KS + d) * PER + i);
      FENCE;
    }
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vb[d], p[1], o[d], 0, 0, 0);
      if constexpr (NEXT) {
        if (d == 0) {
          x = row_max(sn);
          asm volatile("" : "+v"(x));   // (here, not behind the products)
        }
      }
    }
    l += sum[0] + sum[1];
    FENCE;
#undef FENCE
    return x;
  };
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  auto next_stage = [&](int j) {
    // this wave's copies of stage j have landed (those of the AHEAD - 1 stages after it may be in flight)
    if (j + AHEAD <= periods) wait_vm<(AHEAD - 1) * CP>(); else wait_vm<0>();
    if (j < whole0 || j >= whole1) zero_unseen(j);
    barrier_lds();   // stage j complete for every wave; every wave is past stage j - 1, whose slot is free
    if (j + AHEAD < periods) issue(j + AHEAD);
  };
  f32x16 s0, s1;     // scores of even and odd tiles (tile -1: none)
#pragma unroll
  for (int i = 0; i < 16; ++i) s1[i] = -INFINITY;
  // tiles [far0, far1) that no row of the wave sees: from behind the sinks to its first row's (without a gap, the sinks may
  // reach into the run)
  const int far0 = (gap > 0 ? sink_tiles / kTile : a.sinks > 0 ? (a.sinks - 1) / kTile + 1 : 0) - tile0;
  const int far1 = !TREE && a.window > 0 ? (wave_first - a.window + 1 - gap) / kTile - tile0 : 0;
  // plain tiles, in sight of every row of the wave
  const int plain0 = max((max(plain_from - gap, 0) + kTile - 1) / kTile, sink_tiles / kTile) - tile0;
  const uint32_t plain_tiles = max(min(max(wave_first + 1 - gap, 0) / kTile - tile0, wave_tiles) - plain0, 0);
  auto step = [&](int k, f32x16& sn, const f32x16& sc, int t) {   // scores of tile k, values of tile k - 1
    const bool plain = (uint32_t)(k - plain0) < plain_tiles;
    if (!plain) {
      if (k >= wave_tiles) return;
      if (k > far0 && k > 0 && k < far1) {    // (tile far0, too, is all masked: it takes the value product of the one before)
#pragma unroll
        for (int i = 0; i < 16; ++i) sn[i] = -INFINITY;
        return;
      }
    }
    float x = block(yes, sn, sc, t, t);
    if (!plain) {
      mask(sn, slot_of((tile0 + k) * kTile));
      x = row_max(sn);
    }
    move_reference(x);
  };
  for (int j0 = 0; j0 < periods; j0 += L::STAGES) {
#pragma unroll
    for (int x = 0; x < L::STAGES; ++x) {
      const int j = j0 + x;
      if (j >= periods) break;
      next_stage(j);
      step(2 * j, s0, s1, x * L::STAGE);
      step(2 * j + 1, s1, s0, x * L::STAGE + kTile * L::ROW);
      if (wave_tiles >> 1 == j) {   // the value product of the wave's last tile
        if (wave_tiles & 1) s1 = s0;
        block(no, s0, s1, 0, x * L::STAGE + (wave_tiles & 1) * (kTile * L::ROW));
      }
    }
  }

  // ---- the rows' sums (two lanes a row); the second key group's states through LDS
  l += __shfl_xor(l, 32);
  barrier_lds();   // every wave is done with the rings
  if constexpr (KG > 1) {
    float* const far = (float*)(rings + 65536) + wave * (16 * DB * 64) + lane;
    float* const ml = merge_lds + wave * 128 + lane;
    if (kg == 1) {
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) far[(d * 16 + i) * 64] = o[d][i];
      ml[0] = m;
      ml[64] = l;
    }
    __syncthreads();
    if (kg == 0) {
      const float mo = ml[0], M = fmaxf(m, mo);
      const float w = __builtin_amdgcn_exp2f(m - M), wo = __builtin_amdgcn_exp2f(mo - M);
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = o[d][i] * w + far[(d * 16 + i) * 64] * wo;
      l = l * w + ml[64] * wo;
      m = M;
    }
  }
  const bool some = live && l != 0.f;    // (a row that sees a NaN has a NaN sum, and is NaN)
  const float inv = some ? 1.0f / l : 0.f;
  if (a.splits > 1) {   // the piece's rows, in fp32
    const size_t prow = (pset * a.splits + split) * kRowsWg + row;
    if (kg == 0 && row < rows_here) {
      float* const dst = (float*)a.part_o + prow * D + 4 * h;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          f32x4 x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = live ? o[d][i + e] * inv : 0.f;
          *(f32x4*)(dst + d * 32 + 2 * i) = x;
        }
      if (h == 0) *(float2*)(a.part_ml + 2 * prow) = some ? make_float2(m, l) : make_float2(-INFINITY, 0.f);
    }
    merge_set<D, kWaves * KG, false, float>(a, pset, kRowsWg, split, start_old, row0, rows_here, &pieces_lds[0],
                                            &pieces_lds[1]);
    return;
  }
  if (kg == 1) return;
  // ---- the output through LDS, in whole rows
  unsigned char* mine = ring + wave * (kRows * L::ROW);
  auto row_piece = [&](int r, int c) { return mine + r * L::ROW + ((c ^ (r & (L::CPR - 1))) << 4); };
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      bf16x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (__bf16)(live ? o[d][i + e] * inv : 0.f);
      *(bf16x4*)(row_piece(col, d * 4 + (i >> 2)) + 8 * h) = x;
    }
  if (a.lse && h == 0 && row < rows_here) a.lse[row0 + row] = some ? (m + __log2f(l)) * kLn2 : -INFINITY;
  __builtin_amdgcn_s_waitcnt(0xC07F);
  asm volatile("" ::: "memory");
#pragma unroll
  for (int x = 0; x < kRows * L::CPR / 64; ++x) {
    const int e = x * 64 + lane, r = e / L::CPR, c = e - r * L::CPR;
    if (wave * kRows + r < rows_here)
      *(u32x4*)((unsigned char*)a.out + (row0 + wave * kRows + r) * L::ROW + c * 16) = *(const u32x4*)row_piece(r, c);
  }
}

template <int D, int KG, bool TREE>
hipError_t launch(const AttnArgs& a, hipStream_t stream) {
  constexpr int lds = KG * 65536;
  static bool configured[64] = {};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  if (!configured[dev]) {
    e = hipFuncSetAttribute((const void*)paged_rows_bf16_kernel<D, KG, TREE>,
                            hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    configured[dev] = true;
  }
  const unsigned groups = (a.row_groups + a.unit_parts - 1) / a.unit_parts;
  hipLaunchKernelGGL((paged_rows_bf16_kernel<D, KG, TREE>), dim3((unsigned)a.units * a.unit_parts * groups * a.splits),
                     dim3(64 * kWaves * KG), lds, stream, a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_rows(const AttnArgs& a, hipStream_t stream) {
  if (!a.chain) return a.key_groups == 2 ? launch<D, 2, true>(a, stream) : launch<D, 1, true>(a, stream);
  return a.key_groups == 2 ? launch<D, 2, false>(a, stream) : launch<D, 1, false>(a, stream);
}

}  // namespace

hipError_t launch_paged_rows_bf16(const AttnArgs& a, hipStream_t stream) {
  if (a.unit_parts < 1 || a.units * a.unit_parts % 8 != 0 || a.rows_per_wg != kRowsWg ||
      (a.groups_per_head > 0 && a.groups_per_head * a.G != a.row_groups))
    return hipErrorInvalidValue;
  if (a.splits > 1 && (!a.part_o || !a.part_ml || !a.set_ctr || a.ctr_stride < 2)) return hipErrorInvalidValue;
  if (a.D == 128) return launch_rows<128>(a, stream);
  if (a.D == 64) return launch_rows<64>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace dreams
