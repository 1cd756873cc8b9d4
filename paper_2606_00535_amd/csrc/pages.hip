// The bookkeeping of a paged cache: which pages of a pool a sequence holds.  A page's reference count is the number of
// sequences that hold it, 0 marks it free, and pages are handed out lowest number first, so that what a call does
// follows from the state before it alone.
//
//   * pages_take_kernel (reserve and fork): one workgroup.  Its waves read the counts, 64 pages a wave, and leave a word
//     of free bits each; a scan over the words' bit counts ranks the free pages.  Requests are granted in order while
//     the free pages last: where all of them do, their first ranks are a scan of their sizes, else one thread goes
//     through them.  Then a wave per word hands its pages out: the k-th free page goes to the request whose range of
//     ranks holds k (a search over the ranges).
//   * fork_copy_kernel: the partly filled pages of forked sequences, in every layer.
//   * pages_release_kernel: a workgroup per released sequence.
//
// Over small pools all are bound by latency, a chain of a few loads and barriers in one launch each: on 8 sequences of up to
// 91 pages of 32 slots, taking pages 4.4 us, a fork of 6 sequences 6.8 and 4.8 for the copied rows of 32 layers (12 MB read
// and written), a release 3.6.  A launch from a host program costs more than that (8 us), so one workgroup that needs no
// second launch is the split taken.  Its scan reads every count of the pool, one load in flight a wave, so that reserve and
// fork grow with the pool (in a graph, 8 sequences: 600 pages 4.3 and 7.3 us, 8192 6.2 and 9.1, 131072 39 and 42, 524288 143
// and 147); a release does not.
#include "kernels.h"

#include <type_traits>

namespace dreams {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kTakeThreads = 1024;

// inclusive scan of one value a thread over the workgroup
__device__ __forceinline__ int scan_workgroup(int x, int* wave_sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int y = __shfl_up(x, off);
    if (lane >= off) x += y;
  }
  if (lane == 63) wave_sums[wave] = x;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < wave; ++w) before += wave_sums[w];
  __syncthreads();
  return x + before;
}

// exclusive scan of n LDS values in place (saturating sums are the caller's care); returns their sum
__device__ __forceinline__ int scan_lds(int* v, int n, int* wave_sums, int* total) {
  const int per = (n + kTakeThreads - 1) / kTakeThreads;
  const int i0 = min((int)threadIdx.x * per, n), i1 = min(i0 + per, n);
  int sum = 0;
  for (int i = i0; i < i1; ++i) sum += v[i];
  const int incl = scan_workgroup(sum, wave_sums);
  int at = incl - sum;
  for (int i = i0; i < i1; ++i) {
    const int x = v[i];
    v[i] = at;
    at += x;
  }
  if (threadIdx.x == kTakeThreads - 1) *total = incl;
  __syncthreads();
  return *total;
}

// Dynamic LDS: words (8 bytes) of free bits, their ranks, then per request its size, first rank and state.
struct TakeLds {
  uint64_t* bits;
  int* rank;
  int* need;
  int* first;
  int* base;    // fork: the lowest pair that names a sequence as its copy, then the pairs' lengths
};
__host__ __device__ inline size_t take_lds_bytes(int words, int requests, int seqs) {
  return (size_t)words * 12 + (size_t)requests * 8 + (size_t)(requests > seqs ? requests : seqs) * 4 + 16;
}

template <bool FORK>
__global__ __launch_bounds__(kTakeThreads) void pages_take_kernel(PagesArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  __shared__ int wave_sums[kTakeThreads / 64];
  __shared__ int total_lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int words = (a.num_pages + 63) / 64, n = FORK ? a.n : a.B;
  TakeLds s;
  s.bits = (uint64_t*)lds;
  s.rank = (int*)(lds + (size_t)words * 8);
  s.need = s.rank + words;
  s.first = s.need + n;
  s.base = s.first + n;
  const int ps = 1 << a.page_shift;

  // ---- the free pages
  for (int w0 = wave; w0 < words; w0 += kTakeThreads / 64) {
    const int page = w0 * 64 + lane;
    const bool is_free = page < a.num_pages && a.refcount[page] == 0;
    const uint64_t bits = __ballot(is_free);
    if (lane == 0) {
      s.bits[w0] = bits;
      s.rank[w0] = __popcll(bits);
    }
  }
  // ---- the requests
  if constexpr (FORK) {
    for (int i = tid; i < a.B; i += kTakeThreads) s.base[i] = n;
    __syncthreads();
    for (int i = tid; i < n; i += kTakeThreads) {
      const int d = a.dst[i];
      if (d >= 0 && d < a.B) atomicMin(&s.base[d], i);
    }
    __syncthreads();
  }
  for (int i = tid; i < n; i += kTakeThreads) {
    int need = -1;   // refused
    if constexpr (FORK) {
      const int from = a.src[i], to = a.dst[i];
      if (from >= 0 && from < a.B && to >= 0 && to < a.B && from != to && s.base[to] == i && a.count[to] == 0) {
        const int len = a.kv_len[from], have = a.count[from];
        const int hold = len < 0 ? 0x7fffffff : (int)(((long long)len + ps - 1) >> a.page_shift);
        if (hold <= have && hold <= a.width) need = (len & (ps - 1)) ? 1 : 0;
      }
    } else {
      const int have = a.count[i];
      const long long hold = a.want[i] < 0 ? 0 : ((long long)a.want[i] + ps - 1) >> a.page_shift;
      if (have >= 0 && have <= a.width && hold <= a.width) need = hold > have ? (int)hold - have : 0;
    }
    s.need[i] = need;
    s.first[i] = need < 0 ? 0 : need;
  }
  __syncthreads();
  const int free_pages = scan_lds(s.rank, words, wave_sums, &total_lds);
  __syncthreads();
  // (sizes are at most the table's width each: the host has checked that their sum fits)
  const int asked = scan_lds(s.first, n, wave_sums, &total_lds);
  int taken = asked;
  if (asked > free_pages) {
    __syncthreads();
    if (tid == 0) {
      int used = 0;
      for (int i = 0; i < n; ++i) {
        s.first[i] = used;
        if (s.need[i] < 0) continue;
        if (s.need[i] <= free_pages - used) used += s.need[i];
        else s.need[i] = -1;
      }
      total_lds = used;
    }
    __syncthreads();
    taken = total_lds;
  }
  // ---- the state that does not depend on which pages are taken
  if constexpr (FORK) {
    __syncthreads();
    // the sources' lengths, as they are before the call (a source may be another pair's copy)
    for (int i = tid; i < n; i += kTakeThreads) s.base[i] = s.need[i] < 0 ? 0 : a.kv_len[a.src[i]];
    __syncthreads();
    for (int i = wave; i < n; i += kTakeThreads / 64) {
      if (s.need[i] < 0) continue;
      const int from = a.src[i], to = a.dst[i], whole = s.base[i] >> a.page_shift;
      for (int c = lane; c < whole; c += 64) {
        const int id = a.table[(size_t)from * a.width + c];
        a.table[(size_t)to * a.width + c] = id;
        if (id >= 0 && id < a.num_pages) atomicAdd(&a.refcount[id], 1);
      }
    }
  }
  // ---- the pages
  for (int w0 = wave; w0 < words; w0 += kTakeThreads / 64) {
    const uint64_t bits = s.bits[w0];
    const int rank0 = s.rank[w0];
    if (rank0 >= taken || bits == 0) continue;
    const int rank = rank0 + __popcll(bits & ((1ull << lane) - 1));
    if (!((bits >> lane) & 1ull) || rank >= taken) continue;
    // the last request whose first rank is at most this one (one that takes nothing shares its successor's)
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s.first[mid] <= rank) lo = mid; else hi = mid - 1;
    }
    const int page = w0 * 64 + lane;
    int row, column;
    if constexpr (FORK) {
      row = a.dst[lo];
      column = s.base[lo] >> a.page_shift;
    } else {
      row = lo;
      column = a.count[lo] + rank - s.first[lo];
    }
    a.table[(size_t)row * a.width + column] = page;
    a.refcount[page] = 1;
  }
  __syncthreads();   // (every page is placed by the counts before the call)
  for (int i = tid; i < n; i += kTakeThreads) {
    const int need = s.need[i];
    a.granted[i] = need >= 0;
    if (need < 0) continue;
    if constexpr (FORK) {
      a.count[a.dst[i]] = (s.base[i] >> a.page_shift) + need;
      a.kv_len[a.dst[i]] = s.base[i];
    } else if (need > 0) {
      a.count[i] += need;
    }
  }
}

constexpr int kCopyThreads = 256;
constexpr int kCopyBytes = 65536;   // bytes of a page's head that a workgroup copies

// A workgroup per (layer and KV head, piece of its slab, pair): the filled rows of the source's last page.
template <typename Args>
__global__ __launch_bounds__(kCopyThreads) void fork_copy_kernel(Args a) {
  const int i = blockIdx.z;
  if (!a.granted[i]) return;
  const int from = a.src[i], to = a.dst[i];
  const int len = a.kv_len[to];   // (the source's own may be another pair's copy by now)
  const int tail = len & ((1 << a.page_shift) - 1), column = len >> a.page_shift;
  const int64_t bytes = (int64_t)tail * a.row_bytes;
  const int64_t b0 = (int64_t)blockIdx.y * kCopyBytes;
  if (b0 >= bytes) return;
  const int64_t b1 = b0 + kCopyBytes < bytes ? b0 + kCopyBytes : bytes;
  const int p = a.table[(size_t)from * a.width + column], q = a.table[(size_t)to * a.width + column];
  if (p < 0 || p >= a.num_pages || q < 0 || q >= a.num_pages) return;
  const int layer = blockIdx.x / a.Hkv, g = blockIdx.x - layer * a.Hkv;
  const int64_t head = layer * a.layer_stride + (((int64_t)g * a.row_bytes) << a.page_shift);
  const int64_t src = head + (int64_t)p * a.page_stride, dst = head + (int64_t)q * a.page_stride;
  for (int64_t x = b0 + threadIdx.x * 16; x < b1; x += kCopyThreads * 16) {
    const u32x4 k = *(const u32x4*)(a.k + src + x), v = *(const u32x4*)(a.v + src + x);
    *(u32x4*)(a.k + dst + x) = k;
    *(u32x4*)(a.v + dst + x) = v;
  }
  if constexpr (std::is_same_v<Args, PagesArgs8>) {   // the blocks' scales
    if (blockIdx.y > 0) return;
    const int64_t first = layer * a.scales.layer_stride + (((int64_t)g << a.page_shift) / kScaleBlock);
    const int64_t from_s = first + (int64_t)p * a.scales.page_stride, to_s = first + (int64_t)q * a.scales.page_stride;
    for (int x = threadIdx.x; x < (tail + kScaleBlock - 1) / kScaleBlock; x += kCopyThreads) {
      a.scales.k[to_s + x] = a.scales.k[from_s + x];
      a.scales.v[to_s + x] = a.scales.v[from_s + x];
    }
  }
}

constexpr int kReleaseThreads = 256;

__global__ __launch_bounds__(kReleaseThreads) void pages_release_kernel(PagesArgs a) {
  const int i = blockIdx.x, tid = threadIdx.x;
  const int seq = a.dst[i];
  if (seq < 0 || seq >= a.B) return;
  // a sequence that is named twice is released by the first that names it
  bool again = false;
  for (int j = tid; j < i; j += kReleaseThreads) again |= a.dst[j] == seq;
  if (__syncthreads_or(again)) return;
  int have = a.count[seq];
  have = have < 0 ? 0 : (have > a.width ? a.width : have);
  int keep = 0;
  if (a.trim) {
    const int len = a.kv_len[seq];
    keep = len < 0 ? 0 : (int)(((long long)len + (1 << a.page_shift) - 1) >> a.page_shift);
  }
  __syncthreads();
  for (int c = keep + tid; c < have; c += kReleaseThreads) {
    int32_t* entry = a.table + (size_t)seq * a.width + c;
    const int id = *entry;
    *entry = -1;
    if (id >= 0 && id < a.num_pages && atomicSub(&a.refcount[id], 1) <= 0) atomicAdd(&a.refcount[id], 1);
  }
  if (tid == 0) {
    if (keep < have) a.count[seq] = keep;
    if (!a.trim) a.kv_len[seq] = 0;
  }
}

template <bool FORK>
hipError_t launch_take(const PagesArgs& a, hipStream_t stream) {
  static bool configured[64] = {};
  const size_t lds = take_lds_bytes((a.num_pages + 63) / 64, FORK ? a.n : a.B, a.B);
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  if (!configured[dev]) {
    const size_t most = take_lds_bytes((kPagesMaxPages + 63) / 64, kPagesMaxSeqs, kPagesMaxSeqs);
    e = hipFuncSetAttribute((const void*)pages_take_kernel<FORK>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)most);
    if (e != hipSuccess) return e;
    configured[dev] = true;
  }
  hipLaunchKernelGGL(pages_take_kernel<FORK>, dim3(1), dim3(kTakeThreads), lds, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_pages_reserve(const PagesArgs& a, hipStream_t stream) { return launch_take<false>(a, stream); }

namespace {

template <typename Args>
hipError_t launch_fork(const Args& a, hipStream_t stream) {
  hipError_t e = launch_take<true>(a, stream);
  if (e != hipSuccess) return e;
  const int64_t slab = ((int64_t)a.row_bytes << a.page_shift);
  const dim3 grid((unsigned)(a.NL * a.Hkv), (unsigned)((slab + kCopyBytes - 1) / kCopyBytes), (unsigned)a.n);
  hipLaunchKernelGGL(fork_copy_kernel<Args>, grid, dim3(kCopyThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t stream) { return launch_fork(a, stream); }
hipError_t launch_pages_fork_e4m3(const PagesArgs8& a, hipStream_t stream) { return launch_fork(a, stream); }

hipError_t launch_pages_release(const PagesArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(pages_release_kernel, dim3((unsigned)a.n), dim3(kReleaseThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace dreams
