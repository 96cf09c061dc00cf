// Pages of the 4-bit key/value cache: hand out, share, free, pack and copy.  The bookkeeping of a call is one workgroup's work
// (a few hundred slots and pages: latency-bound); the pages' bytes are moved by a launch of their own that reads the list the first one
// left, in 16-byte pieces over all layers (bound by HBM: every byte read and written once).
#include "kernels.hpp"
#include "kv4.hpp"
#include "numeric.hpp"

namespace larosa {

namespace {

constexpr int kBook = 1024;   // lanes of a bookkeeping workgroup

__device__ __forceinline__ int pages_for(int tokens, int page_tokens) { return (tokens + page_tokens - 1) / page_tokens; }

// Exclusive prefix sums of two counts over the workgroup's lanes, and their totals.
struct Sums { unsigned a, b, all_a, all_b; };
__device__ __forceinline__ Sums book_scan(unsigned a, unsigned b) {
  __shared__ unsigned wa[kBook / 64], wb[kBook / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const unsigned ia = wave_scan_inclusive(a, lane), ib = wave_scan_inclusive(b, lane);
  __syncthreads();            // the arrays may still be read from the scan before
  if (lane == 63) {
    wa[wave] = ia;
    wb[wave] = ib;
  }
  __syncthreads();
  Sums s{ia - a, ib - b, 0, 0};
  for (int w = 0; w < kBook / 64; ++w) {
    if (w < wave) {
      s.a += wa[w];
      s.b += wb[w];
    }
    s.all_a += wa[w];
    s.all_b += wb[w];
  }
  return s;
}

// ---- trim -------------------------------------------------------------------------------------------

// One wave per entry.  Exchanges make an entry that is listed twice harmless: the length is the smallest that any entry leaves,
// and a table entry gives its page back once.
__global__ __launch_bounds__(256) void kv4_trim_kernel(larosa_kv4_cache C, const int32_t* slots, const int32_t* keep, int n) {
  const int i = (blockIdx.x * 256 + threadIdx.x) / 64, lane = threadIdx.x & 63;
  if (i >= n) return;
  const int slot = slots[i];
  if (slot < 0 || slot >= C.n_slots) return;
  const int kept = keep ? max(0, keep[i]) : 0;
  int had = 0;
  if (lane == 0) had = atomicMin(&C.length[slot], kept);
  had = __shfl(had, 0);
  const int to = min(pages_for(had, C.page_tokens), C.max_pages);
  for (int p = pages_for(kept, C.page_tokens) + lane; p < to; p += 64) {
    const int page = atomicExch(&C.table[static_cast<size_t>(slot) * C.max_pages + p], -1);
    if (page >= 0 && page < C.n_pages) atomicSub(&C.refs[page], 1);
  }
}

// ---- fork -------------------------------------------------------------------------------------------

// Whether the list is in order.  A free destination is marked by a negative length; a second mark, or a source that carries one,
// gives the fault away.  Marks are taken back where the list is refused, and become lengths in the next launch.
__global__ __launch_bounds__(kBook) void kv4_fork_check_kernel(larosa_kv4_cache C, const int32_t* src, const int32_t* dst, int n,
                                                               int32_t* status) {
  __shared__ int bad;
  if (threadIdx.x == 0) bad = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kBook) {
    const int s = src[i], d = dst[i];
    if (s < 0 || s >= C.n_slots || d < 0 || d >= C.n_slots || atomicCAS(&C.length[d], 0, -1 - i) != 0) bad = 1;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kBook) {
    const int s = src[i];
    if (s >= 0 && s < C.n_slots && atomicAdd(&C.length[s], 0) < 0) bad = 1;
  }
  __syncthreads();
  if (bad)
    for (int i = threadIdx.x; i < n; i += kBook) {
      const int d = dst[i];
      if (d >= 0 && d < C.n_slots) atomicCAS(&C.length[d], -1 - i, 0);
    }
  if (threadIdx.x == 0) *status = bad ? -1 : 0;
}

__global__ __launch_bounds__(256) void kv4_fork_kernel(larosa_kv4_cache C, const int32_t* src, const int32_t* dst,
                                                       const int32_t* status) {
  if (*status != 0) return;
  const int s = src[blockIdx.y], d = dst[blockIdx.y];
  const int p = blockIdx.x * 256 + threadIdx.x;
  if (p == 0) C.length[d] = C.length[s];
  if (p >= C.max_pages) return;
  const int page = C.table[static_cast<size_t>(s) * C.max_pages + p];
  C.table[static_cast<size_t>(d) * C.max_pages + p] = page;
  if (page >= 0 && page < C.n_pages) atomicAdd(&C.refs[page], 1);
}

// ---- grow -------------------------------------------------------------------------------------------

// What a listed slot has and wants.
struct Want {
  int slot, had, count, old_pages, new_pages;
  int page;                   // its last page if that is not full, more tokens come and others share it; else -1
};
__device__ __forceinline__ Want want_of(const larosa_kv4_cache& C, const int32_t* slots, const int32_t* counts, int i) {
  Want w{};
  w.slot = slots[i];
  w.count = counts ? counts[i] : 1;
  w.page = -1;
  if (w.slot < 0 || w.slot >= C.n_slots || w.count < 0) {
    w.slot = -1;
    return w;
  }
  w.had = C.length[w.slot];
  const long room = static_cast<long>(C.max_pages) * C.page_tokens;
  if (w.had < 0 || static_cast<long>(w.had) + w.count > room) {
    w.slot = -1;
    return w;
  }
  w.old_pages = pages_for(w.had, C.page_tokens);
  w.new_pages = pages_for(w.had + w.count, C.page_tokens);
  if (w.count > 0 && w.had % C.page_tokens) {
    const int p = C.table[static_cast<size_t>(w.slot) * C.max_pages + w.old_pages - 1];
    if (p >= 0 && p < C.n_pages && C.refs[p] > 1) w.page = p;
  }
  return w;
}

__global__ __launch_bounds__(kBook) void kv4_grow_kernel(larosa_kv4_cache C, const int32_t* slots, const int32_t* counts, int n,
                                                         int32_t* status, Kv4Scratch x) {
  __shared__ int bad;
  const int tid = threadIdx.x;
  if (tid == 0) {
    bad = 0;
    *x.n_pairs = 0;
  }
  __syncthreads();
  for (int i = tid; i < n; i += kBook) {
    const Want w = want_of(C, slots, counts, i);
    if (w.slot < 0) {
      bad = 1;
      continue;
    }
    atomicExch(&x.mark[w.slot], 0);
    if (w.page >= 0) {
      atomicExch(&x.growing[w.page], 0);
      atomicExch(&x.last[w.page], 0);
    }
  }
  __syncthreads();
  if (!bad)
    for (int i = tid; i < n; i += kBook) {
      const Want w = want_of(C, slots, counts, i);
      if (atomicAdd(&x.mark[w.slot], 1) != 0) bad = 1;
      if (w.page >= 0) {
        atomicAdd(&x.growing[w.page], 1);
        atomicMax(&x.last[w.page], i + 1);
      }
    }
  __syncthreads();
  if (bad) {
    if (tid == 0) *status = -1;
    return;
  }
  // pages for each slot of the list, in its order: a copy of the shared page first, then the new ones
  unsigned wanted = 0, copies = 0;
  for (int i0 = 0; i0 < n; i0 += kBook) {
    const int i = i0 + tid;
    Want w{};
    w.page = -1;
    bool copy = false;
    if (i < n) {
      w = want_of(C, slots, counts, i);
      copy = w.page >= 0 && !(atomicAdd(&x.growing[w.page], 0) == C.refs[w.page] && atomicAdd(&x.last[w.page], 0) == i + 1);
    }
    const Sums s = book_scan(w.new_pages - w.old_pages + copy, copy);
    if (i < n) {
      x.offset[i] = static_cast<int>(wanted + s.a);
      // (more copies than pages: the call is refused below)
      if (copy && copies + s.b < static_cast<unsigned>(C.n_pages)) x.pair_src[copies + s.b] = w.page;
      x.mark[w.slot] = copy ? static_cast<int>(copies + s.b) : -1;      // from here on: which pair is the slot's, or none
    }
    wanted += s.all_a;
    copies += s.all_b;
  }
  // the lowest free pages, eight to a lane at a time
  unsigned found = 0;
  for (int p0 = 0; p0 < C.n_pages && found < wanted; p0 += kBook * 8) {
    unsigned mine = 0;
    uint32_t free8 = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int p = p0 + tid * 8 + k;
      if (p < C.n_pages && C.refs[p] == 0) {
        free8 |= 1u << k;
        ++mine;
      }
    }
    const Sums s = book_scan(mine, 0);
    unsigned at = found + s.a;
    for (int k = 0; k < 8; ++k)
      if (free8 >> k & 1) {
        if (at < wanted) x.free_ids[at] = p0 + tid * 8 + k;
        ++at;
      }
    found += s.all_a;
  }
  if (found < wanted) {
    if (tid == 0) *status = static_cast<int>(wanted - found);
    return;
  }
  __syncthreads();            // the free ids and offsets are written
  for (unsigned k = tid; k < wanted; k += kBook) {
    int lo = 0, hi = n;       // the last slot of the list whose pages begin at or before k
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (static_cast<unsigned>(x.offset[mid]) <= k) lo = mid; else hi = mid;
    }
    const int slot = slots[lo], page = x.free_ids[k], r = static_cast<int>(k) - x.offset[lo], pair = x.mark[slot];
    const int old_pages = pages_for(C.length[slot], C.page_tokens);
    const int p = pair >= 0 ? old_pages - 1 + r : old_pages + r;
    if (pair >= 0 && r == 0) {
      x.pair_dst[pair] = page;
      atomicSub(&C.refs[x.pair_src[pair]], 1);
    }
    C.table[static_cast<size_t>(slot) * C.max_pages + p] = page;
    C.refs[page] = 1;
  }
  __syncthreads();            // the lengths are read above
  for (int i = tid; i < n; i += kBook) C.length[slots[i]] += counts ? counts[i] : 1;
  if (tid == 0) {
    *x.n_pairs = static_cast<int>(copies);
    *status = 0;
  }
}

// ---- compact ------------------------------------------------------------------------------------------

__global__ __launch_bounds__(kBook) void kv4_compact_kernel(larosa_kv4_cache C, int32_t* live, Kv4Scratch x) {
  const int tid = threadIdx.x;
  unsigned n_live = 0;
  for (int p0 = 0; p0 < C.n_pages; p0 += kBook * 8) {
    unsigned mine = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int p = p0 + tid * 8 + k;
      mine += p < C.n_pages && C.refs[p] > 0;
    }
    n_live += book_scan(mine, 0).all_a;
  }
  // free ids below n_live and live ids from it on, both ascending: as many of the one as of the other
  unsigned holes = 0, movers = 0;
  for (int p0 = 0; p0 < C.n_pages; p0 += kBook * 8) {
    uint32_t hole8 = 0, mover8 = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int p = p0 + tid * 8 + k;
      if (p >= C.n_pages) continue;
      const bool used = C.refs[p] > 0;
      hole8 |= (!used && p < static_cast<int>(n_live)) << k;
      mover8 |= (used && p >= static_cast<int>(n_live)) << k;
    }
    const Sums s = book_scan(__popc(hole8), __popc(mover8));
    unsigned a = holes + s.a, b = movers + s.b;
    for (int k = 0; k < 8; ++k) {
      const int p = p0 + tid * 8 + k;
      if (hole8 >> k & 1) x.pair_dst[a++] = p;
      if (mover8 >> k & 1) x.pair_src[b++] = p;
    }
    holes += s.all_a;
    movers += s.all_b;
  }
  __syncthreads();
  for (unsigned k = tid; k < movers; k += kBook) {
    const int from = x.pair_src[k], to = x.pair_dst[k];
    x.free_ids[from] = to;
    C.refs[to] = C.refs[from];
    C.refs[from] = 0;
  }
  if (tid == 0) {
    *x.n_pairs = static_cast<int>(movers);
    if (live) *live = static_cast<int>(n_live);
    x.growing[0] = static_cast<int>(n_live);
  }
}

__global__ __launch_bounds__(256) void kv4_remap_kernel(larosa_kv4_cache C, Kv4Scratch x) {
  const size_t i = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= static_cast<size_t>(C.n_slots) * C.max_pages) return;
  const int page = C.table[i];
  if (page >= x.growing[0] && page < C.n_pages) C.table[i] = x.free_ids[page];
}

// ---- copies -------------------------------------------------------------------------------------------

constexpr int kCopyBytes = 256 * 16 * 4;      // of a workgroup's step

// Pages src[i] into dst[i], all layers; the pairs' number comes from n_pairs or, where that is null, from n.
__global__ __launch_bounds__(256) void kv4_copy_kernel(larosa_kv4_cache C, const int32_t* src, const int32_t* dst,
                                                       const int32_t* n_pairs, int n, size_t page_bytes) {
  if (n_pairs) n = *n_pairs;
  const unsigned steps = static_cast<unsigned>((page_bytes + kCopyBytes - 1) / kCopyBytes);
  const size_t items = static_cast<size_t>(n) * C.n_layers * steps;
  uint8_t* data = static_cast<uint8_t*>(C.data);
  for (size_t it = blockIdx.x; it < items; it += gridDim.x) {
    const unsigned step = static_cast<unsigned>(it % steps);
    const size_t rest = it / steps;
    const int layer = static_cast<int>(rest % C.n_layers);
    const int i = static_cast<int>(rest / C.n_layers);
    const int from = src[i], to = dst[i];
    if (from < 0 || from >= C.n_pages || to < 0 || to >= C.n_pages) continue;
    const size_t base = static_cast<size_t>(layer) * C.n_pages;
    const uint4* a = reinterpret_cast<const uint4*>(data + (base + from) * page_bytes);
    uint4* b = reinterpret_cast<uint4*>(data + (base + to) * page_bytes);
    const size_t at = static_cast<size_t>(step) * (kCopyBytes / 16) + threadIdx.x, end = page_bytes / 16;
    uint4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (at + 256 * k < end) v[k] = a[at + 256 * k];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (at + 256 * k < end) b[at + 256 * k] = v[k];
  }
}

hipError_t launch_copy(const larosa_kv4_cache& C, const int32_t* src, const int32_t* dst, const int32_t* n_pairs, int n, hipStream_t s) {
  const size_t page_bytes = static_cast<size_t>(C.n_kv_heads) * (C.page_tokens / 32) * 34 * C.head_dim;
  const size_t items = static_cast<size_t>(n) * C.n_layers * ((page_bytes + kCopyBytes - 1) / kCopyBytes);
  const unsigned grid = static_cast<unsigned>(items < 2048 ? items : 2048);
  hipLaunchKernelGGL(kv4_copy_kernel, dim3(grid), dim3(256), 0, s, C, src, dst, n_pairs, n, page_bytes);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_trim(const larosa_kv4_cache& C, const int32_t* slots, const int32_t* keep, int n, hipStream_t s) {
  hipLaunchKernelGGL(kv4_trim_kernel, dim3((n + 3) / 4), dim3(256), 0, s, C, slots, keep, n);
  return hipGetLastError();
}

hipError_t launch_kv4_fork(const larosa_kv4_cache& C, const int32_t* src, const int32_t* dst, int n, int32_t* status, hipStream_t s) {
  hipLaunchKernelGGL(kv4_fork_check_kernel, dim3(1), dim3(kBook), 0, s, C, src, dst, n, status);
  if (hipError_t e = hipGetLastError()) return e;
  for (int at = 0; at < n; at += 65535) {
    const dim3 grid((C.max_pages + 255) / 256, n - at < 65535 ? n - at : 65535);
    hipLaunchKernelGGL(kv4_fork_kernel, grid, dim3(256), 0, s, C, src + at, dst + at, status);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

hipError_t launch_kv4_grow(const larosa_kv4_cache& C, const int32_t* slots, const int32_t* counts, int n, int32_t* status,
                           const Kv4Scratch& x, hipStream_t s) {
  hipLaunchKernelGGL(kv4_grow_kernel, dim3(1), dim3(kBook), 0, s, C, slots, counts, n, status, x);
  if (hipError_t e = hipGetLastError()) return e;
  return launch_copy(C, x.pair_src, x.pair_dst, x.n_pairs, n < C.n_pages ? n : C.n_pages, s);
}

hipError_t launch_kv4_compact(const larosa_kv4_cache& C, int32_t* live, const Kv4Scratch& x, hipStream_t s) {
  hipLaunchKernelGGL(kv4_compact_kernel, dim3(1), dim3(kBook), 0, s, C, live, x);
  if (hipError_t e = hipGetLastError()) return e;
  const size_t entries = static_cast<size_t>(C.n_slots) * C.max_pages;
  hipLaunchKernelGGL(kv4_remap_kernel, dim3(static_cast<unsigned>((entries + 255) / 256)), dim3(256), 0, s, C, x);
  if (hipError_t e = hipGetLastError()) return e;
  return launch_copy(C, x.pair_src, x.pair_dst, x.n_pairs, C.n_pages, s);
}

hipError_t launch_kv4_copy_pages(const larosa_kv4_cache& C, const int32_t* src, const int32_t* dst, int n, hipStream_t s) {
  return launch_copy(C, src, dst, nullptr, n, s);
}

}  // namespace larosa
