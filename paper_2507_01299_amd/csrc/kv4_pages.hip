// Pages of the 4-bit key/value cache: hand out, share, free, pack and copy.  The bookkeeping of a call is one workgroup's work
// (a few hundred slots and pages: latency-bound); the pages' bytes are moved by a launch of their own that reads the list the first one
// left, in 16-byte pieces over all layers (bound by HBM: every byte read and written once).
#include "kernels.hpp"
#include "kv4.hpp"
#include "numeric.hpp"

namespace larosa {

namespace {

constexpr int kBook = 1024;   // lanes of a bookkeeping workgroup

// (unsigned: a number of tokens may be up to 2^31 - 1)
__device__ __forceinline__ int pages_for(int tokens, int page_tokens) {
  return static_cast<int>((static_cast<unsigned>(tokens) + page_tokens - 1) / page_tokens);
}

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
  // keep may exceed what the sequence has, by anything: its pages then all stay
  const int from = pages_for(max(0, min(kept, had)), C.page_tokens), to = min(pages_for(max(0, had), C.page_tokens), C.max_pages);
  for (int p = from + lane; p < to; p += 64) {
    const int page = atomicExch(&C.table[static_cast<size_t>(slot) * C.max_pages + p], -1);
    if (page >= 0 && page < C.n_pages) atomicSub(&C.refs[page], 1);
  }
}

// ---- fork -------------------------------------------------------------------------------------------

// Whether the list is in order.  A free destination is marked by a negative length; a second mark, or a source that carries one,
// gives the fault away.  Marks are taken back where the list is refused.  `whole`: the tables are copied here too (few
// entries: the next launch would take longer than they do).
__global__ __launch_bounds__(kBook) void kv4_fork_check_kernel(larosa_kv4_cache C, const int32_t* src, const int32_t* dst, int n,
                                                               int32_t* status, bool whole) {
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
  if (bad || !whole) return;
  for (int i = threadIdx.x; i < n; i += kBook) C.length[dst[i]] = atomicAdd(&C.length[src[i]], 0);
#pragma unroll 4
  for (int e = threadIdx.x; e < n * C.max_pages; e += kBook) {
    const int i = e / C.max_pages, p = e - i * C.max_pages;
    const int page = C.table[static_cast<size_t>(src[i]) * C.max_pages + p];
    C.table[static_cast<size_t>(dst[i]) * C.max_pages + p] = page;
    if (page >= 0 && page < C.n_pages) atomicAdd(&C.refs[page], 1);
  }
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

// Which of the eight pages [p0 + 8 tid, ..) are free, as bits.
__device__ __forceinline__ uint32_t free_bits(const larosa_kv4_cache& C, int p0) {
  int r[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int p = p0 + static_cast<int>(threadIdx.x) * 8 + k;
    r[k] = p < C.n_pages ? C.refs[p] : 1;
  }
  uint32_t bits = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) bits |= (r[k] == 0 ? 1u : 0u) << k;
  return bits;
}

// Latency-bound: a chain of loads (slot, length, table, references), the free pages looked for beside it.  A lane keeps what it found out
// about its slot; lists longer than the workgroup look again.
__global__ __launch_bounds__(kBook) void kv4_grow_kernel(larosa_kv4_cache C, const int32_t* slots, const int32_t* counts,
                                                         int32_t* status, Kv4Scratch x, int n) {
  __shared__ int bad, shared_pages, many;
  __shared__ uint32_t listed[kKv4SlotsMax / 32];
  __shared__ int s_ids[2 * kBook], s_offset[kBook], s_pair[kBook];
  const int tid = threadIdx.x;
  const uint32_t first_free = free_bits(C, 0);
  Want mine{};
  mine.slot = -1;
  if (tid < n) mine = want_of(C, slots, counts, tid);
  auto want = [&](int i) { return i < kBook ? mine : want_of(C, slots, counts, i); };
  for (int k = tid; k < (C.n_slots + 31) / 32; k += kBook) listed[k] = 0;
  if (tid == 0) {
    bad = shared_pages = many = 0;
    *x.n_pairs() = 0;
  }
  __syncthreads();
  for (int i = tid; i < n; i += kBook) {
    const Want w = want(i);
    if (w.slot < 0 || (atomicOr(&listed[w.slot / 32], 1u << (w.slot % 32)) >> (w.slot % 32) & 1)) {
      bad = 1;
      continue;
    }
    if (w.page >= 0) {
      shared_pages = 1;
      atomicExch(&x.growing(C)[w.page], 0);
      atomicExch(&x.last(C)[w.page], 0);
    }
  }
  __syncthreads();
  if (bad) {
    if (tid == 0) *status = -1;
    return;
  }
  if (shared_pages) {
    for (int i = tid; i < n; i += kBook) {
      const Want w = want(i);
      if (w.page >= 0) {
        atomicAdd(&x.growing(C)[w.page], 1);
        atomicMax(&x.last(C)[w.page], i + 1);
      }
    }
    __syncthreads();
  }
  // pages for each slot of the list, in its order: a copy of the shared page first, then the new ones
  int* const offset = n <= kBook ? s_offset : x.offset(C);
  int* const pair = n <= kBook ? s_pair : x.pair(C);
  unsigned wanted = 0, copies = 0;
  for (int i0 = 0; i0 < n; i0 += kBook) {
    const int i = i0 + tid;
    Want w{};
    bool copy = false;
    if (i < n) {
      w = want(i);
      copy = w.page >= 0 && !(atomicAdd(&x.growing(C)[w.page], 0) == C.refs[w.page] && atomicAdd(&x.last(C)[w.page], 0) == i + 1);
    }
    const Sums s = book_scan(w.new_pages - w.old_pages + copy, copy);
    if (i < n) {
      offset[i] = static_cast<int>(wanted + s.a);
      pair[i] = copy ? static_cast<int>(copies + s.b) : -1;
      // (more copies than pages: the call is refused below)
      if (copy && copies + s.b < static_cast<unsigned>(C.n_pages)) x.pair_src(C)[copies + s.b] = w.page;
    }
    wanted += s.all_a;
    copies += s.all_b;
  }
  // the lowest free pages, eight to a lane at a time
  int* const ids = wanted <= 2 * kBook ? s_ids : x.ids(C);
  unsigned found = 0;
  for (int p0 = 0; p0 < C.n_pages && found < wanted; p0 += kBook * 8) {
    const uint32_t free8 = p0 == 0 ? first_free : free_bits(C, p0);
    const Sums s = book_scan(__popc(free8), 0);
    unsigned at = found + s.a;
    for (int k = 0; k < 8; ++k)
      if (free8 >> k & 1) {
        if (at < wanted) ids[at] = p0 + tid * 8 + k;
        ++at;
      }
    found += s.all_a;
  }
  if (found < wanted) {
    if (tid == 0) *status = static_cast<int>(wanted - found);
    return;
  }
  __syncthreads();            // the ids and offsets are written
  auto give = [&](const Want& w, int i, int r) {              // page r of what slot i of the list gets
    const int page = ids[offset[i] + r], copied = pair[i] >= 0 ? 1 : 0;
    C.table[static_cast<size_t>(w.slot) * C.max_pages + w.old_pages - copied + r] = page;
    C.refs[page] = 1;
    if (copied && r == 0) {
      x.pair_dst(C)[pair[i]] = page;
      atomicSub(&C.refs[x.pair_src(C)[pair[i]]], 1);
    }
  };
  constexpr int kFew = 4;     // a lane gives its slot so many; slots that get more are a wave's work each
  for (int i = tid; i < n; i += kBook) {
    const Want w = want(i);
    const int gets = w.new_pages - w.old_pages + (pair[i] >= 0 ? 1 : 0);
    for (int r = 0; r < min(gets, kFew); ++r) give(w, i, r);
    if (gets > kFew) many = 1;
  }
  __syncthreads();
  if (many)
    for (int i = tid / 64; i < n; i += kBook / 64) {
      const Want w = want_of(C, slots, counts, i);
      const int gets = w.new_pages - w.old_pages + (pair[i] >= 0 ? 1 : 0);
      for (int r = kFew + tid % 64; r < gets; r += 64) give(w, i, r);
    }
  __syncthreads();            // the lengths are read above
  for (int i = tid; i < n; i += kBook) {
    const Want w = want(i);
    C.length[w.slot] = w.had + w.count;
  }
  if (tid == 0) {
    *x.n_pairs() = static_cast<int>(copies);
    *status = 0;
  }
}

// ---- compact ------------------------------------------------------------------------------------------

__global__ __launch_bounds__(kBook) void kv4_compact_kernel(larosa_kv4_cache C, int32_t* live, Kv4Scratch x) {
  const int tid = threadIdx.x;
  const uint32_t first_free = free_bits(C, 0);
  auto free8_at = [&](int p0) { return p0 == 0 ? first_free : free_bits(C, p0); };
  unsigned n_free = 0;
  for (int p0 = 0; p0 < C.n_pages; p0 += kBook * 8) n_free += book_scan(__popc(free8_at(p0)), 0).all_a;
  const int n_live = C.n_pages - static_cast<int>(n_free);
  // free ids below n_live and live ids from it on, both ascending: as many of the one as of the other
  unsigned holes = 0, movers = 0;
  for (int p0 = 0; p0 < C.n_pages; p0 += kBook * 8) {
    const uint32_t free8 = free8_at(p0);
    const int p = p0 + tid * 8;
    const uint32_t below = n_live <= p ? 0u : n_live - p >= 8 ? 0xFFu : (1u << (n_live - p)) - 1u;
    const uint32_t there = C.n_pages <= p ? 0u : C.n_pages - p >= 8 ? 0xFFu : (1u << (C.n_pages - p)) - 1u;
    const uint32_t hole8 = free8 & below, mover8 = ~free8 & ~below & there;
    const Sums s = book_scan(__popc(hole8), __popc(mover8));
    unsigned a = holes + s.a, b = movers + s.b;
    for (int k = 0; k < 8; ++k) {
      if (hole8 >> k & 1) x.pair_dst(C)[a++] = p + k;
      if (mover8 >> k & 1) x.pair_src(C)[b++] = p + k;
    }
    holes += s.all_a;
    movers += s.all_b;
  }
  __syncthreads();
  for (unsigned k = tid; k < movers; k += kBook) {
    const int from = x.pair_src(C)[k], to = x.pair_dst(C)[k];
    x.ids(C)[from] = to;
    C.refs[to] = C.refs[from];
    C.refs[from] = 0;
  }
  if (tid == 0) {
    *x.n_pairs() = static_cast<int>(movers);
    *x.n_live() = n_live;
    if (live) *live = n_live;
  }
}

// ---- copies -------------------------------------------------------------------------------------------

constexpr int kCopyUnroll = 4, kCopyPieces = 256 * kCopyUnroll;      // 16-byte pieces of a workgroup's step
typedef uint32_t piece_t __attribute__((ext_vector_type(4)));

template <bool STREAM>
__device__ __forceinline__ void copy_step(const piece_t* a, piece_t* b, unsigned pieces) {
  if (pieces >= kCopyPieces) {
    piece_t v[kCopyUnroll];
#pragma unroll
    for (int k = 0; k < kCopyUnroll; ++k) v[k] = STREAM ? __builtin_nontemporal_load(a + 256 * k + threadIdx.x) : a[256 * k + threadIdx.x];
#pragma unroll
    for (int k = 0; k < kCopyUnroll; ++k) {
      if (STREAM)
        __builtin_nontemporal_store(v[k], b + 256 * k + threadIdx.x);
      else
        b[256 * k + threadIdx.x] = v[k];
    }
  } else {
    for (unsigned k = threadIdx.x; k < pieces; k += 256) b[k] = a[k];
  }
}

// Pages src[i] into dst[i], all layers; the pairs' number comes from n_pairs or, where that is null, from n.  With `remap`, ids
// that a packing has moved change in the tables as well.  Layer by layer, so that neighbouring pages move at the same time (packing
// 170 pages of 2.2 MB: 145 us pair by pair, 120 so; a copy of 4 GiB would take 164 for as much, but part of this stays in the 256 MB cache
// behind the L2s); what that cache does not hold passes them by (128 us without; but 23 MB take 6.4 us through them, 7.4 past them).
__global__ __launch_bounds__(256) void kv4_copy_kernel(larosa_kv4_cache C, const int32_t* src, const int32_t* dst, const int32_t* n_pairs,
                                                       Kv4Scratch remap, int n, unsigned page_pieces, unsigned grid) {
  if (n_pairs) n = *n_pairs;
  if (remap.base) {
    const int32_t* to = remap.ids(C);
    const unsigned entries = static_cast<unsigned>(C.n_slots) * C.max_pages;
    for (unsigned e = blockIdx.x * 256 + threadIdx.x; e < entries; e += grid * 256) {
      const int page = C.table[e];
      if (page >= *remap.n_live() && page < C.n_pages) C.table[e] = to[page];
    }
  }
  const unsigned steps = (page_pieces + kCopyPieces - 1) / kCopyPieces;
  const unsigned items = static_cast<unsigned>(n) * C.n_layers * steps;        // (16 KiB each: far below 2^32 in any memory)
  const bool stream = static_cast<size_t>(n) * C.n_layers * page_pieces * 32 > (static_cast<size_t>(256) << 20);
  piece_t* data = static_cast<piece_t*>(C.data);
  for (unsigned it = blockIdx.x; it < items; it += grid) {
    const unsigned rest = it / steps, first = (it - rest * steps) * kCopyPieces;
    const unsigned layer = rest / n, i = rest - layer * n;
    const int from = src[i], into = dst[i];
    if (from < 0 || from >= C.n_pages || into < 0 || into >= C.n_pages) continue;
    const size_t base = static_cast<size_t>(layer) * C.n_pages;
    const piece_t* a = data + (base + from) * page_pieces + first;
    piece_t* b = data + (base + into) * page_pieces + first;
    if (stream)
      copy_step<true>(a, b, page_pieces - first);
    else
      copy_step<false>(a, b, page_pieces - first);
  }
}

hipError_t launch_copy(const larosa_kv4_cache& C, const int32_t* src, const int32_t* dst, const int32_t* n_pairs, Kv4Scratch remap, int n,
                       hipStream_t s) {
  const unsigned page_pieces = static_cast<unsigned>(C.n_kv_heads) * (C.page_tokens / 32) * 34 * C.head_dim / 16;
  const size_t items = static_cast<size_t>(n) * C.n_layers * ((page_pieces + kCopyPieces - 1) / kCopyPieces);
  // (packing with 758 MB to move: 135.6 us, with 2048 workgroups 145, 65536 138.4; smaller calls take as long with any)
  const unsigned grid = static_cast<unsigned>(items < 16384 ? items : 16384);
  return kv4_launch(kv4_copy_kernel, dim3(grid), dim3(256), s, C, src, dst, n_pairs, remap, n, page_pieces, grid);
}

}  // namespace

hipError_t launch_kv4_trim(const larosa_kv4_cache& C, const int32_t* slots, const int32_t* keep, int n, hipStream_t s) {
  return kv4_launch(kv4_trim_kernel, dim3((n + 3) / 4), dim3(256), s, C, slots, keep, n);
}

hipError_t launch_kv4_fork(const larosa_kv4_cache& C, const int32_t* src, const int32_t* dst, int n, int32_t* status, hipStream_t s) {
  // up to eight entries a lane: 2 us less than with a launch for the tables
  const bool whole = static_cast<long>(n) * C.max_pages <= 8 * kBook;
  if (hipError_t e = kv4_launch(kv4_fork_check_kernel, dim3(1), dim3(kBook), s, C, src, dst, n, status, whole)) return e;
  if (whole) return hipSuccess;
  for (int at = 0; at < n; at += 65535) {
    const dim3 grid((C.max_pages + 255) / 256, n - at < 65535 ? n - at : 65535);
    if (hipError_t e = kv4_launch(kv4_fork_kernel, grid, dim3(256), s, C, src + at, dst + at, static_cast<const int32_t*>(status))) return e;
  }
  return hipSuccess;
}

hipError_t launch_kv4_grow(const larosa_kv4_cache& C, const int32_t* slots, const int32_t* counts, int n, int32_t* status, Kv4Scratch x,
                           hipStream_t s) {
  if (hipError_t e = kv4_launch(kv4_grow_kernel, dim3(1), dim3(kBook), s, C, slots, counts, status, x, n)) return e;
  return launch_copy(C, x.pair_src(C), x.pair_dst(C), x.n_pairs(), Kv4Scratch{nullptr}, n < C.n_pages ? n : C.n_pages, s);
}

hipError_t launch_kv4_compact(const larosa_kv4_cache& C, int32_t* live, Kv4Scratch x, hipStream_t s) {
  if (hipError_t e = kv4_launch(kv4_compact_kernel, dim3(1), dim3(kBook), s, C, live, x)) return e;
  return launch_copy(C, x.pair_src(C), x.pair_dst(C), x.n_pairs(), x, C.n_pages, s);
}

hipError_t launch_kv4_copy_pages(const larosa_kv4_cache& C, const int32_t* src, const int32_t* dst, int n, hipStream_t s) {
  return launch_copy(C, src, dst, nullptr, Kv4Scratch{nullptr}, n, s);
}

}  // namespace larosa
