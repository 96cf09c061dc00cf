// Log probabilities of given tokens, entropy and the most probable tokens, from logits [n_rows, n_vocab].
//
//   z = scale * logit,  M = max z,  S = sum exp(z - M):   log p(i) = z_i - M - ln S,   H = ln S - sum exp(z - M) (z - M) / S
//
// HBM-bound: every logit is read once (2048 x 128256 bf16 with 20 alternatives 118 us, 4.5 TB/s, in
// an unbroken series 122 - 156; the type takes 65 registers there, one more than eight workgroups a compute unit leave; one row of 32000 is
// a chain of 10 us).  A workgroup of four waves takes a row, or a slice of it where rows are few; a wave goes through it
// by itself, chunk after chunk, against the largest logit it has seen.  Slices meet through memory: the workgroup that arrives last joins them.
//  * One logit of the largest value is left out of S and counted: ln S = log1p(the others), which keeps its bits where one token
//    holds nearly all of the probability.
//  * The most probable tokens.  128 logits (the 16 groups of one lane, or of 2, 4, .. lanes with fewer) are a holder, which keeps the largest
//    of them and where it first stood.  The n tokens sought lie among the logits of the n holders with the largest (ties: the earlier
//    place): any other holder's logits are beaten by n of those.  So only these are read again, and the pass over the row does
//    nothing but take maxima, whatever the order of the logits.  One wave selects.  Its code runs once, so what it costs is fetching it:
//    loops are left as loops (unrolled, with a sorting network for each step, 8 alternatives cost 5 us of latency more).
// Exponentials are the hardware's exp2 of (logit - M) times scale / ln 2: the difference first, so that a row of nothing but the type's
// lowest value, a common mask, is a row like any other.
#include "kernels.hpp"
#include "lds_load.hpp"
#include "numeric.hpp"
#include "w8.hpp"

namespace larosa {

namespace {

typedef unsigned long long u64;
constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kLanes = 256;
constexpr int kGroup = 8;                      // logits of a group
constexpr int kHoldersMax = 2048;              // of a slice: one of 262144 logits
constexpr int kSmallSlice = 4096;              // up to here a wave's chunks are of one group a lane, so that all four have some
constexpr int kLeastSlice = 4096, kLeastOfMany = 24576;   // few rows: no shorter slices, from 128 rows on

__device__ __forceinline__ uint32_t& word_of(uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
struct Logits16 {
  static constexpr int kPer = 8, kBytes = 2;   // logits of 16 bytes, bytes of one
};
struct LF16 : Logits16 {
  static constexpr uint32_t kNothing = 0xFC00FC00u;    // -infinity
  static __device__ __forceinline__ void unpack(const uint4 (&r)[1], float (&v)[8]) { unpack8<F16>(r[0], v); }
};
struct LBF16 : Logits16 {
  static constexpr uint32_t kNothing = 0xFF80FF80u;
  static __device__ __forceinline__ void unpack(const uint4 (&r)[1], float (&v)[8]) { unpack8<BF16>(r[0], v); }
};
struct LF32 {
  static constexpr int kPer = 4, kBytes = 4;
  static constexpr uint32_t kNothing = 0xFF800000u;
  static __device__ __forceinline__ void unpack(const uint4 (&r)[2], float (&v)[8]) {
    v[0] = __uint_as_float(r[0].x); v[1] = __uint_as_float(r[0].y); v[2] = __uint_as_float(r[0].z); v[3] = __uint_as_float(r[0].w);
    v[4] = __uint_as_float(r[1].x); v[5] = __uint_as_float(r[1].y); v[6] = __uint_as_float(r[1].z); v[7] = __uint_as_float(r[1].w);
  }
};

// A row whose first logit lies `head` logits behind a 16-byte boundary: places are counted from that boundary, so that groups are
// aligned; places in front of the row or behind its end hold nothing (-infinity).  Only 16-byte pieces that hold a logit are read.
template <typename L>
struct Row {
  const char* base;
  int head, end;                               // places [head, end)
  __device__ __forceinline__ Row(const void* logits, long ld, long row, int n_vocab) {
    const char* p = static_cast<const char*>(logits) + row * ld * L::kBytes;
    const int off = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15);
    base = p - off;
    head = off / L::kBytes;
    end = head + n_vocab;
  }
  // A piece behind the last that holds a logit is read as that one: no lane takes a branch around its loads (trim sees to the rest).
  template <bool STREAM>
  __device__ __forceinline__ void load(int group, uint4 (&raw)[8 / L::kPer]) const {
#pragma unroll
    for (int h = 0; h < 8 / L::kPer; ++h) {
      typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
      const int piece = min(group * (8 / L::kPer) + h, (end - 1) / L::kPer);
      const u32x4* const p = reinterpret_cast<const u32x4*>(base) + piece;
      const u32x4 v = STREAM ? __builtin_nontemporal_load(p) : *p;
      raw[h] = make_uint4(v.x, v.y, v.z, v.w);
    }
  }
  // logit e of a group becomes -infinity where `out`
  static __device__ __forceinline__ void remove(uint4 (&raw)[8 / L::kPer], int e, bool out) {
    uint32_t& w = word_of(raw[L::kBytes == 4 ? e / 4 : 0], L::kBytes == 4 ? e % 4 : e / 2);
    const uint32_t part = L::kBytes == 4 ? 0xFFFFFFFFu : e % 2 ? 0xFFFF0000u : 0x0000FFFFu;
    w = out ? (w & ~part) | (L::kNothing & part) : w;
  }
  // what lies outside the row (or behind group `stop`) becomes -infinity
  __device__ __forceinline__ void trim(int group, int stop, uint4 (&raw)[8 / L::kPer]) const {
    const int last = min(end, stop * 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) remove(raw, e, (group * 8 + e < head) | (group * 8 + e >= last));
  }
  __device__ __forceinline__ float at(int id) const {
    const char* p = base + (static_cast<long>(head) + id) * L::kBytes;
    if constexpr (L::kBytes == 4) return *reinterpret_cast<const float*>(p);
    else return to_f32(L{}, *reinterpret_cast<const uint16_t*>(p));
  }
  static __device__ __forceinline__ float to_f32(LF16, uint16_t b) { return F16::to_f32(b); }
  static __device__ __forceinline__ float to_f32(LBF16, uint16_t b) { return BF16::to_f32(b); }
};

// Order of candidates: the larger value first, then the earlier place; 0 is below every candidate.
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);        // (-0 counts as 0)
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}
__device__ __forceinline__ u64 candidate(float v, int place) {
  return (static_cast<u64>(key_of(v)) << 32) | (0xFFFFFFFFu - static_cast<uint32_t>(place));
}
__device__ __forceinline__ int place_of(u64 c) { return static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(c)); }

// The value of lane ^ D, without an LDS round trip: quads and rows of 16 lanes by DPP, wider by the lane swaps.
template <int D>
__device__ __forceinline__ uint32_t exchanged(uint32_t v) {
  static_assert(D == 1 || D == 2 || D == 4 || D == 8 || D == 16 || D == 32, "a power of two");
  const int i = static_cast<int>(v);
  if constexpr (D == 1) return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(i, i, 0xB1, 0xF, 0xF, false));        // quad_perm 1 0 3 2
  else if constexpr (D == 2) return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(i, i, 0x4E, 0xF, 0xF, false));   // quad_perm 2 3 0 1
  else if constexpr (D == 4) {                 // four lanes up for the even quads, down for the odd ones
    const int up = __builtin_amdgcn_update_dpp(i, i, 0x104, 0xF, 0x5, false);
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(up, i, 0x114, 0xF, 0xA, false));
  } else if constexpr (D == 8) return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(i, i, 0x128, 0xF, 0xF, false));  // row_ror 8
  else {
    const auto x = D == 16 ? __builtin_amdgcn_permlane16_swap(v, v, false, false) : __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return (threadIdx.x & D) ? x[0] : x[1];    // x[0]: the lower half's values in both halves, x[1]: the upper's
  }
}
template <int D>
__device__ __forceinline__ u64 exchanged64(u64 v) {
  const uint32_t lo = exchanged<D>(static_cast<uint32_t>(v)), hi = exchanged<D>(static_cast<uint32_t>(v >> 32));
  return (static_cast<u64>(hi) << 32) | lo;
}
__device__ __forceinline__ u64 reversed(u64 v) {       // lane 63 - l
  return exchanged64<1>(exchanged64<2>(exchanged64<4>(exchanged64<8>(exchanged64<16>(exchanged64<32>(v))))));
}
__device__ __forceinline__ u64 lane_value(u64 v, int lane) {          // lane: uniform
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(v), lane), hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(v >> 32), lane);
  return (static_cast<u64>(hi) << 32) | lo;
}
// One step of a bitonic network: blocks of K lanes fall and rise in turn; J: distance
template <int K, int J>
__device__ __forceinline__ u64 bitonic_step(u64 v, int lane) {
  const u64 other = exchanged64<J>(v);
  const bool larger = ((lane & J) == 0) == ((lane & K) == 0);
  return (v > other) == larger ? v : other;
}
template <int K, int J>
__device__ __forceinline__ u64 bitonic_merge(u64 v, int lane) {
  v = bitonic_step<K, J>(v, lane);
  if constexpr (J > 1) return bitonic_merge<K, J / 2>(v, lane);
  else return v;
}
// the wave's 64 values, largest first
template <int K = 2>
__device__ __forceinline__ u64 sorted(u64 v, int lane) {
  v = bitonic_merge<K, K / 2>(v, lane);
  if constexpr (K < 64) return sorted<2 * K>(v, lane);
  else return v;
}

__device__ __forceinline__ int lanes_before(u64 mask) {        // of the mask's, before this one
  return static_cast<int>(__builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(mask >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(mask), 0)));
}

// The largest 64 of all values offered, in a wave's lanes.
struct Largest {
  u64 best, least;                             // sorted; what an offered value has to reach
  int count, lane, n;
  u64* buf;                                    // [128] of LDS: offered, not yet sorted in
  __device__ __forceinline__ Largest(u64* b, int lane_, int n_, u64 least_) : best(0), least(least_), count(0), lane(lane_), n(n_), buf(b) {}
  static __device__ __forceinline__ void order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  __device__ __forceinline__ void merge(u64 v) {
    v = sorted(v, lane);
    if (best_empty()) {
      best = v;
      return;
    }
    const u64 back = reversed(v);              // beside best: the larger of each pair are the 64 largest of both, falling and rising
    best = bitonic_merge<64, 32>(best > back ? best : back, lane);
  }
  __device__ __forceinline__ void offer(u64 v) {       // 0: nothing
    const bool in = v >= least && v != 0;
    const u64 mask = __ballot(in);
    if (!mask) return;
    const int at = count + lanes_before(mask);
    if (in) buf[at] = v;
    count += __popcll(mask);
    if (count >= 64) {
      order();
      const u64 now = buf[lane], rest = buf[64 + lane];
      order();
      buf[lane] = rest;
      order();
      count -= 64;
      merge(now);
      const u64 nth = lane_value(best, n - 1);
      if (nth > least) least = nth;
    }
  }
  __device__ __forceinline__ bool best_empty() const { return lane_value(best, 0) == 0; }
  __device__ __forceinline__ void done() {
    if (count == 0) return;
    order();
    merge(lane < count ? buf[lane] : 0);
    order();
    count = 0;
  }
};

__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, __uint_as_float(exchanged<32>(__float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(exchanged<16>(__float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(exchanged<8>(__float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(exchanged<4>(__float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(exchanged<2>(__float_as_uint(v))));
  return fmaxf(v, __uint_as_float(exchanged<1>(__float_as_uint(v))));
}

// Holders of W lanes: the largest of each, in all its lanes.
template <int W>
__device__ __forceinline__ u64 holders_largest(u64 v) {
  if constexpr (W > 1) {
    const u64 other = exchanged64<W / 2>(v);
    return holders_largest<W / 2>(v > other ? v : other);
  } else {
    return v;
  }
}

// What is known of a part of a row: its largest logit, how many logits of that value are left out (one at most of a wave's), the sum of
// the other exponentials against it, and the sum of exponential times exponent (in powers of 2).
struct Part { float most, left_out, others, moment; };

// The parts in the lanes, as one (in all lanes).
__device__ __forceinline__ Part joined(Part p, float c) {
  const float M = wave_max(p.most);
  const bool nan = !(p.others < INFINITY);
  if (p.most < M) {
    const float n = p.most > -INFINITY ? p.left_out + p.others : 0.f;
    const float u = fmaxf((p.most - M) * c, -200.f), f = p.most > -INFINITY ? __builtin_amdgcn_exp2f(u) : 0.f;
    p.moment = f * fmaf(n, u, p.moment);
    p.others = n * f;
    p.left_out = 0.f;
  }
  p.others = wave_sum(p.others);
  p.moment = wave_sum(p.moment);
  p.left_out = wave_sum(p.left_out);
  if (__ballot(nan)) p.others = NAN;
  p.most = M;
  return p;
}

// A wave goes through its chunks (64 lanes x G groups, each wave of the workgroup every fourth) with the next one's loads on the way.  Chunks
// are taken against the largest logit so far: sums are rescaled only when it grows, a few times a row.
template <typename L, int G>
__global__ __launch_bounds__(kLanes) void logprobs_kernel(LogprobsArgs a) {
  constexpr int W = 16 / G;                    // lanes of a holder: 16 groups
  constexpr int kHolders = 64 / W;             // of a chunk
  __shared__ __attribute__((aligned(16))) u64 bests[kHoldersMax];
  __shared__ u64 buf[128];
  __shared__ Part parts[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row_int = __builtin_amdgcn_readfirstlane(static_cast<int>(blockIdx.x / static_cast<unsigned>(a.slices)));
  const long row_no = row_int;
  const int slice = static_cast<int>(blockIdx.x) - row_int * a.slices;
  const Row<L> row(a.logits, a.ld, row_no, a.n_vocab);
  const int per = a.slice_len / kGroup, first = slice * per;
  const int stop = min(first + per, (row.end + 7) / 8);                 // groups of the slice
  const int chunks = (per + 64 * G - 1) / (64 * G), count = a.slices * chunks * kHolders;
  const float c = a.scale * kLog2E;

  uint4 raw[G][8 / L::kPer], next[G][8 / L::kPer];
  auto load = [&](int chunk, uint4 (&to)[G][8 / L::kPer]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < G; ++i) {
      row.template load<true>(first + (chunk * G + i) * 64 + lane, to[i]);
    }
  };
  // the given tokens' logits (64 at most) are on their way before they are needed
  int id = -1;
  float id_logit = 0.f;
  if (wave == 0 && lane < a.n_given) {
    id = a.given[row_no * a.n_given + lane];
    if (id >= 0 && id < a.n_vocab) id_logit = row.at(id);
  }

  float M = -INFINITY, left_out = 0.f, sum = 0.f, moment = 0.f;         // of the wave so far; M and left_out uniform
  auto process = [&](int chunk, uint4 (&raw)[G][8 / L::kPer]) __attribute__((always_inline)) {
    const int g0 = first + chunk * G * 64;
    if (g0 * 8 < row.head || (g0 + G * 64) * 8 > row.end || g0 + G * 64 > stop) {       // (uniform: a chunk at an end of the row)
#pragma unroll
      for (int i = 0; i < G; ++i) row.trim(g0 + i * 64 + lane, stop, raw[i]);
    }
    float most = -INFINITY;
    int where = 0;
#pragma unroll
    for (int i = 0; i < G; ++i) {
      float v[8];
      L::unpack(raw[i], v);
      const float m = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
      if (m > most) {
        most = m;
        where = i;
      }
    }
    if (a.n_top > 0) {
      const u64 mine = holders_largest<W>(g0 + lane < stop ? candidate(most, (g0 + where * 64 + lane) * 8) : 0);
      const int at = chunk * kHolders + lane / W;
      if (lane % W == 0) {
        if (a.slices > 1) __hip_atomic_store(a.best + row_no * count + slice * (chunks * kHolders) + at, mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        else bests[at] = mine;
      }
    }
    // the logits wait as they came: without this the compiler would keep them unpacked, in twice the registers
#pragma unroll
    for (int i = 0; i < G; ++i)
#pragma unroll
      for (int h = 0; h < 8 / L::kPer; ++h) asm volatile("" : "+v"(raw[i][h].x), "+v"(raw[i][h].y), "+v"(raw[i][h].z), "+v"(raw[i][h].w));
    const float top = wave_max(most);
    if (top > M) {                             // (uniform) the largest so far: one of it is left out, the one before counts again
      if (M > -INFINITY) {
        const float u = fmaxf((M - top) * c, -200.f), f = __builtin_amdgcn_exp2f(u);
        if (lane == 0) sum += left_out;
        moment = f * fmaf(sum, u, moment);
        sum *= f;
      }
      M = top;
      left_out = 1.f;
      bool out = lane != static_cast<int>(__builtin_ctzll(__ballot(most == top)));
#pragma unroll
      for (int i = 0; i < G; ++i) {
        float v[8];
        L::unpack(raw[i], v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool now = !out & (v[e] == top);
          Row<L>::remove(raw[i], e, now);
          out |= now;
        }
      }
    }
    const float ref = M == -INFINITY ? 0.f : M;
    float s = 0.f, t = 0.f;
#pragma unroll
    for (int i = 0; i < G; ++i) {
      float v[8];
      L::unpack(raw[i], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float u = (v[e] - ref) * c;
        const float x = __builtin_amdgcn_exp2f(u);
        s += x;
        t = fmaf(x, fmaxf(u, -200.f), t);      // (0 times -infinity)
      }
    }
    sum += s;
    moment += t;
  };
  // (two chunks a turn: copied into place, the next one's loads would be waited for at once)
  load(wave, raw);
  for (int chunk = wave; chunk < chunks; chunk += 8) {
    load(chunk + 4, next);
    process(chunk, raw);
    if (chunk + 4 >= chunks) break;
    load(chunk + 8, raw);
    process(chunk + 4, next);
  }
  sum = wave_sum(sum);
  moment = wave_sum(moment);
  if (lane == 0) parts[wave] = Part{M, left_out, sum, moment};

  // ---- the row's slices meet
  // candidates come 16 to a lane (eight 16-byte loads, coherent across the chip); up to 1024 are read once
  constexpr int kAtOnce = 16;
  u64 held_by[kAtOnce];
  auto load_holders = [&](int i0) __attribute__((always_inline)) {
    if (a.slices > 1) {
      typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
      const __amdgpu_buffer_rsrc_t all = __builtin_amdgcn_make_buffer_rsrc(a.best + row_no * count, 0, count * 8, 0x00027000);
#pragma unroll
      for (int i = 0; i < kAtOnce; i += 2) {
        const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(all, (i0 + i * 64 + lane * 2) * 8, 0, 16);
        held_by[i] = (static_cast<u64>(v.y) << 32) | v.x;
        held_by[i + 1] = (static_cast<u64>(v.w) << 32) | v.z;
      }
    } else {
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) held_by[i] = i0 + i * 64 + lane < count ? bests[i0 + i * 64 + lane] : 0;
    }
  };
  if (a.slices > 1) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // the wave's holders
  __syncthreads();
  if (wave != 0) return;
  const Part none{-INFINITY, 0.f, 0.f, 0.f};
  Part p = joined(lane < 4 ? parts[lane & 3] : none, c);
  if (a.slices > 1) {
    float* const sums = a.sums + row_no * a.slices * 4;
    if (lane < 4)
      __hip_atomic_store(sums + slice * 4 + lane, lane == 0 ? p.most : lane == 1 ? p.left_out : lane == 2 ? p.others : p.moment, __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    unsigned old = 0;
    if (lane == 0) old = __hip_atomic_fetch_add(a.counters + row_no, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (__builtin_amdgcn_readfirstlane(old) != static_cast<unsigned>(a.slices - 1)) return;
    if (lane == 0) __hip_atomic_store(a.counters + row_no, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("" ::: "memory");
    if (a.n_top > 0) load_holders(0);          // (with the slices' sums, not behind them)
    Part all = none;
    for (int i0 = 0; i0 < a.slices; i0 += 64) {
      Part q = none;
      if (i0 + lane < a.slices) {
        const float* const from = sums + (i0 + lane) * 4;
        q.most = __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        q.left_out = __hip_atomic_load(from + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        q.others = __hip_atomic_load(from + 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        q.moment = __hip_atomic_load(from + 3, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      q = joined(q, c);
      all = i0 == 0 ? q : joined(lane == 0 ? all : lane == 1 ? q : none, c);
    }
    p = all;
  }
  M = p.most;
  left_out = p.left_out;
  const float others = p.others, moments = p.moment;
  const bool undefined = !(others < INFINITY) || M == INFINITY;
  const bool nothing = M == -INFINITY && !undefined;
  const float log_sum = log1pf(left_out - 1.f + others);
  auto logp_of = [&](float x) __attribute__((always_inline)) {
    if (undefined) return NAN;
    return nothing || x == -INFINITY ? -INFINITY : (x - M) * a.scale - log_sum;
  };
  if (a.entropy && lane == 0) a.entropy[row_no] = undefined ? NAN : nothing ? 0.f : log_sum - kLn2 * moments / (left_out + others);
  for (int i = lane; i < a.n_given; i += 64) {
    if (i >= 64) {
      id = a.given[row_no * a.n_given + i];
      id_logit = id >= 0 && id < a.n_vocab ? row.at(id) : 0.f;
    }
    a.logp[row_no * a.n_given + i] = id < 0 ? 0.f : id < a.n_vocab ? logp_of(id_logit) : NAN;
  }
  if (a.n_top == 0) return;

  // ---- the lanes that hold the most probable tokens, then the tokens
  int* const ids = a.top_id + row_no * a.n_top;
  float* const tops = a.top_logp ? a.top_logp + row_no * a.n_top : nullptr;
  if (undefined) {
    for (int i = lane; i < a.n_top; i += 64) {
      ids[i] = -1;
      if (tops) tops[i] = NAN;
    }
    return;
  }
  const int n = a.n_top;
  // n lanes at least have a largest holder of key t or more, so n candidates do
  u64 mine = 0;
  if (a.slices == 1) load_holders(0);
  for (int i0 = 0; i0 < count; i0 += 64 * kAtOnce) {
    if (i0 > 0) load_holders(i0);
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) mine = held_by[i] > mine ? held_by[i] : mine;
  }
  const uint32_t mine_key = static_cast<uint32_t>(mine >> 32);
  uint32_t t = 0;
#pragma unroll 1
  for (uint32_t bit = 0x80000000u; bit; bit >>= 1)
    if (__popcll(__ballot(mine_key >= (t | bit))) >= n) t |= bit;
  u64 least = static_cast<u64>(t) << 32;
  // holders that reach it: a few more than n, unless logits are alike
  int found = 0;
  for (int i0 = 0; i0 < count; i0 += 64 * kAtOnce) {
    if (count > 64 * kAtOnce) load_holders(i0);
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const bool in = held_by[i] >= least && held_by[i] != 0;
      const u64 mask = __ballot(in);
      const int at = found + lanes_before(mask);
      if (in && at < 64) buf[at] = held_by[i];
      found += __popcll(mask);
    }
  }
  Largest::order();
  u64 mine_held = lane < found ? buf[lane] : 0;
  Largest::order();
  if (found > 64) {                            // the n largest of them
    Largest holders(buf, lane, n, least);
    for (int i = lane; i - lane < count; i += 64)
      holders.offer(i >= count ? 0 : a.slices > 1 ? __hip_atomic_load(a.best + row_no * count + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : bests[i]);
    holders.done();
    found = n;
    mine_held = holders.best;
    least = lane_value(holders.best, n - 1) - 7;       // (its place is its group's first: the logit lies at most 7 further)
  }
  const float least_value = value_of(static_cast<uint32_t>(least >> 32));      // (of nothing: NaN, see below)

  // The holders' logits, 16 lanes to a holder, a group each: straight into LDS, so that all are on their way at once.
  int holder0 = -1, holder_stop = 0;           // of the lane's holder: its first group, where its slice ends
  if (lane < found && mine_held != 0) {
    const int group0 = place_of(mine_held) / 8;        // one of its groups: its lane and its slice
    const int from_slice = group0 / per, in_slice = group0 - from_slice * per;
    holder0 = from_slice * per + in_slice / (64 * G) * (64 * G) + in_slice % 64 / W * W;
    holder_stop = min((from_slice + 1) * per, (row.end + 7) / 8);
  }
  const int within = lane % 16 % W + lane % 16 / W * 64;
  auto group_of = [&](int j) __attribute__((always_inline)) {
    const int h = 4 * j + lane / 16, first = __shfl(holder0, h), end = __shfl(holder_stop, h);   // (both by all lanes)
    return first >= 0 && first + within < end ? first + within : -1;
  };
  constexpr int kPieces = 8 / L::kPer, kReads = kHoldersMax * 8 / (1024 * kPieces);
  const auto buffer = raw_buffer(row.base, static_cast<uint32_t>((row.end - 1) / L::kPer + 1) * 16u);
  const uint32_t staged = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_char*)bests));
  Largest tokens(buf, lane, n, least);
  for (int j0 = 0; 4 * j0 < found; j0 += kReads) {
    const int reads = min(kReads, (found + 3) / 4 - j0);
#pragma unroll 1
    for (int j = 0; j < reads; ++j) {
      const int group = group_of(j0 + j);
#pragma unroll
      for (int h = 0; h < kPieces; ++h)
        load_to_lds(buffer, staged + (j * kPieces + h) * 1024, group < 0 ? kOutside : static_cast<uint32_t>((group * kPieces + h) * 16));
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll 1
    for (int j = 0; j < reads; ++j) {
      const int group = group_of(j0 + j);
      uint4 again[kPieces];
#pragma unroll
      for (int h = 0; h < kPieces; ++h) again[h] = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(bests) + (j * kPieces + h) * 1024 + lane * 16);
      float v[8];
      L::unpack(again, v);
      uint32_t bits = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) bits |= v[e] < least_value ? 0u : 1u << e;
      if (group < 0) bits = 0;
#pragma unroll 1
      while (__ballot(bits != 0)) {
        const int e = __ffs(static_cast<int>(bits)) - 1;
        float x = v[0];
#pragma unroll
        for (int k = 1; k < 8; ++k) x = e == k ? v[k] : x;
        const int place = group * 8 + e;
        tokens.offer(bits != 0 && place >= row.head && place < row.end ? candidate(x, place) : 0);
        bits &= bits - 1;
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
  auto answer = [&](int at, u64 token) __attribute__((always_inline)) {
    ids[at] = place_of(token) - row.head;
    if (tops) tops[at] = logp_of(value_of(static_cast<uint32_t>(token >> 32)));
  };
  if (tokens.best_empty()) {                   // at most 63 came: each finds its place by counting
    Largest::order();
    const u64 token = lane < tokens.count ? buf[lane] : 0;
    int rank = 0;
#pragma unroll 1
    for (int i = 0; i < tokens.count; ++i) rank += lane_value(token, i) > token;
    if (lane < tokens.count && rank < n) answer(rank, token);
  } else {
    tokens.done();
    if (lane < n) answer(lane, tokens.best);
  }
}

template <typename L>
hipError_t launch_type(const LogprobsArgs& a, hipStream_t s) {
  const unsigned grid = static_cast<unsigned>(a.n_rows) * static_cast<unsigned>(a.slices);
  if (a.slice_len <= kSmallSlice) logprobs_kernel<L, 1><<<grid, kLanes, 0, s>>>(a);
  else logprobs_kernel<L, 4><<<grid, kLanes, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

LogprobsPlan plan_logprobs(int n_rows, int n_vocab, int n_top) {
  LogprobsPlan p{};
  const long places = static_cast<long>(n_vocab) + 7;                   // a row may start inside a group
  constexpr long kMost = kHoldersMax / 16 * 2048;                       // a slice's holders lie in LDS
  long slices = (places + kMost - 1) / kMost;
  if (n_rows * slices < kWorkgroupsOfFew) {                             // few rows: slices for all compute units
    const long fine = places / (n_rows < 128 ? kLeastSlice : kLeastOfMany), want = (kWorkgroupsOfFew + n_rows - 1) / n_rows;
    const long more = want < fine ? want : fine;
    if (more > slices) slices = more;
  }
  p.slice_len = static_cast<int>(((places + slices - 1) / slices + kGroup - 1) / kGroup * kGroup);
  p.slices = static_cast<int>((places + p.slice_len - 1) / p.slice_len);
  if (p.slices > 1) {
    p.sums_bytes = static_cast<size_t>(p.slices) * 4 * sizeof(float);
    const int chunk = p.slice_len <= kSmallSlice ? 512 : 2048, holders = chunk / 128;
    p.best_bytes = n_top > 0 ? static_cast<size_t>(p.slices) * ((p.slice_len + chunk - 1) / chunk) * holders * sizeof(u64) : 0;
  }
  return p;
}

hipError_t launch_logprobs(const LogprobsArgs& a, int type, hipStream_t s) {
  if (type == kLogitsF32) return launch_type<LF32>(a, s);
  return type == kLogitsBF16 ? launch_type<LBF16>(a, s) : launch_type<LF16>(a, s);
}

}  // namespace larosa
