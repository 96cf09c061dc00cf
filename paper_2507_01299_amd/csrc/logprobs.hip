// Log probabilities of given tokens, entropy and the most probable tokens, from logits [n_rows, n_vocab].
//
//   z = scale * logit,  M = max z,  S = sum exp(z - M):   log p(i) = z_i - M - ln S,   H = ln S - sum exp(z - M) (z - M) / S
//
// HBM-bound: every logit is read once.  A workgroup of 256 lanes takes a slice of a row, at most 16 groups of 8 logits a lane, which
// wait in registers while the slice's maximum is found: the exponentials are taken once, against the slice's own maximum, and sums are
// never rescaled on the way.  Several slices of a row meet through memory: the workgroup that arrives last at the row joins them.
//  * One logit of the largest value is left out of S and counted: ln S = log1p(the others), which keeps its bits where one token
//    holds nearly all of the probability.
//  * The most probable tokens.  128 logits (the 16 groups of one lane, or of 2, 4, .. lanes with fewer) are a holder, which keeps the largest
//    of them and where it first stood.  The n tokens sought lie among the logits of the n holders with the largest (ties: the earlier
//    place): any other holder's logits are beaten by n of those.  So only these are read again, and the pass over the row does
//    nothing but take maxima, whatever the order of the logits.  One wave selects, in registers, 64 candidates at a time.
// Exponentials are the hardware's exp2 of (logit - M) times scale / ln 2: the difference first, so that a row of nothing but the type's
// lowest value, a common mask, is a row like any other.
#include "kernels.hpp"
#include "numeric.hpp"
#include "w8.hpp"

namespace larosa {

namespace {

typedef unsigned long long u64;
constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kLanes = 256;
constexpr int kGroup = 8;                      // logits of a group

struct Logits16 { using Raw = uint4; static constexpr int kPer = 8, kBytes = 2; };
struct LF16 : Logits16 { static __device__ __forceinline__ void unpack(const uint4 (&r)[1], float (&v)[8]) { unpack8<F16>(r[0], v); } };
struct LBF16 : Logits16 { static __device__ __forceinline__ void unpack(const uint4 (&r)[1], float (&v)[8]) { unpack8<BF16>(r[0], v); } };
struct LF32 {
  static constexpr int kPer = 4, kBytes = 4;   // logits of 16 bytes
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
  __device__ __forceinline__ void load(int group, uint4 (&raw)[8 / L::kPer], bool stream) const {
#pragma unroll
    for (int h = 0; h < 8 / L::kPer; ++h) {
      typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
      const u32x4* p = reinterpret_cast<const u32x4*>(base + (static_cast<long>(group) * 8 + h * L::kPer) * L::kBytes);
      const u32x4 v = group * 8 + h * L::kPer < end ? (stream ? __builtin_nontemporal_load(p) : *p) : u32x4{0u, 0u, 0u, 0u};
      raw[h] = make_uint4(v.x, v.y, v.z, v.w);
    }
  }
  __device__ __forceinline__ void values(int group, const uint4 (&raw)[8 / L::kPer], float (&v)[8]) const {
    L::unpack(raw, v);
    const int first = group * 8;
    if (first < head || first + 8 > end) {     // (the row's two ends)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = first + e >= head && first + e < end ? v[e] : -INFINITY;
    }
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
__device__ __forceinline__ u64 shuffle_from(u64 v, int lane) {
  const int lo = __shfl(static_cast<int>(static_cast<uint32_t>(v)), lane), hi = __shfl(static_cast<int>(v >> 32), lane);
  return (static_cast<u64>(static_cast<uint32_t>(hi)) << 32) | static_cast<uint32_t>(lo);
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
    if (lane_value(best, 0) == 0) {
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
    const int at = count + static_cast<int>(__builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(mask >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(mask), 0)));
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
  __device__ __forceinline__ void done() {
    if (count == 0) return;
    order();
    merge(lane < count ? buf[lane] : 0);
    order();
    count = 0;
  }
};

struct Sums { float most, left_out, others, moment; };   // largest logit, how many of it are left out, sum of the other exponentials, sum of exponential times exponent

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

template <typename L, int G>
__global__ __launch_bounds__(kLanes, 4) void logprobs_kernel(LogprobsArgs a) {
  constexpr int W = 16 / G;                    // lanes of a holder: 16 groups
  constexpr int kHolders = kLanes / W;         // of a slice
  __shared__ __attribute__((aligned(16))) u64 bests[kHolders];
  __shared__ u64 buf[128];
  __shared__ float red[4][4];
  __shared__ int last_flag;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long row_no = blockIdx.x / static_cast<unsigned>(a.slices);
  const int slice = static_cast<int>(blockIdx.x - row_no * a.slices);
  const Row<L> row(a.logits, a.ld, row_no, a.n_vocab);
  const int per = a.slice_len / kGroup, first = slice * per;
  const int stop = min(first + per, (row.end + 7) / 8);                 // groups of the slice

  // ---- the slice, its maxima
  uint4 raw[G][8 / L::kPer];
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const int group = first + i * kLanes + tid;
    if (group < stop) row.load(group, raw[i], true);
  }
  float most = -INFINITY;
  int where = first + tid;
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const int group = first + i * kLanes + tid;
    if (group < stop) {
      float v[8];
      row.values(group, raw[i], v);
      const float m = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
      if (m > most) {
        most = m;
        where = group;
      }
    }
  }
  {
    const float m = wave_max(most);
    if (lane == 0) red[wave][0] = m;
  }
  if (a.n_top > 0) {
    const u64 mine = holders_largest<W>(first + tid < stop ? candidate(most, where * 8) : 0);
    if (tid % W == 0) {
      if (a.slices > 1) __hip_atomic_store(a.best + (row_no * a.slices + slice) * kHolders + tid / W, mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      else bests[tid / W] = mine;
    }
  }
  __syncthreads();
  const float top = fmaxf(fmaxf(red[0][0], red[1][0]), fmaxf(red[2][0], red[3][0]));
  __syncthreads();

  // ---- the exponentials.  The logits wait as they came: without this the compiler would keep them unpacked, in twice the registers.
#pragma unroll
  for (int i = 0; i < G; ++i)
#pragma unroll
    for (int h = 0; h < 8 / L::kPer; ++h) asm volatile("" : "+v"(raw[i][h].x), "+v"(raw[i][h].y), "+v"(raw[i][h].z), "+v"(raw[i][h].w));
  const float c = a.scale * kLog2E;
  const float ref = top == -INFINITY ? 0.f : top;
  float sum = 0.f, moment = 0.f;
  const bool holds = most == top && top > -INFINITY;
  bool out = !holds;                           // one of the largest logits is left out
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const int group = first + i * kLanes + tid;
    if (group < stop) {
      float v[8];
      row.values(group, raw[i], v);
      if (holds) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!out && v[e] == top) {
            v[e] = -INFINITY;
            out = true;
          }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float u = (v[e] - ref) * c;
        const float x = __builtin_amdgcn_exp2f(u);
        sum += x;
        moment = fmaf(x, fmaxf(u, -200.f), moment);    // (0 times -infinity)
      }
    }
  }
  sum = wave_sum(sum);
  moment = wave_sum(moment);
  const int held = __popcll(__ballot(holds));
  if (lane == 0) {
    red[wave][0] = static_cast<float>(held);
    red[wave][1] = sum;
    red[wave][2] = moment;
  }
  __syncthreads();
  Sums s{top, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    s.left_out += red[k][0];
    s.others += red[k][1];
    s.moment += red[k][2];
  }

  // ---- the row's slices meet
  if (a.slices > 1) {
    float* const to = a.sums + (row_no * a.slices + slice) * 4;
    if (tid < 4) {
      const float v = tid == 0 ? s.most : tid == 1 ? s.left_out : tid == 2 ? s.others : s.moment;
      __hip_atomic_store(to + tid, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) {
      const unsigned old = __hip_atomic_fetch_add(a.counters + row_no, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      last_flag = old == static_cast<unsigned>(a.slices - 1);
    }
    __syncthreads();
    if (!last_flag) return;
    if (tid == 0) __hip_atomic_store(a.counters + row_no, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("" ::: "memory");
  }
  if (wave != 0) return;
  float M = s.most, left_out = s.left_out, others = s.others, moments = s.moment;
  if (a.slices > 1) {
    const float* const from = a.sums + row_no * a.slices * 4;
    M = -INFINITY;
    bool nan = false;
    for (int i = lane; i < a.slices; i += 64) M = fmaxf(M, __hip_atomic_load(from + 4 * i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    M = wave_max(M);
    others = moments = left_out = 0.f;
    for (int i = lane; i < a.slices; i += 64) {
      const float m = __hip_atomic_load(from + 4 * i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      const float n = __hip_atomic_load(from + 4 * i + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      const float x = __hip_atomic_load(from + 4 * i + 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      const float t = __hip_atomic_load(from + 4 * i + 3, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      nan = nan || !(x < INFINITY);
      if (m == M) {
        left_out += n;
        others += x;
        moments += t;
      } else if (m > -INFINITY) {
        const float u = (m - M) * c, f = __builtin_amdgcn_exp2f(u);      // the slice's largest against the row's
        others = fmaf(n + x, f, others);
        moments += f * fmaf(n + x, fmaxf(u, -200.f), t);
      }
    }
    others = wave_sum(others);
    moments = wave_sum(moments);
    left_out = wave_sum(left_out);
    if (__ballot(nan)) others = NAN;
  }
  const bool undefined = !(others < INFINITY) || M == INFINITY;
  const bool nothing = M == -INFINITY && !undefined;
  const float log_sum = log1pf(left_out - 1.f + others);
  auto logp_of = [&](float x) __attribute__((always_inline)) {
    if (undefined) return NAN;
    return nothing || x == -INFINITY ? -INFINITY : (x - M) * a.scale - log_sum;
  };
  if (a.entropy && lane == 0) a.entropy[row_no] = undefined ? NAN : nothing ? 0.f : log_sum - kLn2 * moments / (left_out + others);
  for (int i = lane; i < a.n_given; i += 64) {
    const int id = a.given[row_no * a.n_given + i];
    float p = NAN;
    if (id < 0) p = 0.f;
    else if (id < a.n_vocab) p = logp_of(row.at(id));
    a.logp[row_no * a.n_given + i] = p;
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
  // candidates come 16 to a lane (eight 16-byte loads, coherent across the chip); up to 1024 are read once
  const int count = a.slices * kHolders;
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
      for (int i = 0; i < kAtOnce; ++i) held_by[i] = i0 + i * 64 + lane < kHolders ? bests[i0 + i * 64 + lane] : 0;
    }
  };
  u64 mine = 0;
  for (int i0 = 0; i0 < count; i0 += 64 * kAtOnce) {
    load_holders(i0);
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) mine = held_by[i] > mine ? held_by[i] : mine;
  }
  Largest holders(buf, lane, n, lane_value(sorted(mine, lane), n - 1));
  for (int i0 = 0; i0 < count; i0 += 64 * kAtOnce) {
    if (count > 64 * kAtOnce) load_holders(i0);
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) holders.offer(held_by[i]);
  }
  holders.done();
  const u64 nth = lane_value(holders.best, n - 1);
  Largest tokens(buf, lane, n, nth ? nth - 7 : 0);     // (its place is its group's first: the logit lies at most 7 further)
  for (int h0 = 0; h0 < n; h0 += 4) {          // 16 lanes to a holder, a group each
    const int h = h0 + lane / 16;
    const u64 holder = shuffle_from(holders.best, h & 63);
    const int group0 = place_of(holder) / 8;   // one of the holder's groups: its lane and its slice
    const int from_slice = group0 / per, in_slice = group0 - from_slice * per;
    const int group = from_slice * per + in_slice % kLanes / W * W + lane % 16 % W + lane % 16 / W * kLanes;
    const bool valid = h < n && holder != 0 && group < min((from_slice + 1) * per, (row.end + 7) / 8);
    float v[8];
    uint4 again[8 / L::kPer];
    if (valid) {
      row.load(group, again, false);
      row.values(group, again, v);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int place = group * 8 + e;
      tokens.offer(valid && place >= row.head && place < row.end ? candidate(v[e], place) : 0);
    }
  }
  tokens.done();
  if (lane < n) {
    ids[lane] = place_of(tokens.best) - row.head;
    if (tops) tops[lane] = logp_of(value_of(static_cast<uint32_t>(tokens.best >> 32)));
  }
}

template <typename L>
hipError_t launch_type(const LogprobsArgs& a, hipStream_t s) {
  const unsigned grid = static_cast<unsigned>(a.n_rows) * static_cast<unsigned>(a.slices);
  const int groups = (a.slice_len / kGroup + kLanes - 1) / kLanes;
  if (groups <= 1) logprobs_kernel<L, 1><<<grid, kLanes, 0, s>>>(a);
  else if (groups <= 2) logprobs_kernel<L, 2><<<grid, kLanes, 0, s>>>(a);
  else if (groups <= 4) logprobs_kernel<L, 4><<<grid, kLanes, 0, s>>>(a);
  else if (L::kBytes == 4 || groups <= 8) logprobs_kernel<L, 8><<<grid, kLanes, 0, s>>>(a);
  else if constexpr (L::kBytes == 2) logprobs_kernel<L, 16><<<grid, kLanes, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

LogprobsPlan plan_logprobs(int n_rows, int n_vocab, int n_top, int type) {
  LogprobsPlan p{};
  const long places = static_cast<long>(n_vocab) + 7;                   // a row may start inside a group
  const long most = kLanes * kGroup * (type == kLogitsF32 ? 8 : 16);
  long slices = (places + most - 1) / most;
  if (n_rows * slices < 512) {                                          // few rows: slices for all compute units
    const long fine = (places + kLanes * kGroup - 1) / (kLanes * kGroup), want = (512 + n_rows - 1) / n_rows;
    slices = want < fine ? want : fine;
  }
  p.slice_len = static_cast<int>(((places + slices - 1) / slices + kGroup - 1) / kGroup * kGroup);
  p.slices = static_cast<int>((places + p.slice_len - 1) / p.slice_len);
  if (p.slices > 1) {
    p.sums_bytes = static_cast<size_t>(p.slices) * 4 * sizeof(float);
    const int groups = (p.slice_len / kGroup + kLanes - 1) / kLanes;
    const int holders = groups <= 1 ? 16 : groups <= 2 ? 32 : groups <= 4 ? 64 : groups <= 8 ? 128 : 256;    // of a slice
    p.best_bytes = n_top > 0 ? static_cast<size_t>(p.slices) * holders * sizeof(u64) : 0;
  }
  return p;
}

hipError_t launch_logprobs(const LogprobsArgs& a, int type, hipStream_t s) {
  if (type == kLogitsF32) return launch_type<LF32>(a, s);
  return type == kLogitsBF16 ? launch_type<LBF16>(a, s) : launch_type<LF16>(a, s);
}

}  // namespace larosa
