// Key/value cache in 4 bits: new tokens into it (rotary positions, quantisation) and the attention over it.
//
// Format (the byte map is in the public header).  32 neighbouring values of a head share a power of two; a value is a 4-bit
// float (sign, 2 bits of exponent, 1 of mantissa) times it, which gfx950 turns into a pair of 16-bit values per instruction,
// scale included (v_cvt_scalef32_pk_*_fp4).  Both products of the attention then run on 16x16x32 matrix instructions with the
// TOKENS along the rows of K and along the contraction of V, and the bytes of a block lie in the order in which the lanes of a
// wave take them: a lane's operands are its own 16-byte loads (head_dim 128), nothing passes through LDS.
//   S^T [16 tokens, 16 rows] = K Q^T: lane (kq = lane / 16, m = lane mod 16) holds values [kq D/4, (kq+1) D/4) of token m, in
//     the order in which it holds the same values of query row m (a contraction may run in any order);
//   the result leaves tokens 4 kq .. 4 kq + 3 of row n = lane mod 16 in a lane, for two tiles of 16 tokens: 8 tokens, which
//     is what the second product wants of a lane as its B operand, so the weights stay where they are;
//   O^T [D, 16 rows] += V^T P^T: lane (kq, e) holds the same 8 tokens of values [e D/16, (e+1) D/16).
#include "kv4.hpp"
#include "numeric.hpp"

namespace larosa {

namespace {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bfloat8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bfloat2_t __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kBlockTokens = 32;
constexpr uint32_t kScaleNaN = 255;

// f(0), f(1), .. f(N - 1) with the number as a type: operands that have to be constants
template <int I> struct Number { static constexpr int value = I; };
template <int N, int I = 0, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(Number<I>{});
    static_for<N, I + 1>(f);
  }
}

__device__ __forceinline__ size_t block_bytes(int D) { return 34u * static_cast<size_t>(D); }

// ---- 16-bit types on the matrix cores -----------------------------------------------------------

template <typename T> struct Mat;
template <> struct Mat<F16> {
  static __device__ __forceinline__ floatx4 mfma(u32x4_t a, u32x4_t b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
  }
  template <int BYTE> static __device__ __forceinline__ uint32_t pair(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, BYTE));
  }
  static __device__ __forceinline__ uint32_t round2(float lo, float hi) {
    const half2_t v = {static_cast<_Float16>(lo), static_cast<_Float16>(hi)};
    return __builtin_bit_cast(uint32_t, v);
  }
};
template <> struct Mat<BF16> {
  static __device__ __forceinline__ floatx4 mfma(u32x4_t a, u32x4_t b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bfloat8_t, a), __builtin_bit_cast(bfloat8_t, b), c, 0, 0, 0);
  }
  template <int BYTE> static __device__ __forceinline__ uint32_t pair(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE));
  }
  static __device__ __forceinline__ uint32_t round2(float lo, float hi) {
    const bfloat2_t v = {static_cast<__bf16>(lo), static_cast<__bf16>(hi)};
    return __builtin_bit_cast(uint32_t, v);
  }
};

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// whether a byte of v is 255
__device__ __forceinline__ uint32_t any_nan_byte(uint32_t v) { return ((v & 0x7F7F7F7Fu) + 0x01010101u) & v & 0x80808080u; }

// lanes n, n + 16, n + 32, n + 48 together
__device__ __forceinline__ float over_quarters_max(float v) {
  auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
  x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
__device__ __forceinline__ float over_quarters_sum(float v) {
  auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(x[0]) + __uint_as_float(x[1]);
  x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(x[0]) + __uint_as_float(x[1]);
}

// ---- which rows, which tokens --------------------------------------------------------------------

struct Sequence {
  int slot, row0, n_new, len;
  bool real;                  // the slot exists
};

// Sequence s of a batch; n_new is cut to what the batch allows.
__device__ __forceinline__ Sequence sequence(const larosa_kv4_cache& C, const larosa_kv4_batch& b, int s) {
  Sequence q;
  q.row0 = b.starts ? b.starts[s] : s;
  q.n_new = b.starts ? b.starts[s + 1] - q.row0 : 1;
  q.slot = b.slots[s];
  q.real = q.slot >= 0 && q.slot < C.n_slots;
  q.len = q.real ? C.length[q.slot] : 0;
  return q;
}

// Page of token t of a slot, or -1.
__device__ __forceinline__ int page_of(const larosa_kv4_cache& C, int slot, int page_index) {
  if (page_index < 0 || page_index >= C.max_pages) return -1;
  const int p = C.table[static_cast<size_t>(slot) * C.max_pages + page_index];
  return p >= 0 && p < C.n_pages ? p : -1;
}

__device__ __forceinline__ size_t block_at(const larosa_kv4_cache& C, int layer, int page, int head, int block_in_page, int D) {
  const int per_page = C.page_tokens / kBlockTokens;
  return (((static_cast<size_t>(layer) * C.n_pages + page) * C.n_kv_heads + head) * per_page + block_in_page) * block_bytes(D);
}

// ---- append -----------------------------------------------------------------------------------------

// One lane takes 8 neighbouring values of a head, so four neighbouring lanes a group of 32 with one scale.  Bound by the bytes of
// the rows in and out (prompts) or by latency (a decode step).  The partners of a rotation are loaded a second time from the
// cache line's neighbours rather than exchanged between lanes.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv4_append_kernel(Kv4AppendArgs a) {
  constexpr int LP = D / 8;                                   // lanes of a head
  const int s = blockIdx.y;
  const int item = (blockIdx.x * 256 + threadIdx.x) / LP;
  const int c = threadIdx.x % LP;                             // values [8 c, 8 c + 8)
  const int H = a.C.n_kv_heads, heads = a.n_heads + 2 * H;
  const int j = item / heads, head = item - j * heads;
  const Sequence q = sequence(a.C, a.b, s);
  const int row = q.row0 + j;
  if (!q.real || j >= q.n_new || j >= a.b.max_new || row < 0 || row >= a.b.n_rows) return;
  const int place = q.len - q.n_new + j;

  const uint16_t* x = a.qkv + static_cast<size_t>(row) * a.ld_qkv + static_cast<size_t>(head) * D;
  float v[8];
  unpack8<T>(*reinterpret_cast<const uint4*>(x + 8 * c), v);
  const int half = a.r.rot_dim / 2;
  if (a.r.table && head < a.n_heads + H && 8 * c < a.r.rot_dim) {
    // products and sums rounded one by one, so that k is quantised from values that any fp32 program gets
#pragma clang fp contract(off)
    float w[8];                                               // the partners
    const bool upper = !a.r.interleaved && 8 * c >= half;
    if (!a.r.interleaved) unpack8<T>(*reinterpret_cast<const uint4*>(x + 8 * c + (upper ? -half : half)), w);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int f = a.r.interleaved ? 4 * c + i / 2 : 8 * c + i - (upper ? half : 0);
      int p = place;
      if (a.r.positions) {
        int axis = 0;
        for (int end = a.r.axis_pairs[0]; axis + 1 < a.r.n_axes && f >= end; end += a.r.axis_pairs[axis]) ++axis;
        p = a.r.positions[static_cast<size_t>(axis) * a.b.n_rows + row];
      }
      float cs = __uint_as_float(0x7FC00000u), sn = cs;
      if (p >= 0 && p < a.r.n_positions) {
        const float* t = a.r.table + static_cast<size_t>(p) * a.r.rot_dim + f;
        cs = t[0];
        sn = t[half];
      }
      const float other = a.r.interleaved ? v[i ^ 1] : w[i];
      const bool second = a.r.interleaved ? (i & 1) : upper;
      const float p0 = v[i] * cs, p1 = other * sn;
      y[i] = second ? p0 + p1 : p0 - p1;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = y[i];
  }

  if (head >= a.n_heads) {
    // the group's largest magnitude as an integer, so that a NaN is the largest
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
    // exponent of the largest less 2, one more where its mantissa exceeds 1.75: nothing is then further off than half a step
    constexpr bool kBf = sizeof(T) && __is_same(T, BF16);
    int e = static_cast<int>((top + 0x1FFFFFu) >> 23) - 127 - 2;
    e = min(max(e, kBf ? -100 : -23), kBf ? 125 : 13);
    const bool whole = top < 0x7F800000u;
    const float unit = __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
    const uint32_t scale = whole ? static_cast<uint32_t>(e + 127) : kScaleNaN;
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // the borders between neighbouring codes are exact multiples of the unit
      const float m = fabsf(v[i]);
      uint32_t code = 0;
      if (whole)
        code = (m > 0.25f * unit) + (m >= 0.75f * unit) + (m > 1.25f * unit) + (m >= 1.75f * unit) + (m > 2.5f * unit) +
               (m >= 3.5f * unit) + (m > 5.0f * unit);
      // 0, 1/2, 1, 3/2, 2, 3, 4, 6
      const float level = code < 4 ? 0.5f * code : (code == 4 ? 2.f : code == 5 ? 3.f : code == 6 ? 4.f : 6.f);
      const uint32_t sign = __float_as_uint(v[i]) >> 31;
      codes |= (code | sign << 3) << (4 * i);
      v[i] = whole ? (sign ? -level : level) * unit : __uint_as_float(0x7FC00000u);
    }
    const int page = place >= 0 ? page_of(a.C, q.slot, place / a.C.page_tokens) : -1;
    if (page >= 0) {
      constexpr int LB = D / 8, W = LB < 16 ? LB : 16;        // a lane's bytes of a tile, and those of one load
      const int t = place % kBlockTokens, u = t / 16, m = t % 16;
      const bool is_v = head >= a.n_heads + H;
      const int kv = head - a.n_heads - (is_v ? H : 0);
      uint8_t* block = static_cast<uint8_t*>(a.C.data) +
                       block_at(a.C, a.layer, page, kv, place % a.C.page_tokens / kBlockTokens, D);
      auto at = [&](int lane, int byte) { return u * 8 * D + byte / W * 64 * W + lane * W + byte % W; };
      const int g = c / 4;
      if (!is_v) {
        const int i0 = 8 * c;
        *reinterpret_cast<uint32_t*>(block + at(i0 / (D / 4) * 16 + m, i0 % (D / 4) / 2)) = codes;
        if (c % 4 == 0) block[32 * D + u * (D / 2) + 16 * g + m] = static_cast<uint8_t>(scale);
      } else {
        constexpr int PV = D / 16;                            // values of a lane
        const int kq = m / 4, i = m % 4, i0 = 8 * c;
        uint8_t* vb = block + 16 * D;
        if constexpr (PV >= 8) {
          *reinterpret_cast<uint32_t*>(vb + at(kq * 16 + i0 / PV, i * (D / 32) + i0 % PV / 2)) = codes;
        } else {
          *reinterpret_cast<uint16_t*>(vb + at(kq * 16 + i0 / PV, i * (D / 32))) = static_cast<uint16_t>(codes);
          *reinterpret_cast<uint16_t*>(vb + at(kq * 16 + i0 / PV + 1, i * (D / 32))) = static_cast<uint16_t>(codes >> 16);
        }
        if (c % 4 == 0) block[33 * D + u * (D / 2) + (kq * (D / 32) + g) * 4 + i] = static_cast<uint8_t>(scale);
      }
    }
  }
  if (a.out) *reinterpret_cast<uint4*>(a.out + static_cast<size_t>(row) * a.ld_out + static_cast<size_t>(head) * D + 8 * c) = pack8<T>(v);
}

// ---- attention ----------------------------------------------------------------------------------------

// One workgroup: 16 rows (new token, query head of the group) of one key/value head of one sequence; its four waves take every
// fourth block of 32 tokens each and join at the end.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv4_attention_kernel(Kv4AttentionArgs a) {
  constexpr int DW = D / 32;                                  // dwords of a lane's codes in a tile of 16 tokens
  constexpr int NG = D / 32;                                  // scale groups of a head
  constexpr int LW = DW < 4 ? DW : 4;                         // dwords of one load
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = lane & 15, kq = lane >> 4;
  const int head = blockIdx.x % a.C.n_kv_heads;
  const int tile = blockIdx.x / a.C.n_kv_heads;
  const int s = blockIdx.y;
  Sequence sq = sequence(a.C, a.b, s);
  const int news = min(sq.n_new, a.b.max_new);
  if (tile * 16 >= news * a.group) return;
  // this lane's row
  const int r = tile * 16 + n;
  const int j = r / a.group, hq = head * a.group + r % a.group;
  const int row = sq.row0 + j;
  const bool has_row = j < news && row >= 0 && row < a.b.n_rows;
  const int base = sq.len - sq.n_new;                         // place of the sequence's first new token
  const int first_j = tile * 16 / a.group, last_j = min(news - 1, (tile * 16 + 15) / a.group);
  const int seen_to = base + j + 1, seen_from = a.window > 0 ? max(0, seen_to - a.window) : 0;
  const int hi = max(0, min(sq.len, base + last_j + 1));
  const int lo = a.window > 0 ? max(0, base + first_j + 1 - a.window) : 0;
  // every row of the tile sees the tokens in [all_from, all_to)
  const int all_to = base + first_j + 1, all_from = a.window > 0 ? base + last_j + 1 - a.window : 0;

  u32x4_t qf[DW];
#pragma unroll
  for (int k = 0; k < DW; ++k) {
    qf[k] = u32x4_t{0, 0, 0, 0};
    if (has_row)
      qf[k] = *reinterpret_cast<const u32x4_t*>(a.q + static_cast<size_t>(row) * a.ld_q + static_cast<size_t>(hq) * D + kq * (D / 4) + 8 * k);
  }
  floatx4 o[D / 16];
#pragma unroll
  for (int k = 0; k < D / 16; ++k) o[k] = floatx4{0, 0, 0, 0};
  float top = -INFINITY, total = 0.f;

  const int per_page = a.C.page_tokens / kBlockTokens;
  for (int b = lo / kBlockTokens + wave; b * kBlockTokens < hi; b += 4) {
    const int page = page_of(a.C, sq.slot, b / per_page);
    if (page < 0) continue;
    const uint8_t* block = static_cast<const uint8_t*>(a.C.data) + block_at(a.C, a.layer, page, head, b % per_page, D);
    uint32_t kc[2][DW], vc[2][DW], kb[2][2], vs[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int k = 0; k < DW; ++k) {
        kc[u][k] = *reinterpret_cast<const uint32_t*>(block + u * 8 * D + k / LW * 64 * LW * 4 + lane * LW * 4 + k % LW * 4);
        vc[u][k] = *reinterpret_cast<const uint32_t*>(block + 16 * D + u * 8 * D + k / LW * 64 * LW * 4 + lane * LW * 4 + k % LW * 4);
      }
#pragma unroll
      for (int h = 0; h < (D > 128 ? 2 : 1); ++h) kb[u][h] = block[32 * D + u * (D / 2) + 16 * (kq * NG / 4 + h) + n];
      vs[u] = *reinterpret_cast<const uint32_t*>(block + 33 * D + u * (D / 2) + (kq * NG + n * NG / 16) * 4);
    }
    const int t0 = b * kBlockTokens;
    const bool cut = t0 < all_from || t0 + kBlockTokens > all_to;      // some row does not see some token
    uint32_t odd = any_nan_byte(vs[0]) | any_nan_byte(vs[1]) | (kb[0][0] == kScaleNaN) | (kb[1][0] == kScaleNaN);
    if constexpr (D > 128) odd |= (kb[0][1] == kScaleNaN) | (kb[1][1] == kScaleNaN);
    const bool nan_groups = __any(odd != 0);

    float p[8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      floatx4 sc = {0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < DW; ++k) {
        const float f = scale_of(kb[u][k / 4]);
        const u32x4_t kv = {Mat<T>::template pair<0>(kc[u][k], f), Mat<T>::template pair<1>(kc[u][k], f),
                            Mat<T>::template pair<2>(kc[u][k], f), Mat<T>::template pair<3>(kc[u][k], f)};
        sc = Mat<T>::mfma(kv, qf[k], sc);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) p[4 * u + i] = sc[i] * a.scale_log2;
    }
    uint64_t nan_v = 0;                                       // of this lane's row: groups with a NaN value that the row sees
    if (nan_groups || cut) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int t = t0 + 16 * (i / 4) + 4 * kq + i % 4;
        if (nan_groups)
          for (int g = 0; g < NG; ++g)
            if (block[32 * D + i / 4 * (D / 2) + 16 * g + 4 * kq + i % 4] == kScaleNaN) p[i] = __uint_as_float(0x7FC00000u);
        if (t < seen_from || t >= seen_to) p[i] = -INFINITY;
        // what no row of the tile sees may hold anything: its values count as zeros
        if (t < lo || t >= hi) vs[i / 4] &= ~(0xFFu << (8 * (i % 4)));
      }
      if (nan_groups) {
        for (int t = 0; t < kBlockTokens; ++t)
          for (int g = 0; g < NG; ++g) {
            const uint8_t sb = block[33 * D + t / 16 * (D / 2) + (t % 16 / 4 * NG + g) * 4 + t % 4];
            if (sb == kScaleNaN && t0 + t >= seen_from && t0 + t < seen_to) nan_v |= 1ull << g;
          }
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if ((vs[i / 4] >> (8 * (i % 4)) & 0xFFu) == kScaleNaN) vs[i / 4] &= ~(0xFFu << (8 * (i % 4)));
      }
    }
    float m = p[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) m = fmaxf(m, p[i]);
    const float now = fmaxf(top, over_quarters_max(m));
    const float ref = now == -INFINITY ? 0.f : now;
    const float back = __builtin_amdgcn_exp2f(top - ref);     // nothing seen so far: 2^-inf = 0
    top = now;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(p[i] - ref);
      sum += p[i];
    }
    total = total * back + sum;
    // weights to 16 bits: half a step of 2^-8 (bf16) or 2^-11 (f16) relative on each, independent over the tokens
    const u32x4_t pf = {Mat<T>::round2(p[0], p[1]), Mat<T>::round2(p[2], p[3]), Mat<T>::round2(p[4], p[5]), Mat<T>::round2(p[6], p[7])};
    float vf[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) vf[i] = scale_of(vs[i / 4] >> (8 * (i % 4)) & 0xFFu);
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[k][i] *= back;
    static_for<D / 32>([&](auto jb) {                         // two values of the lane's eight tokens
      constexpr int J = decltype(jb)::value;
      uint32_t x[8];
      static_for<8>([&](auto ii) {
        constexpr int I = decltype(ii)::value, B = I % 4 * (D / 32) + J;
        x[I] = Mat<T>::template pair<B % 4>(vc[I / 4][B / 4], vf[I]);
      });
      u32x4_t even, odd2;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        even[h] = __builtin_amdgcn_perm(x[2 * h + 1], x[2 * h], 0x05040100u);
        odd2[h] = __builtin_amdgcn_perm(x[2 * h + 1], x[2 * h], 0x07060302u);
      }
      o[2 * J] = Mat<T>::mfma(even, pf, o[2 * J]);
      o[2 * J + 1] = Mat<T>::mfma(odd2, pf, o[2 * J + 1]);
    });
    if (nan_v) {
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (nan_v >> (((4 * kq + i) * (D / 16) + k) / 32) & 1) o[k][i] = __uint_as_float(0x7FC00000u);
    }
  }
  total = over_quarters_sum(total);

  // join the four waves: a lane's values [kq D/4, (kq+1) D/4) of row n
  __shared__ float s_top[4][16], s_total[4][16];
  __shared__ float s_o[3][64][D / 4 + 1];
  if (kq == 0) {
    s_top[wave][n] = top;
    s_total[wave][n] = total;
  }
  if (wave > 0) {
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) s_o[wave - 1][lane][i * (D / 16) + k] = o[k][i];
  }
  __syncthreads();
  if (wave > 0 || !has_row) return;
  float best = s_top[0][n];
  for (int w = 1; w < 4; ++w) best = fmaxf(best, s_top[w][n]);
  const float ref = best == -INFINITY ? 0.f : best;
  float f[4], sum = 0.f;
  for (int w = 0; w < 4; ++w) {
    f[w] = __builtin_amdgcn_exp2f(s_top[w][n] - ref);
    sum += s_total[w][n] * f[w];
  }
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  uint16_t* dst = a.out + static_cast<size_t>(row) * a.ld_out + static_cast<size_t>(hq) * D + kq * (D / 4);
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int d = 8 * c + e, i = d / (D / 16), k = d % (D / 16);
      float x = o[k][i] * f[0];
      for (int w = 1; w < 4; ++w) x += s_o[w - 1][lane][d] * f[w];
      v[e] = x * inv;
    }
    *reinterpret_cast<uint4*>(dst + 8 * c) = pack8<T>(v);
  }
}

template <typename F>
hipError_t by_type(const larosa_kv4_cache& C, F&& f) {
  const bool bf = C.dtype == LAROSA_BF16;
  switch (C.head_dim) {
    case 64: return bf ? f.template operator()<BF16, 64>() : f.template operator()<F16, 64>();
    case 128: return bf ? f.template operator()<BF16, 128>() : f.template operator()<F16, 128>();
    default: return bf ? f.template operator()<BF16, 256>() : f.template operator()<F16, 256>();
  }
}

struct AppendLaunch {
  const Kv4AppendArgs& a;
  hipStream_t s;
  template <typename T, int D> hipError_t operator()() const {
    const long lanes = static_cast<long>(a.b.max_new) * (a.n_heads + 2 * a.C.n_kv_heads) * (D / 8);
    const dim3 grid(static_cast<unsigned>((lanes + 255) / 256), static_cast<unsigned>(a.b.n_seq));
    hipLaunchKernelGGL((kv4_append_kernel<T, D>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
  }
};

struct AttentionLaunch {
  const Kv4AttentionArgs& a;
  hipStream_t s;
  template <typename T, int D> hipError_t operator()() const {
    const dim3 grid(static_cast<unsigned>(a.row_tiles * a.C.n_kv_heads), static_cast<unsigned>(a.b.n_seq));
    hipLaunchKernelGGL((kv4_attention_kernel<T, D>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
  }
};

}  // namespace

hipError_t launch_kv4_append(const Kv4AppendArgs& a, hipStream_t s) { return by_type(a.C, AppendLaunch{a, s}); }
hipError_t launch_kv4_attention(const Kv4AttentionArgs& a, hipStream_t s) { return by_type(a.C, AttentionLaunch{a, s}); }

}  // namespace larosa
