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
constexpr int kNowhere = 1 << 30;     // past every token

// f(0), f(1), .. f(N - 1) with the number as a type: operands that have to be constants
template <int I> struct Number { static constexpr int value = I; };
template <int N, int I = 0, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(Number<I>{});
    static_for<N, I + 1>(f);
  }
}

// ---- 16-bit types on the matrix cores -----------------------------------------------------------

template <typename T> struct Mat;
template <> struct Mat<F16> {
  static __device__ __forceinline__ floatx4 mfma(u32x4_t a, u32x4_t b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
  }
  // both of a pair to a sum, subnormals too; within 3 2^-24 of it, 2^-26 too small on average (a million random ones)
  static __device__ __forceinline__ float add2(uint32_t pair, float sum) {
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(half2_t, pair), half2_t{1, 1}, sum, false);
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
  static __device__ __forceinline__ float add2(uint32_t pair, float sum) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bfloat2_t, pair), bfloat2_t{1, 1}, sum, false);
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

// Sequence s of a batch (Args: of either kernel), its length left out: a load that waits for the slot's.
template <typename Args>
__device__ __forceinline__ Sequence sequence_rows(const Args& a, int s) {
  Sequence q;
  q.row0 = a.starts ? a.starts[s] : s;
  q.n_new = a.starts ? a.starts[s + 1] - q.row0 : 1;
  q.slot = a.slots[s];
  q.real = q.slot >= 0 && q.slot < static_cast<int>(a.n_slots);
  q.len = 0;
  return q;
}
template <typename Args>
__device__ __forceinline__ Sequence sequence(const Args& a, int s) {
  Sequence q = sequence_rows(a, s);
  if (q.real) q.len = a.length[q.slot];
  return q;
}

// ---- append -----------------------------------------------------------------------------------------

// Cosines and sines for the eight values [8 c, 8 c + 8) of a head at a row's positions.
template <int D>
__device__ __forceinline__ void turn_of(const Kv4AppendArgs& a, int c, int row, int place, float (&cs)[8], float (&sn)[8]) {
  const Kv4AppendArgs& r = a;
  const int half = r.rot_dim / 2;
  const int f0 = r.interleaved ? 4 * c : (8 * c >= half ? 8 * c - half : 8 * c), nf = r.interleaved ? 4 : 8;
  auto axis_of = [&](int f) {
    int axis = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i) axis += f >= static_cast<int>(r.axis_ends >> 8 * i & 255);
    return axis;
  };
  const int axis = r.n_axes > 1 ? axis_of(f0) : 0;
  const bool one = r.n_axes == 1 || axis_of(f0 + nf - 1) == axis;
  auto position = [&](int ax) { return r.positions ? r.positions[static_cast<size_t>(ax) * a.n_rows + row] : place; };
#pragma unroll
  for (int i = 0; i < 8; ++i) cs[i] = sn[i] = __uint_as_float(0x7FC00000u);       // outside the table
  if (one) {
    const int p = position(axis);
    if (p < 0 || p >= r.n_positions) return;
    const float4* t = reinterpret_cast<const float4*>(r.turns + static_cast<size_t>(p) * r.rot_dim + f0);
    const float4* u = reinterpret_cast<const float4*>(r.turns + static_cast<size_t>(p) * r.rot_dim + half + f0);
    const float4 c0 = t[0], s0 = u[0];
    if (r.interleaved) {
      cs[0] = cs[1] = c0.x; cs[2] = cs[3] = c0.y; cs[4] = cs[5] = c0.z; cs[6] = cs[7] = c0.w;
      sn[0] = sn[1] = s0.x; sn[2] = sn[3] = s0.y; sn[4] = sn[5] = s0.z; sn[6] = sn[7] = s0.w;
    } else {
      const float4 c1 = t[1], s1 = u[1];
      cs[0] = c0.x; cs[1] = c0.y; cs[2] = c0.z; cs[3] = c0.w; cs[4] = c1.x; cs[5] = c1.y; cs[6] = c1.z; cs[7] = c1.w;
      sn[0] = s0.x; sn[1] = s0.y; sn[2] = s0.z; sn[3] = s0.w; sn[4] = s1.x; sn[5] = s1.y; sn[6] = s1.z; sn[7] = s1.w;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {                               // the axis changes among the eight
    const int f = f0 + (r.interleaved ? i / 2 : i);
    const int p = position(axis_of(f));
    if (p < 0 || p >= r.n_positions) continue;
    cs[i] = r.turns[static_cast<size_t>(p) * r.rot_dim + f];
    sn[i] = r.turns[static_cast<size_t>(p) * r.rot_dim + half + f];
  }
}

// y = v turned; w: the partners (the other half's values), or v itself where they are neighbours.  Products and sums are rounded one by
// one, so that k is quantised from values that any fp32 program gets.
__device__ __forceinline__ void turn(const Kv4AppendArgs& r, int c, const float (&cs)[8], const float (&sn)[8], const float (&w)[8],
                                     float (&v)[8]) {
#pragma clang fp contract(off)
  const bool upper = 8 * c >= static_cast<int>(r.rot_dim / 2);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float other = r.interleaved ? v[i ^ 1] : w[i];
    const bool second = r.interleaved ? (i & 1) != 0 : upper;
    const float p0 = v[i] * cs[i], p1 = other * sn[i];
    y[i] = second ? p0 + p1 : p0 - p1;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = y[i];
}

__device__ __forceinline__ uint32_t largest_of_four(uint32_t v) {
  const int i = static_cast<int>(v);
  v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(i, i, 0xB1, 0xF, 0xF, false)));      // quad_perm 1, 0, 3, 2
  const int k = static_cast<int>(v);
  return max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(k, k, 0x4E, 0xF, 0xF, false)));   // quad_perm 2, 3, 0, 1
}

// Eight values to codes (value i in nibble i); scale: the byte that the four lanes of a group share.
template <typename T>
__device__ __forceinline__ uint32_t quantise8(const float (&v)[8], uint32_t& scale) {
  // the group's largest magnitude as an integer, so that a NaN is the largest
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  top = largest_of_four(top);
  if (top >= 0x7F800000u) {
    scale = kScaleNaN;
    uint32_t signs = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) signs |= (__float_as_uint(v[i]) >> 31) << (4 * i + 3);
    return signs;
  }
  // exponent of the largest less 2, one more where its mantissa exceeds 1.75: nothing is then further off than half a step
  constexpr bool kBf = __is_same(T, BF16);
  int e = static_cast<int>((top + 0x1FFFFFu) >> 23) - 127 - 2;
  e = min(max(e, kBf ? -100 : -23), kBf ? 125 : 13);
  scale = static_cast<uint32_t>(e + 127);
  // a division by a power of two and a rounding to the nearest code, ties to the even one, more than 6 to 6: one instruction a pair
  const float unit = scale_of(scale);
  uint32_t codes = 0;
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[0], v[1], unit, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[2], v[3], unit, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[4], v[5], unit, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[6], v[7], unit, 3);
}

// A lane takes 8 neighbouring values of HPL heads of a token, four neighbouring lanes a group of 32 with one scale; the cosines and
// sines of its frequencies serve all its heads.  A workgroup takes TW tokens that share a tile of 16 places, so that a tile's
// bytes are written from one place, or one token (TW = 1).  Bound by the rows in and out (prompts) or by latency (a decode step).
template <typename T, int D, int TW, int HPL>
__global__ __launch_bounds__(256) void kv4_append_kernel(Kv4AppendArgs a) {
  constexpr int LP = D / 8;                                   // lanes of a head
  constexpr int HS = 256 / LP / TW;                           // heads at a time
  const int c = threadIdx.x % LP;                             // values [8 c, 8 c + 8)
  const int hs = threadIdx.x / LP % HS, tok = threadIdx.x / LP / HS;
  const int H = a.n_kv_heads, n_heads = a.n_heads, heads = n_heads + 2 * H;
  const Sequence q = sequence(a, blockIdx.y);
  const int base = q.len - q.n_new;
  // j: the token among the sequence's new ones
  const int j = TW == 1 ? static_cast<int>(blockIdx.z) : static_cast<int>(blockIdx.z) * TW + tok - (base & (TW - 1));
  const int row = q.row0 + j;
  if (!q.real || j < 0 || j >= q.n_new || j >= static_cast<int>(a.max_new) || row < 0 || row >= a.n_rows) return;
  const int place = base + j;

  const uint16_t* x = a.qkv + static_cast<size_t>(row) * a.ld_qkv;
  const int half = a.rot_dim / 2;
  const bool turned = a.turns && 8 * c < static_cast<int>(a.rot_dim);
  const int partner = a.interleaved ? 0 : (8 * c >= half ? -half : half);
  uint4 raw[HPL], other[HPL];
#pragma unroll
  for (int k = 0; k < HPL; ++k) {
    const int head = (blockIdx.x * HPL + k) * HS + hs;
    if (head < heads) raw[k] = *reinterpret_cast<const uint4*>(x + static_cast<size_t>(head) * D + 8 * c);
    if (turned && !a.interleaved && head < n_heads + H)
      other[k] = *reinterpret_cast<const uint4*>(x + static_cast<size_t>(head) * D + 8 * c + partner);
  }
  float cs[8], sn[8];
  if (turned) turn_of<D>(a, c, row, place, cs, sn);
  const int page_index = place >> a.page_shift;               // (of no use for a place below zero)
  int page = place >= 0 && page_index < a.max_pages ? a.table[static_cast<size_t>(q.slot) * a.max_pages + page_index] : -1;
  if (page >= a.n_pages) page = -1;
  const unsigned part = (34u * D / kBlockTokens) << a.page_shift;       // bytes of a head's part of a page
#pragma unroll
  for (int k = 0; k < HPL; ++k) {
    const int head = (blockIdx.x * HPL + k) * HS + hs;
    if (head >= heads) break;
    float v[8], w[8];
    unpack8<T>(raw[k], v);
    if (turned && head < n_heads + H) {
      if (!a.interleaved) unpack8<T>(other[k], w);
      turn(a, c, cs, sn, w, v);
    }
    uint4 result;
    if (head < n_heads) {
      result = uint4{Mat<T>::round2(v[0], v[1]), Mat<T>::round2(v[2], v[3]), Mat<T>::round2(v[4], v[5]), Mat<T>::round2(v[6], v[7])};
    } else {
      uint32_t scale;
      const uint32_t codes = quantise8<T>(v, scale);
      // what the codes stand for is exact in 16 bits
      const float unit = scale_of(scale);
      result = uint4{Mat<T>::template pair<0>(codes, unit), Mat<T>::template pair<1>(codes, unit), Mat<T>::template pair<2>(codes, unit),
                     Mat<T>::template pair<3>(codes, unit)};
      if (scale == kScaleNaN) {
        const uint32_t nan2 = Mat<T>::round2(__uint_as_float(0x7FC00000u), __uint_as_float(0x7FC00000u));
        result = uint4{nan2, nan2, nan2, nan2};
      }
      if (page >= 0) {
        constexpr int LB = D / 8, W = LB < 16 ? LB : 16;      // a lane's bytes of a tile in the attention, and those of one load
        const int t = place % kBlockTokens, u = t / 16, m = t % 16;
        const bool is_v = head >= n_heads + H;
        const int kv = head - n_heads - (is_v ? H : 0);
        uint8_t* block = a.data + (static_cast<size_t>(page) * H + kv) * part +
                         ((place & ((1 << a.page_shift) - 1)) / kBlockTokens) * (34 * D);
        auto at = [&](int lane, int byte) { return u * 8 * D + byte / W * 64 * W + lane * W + byte % W; };
        const int g = c / 4;
        if (!is_v) {
          const int i0 = 8 * c;
          *reinterpret_cast<uint32_t*>(block + at(i0 / (D / 4) * 16 + m, i0 % (D / 4) / 2)) = codes;
          if (c % 4 == 0) block[32 * D + u * (D / 2) + 16 * g + m] = static_cast<uint8_t>(scale);
        } else {
          constexpr int PV = D / 16;                          // values of a lane
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
    if (a.out) *reinterpret_cast<uint4*>(a.out + static_cast<size_t>(row) * a.ld_out + static_cast<size_t>(head) * D + 8 * c) = result;
  }
}

// ---- attention ----------------------------------------------------------------------------------------

// What a wave holds of one block of 32 tokens.
template <int D> struct Block {
  static constexpr int DW = D / 32;                           // dwords of a lane's codes in a tile of 16 tokens
  static constexpr int KG = D > 128 ? 2 : 1;                  // scale groups of a lane's part of a key
  uint32_t kc[2][DW], vc[2][DW];
  uint32_t kb[2][KG], vs[2];                                  // scale bytes: of the lane's token; of its four tokens
};

// A block's bytes as a buffer.  Where there is none (present false) its size is zero: loads are issued all the same and come back
// with zeros from no memory, so that the compiler, which counts loads under way, never has to wait for younger ones than it needs.
template <int D>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t block_buffer(const uint8_t* block, bool present) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(block), 0, present ? 34 * D : 0, 0x00027000);
}

// The wave's codes of one block: 16 tokens' keys or values in runs of 64 pieces, one of each lane.  ONCE: no other workgroup
// reads them, so they pass the caches by (64 sequences of up to 16384 tokens: 87.7 -> 79.5 us, 4.7 TB/s).
template <int D, bool ONCE>
__device__ __forceinline__ void load_codes(uint32_t (&c)[2][D / 32], __amdgpu_buffer_rsrc_t block, int at, int lane) {
  constexpr int LW = D < 128 ? D / 32 : 4, kPolicy = ONCE ? 2 : 0;     // 2: nt
  static_assert(LW == 2 || LW == 4, "8 or 16 bytes to a load");
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int p = 0; p < D / 32 / LW; ++p) {
      const int offset = at + u * 8 * D + p * 64 * LW * 4;
      if constexpr (LW == 4) {
        const u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(block, lane * 16, offset, kPolicy);
#pragma unroll
        for (int i = 0; i < 4; ++i) c[u][4 * p + i] = v[i];
      } else {
        typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
        const u32x2_t v = __builtin_amdgcn_raw_buffer_load_b64(block, lane * 8, offset, kPolicy);
        c[u][0] = v[0];
        c[u][1] = v[1];
      }
    }
}
template <int D, bool ONCE>
__device__ __forceinline__ void load_keys(Block<D>& x, __amdgpu_buffer_rsrc_t block, int lane) {
  load_codes<D, ONCE>(x.kc, block, 0, lane);
  const int mine = (lane >> 4) * (D / 32) / 4 * 16 + (lane & 15);
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int h = 0; h < Block<D>::KG; ++h)
      x.kb[u][h] = static_cast<uint8_t>(__builtin_amdgcn_raw_buffer_load_b8(block, mine, 32 * D + u * (D / 2) + 16 * h, 0));
}
template <int D, bool ONCE>
__device__ __forceinline__ void load_values(Block<D>& x, __amdgpu_buffer_rsrc_t block, int lane) {
  load_codes<D, ONCE>(x.vc, block, 16 * D, lane);
  const int mine = ((lane >> 4) * (D / 32) + (lane & 15) * (D / 32) / 16) * 4;
#pragma unroll
  for (int u = 0; u < 2; ++u) x.vs[u] = __builtin_amdgcn_raw_buffer_load_b32(block, mine, 33 * D + u * (D / 2), 0);
}

// What the rows of a tile see together.
struct Seen {
  int lo, hi;                 // no row of the tile sees a token outside
  int all_from, all_to;       // every row of the tile sees all in between
};

// A row's weights are powers of two of its logits less a reference, which need not be the maximum: it is set kLift below the largest
// logit so far, and anew only when a logit exceeds it by more than kTop, which spares most blocks the exchange between lanes and
// the rescaling of the accumulators (8 apart: a prompt of 4096 tokens takes 2 % longer with 4, 7 % with 2).  bf16 has the range of
// fp32.  f16 reaches from 2^16 to 2^-14 with all its bits, so its weights are lifted to the upper end: the largest logit's is between 2^7 and
// 2^15, and one that is 2^21 times smaller still keeps 11 bits (many small ones are all that counts where a key stands out whose own
// value is small).  A lift of less than 8 is at most rounded to 8, however large the logits, so 2^kTop is never exceeded.
template <typename T> constexpr float kLift = __is_same(T, F16) ? 7.f : 0.f;
template <typename T> constexpr float kTop = kLift<T> + 8.f;

// One of a lane's rows: lane mod 16 of 16 rows, values [kq D/4, (kq + 1) D/4) of its query and of its output, the latter in
// o[k][i] = value i D/16 + k.
template <int D> struct Row {
  u32x4_t q[D / 32];
  int from, to;               // the row sees tokens [from, to)
  floatx4 o[D / 16];
  float ref, total;           // total: of the lane's own tokens
};

// One block of tokens t0 .. t0 + 31, in x, for NT times 16 rows: the codes are converted once for all of them.  As soon as x's
// keys are used up those of the block `next` are on their way into the same registers, and so are the values.
template <typename T, int D, int NT, bool ONCE>
__device__ __forceinline__ void attend_block(Block<D>& x, const uint8_t* block, __amdgpu_buffer_rsrc_t next, int t0, const Seen& see,
                                             float scale_log2, int lane, Row<D> (&rows)[NT]) {
  constexpr int DW = D / 32, NG = D / 32;
  const int kq = lane >> 4;
  const bool cut = t0 < see.all_from || t0 + kBlockTokens > see.all_to;       // some row does not see some token
  uint32_t odd = any_nan_byte(x.vs[0]) | any_nan_byte(x.vs[1]);
#pragma unroll
  for (int h = 0; h < Block<D>::KG; ++h) odd |= (x.kb[0][h] == kScaleNaN) | (x.kb[1][h] == kScaleNaN);
  const bool nan_groups = __any(odd != 0);

  float p[NT][8];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    floatx4 sc[NT];
#pragma unroll
    for (int z = 0; z < NT; ++z) sc[z] = floatx4{0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < DW; ++k) {
      const float f = scale_of(x.kb[u][k / 4]);
      const u32x4_t kv = {Mat<T>::template pair<0>(x.kc[u][k], f), Mat<T>::template pair<1>(x.kc[u][k], f),
                          Mat<T>::template pair<2>(x.kc[u][k], f), Mat<T>::template pair<3>(x.kc[u][k], f)};
#pragma unroll
      for (int z = 0; z < NT; ++z) sc[z] = Mat<T>::mfma(kv, rows[z].q[k], sc[z]);
    }
#pragma unroll
    for (int z = 0; z < NT; ++z)
#pragma unroll
      for (int i = 0; i < 4; ++i) p[z][4 * u + i] = sc[z][i] * scale_log2;
  }
  load_keys<D, ONCE>(x, next, lane);
  uint32_t nan_v[NT] = {};                                    // groups with a NaN value that the lane's row sees
  if (nan_groups || cut) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int t = t0 + 16 * (i / 4) + 4 * kq + i % 4;
      bool nan_k = false;
      if (nan_groups)
        for (int g = 0; g < NG; ++g) nan_k |= block[32 * D + i / 4 * (D / 2) + 16 * g + 4 * kq + i % 4] == kScaleNaN;
#pragma unroll
      for (int z = 0; z < NT; ++z) {
        if (nan_k) p[z][i] = __uint_as_float(0x7FC00000u);
        if (t < rows[z].from || t >= rows[z].to) p[z][i] = -INFINITY;
      }
      // what no row of the tile sees may hold anything: its values count as zeros
      if (t < see.lo || t >= see.hi) x.vs[i / 4] &= ~(0xFFu << (8 * (i % 4)));
    }
    if (nan_groups) {
      for (int t = 0; t < kBlockTokens; ++t)
        for (int g = 0; g < NG; ++g) {
          const uint8_t sb = block[33 * D + t / 16 * (D / 2) + (t % 16 / 4 * NG + g) * 4 + t % 4];
#pragma unroll
          for (int z = 0; z < NT; ++z)
            if (sb == kScaleNaN && t0 + t >= rows[z].from && t0 + t < rows[z].to) nan_v[z] |= 1u << g;
        }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if ((x.vs[i / 4] >> (8 * (i % 4)) & 0xFFu) == kScaleNaN) x.vs[i / 4] &= ~(0xFFu << (8 * (i % 4)));
    }
  }
  u32x4_t pf[NT];
#pragma unroll
  for (int z = 0; z < NT; ++z) {
    Row<D>& r = rows[z];
    float m = p[z][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) m = fmaxf(m, p[z][i]);
    // (nothing seen yet: ref is -inf.  The same difference as below: no weight exceeds 2^kTop.)
    if (__any(m - r.ref > kTop<T>)) {
      const float now = fmaxf(r.ref, over_quarters_max(m) - kLift<T>);
      const float back = now == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(r.ref - now);
      r.ref = now;
      r.total *= back;
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) r.o[k][i] *= back;
    }
    const float ref = r.ref == -INFINITY ? 0.f : r.ref;
#pragma unroll
    for (int i = 0; i < 8; ++i) p[z][i] = __builtin_amdgcn_exp2f(p[z][i] - ref);
    // weights to 16 bits, as the values are that they meet on the matrix cores: half a step on each, 2^-8 (bf16) or 2^-11 (f16, from 2^-14
    // on) relative.  Outputs are 2.2e-3 (bf16) or 2.5e-4 (f16) from fp64 so, and 1.7e-3 or 2.0e-4 by the store alone
    pf[z] = u32x4_t{Mat<T>::round2(p[z][0], p[z][1]), Mat<T>::round2(p[z][2], p[z][3]), Mat<T>::round2(p[z][4], p[z][5]),
                    Mat<T>::round2(p[z][6], p[z][7])};
    // summed as rounded, so that what all weights have lost or gained in common cancels
#pragma unroll
    for (int i = 0; i < 4; ++i) r.total = Mat<T>::add2(pf[z][i], r.total);
  }
  float vf[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) vf[i] = scale_of(x.vs[i / 4] >> (8 * (i % 4)) & 0xFFu);
  static_for<D / 32>([&](auto jb) {                           // two values of the lane's eight tokens
    constexpr int J = decltype(jb)::value;
    uint32_t y[8];
    static_for<8>([&](auto ii) {
      constexpr int I = decltype(ii)::value, B = I % 4 * (D / 32) + J;
      y[I] = Mat<T>::template pair<B % 4>(x.vc[I / 4][B / 4], vf[I]);
    });
    u32x4_t even, odd2;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      even[h] = __builtin_amdgcn_perm(y[2 * h + 1], y[2 * h], 0x05040100u);
      odd2[h] = __builtin_amdgcn_perm(y[2 * h + 1], y[2 * h], 0x07060302u);
    }
#pragma unroll
    for (int z = 0; z < NT; ++z) {
      rows[z].o[2 * J] = Mat<T>::mfma(even, pf[z], rows[z].o[2 * J]);
      rows[z].o[2 * J + 1] = Mat<T>::mfma(odd2, pf[z], rows[z].o[2 * J + 1]);
    }
  });
  load_values<D, ONCE>(x, next, lane);
#pragma unroll
  for (int z = 0; z < NT; ++z)
    if (nan_v[z]) {
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (nan_v[z] >> (((4 * kq + i) * (D / 16) + k) / 32) & 1) rows[z].o[k][i] = __uint_as_float(0x7FC00000u);
    }
}

constexpr int kWaves = 4;
template <int D> struct JoinShared {
  float ref[kWaves][16], total[kWaves][16];
  float o[kWaves - 1][64][D / 4 + 1];
};

// The workgroup's waves into wave 0 (every lane calls; only wave 0's r is then of use).  total is a row's on entry and on return.
template <int D>
__device__ __forceinline__ void join_waves(Row<D>& r, JoinShared<D>& sh, int lane, int wave) {
  const int n = lane & 15, kq = lane >> 4;
  if (kq == 0) {
    sh.ref[wave][n] = r.ref;
    sh.total[wave][n] = r.total;
  }
  if (wave > 0) {
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) sh.o[wave - 1][lane][4 * k + i] = r.o[k][i];
  }
  __syncthreads();
  if (wave > 0) return;
  float best = sh.ref[0][n];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) best = fmaxf(best, sh.ref[w][n]);
  const float ref = best == -INFINITY ? 0.f : best;
  r.ref = best;
  float f = __builtin_amdgcn_exp2f(sh.ref[0][n] - ref);
  r.total *= f;
#pragma unroll
  for (int k = 0; k < D / 16; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) r.o[k][i] *= f;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) {
    f = __builtin_amdgcn_exp2f(sh.ref[w][n] - ref);
    r.total += sh.total[w][n] * f;
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) r.o[k][i] += sh.o[w - 1][lane][4 * k + i] * f;
  }
}

// A tile of rows (new token, query head of the group) of one key/value head of one sequence, and its splits.
struct Tile {
  int base;                   // place of the sequence's first new token
  Seen see;
  int b_lo, b_hi, splits;     // blocks that some row sees, and the workgroups they are divided among (1 where there are none)
};
__device__ __forceinline__ Tile find_tile(const Kv4AttentionArgs& a, const Sequence& sq, int news, int tile, int tile_rows) {
  Tile t;
  t.base = sq.len - sq.n_new;
  const int first_j = tile * tile_rows / a.group, last_j = min(news - 1, (tile * tile_rows + tile_rows - 1) / a.group);
  t.see.hi = max(0, min(sq.len, t.base + last_j + 1));
  t.see.lo = a.window > 0 ? max(0, t.base + first_j + 1 - a.window) : 0;
  t.see.all_to = t.base + first_j + 1;
  t.see.all_from = a.window > 0 ? t.base + last_j + 1 - a.window : 0;
  t.b_lo = t.see.lo / kBlockTokens;
  t.b_hi = (t.see.hi + kBlockTokens - 1) / kBlockTokens;
  t.splits = max(1, min(static_cast<int>(a.splits), (t.b_hi - t.b_lo + a.chunk - 1) / a.chunk));
  return t;
}

// Floats of a split's sums: [rows][D], then the rows' references and totals.
__device__ __forceinline__ float* split_sums(const Kv4AttentionArgs& a, int s, int unit_in_seq, int split, int D) {
  const unsigned row_tiles = (a.max_new * a.group + a.tile_rows - 1) / a.tile_rows;
  const size_t unit = static_cast<size_t>(s) * row_tiles * a.n_kv_heads + unit_in_seq;
  return a.partial + (unit * a.splits + split) * kv4_sums_floats(a.partial_rows, D);
}

// Waves of each SIMD that the registers are shared out for.
constexpr int attention_waves(int D, int NT) { return D == 64 ? (NT == 1 ? 4 : 3) : D == 128 ? (NT == 1 ? 3 : 2) : 2; }

// One workgroup: a tile of 16 NT rows and one split of the tokens that they see; its four waves take every fourth block of 32 tokens
// each.  Where a tile has several splits, each leaves its sums for kv4_combine_kernel.  Bound by HBM where there is work for all
// compute units (about 214 vector instructions for a block of 4352 bytes at head_dim 128: 860 cycles of a SIMD, and 1720 at the rate
// of a large read, 6.2 TB/s); a short call is a chain of loads: slot, length and page, keys, output.
template <typename T, int D, int NT, bool ONCE>
__global__ __launch_bounds__(64 * kWaves, attention_waves(D, NT)) void kv4_attention_kernel(Kv4AttentionArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, kq = lane >> 4;
  const int n_kv = a.n_kv_heads;
  const int head = blockIdx.x % n_kv;
  const int tile = blockIdx.x / n_kv;
  const int split = blockIdx.z;
  // Until the first keys are asked for, time goes into loads that wait for one another.  So what depends on the slot (length, pages) and the
  // queries are asked for before any of them is looked at, from addresses that are made valid instead of branches.
  Sequence sq = sequence_rows(a, blockIdx.y);
  const int news = min(sq.n_new, static_cast<int>(a.max_new));
  if (tile * 16 * NT >= news * a.group) return;
  const int slot = sq.real ? sq.slot : 0;
  const int length = a.length[slot];
  // 64 blocks' pages at a time, one to a lane; without a window the first of them do not have to wait for the length
  const int page_shift = a.page_shift - 5;                     // of blocks
  const int32_t* table = a.table + static_cast<size_t>(slot) * a.max_pages;
  auto pages_from = [&](int c0) { return table[min((c0 + lane * kWaves) >> page_shift, a.max_pages - 1)]; };
  int my_page = 0;
  if (a.window == 0) my_page = pages_from(split * a.chunk + wave);
  // this lane's rows: the z-th is row 16 z + n of the tile
  Row<D> rows[NT];
  int row[NT], hq[NT];        // row of the batch (-1: none) and query head
#pragma unroll
  for (int z = 0; z < NT; ++z) {
    const int r = tile * 16 * NT + 16 * z + n, j = r / a.group;
    hq[z] = head * a.group + r - j * a.group;
    row[z] = sq.row0 + j;
    if (j >= news || row[z] >= a.n_rows) row[z] = -1;
    rows[z].to = j + 1;       // (from the place of the first new token on, until the length is known)
    const uint16_t* q = a.q + static_cast<size_t>(max(0, row[z])) * a.ld_q + static_cast<size_t>(hq[z]) * D + kq * (D / 4);
#pragma unroll
    for (int k = 0; k < D / 32; ++k) rows[z].q[k] = *reinterpret_cast<const u32x4_t*>(q + 8 * k);
  }
  sq.len = sq.real ? length : 0;
  const Tile t = find_tile(a, sq, news, tile, 16 * NT);
  if (split >= t.splits) return;
  // the last split takes whatever is left
  const int b0 = t.b_lo + split * a.chunk, b1 = split == t.splits - 1 ? t.b_hi : b0 + a.chunk;
  if (a.window > 0) my_page = pages_from(b0 + wave);
#pragma unroll
  for (int z = 0; z < NT; ++z) {
    if (row[z] < 0)
#pragma unroll
      for (int k = 0; k < D / 32; ++k) rows[z].q[k] = u32x4_t{0, 0, 0, 0};
    rows[z].to += t.base;
    rows[z].from = a.window > 0 ? max(0, rows[z].to - a.window) : 0;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) rows[z].o[k] = floatx4{0, 0, 0, 0};
    rows[z].ref = -INFINITY;
    rows[z].total = 0.f;
  }

  // the head's part of page 0 and the distance to the next page's
  const unsigned part = (34u * D) << page_shift, page_bytes = part * static_cast<unsigned>(n_kv);
  const uint8_t* first_page = a.data + static_cast<size_t>(head) * part;
  for (int c0 = b0 + wave; c0 < b1; c0 += 64 * kWaves) {
    const int mine = min(64, (b1 - c0 + kWaves - 1) / kWaves);
    if (c0 != b0 + wave) my_page = pages_from(c0);
    auto page_at = [&](int i) {                               // -1: a block without a page, which nobody sees
      const int page = __builtin_amdgcn_readlane(my_page, i);
      return page < a.n_pages && (c0 + i * kWaves) >> page_shift < a.max_pages ? page : -1;
    };
    auto address = [&](int i) {                               // (without a page any will do)
      return first_page + static_cast<size_t>(static_cast<unsigned>(max(0, page_at(i)))) * page_bytes +
             ((c0 + i * kWaves) & ((1 << page_shift) - 1)) * (34 * D);
    };
    // two blocks in registers; each is replaced by the one after the next as it is used up
    auto buffer = [&](int i) { return block_buffer<D>(address(min(i, mine - 1)), i < mine); };
    auto work = [&](Block<D>& x, int i) {
      const int t0 = page_at(i) >= 0 ? (c0 + i * kWaves) * kBlockTokens : kNowhere;
      attend_block<T, D, NT, ONCE>(x, address(i), buffer(i + 2), t0, t.see, a.scale_log2, lane, rows);
    };
    Block<D> x, y;
    load_keys<D, ONCE>(x, buffer(0), lane);
    load_values<D, ONCE>(x, buffer(0), lane);
    load_keys<D, ONCE>(y, buffer(1), lane);
    load_values<D, ONCE>(y, buffer(1), lane);
    int i = 0;                                                // (pairs, and a last one by itself: no way out between the two)
    for (; i + 1 < mine; i += 2) {
      work(x, i);
      work(y, i + 1);
    }
    if (i < mine) work(x, i);
  }

  __shared__ JoinShared<D> sh;
#pragma unroll
  for (int z = 0; z < NT; ++z) {
    Row<D>& r = rows[z];
    r.total = over_quarters_sum(r.total);
    if (z > 0) __syncthreads();                               // wave 0 has read the rows before
    join_waves<D>(r, sh, lane, wave);
    if (wave > 0) continue;
    if (t.splits > 1) {
      if (16 * z + n >= static_cast<int>(a.partial_rows)) continue;
      float* sums = split_sums(a, blockIdx.y, blockIdx.x, split, D);
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        floatx4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int d = 4 * c + e;
          v[e] = r.o[d % (D / 16)][d / (D / 16)];
        }
        *reinterpret_cast<floatx4*>(sums + (16 * z + n) * D + kq * (D / 4) + 4 * c) = v;
      }
      if (kq == 0) {
        sums[a.partial_rows * D + 16 * z + n] = r.ref;
        sums[a.partial_rows * (D + 1) + 16 * z + n] = r.total;
      }
      continue;
    }
    if (row[z] < 0) continue;
    const float inv = r.total == 0.f ? 0.f : 1.0f / r.total;
    uint16_t* dst = a.out + static_cast<size_t>(row[z]) * a.ld_out + static_cast<size_t>(hq[z]) * D + kq * (D / 4);
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int d = 8 * c + e;
        v[e] = r.o[d % (D / 16)][d / (D / 16)] * inv;
      }
      *reinterpret_cast<uint4*>(dst + 8 * c) = pack8<T>(v);
    }
  }
}

// A row's splits into its output: WR waves to a row, each with up to 64 of its splits (their references and totals one to a
// lane, the sums 16 bytes to a lane).  Latency-bound: two round trips to what the other launch wrote.
template <typename T, int D, int WR>
__global__ __launch_bounds__(256) void kv4_combine_kernel(Kv4AttentionArgs a) {
  constexpr int PL = D / 4 < 64 ? D / 4 : 64, GL = 64 / PL;   // lanes to a split's sums, splits at a time
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int unit = blockIdx.x;                                // as in kv4_attention_kernel
  const int n_kv = a.n_kv_heads, head = unit % n_kv, tile = unit / n_kv;
  const int n = blockIdx.z * (4 / WR) + wave / WR;            // row of the tile
  const int first = wave % WR;
  // what a split of the plan may have left is read before it is known whether it did: the length takes as long to come
  const size_t stride = static_cast<size_t>(kv4_sums_floats(a.partial_rows, D)) * WR;
  const float* sums = split_sums(a, blockIdx.y, unit, first, D);
  float ref = -INFINITY, total = 0.f;
  const int most = n < static_cast<int>(a.partial_rows) ? (a.splits - first + WR - 1) / WR : 0;
  if (lane < most) {
    ref = sums[lane * stride + a.partial_rows * D + n];
    total = sums[lane * stride + a.partial_rows * (D + 1) + n];
  }
  const int c = lane % PL;
  constexpr int kEarly = 4;
  floatx4 early[kEarly];
#pragma unroll
  for (int e = 0; e < kEarly; ++e) {
    const int k = lane / PL + e * GL;
    early[e] = floatx4{0, 0, 0, 0};
    if (k < most) early[e] = *reinterpret_cast<const floatx4*>(sums + k * stride + n * D + 4 * c);
  }
  const Sequence sq = sequence(a, blockIdx.y);
  const int news = min(sq.n_new, static_cast<int>(a.max_new));
  if (tile * static_cast<int>(a.tile_rows) >= news * a.group) return;           // (uniform over the workgroup, as is the next)
  const Tile t = find_tile(a, sq, news, tile, a.tile_rows);
  if (t.splits == 1) return;
  const int r = tile * static_cast<int>(a.tile_rows) + n, j = r / a.group, row = sq.row0 + j;
  const bool has_row = n < static_cast<int>(a.partial_rows) && j < news && row >= 0 && row < a.n_rows;
  const int mine = has_row ? (t.splits - first + WR - 1) / WR : 0;
  if (lane >= mine) {
    ref = -INFINITY;
    total = 0.f;
  }
  float best = ref;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) best = fmaxf(best, __shfl_xor(best, m));
  const float weight = best == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - best);
  total = wave_sum(total * weight);
  floatx4 o = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < kEarly; ++e) {
    const int k = lane / PL + e * GL;
    const float w = __shfl(weight, k & 63);
    if (k < mine) {
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] += w * early[e][i];
    }
  }
  constexpr int kMore = 8;
  for (int k0 = kEarly * GL; k0 < mine; k0 += kMore * GL) {   // (uniform over the wave: every lane has its weight to give)
    floatx4 more[kMore];
#pragma unroll
    for (int e = 0; e < kMore; ++e) {
      const int k = k0 + e * GL + lane / PL;
      more[e] = floatx4{0, 0, 0, 0};
      if (k < mine) more[e] = *reinterpret_cast<const floatx4*>(sums + k * stride + n * D + 4 * c);
    }
#pragma unroll
    for (int e = 0; e < kMore; ++e) {
      const float w = __shfl(weight, (k0 + e * GL + lane / PL) & 63);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] += w * more[e][i];
    }
  }
#pragma unroll
  for (int m = PL; m < 64; m *= 2)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], m);
  if constexpr (WR > 1) {
    __shared__ floatx4 s_o[4][PL];
    __shared__ float s_best[4], s_total[4];
    if (lane < PL) s_o[wave][lane] = o;
    if (lane == 0) {
      s_best[wave] = best;
      s_total[wave] = total;
    }
    __syncthreads();
    if (wave > 0) return;
    for (int w = 1; w < WR; ++w) best = fmaxf(best, s_best[w]);
    const float all = best == -INFINITY ? 0.f : best;
    total = 0.f;
    o = floatx4{0, 0, 0, 0};
    for (int w = 0; w < WR; ++w) {
      const float f = __builtin_amdgcn_exp2f(s_best[w] - all);
      total += f * s_total[w];
      const floatx4 v = s_o[w][c];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += f * v[e];
    }
  }
  if (!has_row || lane >= PL) return;
  const float inv = total == 0.f ? 0.f : 1.0f / total;
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = o[e] * inv;
  *reinterpret_cast<uint2*>(a.out + static_cast<size_t>(row) * a.ld_out + static_cast<size_t>(head * a.group + r % a.group) * D + 4 * c) =
      pack4<T>(v);
}

template <typename F>
hipError_t by_kind(Kv4Kind kind, F&& f) {
  switch (kind.head_dim) {
    case 64: return kind.bf16 ? f.template operator()<BF16, 64>() : f.template operator()<F16, 64>();
    case 128: return kind.bf16 ? f.template operator()<BF16, 128>() : f.template operator()<F16, 128>();
    default: return kind.bf16 ? f.template operator()<BF16, 256>() : f.template operator()<F16, 256>();
  }
}

struct AppendLaunch {
  const Kv4AppendArgs& a;
  int n_seq;
  hipStream_t s;
  template <typename T, int D> hipError_t operator()() const {
    const int heads = a.n_heads + 2 * a.n_kv_heads, max_new = a.max_new;
    constexpr int kSlots = 256 / (D / 8), TW = kSlots < 16 ? kSlots : 16, HPL = 4;
    if (max_new < TW) return kv4_launch(kv4_append_kernel<T, D, 1, 1>, dim3((heads + kSlots - 1) / kSlots, n_seq, max_new), dim3(256), s, a);
    constexpr int kHeads = HPL * (kSlots / TW);
    return kv4_launch(kv4_append_kernel<T, D, TW, HPL>, dim3((heads + kHeads - 1) / kHeads, n_seq, (max_new + TW - 1 + TW - 1) / TW), dim3(256), s, a);
  }
};

struct AttentionLaunch {
  const Kv4AttentionArgs& a;
  int n_seq, row_tiles;
  hipStream_t s;
  template <typename T, int D> hipError_t operator()() const {
    const dim3 grid(static_cast<unsigned>(row_tiles) * a.n_kv_heads, n_seq, a.splits), block(64 * kWaves);
    const bool once = row_tiles == 1;
    void (*kernel)(Kv4AttentionArgs) = once ? kv4_attention_kernel<T, D, 1, true> : kv4_attention_kernel<T, D, 1, false>;
    if constexpr (D <= 128) {
      if (a.tile_rows == 32) kernel = once ? kv4_attention_kernel<T, D, 2, true> : kv4_attention_kernel<T, D, 2, false>;
    }
    if (hipError_t e = kv4_launch(kernel, grid, block, s, a)) return e;
    if (a.splits == 1) return hipSuccess;
    if (a.splits <= 16) return kv4_launch(kv4_combine_kernel<T, D, 1>, dim3(grid.x, grid.y, (a.partial_rows + 3) / 4), dim3(256), s, a);
    return kv4_launch(kv4_combine_kernel<T, D, 4>, dim3(grid.x, grid.y, a.partial_rows), dim3(256), s, a);
  }
};

}  // namespace

hipError_t launch_kv4_append(const Kv4AppendArgs& a, Kv4Kind kind, int n_seq, hipStream_t s) {
  return by_kind(kind, AppendLaunch{a, n_seq, s});
}
hipError_t launch_kv4_attention(const Kv4AttentionArgs& a, Kv4Kind kind, int n_seq, int row_tiles, hipStream_t s) {
  return by_kind(kind, AttentionLaunch{a, n_seq, row_tiles, s});
}

}  // namespace larosa
