// Host-side launch interface of the operators on 8-bit floating-point weights and of the log probabilities (internal to liblarosa).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace larosa {

// Rows (activations, or a weight's output channels) in e4m3 codes with scales 2^(byte - 127) for 128 neighbours.
struct Held8 {
  const uint8_t* codes;       // [rows, pitch]: pitch = d up to 16, zeros behind d
  const uint8_t* scales;      // rows: [rows, scale_pitch]; a weight: [rows / 128 up, scale_pitch]; scale_pitch = d / 128 up, up to 4
};
inline int pitch8(int d) { return (d + 15) / 16 * 16; }
inline int scale_pitch8(int d) { return ((d + 127) / 128 + 3) / 4 * 4; }

constexpr int kWidthMax8 = 1 << 20;    // channels summed over: a panel of 256 rows stays below 2^28 bytes
constexpr int kOutMax8 = (1 << 21) - 16;    // rows of a weight, values between rows of y: 256 rows of y stay below 2^31 bytes
constexpr int kRowsMax8 = 1 << 24;
constexpr long kTilesMax8 = 1 << 23;   // of 256 threads each
// Bytes of rows' codes, times strips, that the product of few rows makes for itself.  Both sides in us: 4 x 4096 x 4096 8.7 (two launches 10.5), but
// with four strips, whose workgroups are many, 4 x 4096 x 128256 120 (112).
constexpr int kShortRows = 16384;

hipError_t launch_quantize_w8(const uint16_t* W, int d_in, int d_out, uint8_t* codes, uint8_t* scales, bool bf16, hipStream_t s);
// norm_scale nullable; norm_eps < 0: no norm; tiled: pieces of 16 rows x 64 codes, for launch_product8 only
hipError_t launch_quantize_rows8(const uint16_t* x, long ld_x, int n_rows, int d, const uint16_t* norm_scale, float norm_eps,
                                 uint8_t* codes, uint8_t* scales, bool tiled, bool bf16, hipStream_t s);
// bytes of the codes of n_rows rows, tiled
inline size_t tiled_bytes8(int n_rows, int d) { return (static_cast<size_t>(n_rows) + 15) / 16 * 16 * ((pitch8(d) + 63) / 64 * 64); }

// y[m, o] = sum_i x[m, i] w[o, i]
enum : int { kOutF16 = 0, kOutBF16 = 1, kOutF32 = 2 };
struct Product8Args {
  Held8 x, w;
  bool tiled;                 // x's codes (never where plan_product8 says kind 0)
  const uint16_t* x16;        // kind 0: x itself [n_rows, ld_x] instead of its codes, or nullptr; only where takes_rows16 says so
  long ld_x;
  bool x_bf16;
  void* y;                    // [n_rows, ld_y]
  long ld_y;
  int n_rows, d_in, d_out;
  int out;                    // kOutF16, ..
  // split of the work, from plan_product8
  int tiles_m, tiles_o;       // tiles of rows and of output channels
  int splits, blocks_per;     // parts of a tile's sum, blocks of 128 of each
  float* partial;             // [tiles][splits][tile]
  unsigned* counters;         // [tiles], kCounterStride apart, zero on entry and on exit
};
struct Product8Plan {
  int kind;                   // which kernel (0: up to 16 rows, else by its tile)
  int strips;                 // kind 0: of 16 output channels a workgroup
  int tiles_m, tiles_o, splits, blocks_per;
  size_t partial_floats;
};
Product8Plan plan_product8(int n_rows, int d_in, int d_out);      // from 17 rows on the same for 64 k + 1 .. 64 k + 64 rows
constexpr int kRowsOfParts8 = 32768;   // with more rows no sum goes in parts: their tiles, of any kind, fill more than half of the chip
bool plans_product8(int n_rows, int d_out);    // whether there is a plan: not more than kTilesMax8 tiles
inline bool takes_rows16(const Product8Plan& p, int n_rows, int d_in) {
  return p.kind == 0 && n_rows * ((d_in + 127) / 128) * p.strips <= kShortRows / 128;
}
hipError_t launch_product8(const Product8Args& a, const Product8Plan& p, hipStream_t s);

// Log probabilities of logits [n_rows, ld], the first n_vocab of a row.
enum : int { kLogitsF16 = 0, kLogitsBF16 = 1, kLogitsF32 = 2 };
constexpr int kTopMax = 64;
constexpr int kWorkgroupsOfFew = 512;  // fewer rows go in slices, up to this many workgroups in all
constexpr int kVocabMax = 1 << 28;     // bytes of a row are below 2^31
constexpr float kLogitScaleMax = 0x1p126f;     // scale / ln 2 is finite: infinity times a difference of 0 would be NaN
struct LogprobsArgs {
  const void* logits;
  long ld;
  int n_rows, n_vocab;
  float scale;
  const int32_t* given;       // [n_rows, n_given]
  int n_given;
  float* logp;                // [n_rows, n_given]
  float* entropy;             // [n_rows] or nullptr
  int n_top;
  int32_t* top_id;            // [n_rows, n_top]
  float* top_logp;            // [n_rows, n_top] or nullptr
  int slices, slice_len;      // of a row
  float* sums;                // [n_rows][slices][4]
  unsigned long long* best;   // [n_rows][slices][holders]: the largest of 128 logits with its place
  unsigned* counters;         // [n_rows] words, zero on entry and on exit
};
struct LogprobsPlan { int slices, slice_len; size_t sums_bytes, best_bytes; };
LogprobsPlan plan_logprobs(int n_rows, int n_vocab, int n_top);
hipError_t launch_logprobs(const LogprobsArgs& a, int type, hipStream_t s);

}  // namespace larosa
