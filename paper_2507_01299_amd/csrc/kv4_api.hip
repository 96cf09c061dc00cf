// C ABI of the 4-bit key/value cache: argument checks, workspace carving, launch sequencing.
#include "../../include/larosa.h"

#include <hip/hip_runtime.h>

#include <cmath>

#include "kernels.hpp"
#include "kv4.hpp"

using namespace larosa;

namespace {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline hipStream_t stream_of(void* s) { return static_cast<hipStream_t>(s); }
inline int status_of(hipError_t e) { return e == hipSuccess ? LAROSA_OK : LAROSA_EHIP; }

size_t page_bytes_of(const larosa_kv4_cache* C) {
  return static_cast<size_t>(C->n_kv_heads) * (C->page_tokens / 32) * 34 * C->head_dim;
}

// Sizes of a cache; nothing of it is read.
int check_sizes(const larosa_kv4_cache* C) {
  if (!C || C->n_layers < 1 || C->n_pages < 1 || C->n_slots < 1 || C->max_pages < 1 || C->n_kv_heads < 1) return LAROSA_EINVAL;
  if (C->dtype != LAROSA_F16 && C->dtype != LAROSA_BF16) return LAROSA_EINVAL;
  if (C->page_tokens != 32 && C->page_tokens != 64 && C->page_tokens != 128 && C->page_tokens != 256) return LAROSA_EINVAL;
  if (C->head_dim != 64 && C->head_dim != 128 && C->head_dim != 256) return LAROSA_EUNSUPPORTED;
  // places in a sequence and numbers of pages are 32-bit
  if (static_cast<long>(C->max_pages) * C->page_tokens >= (1L << 30) || C->n_kv_heads > kKv4HeadsMax) return LAROSA_EUNSUPPORTED;
  if (C->n_pages > (1 << 28) || C->n_slots > kKv4SlotsMax || C->n_layers > 65535) return LAROSA_EUNSUPPORTED;
  if (static_cast<long>(C->n_slots) * C->max_pages >= (1L << 31)) return LAROSA_EUNSUPPORTED;   // (counts of pages are 32-bit)
  // 8 TiB: pages of all layers, of 2176 bytes at least, are counted in 32 bits; bytes of one layer stay below 2^57
  if (page_bytes_of(C) * C->n_pages > ((size_t{1} << 43) - 1) / C->n_layers) return LAROSA_EUNSUPPORTED;
  return LAROSA_OK;
}

int check_cache(const larosa_kv4_cache* C) {
  if (int rc = check_sizes(C)) return rc;
  if (!C->data || !C->refs || !C->table || !C->length) return LAROSA_EINVAL;
  if (!aligned(C->data, 16) || !aligned(C->refs, 4) || !aligned(C->table, 4) || !aligned(C->length, 4)) return LAROSA_EINVAL;
  return LAROSA_OK;
}

int check_batch(const larosa_kv4_batch* b) {
  if (!b || !b->slots || b->n_seq < 1 || b->n_rows < 1 || b->max_new < 1) return LAROSA_EINVAL;
  if (!aligned(b->slots, 4) || !aligned(b->starts, 4)) return LAROSA_EINVAL;
  if (!b->starts && (b->max_new != 1 || b->n_rows < b->n_seq)) return LAROSA_EINVAL;
  if (b->n_seq > 65535 || b->max_new > kKv4NewMax) return LAROSA_EUNSUPPORTED;      // (sides of a launch)
  return LAROSA_OK;
}

int check_heads(const larosa_kv4_cache* C, int n_heads) {
  if (n_heads < 1 || n_heads % C->n_kv_heads) return LAROSA_EINVAL;
  return n_heads > 65536 ? LAROSA_EUNSUPPORTED : LAROSA_OK;
}

// Attention of so many heads: its tiles of 16 rows lie along one side of a launch (of 256 lanes each, below 2^32).
int check_attention(const larosa_kv4_cache* C, const larosa_kv4_batch* b, int n_heads) {
  if (int rc = check_heads(C, n_heads)) return rc;
  const long rows = static_cast<long>(b->max_new) * (n_heads / C->n_kv_heads);
  return (rows + 15) / 16 * C->n_kv_heads >= (1L << 24) ? LAROSA_EUNSUPPORTED : LAROSA_OK;
}

int check_rotary(const larosa_rotary* r, const larosa_kv4_cache* C) {
  if (!r->table || !aligned(r->table, 16) || !aligned(r->positions, 4) || r->n_positions < 1) return LAROSA_EINVAL;
  if (r->rot_dim < 16 || r->rot_dim % 16 || r->rot_dim > C->head_dim) return LAROSA_EINVAL;
  if (r->n_axes < 1 || r->n_axes > 4 || (r->n_axes > 1 && !r->positions)) return LAROSA_EINVAL;
  if (r->n_axes > 1) {
    int sum = 0;
    for (int i = 0; i < r->n_axes; ++i) {
      if (r->axis_pairs[i] < 0 || r->axis_pairs[i] > r->rot_dim / 2) return LAROSA_EINVAL;
      sum += r->axis_pairs[i];
    }
    if (sum != r->rot_dim / 2) return LAROSA_EINVAL;
  }
  return LAROSA_OK;
}

inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// How an attention call is divided.  A tile of 16 or 32 rows sees `blocks` blocks of 32 tokens; its workgroups take `chunk` each, four waves
// one block at a time, and a second launch adds up what several workgroups of a tile left.  That launch takes 4 us and a
// workgroup 5 us to come to its first block, a block 1 us, so
//  - up to 24 blocks are one workgroup's (333 tokens of an 8B model: 6.3 us, with two workgroups a tile 8.4);
//  - one sequence, or few, are cut into two pieces for each compute unit, of eight blocks at least (100003 tokens of a 70B model: 26.6 us;
//    with three, which are resident at once, 27.1, with 640 or 1024 pieces, which leave compute units idle at the end, 29.3);
//  - else into pieces of 32 blocks, since lengths differ and a piece past a sequence's end costs nothing (9 sequences of up to
//    8191 tokens, 7 new each: 22.9 us; pieces of 24 25.5, of 40 24.6, of 64 27.7), longer ones past 4096 of them (64 sequences of up
//    to 16384 tokens: 75.5 us; past 2048 80.1).
constexpr long kWholeBlocks = 24, kLeastBlocks = 8, kPieceBlocks = 32, kResident = 512, kMostWorkgroups = 4096;
constexpr int kWindowMost = 0x7FFFFFFF - 2 * kKv4NewMax;      // (places with a page are below 2^30)
struct AttentionPlan {
  int tile_rows;
  long row_tiles, units;      // tiles of a key/value head's rows; such tiles of all sequences
  int chunk, splits, partial_rows;
  size_t partial_bytes;
};
AttentionPlan plan_attention(const larosa_kv4_cache* C, const larosa_kv4_batch* b, int n_heads, int window, int max_len) {
  AttentionPlan p{};
  const long rows = static_cast<long>(b->max_new) * (n_heads / C->n_kv_heads);
  const long most = static_cast<long>(C->max_pages) * C->page_tokens;
  long span = max_len > 0 && max_len < most ? max_len : most;
  if (window > 0 && window < span) span = window + b->max_new < span ? window + b->max_new : span;
  const long blocks = (span + 31) / 32 + (window > 0 ? 1 : 0);
  // 32 rows to a tile convert the codes half as often, but leave fewer waves and workgroups: from a thousand pieces of 32 blocks on
  // (a prompt of 4096 tokens, 8B heads: 278 -> 233 us, 32 sequences of 8000 tokens with eight new: 95 -> 80; with less work it goes
  // either way: eight such sequences 27 -> 24, one of 20000 tokens 14.7 -> 16.5).  At head_dim 256 the 16 rows take all registers.
  const long tiles32 = (rows + 31) / 32;
  p.tile_rows = rows > 16 && C->head_dim <= 128 && tiles32 * C->n_kv_heads * b->n_seq * blocks >= 1000 * kPieceBlocks ? 32 : 16;
  p.row_tiles = (rows + p.tile_rows - 1) / p.tile_rows;
  p.units = p.row_tiles * C->n_kv_heads * b->n_seq;
  p.partial_rows = rows < p.tile_rows ? static_cast<int>(rows) : p.tile_rows;
  long chunk = blocks;
  if (blocks > kWholeBlocks) {
    if (b->n_seq == 1 || p.units * ((blocks + kPieceBlocks - 1) / kPieceBlocks) < kResident) {
      const long splits = kResident / p.units > 1 ? kResident / p.units : 1;
      chunk = (blocks + splits - 1) / splits;
      if (chunk < kLeastBlocks) chunk = kLeastBlocks;
    } else {
      chunk = (blocks * p.units + kMostWorkgroups - 1) / kMostWorkgroups;
      if (chunk < kPieceBlocks) chunk = kPieceBlocks;
    }
    if (chunk * kKv4SplitsMax < blocks) chunk = (blocks + kKv4SplitsMax - 1) / kKv4SplitsMax;
    if (chunk > blocks) chunk = blocks;
  }
  const long splits = (blocks + chunk - 1) / chunk;
  p.chunk = static_cast<int>(chunk);
  p.splits = static_cast<int>(splits);
  p.partial_bytes = splits > 1 ? static_cast<size_t>(p.units) * splits * kv4_sums_floats(p.partial_rows, C->head_dim) * 4 : 0;
  return p;
}

// The plan of a call: a window's own only where the workspace, which is sized without it, suffices.
AttentionPlan plan_call(const larosa_kv4_cache* C, const larosa_kv4_batch* b, int n_heads, int window, int max_len) {
  const AttentionPlan p = plan_attention(C, b, n_heads, window, max_len), all = plan_attention(C, b, n_heads, 0, max_len);
  return p.partial_bytes > all.partial_bytes ? all : p;
}

Kv4Scratch scratch_of(void* ws) { return Kv4Scratch{reinterpret_cast<int32_t*>(static_cast<char*>(ws) + kCounterBytes)}; }

Kv4Kind kind_of(const larosa_kv4_cache* C) { return Kv4Kind{C->head_dim, C->dtype == LAROSA_BF16}; }

uint8_t* layer_data(const larosa_kv4_cache* C, int layer) {
  return static_cast<uint8_t*>(C->data) + static_cast<size_t>(layer) * C->n_pages * page_bytes_of(C);
}

// What append and attention have in common.
template <typename Args>
void fill_common(Args& a, const larosa_kv4_cache* C, const larosa_kv4_batch* b, int layer) {
  a.data = layer_data(C, layer);
  a.table = C->table; a.length = C->length;
  a.slots = b->slots; a.starts = b->starts;
  a.n_pages = C->n_pages; a.max_pages = C->max_pages; a.n_slots = C->n_slots; a.n_kv_heads = C->n_kv_heads;
  a.n_rows = b->n_rows; a.max_new = b->max_new;
  a.page_shift = __builtin_ctz(C->page_tokens);
}

// A list of slots and the status it reports to.
int check_list(const larosa_kv4_cache* C, const int32_t* list, int n) {
  if (!list || !aligned(list, 4) || n < 1) return LAROSA_EINVAL;
  return n > C->n_slots ? LAROSA_EINVAL : LAROSA_OK;      // more than there are slots: one is listed twice
}

}  // namespace

extern "C" {

size_t larosa_kv4_page_bytes(int page_tokens, int n_kv_heads, int head_dim) {
  larosa_kv4_cache C{};
  C.n_layers = C.n_pages = C.n_slots = C.max_pages = 1;
  C.page_tokens = page_tokens; C.n_kv_heads = n_kv_heads; C.head_dim = head_dim;
  if (check_sizes(&C) != LAROSA_OK) return 0;
  return page_bytes_of(&C);
}

size_t larosa_kv4_data_bytes(const larosa_kv4_cache* C) {
  if (check_sizes(C) != LAROSA_OK) return 0;
  return static_cast<size_t>(C->n_layers) * C->n_pages * page_bytes_of(C);
}

int larosa_kv4_clear(const larosa_kv4_cache* C, void* stream) {
  if (int rc = check_cache(C)) return rc;
  hipStream_t st = stream_of(stream);
  if (launch_fill_u32(reinterpret_cast<unsigned*>(C->refs), C->n_pages, 0u, st) != hipSuccess) return LAROSA_EHIP;
  if (launch_fill_u32(reinterpret_cast<unsigned*>(C->length), C->n_slots, 0u, st) != hipSuccess) return LAROSA_EHIP;
  return status_of(launch_fill_u32(reinterpret_cast<unsigned*>(C->table), static_cast<size_t>(C->n_slots) * C->max_pages, ~0u, st));
}

int larosa_kv4_append(const larosa_kv4_cache* C, int layer, const larosa_kv4_batch* b, const void* qkv, int ld_qkv, int n_heads,
                      const larosa_rotary* rotary, void* out, int ld_out, void* stream) {
  if (int rc = check_cache(C)) return rc;
  if (int rc = check_batch(b)) return rc;
  if (int rc = check_heads(C, n_heads)) return rc;
  if (layer < 0 || layer >= C->n_layers || !qkv || !aligned(qkv, 16) || !aligned(out, 16)) return LAROSA_EINVAL;
  const long width = (static_cast<long>(n_heads) + 2 * C->n_kv_heads) * C->head_dim;
  if (ld_qkv < width || ld_qkv % 8) return LAROSA_EINVAL;
  if (out && (ld_out < width || ld_out % 8 || (out == qkv && ld_out != ld_qkv))) return LAROSA_EINVAL;
  if (rotary) {
    if (int rc = check_rotary(rotary, C)) return rc;
    if (!out) return LAROSA_EINVAL;
  }
  Kv4AppendArgs a{};
  fill_common(a, C, b, layer);
  a.n_heads = n_heads;
  if (rotary) {
    a.turns = rotary->table; a.positions = rotary->positions;
    a.n_positions = rotary->n_positions; a.rot_dim = rotary->rot_dim;
    a.interleaved = rotary->interleaved != 0; a.n_axes = rotary->n_axes;
    for (int i = 0, end = 0; i < 3; ++i) {
      if (i + 1 < rotary->n_axes) end += rotary->axis_pairs[i];
      a.axis_ends |= static_cast<uint32_t>(i + 1 < rotary->n_axes ? end : 255) << 8 * i;
    }
  }
  a.qkv = static_cast<const uint16_t*>(qkv); a.ld_qkv = ld_qkv;
  a.out = static_cast<uint16_t*>(out); a.ld_out = ld_out;
  return status_of(launch_kv4_append(a, kind_of(C), b->n_seq, stream_of(stream)));
}

size_t larosa_kv4_attention_workspace_bytes(const larosa_kv4_cache* C, const larosa_kv4_batch* b, int n_heads, int max_len) {
  if (check_sizes(C) != LAROSA_OK || check_batch(b) != LAROSA_OK || check_attention(C, b, n_heads) != LAROSA_OK || max_len < 0) return 0;
  return kCounterBytes + round_up(plan_attention(C, b, n_heads, 0, max_len).partial_bytes, 256);
}

int larosa_kv4_attention(const larosa_kv4_cache* C, int layer, const larosa_kv4_batch* b, const void* q, int ld_q, int n_heads,
                         float scale, int window, int max_len, void* out, int ld_out, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_cache(C)) return rc;
  if (int rc = check_batch(b)) return rc;
  if (int rc = check_attention(C, b, n_heads)) return rc;
  if (layer < 0 || layer >= C->n_layers || !q || !out || !aligned(q, 16) || !aligned(out, 16)) return LAROSA_EINVAL;
  const long width = static_cast<long>(n_heads) * C->head_dim;
  if (ld_q < width || ld_q % 8 || ld_out < width || ld_out % 8 || q == out) return LAROSA_EINVAL;
  if (!std::isfinite(scale) || window < 0 || max_len < 0) return LAROSA_EINVAL;
  if (!ws || !aligned(ws, 256) || ws_bytes < larosa_kv4_attention_workspace_bytes(C, b, n_heads, max_len)) return LAROSA_EWORKSPACE;
  Kv4AttentionArgs a{};
  fill_common(a, C, b, layer);
  a.group = n_heads / C->n_kv_heads;
  a.q = static_cast<const uint16_t*>(q); a.ld_q = ld_q;
  a.out = static_cast<uint16_t*>(out); a.ld_out = ld_out;
  a.scale_log2 = scale * 1.4426950408889634f;
  // the kernels take it from the places of a tile's rows, which may lie up to max_new before a sequence's first token
  a.window = window < kWindowMost ? window : kWindowMost;
  const AttentionPlan p = plan_call(C, b, n_heads, window, max_len);
  a.tile_rows = p.tile_rows;
  a.chunk = p.chunk; a.splits = p.splits; a.partial_rows = p.partial_rows;
  a.partial = reinterpret_cast<float*>(static_cast<char*>(ws) + kCounterBytes);
  return status_of(launch_kv4_attention(a, kind_of(C), b->n_seq, static_cast<int>(p.row_tiles), stream_of(stream)));
}

int larosa_kv4_attention_plan(const larosa_kv4_cache* C, const larosa_kv4_batch* b, int n_heads, int window, int max_len, int* plan) {
  if (int rc = check_sizes(C)) return rc;
  if (int rc = check_batch(b)) return rc;
  if (int rc = check_attention(C, b, n_heads)) return rc;
  if (window < 0 || max_len < 0 || !plan) return LAROSA_EINVAL;
  const AttentionPlan p = plan_call(C, b, n_heads, window, max_len);
  plan[0] = p.tile_rows;
  plan[1] = static_cast<int>(p.row_tiles);
  plan[2] = p.chunk;
  plan[3] = p.splits;
  plan[4] = kv4_sums_floats(p.partial_rows, C->head_dim);
  return LAROSA_OK;
}

// ---- pages ---------------------------------------------------------------------------------------

size_t larosa_kv4_pages_workspace_bytes(const larosa_kv4_cache* C) {
  return check_sizes(C) == LAROSA_OK ? kCounterBytes + kv4_scratch_bytes(*C) : 0;
}

int larosa_kv4_grow(const larosa_kv4_cache* C, const int32_t* slots, const int32_t* counts, int n, int32_t* status, void* ws,
                    size_t ws_bytes, void* stream) {
  if (int rc = check_cache(C)) return rc;
  if (int rc = check_list(C, slots, n)) return rc;
  if (!aligned(counts, 4) || !status || !aligned(status, 4)) return LAROSA_EINVAL;
  if (!ws || !aligned(ws, 256) || ws_bytes < larosa_kv4_pages_workspace_bytes(C)) return LAROSA_EWORKSPACE;
  return status_of(launch_kv4_grow(*C, slots, counts, n, status, scratch_of(ws), stream_of(stream)));
}

int larosa_kv4_fork(const larosa_kv4_cache* C, const int32_t* src, const int32_t* dst, int n, int32_t* status, void* stream) {
  if (int rc = check_cache(C)) return rc;
  if (int rc = check_list(C, src, n)) return rc;
  if (int rc = check_list(C, dst, n)) return rc;
  if (!status || !aligned(status, 4)) return LAROSA_EINVAL;
  return status_of(launch_kv4_fork(*C, src, dst, n, status, stream_of(stream)));
}

int larosa_kv4_trim(const larosa_kv4_cache* C, const int32_t* slots, const int32_t* keep, int n, void* stream) {
  if (int rc = check_cache(C)) return rc;
  if (!slots || !aligned(slots, 4) || !aligned(keep, 4) || n < 1) return LAROSA_EINVAL;
  if (n > (1 << 20)) return LAROSA_EUNSUPPORTED;
  return status_of(launch_kv4_trim(*C, slots, keep, n, stream_of(stream)));
}

int larosa_kv4_compact(const larosa_kv4_cache* C, int32_t* live, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_cache(C)) return rc;
  if (!aligned(live, 4)) return LAROSA_EINVAL;
  if (!ws || !aligned(ws, 256) || ws_bytes < larosa_kv4_pages_workspace_bytes(C)) return LAROSA_EWORKSPACE;
  return status_of(launch_kv4_compact(*C, live, scratch_of(ws), stream_of(stream)));
}

int larosa_kv4_copy_pages(const larosa_kv4_cache* C, const int32_t* src, const int32_t* dst, int n, void* stream) {
  if (int rc = check_cache(C)) return rc;
  if (!src || !dst || !aligned(src, 4) || !aligned(dst, 4) || n < 1 || n > C->n_pages) return LAROSA_EINVAL;
  return status_of(launch_kv4_copy_pages(*C, src, dst, n, stream_of(stream)));
}

// ---- a decoder layer with the cache as its attention core -------------------------------------------

namespace {

// Whether a layer, a cache and a batch fit together, for all four steps.
int check_layer_cache(const larosa_layer* L, const larosa_kv4_cache* C, const larosa_kv4_batch* b) {
  if (!L) return LAROSA_EINVAL;
  if (int rc = check_sizes(C)) return rc;
  if (int rc = check_batch(b)) return rc;
  if (L->head_dim != C->head_dim || L->dtype != C->dtype || L->d_kv != C->n_kv_heads * C->head_dim || L->d_q % C->head_dim)
    return LAROSA_EINVAL;
  if (int rc = check_attention(C, b, L->d_q / C->head_dim)) return rc;
  return check_layer_rows(L, b->n_rows);
}

// What the three steps use one after the other; q|k|v, the shortcut and the attention's output lie behind it.
size_t shared_scratch(const larosa_layer* L, const larosa_kv4_cache* C, const larosa_kv4_batch* b, int max_len) {
  const size_t layer = larosa_layer_workspace_bytes(L, b->n_rows);
  const size_t attention = larosa_kv4_attention_workspace_bytes(C, b, L->d_q / C->head_dim, max_len);
  if (!layer || !attention) return 0;
  return round_up(layer > attention ? layer : attention, 256);
}

}  // namespace

size_t larosa_layer_kv4_workspace_bytes(const larosa_layer* L, const larosa_kv4_cache* C, const larosa_kv4_batch* b, int max_len) {
  if (check_layer_cache(L, C, b) != LAROSA_OK) return 0;
  const size_t head = shared_scratch(L, C, b, max_len);
  if (!head) return 0;
  const size_t rows = b->n_rows;
  return head + round_up(rows * (L->d_q + 2 * static_cast<size_t>(L->d_kv)) * 2, 256) + round_up(rows * L->d * 2, 256) +
         round_up(rows * L->d_q * 2, 256);
}

int larosa_layer_forward_kv4(const larosa_layer* L, const larosa_kv4_cache* C, int layer, const larosa_kv4_batch* b,
                             const larosa_rotary* rotary, float scale, int window, int max_len, const void* x, void* x_out,
                             const larosa_trace* trace, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_layer_cache(L, C, b)) return rc;
  if (int rc = check_cache(C)) return rc;
  // everything that one of the steps could refuse, before the first of them is enqueued
  if (layer < 0 || layer >= C->n_layers || !std::isfinite(scale) || window < 0 || max_len < 0) return LAROSA_EINVAL;
  if (!x || !x_out || x == x_out || !aligned(x, 16) || !aligned(x_out, 16)) return LAROSA_EINVAL;
  if (rotary)
    if (int rc = check_rotary(rotary, C)) return rc;
  const size_t need = larosa_layer_kv4_workspace_bytes(L, C, b, max_len);
  if (!ws || !aligned(ws, 256) || ws_bytes < need) return LAROSA_EWORKSPACE;
  const size_t head = shared_scratch(L, C, b, max_len), rows = b->n_rows;
  const int d_qkv = L->d_q + 2 * L->d_kv, heads = L->d_q / C->head_dim;
  char* p = static_cast<char*>(ws) + head;
  void* qkv = p;
  void* s1 = p += round_up(rows * d_qkv * 2, 256);
  void* attn = p += round_up(rows * L->d * 2, 256);
  if (int rc = larosa_layer_qkv(L, x, qkv, s1, b->n_rows, trace, ws, head, stream)) return rc;
  if (int rc = larosa_kv4_append(C, layer, b, qkv, d_qkv, heads, rotary, qkv, d_qkv, stream)) return rc;
  if (int rc = larosa_kv4_attention(C, layer, b, qkv, d_qkv, heads, scale, window, max_len, attn, L->d_q, ws, head, stream)) return rc;
  return larosa_layer_after_attention(L, L->shortcut_attn ? s1 : x, attn, x_out, b->n_rows, trace, ws, head, stream);
}

}  // extern "C"
