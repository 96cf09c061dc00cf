// Host-side launch interface of the 4-bit key/value cache's kernels (internal to liblarosa).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/larosa.h"

namespace larosa {

struct Kv4AppendArgs {
  larosa_kv4_cache C;
  larosa_kv4_batch b;
  larosa_rotary r;            // r.table == nullptr: no rotation
  int layer, n_heads;
  const uint16_t* qkv;
  int ld_qkv;
  uint16_t* out;              // nullable
  int ld_out;
};
hipError_t launch_kv4_append(const Kv4AppendArgs& a, hipStream_t s);

struct Kv4AttentionArgs {
  larosa_kv4_cache C;
  larosa_kv4_batch b;
  int layer, n_heads, group;
  const uint16_t* q;
  int ld_q;
  uint16_t* out;
  int ld_out;
  float scale_log2;           // scale * log2(e): the exponentials are powers of two
  int window;                 // 0: none
  int tile_rows, row_tiles;   // 16 or 32 (new token, query head of the group) pairs to a tile, and tiles of a sequence's head
  // the split of the tokens: `chunk` blocks of 32 to a workgroup, up to `splits` workgroups for a tile
  int chunk, splits;
  float* partial;             // [n_seq][row_tiles * n_kv_heads][splits][partial_rows * (head_dim + 2)] fp32
  int partial_rows;           // rows that a tile can have
};
constexpr int kKv4SplitsMax = 256;            // that one row's sums are joined from
hipError_t launch_kv4_attention(const Kv4AttentionArgs& a, hipStream_t s);

// ---- pages (kv4_pages.hip) -----------------------------------------------------------------------------
// Scratch behind the arrival counters of a workspace.
struct Kv4Scratch {
  int32_t* n_pairs;           // [1] pages to copy
  int32_t* pair_src;          // [n_pages]
  int32_t* pair_dst;          // [n_pages]
  int32_t* free_ids;          // [n_pages] grow: pages to hand out; compact: where a page moves to
  int32_t* growing;           // [n_pages] grow: listed slots that would write into a shared page
  int32_t* last;              // [n_pages] grow: the last of them, by its place in the list, from 1
  int32_t* offset;            // [n_slots] grow: pages handed out before those of a slot of the list
  int32_t* pair;              // [n_slots] grow: its pair of pages to copy, or -1
  int32_t* n_live;            // [1] compact: pages in use
};
constexpr int kKv4SlotsMax = 1 << 18;         // (a bit each in LDS)
hipError_t launch_kv4_grow(const larosa_kv4_cache& C, const int32_t* slots, const int32_t* counts, int n, int32_t* status,
                           const Kv4Scratch& x, hipStream_t s);
hipError_t launch_kv4_fork(const larosa_kv4_cache& C, const int32_t* src, const int32_t* dst, int n, int32_t* status, hipStream_t s);
hipError_t launch_kv4_trim(const larosa_kv4_cache& C, const int32_t* slots, const int32_t* keep, int n, hipStream_t s);
hipError_t launch_kv4_compact(const larosa_kv4_cache& C, int32_t* live, const Kv4Scratch& x, hipStream_t s);
hipError_t launch_kv4_copy_pages(const larosa_kv4_cache& C, const int32_t* src, const int32_t* dst, int n, hipStream_t s);

}  // namespace larosa
