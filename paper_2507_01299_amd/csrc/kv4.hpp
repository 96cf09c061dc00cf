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
  int row_tiles;              // of 16 (new token, query head of the group) pairs
};
hipError_t launch_kv4_attention(const Kv4AttentionArgs& a, hipStream_t s);

}  // namespace larosa
