// Host-side launch interface of the 4-bit key/value cache's kernels (internal to liblarosa).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/larosa.h"

namespace larosa {

// A kernel's launch.  The runtime takes 2.65 us of the host for one whose arguments are at most 112 bytes together and 3.4 for
// more (measured from 16 to 520), which is most of a short call; asking for the last error takes another 0.2.
constexpr size_t kKv4ArgBytes = 112;
template <typename... P>
hipError_t kv4_launch(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t s, P... args) {
  static_assert((sizeof(P) + ...) <= kKv4ArgBytes);
  void* ptrs[] = {static_cast<void*>(&args)...};
  const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, ptrs, 0, s);
  if (e != hipSuccess) (void)hipGetLastError();
  return e;
}

constexpr int kKv4SlotsMax = 1 << 18, kKv4HeadsMax = 1 << 12, kKv4NewMax = 1 << 18;

struct Kv4Kind {              // what picks a kernel
  int head_dim;
  bool bf16;
};

struct Kv4AppendArgs {
  uint8_t* data;              // of the layer
  const int32_t *table, *length, *slots, *starts;
  const uint16_t* qkv;
  uint16_t* out;              // nullable
  const float* turns;         // cosines and sines, nullptr: no rotation
  const int32_t* positions;
  int n_pages, max_pages, n_rows, ld_qkv, ld_out, n_positions;
  uint32_t n_slots : 19, n_kv_heads : 13;
  uint32_t max_new : 19, page_shift : 4;       // page_tokens = 2^page_shift
  uint32_t n_heads : 17, rot_dim : 9, interleaved : 1, n_axes : 3;
  uint32_t axis_ends;         // pairs up to the end of the first, second and third axis, 8 bits each; 255: the last of them or none
};
hipError_t launch_kv4_append(const Kv4AppendArgs& a, Kv4Kind kind, int n_seq, hipStream_t s);

struct Kv4AttentionArgs {
  const uint8_t* data;        // of the layer
  const int32_t *table, *length, *slots, *starts;
  const uint16_t* q;
  uint16_t* out;
  float* partial;             // [n_seq][row tiles * n_kv_heads][splits][kv4_sums_floats] fp32
  int n_pages, max_pages, n_rows, ld_q, ld_out;
  int group;                  // query heads of a key/value head
  int window;                 // 0: none
  int chunk;                  // the split of the tokens: blocks of 32 to a workgroup, up to `splits` workgroups for a tile
  float scale_log2;           // scale * log2(e): the exponentials are powers of two
  uint32_t n_slots : 19, n_kv_heads : 13;
  uint32_t max_new : 19, page_shift : 4, tile_rows : 6;       // tile: 16 or 32 (new token, query head of the group) pairs
  uint32_t splits : 10, partial_rows : 6;      // partial_rows: rows that a tile can have
};
// Floats of one split's sums: rows of head_dim, the rows' references and totals; whole 16-byte pieces, which is how they are moved.
__host__ __device__ constexpr int kv4_sums_floats(int partial_rows, int head_dim) { return (partial_rows * (head_dim + 2) + 3) / 4 * 4; }
hipError_t launch_kv4_attention(const Kv4AttentionArgs& a, Kv4Kind kind, int n_seq, int row_tiles, hipStream_t s);
constexpr int kKv4SplitsMax = 256;            // that one row's sums are joined from

// ---- pages (kv4_pages.hip) -----------------------------------------------------------------------------
// Scratch in a workspace: two words, and from kKv4ScratchHead bytes on arrays of n_pages and of n_slots words, whose addresses a kernel
// works out itself (nine pointers would not fit a cheap launch).
constexpr size_t kKv4ScratchHead = 256;
struct Kv4Scratch {
  int32_t* base;
  __host__ __device__ int32_t* words(const larosa_kv4_cache& C, int pages, int slots) const {
    return base + kKv4ScratchHead / 4 + static_cast<size_t>(pages) * C.n_pages + static_cast<size_t>(slots) * C.n_slots;
  }
  __host__ __device__ int32_t* n_pairs() const { return base; }          // pages to copy
  __host__ __device__ int32_t* n_live() const { return base + 1; }       // compact: pages in use
  __host__ __device__ int32_t* pair_src(const larosa_kv4_cache& C) const { return words(C, 0, 0); }
  __host__ __device__ int32_t* pair_dst(const larosa_kv4_cache& C) const { return words(C, 1, 0); }
  __host__ __device__ int32_t* ids(const larosa_kv4_cache& C) const { return words(C, 2, 0); }       // grow: pages to hand out; compact: where a page moves to
  __host__ __device__ int32_t* growing(const larosa_kv4_cache& C) const { return words(C, 3, 0); }   // grow: listed slots that would write into a shared page
  __host__ __device__ int32_t* last(const larosa_kv4_cache& C) const { return words(C, 4, 0); }      // grow: the last of them, by its place in the list, from 1
  __host__ __device__ int32_t* offset(const larosa_kv4_cache& C) const { return words(C, 5, 0); }    // grow: pages handed out before those of a slot of the list
  __host__ __device__ int32_t* pair(const larosa_kv4_cache& C) const { return words(C, 5, 1); }      // grow: its pair of pages to copy, or -1
};
inline size_t kv4_scratch_bytes(const larosa_kv4_cache& C) {
  return kKv4ScratchHead + (5 * static_cast<size_t>(C.n_pages) + 2 * static_cast<size_t>(C.n_slots)) * 4;
}
hipError_t launch_kv4_grow(const larosa_kv4_cache& C, const int32_t* slots, const int32_t* counts, int n, int32_t* status, Kv4Scratch x,
                           hipStream_t s);
hipError_t launch_kv4_fork(const larosa_kv4_cache& C, const int32_t* src, const int32_t* dst, int n, int32_t* status, hipStream_t s);
hipError_t launch_kv4_trim(const larosa_kv4_cache& C, const int32_t* slots, const int32_t* keep, int n, hipStream_t s);
hipError_t launch_kv4_compact(const larosa_kv4_cache& C, int32_t* live, Kv4Scratch x, hipStream_t s);
hipError_t launch_kv4_copy_pages(const larosa_kv4_cache& C, const int32_t* src, const int32_t* dst, int n, hipStream_t s);

}  // namespace larosa
