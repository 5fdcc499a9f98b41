// Attention in a window: how its matrix-core kernels, of either type, deal tiles to workgroups.
#pragma once
#include "attn_window.h"

namespace fax {

// Workgroup -> item, with neighbouring items on one XCD (workgroups go to the eight XCDs in turn): they share K and V tiles, or Q and dO, in
// its L2.  The grid is xcd_grid(items); items that are none are out of range.
inline unsigned xcd_grid(long long items) { return (unsigned)((items + 7) / 8 * 8); }
__device__ __forceinline__ int xcd_item(int block, int grid) { return (block & 7) * (grid >> 3) + (block >> 3); }

// Tiles of T keys of a run of queries, in order: those of the sinks, then those of the window.
template <int T>
struct KeyTiles {
  int sink_tiles, skip, n;
  __device__ __forceinline__ KeyTiles(const KeyRanges& k) {
    sink_tiles = (k.sink_end + T - 1) / T;
    const int first = max(sink_tiles, k.lo / T);
    skip = first - sink_tiles;
    n = sink_tiles + (k.lo < k.end ? max(0, (k.end + T - 1) / T - first) : 0);
  }
  __device__ __forceinline__ int key(int u) const { return (u < sink_tiles ? u : u + skip) * T; }
};

// Whether queries at p0 .. p1 see all of, or anything of, the keys j0 .. j0 + width - 1.
__device__ __forceinline__ bool sees_all(const WindowArgs& a, int k_len, int p0, int p1, int j0, int width) {
  const int last = j0 + width - 1;
  return last < k_len && last <= p0 && (j0 > p1 - a.window || last < a.sinks);
}
__device__ __forceinline__ bool sees_any(const WindowArgs& a, int k_len, int p0, int p1, int j0, int width) {
  return j0 < k_len && j0 <= p1 && (j0 + width - 1 > p0 - a.window || j0 < a.sinks);
}

// dK and dV.  A workgroup has a tile of keys of one key head and streams the tiles of queries of all its query heads that see some of
// them, head by head.  A stream may be cut into parts, workgroups of their own that leave sums for window_fold_kernel: `sink_splits` of the tiles with
// sinks, which every later query sees, `rest_splits` of the others.  The sinks' workgroups are the first of the launch.
struct KeyGrid {
  int keys, n_tiles, sink_tiles, sink_splits, rest_splits, sink_blocks;
  KeyGrid(const WindowArgs& a, const WindowPlan& p) {
    keys = p.kv_keys;
    n_tiles = (a.Sk + keys - 1) / keys;
    sink_tiles = p.sink_tiles;
    sink_splits = p.sink_splits;
    rest_splits = p.rest_splits;
    sink_blocks = (int)xcd_grid((long long)sink_tiles * a.B * a.Hkv * sink_splits);
  }
  unsigned blocks(const WindowArgs& a) const { return sink_blocks + xcd_grid((long long)(n_tiles - sink_tiles) * a.B * a.Hkv * rest_splits); }
  // Rows of scratch (dK and dV of a key in a part): the sinks' parts [part, key head, key], then the others'.
  __host__ __device__ __forceinline__ long long sink_rows(const WindowArgs& a) const { return sink_splits > 1 ? (long long)sink_splits * a.B * a.Hkv * sink_tiles * keys : 0; }
  long long part_rows(const WindowArgs& a) const {
    return sink_rows(a) + (rest_splits > 1 ? (long long)rest_splits * a.B * a.Hkv * (n_tiles - sink_tiles) * keys : 0);
  }
  __device__ __forceinline__ long long part(const WindowArgs& a, int split, int bh, int j) const {
    const int first = sink_tiles * keys;
    if (j < first) return ((long long)split * a.B * a.Hkv + bh) * first + j;
    return sink_rows(a) + ((long long)split * a.B * a.Hkv + bh) * ((n_tiles - sink_tiles) * keys) + j - first;
  }
  // the keys whose parts are added up: [fold_from, fold_from + fold_keys)
  __host__ __device__ __forceinline__ int fold_from() const { return sink_splits > 1 ? 0 : sink_tiles * keys; }
  __host__ __device__ __forceinline__ int fold_keys(const WindowArgs& a) const {
    const int end = rest_splits > 1 ? a.Sk : sink_tiles * keys;
    return (end < a.Sk ? end : a.Sk) - fold_from();
  }
};
struct KeyItem {
  int bh, tile, split, splits;  // splits 1: whole
  bool ok;
  __device__ __forceinline__ KeyItem(const KeyGrid& k, int heads, int block, int grid) {
    const bool sinks = block < k.sink_blocks;
    const int tiles = max(sinks ? k.sink_tiles : k.n_tiles - k.sink_tiles, 1);
    int i = sinks ? block : xcd_item(block - k.sink_blocks, grid - k.sink_blocks);
    splits = sinks ? k.sink_splits : k.rest_splits;
    split = i % splits;
    i /= splits;
    bh = i / tiles;
    tile = (sinks ? 0 : k.sink_tiles) + i % tiles;
    ok = bh < heads && tile < k.n_tiles;
  }
};

}  // namespace fax
