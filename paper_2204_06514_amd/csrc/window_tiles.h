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
// them, head by head.  The streams of the first `cut_tiles` tiles are cut into `splits` parts, workgroups of their own that leave sums for
// window_fold_kernel: those of the sinks, which every later query sees and not a window's length of them, or of all, where tiles are few.
// They are the first workgroups of the launch; the other tiles follow.
struct KeyGrid {
  int n_tiles, cut_tiles, splits, cut_blocks;  // key tiles of a head; how many of them are cut, into how many parts; workgroups of those
  KeyGrid(const WindowArgs& a, int keys, int cut_tiles_, int splits_) {
    n_tiles = (a.Sk + keys - 1) / keys;
    cut_tiles = splits_ > 1 ? cut_tiles_ : 0;
    splits = splits_;
    cut_blocks = (int)xcd_grid((long long)cut_tiles * a.B * a.Hkv * splits);
  }
  unsigned blocks(int heads) const { return cut_blocks + xcd_grid((long long)(n_tiles - cut_tiles) * heads); }
};
struct KeyItem {
  int bh, tile, split;  // split < 0: whole
  bool ok;
  __device__ __forceinline__ KeyItem(const KeyGrid& k, int heads, int block, int grid) {
    if (block < k.cut_blocks) {
      split = block % k.splits;
      const int r = block / k.splits;
      tile = r % max(k.cut_tiles, 1);
      bh = r / max(k.cut_tiles, 1);
      ok = bh < heads;
    } else {
      const int rest = k.n_tiles - k.cut_tiles, i = xcd_item(block - k.cut_blocks, grid - k.cut_blocks);
      split = -1;
      ok = i < rest * heads;
      tile = k.cut_tiles + i % max(rest, 1);
      bh = i / max(rest, 1);
    }
  }
};

// A part's row of scratch: [part, head, key of the cut tiles, dK | dV, feature].
__device__ __forceinline__ float* part_row(const WindowArgs& a, const KeyGrid& k, float* parts, int split, int bh, int keys, int j) {
  return parts + ((((long long)split * a.B * a.Hkv + bh) * keys + j) * 2) * a.dh;
}

}  // namespace fax
