// Attention in a window on the matrix cores (bf16): the pieces that its kernels share.  Products, registers and LDS tiles are laid out as
// in the full causal attention (attn_mfma_common.h, attn_dkv16.h); what differs:
//   * A workgroup of the forward pass and of dQ has 32 WPG rows of a key head: row r is query r / group, query head r % group of it.  All
//     query heads of a key head share its K and V tiles, single tokens of grouped heads fill one wave's rows, and the rows of a workgroup span
//     few positions, so that few tiles reach past a window's ends.
//   * It streams the tiles of 64 keys that hold the sinks, then those that the window of some row reaches (KeyRanges).  A wave leaves out
//     those that none of its rows sees; only those that some row sees in part take the masks.
//   * Groups (G = 2): two groups of four wavefronts have the same rows and take every other tile, each with LDS buffers of its own, and add up through LDS:
//     where there is a workgroup to a CU or less, whose four wavefronts would be alone on their SIMDs.
//   * Head widths above 128 are computed at 256: accumulators and fragments take 360 to 512 registers and two stages of tiles 128 KB, one workgroup to
//     a CU.  2 x 4096 positions, 16 heads on 4 of 256, window 1024, sinks 4: forward 178 us (680 TFLOP/s), backward 655 us (460).
//   * Rows of a tile from the last key on are loads of the last key (never a read out of bounds, nothing left in LDS that was not loaded).
#pragma once
#include "attn_dkv16.h"
#include "window_tiles.h"

namespace fax {

// The same address for the whole wave, in scalar registers, whatever the compiler keeps it in.
__device__ __forceinline__ const bf16_t* uniform(const bf16_t* p) {
  const unsigned long long v = (unsigned long long)p;
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)v), hi = __builtin_amdgcn_readfirstlane((unsigned)(v >> 32));
  return (const bf16_t*)(((unsigned long long)hi << 32) | lo);
}

// Loads of a wave's share of a 64-row tile, 1 KB segments of RPI rows.  A lane's 16 bytes of segment i lie at its row (lane / NCH, from the segment's
// first) and at the chunk that the swizzle puts there.  The swizzles repeat after 16 rows, so the byte offsets of OFFS segments are kept, and the others'
// are theirs from a base further down.  Of a tile with fewer than 64 rows (at least one) the last row is loaded again; which of the two it is, is asked once
// for all segments (with a branch for each, 8192 of 32 on 8 x 128, window 1024: forward 168 us against 158, backward 632 against 582).
template <int DH, int WAVES, bool SWZ16>
struct TileLoads {
  static constexpr int NCH = DH / 8, RPI = 64 / NCH, NSEG = DH / 8 / WAVES, OFFS = NSEG * RPI <= 16 ? NSEG : 16 / RPI;
  unsigned off[OFFS];
  int wave, ld;
  __device__ __forceinline__ static int chunk_of(int row) {
    return ((threadIdx.x & 63) % NCH) ^ (SWZ16 ? swz16<DH>(row) : swz<DH>(row));
  }
  __device__ __forceinline__ TileLoads(int wave_, long long ld_) {
    wave = wave_;
    ld = (int)ld_;
#pragma unroll
    for (int i = 0; i < OFFS; i++) {
      const int row = (wave * NSEG + i) * RPI + (threadIdx.x & 63) / NCH;
      off[i] = (unsigned)(row * ld) * 2u + chunk_of(row) * 16u;
    }
  }
  // segment i of a whole tile; of one with `rows` rows
  __device__ __forceinline__ void whole(const bf16_t* tile, unsigned lds_tile, int i) const {
    lds_dma16(uniform(tile + (long long)(i / OFFS * OFFS * RPI) * ld), off[i % OFFS], __builtin_amdgcn_readfirstlane(lds_tile + (wave * NSEG + i) * 1024u));
  }
  __device__ __forceinline__ void ragged(const bf16_t* tile, int rows, unsigned lds_tile, int i) const {
    const int row = (wave * NSEG + i) * RPI + (threadIdx.x & 63) / NCH;
    lds_dma16(uniform(tile), (unsigned)(min(row, rows - 1) * ld) * 2u + chunk_of(row) * 16u, __builtin_amdgcn_readfirstlane(lds_tile + (wave * NSEG + i) * 1024u));
  }
};
// Segments of a pair of tiles (K and V; Q and dO) of `rows` rows.
template <int NSEG, typename LoadsA, typename LoadsB>
__device__ __forceinline__ void load_pair(const LoadsA& x, const LoadsB& y, const bf16_t* tx, const bf16_t* ty, int rows, unsigned lds_x, unsigned lds_y,
                                          const bool (&in_head)[NSEG]) {
  if (rows >= TR) {
#pragma unroll
    for (int i = 0; i < NSEG; i++)
      if (in_head[i]) {
        x.whole(tx, lds_x, i);
        y.whole(ty, lds_y, i);
      }
  } else {
#pragma unroll
    for (int i = 0; i < NSEG; i++)
      if (in_head[i]) {
        x.ragged(tx, rows, lds_x, i);
        y.ragged(ty, rows, lds_y, i);
      }
  }
}
// Whether this lane's chunk of segment i lies within the head (masked-edge form).
template <int DH, int WAVES, bool SWZ16>
__device__ __forceinline__ bool lane_in_head(int wave, int i, int chunks) {
  constexpr int NCH = DH / 8, RPI = 64 / NCH, NSEG = DH / 8 / WAVES;
  const int lane = threadIdx.x & 63;
  const int row = (wave * NSEG + i) * RPI + lane / NCH;
  return ((lane % NCH) ^ (SWZ16 ? swz16<DH>(row) : swz<DH>(row))) < chunks;
}

// x and y as bf16 pairs: elements 2 n and 2 n + 1 of hi cut off (not rounded), of lo what that leaves, rounded: 2^-16 off each instead of 2^-8.
__device__ __forceinline__ void split2(float x, float y, bf16x8& hi, bf16x8& lo, int n) {
  typedef __attribute__((ext_vector_type(4))) unsigned u4;
  const unsigned a = __float_as_uint(x), b = __float_as_uint(y);
  u4 h = __builtin_bit_cast(u4, hi);
  h[n] = __builtin_amdgcn_perm(b, a, 0x07060302u);  // upper halves
  hi = __builtin_bit_cast(bf16x8, h);
  lo[2 * n] = (__bf16)(x - __uint_as_float(a & 0xffff0000u));
  lo[2 * n + 1] = (__bf16)(y - __uint_as_float(b & 0xffff0000u));
}

// Which tiles of a stream need no masks: a run of them.
struct FullRun {
  int first;
  unsigned count;
  __device__ __forceinline__ bool has(int u) const { return (unsigned)(u - first) < count; }
  // Keys for rows at p0 .. p1 (by position; tiles of sinks that the window does not reach take the masks even where all of them are seen).
  __device__ __forceinline__ static FullRun keys(const WindowArgs& a, int k_len, int p0, int p1, const KeyTiles<TR>& kt) {
    const int from = max(0, p1 - a.window + 1), to = min(p0 + 1, k_len);  // every row sees [from, to)
    const int t0 = (from + TR - 1) / TR, t1 = to / TR;
    FullRun r;
    r.first = t0 >= kt.sink_tiles ? t0 - kt.skip : t0;
    r.count = (unsigned)max(0, t1 - t0);
    return r;
  }
  // Queries, counted in tiles from i_first, that see all of the keys j0 .. j1.
  __device__ __forceinline__ static FullRun queries(const WindowArgs& a, const WindowSeq& s, int j0, int j1, int i_first) {
    const long long from = max(0, j1 - s.pos0), to = j1 < a.sinks ? a.Sq : min((long long)a.Sq, (long long)j0 + a.window - s.pos0);  // [from, to)
    const int t0 = (int)((max((long long)0, from - i_first) + TR - 1) / TR), t1 = (int)((to - i_first) / TR);
    FullRun r;
    r.first = t0;
    r.count = j1 < s.k_len && to > i_first ? (unsigned)max(0, t1 - t0) : 0u;
    return r;
  }
};

// The rows that a workgroup of the forward pass or of dQ has, and what it streams for them.
template <int WPG>
struct RowTile {
  int b, hk, r0, rows;       // key head; first row of the workgroup, rows of the key head
  int wave, row, i, h, p;    // this lane's row: query, query head, position
  bool ok;                   // there is such a row
  int p0, p1, wp0, wp1;      // positions of the workgroup's rows, of the wave's
  __device__ __forceinline__ RowTile(const WindowArgs& a, const WindowSeq& s, int b_, int hk_, int tile, int wave_) {
    b = b_; hk = hk_;
    rows = a.Sq * a.group;
    r0 = tile * (32 * WPG);
    wave = wave_;
    const int w0 = r0 + wave * 32;
    row = w0 + (threadIdx.x & 31);
    ok = row < rows;
    const int r = min(row, rows - 1);
    i = r / a.group;
    h = hk * a.group + r - i * a.group;
    p = s.pos0 + i;
    p0 = s.pos0 + r0 / a.group;
    p1 = s.pos0 + min(r0 + 32 * WPG - 1, rows - 1) / a.group;
    wp0 = s.pos0 + min(w0, rows - 1) / a.group;
    wp1 = w0 < rows ? s.pos0 + min(w0 + 31, rows - 1) / a.group : -2147483647 - 1;  // (a wave without rows sees nothing)
  }
};

}  // namespace fax
