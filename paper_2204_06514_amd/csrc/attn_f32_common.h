// fp32 attention on the CDNA4 matrix cores: tiles read from memory into operand registers, products of a tile, sums of the wavefronts of a
// workgroup.  Layouts (lane l, h = l >> 5): scores are computed transposed, own row = column l & 31 of the product, so that a
// lane holds, in register v, the score of its own row with row r(v, h) = 8 (v >> 2) + 4 h + (v & 3) of the other tile: the
// softmax reduces over registers plus one exchange with lane l ^ 32, and the registers are, as they stand, the B operand of
// the second product, whose v-th instruction contracts rows r(v, 0) and r(v, 1).
//   rows: operand of a score product, four consecutive features of tile row l & 31 per 16-byte load
//   cols: operand of an output product, feature l & 31 of tile rows r(v, h): 128 contiguous bytes per half-wave
// DH: head width rounded up to 32; features beyond the width are zeros in scores and are not stored.
#pragma once
#include "fax_internal.h"

namespace fax {

typedef __attribute__((ext_vector_type(16))) float f32x16;

// EXACT: the head width is DH.  Tile addresses are a scalar base plus 32-bit lane offsets.
template <int DH, bool EXACT>
struct HeadTile {
  const float* p;  // row 0, feature 0 of this head
  int ld, S, dh;

  __device__ __forceinline__ void rows(int r0, int lane, float4 (&f)[DH / 8]) const {
    const char* tile = reinterpret_cast<const char*>(p + (size_t)r0 * ld);
    const unsigned row = (unsigned)(min(lane & 31, S - 1 - r0) * ld) * 4u, h4 = 4 * (lane >> 5);
#pragma unroll
    for (int t = 0; t < DH / 8; t++) {
      const unsigned c = 8 * t + h4;
      if (EXACT) {
        f[t] = *reinterpret_cast<const float4*>(tile + (row + h4 * 4u) + 32 * t);
      } else {
        f[t] = *reinterpret_cast<const float4*>(tile + (row + min(c, (unsigned)dh - 4u) * 4u));
        if (c >= (unsigned)dh) f[t] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
    }
  }
  __device__ __forceinline__ void cols(int r0, int lane, float (&f)[16][DH / 32]) const {
    const char* tile = reinterpret_cast<const char*>(p + (size_t)r0 * ld);
#pragma unroll
    for (int v = 0; v < 16; v++) {
      const unsigned row = (unsigned)(min(8 * (v >> 2) + 4 * (lane >> 5) + (v & 3), S - 1 - r0) * ld) * 4u;
#pragma unroll
      for (int i = 0; i < DH / 32; i++) {
        if (EXACT) f[v][i] = *reinterpret_cast<const float*>(tile + (row + (lane & 31) * 4u) + 128 * i);
        else f[v][i] = *reinterpret_cast<const float*>(tile + (row + min(32 * i + (lane & 31), dh - 1) * 4u));
      }
    }
  }
  // 32 rows into LDS, whole workgroup
  __device__ __forceinline__ void stage(int r0, float* lds) const {
    for (int c = threadIdx.x; c < 32 * DH / 4; c += 256) {
      const int row = c / (DH / 4), col = c % (DH / 4) * 4;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (col < dh) v = *reinterpret_cast<const float4*>(p + (size_t)min(r0 + row, S - 1) * ld + col);
      *reinterpret_cast<float4*>(lds + row * (DH + 4) + col) = v;
    }
  }
};

template <int DH>
__device__ __forceinline__ f32x16 score_tile(const float4 (&f)[DH / 8], const float* own, int lane) {
  f32x16 s;
#pragma unroll
  for (int v = 0; v < 16; v++) s[v] = 0.f;
  const float* o = own + (lane & 31) * (DH + 4) + 4 * (lane >> 5);
#pragma unroll
  for (int t = 0; t < DH / 8; t++) {
    const float4 b = *reinterpret_cast<const float4*>(o + 8 * t);
    s = __builtin_amdgcn_mfma_f32_32x32x2f32(f[t].x, b.x, s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x2f32(f[t].y, b.y, s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x2f32(f[t].z, b.z, s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x2f32(f[t].w, b.w, s, 0, 0, 0);
  }
  return s;
}

// acc[feature][own row] += sum over the tile's rows of f * w.  `masked`: some w are zero because the pair is masked; a masked row that
// holds an infinity or NaN must not reach the sum as 0 * inf, so such elements are taken out of the product and the
// outputs whose pairs are not masked become NaN instead.
template <int DH>
__device__ __forceinline__ void add_tile(f32x16 (&acc)[DH / 32], float (&f)[16][DH / 32], const float (&w)[16], bool masked,
                                         unsigned pairs) {
  if (masked) {
    auto odd = [](float x) { return !(fabsf(x) <= 3.4028235e38f); };
    bool any = false;
#pragma unroll
    for (int v = 0; v < 16; v++)
#pragma unroll
      for (int i = 0; i < DH / 32; i++) any |= odd(f[v][i]);
    if (__any(any)) {
#pragma unroll
      for (int i = 0; i < DH / 32; i++) {
        f32x16 n;
#pragma unroll
        for (int v = 0; v < 16; v++) n[v] = 0.f;
#pragma unroll
        for (int v = 0; v < 16; v++) {
          asm volatile("" : "+v"(f[v][i]));  // tested again: the answers from above are not worth keeping in registers
          n = __builtin_amdgcn_mfma_f32_32x32x2f32(odd(f[v][i]) ? 1.f : 0.f, (pairs >> v) & 1 ? 1.f : 0.f, n, 0, 0, 0);
          f[v][i] = odd(f[v][i]) ? 0.f : f[v][i];
        }
#pragma unroll
        for (int v = 0; v < 16; v++) acc[i][v] += n[v] > 0.f ? __builtin_nanf("") : 0.f;
      }
    }
  }
#pragma unroll
  for (int v = 0; v < 16; v++)
#pragma unroll
    for (int i = 0; i < DH / 32; i++) acc[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(f[v][i], w[v], acc[i], 0, 0, 0);
}

// a wave's sums into its LDS slot, one row of DH + 4 floats per own row
template <int DH>
__device__ __forceinline__ void put_sums(float* slot, const f32x16 (&acc)[DH / 32], int lane) {
  float* o = slot + (lane & 31) * (DH + 4) + 4 * (lane >> 5);
#pragma unroll
  for (int i = 0; i < DH / 32; i++)
#pragma unroll
    for (int g = 0; g < 4; g++)
      *reinterpret_cast<float4*>(o + 32 * i + 8 * g) = make_float4(acc[i][4 * g], acc[i][4 * g + 1], acc[i][4 * g + 2], acc[i][4 * g + 3]);
}
template <int DH> static constexpr int slot_floats() { return 32 * (DH + 4); }

template <int DH>
__device__ __forceinline__ void zero(f32x16 (&acc)[DH / 32]) {
#pragma unroll
  for (int i = 0; i < DH / 32; i++)
#pragma unroll
    for (int v = 0; v < 16; v++) acc[i][v] = 0.f;
}

// the four waves' sums times `scale`, to rows of `out`
template <int DH>
__device__ __forceinline__ void store_sums(const float* slots, float scale, float* out, int ld, int rows, int dh) {
  for (int c = threadIdx.x; c < 32 * DH / 4; c += 256) {
    const int row = c / (DH / 4), col = c % (DH / 4) * 4;
    if (row >= rows || col >= dh) continue;
    float4 a = *reinterpret_cast<const float4*>(slots + row * (DH + 4) + col);
#pragma unroll
    for (int w = 1; w < 4; w++) {
      const float4 x = *reinterpret_cast<const float4*>(slots + w * slot_floats<DH>() + row * (DH + 4) + col);
      a.x += x.x; a.y += x.y; a.z += x.z; a.w += x.w;
    }
    *reinterpret_cast<float4*>(out + (size_t)row * ld + col) = make_float4(a.x * scale, a.y * scale, a.z * scale, a.w * scale);
  }
}

}  // namespace fax
