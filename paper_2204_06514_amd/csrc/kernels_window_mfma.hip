// Attention in a sliding window with sinks on the CDNA4 matrix cores, bf16: forward pass and dQ (window_mfma.h).
#include "window_dq_mfma.h"

namespace fax {

// ---------------------------------------------------------------------------------------------
// Forward.  Wave w owns rows 32 w .. + 31 of the workgroup's (B operand, in registers); 64-key tiles of K and V stream through two
// LDS buffers: S^T for both 32-key halves, online softmax over the 64 keys, O^T += V^T P^T.
// PART: the workgroup has one of `splits` runs of the tiles and leaves its sums, undivided, with their reference point (in units of the
// unscaled score) and their denominators, for window_join_kernel.
// ---------------------------------------------------------------------------------------------
template <int DW, bool EDGE, int G, int WPG, bool PART>
__global__ __launch_bounds__(64 * G * WPG, DW > 128 ? 1 : 2) void window_fwd_mfma_kernel(WindowArgs a, int n_tiles, int items, int splits, float* __restrict__ part_o,
                                                                      float2* __restrict__ part_ml) {
  constexpr int DH = row_width<DW>();  // row length in LDS
  constexpr int KS = DW / 16, DT = DW / 32, TB = TR * DH * 2;
  constexpr int N = 2 * KS;            // MFMAs per phase
  constexpr int LEAD = N < 8 ? N : 8;  // fragments in flight
  constexpr int NSEG = DH / 8 / WPG;   // 1 KB load instructions per wave per tile
  extern __shared__ __attribute__((aligned(16))) char smem_all[];  // to a group 2 x [K tile | V tile]
  int item = xcd_item(blockIdx.x, gridDim.x);
  if (item >= items) return;
  int split = 0;
  if (PART) { split = item % splits; item /= splits; }
  const int tile_no = item % n_tiles, bh = item / n_tiles;
  const int b = bh / a.Hkv, hk = bh % a.Hkv;
  const WindowSeq sq(a, b);
  const int wave_all = G * WPG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int grp = G == 1 ? 0 : wave_all / WPG, wave = G == 1 ? wave_all : wave_all % WPG;
  const RowTile<WPG> rt(a, sq, b, hk, tile_no, wave);
  char* const smem = smem_all + grp * (4 * TB);
  const int lane = threadIdx.x & 63, g = lane >> 5;
  const int hw = EDGE ? a.dh : DW, nch = hw / 8;
  const bf16_t* kb = strided_row((const bf16_t*)a.k, a.skv, b, 0, hk);
  const bf16_t* vb = strided_row((const bf16_t*)a.v, a.skv, b, 0, hk);
  const float scale = a.scale, c = scale * LOG2E;
  const unsigned sm = lds_addr(smem);
  if (EDGE) clear_lds(smem_all, G * 4 * TB);

  const KeyTiles<TR> kt(KeyRanges(a, sq, rt.p0, rt.p1));
  const int u0 = PART ? (int)((long long)kt.n * split / splits) : 0, u1 = PART ? (int)((long long)kt.n * (split + 1) / splits) : kt.n;

  bf16x8 qf[KS];
  const bf16_t* qp = strided_row((const bf16_t*)a.q, a.sq, b, rt.i, rt.h);
#pragma unroll
  for (int ks = 0; ks < KS; ks++) qf[ks] = __builtin_bit_cast(bf16x8, edge_load16(qp + ks * 16 + g * 8, rt.ok && (!EDGE || ks * 2 + g < nch)));
#pragma unroll
  for (int ks = 0; ks < KS; ks++) settle(qf[ks]);
  float m = -3.4028235e38f, l = 0.f;  // (a row may not see a key for a while, or at all)
  f32x16 oacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; dt++)
#pragma unroll
    for (int v = 0; v < 16; v++) oacc[dt][v] = 0.f;

  const TileLoads<DH, WPG, false> loads(wave, a.skv.row);
  bool in_head[NSEG];
#pragma unroll
  for (int i = 0; i < NSEG; i++) in_head[i] = !EDGE || lane_in_head<DH, WPG, false>(wave, i, nch);
  auto load = [&](int j0, int buf) __attribute__((always_inline)) {
    const long long at = (long long)j0 * a.skv.row;
    load_pair(loads, loads, kb + at, vb + at, sq.k_len - j0, sm + buf * 2 * TB, sm + buf * 2 * TB + TB, in_head);
  };
  const int p = rt.p, last = min(p, sq.k_len - 1), first = p - a.window;  // sees keys in (first, last] and the sinks up to last
  auto tile = [&](auto mask_c, int j0, int buf) __attribute__((always_inline)) {
    constexpr bool MASK = decltype(mask_c)::value;
    int lane_t = lane;
    if (DW > 64) settle(lane_t);  // fragment addresses are formed tile by tile: kept from tile to tile they are some thirty registers
    const char* kt_ = smem + buf * 2 * TB;
    const char* vt_ = kt_ + TB;
    auto row_frag = [&](int i) { return frag_rows<DH>(kt_, (i % 2) * 32, i / 2, lane_t); };
    auto col_frag = [&](int i) { return frag_cols<DH>(vt_, (i % DT) * 32, ((i / DT) % 2) * 32 + ((i / DT) / 2) * 16, lane_t); };
    bf16x8 fr[LEAD], fc[LEAD];
#pragma unroll
    for (int i = 0; i < LEAD; i++) fr[i] = row_frag(i);
    f32x16 s[2];
#pragma unroll
    for (int jt = 0; jt < 2; jt++)
#pragma unroll
      for (int v = 0; v < 16; v++) s[jt][v] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < N; i++) {
      s[i % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[i % LEAD], qf[i / 2], s[i % 2], 0, 0, 0);
      if (i + LEAD < N) fr[i % LEAD] = row_frag(i + LEAD);
      else fc[i + LEAD - N] = col_frag(i + LEAD - N);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    if (MASK) {
#pragma unroll
      for (int jt = 0; jt < 2; jt++)
#pragma unroll
        for (int v = 0; v < 16; v++) {
          const int key = j0 + jt * 32 + (v >> 2) * 8 + g * 4 + (v & 3);
          s[jt][v] = ((key > last) | ((key <= first) & (key >= a.sinks))) ? -INFINITY : s[jt][v];
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int jt = 0; jt < 2; jt++)
#pragma unroll
      for (int v = 0; v < 16; v++) mx = fmaxf(mx, s[jt][v]);
    mx = max32(mx);
    // the reference point follows the running maximum lazily (at most 2^MAX_LAG above it)
    const float mn = fmaxf(m, mx);
    if (__builtin_amdgcn_ballot_w64((mn - m) * c > MAX_LAG) != 0) {
      const float corr = __builtin_amdgcn_exp2f((m - mn) * c);
      l *= corr;
#pragma unroll
      for (int dt = 0; dt < DT; dt++)
#pragma unroll
        for (int v = 0; v < 16; v++) oacc[dt][v] *= corr;
      m = mn;
    }
    const float mc = m * c;
    float rs = 0.f;
    // Probabilities as the second product's factors: bf16, half a step (2^-8) off each (the denominator adds them unrounded), which leaves ctx 1.4 times as
    // far off as its own rounding.  PART, bound by memory: two bf16 numbers, and ctx as good as its rounding.
    bf16x8 pb[2][2], pl[2][2];
#pragma unroll
    for (int jt = 0; jt < 2; jt++)
#pragma unroll
      for (int v = 0; v < 16; v++) {
        const float e = __builtin_amdgcn_exp2f(fmaf(s[jt][v], c, -mc));
        rs += e;
        if (PART) {
          s[jt][v] = e;
          if (v & 1) split2(s[jt][v - 1], e, pb[jt][v >> 3], pl[jt][v >> 3], (v & 7) >> 1);
        } else {
          pb[jt][v >> 3][v & 7] = (__bf16)e;
        }
      }
    l += sum32(rs);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int dt = i % DT, ch = i / DT;
      oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fc[i % LEAD], pb[ch % 2][ch / 2], oacc[dt], 0, 0, 0);
      if (PART) oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fc[i % LEAD], pl[ch % 2][ch / 2], oacc[dt], 0, 0, 0);
      if (i + LEAD < N) fc[i % LEAD] = col_frag(i + LEAD);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
  };

  // (a group without a tile of its own loads the last, and meets the others' barriers)
  if (u0 < u1) {
    load(kt.key(min(u0 + grp, u1 - 1)), 0);
    lds_dma_wait();
    __syncthreads();
    // Runs of tiles that take the masks (or that no row of the wave sees) and of tiles that do not, in loops of their own: one loop over both kinds
    // keeps the accumulators in two places, which does not fit the registers.
    const FullRun full = FullRun::keys(a, sq.k_len, rt.wp0, rt.wp1, kt);
    auto next = [&](int u) __attribute__((always_inline)) {
      if (u + G < u1) load(kt.key(u + G), ((u - u0) / G + 1) & 1);
    };
    auto done = [&]() {
      lds_dma_wait();
      __syncthreads();
    };
    for (int u = u0 + grp; u < u1;) {
      for (; u < u1 && !full.has(u); u += G) {
        next(u);
        if (sees_any(a, sq.k_len, rt.wp0, rt.wp1, kt.key(u), TR)) tile(T_{}, kt.key(u), (u - u0) / G & 1);
        done();
      }
      for (; u < u1 && full.has(u); u += G) {
        next(u);
        tile(F_{}, kt.key(u), (u - u0) / G & 1);
        done();
      }
    }
    if (G > 1)  // every group meets as many barriers as the one with the most tiles
      for (int k = (u1 - u0 + G - 1) / G - (u1 - u0 - grp + G - 1) / G; k > 0; k--) __syncthreads();
  }

  if (G > 1) {
    constexpr int U = DT * 4 + 1;
    float* x = reinterpret_cast<float*>(smem_all);
    if (grp) {
      group_put<U>(x, wave_all - WPG, 0, oacc);
      reinterpret_cast<float4*>(x)[((wave_all - WPG) * U + U - 1) * 64 + lane] = make_float4(m, l, 0.f, 0.f);
    }
    __syncthreads();
    if (grp) return;
#pragma unroll
    for (int o = 0; o < G - 1; o++) {
      const int slot = o * WPG + wave;
      const float4 ml = reinterpret_cast<const float4*>(x)[(slot * U + U - 1) * 64 + lane];
      const float mn = fmaxf(m, ml.x);
      const float a0 = __builtin_amdgcn_exp2f((m - mn) * c), a1 = __builtin_amdgcn_exp2f((ml.x - mn) * c);
      l = fmaf(l, a0, ml.y * a1);
      m = mn;
      group_add<U>(x, slot, 0, oacc, a0, a1);
    }
  }

  const long long row_all = (long long)bh * rt.rows + rt.row;
  if (PART) {
    if (!rt.ok) return;
    const long long at = row_all * splits + split;
    if (g == 0) part_ml[at] = make_float2(m, l);
    float* o = part_o + at * a.dh;
#pragma unroll
    for (int dt = 0; dt < DT; dt++)
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const int d = dt * 32 + q * 8 + g * 4;
        if (!EDGE || dt * 32 + q * 8 < hw) *reinterpret_cast<float4*>(o + d) = make_float4(oacc[dt][q * 4], oacc[dt][q * 4 + 1], oacc[dt][q * 4 + 2], oacc[dt][q * 4 + 3]);
      }
    return;
  }
  const unsigned long long odd = __builtin_amdgcn_ballot_w64(rt.ok && not_finite(oacc, l * 0.f) != 0.f);
  unsigned again = (unsigned)odd | (unsigned)(odd >> 32);
  if (rt.ok && !((again >> (lane & 31)) & 1)) {
    const bool none = l == 0.f;
    store_rows<DW, EDGE>(strided_row((bf16_t*)a.ctx, a.sc, b, rt.i, rt.h), oacc, none ? 0.f : 1.f / l, g, hw);
    if (g == 0 && a.lse) a.lse[((long long)b * a.H + rt.h) * a.Sq + rt.i] = none ? -INFINITY : m * scale + logf(l);
  }
  for (; again; again &= again - 1) {
    const int src = __builtin_ctz(again);
    int lane_r = lane;
    settle(lane_r);
    window_fwd_row<(DW + 63) / 64, bf16_t>(a, b, __shfl(rt.i, src, 64), __shfl(rt.h, src, 64), lane_r);
  }
}

// f(head width as computed, masked edges)
template <typename F>
static int by_width(int dh, F f) {
  if (dh == 64) return f(I<64>{}, F_{});
  if (dh == 128) return f(I<128>{}, F_{});
  return dh < 64 ? f(I<64>{}, T_{}) : dh <= 96 ? f(I<96>{}, T_{}) : dh < 128 ? f(I<128>{}, T_{}) : f(I<256>{}, T_{});
}

int window_fwd_mfma(const WindowArgs& a, int waves, int groups, int splits, float* part_o, void* part_ml, hipStream_t s) {
  const int n_tiles = (int)(((long long)a.Sq * a.group + 32 * waves - 1) / (32 * waves));
  const long long items = (long long)n_tiles * a.B * a.Hkv * splits;
  return by_width(a.dh, [&](auto dw, auto edge) -> int {
    constexpr int DW = decltype(dw)::value;
    constexpr bool E = decltype(edge)::value;
    auto go = [&](auto g, auto wpg, auto part) -> int {
      constexpr size_t lds = decltype(g)::value * 4 * (size_t)TR * row_width<DW>() * 2;
      auto kern = window_fwd_mfma_kernel<DW, E, decltype(g)::value, decltype(wpg)::value, decltype(part)::value>;
      FAX_TRY(set_lds(kern, lds));
      hipLaunchKernelGGL(kern, dim3(xcd_grid(items)), dim3(64 * groups * waves), lds, s, a, n_tiles, (int)items, splits, part_o, (float2*)part_ml);
      return FAX_OK;
    };
    if constexpr (DW <= 128)
      if (groups > 1) return go(I<2>{}, I<4>{}, F_{});
    if (splits > 1) return waves == 1 ? go(I<1>{}, I<1>{}, T_{}) : go(I<1>{}, I<4>{}, T_{});
    return waves == 1 ? go(I<1>{}, I<1>{}, F_{}) : go(I<1>{}, I<4>{}, F_{});
  });
}

int window_dq_mfma(const WindowArgs& a, int waves, int groups, int splits, float* part_dq, float* part_ds, hipStream_t s) {
  if (a.dh > 128) return window_dq_wide(a, waves, splits, part_dq, part_ds, s);
  auto go = [&](auto dw, auto edge) -> int { return dq_launch<decltype(dw)::value, decltype(edge)::value>(a, waves, groups, splits, part_dq, part_ds, s); };
  if (a.dh == 64) return go(I<64>{}, F_{});
  if (a.dh == 128) return go(I<128>{}, F_{});
  return a.dh < 64 ? go(I<64>{}, T_{}) : a.dh <= 96 ? go(I<96>{}, T_{}) : go(I<128>{}, T_{});
}

}  // namespace fax
