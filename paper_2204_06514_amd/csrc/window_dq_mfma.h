// Attention in a sliding window with sinks, bf16: dQ on the matrix cores (window_mfma.h).  For two files that are compiled differently: kernels_window_mfma.hip
// and kernels_window_wide.hip.
#pragma once
#include "window_mfma.h"

namespace fax {

// ---------------------------------------------------------------------------------------------
// dQ, and delta = dctx . ctx by row.  The same tiles; per 32-key half S^T = K Q^T and dP^T = V dO^T, dS^T = P^T (dP^T - delta), dQ^T += K^T dS^T.
// ---------------------------------------------------------------------------------------------
template <int DW, bool EDGE, int G, int WPG, bool PART>
__global__ __launch_bounds__(64 * G * WPG, DW > 128 ? 1 : 2) void window_dq_mfma_kernel(WindowArgs a, int n_tiles, int items, int splits, float* __restrict__ part_dq,
                                                                     float* __restrict__ part_ds) {
  constexpr int DH = row_width<DW>();
  constexpr int KS = DW / 16, DT = DW / 32, TB = TR * DH * 2;
  constexpr int N1 = 2 * KS, N3 = 2 * DT, LEAD = N3;
  constexpr int NSEG = DH / 8 / WPG;
  static_assert(N1 % LEAD == 0, "slot plan");
  extern __shared__ __attribute__((aligned(16))) char smem_all[];
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

  bf16x8 qf[KS], dof[KS];
  const bf16_t* qp = strided_row((const bf16_t*)a.q, a.sq, b, rt.i, rt.h);
  const bf16_t* dop = strided_row((const bf16_t*)a.dctx, a.sc, b, rt.i, rt.h);
  const bf16_t* op = strided_row((const bf16_t*)a.ctx, a.sc, b, rt.i, rt.h);
  const long long stat = ((long long)b * a.H + rt.h) * a.Sq + rt.i;
  float li = rt.ok ? a.lse[stat] * LOG2E : 0.f, di = 0.f;
#pragma unroll
  for (int ks = 0; ks < KS; ks++) {
    const bool ok = rt.ok && (!EDGE || ks * 2 + g < nch);
    qf[ks] = __builtin_bit_cast(bf16x8, edge_load16(qp + ks * 16 + g * 8, ok));
    dof[ks] = __builtin_bit_cast(bf16x8, edge_load16(dop + ks * 16 + g * 8, ok));
    const bf16x8 o = __builtin_bit_cast(bf16x8, edge_load16(op + ks * 16 + g * 8, ok));
#pragma unroll
    for (int e = 0; e < 8; e++) di = fmaf((float)o[e], (float)dof[ks][e], di);
  }
  di = sum32(di);
#pragma unroll
  for (int ks = 0; ks < KS; ks++) { settle(qf[ks]); settle(dof[ks]); }
  settle(li); settle(di);
  f32x16 dq[DT];
#pragma unroll
  for (int dt = 0; dt < DT; dt++)
#pragma unroll
    for (int v = 0; v < 16; v++) dq[dt][v] = 0.f;
  float ds_sum = 0.f;

  const TileLoads<DH, WPG, false> loads(wave, a.skv.row);
  bool in_head[NSEG];
#pragma unroll
  for (int i = 0; i < NSEG; i++) in_head[i] = !EDGE || lane_in_head<DH, WPG, false>(wave, i, nch);
  auto load = [&](int j0, int buf) __attribute__((always_inline)) {
    const long long at = (long long)j0 * a.skv.row;
    load_pair(loads, loads, kb + at, vb + at, sq.k_len - j0, sm + buf * 2 * TB, sm + buf * 2 * TB + TB, in_head);
  };
  const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  const int p = rt.p, last = min(p, sq.k_len - 1), first = p - a.window;
  auto tile = [&](auto mask_c, int j0, int buf) __attribute__((always_inline)) {
    constexpr bool MASK = decltype(mask_c)::value;
    int lane_t = lane;
    if (DW > 64) settle(lane_t);  // fragment addresses are formed tile by tile: kept from tile to tile they are some thirty registers
    const char* kt_ = smem + buf * 2 * TB;
    const char* vt_ = kt_ + TB;
    auto row_frag = [&](int jt, int i) { return frag_rows<DH>((i & 1) ? vt_ : kt_, jt * 32, i / 2, lane_t); };
    auto col_frag = [&](int jt, int i) { return frag_cols<DH>(kt_, (i % DT) * 32, jt * 32 + (i / DT) * 16, lane_t); };
    bf16x8 f[LEAD];
#pragma unroll
    for (int i = 0; i < LEAD; i++) f[i] = row_frag(0, i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int jt = 0; jt < 2; jt++) {
      f32x16 sc, dp;
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < N1; i++) {
        const int ks = i / 2;
        if (i & 1) dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % LEAD], dof[ks], i < 2 ? zero : dp, 0, 0, 0);
        else sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % LEAD], qf[ks], i < 2 ? zero : sc, 0, 0, 0);
        if (i + LEAD < N1) f[i % LEAD] = row_frag(jt, i + LEAD);
        else f[i % LEAD] = col_frag(jt, i + LEAD - N1);
        __builtin_amdgcn_sched_barrier(0);
      }
      bf16x8 db[2], dl[2];  // dS as the second product's factor: two bf16 numbers, the second what the first leaves
      __builtin_amdgcn_s_setprio(0);
#pragma unroll
      for (int v = 0; v < 16; v++) {
        const float e = __builtin_amdgcn_exp2f(fmaf(sc[v], c, -li));
        float d = e * (dp[v] - di);
        const int key = j0 + jt * 32 + (v >> 2) * 8 + g * 4 + (v & 3);
        if (MASK) d = ((key > last) | ((key <= first) & (key >= a.sinks))) ? 0.f : d;
        ds_sum += d;
        dp[v] = d;
        if (v & 1) split2(dp[v - 1], d, db[v >> 3], dl[v >> 3], (v & 7) >> 1);
      }
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < 2 * N3; i++) {  // per k-step all of the first, then all of the second: products on one accumulator stand DT apart
        const int k = i / (2 * DT), n = k * DT + i % DT;
        dq[i % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[n], i / DT % 2 ? dl[k] : db[k], dq[i % DT], 0, 0, 0);
        if (jt == 0 && i / DT % 2) f[n] = row_frag(1, n);
        __builtin_amdgcn_sched_barrier(0);
      }
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
      group_put<U>(x, wave_all - WPG, 0, dq);
      reinterpret_cast<float4*>(x)[((wave_all - WPG) * U + U - 1) * 64 + lane] = make_float4(ds_sum, 0.f, 0.f, 0.f);
    }
    __syncthreads();
    if (grp) return;
#pragma unroll
    for (int o = 0; o < G - 1; o++) {
      const int slot = o * WPG + wave;
      ds_sum += reinterpret_cast<const float4*>(x)[(slot * U + U - 1) * 64 + lane].x;
      group_add<U>(x, slot, 0, dq);
    }
  }
  // The probabilities of a row add up to one, so the sum of its dS is what delta, formed from ctx as it was rounded, lacks: dK gets it with that.
  ds_sum = sum32(ds_sum);
  if (PART) {
    if (!rt.ok) return;
    const long long at = ((long long)bh * rt.rows + rt.row) * splits + split;
    if (g == 0) part_ds[at] = split == 0 ? di + ds_sum : ds_sum;
    float* o = part_dq + at * a.dh;
#pragma unroll
    for (int dt = 0; dt < DT; dt++)
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const int d = dt * 32 + q * 8 + g * 4;
        if (!EDGE || dt * 32 + q * 8 < hw) *reinterpret_cast<float4*>(o + d) = make_float4(dq[dt][q * 4], dq[dt][q * 4 + 1], dq[dt][q * 4 + 2], dq[dt][q * 4 + 3]);
      }
    return;
  }
  di += ds_sum;
  if (g == 0 && rt.ok) a.delta[stat] = di;
  const unsigned long long odd = __builtin_amdgcn_ballot_w64(rt.ok && not_finite(dq, 0.f) != 0.f);
  unsigned again = (unsigned)odd | (unsigned)(odd >> 32);
  if (rt.ok && !((again >> (lane & 31)) & 1)) store_rows<DW, EDGE>(strided_row((bf16_t*)a.dq, a.sq, b, rt.i, rt.h), dq, scale, g, hw);
  if (again) __threadfence();  // delta of this wave's rows, which window_dq_row reads
  for (; again; again &= again - 1) {
    const int src = __builtin_ctz(again);
    int lane_r = lane;
    settle(lane_r);
    window_dq_row<(DW + 63) / 64, bf16_t>(a, b, __shfl(rt.i, src, 64), __shfl(rt.h, src, 64), lane_r);
  }
}

template <typename K>
static int set_lds(K kern, size_t bytes) {
  FAX_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
  return FAX_OK;
}

template <int DW, bool E>
static int dq_launch(const WindowArgs& a, int waves, int groups, int splits, float* part_dq, float* part_ds, hipStream_t s) {
  const int n_tiles = (int)(((long long)a.Sq * a.group + 32 * waves - 1) / (32 * waves));
  const long long items = (long long)n_tiles * a.B * a.Hkv * splits;
  auto go = [&](auto g, auto wpg, auto part) -> int {
    constexpr size_t lds = decltype(g)::value * 4 * (size_t)TR * row_width<DW>() * 2;
    auto kern = window_dq_mfma_kernel<DW, E, decltype(g)::value, decltype(wpg)::value, decltype(part)::value>;
    FAX_TRY(set_lds(kern, lds));
    hipLaunchKernelGGL(kern, dim3(xcd_grid(items)), dim3(64 * groups * waves), lds, s, a, n_tiles, (int)items, splits, part_dq, part_ds);
    return FAX_OK;
  };
  if constexpr (DW <= 128)
    if (groups > 1) return go(I<2>{}, I<4>{}, F_{});
  if (splits > 1) return waves == 1 ? go(I<1>{}, I<1>{}, T_{}) : go(I<1>{}, I<4>{}, T_{});
  return waves == 1 ? go(I<1>{}, I<1>{}, F_{}) : go(I<1>{}, I<4>{}, F_{});
}

}  // namespace fax
