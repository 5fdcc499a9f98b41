// Attention in a sliding window with sinks on the CDNA4 matrix cores, bf16: dK and dV (window_mfma.h).  A wave has 16 keys (16x16x32 products,
// attn_dkv16.h), so that two workgroups share a CU, three up to head width 64.  (32 keys to a wave read half as much from LDS, but there are fewer, longer
// workgroups and fewer of them at once; backward pass, us with 32 | 16: 8 x 2048 positions, 12 heads of 64, window 512  188 | 167; the same, all of it
// 301 | 293; 2 x 4096, 16 heads on 4 of 64, window 1024  181 | 176; 4 x 1000, 12 heads of 48, window 300  46 | 41; 8192, 32 heads on 8 of 128, window
// 1024, where 32 keys leave one wave to a SIMD  706 | 584.)
#include "window_mfma.h"

namespace fax {

static constexpr int WPG = WINDOW_DKV_KEYS / 16;  // wavefronts of a workgroup, which share the streamed tiles: a tile for each would leave room for two on a CU

// The stream of query tiles and its loads.
template <int DH, int WAVES, bool EDGE>
struct QueryStream {
  static constexpr int NSEG = DH / 8 / WAVES, TB = TR * DH * 2, LD_OFF = 2 * TB, STAGE = 2 * TB + 4 * 256;
  const WindowArgs& a;
  int b, hk, wave, lane;
  int i_first, per_head, n;  // first query of a head's first tile; tiles of a head; of all heads
  unsigned sm;
  TileLoads<DH, WAVES, true> q, dout;
  bool in_head[NSEG];
  __device__ __forceinline__ QueryStream(const WindowArgs& a_, int b_, int hk_, const QueryRange& r, int wave_, unsigned sm_, int nch)
      : a(a_), q(wave_, a_.sq.row), dout(wave_, a_.sc.row) {
    b = b_; hk = hk_; wave = wave_; sm = sm_;
    lane = threadIdx.x & 63;
    i_first = r.i0 / TR * TR;
    per_head = r.i0 < r.i1 ? (r.i1 - i_first + TR - 1) / TR : 0;
    n = per_head * a.group;
#pragma unroll
    for (int i = 0; i < NSEG; i++) in_head[i] = !EDGE || lane_in_head<DH, WAVES, true>(wave, i, nch);
  }
  // Tile t of head g (of the key head's) into buffer `buf`: segments of Q and dO, then lse and delta (lanes 0-15 lse, 16-31 delta, the others the
  // same again).
  __device__ __forceinline__ void load(int g, int t, int buf) const {
    const int i0 = i_first + t * TR, h = hk * a.group + g, rows = a.Sq - i0;
    const unsigned st = sm + buf * STAGE;
    load_pair(q, dout, strided_row((const bf16_t*)a.q, a.sq, b, i0, h), strided_row((const bf16_t*)a.dctx, a.sc, b, i0, h), rows, st, st + TB, in_head);
    const long long stat = ((long long)b * a.H + h) * a.Sq + i0;
#pragma unroll
    for (int i = 0; i < 4 / WAVES; i++) {
      const int rb = wave * (4 / WAVES) + i;  // sixteen rows
      lds_dma4(((lane & 16) ? a.delta : a.lse) + stat + min(rb * 16 + (lane & 15), rows - 1), st + LD_OFF + rb * 256);
    }
  }
  // lse or delta of the four rows from `row` on
  __device__ __forceinline__ static float4 stat4(const char* st, int row, int which) {
    return *reinterpret_cast<const float4*>(st + LD_OFF + (row >> 4) * 256 + which * 64 + (row & 15) * 4);
  }
};

// ---------------------------------------------------------------------------------------------
// Per 32-query half: S = Q K^T and dP = dO V^T, P and dS, dV^T += dO^T P and dK^T += Q^T dS.
// ---------------------------------------------------------------------------------------------
template <int DW, bool EDGE>
__global__ __launch_bounds__(64 * WPG, DW <= 64 ? 3 : DW <= 128 ? 2 : 1) void window_dkv_mfma_kernel(WindowArgs a, KeyGrid kg, float* __restrict__ parts) {
  constexpr int DH = row_width<DW>();
  typedef QueryStream<DH, WPG, EDGE> Stream;
  constexpr int KS = DW / 32, DT = DW / 16, TB = Stream::TB;
  constexpr int N = 4 * KS, LEAD = N % 8 == 0 ? 8 : 6;
  static_assert(N == 2 * DT && N % LEAD == 0 && N > 0, "slot plan");
  constexpr int RT = 16 * WPG;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const KeyItem it_(kg, a.B * a.Hkv, blockIdx.x, gridDim.x);
  if (!it_.ok) return;
  const int b = it_.bh / a.Hkv, hk = it_.bh % a.Hkv;
  const WindowSeq sq(a, b);
  const int lane = threadIdx.x & 63, gq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hw = EDGE ? a.dh : DW, nch = hw / 8;
  const float scale = a.scale, c = scale * LOG2E;
  if (EDGE) clear_lds(smem, 2 * Stream::STAGE);
  const int j0w = it_.tile * RT + wave * 16, jk = j0w + (lane & 15);
  Stream qs(a, b, hk, QueryRange(a, sq, it_.tile * RT, min((it_.tile + 1) * RT, a.Sk)), wave, lds_addr(smem), nch);
  const int u0 = (int)((long long)qs.n * it_.split / it_.splits);
  const int u1 = (int)((long long)qs.n * (it_.split + 1) / it_.splits);

  bf16x8 kf[KS], vf[KS];
  const bool key_ok = jk < sq.k_len;
  const bf16_t* kp = strided_row((const bf16_t*)a.k, a.skv, b, min(jk, a.Sk - 1), hk);
  const bf16_t* vp = strided_row((const bf16_t*)a.v, a.skv, b, min(jk, a.Sk - 1), hk);
#pragma unroll
  for (int ks = 0; ks < KS; ks++) {
    const bool ok = key_ok && (!EDGE || ks * 4 + gq < nch);
    kf[ks] = __builtin_bit_cast(bf16x8, edge_load16(kp + ks * 32 + gq * 8, ok));
    vf[ks] = __builtin_bit_cast(bf16x8, edge_load16(vp + ks * 32 + gq * 8, ok));
  }
#pragma unroll
  for (int ks = 0; ks < KS; ks++) { settle(kf[ks]); settle(vf[ks]); }
  f32x4 dk[DT], dv[DT];
#pragma unroll
  for (int dt = 0; dt < DT; dt++)
#pragma unroll
    for (int r = 0; r < 4; r++) dk[dt][r] = dv[dt][r] = 0.f;
  const QueryRange mine(a, sq, jk, jk + 1);
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  auto tile = [&](auto mask_c, int i0, int buf) __attribute__((always_inline)) {
    constexpr bool MASK = decltype(mask_c)::value;
    int lane_t = lane;
    if (DW > 64) settle(lane_t);  // fragment addresses are formed tile by tile: kept from tile to tile they are some thirty registers
    const char* st = smem + buf * Stream::STAGE;
    auto row_frag = [&](int it, int i) { return frag_rows16<DH>(i % 2 ? st + TB : st, it * 32 + ((i / 2) / KS) * 16, (i / 2) % KS, lane_t); };
    auto col_frag = [&](int it, int i) { return frag_cols16<DH>(i % 2 ? st : st + TB, (i / 2) * 16, it * 32, lane_t); };
    bf16x8 f[LEAD];
#pragma unroll
    for (int i = 0; i < LEAD; i++) f[i] = row_frag(0, i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int it = 0; it < 2; it++) {
      f32x4 sc[2], dp[2];
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < N; i++) {
        const int qg = (i / 2) / KS, ks = (i / 2) % KS;
        if (i % 2 == 0) sc[qg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i % LEAD], kf[ks], ks == 0 ? zero : sc[qg], 0, 0, 0);
        else dp[qg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i % LEAD], vf[ks], ks == 0 ? zero : dp[qg], 0, 0, 0);
        if (i + LEAD < N) f[i % LEAD] = row_frag(it, i + LEAD);
        else f[i % LEAD] = col_frag(it, i + LEAD - N);
        __builtin_amdgcn_sched_barrier(0);
      }
      bf16x8 pb, db;  // P and dS as factors: bf16, half a step off
      __builtin_amdgcn_s_setprio(0);
#pragma unroll
      for (int qg = 0; qg < 2; qg++) {
        const int row = it * 32 + qg * 16 + gq * 4;
        const float4 l4 = Stream::stat4(st, row, 0), d4 = Stream::stat4(st, row, 1);
#pragma unroll
        for (int r = 0; r < 4; r++) {
          const int i = i0 + row + r;
          float e = __builtin_amdgcn_exp2f(fmaf(sc[qg][r], c, -LOG2E * f4_get(l4, r)));
          float d = e * (dp[qg][r] - f4_get(d4, r));
          if (MASK) {
            const bool out = (i < mine.i0) | (i >= mine.i1);
            e = out ? 0.f : e;
            d = out ? 0.f : d;
          }
          pb[qg * 4 + r] = (__bf16)e;
          db[qg * 4 + r] = (__bf16)d;
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < N; i++) {
        const int dt = i / 2;
        if (i % 2 == 0) dv[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i % LEAD], pb, dv[dt], 0, 0, 0);
        else dk[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i % LEAD], db, dk[dt], 0, 0, 0);
        if (i + LEAD < N) f[i % LEAD] = col_frag(it, i + LEAD);
        else if (it == 0) f[i % LEAD] = row_frag(1, i + LEAD - N);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
  };

  if (u0 < u1) {
    int g_at = u0 / qs.per_head, t = u0 - g_at * qs.per_head;  // head and tile of u
    qs.load(g_at, t, 0);
    lds_dma_wait();
    __syncthreads();
    // Runs of tiles with and without masks in loops of their own, as in the forward pass.
    const FullRun full = FullRun::queries(a, sq, j0w, j0w + 16 - 1, qs.i_first);
    auto any = [&](int t) __attribute__((always_inline)) {
      const int i0 = qs.i_first + t * TR, p0 = sq.pos0 + i0;
      return sees_any(a, sq.k_len, p0, p0 + min(TR, a.Sq - i0) - 1, j0w, 16);
    };
    auto next = [&](int u) __attribute__((always_inline)) {
      const bool same = t + 1 < qs.per_head;
      if (u + 1 < u1) qs.load(same ? g_at : g_at + 1, same ? t + 1 : 0, (u - u0 + 1) & 1);
    };
    auto done = [&]() __attribute__((always_inline)) {
      lds_dma_wait();
      __syncthreads();
      if (++t == qs.per_head) { t = 0; g_at++; }
    };
    for (int u = u0; u < u1;) {
      for (; u < u1 && !full.has(t); u++) {
        next(u);
        if (any(t)) tile(T_{}, qs.i_first + t * TR, (u - u0) & 1);
        done();
      }
      for (; u < u1 && full.has(t); u++) {
        next(u);
        tile(F_{}, qs.i_first + t * TR, (u - u0) & 1);
        done();
      }
    }
  }

  if (it_.splits > 1) {
    float* o = parts + kg.part(a, it_.split, it_.bh, jk) * 2 * a.dh;
#pragma unroll
    for (int dt = 0; dt < DT; dt++) {
      const int d = dt * 16 + gq * 4;
      if (EDGE && d >= hw) continue;
      *reinterpret_cast<float4*>(o + d) = make_float4(dk[dt][0], dk[dt][1], dk[dt][2], dk[dt][3]);
      *reinterpret_cast<float4*>(o + a.dh + d) = make_float4(dv[dt][0], dv[dt][1], dv[dt][2], dv[dt][3]);
    }
    return;
  }
  const bool store = jk < a.Sk;
  const unsigned long long odd = __builtin_amdgcn_ballot_w64(store && not_finite(dv, not_finite(dk, 0.f)) != 0.f);
  unsigned again = (unsigned)(odd | (odd >> 16) | (odd >> 32) | (odd >> 48)) & 0xffffu;
  if (store && !((again >> (lane & 15)) & 1)) {
    bf16_t* ko = strided_row((bf16_t*)a.dk, a.skv, b, jk, hk);
    bf16_t* vo = strided_row((bf16_t*)a.dv, a.skv, b, jk, hk);
#pragma unroll
    for (int dt = 0; dt < DT; dt++) {
      if (EDGE && dt * 16 + gq * 4 >= hw) continue;
      bf16x4 x, y;
#pragma unroll
      for (int r = 0; r < 4; r++) {
        x[r] = (__bf16)(dk[dt][r] * scale);
        y[r] = (__bf16)dv[dt][r];
      }
      *reinterpret_cast<bf16x4*>(ko + dt * 16 + gq * 4) = x;
      *reinterpret_cast<bf16x4*>(vo + dt * 16 + gq * 4) = y;
    }
  }
  for (; again; again &= again - 1) {
    int lane_r = lane;
    settle(lane_r);
    window_dkv_row<(DW + 63) / 64, bf16_t>(a, b, j0w + __builtin_ctz(again), hk, lane_r);
  }
}

int window_dkv_mfma(const WindowArgs& a, const WindowPlan& p, float* parts, hipStream_t s) {
  const KeyGrid kg(a, p);
  const unsigned grid = kg.blocks(a);
  auto launch = [&](auto kern, size_t row) -> int {
    const size_t lds = 2 * (2 * (size_t)TR * row * 2 + 4 * 256);
    FAX_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    hipLaunchKernelGGL(kern, dim3(grid), dim3(64 * WPG), lds, s, a, kg, parts);
    return FAX_OK;
  };
  if (a.dh == 64) return launch(window_dkv_mfma_kernel<64, false>, 64);
  if (a.dh == 128) return launch(window_dkv_mfma_kernel<128, false>, 128);
  if (a.dh < 64) return launch(window_dkv_mfma_kernel<64, true>, 64);
  if (a.dh <= 96) return launch(window_dkv_mfma_kernel<96, true>, 128);
  if (a.dh < 128) return launch(window_dkv_mfma_kernel<128, true>, 128);
  return launch(window_dkv_mfma_kernel<256, true>, 256);
}

}  // namespace fax
