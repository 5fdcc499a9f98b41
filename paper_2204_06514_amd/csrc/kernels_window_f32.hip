// Attention in a sliding window with sinks, fp32, on the CDNA4 matrix cores (v_mfma_f32_32x32x2_f32): as the full causal attention in
// fp32 (attn_f32_common.h).  A workgroup owns 32 rows of a key head (forward, dQ; row r is query r / group, query head r % group) or 32
// keys (dK, dV); its four wavefronts take the 32-row tiles of the other index that are seen in turn, and their results are added through LDS in wave
// order.  Long streams (single tokens over a cache; the sinks' keys, which every later query sees) are cut over workgroups and joined.
// Bound by the matrix instruction (154 TFLOP/s for a large fp32 product) where streams are long: 2 x 2048 positions, 16 heads on 4 of 128, window 512,
// sinks 4: forward 185 us (82 TFLOP/s), backward 686 us (55; seven products are formed for five); 4 x 1024, 8 heads of 64, window 256: 44 and 125 us.
#include "attn_f32_common.h"
#include "window_tiles.h"

namespace fax {

static constexpr int F32_TILE = 32;

// Rows row0 .. row0 + 31 of the packed rows, as fp32 in LDS; rows beyond the last are the last again.
template <int DH>
__device__ __forceinline__ void stage_rows(const float* base, const FaxStrides& st, int group, int rows, int row0, int dh, float* lds) {
  for (int c = threadIdx.x; c < 32 * DH / 4; c += 256) {
    const int r = min(row0 + c / (DH / 4), rows - 1), col = c % (DH / 4) * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    const int i = r / group;
    if (col < dh) v = *reinterpret_cast<const float4*>(base + (long long)i * st.row + (long long)(r - i * group) * st.head + col);
    *reinterpret_cast<float4*>(lds + c / (DH / 4) * (DH + 4) + col) = v;
  }
}

// Which of a lane's sixteen pairs (own row at position p, keys j0 + r(v, h)) are visible.
__device__ __forceinline__ unsigned seen_keys(const WindowArgs& a, int k_len, int p, int j0, int h) {
  const int last = min(p, k_len - 1), first = p - a.window;
  unsigned pairs = 0;
#pragma unroll
  for (int v = 0; v < 16; v++) {
    const int key = j0 + 8 * (v >> 2) + 4 * h + (v & 3);
    pairs |= (((key <= last) & ((key > first) | (key < a.sinks))) ? 1u : 0u) << v;
  }
  return pairs;
}

template <int DH, bool EXACT, bool PART>
__global__ __launch_bounds__(256, 2) void window_fwd_f32_kernel(WindowArgs a, int n_tiles, int items, int splits, float* __restrict__ part_o,
                                                             float2* __restrict__ part_ml) {
  extern __shared__ __attribute__((aligned(16))) float smem_a[];
  __shared__ float ms[4][32], ls[4][32];
  int item = xcd_item(blockIdx.x, gridDim.x);
  if (item >= items) return;
  int split = 0;
  if (PART) { split = item % splits; item /= splits; }
  const int bh = item / n_tiles, b = bh / a.Hkv, hk = bh % a.Hkv, row0 = item % n_tiles * 32;
  const int rows = a.Sq * a.group, dh = a.dh;
  const WindowSeq sq(a, b);
  const int lane = threadIdx.x & 63, l31 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const HeadTile<DH, EXACT> Kt{strided_row((const float*)a.k, a.skv, b, 0, hk), (int)a.skv.row, sq.k_len, dh};
  const HeadTile<DH, EXACT> Vt{strided_row((const float*)a.v, a.skv, b, 0, hk), (int)a.skv.row, sq.k_len, dh};
  stage_rows<DH>(strided_row((const float*)a.q, a.sq, b, 0, hk * a.group), a.sq, a.group, rows, row0, dh, smem_a);
  __syncthreads();
  const int p = sq.pos0 + min(row0 + l31, rows - 1) / a.group;
  const int p0 = sq.pos0 + row0 / a.group, p1 = sq.pos0 + min(row0 + 31, rows - 1) / a.group;
  const KeyTiles<F32_TILE> kt(KeyRanges(a, sq, p0, p1));
  const int u0 = PART ? (int)((long long)kt.n * split / splits) : 0, u1 = PART ? (int)((long long)kt.n * (split + 1) / splits) : kt.n;
  float m = -3.4028235e38f, l = 0.f;
  f32x16 o[DH / 32];
  zero<DH>(o);
  float4 kf[DH / 8];
  constexpr bool AHEAD = DH <= 64;  // keys one tile ahead where there are registers for them
  if (AHEAD && u0 + wave < u1) Kt.rows(kt.key(u0 + wave), lane, kf);
  for (int u = u0 + wave; u < u1; u += 4) {
    const int j0 = kt.key(u);
    float vf[16][DH / 32];
    if (!AHEAD) Kt.rows(j0, lane, kf);
    if (AHEAD) Vt.cols(j0, lane, vf);
    const f32x16 s = score_tile<DH>(kf, smem_a, lane);
    __builtin_amdgcn_sched_barrier(0);
    if (AHEAD) Kt.rows(kt.key(min(u + 4, u1 - 1)), lane, kf);
    if (!AHEAD) Vt.cols(j0, lane, vf);
    const bool whole = sees_all(a, sq.k_len, p0, p1, j0, F32_TILE);
    const unsigned pairs = whole ? 0xffffu : seen_keys(a, sq.k_len, p, j0, h);
    float e[16], top = -INFINITY;
#pragma unroll
    for (int v = 0; v < 16; v++) {
      e[v] = (pairs >> v) & 1 ? s[v] * a.scale : -INFINITY;
      top = fmaxf(top, e[v]);
    }
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float mn = fmaxf(m, top);
    if (__any(mn != m)) {
      const float corr = expf(m - mn);
      l *= corr;
#pragma unroll
      for (int i = 0; i < DH / 32; i++)
#pragma unroll
        for (int v = 0; v < 16; v++) o[i][v] *= corr;
      m = mn;
    }
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < 16; v++) {
      e[v] = (pairs >> v) & 1 ? expf(e[v] - mn) : 0.f;
      sum += e[v];
    }
    l += sum;
    add_tile<DH>(o, vf, e, !whole, pairs);
  }
  l += __shfl_xor(l, 32, 64);
  __syncthreads();  // every wave is done with the queries
  put_sums<DH>(smem_a + wave * slot_floats<DH>(), o, lane);
  if (h == 0) { ms[wave][l31] = m; ls[wave][l31] = l; }
  __syncthreads();
  for (int c = threadIdx.x; c < 32 * DH / 4; c += 256) {
    const int row = c / (DH / 4), col = c % (DH / 4) * 4, r = row0 + row;
    const float M = fmaxf(fmaxf(ms[0][row], ms[1][row]), fmaxf(ms[2][row], ms[3][row]));
    float L = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < 4; w++) {
      const float f = expf(ms[w][row] - M);
      const float4 y = *reinterpret_cast<const float4*>(smem_a + w * slot_floats<DH>() + row * (DH + 4) + col);
      L = fmaf(ls[w][row], f, L);
      x.x = fmaf(y.x, f, x.x); x.y = fmaf(y.y, f, x.y); x.z = fmaf(y.z, f, x.z); x.w = fmaf(y.w, f, x.w);
    }
    if (r >= rows) continue;
    if (PART) {
      const long long at = ((long long)bh * rows + r) * splits + split;
      if (col < dh) *reinterpret_cast<float4*>(part_o + at * dh + col) = x;
      if (col == 0) part_ml[at] = make_float2(M, L);
      continue;
    }
    const int i = r / a.group, head = hk * a.group + r - i * a.group;
    const bool none = L == 0.f;
    const float inv = none ? 0.f : 1.f / L;
    if (col < dh) *reinterpret_cast<float4*>(strided_row((float*)a.ctx, a.sc, b, i, head) + col) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
    if (col == 0 && a.lse) a.lse[((long long)b * a.H + head) * a.Sq + i] = none ? -INFINITY : M + logf(L);
  }
}

// Both halves of the backward pass in one launch, delta given: the first `kv_blocks` workgroups have keys (dK, dV), the others rows (dQ).
template <int DH, bool EXACT>
__global__ __launch_bounds__(256, DH > 64 ? 1 : 2) void window_bwd_f32_kernel(WindowArgs a, KeyGrid kg, int kv_blocks, int n_tiles, int items, int dq_splits,
                                                                           float* __restrict__ part_dq, float* __restrict__ parts) {
  extern __shared__ __attribute__((aligned(16))) float smem_a[];
  const int lane = threadIdx.x & 63, l31 = lane & 31, h = lane >> 5, dh = a.dh;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float* own_b = smem_a + slot_floats<DH>();
  float* slot = smem_a + wave * slot_floats<DH>();

  if ((int)blockIdx.x >= kv_blocks) {
    int item = xcd_item(blockIdx.x - kv_blocks, gridDim.x - kv_blocks);
    if (item >= items) return;
    const int split = item % dq_splits;
    item /= dq_splits;
    const int bh = item / n_tiles, b = bh / a.Hkv, hk = bh % a.Hkv, row0 = item % n_tiles * 32, rows = a.Sq * a.group;
    const WindowSeq sq(a, b);
    const HeadTile<DH, EXACT> Kt{strided_row((const float*)a.k, a.skv, b, 0, hk), (int)a.skv.row, sq.k_len, dh};
    const HeadTile<DH, EXACT> Vt{strided_row((const float*)a.v, a.skv, b, 0, hk), (int)a.skv.row, sq.k_len, dh};
    stage_rows<DH>(strided_row((const float*)a.q, a.sq, b, 0, hk * a.group), a.sq, a.group, rows, row0, dh, smem_a);
    stage_rows<DH>(strided_row((const float*)a.dctx, a.sc, b, 0, hk * a.group), a.sc, a.group, rows, row0, dh, own_b);
    __syncthreads();
    const int r = min(row0 + l31, rows - 1), i = r / a.group, p = sq.pos0 + i;
    const int p0 = sq.pos0 + row0 / a.group, p1 = sq.pos0 + min(row0 + 31, rows - 1) / a.group;
    const long long stat = ((long long)b * a.H + hk * a.group + r - i * a.group) * a.Sq + i;
    const float li = a.lse[stat], di = a.delta[stat];
    const KeyTiles<F32_TILE> kt(KeyRanges(a, sq, p0, p1));
    f32x16 dq[DH / 32];
    zero<DH>(dq);
    const int u1 = (int)((long long)kt.n * (split + 1) / dq_splits);
    for (int u = (int)((long long)kt.n * split / dq_splits) + wave; u < u1; u += 4) {
      const int j0 = kt.key(u);
      float4 kf[DH / 8], vf[DH / 8];
      float kc[16][DH / 32];
      Kt.rows(j0, lane, kf);
      Vt.rows(j0, lane, vf);
      const f32x16 s = score_tile<DH>(kf, smem_a, lane);
      const f32x16 dp = score_tile<DH>(vf, own_b, lane);
      __builtin_amdgcn_sched_barrier(0);
      Kt.cols(j0, lane, kc);
      const bool whole = sees_all(a, sq.k_len, p0, p1, j0, F32_TILE);
      const unsigned pairs = whole ? 0xffffu : seen_keys(a, sq.k_len, p, j0, h);
      float ds[16];
#pragma unroll
      for (int v = 0; v < 16; v++) ds[v] = (pairs >> v) & 1 ? expf(s[v] * a.scale - li) * (dp[v] - di) : 0.f;
      add_tile<DH>(dq, kc, ds, !whole, pairs);
    }
    __syncthreads();
    put_sums<DH>(slot, dq, lane);
    __syncthreads();
    for (int c = threadIdx.x; c < 32 * DH / 4; c += 256) {
      const int row = c / (DH / 4), col = c % (DH / 4) * 4, rr = row0 + row;
      if (rr >= rows || col >= dh) continue;
      float4 x = *reinterpret_cast<const float4*>(smem_a + row * (DH + 4) + col);
#pragma unroll
      for (int w = 1; w < 4; w++) {
        const float4 y = *reinterpret_cast<const float4*>(smem_a + w * slot_floats<DH>() + row * (DH + 4) + col);
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
      }
      if (dq_splits > 1) {
        *reinterpret_cast<float4*>(part_dq + (((long long)bh * rows + rr) * dq_splits + split) * dh + col) = x;
        continue;
      }
      const int ii = rr / a.group;
      *reinterpret_cast<float4*>(strided_row((float*)a.dq, a.sq, b, ii, hk * a.group + rr - ii * a.group) + col) =
          make_float4(x.x * a.scale, x.y * a.scale, x.z * a.scale, x.w * a.scale);
    }
    return;
  }

  const KeyItem it(kg, a.B * a.Hkv, blockIdx.x, kv_blocks);
  if (!it.ok) return;
  const int b = it.bh / a.Hkv, hk = it.bh % a.Hkv, k0 = it.tile * F32_TILE, keys = min(F32_TILE, a.Sk - k0);
  const WindowSeq sq(a, b);
  // (keys from k_len on have no visible pair: their rows may hold anything, but are there)
  const HeadTile<DH, EXACT> Kt{strided_row((const float*)a.k, a.skv, b, 0, hk), (int)a.skv.row, a.Sk, dh};
  const HeadTile<DH, EXACT> Vt{strided_row((const float*)a.v, a.skv, b, 0, hk), (int)a.skv.row, a.Sk, dh};
  Kt.stage(k0, smem_a);
  Vt.stage(k0, own_b);
  __syncthreads();
  f32x16 dk[DH / 32], dv[DH / 32];
  zero<DH>(dk);
  zero<DH>(dv);
  const QueryRange all(a, sq, k0, k0 + keys), mine(a, sq, min(k0 + l31, a.Sk - 1), min(k0 + l31, a.Sk - 1) + 1);
  const int i_first = all.i0 / F32_TILE * F32_TILE, per_head = all.i0 < all.i1 ? (all.i1 - i_first + F32_TILE - 1) / F32_TILE : 0, n = per_head * a.group;
  const int u0 = (int)((long long)n * it.split / it.splits), u1 = (int)((long long)n * (it.split + 1) / it.splits);
  for (int u = u0 + wave; u < u1; u += 4) {
    const int q0 = i_first + u % per_head * F32_TILE, head = hk * a.group + u / per_head;
    const HeadTile<DH, EXACT> Q{strided_row((const float*)a.q, a.sq, b, 0, head), (int)a.sq.row, a.Sq, dh};
    const HeadTile<DH, EXACT> dO{strided_row((const float*)a.dctx, a.sc, b, 0, head), (int)a.sc.row, a.Sq, dh};
    const float* lrow = a.lse + ((long long)b * a.H + head) * a.Sq;
    const float* drow = a.delta + ((long long)b * a.H + head) * a.Sq;
    float4 qf[DH / 8], of[DH / 8];
    float qc[16][DH / 32], oc[16][DH / 32];
    Q.rows(q0, lane, qf);
    dO.rows(q0, lane, of);
    float li[16], di[16];
    unsigned pairs = 0;
#pragma unroll
    for (int v = 0; v < 16; v++) {
      const int i = q0 + 8 * (v >> 2) + 4 * h + (v & 3), at = min(i, a.Sq - 1);
      li[v] = lrow[at];
      di[v] = drow[at];
      pairs |= (((i >= mine.i0) & (i < mine.i1)) ? 1u : 0u) << v;
    }
    const f32x16 s = score_tile<DH>(qf, smem_a, lane);
    const f32x16 dp = score_tile<DH>(of, own_b, lane);
    __builtin_amdgcn_sched_barrier(0);
    dO.cols(q0, lane, oc);
    Q.cols(q0, lane, qc);
    float e[16], ds[16];
#pragma unroll
    for (int v = 0; v < 16; v++) {
      const bool ok = (pairs >> v) & 1;
      e[v] = ok ? expf(s[v] * a.scale - li[v]) : 0.f;
      ds[v] = ok ? e[v] * (dp[v] - di[v]) : 0.f;
    }
    const bool masked = __any(pairs != 0xffffu);
    add_tile<DH>(dv, oc, e, masked, pairs);
    add_tile<DH>(dk, qc, ds, masked, pairs);
  }
  float* ko = strided_row((float*)a.dk, a.skv, b, k0, hk);
  float* vo = strided_row((float*)a.dv, a.skv, b, k0, hk);
  int ld = (int)a.skv.row, rows = keys;
  float mul = a.scale;
  if (it.splits > 1) {
    ko = parts + kg.part(a, it.split, it.bh, k0) * 2 * dh;
    vo = ko + dh;
    ld = 2 * dh;
    rows = F32_TILE;
    mul = 1.f;
  }
  __syncthreads();
  put_sums<DH>(slot, dk, lane);
  __syncthreads();
  store_sums<DH>(smem_a, mul, ko, ld, rows, dh);
  __syncthreads();
  put_sums<DH>(slot, dv, lane);
  __syncthreads();
  store_sums<DH>(smem_a, 1.f, vo, ld, rows, dh);
}

template <typename F>
static int by_width(int dh, F f) {
  typedef std::true_type Yes;
  typedef std::false_type No;
  if (dh == 32) return f(std::integral_constant<int, 32>{}, Yes{});
  if (dh == 64) return f(std::integral_constant<int, 64>{}, Yes{});
  if (dh == 96) return f(std::integral_constant<int, 96>{}, Yes{});
  if (dh == 128) return f(std::integral_constant<int, 128>{}, Yes{});
  if (dh < 32) return f(std::integral_constant<int, 32>{}, No{});
  if (dh < 64) return f(std::integral_constant<int, 64>{}, No{});
  if (dh < 96) return f(std::integral_constant<int, 96>{}, No{});
  return f(std::integral_constant<int, 128>{}, No{});
}

int window_fwd_f32(const WindowArgs& a, int splits, float* part_o, void* part_ml, hipStream_t s) {
  const int n_tiles = (int)(((long long)a.Sq * a.group + 31) / 32);
  const long long items = (long long)n_tiles * a.B * a.Hkv * splits;
  return by_width(a.dh, [&](auto dw, auto exact) -> int {
    constexpr int DH = decltype(dw)::value;
    constexpr bool E = decltype(exact)::value;
    auto go = [&](auto part) -> int {
      auto kern = window_fwd_f32_kernel<DH, E, decltype(part)::value>;
      constexpr int lds = 4 * slot_floats<DH>() * (int)sizeof(float);
      FAX_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
      hipLaunchKernelGGL(kern, dim3(xcd_grid(items)), dim3(256), lds, s, a, n_tiles, (int)items, splits, part_o, (float2*)part_ml);
      return FAX_OK;
    };
    return splits > 1 ? go(std::true_type{}) : go(std::false_type{});
  });
}

int window_bwd_f32(const WindowArgs& a, const WindowPlan& p, float* part_dq, float* parts, hipStream_t s) {
  const int n_tiles = (int)(((long long)a.Sq * a.group + 31) / 32), heads = a.B * a.Hkv;
  const long long items = (long long)n_tiles * heads * p.dq_splits;
  const KeyGrid kg(a, p);
  const unsigned kv_blocks = kg.blocks(a);
  return by_width(a.dh, [&](auto dw, auto exact) -> int {
    constexpr int DH = decltype(dw)::value;
    auto kern = window_bwd_f32_kernel<DH, decltype(exact)::value>;
    constexpr int lds = 4 * slot_floats<DH>() * (int)sizeof(float);
    FAX_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    hipLaunchKernelGGL(kern, dim3(kv_blocks + xcd_grid(items)), dim3(256), lds, s, a, kg, (int)kv_blocks, n_tiles, (int)items, p.dq_splits, part_dq, parts);
    return FAX_OK;
  });
}

}  // namespace fax
