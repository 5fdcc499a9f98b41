// fp32 causal attention on the CDNA4 matrix cores: v_mfma_f32_32x32x2_f32 for every product, fp32 exponentials and
// sums as in the scalar kernels, which keep the head widths these do not cover (over 128, no multiple of 4).
//
// A workgroup owns 32 queries of one head (forward, dQ) or 32 keys (dK, dV); its four wavefronts take the 32-row tiles
// of the other index in turn (w, w + 4, ...) and their results are combined through LDS in wave order at the end.  So there are
// B H S / 32 workgroups of four waves -- a short sequence of few heads still reaches many CUs -- no barrier inside
// the loop and one writer per output.  The instruction needs 64 clocks for two operand registers, so the tiles are
// read straight from memory (L2 for all but the first reader of a head) into operand registers: 16 KB per 4096 clocks of
// products and wave at head width 64.  Only the workgroup's own rows are kept in LDS.
// Layouts, tiles and products: attn_f32_common.h.
#include "attn_f32_common.h"

namespace fax {

// Bound by the matrix cores and, with few tiles per wave, by the latency of the first loads.  B 4, S 512, 16 heads of 64: 567 us
// on the scalar kernel, 40 here (53 TFLOP/s at the causal half; the matrix cores give 155 in fp32); 1 x 2000 with 4 heads of
// 128: 1207 -> 96.
template <int DH, bool EXACT>
__global__ __launch_bounds__(256, 2) void attn_fwd_f32_kernel(int S, int H, int dh, int BH, const float* __restrict__ qkv,
                                                           float* __restrict__ ctx, float* __restrict__ lse) {
  extern __shared__ __attribute__((aligned(16))) float smem_a[];
  __shared__ float ms[4][32], ls[4][32];
  const int lane = threadIdx.x & 63, l31 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qt = (S + 31) / 32 - 1 - blockIdx.x / BH, bh = blockIdx.x % BH;  // long rows of tiles first
  const int Hd = H * dh, ld = 3 * Hd, q0 = qt * 32;
  const float* base = qkv + (size_t)(bh / H) * S * ld + (bh % H) * dh;
  const HeadTile<DH, EXACT> Q{base, ld, S, dh}, Kt{base + Hd, ld, S, dh}, Vt{base + 2 * Hd, ld, S, dh};
  Q.stage(q0, smem_a);
  __syncthreads();
  const float scale = rsqrtf((float)dh);
  float m = -INFINITY, l = 0.f;
  f32x16 o[DH / 32];
  zero<DH>(o);
  float4 kf[DH / 8];
  // keys one tile ahead where there are registers for them
  constexpr bool AHEAD = DH <= 64;
  if (AHEAD && wave <= qt) Kt.rows(wave * 32, lane, kf);
  for (int kt = wave; kt <= qt; kt += 4) {
    float vf[16][DH / 32];
    if (!AHEAD) Kt.rows(kt * 32, lane, kf);
    if (AHEAD) Vt.cols(kt * 32, lane, vf);
    const f32x16 s = score_tile<DH>(kf, smem_a, lane);
    __builtin_amdgcn_sched_barrier(0);
    if (AHEAD) Kt.rows(min(kt + 4, qt) * 32, lane, kf);
    if (!AHEAD) Vt.cols(kt * 32, lane, vf);
    unsigned pairs = 0xffff;
    if (kt == qt) {
      pairs = 0;
#pragma unroll
      for (int v = 0; v < 16; v++) pairs |= (8 * (v >> 2) + 4 * h + (v & 3) <= l31 ? 1u : 0u) << v;
    }
    float p[16], top = -INFINITY;
#pragma unroll
    for (int v = 0; v < 16; v++) {
      p[v] = (pairs >> v) & 1 ? s[v] * scale : -INFINITY;
      top = fmaxf(top, p[v]);
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
      p[v] = (pairs >> v) & 1 ? expf(p[v] - mn) : 0.f;
      sum += p[v];
    }
    l += sum;
    add_tile<DH>(o, vf, p, kt == qt, pairs);
  }
  l += __shfl_xor(l, 32, 64);
  __syncthreads();  // every wave is done with the queries
  put_sums<DH>(smem_a + wave * slot_floats<DH>(), o, lane);
  if (h == 0) { ms[wave][l31] = m; ls[wave][l31] = l; }
  __syncthreads();
  float* out = ctx + ((size_t)(bh / H) * S + q0) * Hd + (bh % H) * dh;
  for (int c = threadIdx.x; c < 32 * DH / 4; c += 256) {
    const int row = c / (DH / 4), col = c % (DH / 4) * 4;
    const float M = fmaxf(fmaxf(ms[0][row], ms[1][row]), fmaxf(ms[2][row], ms[3][row]));
    float L = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < 4; w++) {
      if (w > qt) break;  // that wave had no tile
      const float e = expf(ms[w][row] - M);
      const float4 x = *reinterpret_cast<const float4*>(smem_a + w * slot_floats<DH>() + row * (DH + 4) + col);
      L = fmaf(ls[w][row], e, L);
      a.x = fmaf(x.x, e, a.x); a.y = fmaf(x.y, e, a.y); a.z = fmaf(x.z, e, a.z); a.w = fmaf(x.w, e, a.w);
    }
    if (q0 + row < S) {
      const float inv = 1.f / L;
      if (col < dh) *reinterpret_cast<float4*>(out + (size_t)row * Hd + col) = make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv);
      if (col == 0) lse[(size_t)bh * S + q0 + row] = M + logf(L);
    }
  }
}

// Both halves of the backward pass in one launch: blockIdx.y = 0 dK and dV of a key tile, 1 dQ of a query tile (less
// work, and fills in behind).  B 4, S 512, 16 heads of 64, with the pass that forms delta: 1617 us on the scalar kernels, 120 here;
// 1 x 2000 with 4 heads of 128: 3462 -> 198.
template <int DH, bool EXACT>
__global__ __launch_bounds__(256, DH > 64 ? 1 : 2) void attn_bwd_f32_kernel(int S, int H, int dh, int BH, const float* __restrict__ qkv,
                                                                         const float* __restrict__ lse,
                                                                         const float* __restrict__ delta,
                                                                         const float* __restrict__ dctx, float* __restrict__ dqkv) {
  extern __shared__ __attribute__((aligned(16))) float smem_a[];
  const int lane = threadIdx.x & 63, l31 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nt = (S + 31) / 32, bh = blockIdx.x % BH;
  const int Hd = H * dh, ld = 3 * Hd;
  const float* base = qkv + (size_t)(bh / H) * S * ld + (bh % H) * dh;
  const HeadTile<DH, EXACT> Q{base, ld, S, dh}, Kt{base + Hd, ld, S, dh}, Vt{base + 2 * Hd, ld, S, dh};
  const HeadTile<DH, EXACT> dO{dctx + (size_t)(bh / H) * S * Hd + (bh % H) * dh, Hd, S, dh};
  float* dout = dqkv + (size_t)(bh / H) * S * ld + (bh % H) * dh;
  const float* lrow = lse + (size_t)bh * S;
  const float* drow = delta + (size_t)bh * S;
  const float scale = rsqrtf((float)dh);
  float* own_b = smem_a + slot_floats<DH>();
  float* slot = smem_a + wave * slot_floats<DH>();

  if (blockIdx.y) {
    const int qt = nt - 1 - blockIdx.x / BH, q0 = qt * 32;
    Q.stage(q0, smem_a);
    dO.stage(q0, own_b);
    __syncthreads();
    const float li = lrow[min(q0 + l31, S - 1)], di = drow[min(q0 + l31, S - 1)];
    f32x16 dq[DH / 32];
    zero<DH>(dq);
    for (int kt = wave; kt <= qt; kt += 4) {
      float4 kf[DH / 8], vf[DH / 8];
      float kc[16][DH / 32];
      Kt.rows(kt * 32, lane, kf);
      Vt.rows(kt * 32, lane, vf);
      const f32x16 s = score_tile<DH>(kf, smem_a, lane);
      const f32x16 dp = score_tile<DH>(vf, own_b, lane);
      __builtin_amdgcn_sched_barrier(0);
      Kt.cols(kt * 32, lane, kc);
      unsigned pairs = 0xffff;
      if (kt == qt) {
        pairs = 0;
#pragma unroll
        for (int v = 0; v < 16; v++) pairs |= (8 * (v >> 2) + 4 * h + (v & 3) <= l31 ? 1u : 0u) << v;
      }
      float ds[16];
#pragma unroll
      for (int v = 0; v < 16; v++) ds[v] = (pairs >> v) & 1 ? expf(s[v] * scale - li) * (dp[v] - di) : 0.f;
      add_tile<DH>(dq, kc, ds, kt == qt, pairs);
    }
    __syncthreads();
    put_sums<DH>(slot, dq, lane);
    __syncthreads();
    store_sums<DH>(smem_a, scale, dout + (size_t)q0 * ld, ld, S - q0, dh);
    return;
  }

  const int kt = blockIdx.x / BH, k0 = kt * 32;
  Kt.stage(k0, smem_a);
  Vt.stage(k0, own_b);
  __syncthreads();
  f32x16 dk[DH / 32], dv[DH / 32];
  zero<DH>(dk);
  zero<DH>(dv);
  for (int qt = kt + wave; qt < nt; qt += 4) {
    const int q0 = qt * 32;
    float4 qf[DH / 8], of[DH / 8];
    float qc[16][DH / 32], oc[16][DH / 32];
    Q.rows(q0, lane, qf);
    dO.rows(q0, lane, of);
    float li[16], di[16];
    const bool tail = q0 + 32 > S;
    unsigned pairs = 0;
#pragma unroll
    for (int v = 0; v < 16; v++) {
      const int r = 8 * (v >> 2) + 4 * h + (v & 3), i = min(q0 + r, S - 1);
      li[v] = lrow[i];
      di[v] = drow[i];
      pairs |= (q0 + r < S && (qt > kt || r >= l31) ? 1u : 0u) << v;
    }
    const f32x16 s = score_tile<DH>(qf, smem_a, lane);
    const f32x16 dp = score_tile<DH>(of, own_b, lane);
    __builtin_amdgcn_sched_barrier(0);
    dO.cols(q0, lane, oc);
    Q.cols(q0, lane, qc);
    float p[16], ds[16];
#pragma unroll
    for (int v = 0; v < 16; v++) {
      const bool ok = (pairs >> v) & 1;
      p[v] = ok ? expf(s[v] * scale - li[v]) : 0.f;
      ds[v] = ok ? p[v] * (dp[v] - di[v]) : 0.f;
    }
    add_tile<DH>(dv, oc, p, qt == kt || tail, pairs);
    add_tile<DH>(dk, qc, ds, qt == kt || tail, pairs);
  }
  __syncthreads();
  put_sums<DH>(slot, dk, lane);
  __syncthreads();
  store_sums<DH>(smem_a, scale, dout + (size_t)k0 * ld + Hd, ld, S - k0, dh);
  __syncthreads();
  put_sums<DH>(slot, dv, lane);
  __syncthreads();
  store_sums<DH>(smem_a, 1.f, dout + (size_t)k0 * ld + 2 * Hd, ld, S - k0, dh);
}

// Head widths in units of the 16-byte loads, and tensors that start on such a unit.  Other widths stay with the scalar
// kernels, which need 567 + 1617 us for 64 heads of 512 x 64 where these need 40 + 120; at one query and key they are even.
bool attn_f32_supported(int dtype, int dh, const void* qkv, const void* ctx, const void* dctx, const void* dqkv) {
  const uintptr_t a = (uintptr_t)qkv | (uintptr_t)ctx | (uintptr_t)dctx | (uintptr_t)dqkv;
  return dtype == FAX_F32 && dh > 0 && dh <= 128 && dh % 4 == 0 && (a & 15) == 0;
}

template <int DH, bool EXACT>
static int attn_fwd_f32_t(int B, int S, int H, int dh, const float* qkv, float* ctx, float* lse, hipStream_t s) {
  constexpr int lds = 4 * slot_floats<DH>() * (int)sizeof(float);
  auto kern = attn_fwd_f32_kernel<DH, EXACT>;
  static bool configured = false;  // benign race: the attribute is idempotent
  if (!configured) {
    FAX_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    configured = true;
  }
  hipLaunchKernelGGL(kern, dim3((S + 31) / 32 * B * H), dim3(256), lds, s, S, H, dh, B * H, qkv, ctx, lse);
  FAX_LAUNCH_CHECK("attn_fwd_f32");
  return FAX_OK;
}

int attn_fwd_f32(int B, int S, int H, int dh, const void* qkv, void* ctx, float* lse, hipStream_t s) {
  if (B * H == 0 || S == 0) return FAX_OK;
  const float* q = (const float*)qkv;
  float* c = (float*)ctx;
  if (dh == 32) return attn_fwd_f32_t<32, true>(B, S, H, dh, q, c, lse, s);
  if (dh == 64) return attn_fwd_f32_t<64, true>(B, S, H, dh, q, c, lse, s);
  if (dh == 96) return attn_fwd_f32_t<96, true>(B, S, H, dh, q, c, lse, s);
  if (dh == 128) return attn_fwd_f32_t<128, true>(B, S, H, dh, q, c, lse, s);
  if (dh < 32) return attn_fwd_f32_t<32, false>(B, S, H, dh, q, c, lse, s);
  if (dh < 64) return attn_fwd_f32_t<64, false>(B, S, H, dh, q, c, lse, s);
  if (dh < 96) return attn_fwd_f32_t<96, false>(B, S, H, dh, q, c, lse, s);
  return attn_fwd_f32_t<128, false>(B, S, H, dh, q, c, lse, s);
}

template <int DH, bool EXACT>
static int attn_bwd_f32_t(int B, int S, int H, int dh, const float* qkv, const float* lse, const float* delta, const float* dctx,
                          float* dqkv, hipStream_t s) {
  constexpr int lds = 4 * slot_floats<DH>() * (int)sizeof(float);
  auto kern = attn_bwd_f32_kernel<DH, EXACT>;
  static bool configured = false;  // benign race: the attribute is idempotent
  if (!configured) {
    FAX_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    configured = true;
  }
  hipLaunchKernelGGL(kern, dim3((S + 31) / 32 * B * H, 2), dim3(256), lds, s, S, H, dh, B * H, qkv, lse, delta, dctx, dqkv);
  FAX_LAUNCH_CHECK("attn_bwd_f32");
  return FAX_OK;
}

int attn_bwd_f32(int B, int S, int H, int dh, const void* qkv, const void* ctx, const float* lse, const void* dctx, void* dqkv,
                 float* delta, hipStream_t s) {
  if (B * H == 0 || S == 0) return FAX_OK;
  FAX_TRY(attn_delta(FAX_F32, B, S, H, dh, ctx, dctx, delta, s));
  const float *q = (const float*)qkv, *g = (const float*)dctx;
  float* o = (float*)dqkv;
  if (dh == 32) return attn_bwd_f32_t<32, true>(B, S, H, dh, q, lse, delta, g, o, s);
  if (dh == 64) return attn_bwd_f32_t<64, true>(B, S, H, dh, q, lse, delta, g, o, s);
  if (dh == 96) return attn_bwd_f32_t<96, true>(B, S, H, dh, q, lse, delta, g, o, s);
  if (dh == 128) return attn_bwd_f32_t<128, true>(B, S, H, dh, q, lse, delta, g, o, s);
  if (dh < 32) return attn_bwd_f32_t<32, false>(B, S, H, dh, q, lse, delta, g, o, s);
  if (dh < 64) return attn_bwd_f32_t<64, false>(B, S, H, dh, q, lse, delta, g, o, s);
  if (dh < 96) return attn_bwd_f32_t<96, false>(B, S, H, dh, q, lse, delta, g, o, s);
  return attn_bwd_f32_t<128, false>(B, S, H, dh, q, lse, delta, g, o, s);
}

}  // namespace fax
