// AdamW over many tensors in one launch, moments of 32 bits or of 8.
//
// Memory bound, one pass: 28 to 30 bytes an element with moments of 32 bits, 16 to 18 with moments of 8.  A workgroup has 1024
// consecutive elements of one tensor, a wave a block that shares a scale; which tensor, it looks up in the table that comes with the launch's arguments
// (MULTI_BATCH tensors: the arguments of a launch are 4 KB).  (4096 elements, four blocks to a wave one after another | 1024, us: 8 tensors of 50000, 8-bit 10.6 | 7.5;
// of 500000 19.5 | 17.0, 32-bit 18.9 | 18.5; of 2 million 56.6 | 52.9, 68.8 | 64.7; of 8 million 216 | 217, 344 | 335.)
// Measured: the 148 tensors of a 12-layer, 768-wide model (125 M elements, fp32 gradients, bf16 copies) 685 us with moments of 32 bits (3.76 GB, 5.5 TB/s)
// and 444 us with moments of 8 (2.26 GB, 5.1 TB/s); a large copy on the same card moves 4.7 to 5.0 TB/s.
#include "adamw.h"

namespace fax {

static constexpr int MULTI_BATCH = 48;
static constexpr int BLOCK = 256;              // elements that share a scale: a wave's, four to a lane
static constexpr int MULTI_CHUNK = 4 * BLOCK;  // elements of a workgroup
static constexpr float E4M3_MAX = 448.f;
static constexpr float M_FLOOR = 7.888609052e-31f;  // 2^-100: below, 448 / maximum would leave fp32
static constexpr uint32_t HASH_C = 0x9E3779B1u, HASH_D = 0x2545F491u;

__host__ __device__ __forceinline__ uint32_t hash32(uint32_t x) {
  x ^= x >> 16;
  x *= HASH_C;
  x ^= x >> 15;
  x *= HASH_D;
  return x ^ (x >> 16);
}

struct MultiEntry {
  float *p, *m_scale, *v_scale;
  void *m, *v;
  const void* g;
  bf16_t* lowp;
  size_t n;
  uint32_t key;     // of this tensor's random bits
  int16_t g_bf16, decay;
};
struct MultiTable {
  MultiEntry t[MULTI_BATCH];
  unsigned first[MULTI_BATCH + 1];  // first workgroup of each tensor
  int count;
};
static_assert(sizeof(MultiTable) + sizeof(AdamScalars) <= 4096, "the arguments of a launch");

// The tensor whose workgroups contain this one.
__device__ __forceinline__ int entry_of(const MultiTable& b, unsigned block) {
  int lo = 0, hi = b.count;  // uniform
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (block >= b.first[mid]) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Elements i .. i + 3 as fp32, those from n on zero.
__device__ __forceinline__ float4 load4(const float* p, size_t i, size_t n) {
  if (i + 4 <= n) return *reinterpret_cast<const float4*>(p + i);
  float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
  if (i < n) r.x = p[i];
  if (i + 1 < n) r.y = p[i + 1];
  if (i + 2 < n) r.z = p[i + 2];
  return r;
}
__device__ __forceinline__ float4 load4(const bf16_t* p, size_t i, size_t n) {
  float r[4] = {0.f, 0.f, 0.f, 0.f};
  if (i + 4 <= n) {
    const uint2 u = *reinterpret_cast<const uint2*>(p + i);
    return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
  }
#pragma unroll
  for (int k = 0; k < 3; k++)
    if (i + k < n) r[k] = (float)p[i + k];
  return make_float4(r[0], r[1], r[2], r[3]);
}
__device__ __forceinline__ uint32_t load4(const uint8_t* p, size_t i, size_t n) {
  if (i + 4 <= n) return *reinterpret_cast<const uint32_t*>(p + i);
  uint32_t r = 0;
#pragma unroll
  for (int k = 0; k < 3; k++)
    if (i + k < n) r |= (uint32_t)p[i + k] << (8 * k);
  return r;
}
__device__ __forceinline__ void store4(float* p, size_t i, size_t n, const float4& v) {
  if (i + 4 <= n) {
    nt_store4(reinterpret_cast<float4*>(p + i), v);
    return;
  }
  if (i < n) p[i] = v.x;
  if (i + 1 < n) p[i + 1] = v.y;
  if (i + 2 < n) p[i + 2] = v.z;
}
__device__ __forceinline__ void store4(bf16_t* p, size_t i, size_t n, const float4& v) {
  union { bf16_t h[4]; uint2 u; } k;
  k.h[0] = (bf16_t)v.x; k.h[1] = (bf16_t)v.y; k.h[2] = (bf16_t)v.z; k.h[3] = (bf16_t)v.w;
  if (i + 4 <= n) {
    nt_store2(reinterpret_cast<uint2*>(p + i), k.u);
    return;
  }
  if (i < n) p[i] = k.h[0];
  if (i + 1 < n) p[i + 1] = k.h[1];
  if (i + 2 < n) p[i + 2] = k.h[2];
}
__device__ __forceinline__ void store4(uint8_t* p, size_t i, size_t n, uint32_t v) {
  if (i + 4 <= n) {
    __builtin_nontemporal_store(v, reinterpret_cast<uint32_t*>(p + i));
    return;
  }
#pragma unroll
  for (int k = 0; k < 3; k++)
    if (i + k < n) p[i + k] = (uint8_t)(v >> (8 * k));
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.4028235e38f; }

// One element.  Every product and sum is rounded by itself (no contraction into multiply-adds): an element's bits do not depend on its place
// or on the compiler, and a code of eight bits that hangs on the last of them can be computed again anywhere.
__device__ __forceinline__ void update(float g, float& p, float& m, float& v, const AdamScalars& a) {
#pragma clang fp contract(off)
  m = a.b1 * m + a.one_m_b1 * g;
  v = a.b2 * v + a.one_m_b2 * g * g;
  const float root = sqrtf(v * a.inv_bc2) + a.eps;
  const float up = m * a.inv_bc1 / root;
  p = p * a.decay - a.lr * up;
}

// x in [0, 448] or NaN, up or down to an e4m3 number: up where the bits cut off and the random ones carry.  Those are the last twenty of
// an fp32 number of at least 2^-6; below, e4m3 numbers are whole multiples of 2^-9, as they are from 2^-6 to 2^-5.
__device__ __forceinline__ float round_random(float x, uint32_t bits20) {
  const bool low = x < 0.015625f;
  float y = low ? x + 0.015625f : x;  // (2^-6)
  y = __uint_as_float((__float_as_uint(y) + bits20) & 0xfff00000u);
  y = low ? y - 0.015625f : y;
  return fminf(y, E4M3_MAX);
}

__device__ __forceinline__ uint32_t pack4(const float (&x)[4]) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
}
__device__ __forceinline__ void unpack4(uint32_t w, float (&x)[4]) {
  x[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
  x[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
  x[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
  x[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
}

template <bool LOW8>
__global__ __launch_bounds__(256) void adamw_table_kernel(MultiTable b, AdamScalars a) {
  const int k = entry_of(b, blockIdx.x);
  const MultiEntry& e = b.t[k];
  const size_t n = e.n;
  if (!e.decay) a.decay = 1.f;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const size_t block = (size_t)(blockIdx.x - b.first[k]) * MULTI_CHUNK + wave * BLOCK, i = block + lane * 4;
  if (block >= n) return;
  float4 p = load4(e.p, i, n);
  const float4 g = e.g_bf16 ? load4((const bf16_t*)e.g, i, n) : load4((const float*)e.g, i, n);
  if constexpr (!LOW8) {
    float4 m = load4((const float*)e.m, i, n), v = load4((const float*)e.v, i, n);
    update(g.x, p.x, m.x, v.x, a);
    update(g.y, p.y, m.y, v.y, a);
    update(g.z, p.z, m.z, v.z, a);
    update(g.w, p.w, m.w, v.w, a);
    store4((float*)e.m, i, n, m);
    store4((float*)e.v, i, n, v);
  } else {
    const size_t at = block / BLOCK;
    const float ms = e.m_scale[at], vs = e.v_scale[at];
    float m[4], v[4];
    unpack4(load4((const uint8_t*)e.m, i, n), m);
    unpack4(load4((const uint8_t*)e.v, i, n), v);
    const float gs[4] = {g.x, g.y, g.z, g.w};
    float ps[4] = {p.x, p.y, p.z, p.w};
    float m_top = 0.f, v_top = 0.f;
#pragma unroll
    for (int q = 0; q < 4; q++) {
      m[q] *= ms;
      v[q] *= vs;
      v[q] *= v[q];
      update(gs[q], ps[q], m[q], v[q], a);
      v[q] = sqrtf(v[q]);
      if (finite(m[q])) m_top = fmaxf(m_top, fabsf(m[q]));
      if (finite(v[q])) v_top = fmaxf(v_top, v[q]);
    }
    p = make_float4(ps[0], ps[1], ps[2], ps[3]);
    m_top = wave_max(m_top);
    v_top = wave_max(v_top);
    if (m_top < M_FLOOR) m_top = 0.f;
    const float m_inv = m_top > 0.f ? 1.f / m_top * E4M3_MAX : 0.f, v_inv = v_top > 0.f ? 1.f / v_top * E4M3_MAX : 0.f;
#pragma unroll
    for (int q = 0; q < 4; q++) {
      const float nan = __builtin_nanf("");
      m[q] = finite(m[q]) ? fminf(fmaxf(m[q] * m_inv, -E4M3_MAX), E4M3_MAX) : nan;
      const uint32_t bits = hash32((uint32_t)(i + q) * HASH_C + e.key) >> 12;
      const float x = v[q];
      v[q] = !finite(x) ? nan : x > 0.f ? fmaxf(round_random(x * v_inv, bits), 0.001953125f) : 0.f;
    }
    store4((uint8_t*)e.m, i, n, pack4(m));
    store4((uint8_t*)e.v, i, n, pack4(v));
    if (lane == 0) {
      e.m_scale[at] = m_top * (1.f / E4M3_MAX);
      e.v_scale[at] = v_top * (1.f / E4M3_MAX);
    }
  }
  store4(e.p, i, n, p);
  if (e.lowp) store4(e.lowp, i, n, p);
}

int adamw_multi(int state, int count, const FaxAdamWTensor* tensors, const FaxAdamW& hp, int step, uint32_t seed, hipStream_t s) {
  MultiTable b;
  b.count = 0;
  b.first[0] = 0;
  double bytes = 0.0;
  const AdamScalars a = adam_scalars(hp, step);
  const uint32_t base = hash32(seed + (uint32_t)step * HASH_C);
  auto flush = [&]() -> int {
    if (b.count == 0) return FAX_OK;
    Timed t_("adamw_multi", WORK_BYTE, bytes, s);
    if (state == FAX_STATE_E4M3) hipLaunchKernelGGL(adamw_table_kernel<true>, dim3(b.first[b.count]), dim3(256), 0, s, b, a);
    else hipLaunchKernelGGL(adamw_table_kernel<false>, dim3(b.first[b.count]), dim3(256), 0, s, b, a);
    FAX_LAUNCH_CHECK("adamw_multi");
    b.count = 0;
    bytes = 0.0;
    return FAX_OK;
  };
  for (int t = 0; t < count; t++) {
    const FaxAdamWTensor& x = tensors[t];
    if (x.n == 0) continue;
    const size_t chunks = (x.n + MULTI_CHUNK - 1) / MULTI_CHUNK;
    if (b.count == MULTI_BATCH || b.first[b.count] + chunks > 0xffffffu) FAX_TRY(flush());  // (fewer than 2^32 threads)
    MultiEntry& e = b.t[b.count];
    e.p = (float*)x.master; e.m = x.m; e.v = x.v; e.g = x.grad; e.lowp = (bf16_t*)x.lowp; e.n = x.n;
    e.m_scale = x.m_scale; e.v_scale = x.v_scale;
    e.key = hash32(base + (uint32_t)t * HASH_C);
    e.g_bf16 = x.grad_dtype == FAX_BF16; e.decay = x.decay != 0;
    b.first[b.count + 1] = b.first[b.count] + (unsigned)chunks;
    b.count++;
    bytes += (double)x.n * (8.0 + (e.g_bf16 ? 2.0 : 4.0) + (x.lowp ? 2.0 : 0.0) + (state == FAX_STATE_E4M3 ? 4.0 + 16.0 / BLOCK : 16.0));
  }
  return flush();
}

}  // namespace fax
