// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// Gradient.  dtable[v] = scale * sum of dout[n] over the positions n that hold id v.  Positions are sorted by id (stably: ascending
// within an id), then every row of dtable has one writer that adds its positions' rows in order: no atomics, the same bits every time.
//   sort     least significant digit first, of SORT_BITS bits at most.  A wave has a run of consecutive positions and ranks 64 at a time by
//            comparing their digits bit by bit (ballots); ranks across waves come from a table of counts by digit and wave, scanned in that order.
//   chunks   of CHUNK sorted positions that all hold the same id are added up into a row of scratch each, so that a frequent id, of which a
//            text has thousands, is not one workgroup's chain.
//   rows     one workgroup to a row: what comes before the first whole chunk, the chunks' sums, what comes after the last.
// Ids outside [0, V) sort behind all others and are not looked at again.
#include "fax_internal.h"

namespace fax {

// ---- lookup -----------------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(int N, int V, int D, const int32_t* __restrict__ tokens, const T* __restrict__ table,
                                                            float scale, T* __restrict__ out) {
  constexpr int E = Vec16<T>::N;
  for (int n = blockIdx.x; n < N; n += gridDim.x) {
    const int id = tokens[n];
    const bool known = id >= 0 && id < V;
    const T* row = table + (size_t)(known ? id : 0) * D;
    T* o = out + (size_t)n * D;
    if (D % E == 0) {
      for (int d = threadIdx.x * E; d < D; d += 256 * E) {
        Vec16<T> x;
        x.load(row + d);
#pragma unroll
        for (int k = 0; k < E; k++) x.set(k, known ? x.get(k) * scale : 0.f);
        x.store(o + d);
      }
    } else {
      for (int d = threadIdx.x; d < D; d += 256) o[d] = from_f<T>(known ? to_f(row[d]) * scale : 0.f);
    }
  }
}

template <typename T>
static int embedding_fwd_t(int N, int V, int D, const int32_t* tokens, const T* table, float scale, T* out, hipStream_t s) {
  hipLaunchKernelGGL(embedding_fwd_kernel<T>, dim3(N), dim3(256), 0, s, N, V, D, tokens, table, scale, out);
  FAX_LAUNCH_CHECK("embedding_fwd");
  return FAX_OK;
}

int embedding_fwd(int dtype, int N, int V, int D, const int32_t* tokens, const void* table, float scale, void* out, hipStream_t s) {
  if (N == 0) return FAX_OK;
  Timed t_("embedding_fwd", WORK_BYTE, 2.0 * N * D * (dtype == FAX_F32 ? 4.0 : 2.0) + 4.0 * N, s);
  if (dtype == FAX_F32) return embedding_fwd_t<float>(N, V, D, tokens, (const float*)table, scale, (float*)out, s);
  return embedding_fwd_t<bf16_t>(N, V, D, tokens, (const bf16_t*)table, scale, (bf16_t*)out, s);
}

// ---- sorting positions by id ------------------------------------------------------------------------
static constexpr int SORT_BITS = 9, BINS = 1 << SORT_BITS;
static constexpr int WAVE_KEYS = 1024;  // positions of a wave, where there are enough of them
static constexpr int CHUNK = 32;

struct SortPlan {
  int bits, passes;   // of a digit, digits
  int per_wave, waves;
};
static SortPlan sort_plan(int N, int V) {
  SortPlan p;
  int bits = 1;
  while (bits < 31 && (V >> bits) != 0) bits++;  // ids 0 .. V
  p.passes = (bits + SORT_BITS - 1) / SORT_BITS;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.per_wave = WAVE_KEYS;
  p.waves = (N + WAVE_KEYS - 1) / WAVE_KEYS;
  return p;
}

// Digit of lane's key, the lanes that have the same one, and this lane's place among them.  Lanes without a key (ok false) match nobody.
__device__ __forceinline__ unsigned long long same_digit(unsigned digit, int bits, bool ok) {
  unsigned long long m = __builtin_amdgcn_ballot_w64(ok);
  for (int b = 0; b < bits; b++) {
    const unsigned long long one = __builtin_amdgcn_ballot_w64((digit >> b) & 1);
    m &= (digit >> b) & 1 ? one : ~one;
  }
  return ok ? m : 0ull;
}
__device__ __forceinline__ int below(unsigned long long m) {
  return __builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0));
}
__device__ __forceinline__ unsigned key_of(int id, int V) { return (unsigned)id < (unsigned)V ? (unsigned)id : (unsigned)V; }

// counts[digit * waves + wave] of one pass.  in_pos NULL: the positions in order (first pass), with keys from the tokens.
__global__ __launch_bounds__(256) void sort_count_kernel(int N, int V, int shift, int bits, int per_wave, int waves, const int32_t* __restrict__ tokens,
                                                         const uint32_t* __restrict__ in_key, uint32_t* __restrict__ counts) {
  __shared__ unsigned hist[4][BINS];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, w = blockIdx.x * 4 + wave;
  const unsigned bins = 1u << bits;
  for (unsigned i = threadIdx.x; i < 4 * BINS; i += 256) (&hist[0][0])[i] = 0;
  __syncthreads();
  if (w < waves) {
    const long long k0 = (long long)w * per_wave;
    for (int k = lane; k < per_wave && k0 + k < N; k += 64) {
      const unsigned key = in_key ? in_key[k0 + k] : key_of(tokens[k0 + k], V);
      atomicAdd(&hist[wave][(key >> shift) & (bins - 1)], 1u);
    }
  }
  __syncthreads();
  if (w < waves)
    for (unsigned d = lane; d < bins; d += 64) counts[(size_t)d * waves + w] = hist[wave][d];
}

// counts -> exclusive prefix sums, in place; one workgroup.
__global__ __launch_bounds__(1024) void sort_scan_kernel(int n, uint32_t* __restrict__ counts) {
  __shared__ unsigned sums[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  unsigned carry = 0;
  for (int base = 0; base < n; base += 1024 * 4) {
    const int i = base + threadIdx.x * 4;
    unsigned c[4], t = 0;
#pragma unroll
    for (int k = 0; k < 4; k++) {
      c[k] = i + k < n ? counts[i + k] : 0u;
      t += c[k];
    }
    unsigned inc = t;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const unsigned x = __shfl_up(inc, o, 64);
      if (lane >= o) inc += x;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = inc;
    __syncthreads();
    unsigned before = 0, total = 0;
    for (int k = 0; k < 16; k++) {
      if (k < wave) before += sums[k];
      total += sums[k];
    }
    unsigned x = carry + before + inc - t;
#pragma unroll
    for (int k = 0; k < 4; k++) {
      if (i + k < n) counts[i + k] = x;
      x += c[k];
    }
    carry += total;
  }
}

__global__ __launch_bounds__(256) void sort_place_kernel(int N, int V, int shift, int bits, int per_wave, int waves, const int32_t* __restrict__ tokens,
                                                         const uint32_t* __restrict__ in_key, const uint32_t* __restrict__ in_pos,
                                                         const uint32_t* __restrict__ starts, uint32_t* __restrict__ out_key, uint32_t* __restrict__ out_pos) {
  __shared__ unsigned next_all[4][BINS];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, w = blockIdx.x * 4 + wave;
  const unsigned bins = 1u << bits;
  if (w >= waves) return;  // (no barrier below: a wave works on its own, its LDS operations are in order)
  volatile unsigned* next = next_all[wave];
  for (unsigned d = lane; d < bins; d += 64) next[d] = starts[(size_t)d * waves + w];
  const long long k0 = (long long)w * per_wave;
  for (int k = 0; k < per_wave && k0 + k < N; k += 64) {
    const bool ok = k + lane < per_wave && k0 + k + lane < N;
    const long long at = k0 + k + lane;
    unsigned key = 0, pos = 0;
    if (ok) {
      key = in_key ? in_key[at] : key_of(tokens[at], V);
      pos = in_pos ? in_pos[at] : (unsigned)at;
    }
    const unsigned digit = (key >> shift) & (bins - 1);
    const unsigned long long m = same_digit(digit, bits, ok);
    const int rank = below(m);
    unsigned to = 0;
    if (ok) to = next[digit] + rank;
    __builtin_amdgcn_wave_barrier();
    if (ok && rank == 0) next[digit] = to + (unsigned)__popcll(m);
    __builtin_amdgcn_wave_barrier();
    if (ok) {
      out_key[to] = key;
      out_pos[to] = pos;
    }
  }
}

// ---- sums -------------------------------------------------------------------------------------------
// acc += rows pos[k0 .. k1) of dout, E features from d0.
template <typename T, int E>
__device__ __forceinline__ void add_rows(float (&acc)[E], const T* __restrict__ dout, int D, int d0, const uint32_t* __restrict__ pos, int k0, int k1) {
  for (int k = k0; k < k1; k++) {
    const T* row = dout + (size_t)pos[k] * D + d0;
    if (E > 1) {
      Vec16<T> x;
      x.load(row);
#pragma unroll
      for (int e = 0; e < E; e++) acc[e] += x.get(e);
    } else {
      acc[0] += to_f(row[0]);
    }
  }
}

template <typename T, int E>
__global__ __launch_bounds__(256) void embedding_chunk_kernel(int N, int V, int D, const uint32_t* __restrict__ key, const uint32_t* __restrict__ pos,
                                                              const T* __restrict__ dout, float* __restrict__ sums) {
  const int k0 = blockIdx.x * CHUNK;
  if (k0 + CHUNK > N) return;
  const unsigned id = key[k0];
  if (id >= (unsigned)V || key[k0 + CHUNK - 1] != id) return;
  for (int d0 = threadIdx.x * E; d0 < D; d0 += 256 * E) {
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; e++) acc[e] = 0.f;
    add_rows<T, E>(acc, dout, D, d0, pos, k0, k0 + CHUNK);
#pragma unroll
    for (int e = 0; e < E; e++) sums[(size_t)blockIdx.x * D + d0 + e] = acc[e];
  }
}

// The first of n sorted keys that is at least v: 64 candidates at a time.
__device__ __forceinline__ int lower_bound(const uint32_t* __restrict__ key, int n, unsigned v) {
  int lo = 0, hi = n;  // the answer is in [lo, hi]
  const int lane = threadIdx.x & 63;
  while (hi - lo > 0) {
    const int step = (hi - lo + 63) / 64;
    const long long at = lo + (long long)lane * step;  // candidates lo, lo + step, ...
    const bool less = at < hi && key[at] < v;
    const int c = __popcll(__builtin_amdgcn_ballot_w64(less));  // sorted: the first c are less
    if (c == 0) return lo;
    const int nlo = lo + (c - 1) * step + 1;
    hi = min(hi, lo + c * step);
    lo = nlo;
  }
  return lo;
}

// BY_ROW: workgroup = row of the table, zeros where no position holds it.  Otherwise workgroup = sorted position, the first of an id adds.
template <typename T, int E, bool BY_ROW>
__global__ __launch_bounds__(256) void embedding_rows_kernel(int N, int V, int D, const uint32_t* __restrict__ key, const uint32_t* __restrict__ pos,
                                                             const T* __restrict__ dout, const float* __restrict__ sums, float scale, int accumulate,
                                                             float* __restrict__ dtable) {
  unsigned v;
  int lo;
  if (BY_ROW) {
    v = blockIdx.x;
    lo = lower_bound(key, N, v);
  } else {
    lo = blockIdx.x;
    v = key[lo];
    if (v >= (unsigned)V || (lo > 0 && key[lo - 1] == v)) return;
  }
  int hi = lo;
  if (lo < N && key[lo] == v) hi = lo + lower_bound(key + lo, N - lo, v + 1);
  const int c0 = (lo + CHUNK - 1) / CHUNK, c1 = hi / CHUNK;  // whole chunks
  for (int d0 = threadIdx.x * E; d0 < D; d0 += 256 * E) {
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; e++) acc[e] = 0.f;
    if (c0 < c1) {
      add_rows<T, E>(acc, dout, D, d0, pos, lo, c0 * CHUNK);
      for (int c = c0; c < c1; c++)
#pragma unroll
        for (int e = 0; e < E; e++) acc[e] += sums[(size_t)c * D + d0 + e];
      add_rows<T, E>(acc, dout, D, d0, pos, c1 * CHUNK, hi);
    } else {
      add_rows<T, E>(acc, dout, D, d0, pos, lo, hi);
    }
    float* o = dtable + (size_t)v * D + d0;
#pragma unroll
    for (int e = 0; e < E; e++) o[e] = accumulate ? fmaf(acc[e], scale, o[e]) : acc[e] * scale;
  }
}

struct EmbeddingWs {
  size_t key[2], pos[2], counts, sums, total;
};
static EmbeddingWs embedding_ws(int N, int V, int D) {
  const SortPlan p = sort_plan(N, V);
  EmbeddingWs w;
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t r = o; o += (bytes + 255) / 256 * 256; return r; };
  for (int i = 0; i < 2; i++) {
    w.key[i] = take((size_t)N * 4);
    w.pos[i] = take((size_t)N * 4);
  }
  w.counts = take((size_t)p.waves * ((size_t)1 << p.bits) * 4);
  w.sums = take((size_t)(N / CHUNK) * D * 4);
  w.total = o;
  return w;
}
size_t embedding_bwd_ws_bytes(int N, int V, int D) { return embedding_ws(N, V, D).total; }

template <typename T, int E>
static int embedding_sums(int N, int V, int D, const uint32_t* key, const uint32_t* pos, const T* dout, float* sums, float scale, float* dtable,
                          bool accumulate, hipStream_t s) {
  if (N >= CHUNK) hipLaunchKernelGGL((embedding_chunk_kernel<T, E>), dim3(N / CHUNK), dim3(256), 0, s, N, V, D, key, pos, dout, sums);
  if (accumulate) hipLaunchKernelGGL((embedding_rows_kernel<T, E, false>), dim3(N), dim3(256), 0, s, N, V, D, key, pos, dout, sums, scale, 1, dtable);
  else hipLaunchKernelGGL((embedding_rows_kernel<T, E, true>), dim3(V), dim3(256), 0, s, N, V, D, key, pos, dout, sums, scale, 0, dtable);
  FAX_LAUNCH_CHECK("embedding_bwd");
  return FAX_OK;
}

int embedding_bwd(int dtype, int N, int V, int D, const int32_t* tokens, const void* dout, float scale, float* dtable, bool accumulate, void* ws,
                  hipStream_t s) {
  if (N == 0) return accumulate ? FAX_OK : fill_zero(dtable, (size_t)V * D * 4, s);
  Timed t_("embedding_bwd", WORK_BYTE, (double)N * D * (dtype == FAX_F32 ? 4.0 : 2.0) + (accumulate ? 8.0 * D * (N < V ? N : V) : 4.0 * V * D), s);
  const SortPlan p = sort_plan(N, V);
  const EmbeddingWs w = embedding_ws(N, V, D);
  char* b = (char*)ws;
  uint32_t* counts = (uint32_t*)(b + w.counts);
  uint32_t *key = nullptr, *pos = nullptr;
  const unsigned grid = (p.waves + 3) / 4;
  for (int i = 0; i < p.passes; i++) {
    uint32_t *ok = (uint32_t*)(b + w.key[i & 1]), *op = (uint32_t*)(b + w.pos[i & 1]);
    hipLaunchKernelGGL(sort_count_kernel, dim3(grid), dim3(256), 0, s, N, V, i * p.bits, p.bits, p.per_wave, p.waves, tokens, key, counts);
    hipLaunchKernelGGL(sort_scan_kernel, dim3(1), dim3(1024), 0, s, p.waves << p.bits, counts);
    hipLaunchKernelGGL(sort_place_kernel, dim3(grid), dim3(256), 0, s, N, V, i * p.bits, p.bits, p.per_wave, p.waves, tokens, key, pos, counts, ok, op);
    key = ok;
    pos = op;
  }
  float* sums = (float*)(b + w.sums);
  if (dtype == FAX_F32)
    return D % 4 == 0 ? embedding_sums<float, 4>(N, V, D, key, pos, (const float*)dout, sums, scale, dtable, accumulate, s)
                      : embedding_sums<float, 1>(N, V, D, key, pos, (const float*)dout, sums, scale, dtable, accumulate, s);
  return D % 8 == 0 ? embedding_sums<bf16_t, 8>(N, V, D, key, pos, (const bf16_t*)dout, sums, scale, dtable, accumulate, s)
                    : embedding_sums<bf16_t, 1>(N, V, D, key, pos, (const bf16_t*)dout, sums, scale, dtable, accumulate, s);
}

}  // namespace fax
