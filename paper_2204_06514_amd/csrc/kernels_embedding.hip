// Embedding lookup with scaling, and its gradient by sorted tokens.  Both are bound by memory.
// Measured at 65536 positions, table of 50304 x 768, frequencies like a text's: lookup (bf16) 22.5 us, 178 MB at 7.9 TB/s (frequent rows come out of the
// caches); gradient (bf16 upstream, fp32 table, 255 MB that have to move: 51 us at the rate of a large copy) 79 us: sorting 34 us, of which the zeros of
// rows without a position, 104 MB, fill 24; the chunks' sums 13 us, the other rows 34 us.  The sort's launches depend on each other, so some 10 us
// of the 34 have the chip idle.
#include <type_traits>

#include "fax_internal.h"

namespace fax {

// x / d for x < 2^31 as a multiplication, d >= 1: q = (x * m) >> s with m = ceil(2^s / d), s = 31 + ceil(log2 d) (Granlund and Montgomery, 1994);
// m is at most 2^32 + 1, the product fits 64 bits.
struct Divider {
  uint64_t m;
  unsigned s, d;
  explicit Divider(unsigned d_) : d(d_) {
    unsigned l = 0;
    while ((1ull << l) < d) l++;
    s = 31 + l;
    m = ((1ull << s) + d - 1) / d;
  }
  __device__ __forceinline__ unsigned operator()(unsigned x) const { return (unsigned)((x * m) >> s); }
};

// ---- lookup -----------------------------------------------------------------------------------------
// A thread has LOOKUPS vectors of the output, 256 apart: their ids, then their rows' vectors are in flight together.  (A workgroup to a row, with a
// thread to a vector, leaves most of 256 threads idle at common widths.)
static constexpr int LOOKUPS = 4;
template <typename T, int E>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(unsigned first_row, unsigned vectors, Divider per_row, int V, int D, const int32_t* __restrict__ tokens,
                                                            const T* __restrict__ table, float scale, T* __restrict__ out) {
  const unsigned base = blockIdx.x * (256u * LOOKUPS) + threadIdx.x;
  int id[LOOKUPS];
  unsigned col[LOOKUPS];
  tokens += first_row;
  out += (size_t)first_row * D;
#pragma unroll
  for (int k = 0; k < LOOKUPS; k++) {
    const unsigned x = base + 256u * k;
    const unsigned row = x < vectors ? per_row(x) : 0;
    col[k] = x - row * per_row.d;
    id[k] = x < vectors ? tokens[row] : -1;
  }
  if constexpr (E == 1) {
#pragma unroll
    for (int k = 0; k < LOOKUPS; k++) {
      const unsigned x = base + 256u * k;
      if (x < vectors) out[x] = from_f<T>(id[k] >= 0 && id[k] < V ? to_f(table[(size_t)id[k] * D + col[k]]) * scale : 0.f);
    }
  } else {
    Vec16<T> v[LOOKUPS];
#pragma unroll
    for (int k = 0; k < LOOKUPS; k++)
      if (id[k] >= 0 && id[k] < V) v[k].load(table + (size_t)id[k] * D + col[k] * E);
#pragma unroll
    for (int k = 0; k < LOOKUPS; k++) {
      const unsigned x = base + 256u * k;
      if (x >= vectors) continue;
      const bool known = id[k] >= 0 && id[k] < V;
      Vec16<T> o;
#pragma unroll
      for (int e = 0; e < E; e++) o.set(e, known ? v[k].get(e) * scale : 0.f);
      o.store_nt(out + (size_t)x * E);
    }
  }
}

template <typename T, int E>
static int embedding_fwd_t(int N, int V, int D, const int32_t* tokens, const T* table, float scale, T* out, hipStream_t s) {
  const unsigned per_row = D / E;
  const Divider div(per_row);
  const int rows = (int)(0x7fffffffu / per_row) < N ? (int)(0x7fffffffu / per_row) : N;  // of a launch: vectors count in 31 bits
  for (int r = 0; r < N; r += rows) {
    const unsigned vectors = (unsigned)(N - r < rows ? N - r : rows) * per_row;
    const unsigned blocks = (unsigned)(((uint64_t)vectors + 256 * LOOKUPS - 1) / (256 * LOOKUPS));
    hipLaunchKernelGGL((embedding_fwd_kernel<T, E>), dim3(blocks), dim3(256), 0, s, (unsigned)r, vectors, div, V, D, tokens, table, scale, out);
  }
  FAX_LAUNCH_CHECK("embedding_fwd");
  return FAX_OK;
}

int embedding_fwd(int dtype, int N, int V, int D, const int32_t* tokens, const void* table, float scale, void* out, hipStream_t s) {
  if (N == 0) return FAX_OK;
  Timed t_("embedding_fwd", WORK_BYTE, 2.0 * N * D * (dtype == FAX_F32 ? 4.0 : 2.0) + 4.0 * N, s);
  if (dtype == FAX_F32)
    return D % 4 == 0 ? embedding_fwd_t<float, 4>(N, V, D, tokens, (const float*)table, scale, (float*)out, s)
                      : embedding_fwd_t<float, 1>(N, V, D, tokens, (const float*)table, scale, (float*)out, s);
  return D % 8 == 0 ? embedding_fwd_t<bf16_t, 8>(N, V, D, tokens, (const bf16_t*)table, scale, (bf16_t*)out, s)
                    : embedding_fwd_t<bf16_t, 1>(N, V, D, tokens, (const bf16_t*)table, scale, (bf16_t*)out, s);
}

// ---- gradient ---------------------------------------------------------------------------------------
// dtable[v] = scale * sum of dout[n] over the positions n that hold id v.  Positions are sorted by id (stably: ascending within an
// id), then every row of dtable has one writer that adds its positions' rows in an order that depends on the ids alone: no floating-point
// atomics, the same bits every time.
//   sort    least significant digit first.  A workgroup has a run of consecutive positions.  A table of counts by run and digit gives where each run's
//           keys of a digit begin (every workgroup adds up what it needs of it); within a run, 64 keys at a time are ranked by comparing their digits bit
//           by bit (ballots).
//   chunks  of CHUNK sorted positions that all hold the same id are added up into a row of scratch each, so that a frequent id, of which a text has
//           thousands, is not one wavefront's chain.
//   rows    a wavefront to pieces of a few rows of dtable.  Rows with whole chunks have a workgroup to a piece: what comes before the first, the chunks' sums in four
//           parts, what comes after the last.
//   zeros   rows that no position holds are most of a table under a text (their frequencies fall like 1 / rank), and sorting leaves most of the chip
//           idle.  The first digit's launches clear and set a byte for each row that is held; workgroups added to the later digits' launches write the
//           zeros of the others, and the rows' kernel goes by position.
// Up to DIRECT positions there is no sort: a wavefront finds a row's positions among all of them.
// Ids outside [0, V) sort behind all others and are not looked at again.
static constexpr int SORT_BITS = 8, BINS = 1 << SORT_BITS;
static constexpr int RUN_KEYS = 1024;  // positions of a run, where that leaves at most MOST_RUNS
static constexpr int MOST_RUNS = 256;
static constexpr int SMALL_KEYS = 4096;  // up to here one workgroup sorts in LDS
static constexpr int DIRECT = 512;
static constexpr int CHUNK = 32;
static constexpr int ZERO_ROWS = 8, IN_FLIGHT = 4;

struct SortPlan {
  int bits, passes;   // of a digit, digits
  int run_keys, runs;
};
static SortPlan sort_plan(int N, int V) {
  SortPlan p;
  int bits = 1;
  while (bits < 31 && (V >> bits) != 0) bits++;  // keys 0 .. V
  p.passes = (bits + SORT_BITS - 1) / SORT_BITS;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.run_keys = RUN_KEYS;
  if (N > RUN_KEYS * MOST_RUNS) p.run_keys = ((N + MOST_RUNS - 1) / MOST_RUNS + RUN_KEYS - 1) / RUN_KEYS * RUN_KEYS;
  p.runs = (N + p.run_keys - 1) / p.run_keys;
  return p;
}

// The lanes that have the same digit as this one.  Lanes without a key (ok false) match nobody.
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

// One pass over a workgroup's keys: `waves` wavefronts with `per_wave` consecutive keys each (a multiple of 64).  get(k): key and position k of the run
// (k < n); next: where each digit's next key goes, by wavefront; put(to, key, position).
template <typename Get, typename Put>
__device__ __forceinline__ void place_keys(int n, int per_wave, int shift, int bits, volatile unsigned* next, Get get, Put put) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int k0 = wave * per_wave, k1 = min(n, k0 + per_wave);
  for (int k = k0; k < k1; k += 64) {
    const bool ok = k + lane < k1;
    unsigned key = 0, pos = 0;
    if (ok) get(k + lane, key, pos);
    const unsigned digit = (key >> shift) & ((1u << bits) - 1);
    const unsigned long long m = same_digit(digit, bits, ok);
    const int rank = below(m);
    unsigned to = 0;
    if (ok) to = next[digit] + rank;
    __builtin_amdgcn_wave_barrier();  // (one wavefront: its LDS operations are in order)
    if (ok && rank == 0) next[digit] = to + (unsigned)__popcll(m);
    __builtin_amdgcn_wave_barrier();
    if (ok) put(to, key, pos);
  }
}

// Exclusive prefix sums over 256 values, one to a thread of the first 256; `tmp`: 4 words of LDS.
__device__ __forceinline__ unsigned scan256(unsigned x, unsigned* tmp) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  unsigned inc = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned y = __shfl_up(inc, o, 64);
    if (lane >= o) inc += y;
  }
  if (wave < 4 && lane == 63) tmp[wave] = inc;
  __syncthreads();
  unsigned before = 0;
  for (int k = 0; k < 4; k++)
    if (k < wave) before += tmp[k];
  return before + inc - x;
}

// What workgroups beyond the sort's do in a launch of it.  held: a byte for each row of the table, NULL: there are none.
struct ZeroRows {
  uint8_t* held;
  float* table;
  int D;
  long long first, end;  // the first pass: bytes to clear (16 to a thread); later: rows to look at, ZERO_ROWS to a wavefront
  unsigned blocks(int threads, bool rows) const { return (unsigned)((end - first + (rows ? threads / 64 * ZERO_ROWS : threads * 16) - 1) / (rows ? threads / 64 * ZERO_ROWS : threads * 16)); }
};
__device__ __forceinline__ void clear_held(const ZeroRows& z, int block) {
  const long long at = ((long long)block * blockDim.x + threadIdx.x) * 16;
  if (at < z.end) *reinterpret_cast<uint4*>(z.held + at) = make_uint4(0u, 0u, 0u, 0u);
}
__device__ __forceinline__ void zero_rows(const ZeroRows& z, int block) {
  const int lane = threadIdx.x & 63;
  const long long r0 = z.first + ((long long)block * (blockDim.x / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * ZERO_ROWS;
  unsigned long long free_ = __builtin_amdgcn_ballot_w64(lane < ZERO_ROWS && r0 + lane < z.end && z.held[min(r0 + lane, z.end - 1)] == 0);
  for (; free_; free_ &= free_ - 1) {
    float* row = z.table + (size_t)(r0 + __builtin_ctzll(free_)) * z.D;
    if (z.D % 4 == 0) {
      Vec16<float> o;
      o.raw = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int d = lane * 4; d < z.D; d += 256) o.store_nt(row + d);
    } else {
      for (int d = lane; d < z.D; d += 64) row[d] = 0.f;
    }
  }
}

// counts[run * BINS + digit].  in_key NULL: the first pass, keys from the tokens.
__global__ __launch_bounds__(256) void sort_count_kernel(int N, int V, int shift, int bits, int run_keys, int runs, const int32_t* __restrict__ tokens,
                                                         const uint32_t* __restrict__ in_key, uint32_t* __restrict__ counts, ZeroRows z) {
  if ((int)blockIdx.x >= runs) {
    if (in_key) zero_rows(z, blockIdx.x - runs);
    else clear_held(z, blockIdx.x - runs);
    return;
  }
  __shared__ unsigned hist[BINS];
  hist[threadIdx.x] = 0;
  __syncthreads();
  const long long k0 = (long long)blockIdx.x * run_keys;
  for (int k = threadIdx.x; k < run_keys && k0 + k < N; k += 256)
    atomicAdd(&hist[((in_key ? in_key[k0 + k] : key_of(tokens[k0 + k], V)) >> shift) & ((1u << bits) - 1)], 1u);
  __syncthreads();
  counts[blockIdx.x * BINS + threadIdx.x] = hist[threadIdx.x];
}

// in_key, in_pos NULL: the first pass, positions in order.
static constexpr int PLACE_WAVES = RUN_KEYS / 64;
__global__ __launch_bounds__(64 * PLACE_WAVES) void sort_place_kernel(int N, int V, int shift, int bits, int run_keys, int runs, const int32_t* __restrict__ tokens,
                                                                      const uint32_t* __restrict__ in_key, const uint32_t* __restrict__ in_pos,
                                                                      const uint32_t* __restrict__ counts, uint32_t* __restrict__ out_key,
                                                                      uint32_t* __restrict__ out_pos, ZeroRows z) {
  if ((int)blockIdx.x >= runs) {
    zero_rows(z, blockIdx.x - runs);
    return;
  }
  constexpr int QUARTERS = PLACE_WAVES * 64 / BINS;
  __shared__ unsigned next[PLACE_WAVES][BINS];
  __shared__ unsigned part[2][QUARTERS][BINS], tmp[4];
  const int run = blockIdx.x, wave = threadIdx.x >> 6, d = threadIdx.x % BINS, quarter = threadIdx.x / BINS;
  const long long k0 = (long long)run * run_keys;
  const int n = (int)min((long long)run_keys, N - k0), per_wave = run_keys / PLACE_WAVES;
  for (int i = threadIdx.x; i < PLACE_WAVES * BINS; i += 64 * PLACE_WAVES) (&next[0][0])[i] = 0;
  // keys of digit d in the runs before this one, and in all
  unsigned before = 0, total = 0;
#pragma unroll 8
  for (int r = quarter; r < runs; r += QUARTERS) {
    const unsigned c = counts[r * BINS + d];
    if (r < run) before += c;
    total += c;
  }
  part[0][quarter][d] = before;
  part[1][quarter][d] = total;
  __syncthreads();
  for (int k = threadIdx.x & 63; k < per_wave && wave * per_wave + k < n; k += 64) {
    const long long at = k0 + wave * per_wave + k;
    atomicAdd(&next[wave][((in_key ? in_key[at] : key_of(tokens[at], V)) >> shift) & ((1u << bits) - 1)], 1u);
  }
  before = total = 0;
#pragma unroll
  for (int q = 0; q < QUARTERS; q++) {
    before += part[0][q][d];
    total += part[1][q][d];
  }
  const unsigned start = scan256(total, tmp) + before;  // (of the first 256 threads; what the others have is not used)
  __syncthreads();
  if (threadIdx.x < BINS) {
    unsigned x = start;
#pragma unroll
    for (int w = 0; w < PLACE_WAVES; w++) {
      const unsigned c = next[w][d];
      next[w][d] = x;
      x += c;
    }
  }
  __syncthreads();
  place_keys(
      n, per_wave, shift, bits, next[wave],
      [&](int k, unsigned& key, unsigned& pos) {
        key = in_key ? in_key[k0 + k] : key_of(tokens[k0 + k], V);
        pos = in_pos ? in_pos[k0 + k] : (unsigned)(k0 + k);
        if (z.held && !in_key && key < (unsigned)V) z.held[key] = 1;  // (whoever holds it writes the same)
      },
      [&](unsigned to, unsigned key, unsigned pos) {
        out_key[to] = key;
        out_pos[to] = pos;
      });
}

// All passes by one workgroup, keys in LDS.
__global__ __launch_bounds__(1024) void sort_small_kernel(int N, int V, int bits, int passes, const int32_t* __restrict__ tokens,
                                                          uint32_t* __restrict__ out_key, uint32_t* __restrict__ out_pos) {
  extern __shared__ unsigned lds[];
  unsigned* next = lds;                // [16][BINS]
  unsigned* tmp = next + 16 * BINS;    // [16]
  unsigned* key[2] = {tmp + 16, tmp + 16 + N};
  unsigned* pos[2] = {tmp + 16 + 2 * N, tmp + 16 + 3 * N};
  const int wave = threadIdx.x >> 6, per_wave = ((N + 15) / 16 + 63) / 64 * 64;
  for (int k = threadIdx.x; k < N; k += 1024) {
    key[0][k] = key_of(tokens[k], V);
    pos[0][k] = k;
  }
  for (int p = 0; p < passes; p++) {
    const int shift = p * bits;
    const unsigned *ik = key[p & 1], *ip = pos[p & 1];
    for (int i = threadIdx.x; i < 16 * BINS; i += 1024) next[i] = 0;
    __syncthreads();
    for (int k = wave * per_wave + (threadIdx.x & 63); k < min(N, (wave + 1) * per_wave); k += 64)
      atomicAdd(&next[wave * BINS + ((ik[k] >> shift) & ((1u << bits) - 1))], 1u);
    __syncthreads();
    unsigned total = 0;
    if (threadIdx.x < BINS)
      for (int w = 0; w < 16; w++) total += next[w * BINS + threadIdx.x];
    unsigned x = scan256(total, tmp);
    if (threadIdx.x < BINS)
      for (int w = 0; w < 16; w++) {
        const unsigned c = next[w * BINS + threadIdx.x];
        next[w * BINS + threadIdx.x] = x;
        x += c;
      }
    __syncthreads();
    unsigned* ok = p + 1 < passes ? key[(p + 1) & 1] : out_key;
    unsigned* op = p + 1 < passes ? pos[(p + 1) & 1] : out_pos;
    place_keys(
        N, per_wave, shift, bits, next + wave * BINS,
        [&](int k, unsigned& a, unsigned& b) {
          a = ik[k];
          b = ip[k];
        },
        [&](unsigned to, unsigned a, unsigned b) {
          ok[to] = a;
          op[to] = b;
        });
    __syncthreads();
  }
}

// ---- sums -------------------------------------------------------------------------------------------
// A wavefront's piece of a row: STEPS x 64 vectors of E elements, from feature d0 on.  Loads beyond the row are loads of its end again: without
// branches, those of several rows are in flight together.
template <int E, int STEPS>
struct Piece {
  static constexpr int WIDTH = STEPS * 64 * E;
  float x[STEPS][E];
  int at[STEPS];  // features of this lane
  __device__ __forceinline__ Piece(int d0) {
#pragma unroll
    for (int s = 0; s < STEPS; s++) {
      at[s] = d0 + (s * 64 + (threadIdx.x & 63)) * E;
#pragma unroll
      for (int e = 0; e < E; e++) x[s][e] = 0.f;
    }
  }
  template <typename T>
  using Vec = std::conditional_t<E == 1, T, std::conditional_t<sizeof(T) == 4, float4, uint2>>;
  template <int R, typename T>
  __device__ __forceinline__ void load(Vec<T> (&v)[R][STEPS], const T* const (&row)[R], int D) const {
#pragma unroll
    for (int r = 0; r < R; r++)
#pragma unroll
      for (int s = 0; s < STEPS; s++) v[r][s] = *reinterpret_cast<const Vec<T>*>(row[r] + min(at[s], D - E));
  }
  template <typename T>
  __device__ __forceinline__ void add(const Vec<T> (&v)[STEPS]) {
#pragma unroll
    for (int s = 0; s < STEPS; s++) {
      if constexpr (E == 1) {
        x[s][0] += to_f(v[s]);
      } else if constexpr (sizeof(T) == 4) {
        x[s][0] += v[s].x; x[s][1] += v[s].y; x[s][2] += v[s].z; x[s][3] += v[s].w;
      } else {
        x[s][0] += __uint_as_float(v[s].x << 16); x[s][1] += __uint_as_float(v[s].x & 0xffff0000u);
        x[s][2] += __uint_as_float(v[s].y << 16); x[s][3] += __uint_as_float(v[s].y & 0xffff0000u);
      }
    }
  }
  // += R rows, in order
  template <int R, typename T>
  __device__ __forceinline__ void add_rows(const T* const (&row)[R], int D) {
    Vec<T> v[R][STEPS];
    load(v, row, D);
#pragma unroll
    for (int r = 0; r < R; r++) add<T>(v[r]);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int s = 0; s < STEPS; s++)
#pragma unroll
      for (int e = 0; e < E; e++) x[s][e] = 0.f;
  }
  // scale, add to what is there where asked, store
  __device__ __forceinline__ void store(float* __restrict__ row, int D, float scale, bool accumulate) const {
#pragma unroll
    for (int s = 0; s < STEPS; s++) {
      if (at[s] >= D) continue;
      float* p = row + at[s];
      if constexpr (E == 1) {
        *p = accumulate ? fmaf(x[s][0], scale, *p) : x[s][0] * scale;
      } else {
        Vec16<float> o;
        o.raw = accumulate ? *reinterpret_cast<const float4*>(p) : make_float4(0.f, 0.f, 0.f, 0.f);
        o.raw.x = fmaf(x[s][0], scale, o.raw.x); o.raw.y = fmaf(x[s][1], scale, o.raw.y);
        o.raw.z = fmaf(x[s][2], scale, o.raw.z); o.raw.w = fmaf(x[s][3], scale, o.raw.w);
        o.store_nt(p);
      }
    }
  }
};

// acc += the rows of the positions in lanes from .. from + n - 1 of `mine`, four (eight) in flight.
template <bool EIGHT = false, typename T, int E, int STEPS>
__device__ __forceinline__ void add_lanes(Piece<E, STEPS>& acc, const T* __restrict__ dout, int D, int mine, int from, int n) {
  auto row = [&](int i) { return dout + (size_t)(unsigned)__builtin_amdgcn_readlane(mine, from + i) * D; };
  int i = 0;
  if constexpr (EIGHT)
    for (; i + 8 <= n; i += 8) {
      const T* const r[8] = {row(i), row(i + 1), row(i + 2), row(i + 3), row(i + 4), row(i + 5), row(i + 6), row(i + 7)};
      acc.add_rows(r, D);
    }
  for (; i + 4 <= n; i += 4) {
    const T* const r[4] = {row(i), row(i + 1), row(i + 2), row(i + 3)};
    acc.add_rows(r, D);
  }
  for (; i < n; i++) {
    const T* const r[1] = {row(i)};
    acc.add_rows(r, D);
  }
}
// acc += the rows of positions pos[k0 .. k1)
template <typename T, int E, int STEPS>
__device__ __forceinline__ void add_positions(Piece<E, STEPS>& acc, const T* __restrict__ dout, int D, const uint32_t* __restrict__ pos, int k0, int k1) {
  const int lane = threadIdx.x & 63;
  for (int k = k0; k < k1; k += 64) {
    const int n = min(64, k1 - k);
    add_lanes(acc, dout, D, (int)(lane < n ? pos[k + lane] : 0u), 0, n);
  }
}

__device__ __forceinline__ bool whole_chunk(const uint32_t* __restrict__ key, int N, int V, int c) {
  const int k = c * CHUNK;
  return c >= 0 && k + CHUNK <= N && key[k] < (unsigned)V && key[k] == key[k + CHUNK - 1];
}

// A wavefront to a piece of a chunk's sum.  (All of the row to a wavefront is three times fewer of them at 768 features, each waiting for loads most of
// its time.)
template <typename T, int E>
__global__ __launch_bounds__(256) void embedding_chunk_kernel(int N, int V, int D, Divider pieces, const uint32_t* __restrict__ key,
                                                              const uint32_t* __restrict__ pos, const T* __restrict__ dout, float* __restrict__ sums) {
  const unsigned item = wide_block() * 4u + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), chunk = pieces(item);
  const int c = (int)chunk;
  if (!whole_chunk(key, N, V, c)) return;
  Piece<E, 1> acc((int)(item - chunk * pieces.d) * Piece<E, 1>::WIDTH);
  add_lanes<true>(acc, dout, D, (int)pos[c * CHUNK + (threadIdx.x & (CHUNK - 1))], 0, CHUNK);
  if (acc.at[0] < D)
#pragma unroll
    for (int e = 0; e < E; e++) sums[(size_t)c * D + acc.at[0] + e] = acc.x[0][e];
}

// The first of n sorted keys that is at least v: 64 candidates at a time.
__device__ __forceinline__ int lower_bound(const uint32_t* __restrict__ key, int n, unsigned v) {
  int lo = 0, hi = n;  // the answer is in [lo, hi]
  const int lane = threadIdx.x & 63;
  while (hi > lo) {
    const int step = (hi - lo + 63) / 64;
    const long long at = lo + (long long)lane * step;  // candidates lo, lo + step, ...
    const bool less = at < hi && key[at] < v;
    const int c = __popcll(__builtin_amdgcn_ballot_w64(less));  // sorted: the first c are less
    if (c == 0) break;
    hi = min(hi, lo + c * step);
    lo += (c - 1) * step + 1;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// A piece of the row of an id that has whole chunks, the first of them c: a workgroup.
template <typename T, int E>
__device__ __forceinline__ void long_row(int N, int D, int c, int piece, const uint32_t* __restrict__ key, const uint32_t* __restrict__ pos, const T* __restrict__ dout,
                                         const float* __restrict__ sums, float scale, bool accumulate, float* __restrict__ dtable, float* lds) {
  const unsigned v = key[c * CHUNK];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  // the positions before the first whole chunk: fewer than CHUNK
  const int back = c * CHUNK - 1 - lane;
  const int lo = c * CHUNK - __popcll(__builtin_amdgcn_ballot_w64(lane < CHUNK && back >= 0 && key[max(back, 0)] == v));
  const int hi = c * CHUNK + lower_bound(key + c * CHUNK, N - c * CHUNK, v + 1);
  const int c1 = hi / CHUNK, per = (c1 - c + 3) / 4;
  Piece<E, 1> acc(piece * Piece<E, 1>::WIDTH);
  if (wave == 0) add_positions(acc, dout, D, pos, lo, c * CHUNK);
  int k = c + wave * per;
  const int end = min(c1, k + per);
  auto row = [&](int i) { return sums + (size_t)i * D; };
  for (; k + 8 <= end; k += 8) {
    const float* const r[8] = {row(k), row(k + 1), row(k + 2), row(k + 3), row(k + 4), row(k + 5), row(k + 6), row(k + 7)};
    acc.add_rows(r, D);
  }
  for (; k < end; k++) {
    const float* const r[1] = {row(k)};
    acc.add_rows(r, D);
  }
  if (wave == 3) add_positions(acc, dout, D, pos, c1 * CHUNK, hi);
  if (wave > 0)
#pragma unroll
    for (int e = 0; e < E; e++) lds[((wave - 1) * E + e) * 64 + lane] = acc.x[0][e];
  __syncthreads();
  if (wave == 0) {
    for (int w = 0; w < 3; w++)
#pragma unroll
      for (int e = 0; e < E; e++) acc.x[0][e] += lds[(w * E + e) * 64 + lane];
    acc.store(dtable + (size_t)v * D, D, scale, accumulate);
  }
}

// The first `chunk_blocks` workgroups: pieces of rows with whole chunks.  The others, a wavefront to a piece: BY_ROW, of `per` rows of the table, with zeros
// where no position holds them; otherwise of `per` sorted positions, of which the first of an id adds (what comes without an id's first is another's).
template <typename T, int E, bool BY_ROW>
__global__ __launch_bounds__(256) void embedding_rows_kernel(int N, int V, int D, int per, int chunk_blocks, Divider pieces, const uint32_t* __restrict__ key,
                                                             const uint32_t* __restrict__ pos, const T* __restrict__ dout, const float* __restrict__ sums,
                                                             float scale, int accumulate, float* __restrict__ dtable) {
  __shared__ float lds[3 * E * 64];
  const int block = (int)wide_block();
  if (block < chunk_blocks) {
    const unsigned at = pieces((unsigned)block);
    const int c = (int)at;
    if (!whole_chunk(key, N, V, c)) return;
    if (whole_chunk(key, N, V, c - 1) && key[c * CHUNK - 1] == key[c * CHUNK]) return;  // not the first of its id
    long_row<T, E>(N, D, c, block - (int)(at * pieces.d), key, pos, dout, sums, scale, accumulate, dtable, lds);
    return;
  }
  const unsigned place = (unsigned)(block - chunk_blocks) * 4u + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int item = (int)pieces(place), d0 = (int)(place - item * pieces.d) * Piece<E, 1>::WIDTH;
  const int lane = threadIdx.x & 63;
  unsigned v, v_end, last;
  int lo, base, stop = N;  // positions are looked for from lo on; 64 sorted keys and their positions are in sight, from `base` on
  unsigned keys;
  int where;
  auto look = [&]() __attribute__((always_inline)) {
    keys = base + lane < N ? key[base + lane] : (unsigned)V;
    where = (int)(base + lane < N ? pos[base + lane] : 0u);
  };
  if (BY_ROW) {
    if ((long long)item * per >= V) return;
    v = item * per;
    v_end = min((unsigned)V, v + per);
    last = v_end - 1;
    lo = base = lower_bound(key, N, v);
    look();
  } else {
    if ((long long)item * per >= N) return;
    base = item * per;
    stop = min(N, base + per);
    const unsigned before = lane < per && base + lane > 0 && base + lane < N ? key[base + lane - 1] : (unsigned)V;
    look();
    const unsigned long long starts = __builtin_amdgcn_ballot_w64(lane < stop - base && keys != before);
    if (starts == 0) return;  // positions of an id that begins before: not this wavefront's
    lo = base + __builtin_ctzll(starts);
    v = __builtin_amdgcn_readlane(keys, lo - base);
    if (v >= (unsigned)V) return;
    last = min((unsigned)__builtin_amdgcn_readlane(keys, stop - base - 1), (unsigned)V - 1);
    v_end = V;
  }
  // Usually the rows' positions are few: then none has a whole chunk, and four positions' rows are loaded at a time, whichever row they belong to.
  const int m = __popcll(__builtin_amdgcn_ballot_w64(base + lane < N && keys <= last));
  if (m < CHUNK) {
    Piece<E, 1> acc(d0);
    unsigned at = v;
    for (int i = lo - base; i < m; i += IN_FLIGHT) {
      const T* r[IN_FLIGHT];
#pragma unroll
      for (int k = 0; k < IN_FLIGHT; k++) r[k] = dout + (size_t)(unsigned)__builtin_amdgcn_readlane(where, min(i + k, m - 1)) * D;
      typename Piece<E, 1>::template Vec<T> x[IN_FLIGHT][1];
      acc.load(x, r, D);
#pragma unroll
      for (int k = 0; k < IN_FLIGHT; k++) {
        if (i + k >= m) break;
        const unsigned id = __builtin_amdgcn_readlane(keys, i + k);
        while (at != id) {
          acc.store(dtable + (size_t)at * D, D, scale, accumulate);
          acc.clear();
          at = BY_ROW ? at + 1 : id;
        }
        acc.template add<T>(x[k]);
      }
    }
    for (; at <= last; at++) {  // (by position: the last id alone)
      acc.store(dtable + (size_t)at * D, D, scale, accumulate);
      acc.clear();
      if (!BY_ROW) break;
    }
    return;
  }
  while (v < v_end) {
    if (lo - base >= 64 - CHUNK) {
      base = lo;
      look();
    }
    // the run [lo, hi) of id v; one that reaches the end of what is in sight holds a whole chunk or ends there
    const int n = __popcll(__builtin_amdgcn_ballot_w64(keys == v && base + lane >= lo));
    const bool beyond = lo + n == base + 64;
    const int hi = beyond ? lo + lower_bound(key + lo, N - lo, v + 1) : lo + n;
    if ((lo + CHUNK - 1) / CHUNK >= hi / CHUNK) {  // (others: a workgroup's)
      Piece<E, 1> acc(d0);
      if (beyond) add_positions(acc, dout, D, pos, lo, hi);
      else add_lanes(acc, dout, D, where, lo - base, hi - lo);
      acc.store(dtable + (size_t)v * D, D, scale, accumulate);
    }
    lo = hi;
    if (BY_ROW) {
      v++;
    } else {
      if (lo >= stop) return;
      v = __builtin_amdgcn_readfirstlane(key[lo]);
    }
  }
}

// Few positions: a wavefront to a row of the table (BY_ROW) or to a position, which does its id's row if it is the first that holds it.
template <typename T, int E, int STEPS, bool BY_ROW>
__global__ __launch_bounds__(256) void embedding_direct_kernel(int N, int V, int D, const int32_t* __restrict__ tokens, const T* __restrict__ dout, float scale,
                                                               int accumulate, float* __restrict__ dtable) {
  const int item = (int)wide_block() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (item >= (BY_ROW ? V : N)) return;
  const int v = BY_ROW ? item : __builtin_amdgcn_readfirstlane(tokens[item]);
  if (!BY_ROW && (v < 0 || v >= V)) return;
  unsigned long long hold[DIRECT / 64];  // which positions hold it
#pragma unroll
  for (int w = 0; w < DIRECT / 64; w++) {
    const int n = w * 64 + lane;
    hold[w] = __builtin_amdgcn_ballot_w64(n < N && tokens[min(n, N - 1)] == v);
  }
  if (!BY_ROW) {
    unsigned long long before = 0;
#pragma unroll
    for (int w = 0; w < DIRECT / 64; w++) {
      const int at = item - w * 64;
      before |= at >= 64 ? hold[w] : at > 0 ? hold[w] & ((1ull << at) - 1) : 0ull;
    }
    if (before) return;
  }
  for (int d0 = 0; d0 < D; d0 += Piece<E, STEPS>::WIDTH) {
    Piece<E, STEPS> acc(d0);
#pragma unroll
    for (int w = 0; w < DIRECT / 64; w++)
      for (unsigned long long m = hold[w]; m; m &= m - 1) {
        const T* const r[1] = {dout + (size_t)(w * 64 + __builtin_ctzll(m)) * D};
        acc.add_rows(r, D);
      }
    acc.store(dtable + (size_t)v * D, D, scale, accumulate);
  }
}

struct EmbeddingWs {
  size_t key[2], pos[2], counts, held, sums, total;
};
static EmbeddingWs embedding_ws(int N, int V, int D) {
  const SortPlan p = sort_plan(N, V);
  EmbeddingWs w = {};
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t r = o; o += (bytes + 255) / 256 * 256; return r; };
  if (N > DIRECT) {
    for (int i = 0; i < 2; i++) {
      w.key[i] = take((size_t)N * 4);
      w.pos[i] = take((size_t)N * 4);
    }
    w.counts = take((size_t)p.runs * BINS * 4);
    w.held = take(V);
    w.sums = take((size_t)(N / CHUNK) * D * 4);
  }
  w.total = o ? o : 256;  // (never none: a caller's empty allocation has no address)
  return w;
}
size_t embedding_bwd_ws_bytes(int N, int V, int D) { return embedding_ws(N, V, D).total; }

template <typename T, int E, int STEPS>
static int embedding_bwd_t(int N, int V, int D, const int32_t* tokens, const T* dout, float scale, float* dtable, bool accumulate, char* ws, hipStream_t s) {
  if (N <= DIRECT) {
    const dim3 grid = wide_grid(((accumulate ? N : V) + 3) / 4);
    if (accumulate) hipLaunchKernelGGL((embedding_direct_kernel<T, E, STEPS, false>), grid, dim3(256), 0, s, N, V, D, tokens, dout, scale, 1, dtable);
    else hipLaunchKernelGGL((embedding_direct_kernel<T, E, STEPS, true>), grid, dim3(256), 0, s, N, V, D, tokens, dout, scale, 0, dtable);
    FAX_LAUNCH_CHECK("embedding_bwd");
    return FAX_OK;
  }
  const SortPlan p = sort_plan(N, V);
  const EmbeddingWs w = embedding_ws(N, V, D);
  uint32_t *key = nullptr, *pos = nullptr;
  bool zeros = false;  // of rows without a position: written beside the sort
  if (N <= SMALL_KEYS) {
    key = (uint32_t*)(ws + w.key[0]);
    pos = (uint32_t*)(ws + w.pos[0]);
    const size_t lds = (16 * BINS + 16 + 4 * (size_t)N) * 4;
    FAX_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(sort_small_kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                (16 * BINS + 16 + 4 * SMALL_KEYS) * 4));
    hipLaunchKernelGGL(sort_small_kernel, dim3(1), dim3(1024), lds, s, N, V, p.bits, p.passes, tokens, key, pos);
  } else {
    uint32_t* counts = (uint32_t*)(ws + w.counts);
    zeros = !accumulate && p.passes > 1;
    ZeroRows z = {zeros ? (uint8_t*)(ws + w.held) : nullptr, dtable, D, 0, zeros ? V : 0};
    const int shares = 2 * (p.passes - 1);
    for (int i = 0; i < p.passes; i++) {
      uint32_t *ok = (uint32_t*)(ws + w.key[i & 1]), *op = (uint32_t*)(ws + w.pos[i & 1]);
      auto share = [&](int k) {  // of the rows, for one of the later digits' launches
        z.first = zeros && k >= 0 ? (long long)V * k / shares : 0;
        z.end = zeros && k >= 0 ? (long long)V * (k + 1) / shares : 0;
      };
      if (i > 0) share(2 * i - 2);
      hipLaunchKernelGGL(sort_count_kernel, dim3(p.runs + z.blocks(256, i > 0)), dim3(256), 0, s, N, V, i * p.bits, p.bits, p.run_keys, p.runs, tokens, key, counts, z);
      share(i > 0 ? 2 * i - 1 : -1);
      hipLaunchKernelGGL(sort_place_kernel, dim3(p.runs + z.blocks(64 * PLACE_WAVES, true)), dim3(64 * PLACE_WAVES), 0, s, N, V, i * p.bits, p.bits, p.run_keys, p.runs,
                         tokens, key, pos, counts, ok, op, z);
      key = ok;
      pos = op;
    }
  }
  float* sums = (float*)(ws + w.sums);
  const int chunks = N / CHUNK;
  const Divider pieces((D + Piece<E, 1>::WIDTH - 1) / Piece<E, 1>::WIDTH);
  hipLaunchKernelGGL((embedding_chunk_kernel<T, E>), wide_grid(((unsigned long long)chunks * pieces.d + 3) / 4), dim3(256), 0, s, N, V, D, pieces, key, pos, dout, sums);
  const bool by_row = !accumulate && !zeros;
  // Rows or positions of a wavefront, us at 768 features by 2, 4, 8 of them:  4000 positions, 50304 rows (by row) 44.6 48.0 50.4;  1000, 8192 (by
  // row) 18.5 18.4 19.0;  16384, 50304 (by position) 54.6 54.4 55.9;  65536, 50304  85.6 81.3 81.1;  262144, 50304  181 163 158;  200000, 1000  132 120 114
  const int per = by_row ? (V > 16384 ? 2 : 4) : N > 65536 ? 8 : 4;
  const unsigned long long items = (((unsigned long long)(by_row ? V : N) + per - 1) / per) * pieces.d;
  const int chunk_blocks = (int)(chunks * pieces.d);
  const dim3 grid = wide_grid(chunk_blocks + (items + 3) / 4);
  if (!by_row) hipLaunchKernelGGL((embedding_rows_kernel<T, E, false>), grid, dim3(256), 0, s, N, V, D, per, chunk_blocks, pieces, key, pos, dout, sums, scale, accumulate, dtable);
  else hipLaunchKernelGGL((embedding_rows_kernel<T, E, true>), grid, dim3(256), 0, s, N, V, D, per, chunk_blocks, pieces, key, pos, dout, sums, scale, 0, dtable);
  FAX_LAUNCH_CHECK("embedding_bwd");
  return FAX_OK;
}

int embedding_bwd(int dtype, int N, int V, int D, const int32_t* tokens, const void* dout, float scale, float* dtable, bool accumulate, void* ws,
                  hipStream_t s) {
  if (N == 0) return accumulate ? FAX_OK : fill_zero(dtable, (size_t)V * D * 4, s);
  Timed t_("embedding_bwd", WORK_BYTE, (double)N * D * (dtype == FAX_F32 ? 4.0 : 2.0) + (accumulate ? 8.0 * D * (N < V ? N : V) : 4.0 * V * D), s);
  // steps of a wavefront across a row: up to four, as even as they come out
  const int e = D % 4 == 0 ? 4 : 1, n = (D + 64 * e - 1) / (64 * e), passes = (n + 3) / 4, steps = (n + passes - 1) / passes;
  auto by_steps = [&](auto rows, auto vec) -> int {
    typedef std::remove_pointer_t<decltype(rows)> T;
    constexpr int E = decltype(vec)::value;
    char* w = (char*)ws;
    const T* d = (const T*)dout;
    switch (steps) {
      case 1: return embedding_bwd_t<T, E, 1>(N, V, D, tokens, d, scale, dtable, accumulate, w, s);
      case 2: return embedding_bwd_t<T, E, 2>(N, V, D, tokens, d, scale, dtable, accumulate, w, s);
      case 3: return embedding_bwd_t<T, E, 3>(N, V, D, tokens, d, scale, dtable, accumulate, w, s);
      default: return embedding_bwd_t<T, E, 4>(N, V, D, tokens, d, scale, dtable, accumulate, w, s);
    }
  };
  typedef std::integral_constant<int, 4> Four;
  typedef std::integral_constant<int, 1> One;
  if (dtype == FAX_F32) return e == 4 ? by_steps((float*)nullptr, Four{}) : by_steps((float*)nullptr, One{});
  return e == 4 ? by_steps((bf16_t*)nullptr, Four{}) : by_steps((bf16_t*)nullptr, One{});
}

}  // namespace fax
