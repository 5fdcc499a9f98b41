// Attention in a sliding window with sinks: the scalar kernels, one wavefront to a row, for any head width up to 256 and any
// alignment, and the choice between them and the matrix-core kernels.
//
// What the matrix-core kernels reach (products of visible pairs only; masked edges of tiles are on top): 8192 positions, 32 heads on 8 of 128, window 1024,
// sinks 4: forward 157 to 188 us (690 to 820 TFLOP/s), dQ 280 to 300 us (650 to 690), dK and dV 335 to 350 us (740 to 770), between a warm and a loaded chip; a
// large bf16 product of the same card 1211 to 1334 TFLOP/s.  8 x 2048 positions, 12 heads of 64, window 512: 59, 89 and 95 us: at width 64 there is
// half the matrix work to a score, and the softmax's instructions and waits are the rest.  Single tokens, 8 sequences of 32 heads on 8 of 128, window 4096: 29 us
// for the 134 MB of keys and values (4.6 TB/s) and 5 us for the join.
// The scalar kernels are for the sizes that nothing else takes: 2048 positions, 8 heads of 256, window 512: 7.9 ms forward, 32 ms backward (1 TFLOP/s); on the matrix cores 35 and 88 us.
#include <initializer_list>

#include "window_tiles.h"

namespace fax {

static constexpr int MAX_R = 4;  // 64-wide pieces of a head width of 256

// Rows in the order (sequence, query, head) or (sequence, key, key head): neighbours share what they stream.
template <typename T, int WHAT>  // 0 forward, 1 dQ, 2 dK and dV, 3 delta
__global__ __launch_bounds__(256) void window_rows_kernel(WindowArgs a) {
  const int lane = threadIdx.x & 63;
  const int heads = WHAT == 2 ? a.Hkv : a.H, S = WHAT == 2 ? a.Sk : a.Sq;
  const long long row = (long long)wide_block() * 4 + (threadIdx.x >> 6), rows = (long long)a.B * S * heads;
  if (row >= rows) return;
  const int h = (int)(row % heads), i = (int)(row / heads % S), b = (int)(row / heads / S);
  if constexpr (WHAT == 0) window_fwd_row<MAX_R, T>(a, b, i, h, lane);
  if constexpr (WHAT == 1) window_dq_row<MAX_R, T>(a, b, i, h, lane);
  if constexpr (WHAT == 2) window_dkv_row<MAX_R, T>(a, b, i, h, lane);
  if constexpr (WHAT == 3) {
    const T* o = strided_row((const T*)a.ctx, a.sc, b, i, h);
    const T* d = strided_row((const T*)a.dctx, a.sc, b, i, h);
    float s = 0.f;
    for (int k = lane; k < a.dh; k += 64) s = fmaf(to_f(o[k]), to_f(d[k]), s);
    s = wave_sum(s);
    if (lane == 0) a.delta[((long long)b * a.H + h) * a.Sq + i] = s;
  }
}

template <int WHAT>
static int rows_launch(const WindowArgs& a, int dtype, hipStream_t s) {
  const long long rows = (long long)a.B * (WHAT == 2 ? (long long)a.Sk * a.Hkv : (long long)a.Sq * a.H);
  const dim3 grid = wide_grid((rows + 3) / 4);
  if (dtype == FAX_F32) hipLaunchKernelGGL((window_rows_kernel<float, WHAT>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((window_rows_kernel<bf16_t, WHAT>), grid, dim3(256), 0, s, a);
  return FAX_OK;
}

static WindowArgs window_args(const FaxWindowDims& d) {
  WindowArgs a = {};
  a.B = d.B; a.Sq = d.Sq; a.Sk = d.Sk; a.H = d.H; a.Hkv = d.Hkv; a.group = d.H / d.Hkv; a.dh = d.dh;
  a.window = d.window < (1 << 30) ? d.window : 1 << 30;
  a.sinks = d.sinks;
  a.scale = (float)(1.0 / sqrt((double)d.dh));
  a.sq = d.q; a.skv = d.kv; a.sc = d.ctx;
  return a;
}

// Joins the parts that the workgroups of a cut row left, their sums undivided, with their reference points and denominators: one wavefront to a
// row.  octaves: of the reference points' unit; unit: of it in scaled scores.  What one wavefront loads at once are all parts' points and up to eight
// parts' sums.
template <int R, typename T>  // R: 64-wide pieces of a head
__global__ __launch_bounds__(256) void window_join_kernel(WindowArgs a, int splits, const float* __restrict__ part_o, const float2* __restrict__ part_ml,
                                                          float octaves, float unit) {
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 6), rows = (long long)a.B * a.Hkv * a.Sq * a.group;
  if (row >= rows) return;
  const int lane = threadIdx.x & 63;
  const long long per_head = (long long)a.Sq * a.group;
  const int bh = (int)(row / per_head), r = (int)(row % per_head);
  const int b = bh / a.Hkv, i = r / a.group, h = bh % a.Hkv * a.group + r % a.group;
  const float2* ml = part_ml + row * splits;
  const float* o = part_o + row * splits * a.dh;
  // part s's point and denominator in lane s
  const float2 mine = lane < splits ? ml[lane] : make_float2(-3.4028235e38f, 0.f);
  const float M = wave_max(mine.x), weight = __builtin_amdgcn_exp2f((mine.x - M) * octaves);
  const float L = wave_sum(mine.y * weight);
  float acc[R] = {};
  for (int s0 = 0; s0 < splits; s0 += 8) {  // (beyond the last part: loads of the last)
    float x[8][R];
#pragma unroll
    for (int k = 0; k < 8; k++) {
      const float* p = o + (long long)min(s0 + k, splits - 1) * a.dh;
#pragma unroll
      for (int c = 0; c < R; c++) x[k][c] = p[min(lane + 64 * c, a.dh - 1)];
    }
#pragma unroll
    for (int k = 0; k < 8; k++) {
      const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), s0 + k));
#pragma unroll
      for (int c = 0; c < R; c++) acc[c] = s0 + k < splits ? fmaf(x[k][c], w, acc[c]) : acc[c];
    }
  }
  bool odd = !(L <= 3.4028235e38f);
#pragma unroll
  for (int c = 0; c < R; c++) odd |= !(fabsf(acc[c]) <= 3.4028235e38f);
  if (__any(odd)) {
    window_fwd_row<R, T>(a, b, i, h, lane);
    return;
  }
  const bool none = L == 0.f;
  const float inv = none ? 0.f : 1.f / L;
  T* out = strided_row((T*)a.ctx, a.sc, b, i, h);
#pragma unroll
  for (int k = 0; k < R; k++) {
    const int d = lane + 64 * k;
    if (d < a.dh) out[d] = from_f<T>(acc[k] * inv);
  }
  if (lane == 0 && a.lse) a.lse[((long long)b * a.H + h) * a.Sq + i] = none ? -INFINITY : M * unit + logf(L);
}

// dQ of cut rows: the parts added in order, one wavefront to a row.  part_ds: the parts of delta (NULL: it is there already).
template <int R, typename T>
__global__ __launch_bounds__(256) void window_fold_dq_kernel(WindowArgs a, int splits, const float* __restrict__ part_dq, const float* __restrict__ part_ds) {
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 6), rows = (long long)a.B * a.Hkv * a.Sq * a.group;
  if (row >= rows) return;
  const int lane = threadIdx.x & 63;
  const long long per_head = (long long)a.Sq * a.group;
  const int bh = (int)(row / per_head), r = (int)(row % per_head);
  const int b = bh / a.Hkv, i = r / a.group, h = bh % a.Hkv * a.group + r % a.group;
  const float* o = part_dq + row * splits * a.dh;
  if (part_ds) {
    const float delta = wave_sum(lane < splits ? part_ds[row * splits + lane] : 0.f);
    if (lane == 0) a.delta[((long long)b * a.H + h) * a.Sq + i] = delta;
  }
  float acc[R] = {}, odd = 0.f;
#pragma unroll 8
  for (int s = 0; s < splits; s++)
#pragma unroll
    for (int c = 0; c < R; c++) acc[c] += o[(long long)s * a.dh + min(lane + 64 * c, a.dh - 1)];
#pragma unroll
  for (int c = 0; c < R; c++) odd = fmaf(acc[c], 0.f, odd);
  if (sizeof(T) == 2 && __any(odd != 0.f)) {  // (the fp32 kernels keep masked rows out of their sums)
    __threadfence();
    window_dq_row<R, T>(a, b, i, h, lane);
    return;
  }
  T* out = strided_row((T*)a.dq, a.sq, b, i, h);
#pragma unroll
  for (int k = 0; k < R; k++) {
    const int d = lane + 64 * k;
    if (d < a.dh) out[d] = from_f<T>(acc[k] * a.scale);
  }
}

// The parts of the cut tiles' keys, added in order: one wavefront to a key.
template <int R, typename T>
__global__ __launch_bounds__(256) void window_fold_kernel(WindowArgs a, KeyGrid kg, const float* __restrict__ parts) {
  const int from = kg.fold_from(), n = kg.fold_keys(a);
  const long long item = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (item >= (long long)n * a.B * a.Hkv) return;
  const int j = from + (int)(item % n), bh = (int)(item / n);
  const int splits = j < kg.sink_tiles * kg.keys ? kg.sink_splits : kg.rest_splits;
  float dk[R] = {}, dv[R] = {}, odd = 0.f;
#pragma unroll 4
  for (int p = 0; p < splits; p++) {
    const float* o = parts + kg.part(a, p, bh, j) * 2 * a.dh;
#pragma unroll
    for (int c = 0; c < R; c++) {
      dk[c] += o[min(lane + 64 * c, a.dh - 1)];
      dv[c] += o[a.dh + min(lane + 64 * c, a.dh - 1)];
    }
  }
#pragma unroll
  for (int c = 0; c < R; c++) odd = fmaf(dk[c], 0.f, fmaf(dv[c], 0.f, odd));
  const int b = bh / a.Hkv, hk = bh % a.Hkv;
  if (__any(odd != 0.f)) {
    window_dkv_row<R, T>(a, b, j, hk, lane);
    return;
  }
  T* ko = strided_row((T*)a.dk, a.skv, b, j, hk);
  T* vo = strided_row((T*)a.dv, a.skv, b, j, hk);
#pragma unroll
  for (int k = 0; k < R; k++) {
    const int d = lane + 64 * k;
    if (d < a.dh) {
      ko[d] = from_f<T>(dk[k] * a.scale);
      vo[d] = from_f<T>(dv[k]);
    }
  }
}

// Rows on 16 bytes, whole 16-byte chunks to a head, offsets within a tile of 64 rows in 32 bits.
static bool strides_fit(const FaxStrides& s, int unit) { return s.batch % unit == 0 && s.row % unit == 0 && s.head % unit == 0 && s.row <= (1 << 24); }

// Into how many parts a stream of `tiles` tiles is cut, with `blocks` workgroups: by an estimate in us.  tile: of a tile, part_tile: of a tile
// in a cut stream; at_once: workgroups that the chip works on side by side without slowing each other down; part_bytes: what a part writes and the joining
// kernel reads.  6 us and 0.04 to a part: the second kernel.
struct StreamCost { double tile, part_tile, at_once; bool whole_rounds; };
static int cut_stream(double blocks, long long tiles, const StreamCost& c, double part_bytes) {
  int best = 1;
  double least = tiles * c.tile;
  for (int n = 2; n <= 64 && n <= tiles; n++) {  // (64: a lane of the joining wavefront each)
    double rounds = blocks * n / c.at_once;
    if (rounds < 1.0) rounds = 1.0;
    else if (c.whole_rounds) rounds = ceil(rounds);
    const double us = 6.0 + 0.04 * n + (double)((tiles + n - 1) / n) * c.part_tile * rounds + part_bytes * n / 2.5e6;
    if (us < 0.97 * least) { least = us; best = n; }
  }
  return best;
}

// Measured, back to back in a graph, us by parts (bf16, heads on key heads x width, window; where there is one part, two groups where the rule has them):
//   forward  512 queries over 2048 keys, 8 on 8 x 128, 2048 (32 workgroups, 34 tiles)  1: 36  4: 28  8: 28  16: 30;  16 on 4 over 8192 (64)  37  37  36  47;
//            two of that (128)  38  4: 47  8: 56;  three (192)  40  2: 67;  16 on 4 x 64, 1024 (64, 18 tiles)  18  2: 29;  1024 of 16 x 64, 300 (128, 7)  13  24
//            tokens over 4096 keys, 32 on 8 x 128: one (8 workgroups)  79  4: 32  8: 20  16: 14  32: 11.7  64: 12.8;  four  81  34  23  21  25;  sixteen  82  52  51  55
//   backward, by parts of dQ's streams  4096 of 2 on 1 x 128, all (64 workgroups, up to 64 tiles)  146  2: 124  4: 99  8: 98  16: 110;  1024 of 16 x 64, 300  27  34  39
//             by those of dK and dV     the same two  231  151  110  99  111;  28  41  47
// and by groups of wavefronts, us with one | with two (forward; backward, where only dQ has them):
//   512 queries over 8192 keys, 16 on 4 x 128, 2048, of two (128 workgroups)  49.8 | 39.9; of four (256)  53.3 | 45.5;  four, x 64, 1024  22.5 | 19.6
//   1024 of 16 x 64, 300 (128, 7 tiles)  13.9 | 12.7; 28.2 | 27.8    1000 of 15 on 5 x 80, 300 (120)  17.7 | 15.3; 49.2 | 45.9
//   2048 of 16 x 64, 512 (256, 10 tiles)  17.8 | 15.9; 46.1 | 44.8   eight of 256 of 16 x 128, all (256, 4 tiles)  14.4 | 14.5; 39.2 | 40.9
//   eight of 128 of 16 x 128, all (128, 2 tiles)  11.0 | 11.3; 24.3 | 26.3
// Head width 256, by parts again:
//   forward  tokens over 4096 keys, 16 heads on 4: one  190  4: 72  8: 43  16: 28  32: 23  64: 21;  four  190  73  44  31  40  57;  sixteen  190  76  83
//            512 queries over them, window 2048 (64 workgroups)  74  2: 68  4: 51  8: 65;  2048 of 8 on 8, 512 (128)  34  43  57
//   backward, by parts of dQ's streams  2048 of 4 on 2, all (64)  177  134  115  132;  2048 of 8 on 8, 512 (128)  88  84  105;  two, 8 on 4 (256)  112  142
//             by those of dK and dV     the same three  218  149  114  125;  87  115  144;  111  137  164
static WindowPlan window_plan(const FaxWindowDims& d) {
  WindowPlan p = {};
  p.form = FAX_ATTENTION_SCALAR;
  p.waves = 1;
  p.fwd_groups = p.dq_groups = p.fwd_splits = p.dq_splits = p.sink_splits = p.rest_splits = 1;
  const int unit = d.dtype == FAX_F32 ? 4 : 8, group = d.H / d.Hkv;
  const long long heads = (long long)d.B * d.Hkv, rows = (long long)d.Sq * group;
  if (d.dh % unit == 0 && d.dh <= (d.dtype == FAX_F32 ? 128 : 256) && strides_fit(d.q, unit) && strides_fit(d.kv, unit) && strides_fit(d.ctx, unit) && rows < (1 << 30)) {
    const bool f32 = d.dtype == FAX_F32;
    p.form = f32 ? FAX_ATTENTION_F32 : d.dh == 64 || d.dh == 128 ? FAX_ATTENTION_MFMA : FAX_ATTENTION_EDGE;
    p.waves = !f32 && rows > 32 ? 4 : 1;
    const double blocks = (double)((rows + 32 * p.waves - 1) / (32 * p.waves) * heads), row_bytes = 8.0 * d.dh * rows * heads;
    const long long span = (rows < 32 * p.waves ? rows : 32 * p.waves) / group + 1;  // positions of a workgroup's rows
    const long long seen = (long long)d.window + d.sinks + span < d.Sk ? d.window + d.sinks + span : d.Sk;
    // A tile is 64 keys (queries), of fp32 a round of 32 for each of the workgroup's four wavefronts, which the matrix cores bound.
    const bool alone = !f32 && p.waves == 1;  // a wavefront with tiles of its own: its workgroups are two to a CU
    const int unit_keys = f32 ? 128 : 64;
    const double w = d.dh / 128.0;
    const bool wide = d.dh > 128;  // bf16: one workgroup to a CU, tiles twice as wide
    const StreamCost fwd = f32 ? StreamCost{1 + 3.4 * w, 1 + 3.4 * w, 256, false} : wide ? StreamCost{3.0, 3.5, 256, alone} : alone ? StreamCost{1.25, 1.25, 512, true} : StreamCost{1.35, 1.7, 384, false};
    const StreamCost dq = f32 ? StreamCost{1 + 5.1 * w, 1 + 5.1 * w, 256, false} : wide ? StreamCost{7.0, 7.0, 256, alone} : alone ? StreamCost{3.0, 3.0, 512, true} : StreamCost{2.0, 2.0, 384, false};
    const StreamCost dkv = f32 ? StreamCost{1 + 6.8 * w, 1 + 6.8 * w, 256, false} : wide ? StreamCost{5.0, 5.0, 256, false} : StreamCost{2.0, 2.0, 400, false};
    auto tiles = [&](long long keys) { return (keys + unit_keys - 1) / unit_keys; };
    p.fwd_splits = cut_stream(blocks, tiles(seen), fwd, row_bytes);
    p.dq_splits = cut_stream(blocks, tiles(seen), dq, row_bytes);
    // Two groups of wavefronts to a workgroup where there is one to a CU: one group's tiles do not fill it, and adding up takes a microsecond or two.
    if (p.waves == 4 && blocks <= 256 && !wide) {
      p.fwd_groups = p.fwd_splits == 1 && tiles(seen) >= 4 ? 2 : 1;
      p.dq_groups = p.dq_splits == 1 && tiles(seen) >= 6 ? 2 : 1;
    }
    // Keys: those among the sinks are seen by every later query, the others by a window's length of them.
    p.kv_keys = f32 ? 32 : WINDOW_DKV_KEYS;
    const long long n = (d.Sk + p.kv_keys - 1) / p.kv_keys, sinks = d.sinks < d.Sk ? d.sinks : d.Sk, all = tiles((long long)d.Sq * group);
    const long long usual = (long long)d.window + p.kv_keys + 64, stream = usual < d.Sq ? tiles(usual * group) : all;
    const double key_bytes = 16.0 * d.dh * p.kv_keys;  // of a tile
    p.sink_tiles = (int)((sinks + p.kv_keys - 1) / p.kv_keys);
    p.rest_splits = cut_stream((double)((n - p.sink_tiles) * heads), stream, dkv, key_bytes * (n - p.sink_tiles) * heads);
    const long long chain = (stream + p.rest_splits - 1) / p.rest_splits;
    if (p.sink_tiles > 0 && 2 * p.sink_tiles <= n) {  // as long as the others' parts, and no more of them than fill the chip several times over
      const long long parts = (all + chain - 1) / chain, room = 1 + 2048 / (p.sink_tiles * heads);
      p.sink_splits = (int)(parts < 64 && parts < room ? parts : room < 64 ? room : 64);
    } else {  // most keys are sinks: one kind of tile
      p.sink_tiles = 0;
      if (sinks > 0) p.rest_splits = cut_stream((double)(n * heads), all, dkv, key_bytes * n * heads);
    }
  }
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t r = o; o += (bytes + 255) / 256 * 256; return r; };
  // forward pass and backward pass take turns in the workspace
  const size_t all_rows = (size_t)d.B * d.H * d.Sq;
  if (p.fwd_splits > 1) {
    p.part_o = take(all_rows * p.fwd_splits * d.dh * 4);
    p.part_ml = take(all_rows * p.fwd_splits * 8);
  }
  const size_t fwd = o;
  o = 0;
  p.delta = take(all_rows * 4);
  if (p.dq_splits > 1) {
    p.part_dq = take(all_rows * p.dq_splits * d.dh * 4);
    p.part_ds = take(all_rows * p.dq_splits * 4);
  }
  if (p.sink_splits > 1 || p.rest_splits > 1) {
    const WindowArgs a = window_args(d);
    p.parts = take((size_t)KeyGrid(a, p).part_rows(a) * 2 * d.dh * 4);
  }
  p.total = o > fwd ? o : fwd;
  return p;
}
size_t window_ws_bytes(const FaxWindowDims& d) { return window_plan(d).total; }
void window_route(const FaxWindowDims& d, FaxWindowRoute* out) {
  const WindowPlan p = window_plan(d);
  out->form = p.form;
  out->waves = p.waves; out->fwd_groups = p.fwd_groups; out->dq_groups = p.dq_groups; out->fwd_splits = p.fwd_splits; out->dq_splits = p.dq_splits;
  out->sink_splits = p.sink_splits; out->key_splits = p.rest_splits;
}
static bool on16(std::initializer_list<const void*> p) {
  uintptr_t all = 0;
  for (const void* x : p) all |= (uintptr_t)x;
  return (all & 15) == 0;
}

// Pairs of a whole batch without k_len and q_pos: what the timing report counts.
static double window_pairs(const FaxWindowDims& d) {
  double n = 0.0;
  const long long first = (long long)d.Sk - d.Sq;
  // query at p sees min(p + 1, window) keys and the sinks before them
  for (int part = 0; part < 2; part++) {
    const long long cap = part ? d.sinks : d.window, shift = part ? d.window : 0;
    const long long a = first + 1 - shift, b = (long long)d.Sk - shift;  // terms min(max(x, 0), cap), x = a .. b
    const long long lo = a > 1 ? a : 1, mid = b < cap ? b : cap;
    if (mid >= lo) n += 0.5 * (double)(lo + mid) * (double)(mid - lo + 1);
    const long long flat = (lo > cap + 1 ? lo : cap + 1);
    if (b >= flat) n += (double)cap * (double)(b - flat + 1);
  }
  return n * d.B * d.H;
}

int window_fwd(const FaxWindowDims& d, const void* q, const void* k, const void* v, const int32_t* q_pos, const int32_t* k_len, void* ctx,
               float* lse, void* ws, hipStream_t s) {
  Timed t_("window_attention_fwd", WORK_FLOP, 4.0 * d.dh * window_pairs(d), s);
  WindowArgs a = window_args(d);
  a.q = q; a.k = k; a.v = v; a.q_pos = q_pos; a.k_len = k_len; a.ctx = ctx; a.lse = lse;
  const WindowPlan p = window_plan(d);
  char* w = (char*)ws;
  if (p.form == FAX_ATTENTION_SCALAR || !on16({q, k, v, ctx})) {
    FAX_TRY(rows_launch<0>(a, d.dtype, s));
  } else {
    float* part_o = (float*)(w + p.part_o);
    float2* part_ml = (float2*)(w + p.part_ml);
    if (p.form == FAX_ATTENTION_F32) FAX_TRY(window_fwd_f32(a, p.fwd_splits, part_o, part_ml, s));
    else FAX_TRY(window_fwd_mfma(a, p.waves, p.fwd_groups, p.fwd_splits, part_o, part_ml, s));
    if (p.fwd_splits > 1) {
      const float log2e = 1.4426950408889634f;
      const dim3 grid((unsigned)(((long long)a.B * a.H * a.Sq + 3) / 4));
      if (d.dtype == FAX_F32) hipLaunchKernelGGL((window_join_kernel<2, float>), grid, dim3(256), 0, s, a, p.fwd_splits, part_o, part_ml, log2e, 1.f);
      else {
        if (d.dh <= 128) hipLaunchKernelGGL((window_join_kernel<2, bf16_t>), grid, dim3(256), 0, s, a, p.fwd_splits, part_o, part_ml, a.scale * log2e, a.scale);
        else hipLaunchKernelGGL((window_join_kernel<4, bf16_t>), grid, dim3(256), 0, s, a, p.fwd_splits, part_o, part_ml, a.scale * log2e, a.scale);
      }
    }
  }
  FAX_LAUNCH_CHECK("window_attention_fwd");
  return FAX_OK;
}

int window_bwd(const FaxWindowDims& d, const void* q, const void* k, const void* v, const int32_t* q_pos, const int32_t* k_len, const void* ctx,
               const float* lse, const void* dctx, void* dq, void* dk, void* dv, void* ws, hipStream_t s) {
  Timed t_("window_attention_bwd", WORK_FLOP, 10.0 * d.dh * window_pairs(d), s);
  WindowArgs a = window_args(d);
  a.q = q; a.k = k; a.v = v; a.q_pos = q_pos; a.k_len = k_len; a.ctx = const_cast<void*>(ctx); a.lse = const_cast<float*>(lse);
  const WindowPlan p = window_plan(d);
  char* w = (char*)ws;
  a.dctx = dctx; a.dq = dq; a.dk = dk; a.dv = dv; a.delta = (float*)(w + p.delta);
  if (p.form == FAX_ATTENTION_SCALAR || !on16({q, k, v, ctx, dctx, dq, dk, dv})) {
    FAX_TRY(rows_launch<3>(a, d.dtype, s));
    FAX_TRY(rows_launch<1>(a, d.dtype, s));
    FAX_TRY(rows_launch<2>(a, d.dtype, s));
  } else {
    float *parts = (float*)(w + p.parts), *part_dq = (float*)(w + p.part_dq), *part_ds = (float*)(w + p.part_ds);
    const unsigned row_blocks = (unsigned)(((long long)a.B * a.H * a.Sq + 3) / 4);
    if (p.form == FAX_ATTENTION_F32) {
      FAX_TRY(rows_launch<3>(a, d.dtype, s));
      FAX_TRY(window_bwd_f32(a, p, part_dq, parts, s));
      if (p.dq_splits > 1) hipLaunchKernelGGL((window_fold_dq_kernel<2, float>), dim3(row_blocks), dim3(256), 0, s, a, p.dq_splits, part_dq, (const float*)nullptr);
    } else {
      // dQ first: it also leaves delta, which dK and dV need
      FAX_TRY(window_dq_mfma(a, p.waves, p.dq_groups, p.dq_splits, part_dq, part_ds, s));
      if (p.dq_splits > 1) {
        if (d.dh <= 128) hipLaunchKernelGGL((window_fold_dq_kernel<2, bf16_t>), dim3(row_blocks), dim3(256), 0, s, a, p.dq_splits, part_dq, part_ds);
        else hipLaunchKernelGGL((window_fold_dq_kernel<4, bf16_t>), dim3(row_blocks), dim3(256), 0, s, a, p.dq_splits, part_dq, part_ds);
      }
      FAX_TRY(window_dkv_mfma(a, p, parts, s));
    }
    if (p.sink_splits > 1 || p.rest_splits > 1) {
      const KeyGrid kg(a, p);
      const dim3 grid((unsigned)(((long long)kg.fold_keys(a) * a.B * a.Hkv + 3) / 4));
      if (d.dtype == FAX_F32) hipLaunchKernelGGL((window_fold_kernel<2, float>), grid, dim3(256), 0, s, a, kg, parts);
      else {
        if (d.dh <= 128) hipLaunchKernelGGL((window_fold_kernel<2, bf16_t>), grid, dim3(256), 0, s, a, kg, parts);
        else hipLaunchKernelGGL((window_fold_kernel<4, bf16_t>), grid, dim3(256), 0, s, a, kg, parts);
      }
    }
  }
  FAX_LAUNCH_CHECK("window_attention_bwd");
  return FAX_OK;
}

}  // namespace fax
