// Attention in a sliding window with sinks: what its kernels share.  The arguments of a pass, which keys a run of queries can see and
// which queries a run of keys, and single rows by one wavefront with scalar FMAs: the kernels for head widths and alignments that the matrix
// cores do not take, and what those run again for a row that came out as NaN (a masked pair enters a matrix product as a zero factor, which an
// infinity or NaN on the other side turns into NaN; the rows here touch visible pairs only).
//
// Query i stands at p = pos0 + i and sees the keys [0, sinks) and (p - window, p], both below k_len.  Runs of queries [p0, p1] therefore see at most
// two ranges of keys, the sinks and the window, and runs of keys [j0, j1) one range of queries.
#pragma once
#include "attn_rows.h"

namespace fax {

struct WindowArgs {
  int B, Sq, Sk, H, Hkv, group, dh, window, sinks;  // group: query heads to a key head; window at most 2^30
  float scale;
  FaxStrides sq, skv, sc;
  const int32_t *q_pos, *k_len;
  const void *q, *k, *v;
  void* ctx;
  float* lse;
  const void* dctx;
  void *dq, *dk, *dv;
  float* delta;
};

// How a size is run (kernels_window.hip), and where its parts lie in the workspace.
struct WindowPlan {
  int form;                                    // FAX_ATTENTION_*
  int waves, fwd_groups, dq_groups, fwd_splits, dq_splits;  // wavefronts of a group of a workgroup of rows, groups; parts of a row's stream of keys
  int kv_keys, sink_tiles, sink_splits, rest_splits;  // keys of a workgroup; tiles of them with sinks, parts of their streams of queries and of the others'
  size_t delta, part_o, part_ml, part_dq, part_ds, parts, total;
};
int window_fwd_mfma(const WindowArgs& a, int waves, int groups, int splits, float* part_o, void* part_ml, hipStream_t s);
int window_dq_wide(const WindowArgs& a, int waves, int splits, float* part_dq, float* part_ds, hipStream_t s);  // head widths above 128
int window_dq_mfma(const WindowArgs& a, int waves, int groups, int splits, float* part_dq, float* part_ds, hipStream_t s);
static constexpr int WINDOW_DKV_KEYS = 64;  // keys of a workgroup
int window_dkv_mfma(const WindowArgs& a, const WindowPlan& p, float* parts, hipStream_t s);
int window_fwd_f32(const WindowArgs& a, int splits, float* part_o, void* part_ml, hipStream_t s);
int window_bwd_f32(const WindowArgs& a, const WindowPlan& p, float* part_dq, float* parts, hipStream_t s);

struct WindowSeq {
  int pos0, k_len;
  __device__ __forceinline__ WindowSeq(const WindowArgs& a, int b) {
    // (b is the same for a wavefront: what follows from these may stay in scalar registers)
    k_len = __builtin_amdgcn_readfirstlane(a.k_len ? min(max(a.k_len[b], 0), a.Sk) : a.Sk);
    pos0 = __builtin_amdgcn_readfirstlane(a.q_pos ? min(max(a.q_pos[b], -(1 << 30)), (1 << 30) - a.Sq) : a.Sk - a.Sq);
  }
};

// Keys that some query at p0 .. p1 sees: [0, sink_end) and [lo, end), sink_end <= lo <= end.
struct KeyRanges {
  int sink_end, lo, end;
  __device__ __forceinline__ KeyRanges(const WindowArgs& a, const WindowSeq& s, int p0, int p1) {
    end = max(0, min(s.k_len, p1 + 1));
    sink_end = min(a.sinks, end);
    lo = min(end, max(sink_end, p0 - a.window + 1));
  }
};

// Queries that some key of [j0, j1) is visible to: [i0, i1).
struct QueryRange {
  int i0, i1;
  __device__ __forceinline__ QueryRange(const WindowArgs& a, const WindowSeq& s, int j0, int j1) {
    j1 = min(j1, s.k_len);
    i0 = min(a.Sq, max(0, j0 - s.pos0));
    const long long last = j0 < a.sinks ? a.Sq : (long long)j1 - 1 + a.window - s.pos0;  // one past
    i1 = j1 <= j0 ? i0 : (int)min((long long)a.Sq, max((long long)i0, last));
  }
};

__device__ __forceinline__ bool window_sees(const WindowArgs& a, const WindowSeq& s, int p, int j) {
  return j < s.k_len && j <= p && (j > p - a.window || j < a.sinks);
}

template <typename T>
__device__ __forceinline__ T* strided_row(T* p, const FaxStrides& s, long long b, long long r, long long h) {
  return p + b * s.batch + r * s.row + h * s.head;
}

// One query.  R: 64-wide pieces of the head width.
template <int R, typename T>
__device__ __forceinline__ void window_fwd_row(const WindowArgs& a, int b, int i, int h, int lane) {
  const WindowSeq sq(a, b);
  const int p = sq.pos0 + i, dh = a.dh, hk = h / a.group;
  const KeyRanges ks(a, sq, p, p);
  const T* q = strided_row((const T*)a.q, a.sq, b, i, h);
  const T* k = strided_row((const T*)a.k, a.skv, b, 0, hk);
  const T* v = strided_row((const T*)a.v, a.skv, b, 0, hk);
  float m = -INFINITY, l = 0.f, acc[R];
#pragma unroll
  for (int r = 0; r < R; r++) acc[r] = 0.f;
  for (int part = 0; part < 2; part++) {
    const int from = part ? ks.lo : 0, to = part ? ks.end : ks.sink_end;
    for (int j0 = from; j0 < to; j0 += 64) {
      const int j = j0 + lane;
      const bool ok = j < to;
      const float sc = ok ? dot_row(q, k + (long long)j * a.skv.row, dh) * a.scale : -INFINITY;
      const float mn = fmaxf(m, wave_max(sc));
      const float ref = mn == -INFINITY ? 0.f : mn;  // (scores that are all -infinity)
      const float e = ok ? expf(sc - ref) : 0.f, corr = expf(m - ref);
      l = l * corr + wave_sum(e);
#pragma unroll
      for (int r = 0; r < R; r++) acc[r] *= corr;
      const int nj = min(64, to - j0);
      for (int jj = 0; jj < nj; jj++) {
        const float ej = __shfl(e, jj, 64);
        const T* vr = v + (long long)(j0 + jj) * a.skv.row;
#pragma unroll
        for (int r = 0; r < R; r++) {
          const int d = lane + 64 * r;
          if (d < dh) acc[r] = fmaf(ej, to_f(vr[d]), acc[r]);
        }
      }
      m = mn;
    }
  }
  const bool none = ks.sink_end + ks.end - ks.lo == 0;
  const float inv = none ? 0.f : 1.f / l;
  T* out = strided_row((T*)a.ctx, a.sc, b, i, h);
#pragma unroll
  for (int r = 0; r < R; r++) {
    const int d = lane + 64 * r;
    if (d < dh) out[d] = from_f<T>(none ? 0.f : acc[r] * inv);
  }
  if (lane == 0 && a.lse) a.lse[((long long)b * a.H + h) * a.Sq + i] = none ? -INFINITY : m + logf(l);
}

template <int R, typename T>
__device__ __forceinline__ void window_dq_row(const WindowArgs& a, int b, int i, int h, int lane) {
  const WindowSeq sq(a, b);
  const int p = sq.pos0 + i, dh = a.dh, hk = h / a.group;
  const KeyRanges ks(a, sq, p, p);
  const T* q = strided_row((const T*)a.q, a.sq, b, i, h);
  const T* dout = strided_row((const T*)a.dctx, a.sc, b, i, h);
  const T* k = strided_row((const T*)a.k, a.skv, b, 0, hk);
  const T* v = strided_row((const T*)a.v, a.skv, b, 0, hk);
  const long long at = ((long long)b * a.H + h) * a.Sq + i;
  const float li = a.lse[at], di = a.delta[at];
  float acc[R];
#pragma unroll
  for (int r = 0; r < R; r++) acc[r] = 0.f;
  for (int part = 0; part < 2; part++) {
    const int from = part ? ks.lo : 0, to = part ? ks.end : ks.sink_end;
    for (int j0 = from; j0 < to; j0 += 64) {
      const int j = j0 + lane;
      float ds = 0.f;
      if (j < to) {
        const float e = expf(dot_row(q, k + (long long)j * a.skv.row, dh) * a.scale - li);
        ds = e * (dot_row(dout, v + (long long)j * a.skv.row, dh) - di);
      }
      const int nj = min(64, to - j0);
      for (int jj = 0; jj < nj; jj++) {
        const float dsj = __shfl(ds, jj, 64);
        const T* kr = k + (long long)(j0 + jj) * a.skv.row;
#pragma unroll
        for (int r = 0; r < R; r++) {
          const int d = lane + 64 * r;
          if (d < dh) acc[r] = fmaf(dsj, to_f(kr[d]), acc[r]);
        }
      }
    }
  }
  T* out = strided_row((T*)a.dq, a.sq, b, i, h);
#pragma unroll
  for (int r = 0; r < R; r++) {
    const int d = lane + 64 * r;
    if (d < dh) out[d] = from_f<T>(acc[r] * a.scale);
  }
}

// One key of key head hk.
template <int R, typename T>
__device__ __forceinline__ void window_dkv_row(const WindowArgs& a, int b, int j, int hk, int lane) {
  const WindowSeq sq(a, b);
  const QueryRange qs(a, sq, j, j + 1);
  const int dh = a.dh;
  const T* kr = strided_row((const T*)a.k, a.skv, b, j, hk);
  const T* vr = strided_row((const T*)a.v, a.skv, b, j, hk);
  float ak[R], av[R];
#pragma unroll
  for (int r = 0; r < R; r++) ak[r] = av[r] = 0.f;
  for (int h = hk * a.group; h < (hk + 1) * a.group; h++) {
    const T* q = strided_row((const T*)a.q, a.sq, b, 0, h);
    const T* dout = strided_row((const T*)a.dctx, a.sc, b, 0, h);
    const long long at = ((long long)b * a.H + h) * a.Sq;
    for (int i0 = qs.i0; i0 < qs.i1; i0 += 64) {
      const int i = i0 + lane;
      float e = 0.f, ds = 0.f;
      if (i < qs.i1) {
        e = expf(dot_row(kr, q + (long long)i * a.sq.row, dh) * a.scale - a.lse[at + i]);
        ds = e * (dot_row(vr, dout + (long long)i * a.sc.row, dh) - a.delta[at + i]);
      }
      const int ni = min(64, qs.i1 - i0);
      for (int ii = 0; ii < ni; ii++) {
        const float ei = __shfl(e, ii, 64), dsi = __shfl(ds, ii, 64);
        const T* qr = q + (long long)(i0 + ii) * a.sq.row;
        const T* dor = dout + (long long)(i0 + ii) * a.sc.row;
#pragma unroll
        for (int r = 0; r < R; r++) {
          const int d = lane + 64 * r;
          if (d < dh) {
            av[r] = fmaf(ei, to_f(dor[d]), av[r]);
            ak[r] = fmaf(dsi, to_f(qr[d]), ak[r]);
          }
        }
      }
    }
  }
  T* dk = strided_row((T*)a.dk, a.skv, b, j, hk);
  T* dv = strided_row((T*)a.dv, a.skv, b, j, hk);
#pragma unroll
  for (int r = 0; r < R; r++) {
    const int d = lane + 64 * r;
    if (d < dh) {
      dk[d] = from_f<T>(ak[r] * a.scale);
      dv[d] = from_f<T>(av[r]);
    }
  }
}

}  // namespace fax
