// Gated linear recurrence along time, forward and backward.
//
//   h_s = a_s h_{s-1} + u_s,  a = sigmoid(f), u = sigmoid(-f) v
//   y_s = h_s sigmoid(o_s)
//   dh_s = dy_s sigmoid(o_s) + a_{s+1} dh_{s+1}
//   dv = dh sigmoid(-f),  df = dh (h_{s-1} - v) sigmoid(f) sigmoid(-f)
//   do = dy h sigmoid(o) sigmoid(-o)
//
// Some 16 (backward 36) operations per element of three (seven) moved: bound
// by memory.  A thread takes V adjacent channels of one row.
#include "seq.h"

namespace st {
namespace ops {
namespace {

constexpr int kStride = ST_SCAN_STRIDE;
constexpr int kThreads = 256;

struct ScanArgs {
  SeqAxes q;
  SeqTensor v, f, o, y;            // y: dy in the backward pass
  SeqTensor dv, df, d_o;
  const float* h;                  // backward: dh_out
  float* h_out;                    // backward: dh
  float* states;
  int cv;
  int64_t lanes;                   // b * cv
  // rows split along time
  int cols;                        // blocks of 64 lanes
  int tiles, subs;                 // tiles of a row, rounds of a tile
  float* ends;                     // [tiles]{A, H}, then the state: [b][c]
};

template <typename T, typename O, int V, bool GATE>
__global__ __launch_bounds__(kThreads) void k_scan(ScanArgs a) {
  constexpr int L = 4;
  const int64_t lane = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (lane >= a.lanes) return;
  const int b = (int)(lane / a.cv), ch = (int)(lane % a.cv) * V;
  const Row r = row_of(a.q, b);
  const int64_t hc = (int64_t)b * a.q.c + ch;
  const int64_t plane = (int64_t)a.q.b * a.q.c;
  float h[V];
#pragma unroll
  for (int e = 0; e < V; ++e) h[e] = a.h ? a.h[hc + e] : 0.f;
  const T* pv = (const T*)a.v.p + (int64_t)b * a.v.sb + ch;
  const T* pf = (const T*)a.f.p + (int64_t)b * a.f.sb + ch;
  const T* po = GATE ? (const T*)a.o.p + (int64_t)b * a.o.sb + ch : nullptr;
  O* py = (O*)a.y.p + (int64_t)b * a.y.sb + ch;
  for (int s = 0; s < r.len; s += L) {
    Pack<T, V> iv[L], jf[L], io[L];
#pragma unroll
    for (int k = 0; k < L; ++k) {
      const int64_t t = time_of(r, min(s + k, r.len - 1));
      iv[k] = load_pack<T, V>(pv + t * a.v.st);
      jf[k] = load_pack<T, V>(pf + t * a.f.st);
      if (GATE) io[k] = load_pack<T, V>(po + t * a.o.st);
    }
    if (a.states && s % kStride == 0)
      store_pack<float, V>(a.states + (s / kStride) * plane + hc, h);
#pragma unroll
    for (int k = 0; k < L; ++k) {
      if (s + k < r.len) {
        const bool cut = reset_at(a.q, r, b, s + k);
        float v[V], f[V], y[V];
        unpack<T, V>(iv[k], v);
        unpack<T, V>(jf[k], f);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float keep, write;
          sigmoids(f[e], keep, write);
          h[e] = __builtin_fmaf(keep, cut ? 0.f : h[e], write * v[e]);
          y[e] = h[e];
        }
        if (GATE) {
          float o[V];
          unpack<T, V>(io[k], o);
#pragma unroll
          for (int e = 0; e < V; ++e) y[e] *= sigmoid(o[e]);
        }
        store_pack<O, V>(py + time_of(r, s + k) * a.y.st, y);
      }
    }
  }
  for (int s = r.len; s < a.q.t; ++s) {
    float z[V];
#pragma unroll
    for (int e = 0; e < V; ++e) z[e] = 0.f;
    store_pack<O, V>(py + (int64_t)s * a.y.st, z);
  }
  if (a.h_out) {
#pragma unroll
    for (int e = 0; e < V; ++e) a.h_out[hc + e] = h[e];
  }
}

// ------------------------------------------------- rows split along time
//
// Few rows and channels, many steps: a thread for each would leave the device
// idle.  h_s = a_s h_{s-1} + u_s joins: a run of steps acts as h -> A h + H
// with A the product of its a.  A block takes 64 lanes (a lane: V adjacent
// channels of a row) over W waves, a wave kSplit steps of each lane, whose
// inputs stay in its registers: the waves exchange their (A, H) through LDS,
// fold those before them in order, and then run their steps from the state
// that enters them.  A tile is `subs` such rounds.  Where a row has several
// tiles a first launch leaves every tile's (A, H); the second folds those
// before it.  All folds run in step order: the same bits in every run.

constexpr int kSplit = 16;       // steps of a wave
constexpr int kWaves = 8;        // waves of a block, along time
constexpr int kRound = kSplit * kWaves;
static_assert(kSplit == kStride, "a wave keeps the state before its steps");

// A reset is a factor of minus zero (gates are never negative), which no value
// passes, not even NaN.
__device__ __forceinline__ bool is_cut(float A) {
  return __float_as_uint(A) == 0x80000000u;
}

// The time of step s, or of the row's nearest (time 0 of a row of none).
__device__ __forceinline__ int64_t time_in(const Row& r, int s) {
  const int64_t t = time_of(r, max(0, min(s, r.len - 1)));
  return t < 0 ? 0 : t;
}

struct LaneAt {
  int b, ch;
  bool on;          // otherwise a copy of the last lane that stores nothing
  int64_t hc;
};
__device__ __forceinline__ LaneAt lane_at(const ScanArgs& a, int v) {
  int64_t lane = (int64_t)(blockIdx.x % a.cols) * 64 + (threadIdx.x & 63);
  LaneAt l;
  l.on = lane < a.lanes;
  if (!l.on) lane = a.lanes - 1;
  l.b = (int)(lane / a.cv);
  l.ch = (int)(lane % a.cv) * v;
  l.hc = (int64_t)l.b * a.q.c + l.ch;
  return l;
}

// Folds `n` entries of (A, H), `step` floats apart, into (A, H) in order.
template <int V>
__device__ __forceinline__ void fold(const float* pa, const float* ph, int n,
                                     int64_t step, float* A, float* H) {
  for (int i = 0; i < n; ++i) {
    float x[V], y[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      x[e] = pa[i * step + e];
      y[e] = ph[i * step + e];
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const bool cut = is_cut(x[e]);
      H[e] = cut ? y[e] : __builtin_fmaf(x[e], H[e], y[e]);
      A[e] = cut ? x[e] : A[e] * x[e];
    }
  }
}

// The (A, H) of a wave's steps [s0, s0 + kSplit).
template <typename T, int V>
__device__ __forceinline__ void wave_ends(const ScanArgs& a, const Row& r,
                                          int b, int s0,
                                          const Pack<T, V>* iv,
                                          const Pack<T, V>* jf, float* A,
                                          float* H) {
#pragma unroll
  for (int e = 0; e < V; ++e) {
    A[e] = 1.f;
    H[e] = 0.f;
  }
#pragma unroll
  for (int k = 0; k < kSplit; ++k) {
    float v[V], f[V];
    unpack<T, V>(iv[k], v);
    unpack<T, V>(jf[k], f);
    const bool live = s0 + k < r.len;
    const bool cut = live && reset_at(a.q, r, b, s0 + k);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float keep, write;
      sigmoids(f[e], keep, write);
      const float h = __builtin_fmaf(keep, cut ? 0.f : H[e], write * v[e]);
      H[e] = live ? h : H[e];
      A[e] = live ? (cut ? -0.f : A[e] * keep) : A[e];
    }
  }
}

template <typename T, int V>
__global__ __launch_bounds__(64 * kWaves) void k_scan_ends(ScanArgs a) {
  __shared__ float sa[kWaves][64 * V], sh[kWaves][64 * V];
  const int wave = threadIdx.x / 64, at = (threadIdx.x & 63) * V;
  const int tile = blockIdx.x / a.cols;
  const LaneAt l = lane_at(a, V);
  const Row r = row_of(a.q, l.b);
  const T* pv = (const T*)a.v.p + (int64_t)l.b * a.v.sb + l.ch;
  const T* pf = (const T*)a.f.p + (int64_t)l.b * a.f.sb + l.ch;
  float TA[V], TH[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    TA[e] = 1.f;
    TH[e] = 0.f;
  }
  for (int sub = 0; sub < a.subs; ++sub) {
    const int s0 = (tile * a.subs + sub) * kRound + wave * kSplit;
    float A[V], H[V];
    if (__any(s0 < r.len)) {
      Pack<T, V> iv[kSplit], jf[kSplit];
#pragma unroll
      for (int k = 0; k < kSplit; ++k) {
        const int64_t tc = time_in(r, s0 + k);
        iv[k] = load_pack<T, V>(pv + tc * a.v.st);
        jf[k] = load_pack<T, V>(pf + tc * a.f.st);
      }
      wave_ends<T, V>(a, r, l.b, s0, iv, jf, A, H);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        A[e] = 1.f;
        H[e] = 0.f;
      }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) {
      sa[wave][at + e] = A[e];
      sh[wave][at + e] = H[e];
    }
    __syncthreads();
    if (wave == 0) fold<V>(&sa[0][at], &sh[0][at], kWaves, 64 * V, TA, TH);
  }
  if (wave == 0 && l.on) {
    const int64_t plane = (int64_t)a.q.b * a.q.c;
    float* o = a.ends + (int64_t)tile * 2 * plane + l.hc;
    store_pack<float, V>(o, TA);
    store_pack<float, V>(o + plane, TH);
    // the state itself too: the second launch may replace it in place
    if (tile == 0) {
      float h[V];
#pragma unroll
      for (int e = 0; e < V; ++e) h[e] = a.h ? a.h[l.hc + e] : 0.f;
      store_pack<float, V>(a.ends + (int64_t)a.tiles * 2 * plane + l.hc, h);
    }
  }
}

template <typename T, typename O, int V, bool GATE>
__global__ __launch_bounds__(64 * kWaves) void k_scan_tiles(ScanArgs a) {
  __shared__ float sa[kWaves][64 * V], sh[kWaves][64 * V];
  const int wave = threadIdx.x / 64, at = (threadIdx.x & 63) * V;
  const int tile = blockIdx.x / a.cols;
  const LaneAt l = lane_at(a, V);
  const Row r = row_of(a.q, l.b);
  const int64_t plane = (int64_t)a.q.b * a.q.c;
  const T* pv = (const T*)a.v.p + (int64_t)l.b * a.v.sb + l.ch;
  const T* pf = (const T*)a.f.p + (int64_t)l.b * a.f.sb + l.ch;
  const T* po =
      GATE ? (const T*)a.o.p + (int64_t)l.b * a.o.sb + l.ch : nullptr;
  O* py = (O*)a.y.p + (int64_t)l.b * a.y.sb + l.ch;
  // the state that enters the tile: waves fold shares of the tiles before it
  float h[V];
  if (a.tiles == 1) {
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = a.h ? a.h[l.hc + e] : 0.f;
  } else {
    float A[V], H[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      A[e] = 1.f;
      H[e] = 0.f;
      h[e] = a.ends[(int64_t)a.tiles * 2 * plane + l.hc + e];
    }
    const int share = (tile + kWaves - 1) / kWaves;
    const int i0 = min(wave * share, tile), i1 = min(i0 + share, tile);
    const float* e0 = a.ends + (int64_t)i0 * 2 * plane + l.hc;
    fold<V>(e0, e0 + plane, i1 - i0, 2 * plane, A, H);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      sa[wave][at + e] = A[e];
      sh[wave][at + e] = H[e];
    }
    __syncthreads();
    fold<V>(&sa[0][at], &sh[0][at], kWaves, 64 * V, A, h);
  }
  for (int sub = 0; sub < a.subs; ++sub) {
    const int s0 = (tile * a.subs + sub) * kRound + wave * kSplit;
    const bool any = __any(s0 < r.len);
    Pack<T, V> iv[kSplit], jf[kSplit], io[kSplit];
    float A[V], H[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      A[e] = 1.f;
      H[e] = 0.f;
    }
    if (any) {
#pragma unroll
      for (int k = 0; k < kSplit; ++k) {
        const int64_t tc = time_in(r, s0 + k);
        iv[k] = load_pack<T, V>(pv + tc * a.v.st);
        jf[k] = load_pack<T, V>(pf + tc * a.f.st);
        if (GATE) io[k] = load_pack<T, V>(po + tc * a.o.st);
      }
      wave_ends<T, V>(a, r, l.b, s0, iv, jf, A, H);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) {
      sa[wave][at + e] = A[e];
      sh[wave][at + e] = H[e];
    }
    __syncthreads();
    float hw[V];
#pragma unroll
    for (int e = 0; e < V; ++e) hw[e] = h[e];
    fold<V>(&sa[0][at], &sh[0][at], wave, 64 * V, A, hw);
    // the round's end: the same sums, carried on to every wave
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = hw[e];
    fold<V>(&sa[wave][at], &sh[wave][at], kWaves - wave, 64 * V, A, h);
    if (any && l.on) {
      if (a.states && s0 < r.len)
        store_pack<float, V>(a.states + (s0 / kStride) * plane + l.hc, hw);
#pragma unroll
      for (int k = 0; k < kSplit; ++k) {
        if (s0 + k < r.len) {
          const bool cut = reset_at(a.q, r, l.b, s0 + k);
          float v[V], f[V], y[V];
          unpack<T, V>(iv[k], v);
          unpack<T, V>(jf[k], f);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            float keep, write;
            sigmoids(f[e], keep, write);
            hw[e] = __builtin_fmaf(keep, cut ? 0.f : hw[e], write * v[e]);
            y[e] = hw[e];
          }
          if (GATE) {
            float o[V];
            unpack<T, V>(io[k], o);
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] *= sigmoid(o[e]);
          }
          store_pack<O, V>(py + time_of(r, s0 + k) * a.y.st, y);
        }
      }
    }
    if (l.on) {
      const int s1 = min(s0 + kSplit, a.q.t);
      for (int s = max(s0, r.len); s < s1; ++s) {
        float z[V];
#pragma unroll
        for (int e = 0; e < V; ++e) z[e] = 0.f;
        store_pack<O, V>(py + (int64_t)s * a.y.st, z);
      }
    }
  }
  if (a.h_out && tile == a.tiles - 1 && wave == 0 && l.on) {
#pragma unroll
    for (int e = 0; e < V; ++e) a.h_out[l.hc + e] = h[e];
  }
}

// A thread walks its row from the last step back, kStride steps at a time:
// the states of these steps come again from the state kept before them.
template <typename T, typename O, int V, bool GATE>
__global__ __launch_bounds__(kThreads) void k_scan_grad(ScanArgs a) {
  const int64_t lane = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (lane >= a.lanes) return;
  const int b = (int)(lane / a.cv), ch = (int)(lane % a.cv) * V;
  const Row r = row_of(a.q, b);
  const int64_t hc = (int64_t)b * a.q.c + ch;
  const int64_t plane = (int64_t)a.q.b * a.q.c;
  float dh[V];
#pragma unroll
  for (int e = 0; e < V; ++e) dh[e] = a.h ? a.h[hc + e] : 0.f;
  const T* pv = (const T*)a.v.p + (int64_t)b * a.v.sb + ch;
  const T* pf = (const T*)a.f.p + (int64_t)b * a.f.sb + ch;
  const T* po = GATE ? (const T*)a.o.p + (int64_t)b * a.o.sb + ch : nullptr;
  const O* pd = (const O*)a.y.p + (int64_t)b * a.y.sb + ch;
  T* pdv = (T*)a.dv.p + (int64_t)b * a.dv.sb + ch;
  T* pdf = (T*)a.df.p + (int64_t)b * a.df.sb + ch;
  T* pdo = GATE ? (T*)a.d_o.p + (int64_t)b * a.d_o.sb + ch : nullptr;
  for (int s = r.len; s < a.q.t; ++s) {
    float z[V];
#pragma unroll
    for (int e = 0; e < V; ++e) z[e] = 0.f;
    store_pack<T, V>(pdv + (int64_t)s * a.dv.st, z);
    store_pack<T, V>(pdf + (int64_t)s * a.df.st, z);
    if (GATE) store_pack<T, V>(pdo + (int64_t)s * a.d_o.st, z);
  }
  for (int s0 = (r.len - 1) / kStride * kStride; s0 >= 0 && r.len > 0;
       s0 -= kStride) {
    Pack<T, V> iv[kStride], jf[kStride];
    float h[V];
    float prev[kStride][V];   // the state that enters each step
#pragma unroll
    for (int k = 0; k < kStride; ++k) {
      const int64_t t = time_of(r, min(s0 + k, r.len - 1));
      iv[k] = load_pack<T, V>(pv + t * a.v.st);
      jf[k] = load_pack<T, V>(pf + t * a.f.st);
    }
    unpack<float, V>(
        load_pack<float, V>(a.states + (s0 / kStride) * plane + hc), h);
#pragma unroll
    for (int k = 0; k < kStride; ++k) {
      float v[V], f[V];
      unpack<T, V>(iv[k], v);
      unpack<T, V>(jf[k], f);
      const bool cut = s0 + k < r.len && reset_at(a.q, r, b, s0 + k);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        float keep, write;
        sigmoids(f[e], keep, write);
        if (cut) h[e] = 0.f;
        prev[k][e] = h[e];
        h[e] = __builtin_fmaf(keep, h[e], write * v[e]);
      }
    }
#pragma unroll
    for (int k = kStride - 1; k >= 0; --k) {
      if (s0 + k < r.len) {
        const int64_t t = time_of(r, s0 + k);
        const bool cut = reset_at(a.q, r, b, s0 + k);
        float v[V], f[V], d[V], gv[V], gf[V];
        unpack<T, V>(iv[k], v);
        unpack<T, V>(jf[k], f);
        unpack<O, V>(load_pack<O, V>(pd + t * a.y.st), d);
        float keep[V], write[V];
#pragma unroll
        for (int e = 0; e < V; ++e) sigmoids(f[e], keep[e], write[e]);
        if (GATE) {
          float o[V], go[V];
          unpack<T, V>(load_pack<T, V>(po + t * a.o.st), o);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float here =
                __builtin_fmaf(keep[e], prev[k][e], write[e] * v[e]);
            float p, n;
            sigmoids(o[e], p, n);
            go[e] = d[e] * here * p * n;
            d[e] *= p;
          }
          store_pack<T, V>(pdo + t * a.d_o.st, go);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
          dh[e] += d[e];
          gv[e] = dh[e] * write[e];
          gf[e] = dh[e] * (prev[k][e] - v[e]) * (keep[e] * write[e]);
          dh[e] = cut ? 0.f : dh[e] * keep[e];
        }
        store_pack<T, V>(pdv + t * a.dv.st, gv);
        store_pack<T, V>(pdf + t * a.df.st, gf);
      }
    }
  }
  if (a.h_out) {
#pragma unroll
    for (int e = 0; e < V; ++e) a.h_out[hc + e] = dh[e];
  }
}

// The backward pass of rows split along time: dh runs from the last step to
// the first, d -> A d + D over a run of steps, and joins the same way.  The
// states come again, wave by wave, from those kept.  (The folds go from the
// last entry down.)
template <int V>
__device__ __forceinline__ void fold_back(const float* pa, const float* pd,
                                          int n, int64_t step, float* A,
                                          float* D) {
  fold<V>(pa + (n - 1) * step, pd + (n - 1) * step, n, -step, A, D);
}

// One step back: dh of the step is d + g; what goes on to the step before.
__device__ __forceinline__ float back(float d, float keep, bool cut) {
  return cut ? 0.f : d * keep;
}

template <typename T, typename O, int V, bool GATE>
__global__ __launch_bounds__(64 * kWaves) void k_scan_grad_ends(ScanArgs a) {
  __shared__ float sa[kWaves][64 * V], sh[kWaves][64 * V];
  const int wave = threadIdx.x / 64, at = (threadIdx.x & 63) * V;
  const int tile = blockIdx.x / a.cols;
  const LaneAt l = lane_at(a, V);
  const Row r = row_of(a.q, l.b);
  const T* pf = (const T*)a.f.p + (int64_t)l.b * a.f.sb + l.ch;
  const T* po =
      GATE ? (const T*)a.o.p + (int64_t)l.b * a.o.sb + l.ch : nullptr;
  const O* pd = (const O*)a.y.p + (int64_t)l.b * a.y.sb + l.ch;
  float TA[V], TD[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    TA[e] = 1.f;
    TD[e] = 0.f;
  }
  for (int sub = a.subs - 1; sub >= 0; --sub) {
    const int s0 = (tile * a.subs + sub) * kRound + wave * kSplit;
    float A[V], D[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      A[e] = 1.f;
      D[e] = 0.f;
    }
    if (__any(s0 < r.len)) {
      Pack<T, V> jf[kSplit], io[kSplit];
      Pack<O, V> id[kSplit];
#pragma unroll
      for (int k = 0; k < kSplit; ++k) {
        const int64_t tc = time_in(r, s0 + k);
        jf[k] = load_pack<T, V>(pf + tc * a.f.st);
        if (GATE) io[k] = load_pack<T, V>(po + tc * a.o.st);
        id[k] = load_pack<O, V>(pd + tc * a.y.st);
      }
#pragma unroll
      for (int k = kSplit - 1; k >= 0; --k) {
        float f[V], d[V];
        unpack<T, V>(jf[k], f);
        unpack<O, V>(id[k], d);
        const bool live = s0 + k < r.len;
        const bool cut = live && reset_at(a.q, r, l.b, s0 + k);
        if (GATE) {
          float o[V];
          unpack<T, V>(io[k], o);
#pragma unroll
          for (int e = 0; e < V; ++e) d[e] *= sigmoid(o[e]);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float keep = sigmoid(f[e]);
          D[e] = live ? back(D[e] + d[e], keep, cut) : D[e];
          A[e] = live ? (cut ? -0.f : A[e] * keep) : A[e];
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) {
      sa[wave][at + e] = A[e];
      sh[wave][at + e] = D[e];
    }
    __syncthreads();
    if (wave == 0)
      fold_back<V>(&sa[0][at], &sh[0][at], kWaves, 64 * V, TA, TD);
  }
  if (wave == 0 && l.on) {
    const int64_t plane = (int64_t)a.q.b * a.q.c;
    float* o = a.ends + (int64_t)tile * 2 * plane + l.hc;
    store_pack<float, V>(o, TA);
    store_pack<float, V>(o + plane, TD);
    if (tile == 0) {   // a copy: dh may replace it in place
      float h[V];
#pragma unroll
      for (int e = 0; e < V; ++e) h[e] = a.h ? a.h[l.hc + e] : 0.f;
      store_pack<float, V>(a.ends + (int64_t)a.tiles * 2 * plane + l.hc, h);
    }
  }
}

template <typename T, typename O, int V, bool GATE>
__global__ __launch_bounds__(64 * kWaves) void k_scan_grad_tiles(ScanArgs a) {
  __shared__ float sa[kWaves][64 * V], sh[kWaves][64 * V];
  const int wave = threadIdx.x / 64, at = (threadIdx.x & 63) * V;
  const int tile = blockIdx.x / a.cols;
  const LaneAt l = lane_at(a, V);
  const Row r = row_of(a.q, l.b);
  const int64_t plane = (int64_t)a.q.b * a.q.c;
  const T* pv = (const T*)a.v.p + (int64_t)l.b * a.v.sb + l.ch;
  const T* pf = (const T*)a.f.p + (int64_t)l.b * a.f.sb + l.ch;
  const T* po =
      GATE ? (const T*)a.o.p + (int64_t)l.b * a.o.sb + l.ch : nullptr;
  const O* pd = (const O*)a.y.p + (int64_t)l.b * a.y.sb + l.ch;
  T* pdv = (T*)a.dv.p + (int64_t)l.b * a.dv.sb + l.ch;
  T* pdf = (T*)a.df.p + (int64_t)l.b * a.df.sb + l.ch;
  T* pdo = GATE ? (T*)a.d_o.p + (int64_t)l.b * a.d_o.sb + l.ch : nullptr;
  // what comes back into the tile's last step
  float dh[V];
  if (a.tiles == 1) {
#pragma unroll
    for (int e = 0; e < V; ++e) dh[e] = a.h ? a.h[l.hc + e] : 0.f;
  } else {
    float A[V], D[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      A[e] = 1.f;
      D[e] = 0.f;
      dh[e] = a.ends[(int64_t)a.tiles * 2 * plane + l.hc + e];
    }
    const int after = a.tiles - 1 - tile;
    const int share = (after + kWaves - 1) / kWaves;
    const int i0 = min(wave * share, after), i1 = min(i0 + share, after);
    const float* e0 = a.ends + (int64_t)(tile + 1 + i0) * 2 * plane + l.hc;
    if (i1 > i0) fold_back<V>(e0, e0 + plane, i1 - i0, 2 * plane, A, D);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      sa[wave][at + e] = A[e];
      sh[wave][at + e] = D[e];
    }
    __syncthreads();
    fold_back<V>(&sa[0][at], &sh[0][at], kWaves, 64 * V, A, dh);
  }
  for (int sub = a.subs - 1; sub >= 0; --sub) {
    const int s0 = (tile * a.subs + sub) * kRound + wave * kSplit;
    const bool any = __any(s0 < r.len);
    Pack<T, V> jf[kSplit];
    float g[kSplit][V];     // dy sigmoid(o)
    float q[kSplit][V];     // h_{s-1} - v
    float A[V], D[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      A[e] = 1.f;
      D[e] = 0.f;
    }
    if (any) {
      Pack<T, V> iv[kSplit], io[kSplit];
      Pack<O, V> id[kSplit];
      float h[V];
#pragma unroll
      for (int k = 0; k < kSplit; ++k) {
        const int64_t tc = time_in(r, s0 + k);
        iv[k] = load_pack<T, V>(pv + tc * a.v.st);
        jf[k] = load_pack<T, V>(pf + tc * a.f.st);
        if (GATE) io[k] = load_pack<T, V>(po + tc * a.o.st);
        id[k] = load_pack<O, V>(pd + tc * a.y.st);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) h[e] = 0.f;
      if (s0 < r.len)
        unpack<float, V>(load_pack<float, V>(
                             a.states + (s0 / kStride) * plane + l.hc),
                         h);
#pragma unroll
      for (int k = 0; k < kSplit; ++k) {
        float v[V], f[V], o[V], go[V];
        unpack<T, V>(iv[k], v);
        unpack<T, V>(jf[k], f);
        unpack<O, V>(id[k], g[k]);
        if (GATE) unpack<T, V>(io[k], o);
        const bool live = s0 + k < r.len;
        const bool cut = live && reset_at(a.q, r, l.b, s0 + k);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float keep, write;
          sigmoids(f[e], keep, write);
          if (cut) h[e] = 0.f;
          q[k][e] = h[e] - v[e];
          h[e] = __builtin_fmaf(keep, h[e], write * v[e]);
          if (GATE) {
            float p, n;
            sigmoids(o[e], p, n);
            go[e] = g[k][e] * h[e] * p * n;
            g[k][e] *= p;
          }
        }
        if (GATE && live && l.on)
          store_pack<T, V>(pdo + time_of(r, s0 + k) * a.d_o.st, go);
      }
#pragma unroll
      for (int k = kSplit - 1; k >= 0; --k) {
        float f[V];
        unpack<T, V>(jf[k], f);
        const bool live = s0 + k < r.len;
        const bool cut = live && reset_at(a.q, r, l.b, s0 + k);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float keep = sigmoid(f[e]);
          D[e] = live ? back(D[e] + g[k][e], keep, cut) : D[e];
          A[e] = live ? (cut ? -0.f : A[e] * keep) : A[e];
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) {
      sa[wave][at + e] = A[e];
      sh[wave][at + e] = D[e];
    }
    __syncthreads();
    float d[V];
#pragma unroll
    for (int e = 0; e < V; ++e) d[e] = dh[e];
    const int later = kWaves - 1 - wave;
    if (later)
      fold_back<V>(&sa[wave + 1][at], &sh[wave + 1][at], later, 64 * V, A, d);
#pragma unroll
    for (int e = 0; e < V; ++e) dh[e] = d[e];
    fold_back<V>(&sa[0][at], &sh[0][at], wave + 1, 64 * V, A, dh);
    if (any && l.on) {
#pragma unroll
      for (int k = kSplit - 1; k >= 0; --k) {
        if (s0 + k < r.len) {
          const int64_t t = time_of(r, s0 + k);
          const bool cut = reset_at(a.q, r, l.b, s0 + k);
          float f[V], gv[V], gf[V];
          unpack<T, V>(jf[k], f);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            float keep, write;
            sigmoids(f[e], keep, write);
            d[e] += g[k][e];
            gv[e] = d[e] * write;
            gf[e] = d[e] * q[k][e] * (keep * write);
            d[e] = back(d[e], keep, cut);
          }
          store_pack<T, V>(pdv + t * a.dv.st, gv);
          store_pack<T, V>(pdf + t * a.df.st, gf);
        }
      }
    }
    if (l.on) {
      const int s1 = min(s0 + kSplit, a.q.t);
      for (int s = max(s0, r.len); s < s1; ++s) {
        float z[V];
#pragma unroll
        for (int e = 0; e < V; ++e) z[e] = 0.f;
        store_pack<T, V>(pdv + (int64_t)s * a.dv.st, z);
        store_pack<T, V>(pdf + (int64_t)s * a.df.st, z);
        if (GATE) store_pack<T, V>(pdo + (int64_t)s * a.d_o.st, z);
      }
    }
  }
  if (a.h_out && tile == 0 && wave == 0 && l.on) {
#pragma unroll
    for (int e = 0; e < V; ++e) a.h_out[l.hc + e] = dh[e];
  }
}

// -------------------------------------------------------------- host side

template <class F>
void with_scan(int v, bool gate, F&& f) {
  auto go = [&](auto vt) {
    if (gate)
      f(vt, std::true_type{});
    else
      f(vt, std::false_type{});
  };
  if (v == 4)
    go(Int<4>{});
  else if (v == 2)
    go(Int<2>{});
  else
    go(Int<1>{});
}

// Which rows are split along time: those of more than 64 steps (a chunk's
// frames, 32 at most, are walked one after another, as they are taken one by
// one: the same bits) of which there are too few to fill the device, a lane
// each.
constexpr int kSerialSteps = 64;
constexpr int64_t kFillWaves = 2048;    // eight to a CU
constexpr int kMaxTiles = 512;

struct ScanCut {
  bool split = false;
  int cols = 0, tiles = 0, subs = 0;
};
ScanCut cut_of(const st_seq_desc& d, int v) {
  ScanCut c;
  const int64_t lanes = (int64_t)d.b * (d.c / v);
  const int64_t cols = ceil_div(lanes, 64);
  if (d.t <= kSerialSteps || cols >= kFillWaves) return c;
  c.split = true;
  c.cols = (int)cols;
  const int64_t rounds = ceil_div(d.t, kRound);
  const int64_t want =
      std::min<int64_t>(kMaxTiles, ceil_div(2 * kFillWaves, cols * kWaves));
  c.subs = (int)ceil_div(rounds, std::min(rounds, want));
  c.tiles = (int)ceil_div(rounds, c.subs);
  return c;
}

uint64_t scan_space(const st_seq_desc& d, bool) {
  uint64_t most = 0;
  for (int v = 4; v >= 1; v /= 2) {
    if (d.c % v || empty(d)) continue;
    const ScanCut c = cut_of(d, v);
    if (c.split && c.tiles > 1)
      most = std::max<uint64_t>(
          most, (uint64_t)(2 * c.tiles + 1) * d.b * d.c * sizeof(float));
  }
  return most;
}

void take_cut(ScanArgs& a, const ScanCut& c, void* ws) {
  a.cols = c.cols;
  a.tiles = c.tiles;
  a.subs = c.subs;
  a.ends = (float*)ws;
}

}  // namespace
}  // namespace ops
}  // namespace st

using namespace st;
using namespace st::ops;

extern "C" st_status st_gated_scan_workspace(const st_seq_desc* d,
                                             int32_t backward,
                                             uint64_t* bytes) {
  return guarded([&]() -> st_status {
    if (const st_status s = check_seq(d); s != ST_OK) return s;
    if (!bytes) return bad("bytes is NULL");
    *bytes = scan_space(*d, backward != 0);
    return ST_OK;
  });
}

extern "C" st_status st_gated_scan(const st_seq_desc* d, const st_seq_ref* v,
                                   const st_seq_ref* f, const st_seq_ref* o,
                                   const float* h, const st_seq_ref* y,
                                   float* h_out, float* states, void* ws,
                                   uint64_t ws_bytes, void* stream) {
  return guarded([&]() -> st_status {
    if (const st_status s = check_seq(d); s != ST_OK) return s;
    if (const st_status s = check_ref(*d, v, false, "v"); s != ST_OK) return s;
    if (const st_status s = check_ref(*d, f, false, "f"); s != ST_OK) return s;
    if (o)
      if (const st_status s = check_ref(*d, o, false, "o"); s != ST_OK)
        return s;
    if (const st_status s = check_ref(*d, y, true, "y"); s != ST_OK) return s;
    if (const st_status s = check_ws(scan_space(*d, false), ws, ws_bytes);
        s != ST_OK)
      return s;
    const int es = esize(d->dtype), eo = esize(d->out_dtype);
    const int64_t plane = (int64_t)d->b * d->c * 4;
    const Span sh = span_of(h, plane);
    if (any_hit({ref_span(*d, y, eo), span_of(h_out, plane),
                 span_of(states, plane * ceil_div(d->t, kStride)),
                 span_of(ws, (int64_t)ws_bytes)},
                {ref_span(*d, v, es), ref_span(*d, f, es),
                 ref_span(*d, o, es), h_out == h ? Span{} : sh,
                 span_of(d->lengths, d->b * 4ll),
                 span_of(d->reset, (int64_t)d->t * d->b)}))
      return bad("an output overlaps an input, another output or the "
                 "workspace");
    if (d->b == 0) return ST_OK;
    (void)hipGetLastError();
    int vec = 4;
    for (; vec > 1; vec /= 2)
      if (d->c % vec == 0 && ops::vec_ok(vec, es, *d, v) &&
          ops::vec_ok(vec, es, *d, f) && ops::vec_ok(vec, es, *d, o) &&
          ops::vec_ok(vec, eo, *d, y) &&
          (uintptr_t)states % (vec * 4) == 0)
        break;
    ScanArgs a{};
    a.q = axes_of(*d);
    a.v = tensor_of(v);
    a.f = tensor_of(f);
    a.o = tensor_of(o);
    a.y = tensor_of(y);
    a.h = h;
    a.h_out = h_out;
    a.states = states;
    a.cv = d->c / vec;
    a.lanes = (int64_t)d->b * a.cv;
    const unsigned grid = (unsigned)ceil_div(a.lanes, kThreads);
    const ScanCut cut = cut_of(*d, vec);
    take_cut(a, cut, ws);
    hipStream_t q = (hipStream_t)stream;
    with_types(d->dtype, d->out_dtype, [&](auto ti, auto to) {
      using T = typename decltype(ti)::type;
      using O = typename decltype(to)::type;
      with_scan(vec, o != nullptr, [&](auto vt, auto gt) {
        constexpr int V = decltype(vt)::value;
        constexpr bool G = decltype(gt)::value;
        if (!cut.split) {
          k_scan<T, O, V, G><<<grid, kThreads, 0, q>>>(a);
          return;
        }
        if (cut.tiles > 1)
          k_scan_ends<T, V>
              <<<cut.cols * cut.tiles, 64 * kWaves, 0, q>>>(a);
        k_scan_tiles<T, O, V, G>
            <<<cut.cols * cut.tiles, 64 * kWaves, 0, q>>>(a);
      });
    });
    return launch_status("gated scan");
  });
}

extern "C" st_status st_gated_scan_backward(
    const st_seq_desc* d, const st_seq_ref* dy, const st_seq_ref* v,
    const st_seq_ref* f, const st_seq_ref* o, const float* states,
    const float* dh_out, const st_seq_ref* dv, const st_seq_ref* df,
    const st_seq_ref* d_o, float* dh, void* ws, uint64_t ws_bytes,
    void* stream) {
  return guarded([&]() -> st_status {
    if (const st_status s = check_seq(d); s != ST_OK) return s;
    struct { const st_seq_ref* r; bool out; const char* name; } refs[] = {
        {dy, false, "dy"}, {v, false, "v"},   {f, false, "f"},
        {dv, true, "dv"},  {df, true, "df"}};
    for (const auto& x : refs)
      if (const st_status s = check_ref(*d, x.r, x.out, x.name); s != ST_OK)
        return s;
    if (!o != !d_o) return bad("o and d_o: both or neither");
    if (o) {
      if (const st_status s = check_ref(*d, o, false, "o"); s != ST_OK)
        return s;
      if (const st_status s = check_ref(*d, d_o, true, "d_o"); s != ST_OK)
        return s;
    }
    if (!states && !empty(*d)) return bad("states is NULL");
    if (const st_status s = check_ws(scan_space(*d, true), ws, ws_bytes);
        s != ST_OK)
      return s;
    const int es = esize(d->dtype), eo = esize(d->out_dtype);
    const int64_t plane = (int64_t)d->b * d->c * 4;
    const std::initializer_list<Span> in = {
        ref_span(*d, dy, eo), ref_span(*d, v, es), ref_span(*d, f, es),
        ref_span(*d, o, es),
        span_of(states, plane * ceil_div(d->t, kStride)),
        dh_out == dh ? Span{} : span_of(dh_out, plane),
        span_of(d->lengths, d->b * 4ll),
        span_of(d->reset, (int64_t)d->t * d->b)};
    const st_seq_ref* out[] = {dv, df, d_o};
    bool hit = false;
    for (int i = 0; i < 3; ++i) {
      if (!out[i]) continue;
      const Span si = ref_span(*d, out[i], es);
      for (const Span& s : in) hit = hit || si.hits(s);
      for (int j = 0; j < i; ++j)
        if (out[j] && si.hits(ref_span(*d, out[j], es)))
          hit = hit || !side_by_side(*d, *out[i], *out[j], es);
      hit = hit || si.hits(span_of(dh, plane)) ||
            si.hits(span_of(ws, (int64_t)ws_bytes));
    }
    if (hit || any_hit({span_of(dh, plane), span_of(ws, (int64_t)ws_bytes)},
                       in))
      return bad("an output overlaps an input, another output or the "
                 "workspace");
    if (d->b == 0) return ST_OK;
    (void)hipGetLastError();
    int vec = 4;
    for (; vec > 1; vec /= 2) {
      bool ok = d->c % vec == 0 && (uintptr_t)states % (vec * 4) == 0 &&
                ops::vec_ok(vec, eo, *d, dy);
      for (const st_seq_ref* r : {v, f, o, dv, df, d_o})
        ok = ok && ops::vec_ok(vec, es, *d, r);
      if (ok) break;
    }
    ScanArgs a{};
    a.q = axes_of(*d);
    a.v = tensor_of(v);
    a.f = tensor_of(f);
    a.o = tensor_of(o);
    a.y = tensor_of(dy);
    a.dv = tensor_of(dv);
    a.df = tensor_of(df);
    a.d_o = tensor_of(d_o);
    a.h = dh_out;
    a.h_out = dh;
    a.states = const_cast<float*>(states);
    a.cv = d->c / vec;
    a.lanes = (int64_t)d->b * a.cv;
    const unsigned grid = (unsigned)ceil_div(a.lanes, kThreads);
    const ScanCut cut = cut_of(*d, vec);
    take_cut(a, cut, ws);
    hipStream_t q = (hipStream_t)stream;
    with_types(d->dtype, d->out_dtype, [&](auto ti, auto to) {
      using T = typename decltype(ti)::type;
      using O = typename decltype(to)::type;
      with_scan(vec, o != nullptr, [&](auto vt, auto gt) {
        constexpr int V = decltype(vt)::value;
        constexpr bool G = decltype(gt)::value;
        if (!cut.split) {
          k_scan_grad<T, O, V, G><<<grid, kThreads, 0, q>>>(a);
          return;
        }
        if (cut.tiles > 1)
          k_scan_grad_ends<T, O, V, G>
              <<<cut.cols * cut.tiles, 64 * kWaves, 0, q>>>(a);
        k_scan_grad_tiles<T, O, V, G>
            <<<cut.cols * cut.tiles, 64 * kWaves, 0, q>>>(a);
      });
    });
    return launch_status("gated scan backward");
  });
}
