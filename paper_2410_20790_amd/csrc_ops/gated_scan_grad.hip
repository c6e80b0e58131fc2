// Gradients of the gated linear recurrence.
//
//   dh_s = dy_s sigmoid(o_s) + a_{s+1} dh_{s+1},  a = sigmoid(f)
//   dv = dh sigmoid(-f),  df = dh (h_{s-1} - v) sigmoid(f) sigmoid(-f)
//   do = dy h sigmoid(o) sigmoid(-o)
//
// Some 36 operations per element of four read and three written: bound by
// memory, with as many instruction slots again for the sigmoids.
#include "gated_scan.h"

namespace st {
namespace ops {
namespace {

// (V is 1: four arrays of 16 steps in registers leave no room for more, and two
// channels to a lane measured 143 us where one takes 127, 9 steps of 2048 rows
// of 1024 channels f32.)
//
// kSplit steps of a lane: their states come again from the one kept before
// them, forward; the gradients go back through them.  All is read once.
template <typename T, typename O, int V, bool GATE>
struct GradSteps {
  float keep[kSplit][V], write[kSplit][V];
  float g[kSplit][V];     // dy sigmoid(o)
  float q[kSplit][V];     // h_{s-1} - v
  Whole whole;
  unsigned cuts;

  // Loads, states, and do.
  __device__ __forceinline__ void forward(const ScanArgs& a, const Row& r,
                                          const LaneAt& l, int s0) {
    whole = whole_wave(a, r, s0, kSplit);
    Pack<T, V> iv[kSplit], jf[kSplit], io[kSplit];
    Pack<O, V> id[kSplit];
    float h[V];
    load_steps<T, V, kSplit>(a.f, whole, a, r, l.b, l.ch, s0, jf);
    load_steps<T, V, kSplit>(a.v, whole, a, r, l.b, l.ch, s0, iv);
    if (GATE)
      load_steps<T, V, kSplit>(a.o, whole, a, r, l.b, l.ch, s0, io);
    load_steps<O, V, kSplit>(a.y, whole, a, r, l.b, l.ch, s0, id);
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = 0.f;
    if (s0 < r.len)
      unpack<float, V>(
          load_pack<float, V>(a.states + (s0 / kStride) *
                                  ((int64_t)a.q.b * a.q.c) + l.hc),
          h);
    cuts = cuts_of<kSplit>(a, r, l.b, s0);
    auto step = [&](int k, float* go) {
      const bool cut = cuts >> k & 1;
      float v[V], f[V], o[V];
      unpack<T, V>(iv[k], v);
      unpack<T, V>(jf[k], f);
      unpack<O, V>(id[k], g[k]);
      if (GATE) unpack<T, V>(io[k], o);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        sigmoids(f[e], keep[k][e], write[k][e]);
        h[e] = cut ? 0.f : h[e];
        q[k][e] = h[e] - v[e];
        h[e] = __builtin_fmaf(keep[k][e], h[e], write[k][e] * v[e]);
        if (GATE) {
          float p, n;
          sigmoids_once(o[e], p, n);
          g[k][e] *= p;
          go[e] = g[k][e] * h[e] * n;
        }
      }
    };
    if (whole.on && __all(l.on)) {
      const WaveWalk<T> w(GATE ? a.d_o : a.dv, whole.t, whole.dir, l.b, l.ch);
#pragma unroll
      for (int k = 0; k < kSplit; ++k) {
        float go[V];
        step(k, go);
        if (GATE) store_pack<T, V>(w.at(k), go);
      }
    } else {
      Walk<T> w(GATE ? a.d_o : a.dv, r, l.b, l.ch, s0);
#pragma unroll
      for (int k = 0; k < kSplit; ++k) {
        if (s0 + k < r.len) {
          float go[V];
          step(k, go);
          if (GATE && l.on) {
            store_pack<T, V>(w.p, go);
            w.next();
          }
        } else {
          // behind the row's end: what comes back passes as it is
#pragma unroll
          for (int e = 0; e < V; ++e) {
            keep[k][e] = 1.f;
            write[k][e] = g[k][e] = q[k][e] = 0.f;
          }
        }
      }
    }
  }

  // What the steps do to a gradient that comes back: d -> A d + D.
  __device__ __forceinline__ void ends(float* A, float* D) const {
    none<V>(A, D);
#pragma unroll
    for (int k = kSplit - 1; k >= 0; --k)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const bool cut = cuts >> k & 1;
        D[e] = cut ? 0.f : (D[e] + g[k][e]) * keep[k][e];
        A[e] = cut ? kCut : A[e] * keep[k][e];
      }
  }

  // dv and df; dh becomes what goes on to the step before.
  __device__ __forceinline__ void back(const ScanArgs& a, const Row& r,
                                       const LaneAt& l, int s0, float* dh) {
    auto step = [&](int k, float* gv, float* gf) {
      const bool cut = cuts >> k & 1;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        dh[e] += g[k][e];
        gv[e] = dh[e] * write[k][e];
        gf[e] = gv[e] * q[k][e] * keep[k][e];
        dh[e] = cut ? 0.f : dh[e] * keep[k][e];
      }
    };
    if (whole.on) {
      const WaveWalk<T> wv(a.dv, whole.t, whole.dir, l.b, l.ch),
          wf(a.df, whole.t, whole.dir, l.b, l.ch);
#pragma unroll
      for (int k = kSplit - 1; k >= 0; --k) {
        float gv[V], gf[V];
        step(k, gv, gf);
        store_pack<T, V>(wv.at(k), gv);
        store_pack<T, V>(wf.at(k), gf);
      }
    } else {
      // back from the last of the steps that the row has
      Walk<T> wv(a.dv, r, l.b, l.ch, s0 + kSplit - 1),
          wf(a.df, r, l.b, l.ch, s0 + kSplit - 1);
#pragma unroll
      for (int k = kSplit - 1; k >= 0; --k) {
        if (s0 + k < r.len) {
          float gv[V], gf[V];
          step(k, gv, gf);
          store_pack<T, V>(wv.p, gv);
          store_pack<T, V>(wf.p, gf);
          wv.p -= wv.step;
          wf.p -= wf.step;
        }
      }
    }
  }
};

// Zeros behind a row's end, of steps [s0, s1).
template <typename T, int V, bool GATE>
__device__ __forceinline__ void zero_behind(const ScanArgs& a, const Row& r,
                                            const LaneAt& l, int s0, int s1) {
  T* pv = (T*)a.dv.p + (int64_t)l.b * a.dv.sb + l.ch;
  T* pf = (T*)a.df.p + (int64_t)l.b * a.df.sb + l.ch;
  T* po = GATE ? (T*)a.d_o.p + (int64_t)l.b * a.d_o.sb + l.ch : nullptr;
  for (int s = max(s0, r.len); s < min(s1, a.q.t); ++s) {
    float z[V];
#pragma unroll
    for (int e = 0; e < V; ++e) z[e] = 0.f;
    store_pack<T, V>(pv + (int64_t)s * a.dv.st, z);
    store_pack<T, V>(pf + (int64_t)s * a.df.st, z);
    if (GATE) store_pack<T, V>(po + (int64_t)s * a.d_o.st, z);
  }
}

// Rows walked from their last step to their first, kSplit steps at a time.
template <typename T, typename O, int V, bool GATE>
__global__ __launch_bounds__(kScanThreads) void k_scan_grad(ScanArgs a) {
  const int64_t lane = (int64_t)blockIdx.x * kScanThreads + threadIdx.x;
  if (lane >= a.lanes) return;
  LaneAt l;
  l.on = true;
  l.b = (int)(lane / a.cv);
  l.ch = (int)(lane % a.cv) * V;
  l.hc = (int64_t)l.b * a.q.c + l.ch;
  const Row r = row_of(a.q, l.b);
  float dh[V];
#pragma unroll
  for (int e = 0; e < V; ++e) dh[e] = a.h ? a.h[l.hc + e] : 0.f;
  zero_behind<T, V, GATE>(a, r, l, 0, a.q.t);
  // (every lane from the last step of all rows: their times stay the same)
  for (int s0 = (a.q.t - 1) / kSplit * kSplit; s0 >= 0; s0 -= kSplit) {
    if (s0 < r.len) {
      GradSteps<T, O, V, GATE> steps;
      steps.forward(a, r, l, s0);
      steps.back(a, r, l, s0, dh);
    }
  }
  if (a.h_out) {
#pragma unroll
    for (int e = 0; e < V; ++e) a.h_out[l.hc + e] = dh[e];
  }
}

// Rows split along time: tiles and waves run from the row's last step.
template <typename T, typename O, int V, bool GATE, int W>
__global__ __launch_bounds__(64 * W) void k_scan_grad_tiles(ScanArgs a) {
  __shared__ TileShared<V, W> sh;
  const int ticket = next_ticket<V, W>(a, sh);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int k_th = ticket / a.cols, col = ticket % a.cols;
  const LaneAt l = lane_at(a, col, V);
  const Row r = row_of(a.q, l.b);
  const int s0 = ((a.tiles - 1 - k_th) * W + W - 1 - wave) * kSplit;
  float dh[V];
#pragma unroll
  for (int e = 0; e < V; ++e) dh[e] = k_th == 0 && a.h ? a.h[l.hc + e] : 0.f;
  const bool any = __any(s0 < r.len);
  GradSteps<T, O, V, GATE> steps;
  float A[V], D[V], TA[V], TD[V];
  none<V>(A, D);
  if (any) {
    steps.forward(a, r, l, s0);
    steps.ends(A, D);
  }
  join_waves<V, W>(sh, wave, A, D, TA, TD);
  float WA[V], WD[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    WA[e] = A[e];
    WD[e] = D[e];
  }
  enter_tile<V, W>(a, sh, k_th, col, wave, TA, TD, dh);
  if (k_th == a.tiles - 1 && a.h_out && wave == 0 && l.on) {
#pragma unroll
    for (int e = 0; e < V; ++e)
      a.h_out[l.hc + e] =
          is_cut(TA[e]) ? TD[e] : __builtin_fmaf(TA[e], dh[e], TD[e]);
  }
#pragma unroll
  for (int e = 0; e < V; ++e)
    dh[e] = is_cut(WA[e]) ? WD[e] : __builtin_fmaf(WA[e], dh[e], WD[e]);
  if (!l.on) return;
  if (any) steps.back(a, r, l, s0, dh);
  zero_behind<T, V, GATE>(a, r, l, s0, s0 + kSplit);
}

}  // namespace

void launch_scan_backward(const ScanArgs& a, int dtype, int out_dtype,
                          bool split, hipStream_t q) {
  with_types(dtype, out_dtype, [&](auto ti, auto to) {
    using T = typename decltype(ti)::type;
    using O = typename decltype(to)::type;
    auto go = [&](auto gt) {
      constexpr bool G = decltype(gt)::value;
      if (split)
        k_scan_grad_tiles<T, O, 1, G, kGradWaves>
            <<<(unsigned)(a.cols * a.tiles), 64 * kGradWaves, 0, q>>>(a);
      else
        k_scan_grad<T, O, 1, G>
            <<<(unsigned)ceil_div(a.lanes, kScanThreads), kScanThreads, 0,
               q>>>(a);
    };
    if (a.o.p)
      go(std::true_type{});
    else
      go(std::false_type{});
  });
}

}  // namespace ops
}  // namespace st
