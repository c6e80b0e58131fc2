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

// (A channel to a lane: four arrays of 16 steps in registers leave no room for
// a second.)
//
// kSplit steps of a lane: their states come again from the one kept before
// them, forward; the gradients go back through them.  All is read once.
template <typename T, typename O, bool GATE>
struct GradSteps {
  float keep[kSplit], write[kSplit];
  float g[kSplit];     // dy sigmoid(o)
  float q[kSplit];     // h_{s-1} - v
  Whole whole;
  unsigned cuts;

  // Loads, states, and do.
  __device__ __forceinline__ void forward(const ScanArgs& a, const Row& r,
                                          const LaneAt& l, int s0) {
    whole = whole_wave(a, r, s0, kSplit);
    Pack<T, 1> iv[kSplit], jf[kSplit], io[kSplit];
    Pack<O, 1> id[kSplit];
    load_steps<T, 1, kSplit>(a.f, whole, a, r, l.b, l.ch, s0, jf);
    load_steps<T, 1, kSplit>(a.v, whole, a, r, l.b, l.ch, s0, iv);
    if (GATE) load_steps<T, 1, kSplit>(a.o, whole, a, r, l.b, l.ch, s0, io);
    load_steps<O, 1, kSplit>(a.y, whole, a, r, l.b, l.ch, s0, id);
    float h = 0.f;
    if (s0 < r.len)
      h = a.states[(s0 / kStride) * ((int64_t)a.q.b * a.q.c) + l.hc];
    cuts = cuts_of<kSplit>(a, r, l.b, s0);
    auto step = [&](int k) {
      const bool cut = cuts >> k & 1;
      const float v = to_f(iv[k].e[0]);
      g[k] = to_f(id[k].e[0]);
      sigmoids(to_f(jf[k].e[0]), keep[k], write[k]);
      h = cut ? 0.f : h;
      q[k] = h - v;
      h = __builtin_fmaf(keep[k], h, write[k] * v);
      if constexpr (GATE) {
        float p, n;
        sigmoids_once(to_f(io[k].e[0]), p, n);
        g[k] *= p;
        return g[k] * h * n;
      } else {
        return 0.f;
      }
    };
    if (whole.on && __all(l.on)) {
      const WaveWalk<T> w(GATE ? a.d_o : a.dv, whole.t, whole.dir, l.b, l.ch);
#pragma unroll
      for (int k = 0; k < kSplit; ++k) {
        const float go = step(k);
        if (GATE) *w.at(k) = from_f<T>(go);
      }
    } else {
      Walk<T> w(GATE ? a.d_o : a.dv, r, l.b, l.ch, s0);
#pragma unroll
      for (int k = 0; k < kSplit; ++k) {
        // behind the row's end: what comes back passes as it is
        keep[k] = 1.f;
        write[k] = g[k] = q[k] = 0.f;
        if (s0 + k < r.len) {
          const float go = step(k);
          if (GATE && l.on) {
            *w.p = from_f<T>(go);
            w.next();
          }
        }
      }
    }
  }

  // What the steps do to a gradient that comes back: d -> A d + D.
  __device__ __forceinline__ void ends(float& A, float& D) const {
    A = 1.f;
    D = 0.f;
#pragma unroll
    for (int k = kSplit - 1; k >= 0; --k) {
      const bool cut = cuts >> k & 1;
      D = cut ? 0.f : (D + g[k]) * keep[k];
      A = cut ? kCut : A * keep[k];
    }
  }

  // dv and df; dh becomes what goes on to the step before.
  __device__ __forceinline__ void back(const ScanArgs& a, const Row& r,
                                       const LaneAt& l, int s0, float& dh) {
    auto step = [&](int k, T* dv, T* df) {
      const bool cut = cuts >> k & 1;
      dh += g[k];
      const float gv = dh * write[k];
      *dv = from_f<T>(gv);
      *df = from_f<T>(gv * q[k] * keep[k]);
      dh = cut ? 0.f : dh * keep[k];
    };
    if (whole.on) {
      const WaveWalk<T> wv(a.dv, whole.t, whole.dir, l.b, l.ch),
          wf(a.df, whole.t, whole.dir, l.b, l.ch);
#pragma unroll
      for (int k = kSplit - 1; k >= 0; --k) step(k, wv.at(k), wf.at(k));
    } else {
      // back from the last of the steps that the row has
      Walk<T> wv(a.dv, r, l.b, l.ch, s0 + kSplit - 1),
          wf(a.df, r, l.b, l.ch, s0 + kSplit - 1);
#pragma unroll
      for (int k = kSplit - 1; k >= 0; --k) {
        if (s0 + k < r.len) {
          step(k, wv.p, wf.p);
          wv.p -= wv.step;
          wf.p -= wf.step;
        }
      }
    }
  }
};

// Zeros behind a row's end, of steps [s0, s1).
template <typename T, bool GATE>
__device__ __forceinline__ void zero_behind(const ScanArgs& a, const Row& r,
                                            const LaneAt& l, int s0, int s1) {
  T* pv = (T*)a.dv.p + (int64_t)l.b * a.dv.sb + l.ch;
  T* pf = (T*)a.df.p + (int64_t)l.b * a.df.sb + l.ch;
  T* po = GATE ? (T*)a.d_o.p + (int64_t)l.b * a.d_o.sb + l.ch : nullptr;
  for (int s = max(s0, r.len); s < min(s1, a.q.t); ++s) {
    pv[(int64_t)s * a.dv.st] = from_f<T>(0.f);
    pf[(int64_t)s * a.df.st] = from_f<T>(0.f);
    if (GATE) po[(int64_t)s * a.d_o.st] = from_f<T>(0.f);
  }
}

// Rows walked from their last step to their first, kSplit steps at a time.
template <typename T, typename O, bool GATE>
__global__ __launch_bounds__(kScanThreads) void k_scan_grad(ScanArgs a) {
  const int64_t lane = (int64_t)blockIdx.x * kScanThreads + threadIdx.x;
  if (lane >= a.lanes) return;
  LaneAt l;
  l.on = true;
  l.b = (int)(lane / a.cv);
  l.ch = (int)(lane % a.cv);
  l.hc = lane;
  const Row r = row_of(a.q, l.b);
  float dh = a.h ? a.h[l.hc] : 0.f;
  zero_behind<T, GATE>(a, r, l, 0, a.q.t);
  // (every lane from the last step of all rows: their times stay the same)
  for (int s0 = (a.q.t - 1) / kSplit * kSplit; s0 >= 0; s0 -= kSplit) {
    if (s0 < r.len) {
      GradSteps<T, O, GATE> steps;
      steps.forward(a, r, l, s0);
      steps.back(a, r, l, s0, dh);
    }
  }
  if (a.h_out) a.h_out[l.hc] = dh;
}

// Rows split along time: tiles and waves run from the row's last step.
template <typename T, typename O, bool GATE, int W>
__global__ __launch_bounds__(64 * W) void k_scan_grad_tiles(ScanArgs a) {
  __shared__ TileShared<W> sh;
  const int ticket = next_ticket(a, sh);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int k_th = ticket / a.cols, col = ticket % a.cols;
  const LaneAt l = lane_at(a, col);
  const Row r = row_of(a.q, l.b);
  const int s0 = ((a.tiles - 1 - k_th) * W + W - 1 - wave) * kSplit;
  float dh = k_th == 0 && a.h ? a.h[l.hc] : 0.f;
  const bool any = __any(s0 < r.len);
  GradSteps<T, O, GATE> steps;
  float A = 1.f, D = 0.f, TA, TD;
  if (any) {
    steps.forward(a, r, l, s0);
    steps.ends(A, D);
  }
  if (k_th == 0) arrived(dh);
  join_waves(sh, wave, A, D, TA, TD);
  const float WA = A, WD = D;     // what runs before the wave in its tile
  enter_tile(a, sh, k_th, col, wave, TA, TD, dh);
  if (k_th == a.tiles - 1 && a.h_out && wave == 0 && l.on)
    a.h_out[l.hc] = after(TA, TD, dh);
  dh = after(WA, WD, dh);
  if (!l.on) return;
  if (any) steps.back(a, r, l, s0, dh);
  zero_behind<T, GATE>(a, r, l, s0, s0 + kSplit);
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
        k_scan_grad_tiles<T, O, G, kGradWaves>
            <<<(unsigned)(a.cols * a.tiles), 64 * kGradWaves, 0, q>>>(a);
      else
        k_scan_grad<T, O, G>
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
