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

// kSplit steps of a lane: their states come again from the one kept before
// them, forward; the gradients go back through them.  All is read once.  (A
// channel to a lane: four arrays of 16 steps in registers leave no room for a
// second.)
//
// TWO: whole waves have a path of their own, without a test at every step.
// Rows split along time gain by it (36 us for 41, 100 steps of 300 rows of 256
// channels); rows that are walked, with all else in the same loop, lose a wave
// of each SIMD to its registers (9 steps of 2048 rows of 1024 channels f32 114
// us for 135).
template <typename T, typename O, bool GATE, bool NARROW, bool TWO>
struct GradSteps {
  float keep[kSplit], write[kSplit];
  float g[kSplit];     // dy sigmoid(o)
  float q[kSplit];     // h_{s-1} - v
  bool whole;          // all lanes of the wave have all steps
  unsigned cuts;

  // Loads, states, and do.
  __device__ __forceinline__ void forward(const ScanArgs& a, const Row& r,
                                          const LaneAt& l, int s0) {
    whole = __all(s0 + kSplit <= r.len);
    Pack<T, 1> iv[kSplit], jf[kSplit], io[kSplit];
    Pack<O, 1> id[kSplit];
    load_steps<kSplit, NARROW>(a.f, a, r, l.b, l.ch, s0, whole, jf);
    load_steps<kSplit, NARROW>(a.v, a, r, l.b, l.ch, s0, whole, iv);
    if (GATE) load_steps<kSplit, NARROW>(a.o, a, r, l.b, l.ch, s0, whole, io);
    load_steps<kSplit, NARROW>(a.y, a, r, l.b, l.ch, s0, whole, id);
    float h = 0.f;
    if (s0 < r.len)
      h = a.states[(s0 / kStride) * ((int64_t)a.q.b * a.q.c) + l.hc];
    cuts = cuts_of<kSplit, NARROW>(a, r, l.b, s0);
    // a step's values; its do, to out
    auto step = [&](int k, T* out, bool put) {
      const float v = to_f(iv[k].e[0]);
      sigmoids(to_f(jf[k].e[0]), keep[k], write[k]);
      h = cuts >> k & 1 ? 0.f : h;
      q[k] = h - v;
      h = __builtin_fmaf(keep[k], h, write[k] * v);
      g[k] = to_f(id[k].e[0]);
      if (GATE) {
        float p, n;
        sigmoids_once(to_f(io[k].e[0]), p, n);
        g[k] *= p;
        const float go = g[k] * h * n;
        if (put) *out = from_f<T>(go);
      }
    };
    const SeqTensor& to = GATE ? a.d_o : a.dv;
    if (TWO && whole && __all(l.on)) {
      const StepsAt<T, NARROW> out(to, a.q, r, l.b, l.ch, s0);
#pragma unroll
      for (int k = 0; k < kSplit; ++k) step(k, out.at(k), true);
    } else {
      const StepsAt<T, NARROW> out(to, a.q, r, l.b, l.ch, s0);
#pragma unroll
      for (int k = 0; k < kSplit; ++k) {
        // behind the row's end: what comes back passes as it is
        keep[k] = 1.f;
        write[k] = g[k] = q[k] = 0.f;
        if (s0 + k < r.len) step(k, out.at(k), l.on);
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
    if (__any(is_zero(A))) {
      bool zero = false;
#pragma unroll
      for (int k = 0; k < kSplit; ++k) zero = zero || is_zero(keep[k]);
      keep_product(A, zero);
    }
  }

  // dv and df; dh becomes what goes on to the step before.
  __device__ __forceinline__ void back(const ScanArgs& a, const Row& r,
                                       const LaneAt& l, int s0, float& dh) {
    auto step = [&](int k, T* dv, T* df) {
      dh += g[k];
      const float gv = dh * write[k];
      *dv = from_f<T>(gv);
      *df = from_f<T>(gv * q[k] * keep[k]);
      dh = cuts >> k & 1 ? 0.f : dh * keep[k];
    };
    if (whole) {
      const StepsAt<T, NARROW> dv(a.dv, a.q, r, l.b, l.ch, s0),
          df(a.df, a.q, r, l.b, l.ch, s0);
#pragma unroll
      for (int k = kSplit - 1; k >= 0; --k) step(k, dv.at(k), df.at(k));
    } else {
      const StepsAt<T, NARROW> dv(a.dv, a.q, r, l.b, l.ch, s0),
          df(a.df, a.q, r, l.b, l.ch, s0);
#pragma unroll
      for (int k = kSplit - 1; k >= 0; --k)
        if (s0 + k < r.len) step(k, dv.at(k), df.at(k));
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
template <typename T, typename O, bool GATE, bool NARROW>
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
      GradSteps<T, O, GATE, NARROW, false> steps;
      steps.forward(a, r, l, s0);
      steps.back(a, r, l, s0, dh);
    }
  }
  if (a.h_out) a.h_out[l.hc] = dh;
}

// Rows split along time: tiles and waves run from the row's last step.
template <typename T, typename O, bool GATE, bool NARROW, int W>
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
  GradSteps<T, O, GATE, NARROW, true> steps;
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
    with_scan_kind(a, [&](auto gt, auto nt) {
      constexpr bool G = decltype(gt)::value, N = decltype(nt)::value;
      if (split)
        k_scan_grad_tiles<T, O, G, N, kGradWaves>
            <<<(unsigned)(a.cols * a.tiles), 64 * kGradWaves, 0, q>>>(a);
      else
        k_scan_grad<T, O, G, N>
            <<<(unsigned)ceil_div(a.lanes, kScanThreads), kScanThreads, 0,
               q>>>(a);
    });
  });
}

}  // namespace ops
}  // namespace st
