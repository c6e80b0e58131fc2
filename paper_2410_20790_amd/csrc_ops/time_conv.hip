// Causal depthwise convolution along time with an activation, forward, and
// the host side of both directions.
//
//   y_s = act(bias + sum_j w_j x_{s - K + 1 + j})
//
// 2 K operations per element moved: bound by memory.  A thread takes V
// adjacent channels of one row over a tile of steps and keeps the K - 1
// inputs before the step in registers, so an input is read once (a tile's
// first K - 1 predecessors again, from the caches).
#include "time_conv.h"

namespace st {
namespace ops {
namespace {

constexpr int kAhead = 4;   // steps whose loads a thread has in flight

template <typename T, typename O, int V, int K, bool NARROW>
__global__ __launch_bounds__(kConvThreads) void k_time_conv(ConvTimeArgs a) {
  const int col = threadIdx.x % a.cols, row = threadIdx.x / a.cols;
  const int cb = blockIdx.x % a.colblocks;
  const int vec = cb * a.cols + col;
  if (row >= a.rows || vec >= a.cv) return;
  const int ch = vec * V;
  float w[K][V], bias[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    bias[e] = a.bias ? a.bias[ch + e] : 0.f;
#pragma unroll
    for (int j = 0; j < K; ++j) w[j][e] = a.weight[(int64_t)j * a.q.c + ch + e];
  }
  const int64_t units = (int64_t)a.tiles * a.q.b;
  const int64_t step = (int64_t)a.gridy * a.rows;
  for (int64_t u = (int64_t)(blockIdx.x / a.colblocks) * a.rows + row;
       u < units; u += step) {
    const int b = (int)(u % a.q.b);
    const int tile = (int)(u / a.q.b);
    const Row r = row_of(a.q, b);
    const int s0 = tile * a.tile, s1 = min(s0 + a.tile, a.q.t);
    const int end = min(s1, r.len);
    float win[K > 1 ? K - 1 : 1][V];
    if (s0 < end) load_window<T, V, K>(a, r, b, ch, s0, win);
    Walk<const T, NARROW> wx(a.x, r, b, ch, s0);
    Walk<O, NARROW> wy(a.y, r, b, ch, s0);
    for (int s = s0; s < end; s += kAhead) {
      Pack<T, V> in[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        in[k] = load_pack<T, V>(wx.here());
        wx.next();
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (s + k < end) {
          float f[V], z[V];
          unpack<T, V>(in[k], f);
          if (reset_at(a.q, r, b, s + k)) {
#pragma unroll
            for (int j = 0; j < K - 1; ++j)
#pragma unroll
              for (int e = 0; e < V; ++e) win[j][e] = 0.f;
          }
#pragma unroll
          for (int e = 0; e < V; ++e) {
            z[e] = bias[e];
#pragma unroll
            for (int j = 0; j < K - 1; ++j)
              z[e] = __builtin_fmaf(w[j][e], win[j][e], z[e]);
            z[e] = __builtin_fmaf(w[K - 1][e], f[e], z[e]);
            z[e] = act_any(a.act, z[e]);
          }
          store_pack<O, V>(wy.here(), z);
          wy.next();
#pragma unroll
          for (int e = 0; e < V; ++e) {
#pragma unroll
            for (int j = 0; j + 1 < K - 1; ++j) win[j][e] = win[j + 1][e];
            if (K > 1) win[K > 1 ? K - 2 : 0][e] = f[e];
          }
        }
      }
    }
    O* y = (O*)a.y.p + (int64_t)b * a.y.sb + ch;
    for (int s = max(s0, r.len); s < s1; ++s) {
      float z[V];
#pragma unroll
      for (int e = 0; e < V; ++e) z[e] = 0.f;
      store_pack<O, V>(y + (int64_t)s * a.y.st, z);
    }
    // The row's window for the next call.  The thread that reads `window`
    // writes it too, and an entry only after those it still needs (entry
    // i + len is read before entry i is written, in rising i), so it may be
    // replaced in place.
    if (K > 1 && tile == 0 && a.window_out) {
      const int cut = last_cut<K>(a, r, b);
      for (int i = 0; i < K - 1; ++i) {
        const int p = r.len - (K - 1) + i;
        const T* from = nullptr;
        if (p >= cut) {
          if (p >= 0)
            from = (const T*)a.x.p + time_of(r, p) * a.x.st +
                   (int64_t)b * a.x.sb + ch;
          else if (a.window)
            from = (const T*)a.window +
                   ((int64_t)(K - 1 + p) * a.q.b + b) * a.q.c + ch;
        }
        Pack<T, V> v{};
        if (from) v = load_pack<T, V>(from);
        *(Pack<T, V>*)((T*)a.window_out +
                       ((int64_t)i * a.q.b + b) * a.q.c + ch) = v;
      }
    }
  }
}

// -------------------------------------------------------------- host side

// Threads that a call is cut for: four waves to a SIMD; the backward pass, whose
// tiles have a longer halo, three (601 steps of 48 rows of 512 channels f16 34
// us, 36 with four and 35 with two; 1000 steps of 64 rows of 512 channels bf16
// 45, 46 and 53).
constexpr int64_t kFillThreads = 256 * 1024, kGradThreads = 192 * 1024;
// Channels to a thread of the backward pass, whose registers hold three
// windows: two, 1000 steps of 64 rows of 512 channels bf16 45 us for 50 with
// one (300 steps of 20 rows of 1024 channels 25 for 23); four take 15% more.
constexpr int kGradVec = 2;
constexpr int kTargetBlocks = 1024;

struct ConvCut {
  int v, cv, cols, rows, colblocks, tile, tiles, gridy;
  size_t part_bytes;
};
ConvCut cut_of(const st_seq_desc& d, int taps, bool backward, int v) {
  ConvCut c{};
  c.v = v;
  c.cv = d.c / v;
  c.colblocks = (int)ceil_div(c.cv, kConvThreads);
  c.cols = (int)ceil_div(c.cv, c.colblocks);
  c.rows = kConvThreads / c.cols;
  // a tile's halo is taps - 1 steps: at least four times as many steps
  const int64_t lanes = (int64_t)d.b * c.cv;
  const int64_t least = std::max(8, 4 * (taps - 1));
  const int64_t want = ceil_div((int64_t)d.t * std::max<int64_t>(lanes, 1),
                                backward ? kGradThreads : kFillThreads);
  c.tile = (int)std::max(least, std::min<int64_t>(want, 1 << 20));
  c.tiles = (int)std::max<int64_t>(1, ceil_div(d.t, c.tile));
  const int64_t need = ceil_div((int64_t)c.tiles * d.b, c.rows);
  // the backward pass keeps sums over its units: fewer, longer lists
  const int64_t most = backward
                           ? std::max<int64_t>(1, kTargetBlocks / c.colblocks)
                           : (int64_t)(1 << 20);
  c.gridy = (int)std::max<int64_t>(1, std::min(need, most));
  c.part_bytes =
      backward ? (size_t)c.gridy * (taps + 1) * d.c * sizeof(float) : 0;
  return c;
}

st_status check_conv(const st_seq_desc* d, int32_t taps, int32_t act) {
  if (const st_status s = check_seq(d); s != ST_OK) return s;
  if (taps < 1 || taps > ST_TIME_CONV_MAX_TAPS)
    return bad("taps must be in [1, 8]");
  if (!act_known(act)) return bad("unknown activation");
  return ST_OK;
}
uint64_t conv_space(const st_seq_desc& d, int taps, bool backward) {
  if (!backward || d.b == 0) return 0;
  uint64_t most = 0;
  for (int v = kGradVec; v >= 1; v /= 2)
    if (d.c % v == 0)
      most = std::max<uint64_t>(most, cut_of(d, taps, true, v).part_bytes);
  return most;
}

}  // namespace

void launch_time_conv(const ConvTimeArgs& a, int dtype, int out_dtype,
                      int taps, int vec, hipStream_t stream) {
  const unsigned grid = (unsigned)(a.colblocks * a.gridy);
  with_types(dtype, out_dtype, [&](auto ti, auto to) {
    using T = typename decltype(ti)::type;
    using O = typename decltype(to)::type;
    with_conv_vec(vec, [&](auto vt) {
      with_taps(taps, [&](auto kt) {
        constexpr int V = decltype(vt)::value, K = decltype(kt)::value;
        if (a.narrow)
          k_time_conv<T, O, V, K, true>
              <<<grid, kConvThreads, 0, stream>>>(a);
        else
          k_time_conv<T, O, V, K, false>
              <<<grid, kConvThreads, 0, stream>>>(a);
      });
    });
  });
}

}  // namespace ops
}  // namespace st

using namespace st;
using namespace st::ops;

extern "C" st_status st_time_conv_workspace(const st_seq_desc* d,
                                            int32_t taps, int32_t backward,
                                            uint64_t* bytes) {
  return guarded([&]() -> st_status {
    if (const st_status s = check_conv(d, taps, 0); s != ST_OK) return s;
    if (!bytes) return bad("bytes is NULL");
    *bytes = conv_space(*d, taps, backward != 0);
    return ST_OK;
  });
}

extern "C" st_status st_time_conv(const st_seq_desc* d, int32_t taps,
                                  int32_t act, const st_seq_ref* x,
                                  const float* weight, const float* bias,
                                  const void* window, const st_seq_ref* y,
                                  void* window_out, void* ws,
                                  uint64_t ws_bytes, void* stream) {
  return guarded([&]() -> st_status {
    if (const st_status s = check_conv(d, taps, act); s != ST_OK) return s;
    const int es = esize(d->dtype), eo = esize(d->out_dtype);
    if (const st_status s = check_ref(*d, x, es, false, "x"); s != ST_OK)
      return s;
    if (const st_status s = check_ref(*d, y, eo, true, "y"); s != ST_OK)
      return s;
    if (!weight) return bad("weight is NULL");
    if (const st_status s = check_addresses({weight, bias},
                                            {window, window_out}, es);
        s != ST_OK)
      return s;
    if (const st_status s = check_ws(0, ws, ws_bytes); s != ST_OK) return s;
    const int64_t wb = (int64_t)(taps - 1) * d->b * d->c * es;
    const Span sx = ref_span(*d, x, es), sy = ref_span(*d, y, eo),
               swo = span_of(window_out, wb), sw = span_of(window, wb),
               sk = span_of(weight, (int64_t)taps * d->c * 4),
               sb = span_of(bias, d->c * 4ll),
               sl = span_of(d->lengths, d->b * 4ll),
               sr = span_of(d->reset, (int64_t)d->t * d->b);
    const Span keep = window_out == window ? Span{} : sw;
    if (any_hit({sy, swo}, {sx, keep, sk, sb, sl, sr}) || sy.hits(sw))
      return bad("an output overlaps an input or another output");
    if (d->b == 0) return ST_OK;
    (void)hipGetLastError();
    int v = 4;
    for (; v > 1; v /= 2)
      if (d->c % v == 0 && ops::vec_ok(v, es, *d, x) &&
          ops::vec_ok(v, eo, *d, y) &&
          (uintptr_t)window % (v * es) == 0 &&
          (uintptr_t)window_out % (v * es) == 0)
        break;
    const ConvCut c = cut_of(*d, taps, false, v);
    ConvTimeArgs a{};
    a.q = axes_of(*d);
    a.x = tensor_of(x);
    a.y = tensor_of(y);
    a.weight = weight;
    a.bias = bias;
    a.window = window;
    a.window_out = window_out;
    a.act = act;
    a.cv = c.cv; a.cols = c.cols; a.rows = c.rows;
    a.colblocks = c.colblocks;
    a.tile = c.tile; a.tiles = c.tiles; a.gridy = c.gridy;
    a.narrow = narrow(*d, x, es, d->t) && narrow(*d, y, eo, d->t);
    launch_time_conv(a, d->dtype, d->out_dtype, taps, v, (hipStream_t)stream);
    return launch_status("time convolution");
  });
}

extern "C" st_status st_time_conv_backward(
    const st_seq_desc* d, int32_t taps, int32_t act, const st_seq_ref* dy,
    const st_seq_ref* x, const float* weight, const float* bias,
    const void* window, const void* dwindow_out, const st_seq_ref* dx,
    float* dweight, float* dbias, void* dwindow, void* ws, uint64_t ws_bytes,
    void* stream) {
  return guarded([&]() -> st_status {
    if (const st_status s = check_conv(d, taps, act); s != ST_OK) return s;
    const int es = esize(d->dtype), eo = esize(d->out_dtype);
    if (const st_status s = check_ref(*d, dy, eo, false, "dy"); s != ST_OK)
      return s;
    if (const st_status s = check_ref(*d, x, es, false, "x"); s != ST_OK)
      return s;
    if (dx)
      if (const st_status s = check_ref(*d, dx, es, true, "dx"); s != ST_OK)
        return s;
    if (!weight) return bad("weight is NULL");
    if (const st_status s = check_addresses(
            {weight, bias, dweight, dbias}, {window, dwindow_out, dwindow},
            es);
        s != ST_OK)
      return s;
    if (const st_status s = check_ws(conv_space(*d, taps, true), ws, ws_bytes);
        s != ST_OK)
      return s;
    const int64_t wb = (int64_t)(taps - 1) * d->b * d->c * es;
    const int64_t kb = (int64_t)taps * d->c * 4, cb = d->c * 4ll;
    if (any_hit({ref_span(*d, dx, es), span_of(dweight, kb),
                 span_of(dbias, cb), span_of(dwindow, wb),
                 span_of(ws, (int64_t)ws_bytes)},
                {ref_span(*d, x, es), ref_span(*d, dy, eo),
                 span_of(weight, kb), span_of(bias, cb), span_of(window, wb),
                 span_of(dwindow_out, wb), span_of(d->lengths, d->b * 4ll),
                 span_of(d->reset, (int64_t)d->t * d->b)}))
      return bad("an output overlaps an input, another output or the "
                 "workspace");
    (void)hipGetLastError();
    int v = kGradVec;
    for (; v > 1; v /= 2)
      if (d->c % v == 0 && ops::vec_ok(v, es, *d, x) &&
          ops::vec_ok(v, eo, *d, dy) && ops::vec_ok(v, es, *d, dx) &&
          (uintptr_t)window % (v * es) == 0 &&
          (uintptr_t)dwindow % (v * es) == 0 &&
          (uintptr_t)dwindow_out % (v * es) == 0)
        break;
    const ConvCut c = cut_of(*d, taps, true, v);
    ConvTimeArgs a{};
    a.q = axes_of(*d);
    a.x = tensor_of(x);
    a.dy = tensor_of(dy);
    a.dx = tensor_of(dx);
    a.weight = weight;
    a.bias = bias;
    a.window = window;
    a.dwindow_out = dwindow_out;
    a.dwindow = dwindow;
    a.part = dweight || dbias ? (float*)ws : nullptr;
    a.dweight = dweight;
    a.dbias = dbias;
    a.act = act;
    a.cv = c.cv; a.cols = c.cols; a.rows = c.rows;
    a.colblocks = c.colblocks;
    a.tile = c.tile; a.tiles = c.tiles;
    a.gridy = d->b == 0 ? 0 : c.gridy;
    a.narrow = narrow(*d, x, es, d->t) && narrow(*d, dy, eo, d->t) &&
               narrow(*d, dx, es, d->t);
    launch_time_conv_backward(a, d->dtype, d->out_dtype, taps, v,
                              (hipStream_t)stream);
    return launch_status("time convolution backward");
  });
}
