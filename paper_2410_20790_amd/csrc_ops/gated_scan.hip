// Gated linear recurrence along time, forward, and the host side of both
// directions.
//
//   h_s = a_s h_{s-1} + u_s,  a = sigmoid(f), u = sigmoid(-f) v
//   y_s = h_s sigmoid(o_s)
//
// Some 16 operations per element of three read and one written; the two
// sigmoids make them about 40 instruction slots, of the some 70 that the vector
// units have while memory moves an element of two bytes each way.
#include "gated_scan.h"

namespace st {
namespace ops {
namespace {

// Rows walked from their first step to their last, one thread to V channels of
// a row, the loads of L steps in flight.
template <typename T, typename O, int V, bool GATE, bool NARROW>
__global__ __launch_bounds__(kScanThreads) void k_scan(ScanArgs a) {
  constexpr int L = kStride / V;
  const int64_t lane = (int64_t)blockIdx.x * kScanThreads + threadIdx.x;
  if (lane >= a.lanes) return;
  const int b = (int)(lane / a.cv), ch = (int)(lane % a.cv) * V;
  const Row r = row_of(a.q, b);
  const int64_t hc = (int64_t)b * a.q.c + ch;
  const int64_t plane = (int64_t)a.q.b * a.q.c;
  float h[V];
#pragma unroll
  for (int e = 0; e < V; ++e) h[e] = a.h ? a.h[hc + e] : 0.f;
  for (int s = 0; s < r.len; s += L) {
    const bool whole = __all(s + L <= r.len);
    Pack<T, V> iv[L], jf[L], io[L];
    load_steps<L, NARROW>(a.f, a, r, b, ch, s, whole, jf);
    load_steps<L, NARROW>(a.v, a, r, b, ch, s, whole, iv);
    if (GATE) load_steps<L, NARROW>(a.o, a, r, b, ch, s, whole, io);
    if (a.states && s % kStride == 0)
      store_pack<float, V>(a.states + (s / kStride) * plane + hc, h);
    auto step = [&](int k, O* y) {
      float v[V], f[V], o[V], z[V];
      unpack<T, V>(iv[k], v);
      unpack<T, V>(jf[k], f);
      if (GATE) unpack<T, V>(io[k], o);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        float keep, write;
        sigmoids(f[e], keep, write);
        h[e] = __builtin_fmaf(keep, h[e], write * v[e]);
        z[e] = GATE ? h[e] * sigmoid_once(o[e]) : h[e];
      }
      store_pack<O, V>(y, z);
    };
    if (whole && !a.q.reset) {
      const StepsAt<O, NARROW> y(a.y, a.q, r, b, ch, s);
#pragma unroll
      for (int k = 0; k < L; ++k) step(k, y.at(k));
    } else {
      const StepsAt<O, NARROW> y(a.y, a.q, r, b, ch, s);
#pragma unroll
      for (int k = 0; k < L; ++k) {
        if (s + k < r.len) {
          if (reset_at(a.q, r, b, s + k)) {
#pragma unroll
            for (int e = 0; e < V; ++e) h[e] = 0.f;
          }
          step(k, y.at(k));
        }
      }
    }
  }
  O* y = (O*)a.y.p + (int64_t)b * a.y.sb + ch;
  for (int s = r.len; s < a.q.t; ++s) {
    float z[V];
#pragma unroll
    for (int e = 0; e < V; ++e) z[e] = 0.f;
    store_pack<O, V>(y + (int64_t)s * a.y.st, z);
  }
  if (a.h_out) {
#pragma unroll
    for (int e = 0; e < V; ++e) a.h_out[hc + e] = h[e];
  }
}

template <typename T, typename O, bool GATE, bool NARROW, int W>
__global__ __launch_bounds__(64 * W) void k_scan_tiles(ScanArgs a) {
  __shared__ TileShared<W> sh;
  const int ticket = next_ticket(a, sh);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int tile = ticket / a.cols, col = ticket % a.cols;
  const LaneAt l = lane_at(a, col);
  const Row r = row_of(a.q, l.b);
  const int64_t plane = (int64_t)a.q.b * a.q.c;
  const int s0 = (tile * W + wave) * kSplit;
  float h = tile == 0 && a.h ? a.h[l.hc] : 0.f;
  const bool any = __any(s0 < r.len);
  const bool whole = __all(s0 + kSplit <= r.len);
  float keep[kSplit], u[kSplit];
  Pack<T, 1> io[kSplit];
  unsigned cuts = 0;
  bool cutting = false;
  float A = 1.f, H = 0.f, TA, TH;
  if (any) {
    cuts = cuts_of<kSplit, NARROW>(a, r, l.b, s0);
    Pack<T, 1> iv[kSplit], jf[kSplit];
    // (one branch over all loads: with one in each, 100 steps of 300 rows of
    // 256 channels take 11% more; the backward pass, of more loads, takes up to
    // 10% less)
    if (s0 < r.len) {
      load_steps<kSplit, NARROW>(a.f, a, r, l.b, l.ch, s0, whole, jf);
      load_steps<kSplit, NARROW>(a.v, a, r, l.b, l.ch, s0, whole, iv);
      if (GATE)
        load_steps<kSplit, NARROW>(a.o, a, r, l.b, l.ch, s0, whole, io);
    }
#pragma unroll
    for (int k = 0; k < kSplit; ++k) {
      float write;
      sigmoids(to_f(jf[k].e[0]), keep[k], write);
      u[k] = write * to_f(iv[k].e[0]);
    }
    // steps behind the row's end keep the state, to the bit
    if (!whole) {
#pragma unroll
      for (int k = 0; k < kSplit; ++k) {
        keep[k] = s0 + k < r.len ? keep[k] : 1.f;
        u[k] = s0 + k < r.len ? u[k] : 0.f;
      }
    }
    cutting = __any(cuts != 0);
    if (cutting) {
#pragma unroll
      for (int k = 0; k < kSplit; ++k) {
        const bool cut = cuts >> k & 1;
        H = __builtin_fmaf(keep[k], cut ? 0.f : H, u[k]);
        A = cut ? kCut : A * keep[k];
      }
    } else {
#pragma unroll
      for (int k = 0; k < kSplit; ++k) {
        H = __builtin_fmaf(keep[k], H, u[k]);
        A *= keep[k];
      }
    }
    if (__any(is_zero(A))) {
      bool zero = false;
#pragma unroll
      for (int k = 0; k < kSplit; ++k) zero = zero || is_zero(keep[k]);
      keep_product(A, zero);
    }
  }
  if (tile == 0) arrived(h);
  join_waves(sh, wave, A, H, TA, TH);
  const float WA = A, WH = H;     // what runs before the wave in its tile
  enter_tile(a, sh, tile, col, wave, TA, TH, h);
  if (tile == a.tiles - 1 && a.h_out && wave == 0 && l.on)
    a.h_out[l.hc] = after(TA, TH, h);
  h = after(WA, WH, h);
  if (!l.on) return;
  if (any) {
    if (a.states && s0 < r.len) a.states[(s0 / kStride) * plane + l.hc] = h;
    auto gated = [&](int k) {
      return GATE ? h * sigmoid_once(to_f(io[k].e[0])) : h;
    };
    const StepsAt<O, NARROW> y(a.y, a.q, r, l.b, l.ch, s0);
    if (whole && !cutting) {
#pragma unroll
      for (int k = 0; k < kSplit; ++k) {
        h = __builtin_fmaf(keep[k], h, u[k]);
        *y.at(k) = from_f<O>(gated(k));
      }
    } else {
#pragma unroll
      for (int k = 0; k < kSplit; ++k) {
        if (s0 + k < r.len) {
          if (cuts >> k & 1) h = 0.f;
          h = __builtin_fmaf(keep[k], h, u[k]);
          *y.at(k) = from_f<O>(gated(k));
        }
      }
    }
  }
  O* y = (O*)a.y.p + (int64_t)l.b * a.y.sb + l.ch;
  const int s1 = min(s0 + kSplit, a.q.t);
  for (int s = max(s0, r.len); s < s1; ++s)
    y[(int64_t)s * a.y.st] = from_f<O>(0.f);
}

// Clears the words and the ticket of a launch.
__global__ __launch_bounds__(256) void k_scan_clear(uint4* w, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n;
       i += (int64_t)gridDim.x * 256)
    w[i] = make_uint4(0, 0, 0, 0);
}

// -------------------------------------------------------------- host side

template <class F>
void with_lane_vec(int v, F&& f) {
  if (v == 4)
    f(Int<4>{});
  else if (v == 2)
    f(Int<2>{});
  else
    f(Int<1>{});
}

// Which rows are split along time: those of more than 32 steps (a chunk's
// frames, so many at most, are walked one after another, as they are taken one
// by one: the same bits) of which there are too few to fill the device, a wave
// for each 64 channels.  What fills it, measured on both sides (us, split and
// walked, bf16, rows of 512 channels unless said):
//   forward   1000 steps, 150 rows 163 and 266, 300 rows 314 and 317;
//             300 steps, 200 rows 76 and 71; 100 steps, 300 rows of 256
//             channels 19 and 26
//   backward  1000 steps, 150 rows 272 and 377, 300 rows 534 and 501;
//             300 steps, 400 rows 227 and 240, 600 rows 337 and 286;
//             100 steps, 300 rows of 256 channels 46 and 38, 200 rows 37 and
//             32; 60 steps of 8 rows 8 and 17
constexpr int kSerialSteps = 32, kShortSteps = 128;
constexpr int64_t kFillWaves = 2048;    // eight to a CU
int64_t split_waves(const st_seq_desc& d, bool backward) {
  if (!backward) return kFillWaves;
  return d.t > kShortSteps ? 2 * kFillWaves : kFillWaves / 2;
}
constexpr int64_t kMaxBlocks = 1 << 22;

constexpr int kTile = kSplit * kWaves, kGradTile = kSplit * kGradWaves;

// Inputs that the last-level cache cannot hold are read past its reuse order:
// 9 steps of 2048 rows of 2048 channels f32 106 us (125); a chunk that it
// does hold would lose, 82 MB 28 us for 25.
constexpr int64_t kCacheBytes = 256 << 20;
int streamed(const st_seq_desc& d, int64_t bytes_of_a_channel) {
  return (int64_t)d.t * d.b * d.c > kCacheBytes / bytes_of_a_channel;
}

struct ScanCut {
  bool split = false;
  int cols = 0, tiles = 0, group = 0;
  uint64_t words = 0;
};
ScanCut cut_of(const st_seq_desc& d, bool backward) {
  const int steps = backward ? kGradTile : kTile;
  ScanCut c;
  const int64_t cols = ceil_div((int64_t)d.b * d.c, 64);
  if (d.t <= kSerialSteps || cols >= split_waves(d, backward))
    return c;
  // (as many blocks as a launch may have; beyond that, rows are walked)
  if (cols * ceil_div(d.t, steps) > kMaxBlocks) return c;
  c.split = true;
  c.cols = (int)cols;
  c.tiles = (int)ceil_div(d.t, steps);
  // a block folds at most group tiles and tiles / group groups
  c.group = 8;
  while ((int64_t)c.group * c.group < c.tiles) c.group *= 2;
  if (c.tiles > 1)
    c.words = kHeadWords +
              (uint64_t)(c.tiles + c.tiles / c.group) * c.cols * 64;
  return c;
}

uint64_t scan_space(const st_seq_desc& d, bool backward) {
  if (empty(d)) return 0;
  const uint64_t words = cut_of(d, backward).words;
  return (words * 8 + 15) / 16 * 16;
}

// Channels to a lane of rows that are walked: as many as a vector has, while
// there are lanes enough.
int lane_vec(const st_seq_desc& d, int vec) {
  while (vec > 1 && (int64_t)d.b * (d.c / vec) < kFillWaves * 64) vec /= 2;
  return vec;
}
// Clears the workspace of a launch of split rows.
void take_cut(ScanArgs& a, const ScanCut& c, void* ws, hipStream_t q) {
  a.cols = c.cols;
  a.tiles = c.tiles;
  a.group = c.group;
  a.ends = ws;
  if (c.words) {
    const int64_t n = (int64_t)(c.words + 1) / 2;
    k_scan_clear<<<(unsigned)std::min<int64_t>(ceil_div(n, 256), 1024), 256,
                   0, q>>>((uint4*)ws, n);
  }
}

}  // namespace

void launch_scan(const ScanArgs& a, int dtype, int out_dtype, int vec,
                 bool split, hipStream_t q) {
  with_types(dtype, out_dtype, [&](auto ti, auto to) {
    using T = typename decltype(ti)::type;
    using O = typename decltype(to)::type;
    with_scan_kind(a, [&](auto gt, auto nt) {
      constexpr bool G = decltype(gt)::value, N = decltype(nt)::value;
      if (split)
        k_scan_tiles<T, O, G, N, kWaves>
            <<<(unsigned)(a.cols * a.tiles), 64 * kWaves, 0, q>>>(a);
      else
        with_lane_vec(vec, [&](auto vt) {
          k_scan<T, O, decltype(vt)::value, G, N>
              <<<(unsigned)ceil_div(a.lanes, kScanThreads), kScanThreads, 0,
                 q>>>(a);
        });
    });
  });
}

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
    const int es = esize(d->dtype), eo = esize(d->out_dtype);
    if (const st_status s = check_ref(*d, v, es, false, "v"); s != ST_OK)
      return s;
    if (const st_status s = check_ref(*d, f, es, false, "f"); s != ST_OK)
      return s;
    if (o)
      if (const st_status s = check_ref(*d, o, es, false, "o"); s != ST_OK)
        return s;
    if (const st_status s = check_ref(*d, y, eo, true, "y"); s != ST_OK)
      return s;
    if (const st_status s = check_addresses({h, h_out, states}, {}, es);
        s != ST_OK)
      return s;
    if (const st_status s = check_ws(scan_space(*d, false), ws, ws_bytes);
        s != ST_OK)
      return s;
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
    a.stream = streamed(*d, (o ? 3 : 2) * es);
    const st_seq_ref rs{nullptr, d->b, 1};
    const int64_t reach = steps_reach(*d);
    a.narrow = narrow(*d, y, eo, reach) && narrow(*d, &rs, 1, reach);
    for (const st_seq_ref* r : {v, f, o})
      a.narrow = a.narrow && narrow(*d, r, es, reach);
    a.h = h;
    a.h_out = h_out;
    a.states = states;
    hipStream_t q = (hipStream_t)stream;
    const ScanCut cut = cut_of(*d, false);
    vec = cut.split ? 1 : lane_vec(*d, vec);
    a.cv = d->c / vec;
    a.lanes = (int64_t)d->b * a.cv;
    take_cut(a, cut, ws, q);
    launch_scan(a, d->dtype, d->out_dtype, vec, cut.split, q);
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
    const int es = esize(d->dtype), eo = esize(d->out_dtype);
    if (!o != !d_o) return bad("o and d_o: both or neither");
    struct { const st_seq_ref* r; int es; bool out; const char* name; }
    refs[] = {{dy, eo, false, "dy"}, {v, es, false, "v"},
              {f, es, false, "f"},   {dv, es, true, "dv"},
              {df, es, true, "df"},  {o, es, false, "o"},
              {d_o, es, true, "d_o"}};
    for (int i = 0; i < (o ? 7 : 5); ++i)
      if (const st_status s = check_ref(*d, refs[i].r, refs[i].es,
                                        refs[i].out, refs[i].name);
          s != ST_OK)
        return s;
    if (const st_status s = check_addresses({states, dh_out, dh}, {}, es);
        s != ST_OK)
      return s;
    if (!states && !empty(*d)) return bad("states is NULL");
    if (const st_status s = check_ws(scan_space(*d, true), ws, ws_bytes);
        s != ST_OK)
      return s;
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
    ScanArgs a{};
    a.q = axes_of(*d);
    a.v = tensor_of(v);
    a.f = tensor_of(f);
    a.o = tensor_of(o);
    a.y = tensor_of(dy);
    a.dv = tensor_of(dv);
    a.df = tensor_of(df);
    a.d_o = tensor_of(d_o);
    a.stream = streamed(*d, (o ? 3 : 2) * es + eo);
    const st_seq_ref rs{nullptr, d->b, 1};
    const int64_t reach = steps_reach(*d);
    a.narrow = narrow(*d, dy, eo, reach) && narrow(*d, &rs, 1, reach);
    for (const st_seq_ref* r : {v, f, o, dv, df, d_o})
      a.narrow = a.narrow && narrow(*d, r, es, reach);
    a.h = dh_out;
    a.h_out = dh;
    a.states = const_cast<float*>(states);
    hipStream_t q = (hipStream_t)stream;
    const ScanCut cut = cut_of(*d, true);
    a.cv = d->c;
    a.lanes = (int64_t)d->b * d->c;
    take_cut(a, cut, ws, q);
    launch_scan_backward(a, d->dtype, d->out_dtype, cut.split, q);
    return launch_status("gated scan backward");
  });
}
