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

uint64_t scan_space(const st_seq_desc&, bool) { return 0; }

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
    with_types(d->dtype, d->out_dtype, [&](auto ti, auto to) {
      using T = typename decltype(ti)::type;
      using O = typename decltype(to)::type;
      with_scan(vec, o != nullptr, [&](auto vt, auto gt) {
        k_scan<T, O, decltype(vt)::value, decltype(gt)::value>
            <<<grid, kThreads, 0, (hipStream_t)stream>>>(a);
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
    with_types(d->dtype, d->out_dtype, [&](auto ti, auto to) {
      using T = typename decltype(ti)::type;
      using O = typename decltype(to)::type;
      with_scan(vec, o != nullptr, [&](auto vt, auto gt) {
        k_scan_grad<T, O, decltype(vt)::value, decltype(gt)::value>
            <<<grid, kThreads, 0, (hipStream_t)stream>>>(a);
      });
    });
    return launch_status("gated scan backward");
  });
}
