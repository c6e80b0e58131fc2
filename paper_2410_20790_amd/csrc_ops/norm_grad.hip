// Gradients of the group norm.
//
//   dz = dy act'(z);  s1 = mean(dz gamma), s2 = mean(dz gamma xh) per group
//   dx = rstd (dz gamma - s1 - xh s2);  dgamma = sum dz xh, dbeta = sum dz
//
// About twenty operations per element moved: bound by memory.
#include <algorithm>

#include "norm.h"

namespace st {
namespace ops {
namespace {

constexpr int kBatch = 4;        // sites whose loads a thread has in flight

// dz and xh of one vector.
template <int V, bool WHOLE, int ACT>
__device__ __forceinline__ void dz_of(const float* x, float* dy,
                                      const Params<V, WHOLE>& q, float* xh) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    xh[i] = (x[i] - q.mu(i)) * q.r(i);
    if constexpr (ACT != ST_ACT_NONE)
      dy[i] *= act_grad<ACT>(__builtin_fmaf(xh[i], q.gamma[i], q.beta[i]));
  }
}

// A thread's sums of dz and dz xh, per channel.
template <typename T, typename O, int V, bool WHOLE, int ACT>
struct Sums {
  float s1[V], s2[V];
  __device__ __forceinline__ Sums() {
#pragma unroll
    for (int i = 0; i < V; ++i) s1[i] = s2[i] = 0.f;
  }
  __device__ __forceinline__ void add(const Pack<T, V>& rx,
                                      const Pack<O, V>& rd,
                                      const Params<V, WHOLE>& q) {
    float f[V], d[V], xh[V];
    unpack<T, V>(rx, f);
    unpack<O, V>(rd, d);
    dz_of<V, WHOLE, ACT>(f, d, q, xh);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      s1[i] += d[i];
      s2[i] = __builtin_fmaf(d[i], xh[i], s2[i]);
    }
  }
};

// Joins the block's sums: per channel, to `ch` (from the block's first channel
// on), and weighted with gamma per group, group j at res[2 j] for all threads.
template <int V, int TH>
__device__ __forceinline__ void block_sums(const NormArgs& a, const Place& p,
                                           const float* s1, const float* s2,
                                           float* ch, float* res) {
  const NormGeom& g = a.g;
  __shared__ float red[TH * V * 2];
  __shared__ float tot[kMaxCols * V * 2];
  const int tid = threadIdx.x;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < V; ++i) {
    red[(tid * V + i) * 2] = s1[i];
    red[(tid * V + i) * 2 + 1] = s2[i];
  }
  __syncthreads();
  const int n = p.nvec * V * 2, line = g.cols * V * 2;
  int lanes = lanes_per_group(TH, n), in = tid & (lanes - 1);
  for (int i = tid / lanes; i < n; i += TH / lanes) {
    float s = 0.f;
    for (int r = in; r < g.rows; r += lanes) s += red[r * line + i];
    s = lanes_sum(s, lanes);
    if (in == 0) {
      tot[i] = s;
      ch[i] = s;
    }
  }
  __syncthreads();
  const int wide = g.cparts == 1 ? g.cpg : p.nvec * V;
  lanes = lanes_per_group(TH, p.ng);
  in = tid & (lanes - 1);
  for (int j = tid / lanes; j < p.ng; j += TH / lanes) {
    float t1 = 0.f, t2 = 0.f;
    for (int c = j * wide + in; c < (j + 1) * wide; c += lanes) {
      const float gm = a.gamma ? a.gamma[p.vec0 * V + c] : 1.f;
      t1 = __builtin_fmaf(tot[c * 2], gm, t1);
      t2 = __builtin_fmaf(tot[c * 2 + 1], gm, t2);
    }
    t1 = lanes_sum(t1, lanes);
    t2 = lanes_sum(t2, lanes);
    if (in == 0) {
      res[j * 2] = t1;
      res[j * 2 + 1] = t2;
    }
  }
  __syncthreads();
}

// Large images, first: the sums of a range of sites.
template <typename T, typename O, int V, bool WHOLE, int ACT>
__device__ __forceinline__ void sums_unit(const NormArgs& a, const Place& p,
                                          float* res) {
  const NormGeom& g = a.g;
  const int col = threadIdx.x % g.cols, row = threadIdx.x / g.cols;
  Sums<T, O, V, WHOLE, ACT> sums;
  if (row < g.rows && col < p.nvec) {
    const int ch = (p.vec0 + col) * V;
    Params<V, WHOLE> q;
    q.load(a, p.n, ch);
    int64_t s = p.s0 + row;
    SiteWalk<const T> x(a.x, p.n, s, ch);
    SiteWalk<const O> dy(a.dy, p.n, s, ch);
    for (; s + (kBatch - 1) * g.rows < p.s1; s += kBatch * g.rows) {
      Pack<T, V> rx[kBatch];
      Pack<O, V> rd[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        rx[k] = load_pack<T, V>(x.p);
        rd[k] = load_pack<O, V>(dy.p);
        x.next();
        dy.next();
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) sums.add(rx[k], rd[k], q);
    }
    for (; s < p.s1; s += g.rows) {
      sums.add(load_pack<T, V>(x.p), load_pack<O, V>(dy.p), q);
      x.next();
      dy.next();
    }
  }
  block_sums<V, kThreads>(
      a, p, sums.s1, sums.s2,
      a.chpart + (((int64_t)p.n * g.slabs + p.slab) * g.c +
                  (int64_t)p.vec0 * V) * 2,
      res);
  const int part = p.slab * g.cparts + p.cb % g.cparts;
  for (int j = threadIdx.x; j < p.ng; j += kThreads) {
    float* o = a.part +
               (((int64_t)p.n * g.groups + p.g0 + j) * a.parts + part) * 2;
    o[0] = res[j * 2];
    o[1] = res[j * 2 + 1];
  }
}

// s1 and s2 of the block's groups from their parts: group j at res[2 j].
__device__ __forceinline__ void join_sums(const NormArgs& a, const Place& p,
                                          float* res) {
  const NormGeom& g = a.g;
  const int lanes = lanes_per_group(kThreads, p.ng);
  const int in = threadIdx.x & (lanes - 1);
  const float m = (float)((double)g.sites * g.cpg);
  for (int j = threadIdx.x / lanes; j < p.ng; j += kThreads / lanes) {
    const float* part =
        a.part + ((int64_t)p.n * g.groups + p.g0 + j) * a.parts * 2;
    float t1 = 0.f, t2 = 0.f;
#pragma unroll 4
    for (int i = in; i < a.parts; i += lanes) {
      t1 += part[i * 2];
      t2 += part[i * 2 + 1];
    }
    t1 = lanes_sum(t1, lanes);
    t2 = lanes_sum(t2, lanes);
    if (in == 0) {
      res[j * 2] = t1 / m;
      res[j * 2 + 1] = t2 / m;
    }
  }
  __syncthreads();
}

// dx of one vector, group statistics s1, s2 of its channels.
template <typename T, typename O, int V, bool WHOLE, int ACT, bool STREAM>
__device__ __forceinline__ void put_dx(T* dx, const Pack<T, V>& rx,
                                       const Pack<O, V>& rd,
                                       const Params<V, WHOLE>& q,
                                       const float* s1, const float* s2) {
  float f[V], d[V], xh[V];
  unpack<T, V>(rx, f);
  unpack<O, V>(rd, d);
  dz_of<V, WHOLE, ACT>(f, d, q, xh);
#pragma unroll
  for (int i = 0; i < V; ++i)
    f[i] = q.r(i) * (__builtin_fmaf(d[i], q.gamma[i], -s1[WHOLE ? 0 : i]) -
                     xh[i] * s2[WHOLE ? 0 : i]);
  if constexpr (STREAM)
    stream_out<T, V>(dx, f);
  else
    store_pack<T, V>(dx, f);
}

// Large images, then: dx of a range of sites.
template <typename T, typename O, int V, bool WHOLE, int ACT>
__device__ __forceinline__ void dx_unit(const NormArgs& a, const Place& p,
                                        float* res) {
  const NormGeom& g = a.g;
  const int col = threadIdx.x % g.cols, row = threadIdx.x / g.cols;
  join_sums(a, p, res);
  if (row >= g.rows || col >= p.nvec) return;
  const int ch = (p.vec0 + col) * V;
  Params<V, WHOLE> q;
  q.load(a, p.n, ch);
  float s1[V], s2[V];
#pragma unroll
  for (int i = 0; i < (WHOLE ? 1 : V); ++i) {
    const int j = (ch + i) / g.cpg - p.g0;
    s1[i] = res[j * 2];
    s2[i] = res[j * 2 + 1];
  }
  int64_t s = p.s0 + row;
  SiteWalk<const T> x(a.x, p.n, s, ch);
  SiteWalk<const O> dy(a.dy, p.n, s, ch);
  SiteWalk<T> dx(a.y, p.n, s, ch);
  for (; s + (kBatch - 1) * g.rows < p.s1; s += kBatch * g.rows) {
    Pack<T, V> rx[kBatch];
    Pack<O, V> rd[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      rx[k] = stream_pack<T, V>(x.p);
      rd[k] = stream_pack<O, V>(dy.p);
      x.next();
      dy.next();
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      put_dx<T, O, V, WHOLE, ACT, true>(dx.p, rx[k], rd[k], q, s1, s2);
      dx.next();
    }
  }
  for (; s < p.s1; s += g.rows) {
    put_dx<T, O, V, WHOLE, ACT, true>(dx.p, load_pack<T, V>(x.p),
                                load_pack<O, V>(dy.p), q, s1, s2);
    x.next();
    dy.next();
    dx.next();
  }
}

// dgamma and dbeta of 32 channels from the sums of all images' site ranges, 8
// lanes of them to a channel, in f64.
__device__ __forceinline__ void sum_channels(const NormArgs& a, int block) {
  __shared__ double red[2][8][32];
  const int cx = threadIdx.x & 31, k = threadIdx.x >> 5;
  const int c = block * 32 + cx;
  double d1 = 0, d2 = 0;
  if (c < a.g.c && k < 8) {
    const int64_t all = (int64_t)a.g.n * a.g.slabs;
#pragma unroll 8
    for (int64_t i = k; i < all; i += 8) {
      d1 += a.chpart[(i * a.g.c + c) * 2];
      d2 += a.chpart[(i * a.g.c + c) * 2 + 1];
    }
  }
  if (k < 8) {
    red[0][k][cx] = d1;
    red[1][k][cx] = d2;
  }
  __syncthreads();
  if (k == 0 && c < a.g.c) {
    for (int i = 1; i < 8; ++i) {
      d1 += red[0][i][cx];
      d2 += red[1][i][cx];
    }
    if (a.dbeta) a.dbeta[c] = (float)d1;
    if (a.dgamma) a.dgamma[c] = (float)d2;
  }
}
__global__ __launch_bounds__(kThreads) void k_norm_channels(NormArgs a) {
  sum_channels(a, blockIdx.x);
}

// A launch over large images: blocks finish the images [end0, end1) and sum up
// [sum0, sum1), in turn; the last launch's first blocks sum the channels.
template <typename T, typename O, int V, bool WHOLE, int ACT>
__global__ __launch_bounds__(kThreads) void k_norm_grad_pass(NormArgs a) {
  __shared__ float res[kMaxCols * (WHOLE ? 1 : V) * 2];
  if ((int)blockIdx.x < a.dblocks) {
    sum_channels(a, blockIdx.x);
    return;
  }
  const int ends = (a.end1 - a.end0) * a.g.units;
  const int all = ends + (a.sum1 - a.sum0) * a.g.units;
  for (int b = blockIdx.x - a.dblocks; b < all;
       b += gridDim.x - a.dblocks) {
    const Turn t(a, b, ends, all);
    const Place p = place_of(a.g, t.n, t.u);
    if (t.end)
      dx_unit<T, O, V, WHOLE, ACT>(a, p, res);
    else
      sums_unit<T, O, V, WHOLE, ACT>(a, p, res);
    __syncthreads();
  }
}

// Images whose groups fit a block's registers: x and dy read once, R sites of
// both to a thread.
template <typename T, typename O, int V, bool WHOLE, int TH, int R>
__global__ __launch_bounds__(TH) void k_norm_grad_held(NormArgs a) {
  const NormGeom& g = a.g;
  __shared__ float res[kMaxCols * (WHOLE ? 1 : V) * 2];
  const int col = threadIdx.x % g.cols, row = threadIdx.x / g.cols;
  const int u = near_block((a.end1 - a.end0) * g.units);
  const Place p = place_of(g, a.end0 + u / g.units, u % g.units);
  const bool on = row < g.rows && col < p.nvec;
  const int ch = (p.vec0 + (on ? col : 0)) * V;
  const int left = on ? (int)g.sites - row : 0;   // sites from its own on
  Pack<T, V> rx[R];
  Pack<O, V> rd[R];
  SiteWalk<const T> x(a.x, p.n, row, ch);
  SiteWalk<const O> dy(a.dy, p.n, row, ch);
#pragma unroll
  for (int k = 0; k < R; ++k) {
    if (k * g.rows < left) {
      rx[k] = load_pack<T, V>(x.p);
      rd[k] = load_pack<O, V>(dy.p);
    }
    x.next();
    dy.next();
  }
  Params<V, WHOLE> q;
  q.load(a, p.n, ch);
  with_activation_of(a.act, [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    Sums<T, O, V, WHOLE, ACT> sums;
#pragma unroll
    for (int k = 0; k < R; ++k)
      if (k * g.rows < left) sums.add(rx[k], rd[k], q);
    block_sums<V, TH>(
        a, p, sums.s1, sums.s2,
        a.chpart + ((int64_t)p.n * g.c + (int64_t)p.vec0 * V) * 2, res);
    const float m = (float)((double)g.sites * g.cpg);
    float s1[V], s2[V];
#pragma unroll
    for (int i = 0; i < (WHOLE ? 1 : V); ++i) {
      const int j = (ch + i) / g.cpg - p.g0;
      s1[i] = res[j * 2] / m;
      s2[i] = res[j * 2 + 1] / m;
    }
    SiteWalk<T> dx(a.y, p.n, row, ch);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (k * g.rows < left)
        put_dx<T, O, V, WHOLE, ACT, false>(dx.p, rx[k], rd[k], q, s1, s2);
      dx.next();
    }
  });
}

}  // namespace

void launch_norm_backward(const NormArgs& a, int dtype, int out_dtype,
                          int held, int batch, hipStream_t q) {
  if (a.g.n == 0) {
    k_norm_channels<<<a.dblocks, kThreads, 0, q>>>(a);
    return;
  }
  with_norm(dtype, out_dtype, a.g, [&](auto ti, auto to, auto vt, auto wt) {
    using T = typename decltype(ti)::type;
    using O = typename decltype(to)::type;
    constexpr int V = decltype(vt)::value;
    constexpr bool W = decltype(wt)::value;
    if (held) {
      with_held(a, [&](const NormArgs& b, unsigned grid) {
        if (held == kFewThreads)
          k_norm_grad_held<T, O, V, W, kFewThreads, kHeld>
              <<<grid, kFewThreads, 0, q>>>(b);
        else
          k_norm_grad_held<T, O, V, W, kManyThreads, kHeld / 2>
              <<<grid, kManyThreads, 0, q>>>(b);
      });
      if (a.dblocks) k_norm_channels<<<a.dblocks, kThreads, 0, q>>>(a);
      return;
    }
    with_activation(a.act, [&](auto act) {
      with_batches(a, batch, [&](NormArgs b, bool last) {
        if (!last) b.dblocks = 0;
        k_norm_grad_pass<T, O, V, W, decltype(act)::value>
            <<<pass_blocks(b) + b.dblocks, kThreads, 0, q>>>(b);
      });
    });
  });
}

}  // namespace ops
}  // namespace st
