// Group norm with an activation on channels-last maps, forward and backward.
//
//   mean, var over an image's sites and the c / groups channels of a group
//   xh = (x - mean) rstd,  z = xh gamma + beta,  y = act(z)
//   dz = dy act'(z);  s1 = mean(dz gamma), s2 = mean(dz gamma xh) per group
//   dx = rstd (dz gamma - s1 - xh s2);  dgamma = sum dz xh, dbeta = sum dz
//
// About ten (backward twenty) operations per element moved: bound by memory.
// The channels of a site are adjacent, so a block takes `cols` vectors of V
// adjacent channels of `rows` sites at a time, and a thread meets the same
// channels at every site: their parameters stay in its registers.
#include <algorithm>
#include <numeric>

#include "ops_common.h"

namespace st {
namespace ops {
namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;        // sites whose loads a thread has in flight
constexpr int kMaxDirectParts = 64;

// How the channels are cut.  A column block holds whole groups, or (groups
// wider than a block) one of `cparts` parts of one group.
struct NormGeom {
  int64_t sites;       // per image
  int h1;              // the sites of an image are w steps of stride_w
  int w;
  int n, c, groups, cpg;
  int v;               // channels per vector
  int whole;           // every vector lies in one group
  int cv;              // vectors per site
  int cols, rows;      // vectors and sites a block takes at a time
  int colblocks, kg, cparts, unit_vec;
  int slabs;           // site ranges per image, per column block
  int64_t slab_sites;
  int64_t units;       // n * slabs * colblocks
};

struct NormArgs {
  NormGeom g;
  const void* x;
  const void* dy;
  void* y;             // y or dx
  int64_t xn, xh, xw, yn, yh, yw, dn, dh, dw;
  const float* gamma;
  const float* beta;
  const float* mean;   // [n][groups]
  const float* rstd;
  float* mean_out;
  float* rstd_out;
  float eps;
  float* part;         // forward: [n][groups][parts] {count, mean, M2};
                       // backward: [n][slabs][c] {sum dz, sum dz xh}
  int parts;
  float* chsum;        // backward: [n][c] {sum dz, sum dz xh}
  float* gsum;         // backward: [n][groups] {s1, s2}
  float* dgamma;
  float* dbeta;
  int dblocks;         // blocks of the last pass that reduce dgamma, dbeta
};

// The block's place: image, site range, vectors and groups.
struct Place {
  int n, slab, cb, vec0, nvec, g0, ng;
  int64_t s0, s1;
};
__device__ __forceinline__ Place place_of(const NormGeom& g, int64_t u) {
  Place p;
  p.cb = (int)(u % g.colblocks);
  const int64_t r = u / g.colblocks;
  p.slab = (int)(r % g.slabs);
  p.n = (int)(r / g.slabs);
  p.s0 = p.slab * g.slab_sites;
  p.s1 = p.s0 + g.slab_sites < g.sites ? p.s0 + g.slab_sites : g.sites;
  if (g.cparts == 1) {
    p.vec0 = p.cb * g.cols;
    p.nvec = min(g.cols, g.cv - p.vec0);
    p.g0 = p.cb * g.kg;
    p.ng = min(g.kg, g.groups - p.g0);
  } else {
    p.g0 = p.cb / g.cparts;
    const int in = (p.cb % g.cparts) * g.cols;
    p.vec0 = p.g0 * g.unit_vec + in;
    p.nvec = min(g.cols, g.unit_vec - in);
    p.ng = 1;
  }
  return p;
}

__device__ __forceinline__ int64_t site_at(const NormGeom& g, int64_t s,
                                           int64_t sh, int64_t sw) {
  if (g.h1) return s * sw;
  const int64_t y = s / g.w;
  return y * sh + (s - y * g.w) * sw;
}

// (na, ma, qa) becomes count, mean and squared deviations of both sets.
template <typename F>
__device__ __forceinline__ void merge(F& na, F& ma, F& qa, F nb, F mb, F qb) {
  if (nb == 0) return;
  if (na == 0) {
    na = nb;
    ma = mb;
    qa = qb;
    return;
  }
  const F n = na + nb, d = mb - ma, w = nb / n;
  ma += d * w;
  qa += qb + d * d * na * w;
  na = n;
}

// Adds a batch of M values to (cnt, mean, m2): the batch's own mean first,
// then its squared deviations from that mean.  Values come relative to one
// value of their group: a mean far from zero costs no digits.
template <int M>
__device__ __forceinline__ void add_batch(const float* f, float& cnt,
                                          float& mean, float& m2) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < M; ++i) s += f[i];
  const float bm = s * (1.f / M);
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < M; ++i) {
    const float d = f[i] - bm;
    q = __builtin_fmaf(d, d, q);
  }
  const float n = cnt + (float)M, d = bm - mean;
  const float w = (float)M * __builtin_amdgcn_rcpf(n);
  m2 += q + d * d * cnt * w;
  mean = __builtin_fmaf(d, w, mean);
  cnt = n;
}

// Tree over a block's rows, then over a group's columns.  WHOLE: one entry
// per thread; otherwise V, one per channel.  Entries of group j end at slot
// j of out (count, mean, M2).
template <int V, bool WHOLE>
__device__ __forceinline__ void block_moments(const NormGeom& g,
                                              const Place& p, float* cnt,
                                              float* mean, float* m2,
                                              float* out) {
  constexpr int S = WHOLE ? 1 : V;
  __shared__ float sc[kThreads * S], sm[kThreads * S], sq[kThreads * S];
  const int tid = threadIdx.x, col = tid % g.cols, row = tid / g.cols;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < S; ++i) {
    sc[tid * S + i] = cnt[i];
    sm[tid * S + i] = mean[i];
    sq[tid * S + i] = m2[i];
  }
  __syncthreads();
  int half = 1;
  while (half * 2 < g.rows) half *= 2;
  for (; half >= 1; half >>= 1) {
    if (row < half && row + half < g.rows) {
      const int a = tid * S, b = (tid + half * g.cols) * S;
      for (int i = 0; i < S; ++i)
        merge(sc[a + i], sm[a + i], sq[a + i], sc[b + i], sm[b + i],
              sq[b + i]);
    }
    __syncthreads();
  }
  if constexpr (WHOLE) {
    const int gw = g.cparts == 1 ? g.unit_vec : p.nvec;  // a group's vectors
    const int in = col % gw;
    half = 1;
    while (half * 2 < gw) half *= 2;
    for (; half >= 1; half >>= 1) {
      if (row == 0 && in < half && in + half < gw && col + half < p.nvec)
        merge(sc[tid], sm[tid], sq[tid], sc[tid + half], sm[tid + half],
              sq[tid + half]);
      __syncthreads();
    }
    if (tid < p.ng) {
      out[tid * 3] = sc[tid * gw];
      out[tid * 3 + 1] = sm[tid * gw];
      out[tid * 3 + 2] = sq[tid * gw];
    }
  } else {
    // fewer than 32 channels to a group here
    for (int j = tid; j < p.ng; j += kThreads) {
      float n = 0.f, m = 0.f, q = 0.f;
      for (int i = j * g.cpg; i < (j + 1) * g.cpg; ++i)
        merge(n, m, q, sc[i], sm[i], sq[i]);
      out[j * 3] = n;
      out[j * 3 + 1] = m;
      out[j * 3 + 2] = q;
    }
  }
}

// The value of a group that its values are taken relative to: the first
// channel of the first site.
template <typename T>
__device__ __forceinline__ float base_of(const NormArgs& a, int n, int gr) {
  return to_f(((const T*)a.x)[n * a.xn + (int64_t)gr * a.g.cpg]);
}

// First pass: count, mean and squared deviations of every site range.
template <typename T, int V, bool WHOLE>
__global__ __launch_bounds__(kThreads) void k_norm_stats(NormArgs a) {
  constexpr int S = WHOLE ? 1 : V;
  const NormGeom& g = a.g;
  __shared__ float res[kThreads * 8 * 3];
  const int col = threadIdx.x % g.cols, row = threadIdx.x / g.cols;
  for (int64_t u = blockIdx.x; u < g.units; u += gridDim.x) {
    const Place p = place_of(g, u);
    float cnt[S], mean[S], m2[S], base[S];
#pragma unroll
    for (int i = 0; i < S; ++i) cnt[i] = mean[i] = m2[i] = 0.f;
    if (row < g.rows && col < p.nvec) {
      const int ch = (p.vec0 + col) * V;
#pragma unroll
      for (int i = 0; i < S; ++i) base[i] = base_of<T>(a, p.n, (ch + i) / g.cpg);
      const T* x = (const T*)a.x + p.n * a.xn + ch;
      int64_t s = p.s0 + row;
      for (; s + (kBatch - 1) * g.rows < p.s1; s += kBatch * g.rows) {
        Pack<T, V> r[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
          r[k] = load_pack<T, V>(
              x + site_at(g, s + k * g.rows, a.xh, a.xw));
        float f[kBatch][V];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          unpack<T, V>(r[k], f[k]);
#pragma unroll
          for (int i = 0; i < V; ++i) f[k][i] -= base[WHOLE ? 0 : i];
        }
        if constexpr (WHOLE) {
          add_batch<kBatch * V>(&f[0][0], cnt[0], mean[0], m2[0]);
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            float t[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) t[k] = f[k][i];
            add_batch<kBatch>(t, cnt[i], mean[i], m2[i]);
          }
        }
      }
      for (; s < p.s1; s += g.rows) {
        float f[V];
        unpack<T, V>(load_pack<T, V>(x + site_at(g, s, a.xh, a.xw)), f);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] -= base[WHOLE ? 0 : i];
        if constexpr (WHOLE) {
          add_batch<V>(f, cnt[0], mean[0], m2[0]);
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i)
            add_batch<1>(f + i, cnt[i], mean[i], m2[i]);
        }
      }
    }
    block_moments<V, WHOLE>(g, p, cnt, mean, m2, res);
    __syncthreads();
    const int part = p.slab * g.cparts + p.cb % g.cparts;
    for (int j = threadIdx.x; j < p.ng; j += kThreads) {
      float* o = a.part +
                 (((int64_t)p.n * g.groups + p.g0 + j) * a.parts + part) * 3;
      o[0] = res[j * 3];
      o[1] = res[j * 3 + 1];
      o[2] = res[j * 3 + 2];
    }
    __syncthreads();
  }
}

// Mean and rstd of one image and group from its parts, by one wave, in f64
// (every lane ends with them).
template <typename T>
__device__ __forceinline__ void join_parts(const NormArgs& a, int64_t ng,
                                           float& mean, float& rstd) {
  const float* part = a.part + ng * a.parts * 3;
  const int lane = threadIdx.x & 63;
  double n = 0, m = 0, q = 0;
  for (int i = lane; i < a.parts; i += 64)
    merge<double>(n, m, q, part[i * 3], part[i * 3 + 1], part[i * 3 + 2]);
  for (int d = 32; d; d >>= 1) {
    const double on = __shfl_down(n, d), om = __shfl_down(m, d),
                 oq = __shfl_down(q, d);
    if (lane + d < 64) merge(n, m, q, on, om, oq);
  }
  const double base =
      base_of<T>(a, (int)(ng / a.g.groups), (int)(ng % a.g.groups));
  mean = (float)(base + __shfl(m, 0));
  rstd = (float)__shfl(1.0 / sqrt(q / n + (double)a.eps), 0);
}

// One wave per image and group.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_norm_join(NormArgs a) {
  const int64_t total = (int64_t)a.g.n * a.g.groups;
  for (int64_t i = blockIdx.x * 4ll + threadIdx.x / 64; i < total;
       i += gridDim.x * 4ll) {
    float m, r;
    join_parts<T>(a, i, m, r);
    if ((threadIdx.x & 63) == 0) {
      a.mean_out[i] = m;
      a.rstd_out[i] = r;
    }
  }
}

// A thread's channels: mean and rstd * gamma, beta.
template <int V>
__device__ __forceinline__ void load_params(const NormArgs& a, int n, int ch,
                                            float* mean, float* rstd,
                                            float* gamma, float* beta) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int64_t at = (int64_t)n * a.g.groups + (ch + i) / a.g.cpg;
    mean[i] = a.mean[at];
    rstd[i] = a.rstd[at];
    gamma[i] = a.gamma ? a.gamma[ch + i] : 1.f;
    beta[i] = a.beta ? a.beta[ch + i] : 0.f;
  }
}

// Last pass: normalise, activate.
template <typename T, typename O, int V, int ACT>
__global__ __launch_bounds__(kThreads) void k_norm_apply(NormArgs a) {
  const NormGeom& g = a.g;
  const int col = threadIdx.x % g.cols, row = threadIdx.x / g.cols;
  for (int64_t u = blockIdx.x; u < g.units; u += gridDim.x) {
    const Place p = place_of(g, u);
    if (row >= g.rows || col >= p.nvec) continue;
    const int ch = (p.vec0 + col) * V;
    float mean[V], scale[V], gamma[V], beta[V];
    load_params<V>(a, p.n, ch, mean, scale, gamma, beta);
#pragma unroll
    for (int i = 0; i < V; ++i) scale[i] *= gamma[i];
    const T* x = (const T*)a.x + p.n * a.xn + ch;
    O* y = (O*)a.y + p.n * a.yn + ch;
    auto put = [&](int64_t s, const Pack<T, V>& r) {
      float f[V];
      unpack<T, V>(r, f);
#pragma unroll
      for (int i = 0; i < V; ++i)
        f[i] = act_fwd<ACT>(
            __builtin_fmaf(f[i] - mean[i], scale[i], beta[i]));
      store_pack<O, V>(y + site_at(g, s, a.yh, a.yw), f);
    };
    int64_t s = p.s0 + row;
    for (; s + (kBatch - 1) * g.rows < p.s1; s += kBatch * g.rows) {
      Pack<T, V> r[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        r[k] = load_pack<T, V>(x + site_at(g, s + k * g.rows, a.xh, a.xw));
#pragma unroll
      for (int k = 0; k < kBatch; ++k) put(s + k * g.rows, r[k]);
    }
    for (; s < p.s1; s += g.rows)
      put(s, load_pack<T, V>(x + site_at(g, s, a.xh, a.xw)));
  }
}

// ---------------------------------------------------------------- backward

// dz and xh of one vector.
template <int V, int ACT>
__device__ __forceinline__ void dz_of(const float* x, float* dy,
                                      const float* mean, const float* rstd,
                                      const float* gamma, const float* beta,
                                      float* xh) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    xh[i] = (x[i] - mean[i]) * rstd[i];
    if constexpr (ACT != ST_ACT_NONE)
      dy[i] *= act_grad<ACT>(__builtin_fmaf(xh[i], gamma[i], beta[i]));
  }
}

// First pass: sums of dz and dz xh per channel and site range.
template <typename T, typename O, int V, int ACT>
__global__ __launch_bounds__(kThreads) void k_norm_grad_sums(NormArgs a) {
  const NormGeom& g = a.g;
  __shared__ float red[kThreads * V * 2];
  const int col = threadIdx.x % g.cols, row = threadIdx.x / g.cols;
  for (int64_t u = blockIdx.x; u < g.units; u += gridDim.x) {
    const Place p = place_of(g, u);
    float s1[V], s2[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s1[i] = s2[i] = 0.f;
    const int ch = (p.vec0 + col) * V;
    if (row < g.rows && col < p.nvec) {
      float mean[V], rstd[V], gamma[V], beta[V];
      load_params<V>(a, p.n, ch, mean, rstd, gamma, beta);
      const T* x = (const T*)a.x + p.n * a.xn + ch;
      const O* dy = (const O*)a.dy + p.n * a.dn + ch;
      auto add = [&](const Pack<T, V>& rx, const Pack<O, V>& rd) {
        float f[V], d[V], xh[V];
        unpack<T, V>(rx, f);
        unpack<O, V>(rd, d);
        dz_of<V, ACT>(f, d, mean, rstd, gamma, beta, xh);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          s1[i] += d[i];
          s2[i] = __builtin_fmaf(d[i], xh[i], s2[i]);
        }
      };
      int64_t s = p.s0 + row;
      for (; s + (kBatch - 1) * g.rows < p.s1; s += kBatch * g.rows) {
        Pack<T, V> rx[kBatch];
        Pack<O, V> rd[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          rx[k] = load_pack<T, V>(x + site_at(g, s + k * g.rows, a.xh, a.xw));
          rd[k] = load_pack<O, V>(dy +
                                  site_at(g, s + k * g.rows, a.dh, a.dw));
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) add(rx[k], rd[k]);
      }
      for (; s < p.s1; s += g.rows)
        add(load_pack<T, V>(x + site_at(g, s, a.xh, a.xw)),
            load_pack<O, V>(dy + site_at(g, s, a.dh, a.dw)));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) {
      red[(threadIdx.x * V + i) * 2] = s1[i];
      red[(threadIdx.x * V + i) * 2 + 1] = s2[i];
    }
    __syncthreads();
    int half = 1;
    while (half * 2 < g.rows) half *= 2;
    for (; half >= 1; half >>= 1) {
      if (row < half && row + half < g.rows) {
        const int x0 = threadIdx.x * V * 2, x1 = x0 + half * g.cols * V * 2;
        for (int i = 0; i < 2 * V; ++i) red[x0 + i] += red[x1 + i];
      }
      __syncthreads();
    }
    float* o = a.part + ((int64_t)p.n * g.slabs + p.slab) * g.c * 2 +
               (int64_t)p.vec0 * V * 2;
    for (int i = threadIdx.x; i < p.nvec * V * 2; i += kThreads) o[i] = red[i];
  }
}

// One block per image and group: sums over the site ranges, per channel
// (kept for dgamma and dbeta) and, weighted, over the group.
__global__ __launch_bounds__(kThreads) void k_norm_grad_join(NormArgs a) {
  const NormGeom& g = a.g;
  __shared__ double r1[kThreads], r2[kThreads];
  const int64_t total = (int64_t)g.n * g.groups;
  for (int64_t u = blockIdx.x; u < total; u += gridDim.x) {
    const int n = (int)(u / g.groups), gr = (int)(u % g.groups);
    // threads of a channel take its site ranges in turn
    int per = 1;
    while (per * 2 * g.cpg <= kThreads && per < g.slabs) per *= 2;
    const int chs = kThreads / per;
    double t1 = 0, t2 = 0;
    for (int c0 = 0; c0 < g.cpg; c0 += chs) {
      const int c = c0 + threadIdx.x % chs, k = threadIdx.x / chs;
      double d1 = 0, d2 = 0;
      if (c < g.cpg) {
        const float* p =
            a.part + ((int64_t)n * g.slabs * g.c + gr * g.cpg + c) * 2;
        for (int s = k; s < g.slabs; s += per) {
          d1 += p[(int64_t)s * g.c * 2];
          d2 += p[(int64_t)s * g.c * 2 + 1];
        }
      }
      __syncthreads();
      r1[threadIdx.x] = d1;
      r2[threadIdx.x] = d2;
      __syncthreads();
      if (k == 0 && c < g.cpg) {
        for (int s = 1; s < per; ++s) {
          d1 += r1[s * chs + threadIdx.x];
          d2 += r2[s * chs + threadIdx.x];
        }
        float* o = a.chsum + ((int64_t)n * g.c + gr * g.cpg + c) * 2;
        o[0] = (float)d1;
        o[1] = (float)d2;
        const double gm = a.gamma ? a.gamma[gr * g.cpg + c] : 1.f;
        t1 += d1 * gm;
        t2 += d2 * gm;
      }
    }
    __syncthreads();
    r1[threadIdx.x] = t1;
    r2[threadIdx.x] = t2;
    __syncthreads();
    for (int d = kThreads / 2; d; d >>= 1) {
      if ((int)threadIdx.x < d) {
        r1[threadIdx.x] += r1[threadIdx.x + d];
        r2[threadIdx.x] += r2[threadIdx.x + d];
      }
      __syncthreads();
    }
    if (threadIdx.x == 0) {
      const double m = (double)g.sites * g.cpg;
      a.gsum[u * 2] = (float)(r1[0] / m);
      a.gsum[u * 2 + 1] = (float)(r2[0] / m);
    }
    __syncthreads();
  }
}

// Last pass: dx; the first `dblocks` blocks sum dgamma and dbeta over the
// images.
template <typename T, typename O, int V, int ACT>
__global__ __launch_bounds__(kThreads) void k_norm_grad_apply(NormArgs a) {
  const NormGeom& g = a.g;
  if ((int)blockIdx.x < a.dblocks) {
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= g.c) return;
    double d1 = 0, d2 = 0;
    for (int n = 0; n < g.n; ++n) {
      d1 += a.chsum[((int64_t)n * g.c + c) * 2];
      d2 += a.chsum[((int64_t)n * g.c + c) * 2 + 1];
    }
    if (a.dbeta) a.dbeta[c] = (float)d1;
    if (a.dgamma) a.dgamma[c] = (float)d2;
    return;
  }
  const int col = threadIdx.x % g.cols, row = threadIdx.x / g.cols;
  for (int64_t u = blockIdx.x - a.dblocks; u < g.units;
       u += gridDim.x - a.dblocks) {
    const Place p = place_of(g, u);
    if (row >= g.rows || col >= p.nvec) continue;
    const int ch = (p.vec0 + col) * V;
    float mean[V], rstd[V], gamma[V], beta[V], s1[V], s2[V];
    load_params<V>(a, p.n, ch, mean, rstd, gamma, beta);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t at = (int64_t)p.n * g.groups + (ch + i) / g.cpg;
      s1[i] = a.gsum[at * 2];
      s2[i] = a.gsum[at * 2 + 1];
    }
    const T* x = (const T*)a.x + p.n * a.xn + ch;
    const O* dy = (const O*)a.dy + p.n * a.dn + ch;
    T* dx = (T*)a.y + p.n * a.yn + ch;
    auto put = [&](int64_t s, const Pack<T, V>& rx, const Pack<O, V>& rd) {
      float f[V], d[V], xh[V];
      unpack<T, V>(rx, f);
      unpack<O, V>(rd, d);
      dz_of<V, ACT>(f, d, mean, rstd, gamma, beta, xh);
#pragma unroll
      for (int i = 0; i < V; ++i)
        f[i] = rstd[i] * (__builtin_fmaf(d[i], gamma[i], -s1[i]) -
                          xh[i] * s2[i]);
      store_pack<T, V>(dx + site_at(g, s, a.yh, a.yw), f);
    };
    int64_t s = p.s0 + row;
    for (; s + (kBatch - 1) * g.rows < p.s1; s += kBatch * g.rows) {
      Pack<T, V> rx[kBatch];
      Pack<O, V> rd[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        rx[k] = load_pack<T, V>(x + site_at(g, s + k * g.rows, a.xh, a.xw));
        rd[k] = load_pack<O, V>(dy + site_at(g, s + k * g.rows, a.dh, a.dw));
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) put(s + k * g.rows, rx[k], rd[k]);
    }
    for (; s < p.s1; s += g.rows)
      put(s, load_pack<T, V>(x + site_at(g, s, a.xh, a.xw)),
          load_pack<O, V>(dy + site_at(g, s, a.dh, a.dw)));
  }
}

// -------------------------------------------------------------- host side

constexpr int kTargetBlocks = 2048;   // eight of 256 threads to a CU
constexpr int kMaxSlabs = 1024;
constexpr int kMinBatches = 2;        // batches a thread has at least

// The cut for vectors of v channels; false where v does not suit the groups.
bool geom(const st_norm_desc& d, int v, NormGeom& g) {
  g = NormGeom{};
  g.sites = (int64_t)d.h * d.w;
  g.w = d.w;
  g.n = d.n;
  g.c = d.c;
  g.groups = d.groups;
  g.cpg = d.c / d.groups;
  g.v = v;
  if (d.c % v) return false;
  g.cv = d.c / v;
  g.whole = g.cpg % v == 0;
  // vectors that straddle groups: only where groups are narrow, so that a
  // group's channels are few to join
  if (!g.whole && g.cpg >= 32) return false;
  const int mul = v / std::gcd(g.cpg, v);   // groups that fill whole vectors
  g.unit_vec = g.cpg * mul / v;
  if (g.unit_vec <= kThreads) {
    const int units = g.groups / mul;
    const int fit = std::min(units, kThreads / g.unit_vec);
    g.colblocks = (int)ceil_div(units, fit);
    const int per = (int)ceil_div(units, g.colblocks);
    g.colblocks = (int)ceil_div(units, per);
    g.cols = per * g.unit_vec;
    g.kg = per * mul;
    g.cparts = 1;
  } else {
    g.cparts = (int)ceil_div(g.unit_vec, kThreads);
    g.cols = (int)ceil_div(g.unit_vec, g.cparts);
    g.cparts = (int)ceil_div(g.unit_vec, g.cols);
    g.colblocks = g.groups * g.cparts;
    g.kg = 1;
  }
  g.rows = kThreads / g.cols;
  const int64_t blocks = (int64_t)g.n * g.colblocks;
  const int64_t most =
      ceil_div(g.sites, (int64_t)g.rows * kBatch * kMinBatches);
  int64_t slabs = std::min<int64_t>(most, ceil_div(kTargetBlocks, blocks));
  slabs = std::max<int64_t>(1, std::min<int64_t>(slabs, kMaxSlabs));
  g.slab_sites = ceil_div(g.sites, slabs);
  g.slabs = (int)ceil_div(g.sites, g.slab_sites);
  g.units = blocks * g.slabs;
  return true;
}

struct NormSpace {
  size_t part = 0, chsum = 0, gsum = 0, stats = 0, bytes = 0;
};
NormSpace space_of(const NormGeom& g, bool backward) {
  NormSpace s;
  size_t top = 0;
  auto take = [&](int64_t floats) {
    const size_t at = top;
    top += (size_t)round_up(floats * 4, (int64_t)kAlign);
    return at;
  };
  const int64_t ng = (int64_t)g.n * g.groups;
  if (backward) {
    s.part = take((int64_t)g.n * g.slabs * g.c * 2);
    s.chsum = take((int64_t)g.n * g.c * 2);
    s.gsum = take(ng * 2);
  } else {
    s.part = take(ng * g.slabs * g.cparts * 3);
    s.stats = take(ng * 2);
  }
  s.bytes = top;
  return s;
}

st_status check_desc(const st_norm_desc* d) {
  if (!d) return bad("descriptor is NULL");
  if (!dtypes_known(d->dtype, d->out_dtype))
    return bad("unknown data types, or a pair that is not offered");
  if (d->n < 0 || d->h < 1 || d->w < 1 || d->c < 1)
    return bad("the map's sizes must be positive (n may be 0)");
  if (d->groups < 1 || d->c % d->groups)
    return bad("groups must divide the channels");
  if (!act_known(d->act)) return bad("unknown activation");
  if (!(d->eps >= 0.f) || d->eps > 3.4e38f)
    return bad("eps must be finite and not negative");
  return ST_OK;
}

// Elements between a map's first and one behind its last.
int64_t reach(const st_norm_desc& d, const st_map_ref& m) {
  return (d.n - 1) * m.stride_n + (d.h - 1) * m.stride_h +
         (d.w - 1) * m.stride_w + d.c;
}
st_status check_map(const st_norm_desc& d, const st_map_ref* m, bool out,
                    const char* name) {
  if (!m || !m->data) return bad(std::string(name) + " is NULL");
  if (m->stride_n < 0 || m->stride_h < 0 || m->stride_w < 0)
    return bad(std::string(name) + " has a negative stride");
  if (!out) return ST_OK;
  // every axis, narrowest stride first, steps over what lies inside it
  int64_t len[3] = {d.n, d.h, d.w};
  int64_t st[3] = {m->stride_n, m->stride_h, m->stride_w};
  int64_t inner = d.c;
  for (int k = 0; k < 3; ++k) {
    int at = -1;
    for (int i = 0; i < 3; ++i)
      if (len[i] > 1 && (at < 0 || st[i] < st[at])) at = i;
    if (at < 0) break;
    if (st[at] < inner)
      return bad(std::string(name) + ": an output's elements overlap");
    inner = st[at] * (len[at] - 1) + inner;
    len[at] = 1;
  }
  return ST_OK;
}
Span map_span(const st_norm_desc& d, const st_map_ref& m, int es) {
  return span_of(m.data, reach(d, m) * es);
}
bool same_map(const st_norm_desc& d, const st_map_ref& a,
              const st_map_ref& b) {
  return a.data == b.data && (d.n < 2 || a.stride_n == b.stride_n) &&
         (d.h < 2 || a.stride_h == b.stride_h) &&
         (d.w < 2 || a.stride_w == b.stride_w);
}

// The widest vector (16 bytes of the widest type at most) that the maps'
// addresses and strides and the groups allow.
struct MapUse {
  const st_map_ref* m;
  int es;
};
NormGeom pick(const st_norm_desc& d, std::initializer_list<MapUse> maps) {
  NormGeom g;
  int v = 16 / std::max(esize(d.dtype), esize(d.out_dtype));
  for (; v > 1; v /= 2) {
    bool ok = true;
    for (const MapUse& u : maps)
      ok = ok && vec_ok(v, u.es, u.m->data, d.n > 1 ? u.m->stride_n : 0,
                        d.h > 1 ? u.m->stride_h : 0,
                        d.w > 1 ? u.m->stride_w : 0);
    if (ok && geom(d, v, g)) break;
  }
  if (v == 1) (void)geom(d, 1, g);
  g.h1 = 1;
  for (const MapUse& u : maps)
    if (d.h > 1 && d.w > 1 && u.m->stride_h != u.m->stride_w * d.w) g.h1 = 0;
  return g;
}
// A map of one column steps by rows.
int64_t step_w(const st_norm_desc& d, const st_map_ref& m) {
  return d.w == 1 ? m.stride_h : m.stride_w;
}

template <class F>
void with_vec(int v, F&& f) {
  if (v == 8)
    f(Int<8>{});
  else if (v == 4)
    f(Int<4>{});
  else if (v == 2)
    f(Int<2>{});
  else
    f(Int<1>{});
}
unsigned grid_of(int64_t units) {
  return (unsigned)std::min<int64_t>(units, 1 << 20);
}

st_status workspace_of(const st_norm_desc* d, int32_t backward,
                       uint64_t* bytes) {
  if (const st_status s = check_desc(d); s != ST_OK) return s;
  if (!bytes) return bad("bytes is NULL");
  // the cut follows the vector, which a call picks by its addresses
  *bytes = 0;
  for (int v = 8; v >= 1 && d->n > 0; v /= 2) {
    NormGeom g;
    if (geom(*d, v, g))
      *bytes = std::max<uint64_t>(*bytes, space_of(g, backward != 0).bytes);
  }
  return ST_OK;
}

st_status check_space(const st_norm_desc& d, bool backward, const void* ws,
                      uint64_t ws_bytes) {
  uint64_t need = 0;
  if (const st_status s = workspace_of(&d, backward, &need); s != ST_OK)
    return s;
  if (need && !ws) return bad("workspace is NULL");
  if ((uintptr_t)ws % kAlign) return bad("workspace must be 256-byte aligned");
  if (ws_bytes < need)
    return fail(nullptr, ST_ERR_WORKSPACE, "workspace too small");
  return ST_OK;
}

}  // namespace
}  // namespace ops
}  // namespace st

using namespace st;
using namespace st::ops;

extern "C" st_status st_group_norm_workspace(const st_norm_desc* d,
                                             int32_t backward,
                                             uint64_t* bytes) {
  return guarded([&] { return workspace_of(d, backward, bytes); });
}

extern "C" st_status st_group_norm(const st_norm_desc* d, const st_map_ref* x,
                                   const float* gamma, const float* beta,
                                   const st_map_ref* y, float* mean,
                                   float* rstd, void* ws, uint64_t ws_bytes,
                                   void* stream) {
  return guarded([&]() -> st_status {
    if (const st_status s = check_desc(d); s != ST_OK) return s;
    if (d->n == 0) return ST_OK;
    if (const st_status s = check_map(*d, x, false, "x"); s != ST_OK) return s;
    if (const st_status s = check_map(*d, y, true, "y"); s != ST_OK) return s;
    if (!mean != !rstd) return bad("mean and rstd: both or neither");
    if (const st_status s = check_space(*d, false, ws, ws_bytes); s != ST_OK)
      return s;
    const int es = esize(d->dtype), eo = esize(d->out_dtype);
    const int64_t ng = (int64_t)d->n * d->groups * 4;
    const Span sy = map_span(*d, *y, eo), sm = span_of(mean, ng),
               sr = span_of(rstd, ng), sw = span_of(ws, (int64_t)ws_bytes),
               sx = map_span(*d, *x, es), sg = span_of(gamma, d->c * 4ll),
               sb = span_of(beta, d->c * 4ll);
    const bool in_place = d->dtype == d->out_dtype && same_map(*d, *x, *y);
    if ((sy.hits(sx) && !in_place) || sy.hits(sg) || sy.hits(sb) ||
        sy.hits(sm) || sy.hits(sr) || sy.hits(sw) || sm.hits(sr) ||
        sm.hits(sx) || sr.hits(sx) || sm.hits(sg) || sm.hits(sb) ||
        sr.hits(sg) || sr.hits(sb) || sw.hits(sx) || sw.hits(sm) ||
        sw.hits(sr) || sw.hits(sg) || sw.hits(sb))
      return bad("an output overlaps an input, another output or the "
                 "workspace");
    (void)hipGetLastError();
    NormArgs a{};
    a.g = pick(*d, {{x, es}, {y, eo}});
    const NormSpace sp = space_of(a.g, false);
    char* w = (char*)ws;
    a.x = x->data;
    a.y = y->data;
    a.xn = x->stride_n; a.xh = x->stride_h; a.xw = step_w(*d, *x);
    a.yn = y->stride_n; a.yh = y->stride_h; a.yw = step_w(*d, *y);
    a.gamma = gamma;
    a.beta = beta;
    a.eps = d->eps;
    a.part = (float*)(w + sp.part);
    a.parts = a.g.slabs * a.g.cparts;
    a.mean_out = mean ? mean : (float*)(w + sp.stats);
    a.rstd_out = rstd ? rstd : a.mean_out + (int64_t)d->n * d->groups;
    a.mean = a.mean_out;
    a.rstd = a.rstd_out;
    hipStream_t q = (hipStream_t)stream;
    with_types(d->dtype, d->out_dtype, [&](auto in, auto out) {
      using T = typename decltype(in)::type;
      using O = typename decltype(out)::type;
      with_vec(a.g.v, [&](auto vt) {
        constexpr int V = decltype(vt)::value;
        if constexpr (V * sizeof(T) <= 16 && V * sizeof(O) <= 16) {
          if constexpr (V == 1)
            k_norm_stats<T, 1, true>
                <<<grid_of(a.g.units), kThreads, 0, q>>>(a);
          else if (a.g.whole)
            k_norm_stats<T, V, true>
                <<<grid_of(a.g.units), kThreads, 0, q>>>(a);
          else
            k_norm_stats<T, V, false>
                <<<grid_of(a.g.units), kThreads, 0, q>>>(a);
          k_norm_join<T><<<grid_of(ceil_div((int64_t)d->n * d->groups, 4)),
                           kThreads, 0, q>>>(a);
          with_activation(d->act, [&](auto act) {
            k_norm_apply<T, O, V, decltype(act)::value>
                <<<grid_of(a.g.units), kThreads, 0, q>>>(a);
          });
        }
      });
    });
    return launch_status("group norm");
  });
}

extern "C" st_status st_group_norm_backward(
    const st_norm_desc* d, const st_map_ref* dy, const st_map_ref* x,
    const float* mean, const float* rstd, const float* gamma,
    const float* beta, const st_map_ref* dx, float* dgamma, float* dbeta,
    void* ws, uint64_t ws_bytes, void* stream) {
  return guarded([&]() -> st_status {
    if (const st_status s = check_desc(d); s != ST_OK) return s;
    hipStream_t q = (hipStream_t)stream;
    NormArgs a{};
    a.dgamma = dgamma;
    a.dbeta = dbeta;
    a.g.c = d->c;
    const int dblocks =
        dgamma || dbeta ? (int)ceil_div(d->c, kThreads) : 0;
    if (d->n == 0) {
      // no image: the parameters' gradients are zero
      if (dblocks) {
        (void)hipGetLastError();
        a.dblocks = dblocks;
        k_norm_grad_apply<float, float, 1, ST_ACT_NONE>
            <<<dblocks, kThreads, 0, q>>>(a);
        return launch_status("group norm backward");
      }
      return ST_OK;
    }
    if (const st_status s = check_map(*d, dy, false, "dy"); s != ST_OK)
      return s;
    if (const st_status s = check_map(*d, x, false, "x"); s != ST_OK) return s;
    if (const st_status s = check_map(*d, dx, true, "dx"); s != ST_OK)
      return s;
    if (!mean || !rstd) return bad("mean or rstd is NULL");
    if (const st_status s = check_space(*d, true, ws, ws_bytes); s != ST_OK)
      return s;
    const int es = esize(d->dtype), eo = esize(d->out_dtype);
    const int64_t ng = (int64_t)d->n * d->groups * 4, cb = d->c * 4ll;
    const Span in[] = {map_span(*d, *dy, eo), map_span(*d, *x, es),
                       span_of(mean, ng),     span_of(rstd, ng),
                       span_of(gamma, cb),    span_of(beta, cb)};
    const Span out[] = {map_span(*d, *dx, es), span_of(dgamma, cb),
                        span_of(dbeta, cb), span_of(ws, (int64_t)ws_bytes)};
    const bool on_dy = d->dtype == d->out_dtype && same_map(*d, *dx, *dy);
    const bool on_x = same_map(*d, *dx, *x);
    bool hit = false;
    for (int o = 0; o < 4; ++o) {
      for (int i = 0; i < 6; ++i)
        if (out[o].hits(in[i]) &&
            !(o == 0 && ((i == 0 && on_dy) || (i == 1 && on_x))))
          hit = true;
      for (int j = 0; j < o; ++j) hit = hit || out[o].hits(out[j]);
    }
    if (hit)
      return bad("an output overlaps an input, another output or the "
                 "workspace");
    (void)hipGetLastError();
    a.g = pick(*d, {{x, es}, {dy, eo}, {dx, es}});
    const NormSpace sp = space_of(a.g, true);
    char* w = (char*)ws;
    a.x = x->data;
    a.dy = dy->data;
    a.y = dx->data;
    a.xn = x->stride_n; a.xh = x->stride_h; a.xw = step_w(*d, *x);
    a.dn = dy->stride_n; a.dh = dy->stride_h; a.dw = step_w(*d, *dy);
    a.yn = dx->stride_n; a.yh = dx->stride_h; a.yw = step_w(*d, *dx);
    a.gamma = gamma;
    a.beta = beta;
    a.mean = mean;
    a.rstd = rstd;
    a.eps = d->eps;
    a.part = (float*)(w + sp.part);
    a.chsum = (float*)(w + sp.chsum);
    a.gsum = (float*)(w + sp.gsum);
    a.dblocks = dblocks;
    with_types(d->dtype, d->out_dtype, [&](auto ti, auto to) {
      using T = typename decltype(ti)::type;
      using O = typename decltype(to)::type;
      with_vec(a.g.v, [&](auto vt) {
        constexpr int V = decltype(vt)::value;
        if constexpr (V * sizeof(T) <= 16 && V * sizeof(O) <= 16) {
          with_activation(d->act, [&](auto act) {
            constexpr int A = decltype(act)::value;
            k_norm_grad_sums<T, O, V, A>
                <<<grid_of(a.g.units), kThreads, 0, q>>>(a);
            k_norm_grad_join<<<grid_of((int64_t)d->n * d->groups), kThreads,
                               0, q>>>(a);
            k_norm_grad_apply<T, O, V, A>
                <<<grid_of(a.g.units) + dblocks, kThreads, 0, q>>>(a);
          });
        }
      });
    });
    return launch_status("group norm backward");
  });
}
