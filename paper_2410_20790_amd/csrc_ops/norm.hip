// Group norm with an activation on channels-last maps, forward, and the host
// side of both directions.
//
//   mean, var over an image's sites and the c / groups channels of a group
//   y = act((x - mean) rstd gamma + beta)
//
// About ten operations per element moved: bound by memory.
#include <algorithm>

#include "norm.h"

namespace st {
namespace ops {
namespace {

// sites whose loads a thread has in flight
constexpr int kBatch = 4, kSumBatch = 8;

// Adds a batch of M values to (cnt, mean, m2): the batch's own mean first,
// then its squared deviations from that mean.  Values come relative to the
// thread's first: a mean far from zero costs no digits, and a value far from
// the others costs those of its own thread alone.
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

// The moments of a vector of values, or (not WHOLE) of each of its channels.
template <int V, bool WHOLE>
struct Moments {
  static constexpr int S = WHOLE ? 1 : V;
  float base[S], cnt[S], mean[S], m2[S];
  __device__ __forceinline__ Moments() {
#pragma unroll
    for (int i = 0; i < S; ++i) base[i] = cnt[i] = mean[i] = m2[i] = 0.f;
  }
  // The base: what the thread has first.
  template <typename T>
  __device__ __forceinline__ void begin(const Pack<T, V>& first) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const float x = to_f(first.e[i]);
      if (cnt[i] == 0.f && __builtin_fabsf(x) < __builtin_inff()) base[i] = x;
    }
  }
  template <typename T, int N>
  __device__ __forceinline__ void add(const Pack<T, V>* r) {
    float f[N][V];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      unpack<T, V>(r[k], f[k]);
#pragma unroll
      for (int i = 0; i < V; ++i) f[k][i] -= base[WHOLE ? 0 : i];
    }
    if constexpr (WHOLE) {
      add_batch<N * V>(&f[0][0], cnt[0], mean[0], m2[0]);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float t[N];
#pragma unroll
        for (int k = 0; k < N; ++k) t[k] = f[k][i];
        add_batch<N>(t, cnt[i], mean[i], m2[i]);
      }
    }
  }
};

// The mean and the squared deviations of values whose distances from `near`, a
// value not far from their mean, add up to `rest` over the lanes, and the
// squares of these (beside deviations of their own) to `q`.
struct Joined {
  float mean, left, m2;    // left: what the mean's rounding left
  __device__ __forceinline__ Joined(float near, float rest, float q, float inv,
                                    int lanes) {
    lanes_sum2(rest, q, lanes);
    const float d = rest * inv;
    const bool finite = __builtin_fabsf(near) < __builtin_inff();
    mean = finite ? near + d : near;
    left = finite ? d - (mean - near) : 0.f;
    q -= rest * d;
    m2 = q < 0.f ? 0.f : q;    // NaN stays
  }
};

// Joins the block's moments: group j of the block ends at out[4 j] (count, mean
// in two parts, squared deviations), for all its threads, over the lanes that
// share a group.  The mean of the threads' means comes first, as the roundings
// leave it; relative to it, what they left out, and the deviations.
template <int V, bool WHOLE, int TH>
__device__ __forceinline__ void block_moments(const NormGeom& g,
                                              const Place& p,
                                              const Moments<V, WHOLE>& m,
                                              float* out) {
  constexpr int S = WHOLE ? 1 : V;
  __shared__ float sc[TH * S], sb[TH * S], sm[TH * S], sq[TH * S];
  const int tid = threadIdx.x;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < S; ++i) {
    sc[tid * S + i] = m.cnt[i];
    sb[tid * S + i] = m.base[i];
    sm[tid * S + i] = m.mean[i];
    sq[tid * S + i] = m.m2[i];
  }
  __syncthreads();
  const int wide = !WHOLE ? g.cpg : g.cparts == 1 ? g.unit_vec : p.nvec;
  const int lanes = lanes_per_group(TH, p.ng), in = tid & (lanes - 1);
  const Entries first(in, lanes, wide);
  const float n = (float)(p.s1 - p.s0) *
                  (float)(g.cparts == 1 ? g.cpg : p.nvec * V);
  const float inv = 1.f / n;
  for (int j = tid / lanes; j < p.ng; j += TH / lanes) {
    float s = 0.f, rest = 0.f, q = 0.f;
    for (Entries e = first; e.row < g.rows; e.next()) {
      const int at = e.row * g.cols * S + j * wide + e.c;
      s += sc[at] * inv * (sb[at] + sm[at]);   // (no sum beyond its values)
    }
    const float near = lanes_sum(s, lanes);
    for (Entries e = first; e.row < g.rows; e.next()) {
      const int at = e.row * g.cols * S + j * wide + e.c;
      const float c = sc[at], d = sb[at] - near + sm[at];
      rest += c * d;    // (no values: all are zero)
      q += sq[at] + c * d * d;
    }
    const Joined r(near, rest, q, inv, lanes);
    if (in == 0) {
      out[j * 4] = n;
      out[j * 4 + 1] = r.mean;
      out[j * 4 + 2] = r.left;
      out[j * 4 + 3] = r.m2;
    }
  }
  __syncthreads();
}

// Large images, first: the moments of a range of sites.
template <typename T, int V, bool WHOLE>
__device__ __forceinline__ void stats_unit(const NormArgs& a, const Place& p,
                                           float* res) {
  const NormGeom& g = a.g;
  const int col = threadIdx.x % g.cols, row = threadIdx.x / g.cols;
  Moments<V, WHOLE> m;
  if (row < g.rows && col < p.nvec) {
    const int ch = (p.vec0 + col) * V;
    int64_t s = p.s0 + row;
    SiteWalk<const T> x(a.x, p.n, s, ch);
    Pack<T, V> r[kSumBatch];
    for (; s + (kSumBatch - 1) * g.rows < p.s1; s += kSumBatch * g.rows) {
#pragma unroll
      for (int k = 0; k < kSumBatch; ++k) {
        r[k] = load_pack<T, V>(x.p);
        x.next();
      }
      m.begin(r[0]);
      m.template add<T, kSumBatch>(r);
    }
    for (; s < p.s1; s += g.rows) {
      r[0] = load_pack<T, V>(x.p);
      x.next();
      m.begin(r[0]);
      m.template add<T, 1>(r);
    }
  }
  block_moments<V, WHOLE, kThreads>(g, p, m, res);
  const int part = p.slab * g.cparts + p.cb % g.cparts;
  for (int j = threadIdx.x; j < p.ng; j += kThreads) {
    ((float4*)a.part)[((int64_t)p.n * g.groups + p.g0 + j) * a.parts + part] =
        make_float4(res[j * 4], res[j * 4 + 1], res[j * 4 + 2],
                    res[j * 4 + 3]);
  }
}

// Mean and rstd of the block's groups from their parts: group j at res[2 j],
// for all threads.
__device__ __forceinline__ void join_parts(const NormArgs& a, const Place& p,
                                           float* res) {
  const NormGeom& g = a.g;
  const int lanes = lanes_per_group(kThreads, p.ng);
  const int in = threadIdx.x & (lanes - 1);
  const float n = (float)((double)g.sites * g.cpg), inv = 1.f / n;
  for (int j = threadIdx.x / lanes; j < p.ng; j += kThreads / lanes) {
    const int64_t at = (int64_t)p.n * g.groups + p.g0 + j;
    const float4* part = (const float4*)a.part + at * a.parts;
    // A part of n of the group's M values whose mean a value D carries off is D
    // / n away, the group's deviation D / sqrt(M) or more: near enough, with
    // hundreds of values in a part and about as many parts.
    const float near = part[0].y;
    float rest = 0.f, q = 0.f;
#pragma unroll 4
    for (int i = in; i < a.parts; i += lanes) {
      const float4 o = part[i];
      const float d = o.y - near + o.z;
      rest += o.x * d;
      q += o.w + o.x * d * d;
    }
    const Joined r(near, rest, q, inv, lanes);
    const float rstd = 1.f / sqrtf(r.m2 / n + a.eps);
    if (in == 0) {
      res[j * 2] = r.mean;
      res[j * 2 + 1] = rstd;
      if (a.mean_out && p.slab == 0 && p.cb % g.cparts == 0) {
        a.mean_out[at] = r.mean;
        a.rstd_out[at] = rstd;
      }
    }
  }
  __syncthreads();
}

// Normalised, scaled, activated.
template <typename T, typename O, int V, bool WHOLE, int ACT, bool STREAM>
__device__ __forceinline__ void put_norm(O* y, const Pack<T, V>& r,
                                         const Params<V, WHOLE>& q,
                                         const float* scale) {
  float f[V];
  unpack<T, V>(r, f);
#pragma unroll
  for (int i = 0; i < V; ++i)
    f[i] = act_fwd<ACT>(
        __builtin_fmaf(f[i] - q.mu(i), scale[i], q.beta[i]));
  if constexpr (STREAM)
    stream_out<O, V>(y, f);
  else
    store_pack<O, V>(y, f);
}

// Large images, then: normalise a range of sites.
template <typename T, typename O, int V, bool WHOLE, int ACT>
__device__ __forceinline__ void apply_unit(const NormArgs& a, const Place& p,
                                           float* res) {
  const NormGeom& g = a.g;
  const int col = threadIdx.x % g.cols, row = threadIdx.x / g.cols;
  join_parts(a, p, res);
  if (row >= g.rows || col >= p.nvec) return;
  const int ch = (p.vec0 + col) * V;
  Params<V, WHOLE> q;
  q.load_affine(a, ch);
  q.load_stats(res, 2, ch, g.cpg, p.g0);
  float scale[V];
#pragma unroll
  for (int i = 0; i < V; ++i) scale[i] = q.r(i) * q.gamma[i];
  int64_t s = p.s0 + row;
  SiteWalk<const T> x(a.x, p.n, s, ch);
  SiteWalk<O> y(a.y, p.n, s, ch);
  Pack<T, V> r[kBatch];
  for (; s + (kBatch - 1) * g.rows < p.s1; s += kBatch * g.rows) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      r[k] = stream_pack<T, V>(x.p);
      x.next();
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      put_norm<T, O, V, WHOLE, ACT, true>(y.p, r[k], q, scale);
      y.next();
    }
  }
  for (; s < p.s1; s += g.rows) {
    put_norm<T, O, V, WHOLE, ACT, true>(y.p, load_pack<T, V>(x.p), q, scale);
    x.next();
    y.next();
  }
}

// A launch over large images: blocks finish the images [end0, end1) and sum up
// [sum0, sum1), in turn, so that reads and writes mix.
template <typename T, typename O, int V, bool WHOLE, int ACT>
__global__ __launch_bounds__(kThreads) void k_norm_pass(NormArgs a) {
  __shared__ float res[kMaxCols * (WHOLE ? 1 : V) * 4];
  const int ends = (a.end1 - a.end0) * a.g.units;
  const int all = ends + (a.sum1 - a.sum0) * a.g.units;
  for (int b = blockIdx.x; b < all; b += gridDim.x) {
    const Turn t(a, b, ends, all);
    const Place p = place_of(a.g, t.n, t.u);
    if (t.end)
      apply_unit<T, O, V, WHOLE, ACT>(a, p, res);
    else
      stats_unit<T, V, WHOLE>(a, p, res);
    __syncthreads();
  }
}

// Images whose groups fit a block's registers: one launch, x read once.  A
// thread holds up to kHeld sites of its vector.
template <typename T, typename O, int V, bool WHOLE, int TH>
__global__ __launch_bounds__(TH) void k_norm_held(NormArgs a) {
  constexpr int S = WHOLE ? 1 : V;
  const NormGeom& g = a.g;
  __shared__ float res[kMaxCols * S * 4];
  const int col = threadIdx.x % g.cols, row = threadIdx.x / g.cols;
  const int u = near_block((a.end1 - a.end0) * g.units);
  const Place p = place_of(g, a.end0 + u / g.units, u % g.units);
  const bool on = row < g.rows && col < p.nvec;
  const int ch = (p.vec0 + (on ? col : 0)) * V;
  const int left = on ? (int)g.sites - row : 0;   // sites from its own on
  Pack<T, V> r[kHeld];
  SiteWalk<const T> x(a.x, p.n, row, ch);
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    if (k * g.rows < left) r[k] = load_pack<T, V>(x.p);
    x.next();
  }
  Moments<V, WHOLE> m;
  Params<V, WHOLE> q;
  q.load_affine(a, ch);
  if (left > 0) m.begin(r[0]);
#pragma unroll
  for (int k = 0; k < kHeld; ++k)
    if (k * g.rows < left) m.template add<T, 1>(r + k);
  block_moments<V, WHOLE, TH>(g, p, m, res);
  for (int j = threadIdx.x; j < p.ng; j += TH) {
    const float rstd = 1.f / sqrtf(res[j * 4 + 3] / res[j * 4] + a.eps);
    res[j * 4 + 2] = rstd;
    if (a.mean_out) {
      const int64_t at = (int64_t)p.n * g.groups + p.g0 + j;
      a.mean_out[at] = res[j * 4 + 1];
      a.rstd_out[at] = rstd;
    }
  }
  __syncthreads();
  float scale[V];
  q.load_stats(res + 1, 4, ch, g.cpg, p.g0);
#pragma unroll
  for (int i = 0; i < V; ++i) scale[i] = q.r(i) * q.gamma[i];
  SiteWalk<O> y(a.y, p.n, row, ch);
  with_activation_of(a.act, [&](auto act) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      if (k * g.rows < left)
        put_norm<T, O, V, WHOLE, decltype(act)::value, false>(y.p, r[k], q,
                                                              scale);
      y.next();
    }
  });
}

// -------------------------------------------------------------- host side

// Rules of the cut, each with what it measured (us, in a replayed graph).  They
// follow an image's own sizes, not the number of images: an image's sums are
// joined in the same order, to the same bits, alone and among others.
// Held blocks take more groups while a site has less than a cache line of them:
// 8x8x320 f32 6.2 for one image and 6.6 for 32 (half a us more with two lines);
// 64x64x256 f16 14 and 57 (12.4 and 90 without).
constexpr int kHeldLine = 128;
// Blocks of 256 threads that an image is cut into, four to a CU, while their
// threads have enough to sum up before they join: as many sites, and as many
// bytes (backward: of x), of vectors that groups or strides keep narrow.
// 16-byte vectors: 9x32x64x2048 bf16 54 (59 with 8 sites), one such image 16
// (14).  One channel to a vector, 61x67x513 f16: four images 28 and one 17 (32
// and 15 with half the bytes, 34 and 23 with twice as many); backward 41 and 23
// (46 and 21 with half the bytes); one channel of 67, backward: nine images of
// 200x300 bf16 133 (167 with half, 125 with twice as many), one 29 (29 and 36).
constexpr int kTargetBlocks = 1024;
constexpr int kMinSites = 16, kMinBytes = 128, kMinGradBytes = 64;
constexpr int kMaxEntries = 4096;     // parts of all groups a block joins
// Bytes of a site to a block, two cache lines: 9x256x512x256 bf16 357 (368
// with four lines, 353 with one, which loses where they are streamed out).
constexpr int kLine = 256;
// Bytes of the images of a batch, read by one launch and again by the next,
// which also writes as many, while the last-level cache holds 256 MiB:
// 9x256x512x256 bf16 329 in six launches (357 in batches of 48 MiB, ten
// launches; 339 in one batch).
constexpr int64_t kBatchBytes = 144 << 20;

// The cut for vectors of v channels; false where v does not suit the groups.
bool geom(const st_norm_desc& d, int v, NormGeom& g) {
  g = NormGeom{};
  g.sites = (int64_t)d.h * d.w;
  g.n = d.n;
  g.c = d.c;
  g.groups = d.groups;
  g.cpg = d.c / d.groups;
  g.v = v;
  if (d.c % v) return false;
  g.cv = d.c / v;
  g.whole = g.cpg % v == 0;
  // vectors that straddle groups: only where groups are narrow, so that a
  // group's channels are few to join, and the vectors' own sums too
  if (!g.whole && (g.cpg >= 32 || v > 4)) return false;
  return true;
}

// Columns for blocks of `threads`, `units` units of the fewest groups that
// fill whole vectors in each.
void columns(NormGeom& g, int threads, int units) {
  const int mul = g.v / std::gcd(g.cpg, g.v);
  g.unit_vec = g.cpg * mul / g.v;
  if (g.unit_vec <= kMaxCols) {
    const int all = g.groups / mul;
    g.colblocks = (int)ceil_div(all, units);
    const int per = (int)ceil_div(all, g.colblocks);
    g.colblocks = (int)ceil_div(all, per);
    g.cols = per * g.unit_vec;
    g.kg = per * mul;
    g.cparts = 1;
  } else {
    g.cparts = (int)ceil_div(g.unit_vec, kMaxCols);
    g.cols = (int)ceil_div(g.unit_vec, g.cparts);
    g.cparts = (int)ceil_div(g.unit_vec, g.cols);
    g.colblocks = g.groups * g.cparts;
    g.kg = 1;
  }
  g.rows = threads / g.cols;
}

// Blocks that hold an image's groups whole, `held` sites a thread at most.
bool hold(NormGeom& g, int es, int threads, int held) {
  const int mul = g.v / std::gcd(g.cpg, g.v);
  const int unit = g.cpg * mul / g.v;
  if (unit > kMaxCols) return false;
  columns(g, threads, 1);
  if (ceil_div(g.sites, g.rows) > held || g.colblocks > kMaxGrid)
    return false;
  NormGeom w = g;
  for (int u = 2; g.cols * g.v * es < kHeldLine && g.colblocks > 1; u *= 2) {
    columns(w, threads, u);
    if (ceil_div(w.sites, w.rows) > held) break;
    g = w;
  }
  g.slabs = 1;
  g.slab_sites = g.sites;
  g.units = g.colblocks;
  return true;
}

// Images of a batch, `es` bytes of each element read by both passes.
int batch_of(const NormGeom& g, int es) {
  return (int)std::max<int64_t>(
      1, std::min<int64_t>(g.n, kBatchBytes / (g.sites * g.c * es)));
}

// Blocks that take a range of an image's sites: columns of at least kLine
// bytes, and no more ranges than a block of the next pass can join.
void split(NormGeom& g, int es, bool backward) {
  const int mul = g.v / std::gcd(g.cpg, g.v);
  const int unit = g.cpg * mul / g.v;
  const int units =
      std::min<int>(kMaxCols / unit,
                    (int)ceil_div(kLine, (int64_t)unit * g.v * es));
  columns(g, kThreads, std::max(1, units));
  // Backward, a second row of columns rather than threads without any:
  // 4x61x67x513 f16, 133 columns or 114, 41 us (53); forward 28 (26).
  constexpr int kHalf = kThreads / 2;
  if (backward && g.cols > kHalf && g.cols * 4 < kThreads * 3 && unit <= kHalf)
    columns(g, kThreads, kHalf / unit);
  const int least =
      std::max(kMinSites, (backward ? kMinGradBytes : kMinBytes) / (g.v * es));
  const int64_t most = ceil_div(g.sites, (int64_t)g.rows * least);
  int64_t slabs =
      std::min<int64_t>(most, ceil_div(kTargetBlocks, g.colblocks));
  slabs = std::min<int64_t>(slabs, kMaxEntries / (g.kg * g.cparts));
  slabs = std::max<int64_t>(1, slabs);
  g.slab_sites = ceil_div(g.sites, slabs);
  g.slabs = (int)ceil_div(g.sites, g.slab_sites);
  g.units = g.slabs * g.colblocks;
}

int read_size(const st_norm_desc& d, bool backward) {
  return esize(d.dtype) + (backward ? esize(d.out_dtype) : 0);
}

struct NormSpace {
  size_t part = 0, chpart = 0, bytes = 0;
};
NormSpace space_of(const NormGeom& g, bool backward, int held) {
  NormSpace s;
  size_t top = 0;
  auto take = [&](int64_t floats) {
    const size_t at = top;
    top += (size_t)round_up(floats * 4, (int64_t)kAlign);
    return at;
  };
  if (!held)
    s.part = take((int64_t)g.n * g.groups * g.slabs * g.cparts *
                  (backward ? 2 : 4));
  if (backward) s.chpart = take((int64_t)g.n * g.slabs * g.c * 2);
  s.bytes = top;
  return s;
}

st_status check_desc(const st_norm_desc* d) {
  if (!d) return bad("descriptor is NULL");
  if (!dtypes_known(d->dtype, d->out_dtype))
    return bad("unknown data types, or a pair that is not offered");
  if (d->n < 0 || d->h < 1 || d->w < 1 || d->c < 1)
    return bad("the map's sizes must be positive (n may be 0)");
  if ((int64_t)d->n * d->c >= (int64_t)1 << 31)
    return bad("n * c must lie below 2^31");
  if ((int64_t)d->h * d->w >= ((int64_t)1 << 40) / d->c)
    return bad("h * w * c must lie below 2^40");
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
st_status check_map(const st_norm_desc& d, const st_map_ref* m, int es,
                    bool out, const char* name) {
  if (!m || !m->data) return bad(std::string(name) + " is NULL");
  if (!aligned(m->data, es)) return bad(std::string(name) + " is misaligned");
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
  return g;
}
// A map for blocks of g.rows sites at a time.
NormMap map_of(const st_norm_desc& d, const st_map_ref& m,
               const NormGeom& g) {
  NormMap r{m.data, m.stride_n, m.stride_h, m.stride_w, d.w, 0, 0, 0};
  if (d.h == 1 || d.w == 1 || m.stride_h == m.stride_w * d.w) {
    // evenly apart: a line to each site
    r.sh = d.w == 1 ? m.stride_h : m.stride_w;
    r.w = 1;
    r.step = g.rows * r.sh;
    return r;
  }
  r.dx = g.rows % d.w;
  r.step = g.rows / d.w * r.sh + r.dx * r.sw;
  r.wrap = r.sh - d.w * r.sw;
  return r;
}
// The threads of the blocks that hold the image's groups (of x and dy in the
// backward pass), or 0 and a cut into site ranges.  (8x47x78x512 f16 20.5 us
// held, 23 in ranges; 16x64x64x256 f16 21 and 22.5, one such image 14 and 14.5;
// 32x8x8x320 f32 6.6 and 11; 9x32x64x512 f32 in 32 groups 27 and 25.)
int hold_or_split(const st_norm_desc& d, NormGeom& g, bool backward) {
  const int es = esize(d.dtype);
  if (hold(g, es, kFewThreads, kHeld)) return kFewThreads;
  if (hold(g, es, kManyThreads, backward ? kHeld / 2 : kHeld))
    return kManyThreads;
  split(g, es, backward);
  return 0;
}

st_status workspace_of(const st_norm_desc* d, int32_t backward,
                       uint64_t* bytes) {
  if (const st_status s = check_desc(d); s != ST_OK) return s;
  if (!bytes) return bad("bytes is NULL");
  // the cut follows the vector, which a call picks by its addresses
  *bytes = 0;
  for (int v = 8; v >= 1 && d->n > 0; v /= 2) {
    NormGeom g;
    if (!geom(*d, v, g)) continue;
    const int held = hold_or_split(*d, g, backward != 0);
    *bytes =
        std::max<uint64_t>(*bytes, space_of(g, backward != 0, held).bytes);
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

void launch_norm(const NormArgs& a, int dtype, int out_dtype, int held,
                 int batch, hipStream_t q) {
  with_norm(dtype, out_dtype, a.g, [&](auto ti, auto to, auto vt, auto wt) {
    using T = typename decltype(ti)::type;
    using O = typename decltype(to)::type;
    constexpr int V = decltype(vt)::value;
    constexpr bool W = decltype(wt)::value;
    if (held) {
      with_held(a, [&](const NormArgs& b, unsigned grid) {
        if (held == kFewThreads)
          k_norm_held<T, O, V, W, kFewThreads><<<grid, kFewThreads, 0, q>>>(b);
        else
          k_norm_held<T, O, V, W, kManyThreads>
              <<<grid, kManyThreads, 0, q>>>(b);
      });
    } else {
      with_activation(a.act, [&](auto act) {
        with_batches(a, batch, [&](const NormArgs& b, bool) {
          k_norm_pass<T, O, V, W, decltype(act)::value>
              <<<pass_blocks(b), kThreads, 0, q>>>(b);
        });
      });
    }
  });
}

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
    const int es = esize(d->dtype), eo = esize(d->out_dtype);
    if (const st_status s = check_map(*d, x, es, false, "x"); s != ST_OK)
      return s;
    if (const st_status s = check_map(*d, y, eo, true, "y"); s != ST_OK)
      return s;
    for (const void* p : {(const void*)gamma, (const void*)beta,
                          (const void*)mean, (const void*)rstd})
      if (!aligned(p, 4)) return bad("an array of floats is misaligned");
    if (!mean != !rstd) return bad("mean and rstd: both or neither");
    if (const st_status s = check_space(*d, false, ws, ws_bytes); s != ST_OK)
      return s;
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
    const int held = hold_or_split(*d, a.g, false);
    a.act = d->act;
    const NormSpace sp = space_of(a.g, false, held);
    char* w = (char*)ws;
    a.x = map_of(*d, *x, a.g);
    a.y = map_of(*d, *y, a.g);
    a.gamma = gamma;
    a.beta = beta;
    a.eps = d->eps;
    a.part = (float*)(w + sp.part);
    a.parts = a.g.slabs * a.g.cparts;
    a.mean_out = mean;
    a.rstd_out = rstd;
    launch_norm(a, d->dtype, d->out_dtype, held,
                batch_of(a.g, read_size(*d, false)), (hipStream_t)stream);
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
    const int es = esize(d->dtype), eo = esize(d->out_dtype);
    for (const void* p : {(const void*)gamma, (const void*)beta,
                          (const void*)mean, (const void*)rstd,
                          (const void*)dgamma, (const void*)dbeta})
      if (!aligned(p, 4)) return bad("an array of floats is misaligned");
    hipStream_t q = (hipStream_t)stream;
    NormArgs a{};
    a.dgamma = dgamma;
    a.dbeta = dbeta;
    a.act = d->act;
    a.g.c = d->c;
    const int dblocks = dgamma || dbeta ? (int)ceil_div(d->c, 32) : 0;
    if (d->n == 0) {
      // no image: the parameters' gradients are zero
      if (dblocks) {
        (void)hipGetLastError();
        a.dblocks = dblocks;
        launch_norm_backward(a, ST_F32, ST_F32, 0, 1, q);
        return launch_status("group norm backward");
      }
      return ST_OK;
    }
    if (const st_status s = check_map(*d, dy, eo, false, "dy"); s != ST_OK)
      return s;
    if (const st_status s = check_map(*d, x, es, false, "x"); s != ST_OK)
      return s;
    if (const st_status s = check_map(*d, dx, es, true, "dx"); s != ST_OK)
      return s;
    if (!mean || !rstd) return bad("mean or rstd is NULL");
    if (const st_status s = check_space(*d, true, ws, ws_bytes); s != ST_OK)
      return s;
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
    const int held = hold_or_split(*d, a.g, true);
    const NormSpace sp = space_of(a.g, true, held);
    char* w = (char*)ws;
    a.x = map_of(*d, *x, a.g);
    a.dy = map_of(*d, *dy, a.g);
    a.y = map_of(*d, *dx, a.g);
    a.gamma = gamma;
    a.beta = beta;
    a.mean = mean;
    a.rstd = rstd;
    a.eps = d->eps;
    a.part = (float*)(w + sp.part);
    a.parts = a.g.slabs * a.g.cparts;
    a.chpart = (float*)(w + sp.chpart);
    a.dblocks = dblocks;
    launch_norm_backward(a, d->dtype, d->out_dtype, held,
                         batch_of(a.g, read_size(*d, true)), q);
    return launch_status("group norm backward");
  });
}
