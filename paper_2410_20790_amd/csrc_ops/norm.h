// Group norm with an activation on channels-last maps: what the forward and
// the backward kernels share.
//
// The channels of a site are adjacent, so a block takes `cols` vectors of V
// adjacent channels of `rows` sites at a time, and a thread meets the same
// channels at every site: their parameters stay in its registers.
#pragma once

#include <algorithm>
#include <numeric>

#include "ops_common.h"

namespace st {
namespace ops {

constexpr int kThreads = 256;
constexpr int kMaxCols = 256;    // vectors a block has side by side

// How the channels are cut.  A column block holds whole groups, or (groups
// wider than a block) one of `cparts` parts of one group.
struct NormGeom {
  int64_t sites;       // per image
  int n, c, groups, cpg;
  int v;               // channels per vector
  int whole;           // every vector lies in one group
  int cv;              // vectors per site
  int cols, rows;      // vectors and sites a block takes at a time
  int colblocks, kg, cparts, unit_vec;
  int slabs;           // site ranges per image, per column block
  int64_t slab_sites;
  int units;           // slabs * colblocks, of one image
};

// A map as a block's threads walk it, `rows` sites at a time.
struct NormMap {
  void* p;
  int64_t sn, sh, sw;
  int w;               // sites of a line; 1 where sites are evenly apart (sh)
  int dx;              // sites into the line that a step moves
  int64_t step, wrap;  // its elements; those that the next line adds
};

struct NormArgs {
  NormGeom g;
  NormMap x, y, dy;    // y: dx in the backward pass
  const float* gamma;
  const float* beta;
  const float* mean;   // [n][groups]
  const float* rstd;
  float* mean_out;
  float* rstd_out;
  float eps;
  int act;
  // Large images: parts of a group's sums, one for each range of sites (and
  // part of a group); forward [n][groups][parts] {count, mean in two
  // parts, M2}, backward {sum dz gamma, sum dz gamma xh}
  float* part;
  int parts;
  // The images that a launch sums up and those that it finishes (held: all).
  int sum0, sum1, end0, end1;
  float* chpart;       // backward: [n][slabs][c] {sum dz, sum dz xh}
  float* dgamma;
  float* dbeta;
  int dblocks;         // blocks that reduce dgamma and dbeta at the end
};

// The block's place: image, site range, vectors and groups.
struct Place {
  int n, slab, cb, vec0, nvec, g0, ng;
  int64_t s0, s1;
};
__device__ __forceinline__ Place place_of(const NormGeom& g, int n, int u) {
  Place p;
  p.n = n;
  p.slab = u / g.colblocks;
  p.cb = u - p.slab * g.colblocks;
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

// The block's unit, so that neighbouring units -- adjacent channels of the
// same sites, which share cache lines -- go to one of the eight dies (blocks
// are dealt out to them in turn) at about the same time.
__device__ __forceinline__ int near_block(int units) {
  const int per = units / 8, b = blockIdx.x;
  return b < per * 8 ? (b % 8) * per + b / 8 : b;
}

// One thread's sites of a map, `rows` apart: a few additions for each, no
// product or quotient.
template <typename T>
struct SiteWalk {
  T* p;
  int64_t step, wrap;
  int x, dx, w;
  __device__ __forceinline__ SiteWalk(const NormMap& m, int n, int64_t s,
                                      int ch)
      : step(m.step), wrap(m.wrap), dx(m.dx), w(m.w) {
    const int64_t line = w == 1 ? s : s / w;
    x = (int)(s - line * w);
    p = (T*)m.p + n * m.sn + line * m.sh + x * m.sw + ch;
  }
  __device__ __forceinline__ void next() {
    p += step;
    x += dx;
    if (x >= w) {
      x -= w;
      p += wrap;
    }
  }
};

// A thread's channels: mean and rstd of their groups, gamma and beta.  WHOLE:
// all in one group, whose statistics are kept once.
template <int V, bool WHOLE>
struct Params {
  static constexpr int S = WHOLE ? 1 : V;
  float mean[S], rstd[S], gamma[V], beta[V];
  __device__ __forceinline__ void load_affine(const NormArgs& a, int ch) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      gamma[i] = a.gamma ? a.gamma[ch + i] : 1.f;
      beta[i] = a.beta ? a.beta[ch + i] : 0.f;
    }
  }
  __device__ __forceinline__ void load(const NormArgs& a, int n, int ch) {
    load_affine(a, ch);
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const int64_t at = (int64_t)n * a.g.groups + (ch + i) / a.g.cpg;
      mean[i] = a.mean[at];
      rstd[i] = a.rstd[at];
    }
  }
  // from a block's own, group j of the block at res[step j]
  __device__ __forceinline__ void load_stats(const float* res, int step,
                                             int ch, int cpg, int g0) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const int j = (ch + i) / cpg - g0;
      mean[i] = res[j * step];
      rstd[i] = res[j * step + 1];
    }
  }
  __device__ __forceinline__ float mu(int i) const {
    return mean[WHOLE ? 0 : i];
  }
  __device__ __forceinline__ float r(int i) const {
    return rstd[WHOLE ? 0 : i];
  }
};

// What block b of a launch over large images does: units that finish images
// and units that sum up the next ones take turns.
struct Turn {
  int n, u;
  bool end;
  __device__ __forceinline__ Turn(const NormArgs& a, int b, int ends,
                                  int all) {
    const int sums = all - ends, pairs = 2 * min(ends, sums);
    int i;
    if (b < pairs) {
      end = b & 1;
      i = b >> 1;
    } else {
      end = ends > sums;
      i = b - pairs / 2;
    }
    n = i / a.g.units;
    u = i - n * a.g.units;
    n += end ? a.end0 : a.sum0;
  }
};

// Lanes that share a group when a block's entries are joined: a power of two,
// within one wave, so that all groups are joined at once if they can be.
__device__ __forceinline__ int lanes_per_group(int threads, int ng) {
  int t = 64;
  while (t > 1 && t * ng > threads) t >>= 1;
  return t;
}
template <typename F>
__device__ __forceinline__ F lanes_sum(F x, int lanes) {
  for (int d = lanes >> 1; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}
__device__ __forceinline__ void lanes_sum2(float& x, float& y, int lanes) {
  for (int d = lanes >> 1; d; d >>= 1) {
    const float a = __shfl_xor(x, d), b = __shfl_xor(y, d);
    x += a;
    y += b;
  }
}
// Places of a block's entries of one group: `wide` adjacent ones of every row,
// `lanes` apart, each lane from its own on.
struct Entries {
  int row, c, down, over, wide;
  __device__ __forceinline__ Entries(int in, int lanes, int wide_)
      : wide(wide_) {
    row = in / wide;
    c = in - row * wide;
    down = lanes / wide;
    over = lanes - down * wide;
  }
  __device__ __forceinline__ void next() {
    row += down;
    c += over;
    if (c >= wide) {
      c -= wide;
      ++row;
    }
  }
};

// -------------------------------------------------------------- host side

// The held kernels: threads of a block, sites a thread holds (backward, where
// it holds x and dy: half as many in the larger blocks).
constexpr int kFewThreads = 256, kManyThreads = 1024;
constexpr int kHeld = 8;

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
// WHOLE or not, for the vectors that may straddle groups.
template <int V, class F>
void with_whole(bool whole, F&& f) {
  if constexpr (V > 1 && V <= 4) {
    if (!whole) {
      f(std::false_type{});
      return;
    }
  }
  f(std::true_type{});
}
constexpr int64_t kMaxGrid = 1 << 20;
inline unsigned grid_of(int64_t units) {
  return (unsigned)std::min<int64_t>(units, kMaxGrid);
}
// Calls f(types, vector, whole) of a call.
template <class F>
void with_norm(int dtype, int out_dtype, const NormGeom& g, F&& f) {
  with_types(dtype, out_dtype, [&](auto ti, auto to) {
    with_vec(g.v, [&](auto vt) {
      constexpr int V = decltype(vt)::value;
      using T = typename decltype(ti)::type;
      using O = typename decltype(to)::type;
      if constexpr (V * sizeof(T) <= 16 && V * sizeof(O) <= 16)
        with_whole<V>(g.whole, [&](auto wt) { f(ti, to, vt, wt); });
    });
  });
}

inline unsigned pass_blocks(const NormArgs& a) {
  return grid_of((int64_t)(a.end1 - a.end0 + a.sum1 - a.sum0) * a.g.units);
}
// Calls f(arguments, blocks) for the launches of blocks that hold whole groups,
// each over as many images as a grid has room for.
template <class F>
void with_held(NormArgs a, F&& f) {
  const int64_t most = std::max<int64_t>(1, kMaxGrid / a.g.units);
  for (int64_t i = 0; i < a.g.n; i += most) {
    a.end0 = (int)i;
    a.end1 = (int)std::min<int64_t>(i + most, a.g.n);
    f(a, (unsigned)((int64_t)(a.end1 - a.end0) * a.g.units));
  }
}
// Calls f(arguments, last) for the launches over large images, each of which sums
// up the images of one batch and finishes those of the batch before: a batch is
// as many images as the last-level cache keeps until they are read again.
template <class F>
void with_batches(NormArgs a, int batch, F&& f) {
  const int n = a.g.n;
  for (int64_t i = 0;; i += batch) {
    a.sum0 = (int)std::min<int64_t>(i, n);
    a.sum1 = (int)std::min<int64_t>(i + batch, n);
    a.end0 = (int)std::max<int64_t>(i - batch, 0);
    a.end1 = (int)std::min<int64_t>(i, n);
    f(a, i >= n);
    if (i >= n) break;
  }
}

// Launches (defined beside their kernels); held: threads of the blocks that
// hold whole groups, or 0 and the images of a batch.
void launch_norm(const NormArgs& a, int dtype, int out_dtype, int held,
                 int batch, hipStream_t q);
void launch_norm_backward(const NormArgs& a, int dtype, int out_dtype,
                          int held, int batch, hipStream_t q);

}  // namespace ops
}  // namespace st
