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
  // rows split along time
  int cols;                        // blocks of 64 lanes
  int tiles, group;                // tiles of a row, tiles of a group
  void* ends;                      // the ticket, then words: tiles, groups
  int narrow;                      // 32-bit offsets within one time
};
constexpr int kHeadWords = 2;

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
          for (int e = 0; e < V; ++e) y[e] *= sigmoid_once(o[e]);
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

// ------------------------------------------------- rows split along time
//
// Few rows and channels, many steps: a thread for each would leave the device
// idle.  h_s = a_s h_{s-1} + u_s joins: a run of steps acts as h -> A h + H
// with A the product of its a (d -> A d + D for the gradient, whose order is
// the reverse).  A block takes a tile: 64 lanes (V adjacent channels of a row
// each) over W waves, a wave kSplit steps of every lane.  Gates and inputs of
// these steps stay in registers, so that all is read once and every gate
// computed once; the tile's (A, H) is published, those of the tiles before it
// are folded, and the steps are run from the state that enters.
//
// Tiles are numbered by a ticket, so a block only waits for blocks that run
// already, and these publish before they wait for anything themselves.  The
// fold is in two levels, groups of `group` tiles and the tiles of the block's
// own group, both in running order and cut by sizes alone: the same bits in
// every run.  (Publishing states instead, each from the one before, would be
// a chain of as many memory round trips as there are tiles; taking whatever
// is there first would change the order of the roundings.)

constexpr int kSplit = ST_SCAN_STRIDE;   // steps of a wave

// A reset is a factor of minus zero (gates are never negative), which no value
// passes, not even NaN.
constexpr float kCut = -0.f;
__device__ __forceinline__ bool is_cut(float A) {
  return __float_as_uint(A) == 0x80000000u;
}

// (A, H), then (x, y): the steps of (x, y) run after those of (A, H).
template <int V>
__device__ __forceinline__ void then(float* A, float* H, const float* x,
                                     const float* y) {
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const bool cut = is_cut(x[e]);
    H[e] = cut ? y[e] : __builtin_fmaf(x[e], H[e], y[e]);
    A[e] = cut ? x[e] : A[e] * x[e];
  }
}
template <int V>
__device__ __forceinline__ void none(float* A, float* H) {
#pragma unroll
  for (int e = 0; e < V; ++e) {
    A[e] = 1.f;
    H[e] = 0.f;
  }
}

// A published value: its bits beside a mark, in one 8-byte word, so that it
// is whole when it is seen.  Words start as zeros.
typedef unsigned long long Word;
__device__ __forceinline__ void publish(Word* w, float x) {
  __hip_atomic_store(w, (1ull << 32) | __float_as_uint(x), __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ Word peek(const Word* w) {
  return __hip_atomic_load(w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The places of published (A, H): entry i of this block's lanes.
struct Ends {
  Word* base;        // of entry 0, this lane
  int64_t plane;     // words of an entry's A (its H follows)
};
template <int V>
__device__ __forceinline__ void put_entry(const Ends& p, int64_t i,
                                          const float* A, const float* H) {
  Word* w = p.base + i * 2 * p.plane;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    publish(w + e, A[e]);
    publish(w + p.plane + e, H[e]);
  }
}
// Folds entries [i0, i1) into (A, H), two at a time, waiting for each.  (Few
// registers: the gates of the block's steps are held meanwhile.)
template <int V>
__device__ __forceinline__ void fold_entries(const Ends& p, int i0, int i1,
                                             float* A, float* H) {
  const Word* q = p.base + (int64_t)i0 * 2 * p.plane;
  for (int i = i0; i < i1; i += 2) {
    const int64_t next = i + 1 < i1 ? 2 * p.plane : 0;
    Word w[2][2 * V];
    bool all;
    do {
      all = true;
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          w[k][e] = peek(q + k * next + e);
          w[k][V + e] = peek(q + k * next + p.plane + e);
        }
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) all = all && (w[k][e] >> 32) != 0;
      if (!all) __builtin_amdgcn_s_sleep(1);
    } while (!all);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (i + k < i1) {
        float x[V], y[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          x[e] = __uint_as_float((uint32_t)w[k][e]);
          y[e] = __uint_as_float((uint32_t)w[k][V + e]);
        }
        then<V>(A, H, x, y);
      }
    }
    q += 2 * next;
  }
}

// A block's lanes and waves, in running order: wave 0 has the first steps to
// run (of the backward pass: the row's last).
template <int V, int W>
struct TileShared {
  float a[W][64 * V], h[W][64 * V];
  int ticket;
};

// Joins the waves' (A, H) in LDS: each wave gets what runs before it in `A, H`
// and every wave the whole in `TA, TH`.
template <int V, int W>
__device__ __forceinline__ void join_waves(TileShared<V, W>& sh, int wave,
                                           float* A, float* H, float* TA,
                                           float* TH) {
  const int at = (threadIdx.x & 63) * V;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < V; ++e) {
    sh.a[wave][at + e] = A[e];
    sh.h[wave][at + e] = H[e];
  }
  __syncthreads();
  none<V>(TA, TH);
#pragma unroll
  for (int w = 0; w < W; ++w) {
    if (w == wave) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        A[e] = TA[e];
        H[e] = TH[e];
      }
    }
    then<V>(TA, TH, &sh.a[w][at], &sh.h[w][at]);
  }
}

// What enters this tile (its k-th in running order): the state `h` after all
// tiles before it, given the tile's own (TA, TH).  h comes in as the state
// before the first tile, which only tile 0 has (the row's state may be
// replaced in place once the last tile has run).
template <int V, int W>
__device__ __forceinline__ void enter_tile(const ScanArgs& a,
                                           TileShared<V, W>& sh, int k,
                                           int col, int wave, float* TA,
                                           float* TH, float* h) {
  if (a.tiles == 1) return;
  Ends p;
  p.plane = (int64_t)a.cols * 64 * V;
  p.base = (Word*)a.ends + kHeadWords +
           ((int64_t)col * 64 + (threadIdx.x & 63)) * V;
  if (k == 0) {
    // nothing enters but h: the tile's end is a state
    if (wave == 0) {
      float cut[V], end[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        cut[e] = kCut;
        end[e] = is_cut(TA[e]) ? TH[e] : __builtin_fmaf(TA[e], h[e], TH[e]);
      }
      put_entry<V>(p, 0, cut, end);
    }
    return;
  }
  if (wave == 0) put_entry<V>(p, k, TA, TH);
  const int g = k / a.group, in = k % a.group;
  float A[V], H[V], PA[V], PH[V];
  // the tiles of its group before it, a share to each wave
  none<V>(A, H);
  const int share = (in + W - 1) / W;
  const int g0 = g * a.group;
  fold_entries<V>(p, g0 + min(wave * share, in),
                  g0 + min((wave + 1) * share, in), A, H);
  join_waves<V, W>(sh, wave, A, H, PA, PH);
  if (in == a.group - 1 && wave == 0 && k < a.tiles - 1) {
    // the last of its group publishes the group
#pragma unroll
    for (int e = 0; e < V; ++e) {
      A[e] = PA[e];
      H[e] = PH[e];
    }
    then<V>(A, H, TA, TH);
    put_entry<V>(p, (int64_t)a.tiles + g, A, H);
  }
  // the groups before its own
  none<V>(A, H);
  const int gs = (g + W - 1) / W;
  fold_entries<V>(p, a.tiles + min(wave * gs, g),
                  a.tiles + min((wave + 1) * gs, g), A, H);
  float GA[V], GH[V];
  join_waves<V, W>(sh, wave, A, H, GA, GH);
  then<V>(GA, GH, PA, PH);
#pragma unroll
  for (int e = 0; e < V; ++e) h[e] = GH[e];
}

// Clears the words and the ticket of a launch.
__global__ __launch_bounds__(256) void k_scan_clear(uint4* w, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n;
       i += (int64_t)gridDim.x * 256)
    w[i] = make_uint4(0, 0, 0, 0);
}

struct LaneAt {
  int b, ch;
  bool on;          // otherwise a copy of the last lane that stores nothing
  int64_t hc;
};
__device__ __forceinline__ LaneAt lane_at(const ScanArgs& a, int col,
                                          int v) {
  int64_t lane = (int64_t)col * 64 + (threadIdx.x & 63);
  LaneAt l;
  l.on = lane < a.lanes;
  if (!l.on) lane = a.lanes - 1;
  l.b = (int)(lane / a.cv);
  l.ch = (int)(lane % a.cv) * v;
  l.hc = (int64_t)l.b * a.q.c + l.ch;
  return l;
}
template <int V, int W>
__device__ __forceinline__ int next_ticket(const ScanArgs& a,
                                           TileShared<V, W>& sh) {
  if (a.tiles == 1) return blockIdx.x;
  if (threadIdx.x == 0)
    sh.ticket = (int)__hip_atomic_fetch_add((unsigned*)a.ends, 1u,
                                            __ATOMIC_RELAXED,
                                            __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(sh.ticket);
}
// Whether all lanes of a wave have all of its steps, at the same times, and
// the time of the first.
struct Whole {
  bool on;
  int64_t t;
  int dir;
};
__device__ __forceinline__ Whole whole_wave(const ScanArgs& a, const Row& r,
                                            int s0) {
  Whole w;
  w.on = a.narrow && !(a.q.lengths && a.q.reverse) &&
         __all(s0 + kSplit <= r.len);
  w.t = a.q.reverse ? a.q.t - 1 - s0 : s0;
  w.dir = a.q.reverse ? -1 : 1;
  return w;
}
template <typename T, int V>
__device__ __forceinline__ void load_steps(const SeqTensor& x, const Whole& w,
                                           const Row& r, int b, int ch,
                                           int s0, Pack<T, V>* out) {
  if (w.on) {
    const WaveWalk<const T> p(x, w.t, w.dir, b, ch);
#pragma unroll
    for (int k = 0; k < kSplit; ++k) out[k] = load_pack<T, V>(p.at(k));
  } else {
    Walk<const T> p(x, r, b, ch, s0);
#pragma unroll
    for (int k = 0; k < kSplit; ++k) {
      out[k] = load_pack<T, V>(p.p);
      p.advance(k);
      // one address at a time, not all of them in registers first
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}
// Bit k: a reset before step s0 + k.
__device__ __forceinline__ unsigned cuts_of(const ScanArgs& a, const Row& r,
                                            int b, int s0) {
  unsigned m = 0;
  if (a.q.reset)
    for (int k = 0; k < kSplit; ++k)
      if (s0 + k < r.len && reset_at(a.q, r, b, s0 + k)) m |= 1u << k;
  return m;
}

template <typename T, typename O, int V, bool GATE, int W>
__global__ __launch_bounds__(64 * W) void k_scan_tiles(ScanArgs a) {
  __shared__ TileShared<V, W> sh;
  const int ticket = next_ticket<V, W>(a, sh);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int tile = ticket / a.cols, col = ticket % a.cols;
  const LaneAt l = lane_at(a, col, V);
  const Row r = row_of(a.q, l.b);
  const int64_t plane = (int64_t)a.q.b * a.q.c;
  const int s0 = (tile * W + wave) * kSplit;
  float h[V];
#pragma unroll
  for (int e = 0; e < V; ++e) h[e] = tile == 0 && a.h ? a.h[l.hc + e] : 0.f;
  const bool any = __any(s0 < r.len);
  const Whole whole = whole_wave(a, r, s0);
  float keep[kSplit][V], u[kSplit][V];
  Pack<T, V> io[kSplit];
  unsigned cuts = 0;
  float A[V], H[V], TA[V], TH[V];
  none<V>(A, H);
  if (any) {
    Pack<T, V> iv[kSplit], jf[kSplit];
    load_steps<T, V>(a.f, whole, r, l.b, l.ch, s0, jf);
    load_steps<T, V>(a.v, whole, r, l.b, l.ch, s0, iv);
    if (GATE) load_steps<T, V>(a.o, whole, r, l.b, l.ch, s0, io);
    cuts = cuts_of(a, r, l.b, s0);
#pragma unroll
    for (int k = 0; k < kSplit; ++k) {
      float v[V], f[V];
      unpack<T, V>(iv[k], v);
      unpack<T, V>(jf[k], f);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        float write;
        sigmoids(f[e], keep[k][e], write);
        u[k][e] = write * v[e];
      }
    }
    // steps behind the row's end keep the state, to the bit
    if (!whole.on) {
#pragma unroll
      for (int k = 0; k < kSplit; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          keep[k][e] = s0 + k < r.len ? keep[k][e] : 1.f;
          u[k][e] = s0 + k < r.len ? u[k][e] : 0.f;
        }
    }
    if (__any(cuts != 0)) {
#pragma unroll
      for (int k = 0; k < kSplit; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const bool cut = cuts >> k & 1;
          H[e] = __builtin_fmaf(keep[k][e], cut ? 0.f : H[e], u[k][e]);
          A[e] = cut ? kCut : A[e] * keep[k][e];
        }
    } else {
#pragma unroll
      for (int k = 0; k < kSplit; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          H[e] = __builtin_fmaf(keep[k][e], H[e], u[k][e]);
          A[e] *= keep[k][e];
        }
    }
  }
  join_waves<V, W>(sh, wave, A, H, TA, TH);
  float WA[V], WH[V];     // what runs before the wave in its tile
#pragma unroll
  for (int e = 0; e < V; ++e) {
    WA[e] = A[e];
    WH[e] = H[e];
  }
  enter_tile<V, W>(a, sh, tile, col, wave, TA, TH, h);
  if (tile == a.tiles - 1 && a.h_out && wave == 0 && l.on) {
#pragma unroll
    for (int e = 0; e < V; ++e)
      a.h_out[l.hc + e] =
          is_cut(TA[e]) ? TH[e] : __builtin_fmaf(TA[e], h[e], TH[e]);
  }
#pragma unroll
  for (int e = 0; e < V; ++e)
    h[e] = is_cut(WA[e]) ? WH[e] : __builtin_fmaf(WA[e], h[e], WH[e]);
  if (!l.on) return;
  if (any) {
    if (a.states && s0 < r.len)
      store_pack<float, V>(a.states + (s0 / kStride) * plane + l.hc, h);
    Walk<O> wy(a.y, r, l.b, l.ch, s0);
    const WaveWalk<O> ww(a.y, whole.t, whole.dir, l.b, l.ch);
#pragma unroll
    for (int k = 0; k < kSplit; ++k) {
      if (s0 + k < r.len) {
        const bool cut = cuts >> k & 1;
        float y[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if (cut) h[e] = 0.f;
          h[e] = __builtin_fmaf(keep[k][e], h[e], u[k][e]);
          y[e] = h[e];
        }
        if (GATE) {
          float o[V];
          unpack<T, V>(io[k], o);
#pragma unroll
          for (int e = 0; e < V; ++e) y[e] *= sigmoid_once(o[e]);
        }
        if (whole.on) {
          store_pack<O, V>(ww.at(k), y);
        } else {
          store_pack<O, V>(wy.p, y);
          wy.advance(k);
        }
      }
    }
  }
  O* py = (O*)a.y.p + (int64_t)l.b * a.y.sb + l.ch;
  const int s1 = min(s0 + kSplit, a.q.t);
  for (int s = max(s0, r.len); s < s1; ++s) {
    float z[V];
#pragma unroll
    for (int e = 0; e < V; ++e) z[e] = 0.f;
    store_pack<O, V>(py + (int64_t)s * a.y.st, z);
  }
}

// The backward pass: tiles and waves run from the row's last step; the states
// of a wave's steps come again from the one kept before them.
template <typename T, typename O, int V, bool GATE, int W>
__global__ __launch_bounds__(64 * W) void k_scan_grad_tiles(ScanArgs a) {
  __shared__ TileShared<V, W> sh;
  const int ticket = next_ticket<V, W>(a, sh);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int k_th = ticket / a.cols, col = ticket % a.cols;
  const LaneAt l = lane_at(a, col, V);
  const Row r = row_of(a.q, l.b);
  const int64_t plane = (int64_t)a.q.b * a.q.c;
  const int s0 = ((a.tiles - 1 - k_th) * W + W - 1 - wave) * kSplit;
  float dh[V];
#pragma unroll
  for (int e = 0; e < V; ++e) dh[e] = k_th == 0 && a.h ? a.h[l.hc + e] : 0.f;
  const bool any = __any(s0 < r.len);
  const Whole whole = whole_wave(a, r, s0);
  float keep[kSplit][V], write[kSplit][V];
  float g[kSplit][V];     // dy sigmoid(o)
  float q[kSplit][V];     // h_{s-1} - v
  unsigned cuts = 0;
  float A[V], D[V], TA[V], TD[V];
  none<V>(A, D);
  if (any) {
    Pack<T, V> iv[kSplit], jf[kSplit], io[kSplit];
    Pack<O, V> id[kSplit];
    float h[V];
    load_steps<T, V>(a.f, whole, r, l.b, l.ch, s0, jf);
    load_steps<T, V>(a.v, whole, r, l.b, l.ch, s0, iv);
    if (GATE) load_steps<T, V>(a.o, whole, r, l.b, l.ch, s0, io);
    load_steps<O, V>(a.y, whole, r, l.b, l.ch, s0, id);
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = 0.f;
    if (s0 < r.len)
      unpack<float, V>(load_pack<float, V>(
                           a.states + (s0 / kStride) * plane + l.hc),
                       h);
    cuts = cuts_of(a, r, l.b, s0);
    Walk<T> wg(GATE ? a.d_o : a.dv, r, l.b, l.ch, s0);
    const WaveWalk<T> wwg(GATE ? a.d_o : a.dv, whole.t, whole.dir, l.b, l.ch);
#pragma unroll
    for (int k = 0; k < kSplit; ++k) {
      float v[V], f[V], o[V], go[V];
      unpack<T, V>(iv[k], v);
      unpack<T, V>(jf[k], f);
      unpack<O, V>(id[k], g[k]);
      if (GATE) unpack<T, V>(io[k], o);
      const bool cut = cuts >> k & 1;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        sigmoids(f[e], keep[k][e], write[k][e]);
        if (cut) h[e] = 0.f;
        q[k][e] = h[e] - v[e];
        h[e] = __builtin_fmaf(keep[k][e], h[e], write[k][e] * v[e]);
        if (GATE) {
          float p, n;
          sigmoids(o[e], p, n);
          go[e] = g[k][e] * h[e] * p * n;
          g[k][e] *= p;
        }
      }
      if (GATE && s0 + k < r.len && l.on) {
        if (whole.on) {
          store_pack<T, V>(wwg.at(k), go);
        } else {
          store_pack<T, V>(wg.p, go);
          wg.advance(k);
        }
      }
    }
    if (!whole.on) {
#pragma unroll
      for (int k = 0; k < kSplit; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          keep[k][e] = s0 + k < r.len ? keep[k][e] : 1.f;
          g[k][e] = s0 + k < r.len ? g[k][e] : 0.f;
        }
    }
    if (__any(cuts != 0)) {
#pragma unroll
      for (int k = kSplit - 1; k >= 0; --k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const bool cut = cuts >> k & 1;
          D[e] = cut ? 0.f : (D[e] + g[k][e]) * keep[k][e];
          A[e] = cut ? kCut : A[e] * keep[k][e];
        }
    } else {
#pragma unroll
      for (int k = kSplit - 1; k >= 0; --k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          D[e] = (D[e] + g[k][e]) * keep[k][e];
          A[e] *= keep[k][e];
        }
    }
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
  if (any) {
    // back from the last of the wave's steps that the row has
    Walk<T> wv(a.dv, r, l.b, l.ch, s0 + kSplit - 1),
        wf(a.df, r, l.b, l.ch, s0 + kSplit - 1);
    const WaveWalk<T> wwv(a.dv, whole.t, whole.dir, l.b, l.ch),
        wwf(a.df, whole.t, whole.dir, l.b, l.ch);
#pragma unroll
    for (int k = kSplit - 1; k >= 0; --k) {
      if (s0 + k < r.len) {
        const bool cut = cuts >> k & 1;
        float gv[V], gf[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          dh[e] += g[k][e];
          gv[e] = dh[e] * write[k][e];
          gf[e] = dh[e] * q[k][e] * (keep[k][e] * write[k][e]);
          dh[e] = cut ? 0.f : dh[e] * keep[k][e];
        }
        if (whole.on) {
          store_pack<T, V>(wwv.at(k), gv);
          store_pack<T, V>(wwf.at(k), gf);
        } else {
          store_pack<T, V>(wv.p, gv);
          store_pack<T, V>(wf.p, gf);
          wv.p -= wv.step;
          wf.p -= wf.step;
        }
      }
    }
  }
  T* pdv = (T*)a.dv.p + (int64_t)l.b * a.dv.sb + l.ch;
  T* pdf = (T*)a.df.p + (int64_t)l.b * a.df.sb + l.ch;
  T* pdo = GATE ? (T*)a.d_o.p + (int64_t)l.b * a.d_o.sb + l.ch : nullptr;
  const int s1 = min(s0 + kSplit, a.q.t);
  for (int s = max(s0, r.len); s < s1; ++s) {
    float z[V];
#pragma unroll
    for (int e = 0; e < V; ++e) z[e] = 0.f;
    store_pack<T, V>(pdv + (int64_t)s * a.dv.st, z);
    store_pack<T, V>(pdf + (int64_t)s * a.df.st, z);
    if (GATE) store_pack<T, V>(pdo + (int64_t)s * a.d_o.st, z);
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

// Which rows are split along time: those of more than 64 steps (a chunk's
// frames, 32 at most, are walked one after another, as they are taken one by
// one: the same bits) of which there are too few to fill the device, a lane
// each.
constexpr int kSerialSteps = 64;
constexpr int64_t kFillWaves = 2048;    // eight to a CU

struct ScanCut {
  bool split = false;
  int cols = 0, tiles = 0, group = 0;
  uint64_t words = 0;
};
ScanCut cut_of(const st_seq_desc& d, int waves) {
  ScanCut c;
  const int64_t cols = ceil_div((int64_t)d.b * d.c, 64);
  if (d.t <= kSerialSteps || cols >= kFillWaves) return c;
  c.split = true;
  c.cols = (int)cols;
  c.tiles = (int)ceil_div(d.t, (int64_t)kSplit * waves);
  // a block folds at most group tiles and tiles / group groups
  c.group = 8;
  while ((int64_t)c.group * c.group < c.tiles) c.group *= 2;
  if (c.tiles > 1)
    c.words = kHeadWords + (uint64_t)(c.tiles + c.tiles / c.group) * 2 *
                               c.cols * 64;
  return c;
}
constexpr int kWaves = 8, kGradWaves = 8;

uint64_t scan_space(const st_seq_desc& d, bool backward) {
  if (empty(d)) return 0;
  return (cut_of(d, backward ? kGradWaves : kWaves).words * 8 + 15) / 16 * 16;
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
    a.narrow = narrow(*d, v, es) && narrow(*d, f, es) && narrow(*d, o, es) &&
               narrow(*d, y, eo);
    a.h = h;
    a.h_out = h_out;
    a.states = states;
    a.cv = d->c / vec;
    a.lanes = (int64_t)d->b * a.cv;
    hipStream_t q = (hipStream_t)stream;
    const ScanCut cut = cut_of(*d, kWaves);
    if (cut.split) {
      vec = 1;
      a.cv = d->c;
      a.lanes = (int64_t)d->b * d->c;
      take_cut(a, cut, ws, q);
    }
    const unsigned grid =
        cut.split ? (unsigned)(cut.cols * cut.tiles)
                  : (unsigned)ceil_div(a.lanes, kThreads);
    with_types(d->dtype, d->out_dtype, [&](auto ti, auto to) {
      using T = typename decltype(ti)::type;
      using O = typename decltype(to)::type;
      with_scan(vec, o != nullptr, [&](auto vt, auto gt) {
        constexpr int V = decltype(vt)::value;
        constexpr bool G = decltype(gt)::value;
        if (!cut.split) {
          k_scan<T, O, V, G><<<grid, kThreads, 0, q>>>(a);
          return;
        }
        if constexpr (V == 1)
          k_scan_tiles<T, O, V, G, kWaves>
              <<<grid, 64 * kWaves, 0, q>>>(a);
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
    a.narrow = narrow(*d, dy, eo);
    for (const st_seq_ref* r : {v, f, o, dv, df, d_o})
      a.narrow = a.narrow && narrow(*d, r, es);
    a.h = dh_out;
    a.h_out = dh;
    a.states = const_cast<float*>(states);
    a.cv = d->c / vec;
    a.lanes = (int64_t)d->b * a.cv;
    hipStream_t q = (hipStream_t)stream;
    const ScanCut cut = cut_of(*d, kGradWaves);
    if (cut.split) {
      vec = 1;
      a.cv = d->c;
      a.lanes = (int64_t)d->b * d->c;
      take_cut(a, cut, ws, q);
    }
    const unsigned grid =
        cut.split ? (unsigned)(cut.cols * cut.tiles)
                  : (unsigned)ceil_div(a.lanes, kThreads);
    with_types(d->dtype, d->out_dtype, [&](auto ti, auto to) {
      using T = typename decltype(ti)::type;
      using O = typename decltype(to)::type;
      with_scan(vec, o != nullptr, [&](auto vt, auto gt) {
        constexpr int V = decltype(vt)::value;
        constexpr bool G = decltype(gt)::value;
        if (!cut.split) {
          k_scan_grad<T, O, V, G><<<grid, kThreads, 0, q>>>(a);
          return;
        }
        if constexpr (V == 1)
          k_scan_grad_tiles<T, O, V, G, kGradWaves>
              <<<grid, 64 * kGradWaves, 0, q>>>(a);
      });
    });
    return launch_status("gated scan backward");
  });
}
