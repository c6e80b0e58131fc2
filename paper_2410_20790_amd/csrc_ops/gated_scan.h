// The gated linear recurrence: what its forward and backward kernels share.
#pragma once

#include "seq.h"

namespace st {
namespace ops {

constexpr int kStride = ST_SCAN_STRIDE;
constexpr int kScanThreads = 256;

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
  int narrow;                      // 32-bit offsets (see StepsAt)
  int stream;                      // inputs larger than the caches
};
constexpr int kHeadWords = 2;

// ------------------------------------------------- rows split along time
//
// Few rows and channels, many steps: a thread for each would leave the device
// idle.  h_s = a_s h_{s-1} + u_s joins: a run of steps acts as h -> A h + H
// with A the product of its a (d -> A d + D for the gradient, whose order is
// the reverse).  A block takes a tile: 64 lanes (a channel of a row each) over
// W waves, a wave kSplit steps of every lane.  Gates and inputs of
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
__device__ __forceinline__ void then(float& A, float& H, float x, float y) {
  const bool cut = is_cut(x);
  H = cut ? y : __builtin_fmaf(x, H, y);
  A = cut ? x : A * x;
}
// A product of gates none of which is zero (nor a cut) does not become zero,
// however many they are: an infinite state passes them, as it passes one after
// another.  (Seen to once for many factors, where the product is zero.)
__device__ __forceinline__ bool is_zero(float A) {
  return __float_as_uint(A) == 0;
}
__device__ __forceinline__ void keep_product(float& A, bool zero_factor) {
  if (is_zero(A) && !zero_factor) A = 0x1p-149f;
}
// The state after the steps of (A, H), from the state h.
__device__ __forceinline__ float after(float A, float H, float h) {
  return is_cut(A) ? H : __builtin_fmaf(A, h, H);
}

// A published (A, H) of a channel, in one 8-byte word, so that it is whole when
// it is seen: H's bits below A's with the sign set, which no factor has (a
// reset, minus zero, goes as minus infinity).  Words start as zeros.
typedef unsigned long long Word;
constexpr uint32_t kCutBits = 0xff800000u;
__device__ __forceinline__ void publish(Word* w, float A, float H) {
  const uint32_t hi =
      is_cut(A) ? kCutBits : __float_as_uint(A) | 0x80000000u;
  __hip_atomic_store(w, (Word)hi << 32 | __float_as_uint(H), __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ Word peek(const Word* w) {
  return __hip_atomic_load(w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The places of published (A, H): entry i of this block's lanes.
struct Ends {
  Word* base;        // of entry 0, this lane
  int64_t plane;     // words of an entry
  __device__ __forceinline__ Word* at(int64_t i) const {
    return base + i * plane;
  }
};
// Folds entries [i0, i1) into (A, H), four at a time, waiting for each.
__device__ __forceinline__ void fold_entries(const Ends& p, int i0, int i1,
                                             float& A, float& H) {
  constexpr int N = 4;
  bool zero = false;
  const Word* q = p.at(i0);
  for (int i = i0; i < i1; i += N) {
    Word w[N];
    bool all;
    do {
      all = true;
#pragma unroll
      for (int k = 0; k < N; ++k)
        w[k] = peek(q + (int64_t)min(k, i1 - 1 - i) * p.plane);
#pragma unroll
      for (int k = 0; k < N; ++k) all = all && (w[k] >> 63) != 0;
      if (!all) __builtin_amdgcn_s_sleep(1);
    } while (!all);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (i + k < i1) {
        const uint32_t hi = (uint32_t)(w[k] >> 32);
        const float x =
            hi == kCutBits ? kCut : __uint_as_float(hi & 0x7fffffffu);
        then(A, H, x, __uint_as_float((uint32_t)w[k]));
        zero = zero || is_zero(x);
      }
    }
    q += N * p.plane;
  }
  keep_product(A, zero);
}

// A block's lanes and waves, in running order: wave 0 has the first steps to
// run (of the backward pass: the row's last).
template <int W>
struct TileShared {
  float a[W][64], h[W][64];
  int ticket;
};

// Joins the waves' (A, H) in LDS: each wave gets what runs before it in `A, H`
// and every wave the whole in `TA, TH`.
template <int W>
__device__ __forceinline__ void join_waves(TileShared<W>& sh, int wave,
                                           float& A, float& H, float& TA,
                                           float& TH) {
  const int at = threadIdx.x & 63;
  __syncthreads();
  sh.a[wave][at] = A;
  sh.h[wave][at] = H;
  __syncthreads();
  TA = 1.f;
  TH = 0.f;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    if (w == wave) {
      A = TA;
      H = TH;
    }
    then(TA, TH, sh.a[w][at], sh.h[w][at]);
  }
  if (__any(is_zero(A) || is_zero(TA))) {
    bool zero = false;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      if (w == wave) keep_product(A, zero);
      zero = zero || is_zero(sh.a[w][at]);
    }
    keep_product(TA, zero);
  }
}

// What enters this tile (its k-th in running order): the state `h` after all
// tiles before it, given the tile's own (TA, TH).  h comes in as the state
// before the first tile, which only tile 0 has (the row's state may be
// replaced in place once the last tile has run).
template <int W>
__device__ __forceinline__ void enter_tile(const ScanArgs& a,
                                           TileShared<W>& sh, int k, int col,
                                           int wave, float TA, float TH,
                                           float& h) {
  if (a.tiles == 1) return;
  Ends p;
  p.plane = (int64_t)a.cols * 64;
  p.base = (Word*)a.ends + kHeadWords + (int64_t)col * 64 +
           (threadIdx.x & 63);
  if (k == 0) {
    // nothing enters but h: the tile's end is a state
    if (wave == 0) publish(p.at(0), kCut, after(TA, TH, h));
    return;
  }
  if (wave == 0) publish(p.at(k), TA, TH);
  const int g = k / a.group, in = k % a.group;
  float A = 1.f, H = 0.f, PA, PH;
  // the tiles of its group before it, a share to each wave
  const int share = (in + W - 1) / W;
  const int g0 = g * a.group;
  fold_entries(p, g0 + min(wave * share, in), g0 + min((wave + 1) * share, in),
               A, H);
  join_waves(sh, wave, A, H, PA, PH);
  if (in == a.group - 1 && wave == 0 && k < a.tiles - 1) {
    // the last of its group publishes the group
    A = PA;
    H = PH;
    then(A, H, TA, TH);
    keep_product(A, is_zero(PA) || is_zero(TA));
    publish(p.at((int64_t)a.tiles + g), A, H);
  }
  // the groups before its own
  A = 1.f;
  H = 0.f;
  const int gs = (g + W - 1) / W;
  fold_entries(p, a.tiles + min(wave * gs, g),
               a.tiles + min((wave + 1) * gs, g), A, H);
  float GA, GH;
  join_waves(sh, wave, A, H, GA, GH);
  then(GA, GH, PA, PH);
  h = GH;
}

// The state before a row's first tile, arrived in all waves of that tile before
// their first barrier: behind it the tile publishes, and the last tile may
// write the state's place.
__device__ __forceinline__ void arrived(float& h) {
  asm volatile("" : "+v"(h));
}

struct LaneAt {
  int b, ch;
  bool on;          // otherwise a copy of the last lane that stores nothing
  int64_t hc;
};
__device__ __forceinline__ LaneAt lane_at(const ScanArgs& a, int col) {
  int64_t lane = (int64_t)col * 64 + (threadIdx.x & 63);
  LaneAt l;
  l.on = lane < a.lanes;
  if (!l.on) lane = a.lanes - 1;
  l.b = (int)(lane / a.cv);
  l.ch = (int)(lane % a.cv);
  l.hc = (int64_t)l.b * a.q.c + l.ch;
  return l;
}
template <int W>
__device__ __forceinline__ int next_ticket(const ScanArgs& a,
                                           TileShared<W>& sh) {
  if (a.tiles == 1) return blockIdx.x;
  if (threadIdx.x == 0)
    sh.ticket = (int)__hip_atomic_fetch_add((unsigned*)a.ends, 1u,
                                            __ATOMIC_RELAXED,
                                            __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(sh.ticket);
}
// N steps of a tensor from step s0 on; for those that the row does not have,
// whatever it has last, or zero if it has none of them: behind its length a row
// is not read, and need not be there.  whole: all lanes of the wave have all.
template <int N, bool NARROW, typename T, int V>
__device__ __forceinline__ void load_steps(const SeqTensor& x,
                                           const ScanArgs& a, const Row& r,
                                           int b, int ch, int s0, bool whole,
                                           Pack<T, V>* out) {
  StepsAt<const T, NARROW> p(x, a.q, r, b, ch, s0);
  if (!whole) {
    if (s0 < r.len) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        out[k] = load_pack<T, V>(p.here());
        p.next(k);
        // (keeps these loads apart from those below: the compiler would form
        // all addresses in registers first and load in one place)
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) out[k] = Pack<T, V>{};
    }
  } else if (a.stream) {
#pragma unroll
    for (int k = 0; k < N; ++k) out[k] = stream_pack<T, V>(p.at(k));
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) out[k] = load_pack<T, V>(p.at(k));
  }
}
// Bit k: a reset before step s0 + k.
template <int N, bool NARROW>
__device__ __forceinline__ unsigned cuts_of(const ScanArgs& a, const Row& r,
                                            int b, int s0) {
  unsigned m = 0;
  if (a.q.reset && s0 < r.len) {
    // all loads at once: none waits for another
    const SeqTensor t{(void*)a.q.reset, a.q.b, 1};
    StepsAt<const uint8_t, NARROW> p(t, a.q, r, b, 0, s0);
    uint8_t x[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      x[k] = *p.here();
      p.next(k);
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (s0 + k < r.len && x[k]) m |= 1u << k;
  }
  return m;
}

// Launches (defined beside their kernels).  Rows split along time: blocks of
// kWaves (backward: kGradWaves) waves, one channel to a lane.  36001 steps of
// 512 channels bf16, forward: 54 us; 40% more with 4 waves, the same with 16
// (shorter rows lose 6%: 300 steps of 30 rows of 1023 channels); two channels
// to a lane and half the steps 17% more.  Backward, 4099 steps of 8 rows: 77;
// 12% more with 8 waves (a block's registers leave no room for a second beside
// it).
constexpr int kWaves = 8, kGradWaves = 4;
// Calls f(gated, narrow).
template <class F>
void with_scan_kind(const ScanArgs& a, F&& f) {
  auto go = [&](auto gt) {
    if (a.narrow)
      f(gt, std::true_type{});
    else
      f(gt, std::false_type{});
  };
  if (a.o.p)
    go(std::true_type{});
  else
    go(std::false_type{});
}
void launch_scan(const ScanArgs& a, int dtype, int out_dtype, int vec,
                 bool split, hipStream_t q);
void launch_scan_backward(const ScanArgs& a, int dtype, int out_dtype,
                          bool split, hipStream_t q);

}  // namespace ops
}  // namespace st
