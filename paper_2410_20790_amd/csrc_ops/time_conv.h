// The causal depthwise convolution along time: what its forward and backward
// kernels share.
#pragma once

#include "seq.h"

namespace st {
namespace ops {

constexpr int kConvThreads = 256;

struct ConvTimeArgs {
  SeqAxes q;
  SeqTensor x, y, dy, dx;
  const float* weight;   // [taps][c]
  const float* bias;
  const void* window;    // [taps - 1][b][c]
  void* window_out;
  const void* dwindow_out;
  void* dwindow;
  float* part;           // backward: [grid rows][taps + 1][c]
  float* dweight;
  float* dbias;
  int act;
  int cv;                // vectors per row of channels
  int cols, rows;        // vectors and units (row, time tile) of a block
  int colblocks;
  int tile, tiles;       // steps per unit, units per row
  int gridy;
  int narrow;            // 32-bit offsets (see Walk)
};

__device__ __forceinline__ float act_any(int act, float z) {
  if (act == ST_ACT_SILU) return act_fwd<ST_ACT_SILU>(z);
  if (act == ST_ACT_RELU) return act_fwd<ST_ACT_RELU>(z);
  return z;
}
__device__ __forceinline__ float act_grad_any(int act, float z) {
  if (act == ST_ACT_SILU) return act_grad<ST_ACT_SILU>(z);
  if (act == ST_ACT_RELU) return act_grad<ST_ACT_RELU>(z);
  return 1.f;
}

// The K - 1 inputs before step s0, oldest first, zero where a reset up to
// s0 - 1 hides them.
template <typename T, int V, int K>
__device__ __forceinline__ void load_window(const ConvTimeArgs& a,
                                            const Row& r, int b, int ch,
                                            int s0, float (*win)[V]) {
#pragma unroll
  for (int i = 0; i < K - 1; ++i) {
    const int p = s0 - (K - 1) + i;
#pragma unroll
    for (int e = 0; e < V; ++e) win[i][e] = 0.f;
    if (p >= 0) {
      if (p < r.len) {
        if (reset_at(a.q, r, b, p)) {
#pragma unroll
          for (int j = 0; j < i; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) win[j][e] = 0.f;
        }
        const T* x = (const T*)a.x.p + time_of(r, p) * a.x.st +
                     (int64_t)b * a.x.sb + ch;
        unpack<T, V>(load_pack<T, V>(x), win[i]);
      }
    } else if (a.window) {
      const T* w = (const T*)a.window +
                   ((int64_t)(K - 1 + p) * a.q.b + b) * a.q.c + ch;
      unpack<T, V>(load_pack<T, V>(w), win[i]);
    }
  }
}

// The last reset among a row's last K - 1 steps (below every position where
// there is none).
template <int K>
__device__ __forceinline__ int last_cut(const ConvTimeArgs& a, const Row& r,
                                        int b) {
  int cut = -K;
  for (int p = max(0, r.len - (K - 1)); p < r.len; ++p)
    if (reset_at(a.q, r, b, p)) cut = p;
  return cut;
}

template <class F>
void with_taps(int k, F&& f) {
  switch (k) {
    case 1: f(Int<1>{}); break;
    case 2: f(Int<2>{}); break;
    case 3: f(Int<3>{}); break;
    case 4: f(Int<4>{}); break;
    case 5: f(Int<5>{}); break;
    case 6: f(Int<6>{}); break;
    case 7: f(Int<7>{}); break;
    default: f(Int<8>{}); break;
  }
}
template <class F>
void with_conv_vec(int v, F&& f) {
  if (v == 4)
    f(Int<4>{});
  else if (v == 2)
    f(Int<2>{});
  else
    f(Int<1>{});
}

// Launches (defined beside their kernels).
void launch_time_conv(const ConvTimeArgs& a, int dtype, int out_dtype,
                      int taps, int vec, hipStream_t stream);
void launch_time_conv_backward(const ConvTimeArgs& a, int dtype,
                               int out_dtype, int taps, int vec,
                               hipStream_t stream);

}  // namespace ops
}  // namespace st
