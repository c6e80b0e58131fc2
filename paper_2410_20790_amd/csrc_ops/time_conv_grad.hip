// Gradients of the causal depthwise convolution along time.
//
//   dz_s = dy_s act'(z_s)
//   dx_p = sum_d w_{K-1-d} dz_{p+d}      (no reset in p < s <= p + d)
//   dw_j = sum_s dz_s x_{s-K+1+j},  db = sum_s dz_s
//
// About 6 K operations per element moved: bound by memory.  A thread walks a
// tile of steps as the forward kernel does, computes z again from the inputs
// in its registers, and carries the K unfinished dx beside them; it runs K - 1
// steps past its tile for its last dx.  The parameters' sums stay in its
// registers over all its tiles, are joined in the block and leave as one part
// per block, which a second launch sums in f64 in a fixed order.
#include "time_conv.h"

namespace st {
namespace ops {
namespace {

constexpr int kAhead = 4;
// PLAIN: no resets, and steps inside a tile have a path of their own that tests
// for nothing.  It takes a quarter more registers: for tiles (or rows) of some
// length, and as many channels and taps as still leave four waves to a SIMD.
// us, with and without: 601 steps of 48 rows of 512 channels f16, 4 taps 34 and
// 38; 300 steps of 30 rows of 1023 channels, 5 taps 28 and 33; 9 steps of 2048
// rows of 512 channels f32 45 and 39; 64 steps of 512 rows of 256 channels, 8
// taps 40 and 37.
constexpr int kPlainSteps = 16, kPlainTaps = 10;   // taps times channels

template <typename T, typename O, int V, int K, bool NARROW, bool PLAIN>
__global__ __launch_bounds__(kConvThreads) void k_time_conv_grad(
    ConvTimeArgs a) {
  const int col = threadIdx.x % a.cols, row = threadIdx.x / a.cols;
  const int cb = blockIdx.x % a.colblocks, by = blockIdx.x / a.colblocks;
  const int vec = cb * a.cols + col;
  const bool active = row < a.rows && vec < a.cv;
  const int ch = active ? vec * V : 0;
  float w[K][V], bias[V], dw[K][V], db[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    bias[e] = a.bias ? a.bias[ch + e] : 0.f;
    db[e] = 0.f;
#pragma unroll
    for (int j = 0; j < K; ++j) {
      w[j][e] = a.weight[(int64_t)j * a.q.c + ch + e];
      dw[j][e] = 0.f;
    }
  }
  const int64_t units = active ? (int64_t)a.tiles * a.q.b : 0;
  const int64_t step = (int64_t)a.gridy * a.rows;
  for (int64_t u = (int64_t)by * a.rows + row; u < units; u += step) {
    const int b = (int)(u % a.q.b);
    const int tile = (int)(u / a.q.b);
    const Row r = row_of(a.q, b);
    const int s0 = tile * a.tile, s1 = min(s0 + a.tile, a.q.t);
    const int own = min(s1, r.len);             // steps [s0, own) are its own
    const int end = min(s1 + K - 1, r.len);     // steps it needs dz of
    const int first = tile == 0 ? -(K - 1) : s0;  // positions [first, own)
    const int cut_end = a.dwindow_out ? last_cut<K>(a, r, b) : 0;
    float win[K > 1 ? K - 1 : 1][V];
    float acc[K][V];                            // dx of s - K + 1 .. s
#pragma unroll
    for (int i = 0; i < K; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) acc[i][e] = 0.f;
    // the finished dx of position p (in rising order)
    Walk<T, NARROW> dx(a.dx, r, b, ch, s0);
    auto put = [&](int p, float* v) {
      if (p < first || p >= own) return;
      const int i = p - (r.len - (K - 1));      // its place in window_out
      if (K > 1 && i >= 0 && a.dwindow_out && p >= cut_end) {
        float g[V];
        unpack<T, V>(load_pack<T, V>((const T*)a.dwindow_out +
                                     ((int64_t)i * a.q.b + b) * a.q.c + ch),
                     g);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] += g[e];
      }
      if (p >= 0) {
        if (a.dx.p) store_pack<T, V>(dx.here(), v);
        dx.next();
      } else if (a.dwindow) {
        store_pack<T, V>((T*)a.dwindow +
                             ((int64_t)(K - 1 + p) * a.q.b + b) * a.q.c + ch,
                         v);
      }
    };
    if (s0 < own || (tile == 0 && K > 1)) {
      int open = K;    // taps back that no reset hides
      if (s0 < own) load_window<T, V, K>(a, r, b, ch, s0, win);
      int s = s0;
      Walk<const T, NARROW> x(a.x, r, b, ch, s0);
      Walk<const O, NARROW> dy(a.dy, r, b, ch, s0);
      // the next steps' loads are in flight while these are worked on
      Pack<T, V> xn[kAhead];
      Pack<O, V> dn[kAhead];
      auto fetch = [&] {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          xn[k] = load_pack<T, V>(x.here());
          dn[k] = load_pack<O, V>(dy.here());
          x.next();
          dy.next();
        }
      };
      if (s < end) fetch();
      for (; s < end; s += kAhead) {
        Pack<T, V> xi[kAhead];
        Pack<O, V> di[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          xi[k] = xn[k];
          di[k] = dn[k];
        }
        if (s + kAhead < end) fetch();
        auto step = [&](int k, auto pt) __attribute__((always_inline)) {
          constexpr bool P = decltype(pt)::value;
          float f[V], d[V], out[V];
          unpack<T, V>(xi[k], f);
          unpack<O, V>(di[k], d);
          if (!PLAIN && reset_at(a.q, r, b, s + k)) {
            open = 0;
#pragma unroll
            for (int j = 0; j < K - 1; ++j)
#pragma unroll
              for (int e = 0; e < V; ++e) win[j][e] = 0.f;
          }
          const bool mine = P || s + k < s1;
#pragma unroll
          for (int e = 0; e < V; ++e) {
            if (a.act != ST_ACT_NONE) {
              float z = bias[e];
#pragma unroll
              for (int j = 0; j < K - 1; ++j)
                z = __builtin_fmaf(w[j][e], win[j][e], z);
              z = __builtin_fmaf(w[K - 1][e], f[e], z);
              d[e] *= act_grad_any(a.act, z);
            }
            const float m = mine ? d[e] : 0.f;
            db[e] += m;
#pragma unroll
            for (int j = 0; j < K - 1; ++j)
              dw[j][e] = __builtin_fmaf(m, win[j][e], dw[j][e]);
            dw[K - 1][e] = __builtin_fmaf(m, f[e], dw[K - 1][e]);
            // acc[j] is position s + k - (K - 1) + j, tap j
#pragma unroll
            for (int j = 0; j < K; ++j)
              if (PLAIN || K - 1 - j <= open)
                acc[j][e] = __builtin_fmaf(w[j][e], d[e], acc[j][e]);
            out[e] = acc[0][e];
#pragma unroll
            for (int j = 0; j + 1 < K; ++j) acc[j][e] = acc[j + 1][e];
            acc[K - 1][e] = 0.f;
#pragma unroll
            for (int j = 0; j + 1 < K - 1; ++j) win[j][e] = win[j + 1][e];
            if (K > 1) win[K > 1 ? K - 2 : 0][e] = f[e];
          }
          if constexpr (P) {
            if (a.dx.p) store_pack<T, V>(dx.here(), out);
            dx.next();
          } else {
            open = min(open + 1, K);
            put(s + k - (K - 1), out);
          }
        };
        if (PLAIN && __all(s >= s0 + K - 1 && s + kAhead <= own)) {
#pragma unroll
          for (int k = 0; k < kAhead; ++k) step(k, std::true_type{});
        } else {
#pragma unroll
          for (int k = 0; k < kAhead; ++k)
            if (s + k < end) step(k, std::false_type{});
        }
      }
      // positions that no further step reaches
      const int at = max(s0, end);
#pragma unroll
      for (int j = 0; j < K - 1; ++j) put(at - (K - 1) + j, acc[j]);
    }
    if (a.dx.p) {
      T* q = (T*)a.dx.p + (int64_t)b * a.dx.sb + ch;
      for (int s = max(s0, r.len); s < s1; ++s) {
        float z[V];
#pragma unroll
        for (int e = 0; e < V; ++e) z[e] = 0.f;
        store_pack<T, V>(q + (int64_t)s * a.dx.st, z);
      }
    }
  }
  if (!a.part) return;
  // join the block's rows, tap by tap
  __shared__ float red[kConvThreads * V];
#pragma unroll
  for (int j = 0; j <= K; ++j) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e)
      red[threadIdx.x * V + e] = !active ? 0.f : j < K ? dw[j < K ? j : 0][e]
                                                       : db[e];
    __syncthreads();
    for (int i = threadIdx.x; i < a.cols * V; i += kConvThreads) {
      const int c = cb * a.cols * V + i;
      if (c < a.q.c) {
        float s = 0.f;
        for (int k = 0; k < a.rows; ++k) s += red[k * a.cols * V + i];
        a.part[((int64_t)by * (K + 1) + j) * a.q.c + c] = s;
      }
    }
  }
}

// Sums the blocks' parts in f64: 16 channels by 16 lanes of parts in a block.
__global__ __launch_bounds__(256) void k_time_conv_join(ConvTimeArgs a,
                                                        int taps) {
  __shared__ double red[16][16];
  const int cx = threadIdx.x & 15, k = threadIdx.x >> 4;
  const int64_t total = (int64_t)(taps + 1) * a.q.c;
  for (int64_t i0 = blockIdx.x * 16ll; i0 < total; i0 += gridDim.x * 16ll) {
    const int64_t i = i0 + cx;
    double s = 0;
    if (i < total) {
#pragma unroll 8
      for (int p = k; p < a.gridy; p += 16) s += a.part[p * total + i];
    }
    __syncthreads();
    red[k][cx] = s;
    __syncthreads();
    if (k == 0 && i < total) {
      for (int p = 1; p < 16; ++p) s += red[p][cx];
      const int64_t j = i / a.q.c;
      if (j < taps) {
        if (a.dweight) a.dweight[i] = (float)s;
      } else if (a.dbias) {
        a.dbias[i - (int64_t)taps * a.q.c] = (float)s;
      }
    }
  }
}

}  // namespace

void launch_time_conv_backward(const ConvTimeArgs& a, int dtype,
                               int out_dtype, int taps, int vec,
                               hipStream_t stream) {
  const unsigned grid = (unsigned)(a.colblocks * a.gridy);
  if (grid)
    with_types(dtype, out_dtype, [&](auto ti, auto to) {
      using T = typename decltype(ti)::type;
      using O = typename decltype(to)::type;
      with_conv_vec(vec, [&](auto vt) {
        with_taps(taps, [&](auto kt) {
          constexpr int V = decltype(vt)::value, K = decltype(kt)::value;
          if constexpr (V <= 2) {
            constexpr bool fits = V * K <= kPlainTaps;
            if (!a.narrow)
              k_time_conv_grad<T, O, V, K, false, false>
                  <<<grid, kConvThreads, 0, stream>>>(a);
            else if (fits && !a.q.reset &&
                     std::min(a.tile, a.q.t) >= kPlainSteps)
              k_time_conv_grad<T, O, V, K, true, fits>
                  <<<grid, kConvThreads, 0, stream>>>(a);
            else
              k_time_conv_grad<T, O, V, K, true, false>
                  <<<grid, kConvThreads, 0, stream>>>(a);
          }
        });
      });
    });
  if (a.dweight || a.dbias) {
    const int64_t total = (int64_t)(taps + 1) * a.q.c;
    k_time_conv_join<<<(unsigned)std::min<int64_t>(ceil_div(total, 16), 4096),
                       256, 0, stream>>>(a, taps);
  }
}

}  // namespace ops
}  // namespace st
