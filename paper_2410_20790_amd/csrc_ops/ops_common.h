// What the operators behind the encoder share: vectors of adjacent channels,
// gates, and the host's checks of their arguments.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <exception>
#include <string>
#include <type_traits>

#include "../../include/sparsetem.h"
#include "../csrc/st_device.h"
#include "../csrc/st_internal.h"

namespace st {
namespace ops {

// ------------------------------------------------------------ device side

// V adjacent elements, loaded and stored at once (V * sizeof(T) <= 16 bytes,
// the address aligned to that).
template <typename T, int V>
struct alignas(sizeof(T) * V) Pack {
  T e[V];
};
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T* p) {
  return *(const Pack<T, V>*)p;
}
// The same past the caches' reuse order: for data that is streamed through
// once.  Whole lines only (a store of part of one costs a read of the rest).
template <int N> struct Bits;
template <> struct Bits<2> { typedef uint16_t type; };
template <> struct Bits<4> { typedef uint32_t type; };
template <> struct Bits<8> {
  typedef uint32_t type __attribute__((ext_vector_type(2)));
};
template <> struct Bits<16> {
  typedef uint32_t type __attribute__((ext_vector_type(4)));
};
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> stream_pack(const T* p) {
  typedef typename Bits<sizeof(T) * V>::type B;
  const B b = __builtin_nontemporal_load((const B*)p);
  return __builtin_bit_cast(Pack<T, V>, b);
}
template <typename T, int V>
__device__ __forceinline__ void stream_out(T* p, const float* f) {
  typedef typename Bits<sizeof(T) * V>::type B;
  Pack<T, V> r;
#pragma unroll
  for (int i = 0; i < V; ++i) r.e[i] = from_f<T>(f[i]);
  __builtin_nontemporal_store(__builtin_bit_cast(B, r), (B*)p);
}
template <typename T, int V>
__device__ __forceinline__ void unpack(const Pack<T, V>& p, float* f) {
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = to_f(p.e[i]);
}
template <typename T, int V>
__device__ __forceinline__ void store_pack(T* p, const float* f) {
  Pack<T, V> r;
#pragma unroll
  for (int i = 0; i < V; ++i) r.e[i] = from_f<T>(f[i]);
  *(Pack<T, V>*)p = r;
}

// e^x for x <= 0, to about an ulp: 2^(x log2 e) with the product's rounding
// error and the constant's tail brought back.  (Below -104 the result is zero;
// -inf would make the correction NaN.)
__device__ __forceinline__ float exp_nonpos(float x) {
  const float hi = 1.44269502162933349609f, lo = 1.92596299e-8f;
  x = x < -104.f ? -104.f : x;   // NaN stays
  const float t = x * hi;
  const float r = __builtin_fmaf(x, lo, __builtin_fmaf(x, hi, -t));
  const float e = __builtin_amdgcn_exp2f(t);
  return __builtin_fmaf(e * r, 0.693147180559945f, e);
}
// 1 / d for 1 <= d <= 2: the hardware's estimate and one Newton step.
__device__ __forceinline__ float rcp_1to2(float d) {
  const float r = __builtin_amdgcn_rcpf(d);
  return __builtin_fmaf(__builtin_fmaf(-d, r, 1.f), r, r);
}
// sigmoid(x) and sigmoid(-x), both to full relative accuracy: neither is
// formed as one minus the other, so that a gate that holds for 10^8 steps
// still lets its 10^-8 in.
__device__ __forceinline__ void sigmoids(float x, float& pos, float& neg) {
  const float e = exp_nonpos(-__builtin_fabsf(x));
  const float big = rcp_1to2(1.f + e), small = e * big;
  pos = x >= 0.f ? big : small;
  neg = x >= 0.f ? small : big;
}

// sigmoid(x) where it scales a value once: off by some (4 + 1.25 |x|) 2^-24 of
// itself, which is 5 * 2^-24 at most (the exponent's rounding, the exponential,
// the reciprocal), at half the instructions.  For f32 results too: there the
// full accuracy of sigmoids() takes 1 to 3% more of the convolution and the
// recurrence, and of norms held in registers 5 to 17% (32x64x512 in 32 groups,
// one image 12.9 us for 11.0, nine 29.8 for 26.5).
__device__ __forceinline__ float sigmoid_once(float x) {
  const float e = __builtin_amdgcn_exp2f(x * -1.44269502162933349609f);
  return __builtin_amdgcn_rcpf(1.f + e);
}

// sigmoid(x) and sigmoid(-x) likewise.  (n as e p rather than 1 - p, whose
// error a large factor would magnify; beyond 2^126, where p is no normal number
// any more, every result is zero.)
__device__ __forceinline__ void sigmoids_once(float x, float& p, float& n) {
  const float e = __builtin_amdgcn_exp2f(x * -1.44269502162933349609f);
  p = __builtin_amdgcn_rcpf(1.f + e);
  n = fminf(e, 0x1p126f) * p;
}

// f(z) and its derivative for the activation ACT (ST_ACT_*).
template <int ACT>
__device__ __forceinline__ float act_fwd(float z) {
  if constexpr (ACT == ST_ACT_RELU)
    return z < 0.f ? 0.f : z;  // NaN stays
  else if constexpr (ACT == ST_ACT_SILU)
    return z * sigmoid_once(z);
  else
    return z;
}
template <int ACT>
__device__ __forceinline__ float act_grad(float z) {
  if constexpr (ACT == ST_ACT_RELU) {
    return z > 0.f ? 1.f : 0.f;
  } else if constexpr (ACT == ST_ACT_SILU) {
    float p, n;
    sigmoids_once(z, p, n);
    return p * __builtin_fmaf(z, n, 1.f);
  } else {
    return 1.f;
  }
}

// Calls f(std::integral_constant<int, ACT>{}) for the activation act.
template <class F>
__device__ __forceinline__ void with_activation_of(int act, F&& f) {
  if (act == ST_ACT_RELU)
    f(std::integral_constant<int, ST_ACT_RELU>{});
  else if (act == ST_ACT_SILU)
    f(std::integral_constant<int, ST_ACT_SILU>{});
  else
    f(std::integral_constant<int, ST_ACT_NONE>{});
}

// -------------------------------------------------------------- host side

inline bool act_known(int32_t a) { return a >= ST_ACT_NONE && a <= ST_ACT_SILU; }
inline bool dtypes_known(int32_t in, int32_t out) {
  const bool ok = in == ST_F32 || in == ST_F16 || in == ST_BF16;
  const bool ok_out = out == ST_F32 || out == ST_F16 || out == ST_BF16;
  return ok && ok_out && (in == out || in == ST_F32);
}
inline int esize(int32_t dt) { return dt == ST_F32 ? 4 : 2; }

inline st_status bad(const std::string& msg) {
  return fail(nullptr, ST_ERR_INVALID_ARG, msg);
}

// Runs a call's body; no exception leaves it.
template <class F>
st_status guarded(F&& body) noexcept {
  try {
    return body();
  } catch (const std::exception&) {
    // (a message this short takes no memory)
    return fail(nullptr, ST_ERR_HIP, "no host memory");
  }
}

inline st_status launch_status(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return ST_OK;
  return fail(nullptr, ST_ERR_HIP,
              std::string(what) + ": " + hipGetErrorString(e));
}

// The bytes a call may touch behind a pointer, for the overlap checks.
struct Span {
  const char* lo = nullptr;
  const char* hi = nullptr;
  bool hits(const Span& o) const {
    return lo != hi && o.lo != o.hi && lo < o.hi && o.lo < hi;
  }
};
inline Span span_of(const void* p, int64_t bytes) {
  return p ? Span{(const char*)p, (const char*)p + bytes} : Span{};
}

// Whether an address that may be absent is one of elements of `es` bytes.
inline bool aligned(const void* p, int es) { return (uintptr_t)p % es == 0; }

// Calls f(type tags) for a known pair of data types.
template <typename T> struct Tag { using type = T; };
template <class F>
void with_types(int32_t in, int32_t out, F&& f) {
  if (in == ST_F16)
    f(Tag<_Float16>{}, Tag<_Float16>{});
  else if (in == ST_BF16)
    f(Tag<bf16_t>{}, Tag<bf16_t>{});
  else if (out == ST_F32)
    f(Tag<float>{}, Tag<float>{});
  else if (out == ST_F16)
    f(Tag<float>{}, Tag<_Float16>{});
  else
    f(Tag<float>{}, Tag<bf16_t>{});
}
template <int I> using Int = std::integral_constant<int, I>;
template <class F>
void with_activation(int32_t act, F&& f) {
  if (act == ST_ACT_RELU)
    f(Int<ST_ACT_RELU>{});
  else if (act == ST_ACT_SILU)
    f(Int<ST_ACT_SILU>{});
  else
    f(Int<ST_ACT_NONE>{});
}

// Whether V elements of every listed size may be moved at once: address and
// strides are multiples of the vector.
inline bool vec_ok(int v, int es, const void* p, int64_t a, int64_t b,
                   int64_t c = 0) {
  return (uintptr_t)p % (uint64_t)(v * es) == 0 && a % v == 0 && b % v == 0 &&
         c % v == 0;
}

}  // namespace ops
}  // namespace st
