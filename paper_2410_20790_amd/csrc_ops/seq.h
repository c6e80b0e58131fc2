// What the sequence operators share: a row's steps, the cut of channels into
// vectors, and the host's checks.
#pragma once

#include <algorithm>
#include <initializer_list>

#include "ops_common.h"

namespace st {
namespace ops {

// The axes on the device.
struct SeqAxes {
  int t, b, c;
  int reverse;
  const int* lengths;
  const uint8_t* reset;
};
// A tensor [t][b][c] on the device.
struct SeqTensor {
  void* p;
  int64_t st, sb;
};

// One row: its length, and the time of a running step.
struct Row {
  int len;
  int64_t t0;   // time of step 0
  int dir;
};
__device__ __forceinline__ Row row_of(const SeqAxes& q, int b) {
  Row r;
  r.len = q.t;
  if (q.lengths) r.len = max(0, min(q.lengths[b], q.t));
  r.dir = q.reverse ? -1 : 1;
  r.t0 = q.reverse ? r.len - 1 : 0;
  return r;
}
__device__ __forceinline__ int64_t time_of(const Row& r, int s) {
  return r.t0 + (int64_t)r.dir * s;
}
__device__ __forceinline__ bool reset_at(const SeqAxes& q, const Row& r,
                                         int b, int s) {
  return q.reset && q.reset[time_of(r, s) * q.b + b] != 0;
}

// A row's elements in running order, from step s0 on: next() goes to the next
// step, or stays where the row ends.  One addition per step; the products that
// a time and its stride make up are formed once.  NARROW: offsets of 32 bits
// into the tensor.
template <typename T, bool NARROW>
struct Walk {
  typedef std::conditional_t<NARROW, uint32_t, int64_t> Off;
  char* p;
  Off off, step;
  int left;    // steps that may follow
  __device__ __forceinline__ Walk(const SeqTensor& x, const Row& r, int b,
                                  int ch, int s0) {
    const int last = max(r.len - 1, 0), s = min(s0, last);
    const int64_t t = r.len > 0 ? time_of(r, s) : 0, es = sizeof(T);
    p = (char*)x.p;
    off = (Off)((t * x.st + (int64_t)b * x.sb + ch) * es);
    step = (Off)(r.dir * x.st * es);
    left = last - s;
  }
  __device__ __forceinline__ T* here() const {
    Off o = off;
    // (added to the address here, as the instruction does by itself)
    if constexpr (NARROW) asm volatile("" : "+v"(o));
    return (T*)(p + o);
  }
  __device__ __forceinline__ void next() {
    off += left > 0 ? step : 0;
    --left;
  }
};

// Running steps s0, s0 + 1, ... of a row: a scalar address that moves by steps
// and one offset per lane (NARROW: of 32 bits), so that the addresses of many
// loads in flight take no vector registers.  Times differ from lane to lane
// only where rows of their own lengths run backwards; there the offset holds
// the row's time.  Offsets never fall below zero: rows that run backwards begin
// kAheadSteps steps into theirs.
constexpr int kAheadSteps = ST_SCAN_STRIDE;   // steps of one of these, at most
template <typename T, bool NARROW>
struct StepsAt {
  typedef std::conditional_t<NARROW, uint32_t, int64_t> Off;
  char* p;
  int64_t step;
  Off off;
  int left;      // steps that the row has after s0
  __device__ __forceinline__ StepsAt(const SeqTensor& x, const SeqAxes& q,
                                     const Row& r, int b, int ch, int s0) {
    const int64_t es = sizeof(T);
    left = max(r.len - 1 - s0, 0);
    int64_t at = (int64_t)b * x.sb + ch, t = s0;
    if (q.reverse) {
      t = q.t - 1 - s0;
      if (q.lengths) {
        t = 0;
        at += left * x.st;
      } else {
        t -= kAheadSteps;
        at += kAheadSteps * x.st;
      }
    }
    p = (char*)x.p + t * x.st * es;
    step = q.reverse ? -x.st * es : x.st * es;
    off = (Off)(at * es);
    // (formed anew wherever it is used: across blocks the compiler would keep
    // it added to the address, two registers for every load in flight.  Walked
    // rows form one in each branch for that: above the branch, 300 steps of 600
    // rows of 512 channels bf16 take 186 us for 166)
    if constexpr (NARROW) asm volatile("" : "+v"(off));
  }
  // Step s0 + k, which the row must have.
  __device__ __forceinline__ T* at(int k) const {
    return (T*)(p + k * step + off);
  }
  // The same one by one, of a row that has step s0: on to the next step, or to
  // where the row ends.
  __device__ __forceinline__ T* here() const { return (T*)(p + off); }
  __device__ __forceinline__ void next(int k) {     // from step s0 + k
    off += k < left ? (Off)step : 0;
  }
};

// -------------------------------------------------------------- host side

// Whether offsets into `times` times of a tensor fit 32 bits.
inline bool narrow(const st_seq_desc& d, const st_seq_ref* r, int es,
                   int64_t times) {
  return !r || ((d.b - 1) * r->stride_b + times * r->stride_t + d.c) * es <
                   (int64_t)1 << 31;
}
// The times that StepsAt reaches over: all of them where rows of their own
// lengths run backwards.
inline int64_t steps_reach(const st_seq_desc& d) {
  return d.lengths && d.reverse ? d.t : kAheadSteps;
}
inline SeqAxes axes_of(const st_seq_desc& d) {
  return SeqAxes{d.t, d.b, d.c, d.reverse != 0, d.lengths, d.reset};
}
inline SeqTensor tensor_of(const st_seq_ref* r) {
  return r ? SeqTensor{r->data, r->stride_t, r->stride_b}
           : SeqTensor{nullptr, 0, 0};
}
inline bool empty(const st_seq_desc& d) { return d.t == 0 || d.b == 0; }

inline st_status check_seq(const st_seq_desc* d) {
  if (!d) return bad("descriptor is NULL");
  if (!dtypes_known(d->dtype, d->out_dtype))
    return bad("unknown data types, or a pair that is not offered");
  if (d->t < 0 || d->b < 0 || d->c < 1)
    return bad("t and b must not be negative, c must be positive");
  if (d->t > 1 << 30) return bad("t must not lie above 2^30");
  if ((int64_t)d->b * d->c >= (int64_t)1 << 31)
    return bad("b * c must lie below 2^31");
  if (!aligned(d->lengths, 4)) return bad("lengths is misaligned");
  return ST_OK;
}
// Float arrays and tensors of `es` bytes that may be absent.
inline st_status check_addresses(std::initializer_list<const void*> floats,
                                 std::initializer_list<const void*> others,
                                 int es) {
  for (const void* p : floats)
    if (!aligned(p, 4)) return bad("an array of floats is misaligned");
  for (const void* p : others)
    if (!aligned(p, es)) return bad("a window is misaligned");
  return ST_OK;
}
inline st_status check_ref(const st_seq_desc& d, const st_seq_ref* r,
                           int es, bool out, const char* name) {
  if (!r || (!r->data && !empty(d)))
    return bad(std::string(name) + " is NULL");
  if (!aligned(r->data, es)) return bad(std::string(name) + " is misaligned");
  if (r->stride_t < 0 || r->stride_b < 0)
    return bad(std::string(name) + " has a negative stride");
  if (out && !empty(d)) {
    const bool ts = d.t > 1, bs = d.b > 1;
    const int64_t a = ts ? r->stride_t : 0, b = bs ? r->stride_b : 0;
    bool ok = (!ts || a >= d.c) && (!bs || b >= d.c);
    if (ts && bs)
      ok = ok && (a <= b ? b >= a * (d.t - 1) + d.c
                         : a >= b * (d.b - 1) + d.c);
    if (!ok) return bad(std::string(name) + ": an output's elements overlap");
  }
  return ST_OK;
}
inline Span ref_span(const st_seq_desc& d, const st_seq_ref* r, int es) {
  if (!r || !r->data || empty(d)) return Span{};
  return span_of(r->data, ((d.t - 1) * r->stride_t + (d.b - 1) * r->stride_b +
                           d.c) * es);
}
// Two tensors of one type whose spans cross but whose elements do not: equal
// strides, and channels side by side (slices of one wider tensor, whose outer
// axis steps over the inner one whole).
inline bool side_by_side(const st_seq_desc& d, const st_seq_ref& a,
                         const st_seq_ref& b, int es) {
  if ((d.t > 1 && a.stride_t != b.stride_t) ||
      (d.b > 1 && a.stride_b != b.stride_b))
    return false;
  if (d.t > 1 && d.b > 1 &&
      (a.stride_t <= a.stride_b ? a.stride_b < a.stride_t * d.t
                                : a.stride_t < a.stride_b * d.b))
    return false;
  const int64_t bytes = std::abs((const char*)a.data - (const char*)b.data);
  int64_t room = INT64_MAX;   // the narrowest step of the two axes
  if (d.t > 1) room = std::min(room, a.stride_t);
  if (d.b > 1) room = std::min(room, a.stride_b);
  return bytes >= (int64_t)d.c * es &&
         (room == INT64_MAX || bytes <= (room - d.c) * es);
}
inline bool any_hit(std::initializer_list<Span> out,
                    std::initializer_list<Span> in) {
  for (const Span& o : out)
    for (const Span& i : in)
      if (o.hits(i)) return true;
  for (const Span* a = out.begin(); a != out.end(); ++a)
    for (const Span* b = out.begin(); b != a; ++b)
      if (a->hits(*b)) return true;
  return false;
}
inline st_status check_ws(uint64_t need, const void* ws, uint64_t ws_bytes) {
  if (need && !ws) return bad("workspace is NULL");
  if ((uintptr_t)ws % kAlign) return bad("workspace must be 256-byte aligned");
  if (ws_bytes < need)
    return fail(nullptr, ST_ERR_WORKSPACE, "workspace too small");
  return ST_OK;
}

inline bool vec_ok(int v, int es, const st_seq_desc& d, const st_seq_ref* r) {
  return !r || !r->data ||
         vec_ok(v, es, r->data, d.t > 1 ? r->stride_t : 0,
                d.b > 1 ? r->stride_b : 0);
}

}  // namespace ops
}  // namespace st
