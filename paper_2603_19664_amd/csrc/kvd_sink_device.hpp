// What kvd_sink.hip and kvd_mx.hip share: which keys of a cache a block of query rows sees
// and where they lie, and the 4-bit numbers.
#pragma once

#include "kvd_device.hpp"
#include "kvd_launch.h"

namespace kvd {

// What sequence b brings: tokens len, the last n of them new (both clamped to the call's sizes).
struct SinkSeq {
  int len, n;
};
__device__ __forceinline__ SinkSeq sink_seq(const int32_t* kv_len, const int32_t* n_new, int T, int N, int b) {
  SinkSeq s;
  s.len = kv_len != nullptr ? min(max(kv_len[b], 0), T) : T;
  s.n = n_new != nullptr ? min(max(n_new[b], 0), N) : N;
  return s;
}

// Row of token t (counted from the view's t_off): a cache that holds every token (ring 0) keeps it in
// row t, others below sink, and behind that in a ring.
__device__ __forceinline__ int sink_row(int t, int sink, int ring) {
  return ring == 0 || t < sink ? t : sink + (t - sink) % ring;
}

// The keys that the new tokens at positions p0 .. p1 see between them, in order: x = 0 .. n - 1
// are tokens 0 .. ns - 1 (sinks before the first one's window), then the tokens from w0 on to p1.
// The row of x is x + d behind the sinks, less ring from row cap on (at most once: a ring holds
// the windows of all new tokens).
struct SinkKeys {
  int n, ns, skip, d, cap, ring;  // skip: tokens left out before w0
  __device__ __forceinline__ int row(int x) const {
    const int y = x < ns ? x : x + d;
    return y < cap ? y : y - ring;
  }
};
__device__ __forceinline__ SinkKeys sink_keys(const SinkArgs& a, int p0, int p1) {
  SinkKeys k;
  const int w0 = max(max(p0, -1) - a.window + 1, 0);  // window <= T
  k.ns = min(a.sink, w0);
  k.skip = w0 - k.ns;
  k.n = p1 < 0 ? 0 : p1 + 1 - k.skip;
  k.d = sink_row(w0, a.sink, a.ring) - k.ns;
  k.cap = a.cap;
  k.ring = a.ring;
  return k;
}
// Of those, the token at position p sees x < hi with x < sink or x >= lo.
struct SinkRow {
  int lo, hi;
};
__device__ __forceinline__ SinkRow sink_row_of(const SinkArgs& a, const SinkKeys& k, int p) {
  p = max(p, -1);
  return SinkRow{p - a.window + 1 - k.skip, p + 1 - k.skip};
}

// 4-bit numbers: a sign and 0, 1/2, 1, 3/2, 2, 3, 4, 6, times a power of two that 32 neighbours
// share, held as its fp32 exponent in a byte (255: all 32 are NaN).  bf16 holds their values
// exactly, and the conversions below are single instructions: elements 2 SEL and 2 SEL + 1 of a
// word's eight.
__device__ __forceinline__ float mx_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
template <int SEL>
__device__ __forceinline__ uint32_t mx_bf16x2(uint32_t word, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, SEL));
}

}  // namespace kvd
