// Attention of new tokens over a sequence's first tokens and a sliding window: kvd_sink_attn
// (K/V of the shape's dtype) and kvd_mx_attn (a 4-bit cache).
//
//   sink_row_kernel    one query row per workgroup, keys to its 4 waves in turn.
//
// Scores are kept in the log2 domain; a row that sees no key gives 0.
#include <hip/hip_runtime.h>

#include "kvd_sink_device.hpp"

namespace kvd {

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// Elements E lane .. of row `row` of K or V: type T, or 4-bit numbers (scale not null).
template <typename T, int HD, bool MX>
__device__ __forceinline__ void sink_load(const void* base, const uint8_t* scale, size_t row, int lane,
                                          float (&x)[HD / 64]) {
  constexpr int E = HD / 64;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int c = E * lane + e;
    if constexpr (MX) {
      const uint32_t b = static_cast<const uint8_t*>(base)[row * (HD / 2) + (c >> 1)];
      const uint32_t v = mx_bf16x2<0>(b, mx_scale(scale[row * (HD / kMxGroup) + c / kMxGroup]));
      x[e] = c & 1 ? bf_hi(v) : bf_lo(v);
    } else if constexpr (sizeof(T) == 2) {
      x[e] = bf_lo(static_cast<const uint16_t*>(base)[row * HD + c]);
    } else {
      x[e] = static_cast<const float*>(base)[row * HD + c];
    }
  }
}

// One workgroup per query row (b, i, h).  A wave's keys: x = w, w + 4, ..; the lanes hold a
// key's elements between them.  Bound by the latency of a key's loads and the sum over the wave.
template <typename T, int HD, bool MX>
__global__ __launch_bounds__(256) void sink_row_kernel(SinkArgs a) {
  constexpr int E = HD / 64;
  __shared__ float part[4][HD], ml[4][2];
  const int lane = threadIdx.x & 63, w = wave_id();
  const int row = (int)blockIdx.x, h = row % a.n_q, bi = row / a.n_q, i = bi % a.N, b = bi / a.N;
  const int j = h / a.g;
  const SinkSeq sq = sink_seq(a.kv_len, a.n_new, a.T, a.N, b);
  if (i >= sq.n) return;
  const int p = sq.len - sq.n + i;
  const SinkKeys keys = sink_keys(a, p, p);
  const size_t base = ((size_t)b * a.n_kv + j) * a.t_cap + a.t_off;
  float q[E], o[E], m = -INFINITY, l = 0.0f;
  sink_load<T, HD, false>(a.q, nullptr, (size_t)row, lane, q);
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.0f;
  for (int x = w; x < keys.n; x += 4) {
    const size_t r = base + keys.row(x);
    float k[E], v[E], s = 0.0f;
    sink_load<T, HD, MX>(a.k, a.ks, r, lane, k);
    sink_load<T, HD, MX>(a.v, a.vs, r, lane, v);
#pragma unroll
    for (int e = 0; e < E; ++e) s = fmaf(q[e], k[e], s);
    s = wave_sum(s) * ScoreScale<HD>::v;
    const float m_new = fmaxf(m, s), mu = m_new == -INFINITY ? 0.0f : m_new;
    const float alpha = exp2_hw(m - mu), pw = exp2_hw(s - mu);
    m = m_new;
    l = fmaf(l, alpha, pw);
#pragma unroll
    for (int e = 0; e < E; ++e)
      o[e] = fabsf(o[e]) < INFINITY ? fabsf(v[e]) < INFINITY ? fmaf(pw, v[e], alpha * o[e]) : v[e] : o[e] + v[e] * 0.0f;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) part[w][E * lane + e] = o[e];
  if (lane == 0) {
    ml[w][0] = m;
    ml[w][1] = l;
  }
  __syncthreads();
  if (threadIdx.x >= HD) return;
  float M = -INFINITY, L = 0.0f, y = 0.0f;
  for (int v = 0; v < 4; ++v) M = fmaxf(M, ml[v][0]);
  const float Mu = M == -INFINITY ? 0.0f : M;
  for (int v = 0; v < 4; ++v) {
    const float wt = exp2_hw(ml[v][0] - Mu), z = part[v][threadIdx.x];
    L = fmaf(wt, ml[v][1], L);
    y = fabsf(z) < INFINITY ? fmaf(wt, z, y) : y + z;
  }
  y = L != 0.0f ? y / L : 0.0f;
  if constexpr (sizeof(T) == 2)
    static_cast<uint16_t*>(a.out)[(size_t)row * HD + threadIdx.x] = (uint16_t)pack_bf16x2(y, y);
  else
    static_cast<float*>(a.out)[(size_t)row * HD + threadIdx.x] = y;
}

template <typename T, int HD>
static hipError_t launch_sink_t(const SinkArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((long long)a.B * a.N * a.n_q));
  if (a.ks != nullptr)
    hipLaunchKernelGGL((sink_row_kernel<T, HD, true>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((sink_row_kernel<T, HD, false>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_sink(const SinkArgs& a, int dtype_bf16, int hd, hipStream_t st) {
  switch (hd) {
    case 64: return dtype_bf16 ? launch_sink_t<uint16_t, 64>(a, st) : launch_sink_t<float, 64>(a, st);
    case 128: return dtype_bf16 ? launch_sink_t<uint16_t, 128>(a, st) : launch_sink_t<float, 128>(a, st);
    case 256: return dtype_bf16 ? launch_sink_t<uint16_t, 256>(a, st) : launch_sink_t<float, 256>(a, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace kvd
