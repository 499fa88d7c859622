// Rows of a 4-bit cache, written from K/V of the shape's dtype (kvd_mx_store) and read
// back (kvd_mx_load).
//
// 32 neighbouring elements of a row share 2^E, E the smallest with every |x| <= 7 2^E: the
// largest then rounds to at most 6, the largest number there is.  (Against N(0, 1) in bf16 the rms
// error is 0.1119 so; with E the exponent of the largest less 2, which clips up to 8 to 6, 0.1149, and with the
// largest at most 6, 0.1155.)  Powers of two make every step exact, so that a row has one
// 4-bit form, whatever computes it.
//
// HBM-bound: a thread takes 8 elements (16 or 32 bytes) of one row, the four of a group of 32
// find its largest between them.  (6503 rows of 4 heads of 256, K and V: 10 us to store, 9.6 to load, 3.4 to
// 3.5 TB/s; 32 rows of 2 heads of 128: 2.8 and 2.6 us, launch and round trip.)
#include <hip/hip_runtime.h>

#include "kvd_sink_device.hpp"

namespace kvd {

// What a thread works on: 8 elements (chunk c of hd / 8) of new token i of (b, j), in K or V.
struct MxItem {
  bool on;
  size_t plain, held;  // the row in the plain tensor and in the cache
  int c;
};
template <int HD>
__device__ __forceinline__ MxItem mx_item(const MxArgs& a) {
  constexpr uint32_t CPR = HD / 8;
  const uint32_t id = blockIdx.x * 256u + threadIdx.x;  // (a call has fewer than 2^31)
  MxItem it;
  it.c = (int)(id % CPR);
  const uint32_t row = id / CPR;  // (b n_kv + j) N + i
  const uint32_t bj = row / (uint32_t)a.N;
  const int i = (int)(row - bj * (uint32_t)a.N);
  it.on = bj < (uint32_t)a.B * (uint32_t)a.n_kv;
  if (!it.on) return it;
  const SinkSeq s = sink_seq(a.kv_len, a.n_new, a.T, a.N, (int)(bj / (uint32_t)a.n_kv));
  const int t = s.len - s.n + i;
  it.on = i < s.n && t >= 0;
  if (!it.on) return it;
  it.plain = (size_t)bj * a.p_cap + a.p_off + i;
  it.held = (size_t)bj * a.t_cap + a.t_off + sink_row(t, a.sink, a.ring);
  return it;
}

template <typename T, int HD>
__global__ __launch_bounds__(256) void mx_store_kernel(MxArgs a) {
  const MxItem it = mx_item<HD>(a);
  if (!it.on) return;  // the four threads of a group take the same row
  const bool is_v = blockIdx.y != 0;
  const T* src = static_cast<const T*>(is_v ? a.pv : a.pk) + it.plain * HD + 8 * it.c;
  uint32_t top = 0;  // the largest magnitude's bits: infinities and NaN above all numbers
  u32x4_t x[sizeof(T) / 2];
  if constexpr (sizeof(T) == 2) {
    x[0] = *reinterpret_cast<const u32x4_t*>(src);
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, max(x[0][e] << 16 & 0x7fff0000u, x[0][e] & 0x7fff0000u));
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      x[h] = *reinterpret_cast<const u32x4_t*>(src + 4 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) top = max(top, x[h][e] & 0x7fffffffu);
    }
  }
  top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
  // 1.75 2^2 = 7: one more where the significand is larger
  int byte = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  byte = min(max(byte, kMxLeast), kMxMost);
  const float scale = mx_scale((uint32_t)byte);
  uint32_t code = 0;
  if (top >= 0x7f800000u) {
    byte = 255;
  } else if constexpr (sizeof(T) == 2) {
    const auto two = [&](int i) {
      const uint32_t w = x[0][i];  // a bit cast of the vector's element itself takes element 0
      return __builtin_bit_cast(bf16x2_t, w);
    };
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, two(0), scale, 0);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, two(1), scale, 1);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, two(2), scale, 2);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, two(3), scale, 3);
  } else {
    const auto f = [&](int e) { return __uint_as_float(x[e >> 2][e & 3]); };
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, f(0), f(1), scale, 0);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, f(2), f(3), scale, 1);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, f(4), f(5), scale, 2);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, f(6), f(7), scale, 3);
  }
  *reinterpret_cast<uint32_t*>((is_v ? a.v : a.k) + it.held * (HD / 2) + 4 * it.c) = code;
  if ((it.c & 3) == 0) (is_v ? a.vs : a.ks)[it.held * (HD / kMxGroup) + (it.c >> 2)] = (uint8_t)byte;
}

template <typename T, int HD>
__global__ __launch_bounds__(256) void mx_load_kernel(MxArgs a) {
  const MxItem it = mx_item<HD>(a);
  if (!it.on) return;
  const bool is_v = blockIdx.y != 0;
  const uint32_t code = *reinterpret_cast<const uint32_t*>((is_v ? a.v : a.k) + it.held * (HD / 2) + 4 * it.c);
  const float scale = mx_scale((is_v ? a.vs : a.ks)[it.held * (HD / kMxGroup) + (it.c >> 2)]);
  const u32x4_t x = {mx_bf16x2<0>(code, scale), mx_bf16x2<1>(code, scale), mx_bf16x2<2>(code, scale),
                     mx_bf16x2<3>(code, scale)};
  T* dst = static_cast<T*>(is_v ? a.pv : a.pk) + it.plain * HD + 8 * it.c;
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<u32x4_t*>(dst) = x;
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<u32x4_t*>(dst + 4 * h) = u32x4_t{x[2 * h] << 16, x[2 * h] & 0xffff0000u, x[2 * h + 1] << 16,
                                                         x[2 * h + 1] & 0xffff0000u};
  }
}

template <typename T, int HD>
static hipError_t launch_mx_t(const MxArgs& a, bool store, hipStream_t st) {
  const long long threads = (long long)a.B * a.n_kv * a.N * (HD / 8);
  const dim3 grid((unsigned)((threads + 255) / 256), 2);
  if (store)
    hipLaunchKernelGGL((mx_store_kernel<T, HD>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((mx_load_kernel<T, HD>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_mx(const MxArgs& a, int dtype_bf16, int hd, int store, hipStream_t st) {
  switch (hd) {
    case 64: return dtype_bf16 ? launch_mx_t<uint16_t, 64>(a, store, st) : launch_mx_t<float, 64>(a, store, st);
    case 128: return dtype_bf16 ? launch_mx_t<uint16_t, 128>(a, store, st) : launch_mx_t<float, 128>(a, store, st);
    case 256: return dtype_bf16 ? launch_mx_t<uint16_t, 256>(a, store, st) : launch_mx_t<float, 256>(a, store, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace kvd
