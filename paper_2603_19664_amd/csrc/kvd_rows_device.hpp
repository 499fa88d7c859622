// What kvd_rows.hip and kvd_sink.hip share: LDS tiles of bf16 keys and values as MFMA
// operands, their copies, and the arithmetic of infinities.
#pragma once

#include "kvd_device.hpp"
#include "kvd_launch.h"

namespace kvd {

// v_exp_f32: one ulp, results below 2^-126 become 0 (weights that no sum feels).
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// Token of a row (r / g): the high half of r ceil(2^32 / g), exact below 2^28 rows (g <= 16);
// a division costs some 30 instructions, and copies of query rows take one per row.
template <class Args>  // RowsArgs or SinkArgs
__device__ __forceinline__ int token_of(const Args& a, int r) {
  return a.g == 1 ? r : (int)__umulhi((uint32_t)r, a.g_inv);
}

// Keys per LDS tile: 32 KiB of K and V.
constexpr int rows_kt(int hd) { return hd == 256 ? 32 : 64; }

// LDS tiles hold rows of HD elements with their 16-byte chunks permuted, row r's chunk c at
// chunk c ^ swz(r), so that every read touches all 64 banks evenly.  The score operand is
// one chunk of 32 rows, 16 rows at a time: swz = r % 16 (two 128-byte rows of head_dim 64
// fill the banks: r / 2 % 8).  The transposing V reads take 64 bytes of 4 rows: swz = 4 (r %
// 4) (head_dim 64: 4 (r / 2 % 2)).  (With 8 rows, or 32 bytes of 4, half of the cycles were
// conflicts.)
template <int HD>
__device__ __forceinline__ int score_swz(int r) { return HD == 64 ? (r >> 1) & 7 : r & 15; }
template <int HD>
__device__ __forceinline__ int v_swz(int r) { return HD == 64 ? 4 * ((r >> 1) & 1) : 4 * (r & 3); }

// A value that the compiler must compute again where it is used: offsets derived from it
// are not kept in registers across a loop (the row tiles of head_dim 256 have none to spare:
// their scores ran on one register quad for K, read, wait, multiply).
__device__ __forceinline__ uint32_t fresh(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Copies KT rows of HD elements from global memory straight into the LDS tile dst (rows
// past n - 1 repeat row n - 1).  Thread tid copies chunk tid % CPR of rows r0 + RPI i, r0 =
// tid / CPR: a full tile takes its rows' offsets from the thread once, 4096 i as a scalar.
template <int HD, int KT, bool SCORE>
__device__ __forceinline__ void copy_tile(const uint16_t* src, int n, uint16_t* dst) {
  constexpr int CPR = HD / 8, RPI = 256 / CPR, CH = KT / RPI;
  const int tid = (int)fresh(threadIdx.x), w = wave_id();
  const int r0 = tid / CPR, ch = tid % CPR;
  const __amdgpu_buffer_rsrc_t res =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(src), (short)0, KT * HD * 2, 0x00027000);
  const bool full = n >= KT;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int r = r0 + RPI * i;
    const int col = 16 * (ch ^ (SCORE ? score_swz<HD>(r) : v_swz<HD>(r)));
    __builtin_amdgcn_raw_ptr_buffer_load_lds(res, (__attribute__((address_space(3))) void*)(dst + 512 * w + 2048 * i), 16,
                                             (full ? r0 * HD * 2 : min(r, n - 1) * HD * 2) + col, full ? 4096 * i : 0,
                                             0, 0);
  }
}

typedef short i16x4_t __attribute__((ext_vector_type(4)));

// Byte offsets of a lane's operands in the LDS tiles.
// Score operand: row lane % 32, elements 16 kk + 8 (lane / 32) ..; 32 rows on: + 64 HD.
template <int HD>
__device__ __forceinline__ uint32_t score_base(int lane) {
  return (lane & 31) * HD * 2 + (((lane >> 5) ^ score_swz<HD>(lane & 31)) << 4);
}
__device__ __forceinline__ bf16x8_t score_operand(const uint16_t* tile, uint32_t base, int kk, int rows) {
  return *reinterpret_cast<const bf16x8_t*>(reinterpret_cast<const char*>(tile) + (base ^ (kk << 5)) + rows);
}
// V^T operand of a 32-row block db of O^T for the 16 keys at k0: two transposing reads
// (in a group of 16 lanes, lane s names 4 columns of row s / 4 of a 4-key group, and lane
// i receives column i of the 4 keys).  Lane half hl gets keys k0 + 4 hl + {0..3, 8..11},
// the ones whose scores it holds.
template <int HD>
__device__ __forceinline__ uint32_t v_base(int lane) {
  const int row = 4 * (lane >> 5) + ((lane & 15) >> 2);
  return row * HD * 2 + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ v_swz<HD>(row)) << 4) + 8 * (lane & 1);
}
template <int HD>
__device__ __forceinline__ bf16x8_t v_operand(const uint16_t* vs, uint32_t base, int k0, int db) {
  const char* p = reinterpret_cast<const char*>(vs) + (base ^ (db << 6)) + k0 * HD * 2;
  const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4_t*)p);
  const i16x4_t hi =
      __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4_t*)(p + 16 * HD));
  return __builtin_bit_cast(bf16x8_t, make_uint4(__builtin_bit_cast(uint2, lo).x, __builtin_bit_cast(uint2, lo).y,
                                                 __builtin_bit_cast(uint2, hi).x, __builtin_bit_cast(uint2, hi).y));
}

// Two bf16 in a word: nonzero where one is infinite or NaN (the exponent's carry).
__device__ __forceinline__ uint32_t nonfinite2(uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
// A code for a non-finite value that sums over up to 127 keys keep apart, and back.
__device__ __forceinline__ float code_of(float v) {
  return v == INFINITY ? 1.0f : v == -INFINITY ? 128.0f : 16384.0f;
}
__device__ __forceinline__ float poison_of(float codes) {
  if (codes == 0.0f) return 0.0f;
  const int c = (int)codes;
  const bool pos = (c & 127) != 0, neg = ((c >> 7) & 127) != 0;
  return c >= 16384 || (pos && neg) ? __uint_as_float(0x7fc00000u) : pos ? INFINITY : -INFINITY;
}
// x + w y of partial sums, where a weight that 32 bits took as 0 does not make an infinity NaN.
__device__ __forceinline__ float add_state(float x, float w, float y) {
  return fabsf(y) < INFINITY ? fmaf(w, y, x) : x + y;
}

// V in a wave's LDS slice of few rows: see copy16.
template <int HD>
__device__ __forceinline__ int few_v_swz(int r) { return HD == 64 ? 2 * ((r >> 1) & 3) : 2 * (r & 7); }
// Waits until at most N of the wave's vector memory operations are in flight (they complete
// in order), and keeps the LDS reads that follow behind it.
template <int N>
__device__ __forceinline__ void wait_copies() {
  static_assert(N < 64, "a count of six bits");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4) << 14);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

}  // namespace kvd
