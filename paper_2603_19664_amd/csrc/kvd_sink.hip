// Attention of new tokens over a sequence's first tokens and a sliding window: kvd_sink_attn
// (K/V of the shape's dtype) and kvd_mx_attn (a 4-bit cache).
//
//   sink_few_kernel     blocks of 16 query rows, whose waves stream 32 keys at a time each on
//                       its own (bf16: single tokens and short drafts; 4 bits with fp32 queries: every call).
//   sink_tile_kernel    bf16: 128 rows per workgroup that share key tiles in LDS.
//   sink_f32_kernel     fp32 K/V: blocks of 16 rows, both products on MFMA 16x16x4 f32.
//   sink_merge_kernel, sink_finish_kernel
//                       merge the slots' softmax states into out.
//
// Rows.  The rows of (sequence b, KV head j) are (token i, head h of the group), r = i g + h.
// A block of them sees the keys x = 0 .. n - 1 that sink_keys names, in slots of C; slot s
// leaves the partial states
//   acc [S][n_kv][B R][hd], ml [S][n_kv][B R][2]  (sum 2^(s - max) V; max, sum),
// in the log2 domain.  A block whose keys are one slot writes out itself.
#include <hip/hip_runtime.h>

#include "kvd_rows_device.hpp"
#include "kvd_rows_layout.h"
#include "kvd_sink_device.hpp"

namespace kvd {

// A block of rows of (b, j) and its share of their keys: slot s of slots.
struct SinkItem {
  int b, j, r0, nr;  // rows r0 .. r0 + nr - 1
  int s, slots, x0, n;  // keys x0 .. x0 + n - 1
  int p0;            // position of the sequence's first new token
  SinkKeys keys;
};
__device__ __forceinline__ int sink_slots(const SinkArgs& a, const SinkKeys& k) {
  return max((int)(((uint32_t)k.n + (uint32_t)a.C - 1u) / (uint32_t)a.C), 1);
}

// Grid: B n_kv (sequence, KV head), slots, blocks.  False where the workgroup has nothing to do.
template <int RB>
__device__ __forceinline__ bool sink_item(const SinkArgs& a, SinkItem& it) {
  it.b = (int)(blockIdx.x / (uint32_t)a.n_kv);
  it.j = (int)blockIdx.x - it.b * a.n_kv;
  // from another slot in every block: XCDs (workgroups in turn) share early and late keys
  it.s = a.S == 1 ? 0 : (int)((blockIdx.y + blockIdx.z) % (uint32_t)a.S);
  it.r0 = (int)(gridDim.z - 1 - blockIdx.z) * RB;  // heavy blocks, the last tokens, first
  const SinkSeq sq = sink_seq(a.kv_len, a.n_new, a.T, a.N, it.b);
  it.nr = min(RB, sq.n * a.g - it.r0);
  if (it.nr <= 0) return false;
  it.p0 = sq.len - sq.n;
  it.keys = sink_keys(a, it.p0 + token_of(a, it.r0), it.p0 + token_of(a, it.r0 + it.nr - 1));
  it.slots = sink_slots(a, it.keys);
  if (it.s >= it.slots) return false;
  it.x0 = it.s * a.C;
  it.n = min(a.C, it.keys.n - it.x0);
  return true;
}
__device__ __forceinline__ size_t sink_state(const SinkArgs& a, int s, int b, int j, int r) {
  return ((size_t)s * a.n_kv + j) * ((size_t)a.B * a.R) + (size_t)b * a.R + r;
}

// The item's keys in blocks of KB that lie in neighbouring rows each: those of the sinks, of the
// window up to the ring's end, and behind it.  All of it is uniform.
template <int KB>
struct SinkBlocks {
  int e0, e1, n, n0, n1, blocks;  // ends of the first two parts, keys; blocks of the first part, of the first two, in all
  int row0, d, ring;
  __device__ __forceinline__ SinkBlocks(const SinkItem& it) {
    n = it.n;
    e0 = min(max(it.keys.ns - it.x0, 0), n);
    e1 = min(max(it.keys.cap - it.keys.d - it.x0, e0), n);
    n0 = (e0 + KB - 1) / KB;
    n1 = n0 + (e1 - e0 + KB - 1) / KB;
    blocks = n1 + (n - e1 + KB - 1) / KB;
    row0 = it.x0;
    d = it.keys.d;
    ring = it.keys.ring;
  }
  // block i: keys x .. end - 1 (at most KB of them), from cache row `row` on
  struct Block {
    int x, end, row;
  };
  __device__ __forceinline__ Block at(int i) const {
    Block b;
    if (i < n0) {
      b.x = KB * i;
      b.end = e0;
      b.row = row0 + b.x;
    } else if (i < n1) {
      b.x = e0 + KB * (i - n0);
      b.end = e1;
      b.row = row0 + b.x + d;
    } else {
      b.x = e1 + KB * (i - n1);
      b.end = n;
      b.row = row0 + b.x + d - ring;
    }
    b.x = __builtin_amdgcn_readfirstlane(b.x);
    b.end = __builtin_amdgcn_readfirstlane(min(b.end, b.x + KB));
    b.row = __builtin_amdgcn_readfirstlane(b.row);
    return b;
  }
};

// Rows row .. row + n - 1 of an array with `bytes` to a row: reads behind them give 0.  The range check is of
// the vector offset with the immediate: offsets of rows are in these whole, and the scalar offset is 0.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_resource(const void* p, size_t row, int n, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(p)) + row * bytes, (short)0,
                                           n * bytes, 0x00027000);
}

// Element offset of row r of (b, j) in q and out.
__device__ __forceinline__ size_t sink_q(const SinkArgs& a, int b, int j, int r, int hd) {
  const int i = token_of(a, r);
  return (((size_t)b * a.N + i) * a.n_q + (size_t)j * a.g + (r - i * a.g)) * hd;
}

// Where 16-byte chunk e of group g of a 4-bit row's values goes within the group's 64 bytes of
// LDS, beside the swizzle of the row: a store instruction writes chunk e of 8 groups at a time.
__device__ __forceinline__ constexpr int mx_swz(int g) { return (g & 3) ^ (g >> 2 & 1); }

// 32 4-bit numbers as 4 chunks of 8 bf16 into LDS at row_at + 16 (4 g + e ^ swz).
__device__ __forceinline__ void mx_put(u32x4_t code, float scale, char* row_at, int g, int swz) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t w = code[e];
    *reinterpret_cast<u32x4_t*>(row_at + ((4 * g + e) ^ swz ^ mx_swz(g)) * 16) =
        u32x4_t{mx_bf16x2<0>(w, scale), mx_bf16x2<1>(w, scale), mx_bf16x2<2>(w, scale), mx_bf16x2<3>(w, scale)};
  }
}

// 32 rows of V by direct copies into a wave's slice of LDS, 16-byte chunks permuted (few_v_swz).
template <int HD>
__device__ __forceinline__ void copy_v32(__amdgpu_buffer_rsrc_t res, char* dst) {
  constexpr int CPR = HD / 8, RPI = 64 / CPR;
  const int lane = (int)fresh(threadIdx.x & 63);
#pragma unroll
  for (int l = 0; l < 32 / RPI; ++l)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        res, (__attribute__((address_space(3))) void*)(dst + 1024 * l), 16,
        (lane / CPR) * HD * 2 + 16 * (lane % CPR ^ few_v_swz<HD>(lane / CPR + RPI * l)) + 1024 * l, 0, 0, 0);
}

// x as a sum of bf16 parts, rounded (P parts), returned as the packed pairs of (x, y).
template <int P>
__device__ __forceinline__ void split2(float x, float y, uint32_t (&w)[P]) {
#pragma unroll
  for (int i = 0; i < P; ++i) {
    w[i] = pack_bf16x2(x, y);
    x -= bf_lo(w[i]);
    y -= bf_hi(w[i]);
  }
}
// The same by truncation, which overflows nowhere; an infinity or NaN is the first part alone.
template <int P>
__device__ __forceinline__ void split2_trunc(float x, float y, uint32_t (&w)[P]) {
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const uint32_t hx = __float_as_uint(x) & 0xffff0000u, hy = __float_as_uint(y) & 0xffff0000u;
    // a NaN keeps a bit of its significand
    w[i] = (x == x ? hx : 0x7fc00000u) >> 16 | (y == y ? hy : 0x7fc00000u);
    x = fabsf(x) < INFINITY ? x - __uint_as_float(hx) : 0.0f;
    y = fabsf(y) < INFINITY ? y - __uint_as_float(hy) : 0.0f;
  }
}

// Sums of finite values may pass 2^128 where their weighted mean does not.  A wave's sums of 2^117 and more send it
// through its keys once more, with weights of at most 2^-sum_room(keys that the block sees): all of the block's states
// together stay below 2^127 then, and those of up to 512 others below 2^126, so no merge overflows.
__device__ __forceinline__ float too_large(float o, float x) { return fmaf(o * 0x1p11f, 0.0f, x); }  // x, NaN if it is
__device__ __forceinline__ float sum_room(int n) { return (float)(33 - __clz(n)); }

// ------------------------------------------------------------------ blocks of 16 rows

// Workgroups per CU that the registers are to leave room for.
constexpr int few_wgs(int hd, bool bf) {
  return hd == 256 ? (bf ? 2 : 1) : hd == 128 ? 3 : 4;
}

// One workgroup of 4 waves per (16-row block, slot).  The slot's 32-key blocks go to the waves in
// turn, each wave with its own slice of LDS and no barrier: HBM-bound, so what matters is
// loads in flight.
//
// Scores S^T = K Q^T on MFMA 16x16x32, 16 keys at a time, K straight from memory: lane (key lane %
// 16, lg = lane / 16) brings 8 elements of a key to every step.  Plain: elements 32 c + 8 lg ..
// of step c.  4 bits: the lane's 16 bytes are one group of 32, a quarter of it for each step, and one scale:
// which elements meet in a step does not matter as long as K's and Q's are the same.
// O^T += V^T P^T on 16x16x32 with P^T straight from the score registers, as the sum of bf16 parts
// (two for bf16 queries: 2^-17 of a weight is lost; three for fp32), V through LDS: plain by direct copies,
// 4 bits as the bf16 numbers that they are (one instruction for two), read transposed.
// K of the next block is asked for when the scores are taken, V after its product.
// Measured (several caches in turn, so that HBM is read): 64 streams of 1028 bf16 rows, 4 KV heads of 256, 49.2 us,
// 5.5 TB/s; in 4 bits 8 x 32768 rows of them 57 us, 5.0 TB/s; 64 x 4096 .. 8192 rows of 2 heads of 128 27 us, 3.9 TB/s:
// half the bytes to a block's fixed work, waves waiting for memory 44% of their time.  (Two blocks of these on
// their way, 204 registers: 37 us.)  A call of few keys takes 5 us, at head_dim 256 7 to 8, most of it instructions.
template <int HD, bool MX, typename QT>
__global__ __launch_bounds__(256, few_wgs(HD, sizeof(QT) == 2)) void sink_few_kernel(SinkArgs a) {
  constexpr bool BF = sizeof(QT) == 2;
  constexpr int NW = 4, KB = 32, KC = HD / 32, DB = HD / 16, kLead = 4;
  constexpr int QP = BF ? 1 : 3, PP = BF ? 2 : 3;  // parts of a query element and of a weight
  constexpr int KW = HD == 64 ? 2 : 4;             // words of 4-bit codes a lane loads at once
  constexpr int KL = HD / 32 / KW;                 // how many times (MX)
  constexpr int G = HD / kMxGroup, NV = HD / 64;   // groups of a row; groups of V a lane turns into bf16
  __shared__ __align__(1024) uint16_t vbuf[NW][KB * HD];
  __shared__ float ml[NW][16][2];
  __shared__ unsigned long long bads[NW];
  const int tid = threadIdx.x, lane = tid & 63, w = wave_id(), hq = lane & 15, lg = lane >> 4;
  SinkItem it;
  if (!sink_item<16>(a, it)) return;
  const SinkBlocks<KB> blk(it);
  const int nb = blk.blocks > w ? (blk.blocks - 1 - w) / NW + 1 : 0;  // this wave's blocks: w, w + NW, ..
  const size_t base = ((size_t)it.b * a.n_kv + it.j) * a.t_cap + a.t_off;
  // keys of this slot that the lane's row sees: x < hi with x < sink or x >= lo; that every row sees
  const auto seen_by = [&](int r) {
    SinkRow s = sink_row_of(a, it.keys, it.p0 + token_of(a, it.r0 + min(r, it.nr - 1)));
    return SinkRow{max(s.lo, 0) - it.x0, min(s.hi - it.x0, it.n)};
  };
  const int sink = max(a.sink - it.x0, 0);
  const SinkRow mine = seen_by(hq);
  const int all_hi = seen_by(0).hi, all_lo = seen_by(15).lo;

  // queries
  uint32_t qw[QP][KC][4];
  {
    const QT* qs = static_cast<const QT*>(a.q) + sink_q(a, it.b, it.j, it.r0 + min(hq, it.nr - 1), HD);
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const int d = MX ? 8 * KW * (lg + 4 * (c / KW)) + 8 * (c % KW) : 32 * c + 8 * lg;
      if constexpr (BF) {
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(qs + d);
#pragma unroll
        for (int e = 0; e < 4; ++e) qw[0][c][e] = v[e];
      } else {
        const f32x4_t u = *reinterpret_cast<const f32x4_t*>(qs + d), v = *reinterpret_cast<const f32x4_t*>(qs + d + 4);
        const float x[8] = {u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t part[QP];
          split2_trunc<QP>(x[2 * e], x[2 * e + 1], part);
#pragma unroll
          for (int i = 0; i < QP; ++i) qw[i][c][e] = part[i];
        }
      }
    }
  }

  // K of a block: two sets of 16 keys
  u32x4_t kp[2][MX ? 1 : KC];
  uint32_t kc[2][MX ? KL : 1][KW];
  uint8_t ks[2][MX ? KL : 1];  // (as 32 bits, their extension waited for the load that it follows)
  u32x4_t vc[MX ? NV : 1];
  uint8_t vs[MX ? NV : 1];
  char* const vl = reinterpret_cast<char*>(vbuf[w]);
  typedef typename SinkBlocks<KB>::Block Block;
  auto load_k = [&](const Block& kb) {
    const auto res = rows_resource(a.k, base + kb.row, kb.end - kb.x, MX ? HD / 2 : HD * 2);
    if constexpr (MX) {
      const auto sres = rows_resource(a.ks, base + kb.row, kb.end - kb.x, G);
      const int at = hq * (HD / 2) + 4 * KW * lg, sat = hq * G + (HD == 64 ? lg >> 1 : lg);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int l = 0; l < KL; ++l) {
          if constexpr (KW == 4) {
            const auto v = __builtin_amdgcn_raw_buffer_load_b128(res, at + 16 * t * (HD / 2) + 64 * l, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) kc[t][l][e] = v[e];
          } else {
            const auto v = __builtin_amdgcn_raw_buffer_load_b64(res, at + 16 * t * (HD / 2), 0, 0);
            kc[t][l][0] = v[0];
            kc[t][l][1] = v[1];
          }
          ks[t][l] = __builtin_amdgcn_raw_buffer_load_b8(sres, sat + 16 * t * G + 4 * l, 0, 0);
        }
    } else {
      const int at = hq * HD * 2 + 16 * lg;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int c = 0; c < KC; ++c)
          kp[t][c] = __builtin_amdgcn_raw_buffer_load_b128(res, at + 64 * c + 32 * t * HD, 0, 0);
    }
  };
  auto load_v = [&](const Block& kb) {
    const auto res = rows_resource(a.v, base + kb.row, kb.end - kb.x, MX ? HD / 2 : HD * 2);
    if constexpr (MX) {
      const auto sres = rows_resource(a.vs, base + kb.row, kb.end - kb.x, G);
#pragma unroll
      for (int l = 0; l < NV; ++l) {
        vc[l] = __builtin_amdgcn_raw_buffer_load_b128(res, 16 * lane + 1024 * l, 0, 0);
        vs[l] = __builtin_amdgcn_raw_buffer_load_b8(sres, lane + 64 * l, 0, 0);
      }
    } else {
      copy_v32<HD>(res, vl);
    }
  };
  // every LDS read of the wave is done: its slice may be written again
  auto reads_done = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
  };
  // byte offsets in LDS: of the lane's V operands, and of the bf16 numbers that it makes (group lane % G of row lane /
  // G; 64 lanes on, the swizzles are the same)
  char* const lds = reinterpret_cast<char*>(&vbuf[0][0]);
  const int vrow = 4 * lg + (hq >> 2), prow = lane / G, pg = lane % G;
  const uint32_t vrow_at = (w * KB + vrow) * HD * 2 + ((((hq & 3) >> 1) ^ few_v_swz<HD>(vrow)) << 4) + 8 * (hq & 1);
  const uint32_t put_at = (w * KB + prow) * HD * 2 + ((4 * pg ^ few_v_swz<HD>(prow) ^ mx_swz(pg)) << 4);

  f32x4_t o[DB];
  float m_run, l_run;
  // A second pass where an infinite or NaN value met a weight of 0: such values count as 0 there and
  // are added afterwards where they are seen.  A third one for sums that are too large.
  int pass = 0;
  float lag = 8.0f, room = 0.0f;  // how far the maximum may lie behind; weights are 2^-room of what they would be
  unsigned long long bad = 0;  // bit i % 64: block i of the wave holds such a value
again:
  Block kb{0, 0, 0};
  if (nb > 0) {
    kb = blk.at(w);
    load_k(kb);
    load_v(kb);
  }
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  m_run = -INFINITY;
  l_run = 0.0f;
  // One copy of the code, also for a wave's last block, whose successor is empty: a small call waits for its
  // instructions (60 ns for 64 bytes).  (The waits for K are shorter than the loads behind it would allow: to the
  // compiler the queries' loads may still be pending, as they are past the branch of a wave without blocks.)
  auto step = [&](auto second, int i) {
    constexpr bool SECOND = decltype(second)::value != 0;
    const Block kb1 = i + 1 < nb ? blk.at(w + NW * (i + 1)) : Block{0, 0, 0};
    const bool masked = kb.x + KB > min(all_hi, kb.end) || (kb.end > sink && all_lo > max(kb.x, sink));
    f32x4_t st[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
      for (int t = 0; t < 2; ++t) {  // two chains of products
        u32x4_t kf;
        if constexpr (MX) {
          const uint32_t code = kc[t][c / KW][c % KW];
          const float scale = mx_scale(ks[t][c / KW]);
          kf = u32x4_t{mx_bf16x2<0>(code, scale), mx_bf16x2<1>(code, scale), mx_bf16x2<2>(code, scale),
                       mx_bf16x2<3>(code, scale)};
        } else {
          kf = kp[t][c];
        }
#pragma unroll
        for (int e = 0; e < QP; ++e)
          st[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              __builtin_bit_cast(bf16x8_t, kf),
              __builtin_bit_cast(bf16x8_t, make_uint4(qw[e][c][0], qw[e][c][1], qw[e][c][2], qw[e][c][3])), st[t], 0, 0,
              0);
      }
    load_k(kb1);
    if constexpr (MX) {
      const uint32_t to = fresh(put_at);
      uint32_t found = 0;
#pragma unroll
      for (int l = 0; l < NV; ++l) {
        u32x4_t code = vc[l];
        uint32_t byte = vs[l];
        if (SECOND && byte == 255) {
          found = 1;
          byte = 127;
          code = u32x4_t{0u, 0u, 0u, 0u};
        }
        const float scale = mx_scale(byte);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t cw = code[e];
          *reinterpret_cast<u32x4_t*>(lds + (to ^ (e << 4)) + l * (64 / G) * HD * 2) =
              u32x4_t{mx_bf16x2<0>(cw, scale), mx_bf16x2<1>(cw, scale), mx_bf16x2<2>(cw, scale), mx_bf16x2<3>(cw, scale)};
        }
      }
      if (SECOND && __any(found != 0)) bad |= 1ull << (i & 63);
      load_v(kb1);
    }
    // st[t][r]: key kb.x + 16 t + 4 lg + r, row hq
    if (masked) {
      asm volatile("");  // one branch
      const int hi = min(mine.hi, kb.end);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int x = kb.x + 16 * (e >> 2) + 4 * lg + (e & 3);
        st[e >> 2][e & 3] = (x < hi) & ((x < sink) | (x >= mine.lo)) ? st[e >> 2][e & 3] : -INFINITY;
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) mx = fmaxf(mx, st[e >> 2][e & 3]);
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * ScoreScale<HD>::v;
    const bool grow = mx > m_run + lag;
    if (__any(grow)) {
      const float m_new = grow ? mx : m_run;
      const float alpha = exp2_hw(grow ? m_run - m_new : 0.0f);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= alpha;
    }
    const float m_use = (m_run == -INFINITY ? 0.0f : m_run) + room;
    uint32_t pw[PP][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 2 * (e & 1);
      const float pa = exp2_hw(fmaf(st[e >> 1][r], ScoreScale<HD>::v, -m_use));
      const float pb = exp2_hw(fmaf(st[e >> 1][r + 1], ScoreScale<HD>::v, -m_use));
      l_run += pa + pb;
      uint32_t part[PP];
      split2<PP>(pa, pb, part);
#pragma unroll
      for (int p = 0; p < PP; ++p) pw[p][e] = part[p];
    }
    if constexpr (!MX) {
      // V, in order after which the next block's K was asked for
      wait_copies<2 * KC>();
      if (pass != 0) {
        uint32_t found = 0;
#pragma unroll 1
        for (int x = lane; x < KB * HD / 2; x += 64) {
          uint32_t* at = reinterpret_cast<uint32_t*>(vl) + x;
          const uint32_t f = nonfinite2(*at);
          found |= f;
          if (f != 0) *at &= (f & 0x8000u ? 0u : 0xffffu) | (f & 0x80000000u ? 0u : 0xffff0000u);
        }
        if (__any(found != 0)) bad |= 1ull << (i & 63);
      }
    }
    const uint32_t vbase = fresh(vrow_at);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const char* at = lds + (vbase ^ (db << 5) ^ (MX ? mx_swz(db >> 1) << 4 : 0));
      const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4_t*)at);
      const i16x4_t hi =
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4_t*)(at + 16 * HD * 2));
      const uint2 vlo = __builtin_bit_cast(uint2, lo), vhi = __builtin_bit_cast(uint2, hi);
      const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, make_uint4(vlo.x, vlo.y, vhi.x, vhi.y));
#pragma unroll
      for (int p = 0; p < PP; ++p)
        o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            vf, __builtin_bit_cast(bf16x8_t, make_uint4(pw[p][0], pw[p][1], pw[p][2], pw[p][3])), o[db], 0, 0, 0);
    }
    // V operands kLead products ahead: all at once they would take the registers that K waits in.  (A hint: in 4 bits
    // at head_dim 64, and at 128 with fp32 queries, every operand is waited for where it is used, and in the plain
    // kernel at 256 every wait is one for all reads.)
    __builtin_amdgcn_sched_group_barrier(0x100, 2 * kLead, 0);
#pragma unroll
    for (int db = 0; db < DB - kLead; ++db) {
      __builtin_amdgcn_sched_group_barrier(0x008, PP, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, PP * kLead, 0);
    if constexpr (!MX) {
      reads_done();
      load_v(kb1);
    }
    kb = kb1;
  };
  if (!MX || pass == 0) {
    for (int i = 0; i < nb; ++i) step(IC<0>{}, i);
  } else {
    for (int i = 0; i < nb; ++i) step(IC<1>{}, i);
  }
  l_run += __shfl_xor(l_run, 16, 64);
  l_run += __shfl_xor(l_run, 32, 64);
  if (pass < 2) {
    float x = 0.0f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 4; ++e) x = too_large(o[db][e], x);
    x += __shfl_xor(x, 16, 64);
    x += __shfl_xor(x, 32, 64);
    const bool odd = hq < it.nr && x != 0.0f && (pass == 0 || l_run < INFINITY);  // (a NaN score stays one)
    if (__any(odd)) {
      if (++pass == 2 && odd) {  // for such a row alone: what it does not see changes no bit of another
        lag = 0.0f;
        room = sum_room(it.keys.n);
      }
      if constexpr (!MX) wait_copies<0>();  // the last, empty block's copy is no longer on its way into the slice
      goto again;
    }
  }

  // The waves' states into LDS (16-byte chunks permuted by the row), then merged in wave order:
  // the slot's state, or with one slot the output.
  if constexpr (!MX) wait_copies<0>();
  __syncthreads();
  constexpr int CM = HD / 4 - 1;
  float* f = reinterpret_cast<float*>(&vbuf[0][0]);
  if (lg == 0) {
    ml[w][hq][0] = m_run + room;
    ml[w][hq][1] = l_run;
  }
  if (lane == 0) bads[w] = bad;
#pragma unroll
  for (int db = 0; db < DB; ++db)
    *reinterpret_cast<f32x4_t*>(f + (w * 16 + hq) * HD + 4 * ((4 * db + lg) ^ (hq & CM))) = o[db];
  __syncthreads();
  for (int i = tid; i < it.nr * (HD / 4); i += 64 * NW) {
    const int h = i / (HD / 4), c4 = i - h * (HD / 4);
    float M = -INFINITY;
#pragma unroll
    for (int v = 0; v < NW; ++v) M = fmaxf(M, ml[v][h][0]);
    const float Mu = M == -INFINITY ? 0.0f : M;
    f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
    float L = 0.0f;
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      const float wt = exp2_hw(ml[v][h][0] - Mu);
      const f32x4_t y = *reinterpret_cast<const f32x4_t*>(f + (v * 16 + h) * HD + 4 * (c4 ^ (h & CM)));
      x += wt * y;  // (no state holds an infinity, and no sum of them passes 2^128)
      L = fmaf(wt, ml[v][h][1], L);
    }
    // the values that a second pass took as 0, where the row sees them
#pragma unroll 1
    for (int v = 0; v < NW; ++v) {
      if (bads[v] == 0) continue;
      const SinkRow see = seen_by(h);
#pragma unroll 1
      for (int k = 0; v + NW * k < blk.blocks; ++k) {
        if ((bads[v] >> (k & 63) & 1) == 0) continue;
        const auto kb = blk.at(v + NW * k);
#pragma unroll 1
        for (int y = kb.x; y < kb.end; ++y) {
          if (!((y < see.hi) & ((y < sink) | (y >= see.lo)))) continue;
          const size_t r = base + kb.row + (y - kb.x);
          float z[4];
          if constexpr (MX) {
            z[0] = z[1] = z[2] = z[3] = a.vs[r * G + (c4 >> 3)] == 255 ? __uint_as_float(0x7fc00000u) : 0.0f;
          } else {
            const uint2 u = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(a.v) + r * HD + 4 * c4);
            z[0] = bf_lo(u.x), z[1] = bf_hi(u.x), z[2] = bf_lo(u.y), z[3] = bf_hi(u.y);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] += fabsf(z[e]) < INFINITY ? 0.0f : z[e];
        }
      }
    }
    if (it.slots == 1) {
      QT* dst = static_cast<QT*>(a.out) + sink_q(a, it.b, it.j, it.r0 + h, HD) + 4 * c4;
      if constexpr (BF) {
        const float inv = L != 0.0f ? 1.0f / L : 0.0f;
        uint2 y = make_uint2(0u, 0u);
        if (L != 0.0f) y = make_uint2(pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv));
        *reinterpret_cast<uint2*>(dst) = y;
      } else {
        *reinterpret_cast<f32x4_t*>(dst) =
            L != 0.0f ? f32x4_t{x[0] / L, x[1] / L, x[2] / L, x[3] / L} : f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
      }
    } else {
      const size_t row = sink_state(a, it.s, it.b, it.j, it.r0 + h);
      *reinterpret_cast<f32x4_t*>(a.acc + row * HD + 4 * c4) = x;
      if (c4 == 0) {
        a.ml[2 * row] = Mu;
        a.ml[2 * row + 1] = L;
      }
    }
  }
}

// ------------------------------------------------------------------ 128-row tiles (bf16)

// One workgroup of 4 waves per (128-row block, slot), 32 rows per wave, through the slot's key
// tiles; the products, the running maximum and the two parts of a weight as in rows_tile
// (kvd_rows.hip).  Plain K and V are copied straight into the other LDS buffer while a tile is
// computed; the rows of a tile that the sinks' or the ring's end cuts are copied one by one.  4 bits: the
// next tile's numbers wait as they are and become bf16 in LDS once for the 128 rows.  A
// wave skips the tiles that none of its rows sees.
// Measured: 8192 tokens, window 1024, 8 heads of 256: 113 us, 0.57 PFLOP/s of the formula's flops, 0.86 of products
// (a large matrix product reaches 1.17); MFMA is busy in half of the cycles, at 1.6 GHz.  The next tile's scores
// between a tile's weights and its product cost registers and time (2 x 512 tokens over 4611 keys of 128: 44 -> 51
// us), tiles of 32 keys and three workgroups per CU too (47).
template <int HD, bool MX>
__global__ __launch_bounds__(256, 2) void sink_tile_kernel(SinkArgs a) {
  constexpr int KT = rows_kt(HD), KH = KT / 32, KS = HD / 16, DB = HD / 32, kLead = 4;
  constexpr int G = HD / kMxGroup, NC = KT * G >= 256 ? KT * G / 256 : 1;  // groups of a row; groups a thread brings
  __shared__ __align__(1024) uint16_t buf0[2 * KT * HD], buf1[2 * KT * HD];
  // Where a thread's own groups of the next tile wait: head_dim 256 has no registers for them (63 us so, 52 through LDS:
  // 2 x 256 tokens over 4000 keys), the others no time to spare (8 x 256 tokens over 8448 keys: 160, 176).
  constexpr bool RAW = MX && HD == 256;
  __shared__ __align__(1024) u32x4_t raw[RAW ? 2 * 256 * NC : 1];
  const int lane = threadIdx.x & 63, w = wave_id(), hl = lane >> 5;
  SinkItem it;
  if (!sink_item<kRowsTile>(a, it)) return;
  const int nt = (it.n + KT - 1) / KT;
  const size_t base = ((size_t)it.b * a.n_kv + it.j) * a.t_cap + a.t_off;

  // this lane's row, and what it and the wave's first and last row see: x < hi with x < sink or x >= lo
  const int rl = 32 * w + (lane & 31);
  const bool wave_on = 32 * w < it.nr;
  const auto seen_by = [&](int r) {
    SinkRow s = sink_row_of(a, it.keys, it.p0 + token_of(a, it.r0 + min(r, it.nr - 1)));
    return SinkRow{max(s.lo, 0) - it.x0, min(s.hi - it.x0, it.n)};
  };
  const int sink = max(a.sink - it.x0, 0);
  const SinkRow mine = seen_by(rl), first = seen_by(32 * w), last = seen_by(32 * w + 31);
  bf16x8_t qf[KS];
  {
    const uint16_t* qs = static_cast<const uint16_t*>(a.q) + sink_q(a, it.b, it.j, it.r0 + min(rl, it.nr - 1), HD) + 8 * hl;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8_t*>(qs + 16 * ks);
  }
  f32x16_t o[DB];
  float m_run, l_run;  // in units of the scaled score

  // plain: tile t into buf
  auto load = [&](int t, uint16_t* buf) {
    const int k0 = it.x0 + KT * t, n = it.n - KT * t;
    const int r0 = it.keys.row(k0);
    if (n >= KT && it.keys.row(k0 + KT - 1) == r0 + KT - 1) {  // rows in order
      copy_tile<HD, KT, true>(static_cast<const uint16_t*>(a.k) + (base + r0) * HD, KT, buf);
      copy_tile<HD, KT, false>(static_cast<const uint16_t*>(a.v) + (base + r0) * HD, KT, buf + KT * HD);
      return;
    }
    constexpr int CPR = HD / 8, RPI = 256 / CPR;
    const int tid = (int)fresh(threadIdx.x);
#pragma unroll 2
    for (int i = 0; i < KT / RPI; ++i) {
      const int r = tid / CPR + RPI * i, ch = tid % CPR;
      const size_t row = (base + it.keys.row(k0 + min(r, n - 1))) * HD;
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)(static_cast<const uint16_t*>(a.k) + row + 8 * (ch ^ score_swz<HD>(r))),
          (__attribute__((address_space(3))) void*)(buf + 512 * w + 2048 * i), 16, 0, 0);
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)(static_cast<const uint16_t*>(a.v) + row + 8 * (ch ^ v_swz<HD>(r))),
          (__attribute__((address_space(3))) void*)(buf + KT * HD + 512 * w + 2048 * i), 16, 0, 0);
    }
  };
  // 4 bits: tile t's numbers on their way, and from there into buf
  u32x4_t kc[RAW ? 1 : NC], vc[RAW ? 1 : NC];
  uint8_t kb[NC], vb[NC];
  auto fetch = [&](int t) {
    if constexpr (RAW) {  // the wave's reads of its places are done
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
      __builtin_amdgcn_sched_barrier(0);
    }
    const int k0 = it.x0 + KT * t, n = it.n - KT * t;
    const int tid = RAW ? (int)fresh(threadIdx.x) : (int)threadIdx.x;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int id = tid + 256 * i, r = id / G, g = id % G;
      if (KT * G < 256 && r >= KT) break;
      const size_t row = base + it.keys.row(k0 + min(r, n - 1));
      const uint8_t* ksrc = static_cast<const uint8_t*>(a.k) + row * (HD / 2) + 16 * g;
      const uint8_t* vsrc = static_cast<const uint8_t*>(a.v) + row * (HD / 2) + 16 * g;
      if constexpr (RAW) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)ksrc,
                                         (__attribute__((address_space(3))) void*)(raw + 256 * i + 64 * w), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)vsrc,
                                         (__attribute__((address_space(3))) void*)(raw + 256 * (NC + i) + 64 * w), 16, 0, 0);
      } else {
        kc[i] = *reinterpret_cast<const u32x4_t*>(ksrc);
        vc[i] = *reinterpret_cast<const u32x4_t*>(vsrc);
      }
      kb[i] = a.ks[row * G + g];
      vb[i] = a.vs[row * G + g];
    }
  };
  auto put = [&](uint16_t* buf) {
    if constexpr (RAW) wait_copies<0>();
    const int tid = RAW ? (int)fresh(threadIdx.x) : (int)threadIdx.x;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int id = tid + 256 * i, r = id / G, g = id % G;
      if (KT * G < 256 && r >= KT) break;
      mx_put(RAW ? raw[id] : kc[RAW ? 0 : i], mx_scale(kb[i]), reinterpret_cast<char*>(buf) + r * HD * 2, g, score_swz<HD>(r));
      mx_put(RAW ? raw[256 * NC + id] : vc[RAW ? 0 : i], mx_scale(vb[i]), reinterpret_cast<char*>(buf + KT * HD) + r * HD * 2, g,
             v_swz<HD>(r));
    }
  };

  // A second pass where an infinite or NaN value met a weight of 0 (a row that does not
  // see it): such values count as 0 there and are added afterwards where they are seen.
  // A third one for sums that are too large.
  int pass = 0;
  float lag = 8.0f, room = 0.0f;  // as in sink_few_kernel
  unsigned long long bad = 0;  // bit t % 64: tile t holds such a value
again:
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.0f;
  m_run = -INFINITY;
  l_run = 0.0f;
  bool odd = false;
  auto step = [&](int t, uint16_t* buf, uint16_t* next) {
    uint16_t *ks = buf, *vs = buf + KT * HD;
    if constexpr (!MX) __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wave's share of tile t is in LDS
    __syncthreads();                                        // every wave's share, and tile t - 1 is no longer read
    if constexpr (MX) {
      if (t + 1 < nt) {
        put(next);
        if (t + 2 < nt) fetch(t + 2);
      }
    } else {
      if (t + 1 < nt) load(t + 1, next);
    }
    if (pass != 0) {
      uint32_t found = 0;
      for (int i = threadIdx.x; i < KT * HD / 2; i += 256) {
        uint32_t* x = reinterpret_cast<uint32_t*>(vs) + i;
        const uint32_t nf = nonfinite2(*x);
        found |= nf;
        if (nf != 0) *x &= (nf & 0x8000u ? 0u : 0xffffu) | (nf & 0x80000000u ? 0u : 0xffff0000u);
      }
      if (__syncthreads_or(found != 0)) bad |= 1ull << (t & 63);
    }
    const int k0 = KT * t;
    if (!wave_on || k0 >= last.hi || (k0 >= sink && k0 + KT <= first.lo)) return;
    const bool masked = k0 + KT > first.hi || (k0 + KT > sink && last.lo > max(k0, sink));

    f32x16_t st[KH];
    const uint32_t kbase = fresh(score_base<HD>(lane));
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int kh = 0; kh < KH; ++kh)
#pragma unroll
      for (int i = 0; i < 16; ++i) st[kh][i] = 0.0f;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
#pragma unroll
      for (int kh = 0; kh < KH; ++kh) {
        const bf16x8_t kf = score_operand(ks, MX ? kbase ^ mx_swz(kk >> 1) << 4 : kbase, kk, 64 * HD * kh);
        st[kh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[kk], st[kh], 0, 0, 0);
      }
    }
    // reads kLead operands ahead of the products (a hint: with copies of single rows in the loop, global_load_lds, the
    // compiler makes every wait for LDS one for all reads, so that the lead ends at every fourth operand)
    __builtin_amdgcn_sched_group_barrier(0x100, kLead, 0);
#pragma unroll
    for (int i = 0; i < KS * KH - kLead; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, kLead, 0);
    __builtin_amdgcn_s_setprio(0);
    if (masked) {
      asm volatile("");  // a branch: as selects they would run for every tile
#pragma unroll
      for (int kh = 0; kh < KH; ++kh)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = k0 + 32 * kh + 8 * (r >> 2) + 4 * hl + (r & 3);
          st[kh][r] = (key < mine.hi) & ((key < sink) | (key >= mine.lo)) ? st[kh][r] : -INFINITY;
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kh = 0; kh < KH; ++kh)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[kh][r]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * ScoreScale<HD>::v;
    const bool grow = mx > m_run + lag;
    if (__any(grow)) {
      const float m_new = grow ? mx : m_run;
      const float alpha = exp2_hw(grow ? m_run - m_new : 0.0f);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
    }
    const float m_use = (m_run == -INFINITY ? 0.0f : m_run) + room;
    // P as two bf16 parts, p = hi + lo: hi's rounding error is lo
    bf16x8_t hi[2 * KH], lo[2 * KH];
    float sum = 0.0f;
#pragma unroll
    for (int tt = 0; tt < 2 * KH; ++tt) {
      uint32_t hw[4], lw[4];
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const int r = 8 * (tt & 1) + e;
        const float pa = exp2_hw(fmaf(st[tt >> 1][r], ScoreScale<HD>::v, -m_use));
        const float pb = exp2_hw(fmaf(st[tt >> 1][r + 1], ScoreScale<HD>::v, -m_use));
        sum += pa + pb;
        hw[e >> 1] = pack_bf16x2(pa, pb);
        lw[e >> 1] = pack_bf16x2(pa - bf_lo(hw[e >> 1]), pb - bf_hi(hw[e >> 1]));
      }
      hi[tt] = __builtin_bit_cast(bf16x8_t, make_uint4(hw[0], hw[1], hw[2], hw[3]));
      lo[tt] = __builtin_bit_cast(bf16x8_t, make_uint4(lw[0], lw[1], lw[2], lw[3]));
    }
    l_run += sum;  // this lane's keys; lane ^ 32 holds the others
    const uint32_t vbase = fresh(v_base<HD>(lane));
#pragma unroll
    for (int tt = 0; tt < 2 * KH; ++tt)
#pragma unroll
      for (int db = 0; db < DB; db += 2) {
        const bf16x8_t v0 = v_operand<HD>(vs, MX ? vbase ^ mx_swz(db) << 4 : vbase, 16 * tt, db);
        const bf16x8_t v1 = v_operand<HD>(vs, MX ? vbase ^ mx_swz(db + 1) << 4 : vbase, 16 * tt, db + 1);
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v0, hi[tt], o[db], 0, 0, 0);
        o[db + 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v1, hi[tt], o[db + 1], 0, 0, 0);
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v0, lo[tt], o[db], 0, 0, 0);
        o[db + 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v1, lo[tt], o[db + 1], 0, 0, 0);
      }
  };
  if (nt > 0) {
    if constexpr (MX) {
      fetch(0);
      put(buf0);
      if (nt > 1) fetch(1);
    } else {
      load(0, buf0);
    }
  }
  for (int t = 0; t < nt; t += 2) {
    step(t, buf0, buf1);
    if (t + 1 < nt) step(t + 1, buf1, buf0);
  }
  const bool wanted = rl < it.nr;
  l_run += __shfl_xor(l_run, 32, 64);
  if (pass < 2) {
    float x = 0.0f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) x = too_large(o[db][i], x);
    x += __shfl_xor(x, 32, 64);
    odd = wanted && x != 0.0f && (pass == 0 || l_run < INFINITY);
  }
  if (pass < 2 && __syncthreads_or(odd)) {
    if (++pass == 2 && odd) {
      lag = 0.0f;
      room = sum_room(it.keys.n);
    }
    goto again;
  }

  if (pass != 0) {
    // the infinite and NaN values that were taken as 0, for the rows that see them
#pragma unroll 1
    for (int t = 0; t < nt; ++t) {
      if ((bad >> (t & 63) & 1) == 0 || !wave_on) continue;
#pragma unroll 1
      for (int x = KT * t; x < min(KT * t + KT, mine.hi); ++x) {
        if (x >= sink && x < mine.lo) continue;
        const size_t row = base + it.keys.row(it.x0 + x);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            float v[4];
            if constexpr (MX) {
              v[0] = v[1] = v[2] = v[3] = a.vs[row * G + db] == 255 ? __uint_as_float(0x7fc00000u) : 0.0f;
            } else {
              const uint2 y = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(a.v) + row * HD + 4 * hl + 32 * db +
                                                              8 * q4);
              v[0] = bf_lo(y.x), v[1] = bf_hi(y.x), v[2] = bf_lo(y.y), v[3] = bf_hi(y.y);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) o[db][4 * q4 + e] += fabsf(v[e]) < INFINITY ? 0.0f : v[e];
          }
      }
    }
  }
  if (!wanted) return;
  if (it.slots == 1) {
    const float inv = l_run != 0.0f ? 1.0f / l_run : 0.0f;
    uint16_t* dst = static_cast<uint16_t*>(a.out) + sink_q(a, it.b, it.j, it.r0 + rl, HD);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        // with no key o is 0
        const uint2 v = make_uint2(pack_bf16x2(o[db][4 * q4 + 0] * inv, o[db][4 * q4 + 1] * inv),
                                   pack_bf16x2(o[db][4 * q4 + 2] * inv, o[db][4 * q4 + 3] * inv));
        *reinterpret_cast<uint2*>(dst + 32 * db + 8 * q4 + 4 * hl) = v;
      }
    return;
  }
  const size_t row = sink_state(a, it.s, it.b, it.j, it.r0 + rl);
  if (hl == 0) {
    a.ml[2 * row] = m_run == -INFINITY ? 0.0f : m_run + room;
    a.ml[2 * row + 1] = l_run;
  }
  if (l_run != 0.0f) {
    float* dst = a.acc + row * HD;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<float4*>(dst + 32 * db + 8 * q4 + 4 * hl) =
            make_float4(o[db][4 * q4 + 0], o[db][4 * q4 + 1], o[db][4 * q4 + 2], o[db][4 * q4 + 3]);
  }
}

// ------------------------------------------------------------------ fp32 K/V

// One workgroup per (16-row block, slot), 16-key blocks to the waves in turn; the
// products, lanes and infinities as in rows_f32_kernel (kvd_rows.hip).  Bound by round trips: no
// load is in flight behind the products (one token over 132 keys of 64: 7.2 us).
constexpr int sink_f32_waves(int hd) { return hd == 64 ? 8 : 4; }  // (8 do not leave the registers for longer rows)
template <int HD>
__global__ __launch_bounds__(64 * sink_f32_waves(HD)) void sink_f32_kernel(SinkArgs a) {
  constexpr int NW = sink_f32_waves(HD), KC = HD / 16, VU = HD / 64;
  __shared__ __align__(16) float part[NW - 1][16][HD + 4];
  __shared__ float ml[NW][16][2];
  const int lane = threadIdx.x & 63, w = wave_id(), rq = lane & 15, lg = lane >> 4;
  SinkItem it;
  if (!sink_item<kRowsWave>(a, it)) return;
  const int nt = (it.n + 15) / 16;
  const size_t base = ((size_t)it.b * a.n_kv + it.j) * a.t_cap + a.t_off;
  const auto row_at = [&](int x) { return (base + it.keys.row(it.x0 + min(x, it.n - 1))) * HD; };
  const int sink = max(a.sink - it.x0, 0);
  SinkRow mine = sink_row_of(a, it.keys, it.p0 + token_of(a, it.r0 + min(rq, it.nr - 1)));
  mine = SinkRow{max(mine.lo, 0) - it.x0, min(mine.hi - it.x0, it.n)};
  const auto sees = [&](int x) { return (x < mine.hi) & ((x < sink) | (x >= mine.lo)); };
  const float* K = static_cast<const float*>(a.k);
  const float* V = static_cast<const float*>(a.v);
  f32x4_t q[KC];
  {
    const float* qs = static_cast<const float*>(a.q) + sink_q(a, it.b, it.j, it.r0 + min(rq, it.nr - 1), HD) + 4 * lg;
#pragma unroll
    for (int c = 0; c < KC; ++c) q[c] = *reinterpret_cast<const f32x4_t*>(qs + 16 * c);
  }
  f32x4_t o[VU][4];
  float m_run, l_run;
  int pass = 0;
  float room = 0.0f;  // as in sink_few_kernel
again:
#pragma unroll
  for (int u = 0; u < VU; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[u][e] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  m_run = -INFINITY;
  l_run = 0.0f;
  for (int t = w; t < nt; t += NW) {
    const int k0 = 16 * t;
    f32x4_t kf[KC], vf[4][VU];
    const float* ks = K + row_at(k0 + rq) + 4 * lg;
#pragma unroll
    for (int c = 0; c < KC; ++c) kf[c] = *reinterpret_cast<const f32x4_t*>(ks + 16 * c);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float* vs = V + row_at(k0 + 4 * lg + i) + 4 * rq;
#pragma unroll
      for (int u = 0; u < VU; ++u) vf[i][u] = *reinterpret_cast<const f32x4_t*>(vs + 64 * u);
    }
    f32x4_t s0 = {0.0f, 0.0f, 0.0f, 0.0f}, s1 = s0;
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[c][e], q[c][e], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[c][e + 1], q[c][e + 1], s1, 0, 0, 0);
      }
    // key k0 + 4 lg + r, row rq
    float sv[4], mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      sv[r] = sees(k0 + 4 * lg + r) ? (s0[r] + s1[r]) * ScoreScale<HD>::v : -INFINITY;
      mx = fmaxf(mx, sv[r]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float m_new = fmaxf(m_run, mx);
    const float m_use = m_new == -INFINITY ? 0.0f : m_new;
    const float alpha = exp2_hw(m_run - m_use);
    m_run = m_new;
    float p[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) p[r] = exp2_hw(sv[r] - (m_use + room));
    l_run = fmaf(l_run, alpha, (p[0] + p[1]) + (p[2] + p[3]));
#pragma unroll
    for (int u = 0; u < VU; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[u][e] *= alpha;
    if (pass != 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int u = 0; u < VU; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) vf[i][u][e] = fabsf(vf[i][u][e]) < INFINITY ? vf[i][u][e] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int u = 0; u < VU; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          o[u][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[i][u][e], p[i], o[u][e], 0, 0, 0);
  }
  l_run += __shfl_xor(l_run, 16, 64);
  l_run += __shfl_xor(l_run, 32, 64);
  if (pass < 2) {
    float x = 0.0f;
#pragma unroll
    for (int u = 0; u < VU; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r) x = too_large(o[u][e][r], x);
    x += __shfl_xor(x, 16, 64);
    x += __shfl_xor(x, 32, 64);
    const bool odd = rq < it.nr && x != 0.0f && (pass == 0 || l_run < INFINITY);
    if (__any(odd)) {
      if (++pass == 2 && odd) room = sum_room(it.keys.n);
      goto again;
    }
  }
  if (pass != 0) {
    // the values that were taken as 0, for the rows that see them
#pragma unroll 1
    for (int t = w; t < nt; t += NW) {
      const int k0 = 16 * t;
#pragma unroll
      for (int u = 0; u < VU; ++u) {
        f32x4_t vf[4];
        float x = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          vf[i] = *reinterpret_cast<const f32x4_t*>(V + row_at(k0 + 4 * lg + i) + 4 * rq + 64 * u);
#pragma unroll
          for (int e = 0; e < 4; ++e) x = fmaf(vf[i][e], 0.0f, x);
        }
        if (!__any(x != 0.0f)) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f32x4_t codes = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int i = 0; i < 4; ++i)
            codes = __builtin_amdgcn_mfma_f32_16x16x4f32(fabsf(vf[i][e]) < INFINITY ? 0.0f : code_of(vf[i][e]),
                                                         sees(k0 + 4 * lg + i) ? 1.0f : 0.0f, codes, 0, 0, 0);
#pragma unroll
          for (int r = 0; r < 4; ++r) o[u][e][r] += poison_of(codes[r]);
        }
      }
    }
  }
  m_run += room;
  // the waves' states, merged by the first in wave order.  o[u][e][r]: dim 64 u + 16 lg + 4 r + e
  if (lg == 0) {
    ml[w][rq][0] = m_run;
    ml[w][rq][1] = l_run;
  }
  if (w > 0) {
#pragma unroll
    for (int u = 0; u < VU; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<float4*>(&part[w - 1][rq][64 * u + 16 * lg + 4 * r]) =
            make_float4(o[u][0][r], o[u][1][r], o[u][2][r], o[u][3][r]);
  }
  __syncthreads();
  if (w > 0 || rq >= it.nr) return;
  float M = m_run;
#pragma unroll
  for (int v = 1; v < NW; ++v) M = fmaxf(M, ml[v][rq][0]);
  const float Mu = M == -INFINITY ? 0.0f : M;
  const float w0 = exp2_hw(m_run - Mu);
  l_run *= w0;
#pragma unroll
  for (int u = 0; u < VU; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int r = 0; r < 4; ++r) o[u][e][r] = add_state(0.0f, w0, o[u][e][r]);
#pragma unroll
  for (int v = 1; v < NW; ++v) {
    const float wt = exp2_hw(ml[v][rq][0] - Mu);
    l_run = fmaf(wt, ml[v][rq][1], l_run);
#pragma unroll
    for (int u = 0; u < VU; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const f32x4_t y = *reinterpret_cast<const f32x4_t*>(&part[v - 1][rq][64 * u + 16 * lg + 4 * r]);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[u][e][r] = add_state(o[u][e][r], wt, y[e]);
      }
  }
  const bool direct = it.slots == 1;
  const size_t row = sink_state(a, it.s, it.b, it.j, it.r0 + rq);
  if (!direct && lg == 0) {
    a.ml[2 * row] = Mu;
    a.ml[2 * row + 1] = l_run;
  }
  if (direct || l_run != 0.0f) {
    float* dst = direct ? static_cast<float*>(a.out) + sink_q(a, it.b, it.j, it.r0 + rq, HD) : a.acc + row * HD;
#pragma unroll
    for (int u = 0; u < VU; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float4 v = make_float4(o[u][0][r], o[u][1][r], o[u][2][r], o[u][3][r]);
        if (direct)
          v = l_run != 0.0f ? make_float4(v.x / l_run, v.y / l_run, v.z / l_run, v.w / l_run)
                            : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        *reinterpret_cast<float4*>(dst + 64 * u + 16 * lg + 4 * r) = v;
      }
  }
}

// ------------------------------------------------------------------ merge

// Rows of up to 8 states, or many rows: a thread takes 4 elements of a row, its states 8 at a time in flight.
// Bound by the states' traffic (2 x 512 tokens of 12 heads of 128, up to 5 states a row: 9 us; with a wave to a row
// 9.9).  RB: rows of the attention's blocks, which know how many slots they have.
template <typename T, int HD, int RB>
__global__ __launch_bounds__(256) void sink_merge_kernel(SinkArgs a) {
  constexpr int TPR = HD / 4;
  const long long idx = (long long)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
  const int c = 4 * (threadIdx.x % TPR);
  const int u = (int)(idx / a.R), r = (int)(idx - (long long)u * a.R);  // neighbours' states lie side by side
  if (u >= a.B * a.n_kv) return;
  const int j = u / a.B, b = u - j * a.B;
  const SinkSeq sq = sink_seq(a.kv_len, a.n_new, a.T, a.N, b);
  const int rows = sq.n * a.g;
  if (r >= rows) return;
  const int r0 = r / RB * RB, p0 = sq.len - sq.n;
  const int S = sink_slots(a, sink_keys(a, p0 + token_of(a, r0), p0 + token_of(a, min(r0 + RB, rows) - 1)));
  if (S == 1) return;
  const size_t step = (size_t)a.n_kv * a.B * a.R, first = sink_state(a, 0, b, j, r);
  const float2* st = reinterpret_cast<const float2*>(a.ml) + first;
  const float* acc = a.acc + first * HD + c;
  float M = -INFINITY, L = 0.0f;
  f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = 0; s0 < S; s0 += 8) {
    float2 ml[8];
    f32x4_t y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      ml[i] = make_float2(-INFINITY, 0.0f);
      if (s0 + i < S) ml[i] = st[(s0 + i) * step];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (s0 + i < S) y[i] = *reinterpret_cast<const f32x4_t*>(acc + (s0 + i) * step * HD);
    float m = M;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (ml[i].y != 0.0f) m = fmaxf(m, ml[i].x);
    const float mu = m == -INFINITY ? 0.0f : m, old = exp2_hw(M - mu);
    M = m;
    L *= old;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = add_state(0.0f, old, x[e]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (ml[i].y == 0.0f) continue;  // an empty state has no acc
      const float wt = exp2_hw(ml[i].x - mu);
      L = fmaf(wt, ml[i].y, L);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = add_state(x[e], wt, y[i][e]);
    }
  }
  T* dst = static_cast<T*>(a.out) + sink_q(a, b, j, r, HD) + c;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = L != 0.0f ? x[e] / L : 0.0f;
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
  else
    *reinterpret_cast<f32x4_t*>(dst) = x;
}

// Few rows of many states: a row by 4 waves (each every 4th state, 8 in flight), lane s taking the
// (max, sum) of state s.
template <typename T, int HD, int RB>
__global__ __launch_bounds__(256) void sink_finish_kernel(SinkArgs a) {
  constexpr int E = HD / 64, WPR = 4;
  __shared__ float part[WPR][HD];
  const int lane = threadIdx.x & 63, w = wave_id();
  const int units = a.B * a.n_kv, r = (int)(blockIdx.x / (uint32_t)units), u = (int)blockIdx.x - r * units;
  const int j = u % a.n_kv, b = u / a.n_kv;
  const SinkSeq sq = sink_seq(a.kv_len, a.n_new, a.T, a.N, b);
  const int rows = sq.n * a.g;
  if (r >= rows) return;
  const int r0 = r / RB * RB, p0 = sq.len - sq.n;
  const SinkKeys keys = sink_keys(a, p0 + token_of(a, r0), p0 + token_of(a, min(r0 + RB, rows) - 1));
  const int S = sink_slots(a, keys);
  if (S == 1) return;
  float2 st = make_float2(-INFINITY, 0.0f);
  if (lane < S) st = *reinterpret_cast<const float2*>(a.ml + 2 * sink_state(a, lane, b, j, r));
  if (st.y == 0.0f) st.x = -INFINITY;
  const float M = wave_max(st.x), Mu = M == -INFINITY ? 0.0f : M;
  const float wt = exp2_hw(st.x - Mu), L = wave_sum(st.y * wt);
  float x[E];
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = 0.0f;
  const float* src = a.acc + sink_state(a, 0, b, j, r) * HD + E * lane;
  const size_t step = (size_t)a.n_kv * a.B * a.R * HD;
  unsigned long long left = __ballot(st.y != 0.0f && lane % WPR == w % WPR);  // an empty state has no acc
  while (left != 0) {
    float y[8][E], ws[8];
    const int n = __popcll(left);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int s = left != 0 ? __builtin_ctzll(left) : 0;
      ws[i] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, wt), s));
      if (left != 0) {
        const float* at = src + (size_t)s * step;
        if constexpr (E == 1) y[i][0] = *at;
        if constexpr (E == 2) {
          const float2 v = *reinterpret_cast<const float2*>(at);
          y[i][0] = v.x, y[i][1] = v.y;
        }
        if constexpr (E == 4) {
          const float4 v = *reinterpret_cast<const float4*>(at);
          y[i][0] = v.x, y[i][1] = v.y, y[i][2] = v.z, y[i][3] = v.w;
        }
      }
      left &= left - 1;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = i >= n ? x[e] : add_state(x[e], ws[i], y[i][e]);
  }
#pragma unroll
  for (int e = 0; e < E; ++e) part[w][E * lane + e] = x[e];
  __syncthreads();
  if (w > 0) return;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    x[e] = part[0][E * lane + e];
#pragma unroll
    for (int v = 1; v < WPR; ++v) x[e] += part[v][E * lane + e];
  }
  T* dst = static_cast<T*>(a.out) + sink_q(a, b, j, r, HD) + E * lane;
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = L != 0.0f ? x[e] / L : 0.0f;
  if constexpr (sizeof(T) == 2) {
    if constexpr (E == 1) *dst = (uint16_t)pack_bf16x2(x[0], x[0]);
    if constexpr (E == 2) *reinterpret_cast<uint32_t*>(dst) = pack_bf16x2(x[0], x[1]);
    if constexpr (E == 4)
      *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) dst[e] = x[e];
  }
}

// ------------------------------------------------------------------ launchers

// bf16 calls of more than kRowsFew rows go to the tiles (us per call in blocks of 16 rows, and in tiles).  Plain, 8
// sequences over 4096 keys: 30 rows of 128 14.6, 16.1; 96 rows 27.7, 19.4; 18 rows of 256 48.5, 36.5; 96 rows 96.7,
// 50.7; with windows of 1024 (16 sequences) 18 rows of 256 25.5, 27.3, 96 rows 49.5, 35.8.  4 bits at head_dim 128 are
// even (18 rows 13.0, 12.8; 96 rows 20.3, 19.1; 16 windows of 1024 16.4, 19.8), at 256 blocks of 16 would be faster
// up to 96 rows (18 rows 21.5, 27.3; 96 rows 41.6, 49.7; windows 17.9, 24.6 and 35.4, 37.6): left to do.

// From as many rows on, those of more than 8 states too are merged by rows side by side (5000 keys of 128: 1200 rows
// 7.2 us, by four waves each 5.1; 3600 rows 6.8 and 9.0).
constexpr long long kSinkManyRows = 2048;

template <typename T, int HD>
static hipError_t launch_sink_t(const SinkArgs& a, hipStream_t st) {
  constexpr bool BF = sizeof(T) == 2;
  const bool mx = a.ks != nullptr, tile = BF && a.R > kRowsFew;
  const int RB = tile ? kRowsTile : kRowsWave;
  const dim3 grid((unsigned)(a.B * a.n_kv), (unsigned)a.S, (unsigned)((a.R + RB - 1) / RB));
  if (tile) {
    if constexpr (BF) {
      if (mx)
        hipLaunchKernelGGL((sink_tile_kernel<HD, true>), grid, dim3(256), 0, st, a);
      else
        hipLaunchKernelGGL((sink_tile_kernel<HD, false>), grid, dim3(256), 0, st, a);
    }
  } else if (mx) {
    hipLaunchKernelGGL((sink_few_kernel<HD, true, T>), grid, dim3(256), 0, st, a);
  } else {
    if constexpr (BF)
      hipLaunchKernelGGL((sink_few_kernel<HD, false, T>), grid, dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL(sink_f32_kernel<HD>, grid, dim3(64 * sink_f32_waves(HD)), 0, st, a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.S == 1) return e;
  const long long rows = (long long)a.B * a.n_kv * a.R;
  const auto finish = [&](auto rb) {
    constexpr int RB_ = decltype(rb)::value, per = 256 / (HD / 4);
    if (a.S > 8 && rows < kSinkManyRows)
      hipLaunchKernelGGL((sink_finish_kernel<T, HD, RB_>), dim3((unsigned)rows), dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL((sink_merge_kernel<T, HD, RB_>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, st, a);
  };
  if (tile)
    finish(IC<kRowsTile>{});
  else
    finish(IC<kRowsWave>{});
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
