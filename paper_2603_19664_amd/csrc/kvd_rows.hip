// Attention of several query rows over stored keys that rows may share:
// kvd_prefix_attn (a prefix that the whole batch attends, then each sequence's own
// rows) and kvd_weighted_attn (the weight every cached key received).
//
//   rows_bf16_kernel    bf16, one launch for both kinds of items: rows_few, at most 16
//                       rows per key range (single tokens), whose waves stream 16-key
//                       blocks each on its own; rows_tile, 128 rows per workgroup that
//                       share key tiles in LDS.  Both products on MFMA.
//   rows_f32_kernel     fp32: 16 rows per workgroup, both products on MFMA 16x16x4 f32.
//   rows_finish_kernel  merges the key ranges' softmax states into out, and adds up
//                       the streamed scores' weights.
//   weight_tile_kernel, weight_f32_kernel
//                       weights of a key tile: its scores once more against every
//                       row that sees it, weighed with the rows' final sums.
//
// Rows.  The rows that read KV head j are (sequence b, token i, head h of the group),
// flat index fr = (b N + i) g + h: a prefix range takes them all, an own range the R =
// N g of one sequence.  Every key range is one slot s of the partial states
//   acc [S][n_kv][B R][hd], ml [S][n_kv][B R][2]  (sum 2^(s - max) V; max, sum),
// in the log2 domain.  A state with sum 0 has no acc.
#include <hip/hip_runtime.h>

#include "kvd_device.hpp"
#include "kvd_launch.h"
#include "kvd_rows_device.hpp"
#include "kvd_rows_layout.h"

namespace kvd {

// What sequence b brings: own rows len, new tokens n (both clamped to the call's sizes).
struct Seq {
  int len, n;
};
__device__ __forceinline__ Seq seq_of(const RowsArgs& a, int b) {
  Seq s;
  s.len = a.own_len != nullptr ? min(max(a.own_len[b], 0), a.T_own) : a.T_own;
  s.n = a.n_new != nullptr ? min(max(a.n_new[b], 0), a.N) : a.N;
  return s;
}
// Own rows that token i of n sees: those up to its own.
__device__ __forceinline__ int rows_seen(const Seq& s, int i) { return i < s.n ? max(s.len - s.n + i + 1, 0) : 0; }

// Whether flat row fr belongs to a new token (the rows behind a sequence's n are left alone).
__device__ __forceinline__ bool row_wanted(const RowsArgs& a, int fr) {
  if (a.n_new == nullptr) return true;
  const int b = fr / a.R;
  return token_of(a, fr - b * a.R) < seq_of(a, b).n;
}

__device__ __forceinline__ size_t slot_row(const RowsArgs& a, int s, int j, int fr) {
  return ((size_t)s * a.n_kv + j) * ((size_t)a.B * a.R) + fr;
}
// Element offset of flat row fr of KV head j in q and out.
__device__ __forceinline__ size_t q_off(const RowsArgs& a, int j, int fr, int hd) {
  const int tok = token_of(a, fr);
  return ((size_t)tok * a.n_q + (size_t)j * a.g + (fr - tok * a.g)) * hd;
}

// Whether the rb rows from row r_blk on of a sequence see no key beyond the call's first slot
// (the first rows of a causal prompt): that slot's workgroup writes out itself, the others
// nothing, and no state is merged (a 3001-token prompt 120.3 us instead of 122.7).
__device__ __forceinline__ bool any_sole_slot(const RowsArgs& a) {  // of a call of several slots
  return a.S_prefix == 0 && !a.own_few && a.sc == nullptr && (a.joint ? a.T_prefix : 0) < a.C_own &&
         (a.own_len != nullptr || a.T_own - a.N < a.C_own);
}
__device__ __forceinline__ bool sole_slot(const RowsArgs& a, const Seq& sq, int r_blk, int rb) {
  if (a.S_prefix + a.S_own == 1) return true;
  if (!any_sole_slot(a)) return false;
  const int seen = rows_seen(sq, token_of(a, min(r_blk + rb, sq.n * a.g) - 1));
  return (long long)(a.joint ? a.T_prefix : 0) + seen <= a.C_own;
}

// A range of keys [k0, k1) of KV head j: of the prefix, or of sequence b's own rows.
struct KeyRange {
  size_t row;  // first key's row in the K and V arrays
  int n;
};
__device__ __forceinline__ KeyRange prefix_range(const RowsArgs& a, int j, int k0, int k1) {
  return KeyRange{(size_t)j * a.p_cap + a.p_off + k0, max(k1 - k0, 0)};
}
__device__ __forceinline__ KeyRange own_range(const RowsArgs& a, int b, int j, int k0, int k1) {
  return KeyRange{((size_t)b * a.n_kv + j) * a.t_cap + a.t_off + k0, max(k1 - k0, 0)};
}

// ------------------------------------------------------------------ 128-row tiles (bf16)

// One workgroup of 4 waves per (128-row block, key range), 32 rows per wave, through
// the range's key tiles: first its prefix keys, then its own ones (one of them empty
// unless the call is joint).  Tile t + 1 is copied into the other LDS buffer while tile
// t is computed.  S^T = K Q^T (A: 32 keys from LDS, B: the wave's rows, in registers):
// a lane holds scores of one row, so its running maximum and sum need one exchange with
// lane ^ 32.  The maximum moves only by steps of more than 2^8, so that O is rescaled
// in few tiles.  O^T += V^T P^T with P^T straight from the score registers, as the sum of
// two bf16 parts (2^-17 of a weight is lost).  Rounded to one part, each weight was off by up to
// 2^-8: the output's error grew from 1.7e-3 to 2.3e-3, and a token's precision hung on how many
// shared its batch (8 prompts over 8192 keys 128 us so, 154 with both parts; a 3001-token
// prompt 110 and 120).
template <int HD>
__device__ __forceinline__ void rows_tile(const RowsArgs& a, int item, uint16_t* buf0, uint16_t* buf1) {
  constexpr int KT = rows_kt(HD), KH = KT / 32, KS = HD / 16, DB = HD / 32, kLead = 4;
  const int lane = threadIdx.x & 63, w = wave_id(), hl = lane >> 5;
  // the item: own (or joint) row blocks first, then the prefix's
  const int nbo = (a.R + kRowsTile - 1) / kRowsTile;
  const int own_items = a.own_few ? 0 : a.B * a.n_kv * nbo * a.S_own;
  const bool own = item < own_items;
  int blk, s, j, b;
  if (own) {
    const int units = a.B * a.n_kv, x = item / units, u = item - x * units;
    j = u % a.n_kv;
    b = u / a.n_kv;
    s = (x + x / a.S_own) % a.S_own;  // from another slot in every block: XCDs (item % 8) share early and late keys
    blk = nbo - 1 - x / a.S_own;  // the last rows see the most keys: first
  } else {
    item -= own_items;
    const int units = a.n_kv * a.S_prefix;
    blk = item / units;
    const int u = item - blk * units;
    j = u % a.n_kv;
    s = u / a.n_kv;
    b = 0;
  }
  const int nr = own ? a.R : a.B * a.R;
  const int fr0 = own ? b * a.R : 0;
  Seq sq{0, 0};
  if (own) sq = seq_of(a, b);
  const int slot = own ? a.S_prefix + s : s;
  const int r_blk = blk * kRowsTile;
  if (own && r_blk >= sq.n * a.g) return;  // no row of this block is asked for
  const bool direct = own ? sole_slot(a, sq, r_blk, kRowsTile) : a.S_prefix + a.S_own == 1;
  if (direct && s > 0) return;
  // key range of the item
  int p0 = 0, p1 = 0, o0 = 0, o1 = 0;
  if (!own) {
    p0 = s * a.C_prefix;
    p1 = min(p0 + a.C_prefix, a.T_prefix);
  } else {
    const int last = min(r_blk + kRowsTile, sq.n * a.g) - 1;
    const int seen = rows_seen(sq, token_of(a, last));  // the block's longest row
    const int base = a.joint ? a.T_prefix : 0;
    const long long k0 = (long long)s * a.C_own, k1 = k0 + a.C_own;
    p0 = (int)min(k0, (long long)base);
    p1 = (int)min(k1, (long long)base);
    o0 = (int)max(k0 - base, 0ll);
    o1 = (int)min(max(k1 - base, 0ll), (long long)seen);
  }
  const KeyRange kp = prefix_range(a, j, p0, p1), ko = own_range(a, b, j, o0, o1);
  const int np = (kp.n + KT - 1) / KT, nt = np + (ko.n + KT - 1) / KT;
  const uint16_t* Kp = static_cast<const uint16_t*>(a.pk) + kp.row * HD;
  const uint16_t* Vp = static_cast<const uint16_t*>(a.pv) + kp.row * HD;
  const uint16_t* Ko = static_cast<const uint16_t*>(a.k) + ko.row * HD;
  const uint16_t* Vo = static_cast<const uint16_t*>(a.v) + ko.row * HD;

  // this lane's row
  const int rl = r_blk + 32 * w + (lane & 31);
  const bool wave_on = r_blk + 32 * w < (own ? sq.n * a.g : nr);
  const int fr = fr0 + min(rl, nr - 1);
  // keys of the item's own range that the row sees; every prefix key is seen
  const int lim = own && rl < nr ? min(rows_seen(sq, token_of(a, rl)) - o0, ko.n) : 0;
  // own keys that every row of the wave's block sees
  const int all = own ? min(rows_seen(sq, token_of(a, min(r_blk + 32 * w, nr - 1))) - o0, ko.n) : 0;
  bf16x8_t qf[KS];
  {
    const uint16_t* qs = static_cast<const uint16_t*>(a.q) + q_off(a, j, fr, HD) + 8 * hl;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8_t*>(qs + 16 * ks);
  }
  f32x16_t o[DB];
  float m_run, l_run;  // in units of the scaled score

  auto load = [&](int t, uint16_t* buf) {
    const int k = (t < np ? t : t - np) * KT, n = (t < np ? kp.n : ko.n) - k;
    copy_tile<HD, KT, true>((t < np ? Kp : Ko) + (size_t)k * HD, n, buf);
    copy_tile<HD, KT, false>((t < np ? Vp : Vo) + (size_t)k * HD, n, buf + KT * HD);
  };
  // A second pass where an infinite or NaN value met a weight of 0 (a row that does not
  // see it): such values count as 0 there and are added afterwards where they are seen.
  int pass = 0;
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
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wave's share of tile t is in LDS
    __syncthreads();                     // every wave's share, and tile t - 1 is no longer read
    if (t + 1 < nt) load(t + 1, next);
    if (pass == 1) {
      uint32_t found = 0;
      for (int i = threadIdx.x; i < KT * HD / 2; i += 256) {
        uint32_t* x = reinterpret_cast<uint32_t*>(vs) + i;
        const uint32_t nf = nonfinite2(*x);
        found |= nf;
        if (nf != 0) *x &= (nf & 0x8000u ? 0u : 0xffffu) | (nf & 0x80000000u ? 0u : 0xffff0000u);
      }
      if (__syncthreads_or(found != 0)) bad |= 1ull << (t & 63);
    }
    if (!wave_on) return;
    const bool is_own = t >= np;
    const int k0 = (is_own ? t - np : t) * KT;
    const int row_lim = is_own ? lim : kp.n;
    const bool masked = k0 + KT > (is_own ? all : kp.n);

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
        const bf16x8_t kf = score_operand(ks, kbase, kk, 64 * HD * kh);
        st[kh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[kk], st[kh], 0, 0, 0);
      }
    }
    // reads kLead operands ahead of the products
    __builtin_amdgcn_sched_group_barrier(0x100, kLead, 0);
#pragma unroll
    for (int i = 0; i < KS * KH - kLead; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, kLead, 0);
    __builtin_amdgcn_s_setprio(0);
    if (masked) {
      asm volatile("");  // a branch: as selects they ran for every tile (a third of its VALU work)
#pragma unroll
      for (int kh = 0; kh < KH; ++kh)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = k0 + 32 * kh + 8 * (r >> 2) + 4 * hl + (r & 3);
          st[kh][r] = key < row_lim ? st[kh][r] : -INFINITY;
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kh = 0; kh < KH; ++kh)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[kh][r]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * ScoreScale<HD>::v;
    const bool grow = mx > m_run + 8.0f;
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
    const float m_use = m_run == -INFINITY ? 0.0f : m_run;
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
        const bf16x8_t v0 = v_operand<HD>(vs, vbase, 16 * tt, db), v1 = v_operand<HD>(vs, vbase, 16 * tt, db + 1);
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v0, hi[tt], o[db], 0, 0, 0);
        o[db + 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v1, hi[tt], o[db + 1], 0, 0, 0);
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v0, lo[tt], o[db], 0, 0, 0);
        o[db + 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v1, lo[tt], o[db + 1], 0, 0, 0);
      }
  };
  if (nt > 0) load(0, buf0);
  for (int t = 0; t < nt; t += 2) {
    step(t, buf0, buf1);
    if (t + 1 < nt) step(t + 1, buf1, buf0);
  }
  // O holds no infinity or NaN unless V or the scores did; rows nobody asked for may
  const bool wanted = rl < nr && row_wanted(a, fr);
  if (pass == 0 && wanted) {
    float x = 0.0f;  // 0 o: 4 bytes of code each; a small call waits for its instructions, 60 ns for 64 bytes
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) x = fmaf(o[db][i], 0.0f, x);
    odd = x != 0.0f;
  }
  if (pass == 0 && __syncthreads_or(odd)) {
    pass = 1;
    goto again;
  }
  l_run += __shfl_xor(l_run, 32, 64);

  if (pass == 1) {
    // the infinite and NaN values that pass 1 took as 0, for the rows that see them
#pragma unroll 1
    for (int t = 0; t < nt; ++t) {
      if ((bad >> (t & 63) & 1) == 0 || !wave_on) continue;
      const bool is_own = t >= np;
      const int k0 = (is_own ? t - np : t) * KT;
#pragma unroll 1
      for (int k = k0; k < min(k0 + KT, is_own ? lim : kp.n); ++k) {
        const uint16_t* vr = (is_own ? Vo : Vp) + (size_t)k * HD + 4 * hl;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const uint2 y = *reinterpret_cast<const uint2*>(vr + 32 * db + 8 * q4);
            const float v[4] = {bf_lo(y.x), bf_hi(y.x), bf_lo(y.y), bf_hi(y.y)};
#pragma unroll
            for (int e = 0; e < 4; ++e) o[db][4 * q4 + e] += fabsf(v[e]) < INFINITY ? 0.0f : v[e];
          }
      }
    }
  }
  if (!wanted) return;
  const float m_out = m_run == -INFINITY ? 0.0f : m_run;
  const size_t row = slot_row(a, slot, j, fr);
  if (hl == 0) {
    a.ml[2 * row] = m_out;
    a.ml[2 * row + 1] = l_run;
    if (direct && a.lse != nullptr)
      a.lse[(size_t)j * a.B * a.R + fr] = l_run != 0.0f ? m_out + __builtin_amdgcn_logf(l_run) : INFINITY;
  }
  if (direct) {
    const float inv = l_run != 0.0f ? 1.0f / l_run : 0.0f;
    uint16_t* dst = static_cast<uint16_t*>(a.out) + q_off(a, j, fr, HD);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        // with no key o is 0
        const uint2 v = make_uint2(pack_bf16x2(o[db][4 * q4 + 0] * inv, o[db][4 * q4 + 1] * inv),
                                   pack_bf16x2(o[db][4 * q4 + 2] * inv, o[db][4 * q4 + 3] * inv));
        *reinterpret_cast<uint2*>(dst + 32 * db + 8 * q4 + 4 * hl) = v;
      }
  } else if (l_run != 0.0f) {
    float* dst = a.acc + row * HD;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<float4*>(dst + 32 * db + 8 * q4 + 4 * hl) =
            make_float4(o[db][4 * q4 + 0], o[db][4 * q4 + 1], o[db][4 * q4 + 2], o[db][4 * q4 + 3]);
  }
}

// ------------------------------------------------------------------ at most 16 rows (bf16)

// Copies 16 rows of HD elements into a wave's LDS slice (rows past n - 1 repeat row n - 1),
// chunks permuted: score operands as in copy_tile; V by 2 (r % 8) (head_dim 64: 2 (r / 2 %
// 4)), its reads taking 32 bytes of 8 rows at a time.
template <int HD, bool SCORE>
__device__ __forceinline__ void copy16(const uint16_t* src, int n, uint16_t* dst) {
  constexpr int CPR = HD / 8, RPI = 64 / CPR, CH = 16 / RPI;
  const int lane = threadIdx.x & 63, r0 = lane / CPR, ch = lane % CPR;
  const __amdgpu_buffer_rsrc_t res =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(src), (short)0, 16 * HD * 2, 0x00027000);
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int r = r0 + RPI * i;
    const int col = 16 * (ch ^ (SCORE ? score_swz<HD>(r) : few_v_swz<HD>(r)));
    __builtin_amdgcn_raw_ptr_buffer_load_lds(res, (__attribute__((address_space(3))) void*)(dst + 512 * i), 16,
                                             min(r, n - 1) * HD * 2 + col, 0, 0, 0);
  }
}

// One workgroup of 4 waves per (unit, split): units 0 .. B n_kv - 1 are the own rows of (b,
// j) in S_own splits (of a joint call all keys, prefix and own, at once), the rest the prefix
// of KV head j in S_prefix splits.  A split's 16-key
// blocks go to the waves in turn, and each wave streams its own through its own slice of
// LDS, with no barrier: HBM-bound, so what matters is loads in flight (head_dim 256: K and
// V of one block, K refilled as soon as the scores are taken, V after its product; smaller
// ones: two blocks).  Scores S^T = K Q^T on MFMA 16x16x32, one row per column; O^T += V^T P^T
// on 16x16x16 with P^T straight from the score registers, as the sum of two bf16 parts
// (2^-17 of a weight is lost; the matrix unit idles here anyway).  The waves' states meet in
// LDS.  With a.sc the scores of own keys are kept for the weights.
template <int HD>
__device__ __forceinline__ void rows_few(const RowsArgs& a, int item, uint16_t* buf0, uint16_t* buf1,
                                         float (*ml)[16][2]) {
  constexpr int NW = 4, KC = HD / 32, DB = HD / 16;
  constexpr bool ONE = HD == 256;  // one block at a time: K in buf0, V in buf1
  constexpr int SLICE = rows_kt(HD) * HD / 2;
  typedef short s16x4_t __attribute__((ext_vector_type(4)));
  const int tid = threadIdx.x, lane = tid & 63, w = wave_id(), hq = lane & 15, lg = lane >> 4;
  const int own_items = a.own_few ? a.B * a.n_kv * a.S_own : 0;
  const bool own = item < own_items;
  if (!own) item -= own_items;
  const int units = own ? a.B * a.n_kv : a.n_kv;
  const int S = own ? a.S_own : a.S_prefix;
  const int s = item / units, u = item - s * units;
  const int j = u % a.n_kv, b = u / a.n_kv;
  const int slot = own ? a.S_prefix + s : s;
  const int nr = own ? a.R : a.B * a.R;
  const int fr0 = own ? b * a.R : 0;
  Seq sq{0, 0};
  if (own) sq = seq_of(a, b);
  if (own && sq.n == 0) return;  // no row of this sequence is asked for
  // the split's keys: of the prefix (a prefix unit's split; all of a joint call's), then of
  // the sequence's own rows
  const int T = own ? sq.len : a.T_prefix;
  const int nblk_all = (T + kSaBlock - 1) / kSaBlock;
  const int k0 = kSaBlock * sa_first_block(s, nblk_all, S);
  const int nk = max(min(T, kSaBlock * sa_first_block(s + 1, nblk_all, S)) - k0, 0);
  const KeyRange kp = own ? prefix_range(a, j, 0, a.joint ? a.T_prefix : 0) : prefix_range(a, j, k0, k0 + nk);
  const KeyRange ko = own ? own_range(a, b, j, k0, k0 + nk) : KeyRange{0, 0};
  const int pblk = (kp.n + kSaBlock - 1) / kSaBlock, nblk = pblk + (ko.n + kSaBlock - 1) / kSaBlock;
  const int nb = nblk > w ? (nblk - 1 - w) / NW + 1 : 0;  // this wave's blocks: w, w + NW, ..
  const uint16_t* Kp = static_cast<const uint16_t*>(a.pk) + kp.row * HD;
  const uint16_t* Vp = static_cast<const uint16_t*>(a.pv) + kp.row * HD;
  const uint16_t* Ko = static_cast<const uint16_t*>(a.k) + ko.row * HD;
  const uint16_t* Vo = static_cast<const uint16_t*>(a.v) + ko.row * HD;
  // own keys of this split that the lane's row sees, and that every row sees
  const int lim = hq < nr && own ? min(rows_seen(sq, token_of(a, hq)) - k0, ko.n) : 0;
  const int all = own ? min(rows_seen(sq, 0) - k0, ko.n) : 0;
  float* sc_row = a.sc != nullptr && own && hq < nr
                      ? a.sc + (((size_t)b * a.n_kv + j) * a.R + hq) * a.sc_ld + k0 + 4 * lg
                      : nullptr;

  uint16_t* const sl0 = buf0 + SLICE * w;
  uint16_t* const sl1 = buf1 + SLICE * w;
  auto load_k = [&](int i, uint16_t* dst) {
    const int x = w + NW * i;
    const int kb = kSaBlock * (x < pblk ? x : x - pblk), n = x < pblk ? kp.n : ko.n;
    copy16<HD, true>((x < pblk ? Kp : Ko) + (size_t)kb * HD, n - kb, dst);
  };
  auto load_v = [&](int i, uint16_t* dst) {
    const int x = w + NW * i;
    const int kb = kSaBlock * (x < pblk ? x : x - pblk), n = x < pblk ? kp.n : ko.n;
    copy16<HD, false>((x < pblk ? Vp : Vo) + (size_t)kb * HD, n - kb, dst);
  };
  // every LDS read of the wave is done: its slice may be written again
  auto reads_done = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
  };
  // queries first: the loop's wait for them then leaves the copies in flight
  bf16x8_t qf[KC];
  {
    const uint16_t* qs = static_cast<const uint16_t*>(a.q) + q_off(a, j, fr0 + min(hq, nr - 1), HD) + 8 * lg;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      u32x4_t v = *reinterpret_cast<const u32x4_t*>(qs + 32 * c);
      if (hq >= nr) v = u32x4_t{0u, 0u, 0u, 0u};
      qf[c] = __builtin_bit_cast(bf16x8_t, v);
    }
  }
  if constexpr (ONE) {
    if (nb > 0) {
      load_k(0, sl0);
      load_v(0, sl1);
    }
  } else {
    if (nb > 0) {
      load_k(0, sl0);
      load_v(0, sl0 + SLICE / 2);
    }
    if (nb > 1) {
      load_k(1, sl1);
      load_v(1, sl1 + SLICE / 2);
    }
  }

  const uint32_t kbase = hq * HD * 2 + ((lg ^ score_swz<HD>(hq)) << 4);
  const int vrow = 4 * lg + (hq >> 2);
  const uint32_t vbase = vrow * HD * 2 + ((((hq & 3) >> 1) ^ few_v_swz<HD>(vrow)) << 4) + 8 * (hq & 1);

  f32x4_t o[DB];
  float m_run, l_run;
  // as in rows_tile: a second pass without infinite and NaN values, which the parts of a weight
  // (lo is 0 or negative as often as not) and the weights of rows that do not see them make NaN
  int pass = 0;
  unsigned long long bad = 0;  // bit i % 64: block i of the wave holds such a value
again:
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  m_run = -INFINITY;
  l_run = 0.0f;
  bool odd = false;
  // NEXT (head_dim 256): whether another block follows; a condition inside the loop made the
  // compiler wait for V before K was read
  auto step = [&](auto next, int i, uint16_t* ks, uint16_t* vs) {
    constexpr bool NEXT = decltype(next)::value != 0;
    const bool is_own = w + NW * i >= pblk;
    const int kb = kSaBlock * (w + NW * i - (is_own ? pblk : 0));
    const int row_lim = is_own ? lim : kp.n;
    const bool masked = kb + kSaBlock > (is_own ? all : kp.n);
    // this block's K (head_dim 256; V was issued after it), or K and V (the next block's
    // were): copies complete in order
    if (ONE || i + 1 < nb)
      wait_copies<ONE ? KC : 2 * KC>();
    else
      wait_copies<0>();
    f32x4_t st = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < KC; ++c)
      st = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
          *reinterpret_cast<const bf16x8_t*>(reinterpret_cast<const char*>(ks) + (kbase ^ (c << 6))), qf[c], st, 0, 0,
          0);
    if constexpr (ONE) {
      reads_done();
      if constexpr (NEXT) load_k(i + 1, ks);
    }
    // st[r]: key kb + 4 lg + r, row hq
    float sv[4], mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      sv[r] = st[r] * ScoreScale<HD>::v;
      if (masked) sv[r] = kb + 4 * lg + r < row_lim ? sv[r] : -INFINITY;
      mx = fmaxf(mx, sv[r]);
    }
    if (sc_row != nullptr && is_own && pass == 0)
      *reinterpret_cast<float4*>(sc_row + kb) = make_float4(sv[0], sv[1], sv[2], sv[3]);
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const bool grow = mx > m_run + 8.0f;
    if (__any(grow)) {
      const float m_new = grow ? mx : m_run;
      const float alpha = exp2_hw(grow ? m_run - m_new : 0.0f);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= alpha;
    }
    const float m_use = m_run == -INFINITY ? 0.0f : m_run;
    float p[4], lo[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) p[r] = exp2_hw(sv[r] - m_use);
    l_run += (p[0] + p[1]) + (p[2] + p[3]);
    const uint2 ph = make_uint2(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]));
    lo[0] = p[0] - bf_lo(ph.x);
    lo[1] = p[1] - bf_hi(ph.x);
    lo[2] = p[2] - bf_lo(ph.y);
    lo[3] = p[3] - bf_hi(ph.y);
    const uint2 pl = make_uint2(pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3]));
    const s16x4_t pfh = __builtin_bit_cast(s16x4_t, ph), pfl = __builtin_bit_cast(s16x4_t, pl);
    if constexpr (ONE) wait_copies<NEXT ? KC : 0>();  // V; the next block's K was issued after it
    if (pass == 1) {
      uint32_t found = 0;
#pragma unroll 1
      for (int x = lane; x < 16 * HD / 2; x += 64) {
        uint32_t* at = reinterpret_cast<uint32_t*>(vs) + x;
        const uint32_t f = nonfinite2(*at);
        found |= f;
        if (f != 0) *at &= (f & 0x8000u ? 0u : 0xffffu) | (f & 0x80000000u ? 0u : 0xffff0000u);
      }
      if (__any(found != 0)) bad |= 1ull << (i & 63);
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const s16x4_t vf = __builtin_bit_cast(
          s16x4_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4_t*)(
                       reinterpret_cast<char*>(vs) + (vbase ^ (db << 5)))));
      o[db] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vf, pfh, o[db], 0, 0, 0);
      o[db] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vf, pfl, o[db], 0, 0, 0);
    }
    reads_done();
    if constexpr (ONE) {
      if constexpr (NEXT) load_v(i + 1, vs);
    } else {
      if (i + 2 < nb) {
        load_k(i + 2, ks);
        load_v(i + 2, vs);
      }
    }
  };
  if constexpr (ONE) {
    for (int i = 0; i + 1 < nb; ++i) step(IC<1>{}, i, sl0, sl1);
    if (nb > 0) step(IC<0>{}, nb - 1, sl0, sl1);
  } else {
    for (int i = 0; i < nb; i += 2) {
      step(IC<0>{}, i, sl0, sl0 + SLICE / 2);
      if (i + 1 < nb) step(IC<0>{}, i + 1, sl1, sl1 + SLICE / 2);
    }
  }
  if (pass == 0 && hq < nr && row_wanted(a, fr0 + hq)) {
    float x = 0.0f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 4; ++e) x = fmaf(o[db][e], 0.0f, x);
    odd = x != 0.0f;
  }
  if (pass == 0 && __any(odd)) {
    pass = 1;
    if constexpr (ONE) {
      load_k(0, sl0);
      load_v(0, sl1);
    } else {
      load_k(0, sl0);
      load_v(0, sl0 + SLICE / 2);
      if (nb > 1) {
        load_k(1, sl1);
        load_v(1, sl1 + SLICE / 2);
      }
    }
    goto again;
  }
  if (pass == 1) {
    // the values that pass 1 took as 0, for the rows that see them
#pragma unroll 1
    for (int i = 0; i < nb; ++i) {
      if ((bad >> (i & 63) & 1) == 0) continue;
      const bool is_own = w + NW * i >= pblk;
      const int kb = kSaBlock * (w + NW * i - (is_own ? pblk : 0));
#pragma unroll 1
      for (int t = kb; t < min(kb + kSaBlock, is_own ? lim : kp.n); ++t) {
        const uint16_t* vr = (is_own ? Vo : Vp) + (size_t)t * HD + 4 * lg;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const uint2 y = *reinterpret_cast<const uint2*>(vr + 16 * db);
          const float v[4] = {bf_lo(y.x), bf_hi(y.x), bf_lo(y.y), bf_hi(y.y)};
#pragma unroll
          for (int e = 0; e < 4; ++e) o[db][e] += fabsf(v[e]) < INFINITY ? 0.0f : v[e];
        }
      }
    }
  }
  l_run += __shfl_xor(l_run, 16, 64);
  l_run += __shfl_xor(l_run, 32, 64);

  // The waves' states into LDS (elements below HD / 2 of the 16 rows in buf0, the others
  // in buf1, 16-byte chunks permuted by the row), then merged in wave order: the slot's
  // state, or with one slot the output.
  __syncthreads();
  constexpr int HH = HD / 2, CM = HH / 4 - 1;
  float* f0 = reinterpret_cast<float*>(buf0);
  float* f1 = reinterpret_cast<float*>(buf1);
  if (lg == 0) {
    ml[w][hq][0] = m_run;
    ml[w][hq][1] = l_run;
  }
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    float* f = db < DB / 2 ? f0 : f1;
    const int c = (4 * db + lg) & CM;
    *reinterpret_cast<f32x4_t*>(f + (w * 16 + hq) * HH + 4 * (c ^ (hq & CM))) = o[db];
  }
  __syncthreads();
  const bool direct = a.S_prefix + a.S_own == 1;
  for (int i = tid; i < nr * (HD / 4); i += 64 * NW) {
    const int h = i / (HD / 4), c4 = i - h * (HD / 4);
    const float* f = c4 <= CM ? f0 : f1;
    float M = -INFINITY;
#pragma unroll
    for (int v = 0; v < NW; ++v) M = fmaxf(M, ml[v][h][0]);
    const float Mu = M == -INFINITY ? 0.0f : M;
    f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
    float L = 0.0f;
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      const float wt = exp2_hw(ml[v][h][0] - Mu);
      x += wt * *reinterpret_cast<const f32x4_t*>(f + (v * 16 + h) * HH + 4 * ((c4 & CM) ^ (h & CM)));
      L = fmaf(wt, ml[v][h][1], L);
    }
    if (fmaf(x[0], 0.0f, fmaf(x[1], 0.0f, fmaf(x[2], 0.0f, x[3] * 0.0f))) != 0.0f) {  // 0 x infinity, perhaps
      x = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
      for (int v = 0; v < NW; ++v) {
        const float wt = exp2_hw(ml[v][h][0] - Mu);
        const f32x4_t y = *reinterpret_cast<const f32x4_t*>(f + (v * 16 + h) * HH + 4 * ((c4 & CM) ^ (h & CM)));
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = add_state(x[e], wt, y[e]);
      }
    }
    const size_t row = slot_row(a, slot, j, fr0 + h);
    if (direct) {
      if (row_wanted(a, fr0 + h)) {
        const float inv = L != 0.0f ? 1.0f / L : 0.0f;
        uint2 y = make_uint2(0u, 0u);
        if (L != 0.0f) y = make_uint2(pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv));
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + q_off(a, j, fr0 + h, HD) + 4 * c4) = y;
      }
    } else {
      *reinterpret_cast<f32x4_t*>(a.acc + row * HD + 4 * c4) = x;
    }
    if (c4 == 0) {
      a.ml[row * 2] = Mu;
      a.ml[row * 2 + 1] = L;
    }
  }
}

// Workgroups 0 .. tile_items - 1 take tiles, the rest few-row splits: the matrix work of the
// ones runs beside the memory traffic of the others.  The two buffers are two objects,
// every access naming one: a copy in flight into one is then known not to touch the other
// (of one array, every LDS read waited for all copies: 8 prompts over 8192 keys 160 us
// instead of 147, both with weights of one part).
template <int HD>
__global__ __launch_bounds__(256, 2) void rows_bf16_kernel(RowsArgs a, int tile_items) {
  constexpr int KT = rows_kt(HD);
  __shared__ __align__(1024) uint16_t buf0[2 * KT * HD], buf1[2 * KT * HD];
  __shared__ float ml[4][16][2];
  if ((int)blockIdx.x < tile_items)
    rows_tile<HD>(a, (int)blockIdx.x, buf0, buf1);
  else
    rows_few<HD>(a, (int)blockIdx.x - tile_items, buf0, buf1, ml);
}

// ------------------------------------------------------------------ fp32

// One workgroup of 4 waves per (16-row block, key range); the range's 16-key blocks go to
// the waves in turn, on v_mfma_f32_16x16x4_f32.
// Scores S^T = K Q^T: lane (row lane % 16, group lg = lane / 16) holds elements 16 c + 4
// lg .. + 3 of a key (A) and of its query row (B); MFMA e of chunk c takes element e.
// P V: O^T = V^T P^T, step t takes the keys 4 lg + t, whose weights the lanes hold; a
// lane's 16 bytes of V row 4 lg + t (dims 64 u + 4 (lane % 16) ..) are the A operands of
// four MFMAs, MFMA e giving dims 64 u + 4 i + e.  Both operands come straight from memory;
// LDS only merges the waves.  With a.sc (at most 16 rows) the scores of own keys are kept
// for the weights.  Masked keys: score -inf.  Where O comes out non-finite, a second pass takes
// V's non-finite values out of the products, and their codes (code_of), summed over the
// keys of a block that a row sees, put them back after the last rescaling.
template <int HD>
__global__ __launch_bounds__(256) void rows_f32_kernel(RowsArgs a) {
  constexpr int KC = HD / 16, VU = HD / 64;
  __shared__ __align__(16) float part[3][16][HD + 4];
  __shared__ float ml[4][16][2];
  __shared__ int passes[4];
  const int lane = threadIdx.x & 63, w = wave_id(), rq = lane & 15, lg = lane >> 4;
  const int nbo = (a.R + kRowsWave - 1) / kRowsWave;
  const int own_items = a.B * a.n_kv * nbo * a.S_own;
  const bool own = (int)blockIdx.x < own_items;
  int blk, s, j, b;
  if (own) {
    const int units = a.B * a.n_kv, x = (int)blockIdx.x / units, u = (int)blockIdx.x - x * units;
    j = u % a.n_kv;
    b = u / a.n_kv;
    s = (x + x / a.S_own) % a.S_own;  // from another slot in every block: XCDs (item % 8) share early and late keys
    blk = nbo - 1 - x / a.S_own;
  } else {
    const int item = (int)blockIdx.x - own_items, units = a.n_kv * a.S_prefix;
    blk = item / units;
    const int u = item - blk * units;
    j = u % a.n_kv;
    s = u / a.n_kv;
    b = 0;
  }
  const int nr = own ? a.R : a.B * a.R;
  const int fr0 = own ? b * a.R : 0;
  Seq sq{0, 0};
  if (own) sq = seq_of(a, b);
  const int slot = own ? a.S_prefix + s : s;
  const int r_blk = blk * kRowsWave;
  if (own && r_blk >= sq.n * a.g) return;
  const bool direct = own ? sole_slot(a, sq, r_blk, kRowsWave) : a.S_prefix + a.S_own == 1;
  if (direct && s > 0) return;
  int p0 = 0, p1 = 0, o0 = 0, o1 = 0;
  if (!own) {
    p0 = s * a.C_prefix;
    p1 = min(p0 + a.C_prefix, a.T_prefix);
  } else {
    const int last = min(r_blk + kRowsWave, sq.n * a.g) - 1;
    const int seen = rows_seen(sq, token_of(a, last));
    const int base = a.joint ? a.T_prefix : 0;
    const long long k0 = (long long)s * a.C_own, k1 = k0 + a.C_own;
    p0 = (int)min(k0, (long long)base);
    p1 = (int)min(k1, (long long)base);
    o0 = (int)max(k0 - base, 0ll);
    o1 = (int)min(max(k1 - base, 0ll), (long long)seen);
  }
  const KeyRange kp = prefix_range(a, j, p0, p1), ko = own_range(a, b, j, o0, o1);
  const int np = (kp.n + 15) / 16, nt = np + (ko.n + 15) / 16;
  const int rl = r_blk + rq;
  const int fr = fr0 + min(rl, nr - 1);
  const int lim = own && rl < nr ? min(rows_seen(sq, token_of(a, rl)) - o0, ko.n) : 0;

  f32x4_t q[KC];
  {
    const float* qs = static_cast<const float*>(a.q) + q_off(a, j, fr, HD) + 4 * lg;
#pragma unroll
    for (int c = 0; c < KC; ++c) q[c] = *reinterpret_cast<const f32x4_t*>(qs + 16 * c);
  }
  f32x4_t o[VU][4];
  float m_run, l_run;
  const bool wanted = rl < nr && row_wanted(a, fr);
  int pass = 0;
again:
#pragma unroll
  for (int u = 0; u < VU; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[u][e] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  m_run = -INFINITY;
  l_run = 0.0f;
  for (int t = w; t < nt; t += 4) {
    const bool is_own = t >= np;
    const KeyRange& kr = is_own ? ko : kp;
    const float* K = static_cast<const float*>(is_own ? a.k : a.pk) + kr.row * HD;
    const float* V = static_cast<const float*>(is_own ? a.v : a.pv) + kr.row * HD;
    const int k0 = 16 * (is_own ? t - np : t);
    const int row_lim = is_own ? lim : kp.n;
    f32x4_t kf[KC], vf[4][VU];
    const float* ks = K + (size_t)min(k0 + rq, kr.n - 1) * HD + 4 * lg;
#pragma unroll
    for (int c = 0; c < KC; ++c) kf[c] = *reinterpret_cast<const f32x4_t*>(ks + 16 * c);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float* vs = V + (size_t)min(k0 + 4 * lg + i, kr.n - 1) * HD + 4 * rq;
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
      sv[r] = k0 + 4 * lg + r < row_lim ? (s0[r] + s1[r]) * ScoreScale<HD>::v : -INFINITY;
      mx = fmaxf(mx, sv[r]);
    }
    if (a.sc != nullptr && is_own && rl < nr && pass == 0) {
      float* sc = a.sc + (((size_t)b * a.n_kv + j) * a.R + rl) * a.sc_ld + o0 + k0 + 4 * lg;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (k0 + 4 * lg + r < ko.n) sc[r] = sv[r];
    }
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float m_new = fmaxf(m_run, mx);
    const float m_use = m_new == -INFINITY ? 0.0f : m_new;
    const float alpha = exp2_hw(m_run - m_use);
    m_run = m_new;
    float p[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) p[r] = exp2_hw(sv[r] - m_use);
    l_run = fmaf(l_run, alpha, (p[0] + p[1]) + (p[2] + p[3]));
#pragma unroll
    for (int u = 0; u < VU; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[u][e] *= alpha;
    if (pass == 1) {
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
  if (pass == 0) {
    float x = 0.0f;
#pragma unroll
    for (int u = 0; u < VU; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r) x = fmaf(o[u][e][r], 0.0f, x);
    if (__any(wanted && x != 0.0f)) {
      pass = 1;
      goto again;
    }
  } else {
    // the values that pass 1 took as 0, for the rows that see them
#pragma unroll 1
    for (int t = w; t < nt; t += 4) {
      const bool is_own = t >= np;
      const KeyRange& kr = is_own ? ko : kp;
      const float* V = static_cast<const float*>(is_own ? a.v : a.pv) + kr.row * HD;
      const int k0 = 16 * (is_own ? t - np : t), row_lim = is_own ? lim : kp.n;
#pragma unroll
      for (int u = 0; u < VU; ++u) {
        f32x4_t vf[4];
        float x = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          vf[i] = *reinterpret_cast<const f32x4_t*>(V + (size_t)min(k0 + 4 * lg + i, kr.n - 1) * HD + 4 * rq + 64 * u);
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
                                                         k0 + 4 * lg + i < row_lim ? 1.0f : 0.0f, codes, 0, 0, 0);
#pragma unroll
          for (int r = 0; r < 4; ++r) o[u][e][r] += poison_of(codes[r]);
        }
      }
    }
  }
  l_run += __shfl_xor(l_run, 16, 64);
  l_run += __shfl_xor(l_run, 32, 64);
  // the waves' states, merged by the first in wave order.  o[u][e][r]: dim 64 u + 16 lg + 4
  // r + e
  if (lg == 0) {
    ml[w][rq][0] = m_run;
    ml[w][rq][1] = l_run;
  }
  if (lane == 0) passes[w] = pass;
  if (w > 0) {
#pragma unroll
    for (int u = 0; u < VU; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<float4*>(&part[w - 1][rq][64 * u + 16 * lg + 4 * r]) =
            make_float4(o[u][0][r], o[u][1][r], o[u][2][r], o[u][3][r]);
  }
  __syncthreads();
  if (w > 0 || !wanted) return;
  float M = m_run;
#pragma unroll
  for (int v = 1; v < 4; ++v) M = fmaxf(M, ml[v][rq][0]);
  const float Mu = M == -INFINITY ? 0.0f : M;
  // SPOILT: a wave took its second pass, so that states may hold infinities
  auto merge = [&](auto spoilt) {
    constexpr bool SPOILT = decltype(spoilt)::value != 0;
    const float w0 = exp2_hw(m_run - Mu);
    l_run *= w0;
#pragma unroll
    for (int u = 0; u < VU; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[u][e][r] = SPOILT ? add_state(0.0f, w0, o[u][e][r]) : w0 * o[u][e][r];
#pragma unroll
    for (int v = 1; v < 4; ++v) {
      const float wt = exp2_hw(ml[v][rq][0] - Mu);
      l_run = fmaf(wt, ml[v][rq][1], l_run);
#pragma unroll
      for (int u = 0; u < VU; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const f32x4_t y = *reinterpret_cast<const f32x4_t*>(&part[v - 1][rq][64 * u + 16 * lg + 4 * r]);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            o[u][e][r] = SPOILT ? add_state(o[u][e][r], wt, y[e]) : fmaf(wt, y[e], o[u][e][r]);
        }
    }
  };
  if (passes[0] + passes[1] + passes[2] + passes[3] > 0)
    merge(IC<1>{});
  else
    merge(IC<0>{});
  const size_t row = slot_row(a, slot, j, fr);
  if (lg == 0) {
    a.ml[2 * row] = Mu;
    a.ml[2 * row + 1] = l_run;
    if (direct && a.lse != nullptr)
      a.lse[(size_t)j * a.B * a.R + fr] = l_run != 0.0f ? Mu + __builtin_amdgcn_logf(l_run) : INFINITY;
  }
  if (direct || l_run != 0.0f) {
    float* dst = direct ? static_cast<float*>(a.out) + q_off(a, j, fr, HD) : a.acc + row * HD;
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

// ------------------------------------------------------------------ merge and streamed weights

// A row's S <= 128 states, by one wave: lane s takes the (max, sum) of states s and s + 64.
// Their merged max M and sum L, and the weights 2^(max - M) (0 for an empty state).
struct Merge {
  float M, L, w0, w1;
};
__device__ __forceinline__ void load_states(const RowsArgs& a, int S, int j, int fr, int lane, float2& x, float2& y) {
  x = y = make_float2(-INFINITY, 0.0f);
  if (lane < S) x = *reinterpret_cast<const float2*>(a.ml + 2 * slot_row(a, lane, j, fr));
  if (lane + 64 < S) y = *reinterpret_cast<const float2*>(a.ml + 2 * slot_row(a, lane + 64, j, fr));
}
__device__ __forceinline__ Merge merge_states(float2 x, float2 y) {
  if (x.y == 0.0f) x.x = -INFINITY;
  if (y.y == 0.0f) y.x = -INFINITY;
  Merge m;
  m.M = wave_max(fmaxf(x.x, y.x));
  const float Mu = m.M == -INFINITY ? 0.0f : m.M;
  m.w0 = exp2_hw(x.x - Mu);
  m.w1 = exp2_hw(y.x - Mu);
  m.L = wave_sum(fmaf(x.y, m.w0, y.y * m.w1));
  return m;
}

constexpr int kFinishKeys = 256;   // keys per workgroup of the streamed weights

// Workgroups 0 .. merge_wgs - 1 merge 4 / WPR rows each (out, and their max + log2(sum)
// where the weights of tiles need them); the rest add up the weights of 256 own keys of one
// (b, j) from the kept scores: weight = decay weight + sum_rows 2^(score - max) / sum.
template <typename T, int HD, int WPR>
__global__ __launch_bounds__(256) void rows_finish_kernel(RowsArgs a, int merge_wgs) {
  constexpr int E = HD / 64;
  const int lane = threadIdx.x & 63, w = wave_id();
  const int S = a.S_prefix + a.S_own;
  if ((int)blockIdx.x < merge_wgs) {
    const long long idx = (long long)blockIdx.x * (4 / WPR) + w / WPR;
    const int Rt = a.B * a.R;
    const bool in = idx < (long long)Rt * a.n_kv;
    const int j = in ? (int)(idx / Rt) : 0, fr = in ? (int)(idx - (long long)j * Rt) : 0;
    bool on = in && row_wanted(a, fr);
    if (any_sole_slot(a) && on) {
      constexpr int RB = sizeof(T) == 2 ? kRowsTile : kRowsWave;
      const int b = fr / a.R;
      on = !sole_slot(a, seq_of(a, b), (fr - b * a.R) / RB * RB, RB);
    }
    if (WPR == 1 && !on) return;
    float2 s0, s1;
    load_states(a, S, j, fr, lane, s0, s1);
    const Merge m = merge_states(s0, s1);
    if (a.lse != nullptr && on && lane == 0 && w % WPR == 0)
      a.lse[(size_t)j * Rt + fr] = m.L != 0.0f ? m.M + __builtin_amdgcn_logf(m.L) : INFINITY;
    float x[E];
    // the states that hold keys (every WPR-th of them), 8 at a time in flight; an empty
    // state has no acc
    const float* src = a.acc + slot_row(a, 0, j, fr) * HD + E * lane;
    const size_t step = (size_t)a.n_kv * Rt * HD;
    auto gather = [&](auto spoilt) {
      constexpr bool SPOILT = decltype(spoilt)::value != 0;
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = 0.0f;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const float wv = half == 0 ? m.w0 : m.w1, sum = half == 0 ? s0.y : s1.y;
        unsigned long long left = __ballot(sum != 0.0f && lane % WPR == w % WPR);
        while (left != 0) {
          float y[8][E], wt[8];
          const int n = __popcll(left);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int s = left != 0 ? __builtin_ctzll(left) : 0;
            wt[i] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, wv), s));
            if (left != 0) load_e<E>(src + (size_t)(s + 64 * half) * step, y[i]);
            left &= left - 1;
          }
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e)
              x[e] = i >= n ? x[e] : SPOILT ? add_state(x[e], wt[i], y[i][e]) : fmaf(y[i][e], wt[i], x[e]);
        }
      }
    };
    gather(IC<0>{});
    float z = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) z = fmaf(x[e], 0.0f, z);
    if (__any(z != 0.0f)) gather(IC<1>{});  // 0 x infinity, perhaps
    if constexpr (WPR > 1) {  // one row per workgroup: its waves' sums in wave order
      __shared__ float part[WPR][HD];
#pragma unroll
      for (int e = 0; e < E; ++e) part[w][E * lane + e] = x[e];
      __syncthreads();
      if (w > 0 || !on) return;
#pragma unroll
      for (int v = 1; v < WPR; ++v)
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] += part[v][E * lane + e];
    }
    T* dst = static_cast<T*>(a.out) + q_off(a, j, fr, HD) + E * lane;
#pragma unroll
    for (int e = 0; e < E; ++e) dst[e] = from_f<T>(m.L != 0.0f ? x[e] / m.L : 0.0f);
    return;
  }
  __shared__ float lse[kMaxGroup];
  const int item = (int)blockIdx.x - merge_wgs, units = a.B * a.n_kv;
  const int c = item / units, u = item - c * units;
  const int j = u % a.n_kv, b = u / a.n_kv;
  const Seq sq = seq_of(a, b);
  const int nr = sq.n * a.g, t = c * kFinishKeys + threadIdx.x;
  // the earlier weight and the first four rows' scores while the rows' sums are merged
  const bool in = t < sq.len;
  float* wp = a.weight + ((size_t)b * a.n_kv + j) * a.t_cap + a.t_off + t;
  const float* sc = a.sc + ((size_t)b * a.n_kv + j) * a.R * a.sc_ld + t;
  const float old = in && a.decay != 0.0f ? a.decay * *wp : 0.0f;
  float x[4];
  auto scores = [&](int r0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = in && r0 + i < nr ? sc[(size_t)(r0 + i) * a.sc_ld] : -INFINITY;
  };
  scores(0);
  float2 s0[4], s1[4];  // of rows w, w + 4, ..
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (w + 4 * i < nr) load_states(a, S, j, b * a.R + w + 4 * i, lane, s0[i], s1[i]);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (w + 4 * i < nr) {
      const Merge m = merge_states(s0[i], s1[i]);
      if (lane == 0) lse[w + 4 * i] = m.L != 0.0f ? m.M + __builtin_amdgcn_logf(m.L) : INFINITY;
    }
  __syncthreads();
  float sum = 0.0f;
  for (int r = 0; r < nr; r += 4) {
    float p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = x[i] == -INFINITY ? 0.0f : exp2_hw(x[i] - lse[min(r + i, nr - 1)]);
    if (r + 4 < nr) scores(r + 4);
    sum += (p[0] + p[1]) + (p[2] + p[3]);
  }
  if (in) *wp = old + sum;
}

// ------------------------------------------------------------------ weights of a key tile

// Rows [r0, r1) of part c, P_w rows each, of the rows that see key k0 of sequence sq: early
// keys have more parts than late ones, all of one size (a 3001-token prompt: 35 us; with the
// same number for each key, the first tiles' the longest, 37).
struct RowSpan {
  int r0, r1;
};
__device__ __forceinline__ RowSpan rows_of_part(const RowsArgs& a, const Seq& sq, int k0, int c) {
  const int i0 = min(max(k0 - (sq.len - sq.n), 0), sq.n);  // the first token that sees key k0
  const long long r0 = (long long)i0 * a.g + (long long)c * a.P_w, end = (long long)sq.n * a.g;
  return RowSpan{(int)min(r0, end), (int)min(r0 + a.P_w, end)};
}
__device__ __forceinline__ void put_weight(const RowsArgs& a, int c, int b, int j, int t, float sum) {
  const size_t bj = (size_t)b * a.n_kv + j;
  if (a.S_w == 1) {
    float* wp = a.weight + bj * a.t_cap + a.t_off + t;
    *wp = a.decay != 0.0f ? fmaf(a.decay, *wp, sum) : sum;
  } else {
    a.wpart[((size_t)c * a.B * a.n_kv + bj) * a.T_own + t] = sum;
  }
}

constexpr int kWtKeys = 128, kWtRows = 64;

// Byte offset of the thread's i-th chunk of a tile of `rows` query rows from the first one's
// token, whose row `at` it is (at most 65 tokens: 32 bits), and its copy into LDS.
template <int HD>
__device__ __forceinline__ uint32_t chunk_offset(const RowsArgs& a, int i, int at, int rows) {
  constexpr int CPR = HD / 8;
  const int r = threadIdx.x / CPR + 256 / CPR * i, x = at + min(r, rows - 1), tok = token_of(a, x);
  return ((uint32_t)x + (uint32_t)tok * (uint32_t)(a.n_q - a.g)) * (HD * 2) +
         16u * ((threadIdx.x % CPR) ^ score_swz<HD>(r));
}
__device__ __forceinline__ void copy_chunk(const uint16_t* src, uint32_t off, uint16_t* dst) {
  const __amdgpu_buffer_rsrc_t res =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(src), (short)0, -1, 0x00027000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(res, (__attribute__((address_space(3))) void*)dst, 16, off, 0, 0, 0);
}

// bf16: one workgroup of 4 waves per (128 keys of (b, j), part of the rows).  A wave
// keeps its 32 keys as MFMA A operands; the rows pass through LDS 64 at a time
// (layout of copy_tile's score operands), two buffers.  A lane holds the scores of one row and
// adds 2^(score - lse) into 16 sums, one per key.
template <int HD>
__global__ __launch_bounds__(256, 2) void weight_tile_kernel(RowsArgs a) {
  constexpr int KS = HD / 16, CPR = HD / 8, CH = kWtRows * CPR / 256, kLead = 4;
  __shared__ __align__(1024) uint16_t q_a[kWtRows * HD], q_b[kWtRows * HD];  // two objects: see rows_bf16_kernel
  const int tid = threadIdx.x, lane = tid & 63, w = wave_id(), hl = lane >> 5;
  const int units = a.B * a.n_kv, x = (int)blockIdx.x / units, u = (int)blockIdx.x - x * units;
  const int j = u % a.n_kv, b = u / a.n_kv;
  const int c = x % a.S_w, tile = x / a.S_w;
  const Seq sq = seq_of(a, b);
  const int k0 = tile * kWtKeys;
  if (k0 >= sq.len) return;
  const RowSpan rs = rows_of_part(a, sq, k0, c);
  if (c > 0 && rs.r0 >= rs.r1) return;  // the first part writes in any case
  const KeyRange kr = own_range(a, b, j, 0, sq.len);
  const uint32_t qbase = score_base<HD>(lane);
  // The keys through the rows' buffers, whole lines at a time (straight into the registers a
  // load takes 32 bytes of 32 rows: 32.0 us instead of 31.1).
  bf16x8_t kf[KS];
  {
    const uint16_t* ks = static_cast<const uint16_t*>(a.k) + kr.row * HD;
    const int k1 = min(k0 + 64, sq.len - 1);
    copy_tile<HD, 64, true>(ks + (size_t)k0 * HD, sq.len - k0, q_a);
    copy_tile<HD, 64, true>(ks + (size_t)k1 * HD, sq.len - k1, q_b);
    __builtin_amdgcn_s_waitcnt(0x0f70);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < KS; ++i) kf[i] = score_operand(w < 2 ? q_a : q_b, qbase, i, 64 * HD * (w & 1));
    __syncthreads();
  }
  float sum[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) sum[r] = 0.0f;
  const int fr0 = b * a.R;
  const int nt = rs.r1 > rs.r0 ? (rs.r1 - rs.r0 + kWtRows - 1) / kWtRows : 0;
  // A group size that divides 64: every tile starts with a token, and a thread's rows have
  // the same offsets from it (64-bit offsets of every row: 35 us instead of 32).
  const bool same = kWtRows % a.g == 0;
  uint32_t off[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) off[i] = chunk_offset<HD>(a, i, 0, kWtRows);
  auto load = [&](int t, uint16_t* dst) {
    const int first = rs.r0 + t * kWtRows, left = rs.r1 - first, at = first - token_of(a, first) * a.g;
    const uint16_t* src = static_cast<const uint16_t*>(a.q) + q_off(a, j, fr0 + first - at, HD);
    const bool full = same && left >= kWtRows;
#pragma unroll
    for (int i = 0; i < CH; ++i)
      copy_chunk(src, full ? off[i] : chunk_offset<HD>(a, i, at, left), dst + 512 * w + 2048 * i);
  };
  // max + log2(sum) of the lane's two rows of a tile, loaded a tile ahead and before that
  // tile's copies (a load is waited for with everything issued before it); rows past the
  // part get +inf, weight 0
  const float* lse_row = a.lse + (size_t)j * a.B * a.R + fr0;
  float lse_next[2];
  auto load_lse = [&](int t) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = rs.r0 + t * kWtRows + 32 * h + (lane & 31);
      lse_next[h] = lse_row[min(r, rs.r1 - 1)];
      if (r >= rs.r1) lse_next[h] = INFINITY;
    }
  };
  auto step = [&](int t, const uint16_t* qs, uint16_t* next) {
    __builtin_amdgcn_s_waitcnt(0x0f70);
    __syncthreads();
    const float lse[2] = {lse_next[0], lse_next[1]};
    if (t + 1 < nt) {
      load_lse(t + 1);
      load(t + 1, next);
    }
    // whether every row of the tile sees every key of the workgroup
    const int first = rs.r0 + t * kWtRows;
    const bool masked = rows_seen(sq, token_of(a, first)) < k0 + kWtKeys;
    f32x16_t sts[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 16; ++i) sts[h][i] = 0.0f;
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < KS; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        sts[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i], score_operand(qs, qbase, i, 64 * HD * h), sts[h], 0, 0, 0);
    // reads kLead operands ahead of the products
    __builtin_amdgcn_sched_group_barrier(0x100, kLead, 0);
#pragma unroll
    for (int i = 0; i < 2 * KS - kLead; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, kLead, 0);
    __builtin_amdgcn_s_setprio(0);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x16_t st = sts[h];
      float p[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = exp2_hw(fmaf(st[i], ScoreScale<HD>::v, -lse[h]));
      if (masked) {
        asm volatile("");
        const int r = first + 32 * h + (lane & 31);
        const int lim = r < rs.r1 ? rows_seen(sq, token_of(a, r)) - k0 - 32 * w : 0;  // keys of the wave that the row sees
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = 8 * (i >> 2) + 4 * hl + (i & 3) < lim ? p[i] : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[i] += p[i];
    }
  };
  if (nt > 0) load_lse(0);
  if (nt > 0) load(0, q_a);
  for (int t = 0; t < nt; t += 2) {
    step(t, q_a, q_b);
    if (t + 1 < nt) step(t + 1, q_b, q_a);
  }
  // over the 32 lanes: each exchange adds half of the keys and hands the other half over
#pragma unroll
  for (int o = 1, n = 8; o < 16; o <<= 1, n >>= 1) {
    const bool up = (lane & o) != 0;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float give = up ? sum[i] : sum[i + n];
      sum[i] = (up ? sum[i + n] : sum[i]) + __shfl_xor(give, o, 64);
    }
  }
  const float total = sum[0] + __shfl_xor(sum[0], 16, 64);
  const int i = (lane & 1) * 8 + (lane & 2) * 2 + ((lane & 4) >> 1) + ((lane & 8) >> 3);  // the lane's key
  const int t = k0 + 32 * w + 8 * (i >> 2) + 4 * hl + (i & 3);
  if ((lane & 16) == 0 && t < sq.len) put_weight(a, c, b, j, t, total);
}

// fp32: one workgroup of 4 waves per (16 keys of (b, j), part of the rows), 16 rows at a step
// and wave in turn (a wave's steps are round trips: 3 x 512 tokens of 9 heads 38 us with one
// wave per workgroup, 19 with four), the waves' sums in wave order.
template <int HD>
__global__ __launch_bounds__(256) void weight_f32_kernel(RowsArgs a) {
  constexpr int KC = HD / 16;
  __shared__ float part[4][16];
  const int lane = threadIdx.x & 63, wv = wave_id(), rq = lane & 15, lg = lane >> 4;
  const int units = a.B * a.n_kv, x = (int)blockIdx.x / units, u = (int)blockIdx.x - x * units;
  const int j = u % a.n_kv, b = u / a.n_kv;
  const int c = x % a.S_w, tile = x / a.S_w;
  const Seq sq = seq_of(a, b);
  const int k0 = tile * 16;
  if (k0 >= sq.len) return;
  const RowSpan rs = rows_of_part(a, sq, k0, c);
  if (c > 0 && rs.r0 >= rs.r1) return;  // the first part writes in any case
  const KeyRange kr = own_range(a, b, j, 0, sq.len);
  f32x4_t kf[KC];
  const float* ks = static_cast<const float*>(a.k) + (kr.row + min(k0 + rq, sq.len - 1)) * HD + 4 * lg;
#pragma unroll
  for (int i = 0; i < KC; ++i) kf[i] = *reinterpret_cast<const f32x4_t*>(ks + 16 * i);
  float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int r0 = rs.r0 + 16 * wv; r0 < rs.r1; r0 += 64) {
    const int r = r0 + rq, fr = b * a.R + min(r, rs.r1 - 1);
    const float* qs = static_cast<const float*>(a.q) + q_off(a, j, fr, HD) + 4 * lg;
    f32x4_t s0 = {0.0f, 0.0f, 0.0f, 0.0f}, s1 = s0;
#pragma unroll
    for (int i = 0; i < KC; ++i) {
      const f32x4_t qf = *reinterpret_cast<const f32x4_t*>(qs + 16 * i);
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[i][e], qf[e], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[i][e + 1], qf[e + 1], s1, 0, 0, 0);
      }
    }
    const float lse = r < rs.r1 ? a.lse[(size_t)j * a.B * a.R + fr] : INFINITY;
    const int lim = r < rs.r1 ? rows_seen(sq, token_of(a, r)) - k0 : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = exp2_hw((s0[i] + s1[i]) * ScoreScale<HD>::v - lse);
      sum[i] += 4 * lg + i < lim ? p : 0.0f;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) sum[i] += __shfl_xor(sum[i], o, 64);
    if (rq == 0) part[wv][4 * lg + i] = sum[i];
  }
  __syncthreads();
  const int k = threadIdx.x;
  if (k < 16 && k0 + k < sq.len) put_weight(a, c, b, j, k0 + k, (part[0][k] + part[1][k]) + (part[2][k] + part[3][k]));
}

// weight = decay weight + the sums of the parts that key t's tile has, in part order.
__global__ __launch_bounds__(256) void weight_sum_kernel(RowsArgs a, int tile_keys) {
  const int chunks = (a.T_own + 255) / 256;
  const int bj = (int)blockIdx.x / chunks, t = ((int)blockIdx.x - bj * chunks) * 256 + threadIdx.x;
  const Seq sq = seq_of(a, bj / a.n_kv);
  if (t >= sq.len) return;
  const RowSpan rs = rows_of_part(a, sq, t / tile_keys * tile_keys, 0);
  const int parts = max((sq.n * a.g - rs.r0 + a.P_w - 1) / a.P_w, 1);
  float sum = 0.0f;
#pragma unroll 4
  for (int c = 0; c < parts; ++c) sum += a.wpart[((size_t)c * a.B * a.n_kv + bj) * a.T_own + t];
  float* wp = a.weight + (size_t)bj * a.t_cap + a.t_off + t;
  *wp = a.decay != 0.0f ? fmaf(a.decay, *wp, sum) : sum;
}

// ------------------------------------------------------------------ launchers

#define KVD_LAUNCH_TRY(expr)          \
  do {                                \
    hipError_t _e = (expr);           \
    if (_e != hipSuccess) return _e;  \
  } while (0)

template <typename T, int HD>
static hipError_t launch_rows_t(const RowsArgs& a, hipStream_t st) {
  constexpr bool BF = sizeof(T) == 2;
  const int RB = BF ? kRowsTile : kRowsWave;
  const long long nbo = (a.R + RB - 1) / RB, nbp = ((long long)a.B * a.R + RB - 1) / RB;
  const int S_prefix = a.S_prefix;
  long long few_items = 0, tile_items = 0;
  (a.own_few ? few_items : tile_items) += (long long)a.B * a.n_kv * a.S_own * (a.own_few ? 1 : nbo);
  (a.prefix_few ? few_items : tile_items) += (long long)a.n_kv * S_prefix * (a.prefix_few ? 1 : nbp);
  if constexpr (BF)
    hipLaunchKernelGGL(rows_bf16_kernel<HD>, dim3((unsigned)(tile_items + few_items)), dim3(256), 0, st, a,
                       (int)tile_items);
  else
    hipLaunchKernelGGL(rows_f32_kernel<HD>, dim3((unsigned)tile_items), dim3(256), 0, st, a);
  KVD_LAUNCH_TRY(hipGetLastError());
  const int S = S_prefix + a.S_own;
  const bool sums = a.weight != nullptr && a.T_own > 0;
  const long long rows = (long long)a.B * a.R * a.n_kv;
  const int per = 4 / rows_finish_waves(S);  // merged rows per workgroup
  const int merge_wgs = S > 1 ? (int)((rows + per - 1) / per) : 0;
  const int weight_wgs = sums && a.sc != nullptr ? a.B * a.n_kv * ((a.T_own + kFinishKeys - 1) / kFinishKeys) : 0;
  if (merge_wgs + weight_wgs > 0) {
    if (rows_finish_waves(S) == 4)
      hipLaunchKernelGGL((rows_finish_kernel<T, HD, 4>), dim3(merge_wgs + weight_wgs), dim3(256), 0, st, a, merge_wgs);
    else
      hipLaunchKernelGGL((rows_finish_kernel<T, HD, 1>), dim3(merge_wgs + weight_wgs), dim3(256), 0, st, a, merge_wgs);
    KVD_LAUNCH_TRY(hipGetLastError());
  }
  if (sums && a.sc == nullptr) {
    const int keys = BF ? kWtKeys : 16;
    const unsigned items = (unsigned)((long long)a.B * a.n_kv * a.S_w * ((a.T_own + keys - 1) / keys));
    if constexpr (BF)
      hipLaunchKernelGGL(weight_tile_kernel<HD>, dim3(items), dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL(weight_f32_kernel<HD>, dim3(items), dim3(256), 0, st, a);
    KVD_LAUNCH_TRY(hipGetLastError());
    if (a.S_w > 1) {
      hipLaunchKernelGGL(weight_sum_kernel, dim3((unsigned)(a.B * a.n_kv * ((a.T_own + 255) / 256))), dim3(256), 0, st,
                         a, keys);
      KVD_LAUNCH_TRY(hipGetLastError());
    }
  }
  return hipSuccess;
}

hipError_t launch_rows(const RowsArgs& a, int dtype_bf16, int hd, hipStream_t st) {
  switch (hd) {
    case 64: return dtype_bf16 ? launch_rows_t<uint16_t, 64>(a, st) : launch_rows_t<float, 64>(a, st);
    case 128: return dtype_bf16 ? launch_rows_t<uint16_t, 128>(a, st) : launch_rows_t<float, 128>(a, st);
    case 256: return dtype_bf16 ? launch_rows_t<uint16_t, 256>(a, st) : launch_rows_t<float, 256>(a, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace kvd
