// Eviction from a cache by accumulated attention weight (kvd_evict): every (sequence,
// KV head) keeps its n' = min(len, keep) foremost rows.
//
//   evict_one_kernel     keep = T - 1, a decode step's call: the lightest row of each
//                        cache, and the move of its last one, in one launch.
//   evict_select_kernel  otherwise, one workgroup per (b, j): the rows' ranks, the rank of
//                        the last row kept, and who moves where.
//   evict_move_kernel    then the moves themselves.
//
// Kept rows in slots >= n' move into the freed slots < n', both in slot order: sources
// and destinations are disjoint sets, so the copies need no order, and no fewer rows
// could move.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kvd_device.hpp"
#include "kvd_launch.h"

namespace kvd {

constexpr int kNtEvict = 1024;

// A row's rank: larger stays longer.  Protected rows above every weight, NaN below, -0
// as +0; the float order otherwise.
__device__ __forceinline__ uint32_t rank_of(const EvictArgs& a, float w, int pos, int newest) {
  if (a.pos != nullptr && (pos < a.sink || (a.recent > 0 && (long long)pos > (long long)newest - a.recent)))
    return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t x = __float_as_uint(w + 0.0f);
  return x ^ ((x >> 31) != 0 ? 0xffffffffu : 0x80000000u);
}

// Inclusive sum over the workgroup's threads of v, in thread order, and the total;
// `buf` holds one word per wave.  Ends with a barrier.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* buf, uint32_t& total) {
  const int lane = threadIdx.x & 63, w = wave_id();
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t x = __shfl_up(v, o, 64);
    if (lane >= o) v += x;
  }
  if (lane == 63) buf[w] = v;
  __syncthreads();
  uint32_t before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < kNtEvict / 64; ++i) {
    const uint32_t x = buf[i];
    before += i < w ? x : 0u;
    total += x;
  }
  __syncthreads();
  return v + before;
}

constexpr int kEvictBins = 2 * kNtEvict;

// f(i) for the slots i < N of a thread (rows t, t + 1024, ..) that `rows` rows reach into; the code
// of the others is jumped over (fetching it costs more than running it), and i is a constant, so
// that arrays indexed by it stay in registers.
template <int I, int N, typename F>
__device__ __forceinline__ void slots_with_rows(int rows, const F& f) {
  if constexpr (I < N) {
    if (I * kNtEvict < rows) {
      f(I);
      slots_with_rows<I + 1, N>(rows, f);
    }
  }
}

// The rank of the last row kept: each pass spreads the ranks that can still be it, [lo,
// hi], over 2048 equal bins (a first pass over the ranks that occur, so that weights of
// like size do not share a bin, whose counter they would take turns at; protected and
// NaN rows are counted apart) and goes on with the bin that holds it, at most three times;
// a bin of up to 64 rows (the first one as a rule) is settled by one wave that compares
// them.  Then rows are taken thread by thread in slot order: c consecutive slots each, c
// odd (LDS banks), one prefix sum for freed slots and movers, and before it one for the rows
// that tie with the last rank unless all of those stay.  Latency-bound: a thread keeps the
// ranks of its rows (t, t + 1024, .., at most PER) in registers, all its loads in flight at once,
// and LDS turns them into slot order.  PER = 0: any length, ranks in the workspace.  16 caches of
// 8192 .. 16385 rows to 2048: 88 us with 8-bit digits of the whole rank and serial bin walks, 28
// us with ranks read from LDS in every pass and four loads in flight, 26 us with three passes
// always, 22 us so.
template <int PER>
__global__ __launch_bounds__(kNtEvict) void evict_select_kernel(EvictArgs a) {
  __shared__ uint32_t lkeys[PER > 0 ? PER * kNtEvict : 1];
  __shared__ uint32_t hist[kEvictBins];
  __shared__ uint32_t buf[kNtEvict / 64];
  __shared__ uint32_t list[64];
  __shared__ uint32_t s_lo, s_hi, s_top, s_bin, s_need, s_count, s_fill;
  const int tid = threadIdx.x, lane = tid & 63;
  const int bj = blockIdx.x, b = bj / a.n_kv;
  float* wt = a.weight + (size_t)bj * a.t_cap + a.t_off;
  int32_t* ps = a.pos != nullptr ? a.pos + (size_t)bj * a.t_cap + a.t_off : nullptr;
  uint32_t* keys = PER > 0 ? lkeys : a.keys + (size_t)bj * a.T;
  // the weights and positions of all T rows, before the length is known
  constexpr int N = PER > 0 ? PER : 1;
  float x[N];
  int p[N];
  auto each = [&](auto f) {
    int rows = a.T;
    asm volatile("" : "+s"(rows));  // compared again in each loop: the results of all slots took 148 scalar registers
    slots_with_rows<0, N>(rows, f);
  };
  if constexpr (PER > 0) {
    each([&](int i) { x[i] = wt[(uint32_t)min(tid + i * kNtEvict, a.T - 1)]; });
    if (ps != nullptr) each([&](int i) { p[i] = ps[(uint32_t)min(tid + i * kNtEvict, a.T - 1)]; });
  }
  const int n = a.len != nullptr ? min(max(a.len[b], 0), a.T) : a.T;
  const int newest = a.last_pos != nullptr ? a.last_pos[b] : 0;
  const int left = min(n, a.keep);
  if (n == left) {
    if (tid == 0) a.n_moves[bj] = 0;
    return;
  }
  if (tid == 0) {
    s_lo = 0xffffffffu;
    s_hi = 0u;
    s_top = 0u;
  }
  for (int i = tid; i < kEvictBins; i += kNtEvict) hist[i] = 0u;
  __syncthreads();
  uint32_t lo = 0xffffffffu, hi = 0u, top = 0u;
  uint32_t k[N];
  auto take = [&](uint32_t r) {
    if (r == 0xffffffffu) {
      ++top;
    } else if (r != 0u) {
      lo = min(lo, r);
      hi = max(hi, r);
    }
  };
  if constexpr (PER > 0) {
    each([&](int i) {
      const int t = tid + i * kNtEvict;
      k[i] = t < n ? rank_of(a, x[i], ps != nullptr ? p[i] : 0, newest) : 0u;  // past the rows: as NaN, never counted
      lkeys[t] = k[i];
      take(k[i]);
    });
  } else {
    for (int t = tid; t < n; t += kNtEvict) {
      const uint32_t r = rank_of(a, wt[t], ps != nullptr ? ps[t] : 0, newest);
      keys[t] = r;
      take(r);
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    lo = min(lo, (uint32_t)__shfl_xor(lo, o, 64));
    hi = max(hi, (uint32_t)__shfl_xor(hi, o, 64));
    top += __shfl_xor(top, o, 64);
  }
  if (lane == 0) {
    atomicMin(&s_lo, lo);
    atomicMax(&s_hi, hi);
    atomicAdd(&s_top, top);
  }
  __threadfence_block();
  __syncthreads();
  lo = s_lo;
  hi = s_hi;
  uint32_t need = (uint32_t)left;  // rows still to be kept among those of rank <= hi
  uint32_t last = 0u;              // rank of the last row kept
  bool found = false, whole = false;  // whole: every row of that rank stays
  if (need <= s_top) {
    last = 0xffffffffu;
    whole = need == s_top;
    found = true;
  } else {
    need -= s_top;
    if (lo > hi) found = true;  // nothing but NaN left
  }
  while (!found) {
    // bin width 2^shift: the least that covers [lo, hi] with 2048 bins
    const uint32_t range = hi - lo;
    const int shift = range < (uint32_t)kEvictBins ? 0 : 21 - __clz(range);
    if (tid == 0) {
      s_bin = 0xffffffffu;
      s_fill = 0u;
    }
    if constexpr (PER > 0) {
      each([&](int i) {
        if (k[i] >= lo && k[i] <= hi) atomicAdd(&hist[(k[i] - lo) >> shift], 1u);
      });
    } else {
      for (int t = tid; t < n; t += kNtEvict) {
        const uint32_t r = keys[t];
        if (r >= lo && r <= hi) atomicAdd(&hist[(r - lo) >> shift], 1u);
      }
    }
    __syncthreads();
    // thread i takes the i-th pair of bins from the top, and leaves them at zero
    const uint32_t h1 = hist[kEvictBins - 1 - 2 * tid], h0 = hist[kEvictBins - 2 - 2 * tid];
    hist[kEvictBins - 1 - 2 * tid] = 0u;
    hist[kEvictBins - 2 - 2 * tid] = 0u;
    uint32_t total;
    const uint32_t upto = block_scan(h0 + h1, buf, total);
    const uint32_t before = upto - h0 - h1;
    if (before < need && need <= upto) {
      const bool first = need <= before + h1;
      s_bin = kEvictBins - 1 - 2 * tid - (first ? 0 : 1);
      s_need = need - before - (first ? 0u : h1);
      s_count = first ? h1 : h0;
    }
    __syncthreads();
    if (s_bin == 0xffffffffu) {  // every number stays, and some NaN
      need -= total;
      found = true;
    } else {
      need = s_need;
      lo += s_bin << shift;
      hi = lo + ((1u << shift) - 1u);
      if (shift == 0) {
        last = lo;
        whole = need == s_count;
        found = true;
      } else if (s_count <= 64u) {  // the bin's rows, compared by the first wave
        const auto gather = [&](uint32_t r) {
          if (r >= lo && r <= hi) list[atomicAdd(&s_fill, 1u)] = r;
        };
        if constexpr (PER > 0) {
          each([&](int i) { gather(k[i]); });
        } else {
          for (int t = tid; t < n; t += kNtEvict) gather(keys[t]);
        }
        __syncthreads();
        if (tid < 64) {
          const int count = (int)s_count;
          const uint32_t mine = list[min(lane, count - 1)];
          uint32_t above = 0, same = 0;
          for (int i = 0; i < count; ++i) {
            const uint32_t r = list[i];
            above += r > mine ? 1u : 0u;
            same += r == mine ? 1u : 0u;
          }
          if (lane < count && above < need && need <= above + same) {
            s_bin = mine;
            s_need = need - above;
            s_count = same;
          }
        }
        __syncthreads();
        last = s_bin;
        need = s_need;
        whole = need == s_count;
        found = true;
      }
    }
    __syncthreads();
  }
  const uint32_t ties = need;  // rows of rank `last` that stay: the lowest slots
  const int c = ((n + kNtEvict - 1) / kNtEvict) | 1;
  const int t0 = (int)min((long long)tid * c, (long long)n), t1 = min(t0 + c, n);
  uint32_t eq0 = 0, total;
  if (!whole) {
    uint32_t eq = 0;
#pragma unroll 8
    for (int t = t0; t < t1; ++t) eq += keys[t] == last ? 1u : 0u;
    eq0 = block_scan(eq, buf, total) - eq;
  }
  uint32_t e = eq0;
  auto kept = [&](uint32_t r) { return r > last || (r == last && (whole || e++ < ties)); };
  // freed slots below `left` and, as many, movers behind it, in one sum
  uint32_t count = 0;
#pragma unroll 8
  for (int t = t0; t < t1; ++t) count += kept(keys[t]) == (t >= left) ? 1u : 0u;
  uint32_t at = block_scan(count, buf, total) - count;
  int2* mv = a.moves + (size_t)bj * a.max_moves;
  e = eq0;
#pragma unroll 8
  for (int t = t0; t < t1; ++t) {
    const bool stays = kept(keys[t]);
    if (t < left) {
      if (!stays) mv[at++].x = t;
    } else if (stays) {
      mv[at++ - total / 2].y = t;
    } else if (keys[t] == last) {
      wt[t] = 0.0f;
    }
  }
  // weights of the freed slots from `left` on: ranks below the last one here, ties that do
  // not stay above, a mover's when it has moved
  if constexpr (PER > 0) {
    each([&](int i) {
      const int t = tid + i * kNtEvict;
      if (t >= left && t < n && k[i] < last) wt[t] = 0.0f;
    });
  } else {
    for (int t = left + tid; t < n; t += kNtEvict)
      if (keys[t] < last) wt[t] = 0.0f;
  }
  if (tid == 0) a.n_moves[bj] = (int)(total / 2);
}

// keep = T - 1: a cache of T rows loses its lightest one (of equal ones the highest slot),
// and row T - 1 takes its place.  A workgroup takes `heads` caches of one sequence, 16 /
// heads waves each: all of a sequence's where its length has to be set (nothing may read it
// after that), one otherwise.
__global__ __launch_bounds__(kNtEvict) void evict_one_kernel(EvictArgs a, int heads) {
  constexpr int NW = kNtEvict / 64;
  __shared__ unsigned long long best[NW];
  const int lane = threadIdx.x & 63, w = wave_id();
  const int wph = heads >= NW ? 1 : NW / heads;  // waves per head
  const int groups = a.n_kv / heads;
  const int b = (int)blockIdx.x / groups, j0 = ((int)blockIdx.x - b * groups) * heads;
  const int n = a.len != nullptr ? min(max(a.len[b], 0), a.T) : a.T;
  const int newest = a.last_pos != nullptr ? a.last_pos[b] : 0;
  if (n < a.T) {  // this sequence keeps all of its rows
    if (a.len != nullptr && threadIdx.x == 0) a.len[b] = n;
    return;
  }
  const int hw = w / wph, part = w - hw * wph;
  for (int h0 = 0; h0 < heads; h0 += NW / wph) {
    const bool on = hw < NW / wph && h0 + hw < heads;
    const size_t row0 = ((size_t)b * a.n_kv + j0 + h0 + hw) * a.t_cap + a.t_off;
    // the least rank, of equal ones the highest slot
    unsigned long long least = ~0ull;
    if (on) {
      const float* wt = a.weight + row0;
      const int32_t* ps = a.pos != nullptr ? a.pos + row0 : nullptr;
      for (int t0 = part * 64 + lane; t0 < n; t0 += 8 * 64 * wph) {
        float x[8];
        int p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int t = min(t0 + i * 64 * wph, n - 1);
          x[i] = wt[t];
          p[i] = ps != nullptr ? ps[t] : 0;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int t = min(t0 + i * 64 * wph, n - 1);  // the last row again: the same candidate
          const unsigned long long k =
              ((unsigned long long)rank_of(a, x[i], p[i], newest) << 32) | (0xffffffffu - (uint32_t)t);
          least = k < least ? k : least;
        }
      }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const unsigned long long x = __shfl_xor(least, o, 64);
      least = x < least ? x : least;
    }
    __syncthreads();
    if (lane == 0) best[w] = least;
    __syncthreads();
    if (on && part == 0) {
      for (int i = 1; i < wph; ++i) least = best[w + i] < least ? best[w + i] : least;
      const int gone = (int)(0xffffffffu - (uint32_t)least), from = n - 1;
      const int cpr = a.row_bytes / 16;
      if (gone != from) {
        uint4* k = reinterpret_cast<uint4*>(a.k) + row0 * cpr;
        uint4* v = reinterpret_cast<uint4*>(a.v) + row0 * cpr;
        if (lane < cpr) {
          const uint4 x = k[(size_t)from * cpr + lane], y = v[(size_t)from * cpr + lane];
          k[(size_t)gone * cpr + lane] = x;
          v[(size_t)gone * cpr + lane] = y;
        }
        if (lane == 0) {
          a.weight[row0 + gone] = a.weight[row0 + from];
          if (a.pos != nullptr) a.pos[row0 + gone] = a.pos[row0 + from];
        }
      }
      if (lane == 0) a.weight[row0 + from] = 0.0f;
    }
  }
  if (a.len != nullptr && threadIdx.x == 0) a.len[b] = a.keep;
}

// `parts` workgroups per (b, j) copy its moves, 16 bytes of K and V per lane, weights and
// positions beside a row's first.  Also the lengths.
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a, int parts) {
  const int bj = (int)(blockIdx.x / (unsigned)parts), part = (int)blockIdx.x - bj * parts, b = bj / a.n_kv;
  const int n = a.n_moves[bj];
  const int cpr = a.row_bytes / 16;
  const size_t row0 = (size_t)bj * a.t_cap + a.t_off;
  uint4* k = reinterpret_cast<uint4*>(a.k) + row0 * cpr;
  uint4* v = reinterpret_cast<uint4*>(a.v) + row0 * cpr;
  const int2* mv = a.moves + (size_t)bj * a.max_moves;
  const long long chunks = (long long)n * cpr;
  for (long long i = (long long)part * 256 + threadIdx.x; i < chunks; i += (long long)parts * 256) {
    const int m = (int)(i / cpr), c = (int)(i - (long long)m * cpr);
    const int2 d = mv[m];
    const size_t dst = (size_t)d.x * cpr + c, src = (size_t)d.y * cpr + c;
    const uint4 x = k[src], y = v[src];
    k[dst] = x;
    v[dst] = y;
    if (c == 0) {
      a.weight[row0 + d.x] = a.weight[row0 + d.y];
      a.weight[row0 + d.y] = 0.0f;
      if (a.pos != nullptr) a.pos[row0 + d.x] = a.pos[row0 + d.y];
    }
  }
  if (a.len != nullptr && bj == b * a.n_kv && part == 0 && threadIdx.x == 0)
    a.len[b] = min(min(max(a.len[b], 0), a.T), a.keep);
}

hipError_t launch_evict(const EvictArgs& a, hipStream_t st) {
  const int bjs = a.B * a.n_kv;
  if (a.keep == a.T - 1) {
    const int heads = a.len != nullptr ? a.n_kv : 1;
    hipLaunchKernelGGL(evict_one_kernel, dim3(bjs / heads), dim3(kNtEvict), 0, st, a, heads);
    return hipGetLastError();
  }
  const auto select = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(bjs), dim3(kNtEvict), 0, st, a); };
  // Rows per thread in registers: 8, 16 or 32, all without spills (32: 101 VGPRs, 140 KB of LDS
  // for the ranks), each for twice the length of the one before, because a slot that holds no row
  // costs 0.1 us (8192 rows: 13.5 us with 8, 14.2 with 16, 15.7 with 32; both launches of a call,
  // 16 caches).  Beyond, ranks in the workspace (32768 rows: 33 us with 32, 59 so; 60000: 101).
  if (a.T <= 8 * kNtEvict)
    select(evict_select_kernel<8>);
  else if (a.T <= 16 * kNtEvict)
    select(evict_select_kernel<16>);
  else if (a.T <= 32 * kNtEvict)
    select(evict_select_kernel<32>);
  else
    select(evict_select_kernel<0>);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const long long work = (long long)a.max_moves * (a.row_bytes / 16);
  const int parts = (int)std::max<long long>(1, std::min<long long>((work + 1023) / 1024, 2048 / bjs));
  hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)parts * bjs), dim3(256), 0, st, a, parts);
  return hipGetLastError();
}

}  // namespace kvd
