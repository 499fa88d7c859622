// Eviction from a cache by accumulated attention weight (kvd_evict): every (sequence,
// KV head) keeps its n' = min(len, keep) foremost rows.
//
//   evict_select_kernel  one workgroup per (b, j): the rows' ranks, the rank of the last
//                        row kept (radix selection), and who moves where; weights and
//                        positions are moved here.
//   evict_move_kernel    the K and V rows.
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

// Number of lanes below this one whose predicate holds, and in the whole wave.
__device__ __forceinline__ int lanes_below(unsigned long long m, int lane) {
  return __popcll(m & ((1ull << lane) - 1));
}

__global__ __launch_bounds__(kNtEvict) void evict_select_kernel(EvictArgs a) {
  constexpr int NW = kNtEvict / 64;
  __shared__ int hist[256];
  __shared__ int wsum[2][NW];
  __shared__ uint32_t s_prefix;
  __shared__ int s_need;
  const int tid = threadIdx.x, lane = tid & 63, w = wave_id();
  const int bj = blockIdx.x, b = bj / a.n_kv;
  const int n = a.len != nullptr ? min(max(a.len[b], 0), a.T) : a.T;
  const int left = min(n, a.keep);
  if (n == left) {
    if (tid == 0) a.n_moves[bj] = 0;
    return;
  }
  float* wt = a.weight + (size_t)bj * a.t_cap + a.t_off;
  int32_t* ps = a.pos != nullptr ? a.pos + (size_t)bj * a.t_cap + a.t_off : nullptr;
  uint32_t* keys = a.keys + (size_t)bj * a.T;
  const int newest = a.last_pos != nullptr ? a.last_pos[b] : 0;
  for (int t = tid; t < n; t += kNtEvict) keys[t] = rank_of(a, wt[t], ps != nullptr ? ps[t] : 0, newest);
  // the left-th largest rank, 8 bits at a time
  if (tid == 0) {
    s_prefix = 0;
    s_need = left;
  }
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    const uint32_t prefix = s_prefix;
    const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
    for (int t = tid; t < n; t += kNtEvict) {
      const uint32_t k = keys[t];
      if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    if (tid == 0) {
      int need = s_need, d = 255;
      for (; d > 0 && hist[d] < need; --d) need -= hist[d];
      s_need = need;
      s_prefix = prefix | ((uint32_t)d << shift);
    }
    __syncthreads();
  }
  const uint32_t last = s_prefix;  // rank of the last row kept
  const int ties = s_need;         // rows of that rank that stay: the lowest slots
  // slots in order: freed ones below `left`, kept ones from there on
  int eq0 = 0, holes = 0, movers = 0;
  int2* mv = a.moves + (size_t)bj * a.max_moves;
  for (int t0 = 0; t0 < n; t0 += kNtEvict) {
    const int t = t0 + tid;
    const uint32_t k = t < n ? keys[t] : 0u;
    const bool eq = t < n && k == last;
    const unsigned long long me = __ballot(eq);
    __syncthreads();
    if (lane == 0) wsum[0][w] = __popcll(me);
    __syncthreads();
    int before = eq0, total = 0;
    for (int i = 0; i < NW; ++i) {
      before += i < w ? wsum[0][i] : 0;
      total += wsum[0][i];
    }
    before += lanes_below(me, lane);
    eq0 += total;
    const bool kept = t < n && (k > last || (eq && before < ties));
    const bool hole = t < left && !kept, mover = t >= left && kept;
    const unsigned long long mh = __ballot(hole), mm = __ballot(mover);
    __syncthreads();
    if (lane == 0) {
      wsum[0][w] = __popcll(mh);
      wsum[1][w] = __popcll(mm);
    }
    __syncthreads();
    int hb = holes, mb = movers, ht = 0, mt = 0;
    for (int i = 0; i < NW; ++i) {
      hb += i < w ? wsum[0][i] : 0;
      mb += i < w ? wsum[1][i] : 0;
      ht += wsum[0][i];
      mt += wsum[1][i];
    }
    if (hole) mv[hb + lanes_below(mh, lane)].x = t;
    if (mover) mv[mb + lanes_below(mm, lane)].y = t;
    holes += ht;
    movers += mt;
  }
  __threadfence_block();
  __syncthreads();
  if (tid == 0) a.n_moves[bj] = movers;
  for (int i = tid; i < movers; i += kNtEvict) {
    const int2 m = mv[i];
    wt[m.x] = wt[m.y];
    if (ps != nullptr) ps[m.x] = ps[m.y];
  }
  __syncthreads();
  for (int t = left + tid; t < n; t += kNtEvict) wt[t] = 0.0f;
}

// `parts` workgroups per (b, j) copy its moves, 16 bytes per lane.  Also the lengths.
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
    k[dst] = k[src];
    v[dst] = v[src];
  }
  if (a.len != nullptr && bj == b * a.n_kv && part == 0 && threadIdx.x == 0)
    a.len[b] = min(min(max(a.len[b], 0), a.T), a.keep);
}

hipError_t launch_evict(const EvictArgs& a, hipStream_t st) {
  const int bjs = a.B * a.n_kv;
  hipLaunchKernelGGL(evict_select_kernel, dim3(bjs), dim3(kNtEvict), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const long long work = (long long)a.max_moves * (a.row_bytes / 16);
  const int parts = (int)std::max<long long>(1, std::min<long long>((work + 1023) / 1024, 2048 / bjs));
  hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)parts * bjs), dim3(256), 0, st, a, parts);
  return hipGetLastError();
}

}  // namespace kvd
