// Running sums over a wave and a workgroup.
#pragma once

#include "esp_internal.h"

// A wave's running sums and reductions by data-parallel-primitive moves (a dozen cycles each; exchanges through LDS take ten times that, and where a
// workgroup decides something such chains are most of what it does): lanes 1, 2, 4, 8 back in a row of 16, then the last of a row to the next one, of two to the others.
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned moved(unsigned v, unsigned idle) {
  return (unsigned)__builtin_amdgcn_update_dpp((int)idle, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t moved(uint64_t v, unsigned) {
  return (uint64_t)moved<CTRL, ROWS>((unsigned)(v >> 32), 0u) << 32 | moved<CTRL, ROWS>((unsigned)v, 0u);
}
template <typename V, typename OP>
__device__ __forceinline__ V running(V v, unsigned idle, OP op) {
  v = op(v, moved<0x111, 0xf>(v, idle));
  v = op(v, moved<0x112, 0xf>(v, idle));
  v = op(v, moved<0x114, 0xf>(v, idle));
  v = op(v, moved<0x118, 0xf>(v, idle));
  v = op(v, moved<0x142, 0xa>(v, idle));
  return op(v, moved<0x143, 0xc>(v, idle));
}
// of a row of 16 lanes: the four steps inside it
template <typename V, typename OP>
__device__ __forceinline__ V running_row(V v, unsigned idle, OP op) {
  v = op(v, moved<0x111, 0xf>(v, idle));
  v = op(v, moved<0x112, 0xf>(v, idle));
  v = op(v, moved<0x114, 0xf>(v, idle));
  return op(v, moved<0x118, 0xf>(v, idle));
}
struct Plus { template <typename V> __device__ __forceinline__ V operator()(V a, V b) const { return a + b; } };
struct Least { __device__ __forceinline__ unsigned operator()(unsigned a, unsigned b) const { return min(a, b); } };
struct Most { __device__ __forceinline__ unsigned operator()(unsigned a, unsigned b) const { return max(a, b); } };
template <typename V>
__device__ __forceinline__ V running_sum(V v) { return running(v, 0u, Plus()); }
__device__ __forceinline__ unsigned lane_of(unsigned v, int l) { return __builtin_amdgcn_readlane(v, l); }
__device__ __forceinline__ uint64_t lane_of(uint64_t v, int l) { return (uint64_t)lane_of((unsigned)(v >> 32), l) << 32 | lane_of((unsigned)v, l); }
template <typename V>
__device__ __forceinline__ V wave_total(V v) { return lane_of(running_sum(v), 63); }

// Of a workgroup's waves (16 at most), in LDS.  Two places that take turns: what is written at one call is read before anybody is past the next one's barrier,
// so a call has one barrier.
template <int WAVES>
struct WaveSums {
  uint64_t sum[2][WAVES];
  unsigned cnt[2][WAVES];
};
// sums of the threads before this one, in place; returns all threads'
template <int WAVES, typename V>
__device__ __forceinline__ V before_in(V (&place)[WAVES], V& v) {
  static_assert(WAVES <= 16, "a row of lanes");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const V q = running_sum(v);
  if (lane == 63) place[wave] = q;
  __syncthreads();
  const V of = running_row(lane < WAVES ? place[lane & (WAVES - 1)] : (V)0, 0u, Plus());
  const int last = __builtin_amdgcn_readfirstlane(wave) - 1;
  v = q - v + (last >= 0 ? lane_of(of, max(last, 0)) : (V)0);
  return lane_of(of, WAVES - 1);
}
template <int WAVES>
__device__ __forceinline__ uint64_t before(WaveSums<WAVES>& s, int& turn, uint64_t& sum) { turn ^= 1; return before_in(s.sum[turn], sum); }
template <int WAVES>
__device__ __forceinline__ unsigned before(WaveSums<WAVES>& s, int& turn, unsigned& cnt) { turn ^= 1; return before_in(s.cnt[turn], cnt); }
// both at once; returns the sum
template <int WAVES>
__device__ __forceinline__ uint64_t before(WaveSums<WAVES>& s, int& turn, uint64_t& sum, unsigned& cnt) {
  static_assert(WAVES <= 16, "a row of lanes");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  turn ^= 1;
  const uint64_t q = running_sum(sum);
  const unsigned c = running_sum(cnt);
  if (lane == 63) { s.sum[turn][wave] = q; s.cnt[turn][wave] = c; }
  __syncthreads();
  const uint64_t q_of = running_row(lane < WAVES ? s.sum[turn][lane & (WAVES - 1)] : (uint64_t)0, 0u, Plus());
  const unsigned c_of = running_row(lane < WAVES ? s.cnt[turn][lane & (WAVES - 1)] : 0u, 0u, Plus());
  const int last = __builtin_amdgcn_readfirstlane(wave) - 1;
  sum = q - sum + (last >= 0 ? lane_of(q_of, max(last, 0)) : (uint64_t)0);
  cnt = c - cnt + (last >= 0 ? lane_of(c_of, max(last, 0)) : 0u);
  return lane_of(q_of, WAVES - 1);
}
