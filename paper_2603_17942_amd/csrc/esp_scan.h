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
template <typename V>
__device__ __forceinline__ V running_sum(V v) { return running(v, 0u, [](V a, V b) { return a + b; }); }
__device__ __forceinline__ unsigned lane_of(unsigned v, int l) { return __builtin_amdgcn_readlane(v, l); }
__device__ __forceinline__ uint64_t lane_of(uint64_t v, int l) { return (uint64_t)lane_of((unsigned)(v >> 32), l) << 32 | lane_of((unsigned)v, l); }
template <typename V>
__device__ __forceinline__ V wave_total(V v) { return lane_of(running_sum(v), 63); }

template <int WAVES>
struct WaveSums {                      // of a workgroup's waves, in LDS
  uint64_t sum[WAVES];
  unsigned cnt[WAVES];
};
// sums of the threads before this one, in place; returns all threads'
template <int WAVES>
__device__ __forceinline__ uint64_t before(WaveSums<WAVES>& s, uint64_t& sum) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t q = running_sum(sum);
  __syncthreads();
  if (lane == 63) s.sum[wave] = q;
  __syncthreads();
  const uint64_t of = running_sum(lane < WAVES ? s.sum[lane & (WAVES - 1)] : (uint64_t)0);
  const int last = __builtin_amdgcn_readfirstlane(wave) - 1;
  sum = q - sum + (last >= 0 ? lane_of(of, max(last, 0)) : (uint64_t)0);
  return lane_of(of, WAVES - 1);
}
template <int WAVES>
__device__ __forceinline__ unsigned before(WaveSums<WAVES>& s, unsigned& cnt) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const unsigned c = running_sum(cnt);
  __syncthreads();
  if (lane == 63) s.cnt[wave] = c;
  __syncthreads();
  const unsigned of = running_sum(lane < WAVES ? s.cnt[lane & (WAVES - 1)] : 0u);
  const int last = __builtin_amdgcn_readfirstlane(wave) - 1;
  cnt = c - cnt + (last >= 0 ? lane_of(of, max(last, 0)) : 0u);
  return lane_of(of, WAVES - 1);
}
