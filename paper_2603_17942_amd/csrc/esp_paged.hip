// Rotary positions with head norms, the append into a paged KV cache, the move of accepted rows, and the way back to
// plain rows.  The attention over the pages is in esp_paged_attn.hip.
#include <algorithm>

#include "esp_paged.h"

namespace {

// sine and cosine of t revolutions: whole and quarter turns come off in fp64, so a far position costs nothing (position 2^20 at one
// radian a position is 1.7e5 turns, known to 2^-36), and what is left, an eighth of a turn at most, is exact to half a step of fp32
__device__ __forceinline__ void turn_sincos(double t, float& s, float& c) {
  t -= rint(t);
  const double q = rint(4.0 * t);
  float s0, c0;
  sincospif((float)(2.0 * (t - 0.25 * q)), &s0, &c0);
  const int quarter = (int)q & 3;
  const float a = quarter & 1 ? c0 : s0, b = quarter & 1 ? s0 : c0;
  s = quarter & 2 ? -a : a;
  c = (quarter == 1 || quarter == 2) ? -b : b;
}

// eight consecutive elements; VEC: 16-byte aligned
template <bool VEC, typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  if constexpr (VEC && sizeof(T) == 4) {
    const f32x4_t a = *reinterpret_cast<const f32x4_t*>(p), b = *reinterpret_cast<const f32x4_t*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
  } else if constexpr (VEC) {
    const bf16x8_t a = *reinterpret_cast<const bf16x8_t*>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)a[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = to_f32(p[e]);
  }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  if constexpr (VEC && sizeof(T) == 4) {
    *reinterpret_cast<f32x4_t*>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4_t*>(p + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
  } else if constexpr (VEC) {
    bf16x8_t a;
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = (bf16_t)v[e];
    *reinterpret_cast<bf16x8_t*>(p) = a;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = from_f32<T>(v[e]);
  }
}

// The sequence that holds row m, by the whole wave: the first that is in order and has it among its rows; -1: none.  (Asked of every sequence, since
// where row0 descends the one that begins last before a row need not hold it.)
__device__ __forceinline__ int find_seq(const PagedDev& kv, const ChunkDev& ch, int m, int lane, ChunkSeq& s) {
  for (int b0 = 0; b0 < kv.batch; b0 += 64) {
    const int b = b0 + lane;
    const ChunkSeq x = chunk_seq(kv, ch, min(b, kv.batch - 1));
    const uint64_t holds = __builtin_amdgcn_ballot_w64(b < kv.batch && x.ok && m >= x.row0 && m - x.row0 < x.rows);
    if (holds) {
      const int l = __builtin_ctzll(holds);
      s = ChunkSeq{__builtin_amdgcn_readlane(x.row0, l), __builtin_amdgcn_readlane(x.rows, l), __builtin_amdgcn_readlane(x.len, l), true};
      return b0 + l;
    }
  }
  return -1;
}

// Sixteen features of a head in two pieces of eight, one thread: of a part that turns the pieces hold its pairs, so a thread
// needs nothing of its neighbours.  HD / 16 threads of a head lie side by side in a wave and add up the squares for the norm.
template <typename T, int HD>
__device__ __forceinline__ void norm_rotate(const RopeRows& a, const T* gain, int j, int u0, int u1, const float2* cs, float (&x0)[8],
                                            float (&x1)[8]) {
  if (gain) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += x0[e] * x0[e] + x1[e] * x1[e];
#pragma unroll
    for (int o = HD / 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o, 64);
    const float inv = 1.0f / sqrtf(ss / (float)HD + a.eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x0[e] *= inv * to_f32(gain[8 * u0 + e]);
      x1[e] *= inv * to_f32(gain[8 * u1 + e]);
    }
  }
  if (16 * j < a.rot) {
    if (a.interleaved) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float2 t0 = cs[4 * u0 + e / 2], t1 = cs[4 * u1 + e / 2];
        const float p0 = x0[e], p1 = x1[e];
        x0[e] = p0 * t0.x - x0[e + 1] * t0.y;
        x0[e + 1] = x0[e + 1] * t0.x + p0 * t0.y;
        x1[e] = p1 * t1.x - x1[e + 1] * t1.y;
        x1[e + 1] = x1[e + 1] * t1.x + p1 * t1.y;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 t = cs[8 * j + e];
        const float p = x0[e];
        x0[e] = p * t.x - x1[e] * t.y;
        x1[e] = x1[e] * t.x + p * t.y;
      }
    }
  }
}
// the two pieces of thread j of a head: pairs (j, j + rot/16) where the head turns, neighbours behind that
__device__ __forceinline__ void pieces_of(int j, int rot, int& u0, int& u1) {
  const bool turns = 16 * j < rot;
  u0 = turns ? j : 2 * j;
  u1 = turns ? j + rot / 16 : 2 * j + 1;
}

// R rows a workgroup, a wave finds a row's place and fills its table of cosines and sines, then all threads take the heads.  One row's chain
// of loads takes 3.5 us; from 1024 rows on four a workgroup: 8192 rows of 32 + 8 heads with norms 36 us, 4.6 TB/s (a copy 4.9).
template <typename T, int HD, bool PAGED, bool VEC, int R>
__device__ __forceinline__ void rope_rows(const RopeRows& a, const PagedDev& kv, const ChunkDev& ch, int hkv, int block) {
  constexpr int LPH = HD / 16;
  __shared__ float2 cs[R][HD / 2];
  __shared__ int page_of[R], slot_of[R];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m0 = block * R;
  for (int i = wave; i < R; i += 4) {
    const int m = m0 + i;
    int page = -1, slot = 0, pos = 0;
    if (m < a.rows) {
      if (PAGED) {
        ChunkSeq s;
        const int seq = find_seq(kv, ch, m, lane, s);
        if (seq >= 0) {
          slot = s.len + (m - s.row0);
          pos = slot;
          page = kv.table[(size_t)seq * kv.stride + slot / kv.page_size];
          slot %= kv.page_size;
          if ((unsigned)page >= (unsigned)kv.n_pages) {
            if (lane == 0) set_status(kv.status, ESP_DEV_BAD_PAGE);
            page = -2;                                    // the query is there, the slot is not
          }
        }
      } else {
        page = 0;
      }
      if (a.positions) pos = a.positions[m];
    }
    if (lane == 0) { page_of[i] = page; slot_of[i] = slot; }
    if (page != -1 && lane < a.rot / 2) {
      float s, c;
      turn_sincos((double)pos * a.turns[lane], s, c);
      cs[i][lane] = float2{c * a.amplitude, s * a.amplitude};
    }
  }
  if (PAGED && block == 0)
    for (int b = tid; b < kv.batch; b += 256)
      if (!chunk_seq(kv, ch, b).ok) set_status(kv.status, chunk_fault(ch, b));
  __syncthreads();
  const int heads = a.hq + (PAGED ? 2 : 1) * hkv, per_row = heads * LPH;
  for (int t = tid; t < R * per_row; t += 256) {
    const int i = t / per_row, head = (t - i * per_row) / LPH, j = t % LPH, m = m0 + i;
    const int page = page_of[i];
    if (page == -1) continue;
    float x0[8], x1[8];
    if (head >= a.hq + hkv) {
      if (page < 0) continue;
      const int kvh = head - a.hq - hkv;
      const T* src = (const T*)a.v + (int64_t)m * a.v_stride + kvh * HD;
      load8<VEC>(src + 8 * j, x0);
      load8<VEC>(src + 8 * (j + LPH), x1);
      T* dst = (T*)kv.v + page_plane(page, kvh, kv.hkv, kv.page_size, HD);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dst[v_off(slot_of[i], 8 * j + e, HD)] = from_f32<T>(x0[e]);
        dst[v_off(slot_of[i], 8 * (j + LPH) + e, HD)] = from_f32<T>(x1[e]);
      }
      continue;
    }
    int u0, u1;
    pieces_of(j, a.rot, u0, u1);
    const bool is_q = head < a.hq;
    const T* src = is_q ? (const T*)a.q + (int64_t)m * a.q_stride + head * HD : (const T*)a.k + (int64_t)m * a.k_stride + (head - a.hq) * HD;
    load8<VEC>(src + 8 * u0, x0);
    load8<VEC>(src + 8 * u1, x1);
    norm_rotate<T, HD>(a, (const T*)(is_q ? a.q_gain : a.k_gain), j, u0, u1, cs[i], x0, x1);
    if (is_q) {
      T* dst = (T*)a.q_out + (int64_t)m * a.q_out_stride + head * HD;
      store8<VEC>(dst + 8 * u0, x0);
      store8<VEC>(dst + 8 * u1, x1);
    } else if (PAGED) {
      if (page < 0) continue;
      T* dst = (T*)kv.k + page_plane(page, head - a.hq, kv.hkv, kv.page_size, HD);
      store8<true>(dst + k_off(slot_of[i], 8 * u0, HD), x0);
      store8<true>(dst + k_off(slot_of[i], 8 * u1, HD), x1);
    } else {
      T* dst = (T*)a.k_out + (int64_t)m * a.k_out_stride + (head - a.hq) * HD;
      store8<VEC>(dst + 8 * u0, x0);
      store8<VEC>(dst + 8 * u1, x1);
    }
  }
}

template <typename T, int HD, bool PAGED, bool VEC, int R>
__global__ __launch_bounds__(256) void k_rope_rows(RopeRows a, PagedDev kv, ChunkDev ch) {
  rope_rows<T, HD, PAGED, VEC, R>(a, kv, ch, a.hkv, blockIdx.x);
}

// The same for chunks of many rows: K and V go by blocks of the cache, a workgroup takes 32 slots and HEADS kv heads and writes
// whole 128-byte lines, V turned from rows to columns through LDS; the queries go by rows, in the workgroups behind these.  (By rows
// a V row is HD stores of one element.)  Four chunks of 700 to 2048 rows, 143 MB: 66 us by rows, 37 by blocks, 3.9 TB/s (31 and 4.7 with
// the rows in the last cache, as behind a projection)
template <int HD> constexpr int BLOCK_HEADS = 128 / HD;
template <typename T, int HD, bool VEC, int R>
__global__ __launch_bounds__(256) void k_append_blocks(RopeRows a, PagedDev kv, ChunkDev ch, int block_groups, int head_groups) {
  constexpr int LPH = HD / 16, HEADS = BLOCK_HEADS<HD>;
  typedef T piece_t __attribute__((ext_vector_type(8)));
  if ((int)blockIdx.x >= block_groups) {
    rope_rows<T, HD, true, VEC, R>(a, kv, ch, 0, blockIdx.x - block_groups);
    return;
  }
  __shared__ float2 cs[32][HD / 2];
  __shared__ __align__(16) T vt[HEADS][32][HD + 8];
  const int tid = threadIdx.x, lane = tid & 63;
  const int kvh0 = blockIdx.x % head_groups * HEADS;
  // the blocks of the sequences, one after the other: which one is this?
  const int x = blockIdx.x / head_groups;
  if (blockIdx.x == 0 && a.hq == 0)
    for (int b = tid; b < kv.batch; b += 256)
      if (!chunk_seq(kv, ch, b).ok) set_status(kv.status, chunk_fault(ch, b));
  int seq = -1, block = 0;
  for (int b0 = 0, base = 0; b0 < kv.batch && seq < 0; b0 += 64) {
    const ChunkSeq s = chunk_seq(kv, ch, min(b0 + lane, kv.batch - 1));
    const int first = s.len >> 5, mine = s.ok && s.rows > 0 && b0 + lane < kv.batch ? ((s.len + s.rows - 1) >> 5) - first + 1 : 0;
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(upto, o, 64);
      if (lane >= o) upto += y;
    }
    const uint64_t here = __builtin_amdgcn_ballot_w64(base + upto > x);
    if (here) {
      const int l = __builtin_ctzll(here);
      seq = b0 + l;
      block = __builtin_amdgcn_readlane(first, l) + x - base - __builtin_amdgcn_readlane(upto - mine, l);
    }
    base += __builtin_amdgcn_readlane(upto, 63);
  }
  if (seq < 0) return;
  const ChunkSeq s = chunk_seq(kv, ch, seq);
  const int slot0 = 32 * block, page = kv.table[(size_t)seq * kv.stride + slot0 / kv.page_size], inside = slot0 % kv.page_size;
  const int lo = max(s.len - slot0, 0), hi = min(s.len + s.rows - slot0, 32);       // of the block's slots
  const int m0 = s.row0 + slot0 - s.len;                                            // row of its first slot
  if ((unsigned)page >= (unsigned)kv.n_pages) {
    if (tid == 0) set_status(kv.status, ESP_DEV_BAD_PAGE);
    return;
  }
  const int i = tid / LPH % 32, j = tid % LPH, h = tid / (LPH * 32), kvh = kvh0 + h, m = m0 + i;
  const bool mine = i >= lo && i < hi && kvh < a.hkv;
  int u0, u1;
  pieces_of(j, a.rot, u0, u1);
  float k0[8], k1[8], v0[8], v1[8];
  if (mine) {
    const T* ks = (const T*)a.k + (int64_t)m * a.k_stride + kvh * HD;
    const T* vs = (const T*)a.v + (int64_t)m * a.v_stride + kvh * HD;
    load8<VEC>(ks + 8 * u0, k0);
    load8<VEC>(ks + 8 * u1, k1);
    load8<VEC>(vs + 8 * j, v0);
    load8<VEC>(vs + 8 * (j + LPH), v1);
  }
  for (int t = tid; t < 32 * (a.rot / 2); t += 256) {
    const int r = t / (a.rot / 2), e = t - r * (a.rot / 2);
    if (r < lo || r >= hi) continue;
    float sn, c;
    turn_sincos((double)(a.positions ? a.positions[m0 + r] : slot0 + r) * a.turns[e], sn, c);
    cs[r][e] = float2{c * a.amplitude, sn * a.amplitude};
  }
  if (mine) {
    store8<true>(&vt[h][i][8 * j], v0);
    store8<true>(&vt[h][i][8 * (j + LPH)], v1);
  }
  __syncthreads();
  if (mine) {
    norm_rotate<T, HD>(a, (const T*)a.k_gain, j, u0, u1, cs[i], k0, k1);
    T* dst = (T*)kv.k + page_plane(page, kvh, kv.hkv, kv.page_size, HD);
    store8<true>(dst + k_off(inside + i, 8 * u0, HD), k0);
    store8<true>(dst + k_off(inside + i, 8 * u1, HD), k1);
  }
#pragma unroll
  for (int t = tid; t < HEADS * HD * 4; t += 256) {           // 16-byte pieces of V's block
    const int hv = t / (HD * 4), at = t % (HD * 4), frag = at >> 6, l = at & 63, d = (frag >> 1) * 32 + (l & 31), key0 = (frag & 1) * 16 + 4 * (l >> 5);
    if (kvh0 + hv >= a.hkv) continue;
    T* dst = (T*)kv.v + page_plane(page, kvh0 + hv, kv.hkv, kv.page_size, HD) + (size_t)(inside >> 5) * (32 * HD) + at * 8;
    piece_t p;
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = vt[hv][key0 + (e & 3) + 8 * (e >> 2)][d];
    if (key0 >= lo && key0 + 12 <= hi) {
      *reinterpret_cast<piece_t*>(dst) = p;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = key0 + (e & 3) + 8 * (e >> 2);
        if (key >= lo && key < hi) dst[e] = p[e];
      }
    }
  }
}

// What is wrong with a sequence's path (0: nothing): its rows ascend from 1 on, and rows and places lie in the table.
__device__ __forceinline__ int path_fault(const PagedDev& kv, int L, int n, const int32_t* path) {
  const int64_t cap = (int64_t)kv.stride * kv.page_size;
  if (n < 0 || n > ESP_MAX_MASKS + 1) return ESP_DEV_BAD_PATH;
  if (L < 0 || L > kv.len_bound || (int64_t)L + n > cap) return ESP_DEV_LEN_OVER_BOUND;
  bool ok = true;
#pragma unroll
  for (int i = 1; i <= ESP_MAX_MASKS; ++i) {
    const int r = path[i], before = i > 1 ? path[i - 1] : 0;
    ok &= i >= n || ((r > before) & ((int64_t)L + r < cap));
  }
  return ok ? 0 : ESP_DEV_BAD_PATH;
}

// A wave moves one (layer, kv head) of a sequence's path: everything is read before anything is written, since a row's place may be another's
// source.  A V row is HD single elements 16 bytes apart, a sector of memory each: 16 sequences in 32 layers 12.5 us (15.4 with a workgroup a
// plane); one sequence, and the launch that advances len in place, 4.9.
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_paged_commit(PagedDev kv, int planes, const int32_t* __restrict__ n_emit, const int32_t* __restrict__ accepted,
                                                      int32_t* len_out) {
  constexpr int MOST = ESP_MAX_MASKS;                  // rows that can move
  typedef T piece_t __attribute__((ext_vector_type(8)));
  const int seq = blockIdx.y, plane_of = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int layer = plane_of / kv.hkv, kvh = plane_of % kv.hkv;
  const int L = kv.len[seq], n = n_emit[seq];
  const int32_t* path = accepted + (size_t)seq * (ESP_MAX_MASKS + 1);
  const int fault = path_fault(kv, L, n, path);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (fault) set_status(kv.status, fault);
    if (len_out) len_out[seq] = fault ? L : L + n;
  }
  if (fault || plane_of >= planes) return;
  const size_t layer0 = (size_t)layer * kv.n_pages * kv.hkv * kv.page_size * HD;
  T* kp = (T*)kv.k + layer0;
  T* vp = (T*)kv.v + layer0;
  const int32_t* table = kv.table + (size_t)seq * kv.stride;
  // where rows lie and go: the same for the whole wave
  size_t from[MOST], to[MOST];
  int from_in[MOST], to_in[MOST];
  bool moves[MOST], lands[MOST];
  auto place = [&](int s, size_t& plane, int& inside) {
    const int page = table[s / kv.page_size];
    inside = s % kv.page_size;
    const bool there = (unsigned)page < (unsigned)kv.n_pages;
    if (!there && lane == 0) set_status(kv.status, ESP_DEV_BAD_PAGE);
    plane = page_plane(there ? page : 0, kvh, kv.hkv, kv.page_size, HD);
    return there;
  };
#pragma unroll
  for (int i = 0; i < MOST; ++i) {
    moves[i] = i + 1 < n && path[i + 1] != i + 1 && place(L + path[i + 1], from[i], from_in[i]);
    lands[i] = moves[i] && place(L + i + 1, to[i], to_in[i]);
  }
  constexpr int VE = HD / 64, PIECES = HD / 8;
  T v[MOST][VE];
  piece_t k[MOST];
#pragma unroll
  for (int i = 0; i < MOST; ++i) {
    if (!moves[i]) continue;
#pragma unroll
    for (int e = 0; e < VE; ++e) v[i][e] = vp[from[i] + v_off(from_in[i], lane + 64 * e, HD)];
    if (lane < PIECES) k[i] = *reinterpret_cast<const piece_t*>(kp + from[i] + k_off(from_in[i], 8 * lane, HD));
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
  for (int i = 0; i < MOST; ++i) {
    if (!lands[i]) continue;
#pragma unroll
    for (int e = 0; e < VE; ++e) vp[to[i] + v_off(to_in[i], lane + 64 * e, HD)] = v[i][e];
    if (lane < PIECES) *reinterpret_cast<piece_t*>(kp + to[i] + k_off(to_in[i], 8 * lane, HD)) = k[i];
  }
}

// the lengths, where they are advanced in place: the workgroups that move rows read them
__global__ void k_paged_advance(PagedDev kv, const int32_t* __restrict__ n_emit, const int32_t* __restrict__ accepted, int32_t* len) {
  const int seq = blockIdx.x * blockDim.x + threadIdx.x;
  if (seq >= kv.batch) return;
  const int L = len[seq], n = n_emit[seq];
  if (path_fault(kv, L, n, accepted + (size_t)seq * (ESP_MAX_MASKS + 1)) == 0) len[seq] = L + n;
}

template <typename T, int HD>
__global__ __launch_bounds__(256) void k_paged_load(PagedDev kv, int seq, int first_slot, size_t n, T* __restrict__ k_rows,
                                                    T* __restrict__ v_rows) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const int d = (int)(i % HD), kvh = (int)(i / HD % kv.hkv), s = first_slot + (int)(i / ((size_t)HD * kv.hkv));
  const int page = kv.table[(size_t)seq * kv.stride + s / kv.page_size], inside = s % kv.page_size;
  T k = from_f32<T>(0.f), v = k;
  if ((unsigned)page < (unsigned)kv.n_pages) {
    const size_t plane = page_plane(page, kvh, kv.hkv, kv.page_size, HD);
    k = ((const T*)kv.k)[plane + k_off(inside, d, HD)];
    v = ((const T*)kv.v)[plane + v_off(inside, d, HD)];
  } else {
    set_status(kv.status, ESP_DEV_BAD_PAGE);
  }
  k_rows[i] = k;
  v_rows[i] = v;
}

template <typename T>
bool rows_aligned(const RopeRows& a, bool paged) {
  auto fits = [](const void* p, int64_t stride) { return (uintptr_t)p % 16 == 0 && stride * (int64_t)sizeof(T) % 16 == 0; };
  bool ok = true;
  if (a.hq) ok = ok && fits(a.q, a.q_stride) && fits(a.q_out, a.q_out_stride);
  if (a.hkv) ok = ok && fits(a.k, a.k_stride) && (paged ? fits(a.v, a.v_stride) : fits(a.k_out, a.k_out_stride));
  return ok;
}

template <typename T, int HD, bool PAGED>
hipError_t launch_rows(hipStream_t st, const RopeRows& a, const PagedDev& kv, const ChunkDev& ch) {
  const bool vec = rows_aligned<T>(a, PAGED);
  const int r = a.rows >= 1024 ? 4 : 1;
  const dim3 grid((unsigned)((a.rows + r - 1) / r));
#define ESP_ROPE_ROWS(V_, R_) hipLaunchKernelGGL((k_rope_rows<T, HD, PAGED, V_, R_>), grid, dim3(256), 0, st, a, kv, ch)
  if (r == 4) { if (vec) ESP_ROPE_ROWS(true, 4); else ESP_ROPE_ROWS(false, 4); }
  else { if (vec) ESP_ROPE_ROWS(true, 1); else ESP_ROPE_ROWS(false, 1); }
#undef ESP_ROPE_ROWS
  return hipGetLastError();
}

template <typename T, int HD>
hipError_t launch_append(hipStream_t st, const RopeRows& a, const PagedDev& kv, const ChunkDev& ch) {
  const int r = a.rows >= 1024 ? 4 : 1, head_groups = (a.hkv + BLOCK_HEADS<HD> - 1) / BLOCK_HEADS<HD>;
  const int64_t block_groups = ((int64_t)a.rows / 32 + 2 * (int64_t)kv.batch) * head_groups, grid = block_groups + (a.hq ? (a.rows + r - 1) / r : 0);
  // by rows / by blocks, 32/8 heads of 128 in bf16, us: 64 rows 5.3 / 7.0, 320 7.5 / 7.3, 32 x 8 7.0 / 7.6, 32 x 16 9.0 / 7.6, 8192 61 / 40
  if (a.rows < 256 || a.rows < 16 * kv.batch || grid > MOST_WORKGROUPS) return launch_rows<T, HD, true>(st, a, kv, ch);
  const bool vec = rows_aligned<T>(a, true);
#define ESP_APPEND(V_, R_) \
  hipLaunchKernelGGL((k_append_blocks<T, HD, V_, R_>), dim3((unsigned)grid), dim3(256), 0, st, a, kv, ch, (int)block_groups, head_groups)
  if (r == 4) { if (vec) ESP_APPEND(true, 4); else ESP_APPEND(false, 4); }
  else { if (vec) ESP_APPEND(true, 1); else ESP_APPEND(false, 1); }
#undef ESP_APPEND
  return hipGetLastError();
}

template <typename T, int HD>
hipError_t launch_commit(hipStream_t st, const PagedDev& kv, int layers, const int32_t* n_emit, const int32_t* accepted, int32_t* len_out) {
  const bool in_place = len_out == kv.len;
  hipLaunchKernelGGL((k_paged_commit<T, HD>), dim3((layers * kv.hkv + 3) / 4, kv.batch), dim3(256), 0, st, kv, layers * kv.hkv, n_emit, accepted, in_place ? nullptr : len_out);
  if (in_place) hipLaunchKernelGGL(k_paged_advance, dim3((kv.batch + 255) / 256), dim3(256), 0, st, kv, n_emit, accepted, len_out);
  return hipGetLastError();
}
template <typename T, int HD>
hipError_t launch_load(hipStream_t st, const PagedDev& kv, int seq, int first_slot, int n_slots, void* k_rows, void* v_rows) {
  const int64_t row = (int64_t)kv.hkv * HD, at_once = 256 * MOST_WORKGROUPS / row;
  for (int64_t done = 0; done < n_slots; done += at_once) {
    const size_t n = (size_t)(std::min(at_once, n_slots - done) * row);
    hipLaunchKernelGGL((k_paged_load<T, HD>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, kv, seq, first_slot + (int)done, n,
                       (T*)k_rows + done * row, (T*)v_rows + done * row);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

#define ESP_BY_TYPE(CALL)                                                        \
  (dtype == ESP_F32 ? (hd == 64 ? CALL(float, 64) : CALL(float, 128)) : (hd == 64 ? CALL(bf16_t, 64) : CALL(bf16_t, 128)))

hipError_t launch_rope_rows(hipStream_t st, int dtype, int hd, const RopeRows& a) {
#define ESP_CALL(T_, HD_) (launch_rows<T_, HD_, false>(st, a, PagedDev{}, ChunkDev{}))
  return ESP_BY_TYPE(ESP_CALL);
#undef ESP_CALL
}

hipError_t launch_paged_append(hipStream_t st, int dtype, int hd, const PagedDev& kv, const ChunkDev& ch, const RopeRows& a) {
#define ESP_CALL(T_, HD_) (launch_append<T_, HD_>(st, a, kv, ch))
  return ESP_BY_TYPE(ESP_CALL);
#undef ESP_CALL
}

hipError_t launch_paged_commit(hipStream_t st, int dtype, int hd, const PagedDev& kv, int layers, const int32_t* n_emit,
                               const int32_t* accepted, int32_t* len_out) {
#define ESP_CALL(T_, HD_) (launch_commit<T_, HD_>(st, kv, layers, n_emit, accepted, len_out))
  return ESP_BY_TYPE(ESP_CALL);
#undef ESP_CALL
}

hipError_t launch_paged_load(hipStream_t st, int dtype, int hd, const PagedDev& kv, int seq, int first_slot, int n_slots, void* k_rows,
                             void* v_rows) {
#define ESP_CALL(T_, HD_) (launch_load<T_, HD_>(st, kv, seq, first_slot, n_slots, k_rows, v_rows))
  return ESP_BY_TYPE(ESP_CALL);
#undef ESP_CALL
}
