// How much attention a chunk's rows give to each cached token (esp_paged_weigh): mass[t] = before[t] + sum over counted rows r and the kv
// head's queries g of softmax_t(scale q_rg . k_t), causal.
//
// A token's sum needs every row's largest score and sum of exponentials first, so there are two looks at the scores.  Few columns (row, query
// head of the kv head: up to 32, a decode step's): K is what has to be read, once; the scores, 4 bytes each, go to scratch with the share's
// statistics, and a second kernel adds up their exponentials, a thread a token.  Many columns (a prompt's): the products are what costs, and are
// taken twice.  First a wave has 32 columns (bf16: 64) and goes over the keys, for the statistics; then a wave has 32 keys (bf16: 64) and goes over the
// columns, whose tiles four waves share through LDS, so that a token's sum stays in a lane and nothing is added by atomics: the same bits every time.
//
// What bounds them, at 32 query and 8 kv heads of 128 in bf16: 32 ragged sequences' single rows read 522 MB of K, 101 us at the rate of a copy, and take
// 121 (scores 108, sums 14).  A prompt of 4096 takes its 137 GF of products in twice 120 to 133 us, 45% of the rate of a large product: matrix
// instructions for 25% of the time, the exponentials' vector instructions for 40%, and 1.1 and 1.7 waves a SIMD on average, too few for one to hide behind
// the other.  The registers (217 and 164) leave room for 2 and 3: the workgroups have unequal work, as shares and parts are of equal size and what a row sees is a
// triangle, so CUs stand idle towards the end (counted in units, with workgroups taken in turn, at most 1.6 and 2.1 waves a SIMD on average; with equal ones 2 and 2.7).
//
// Scores are S = Q K^T on 32 x 32 matrix instructions.  With keys as the second operand a lane has one key and the columns
// 8 (v / 4) + 4 half + v % 4 in its 16 registers; with keys first (the statistics of many columns) one column and those keys.
#include <algorithm>
#include <cfloat>

#include "esp_attn_unit.h"
#include "esp_paged.h"

namespace {

constexpr int WAVES = 4, THREADS = 64 * WAVES;
constexpr int stat_tiles(bool bf16) { return bf16 ? 2 : 1; }      // column tiles of a wave of the statistics

struct WeighSeq {            // a sequence's counted rows: the last `rows` of its chunk
  int first_row;             // in the chunk
  int first, rows, len, total;       // total: len and all rows
  bool ok;
};
__device__ __forceinline__ WeighSeq weigh_seq(const PagedDev& kv, const ChunkDev& ch, int seq, int last, int slots) {
  const ChunkSeq c = chunk_seq(kv, ch, seq);
  const bool ok = c.ok && (int64_t)c.len + c.rows <= slots;
  const int n = last > 0 ? min(c.rows, last) : c.rows;
  return {c.row0, c.rows - n, n, c.len, c.len + c.rows, ok};
}

// Units of 32 keys of a sequence and kv head, one after the other: a lane has the page of one of 64 pages ahead, so that a unit's address takes no look
// into the table of its own.
template <typename T>
struct Units {
  const int32_t* table;
  const T* k;                          // of the layer
  size_t plane;                        // elements of a page and kv head, before it those of the page's other heads
  int hkv, kvh, n_pages, pages_end, of_page, first_page, pages;
  __device__ __forceinline__ Units(const PagedDev& kv, int seq, int kvh_, int hd)
      : table(kv.table + (size_t)seq * kv.stride), k((const T*)kv.k), plane((size_t)kv.page_size * hd), hkv(kv.hkv), kvh(kvh_), n_pages(kv.n_pages),
        pages_end(kv.stride), of_page(kv.page_size / 32), first_page(-64), pages(0) {}
  // first element of a unit; null: its page is outside the pool
  __device__ __forceinline__ const T* at(int unit, int page, int hd) {
    if (page >= first_page + 64 || page < first_page) {
      first_page = page;
      const int i = page + (int)(threadIdx.x & 63);
      pages = i < pages_end ? table[i] : -1;
    }
    const int id = __builtin_amdgcn_readlane(pages, page - first_page);
    if (id < 0 || id >= n_pages) return nullptr;
    return k + ((size_t)id * hkv + kvh) * plane + (size_t)(unit - page * of_page) * 32 * hd;
  }
  __device__ __forceinline__ const T* at(int unit, int hd) { return at(unit, unit / of_page, hd); }
};
template <typename T, int HD>
__device__ __forceinline__ void load_unit(const T* p, int lane, typename AttnFrag<T>::type (&k)[HD / 16]) {
  typedef typename AttnFrag<T>::type F;
#pragma unroll
  for (int s = 0; s < HD / 16; ++s) k[s] = *reinterpret_cast<const F*>(p + (s * 64 + lane) * 8);
}
// eight features of q (null: zeros); WHOLE: 16-byte loads
template <typename T>
__device__ __forceinline__ typename AttnFrag<T>::type load_eight(const T* p, bool whole) {
  typedef typename AttnFrag<T>::type F;
  F f = {};
  if (p && whole) {
    f = *reinterpret_cast<const F*>(p);
  } else if (p) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = p[e];
  }
  return f;
}
// features of one column as operand: 16 s + 8 half + 0..7
template <typename T, int HD>
__device__ __forceinline__ void load_column(const T* p, int half, bool whole, typename AttnFrag<T>::type (&q)[HD / 16]) {
#pragma unroll
  for (int s = 0; s < HD / 16; ++s) q[s] = load_eight<T>(p ? p + 16 * s + 8 * half : nullptr, whole);
}

// (reference, sum of exponentials against it).  The reference is the largest score times the scale, rounded, and is the same number
// wherever it is taken away: scale times a difference of two scores is not, by 2^-24 of the references.
__device__ __forceinline__ float2 join(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  return {m, a.y * __builtin_amdgcn_exp2f(a.x - m) + b.y * __builtin_amdgcn_exp2f(b.x - m)};
}
// (reference, 1 / sum): a row that saw nothing gives nothing
__device__ __forceinline__ float2 finish(float2 a) { return {a.x, a.y == 0.f ? 0.f : 1.f / a.y}; }

// ---- few columns ---------------------------------------------------------------------------------------------

// What a score is where a column does not see the token.  Not minus infinity: a score can be that, which weighs nothing, but is NaN in a row that is.
constexpr float NOT_SEEN = -FLT_MAX;

// scores [seq][kvh][t][width] of columns below `width`; stats [seq][kvh][share][width].  K's bytes are what bounds it.  (bf16 with up to eight columns: 128 registers
// and four waves a SIMD instead of 132 and three, 123 us instead of 128 for 32 ragged sequences, sums included)
template <typename T, int HD, int NV>      // NV: groups of eight columns
__global__ __launch_bounds__(THREADS, sizeof(T) == 2 && NV == 1 ? 4 : 1) void k_weigh_scores(PagedDev kv, ChunkDev ch, WeighArgs a, WeighPlan p) {
  typedef typename AttnFrag<T>::type F;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
  const int share = blockIdx.x, kvh = blockIdx.y, seq = blockIdx.z;
  const WeighSeq c = weigh_seq(kv, ch, seq, a.last, a.slots);
  if (!c.ok) {
    if (share == 0 && kvh == 0 && tid == 0) set_status(kv.status, chunk_fault(ch, seq));
    return;
  }
  const int units = (c.total + 31) / 32, begin = share * p.share_units, end = min(begin + p.share_units, units);
  if (c.rows == 0 || begin >= end) return;
  const int G = a.hq / kv.hkv, cols = c.rows * G;
  F q[HD / 16], k[HD / 16], next[HD / 16] = {};
  const int mine = lane & 31;
  load_column<T, HD>(mine < cols ? (const T*)a.q + (int64_t)(c.first_row + c.first + mine / G) * a.q_stride + (int64_t)(kvh * G + mine % G) * HD : nullptr, half, a.whole, q);
  int sees[4 * NV];                    // last slot that a column sees
  float m[4 * NV], l[4 * NV];
#pragma unroll
  for (int v = 0; v < 4 * NV; ++v) {
    const int col = 8 * (v >> 2) + 4 * half + (v & 3);
    sees[v] = col < cols ? c.len + c.first + col / G : -1;
    m[v] = ATTN_UNSEEN;
    l[v] = 0.f;
  }
  float* scores = a.scratch + p.stats_floats + ((int64_t)seq * kv.hkv + kvh) * p.tokens * p.width;
  Units<T> units_of(kv, seq, kvh, HD);
  const int w0 = __builtin_amdgcn_readfirstlane(wave);
  const T* at = begin + w0 < end ? units_of.at(begin + w0, HD) : nullptr;
  if (at) load_unit<T, HD>(at, lane, next);
  for (int u = begin + w0; u < end; u += WAVES) {
    const bool there = at != nullptr;
    if (!there && lane == 0) set_status(kv.status, ESP_DEV_BAD_PAGE);
#pragma unroll
    for (int s = 0; s < HD / 16; ++s) k[s] = next[s];
    if (u + WAVES < end) {
      at = units_of.at(u + WAVES, HD);
      if (at) load_unit<T, HD>(at, lane, next);
    }
    f32x16_t x = {};
#pragma unroll
    for (int s = 0; s < HD / 16; ++s) x = attn_mma(q[s], k[s], x);
    const int slot = 32 * u + mine;
#pragma unroll
    for (int v = 0; v < 4 * NV; ++v) {
      const bool seen = there && slot <= sees[v];
      const float top = seen ? fmaxf(m[v], x[v] * a.scale) : m[v];
      const float e = seen ? __builtin_amdgcn_exp2f(fmaf(x[v], a.scale, -top)) : 0.f;
      l[v] = l[v] * __builtin_amdgcn_exp2f(m[v] - top) + e;
      m[v] = top;
      x[v] = seen ? x[v] : NOT_SEEN;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (8 * i + 4 * half < p.width && slot < c.total)
        *reinterpret_cast<f32x4_t*>(scores + (int64_t)slot * p.width + 8 * i + 4 * half) = f32x4_t{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
  }
  __shared__ float2 part[WAVES][32];
#pragma unroll
  for (int v = 0; v < 4 * NV; ++v) {
    float2 r = {m[v], l[v]};
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) r = join(r, float2{__shfl_xor(r.x, o, 64), __shfl_xor(r.y, o, 64)});
    if (mine == 0) part[wave][8 * (v >> 2) + 4 * half + (v & 3)] = r;
  }
  __syncthreads();
  if (tid < p.width) {
    float2 r = part[0][tid];
    for (int w = 1; w < WAVES; ++w) r = join(r, part[w][tid]);
    reinterpret_cast<float2*>(a.scratch)[(((int64_t)seq * kv.hkv + kvh) * p.shares + share) * p.width + tid] = r;
  }
}

template <int EACH>                     // tokens of a thread
__global__ __launch_bounds__(THREADS) void k_weigh_sum(PagedDev kv, ChunkDev ch, WeighArgs a, WeighPlan p) {
  const int tid = threadIdx.x, kvh = blockIdx.y, seq = blockIdx.z, slot0 = blockIdx.x * THREADS * EACH;
  const WeighSeq c = weigh_seq(kv, ch, seq, a.last, a.slots);
  if (!c.ok || c.rows == 0 || slot0 >= c.total) return;
  __shared__ float2 col[THREADS];
  const int64_t head = (int64_t)seq * kv.hkv + kvh;
  // thread: column tid % width, shares tid / width and every THREADS / width on
  const int shares = ((c.total + 31) / 32 + p.share_units - 1) / p.share_units;
  const float2* s = reinterpret_cast<const float2*>(a.scratch) + head * p.shares * p.width;
  float2 r = {ATTN_UNSEEN, 0.f};
  for (int i = tid / p.width; i < shares; i += THREADS / p.width) r = join(r, s[i * p.width + tid % p.width]);
  col[tid] = r;
  for (int n = THREADS / 2; n >= p.width; n /= 2) {
    __syncthreads();
    if (tid < n) col[tid] = join(col[tid], col[tid + n]);
  }
  if (tid < p.width) col[tid] = finish(col[tid]);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const int slot = slot0 + j * THREADS + tid;
    if (slot >= c.total) return;
    const float* x = a.scratch + p.stats_floats + (head * p.tokens + slot) * p.width;
    const int64_t at = head * a.slots + slot;
    const float old = a.before && slot < c.len ? a.before[at] : 0.f;
    float sum = 0.f;
    for (int i = 0; i < p.width; i += 4) {
      const f32x4_t v = *reinterpret_cast<const f32x4_t*>(x + i);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sum = v[e] == NOT_SEEN ? sum : fmaf(__builtin_amdgcn_exp2f(fmaf(v[e], a.scale, -col[i + e].x)), col[i + e].y, sum);
    }
    a.mass[at] = old + sum;
  }
}

// ---- many columns --------------------------------------------------------------------------------------------

// columns of a sequence and kv head begin at this one of the statistics
__device__ __forceinline__ int64_t first_column(const WeighPlan& p, const WeighSeq& c, const PagedDev& kv, int G, int seq, int kvh) {
  return p.packed ? ((int64_t)c.first_row * kv.hkv + (int64_t)kvh * (c.total - c.len)) * G : ((int64_t)seq * kv.hkv + kvh) * p.most_rows * G;
}

// CT column tiles a wave: what it loads of K serves them all
template <typename T, int HD, int CT>
__global__ __launch_bounds__(THREADS, 2) void k_weigh_stats(PagedDev kv, ChunkDev ch, WeighArgs a, WeighPlan p) {
  typedef typename AttnFrag<T>::type F;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
  // Late columns have the most to do and come first.  Workgroups go to the XCDs in turn, and early columns have no last shares: column groups lie next to
  // each other, shares far apart (eight shares next to each other: 204 us for a prompt of 4096, half of the XCDs idle most of the time; so 158), and
  // groups are turned by one from head to head.  (With units' scores among exponentials, below: 120.)
  const int block = gridDim.x - 1 - blockIdx.x, groups = gridDim.x / p.shares, kvh = blockIdx.y, seq = blockIdx.z;
  const int share = block / groups, tile = ((block + kvh) % groups * WAVES + wave) * CT;
  const WeighSeq c = weigh_seq(kv, ch, seq, a.last, a.slots);
  if (!c.ok) {
    if (blockIdx.x == 0 && kvh == 0 && tid == 0) set_status(kv.status, chunk_fault(ch, seq));
    return;
  }
  const int G = a.hq / kv.hkv, cols = c.rows * G;
  if (32 * tile >= cols) return;       // (no barrier below)
  const int top_row = c.first + min(32 * (tile + CT) - 1, cols - 1) / G;
  const int begin = share * p.share_units, end = min(begin + p.share_units, (c.len + top_row) / 32 + 1);
  float2* out = reinterpret_cast<float2*>(a.scratch) + share * p.columns + first_column(p, c, kv, G, seq, kvh);
  if (begin >= end) {                  // (none of the share's units is seen: then there are several)
    for (int col = 32 * tile + lane; col < min(32 * (tile + CT), cols); col += 64) out[col] = {ATTN_UNSEEN, 0.f};
    return;
  }
  F q[CT][HD / 16], k[HD / 16] = {}, next[HD / 16] = {};
  Units<T> units(kv, seq, kvh, HD);
  bool there = false, next_there = false;
  auto fetch = [&](int u, F (&key)[HD / 16], bool& is_there) {
    const T* at = u < end ? units.at(u, HD) : nullptr;
    is_there = at != nullptr;
    if (at) load_unit<T, HD>(at, lane, key);
    else if (u < end && lane == 0) set_status(kv.status, ESP_DEV_BAD_PAGE);
  };
  fetch(begin, k, there);
  int sees[CT];
  float m[CT], l[CT];
#pragma unroll
  for (int i = 0; i < CT; ++i) {
    const int col = 32 * (tile + i) + (lane & 31), row = c.first + min(col, cols - 1) / G;
    load_column<T, HD>(col < cols ? (const T*)a.q + (int64_t)(c.first_row + row) * a.q_stride + (int64_t)(kvh * G + col % G) * HD : nullptr, half,
                       a.whole, q[i]);
    sees[i] = c.len + row;
    m[i] = ATTN_UNSEEN;
    l[i] = 0.f;
  }
  auto scores = [&](const F (&key)[HD / 16], f32x16_t (&x)[CT]) {
#pragma unroll
    for (int i = 0; i < CT; ++i) x[i] = f32x16_t{};
#pragma unroll
    for (int s = 0; s < HD / 16; ++s)
#pragma unroll
      for (int i = 0; i < CT; ++i) x[i] = attn_mma(key[s], q[i][s], x[i]);
  };
  // what a unit's scores add to the statistics
  auto add = [&](const f32x16_t (&x)[CT]) {
#pragma unroll
    for (int i = 0; i < CT; ++i) {
      float top = attn_max3(x[i][0], x[i][1], x[i][2]);
#pragma unroll
      for (int v = 3; v < 15; v += 2) top = attn_max3(top, x[i][v], x[i][v + 1]);
      const float ref = fmaxf(m[i], fmaxf(top, x[i][15]) * a.scale);
      float sum = 0.f;
#pragma unroll
      for (int v = 0; v < 16; ++v) sum += __builtin_amdgcn_exp2f(fmaf(x[i][v], a.scale, -ref));
      l[i] = fmaf(l[i], __builtin_amdgcn_exp2f(m[i] - ref), sum);
      m[i] = ref;
    }
  };
  // Units that all columns see whole, as long as their pages are there: one's scores among the other's exponentials (a wave has its SIMD to itself much of the
  // time, and the matrix core would wait for the exponentials and they for it).
  auto both = [&](const F (&key)[HD / 16], f32x16_t (&next_x)[CT], const f32x16_t (&x)[CT]) {
    scores(key, next_x);
    add(x);
#pragma unroll
    for (int i = 0; i < CT * HD / 16 * (sizeof(T) == 2 ? 1 : 8); ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);       // a matrix instruction
      __builtin_amdgcn_sched_group_barrier(0x002, sizeof(T) == 2 ? 8 : 1, 0);
    }
  };
  int u = begin;
  const int end_whole = min(end, (c.len + c.first + 32 * tile / G + 1) / 32);
  f32x16_t x[CT], y[CT];
  if (there && u + 1 < end_whole) {
    fetch(u + 1, next, next_there);
    scores(k, x);
    while (next_there && u + 2 < end_whole) {          // x: scores of unit u; next: keys of the one after
      fetch(u + 2, k, there);
      both(next, y, x);
      ++u;
      if (!there || u + 2 >= end_whole) {
#pragma unroll
        for (int i = 0; i < CT; ++i) x[i] = y[i];
#pragma unroll
        for (int s = 0; s < HD / 16; ++s) next[s] = k[s];
        next_there = there;
        break;
      }
      fetch(u + 2, next, next_there);
      both(k, x, y);
      ++u;
    }
    add(x);
    ++u;
#pragma unroll
    for (int s = 0; s < HD / 16; ++s) k[s] = next[s];
    there = next_there;
  }
  for (; u < end; ++u) {
    if (there) {
      scores(k, x);
#pragma unroll
      for (int i = 0; i < CT; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) x[i][v] = 32 * u + 8 * (v >> 2) + 4 * half + (v & 3) <= sees[i] ? x[i][v] : -INFINITY;
    }
    const bool was_there = there;
    fetch(u + 1, k, there);
    if (was_there) add(x);
  }
#pragma unroll
  for (int i = 0; i < CT; ++i) {
    const float2 r = join(float2{m[i], l[i]}, float2{__shfl_xor(m[i], 32, 64), __shfl_xor(l[i], 32, 64)});
    const int col = 32 * (tile + i) + (lane & 31);
    if (half == 0 && col < cols) out[col] = p.shares > 1 ? r : finish(r);
  }
}

// the shares' statistics together, in the first one's place
__global__ __launch_bounds__(THREADS) void k_weigh_join(PagedDev kv, ChunkDev ch, WeighArgs a, WeighPlan p) {
  const int kvh = blockIdx.y, seq = blockIdx.z, col = blockIdx.x * THREADS + threadIdx.x;
  const WeighSeq c = weigh_seq(kv, ch, seq, a.last, a.slots);
  const int G = a.hq / kv.hkv;
  if (!c.ok || col >= c.rows * G) return;
  float2* s = reinterpret_cast<float2*>(a.scratch) + first_column(p, c, kv, G, seq, kvh) + col;
  const int shares = (c.total + 31) / 32;
  float2 r = s[0];
  for (int i = 1; i < p.shares && i * p.share_units < shares; ++i) r = join(r, s[i * p.columns]);
  *s = finish(r);
}

// KU units of 32 keys a wave.  Column tiles go through two places in LDS: the next one is on its way while this one is used.  (Three places, and the next tile's
// scores among this one's exponentials as in the statistics: 236 registers and a wave a SIMD less, 268 us for a prompt of 4096 instead of 240.)
template <typename T, int HD, int KU>
__global__ __launch_bounds__(THREADS, 2) void k_weigh_add(PagedDev kv, ChunkDev ch, WeighArgs a, WeighPlan p) {
  typedef typename AttnFrag<T>::type F;
  constexpr int EIGHTS = HD / 8 * 32 / THREADS;        // of eight features, a thread's of a tile
  // (columns of a step and half exchanged by the step's number: rows are written eight features a lane, and would all meet in the same banks)
  __shared__ __align__(16) F tile_q[2][HD / 16 * 64];
  __shared__ __align__(16) float ref[2][32], inv[2][32];
  __shared__ int sees[2][32];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
  // (parts turned by one from key tile to key tile: workgroups go to the XCDs in turn, and a tile's first parts may have nothing to do)
  const int tile = blockIdx.x / p.parts, part = p.parts - 1 - (blockIdx.x + tile) % p.parts, kvh = blockIdx.y, seq = blockIdx.z;
  const WeighSeq c = weigh_seq(kv, ch, seq, a.last, a.slots);
  const int tile0 = tile * WAVES * KU * 32;
  if (!c.ok || c.rows == 0 || tile0 >= c.total) return;
  const int G = a.hq / kv.hkv, cols = c.rows * G;
  F k[KU][HD / 16];
  bool there[KU];
  float sum[KU];
  const int unit0 = tile0 / 32 + __builtin_amdgcn_readfirstlane(wave) * KU;
  Units<T> units(kv, seq, kvh, HD);
#pragma unroll
  for (int i = 0; i < KU; ++i) {
    const T* at = 32 * (unit0 + i) < c.total ? units.at(unit0 + i, HD) : nullptr;
    there[i] = at != nullptr;
    sum[i] = 0.f;
#pragma unroll
    for (int s = 0; s < HD / 16; ++s) k[i][s] = F{};
    if (at) load_unit<T, HD>(at, lane, k[i]);
  }
  const float2* stats = reinterpret_cast<const float2*>(a.scratch) + first_column(p, c, kv, G, seq, kvh);
  const T* q0 = (const T*)a.q + (int64_t)(c.first_row + c.first) * a.q_stride + (int64_t)kvh * G * HD;
  // column tiles of this part, less those whose rows all end before the first key
  const int tiles = (cols + 31) / 32, each = (tiles + p.parts - 1) / p.parts;
  const int first_needed = (int)((int64_t)max(0, tile0 - c.len - c.first) * G / 32);
  const int t0 = max(part * each, first_needed), t1 = min((part + 1) * each, tiles);
  F q_next[EIGHTS];
  float2 s_next = {0.f, 0.f};
  // row and query head of this thread's columns of the next tile to be asked for, tile after tile without dividing
  int row[EIGHTS], g[EIGHTS], stat_row = (32 * t0 + (tid & 31)) / G, stat_g = (32 * t0 + (tid & 31)) % G;
  const int more_rows = 32 / G, more_g = 32 % G;
  auto step = [&](int& r, int& h) {
    r += more_rows; h += more_g;
    if (h >= G) { h -= G; ++r; }
  };
#pragma unroll
  for (int i = 0; i < EIGHTS; ++i) {
    const int col = 32 * t0 + (i * THREADS + tid) / (HD / 8);
    row[i] = col / G; g[i] = col % G;
  }
  auto fetch = [&](int t) {
#pragma unroll
    for (int i = 0; i < EIGHTS; ++i) {
      const int e = i * THREADS + tid, f = e % (HD / 8);
      q_next[i] = load_eight<T>(row[i] < c.rows ? q0 + row[i] * a.q_stride + g[i] * HD + 8 * f : nullptr, a.whole);
      step(row[i], g[i]);
    }
    if (tid < 32) {
      const int col = 32 * t + tid;
      s_next = {0.f, 0.f};
      if (col < cols && !p.join_here) s_next = stats[col];
      if (col < cols && p.join_here) {
        s_next = stats[col];
        for (int i = 1; i < p.shares; ++i) s_next = join(s_next, stats[i * p.columns + col]);
        s_next = finish(s_next);
      }
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < EIGHTS; ++i) {
      const int e = i * THREADS + tid, f = e % (HD / 8);
      tile_q[buf][(f >> 1) * 64 + (f & 1) * 32 + ((e / (HD / 8)) ^ (f & 7))] = q_next[i];
    }
    if (tid < 32) {
      ref[buf][tid] = s_next.x; inv[buf][tid] = s_next.y;
      sees[buf][tid] = stat_row < c.rows ? c.len + c.first + stat_row : -1;
      step(stat_row, stat_g);
    }
  };
  int low_row = 32 * t0 / G, low_g = 32 * t0 % G;      // of a tile's first column
  if (t0 < t1) { fetch(t0); put(0); }
  __syncthreads();
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1;
    if (t + 1 < t1) fetch(t + 1);
    f32x16_t x[KU] = {};
    float of_tile[KU] = {};            // (tiles by themselves: 16 and then hundreds of additions in a row, not thousands)
#pragma unroll
    for (int s = 0; s < HD / 16; ++s) {
      const F q = tile_q[buf][s * 64 + 32 * half + ((lane & 31) ^ ((2 * s + half) & 7))];
#pragma unroll
      for (int i = 0; i < KU; ++i) x[i] = attn_mma(q, k[i][s], x[i]);
    }
    // (whole: all columns of the tile see all keys of the wave; the last tile's columns past the end have a weight of zero)
    const bool whole = 32 * t + 32 <= cols && 32 * (unit0 + KU) - 1 <= c.len + c.first + low_row;
    step(low_row, low_g);
    if (whole) {
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4) {
        const f32x4_t r = *reinterpret_cast<const f32x4_t*>(&ref[buf][8 * g4 + 4 * half]), w = *reinterpret_cast<const f32x4_t*>(&inv[buf][8 * g4 + 4 * half]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int i = 0; i < KU; ++i) of_tile[i] = fmaf(__builtin_amdgcn_exp2f(fmaf(x[i][4 * g4 + e], a.scale, -r[e])), w[e], of_tile[i]);
      }
    } else {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int col = 8 * (v >> 2) + 4 * half + (v & 3), last = sees[buf][col];
        const float r = ref[buf][col], w = inv[buf][col];
#pragma unroll
        for (int i = 0; i < KU; ++i) {
          const float y = fmaf(__builtin_amdgcn_exp2f(fmaf(x[i][v], a.scale, -r)), w, of_tile[i]);
          of_tile[i] = 32 * (unit0 + i) + (lane & 31) <= last ? y : of_tile[i];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < KU; ++i) sum[i] += of_tile[i];
    if (t + 1 < t1) put(buf ^ 1);               // (nobody reads that one: all have passed the barrier behind its tile)
    __syncthreads();
  }
  const int64_t head = (int64_t)seq * kv.hkv + kvh;
#pragma unroll
  for (int i = 0; i < KU; ++i) {
    const float all = there[i] ? attn_sum_of_halves(sum[i]) : 0.f;
    const int slot = 32 * (unit0 + i) + (lane & 31);
    if (half == 0 && slot < c.total) {
      const int64_t at = head * a.slots + slot;
      if (p.parts > 1) a.scratch[p.stats_floats + (part * (int64_t)kv.batch * kv.hkv + head) * p.tokens + slot] = all;
      else a.mass[at] = (a.before && slot < c.len ? a.before[at] : 0.f) + all;
    }
  }
}

__global__ __launch_bounds__(THREADS) void k_weigh_parts(PagedDev kv, ChunkDev ch, WeighArgs a, WeighPlan p) {
  const int kvh = blockIdx.y, seq = blockIdx.z, slot = blockIdx.x * THREADS + threadIdx.x;
  const WeighSeq c = weigh_seq(kv, ch, seq, a.last, a.slots);
  if (!c.ok || c.rows == 0 || slot >= c.total) return;
  const int64_t head = (int64_t)seq * kv.hkv + kvh, at = head * a.slots + slot;
  const float* s = a.scratch + p.stats_floats + head * p.tokens + slot;
  float sum = 0.f;
  for (int i = 0; i < p.parts; ++i) sum += s[i * (int64_t)kv.batch * kv.hkv * p.tokens];
  a.mass[at] = (a.before && slot < c.len ? a.before[at] : 0.f) + sum;
}

template <typename T, int HD>
hipError_t launch(hipStream_t st, const PagedDev& kv, const ChunkDev& ch, const WeighArgs& a, const WeighPlan& p) {
  const dim3 tokens((unsigned)((p.tokens + THREADS - 1) / THREADS), kv.hkv, kv.batch), wg(THREADS);
  if (p.width) {
    const dim3 grid(p.shares, kv.hkv, kv.batch);
    if (p.width <= 8) hipLaunchKernelGGL((k_weigh_scores<T, HD, 1>), grid, wg, 0, st, kv, ch, a, p);
    else if (p.width <= 16) hipLaunchKernelGGL((k_weigh_scores<T, HD, 2>), grid, wg, 0, st, kv, ch, a, p);
    else hipLaunchKernelGGL((k_weigh_scores<T, HD, 4>), grid, wg, 0, st, kv, ch, a, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // Four tokens a thread where there are many, as the shares are joined by every workgroup.  Whole calls of a row a sequence, one / four a thread: 2^14 tokens of all
    // heads 8.8 / 10.4 us, 2^18 21.5 / 22.6, 2^19 33.2 / 33.1, 2^20 62.6 / 59.4 (one sequence of 131072: 71.7 / 64.0), 2^22 252 / 239.
    if (p.tokens * kv.hkv * kv.batch >= (1 << 20)) hipLaunchKernelGGL(k_weigh_sum<4>, dim3((tokens.x + 3) / 4, tokens.y, tokens.z), wg, 0, st, kv, ch, a, p);
    else hipLaunchKernelGGL(k_weigh_sum<1>, tokens, wg, 0, st, kv, ch, a, p);
    return hipGetLastError();
  }
  const int G = a.hq / kv.hkv, tiles = (int)(((int64_t)p.most_rows * G + 31) / 32);
  constexpr int CT = stat_tiles(sizeof(T) == 2);
  hipLaunchKernelGGL((k_weigh_stats<T, HD, CT>), dim3((tiles + WAVES * CT - 1) / (WAVES * CT) * p.shares, kv.hkv, kv.batch), wg, 0, st, kv, ch, a, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (p.shares > 1 && !p.join_here) {
    hipLaunchKernelGGL(k_weigh_join, dim3((32 * tiles + THREADS - 1) / THREADS, kv.hkv, kv.batch), wg, 0, st, kv, ch, a, p);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  constexpr int KU = sizeof(T) == 2 ? 2 : 1, KEYS = WAVES * KU * 32;
  hipLaunchKernelGGL((k_weigh_add<T, HD, KU>), dim3((unsigned)((p.tokens + KEYS - 1) / KEYS) * p.parts, kv.hkv, kv.batch), wg, 0, st, kv, ch, a, p);
  e = hipGetLastError();
  if (e != hipSuccess || p.parts == 1) return e;
  hipLaunchKernelGGL(k_weigh_parts, tokens, wg, 0, st, kv, ch, a, p);
  return hipGetLastError();
}

}  // namespace

WeighPlan weigh_plan(int dtype, int batch, int hq, int hkv, int total_rows, int max_rows, int last, int len_bound) {
  WeighPlan p{};
  const int G = hq / hkv, rows = std::min(std::min(max_rows, total_rows), last > 0 ? last : max_rows);
  const int64_t cols = (int64_t)rows * G, heads = (int64_t)batch * hkv;
  p.most_rows = rows;
  p.tokens = ((int64_t)len_bound + std::min(max_rows, total_rows) + 31) / 32 * 32;
  const int units = (int)(p.tokens / 32);
  if (cols <= 32) {
    p.width = cols <= 4 ? 4 : cols <= 8 ? 8 : cols <= 16 ? 16 : 32;
    // Shares of a sequence and kv head: small ones, as sequences differ in length (32 of 1000 to 16384, 256 heads together: 152 us with 2048 in all, 145 with 4096,
    // 127 with 8192, 123 with 16384, 132 with 32768), of a unit a wave at least.
    const int64_t most = std::max<int64_t>(1, 16384 / heads);
    p.share_units = (int)std::max<int64_t>(4, (units + most - 1) / most);
    p.shares = (units + p.share_units - 1) / p.share_units;
    p.stats_floats = 2 * heads * p.shares * p.width;
    p.scratch_floats = p.stats_floats + heads * p.tokens * p.width;
    return p;
  }
  p.packed = (int64_t)total_rows < (int64_t)batch * rows;
  p.columns = (p.packed ? (int64_t)total_rows : (int64_t)batch * rows) * hq;
  const int of_group = WAVES * stat_tiles(dtype == ESP_BF16);
  const int64_t groups = ((cols + 31) / 32 + of_group - 1) / of_group * heads;
  // About 2048 workgroups for the statistics, of 16 units at least where there are many units; four shares at most, of two units, where there are few units or
  // many columns.  Few: 64 rows of 32 heads over 16 to 62 units take the same time either way, 512 rows by themselves (16 units) 28.3 us instead of 33.0; over
  // 96 and 126 units the 64 rows take 40.9 and 44.8 instead of 32.2 and 32.0.  The sums: up to 2048 also.  (A prompt of 4096: 229 to 231 us; with 1024 or 4096 of the first
  // 234 and 239, of the second 234 and 228.  Four of 1500 rows: 155; 152 and 168, 154 and 147.)
  const int64_t most = std::max<int64_t>(1, 2048 / groups);
  if (most <= 4 || units <= 64) p.share_units = (int)std::max<int64_t>(2, (units + std::min<int64_t>(4, most) - 1) / std::min<int64_t>(4, most));
  else p.share_units = (int)std::max<int64_t>(16, (units + most - 1) / most);
  p.shares = (units + p.share_units - 1) / p.share_units;
  // Few columns: the sums join the shares, a tile of columns a time and a share after the other, which costs less than a launch does (448 tokens, bf16 of 128 and four
  // shares, joined there / in a launch: 36 columns 14.3 / 15.7 us, 96 16.5 / 16.6, 128 18.3 / 17.5, 256 28.0 / 23.5; fp32 of 64 16.4 / 17.7, 20.6 / 20.5, 23.1 / 22.1,
  // 33.6 / 29.9; at 960 and 1900 tokens and eight sequences the same turn at 96).
  p.join_here = p.shares > 1 && p.shares <= 4 && cols <= 96;
  p.stats_floats = 2 * p.columns * p.shares;
  const int keys = WAVES * 32 * (dtype == ESP_BF16 ? 2 : 1);
  const int64_t key_groups = (p.tokens + keys - 1) / keys * heads;
  p.parts = (int)std::max<int64_t>(1, std::min<int64_t>((cols + 255) / 256, 2048 / key_groups));
  p.scratch_floats = p.stats_floats + (p.parts > 1 ? p.parts * heads * p.tokens : 0);
  return p;
}

int64_t weigh_workgroups(const WeighPlan& p, int batch, int hkv, int G) {
  const int64_t tiles = ((int64_t)p.most_rows * G + 31) / 32, heads = (int64_t)batch * hkv;
  return std::max<int64_t>({p.tokens / 128 + 1, (tiles / WAVES + 1) * p.shares, (p.tokens / 128 + 1) * std::max(1, p.parts)}) * heads;
}

hipError_t launch_paged_weigh(hipStream_t st, int dtype, int hd, const PagedDev& kv, const ChunkDev& ch, const WeighArgs& a, const WeighPlan& p) {
  if (dtype == ESP_BF16) return hd == 128 ? launch<bf16_t, 128>(st, kv, ch, a, p) : launch<bf16_t, 64>(st, kv, ch, a, p);
  return hd == 128 ? launch<float, 128>(st, kv, ch, a, p) : launch<float, 64>(st, kv, ch, a, p);
}
