// Grouped-query attention of a chunk of new rows over a paged KV cache, causal or under ancestor bitsets.
//
// The G = n_q / n_kv query heads of a kv head times a sequence's rows are its query columns.  A workgroup has a group of columns of one
// (sequence, kv head) and one split of the key range; where there are several splits they leave (m, l, O) in memory, and k_paged_merge
// adds them up in split order, so results do not depend on scheduling.
#include <algorithm>

#include "esp_attn_unit.h"
#include "esp_paged.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f;

struct Partials {               // [split][row][head][HD], then (m in powers of two, l) [split][row][head][2]
  float* o;
  float* ml;
};
__device__ __forceinline__ Partials partials_of(float* base, int nsplit, int total, int hq, int hd) {
  return {base, base + (size_t)nsplit * total * hq * hd};
}

// which workgroup this is.  Groups (split, sequence, kv head) are dealt to the XCDs round-robin, and the workgroups of a group, which read
// the same keys, come out on the same one; the last columns, which see the most keys, come first.
struct PagedWork { int seq, kvh, split, qt; bool any; };
__device__ __forceinline__ PagedWork work_of(int block, int batch, int hkv, int nsplit, int q_tiles) {
  const int groups = batch * hkv * nsplit, step = q_tiles > 1 && groups >= 8 ? (groups + 7) & ~7 : groups;
  const int g = block % step;
  return {g / hkv % batch, g % hkv, g / hkv / batch, q_tiles - 1 - block / step, g < groups};
}
inline int64_t work_grid(int batch, int hkv, int nsplit, int q_tiles) {
  const int64_t groups = (int64_t)batch * hkv * nsplit, step = q_tiles > 1 && groups >= 8 ? (groups + 7) & ~7ll : groups;
  return step * q_tiles;
}

template <typename T>
__device__ __forceinline__ typename AttnFrag<T>::type load_frag(const T* p) {
  return *reinterpret_cast<const typename AttnFrag<T>::type*>(p);
}
// eight features of a query, which may lie at any element
template <typename T>
__device__ __forceinline__ typename AttnFrag<T>::type load_query(const T* p, bool vec) {
  if (vec) return load_frag(p);
  typename AttnFrag<T>::type f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = p[e];
  return f;
}
__device__ __forceinline__ void store4(float* p, f32x4_t v, bool vec) {
  if (vec) { *reinterpret_cast<f32x4_t*>(p) = v; return; }
#pragma unroll
  for (int e = 0; e < 4; ++e) p[e] = v[e];
}
__device__ __forceinline__ void store4(bf16_t* p, f32x4_t v, bool vec) {
  const bf16x4_t o = {(bf16_t)v[0], (bf16_t)v[1], (bf16_t)v[2], (bf16_t)v[3]};
  if (vec) { *reinterpret_cast<bf16x4_t*>(p) = o; return; }
#pragma unroll
  for (int e = 0; e < 4; ++e) p[e] = o[e];
}

// --------------------------------------------------------------------------------------------------
// k_paged_stream: up to 32 query columns a workgroup, four waves that share them and take the units of the split's keys in
// turn.  Nothing is used twice, so K and V go from memory to registers and straight into the matrix instructions; a
// wave asks for its next unit's K as soon as its scores are done and for the next V behind the product with this one.
constexpr int STREAM_WAVES = 4;
constexpr int STREAM_MOST = 64 * STREAM_WAVES * 32;     // keys of a split: a wave keeps its units' places in one register, one a lane

template <typename T, int HD>
__global__ __launch_bounds__(64 * STREAM_WAVES, sizeof(T) * HD <= 256 ? 2 : 1) void k_paged_stream(PagedDev kv, ChunkDev ch, PagedAttnArgs a,
                                                                                               int nsplit, int chunk, int q_tiles, bool vec_q,
                                                                                               bool vec_out) {
  constexpr int NS = HD / 16, DB = HD / 32, W = STREAM_WAVES, BLOCK = 32 * HD;
  typedef typename AttnFrag<T>::type frag_t;
  __shared__ __align__(16) float xo[W][32][HD];
  __shared__ float xm[W][32], xl[W][32];
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, lg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const PagedWork w = work_of(blockIdx.x, kv.batch, kv.hkv, nsplit, q_tiles);
  if (!w.any) return;
  const int G = a.hq / kv.hkv, blocks = kv.page_size >> 5;
  const int key_lo = w.split * chunk;
  // this wave's units: unit i at key_lo + 32 (wave + W i), its place looked up by lane i
  int place;
  bool bad;
  {
    const int n = (key_lo >> 5) + wave + W * lane, pg = min(n / blocks, kv.stride - 1);
    const int page = kv.table[(size_t)w.seq * kv.stride + pg];
    bad = (unsigned)page >= (unsigned)kv.n_pages;
    place = bad ? -1 : (page * kv.hkv + w.kvh) * blocks + n % blocks;
  }
  const ChunkSeq s = chunk_seq(kv, ch, w.seq);
  if (!s.ok) {
    if (w.kvh == 0 && w.split == 0 && w.qt == 0 && tid == 0) set_status(kv.status, chunk_fault(kv, ch, w.seq));
    return;
  }
  const int ncols = s.rows * G, col0 = w.qt * 32;
  if (col0 >= ncols) return;
  const int r_lo = col0 / G, r_hi = min(s.rows - 1, (col0 + 31) / G), total = s.len + s.rows;
  const int key_end = a.anc ? total : s.len + r_hi + 1;
  const int key_hi = min(key_lo + chunk, key_end);
  if (key_lo >= key_hi) return;
  const int units = max(0, (((key_hi - key_lo + 31) >> 5) - wave + W - 1) / W);
  if (bad && lane < units) set_status(kv.status, ESP_DEV_BAD_PAGE);

  const int col = col0 + lr;
  const bool live = col < ncols;
  const int r = live ? col / G : 0, h = w.kvh * G + (live ? col % G : 0);
  const int64_t row = s.row0 + r;
  frag_t qf[NS];
  {
    const T* qp = (const T*)a.q + row * a.q_stride + h * HD + 8 * lg;
#pragma unroll
    for (int i = 0; i < NS; ++i) qf[i] = load_query(qp + 16 * i, vec_q);
  }
  const uint64_t* anc = a.anc ? a.anc + row * a.anc_words : nullptr;
  f32x16_t o[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[i][v] = 0.f;
  float m = ATTN_UNSEEN, l = 0.f;

  frag_t kf[NS], vf[2 * DB];
  auto base = [&](const void* pool, int i) {
    const int p = __builtin_amdgcn_readlane(place, i);
    return (const T*)pool + (size_t)max(p, 0) * BLOCK + lane * 8;
  };
  if (units > 0) {
    const T *kb = base(kv.k, 0), *vb = base(kv.v, 0);
#pragma unroll
    for (int i = 0; i < NS; ++i) kf[i] = load_frag(kb + i * 512);
#pragma unroll
    for (int i = 0; i < 2 * DB; ++i) vf[i] = load_frag(vb + i * 512);
  }
  for (int i = 0; i < units; ++i) {
    const int key0 = key_lo + 32 * (wave + W * i), c_lo = key0 - s.len, left = total - key0;
    const bool there = __builtin_amdgcn_readlane(place, i) >= 0;
    const int next = min(i + 1, units - 1);
    f32x16_t sc;
#pragma unroll
    for (int v = 0; v < 16; ++v) sc[v] = 0.f;
#pragma unroll
    for (int j = 0; j < NS; ++j) sc = attn_mma(kf[j], qf[j], sc);
    __builtin_amdgcn_sched_barrier(0);
    {
      const T* kb = base(kv.k, next);
#pragma unroll
      for (int j = 0; j < NS; ++j) kf[j] = load_frag(kb + j * 512);
    }
    __builtin_amdgcn_sched_barrier(0);
    const bool masked = !there || c_lo + 32 > (a.anc ? 0 : r_lo + 1);
    unsigned window = ~0u;
    if (masked) window = there ? attn_window(anc, a.anc_words, r, c_lo, s.rows) : 0u;
    frag_t pf[2];
    attn_softmax<T, DB>(sc, masked, window >> (4 * lg), a.scale, o, m, l, pf);
    if (masked) {
      bool odd = false;
#pragma unroll
      for (int j = 0; j < 2 * DB; ++j) {
        if (left < 32) vf[j] = attn_zero_tail(vf[j], j & 1, lane, left);
        odd |= attn_not_finite(vf[j]);
      }
      if (__builtin_amdgcn_ballot_w64(odd) != 0ull) attn_keep_hidden<T, DB>(vf, window >> (4 * lg), o);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] = attn_mma(vf[2 * db + u], pf[u], o[db]);
    __builtin_amdgcn_sched_barrier(0);
    {
      const T* vb = base(kv.v, next);
#pragma unroll
      for (int j = 0; j < 2 * DB; ++j) vf[j] = load_frag(vb + j * 512);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  l += __shfl_xor(l, 32, 64);
  // the waves' parts meet in LDS, a column's features side by side in pieces of four, which are shuffled by the column's number so
  // that the columns of a store fall on different banks
  constexpr int PIECES = HD / 4;
  if (live) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int v = 0; v < 16; v += 4) {
        const int piece = db * 8 + 2 * (v >> 2) + lg;
        *reinterpret_cast<f32x4_t*>(&xo[wave][lr][4 * (piece ^ (lr & (PIECES - 1)))]) = f32x4_t{o[db][v], o[db][v + 1], o[db][v + 2], o[db][v + 3]};
      }
    if (lg == 0) { xm[wave][lr] = m; xl[wave][lr] = l; }
  }
  __syncthreads();
  const int n_live = min(32, ncols - col0);
  for (int t = tid; t < n_live * PIECES; t += 64 * W) {
    const int c = t / PIECES, piece = t % PIECES;
    float top = xm[0][c];
#pragma unroll
    for (int i = 1; i < W; ++i) top = fmaxf(top, xm[i][c]);
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    float lt = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float f = attn_weight(xm[i][c], top, a.scale);
      lt += xl[i][c] * f;
      acc += *reinterpret_cast<const f32x4_t*>(&xo[i][c][4 * (piece ^ (c & (PIECES - 1)))]) * f;
    }
    const int cc = col0 + c;
    const int64_t rr = s.row0 + cc / G, item = rr * a.hq + w.kvh * G + cc % G;
    if (nsplit == 1) {
      store4((T*)a.out + item * HD + 4 * piece, acc * (lt > 0.f ? 1.f / lt : 0.f), vec_out);
    } else {
      const Partials p = partials_of(a.partials, nsplit, ch.total, a.hq, HD);
      const int64_t at = (int64_t)w.split * ch.total * a.hq + item;
      *reinterpret_cast<f32x4_t*>(p.o + at * HD + 4 * piece) = acc;
      if (piece == 0) { p.ml[2 * at] = top * a.scale; p.ml[2 * at + 1] = lt; }
    }
  }
}

// --------------------------------------------------------------------------------------------------
// The splits of a (row, head), in split order: HD / 4 threads, four features each.
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_paged_merge(PagedDev kv, ChunkDev ch, PagedAttnArgs a, int nsplit, int chunk, bool vec_out) {
  constexpr int PER = HD / 4;
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t item = (int64_t)blockIdx.x * (256 / PER) + tid / PER;
  const int row = (int)min(item / a.hq, (int64_t)ch.total - 1), d = 4 * (tid % PER);
  // the sequence: the last that begins at or before the row; a wave's items are of two rows at most where there are two heads or more,
  // so every thread looks for itself
  int seq = -1;
  {
    int lo = 0, hi = kv.batch;                      // row0 ascends: the first sequence that begins behind the row
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (ch.row0[mid] <= row) lo = mid + 1; else hi = mid;
    }
    seq = lo - 1;
  }
  (void)lane;
  if (item >= (int64_t)ch.total * a.hq || seq < 0) return;
  const ChunkSeq s = chunk_seq(kv, ch, seq);
  if (!s.ok || row < s.row0 || row >= s.row0 + s.rows) return;
  const int end = a.anc ? s.len + s.rows : s.len + (row - s.row0) + 1;
  const int n = min(nsplit, (end + chunk - 1) / chunk);
  const Partials p = partials_of(a.partials, nsplit, ch.total, a.hq, HD);
  const int64_t step = (int64_t)ch.total * a.hq;
  float top = ATTN_UNSEEN;
  for (int i = 0; i < n; ++i) top = fmaxf(top, p.ml[2 * (item + i * step)]);
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  float lt = 0.f;
  for (int i = 0; i < n; ++i) {
    const int64_t at = item + i * step;
    const float m = p.ml[2 * at], l = p.ml[2 * at + 1];
    const float f = l > 0.f ? __builtin_amdgcn_exp2f(m - top) : 0.f;
    lt += l * f;
    acc += *reinterpret_cast<const f32x4_t*>(p.o + at * HD + d) * f;
  }
  store4((T*)a.out + item * HD + d, acc * (lt > 0.f ? 1.f / lt : 0.f), vec_out);
}

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

template <typename T, int HD>
hipError_t launch(hipStream_t st, const PagedDev& kv, const ChunkDev& ch, const PagedAttnArgs& a, const PagedAttnPlan& p) {
  const bool vec_q = (uintptr_t)a.q % 16 == 0 && a.q_stride * (int64_t)sizeof(T) % 16 == 0, vec_out = (uintptr_t)a.out % 16 == 0;
  const int64_t grid = work_grid(kv.batch, kv.hkv, p.nsplit, p.q_tiles);
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  hipLaunchKernelGGL((k_paged_stream<T, HD>), dim3((unsigned)grid), dim3(64 * STREAM_WAVES), 0, st, kv, ch, a, p.nsplit, p.chunk, p.q_tiles,
                     vec_q, vec_out);
  if (p.nsplit > 1) {
    const int64_t items = (int64_t)ch.total * a.hq;
    hipLaunchKernelGGL((k_paged_merge<T, HD>), dim3((unsigned)ceil_div(items, 256 / (HD / 4))), dim3(256), 0, st, kv, ch, a, p.nsplit, p.chunk, vec_out);
  }
  return hipGetLastError();
}

}  // namespace

// Splits where the columns alone do not fill the CUs, of 256 keys or more.
PagedAttnPlan paged_attn_plan(int dtype, int hd, int batch, int hq, int hkv, int total_rows, int max_rows, int len_bound) {
  PagedAttnPlan p;
  const int G = hq / hkv;
  p.q_tiles = std::max(1, ceil_div((int64_t)max_rows * G, 32));
  const int64_t keys = (int64_t)len_bound + max_rows;
  const int64_t groups = (int64_t)hkv * std::min<int64_t>((int64_t)batch * p.q_tiles, ((int64_t)total_rows * G + 31) / 32 + batch);
  int64_t n = std::max<int64_t>(1, 1024 / std::max<int64_t>(groups, 1));
  n = std::min<int64_t>(n, std::max<int64_t>(1, keys / 256));
  n = std::max<int64_t>(n, (keys + STREAM_MOST - 1) / STREAM_MOST);
  const int unit = 32 * STREAM_WAVES;
  p.chunk = (int)std::min<int64_t>((keys + n * unit - 1) / (n * unit) * unit, STREAM_MOST);
  p.nsplit = std::max(1, ceil_div(keys, p.chunk));
  return p;
}

hipError_t launch_paged_attn(hipStream_t st, int dtype, int hd, const PagedDev& kv, const ChunkDev& ch, const PagedAttnArgs& a,
                             const PagedAttnPlan& p) {
  PagedAttnArgs x = a;
  x.scale = a.scale * LOG2E;
  if (dtype == ESP_F32) return hd == 64 ? launch<float, 64>(st, kv, ch, x, p) : launch<float, 128>(st, kv, ch, x, p);
  return hd == 64 ? launch<bf16_t, 64>(st, kv, ch, x, p) : launch<bf16_t, 128>(st, kv, ch, x, p);
}
