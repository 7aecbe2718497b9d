// Grouped-query attention of a chunk of new rows over a paged KV cache, causal or under ancestor bitsets.
//
// The G = n_q / n_kv query heads of a kv head times a sequence's rows are its query columns, in tiles of 32.  An item is a group of up to
// CAP column tiles of one (sequence, kv head) over all keys they see, which are walked in key tiles of TK.  Either a workgroup has an item
// (the launch has enough of them to even out, or they are too short to be cut), or the items form a line of work that is cut into equal
// shares, one a workgroup: the pieces of an item that a cut went through leave (m, l, O) in memory, and k_paged_merge adds them up in the
// line's order, so results do not depend on scheduling.  Only the device knows lengths and rows; every workgroup looks its share up.
//
// k_paged_stream (up to 32 columns an item, four waves that share them, TK 128) is for decoding, bound by the memory that K and V come
// from; k_paged_tile (up to 256 columns, eight waves around a ring of key tiles in LDS, TK 64) for chunks and trees, bound by the matrix cores.
#include <algorithm>
#include <atomic>

#include "esp_attn_unit.h"
#include "esp_paged.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int STREAM_WAVES = 4, STREAM_TK = 32 * STREAM_WAVES;
constexpr int TILE_WAVES = 8, TILE_TK = 64, TILE_CAP = 8;

// ---- the line of work --------------------------------------------------------------------------------------------
struct Item { int seq, kvh, qt; };
struct Cut { Item item; int tile; };            // before key tile `tile` of the item

// what a sequence's items are: n of them for each kv head, of `per` column tiles (the last may have fewer)
struct Items { int n, per; };
__host__ __device__ __forceinline__ Items items_of(int rows, int G, int cap) {
  const int ct = (int)(((int64_t)rows * G + 31) / 32), n = (ct + cap - 1) / cap;
  return {n, n ? (ct + n - 1) / n : 0};
}
// keys that item qt sees
__device__ __forceinline__ int keys_of(const ChunkSeq& s, int G, int per, int qt, bool causal) {
  const int rows = causal ? min(s.rows, (int)((((int64_t)qt + 1) * per * 32 + G - 1) / G)) : s.rows;
  return s.len + rows;
}
// Weights along the line, in keys x G x time of a key tile: an item counts START keys for its beginning and end and the keys that it
// sees.  Cuts need not be exact, only the same for everybody.
struct Weights {
  int64_t first, slope;                         // item k weighs first + slope (k + 1)
  int64_t tile, start;
  __device__ __forceinline__ int64_t upto(int64_t k) const { return first * k + slope * (k * (k + 1) / 2); }
};
template <int CAP>
__device__ __forceinline__ Weights weights_of(const ChunkSeq& s, int G, int per, bool causal) {
  // time of a key tile with that many column tiles (k_paged_tile): 0.7 us with one to 1.5 us with eight; START is 4 us of the latter
  constexpr int TK = CAP == 1 ? STREAM_TK : TILE_TK, START = CAP == 1 ? 64 : 160;
  const int64_t t = CAP == 1 ? 1 : 5 + per;
  return {t * G * ((int64_t)START * (CAP == 1 ? 1 : 13) / t + s.len + (causal ? 0 : s.rows)), causal ? t * per * 32 : 0, t * G * TK,
          (int64_t)G * START * (CAP == 1 ? 1 : 13)};
}

// exclusive sum over the workgroup's threads; total: of all.  sums: LDS, NT / 64 of them
template <int NT>
__device__ __forceinline__ int64_t sum_before(int64_t x, int64_t* sums, int64_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t upto = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(upto, o, 64);
    if (lane >= o) upto += y;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int64_t before = upto - x;
  total = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    if (w < wave) before += sums[w];
    total += sums[w];
  }
  __syncthreads();
  return before;
}

// Where share w of `shares` begins and ends.  Order of the line: kv heads, sequences, column groups from the last.  The device may use fewer
// shares than were launched: none with less than `least` of weight in key tiles.  False: no such share.
template <int NT, int CAP>
__device__ bool share_of(const PagedDev& kv, const ChunkDev& ch, int hq, bool causal, int w, int shares, int least, Cut& lo, Cut& hi) {
  __shared__ int64_t sums[NT / 64];
  __shared__ Cut cuts[2];
  const int tid = threadIdx.x, G = hq / kv.hkv;
  constexpr int TK = CAP == 1 ? STREAM_TK : TILE_TK;
  auto weight = [&](int b, ChunkSeq& s, Items& it, Weights& wt) -> int64_t {
    if (b >= kv.batch) return 0;
    s = chunk_seq(kv, ch, b);
    if (!s.ok) return 0;
    it = items_of(s.rows, G, CAP);
    wt = weights_of<CAP>(s, G, it.per, causal);
    return wt.upto(it.n);
  };
  ChunkSeq s;
  Items it;
  Weights wt;
  int64_t per_head = 0, mine = 0, before = 0;
  for (int b0 = 0; b0 < kv.batch; b0 += NT) {
    int64_t total;
    mine = weight(b0 + tid, s, it, wt);
    before = sum_before<NT>(mine, sums, total);
    per_head += total;
  }
  const int64_t all = per_head * kv.hkv;
  const int64_t tile_weight = (int64_t)(CAP == 1 ? 1 : 13) * G * TK;
  const int n = (int)max((int64_t)1, min((int64_t)shares, all / (tile_weight * least)));
  if (w >= n || all == 0) return false;
  // position x * all / n on the line, without overflow
  auto at = [&](int x) { return all / n * x + all % n * x / n; };
  const int64_t want[2] = {at(w), at(w + 1)};
  if (tid < 2) cuts[tid] = Cut{{kv.batch, kv.hkv, 0}, 0};           // the line's end
  __syncthreads();
  int64_t base = 0;
  for (int b0 = 0; b0 < kv.batch; b0 += NT) {
    if (kv.batch > NT) {
      int64_t total;
      mine = weight(b0 + tid, s, it, wt);
      before = base + sum_before<NT>(mine, sums, total);
      base += total;
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int64_t head = want[e] / per_head, off = want[e] - head * per_head - before;
      if (head >= kv.hkv || off < 0 || off >= mine) continue;
      // item j of the line is column group n - 1 - j, so what is in front is all behind group k: weight of groups 0 .. k is more than rest
      const int64_t rest = mine - off;                              // weight from here to the sequence's end, > 0
      int64_t k;                                                    // the group with upto(k) < rest <= upto(k + 1)
      if (wt.slope > 0) {
        const double a = 0.5 * (double)wt.slope, c = (double)wt.first + a;
        k = (int64_t)((sqrt(c * c + 4.0 * a * (double)rest) - c) / (2.0 * a));
      } else {
        k = rest / wt.first;
      }
      k = max((int64_t)0, min(k, (int64_t)it.n - 1));
      while (k > 0 && wt.upto(k) >= rest) --k;
      while (k + 1 < it.n && wt.upto(k + 1) < rest) ++k;
      const int64_t into = wt.upto(k + 1) - rest - wt.start;        // weight of this item in front of the cut, but for its start
      const int tiles = (keys_of(s, G, it.per, (int)k, causal) + TK - 1) / TK;
      const int tile = into <= 0 ? 0 : (int)min((into + wt.tile - 1) / wt.tile, (int64_t)tiles);
      cuts[e] = Cut{{b0 + tid, (int)head, (int)k}, tile};
    }
  }
  __syncthreads();
  auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  auto take = [&](const Cut& c) { return Cut{{uniform(c.item.seq), uniform(c.item.kvh), uniform(c.item.qt)}, uniform(c.tile)}; };
  lo = take(cuts[0]);
  hi = take(cuts[1]);
  return true;
}
// a sequence's scalars, the same for the whole wave
__device__ __forceinline__ ChunkSeq uniform_seq(const PagedDev& kv, const ChunkDev& ch, int seq) {
  const ChunkSeq s = chunk_seq(kv, ch, seq);
  return {__builtin_amdgcn_readfirstlane(s.row0), __builtin_amdgcn_readfirstlane(s.rows), __builtin_amdgcn_readfirstlane(s.len),
          (bool)__builtin_amdgcn_readfirstlane((int)s.ok)};
}
__device__ __forceinline__ bool same(const Item& a, const Item& b) { return a.seq == b.seq && a.kvh == b.kvh && a.qt == b.qt; }

// Partials: slots of CAP x 32 columns, [slot][column][HD] then (m in powers of two, l) [slot][column][2].  Share w has slots 2 w, for the piece
// that it begins with if that is not an item's first, and 2 w + 1, for the piece that it ends with if that is an item's first and not its last.
// What a share leaves for the merge: the item that begins in slot 2 w + 1 (seq -1: none), and of slot 2 w whether there is anything in it
// (HAS) and whether the item ends in this share, or there is none (ENDS).
struct ShareNote { Item begun; int first; };
enum { HAS = 1, ENDS = 2 };
struct Partials {
  ShareNote* notes;
  float *o, *ml;
};
__host__ __device__ inline size_t notes_floats(int shares) { return ((size_t)shares * sizeof(ShareNote) / 4 + 3) / 4 * 4; }
__device__ __forceinline__ Partials partials_of(float* base, int shares, int cols, int hd) {
  float* o = base + notes_floats(shares);
  return {(ShareNote*)base, o, o + (size_t)2 * shares * cols * hd};
}

// Walks the pieces of a workgroup: run(item, sequence, its items, first and last key tile, slot of the partial or -1 for a whole item).
template <int NT, int CAP, typename RUN>
__device__ __forceinline__ void walk(const PagedDev& kv, const ChunkDev& ch, const PagedAttnArgs& a, int shares, int least, int q_tiles, RUN run) {
  constexpr int TK = CAP == 1 ? STREAM_TK : TILE_TK;
  const bool causal = a.anc == nullptr;
  const int G = a.hq / kv.hkv;
  int w = 0;
  Cut lo, hi;
  if (shares == 0) {
    // an item each.  Groups (sequence, kv head) are dealt to the XCDs round-robin, and a group's items, which read the same keys, come out on the
    // same one; the last columns, which see the most keys, come first.
    const int groups = kv.batch * kv.hkv, step = q_tiles > 1 && groups >= 8 ? (groups + 7) & ~7 : groups;
    const int g = blockIdx.x % step;
    if (g >= groups) return;
    lo = Cut{{g / kv.hkv, g % kv.hkv, q_tiles - 1 - (int)(blockIdx.x / step)}, 0};
    hi = Cut{lo.item, INT32_MAX};
    if (lo.item.kvh == 0 && lo.item.qt == 0 && threadIdx.x == 0 && !chunk_seq(kv, ch, lo.item.seq).ok)
      set_status(kv.status, chunk_fault(kv, ch, lo.item.seq));
  } else {
    if (blockIdx.x == 0)
      for (int b = threadIdx.x; b < kv.batch; b += NT)
        if (!chunk_seq(kv, ch, b).ok) set_status(kv.status, chunk_fault(kv, ch, b));
    // shares next to each other on the line, which read the same keys, on one XCD
    const int per_xcd = (shares + 7) >> 3;
    w = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if (w >= shares) return;
    if (!share_of<NT, CAP>(kv, ch, a.hq, causal, w, shares, least, lo, hi)) lo = Cut{{0, kv.hkv, 0}, 0};
  }
  ShareNote note{{-1, 0, 0}, ENDS};
  Item item = lo.item;
  int t0 = lo.tile;
  while (item.kvh < kv.hkv) {
    const ChunkSeq s = uniform_seq(kv, ch, item.seq);
    const Items it = items_of(s.rows, G, CAP);
    if (s.ok && item.qt < 0) item.qt = it.n - 1;
    const bool last = same(item, hi.item);
    if (s.ok && item.qt >= 0 && item.qt < it.n) {
      const int tiles = (keys_of(s, G, it.per, item.qt, causal) + TK - 1) / TK, t1 = last ? min(hi.tile, tiles) : tiles;
      const bool ends = t1 >= tiles;
      if (t0 > 0) note.first = (t1 > t0 ? HAS : 0) | (ends ? ENDS : 0);
      else if (!ends && t1 > 0) note.begun = item;
      if (t1 > t0) run(item, s, it, t0, t1, t0 > 0 ? 2 * w : ends ? -1 : 2 * w + 1);
    }
    if (last) break;
    t0 = 0;
    if (s.ok && item.qt > 0) {
      --item.qt;
    } else {                                      // the next sequence's last group, or the next kv head's first sequence
      item.qt = -1;
      if (++item.seq == kv.batch) { item.seq = 0; ++item.kvh; }
    }
  }
  if (shares != 0 && threadIdx.x == 0) ((ShareNote*)a.partials)[w] = note;
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
// A wave's O^T as columns in LDS, [32][HD]: features in pieces of four, which are shuffled by the column's number so that the columns
// of an access fall on different banks.
template <int HD>
__device__ __forceinline__ float* column_piece(float* xo, int col, int piece) { return xo + col * HD + 4 * (piece ^ (col & (HD / 4 - 1))); }
template <int HD>
__device__ __forceinline__ void put_columns(float* xo, const f32x16_t (&o)[HD / 32], int lane) {
#pragma unroll
  for (int db = 0; db < HD / 32; ++db)
#pragma unroll
    for (int v = 0; v < 16; v += 4)
      *reinterpret_cast<f32x4_t*>(column_piece<HD>(xo, lane & 31, db * 8 + 2 * (v >> 2) + (lane >> 5))) = f32x4_t{o[db][v], o[db][v + 1], o[db][v + 2], o[db][v + 3]};
}

// --------------------------------------------------------------------------------------------------
// k_paged_stream: nothing of K and V is used twice, so they go from memory to registers and straight into the matrix
// instructions.  The waves take the 32-key units of a piece in turn; a wave asks for its next unit's K as soon as its scores are done and
// for the next V behind the product with this one.
template <typename T, int HD>
__global__ __launch_bounds__(64 * STREAM_WAVES, sizeof(T) * HD <= 256 ? 2 : 1) void k_paged_stream(PagedDev kv, ChunkDev ch, PagedAttnArgs a,
                                                                                               int shares, int least, int q_tiles, bool vec_q,
                                                                                               bool vec_out) {
  constexpr int NS = HD / 16, DB = HD / 32, W = STREAM_WAVES, BLOCK = 32 * HD, PIECES = HD / 4;
  typedef typename AttnFrag<T>::type frag_t;
  __shared__ __align__(16) float xo[W][32 * HD];
  __shared__ float xm[W][32], xl[W][32];
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, lg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.hq / kv.hkv, blocks = kv.page_size >> 5;

  walk<64 * W, 1>(kv, ch, a, shares, least, q_tiles, [&](const Item& item, const ChunkSeq& s, const Items&, int t0, int t1, int slot) {
    const int ncols = s.rows * G, col0 = item.qt * 32, total = s.len + s.rows;
    const int key_end = keys_of(s, G, 1, item.qt, a.anc == nullptr), key_lo = t0 * STREAM_TK;
    const int key_hi = min(t1 * STREAM_TK, key_end);
    const int r_lo = col0 / G;
    const int units = max(0, (((key_hi - key_lo + 31) >> 5) - wave + W - 1) / W);
    const int col = col0 + lr;
    const bool live = col < ncols;
    const int r = live ? col / G : 0, h = item.kvh * G + (live ? col % G : 0);
    const int64_t row = s.row0 + r;
    // Places of this wave's units, unit i at key_lo + 32 (wave + W i): one a lane, 64 units at a time
    int place = 0;
    auto look_up = [&](int i0) {
      const int i = i0 + lane, n = (key_lo >> 5) + wave + W * i, pg = n / blocks;
      if (i >= units) return;
      const int page = kv.table[(size_t)item.seq * kv.stride + pg];
      const bool bad = (unsigned)page >= (unsigned)kv.n_pages;
      if (bad) set_status(kv.status, ESP_DEV_BAD_PAGE);
      place = bad ? -1 : (page * kv.hkv + item.kvh) * blocks + n % blocks;
    };
    look_up(0);                                   // (on its way while the queries are)
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
    bool odd = false;
    auto add_odd = [&](int n, int c_lo, int left) {
      const int page = __builtin_amdgcn_readfirstlane(kv.table[(size_t)item.seq * kv.stride + n / blocks]);
      if ((unsigned)page >= (unsigned)kv.n_pages) return;
      attn_add_odd<T, HD>((const T*)kv.v + ((size_t)(page * kv.hkv + item.kvh) * blocks + n % blocks) * BLOCK,
                          attn_window(anc, a.anc_words, r, c_lo, s.rows) >> (4 * lg), left, lane, o);
    };

    frag_t kf[NS], vf[2 * DB];
    auto load_k = [&](int p) {
      const T* b = (const T*)kv.k + (size_t)max(p, 0) * BLOCK + lane * 8;
#pragma unroll
      for (int i = 0; i < NS; ++i) kf[i] = load_frag(b + i * 512);
    };
    auto load_v = [&](int p) {
      const T* b = (const T*)kv.v + (size_t)max(p, 0) * BLOCK + lane * 8;
#pragma unroll
      for (int i = 0; i < 2 * DB; ++i) vf[i] = load_frag(b + i * 512);
    };
    for (int i0 = 0; i0 < units; i0 += 64) {
    if (i0) look_up(i0);
    const int upto = min(64, units - i0);
    int here = __builtin_amdgcn_readlane(place, 0);
    __builtin_amdgcn_sched_barrier(0);            // (K first: the wait for it at the top of the loop is for as many younger loads as there are on every way)
    load_k(here);
    __builtin_amdgcn_sched_barrier(0);
    load_v(here);
    __builtin_amdgcn_sched_barrier(0);
    for (int i = 0; i < upto; ++i) {
      const int key0 = key_lo + 32 * (wave + W * (i0 + i)), c_lo = key0 - s.len, left = total - key0;
      const bool there = here >= 0;
      const int next = __builtin_amdgcn_readlane(place, min(i + 1, upto - 1));
      f32x16_t sc;
#pragma unroll
      for (int v = 0; v < 16; ++v) sc[v] = 0.f;
#pragma unroll
      for (int j = 0; j < NS; ++j) sc = attn_mma(kf[j], qf[j], sc);
      __builtin_amdgcn_sched_barrier(0);
      load_k(next);                               // (behind the last unit that one again, and for nothing: a branch would cost registers)
      __builtin_amdgcn_sched_barrier(0);
      const bool masked = !there || c_lo + 32 > (a.anc ? 0 : r_lo + 1);
      unsigned window = ~0u;
      if (masked) window = there ? attn_window(anc, a.anc_words, r, c_lo, s.rows) : 0u;
      frag_t pf[2];
      attn_softmax<T, DB>(sc, masked, window >> (4 * lg), a.scale, o, m, l, pf);
      if (masked) {
#pragma unroll
        for (int j = 0; j < 2 * DB; ++j) {
          if (left < 32) vf[j] = attn_zero_tail(vf[j], j & 1, lane, left);
          odd |= attn_any(attn_take_odd(vf[j]));
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] = attn_mma(vf[2 * db + u], pf[u], o[db]);
      __builtin_amdgcn_sched_barrier(0);
      load_v(next);
      __builtin_amdgcn_sched_barrier(0);
      here = next;
    }
    }
    if (__builtin_amdgcn_ballot_w64(odd) != 0ull)
      for (int i = 0; i < units; ++i) {
        const int n = (key_lo >> 5) + wave + W * i, c_lo = 32 * n - s.len;
        if (c_lo + 32 > 0) add_odd(n, c_lo, total - 32 * n);
      }
    l += __shfl_xor(l, 32, 64);
    // the waves' parts meet in LDS
    if (live) {
      put_columns<HD>(xo[wave], o, lane);
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
        acc += *reinterpret_cast<const f32x4_t*>(column_piece<HD>(xo[i], c, piece)) * f;
      }
      const int cc = col0 + c;
      if (slot < 0) {
        const int64_t at = ((int64_t)s.row0 + cc / G) * a.hq + item.kvh * G + cc % G;
        store4((T*)a.out + at * HD + 4 * piece, acc * (lt > 0.f ? 1.f / lt : 0.f), vec_out);
      } else {
        const Partials p = partials_of(a.partials, shares, 32, HD);
        const int64_t at = (int64_t)slot * 32 + c;
        *reinterpret_cast<f32x4_t*>(p.o + at * HD + 4 * piece) = acc;
        if (piece == 0) { p.ml[2 * at] = top * a.scale; p.ml[2 * at + 1] = lt; }
      }
    }
    __syncthreads();                              // the next piece's parts go there
  });
}

// --------------------------------------------------------------------------------------------------
// k_paged_tile: key tiles of 64 go from memory straight into a ring of LDS stages (a linear copy, the cache's blocks being in
// operand order), each brought by all eight waves and read by all of them.  A wave has a column tile, or, of the first or second half
// of each key tile's keys, shares one with its neighbour: waves go to SIMDs round-robin, and eight waves over 1 to 8 column tiles
// come out with the SIMDs' loads as even as they can be (5 tiles: 3, 3, 2, 2 half tiles of keys instead of 4, 2, 2, 2).
template <typename T, int HD> struct TileRing {
  static constexpr int BLOCK = 32 * HD * sizeof(T);               // 32 keys of K, or of V
  static constexpr int STAGE = 4 * BLOCK;                         // K and V of a tile
  static constexpr int STAGES = STAGE > 32768 ? 2 : 4;
  static constexpr int LPW = STAGE / TILE_WAVES / 1024;           // 1 KB loads of a wave for a tile
  static constexpr int BYTES = STAGE * STAGES;
  static_assert(BYTES >= TILE_WAVES * 32 * HD * 4, "the columns of all waves go there at the end");
};

template <int LPW>
__device__ __forceinline__ void load_run(const unsigned char* src, uint32_t lane_off, uint32_t dst) {
  load_to_lds16_sbase<0>(src, lane_off, dst);
  if constexpr (LPW > 1) load_to_lds16_sbase<1024>(src, lane_off, dst);
  if constexpr (LPW > 2) load_to_lds16_sbase<2048>(src, lane_off, dst);
  if constexpr (LPW > 3) load_to_lds16_sbase<3072>(src, lane_off, dst);
  if constexpr (LPW > 4) load_run<LPW - 4>(src + 4096, lane_off, dst + 4096);
}
// all but the youngest n tiles' loads of this wave have landed
template <int LPW>
__device__ __forceinline__ void wait_tiles_but(int n) {
  if (n >= 2) wait_loads_but<2 * LPW>();
  else if (n == 1) wait_loads_but<LPW>();
  else wait_loads_but<0>();
}

typedef const int __attribute__((address_space(4))) scalar_int;     // memory that no kernel writes meanwhile, read through the scalar cache

template <typename T, int HD>
__global__ __launch_bounds__(64 * TILE_WAVES) void k_paged_tile(PagedDev kv, ChunkDev ch, PagedAttnArgs a, int shares, int least, int q_tiles,
                                                               bool vec_q, bool vec_out) {
  typedef TileRing<T, HD> R;
  typedef typename AttnFrag<T>::type frag_t;
  constexpr int NS = HD / 16, DB = HD / 32, PIECES = HD / 4;
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ float xm[TILE_WAVES][32], xl[TILE_WAVES][32];
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, lg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.hq / kv.hkv, blocks = kv.page_size >> 5;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  // what this wave brings of a tile: a run of one block of K (waves 0-3) or V
  const int my_block = (wave >> 1) & 1;
  const size_t my_off = (size_t)(wave & 1) * (R::BLOCK / 2);
  const unsigned char* my_pool = (const unsigned char*)(wave < 4 ? kv.k : kv.v) + my_off;
  const uint32_t my_lds = lds0 + (uint32_t)((wave < 4 ? 0 : 2 * R::BLOCK) + my_block * R::BLOCK + my_off);

  walk<64 * TILE_WAVES, TILE_CAP>(kv, ch, a, shares, least, q_tiles, [&](const Item& item, const ChunkSeq& s, const Items& it, int t0, int t1, int slot) {
    const int seq = __builtin_amdgcn_readfirstlane(item.seq), kvh = __builtin_amdgcn_readfirstlane(item.kvh);
    const int qt = __builtin_amdgcn_readfirstlane(item.qt);
    const bool causal = a.anc == nullptr;
    const int ncols = s.rows * G, total = s.len + s.rows, keys = keys_of(s, G, it.per, qt, causal);
    const int nt = t1 - t0;
    const int ct = min(it.per, (ncols + 31) / 32 - qt * it.per);              // column tiles of this item
    const int pairs = min(ct, TILE_WAVES - ct), full = ct - pairs;             // tiles shared by two waves, and those that have one
    const bool paired = wave >= full;
    const int ctl = paired ? full + ((wave - full) >> 1) : wave;
    const int kh0 = paired ? (wave - full) & 1 : 0, kh1 = paired ? kh0 : 1;    // halves of the key tiles
    const bool works = ctl < ct;
    const int col = (qt * it.per + ctl) * 32 + lr;
    const bool live = works && col < ncols;
    const int r = live ? col / G : 0, h = kvh * G + (live ? col % G : 0);
    const int r_lo = works ? (qt * it.per + ctl) * 32 / G : 0, r_hi = min(s.rows - 1, ((qt * it.per + ctl) * 32 + 31) / G);
    const int64_t row = s.row0 + r;
    scalar_int* table = (scalar_int*)(uintptr_t)(kv.table + (size_t)seq * kv.stride);

    // are all pages there?  (Where one is not, its keys are looked at one block after the other.)
    bool bad = false;
    const int last_block = (min(keys, t1 * TILE_TK) - 1) >> 5;
    for (int p = 2 * t0 / blocks + tid; p <= last_block / blocks; p += 64 * TILE_WAVES)
      bad |= (unsigned)kv.table[(size_t)seq * kv.stride + p] >= (unsigned)kv.n_pages;
    if (bad) set_status(kv.status, ESP_DEV_BAD_PAGE);
    const bool any_bad = __syncthreads_or(bad);

    // this wave's next block: page number in the table, place in it; a block behind the last that is needed is that one
    int n = 2 * t0 + my_block, pg = min(n, last_block) / blocks, in = min(n, last_block) - pg * blocks;
    int page = table[pg];
    auto issue = [&](int i) {                     // tile t0 + i into stage i % STAGES; called for i = 0, 1, 2, ...
      const int p = (unsigned)page < (unsigned)kv.n_pages ? page : 0;
      const unsigned char* src = my_pool + ((size_t)(p * kv.hkv + kvh) * blocks + in) * R::BLOCK;
      load_run<R::LPW>(src, (uint32_t)lane * 16, my_lds + (uint32_t)(i % R::STAGES) * R::STAGE);
      n += 2;
      if (n <= last_block) {
        in += 2;
        while (in >= blocks) { in -= blocks; ++pg; }
        page = table[pg];
      } else if (n - 1 == last_block) {
        in += 1;
        if (in >= blocks) { in -= blocks; ++pg; }
        page = table[pg];
      }
    };
    issue(0);
    // The queries between the first tile's loads and the others': the compiler's wait for them, held here by the empty statement, covers
    // the first tile too, and no load that the compiler knows of is in flight in the loop (its wait would drain the ring).
    frag_t qf[NS];
    {
      const T* qp = (const T*)a.q + row * a.q_stride + h * HD + 8 * lg;
#pragma unroll
      for (int i = 0; i < NS; ++i) qf[i] = load_query(qp + 16 * i, vec_q);
#pragma unroll
      for (int i = 0; i < NS; ++i) asm volatile("" : "+v"(qf[i])::"memory");
    }
    for (int i = 1; i < R::STAGES - 1; ++i)
      if (i < nt) issue(i);
    const uint64_t* anc = causal ? nullptr : a.anc + row * a.anc_words;
    f32x16_t o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[i][v] = 0.f;
    float m = ATTN_UNSEEN, l = 0.f;
    bool odd = false;

    const unsigned char* frag = lds + lane * 8 * sizeof(T);
    for (int i = 0; i < nt; ++i) {
      // tile i has landed (this wave's loads retire in order; the barrier covers the other waves'), and every wave is done with tile i - 1,
      // whose stage takes tile i + STAGES - 1
      wait_tiles_but<R::LPW>(min(R::STAGES - 2, nt - 1 - i));
      __syncthreads();
      if (i + R::STAGES - 1 < nt) issue(i + R::STAGES - 1);
      if (!works) continue;
      const unsigned char* st = frag + (i % R::STAGES) * R::STAGE;
      for (int kh = kh0; kh <= kh1; ++kh) {
        const int key0 = (t0 + i) * TILE_TK + 32 * kh, c_lo = key0 - s.len;
        if (key0 >= total || (causal && c_lo > r_hi)) continue;                 // nobody here sees any of it
        bool there = true;
        if (any_bad) there = (unsigned)table[(key0 >> 5) / blocks] < (unsigned)kv.n_pages;
        const bool masked = !there || c_lo + 32 > (causal ? r_lo + 1 : 0);
        unsigned window = ~0u;
        if (masked) window = there ? attn_window(anc, a.anc_words, r, c_lo, s.rows) : 0u;
        attn_unit<T, HD>(st + kh * R::BLOCK, st + (2 + kh) * R::BLOCK, masked, window, total - key0, lane, a.scale, qf, o, m, l, odd);
      }
    }
    if (__builtin_amdgcn_ballot_w64(odd) != 0ull)
      for (int i = 0; i < 2 * nt; ++i) {
        const int n = 2 * t0 + i, c_lo = 32 * n - s.len;
        if ((i & 1) < kh0 || (i & 1) > kh1 || 32 * n >= keys || c_lo + 32 <= 0) continue;
        const int p = table[n / blocks];
        if ((unsigned)p >= (unsigned)kv.n_pages) continue;
        attn_add_odd<T, HD>((const T*)kv.v + ((size_t)(p * kv.hkv + kvh) * blocks + n % blocks) * (32 * HD),
                            attn_window(anc, a.anc_words, r, c_lo, s.rows) >> (4 * lg), total - 32 * n, lane, o);
      }
    l += __shfl_xor(l, 32, 64);

    // the ring is done with: columns of wave w at its place in it
    __syncthreads();
    float* xo = reinterpret_cast<float*>(lds) + wave * (32 * HD);
    if (works && kh0 == 1) {
      put_columns<HD>(xo, o, lane);
      if (lg == 0) { xm[wave][lr] = m; xl[wave][lr] = l; }
    }
    __syncthreads();
    if (works && kh0 == 0) {
      float fa = 1.f, fb = 0.f, mo = ATTN_UNSEEN, lo = 0.f;
      if (paired) {
        mo = xm[wave + 1][lr];
        lo = xl[wave + 1][lr];
        const float top = fmaxf(m, mo);
        fa = attn_weight(m, top, a.scale);
        fb = attn_weight(mo, top, a.scale);
        l = l * fa + lo * fb;
        m = top;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int v = 0; v < 16; v += 4) {
            const f32x4_t x = *reinterpret_cast<const f32x4_t*>(column_piece<HD>(xo + 32 * HD, lr, db * 8 + 2 * (v >> 2) + lg));
#pragma unroll
            for (int e = 0; e < 4; ++e) o[db][v + e] = o[db][v + e] * fa + x[e] * fb;
          }
      }
      const float inv = l > 0.f ? 1.f / l : 0.f;
      if (slot < 0) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[db][v] *= inv;
      }
      put_columns<HD>(xo, o, lane);
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");       // (a wave's LDS accesses are done in order: for the compiler)
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      const int c0 = (qt * it.per + ctl) * 32, n_live = min(32, ncols - c0);
      if (slot < 0) {
        for (int t = lane; t < n_live * PIECES; t += 64) {
          const int c = t / PIECES, piece = t % PIECES, cc = c0 + c;
          const int64_t at = ((int64_t)s.row0 + cc / G) * a.hq + kvh * G + cc % G;
          store4((T*)a.out + at * HD + 4 * piece, *reinterpret_cast<const f32x4_t*>(column_piece<HD>(xo, c, piece)), vec_out);
        }
      } else {
        const Partials p = partials_of(a.partials, shares, 32 * TILE_CAP, HD);
        const int64_t at = (int64_t)slot * (32 * TILE_CAP) + ctl * 32;
        for (int t = lane; t < n_live * PIECES; t += 64) {
          const int c = t / PIECES, piece = t % PIECES;
          *reinterpret_cast<f32x4_t*>(p.o + (at + c) * HD + 4 * piece) = *reinterpret_cast<const f32x4_t*>(column_piece<HD>(xo, c, piece));
        }
        if (lg == 0 && lr < n_live) { p.ml[2 * (at + lr)] = m * a.scale; p.ml[2 * (at + lr) + 1] = l; }
      }
    }
    // the stores do not count as loads of the next piece, whose ring goes where the columns are
    wait_loads_but<0>();
    __syncthreads();
  });
}

// --------------------------------------------------------------------------------------------------
// The pieces of an item that begins in share w and does not end there: those of the shares behind it, up to the one that ends it.
// A workgroup has 32 columns, HD / 4 threads and more a column.
template <typename T, int HD, int CAP>
__global__ __launch_bounds__(256) void k_paged_merge(PagedDev kv, ChunkDev ch, PagedAttnArgs a, int shares, bool vec_out) {
  constexpr int PIECES = HD / 4, COLS = 32 * CAP;
  const int w = blockIdx.x, ctl = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const Partials p = partials_of(a.partials, shares, COLS, HD);
  const Item item = p.notes[w].begun;
  if (item.seq < 0) return;
  const ChunkSeq s = chunk_seq(kv, ch, item.seq);
  const int G = a.hq / kv.hkv, ncols = s.rows * G;
  const Items it = items_of(s.rows, G, CAP);
  const int c0 = (item.qt * it.per + ctl) * 32, n_live = min(32, ncols - c0);
  if (ctl >= it.per || n_live <= 0) return;
  for (int t = tid; t < n_live * PIECES; t += 256) {
    const int c = t / PIECES, piece = t % PIECES, cc = c0 + c;
    const int64_t col = ctl * 32 + c;
    int64_t at = (int64_t)(2 * w + 1) * COLS + col;
    float top = p.ml[2 * at], lt = p.ml[2 * at + 1];
    f32x4_t acc = *reinterpret_cast<const f32x4_t*>(p.o + at * HD + 4 * piece);
    if (!(lt > 0.f)) top = -INFINITY;
    for (int x = w + 1; x < shares; ++x) {
      const int first = p.notes[x].first;
      if (first & HAS) {
        at = (int64_t)(2 * x) * COLS + col;
        const float m = p.ml[2 * at], l = p.ml[2 * at + 1];
        const f32x4_t o = *reinterpret_cast<const f32x4_t*>(p.o + at * HD + 4 * piece);
        const float now = l > 0.f ? fmaxf(top, m) : top;
        const float fa = top > -INFINITY ? __builtin_amdgcn_exp2f(top - now) : 0.f, fb = l > 0.f ? __builtin_amdgcn_exp2f(m - now) : 0.f;
        lt = lt * fa + l * fb;
        acc = acc * fa + o * fb;
        top = now;
      }
      if (first & ENDS) break;
    }
    (void)lane;
    const int64_t out = ((int64_t)s.row0 + cc / G) * a.hq + item.kvh * G + cc % G;
    store4((T*)a.out + out * HD + 4 * piece, acc * (lt > 0.f ? 1.f / lt : 0.f), vec_out);
  }
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// the attribute for more than 64 KB of LDS, once a device
template <typename T, int HD>
hipError_t allow_lds(unsigned bytes) {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (done.load(std::memory_order_relaxed) & bit) return hipSuccess;
  e = hipFuncSetAttribute((const void*)k_paged_tile<T, HD>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

template <typename T, int HD>
hipError_t launch(hipStream_t st, const PagedDev& kv, const ChunkDev& ch, const PagedAttnArgs& a, const PagedAttnPlan& p) {
  const bool vec_q = (uintptr_t)a.q % 16 == 0 && a.q_stride * (int64_t)sizeof(T) % 16 == 0, vec_out = (uintptr_t)a.out % 16 == 0;
  int64_t grid = (p.shares + 7) / 8 * 8;
  if (p.shares == 0) {
    const int64_t groups = (int64_t)kv.batch * kv.hkv;
    grid = (p.q_tiles > 1 && groups >= 8 ? (groups + 7) & ~7ll : groups) * p.q_tiles;
  }
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  if (p.tile) {
    constexpr unsigned bytes = TileRing<T, HD>::BYTES;
    const hipError_t e = allow_lds<T, HD>(bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_paged_tile<T, HD>), dim3((unsigned)grid), dim3(64 * TILE_WAVES), bytes, st, kv, ch, a, p.shares, p.least, p.q_tiles,
                       vec_q, vec_out);
    if (p.shares) hipLaunchKernelGGL((k_paged_merge<T, HD, TILE_CAP>), dim3(p.shares, TILE_CAP), dim3(256), 0, st, kv, ch, a, p.shares, vec_out);
  } else {
    hipLaunchKernelGGL((k_paged_stream<T, HD>), dim3((unsigned)grid), dim3(64 * STREAM_WAVES), 0, st, kv, ch, a, p.shares, p.least, p.q_tiles, vec_q,
                       vec_out);
    if (p.shares) hipLaunchKernelGGL((k_paged_merge<T, HD, 1>), dim3(p.shares, 1), dim3(256), 0, st, kv, ch, a, p.shares, vec_out);
  }
  return hipGetLastError();
}

}  // namespace

PagedAttnPlan paged_attn_plan(int dtype, int hd, int batch, int hq, int hkv, int total_rows, int max_rows, int len_bound) {
  PagedAttnPlan p;
  const int G = hq / hkv;
  const int64_t cols = (int64_t)max_rows * G, keys = (int64_t)len_bound + max_rows;
  p.tile = cols > 32;
  const int cap = p.tile ? TILE_CAP : 1, tk = p.tile ? TILE_TK : STREAM_TK;
  p.q_tiles = (int)std::max<int64_t>(1, ceil_div(ceil_div(cols, 32), cap));
  // items that there can be, and workgroups that have a place at once
  const int64_t items = (int64_t)hkv * std::min<int64_t>((int64_t)batch * p.q_tiles, ceil_div((int64_t)total_rows * G, 32 * cap) + batch);
  const bool big = dtype == ESP_F32 || hd == 128;
  const int64_t places = 256 * (p.tile ? 1 : dtype == ESP_F32 && hd == 128 ? 1 : 2);
  (void)big;
  p.least = p.tile ? 4 : 2;
  const int64_t tiles = ceil_div(keys, tk);
  if (tiles > p.least && items < 4 * places) p.shares = (int)std::min(places, ceil_div(items * tiles, p.least));
  return p;
}
size_t paged_attn_partial_floats(const PagedAttnPlan& p, int hd) {
  return p.shares ? notes_floats(p.shares) + (size_t)2 * p.shares * 32 * (p.tile ? TILE_CAP : 1) * (hd + 2) : 0;
}

hipError_t launch_paged_attn(hipStream_t st, int dtype, int hd, const PagedDev& kv, const ChunkDev& ch, const PagedAttnArgs& a,
                             const PagedAttnPlan& p) {
  PagedAttnArgs x = a;
  x.scale = a.scale * LOG2E;
  if (dtype == ESP_F32) return hd == 64 ? launch<float, 64>(st, kv, ch, x, p) : launch<float, 128>(st, kv, ch, x, p);
  return hd == 64 ? launch<bf16_t, 64>(st, kv, ch, x, p) : launch<bf16_t, 128>(st, kv, ch, x, p);
}
