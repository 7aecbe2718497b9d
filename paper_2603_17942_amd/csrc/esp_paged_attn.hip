// Grouped-query attention of a chunk of new rows over a paged KV cache, causal or under ancestor bitsets.
//
// The G = n_q / n_kv query heads of a kv head times a sequence's rows are its query columns, in tiles of 32.  An item is a group of up to
// CAP column tiles of one (sequence, kv head) over all keys they see, which are walked in key tiles of TK.  Either a workgroup has an item
// (the launch has enough of them to even out, or they are too short to be cut), or the items form a line of work that is cut into equal
// shares, one a workgroup: the pieces of an item that a cut went through leave (m, l, O) in memory, and k_paged_merge adds them up in the
// line's order, so results do not depend on scheduling.  Only the device knows lengths and rows; every workgroup looks its share up.
//
// k_paged_stream (32 columns an item, four waves that share them) is for decoding and for little work, bound by the memory that K and V
// come from; k_paged_tile (up to 256 columns in bf16, 128 in fp32) for much of it, bound by the matrix cores: it walks a ring of key tiles in
// LDS.  paged_attn_plan chooses.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "esp_attn_unit.h"
#include "esp_paged.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int MOST_SHARES = 512;
constexpr int STREAM_WAVES = 4, STREAM_TK = 32 * STREAM_WAVES;
constexpr int TILE_WAVES = 4, TILE_TK = 64;
template <typename T> constexpr int TILE_NT = sizeof(T) == 2 ? 2 : 1;              // column tiles of a wave
template <typename T> constexpr int TILE_CAP = TILE_WAVES * TILE_NT<T>;            // and of an item at most

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
// a value that the compiler does not see through: what is computed from it stays where it is used.  (Addresses that it takes out of a loop
// cost registers over all of it, and a register that it saves to memory it has restored in front of the end of a branch, with the
// branch's lanes only.  The kernels here are to save no vector register; scalar ones, up to 171 of a kernel, are kept in lanes of vector registers.)
__device__ __forceinline__ int opaque(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// does a thread of the workgroup say so; said: LDS, a word a wave
template <int WAVES>
__device__ __forceinline__ bool any_thread(bool here, int* said) {
  const bool mine = __builtin_amdgcn_ballot_w64(here) != 0ull;
  said[threadIdx.x >> 6] = mine;                  // (all lanes the same)
  __syncthreads();
  int any = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) any |= said[w];
  return uniform(any) != 0;
}

// ---- the line of work --------------------------------------------------------------------------------------------
struct Item { int seq, kvh, qt; };
struct Place { int seq, kvh, at; };             // item `at` of a sequence and kv head in the line's order
struct Cut { Place place; int tile; };          // before key tile `tile` of the item there

// what a sequence's items are: n of them for each kv head, of `per` column tiles, the last one of what is left
struct Items { int n, per; };
__host__ __device__ __forceinline__ Items items_of(int rows, int G, int cap) {
  const int ct = (rows * G + 31) / 32, n = (ct + cap - 1) / cap;      // (the host has checked rows * G)
  return {n, n ? (ct + n - 1) / n : 0};
}
// keys that item qt sees
__device__ __forceinline__ int keys_of(const ChunkSeq& s, int G, int per, int qt, bool causal) {
  const int rows = causal ? min(s.rows, ((qt + 1) * per * 32 + G - 1) / G) : s.rows;
  return s.len + rows;
}
// The line's order of a sequence's items: the last (which sees the most keys), the first, the last but one, the second ..., so that two
// neighbours weigh the same.
__device__ __forceinline__ int item_at(int n, int at) { return at & 1 ? at >> 1 : n - 1 - (at >> 1); }
// Weights along the line, in keys x time of a key tile: an item counts `start` for its beginning and end and its keys.  Cuts need not be
// exact, only the same for everybody, and never before the one in front.
struct Weights {
  float first, slope;                             // item k weighs first + slope (k + 1)
  __device__ __forceinline__ float of(int k) const { return first + slope * (float)(k + 1); }
  __device__ __forceinline__ float sum(int n) const { return first * (float)n + slope * (0.5f * (float)n * (float)(n + 1)); }
};
constexpr int SNAP = 4;                           // a cut this near to an item's beginning or end (key tiles, at most a quarter of a share) goes there
// time of a key tile of an item with that many column tiles, and of its start and end, in units of a key's time (tile kernel: 64 keys take
// 1.95 us with more than four column tiles, 1.4 with three or four, 1 with less; a start and end 13)
template <bool STREAM>
__host__ __device__ constexpr int tile_time(int per) { return STREAM ? 1 : per > 4 ? 10 : per > 2 ? 7 : 5; }
template <bool STREAM>
constexpr int start_time() { return STREAM ? 64 : 4000; }
template <bool STREAM>
__device__ __forceinline__ Weights weights_of(const ChunkSeq& s, int G, int per, bool causal) {
  const float t = (float)tile_time<STREAM>(per);
  return {(float)start_time<STREAM>() + t * (float)(s.len + (causal ? 0 : s.rows)), causal ? t * (float)(per * 32) / (float)G : 0.f};
}

// Share of a workgroup if n of them have work: the ones next to each other on the line, which read the same keys, on one XCD; those that have
// none behind them.
__device__ __forceinline__ int share_at(int block, int n) {
  const int per_xcd = (n + 7) >> 3;
  return block >> 3 < per_xcd ? (block & 7) * per_xcd + (block >> 3) : block;
}

// Where a workgroup's share w of `shares` begins and ends.  Order of the line: kv heads, sequences, column groups from the last.  The device may use fewer
// shares than were launched: none with less than `least` key tiles.  False: no such share.  Every wave finds out for itself: a lane a
// sequence, 64 at a time, then even lanes for the beginning and odd ones for the end.
template <bool STREAM>
__device__ __forceinline__ bool share_of(const PagedDev& kv, const ChunkDev& ch, int G, int cap, bool causal, int block, int shares, int least, int& w,
                                         Cut& lo, Cut& hi) {
  constexpr int TK = STREAM ? STREAM_TK : TILE_TK;
  const int lane = threadIdx.x & 63;
  const bool one = kv.batch == 1;                 // (then every lane holds that sequence)
  ChunkSeq s;
  Items it;
  Weights wt;
  float mine, upto;
  auto weigh = [&](int b) {
    s = chunk_seq(kv, ch, min(b, kv.batch - 1));
    it = items_of(s.rows, G, cap);
    wt = weights_of<STREAM>(s, G, it.per, causal);
    mine = upto = s.ok && (one || b < kv.batch) ? wt.sum(it.n) : 0.f;
    if (one) return;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const float y = __shfl_up(upto, o, 64);
      if (lane >= o) upto += y;
    }
  };
  float per_head = 0.f;
  for (int b0 = 0; b0 < kv.batch; b0 += 64) {
    weigh(b0 + lane);
    per_head += one ? upto : __shfl(upto, 63, 64);
  }
  const float all = per_head * (float)kv.hkv;
  w = block;
  if (uniform(all > 0.f) == 0) return false;
  int n = uniform(max(1, (int)min((float)shares, all / (float)(tile_time<STREAM>(cap) * TK * least))));
  if (one && n > it.n * kv.hkv) n = uniform(n - n % (it.n * kv.hkv));         // (as the host does where the bound is the length)
  w = share_at(block, n);
  if (w >= n) return false;
  const float at = all / (float)n * (float)(w + (lane & 1));
  const int head = min((int)(at / per_head), kv.hkv - 1);
  const float off = max(at - (float)head * per_head, 0.f);
  // the last sequence with work that begins at or before this place
  float begin = 0.f, base = 0.f;
  int seq = 0;
  if (!one) {
    Weights fw = wt;
    ChunkSeq fs = s;
    for (int b0 = 0; b0 < kv.batch; b0 += 64) {
      if (kv.batch > 64) weigh(b0 + lane);
      const float before = base + (upto - mine), off0 = __shfl(off, 0, 64), off1 = __shfl(off, 1, 64);
      const uint64_t in0 = __builtin_amdgcn_ballot_w64(mine > 0.f && before <= off0), in1 = __builtin_amdgcn_ballot_w64(mine > 0.f && before <= off1);
      const uint64_t in = lane & 1 ? in1 : in0;
      const int l = in ? 63 - __clzll((long long)in) : 0;
      const float b_ = __shfl(before, l, 64);
      const Weights w_{__shfl(wt.first, l, 64), __shfl(wt.slope, l, 64)};
      const int r_ = __shfl(s.rows, l, 64), n_ = __shfl(s.len, l, 64);
      if (in) { begin = b_; fw = w_; fs.rows = r_; fs.len = n_; seq = b0 + l; }
      base += __shfl(upto, 63, 64);
    }
    wt = fw;
    s = fs;
    it = items_of(s.rows, G, cap);
  }
  const float into = max(off - begin, 0.f), pair = 2.f * wt.first + wt.slope * (float)(it.n + 1);
  const int j = min((int)(into / pair), (it.n - 1) >> 1);
  float in_item = max(into - (float)j * pair, 0.f);
  const float heavy = wt.of(it.n - 1 - j);
  int at_ = 2 * j;
  if (in_item >= heavy && at_ + 1 < it.n) { in_item -= heavy; ++at_; }
  in_item -= (float)start_time<STREAM>();
  const float of_tile = (float)(tile_time<STREAM>(it.per) * TK);
  const int tiles = (keys_of(s, G, it.per, item_at(it.n, at_), causal) + TK - 1) / TK;
  int tile = in_item > 0.f ? (int)min(ceilf(in_item / of_tile), (float)tiles) : 0;
  // (an item that is cut costs a beginning, an end and two partials more than one that is not)
  if (!STREAM) {
    const int snap = min(SNAP, (int)(all / (float)n / (4.f * of_tile)));
    tile = tile <= min(snap, tiles >> 1) ? 0 : tiles - tile <= snap ? tiles : tile;
  }
  auto take = [&](int x, int e) { return uniform(__shfl(x, e, 64)); };
  lo = Cut{{take(seq, 0), take(head, 0), take(at_, 0)}, take(tile, 0)};
  hi = w + 1 == n ? Cut{{kv.batch, kv.hkv, 0}, 0} : Cut{{take(seq, 1), take(head, 1), take(at_, 1)}, take(tile, 1)};
  return true;
}
// a sequence's scalars, the same for the whole wave
__device__ __forceinline__ ChunkSeq uniform_seq(const PagedDev& kv, const ChunkDev& ch, int seq) {
  const ChunkSeq s = chunk_seq(kv, ch, seq);
  return {uniform(s.row0), uniform(s.rows), uniform(s.len), uniform((int)s.ok) != 0};
}
__device__ __forceinline__ bool same(const Place& a, const Place& b) { return a.seq == b.seq && a.kvh == b.kvh && a.at == b.at; }

// Partials: a slot of 32 columns for each of an item's column tiles: their HD sums, then for every column m in powers of two and l.  Share w
// has slots 2 w, for the piece that it begins with if that is not an item's first, and 2 w + 1, for the piece that it ends with if that is an
// item's first and not its last.
// What a share leaves for the merge: the item that begins in slot 2 w + 1 (columns 0: none), and of slot 2 w whether there is anything in
// it (HAS) and whether the item ends in this share, or there is none (ENDS).
struct alignas(16) ShareNote { int columns, col0, row0, kvh, first, pad[3]; };
enum { HAS = 1, ENDS = 2 };
inline size_t notes_floats(int shares) { return (size_t)shares * sizeof(ShareNote) / 4; }
__host__ __device__ constexpr size_t slot_floats(int cols, int hd) { return (size_t)cols * (hd + 2); }
struct Partials {
  ShareNote* notes;
  float* first;
  int cols, hd;
  __device__ __forceinline__ float* sums(int slot) const { return first + slot_floats(cols, hd) * slot; }
  __device__ __forceinline__ float* stats(int slot) const { return sums(slot) + cols * hd; }
};
__device__ __forceinline__ Partials partials_of(float* base, int shares, int cols, int hd) {
  return {(ShareNote*)base, base + (size_t)shares * sizeof(ShareNote) / 4, cols, hd};
}

// Walks the pieces of a workgroup: run(item, sequence, its items, first and last key tile, slot of the partial or -1 for a whole item).
template <int NT, bool STREAM, typename RUN>
__device__ __forceinline__ void walk(const PagedDev& kv, const ChunkDev& ch, const PagedAttnArgs& a, const PagedAttnPlan& plan, RUN run) {
  constexpr int TK = STREAM ? STREAM_TK : TILE_TK;
  const int shares = plan.shares, q_tiles = plan.q_tiles, CAP = STREAM ? 1 : plan.cap;
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
    hi = Cut{lo.place, INT32_MAX};
    if (lo.place.kvh == 0 && lo.place.at == 0 && threadIdx.x == 0 && !chunk_seq(kv, ch, lo.place.seq).ok)
      set_status(kv.status, chunk_fault(ch, lo.place.seq));
  } else {
    if (blockIdx.x == 0)
      for (int b = threadIdx.x; b < kv.batch; b += NT)
        if (!chunk_seq(kv, ch, b).ok) set_status(kv.status, chunk_fault(ch, b));
    if (!share_of<STREAM>(kv, ch, G, CAP, causal, blockIdx.x, shares, plan.least, w, lo, hi)) lo = Cut{{0, kv.hkv, 0}, 0};
    if (w >= shares) return;
  }
  ShareNote note{0, 0, 0, 0, ENDS, {0, 0, 0}};
  Place pl = lo.place;
  int t0 = lo.tile;
  while (pl.kvh < kv.hkv) {
    const ChunkSeq s = uniform_seq(kv, ch, pl.seq);
    const Items it = items_of(s.rows, G, CAP);
    const bool last = same(pl, hi.place), there = s.ok && pl.at < it.n;
    if (there) {
      const int qt = shares == 0 ? pl.at : item_at(it.n, pl.at);
      const int tiles = (keys_of(s, G, it.per, qt, causal) + TK - 1) / TK, t1 = last ? min(hi.tile, tiles) : tiles;
      const bool ends = t1 >= tiles;
      if (t0 > 0) note.first = (t1 > t0 ? HAS : 0) | (ends ? ENDS : 0);
      else if (!ends && t1 > 0) {
        const int col0 = qt * it.per * 32;
        note.columns = min(it.per * 32, s.rows * G - col0); note.col0 = col0; note.row0 = s.row0; note.kvh = pl.kvh;
      }
      if (t1 > t0)
        run(Item{uniform(pl.seq), uniform(pl.kvh), uniform(qt)}, s, it, uniform(t0), uniform(t1), t0 > 0 ? 2 * w : ends ? -1 : 2 * w + 1);
    }
    if (last) break;
    t0 = 0;
    if (there && pl.at + 1 < it.n) {
      ++pl.at;
    } else {                                      // the next sequence's, or the next kv head's first sequence's
      pl.at = 0;
      if (++pl.seq == kv.batch) { pl.seq = 0; ++pl.kvh; }
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
// for the next V behind the product with this one: four waves, two workgroups a CU, have 128 KB of it on their way.  Measured, 32/8 heads of
// 128 in bf16: 32 rows over 8192 keys each 192 us, 5.6 TB/s (a plain read on this card 6.1); one over 2048 keys 13 us, of which 8 here (2 to
// look the share up, 2 until the first keys are there) and 5 in the merge.
template <typename T, int HD>
__global__ __launch_bounds__(64 * STREAM_WAVES, sizeof(T) * HD <= 256 ? 2 : 1) void k_paged_stream(PagedDev kv, ChunkDev ch, PagedAttnArgs a,
                                                                                               PagedAttnPlan plan, bool vec_q, bool vec_out) {
  constexpr int NS = HD / 16, DB = HD / 32, W = STREAM_WAVES, BLOCK = 32 * HD, PIECES = HD / 4;
  typedef typename AttnFrag<T>::type frag_t;
  __shared__ __align__(16) float xo[W][32 * HD];
  __shared__ float xm[W][32], xl[W][32];
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, lg = lane >> 5;
  const int wave = uniform(tid >> 6);
  const int G = a.hq / kv.hkv, blocks = kv.page_size >> 5;

  walk<64 * W, true>(kv, ch, a, plan, [&](const Item& item, const ChunkSeq& s, const Items&, int t0, int t1, int slot) {
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
        const int lane = opaque(threadIdx.x) & 63;
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
    l = attn_sum_of_halves(l);
    // the waves' parts meet in LDS
    const int tid = opaque(threadIdx.x), lane = tid & 63;
    if (live) {
      put_columns<HD>(xo[wave], o, lane);
      if (lane < 32) { xm[wave][lane] = m; xl[wave][lane] = l; }
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
        const Partials p = partials_of(a.partials, plan.shares, 32, HD);
        *reinterpret_cast<f32x4_t*>(p.sums(slot) + c * HD + 4 * piece) = acc;
        if (piece == 0) { p.stats(slot)[2 * c] = top * a.scale; p.stats(slot)[2 * c + 1] = lt; }
      }
    }
    __syncthreads();                              // the next piece's parts go there
  });
}

// piece J of a run of 1 KB pieces: a wave-uniform address and 16 bytes a lane, to dst + 16 x lane.  As text: the waits are counted by hand.
template <int J>
__device__ __forceinline__ void load_piece(const unsigned char* src, uint32_t lane_off, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 offset:%3" ::"s"(dst + (J >> 2) * 4096), "v"(lane_off),
               "s"(src + (J >> 2) * 4096), "n"((J & 3) * 1024)
               : "memory", "m0");
}
template <int FROM, int TO>
__device__ __forceinline__ void load_pieces(const unsigned char* src, uint32_t lane_off, uint32_t dst) {
  if constexpr (FROM < TO) {
    load_piece<FROM>(src, lane_off, dst);
    load_pieces<FROM + 1, TO>(src, lane_off, dst);
  }
}
// all but the youngest n tiles' loads of this wave have landed
template <int LPW>
__device__ __forceinline__ void wait_tiles_but(int n) {
  if (n >= 2) wait_loads_but<2 * LPW>();
  else if (n == 1) wait_loads_but<LPW>();
  else wait_loads_but<0>();
}

typedef const int __attribute__((address_space(4))) scalar_int;     // memory that no kernel writes meanwhile, read through the scalar cache

// --------------------------------------------------------------------------------------------------
// k_paged_tile: key tiles of 64 go from memory straight into a ring of LDS stages (a linear copy, the cache's blocks being in operand order),
// a block by each of four waves, and are read by all of them.  A fragment that feeds one 32 x 32 x 16 instruction is read from LDS at the full
// rate of LDS (1 KB in the 32 clocks that the instruction takes on each of four SIMDs), so eight waves with 32 columns each waited for LDS
// (2.4 us a key tile and 256 columns).  In bf16 a wave has 64 columns, two tiles that share every fragment, and 512 registers: one wave a SIMD, which has to overlap its
// own matrix work and softmax.  Its two column tiles run half a unit apart: while one's scores or outputs are on the matrix
// cores, the other's exponentials are computed between the instructions, in four groups a unit of 32 keys:
//   scores of tile 0, next unit  | exponentials of tile 1        outputs of tile 0            | exponentials of tile 1; maximum of tile 0, next unit
//   scores of tile 1, next unit  | exponentials of tile 0, next  outputs of tile 1            | exponentials of tile 0, next; maximum of tile 1, next
// Outputs and queries sit in AGPRs (the instructions that touch the outputs are text, so that the compiler moves neither).  In fp32 a wave has
// one tile: its matrix instructions take 16 times as long, and softmax beside them is an eighth.
// Measured, 32/8 heads of 128: 1.95 us a key tile of 256 columns; 8192 rows from none 522 us, 1055 TF/s (of which the matrix instructions alone
// take 410; a product of 8192 x 8192 x 8192 on this card 1388 TF/s), 512 rows over 32768 keys 1025 TF/s.  A piece takes 13 us beside its
// tiles: 2 to look its share up, 4 until the first tile and the queries are there, 1.5 for the look at outputs where rows are hidden, 2 to 4
// to store them.
template <typename T, int HD> struct TileRing {
  static constexpr int BLOCK = 32 * HD * sizeof(T), STAGE = 4 * BLOCK, STAGES = STAGE > 32768 ? 2 : 4, LPW = BLOCK / 1024;
  // Tiles that are asked for ahead.  With two column tiles a wave is half a tile into the next scores when it stops at the barrier, so
  // the stage it came from is not free yet.
  static constexpr int AHEAD = STAGES - (TILE_NT<T> - 1);
  static constexpr int BYTES = STAGE * STAGES;
  static_assert((BYTES & (BYTES - 1)) == 0);
  static_assert(BYTES >= TILE_CAP<T> * 32 * HD * 4, "the columns of all waves go there at the end");
};
constexpr int TILE_ANC = 2560;                    // 64-bit words of ancestor bitsets that are kept in LDS

__device__ __forceinline__ void tile_out(f32x16_t& o, bf16x8_t v, bf16x8_t p) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(o) : "v"(v), "v"(p));
}
// The text's matrix instructions, of which the compiler knows nothing, have their results before it reads these registers ...
template <int DB>
__device__ __forceinline__ void tile_settle(f32x16_t (&o)[DB]) {
  asm volatile("s_nop 15\n\ts_nop 15" : "+a"(o[0]));
#pragma unroll
  for (int i = 1; i < DB; ++i) asm volatile("" : "+a"(o[i]));
}
// ... and begin two instructions or more behind the last that wrote one of their operands
__device__ __forceinline__ void tile_begin() { asm volatile("s_nop 1"); }
__device__ __forceinline__ void tile_zero(f32x16_t& x) {
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = 0.f;
}

// A column tile of a wave
template <typename T, int HD> struct ColumnTile {
  f32x16_t sc;                                    // scores of a unit
  float m, mb, l, limit;                          // reference of the exponents, the same scaled, sum, and the score from which the reference moves
  typename AttnFrag<T>::type p[2];                // probabilities: rounded to bf16 for the product, their sum is of the unrounded ones
  __device__ __forceinline__ void start() {
    m = ATTN_UNSEEN; mb = 0.f; l = 0.f; limit = ATTN_UNSEEN;
  }
  // Step s of a unit's exponentials, -2 .. 15: element s + 2 gets its exponent, s + 1 is raised, s goes to the sum and the operand.  A wave has
  // its SIMD to itself, so what depends on each other is a step apart.  (The empty statements keep it beside the matrix instructions: the
  // results are used blocks of code later, and the compiler would compute them there.)
  __device__ __forceinline__ void exp_step(int s, float scale) {
    if (s + 2 < 16) {
      float x = fmaf(sc[s + 2], scale, -mb);
      asm volatile("" : "+v"(x));
      sc[s + 2] = x;
    }
    if (s + 1 >= 0 && s + 1 < 16) {
      float x = __builtin_amdgcn_exp2f(sc[s + 1]);
      asm volatile("" : "+v"(x));
      sc[s + 1] = x;
    }
    if (s >= 0) {
      l += sc[s];
      asm volatile("" : "+v"(l));
      p[s >> 3][s & 7] = from_f32<T>(sc[s]);
    }
  }
  __device__ __forceinline__ void hide(unsigned seen) {
#pragma unroll
    for (int v = 0; v < 16; ++v) sc[v] = ((seen >> (8 * (v >> 2) + (v & 3))) & 1u) ? sc[v] : ATTN_UNSEEN;
  }
  __device__ __forceinline__ void top_of(float& top, int i) { top = attn_max3(top, sc[2 * i], sc[2 * i + 1]); }
  // Moves the reference where a score is above its limit; o: the outputs so far, all of whose sums are of units before this one.
  __device__ __forceinline__ void follow(float top, float scale, float slack, f32x16_t (&o)[HD / 32]) {
    if (__builtin_amdgcn_ballot_w64(top > limit) == 0ull) return;
    top = attn_max_of_halves(top);
    const float was = mb;
    const bool moves = top > limit, had = m > 0.5f * ATTN_UNSEEN;
    if (moves) { m = top; mb = top * scale; limit = top + slack; }
    if (__builtin_amdgcn_ballot_w64(moves && had) == 0ull) return;
    const float f = moves && had ? __builtin_amdgcn_exp2f(was - mb) : 1.f;
    l *= f;
    tile_settle(o);
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) {
#pragma unroll
      for (int v = 0; v < 16; ++v) o[i][v] *= f;
      asm volatile("" : "+a"(o[i]));              // (back where it was, one after the other)
    }
  }
};

template <typename T, int HD>
__global__ __launch_bounds__(64 * TILE_WAVES, 1) void k_paged_tile(PagedDev kv, ChunkDev ch, PagedAttnArgs a, PagedAttnPlan plan, bool vec_q,
                                                                  bool vec_out) {
  typedef TileRing<T, HD> R;
  typedef typename AttnFrag<T>::type frag_t;
  constexpr int NT = TILE_NT<T>, NS = HD / 16, DB = HD / 32, PIECES = HD / 4, EPI = 8 / NS;   // EPI: exponentials beside a matrix instruction
  extern __shared__ __align__(16) unsigned char lds[];
  uint64_t* anc_lds = reinterpret_cast<uint64_t*>(lds + R::BYTES);
  __shared__ float xm[TILE_WAVES][32], xl[TILE_WAVES][32];
  __shared__ int said[2][TILE_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, lg = lane >> 5;
  const int wave = uniform(tid >> 6);
  const int G = a.hq / kv.hkv, blocks = kv.page_size >> 5;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  const bool causal = a.anc == nullptr;
  const float slack = ATTN_SLACK / a.scale;
  // what this wave brings of a tile: a block of K (waves 0 and 1) or V
  const unsigned char* my_pool = (const unsigned char*)(wave < 2 ? kv.k : kv.v);
  const uint32_t my_lds = lds0 + (uint32_t)wave * R::BLOCK;

  walk<64 * TILE_WAVES, false>(kv, ch, a, plan, [&](const Item& item, const ChunkSeq& s, const Items& it, int t0, int t1, int slot) {
    const int seq = item.seq, kvh = item.kvh, qt = item.qt;
    const int ncols = s.rows * G, total = s.len + s.rows, keys = keys_of(s, G, it.per, qt, causal);
    const int nt = t1 - t0, col0 = qt * it.per * 32;
    const int ct = min(it.per, (ncols - col0 + 31) / 32);                     // column tiles of this item
    // Wave w has tiles w and w + 4.  One or two tiles are shared by two waves each, which have the halves of every key tile.
    const bool halves = ct <= 2;
    const int kh0 = halves ? wave >> 1 : 0, kh1 = halves ? kh0 : 1, ct0 = halves ? wave & 1 : wave;
    const int mine = ct0 >= ct ? 0 : NT == 2 && ct0 + 4 < ct ? 2 : 1;
    scalar_int* table = (scalar_int*)(uintptr_t)(kv.table + (size_t)seq * kv.stride);

    int col[NT], r[NT], r_lo[NT];
    bool live[NT];
#pragma unroll
    for (int c = 0; c < NT; ++c) {
      const int first = col0 + (ct0 + 4 * c) * 32;
      col[c] = first + lr;
      live[c] = c < mine && col[c] < ncols;
      r[c] = live[c] ? col[c] / G : 0;
      r_lo[c] = first / G;
    }
    // ancestor bitsets of the item's rows in LDS, where they fit
    const int row_lo = col0 / G, n_rows = (min(ncols, col0 + ct * 32) - 1) / G - row_lo + 1;
    const bool anc_here = !causal && (int64_t)n_rows * a.anc_words <= TILE_ANC;
    if (anc_here) {
      const uint64_t* from = a.anc + (size_t)(s.row0 + row_lo) * a.anc_words;
      const int words = n_rows * a.anc_words;
      for (int i = opaque(tid); i < words; i += 4 * 64 * TILE_WAVES) {                       // (four on their way)
        uint64_t w[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) w[x] = from[min(i + x * 64 * TILE_WAVES, words - 1)];
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (i + x * 64 * TILE_WAVES < words) anc_lds[i + x * 64 * TILE_WAVES] = w[x];
      }
    }
    auto window_of = [&](int c, int c_lo) {
      const int row = opaque(r[c]);               // (of a dead column: the first)
      if (causal) return attn_low_bits(row + 1 - c_lo);
      if (anc_here) {
        const uint64_t* w = anc_lds + max(row - row_lo, 0) * a.anc_words;
        return attn_tree_window([&](int i) { return i < a.anc_words ? w[i] : 0ull; }, c_lo, s.rows);
      }
      const uint64_t* w = a.anc + (size_t)(s.row0 + row) * a.anc_words;
      return attn_tree_window([&](int i) { return i < a.anc_words ? w[i] : 0ull; }, c_lo, s.rows);
    };

    const int last_block = (min(keys, t1 * TILE_TK) - 1) >> 5;
    bool any_bad = false;
    // some key of the piece may be hidden from some column (from a single row only by its own bit)
    const bool hides = (int64_t)t1 * TILE_TK > s.len && (s.rows > 1 || !causal);

    frag_t qf[NT][NS];
    f32x16_t o[NT][DB];
    ColumnTile<T, HD> tile[NT];
    // Once; and where the outputs hold infinities or NaN that may come from values which some columns do not see (0 times them), again with
    // these taken out of the tiles (safe), and infinities added where they are seen.
    for (int safe = 0;; ++safe) {
      int n = 2 * t0 + (wave & 1), pg = min(n, last_block) / blocks, in = min(n, last_block) - pg * blocks;
      int page = table[pg];
      // where this wave's part of the tile after the last that was asked for lies, and on to the next one
      auto source = [&]() {
        const int p = (unsigned)page < (unsigned)kv.n_pages ? page : 0;
        return my_pool + ((size_t)(p * kv.hkv + kvh) * blocks + in) * R::BLOCK;
      };
      auto advance = [&]() {
        n += 2;
        const int on = n <= last_block ? 2 : n - 1 == last_block ? 1 : 0;     // (a block behind the last that is needed is that one)
        if (on) {
          in += on;
          while (in >= blocks) { in -= blocks; ++pg; }
          page = table[pg];
        }
      };
      auto stage_of = [&](int i) { return my_lds + (uint32_t)(i % R::STAGES) * R::STAGE; };
      auto issue = [&](int i) {                   // tile t0 + i; called for i = 0, 1, 2, ...
        load_pieces<0, R::LPW>(source(), (uint32_t)lane * 16, stage_of(i));
        advance();
      };
      // The last tile of the sequence: V of keys past its end as zeros (memory there may hold anything), and so V of blocks whose page is not
      // there (page 0 stands in for it).  Safe: infinities and NaN out of all tiles with rows of the chunk.
      const int odd_from = s.len / TILE_TK - t0;
      int clean_from = 0;                         // (set when it is known whether all pages are there)
      auto clean = [&](int i) {
        if (i < clean_from) return;
        const int left = total - (t0 + i) * TILE_TK;
        const bool odd = safe && i >= odd_from;
        auto left_of = [&](int b) {               // keys of block b of the tile that are there
          if (any_bad && (unsigned)table[min(2 * (t0 + i) + b, last_block) / blocks] >= (unsigned)kv.n_pages) return 0;
          return left - 32 * b;
        };
        const int left0 = left_of(0), left1 = left_of(1);
        unsigned char* v = lds + (i % R::STAGES) * R::STAGE + 2 * R::BLOCK;
        constexpr int PIECE = 8 * sizeof(T), IN = R::BLOCK / PIECE;
        for (int x = opaque(tid); x < 2 * IN; x += 64 * TILE_WAVES) {          // piece x: block, fragment (db, u), lane
          const int in_block = x % IN, u = (in_block >> 6) & 1;
          frag_t f = *reinterpret_cast<const frag_t*>(v + x * PIECE);
          const int here = x >= IN ? left1 : left0;
          if (here < 32) f = attn_zero_tail(f, u, in_block & 63, here);
          if (odd) attn_take_odd(f);
          *reinterpret_cast<frag_t*>(v + x * PIECE) = f;
        }
        __syncthreads();
      };
      issue(0);
      // The queries between the first tile's loads and the others': the compiler's wait for them, held here by the empty statement, covers
      // the first tile too, and no load that the compiler knows of is in flight in the loop (its wait would drain the ring).
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        const T* qp = (const T*)a.q + (int64_t)(s.row0 + r[c]) * a.q_stride + (kvh * G + (live[c] ? col[c] % G : 0)) * HD + 8 * lg;
#pragma unroll
        for (int i = 0; i < NS; ++i) qf[c][i] = load_query(qp + 16 * i, vec_q);
      }
      // are all pages there?  (Where one is not, its keys are looked at one block after the other.)
      bool bad = false;
      for (int p = 2 * t0 / blocks + opaque(tid); p <= last_block / blocks; p += 64 * TILE_WAVES)
        bad |= (unsigned)kv.table[(size_t)seq * kv.stride + p] >= (unsigned)kv.n_pages;
#pragma unroll
      for (int c = 0; c < NT; ++c) {
#pragma unroll
        for (int i = 0; i < NS; ++i) asm volatile("" : "+a"(qf[c][i])::"memory");
#pragma unroll
        for (int i = 0; i < DB; ++i) {
#pragma unroll
          for (int v = 0; v < 16; ++v) o[c][i][v] = 0.f;
          asm volatile("" : "+a"(o[c][i]));
        }
        tile[c].start();
      }
      for (int i = 1; i < R::AHEAD; ++i)
        if (i < nt) issue(i);
      // tile 0 is here for everybody (this wave's loads retire in order, the barrier covers the others')
      wait_tiles_but<R::LPW>(min(R::AHEAD - 1, nt - 1));
      any_bad = any_thread<TILE_WAVES>(bad, said[0]);                          // (with its barrier)
      clean_from = any_bad ? 0 : (safe ? s.len : total) / TILE_TK - t0;
      clean(0);
      // Tile i + 1 is here, and all are done with tile i (with two column tiles: i - 1), whose stage takes the next that is asked for.
      auto next_tile = [&](int i) {
        if (i + 1 >= nt) return;
        wait_tiles_but<R::LPW>(min(R::AHEAD - 2, nt - 2 - i));
        __syncthreads();
        if (NT == 1 && i + R::AHEAD < nt) issue(i + R::AHEAD);
        clean(i + 1);
      };
      const unsigned char* frag = lds + lane * 8 * sizeof(T);
      // units from hide_at[c] on hold keys that some column of tile c does not see
      int hide_at[NT];
#pragma unroll
      for (int c = 0; c < NT; ++c)
        hide_at[c] = any_bad ? 0 : max(0, ((s.len - 32 - t0 * TILE_TK + (causal ? r_lo[c] + 1 : 0)) >> 5) + 1);
      auto seen_of = [&](int c, int u) -> unsigned {                          // bits of this lane's keys of unit u
        const int key0 = t0 * TILE_TK + 32 * u;
        if (any_bad && (key0 >= keys || (unsigned)table[(key0 >> 5) / blocks] >= (unsigned)kv.n_pages)) return 0u;
        return window_of(c, key0 - s.len) >> (opaque(lane) >> 5 << 2);
      };

      auto two_tiles = [&]() {
        if constexpr (NT == 2) {
          bf16x8_t kf[NS], vf[NS];                // V: fragment (db, u) at 2 db + u
          auto read = [&](bf16x8_t (&f)[NS], const unsigned char* at, int j) { f[j] = *reinterpret_cast<const bf16x8_t*>(at + j * 1024); };
#pragma unroll
          for (int j = 0; j < NS; ++j) read(kf, frag, j);
#pragma unroll
          for (int c = 0; c < NT; ++c) {
            tile_zero(tile[c].sc);
#pragma unroll
            for (int j = 0; j < NS; ++j) tile[c].sc = attn_mma(kf[j], qf[c][j], tile[c].sc);
            if (hide_at[c] <= 0) tile[c].hide(seen_of(c, 0));
            float top = ATTN_UNSEEN;
#pragma unroll
            for (int e = 0; e < 8; ++e) tile[c].top_of(top, e);
            tile[c].follow(top, a.scale, slack, o[c]);
          }
#pragma unroll
          for (int e = -2; e < 16; ++e) tile[0].exp_step(e, a.scale);
          tile[1].exp_step(-2, a.scale);
          tile[1].exp_step(-1, a.scale);
#pragma unroll
          for (int j = 0; j < NS; ++j) read(kf, frag + R::BLOCK, j);
          const int hide0 = hide_at[0] - 1, hide1 = hide_at[1] - 1;
          uint32_t here = 0, then = R::STAGE;     // stages of this tile and the next
          // One unit.  Everything scalar that can wait is put between matrix instructions too: a wave that does 30 scalar instructions in a
          // row has let its matrix core run dry.  Behind the piece's last unit the scores are of what lies in LDS, and for nothing.
          float l0 = 0.f;
          auto unit = [&](auto odd_unit, int i) {
            constexpr bool ODD = decltype(odd_unit)::value;
            const int u = 2 * i + ODD;
            const unsigned char* v = frag + here + (2 + ODD) * R::BLOCK;
            f32x16_t next;
            float top = ATTN_UNSEEN;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < NS; ++j) {
              if (j < NS / 2) { read(vf, v, 2 * j); read(vf, v, 2 * j + 1); }         // (half a group ahead of their use)
              if (j == 0) tile_zero(next);
              next = attn_mma(kf[j], qf[0][j], next);
#pragma unroll
              for (int e = 0; e < EPI; ++e) tile[1].exp_step(j * EPI + e, a.scale);
              __builtin_amdgcn_sched_barrier(0);
            }
            tile[0].sc = next;
            if (u >= hide0) tile[0].hide(seen_of(0, u + 1));
            // (in the second unit of a tile the tile after next is asked for)
            const bool ask = ODD && i + R::AHEAD < nt;
            const unsigned char* src = nullptr;
            uint32_t dst = 0;
            tile_begin();
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < NS; ++j) {
              tile_out(o[0][j % DB], vf[2 * (j % DB) + j / DB], tile[0].p[j / DB]);
#pragma unroll
              for (int e = 0; e < EPI; ++e) tile[1].exp_step(8 + j * EPI + e, a.scale);
              if (ODD && j == 1) {
                src = source();
                dst = stage_of(i + R::AHEAD);
              }
              if (j >= NS / 2) {         // (the scores are there by now)
#pragma unroll
                for (int e = 0; e < 2 * EPI; ++e) tile[0].top_of(top, (j - NS / 2) * 2 * EPI + e);
              }
              __builtin_amdgcn_sched_barrier(0);
            }
            tile[0].follow(top, a.scale, slack, o[0]);
            l0 = tile[0].l;
            tile[0].exp_step(-2, a.scale);
            tile[0].exp_step(-1, a.scale);
            tile_zero(next);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < NS; ++j) {
              next = attn_mma(kf[j], qf[1][j], next);
              if (ODD && j % 2 == 0 && ask) {
                constexpr int Q = R::LPW / (NS / 2);
                if (j == 0) load_pieces<0, Q>(src, (uint32_t)lane * 16, dst);
                if (j == 2) load_pieces<Q, 2 * Q>(src, (uint32_t)lane * 16, dst);
                if (j == 4) load_pieces<2 * Q, 3 * Q>(src, (uint32_t)lane * 16, dst);
                if (j == 6) load_pieces<3 * Q, 4 * Q>(src, (uint32_t)lane * 16, dst);
              }
#pragma unroll
              for (int e = 0; e < EPI; ++e) tile[0].exp_step(j * EPI + e, a.scale);
              __builtin_amdgcn_sched_barrier(0);
            }
            tile[1].sc = next;
            if (u >= hide1) tile[1].hide(seen_of(1, u + 1));
            if constexpr (!ODD) next_tile(i);
            const unsigned char* k = frag + then + ODD * R::BLOCK;
            top = ATTN_UNSEEN;
            tile_begin();
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < NS; ++j) {
              tile_out(o[1][j % DB], vf[2 * (j % DB) + j / DB], tile[1].p[j / DB]);
              if (j < NS / 2) { read(kf, k, 2 * j); read(kf, k, 2 * j + 1); }
#pragma unroll
              for (int e = 0; e < EPI; ++e) tile[0].exp_step(8 + j * EPI + e, a.scale);
              if (ODD && j == NS / 2 && ask) advance();
              if (j >= NS / 2) {
#pragma unroll
                for (int e = 0; e < 2 * EPI; ++e) tile[1].top_of(top, (j - NS / 2) * 2 * EPI + e);
              }
              __builtin_amdgcn_sched_barrier(0);
            }
            tile[1].follow(top, a.scale, slack, o[1]);
            tile[1].exp_step(-2, a.scale);
            tile[1].exp_step(-1, a.scale);
          };
          for (int i = 0; i < nt; ++i) {
            unit(std::false_type{}, i);
            if (i + 1 == nt) tile[0].limit = tile[1].limit = INFINITY;        // (nothing moves the references any more)
            unit(std::true_type{}, i);
            here = then;
            then = (then + R::STAGE) & (R::BYTES - 1);
          }
          tile[0].l = l0;
        }
      };
      // one column tile: a unit's steps one after the other
      auto one_tile = [&](int u, const unsigned char* at) {
        const bool masked = u >= hide_at[0];
        if constexpr (NT == 1) {
          attn_unit<HD>(at, at + 2 * R::BLOCK, masked, masked ? seen_of(0, u) : ~0u, a.scale, qf[0], o[0], tile[0].m, tile[0].l);
        } else {
          bf16x8_t f[NS];
#pragma unroll
          for (int j = 0; j < NS; ++j) f[j] = *reinterpret_cast<const bf16x8_t*>(at + j * 1024);
          tile_zero(tile[0].sc);
#pragma unroll
          for (int j = 0; j < NS; ++j) tile[0].sc = attn_mma(f[j], qf[0][j], tile[0].sc);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int j = 0; j < NS; ++j) f[j] = *reinterpret_cast<const bf16x8_t*>(at + 2 * R::BLOCK + j * 1024);
          if (masked) tile[0].hide(seen_of(0, u));
          float top = ATTN_UNSEEN;
#pragma unroll
          for (int e = 0; e < 8; ++e) tile[0].top_of(top, e);
          tile[0].follow(top, a.scale, slack, o[0]);
#pragma unroll
          for (int e = -2; e < 16; ++e) tile[0].exp_step(e, a.scale);
          tile_begin();
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int j = 0; j < NS; ++j) tile_out(o[0][j % DB], f[2 * (j % DB) + j / DB], tile[0].p[j / DB]);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      if (bad) set_status(kv.status, ESP_DEV_BAD_PAGE);
      if (mine == 2) {
        two_tiles();
      } else {
        for (int i = 0; i < nt; ++i) {
          if (mine == 1)
            for (int kh = kh0; kh <= kh1; ++kh) one_tile(2 * i + kh, frag + (i % R::STAGES) * R::STAGE + kh * R::BLOCK);
          next_tile(i);
          if (NT == 2 && i + R::AHEAD < nt) issue(i + R::AHEAD);
        }
      }
#pragma unroll
      for (int c = 0; c < NT; ++c) tile_settle(o[c]);
      if (safe) {
        for (int u = 0; u < 2 * nt; ++u) {
          const int n = 2 * t0 + u, key0 = 32 * n;
          if ((key0 & ~(TILE_TK - 1)) + TILE_TK <= s.len || key0 >= keys || (halves && (u & 1) != kh0)) continue;
          const int p = table[n / blocks];
          if ((unsigned)p >= (unsigned)kv.n_pages) continue;
          const T* v = (const T*)kv.v + ((size_t)(p * kv.hkv + kvh) * blocks + n % blocks) * (32 * HD);
#pragma unroll
          for (int c = 0; c < NT; ++c)
            if (c < mine) attn_add_odd<T, HD>(v, window_of(c, key0 - s.len) >> (opaque(lane) >> 5 << 2), total - key0, opaque(lane), o[c]);
        }
        break;
      }
      if (!hides) break;
      float zero[4] = {0.f, 0.f, 0.f, 0.f};       // (0 x infinity is NaN, and that stays)
#pragma unroll
      for (int c = 0; c < NT; ++c)
        if (c < mine) {
#pragma unroll
          for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) zero[v & 3] = fmaf(o[c][i][v], 0.f, zero[v & 3]);
        }
      if (!any_thread<TILE_WAVES>(!((zero[0] + zero[1]) + (zero[2] + zero[3]) == 0.f), said[1])) break;
    }

    // the ring is done with: a wave's columns, [tile][32][HD], one wave's behind the other's
    __syncthreads();
    const int lane = opaque(threadIdx.x) & 63, lr = lane & 31, lg = lane >> 5;
    float* xo = reinterpret_cast<float*>(lds) + wave * (32 * NT * HD);
#pragma unroll
    for (int c = 0; c < NT; ++c) tile[c].l = attn_sum_of_halves(tile[c].l);
    if (halves) {                                 // the second half of the keys goes to the wave that has the first
      if (mine == 1 && kh0 == 1) {
        put_columns<HD>(xo, o[0], lane);
        if (lg == 0) { xm[wave][lr] = tile[0].m; xl[wave][lr] = tile[0].l; }
      }
      __syncthreads();
      if (mine == 1 && kh0 == 0) {
        const float mo = xm[wave + 2][lr], lo = xl[wave + 2][lr], top = fmaxf(tile[0].m, mo);
        const float fa = attn_weight(tile[0].m, top, a.scale), fb = attn_weight(mo, top, a.scale);
        tile[0].l = tile[0].l * fa + lo * fb;
        tile[0].m = top;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int v = 0; v < 16; v += 4) {
            const f32x4_t x = *reinterpret_cast<const f32x4_t*>(column_piece<HD>(xo + 2 * (32 * NT * HD), lr, db * 8 + 2 * (v >> 2) + lg));
#pragma unroll
            for (int e = 0; e < 4; ++e) o[0][db][v + e] = o[0][db][v + e] * fa + x[e] * fb;
          }
      }
    }
    const Partials part = partials_of(a.partials, plan.shares, 32 * plan.cap, HD);
#pragma unroll
    for (int c = 0; c < NT; ++c) {
      if (c >= mine || kh0 != 0) continue;
      const int tc = ct0 + 4 * c, c0 = col0 + tc * 32, n_live = min(32, ncols - c0);
      if (slot >= 0) {                            // a partial as the registers hold it: [four features][column][4]
        float* po = part.sums(slot) + tc * 32 * HD + (lg * 32 + lr) * 4;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int v = 0; v < 16; v += 4)
            *reinterpret_cast<f32x4_t*>(po + (db * 8 + 2 * (v >> 2)) * 128) = f32x4_t{o[c][db][v], o[c][db][v + 1], o[c][db][v + 2], o[c][db][v + 3]};
        if (lg == 0) {
          float* ml = part.stats(slot) + 2 * (tc * 32 + lr);
          ml[0] = tile[c].m * a.scale;
          ml[1] = tile[c].l;
        }
        continue;
      }
      const float inv = tile[c].l > 0.f ? 1.f / tile[c].l : 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[c][db][v] *= inv;
      put_columns<HD>(xo, o[c], lane);
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");       // (a wave's LDS accesses are done in order: for the compiler)
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll 4
      for (int t = lane; t < 32 * PIECES; t += 64) {
        const int i = t / PIECES, piece = t % PIECES, row = (c0 + i) / G;
        const f32x4_t x = *reinterpret_cast<const f32x4_t*>(column_piece<HD>(xo, i, piece));
        if (i < n_live) store4((T*)a.out + ((int64_t)(s.row0 + row) * a.hq + kvh * G + (c0 + i) - row * G) * HD + 4 * piece, x, vec_out);
      }
      xo += 32 * HD;
    }
    // the stores do not count as loads of the next piece, whose ring goes where the columns are
    wait_loads_but<0>();
    __syncthreads();
  });
}

// --------------------------------------------------------------------------------------------------
// The pieces of an item that begins in share w and does not end there: that one and those of the shares behind it, up to the one that ends
// it.  Four features of a column are a thread's, and where fewer than all threads have any, as many groups of them as there is room for take
// the pieces in turn: nearly all of it is waiting for memory, so all loads are to be on their way at once.  A workgroup has the 32 columns of
// a decoding item (64 pieces of 4 columns: 5.9 us) or 8 of a tile item's, whole lines (16 items of 16 pieces, 34 MB: 9.8 us).
template <bool STREAM> constexpr int MERGE_THREADS = STREAM ? 1024 : 256;
template <bool STREAM, int HD> constexpr int MERGE_COLUMNS = STREAM ? 32 : 4 * MERGE_THREADS<STREAM> / HD;
template <typename T, int HD, bool STREAM>
__global__ __launch_bounds__(MERGE_THREADS<STREAM>) void k_paged_merge(PagedAttnArgs a, int hkv, int shares, int cols, bool vec_out) {
  constexpr int NT = MERGE_THREADS<STREAM>, NC = MERGE_COLUMNS<STREAM, HD>, PIECES = HD / 4, U = 8;
  __shared__ int slots[2 * MOST_SHARES];
  __shared__ __align__(16) f32x4_t part[NT];
  __shared__ float part_m[NT], part_l[NT];
  // The items that began in shares are often a multiple of 8 shares apart: a tile item's workgroups go to all XCDs, decoding items' are spread
  // over the XCDs as the shares are.  (All on one XCD: 43 us for 9.8.)
  const int of_share = cols / NC, w = STREAM ? share_at(blockIdx.x, shares) : blockIdx.x / of_share;
  const int c0 = STREAM ? 0 : blockIdx.x % of_share * NC, tid = threadIdx.x, lane = tid & 63;
  if (w >= shares) return;
  const Partials p = partials_of(a.partials, shares, cols, HD);
  const ShareNote note = p.notes[w];
  int first = w + 1 + lane < shares ? p.notes[w + 1 + lane].first : ENDS;
  if (note.columns <= c0) return;
  // the pieces' slots, in order, by every wave alike
  int n = 1;
  if (tid == 0) slots[0] = 2 * w + 1;
  for (int x0 = w + 1;; x0 += 64) {
    if (x0 > w + 1) first = x0 + lane < shares ? p.notes[x0 + lane].first : ENDS;
    const uint64_t ends = __builtin_amdgcn_ballot_w64((first & ENDS) != 0);
    const uint64_t upto = ends ? (2ull << __builtin_ctzll(ends)) - 1ull : ~0ull;
    const uint64_t has = __builtin_amdgcn_ballot_w64((first & HAS) != 0) & upto;
    if (has >> lane & 1) slots[n + __popcll(has & ((1ull << lane) - 1ull))] = 2 * (x0 + lane);
    n += __popcll(has);
    if (ends) break;
  }
  __syncthreads();
  const int G = a.hq / hkv, live = min(NC, note.columns - c0), work = live * PIECES, groups = min(NT / work, n);
  const int g = tid / work, t = tid - g * work, c = c0 + (STREAM ? t / PIECES : t % live), piece = STREAM ? t % PIECES : t / live;
  // where these four features of a slot are: [column][HD], or of a tile of 32 columns [four features][column][4]
  const int in_slot = STREAM ? c * HD + 4 * piece : (c & ~31) * HD + (piece * 32 + (c & 31)) * 4;
  float top = -INFINITY, lt = 0.f;
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](float m, float l, f32x4_t o) {
    const float now = l > 0.f ? fmaxf(top, m) : top;
    const float fa = top > -INFINITY ? __builtin_amdgcn_exp2f(top - now) : 0.f, fb = l > 0.f ? __builtin_amdgcn_exp2f(m - now) : 0.f;
    lt = lt * fa + l * fb;
    acc = acc * fa + o * fb;
    top = now;
  };
  if (g < groups)
    for (int i = g; i < n; i += U * groups) {
      float m[U], l[U];
      f32x4_t o[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int slot = slots[min(i + u * groups, n - 1)];
        m[u] = p.stats(slot)[2 * c];
        l[u] = p.stats(slot)[2 * c + 1];
        o[u] = *reinterpret_cast<const f32x4_t*>(p.sums(slot) + in_slot);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u * groups < n) add(m[u], l[u], o[u]);
    }
  if (groups > 1) {
    part[tid] = acc;
    part_m[tid] = top;
    part_l[tid] = lt;
    __syncthreads();
    if (g == 0)
      for (int x = 1; x < groups; ++x) add(part_m[x * work + t], part_l[x * work + t], part[x * work + t]);
  }
  if (g > 0) return;
  const int cc = note.col0 + c;
  const int64_t out = ((int64_t)note.row0 + cc / G) * a.hq + note.kvh * G + cc % G;
  store4((T*)a.out + out * HD + 4 * piece, acc * (lt > 0.f ? 1.f / lt : 0.f), vec_out);
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
  const dim3 g((unsigned)paged_attn_workgroups(p, kv.batch, kv.hkv));
  if (p.cap == 1) {
    hipLaunchKernelGGL((k_paged_stream<T, HD>), g, dim3(64 * STREAM_WAVES), 0, st, kv, ch, a, p, vec_q, vec_out);
    if (p.shares)
      hipLaunchKernelGGL((k_paged_merge<T, HD, true>), dim3((p.shares + 7) & ~7), dim3(MERGE_THREADS<true>), 0, st, a, kv.hkv, p.shares, 32, vec_out);
  } else {
    constexpr unsigned bytes = TileRing<T, HD>::BYTES + TILE_ANC * 8;
    const hipError_t e = allow_lds<T, HD>(bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_paged_tile<T, HD>), g, dim3(64 * TILE_WAVES), bytes, st, kv, ch, a, p, vec_q, vec_out);
    if (p.shares)
      hipLaunchKernelGGL((k_paged_merge<T, HD, false>), dim3(p.shares * (32 * p.cap / MERGE_COLUMNS<false, HD>)),
                         dim3(MERGE_THREADS<false>), 0, st, a, kv.hkv, p.shares, 32 * p.cap, vec_out);
  }
  return hipGetLastError();
}

}  // namespace

// Which kernel, and how many shares.  The times are of bf16 with 32/8 heads of 128, in us, and fit what was measured from 1 to 32 sequences.
// Stream or tile kernel: the stream kernel begins and ends sooner (7 against 13) and has the work in pieces of 32 columns for every place, but
// reads every key again for each 32 columns, at best from its XCD's 4 MB of L2.  128 rows over 2048 / 8000 keys: 19 / 42 against 28 / 43;
// 320 rows over 2048 / 8000: 31 / 78 against 39 / 70; 2048 rows from none: 64 against 72; 2000 in fp32: 332 against 299; 4 x 100 rows over
// 4000, whose keys are too much for L2: 85 against 58; 32 x 40 over 1000: 115 against 48.  Two column tiles each of more pairs than CUs: 64 x 16
// rows over 200 / 500 / 1000 / 2000: 28 / 48 / 88 / 190 against 35 / 46 / 63 / 122; of fewer, 16 x 16 over 2000: 26 against 30.
// Stream kernel, shares or an item a workgroup: an item alone takes 7 and 0.57 for 128 keys (64 KB: a CU takes in 110 GB/s, and more waves on
// an item do not change that); shares with their merge 13.5 and what K and V take.  One row over 1000 / 4000 keys: 11.2 / 25.7 alone,
// 12.9 / 17.5 in shares; 32 sequences of 2000 / 4000: 45 / 97, 53 / 105 (but alone a batch takes as long as its longest sequence, so a longer
// one is shared out).
// Tile kernel: 2 for 64 keys, 13 for an item's beginning and end, 8 for the merge and 1/20 for a partial.  (These are taken for heads of 64 and
// for fp32 too, whose key tiles take half as long and, by their operations, 3.5 times.)  With as many items as places, one sequence's go to the places by weight: 4096 rows from none 150 against 190 in shares.  So do a batch's if they are short; else they are
// shared out, since nothing is known here of how their lengths differ (8 chunks of 189 to 512 rows over up to 8192 keys: 215 against 361;
// 8 x 512 rows over 4096 each: 308 against 296).
PagedAttnPlan paged_attn_plan(int dtype, int hd, int batch, int hq, int hkv, int total_rows, int max_rows, int len_bound) {
  PagedAttnPlan p;
  const int G = hq / hkv;
  const int64_t cols = (int64_t)max_rows * G, keys = (int64_t)len_bound + max_rows, tiles = std::max<int64_t>(1, ceil_div(cols, 32));
  // items that there can be with a cap
  auto items = [&](int cap) {
    return (int64_t)hkv * std::min<int64_t>((int64_t)batch * ceil_div(tiles, cap), ceil_div((int64_t)total_rows * G, 32 * cap) + batch);
  };
  const int64_t kv_bytes = ceil_div((int64_t)batch * hkv, 8) * keys * hd * (dtype == ESP_F32 ? 8 : 4);     // of an XCD's sequences and heads
  const int64_t work = items(1) * (len_bound + max_rows / 2) * hd * (dtype == ESP_F32 ? 4 : 2);
  const bool small = work <= (int64_t)1 << 29 && (kv_bytes <= 5 << 20 || (tiles <= 2 && (items(1) <= 256 || keys <= 700)));
  p.cap = tiles == 1 || small ? 1 : dtype == ESP_F32 ? TILE_CAP<float> : TILE_CAP<bf16_t>;
  while (p.cap > 2 && p.cap / 2 >= tiles && items(p.cap) < 256) p.cap /= 2;
  const int64_t n = items(p.cap), key_tiles = ceil_div(keys, p.cap == 1 ? STREAM_TK : TILE_TK);
  p.q_tiles = (int)ceil_div(tiles, p.cap);
  if (p.cap == 1) {
    const int64_t places = dtype == ESP_F32 && hd == 128 ? 256 : 512;        // workgroups that have a place at once
    const double tile_us = dtype == ESP_F32 ? 3.5 * hd / 128 : 0.17 + 0.4 * hd / 128;
    p.least = 2;
    if (n < 4 * places && tile_us * key_tiles > 6.5 + 0.09 * std::min<int64_t>(n, 64)) {
      p.shares = (int)std::min(places, ceil_div(n * key_tiles, p.least));
      if (batch == 1 && p.shares > n) p.shares = (int)(p.shares / n * n);    // (whole items come out: 17 us with two more shares, 14 without)
    }
  } else if (n < (batch == 1 || key_tiles <= 20 ? 256 : 4 * 256)) {
    const double alone = 2. * key_tiles + 13., parts = std::min(sqrt(40. * key_tiles / n), 256. / n);
    p.least = 4;
    if (batch > 1 && key_tiles > 20) p.shares = (int)std::min(256., std::max(n * parts, (double)n));
    else if (parts >= 2. && 2. * key_tiles / parts + 0.05 * n * parts + 21. < alone) p.shares = (int)(n * std::floor(parts));
  }
  return p;
}
int64_t paged_attn_workgroups(const PagedAttnPlan& p, int batch, int hkv) {
  if (p.shares) return (p.shares + 7) / 8 * 8;
  const int64_t groups = (int64_t)batch * hkv;
  return (p.q_tiles > 1 && groups >= 8 ? (groups + 7) & ~7ll : groups) * p.q_tiles;
}
size_t paged_attn_partial_floats(const PagedAttnPlan& p, int hd) {
  return p.shares ? notes_floats(p.shares) + 2 * p.shares * slot_floats(32 * p.cap, hd) : 0;
}

hipError_t launch_paged_attn(hipStream_t st, int dtype, int hd, const PagedDev& kv, const ChunkDev& ch, const PagedAttnArgs& a,
                             const PagedAttnPlan& p) {
  PagedAttnArgs x = a;
  x.scale = a.scale * LOG2E;
  if (dtype == ESP_F32) return hd == 64 ? launch<float, 64>(st, kv, ch, x, p) : launch<float, 128>(st, kv, ch, x, p);
  return hd == 64 ? launch<bf16_t, 64>(st, kv, ch, x, p) : launch<bf16_t, 128>(st, kv, ch, x, p);
}
