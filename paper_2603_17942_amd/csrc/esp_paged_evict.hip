// Bounded caches (esp_paged_evict): of a sequence with more than `keep` tokens the first, the last and those of most weight stay, by the weights of
// each layer and kv head, and move up in their order.
//
// k_evict_choose, a workgroup a layer, sequence and kv head: the weight at which the cut lies by counting keys (the weight's bits in unsigned order) in
// three steps of 12, 12 and 8 bits; a thread then has a run of consecutive slots, and one sum over the threads before it says where its kept
// ones go and how many of those at the cut are in.  Integers alone: the same list every time.
// k_evict_move: the list's tokens go to slots 0, 1, ...; a token never moves back, so a plane's blocks of 32 new slots are filled one after the other and what
// is still to be read lies behind what is written, also where old and new pages are the same.
//
// The move is bound by memory: a token's K lies in 16-byte pieces (32 tokens of eight features side by side) and its V in single elements, so where half of
// a block stays all of its lines are read.  4096 to 2048 tokens of 32 layers and 8 kv heads, bf16, 128: 540 MB read and 268 written in 172 us, 4.7 TB/s (a copy:
// 5.1); 16 ragged sequences 1094 and 534 in 336.  Choosing is a chain of some 20 barriers, 20 to 26 us.
#include "esp_paged.h"
#include "esp_scan.h"

namespace {

constexpr int CHOOSERS = 512, DIGIT_BINS = 4096, EACH = DIGIT_BINS / CHOOSERS;

// larger weights have larger keys; NaN has the least of all
__device__ __forceinline__ unsigned weight_key(float x) {
  const unsigned b = __float_as_uint(x + 0.f);
  return x != x ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
}

__global__ __launch_bounds__(CHOOSERS) void k_evict_choose(PagedDev kv, EvictArgs a) {
  __shared__ unsigned bins[DIGIT_BINS];
  __shared__ WaveSums<CHOOSERS / 64> sums;
  __shared__ unsigned found[2];
  int turn = 0;
  const int tid = threadIdx.x, kvh = blockIdx.x, seq = blockIdx.y, layer = blockIdx.z;
  const int64_t head = ((int64_t)layer * kv.batch + seq) * kv.hkv + kvh;
  const float* mass = a.mass + head * a.slots;
  float* mass_out = a.mass_out + head * a.out_slots;
  int32_t* kept = a.kept + head * a.keep;
  const int len = kv.len[seq];
  const bool ok = len >= 0 && len <= kv.len_bound && (int64_t)len <= (int64_t)kv.stride * kv.page_size && len <= a.slots;
  if (!ok || len <= a.keep) {
    if (!ok && tid == 0 && kvh == 0 && layer == 0) set_status(kv.status, ESP_DEV_LEN_OVER_BOUND);
    for (int i = tid; i < a.keep; i += CHOOSERS) {
      const bool there = ok && i < len;
      kept[i] = there ? i : -1;
      if (there && mass != mass_out) mass_out[i] = mass[i];
    }
    return;
  }
  // how many between the first and the last ones stay, and the key of the last of these in the order
  const int lo = a.first, hi = len - a.recent;
  unsigned want = (unsigned)(a.keep - a.first - a.recent), cut = 0;
  if (want > 0) {
    int shift = 20, bits = 12;
    for (int step = 0; step < 3; ++step) {
      for (int i = tid; i < DIGIT_BINS; i += CHOOSERS) bins[i] = 0;
      __syncthreads();
      for (int i = lo + tid; i < hi; i += CHOOSERS) {
        const unsigned k = weight_key(mass[i]);
        if (step == 0 || (k >> (shift + bits)) == (cut >> (shift + bits))) atomicAdd(&bins[(k >> shift) & ((1u << bits) - 1u)], 1u);
      }
      __syncthreads();
      // thread t has EACH bins, from the largest down
      unsigned n[EACH], at = 0;
#pragma unroll
      for (int i = 0; i < EACH; ++i) { n[i] = bins[DIGIT_BINS - 1 - (EACH * tid + i)]; at += n[i]; }
      before(sums, turn, at);
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        if (at < want && want <= at + n[i]) { found[0] = DIGIT_BINS - 1 - (EACH * tid + i); found[1] = at; }
        at += n[i];
      }
      __syncthreads();
      cut |= found[0] << shift;
      want -= found[1];
      bits = step == 0 ? 12 : 8;
      shift = step == 0 ? 8 : 0;
      __syncthreads();
    }
  }
  // `want` of those at the cut are in
  const int run = (len + CHOOSERS - 1) / CHOOSERS, begin = min(tid * run, len), end = min(begin + run, len);
  const bool none = a.keep == a.first + a.recent;
  unsigned certain = 0, equal = 0;     // in, and at the cut
  for (int i = begin; i < end; ++i) {
    if (i < lo || i >= hi) { ++certain; continue; }
    if (none) continue;
    const unsigned k = weight_key(mass[i]);
    certain += k > cut;
    equal += k == cut;
  }
  before(sums, turn, certain);
  before(sums, turn, equal);
  unsigned ties = equal, place = certain + min(equal, want);
  for (int i = begin; i < end; ++i) {
    bool in = i < lo || i >= hi;
    if (!in && !none) {
      const unsigned k = weight_key(mass[i]);
      in = k > cut || (k == cut && ties++ < want);
    }
    if (in) kept[place++] = i;
  }
  __syncthreads();
  for (int i0 = 0; i0 < a.keep; i0 += CHOOSERS) {      // (a token's weight moves down: what is read later lies behind)
    const int i = i0 + tid;
    const float w = i < a.keep ? mass[kept[i]] : 0.f;
    __syncthreads();
    if (i < a.keep) mass_out[i] = w;
    __syncthreads();
  }
}

// Tokens in batches of 64 (two blocks), a thread HD / 64 pieces of eight elements of K and of V each.  The next batch is on its way while one is written, and
// where a token of the one after lies is looked up meanwhile.  A piece of V has eight tokens' elements of one feature: eight loads whose lanes have
// neighbouring features, 16 bytes (of the type's size, eight elements) apart, so a wave's loads of a block come from lines that they share.
constexpr int MOVERS = 512, BATCH = 64;
// an empty statement that takes a value, which therefore has arrived
template <typename V> __device__ __forceinline__ void wait_for(const V& v) {
  typedef __attribute__((ext_vector_type(sizeof(V) / 4))) uint32_t words;
  const words w = __builtin_bit_cast(words, v);
#pragma unroll
  for (int i = 0; i < (int)sizeof(V) / 4; ++i) { const uint32_t x = w[i]; asm volatile("" ::"v"(x)); }
}
template <typename T> struct Raw { typedef uint32_t type; };
template <> struct Raw<bf16_t> { typedef uint16_t type; };
struct Source { int64_t at; int key; };                // first element of the block (-1: outside the pool), place in it

template <typename T, int HD>
__global__ __launch_bounds__(MOVERS) void k_evict_move(PagedDev kv, EvictArgs a) {
  typedef __attribute__((ext_vector_type(8))) T vec;
  typedef typename Raw<T>::type raw;                   // (loads into halves of a register would wait for one another)
  constexpr int PIECES = HD / 64;                      // of K, and of V
  __shared__ Source src[4][BATCH];                     // of the batch that is written, the one on its way, the one after, and one that others may still read
  __shared__ int64_t dst[4][2];                        // of the batch's blocks; -1: not to be written
  __shared__ int bad[4];                               // tokens of it lie outside the pool
  __shared__ int counted[MOVERS / 64];
  const int tid = threadIdx.x, kvh = blockIdx.x, seq = blockIdx.y, layer = blockIdx.z;
  const int32_t* kept = a.kept + (((int64_t)layer * kv.batch + seq) * kv.hkv + kvh) * a.keep;
  const size_t of_layer = (size_t)layer * kv.n_pages * kv.hkv * kv.page_size * HD;
  T* kp = (T*)kv.k + of_layer;
  T* vp = (T*)kv.v + of_layer;
  const int32_t* table = kv.table + (size_t)seq * kv.stride;
  const int32_t* table_out = a.table_out + (size_t)seq * a.out_stride;

  int n = 0;
  for (int i = tid; i < a.keep; i += MOVERS) n += kept[i] >= 0;
  n = (int)wave_total((unsigned)n);
  if ((tid & 63) == 0) counted[tid >> 6] = n;
  __syncthreads();
  n = 0;
#pragma unroll
  for (int w = 0; w < MOVERS / 64; ++w) n += counted[w];
  // (of the workgroups here only this one looks at the length, so len_out may be where it came from)
  if (tid == 0 && kvh == 0 && layer == 0) a.len_out[seq] = n > 0 ? n : kv.len[seq];
  if (n == 0 || (a.table_out == kv.table && kept[n - 1] == n - 1)) return;       // (all where they are)

  auto block_at = [&](int page, int slot_in_page) {
    return page < 0 || page >= kv.n_pages ? (int64_t)-1
                                          : (int64_t)(page_plane(page, kvh, kv.hkv, kv.page_size, HD) + (size_t)(slot_in_page >> 5) * 32 * HD);
  };
  // lane l < 64: old slot of token l of a batch; its page; and so on one step later each
  auto old_slot = [&](int batch) {
    const int i = batch * BATCH + tid;
    return tid < BATCH && i < n ? kept[i] : -1;
  };
  auto page_of = [&](int slot) { return slot >= 0 ? table[slot / kv.page_size] : 0; };
  auto put = [&](int batch, int slot, int page) {
    if (tid >= BATCH) return;
    const int buf = batch & 3;
    int64_t at = -1;
    if (slot >= 0) {
      at = block_at(page, slot % kv.page_size);
      if (at < 0) set_status(kv.status, ESP_DEV_BAD_PAGE);
    }
    src[buf][tid] = {at, slot & 31};
    const bool outside = __builtin_amdgcn_ballot_w64(slot >= 0 && at < 0) != 0ull;
    if (tid == 0) bad[buf] = outside;
    if ((tid & 31) == 0) {
      const int first = batch * BATCH + tid, last = min(first + 31, n - 1);
      int64_t to = -1;
      if (first < n) {
        const int new_page = table_out[first / kv.page_size];
        to = block_at(new_page, first % kv.page_size);
        if (to < 0) set_status(kv.status, ESP_DEV_BAD_PAGE);
        else if (kept[last] == last && table[first / kv.page_size] == new_page) to = -1;       // (all where they are)
      }
      dst[buf][tid >> 5] = to;
    }
  };
  // K: piece p of a block is features 8 (p / 32) .. of token p % 32.  V: feature 32 (p / 128) + p % 32, tokens 16 (p / 64 % 2) + 4 (p / 32 % 2) + 0..3 and 8 more.
  // (what is not there is read at the pool's beginning)
  auto fetch = [&](int batch, vec (&k)[PIECES], raw (&v)[PIECES][8]) {
    const int buf = batch & 3;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int piece = i * MOVERS + tid, block = piece / (4 * HD), p = piece % (4 * HD);
      const Source s = src[buf][32 * block + p % 32];
      k[i] = *reinterpret_cast<const vec*>(kp + max(s.at, (int64_t)0) + (p / 32 * 32 + s.key) * 8);
      const int d = 32 * (p / 128) + p % 32, first = 16 * (p / 64 % 2) + 4 * (p / 32 % 2);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const Source t = src[buf][32 * block + first + 8 * (e >> 2) + (e & 3)];
        v[i][e] = reinterpret_cast<const raw*>(vp)[max(t.at, (int64_t)0) + v_off(t.key, d, HD)];
      }
    }
  };
  auto store = [&](int batch, const vec (&k)[PIECES], const vec (&v)[PIECES]) {
    const int buf = batch & 3;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int piece = i * MOVERS + tid, block = piece / (4 * HD), p = piece % (4 * HD);
      const int64_t to = dst[buf][block];
      if (to < 0) continue;
      const int left = n - batch * BATCH - 32 * block, first = 16 * (p / 64 % 2) + 4 * (p / 32 % 2);
      if (p % 32 < left) *reinterpret_cast<vec*>(kp + to + p * 8) = k[i];
      if (first + 11 < left) {
        *reinterpret_cast<vec*>(vp + to + p * 8) = v[i];
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (first + 8 * (e >> 2) + (e & 3) < left) vp[to + p * 8 + e] = v[i][e];
      }
    }
  };

  const int batches = (n + BATCH - 1) / BATCH;
  put(0, old_slot(0), page_of(old_slot(0)));
  put(1, old_slot(1), page_of(old_slot(1)));
  int slot2 = old_slot(2), page2 = page_of(slot2), slot3 = old_slot(3);
  vec k[PIECES], v[PIECES], next_k[PIECES];
  raw next_v[PIECES][8];
  __syncthreads();
  fetch(0, next_k, next_v);
  for (int b = 0; b < batches; ++b) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      k[i] = next_k[i];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = __builtin_bit_cast(T, next_v[i][e]);
    }
    if (bad[b & 3]) {                  // zeros in their place
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int piece = i * MOVERS + tid, block = piece / (4 * HD), p = piece % (4 * HD), first = 16 * (p / 64 % 2) + 4 * (p / 32 % 2);
        if (src[b & 3][32 * block + p % 32].at < 0) k[i] = vec{};
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (src[b & 3][32 * block + first + 8 * (e >> 2) + (e & 3)].at < 0) v[i][e] = from_f32<T>(0.f);
      }
    }
    if (b + 1 < batches) fetch(b + 1, next_k, next_v);
    put(b + 2, slot2, page2);
    slot2 = slot3;
    page2 = page_of(slot2);
    slot3 = old_slot(b + 4);
    // what anybody reads of this batch has arrived (k and v are made of it) before anything of it is written
#pragma unroll
    for (int i = 0; i < PIECES; ++i) { wait_for(k[i]); wait_for(v[i]); }
    __syncthreads();
    store(b, k, v);
  }
}

template <typename T, int HD>
void move(hipStream_t st, const PagedDev& kv, const EvictArgs& a) {
  hipLaunchKernelGGL((k_evict_move<T, HD>), dim3(kv.hkv, kv.batch, a.layers), dim3(MOVERS), 0, st, kv, a);
}

}  // namespace

hipError_t launch_paged_evict(hipStream_t st, int dtype, int hd, const PagedDev& kv, const EvictArgs& a) {
  hipLaunchKernelGGL(k_evict_choose, dim3(kv.hkv, kv.batch, a.layers), dim3(CHOOSERS), 0, st, kv, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (dtype == ESP_BF16) hd == 128 ? move<bf16_t, 128>(st, kv, a) : move<bf16_t, 64>(st, kv, a);
  else hd == 128 ? move<float, 128>(st, kv, a) : move<float, 64>(st, kv, a);
  return hipGetLastError();
}
