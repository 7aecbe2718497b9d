// Bounded caches (esp_paged_evict): of a sequence with more than `keep` tokens the first, the last and those of most weight stay, by the weights of
// each layer and kv head, and move up in their order.
//
// k_evict_choose, a workgroup a layer, sequence and kv head: the weight at which the cut lies by counting keys (the weight's bits in unsigned order) in
// three steps of 12, 12 and 8 bits; a thread then has a run of consecutive slots, and one sum over the threads before it says where its kept
// ones go and how many of those at the cut are in.  Integers alone: the same list every time.
// k_evict_move: the list's tokens go to slots 0, 1, ...; a token never moves back, so a plane's blocks of 32 new slots are filled one after the other and what
// is still to be read lies behind what is written, also where old and new pages are the same.
#include "esp_paged.h"

namespace {

constexpr int CHOOSERS = 1024, DIGIT_BINS = 4096;

// larger weights have larger keys; NaN has the least of all
__device__ __forceinline__ unsigned weight_key(float x) {
  const unsigned b = __float_as_uint(x + 0.f);
  return x != x ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
}

// sums over the threads before this one, and of all
__device__ __forceinline__ uint2 sums_before(uint2 v, uint2& all, uint2* of_wave) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint2 at = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned x = __shfl_up(at.x, o, 64), y = __shfl_up(at.y, o, 64);
    if (lane >= o) { at.x += x; at.y += y; }
  }
  __syncthreads();
  if (lane == 63) of_wave[wave] = at;
  __syncthreads();
  all = {0, 0};
  uint2 r = {at.x - v.x, at.y - v.y};
  for (int w = 0; w < CHOOSERS / 64; ++w) {
    const uint2 t = of_wave[w];
    if (w < wave) { r.x += t.x; r.y += t.y; }
    all.x += t.x; all.y += t.y;
  }
  return r;
}

__global__ __launch_bounds__(CHOOSERS) void k_evict_choose(PagedDev kv, EvictArgs a) {
  __shared__ unsigned bins[DIGIT_BINS];
  __shared__ uint2 of_wave[CHOOSERS / 64];
  __shared__ unsigned found[2];
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
      // thread t has the bins 4 t .. from the largest down
      unsigned n[4], mine = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) { n[i] = bins[DIGIT_BINS - 1 - (4 * tid + i)]; mine += n[i]; }
      uint2 all;
      unsigned at = sums_before({mine, 0}, all, of_wave).x;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (at < want && want <= at + n[i]) { found[0] = DIGIT_BINS - 1 - (4 * tid + i); found[1] = at; }
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
  uint2 mine = {0, 0};                 // in for certain, at the cut
  for (int i = begin; i < end; ++i) {
    if (i < lo || i >= hi) { ++mine.x; continue; }
    const unsigned k = weight_key(mass[i]);
    if (none) continue;
    mine.x += k > cut;
    mine.y += k == cut;
  }
  uint2 all;
  const uint2 before = sums_before(mine, all, of_wave);
  unsigned ties = before.y, place = before.x + min(before.y, want);
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

template <typename T, int HD>
__global__ __launch_bounds__(256) void k_evict_move(PagedDev kv, EvictArgs a) {
  typedef __attribute__((ext_vector_type(8))) T vec;
  constexpr int PIECES = HD / 8;                       // of eight features, of a slot of K
  constexpr int KN = 32 * PIECES / 256, VN = 32 * HD / 256;
  __shared__ int from[32];
  const int tid = threadIdx.x, kvh = blockIdx.x, seq = blockIdx.y, layer = blockIdx.z;
  const int32_t* kept = a.kept + (((int64_t)layer * kv.batch + seq) * kv.hkv + kvh) * a.keep;
  const size_t of_layer = (size_t)layer * kv.n_pages * kv.hkv * kv.page_size * HD;
  T* kp = (T*)kv.k + of_layer;
  T* vp = (T*)kv.v + of_layer;
  int n = 0;
  for (int b = 0; b < a.keep; b += 32) {
    __syncthreads();
    if (tid < 32) from[tid] = b + tid < a.keep ? kept[b + tid] : -1;
    __syncthreads();
    if (from[0] < 0) break;
    const int last = 31 - __clz((int)__builtin_amdgcn_ballot_w64((threadIdx.x & 63) < 32 && from[threadIdx.x & 31] >= 0));
    n = b + last + 1;
    const int to_page = a.table_out[(size_t)seq * a.out_stride + b / kv.page_size], inside = b % kv.page_size;
    const bool to_ok = to_page >= 0 && to_page < kv.n_pages;
    if (!to_ok) {
      if (tid == 0) set_status(kv.status, ESP_DEV_BAD_PAGE);
      continue;
    }
    if (from[last] == b + last && kv.table[(size_t)seq * kv.stride + b / kv.page_size] == to_page) continue;     // (all where they are)
    auto plane_of = [&](int slot, int& in_page) -> int64_t {
      const int at = slot / kv.page_size, page = kv.table[(size_t)seq * kv.stride + at];
      in_page = slot - at * kv.page_size;
      if (page < 0 || page >= kv.n_pages) return -1;
      return (int64_t)page_plane(page, kvh, kv.hkv, kv.page_size, HD);
    };
    vec k[KN];
    T v[VN];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < KN; ++i) {
      const int piece = i * 256 + tid, slot = from[piece % 32];
      k[i] = vec{};
      if (slot >= 0) {
        int in;
        const int64_t plane = plane_of(slot, in);
        if (plane >= 0) k[i] = *reinterpret_cast<const vec*>(kp + plane + k_off(in, piece / 32 * 8, HD));
        bad |= plane < 0;
      }
    }
#pragma unroll
    for (int i = 0; i < VN; ++i) {
      const int e = i * 256 + tid, slot = from[e % 32];
      v[i] = from_f32<T>(0.f);
      if (slot >= 0) {
        int in;
        const int64_t plane = plane_of(slot, in);
        if (plane >= 0) v[i] = vp[plane + v_off(in, e / 32, HD)];
      }
    }
    if (bad) set_status(kv.status, ESP_DEV_BAD_PAGE);
    __syncthreads();
    const size_t to = page_plane(to_page, kvh, kv.hkv, kv.page_size, HD);
#pragma unroll
    for (int i = 0; i < KN; ++i) {
      const int piece = i * 256 + tid, s = piece % 32;
      if (s <= last) *reinterpret_cast<vec*>(kp + to + k_off(inside + s, piece / 32 * 8, HD)) = k[i];
    }
#pragma unroll
    for (int i = 0; i < VN; ++i) {
      const int e = i * 256 + tid, s = e % 32;
      if (s <= last) vp[to + v_off(inside + s, e / 32, HD)] = v[i];
    }
  }
  // (of the workgroups here only this one looks at the length, so len_out may be where it came from)
  if (tid == 0 && kvh == 0 && layer == 0) a.len_out[seq] = n > 0 ? n : kv.len[seq];
}

template <typename T, int HD>
void move(hipStream_t st, const PagedDev& kv, const EvictArgs& a) {
  hipLaunchKernelGGL((k_evict_move<T, HD>), dim3(kv.hkv, kv.batch, a.layers), dim3(256), 0, st, kv, a);
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
