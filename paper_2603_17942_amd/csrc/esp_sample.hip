// One token a row from its logits: temperature, top-k, top-p, min-p, inverse distribution function over ids (esp_sample).
//
// Weights are integers: q_i = rint(2^S exp((l_i - max) / T)), the exponential in fp64, S as large as leaves room for the sum of a row's in 63
// bits (50 at most).  Sums of them are the same in any order, so neither the histogram's atomics nor the division of the row among lanes
// can move a border between two tokens.  fp32 weights would: with 1e-7 each, the borders of 128256 tokens of which a few thousand count
// move by 1e-4 of all draws together.
//
// A workgroup has a row, a wave a sixteenth of it that lies in one piece, so that what waves add up is in the order of ids.  Passes over the row (the
// first from memory, the others from the caches): the largest; then, where top-k or top-p can cut, a histogram of counts and sums over 4096
// equal steps of log w, which says in what step the cut lies and with what count and sum before it.  The step's tokens go to LDS and are
// divided further, by the bits of their logits, until a few (ranked by comparing all with all) or equal ones (arithmetic) are left: the cut is
// a logit and how many of those equal to it are in.  Top-k first, as top-p is of its sum.  A last pass adds up what is in, by waves; the wave's
// piece in which the target lies is looked through by all.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "esp_internal.h"

namespace {

constexpr int WAVES = 16, THREADS = 64 * WAVES;
constexpr int BINS = 4096;             // of the first division, 12 bytes each
constexpr int SUB = THREADS;           // of the further ones: a thread each
constexpr int LIST = 4096;             // tokens of one bin that go to LDS
constexpr int FEW = 64;                // that are ranked by comparing all with all

struct SampleArgs {
  const void* logits;
  int64_t stride;
  int rows, vocab, shift;              // shift: S
  const float* temperature;
  const int32_t* top_k;
  const float *top_p, *min_p, *u;
  int32_t* ids;
  float* probs;
};

// fp32 order as unsigned order; both zeros are one
__device__ __forceinline__ unsigned key_of(float x) {
  const unsigned b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// rint(2^shift 2^t), t <= 0: 2^t = 2^n 2^f, |f| <= 1/2, the series of exp(f ln 2) up to f^9 (7e-12 is left out), the integer from the low bits of
// its sum with 2^52
struct Weigher {
  double top, scale;                   // of (l - top) scale: log2 of the weight
  float floor_t;                       // from here down there is nothing
  int shift;
  __device__ __forceinline__ double log2w(float l) const { return ((double)l - top) * scale; }
  __device__ __forceinline__ uint64_t of_log(double t) const {
    const double n = __builtin_rint(t), f = t - n;
    double p = 1.01780860092396997e-7;                  // (ln 2)^i / i!
    p = __builtin_fma(p, f, 1.32154867901443095e-6);
    p = __builtin_fma(p, f, 1.52527338040598403e-5);
    p = __builtin_fma(p, f, 1.54035303933816099e-4);
    p = __builtin_fma(p, f, 1.33335581464284434e-3);
    p = __builtin_fma(p, f, 9.61812910762847716e-3);
    p = __builtin_fma(p, f, 5.55041086648215800e-2);
    p = __builtin_fma(p, f, 2.40226506959100712e-1);
    p = __builtin_fma(p, f, 6.93147180559945309e-1);
    p = __builtin_fma(p, f, 1.0);
    const double w = __builtin_ldexp(p, (int)n + shift) + 0x1p52;
    return (uint64_t)__double_as_longlong(w) & 0xfffffffffffffull;
  }
  // 0 for what is no number, minus infinity, or too far down
  __device__ __forceinline__ uint64_t operator()(float l) const {
    const double t = log2w(l);
    return t > (double)floor_t ? of_log(t) : 0ull;
  }
};

__device__ __forceinline__ uint64_t shfl_up64(uint64_t v, int by) {
  const unsigned lo = __shfl_up((unsigned)v, by, 64), hi = __shfl_up((unsigned)(v >> 32), by, 64);
  return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t shfl_xor64(uint64_t v, int by) {
  const unsigned lo = __shfl_xor((unsigned)v, by, 64), hi = __shfl_xor((unsigned)(v >> 32), by, 64);
  return (uint64_t)hi << 32 | lo;
}

struct Shared {
  uint64_t sum[BINS];
  uint64_t sub_sum[SUB];
  uint64_t list[LIST];                 // key << 32 | ~id: larger is earlier in the order
  unsigned cnt[BINS];
  unsigned sub_cnt[SUB];
  uint64_t wave_sum[WAVES];
  unsigned wave_cnt[WAVES];
  float wave_max[WAVES];
  int wave_id[WAVES];
  // what one thread found
  uint64_t found_sum, few_sum;
  unsigned found_cnt, found_n, key_lo, key_hi, list_n, few_n, few_key, few_ties;
  int found_bin;
};

// sums of the threads before this one
__device__ __forceinline__ void before(Shared& s, unsigned& cnt, uint64_t& sum) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const unsigned own_c = cnt;
  const uint64_t own_s = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned c = __shfl_up(cnt, o, 64);
    const uint64_t q = shfl_up64(sum, o);
    if (lane >= o) { cnt += c; sum += q; }
  }
  __syncthreads();
  if (lane == 63) { s.wave_cnt[wave] = cnt; s.wave_sum[wave] = sum; }
  __syncthreads();
  cnt -= own_c; sum -= own_s;
  for (int w = 0; w < wave; ++w) { cnt += s.wave_cnt[w]; sum += s.wave_sum[w]; }
}

template <typename T> struct Piece;
template <> struct Piece<float> {
  static constexpr int N = 4;
  f32x4_t v;
  __device__ __forceinline__ float operator[](int i) const { return v[i]; }
};
template <> struct Piece<bf16_t> {
  static constexpr int N = 8;
  bf16x8_t v;
  __device__ __forceinline__ float operator[](int i) const { return (float)v[i]; }
};

// A row; a lane takes pieces of N consecutive logits, 16 bytes.
template <typename T, bool ALIGNED>
struct Row {
  static constexpr int N = Piece<T>::N;
  const T* p;
  int vocab;
  bool has_inf;                        // (then infinity is as the largest finite value)
  __device__ __forceinline__ void load(int at, float (&x)[N]) const {
    if (ALIGNED && at + N <= vocab) {
      Piece<T> q;
      q.v = *reinterpret_cast<const decltype(q.v)*>(p + at);
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = q[i];
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = at + i < vocab ? to_f32(p[at + i]) : -INFINITY;
    }
  }
  // f(id of the first, N logits) for this wave's pieces of [lo, hi), in ascending order for each lane; lo a multiple of N
  template <typename F> __device__ __forceinline__ void each(int lo, int hi, F f) const {
    constexpr int AHEAD = 32 / N;      // pieces on their way at once
    const int lane = threadIdx.x & 63;
    for (int b = lo; b < hi; b += 64 * N * AHEAD) {
      float x[AHEAD][N];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int at = b + (j * 64 + lane) * N;
        load(at < hi ? at : vocab, x[j]);
      }
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int at = b + (j * 64 + lane) * N;
        if (at >= hi) break;
        if (has_inf) {
#pragma unroll
          for (int i = 0; i < N; ++i) x[j][i] = x[j][i] == INFINITY ? FLT_MAX : x[j][i];
        }
        f(at, x[j]);
      }
    }
  }
};

struct Cut {
  unsigned key;                        // what is above it is in
  unsigned ties;                       // and so many of those at it, by id
  uint64_t sum;                        // of all that is in
};

template <typename T, bool ALIGNED>
__global__ __launch_bounds__(THREADS) void k_sample(SampleArgs a) {
  __shared__ Shared s;
  constexpr int N = Piece<T>::N;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.x;
  const int vocab = a.vocab;
  Row<T, ALIGNED> r{(const T*)a.logits + (int64_t)row * a.stride, vocab, false};
  const int piece = ((vocab + WAVES - 1) / WAVES + 64 * N - 1) / (64 * N) * (64 * N);       // a wave's
  const int lo = min(wave * piece, vocab), hi = min(lo + piece, vocab);

  const float temperature = a.temperature ? a.temperature[row] : 1.f;
  const float top_p = a.top_p ? a.top_p[row] : 1.f;
  const float min_p = a.min_p ? a.min_p[row] : 0.f;
  const int top_k = a.top_k ? a.top_k[row] : 0;
  const bool valid = temperature >= 0.f && temperature < INFINITY && top_p == top_p && min_p == min_p;

  // the largest, and where it is first
  float best = -INFINITY;
  int best_at = -1;
  if (valid)
    r.each(lo, hi, [&](int at, const float (&x)[N]) {
      float m = x[0];
#pragma unroll
      for (int i = 1; i < N; ++i) m = fmaxf(m, x[i]);
      if (m > best) { best = m; best_at = at; }
    });
  if (best_at >= 0) {
    float x[N];
    r.load(best_at, x);
    int e = 0;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) e = x[i] == best ? i : e;
    best_at += e;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const float m = __shfl_xor(best, o, 64);
    const int at = __shfl_xor(best_at, o, 64);
    if (m > best || (m == best && at >= 0 && (unsigned)at < (unsigned)best_at)) { best = m; best_at = at; }
  }
  if (lane == 0) { s.wave_max[wave] = best; s.wave_id[wave] = best_at; }
  __syncthreads();
  for (int w = 0; w < WAVES; ++w)      // (waves have ascending ids)
    if (s.wave_max[w] > best || (s.wave_max[w] == best && (unsigned)s.wave_id[w] < (unsigned)best_at)) { best = s.wave_max[w]; best_at = s.wave_id[w]; }
  if (best_at < 0 || temperature == 0.f) {             // nothing to choose, or the first of the order
    if (tid == 0) {
      a.ids[row] = best_at;
      if (a.probs) a.probs[row] = best_at < 0 ? 0.f : 1.f;
    }
    return;
  }
  if (best == INFINITY) { r.has_inf = true; best = FLT_MAX; }

  const Weigher weight{(double)best, 1.4426950408889634 / (double)temperature, -(float)(a.shift + 2), a.shift};
  const uint64_t least = min_p > 0.f ? max(1ull, (uint64_t)__builtin_rint(__builtin_ldexp((double)fminf(min_p, 1.f), a.shift))) : 1ull;
  Cut cut{0u, 0u, 0ull};               // all is in
  const bool by_count = top_k > 0 && top_k < vocab, by_sum = top_p < 1.f;

  if (by_count || by_sum) {
    const double steps = (double)BINS / (a.shift + 2);
    auto bin_of = [&](double t) { return min((int)(-t * steps), BINS - 1); };
    for (int i = tid; i < BINS; i += THREADS) { s.cnt[i] = 0; s.sum[i] = 0; }
    __syncthreads();
    r.each(lo, hi, [&](int, const float (&x)[N]) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const double t = weight.log2w(x[i]);
        if (t > (double)weight.floor_t) {
          const uint64_t q = weight.of_log(t);
          if (q) {
            const int b = bin_of(t);
            atomicAdd(&s.cnt[b], 1u);
            atomicAdd((unsigned long long*)&s.sum[b], (unsigned long long)q);
          }
        }
      }
    });
    __syncthreads();
    constexpr int EACH = BINS / THREADS;
    unsigned total_c = 0;
    uint64_t total_s = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) { total_c += s.cnt[tid * EACH + i]; total_s += s.sum[tid * EACH + i]; }
    unsigned before_c = total_c;
    uint64_t before_s = total_s;
    before(s, before_c, before_s);
    if (tid == THREADS - 1) { s.found_cnt = before_c + total_c; s.found_sum = before_s + total_s; }
    __syncthreads();
    const unsigned alive = s.found_cnt;
    cut.sum = s.found_sum;
    __syncthreads();

    // The cut after `count` tokens, or before the first one with `sum` or more before it, whichever comes first; it is there.
    auto find = [&](unsigned count, uint64_t sum) {
      unsigned c = before_c;
      uint64_t q = before_s;
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const unsigned n = s.cnt[tid * EACH + i];
        const uint64_t w = s.sum[tid * EACH + i];
        if (n && c < count && q < sum && (c + n >= count || q + w >= sum)) { s.found_bin = tid * EACH + i; s.found_cnt = c; s.found_sum = q; s.found_n = n; }
        c += n; q += w;
      }
      if (tid == 0) { s.key_lo = ~0u; s.key_hi = 0u; s.list_n = 0; }
      __syncthreads();
      const int bin = s.found_bin;
      r.each(lo, hi, [&](int at, const float (&x)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const double t = weight.log2w(x[i]);
          if (t > (double)weight.floor_t && bin_of(t) == bin && weight.of_log(t)) {
            const unsigned k = key_of(x[i]), place = atomicAdd(&s.list_n, 1u);
            if (place < LIST) s.list[place] = (uint64_t)k << 32 | (unsigned)~(at + i);
            atomicMin(&s.key_lo, k);
            atomicMax(&s.key_hi, k);
          }
        }
      });
      __syncthreads();
      const bool listed = s.list_n <= LIST;
      const unsigned listed_n = s.list_n;
      for (int level = 0; level < 6; ++level) {        // (32 bits, ten at a time, and the last look)
        const unsigned k_lo = s.key_lo, k_hi = s.key_hi, n = s.found_n, c0 = s.found_cnt;
        const uint64_t q0 = s.found_sum;
        if (k_lo == k_hi) {            // equal ones: as many as there is room for
          const uint64_t q = weight(of_key(k_lo));
          uint64_t m = min((uint64_t)n, (uint64_t)(count - c0));
          m = min(m, (sum - q0 - 1) / q + 1);
          cut = {k_lo, (unsigned)m, q0 + m * q};
          __syncthreads();
          return;
        }
        auto members = [&](auto f) {   // f(key, id) for what is between the two keys
          if (listed) {
            for (unsigned i = tid; i < listed_n; i += THREADS) {
              const unsigned k = (unsigned)(s.list[i] >> 32);
              if (k >= k_lo && k <= k_hi) f(k, (int)~(unsigned)s.list[i]);
            }
          } else {
            r.each(lo, hi, [&](int at, const float (&x)[N]) {
#pragma unroll
              for (int i = 0; i < N; ++i) {
                if (x[i] > -INFINITY) {
                  const unsigned k = key_of(x[i]);
                  if (k >= k_lo && k <= k_hi) f(k, at + i);
                }
              }
            });
          }
        };
        if (n <= FEW) {                // (their places in sub_sum)
          if (tid == 0) { s.few_n = 0; s.few_sum = 0; }
          __syncthreads();
          members([&](unsigned k, int id) { s.sub_sum[atomicAdd(&s.few_n, 1u)] = (uint64_t)k << 32 | (unsigned)~id; });
          __syncthreads();
          if (wave == 0) {
            const uint64_t mine = lane < (int)n ? s.sub_sum[lane] : 0ull;
            const unsigned k = (unsigned)(mine >> 32);
            const uint64_t w = lane < (int)n ? weight(of_key(k)) : 0ull;
            unsigned rank = 0;
            uint64_t ahead = 0;
            for (int j = 0; j < (int)n; ++j) {
              const uint64_t other = s.sub_sum[j];
              const unsigned lo_w = __shfl((unsigned)w, j, 64), hi_w = __shfl((unsigned)(w >> 32), j, 64);
              const uint64_t wj = (uint64_t)hi_w << 32 | lo_w;
              if (other > mine) { ++rank; ahead += wj; }
            }
            const bool in = lane < (int)n && c0 + rank < count && q0 + ahead < sum;
            const int last = __popcll(__builtin_amdgcn_ballot_w64(in)) - 1;      // (what is in is a prefix of the ranking)
            if (in && (int)rank == last) { s.few_key = k; s.few_sum = q0 + ahead + w; }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const int ties = __popcll(__builtin_amdgcn_ballot_w64(in && k == s.few_key));
            if (lane == 0) s.few_ties = ties;
          }
          __syncthreads();
          cut = {s.few_key, s.few_ties, s.few_sum};
          __syncthreads();
          return;
        }
        const int bits = 32 - __clz(k_hi - k_lo), by = max(0, bits - 10);          // SUB = 2^10 of them
        s.sub_cnt[tid] = 0; s.sub_sum[tid] = 0;
        __syncthreads();
        members([&](unsigned k, int) {
          const unsigned b = (k_hi - k) >> by;
          atomicAdd(&s.sub_cnt[b], 1u);
          atomicAdd((unsigned long long*)&s.sub_sum[b], (unsigned long long)weight(of_key(k)));
        });
        __syncthreads();
        const unsigned m = s.sub_cnt[tid];
        const uint64_t w = s.sub_sum[tid];
        unsigned c1 = m;
        uint64_t q1 = w;
        before(s, c1, q1);
        c1 += c0; q1 += q0;
        __syncthreads();
        if (m && c1 < count && q1 < sum && (c1 + m >= count || q1 + w >= sum)) {
          s.found_cnt = c1; s.found_sum = q1; s.found_n = m;
          s.key_hi = k_hi - ((unsigned)tid << by);
          const uint64_t down = ((uint64_t)tid + 1) << by;
          s.key_lo = down - 1 >= (uint64_t)(k_hi - k_lo) ? k_lo : k_hi - (unsigned)(down - 1);
        }
        __syncthreads();
      }
    };
    if (by_count && (unsigned)top_k < alive) find((unsigned)top_k, ~0ull);
    if (by_sum) {
      const double p = fmaxf(top_p, 0.f) * (double)cut.sum;
      const uint64_t goal = max(1ull, (uint64_t)__builtin_ceil(p));            // (the first is in)
      if (goal <= cut.sum) find(~0u, goal);
    }
  }

  // what is in, by waves
  uint64_t sum = 0;
  unsigned ties = 0;
  auto take = [&](float x, uint64_t& q_in, unsigned& tie) {
    const uint64_t q = weight(x);
    const unsigned k = key_of(x);
    q_in = q >= least && k > cut.key ? q : 0ull;
    tie = q >= least && k == cut.key ? 1u : 0u;
  };
  r.each(lo, hi, [&](int, const float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint64_t q; unsigned t;
      take(x[i], q, t);
      sum += q; ties += t;
    }
  });
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) { sum += shfl_xor64(sum, o); ties += __shfl_xor(ties, o, 64); }
  __syncthreads();
  if (lane == 0) { s.wave_sum[wave] = sum; s.wave_cnt[wave] = ties; }
  __syncthreads();
  const uint64_t tie_q = cut.key ? weight(of_key(cut.key)) : 0ull;
  uint64_t all = 0;
  unsigned tied = 0;
  for (int w = 0; w < WAVES; ++w) { all += s.wave_sum[w]; tied += s.wave_cnt[w]; }
  all += tie_q * min(tied, cut.ties);
  const float u = a.u[row];
  const double uu = u > 0.f ? (double)fminf(u, 0.99999994f) : 0.0;
  const uint64_t target = min((uint64_t)(uu * (double)all), all - 1);
  int in_wave = WAVES - 1;
  uint64_t ahead = 0;
  unsigned ties_ahead = 0;
  for (int w = 0; w < WAVES; ++w) {
    const unsigned left = cut.ties - min(ties_ahead, cut.ties);
    const uint64_t q = s.wave_sum[w] + tie_q * min(s.wave_cnt[w], left);
    if (target < ahead + q) { in_wave = w; break; }
    ahead += q; ties_ahead += s.wave_cnt[w];
  }
  // that piece, a run of consecutive ids for every thread
  const int start = min(in_wave * piece, vocab), end = min(start + piece, vocab);
  const int run = (piece / THREADS + N) / N * N;
  const int mine = min(start + tid * run, end), mine_end = min(mine + run, end);
  sum = 0; ties = 0;
  for (int at = mine; at < mine_end; at += N) {
    float x[N];
    r.load(at, x);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint64_t q; unsigned t;
      if (r.has_inf && x[i] == INFINITY) x[i] = FLT_MAX;
      take(x[i], q, t);
      if (at + i < mine_end) { sum += q; ties += t; }
    }
  }
  uint64_t q1 = sum;
  unsigned c1 = ties;
  before(s, c1, q1);
  c1 += ties_ahead;
  const unsigned left0 = cut.ties - min(ties_ahead, cut.ties), left1 = cut.ties - min(c1, cut.ties);
  uint64_t at_q = ahead + q1 + tie_q * (left0 - left1);
  if (target >= at_q && target < at_q + sum + tie_q * min(ties, left1)) {
    unsigned left = left1;
    for (int at = mine; at < mine_end; ++at) {
      float x = to_f32(r.p[at]);
      if (r.has_inf && x == INFINITY) x = FLT_MAX;
      uint64_t q; unsigned t;
      take(x, q, t);
      if (t && left) { q = tie_q; --left; }
      if (target < at_q + q) {
        a.ids[row] = at;
        if (a.probs) a.probs[row] = (float)((double)q / (double)all);
        break;
      }
      at_q += q;
    }
  }
}

template <typename T>
hipError_t launch(hipStream_t st, const SampleArgs& a) {
  const bool aligned = (uintptr_t)a.logits % 16 == 0 && a.stride * sizeof(T) % 16 == 0;
  auto* f = aligned ? k_sample<T, true> : k_sample<T, false>;
  hipLaunchKernelGGL(f, dim3(a.rows), dim3(THREADS), 0, st, a);
  return hipGetLastError();
}

}  // namespace

extern "C" esp_status esp_sample(void* stream, int32_t dtype, const void* logits, int64_t row_stride, int32_t rows, int32_t vocab,
                                 const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, const float* u,
                                 int32_t* ids, float* probs) {
  if (!logits || !u || !ids || rows < 0 || vocab < 1) return ESP_EINVAL;
  if (dtype != ESP_F32 && dtype != ESP_BF16) return ESP_EDTYPE;
  if (row_stride < vocab) return ESP_ESHAPE;
  // ids are counted in 31 bits with room for a workgroup's pieces behind the last; a launch counts threads in 32
  if (vocab > (1 << 24) || rows >= (1 << 22)) return ESP_ECAPACITY;
  if (rows == 0) return ESP_OK;
  int log2_vocab = 0;
  while ((1 << log2_vocab) < vocab) ++log2_vocab;
  const SampleArgs a{logits, row_stride, rows, vocab, std::min(50, 62 - log2_vocab), temperature, top_k, top_p, min_p, u, ids, probs};
  const hipError_t e = dtype == ESP_F32 ? launch<float>((hipStream_t)stream, a) : launch<bf16_t>((hipStream_t)stream, a);
  return e == hipSuccess ? ESP_OK : ESP_EDEVICE;
}
