// One token a row from its logits: temperature, top-k, top-p, min-p, inverse distribution function over ids (esp_sample).
//
// w = exp((l - largest) / T) is computed in fp64 (1.1e-12 of itself) and added up in integers or, within a part of a row, in fp64 in a fixed order.
// fp32 would not do: with 1e-7 for each weight the borders of 128256 tokens of which a few thousand count move by 1e-4 of all draws together.
//
// What goes over logits has them in registers, 4096 or 8192 a workgroup (a part of a row), so that one row is spread over many CUs; what decides has a
// workgroup a row and looks at what the parts left.
//   k_sample_parts  a part's largest logit and the first id that has it; where all tokens' weights count (no limit, or top-p without top-k) their sum
//                   against that largest one; for top-k and top-p a histogram over equal steps of log w: how many tokens, and where in the step they lie
//   k_sample_edges  the histograms together say in which steps the cut lies, for certain: counts are exact, weights known to 1e-4 from the places
//   k_sample_collect the tokens of these steps to a list, what lies before them added up by parts (threads whose largest logit is below do not look again)
//   k_sample_pick   the list is divided, by equal steps and then by the bits of its logits, until a few tokens (ranked by comparing all with all) or equal
//                   ones (arithmetic) are left: the cut is a logit and how many of those equal to it are in.  Top-k first, as top-p is of what it leaves.
//                   The part in which the target lies is looked through.
// The two in the middle are launched where there are limits and more than 4096 tokens: so many are a list by themselves (top-k of one row: 4096 tokens 14.4 us,
// 4100 with all four kernels 22.5; top-p 17.0 and 27.9).  Rows that they cannot narrow down (more than 4096 tokens in the steps of the cut, or
// logits above 2^20 steps) are divided in k_sample_pick by going over the row again and again.  Logits of a normal distribution of 1e-3, with top-k 50 / top-p 0.9 /
// top-k 5000 and top-p 0.9: 154 / 286 / 339 us for a row of 128256, 63 / 109 / 118 for one of 40000, 184 / 324 / 384 and 72 / 117 / 139 for 64 of them side by side.
//
// What bounds it: 320 rows of 151936 bf16 without limits are 97 MB, 19 us at the rate of a copy, and take 51, as the sum is some 20 fp64 and other
// instructions a weight (64% of the issue slots; with 13 instead of 17 in fp64 and as many more in fp32 2 us more).  256 rows of 128256 with limits are 131 MB, 26 us, and take
// 84: parts 36, edges 8, collect 22, pick 18.  A single row is a chain of launches (4, of which parts and collect are 5 us each) and of exchanges inside
// the two that decide: 24 us with top-k, 32 with top-p, 9.5 without limits.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>

#include "esp_internal.h"
#include "esp_scan.h"

namespace {

constexpr int PART_THREADS = 256;      // of what goes over logits
constexpr int THREADS = 1024, WAVES = THREADS / 64;    // of what decides
constexpr int BINS = 1024;             // steps of log w, 47 powers of two at most
constexpr int PLACES = 512;            // that are told apart in a step.  A bin: tokens (up to 8192) << 44 | sum of places << 22 | of their squares / PLACES
constexpr int LIST = 4096;             // tokens that may be listed
constexpr int FEW = 64;                // that are ranked by comparing all with all
constexpr int MOST_PARTS = THREADS;
constexpr int ROWS_AT_ONCE = 1024;     // that the workspace is for; more are done one lot after the other
constexpr float FAR_STEPS = 0x1p20f;   // logits of more steps than that have no place in one

struct Part {
  float top;                           // largest logit (infinity: as the largest finite value), and the first id that has it (-1: none)
  int at;
  double sum;                          // of the weights against it
};
struct PartSums { uint64_t all, in; }; // of what is before the list; less what min-p takes and what is below half a unit
enum { AS_IT_IS = 0, COLLECT = 1, DIVIDE = 2 };        // without list; with it; by going over the row
struct RowState {
  int mode, first, last;               // steps of the list; what is before `first` is added up
  unsigned before;                     // tokens before the list
  int list_n;
  float top, base;                     // the largest logit, its step
};

struct SampleArgs {
  const void* logits;
  int64_t stride;
  int vocab, shift;                    // shift: of the integers, S
  int part, parts;                     // logits of a part, parts of a row
  const float* temperature;
  const int32_t* top_k;
  const float *top_p, *min_p, *u;
  int32_t* ids;
  float* probs;
  // workspace: [rows][parts] and [rows]
  Part* tops;
  PartSums* sums;
  uint64_t* bins;                      // [BINS]
  float* maxima;                       // [PART_THREADS]
  RowState* state;
  uint64_t* list;                      // [LIST]  key << 32 | ~id: larger is earlier in the order
};

struct Limits {
  float temperature, top_p, min_p;
  int top_k;
  bool valid, by_count, by_sum, by_part;
};
__device__ __forceinline__ Limits limits(const SampleArgs& a, int row) {
  Limits m;
  const float t = a.temperature ? a.temperature[row] : 1.f;
  m.top_p = a.top_p ? a.top_p[row] : 1.f;
  m.min_p = a.min_p ? a.min_p[row] : 0.f;
  m.top_k = a.top_k ? a.top_k[row] : 0;
  m.valid = t >= 0.f && t < INFINITY && m.top_p == m.top_p && m.min_p == m.min_p;
  m.temperature = t > 0.f ? fminf(fmaxf(t, 1e-20f), 1e20f) : t;
  m.by_count = m.top_k > 0 && m.top_k < a.vocab;
  m.by_sum = m.top_p < 1.f;
  m.by_part = m.min_p > 0.f;
  return m;
}
// all tokens are the list
__device__ __forceinline__ bool one_list(const SampleArgs& a) { return a.vocab <= LIST; }
__device__ __forceinline__ bool draws(const Limits& m) { return m.valid && m.temperature > 0.f; }
__device__ __forceinline__ bool limited(const Limits& m) { return m.by_count || m.by_sum || m.by_part; }
// do the weights of all tokens count
__device__ __forceinline__ bool all_count(const Limits& m) { return !m.by_count && (m.by_sum || !m.by_part); }

// powers of two, and steps of log w, that a unit of the logits is
__device__ __forceinline__ double octaves(const Limits& m) { return 1.4426950408889634 / (double)m.temperature; }
__device__ __forceinline__ float steps(const SampleArgs& a, const Limits& m) { return (float)(octaves(m) * (BINS / (double)(a.shift + 2))); }
__device__ __forceinline__ float step_of(float x, float per) { return floorf(x * per); }

// fp32 order as unsigned order; both zeros are one
__device__ __forceinline__ unsigned key_of(float x) {
  const unsigned b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// Weights against a largest logit.  2^t = 2^n 2^f with |f| <= 1/2: n and the fraction by adding 1.5 2^52, 2^f = 1 + f p(f) with p of degree 7
// (equal ripples of the relative error, 1.1e-12, found by exchange), n into the exponent.
struct Weigher {
  double top, scale;                   // of (l - top) scale: log2 of the weight
  // 2^up w, up >= 0; what is no number, minus infinity or below 2^-900 weighs 2^-900
  __device__ __forceinline__ double real(float l, int up) const {
    const double t = __builtin_fmax(((double)l - top) * scale, -900.0);
    const double k = t + 0x1.8p52, f = t - (k - 0x1.8p52);
    double p = 1.3344183709045696e-06;
    p = __builtin_fma(p, f, 1.5314209233228402e-05);
    p = __builtin_fma(p, f, 0.00015403098285429032);
    p = __builtin_fma(p, f, 0.001333343415751413);
    p = __builtin_fma(p, f, 0.009618129558840711);
    p = __builtin_fma(p, f, 0.05550410959228873);
    p = __builtin_fma(p, f, 0.24022650694742584);
    p = __builtin_fma(p, f, 0.6931471805412327);
    p = __builtin_fma(p, f, 1.0);
    const int n = (int)__double_as_longlong(k) + up;
    return __longlong_as_double(__double_as_longlong(p) + ((int64_t)n << 52));
  }
  // rint(2^up w), up <= 50: the low bits of its sum with 2^52
  __device__ __forceinline__ uint64_t whole(float l, int up) const {
    return (uint64_t)__double_as_longlong(real(l, up) + 0x1p52) & 0xfffffffffffffull;
  }
};

__device__ __forceinline__ unsigned wave_most(unsigned float_bits) {
  return lane_of(running(float_bits, __float_as_uint(-INFINITY), [](unsigned a, unsigned b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }), 63);
}
// the largest of a wave's logits, the lowest id of equal ones
__device__ __forceinline__ void wave_largest(float& top, int& at) {
  const float m = __uint_as_float(wave_most(__float_as_uint(top)));
  at = (int)lane_of(running(top == m ? (unsigned)at : ~0u, ~0u, Least()), 63);
  top = m;
}

// A row; a thread takes pieces of N consecutive logits, 16 bytes.
template <typename T, bool ALIGNED>
struct Row {
  static constexpr int N = 16 / sizeof(T);
  const T* p;
  int vocab;
  __device__ __forceinline__ Row(const SampleArgs& a, int row) : p((const T*)a.logits + (int64_t)row * a.stride), vocab(a.vocab) {}
  template <int M>                     // a divisor of N; `at` is divided by it
  __device__ __forceinline__ void load(int at, float (&x)[M]) const {
    typedef __attribute__((ext_vector_type(M))) T vec;
    if (ALIGNED && at + M <= vocab) {
      const vec v = *reinterpret_cast<const vec*>(p + at);
#pragma unroll
      for (int i = 0; i < M; ++i) x[i] = (float)v[i];
    } else {
#pragma unroll
      for (int i = 0; i < M; ++i) x[i] = at + i < vocab ? to_f32(p[at + i]) : -INFINITY;
    }
  }
};
// infinity is as the largest finite value
__device__ __forceinline__ float tame(float x) { return x == INFINITY ? FLT_MAX : x; }

template <typename T, bool ALIGNED, int PER>           // PER logits a thread
__global__ __launch_bounds__(PART_THREADS) void k_sample_parts(SampleArgs a) {
  constexpr int N = Row<T, ALIGNED>::N, PIECES = PER / N;
  __shared__ float wave_top[4];
  __shared__ int first_at;
  __shared__ double wave_sum[4];
  __shared__ uint64_t bins[BINS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, part = blockIdx.x, row = blockIdx.y;
  const int64_t mine = (int64_t)row * a.parts + part;
  const Limits m = limits(a, row);
  const Row<T, ALIGNED> r(a, row);
  const int lo = part * (PART_THREADS * PER);
  float x[PIECES][N];
  float own = -INFINITY;
#pragma unroll
  for (int j = 0; j < PIECES; ++j) r.load(min(lo + (j * PART_THREADS + tid) * N, a.vocab), x[j]);
#pragma unroll
  for (int j = 0; j < PIECES; ++j)
#pragma unroll
    for (int i = 0; i < N; ++i) own = fmaxf(own, x[j][i]);
  if (own == INFINITY) {
    own = FLT_MAX;
#pragma unroll
    for (int j = 0; j < PIECES; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i) x[j][i] = tame(x[j][i]);
  }
  // the largest of all, then its first id among the few threads that have it
  const float of_wave = __uint_as_float(wave_most(__float_as_uint(own)));
  if (lane == 0) wave_top[wave] = of_wave;
  if (tid == 0) first_at = INT_MAX;
  __syncthreads();
  const float top = fmaxf(fmaxf(wave_top[0], wave_top[1]), fmaxf(wave_top[2], wave_top[3]));
  if (own == top && top > -INFINITY) {
    int at = INT_MAX;
#pragma unroll
    for (int j = PIECES - 1; j >= 0; --j)
#pragma unroll
      for (int i = N - 1; i >= 0; --i) at = x[j][i] == top ? lo + (j * PART_THREADS + tid) * N + i : at;
    atomicMin(&first_at, at);
  }
  if (draws(m) && limited(m) && !one_list(a)) a.maxima[mine * PART_THREADS + tid] = own;
  double sum = 0.0;
  if (draws(m) && top > -INFINITY) {
    if (all_count(m)) {
      const Weigher weight{(double)top, octaves(m)};
      double s[2] = {0.0, 0.0};
#pragma unroll
      for (int j = 0; j < PIECES; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) s[i & 1] += weight.real(x[j][i], 0);
      sum = s[0] + s[1];
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
      if (lane == 0) wave_sum[wave] = sum;
      __syncthreads();
      sum = (wave_sum[0] + wave_sum[1]) + (wave_sum[2] + wave_sum[3]);
    }
    if ((m.by_count || m.by_sum) && !one_list(a)) {
      for (int i = tid; i < BINS; i += PART_THREADS) bins[i] = 0;
      __syncthreads();
      const float per = steps(a, m), base = step_of(top, per);
#pragma unroll
      for (int j = 0; j < PIECES; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float s = x[j][i] * per, step = base - floorf(s);
          if (step < (float)BINS) {
            const unsigned f = (unsigned)(__builtin_amdgcn_fractf(s) * PLACES);         // (below 1, which s - floor(s) is not for a little less than 0)
            atomicAdd((unsigned long long*)&bins[(int)step], 1ull << 44 | (uint64_t)f << 22 | (f * f / PLACES));
          }
        }
      __syncthreads();
      for (int i = tid; i < BINS; i += PART_THREADS) a.bins[mine * BINS + i] = bins[i];
    }
  }
  __syncthreads();
  if (tid == 0) a.tops[mine] = {top, top > -INFINITY ? first_at : -1, sum};
}

// ---- a workgroup a row -----------------------------------------------------------------------------------------

typedef WaveSums<WAVES> Sums;

// The parts of a row.  Every wave looks at all of them, a lane at `each` consecutive ones (as a rule one), so nothing is exchanged between waves: an exchange with its
// barrier and two rounds of running sums takes half a microsecond, and there were ten of them.
struct Parts {
  const Part* p;
  int n, each, first;
  Part mine;                           // this lane's first
  __device__ __forceinline__ Parts(const SampleArgs& a, int row)
      : p(a.tops + (int64_t)row * a.parts), n(a.parts), each((a.parts + 63) / 64), first((int)(threadIdx.x & 63) * each) {
    mine = first < n ? p[first] : Part{-INFINITY, -1, 0.0};
  }
  template <typename F>
  __device__ __forceinline__ void all(F f) const {     // of this lane
    f(first, mine);
    for (int i = 1; i < each; ++i)
      if (first + i < n) f(first + i, p[first + i]);
  }
  __device__ __forceinline__ void largest(float& top, int& at) const {
    top = -INFINITY; at = -1;
    all([&](int, const Part& q) { if (q.top > top) { top = q.top; at = q.at; } });
    wave_largest(top, at);
  }
};
// a part's weights in units of 2^-shift of the largest logit's
__device__ __forceinline__ uint64_t part_weight(const Part& p, const Weigher& weight, int shift) {
  return p.at >= 0 ? (uint64_t)__builtin_rint(p.sum * weight.real(p.top, shift)) : 0ull;
}
__device__ __forceinline__ uint64_t sum_goal(float top_p, uint64_t sum) {        // (the first is in)
  return max(1ull, (uint64_t)__builtin_ceil((double)fmaxf(top_p, 0.f) * (double)sum));
}

static_assert(BINS == THREADS, "k_sample_edges: a thread a step");
__global__ __launch_bounds__(THREADS) void k_sample_edges(SampleArgs a) {
  __shared__ Sums s;
  __shared__ int found[4];
  int turn = 0;
  const int tid = threadIdx.x, row = blockIdx.x;
  const Parts parts(a, row);
  const Limits m = limits(a, row);
  RowState& out = a.state[row];
  if (!draws(m) || !limited(m)) {
    if (tid == 0) out.mode = AS_IT_IS;
    return;
  }
  float top;
  int top_at;
  parts.largest(top, top_at);
  const float per = steps(a, m), base = step_of(top, per);
  const double octave = (double)(a.shift + 2) / BINS;  // of a step
  RowState st{COLLECT, 0, -1, 0u, 0, top, base};
  // (largest logits between which the parts' differ by 2^20 steps and more differ by more than 47 powers of two: nothing there counts)
  if (top_at < 0 || !(fabsf(top * per) < FAR_STEPS)) {
    if (tid == 0) { st.mode = top_at < 0 ? AS_IT_IS : DIVIDE; out = st; }
    return;
  }
  if (!m.by_count && !m.by_sum) {      // min-p: what can weigh that much, a step more and the one that the largest is in
    st.first = (int)fminf(-__builtin_amdgcn_logf(fminf(m.min_p, 1.f)) * (float)(1.0 / octave) * 1.001f + 3.f, (float)BINS);
    if (tid == 0) out = st;
    return;
  }
  if (tid < 4) found[tid] = tid == 1 ? BINS - 1 : 0;
  unsigned n = 0, places = 0, squares = 0;
  for (int p0 = 0; p0 < a.parts; p0 += 64) {
    // lane l: by how many steps part p0 + l begins below the row's largest (BINS: by all of them)
    const int p = p0 + (tid & 63);
    const Part of = parts.each == 1 ? parts.mine : p < a.parts ? parts.p[p] : Part{0.f, -1, 0.0};
    const float d = of.at < 0 ? (float)BINS : fminf(base - step_of(of.top, per), (float)BINS);
    const int by = (int)d;
    for (int e0 = 0; e0 < min(64, a.parts - p0); e0 += 16) {       // (sixteen parts' on their way at once)
      uint64_t v[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int i = tid - __builtin_amdgcn_readlane(by, e0 + e);
        v[e] = i >= 0 ? a.bins[((int64_t)row * a.parts + p0 + e0 + e) * BINS + i] : 0ull;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) { n += (unsigned)(v[e] >> 44); places += (unsigned)(v[e] >> 22) & 0x3fffffu; squares += (unsigned)v[e] & 0x3fffffu; }
    }
  }
  // Sums of weights in units of 2^-40.  A token at place f of a step weighs 1 + k f + (k f)^2 / 2 + up to k^3 / 5 times what one at its lower end does,
  // k = ln 2 octave = 0.032: 6.6e-6 for the last, k / PLACES = 6e-5 for the place, k^2 / PLACES = 2e-6 for its square; the first two taken at their
  // middle, sums are off by 4e-5, by what the step's number is off, and by 1e-6 for the exponential.
  const double k = 0.6931471805599453 * octave, up = top * per - base;
  const double middle = (double)n * (1 + 0.5 * k / PLACES) + k / PLACES * ((double)places + 0.5 * k * (double)squares);
  const uint64_t w = (uint64_t)(middle * (double)__builtin_amdgcn_exp2f((float)(40.0 - (tid + up) * octave)));
  unsigned c0 = n;
  uint64_t q0 = w;
  const unsigned alive = before(s, turn, c0);
  if (!m.by_count) before(s, turn, q0);
  if (m.by_count) {                    // (no cut, if fewer weigh anything: the last step)
    const unsigned want = min((unsigned)m.top_k, alive);
    if (c0 < want && want <= c0 + n) found[0] = found[1] = tid;
  } else {
    uint64_t all = 0;
    parts.all([&](int, const Part& q) { all += part_weight(q, Weigher{(double)top, octaves(m)}, a.shift); });
    const uint64_t goal = sum_goal(m.top_p, wave_total(all));
    const double g = __builtin_ldexp((double)goal, 40 - a.shift), off = 1e-4 + 0.1 * 0x1p-23 * fabsf(top * per);
    const uint64_t reach = max(1ull, (uint64_t)(g * (1 - off))), surely = (uint64_t)(g * (1 + off)) + BINS;
    if (q0 < reach && reach <= q0 + w) found[0] = tid;
    if (q0 < surely && surely <= q0 + w) found[1] = tid;
  }
  __syncthreads();
  const int first = found[0], last = found[1];
  __syncthreads();
  if (tid == first) found[2] = (int)c0;
  if (tid == last) found[3] = (int)(c0 + n);
  __syncthreads();
  if (tid == 0) {
    const unsigned ahead = (unsigned)found[2], end = (unsigned)found[3];
    // All tokens from the first on, if there is room: top-p after top-k needs that, and so does top-k where all that weighs anything is in.
    st.last = last;
    if (end > LIST) {
      st.first = first; st.before = ahead;
      if (end - ahead > LIST || (m.by_count && (m.by_sum || (unsigned)m.top_k >= alive))) st.mode = DIVIDE;
    }
    out = st;
  }
}

template <typename T, bool ALIGNED, int PER>
__global__ __launch_bounds__(PART_THREADS) void k_sample_collect(SampleArgs a) {
  constexpr int N = Row<T, ALIGNED>::N, PIECES = PER / N;
  __shared__ unsigned short list[LIST];                // places in the part
  __shared__ double wave_sum[4][2];
  __shared__ unsigned list_n, place;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, part = blockIdx.x, row = blockIdx.y;
  const int64_t mine = (int64_t)row * a.parts + part;
  const RowState st = a.state[row];
  if (st.mode != COLLECT) return;
  const Limits m = limits(a, row);
  const Row<T, ALIGNED> r(a, row);
  // step < n is x per >= base - n + 1
  const float per = steps(a, m), ahead = st.base - (float)st.first + 1.f, listed = st.base - (float)max(st.first, st.last + 1) + 1.f;
  if (tid == 0) list_n = 0;
  const float own = a.maxima[mine * PART_THREADS + tid];
  const Weigher weight{(double)st.top, octaves(m)};
  __syncthreads();
  // In is what weighs min_p and half a unit; without min-p that is all, unless the steps before the list reach so far down.
  const double least = (m.by_part ? fmax(__builtin_rint(__builtin_ldexp((double)fminf(m.min_p, 1.f), a.shift)), 1.0) : 1.0) - 0.5;
  const bool some_out = m.by_part || (int64_t)st.first * (a.shift + 2) > (int64_t)(a.shift + 1) * BINS;
  double all = 0.0, in = 0.0;
  if (own * per >= listed) {
    float x[PIECES][N];
#pragma unroll
    for (int j = 0; j < PIECES; ++j) r.load(min(part * (PART_THREADS * PER) + (j * PART_THREADS + tid) * N, a.vocab), x[j]);
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
      float most = x[j][0] = tame(x[j][0]);
#pragma unroll
      for (int i = 1; i < N; ++i) { x[j][i] = tame(x[j][i]); most = fmaxf(most, x[j][i]); }
      if (most * per >= ahead) {
#pragma unroll
        for (int i = 0; i < N; ++i) {  // (the piece's others weigh 2^-900: side by side they take less time than branches do)
          const double w = weight.real(x[j][i] * per >= ahead ? x[j][i] : -INFINITY, a.shift);
          all += w;
          if (some_out) in += w >= least ? w : 0.0;
        }
      }
      if (most * per >= listed && st.first <= st.last) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float t = x[j][i] * per;
          if (t >= listed && t < ahead) {
            const unsigned n = atomicAdd(&list_n, 1u);
            if (n < LIST) list[n] = (unsigned short)((j * PART_THREADS + tid) * N + i);
          }
        }
      }
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) { all += __shfl_xor(all, o); if (some_out) in += __shfl_xor(in, o); }
  if (lane == 0) { wave_sum[wave][0] = all; wave_sum[wave][1] = some_out ? in : all; }
  __syncthreads();
  if (tid == 0) {
    a.sums[mine] = {(uint64_t)__builtin_rint((wave_sum[0][0] + wave_sum[1][0]) + (wave_sum[2][0] + wave_sum[3][0])),
                    (uint64_t)__builtin_rint((wave_sum[0][1] + wave_sum[1][1]) + (wave_sum[2][1] + wave_sum[3][1]))};
    place = list_n ? atomicAdd((unsigned*)&a.state[row].list_n, list_n) : 0u;
  }
  __syncthreads();
  for (unsigned i = tid; i < min(list_n, (unsigned)LIST); i += PART_THREADS)
    if (place + i < LIST) {
      const int id = part * (PART_THREADS * PER) + list[i];
      a.list[(int64_t)row * LIST + place + i] = (uint64_t)key_of(tame(to_f32(r.p[id]))) << 32 | (unsigned)~id;
    }
}

struct Tally { uint64_t sum; unsigned cnt, lo, hi; };          // of tokens: what they weigh, how many, least and largest key
struct Shared {
  Sums sums;
  Tally tallies[2][WAVES];
  uint64_t sub_sum[THREADS];           // a division: a thread a bin
  unsigned sub_cnt[THREADS];
  uint64_t part_sum[MOST_PARTS];       // what is in
  unsigned part_ties[MOST_PARTS];
  uint64_t few[FEW], few_weight[FEW], ranked[FEW], ranked_weight[FEW];
  // what one thread found
  uint64_t found_sum;
  unsigned found_cnt, found_n, found_bin, few_n;
};
struct Cut {
  unsigned key;                        // what is above it is in
  unsigned ties;                       // and so many of those at it, by id
};

// LIMITS: of some row.  The list's tokens and their weights are in registers, EACH a thread.
template <typename T, bool ALIGNED, bool LIMITS>
__global__ __launch_bounds__(THREADS, 4) void k_sample_pick(SampleArgs a) {
  __shared__ Shared s;
  constexpr int N = Row<T, ALIGNED>::N, EACH = LIST / THREADS;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.x, vocab = a.vocab, shift = a.shift;
  int turn = 0, tally_turn = 0;
  // all that may be wanted is asked for at once
  const Limits lim = limits(a, row);
  const Row<T, ALIGNED> r(a, row);
  const Parts parts(a, row);
  const float u = a.u[row];
  RowState st{COLLECT, 0, -1, 0u, vocab, 0.f, 0.f};
  PartSums mine{0, 0};
  uint64_t listed_first = 0;
  if (LIMITS && !one_list(a)) {
    st = a.state[row];
    if (tid < a.parts) mine = a.sums[(int64_t)row * a.parts + tid];
    listed_first = a.list[(int64_t)row * LIST + tid];
  }
  float top;
  int top_at;
  parts.largest(top, top_at);
  if (!draws(lim) || top_at < 0) {     // nothing to choose, or the first of the order
    if (tid == 0) {
      const bool none = !lim.valid || top_at < 0;
      a.ids[row] = none ? -1 : top_at;
      if (a.probs) a.probs[row] = none ? 0.f : 1.f;
    }
    return;
  }
  const bool narrow = LIMITS && limited(lim);
  const Weigher weight{(double)top, octaves(lim)};
  const double uu = u > 0.f ? (double)fminf(u, 0.99999994f) : 0.0;
  const uint64_t least = lim.by_part ? max(1ull, (uint64_t)__builtin_rint(__builtin_ldexp((double)fminf(lim.min_p, 1.f), shift))) : 1ull;
  Cut cut{0u, 0u};                     // all is in
  uint64_t own = 0;                    // of this lane's parts: what is in
  unsigned own_ties = 0;

  if (narrow) {
    const bool listed = st.mode == COLLECT;
    const unsigned listed_n = listed ? min((unsigned)st.list_n, (unsigned)LIST) : 0u;
    const bool from_top = listed && st.first == 0;
    unsigned key[EACH];
    int id[EACH];
    uint64_t q_of[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const unsigned i = tid + e * THREADS;
      key[e] = 0; id[e] = 0; q_of[e] = 0;
      if (i < listed_n) {
        if (one_list(a)) {
          key[e] = key_of(tame(to_f32(r.p[i])));
          id[e] = (int)i;
        } else {
          const uint64_t l = e == 0 ? listed_first : a.list[(int64_t)row * LIST + i];
          key[e] = (unsigned)(l >> 32);
          id[e] = (int)~(unsigned)l;
        }
        q_of[e] = weight.whole(of_key(key[e]), shift);
      }
    }
    // f(key, id, weight) for the listed tokens, or all of the row, that weigh anything and whose key passes
    auto tokens = [&](auto pass, auto f) {
      if (listed) {
#pragma unroll
        for (int e = 0; e < EACH; ++e)
          if (q_of[e] && pass(key[e])) f(key[e], id[e], q_of[e]);
      } else {
#pragma unroll 1
        for (int at = tid * N; at < vocab; at += THREADS * N) {
          float x[N];
          r.load(at, x);
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const unsigned k = key_of(tame(x[i]));
            const uint64_t q = x[i] > -INFINITY && pass(k) ? weight.whole(of_key(k), shift) : 0ull;
            if (q) f(k, at + i, q);
          }
        }
      }
    };
    auto tally = [&](auto pass) {
      Tally v{0, 0u, ~0u, 0u};
      tokens(pass, [&](unsigned k, int, uint64_t q) { v.sum += q; ++v.cnt; v.lo = min(v.lo, k); v.hi = max(v.hi, k); });
      v = {wave_total(v.sum), wave_total(v.cnt), lane_of(running(v.lo, ~0u, Least()), 63), lane_of(running(v.hi, 0u, Most()), 63)};
      tally_turn ^= 1;
      if (lane == 0) s.tallies[tally_turn][wave] = v;
      __syncthreads();
      v = s.tallies[tally_turn][lane & (WAVES - 1)];
      constexpr int LAST = WAVES - 1;
      return Tally{lane_of(running_row(v.sum, 0u, Plus()), LAST), lane_of(running_row(v.cnt, 0u, Plus()), LAST),
                    lane_of(running_row(v.lo, ~0u, Least()), LAST), lane_of(running_row(v.hi, 0u, Most()), LAST)};
    };
    if (tid == 0) s.few_n = 0;
    s.part_sum[tid] = listed ? mine.in : 0ull;
    s.part_ties[tid] = 0;
    const uint64_t q0 = from_top || !listed ? 0ull : before(s.sums, turn, mine.all);         // of those before the list
    const unsigned c0 = listed && !from_top ? st.before : 0u;
    Tally left = tally([](unsigned) { return true; });       // (its barrier: all of the above is there)
    const uint64_t all_in = q0 + left.sum;
    // Among the tokens of `left`, c0 and q0 before them: the cut after `count` tokens (by_sum: before the first one with `goal` or more before it).
    auto find = [&](const bool by_sum, unsigned count, uint64_t goal) {
      unsigned n = left.cnt, c = c0, k_lo = left.lo, k_hi = left.hi, bin = 0;
      uint64_t q = q0;
      // Equal steps of the logits first, as what is listed is spread over them.  Then, where more than a few lie in one of them, the keys' bits, ten at a time.
      bool equal_steps = true, in_step = false;
      const float hi = of_key(k_hi), per = ((float)THREADS - 0.1f) / (hi - of_key(k_lo));
      auto step = [&](unsigned k) { return min((unsigned)((hi - of_key(k)) * per), (unsigned)THREADS - 1u); };
#pragma unroll 1
      for (int level = 0; level < 8; ++level) {
        if (k_lo == k_hi) {            // equal ones: as many as there is room for
          const uint64_t w = max(1ull, weight.whole(of_key(k_lo), shift));
          cut = {k_lo, (unsigned)(by_sum ? min((uint64_t)n, (goal - q - 1) / w + 1) : (uint64_t)min(n, count - c))};
          return;
        }
        auto pass = [&](unsigned k) { return k >= k_lo && k <= k_hi && (!in_step || step(k) == bin); };
        if (n <= FEW) {                // each one's rank by comparing it with all
          tokens(pass, [&](unsigned k, int i, uint64_t w) {
            const unsigned at = atomicAdd(&s.few_n, 1u) & (FEW - 1);
            s.few[at] = (uint64_t)k << 32 | (unsigned)~i;
            s.few_weight[at] = w;
          });
          __syncthreads();
          if (tid == 0) s.few_n = 0;
          const uint64_t token = lane < (int)n ? s.few[lane] : 0ull;
#pragma unroll
          for (int e = 0; e < FEW / WAVES; ++e) {
            const int i = __builtin_amdgcn_readfirstlane(wave) * (FEW / WAVES) + e;
            const int rank = __popcll(__builtin_amdgcn_ballot_w64(token > lane_of(token, i)));
            if (lane == i && i < (int)n) { s.ranked[rank] = token; s.ranked_weight[rank] = s.few_weight[i]; }
          }
          __syncthreads();
          const unsigned k = lane < (int)n ? (unsigned)(s.ranked[lane] >> 32) : 0u;
          bool in = lane < (int)n;
          if (by_sum) {
            const uint64_t w = in ? s.ranked_weight[lane] : 0ull;
            in = in && q + running_sum(w) - w < goal;
          } else {
            in = in && c + lane < count;
          }
          const unsigned last = lane_of(k, max(__popcll(__builtin_amdgcn_ballot_w64(in)) - 1, 0));          // (what is in is a prefix of the ranking)
          cut = {last, (unsigned)__popcll(__builtin_amdgcn_ballot_w64(in && k == last))};
          return;
        }
        if (in_step) {                 // more than a few in one step: their keys
          left = tally(pass);
          k_lo = left.lo; k_hi = left.hi;
          in_step = false;
          continue;
        }
        const int by = max(0, 32 - __clz(k_hi - k_lo) - 10);   // THREADS = 2^10 bins
        s.sub_cnt[tid] = 0;
        if (by_sum) s.sub_sum[tid] = 0;
        __syncthreads();
        tokens(pass, [&](unsigned k, int, uint64_t w) {
          const unsigned b = equal_steps ? step(k) : (k_hi - k) >> by;
          atomicAdd(&s.sub_cnt[b], 1u);
          if (by_sum) atomicAdd((unsigned long long*)&s.sub_sum[b], (unsigned long long)w);
        });
        __syncthreads();
        const unsigned m = s.sub_cnt[tid];
        if (by_sum) {
          const uint64_t w = s.sub_sum[tid];
          uint64_t ahead = w;
          before(s.sums, turn, ahead);
          ahead += q;
          if (m && ahead < goal && goal <= ahead + w) { s.found_sum = ahead; s.found_n = m; s.found_bin = tid; }
        } else {
          unsigned ahead = m;
          before(s.sums, turn, ahead);
          ahead += c;
          if (m && ahead < count && count <= ahead + m) { s.found_cnt = ahead; s.found_n = m; s.found_bin = tid; }
        }
        __syncthreads();
        bin = s.found_bin; n = s.found_n;
        if (by_sum) q = s.found_sum;
        else c = s.found_cnt;
        if (equal_steps) {
          equal_steps = false;
          in_step = true;
        } else {
          const uint64_t down = ((uint64_t)bin + 1) << by;
          const unsigned below = down - 1 >= (uint64_t)(k_hi - k_lo) ? k_lo : k_hi - (unsigned)(down - 1);
          k_hi -= bin << by;
          k_lo = below;
        }
      }
    };
    uint64_t to_cut = all_in;          // what is in by count
    if (lim.by_count && (unsigned)lim.top_k <= c0 + left.cnt) {        // (otherwise no more than that weigh anything)
      find(false, (unsigned)lim.top_k, 0);
      if (lim.by_sum) {                // (all that weighs anything is in the list)
        const unsigned in = cut.key;
        left = tally([&](unsigned k) { return k >= in; });
        to_cut = left.sum - (left.cnt - (unsigned)lim.top_k) * weight.whole(of_key(in), shift);
      }
    }
    if (lim.by_sum) {
      uint64_t of = to_cut;
      if (!lim.by_count) {             // of all tokens, by the parts' sums, however the cut is found
        of = 0;
        parts.all([&](int, const Part& p) { of += part_weight(p, weight, shift); });
        of = wave_total(of);
      }
      // (tokens of less than half a unit count in the parts' sums: nothing behind the list)
      find(true, ~0u, min(sum_goal(lim.top_p, of), to_cut));
    }
    // what of the list is in, by parts
    const int log2_part = 31 - __clz(a.part);
    uint64_t in = 0;
    unsigned ties = 0;
    tokens([&](unsigned k) { return k >= cut.key; }, [&](unsigned k, int i, uint64_t q) {
      if (q < least) return;
      if (a.parts == 1) {
        if (k > cut.key) in += q;
        else ++ties;
      } else if (k > cut.key) {
        atomicAdd((unsigned long long*)&s.part_sum[i >> log2_part], (unsigned long long)q);
      } else {
        atomicAdd(&s.part_ties[i >> log2_part], 1u);
      }
    });
    if (a.parts == 1) {                // (all atomics would meet in one place)
      in = wave_total(in);
      ties = wave_total(ties);
      if (lane == 0 && in) atomicAdd((unsigned long long*)&s.part_sum[0], (unsigned long long)in);
      if (lane == 0 && ties) atomicAdd(&s.part_ties[0], ties);
    }
    __syncthreads();
  }

  // the part in which the target lies; of tokens at the cut's logit the first by id are in
  const uint64_t tie_q = cut.key ? weight.whole(of_key(cut.key), shift) : 0ull;
  // Of half a unit and more, against the row's largest.  Without limits a part's sum has what is less in it also: a part of nothing else has no weight, and of
  // another's tokens those of less are not taken, whatever they are against its own largest.
  auto counts = [&](float l) { return ((double)l - weight.top) * weight.scale > -(double)(shift + 1); };
  auto of_part = [&](int p, const Part& part, unsigned& ties) {        // ties aside
    ties = narrow && p < a.parts ? s.part_ties[p] : 0u;
    return narrow ? (p < a.parts ? s.part_sum[p] : 0ull) : counts(part.top) ? part_weight(part, weight, shift) : 0ull;
  };
  parts.all([&](int p, const Part& part) {
    unsigned ties;
    own += of_part(p, part, ties);
    own_ties += ties;
  });
  auto taken = [&](unsigned ties, unsigned ahead) { return tie_q * min(ties, cut.ties - min(ahead, cut.ties)); };
  unsigned ties_ahead = running_sum(own_ties) - own_ties;
  own += taken(own_ties, ties_ahead);
  uint64_t ahead = running_sum(own);
  const uint64_t total = lane_of(ahead, 63), target = min((uint64_t)(uu * (double)total), total - 1);
  ahead -= own;
  const int at_lane = max(__ffsll((unsigned long long)__builtin_amdgcn_ballot_w64(target >= ahead && target < ahead + own)) - 1, 0);
  int part = at_lane * parts.each;
  float part_top = __uint_as_float(lane_of(__float_as_uint(parts.mine.top), at_lane));
  uint64_t part_in = lane_of(own, at_lane), part_ahead = lane_of(ahead, at_lane);
  unsigned part_ties = lane_of(ties_ahead, at_lane);
  if (parts.each > 1) {                // which one of the lane's
#pragma unroll 1
    for (;; ++part) {
      const Part p = part < a.parts ? parts.p[part] : Part{-INFINITY, -1, 0.0};
      unsigned ties;
      part_in = of_part(part, p, ties);
      part_in += taken(ties, part_ties);
      part_top = p.top;
      if (target < part_ahead + part_in || part + 1 >= a.parts) break;
      part_ahead += part_in;
      part_ties += ties;
    }
  }
  // A run of its logits for every thread.  Without limits weights are taken against the part's largest, as its sum was.
  const Weigher local{narrow ? (double)top : (double)part_top, weight.scale};
  constexpr int RUN = 8, HALF = 4;     // (a part has 4 or 8 times THREADS)
  const int run = a.part / THREADS, from = part * a.part + tid * run, to = min(min(from + run, (part + 1) * a.part), vocab);
  float x[RUN];
#pragma unroll
  for (int i = 0; i < RUN; i += HALF) {
    float v[HALF];
    r.load(i < run ? min(from + i, vocab) : vocab, v);
#pragma unroll
    for (int e = 0; e < HALF; ++e) x[i + e] = v[e];
  }
  // the weight of what is in for certain, and whether it is one of the equal ones at the cut
  auto take = [&](float v, int i, bool& tie) {
    v = tame(v);
    const unsigned k = key_of(v);
    const uint64_t q = from + i < to && v > -INFINITY && k >= cut.key && (narrow || counts(v)) ? local.whole(v, shift) : 0ull;
    tie = q >= least && k == cut.key;
    return q >= least && k > cut.key ? q : 0ull;
  };
  uint64_t sum = 0, q_of[RUN];
  unsigned ties = 0, tie_at = 0;
#pragma unroll
  for (int i = 0; i < RUN; ++i) {
    bool tie;
    sum += q_of[i] = take(x[i], i, tie);
    ties += tie;
    tie_at |= (unsigned)tie << i;
  }
  const uint64_t own_sum = sum;
  const unsigned own_count = ties;
  unsigned all_ties = 0;
  uint64_t in_part = before(s.sums, turn, sum, ties);  // of the threads before
  all_ties = lane_of(running_row(s.sums.cnt[turn][lane & (WAVES - 1)], 0u, Plus()), WAVES - 1);
  const unsigned left0 = cut.ties - min(part_ties, cut.ties), left = cut.ties - min(part_ties + ties, cut.ties);
  // The part's sum was of weights before they were rounded, or against its own largest: the target in the units of this one.
  in_part += tie_q * min(all_ties, left0);
  if (in_part == 0) {                  // (a part of nothing but less than half units: the largest stands for it)
    if (tid == 0) {
      a.ids[row] = top_at;
      if (a.probs) a.probs[row] = (float)(__builtin_ldexp(1.0, shift) / (double)total);
    }
    return;
  }
  const uint64_t goal = min((uint64_t)((double)(target - part_ahead) / (double)part_in * (double)in_part), in_part - 1);
  const double share = (double)part_in / (double)in_part / (double)total;
  uint64_t at_q = sum + tie_q * (left0 - left);
  if (goal >= at_q && goal < at_q + own_sum + tie_q * min(own_count, left)) {
    unsigned more = left;
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
      uint64_t q = q_of[i];
      if (tie_at >> i & 1u && more) { q = tie_q; --more; }
      if (goal >= at_q && goal < at_q + q) {
        a.ids[row] = from + i;
        if (a.probs) a.probs[row] = (float)((double)q * share);
      }
      at_q += q;
    }
  }
}

// Logits of a part: as many as a thread's registers hold with ease (32) where there are many; half of them where a short launch is spread over more CUs.  Measured
// with halves and wholes, no limits / top-k 50 / top-p 0.9 / both, us: 1 row of 128256  9.5 / 23.9 / 31.8 / 27.4 and 10.8 / 24.2 / 33.6 / 27.7; 8 rows  9.6 / 26.3 / 34.2 /
// 29.8 and 11.3 / 25.1 / 36.0 / 28.5; 32 rows (1024 parts, the last halves)  12.2 / 31.2 / 42.8 / 34.6 and 13.0 / 27.8 / 40.9 / 31.1; 64 rows  16.6 / 36.4 / 53.4 / 40.0 and
// 17.8 / 32.7 / 53.4 / 36.0; 128 rows  24.1 / 46.7 / 74.3 / 50.7 and 24.8 / 40.3 / 73.1 / 44.7.  Without limits halves are ahead up to 128 rows, with top-k wholes from 8 on:
// the rule lies between them.  It looks at no limits, so that a row with limits that leave everything has the parts, and the sums to the bit, of one without.
constexpr int SMALL_PARTS = 1024;
void divide(SampleArgs& a, int rows) {
  a.part = (int64_t)rows * ((a.vocab + 4095) / 4096) > SMALL_PARTS ? 8192 : 4096;
  a.parts = (a.vocab + a.part - 1) / a.part;
}

// the workspace's arrays for so many rows, behind one another; its bytes
size_t place(SampleArgs& a, int rows, char* base) {
  const size_t parts = (size_t)rows * a.parts;
  size_t at = 0;
  auto take = [&](size_t bytes) { char* p = base + at; at += (bytes + 15) / 16 * 16; return p; };
  a.tops = (Part*)take(parts * sizeof(Part));
  if (a.vocab <= LIST) return at;
  a.sums = (PartSums*)take(parts * sizeof(PartSums));
  a.bins = (uint64_t*)take(parts * BINS * 8);
  a.maxima = (float*)take(parts * PART_THREADS * 4);
  a.state = (RowState*)take(rows * sizeof(RowState));
  a.list = (uint64_t*)take((size_t)rows * LIST * 8);
  return at;
}

template <typename T, bool ALIGNED>
hipError_t launch(hipStream_t st, const SampleArgs& a, int rows) {
  const dim3 grid(a.parts, rows), wg(PART_THREADS);
  const bool wide = a.part == 8192;
  if (wide) hipLaunchKernelGGL((k_sample_parts<T, ALIGNED, 32>), grid, wg, 0, st, a);
  else hipLaunchKernelGGL((k_sample_parts<T, ALIGNED, 16>), grid, wg, 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if ((a.top_k || a.top_p || a.min_p) && a.vocab > LIST) {
    hipLaunchKernelGGL(k_sample_edges, dim3(rows), dim3(THREADS), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (wide) hipLaunchKernelGGL((k_sample_collect<T, ALIGNED, 32>), grid, wg, 0, st, a);
    else hipLaunchKernelGGL((k_sample_collect<T, ALIGNED, 16>), grid, wg, 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.top_k || a.top_p || a.min_p) hipLaunchKernelGGL((k_sample_pick<T, ALIGNED, true>), dim3(rows), dim3(THREADS), 0, st, a);
  else hipLaunchKernelGGL((k_sample_pick<T, ALIGNED, false>), dim3(rows), dim3(THREADS), 0, st, a);
  return hipGetLastError();
}

// A lot of rows at a time; the rows' arrays move along.
template <typename T>
hipError_t launch_rows(hipStream_t st, SampleArgs a, int rows) {
  const bool aligned = (uintptr_t)a.logits % 16 == 0 && (rows == 1 || a.stride * sizeof(T) % 16 == 0);       // (of one row the stride is not used)
  for (int i = 0;; ++i) {
    const auto [done, n] = sample_lot(rows, i);
    if (n == 0) return hipSuccess;
    SampleArgs b = a;
    b.logits = (const T*)a.logits + done * a.stride;
    if (a.temperature) b.temperature += done;
    if (a.top_k) b.top_k += done;
    if (a.top_p) b.top_p += done;
    if (a.min_p) b.min_p += done;
    b.u += done; b.ids += done;
    if (a.probs) b.probs += done;
    const hipError_t e = aligned ? launch<T, true>(st, b, n) : launch<T, false>(st, b, n);
    if (e != hipSuccess) return e;
  }
}

bool too_large(int vocab) { return vocab > MOST_PARTS * 4096; }

}  // namespace

SampleLot sample_lot(int rows, int i) {
  const int64_t first = std::min<int64_t>((int64_t)i * ROWS_AT_ONCE, rows);
  return {first, (int)std::min<int64_t>(rows - first, ROWS_AT_ONCE)};
}

extern "C" size_t esp_sample_scratch_bytes(int32_t rows, int32_t vocab) {
  if (rows < 1 || vocab < 1 || too_large(vocab)) return 0;
  // (what the most rows with small parts want can be more than what more rows do: enough for those also)
  const int small = std::min(rows, SMALL_PARTS / ((vocab + 4095) / 4096));
  size_t most = 0;
  for (const int n : {std::min(rows, ROWS_AT_ONCE), std::min(std::max(small, 1), ROWS_AT_ONCE)}) {
    SampleArgs a{};
    a.vocab = vocab;
    divide(a, n);
    most = std::max(most, place(a, n, nullptr));
  }
  return most;
}

extern "C" esp_status esp_sample(void* stream, int32_t dtype, const void* logits, int64_t row_stride, int32_t rows, int32_t vocab,
                                 const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, const float* u,
                                 int32_t* ids, float* probs, void* scratch, size_t scratch_bytes) {
  if (!logits || !u || !ids || rows < 0 || vocab < 1) return ESP_EINVAL;
  if (dtype != ESP_F32 && dtype != ESP_BF16) return ESP_EDTYPE;
  if (row_stride < vocab) return ESP_ESHAPE;
  if (too_large(vocab)) return ESP_ECAPACITY;
  if (rows == 0) return ESP_OK;
  if (!scratch || scratch_bytes < esp_sample_scratch_bytes(rows, vocab)) return ESP_ECAPACITY;
  if ((uintptr_t)scratch % 16) return ESP_EINVAL;
  int log2_vocab = 0;
  while ((1 << log2_vocab) < vocab) ++log2_vocab;
  SampleArgs a{};
  a.logits = logits; a.stride = row_stride; a.vocab = vocab;
  a.shift = std::min(45, 62 - log2_vocab);
  divide(a, std::min(rows, ROWS_AT_ONCE));
  a.temperature = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p; a.u = u; a.ids = ids; a.probs = probs;
  place(a, std::min(rows, ROWS_AT_ONCE), (char*)scratch);
  const hipError_t e = dtype == ESP_F32 ? launch_rows<float>((hipStream_t)stream, a, rows) : launch_rows<bf16_t>((hipStream_t)stream, a, rows);
  return e == hipSuccess ? ESP_OK : ESP_EDEVICE;
}
