// What the kernels of the paged attention share: one unit of 32 keys for a wave's 32 query columns, bf16 or fp32.
//
// S^T = K Q^T and O^T = V^T P^T on 32 x 32 matrix instructions (bf16: 16 features or keys at a time; fp32: two).  Computing the
// transposed scores leaves a lane with one query column and 16 keys of the unit, register v <-> key 8 (v / 4) + 4 half + v % 4, which is
// the operand layout P^T needs: the probabilities never leave registers.  The cache's block order (esp_kv) is what the other operands
// need, a lane's share of a fragment being eight consecutive elements: of K the features 16 s + 8 half + 0..7 of key lane % 32, of V the
// keys 16 u + 8 (j / 4) + 4 half + j % 4 of feature lane % 32.
#pragma once

#include "esp_internal.h"

typedef __attribute__((ext_vector_type(8))) float f32x8_t;
template <typename T> struct AttnFrag;
template <> struct AttnFrag<bf16_t> { typedef bf16x8_t type; };
template <> struct AttnFrag<float> { typedef f32x8_t type; };

__device__ __forceinline__ f32x16_t attn_mma(bf16x8_t a, bf16x8_t b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
// element e of both halves: two of the contraction's terms an instruction
__device__ __forceinline__ f32x16_t attn_mma(f32x8_t a, f32x8_t b, f32x16_t c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

__device__ __forceinline__ float attn_sum_of_halves(float v) {
  const unsigned u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

constexpr float ATTN_UNSEEN = -1.0e30f;      // score of a hidden key, and start of a column's running maximum
constexpr float ATTN_SLACK = 24.0f;          // powers of two by which a score may exceed the exponents' reference before that moves

// written as text: of fmaxf the compiler makes a second instruction for every operand that might be a signalling NaN
__device__ __forceinline__ float attn_max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
// max with the lane 32 places away, which holds the column's other keys
__device__ __forceinline__ float attn_max_of_halves(float v) {
  const unsigned u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const float a = __uint_as_float(r[0]), b = __uint_as_float(r[1]);
  return attn_max3(a, b, b);
}

// Online softmax of a unit's scores: p = 2^(scale s - scale m) with m the running maximum, followed lazily (the sums hold 2^24 times the
// largest probability without loss), the probabilities as operand fragments (bf16: rounded to it, 2^-8 of a probability at most, as the
// matrix product takes them; the sum l is of the unrounded ones).  seen: bits of this lane's keys, at 8 (v / 4) + v % 4.
template <typename T, int DB>
__device__ __forceinline__ void attn_softmax(f32x16_t& sc, bool masked, unsigned seen, float scale, f32x16_t (&o)[DB], float& m, float& l,
                                             typename AttnFrag<T>::type (&p)[2]) {
  if (masked) {
#pragma unroll
    for (int v = 0; v < 16; ++v) sc[v] = ((seen >> (8 * (v >> 2) + (v & 3))) & 1u) ? sc[v] : ATTN_UNSEEN;
  }
  float top = sc[0];
#pragma unroll
  for (int v = 1; v < 15; v += 2) top = attn_max3(top, sc[v], sc[v + 1]);
  top = attn_max3(top, sc[15], sc[15]);
  top = attn_max_of_halves(top);
  const float m_new = top * scale > m * scale + ATTN_SLACK ? top : m;
  // nothing seen so far: any finite reference makes the hidden keys' probabilities zero
  const float mb = m_new > 0.5f * ATTN_UNSEEN ? m_new * scale : 0.f;
  const bool moved = m_new != m && m > 0.5f * ATTN_UNSEEN;
  if (__builtin_amdgcn_ballot_w64(moved) != 0ull) {
    const float alpha = m > 0.5f * ATTN_UNSEEN ? __builtin_amdgcn_exp2f(m * scale - mb) : 1.0f;
    l *= alpha;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[i][v] *= alpha;
  }
  m = m_new;
  __builtin_amdgcn_sched_barrier(0);
  float sum = 0.f;
#pragma unroll
  for (int c = 0; c < 4; ++c) {       // four at a time: sixteen exponentials in flight would cost the registers of other operands
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int v = 4 * c + e;
      const float x = __builtin_amdgcn_exp2f(fmaf(sc[v], scale, -mb));
      sum += x;
      p[v >> 3][v & 7] = from_f32<T>(x);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  l += sum;
}

// (m, l) of two parts of a column's keys, weights for what each has summed up; a part that saw no key weighs nothing
__device__ __forceinline__ float attn_weight(float m, float top, float scale) {
  return m > 0.5f * ATTN_UNSEEN ? __builtin_amdgcn_exp2f((m - top) * scale) : 0.f;
}

// Bits of 32 keys of a unit that begins c_lo places behind the first row of the chunk (negative: before it), of nr rows: committed keys, and
// of the chunk the rows up to r (anc null) or those in the row's ancestor bitset.
__device__ __forceinline__ unsigned attn_low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }
template <typename WORD>                          // word(i): of the row's ancestor bitset, 0 from its end on
__device__ __forceinline__ unsigned attn_tree_window(WORD word, int c_lo, int nr) {
  if (c_lo <= -32) return ~0u;
  uint64_t w;
  if (c_lo < 0) {
    w = (word(0) << -c_lo) | ((1ull << -c_lo) - 1ull);
  } else {
    const int i = c_lo >> 6, sh = c_lo & 63;
    const uint64_t a = word(i), b = word(i + 1);
    w = sh ? (a >> sh) | (b << (64 - sh)) : a;
  }
  return (unsigned)w & attn_low_bits(nr - c_lo);  // (keys of the sequence in the unit)
}
__device__ __forceinline__ unsigned attn_window(const uint64_t* anc, int anc_words, int r, int c_lo, int nr) {
  if (!anc) return c_lo <= -32 ? ~0u : attn_low_bits(min(r, nr - 1) + 1 - c_lo);
  return attn_tree_window([&](int i) { return i < anc_words ? anc[i] : 0ull; }, c_lo, nr);
}

// takes infinities and NaN (all bits of the exponent set) out of a fragment; ones in their places, zeros elsewhere
__device__ __forceinline__ bf16x8_t attn_take_odd(bf16x8_t& f) {
  u32x4_t w = __builtin_bit_cast(u32x4_t, f), ones;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned t = ((w[i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u, odd = (t >> 15) * 0xffffu;
    ones[i] = odd & 0x3f803f80u;
    w[i] &= ~odd;
  }
  f = __builtin_bit_cast(bf16x8_t, w);
  return __builtin_bit_cast(bf16x8_t, ones);
}
__device__ __forceinline__ f32x8_t attn_take_odd(f32x8_t& f) {
  f32x8_t ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool odd = (__float_as_uint(f[i]) & 0x7f800000u) == 0x7f800000u;
    ones[i] = odd ? 1.f : 0.f;
    f[i] = odd ? 0.f : f[i];
  }
  return ones;
}
// what is in a fragment's places: infinities 1, negative ones 64, NaN 4096, anything else 0, so that up to 63 of each can be told from their sum
__device__ __forceinline__ float attn_odd_mark(unsigned f32_bits) {
  if ((f32_bits & 0x7f800000u) != 0x7f800000u) return 0.f;
  return f32_bits & 0x007fffffu ? 4096.f : f32_bits >> 31 ? 64.f : 1.f;
}
__device__ __forceinline__ bf16x8_t attn_odd_marks(bf16x8_t f) {
  u32x4_t w = __builtin_bit_cast(u32x4_t, f);
#pragma unroll
  for (int i = 0; i < 4; ++i) {                    // (1, 64 and 4096 are bf16 numbers)
    const unsigned lo = __float_as_uint(attn_odd_mark(w[i] << 16)), hi = __float_as_uint(attn_odd_mark(w[i] & 0xffff0000u));
    w[i] = lo >> 16 | hi;
  }
  return __builtin_bit_cast(bf16x8_t, w);
}
__device__ __forceinline__ f32x8_t attn_odd_marks(f32x8_t f) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = attn_odd_mark(__float_as_uint(f[i]));
  return f;
}
__device__ __forceinline__ bool attn_any(bf16x8_t f) {
  const u32x4_t w = __builtin_bit_cast(u32x4_t, f);
  return (w[0] | w[1] | w[2] | w[3]) != 0;
}
__device__ __forceinline__ bool attn_any(f32x8_t f) {
  float any = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) any += f[i];
  return any > 0.f;
}

// V of keys past the sequence's end (left keys of the unit are there) as zeros: memory there may hold anything, and 0 times NaN is NaN
__device__ __forceinline__ f32x8_t attn_zero_tail(f32x8_t f, int u, int lane, int left) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (16 * u + 8 * (j >> 2) + 4 * (lane >> 5) + (j & 3) >= left) f[j] = 0.f;
  return f;
}
__device__ __forceinline__ bf16x8_t attn_zero_tail(bf16x8_t f, int u, int lane, int left) {
  u32x4_t w = __builtin_bit_cast(u32x4_t, f);
#pragma unroll
  for (int i = 0; i < 4; ++i) {                   // a word holds keys k and k + 1
    const int k = 16 * u + 8 * (i >> 1) + 4 * (lane >> 5) + 2 * (i & 1);
    w[i] &= k + 1 < left ? 0xffffffffu : k < left ? 0x0000ffffu : 0u;
  }
  return __builtin_bit_cast(bf16x8_t, w);
}

// In a unit some of whose keys not every column sees, infinities and NaN among the values would reach the columns that do not see them, as 0
// times them.  So they are taken out there, and where that took any out (odd) the columns that do see them get theirs when all else is
// done: this adds what they see to the outputs, an infinity of its sign, or NaN for a NaN and for infinities of both signs.  v: the unit's
// fragments in memory; seen: bits of this lane's keys.
template <typename T, int HD>
__device__ __forceinline__ void attn_add_odd(const T* v, unsigned seen, int left, int lane, f32x16_t (&o)[HD / 32]) {
  typedef typename AttnFrag<T>::type frag_t;
  frag_t s[2];
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i >> 3][i & 7] = from_f32<T>((seen >> (8 * (i >> 2) + (i & 3))) & 1u ? 1.f : 0.f);
#pragma unroll
  for (int db = 0; db < HD / 32; ++db) {
    f32x16_t n;
#pragma unroll
    for (int i = 0; i < 16; ++i) n[i] = 0.f;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const frag_t f = attn_zero_tail(*reinterpret_cast<const frag_t*>(v + (2 * db + u) * 512 + lane * 8), u, lane, left);
      n = attn_mma(attn_odd_marks(f), s[u], n);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int marks = (int)n[i];                 // (32 keys: 32 of a kind at most)
      const float up = marks & 63 ? __builtin_inff() : 0.f, down = marks & 63 << 6 ? __builtin_inff() : 0.f, none = marks >> 12 ? __builtin_nanf("") : 0.f;
      o[db][i] += up - down + none;                // (infinity less infinity is NaN)
    }
  }
}

// One unit out of LDS, in fp32.  k, v: this lane's share of the unit's first K and first V fragment, fragments FRAG bytes apart, of V (db, u) at
// 2 db + u.  seen: bits of this lane's keys, looked at where `masked`.
// Fragments are read a matrix step ahead and held there (left to itself the compiler reads them all and runs out of registers); the matrix
// phases run at raised wave priority, so that of the waves of a SIMD one has matrix work and the others fill in with their softmax.
template <int HD>
__device__ __forceinline__ void attn_unit(const unsigned char* k, const unsigned char* v, bool masked, unsigned seen, float scale,
                                          const f32x8_t (&q)[HD / 16], f32x16_t (&o)[HD / 32], float& m, float& l) {
  typedef f32x8_t frag_t;
  constexpr int NS = HD / 16, DB = HD / 32, FRAG = 512 * sizeof(float), PF = 1, NF = PF + 1;
  frag_t fr[NF];
  // fragment j: K steps 0 .. NS - 1, then V in the order (u, db)
  auto frag_at = [&](int j) {
    const int i = j - NS;
    return j < NS ? *reinterpret_cast<const frag_t*>(k + j * FRAG) : *reinterpret_cast<const frag_t*>(v + (i % DB * 2 + i / DB) * FRAG);
  };
  f32x16_t sc;
#pragma unroll
  for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
  for (int j = 0; j < PF; ++j) fr[j] = frag_at(j);
  __builtin_amdgcn_s_setprio(2);
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    fr[(j + PF) % NF] = frag_at(j + PF);
    __builtin_amdgcn_sched_barrier(0);
    sc = attn_mma(fr[j % NF], q[j], sc);
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_setprio(0);
  frag_t p[2];
  attn_softmax<float, DB>(sc, masked, seen, scale, o, m, l, p);
  __builtin_amdgcn_s_setprio(2);
#pragma unroll
  for (int i = 0; i < 2 * DB; ++i) {              // i = u DB + db
    if (i + PF < 2 * DB) fr[(NS + i + PF) % NF] = frag_at(NS + i + PF);
    __builtin_amdgcn_sched_barrier(0);
    o[i % DB] = attn_mma(fr[(NS + i) % NF], p[i / DB], o[i % DB]);
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_setprio(0);
}
