// Device helpers shared by the routing kernels.
#pragma once

#include "rr_internal.h"

namespace rr {

constexpr int kMaxRank = kMaxK + 1;

// Ranking key of a (score, expert) pair: the order-preserving image of the score, then the complement of the expert index
// (Eq. 1 argtopk, ties -> lower expert index).  A greater key is a better rank and the keys of different experts never
// tie.  The 38 bits sit in the bits of a positive double - 18 bits of the image behind an exponent that keeps it normal, the
// other 14 and the 6 of the expert in the low word - so the order is that of doubles, and a compare-exchange is one v_max_f64
// and one v_min_f64 (a comparison of 64-bit integers and four selects before; figures at topk_rank_kernel).
// 0.0 lies below every real key and decodes to expert -1.
typedef double rank_t;
__device__ inline rank_t rank_key(float v, int e) {
  const u32 image = score_key(v);
  const u32 hi = 0x40000000u | (image >> 14), lo = (image << 18) | ((u32)(kMaxE - 1 - e) << 12);
  return __builtin_bit_cast(double, ((unsigned long long)hi << 32) | lo);
}
__device__ inline u32 rank_key_score(rank_t key) {
  return (u32)(__builtin_bit_cast(unsigned long long, key) >> 18);
}
__device__ inline int rank_key_expert(rank_t key) {
  const unsigned long long bits = __builtin_bit_cast(unsigned long long, key);
  return bits ? kMaxE - 1 - (int)((u32)bits >> 12 & (kMaxE - 1)) : -1;
}
static_assert(kMaxE == 64, "six bits of a ranking key hold the expert");
__device__ __forceinline__ rank_t rank_max(rank_t a, rank_t b) {
  rank_t r;
  asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ rank_t rank_min(rank_t a, rank_t b) {
  rank_t r;
  asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ inline rank_t rank_of_lane(rank_t key, int off) {  // the key of lane ^ off
  const unsigned long long bits = __builtin_bit_cast(unsigned long long, key);
  const u32 lo = __shfl_xor((u32)bits, off), hi = __shfl_xor((u32)(bits >> 32), off);
  return __builtin_bit_cast(double, ((unsigned long long)hi << 32) | lo);
}

// b[0] > b[1] > ... > b[N-1] are the N greatest keys seen so far: one compare-exchange per position.
template <int N>
__device__ inline void insert_key(rank_t (&b)[N], rank_t a) {
#pragma unroll
  for (int q = 0; q < N; ++q) {
    const rank_t hi = rank_max(a, b[q]);
    if (q + 1 < N) a = rank_min(a, b[q]);
    b[q] = hi;
  }
}

// Eq. 1 argtopk over experts [e0, e1) of one row of scores held in LDS: the N best keys, best first
// (positions past the number of experts stay 0).
template <int N>
__device__ inline void top_keys_of_range(const float *row, int e0, int e1, rank_t (&b)[N]) {
#pragma unroll
  for (int q = 0; q < N; ++q) b[q] = 0.0;
  for (int e = e0; e < e1; ++e) insert_key(b, rank_key(row[e], e));
}

// Sec. 4.1: best expert among those of one group, ties -> lower expert index.
__device__ inline void best_in_group(const float *row, int e0, int e1, float &best, int &arg) {
  best = row[e0];
  arg = e0;
  for (int e = e0 + 1; e < e1; ++e) {
    float v = row[e];
    if (v > best) { best = v; arg = e; }
  }
}

__device__ inline int lane_id() { return threadIdx.x & (kWave - 1); }

// Workgroup -> token block for kernels whose neighbouring token blocks write neighbouring words of
// the same per-expert arrays.  Workgroups are dealt to the 8 XCDs round-robin and each XCD has its
// own L2: with block = workgroup, one cache line would be completed piecewise from 8 L2s.  Here XCD
// x walks its own contiguous eighth of the blocks, so the pieces of a line meet in one L2.
__device__ inline int xcd_block(int g, int NB) {
  const int per = NB >> 3, main = per << 3;
  return g < main ? (g & 7) * per + (g >> 3) : g;
}

// Four words of random bits: Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as
// 1, 2, 3", SC 2011) at counter words (low, high, 0, 0) with the two words of `seed` as key.
__device__ inline void philox4x32_10(unsigned long long counter, unsigned long long seed, u32 (&out)[4]) {
  u32 c0 = (u32)counter, c1 = (u32)(counter >> 32), c2 = 0u, c3 = 0u, k0 = (u32)seed, k1 = (u32)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
    c0 = (u32)(b >> 32) ^ c1 ^ k0;
    c1 = (u32)b;
    c2 = (u32)(a >> 32) ^ c3 ^ k1;
    c3 = (u32)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  out[0] = c0; out[1] = c1; out[2] = c2; out[3] = c3;
}

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
// two fp32 -> packed bf16 pair, round to nearest even (v_cvt_pk_bf16_f32), first value in the low half
__device__ inline u32 pack_bf16(float a, float b) {
  const f32x2_t f = {a, b};
  return __builtin_bit_cast(u32, __builtin_convertvector(f, bf16x2_t));
}

// g Phi(g).  (A single polynomial for erfc in 1 / (1 + 0.45 |g|) is 3 us less of a 6161 x 2728 up projection, 55 us, but
// 5 times the error for |g| < 1: 41 of 2^20 normal arguments of sigma 0.3 round to another bf16 than g Phi(g) does, here 3.)
__device__ inline float gelu_erf(float g) { return 0.5f * g * (1.0f + erff(g * 0.70710678118654752f)); }

// exp(x) for x <= 0 to 2 u: 2^t with t the rounded x / ln 2, times 1 + ln 2 (x / ln 2 - t); 0 where it is below 2^-126, and for
// -infinity.  (Half of expf's instructions, which bind the loss.)
__device__ inline float exp_short(float x) {
  constexpr float kLog2e = 1.44269504088896341f, kLog2eLow = (float)(1.44269504088896341 - (double)kLog2e), kLn2 = 0.69314718055994531f;
  x = x < -104.0f ? -104.0f : x;  // (NaN stays)
  const float t = x * kLog2e, r = fmaf(x, kLog2eLow, fmaf(x, kLog2e, -t)), e = __builtin_amdgcn_exp2f(t);
  return fmaf(e * r, kLn2, e);
}

}  // namespace rr
