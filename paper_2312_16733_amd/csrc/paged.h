// What the autoregressive serving kernels share: the step's sequences, the paged key / value cache, 16-bit element types.
#pragma once
#include "common.h"
#include "paged_plan.h"

namespace sna {

typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

// Element types: eight of them are one 16-byte access and one operand of the matrix instructions.
struct Bf16 {
  static constexpr unsigned kInf = 0x7f80u, kOne = 0x3f80u;
  static constexpr bool kNarrow = false;                             // few powers of two: see Reference
  typedef __attribute__((ext_vector_type(8))) __bf16 v8;
  typedef __attribute__((ext_vector_type(4))) __bf16 v4;
  static __device__ __forceinline__ f32x4 mma16(u32x4 a, u32x4 b, f32x4 c) {     // 16 x 16 += 16 x 32 by 32 x 16
#if defined(__HIP_DEVICE_COMPILE__)
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
#endif
    return c;
  }
  static __device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c) {     // 32 x 32 += 32 x 16 by 16 x 32
#if defined(__HIP_DEVICE_COMPILE__)
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
#endif
    return c;
  }
};
struct Fp16 {
  static constexpr unsigned kInf = 0x7c00u, kOne = 0x3c00u;
  static constexpr bool kNarrow = true;
  typedef __attribute__((ext_vector_type(8))) _Float16 v8;
  typedef __attribute__((ext_vector_type(4))) _Float16 v4;
  static __device__ __forceinline__ f32x4 mma16(u32x4 a, u32x4 b, f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
    c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
#endif
    return c;
  }
  static __device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c) {
#if defined(__HIP_DEVICE_COMPILE__)
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
#endif
    return c;
  }
};
template <class T>
__device__ __forceinline__ f32x8 to_f32(u32x4 u) { return __builtin_convertvector(__builtin_bit_cast(typename T::v8, u), f32x8); }
template <class T>
__device__ __forceinline__ u32x4 to_16(f32x8 x) { return __builtin_bit_cast(u32x4, __builtin_convertvector(x, typename T::v8)); }   // to the nearest, ties to even

// Values that are no numbers, where the rows of a product differ in the keys they see: 0 * inf is not 0, so that such a value
// would reach rows that do not see its key.  They are taken out of the product, and counted for the rows that do see them by
// products of ones.  All of it happens in a second pass over the keys, of waves whose sums come out as no numbers: in the first,
// a look at the values of such tiles alone cost 4 to 11 % of a chunk.
enum Odd { ODD_NAN, ODD_INF, ODD_MINUS_INF, ODD_KINDS };
// In integers throughout: a comparison for each of a wave's values would take the scalar registers of the ordinary case.
__device__ __forceinline__ int ones_if_zero(int x) { return (x - 1) >> 31; }             // all ones, for x >= 0
template <class T>
__device__ __forceinline__ u32x4 without_odd(u32x4 v) {
#pragma unroll
  for (int w = 0; w < 4; ++w)
    v[w] &= ~((unsigned)ones_if_zero((int)(~v[w] & T::kInf)) & 0xffffu) & ~((unsigned)ones_if_zero((int)(~v[w] >> 16 & T::kInf)) << 16);
  return v;
}
template <class T>
__device__ __forceinline__ unsigned one_if_odd(unsigned h, int kind) {
  const int m = kind == ODD_NAN ? ((int)T::kInf - (int)(h & 0x7fffu)) >> 31 : ones_if_zero((int)(h ^ (kind == ODD_INF ? T::kInf : T::kInf | 0x8000u)));
  return (unsigned)m & T::kOne;
}
template <class T>
__device__ __forceinline__ u32x4 ones_where_odd(u32x4 v, int kind) {
#pragma unroll
  for (int w = 0; w < 4; ++w) v[w] = one_if_odd<T>(v[w] & 0xffffu, kind) | one_if_odd<T>(v[w] >> 16, kind) << 16;
  return v;
}
// Ones for the keys of key .. key + 7 that a row sees
template <class T>
__device__ __forceinline__ u32x4 ones_where_seen(int key, int low, int lim) {
  u32x4 v;
  const auto one = [&](int k) { return (unsigned)(~((k - low) | (lim - k)) >> 31) & T::kOne; };
#pragma unroll
  for (int w = 0; w < 4; ++w) v[w] = one(key + 2 * w) | one(key + 2 * w + 1) << 16;
  return v;
}
__device__ __forceinline__ float odd_sum(bool some, int kind) {      // what they add
  return some ? kind == ODD_NAN ? __builtin_nanf("") : kind == ODD_INF ? INFINITY : -INFINITY : 0.f;
}

// The rows of a step.  Sequence b brings rows starts[b] .. starts[b + 1] - 1; with them lens[b] of its tokens are cached.
// The arrays are the device's: what they hold is not known to the host, so every use below is clamped to what the host
// does know (T rows, `width` table columns, n_pages pages), and wrong contents give wrong results, never a wild access.
struct PagedSeqs {
  const int* starts; const int* lens; const int* table;
  int B, T, width, tstride;
  int max_len;                       // longer ones are taken to be this long
};
struct PagedKV {
  char* k; char* v;                  // [page][head][slot][dim], [page][head][dim][slot]
  long kstride, vstride;             // bytes between pages
  int n_pages, lps, heads;           // lps: log2(slots of a page)
};
struct Seq { int row0, n, len; };    // first row, new tokens, cached tokens with them

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }      // in scalar registers
__device__ __forceinline__ int clamped(int x, int lo, int hi) { return min(max(x, lo), hi); }
__device__ __forceinline__ Seq sequence(const PagedSeqs& s, int b) {
  const int r0 = clamped(s.starts[b], 0, s.T), r1 = clamped(s.starts[b + 1], 0, s.T);
  return Seq{r0, max(r1 - r0, 0), clamped(s.lens[b], 0, s.max_len)};
}
__device__ __forceinline__ Seq uniform(const Seq& q) { return Seq{uniform(q.row0), uniform(q.n), uniform(q.len)}; }
// The largest i of [0, n) with f(i) <= x, for a rising f with f(0) <= x: 64 places at a time, one of them a lane, so that
// up to 64 sequences cost one round trip to memory and up to 4096 two.
template <class F>
__device__ __forceinline__ int last_at_most(int n, int x, F f) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) >> 6, i = lo + lane * step;
    const bool in = lane == 0 || (i < hi && f(i < hi ? i : lo) <= x);
    lo += (__popcll(__ballot(in)) - 1) * step;
    hi = min(hi, lo + step);
  }
  return uniform(lo);
}

// Over the two lanes that share lane % 32
__device__ __forceinline__ float max_of_2(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
#endif
  return v;
}
__device__ __forceinline__ float sum_of_2(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
#endif
  return v;
}
// Over the four lanes that share lane % 16
__device__ __forceinline__ float max_of_4(float v) {
  v = max_of_2(v);
#if defined(__HIP_DEVICE_COMPILE__)
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
#endif
  return v;
}
__device__ __forceinline__ float sum_of_4(float v) {
  v = sum_of_2(v);
#if defined(__HIP_DEVICE_COMPILE__)
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
#endif
  return v;
}

// What a row's exponentials, their sum and the products are relative to, in powers of two: p = 2^(score - at).  It moves only where
// a tile's largest score x lies too far from it, so that the sums stay untouched in most tiles.  All lanes of a wave move at once.
//   bf16 has fp32's powers of two: `at` is the largest score at the last move, and goes up where x exceeds it by 2^8; p and the
//   products are as exact there as they are at 1.
//   fp16 loses bits below 2^-14 and everything below 2^-25: with one key that takes nearly all of the weight, the others' p would
//   vanish from the products while the sum still counts them (of 32768 keys with 0.001 of the weight, 2 % of their value).  So a
//   tile's largest p is kept within 2^-1 .. 2^15: `at` also goes down, after the high keys, 2^60 below the largest score at most,
//   behind which a tile is nothing in fp32 sums and the sums would leave fp32.  What 64 keys lose below 2^-14 is then less than
//   2^-18 of the largest's part.
template <class T>
struct Reference {
  float at, high;
  __device__ __forceinline__ void clear() { at = high = -INFINITY; }
  __device__ __forceinline__ bool moves(float x) {
    if (!T::kNarrow) return x - at > 8.f;
    high = fmaxf(high, x);
    return x - at > 15.f || (x - at < -1.f && x != -INFINITY && at > high - 60.f);
  }
  __device__ __forceinline__ float move(float x) {                   // what the sums are scaled by
    const float was = at;
    if (!T::kNarrow) at = fmaxf(at, x);
    else if (x != -INFINITY) at = fmaxf(x - 7.f, high - 60.f);
    return __builtin_amdgcn_exp2f(was - from());
  }
  __device__ __forceinline__ float from() const { return at == -INFINITY ? 0.f : at; }             // nothing seen so far: p is 0 anyway
};

// A launch has fewer than 2^32 threads along x: steps of more are refused, not cut off
inline bool fits_a_launch(long blocks, int threads) { return blocks * threads < 1l << 32; }

struct AppendArgs {
  PagedSeqs s;
  PagedKV kv;
  const char *q, *k, *v;
  char* qo;
  const float *inv_freq, *q_norm, *k_norm;
  long q_t, q_h, k_t, k_h, v_t, v_h, o_t, o_h;   // bytes between tokens / heads
  int Hq, half;                                  // half: rotated pairs of a head
  float eps;
  int interleaved, one;                          // one: every sequence brings exactly one token
  int q_parts, k_parts, v_parts, qk_tiles;       // filled by the launcher
};
hipError_t launch_append(const AppendArgs& a, int dtype, int head_dim, hipStream_t s);

struct PagedAttnArgs {
  PagedSeqs s;
  PagedKV kv;
  const char* q;
  char* o;
  long q_t, q_h, o_t, o_h;                       // bytes between tokens / heads
  int G;                                         // query heads of a key / value head
  int window;                                    // keys that a token sees, its own among them; INT_MAX: all
  float scale2;                                  // scale * log2(e)
  int max_new;
  // filled by the launchers
  int most;                                      // tokens of a sequence up to which the few-rows kernel takes it, not the other
  void* parts;                                   // parts of sums, where the keys are shared out over blocks
  int waves;                                     // of a block (few rows: of one that walks all keys of its rows)
  int tpt;                                       // tokens of a tile of rows
  FastDiv by_tpt;
  int rows_cap, least, blocks;                   // rows of a part; least tiles of a share; blocks that share
  int splits;                                    // many rows: shares of the keys
};
size_t paged_attention_workspace(int n_seqs, int n_tokens, int kv_heads, int group, int max_new, int max_len, int window, int head_dim);
bool chunks_fit_a_launch(const PagedAttnArgs& a);
hipError_t launch_paged_chunks(const PagedAttnArgs& a, int dtype, int head_dim, hipStream_t s);
hipError_t launch_paged_attention(PagedAttnArgs a, int dtype, int head_dim, int max_len, void* workspace, hipStream_t s);

struct VerifyArgs {
  const float *target, *draft;                   // [seq][K + 1][V], [seq][K][V] or nullptr
  long t_seq, t_row, d_seq, d_row;               // elements between sequences / rows
  const void* tokens;                            // [seq][K]
  const float* uniforms;                         // [seq][K + 1]
  const int* counts;                             // [seq] or nullptr
  int* out;                                      // [seq][K + 1]
  int* accepted;                                 // [seq]
  int K, V;
};
hipError_t launch_verify(const VerifyArgs& a, int token_bytes, int n_seqs, hipStream_t s);

}  // namespace sna
