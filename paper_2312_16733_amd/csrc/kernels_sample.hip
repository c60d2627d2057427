// A token of each row of logits, from a given random number.
//   w_i = exp((l_i - max) / temperature);  in the order of falling l (then rising i):  the first top_k;  of these the fewest whose
//   weights make top_p of theirs;  of these the ones with w_i >= min_p.  The token is the smallest i for which the weights of the
//   ones that are left, up to i in the vocabulary's order, make more than u of all of them.
// Weights are formed in 64 bits and summed as whole numbers, steps of 2^-scale_bits of the largest (2^-44 for 2^18 logits): the sums
// of many do not depend on their order, so that they can come together through atomics, and are as exact as 64-bit floats would be.
// Nothing is sorted.  Where the order is cut, and where the draw falls, is found digit by digit of the logits' bit patterns (or of
// the index): sums by digit in LDS, the digit that the wanted sum falls into, then the same among what has that digit.
// Rows of up to 4096 logits take one launch, a block a row with its logits in registers.  Longer ones are read three times, by as
// many blocks as fill the chip: for the largest; for counts or weights by distance from it (where a row is cut); and for what lies at
// the cut, a short list, and the sums of what is kept for certain, by runs of 512.  Then one block a row has the list and the sums.
#include <algorithm>

#include "paged.h"

namespace sna {

typedef unsigned long long u64;
constexpr int SM_BINS = 2048;      // values of a digit; distances told apart; runs of a row, at most
constexpr int SM_SMALL = 4096;     // logits of a row that one block takes in one launch
constexpr int SM_LIST = 4096;      // logits at a row's cut
constexpr int SM_MOST = SM_LIST / 2;             // top_k up to which a row's list is to hold all that it keeps
constexpr int SM_RUN = 512;        // logits of a wave's turn, and of a sum
constexpr int SM_T = 512;          // threads of the blocks that share a row
constexpr int SM_FINAL = 1024;     // of the one that ends it

__device__ __forceinline__ float logit(const float* p, long i) { return p[i]; }
__device__ __forceinline__ float logit(const __bf16* p, long i) { return (float)p[i]; }
__device__ __forceinline__ float logit(const _Float16* p, long i) { return (float)p[i]; }
// What a row's logit counts as: no number as none, both zeros as one
__device__ __forceinline__ float taken(float x) { return x == x ? x + 0.f : -INFINITY; }
// Rises as the logit falls; an order of all floats
__device__ __forceinline__ unsigned falling(float x) {
  const unsigned u = __float_as_uint(x);
  return ~(u ^ (unsigned)((int)u >> 31 | (int)0x80000000));
}
__device__ __forceinline__ float of_falling(unsigned f) {
  const unsigned u = ~f;
  return __uint_as_float(u ^ (u >> 31 ? 0x80000000u : ~0u));
}
__device__ __forceinline__ u64 place(float x, int i) { return (u64)falling(x) << 32 | (unsigned)i; }

struct Row {                       // of logits, and what is wanted of it
  float top;
  double inv_t, magic, min_p;
  u64 cut;                         // place of the last one kept
  float top_p;
  int top_k;                       // 0: all
  __device__ __forceinline__ double weight(float x) const { return x == top ? 1.0 : exp(((double)x - (double)top) * inv_t); }
  // In steps: the sum with a power of two whose last place is a step
  __device__ __forceinline__ u64 steps(double w) const { return (u64)__double_as_longlong(w + magic) & 0xfffffffffffffull; }
  __device__ __forceinline__ u64 weight_of(float x) const { return x > -INFINITY ? steps(weight(x)) : 0; }
  __device__ __forceinline__ double kept(float x, int i) const {       // the weight of one that is left
    if (!(x > -INFINITY && place(x, i) <= cut)) return 0.0;
    const double w = weight(x);
    return w >= min_p ? w : 0.0;
  }
};
__device__ __forceinline__ Row row_of(const SampleArgs& a, int row) {
  Row r;
  const float t = a.temperature_of ? a.temperature_of[row] : a.temperature;
  const int k = a.top_k_of ? a.top_k_of[row] : a.top_k;
  r.inv_t = t > 0.f ? 1.0 / (double)fminf(t, 3.4028235e38f) : 0.0;
  r.min_p = fmin(fmax((double)(a.min_p_of ? a.min_p_of[row] : a.min_p), 0.0), 1.0);       // what is no number cuts nothing, and the largest stays
  r.magic = __longlong_as_double((long long)(1023 + 52 - a.scale_bits) << 52);
  r.top_p = a.top_p_of ? a.top_p_of[row] : a.top_p;
  r.top_k = t > 0.f ? k > 0 && k < a.V ? k : 0 : 1;
  r.cut = ~0ull;
  return r;
}

__device__ __forceinline__ u64 scan_up(u64 v) {                      // inclusive, of a wave
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const u64 x = __shfl_up(v, m, 64);
    if (lane >= m) v += x;
  }
  return v;
}
__device__ __forceinline__ u64 sum_of_wave(u64 v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, 64);
  return v;
}
__device__ __forceinline__ float max_of_wave(float v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v = fmaxf(v, __shfl_xor(v, m, 64));
  return v;
}

template <int NT>
struct SampleLds {
  u64 sums[SM_BINS], waves[NT / 64], ups[NT / 64], before, found;
  int digit, n;
  float top[NT / 64];
};
template <int NT>
__device__ __forceinline__ u64 sum_of_block(SampleLds<NT>& lds, u64 v) {
  v = sum_of_wave(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds.waves[threadIdx.x >> 6] = v;
  __syncthreads();
  u64 s = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) s += lds.waves[w];
  return s;
}
template <int NT>
__device__ __forceinline__ float max_of_block(SampleLds<NT>& lds, float v) {
  v = max_of_wave(v);
  if ((threadIdx.x & 63) == 0) lds.top[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) v = fmaxf(v, lds.top[w]);
  return v;
}

// The bin of lds.sums at which their running sum reaches `want` (1 or more, at most the sum of all), and what comes before it.
// All threads get both; the sums are complete when it is called, and may be overwritten when it returns.
template <int NT>
__device__ __forceinline__ int crossing(SampleLds<NT>& lds, u64 want, u64& before) {
  constexpr int N = SM_BINS / NT;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  u64 v[N], mine = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) mine += v[i] = lds.sums[N * tid + i];
  const u64 up = scan_up(mine);
  if (lane == 63) lds.ups[wave] = up;
  __syncthreads();
  u64 at = up - mine;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) at += w < wave ? lds.ups[w] : 0;
  if (at < want && want <= at + mine)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (at < want && want <= at + v[i]) { lds.digit = N * tid + i; lds.before = at; }
      at += v[i];
    }
  __syncthreads();
  before = lds.before;
  return lds.digit;
}

// Of all (order, weight) that `each` visits, in rising order: the order at which the running sum of weights reaches `want`, which is
// 1 .. the sum of all.  Orders differ in their last `bits` bits only.  All threads.
template <int NT, class Each>
__device__ __forceinline__ u64 select(SampleLds<NT>& lds, int bits, u64 want, const Each& each) {
  u64 lo = 0;
  bool first = true;
  for (int left = bits; left > 0; first = false) {
    const int width = min(left, 11), shift = left - width;
    const u64 mask = left == 64 ? ~0ull : (1ull << left) - 1, same = lo >> shift >> width;      // left == 64: no bits above
    __syncthreads();
    for (int i = threadIdx.x; i < SM_BINS; i += NT) lds.sums[i] = 0;
    if (threadIdx.x == 0) lds.n = 0;
    __syncthreads();
    each([&](u64 order, u64 w) {
      if (w && (first || order >> shift >> width == same)) atomicAdd(&lds.sums[(order & mask) >> shift], w);
    });
    __syncthreads();
    u64 before;
    const u64 digit = crossing(lds, want, before);
    want -= before;
    if (first) {                                                     // the bits that all share
      each([&](u64 order, u64 w) {
        if (w && (order & mask) >> shift == digit) {
          atomicAdd(&lds.n, 1);
          lds.found = order;
        }
      });
      __syncthreads();
      lo = (lds.found & ~mask) | digit << shift;
    } else {
      lo |= digit << shift;
      each([&](u64 order, u64 w) {
        if (w && order >> shift == lo >> shift) {
          atomicAdd(&lds.n, 1);
          lds.found = order;
        }
      });
      __syncthreads();
    }
    if (lds.n == 1) return lds.found;
    left = shift;
  }
  return lo;
}
// A fraction f of a sum of s steps, upwards, as a sum that can be reached
__device__ __forceinline__ u64 part_of(double f, u64 s) {
  const u64 want = (u64)ceil(fmax(f, 0.0) * (double)s);
  return want < 1 ? 1 : want > s ? s : want;
}
// What the running sum of `total` steps has to reach for the draw
__device__ __forceinline__ u64 drawn_at(const SampleArgs& a, int row, u64 total) {
  const u64 want = (u64)(fmin(fmax((double)a.u[row], 0.0), 1.0) * (double)total) + 1;
  return want > total ? total : want;
}
// 1 over the sum of what is left
__device__ __forceinline__ double share_of(const SampleArgs& a, u64 total) { return 1.0 / ((double)total * __longlong_as_double((long long)(1023 - a.scale_bits) << 52)); }
__device__ __forceinline__ int index_bits(int V) { return 32 - __builtin_clz(V); }

// The cuts of logits that `each` visits (logit, index) into r.cut, top_k and then top_p
template <int NT, class Each>
__device__ __forceinline__ void cut_row(SampleLds<NT>& lds, Row& r, const Each& each) {
  if (r.top_k) {
    u64 n = 0;
    each([&](float x, int) { n += x > -INFINITY; });
    n = sum_of_block(lds, n);
    if (n >= (u64)r.top_k)                                           // also of a list that holds no more than these
      r.cut = select(lds, 64, (u64)r.top_k, [&](const auto& f) { each([&](float x, int i) { f(place(x, i), x > -INFINITY ? 1 : 0); }); });
  }
  if (r.top_p < 1.f) {
    const u64 cut = r.cut;
    u64 n = 0;
    each([&](float x, int i) { if (place(x, i) <= cut) n += r.weight_of(x); });
    n = sum_of_block(lds, n);
    r.cut = select(lds, 64, part_of(r.top_p, n), [&](const auto& f) { each([&](float x, int i) { f(place(x, i), place(x, i) <= cut ? r.weight_of(x) : 0); }); });
  }
}
// The draw among those of them that are left, and the sum of these
template <int NT, class Each>
__device__ __forceinline__ int draw_row(SampleLds<NT>& lds, const SampleArgs& a, int row, const Row& r, u64& total, const Each& each) {
  total = 0;
  each([&](float x, int i) { total += r.steps(r.kept(x, i)); });
  total = sum_of_block(lds, total);
  return (int)select(lds, index_bits(a.V), drawn_at(a, row, total), [&](const auto& f) { each([&](float x, int i) { f((u64)i, r.steps(r.kept(x, i))); }); });
}

// ---- rows of a block -----------------------------------------------------------------------------------------------------------
template <class X, int NT>
__global__ __launch_bounds__(NT) void sample_small_kernel(const SampleArgs a) {
  constexpr int N = 4;
  __shared__ SampleLds<NT> lds;
  const int tid = threadIdx.x, row = blockIdx.x, V = a.V;
  const X* logits = (const X*)a.logits + row * a.stride;
  float x[N], top = -INFINITY;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int i = j * NT + tid;
    x[j] = i < V ? taken(logit(logits, i)) : -INFINITY;
  }
  Row r = row_of(a, row);
#pragma unroll
  for (int j = 0; j < N; ++j) top = fmaxf(top, x[j]);
  r.top = max_of_block(lds, top);
  u64 total = 0;
  const bool some = r.top > -INFINITY;
  if (some) {
    const auto each = [&](const auto& f) {
#pragma unroll
      for (int j = 0; j < N; ++j) f(x[j], j * NT + tid);
    };
    cut_row(lds, r, each);
    const int token = draw_row(lds, a, row, r, total, each);
    if (tid == 0) a.tokens[row] = token;
  } else if (tid == 0) {
    a.tokens[row] = -1;                                              // nothing to draw from
  }
  if (a.probs) {
    const double f = some ? share_of(a, total) : 0.0;
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j * NT + tid < V) a.probs[row * a.p_stride + j * NT + tid] = some ? (float)(r.kept(x[j], j * NT + tid) * f) : 0.f;
  }
}

// ---- rows of several blocks ------------------------------------------------------------------------------------------------------
// What a row needs between launches
struct RowWork {
  u64 weights[SM_BINS];            // by distance from the largest
  unsigned counts[SM_BINS];
  u64 list[SM_LIST];               // places
  unsigned listed, pad;            // more than SM_LIST: not all of them are there
  u64 cut;                         // what the row comes to
  double share;
};
// How a row is cut
enum Kind { CUT_NONE, CUT_COUNT, CUT_WEIGHT, CUT_SLOWLY };           // all that is kept in the list; the list at the cut; digit by digit of the whole row
__device__ __forceinline__ Kind kind_of(const Row& r) {
  if (r.top_k) return r.top_k <= SM_MOST ? CUT_COUNT : CUT_SLOWLY;
  return r.top_p < 1.f ? CUT_WEIGHT : CUT_NONE;
}
struct Work {                      // of a call
  RowWork* rows;                   // [n]
  float* tops;                     // [n][parts]
  u64* runs;                       // [n][runs]
  int parts, len, n_runs;          // blocks of a row, logits of one, sums of a row
};

// Rises as x falls.  Even steps of 1 / 64 of the temperature for 16 of it, then 64 to an octave
__device__ __forceinline__ int distance(const Row& r, float x) {
  const float d = x == r.top ? 0.f : (r.top - x) * (r.inv_t > 0.0 ? (float)(r.inv_t * (1.0 / 16)) : 1.f);
  return d < 1.f ? (int)(d * (SM_BINS / 2)) : min(SM_BINS / 2 + (int)((__float_as_uint(d) - 0x3f800000u) >> 17), SM_BINS - 1);
}

// Runs of the block's part of a row, a wave's turn each: eight logits a lane
template <class X>
struct Eight;
template <>
struct Eight<float> {
  typedef __attribute__((ext_vector_type(4), aligned(4))) float v4;
  static __device__ __forceinline__ void load(const float* p, float (&x)[8]) {
    const v4 a = *(const v4*)p, b = *(const v4*)(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
  }
};
template <class H>
struct EightHalves {
  typedef __attribute__((ext_vector_type(8), aligned(2))) H v8;
  static __device__ __forceinline__ void load(const H* p, float (&x)[8]) {
    const v8 a = *(const v8*)p;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)a[e];
  }
};
template <>
struct Eight<__bf16> : EightHalves<__bf16> {};
template <>
struct Eight<_Float16> : EightHalves<_Float16> {};

// f(logits, index of the first, run), run by run; what lies behind the row is -inf
template <class X, class F>
__device__ __forceinline__ void each_run(const SampleArgs& a, const Work& w, int row, int part, const F& f) {
  const X* logits = (const X*)a.logits + row * a.stride;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, end = min((part + 1) * w.len, a.V);
  for (int i0 = part * w.len + wave * SM_RUN; i0 < end; i0 += SM_T / 64 * SM_RUN) {
    const int i = i0 + 8 * lane;
    float x[8];
    if (i + 8 <= a.V) {
      Eight<X>::load(logits + i, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = taken(x[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = i + e < a.V ? taken(logit(logits, i + e)) : -INFINITY;
    }
    f(x, i, i0 / SM_RUN);
  }
}
__device__ __forceinline__ float top_of(const Work& w, int row) {
  float top = -INFINITY;
  for (int p = threadIdx.x & 63; p < w.parts; p += 64) top = fmaxf(top, w.tops[row * w.parts + p]);
  return max_of_wave(top);
}

template <class X>
__global__ __launch_bounds__(SM_T) void sample_top_kernel(const SampleArgs a, const Work w) {
  __shared__ SampleLds<SM_T> lds;
  const int row = blockIdx.x / w.parts, part = blockIdx.x % w.parts;
  RowWork& rw = w.rows[row];
  if (part == 0)
    for (int i = threadIdx.x; i < SM_BINS; i += SM_T) {
      rw.weights[i] = 0;
      rw.counts[i] = 0;
    }
  if (part == 0 && threadIdx.x == 0) rw.listed = 0;
  float top = -INFINITY;
  each_run<X>(a, w, row, part, [&](const float (&x)[8], int, int) {
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, x[e]);
  });
  top = max_of_block(lds, top);
  if (threadIdx.x == 0) w.tops[blockIdx.x] = top;
}

template <class X>
__global__ __launch_bounds__(SM_T) void sample_sums_kernel(const SampleArgs a, const Work w) {
  __shared__ u64 weights[SM_BINS];
  __shared__ unsigned counts[SM_BINS];
  const int row = blockIdx.x / w.parts, part = blockIdx.x % w.parts;
  Row r = row_of(a, row);
  const Kind kind = kind_of(r);
  if (kind != CUT_COUNT && kind != CUT_WEIGHT) return;
  r.top = top_of(w, row);
  if (r.top == -INFINITY) return;
  RowWork& rw = w.rows[row];
  for (int i = threadIdx.x; i < SM_BINS; i += SM_T) {
    if (kind == CUT_COUNT) counts[i] = 0;
    else weights[i] = 0;
  }
  __syncthreads();
  if (kind == CUT_COUNT)
    each_run<X>(a, w, row, part, [&](const float (&x)[8], int, int) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (x[e] > -INFINITY) atomicAdd(&counts[distance(r, x[e])], 1u);
    });
  else
    each_run<X>(a, w, row, part, [&](const float (&x)[8], int, int) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const u64 s = r.weight_of(x[e]);
        if (s) atomicAdd(&weights[distance(r, x[e])], s);
      }
    });
  __syncthreads();
  for (int i = threadIdx.x; i < SM_BINS; i += SM_T) {
    if (kind == CUT_COUNT) {
      if (counts[i]) atomicAdd(&rw.counts[i], counts[i]);
    } else {
      if (weights[i]) atomicAdd(&rw.weights[i], weights[i]);
    }
  }
}

// The distance that the row's cut lies at, and what is wanted of it there; SM_BINS: it is not cut
template <int NT>
__device__ __forceinline__ int cut_at(SampleLds<NT>& lds, const Row& r, Kind kind, const RowWork& rw, u64& want) {
  u64 all = 0;
  for (int i = threadIdx.x; i < SM_BINS; i += NT) all += lds.sums[i] = kind == CUT_COUNT ? rw.counts[i] : rw.weights[i];
  all = sum_of_block(lds, all);                                      // and the sums are there
  want = kind == CUT_COUNT ? (u64)r.top_k : part_of(r.top_p, all);
  if (kind == CUT_COUNT && all <= want) return SM_BINS;
  u64 before;
  const int d = crossing(lds, want, before);
  want -= before;
  return d;
}

template <class X>
__global__ __launch_bounds__(SM_T) void sample_list_kernel(const SampleArgs a, const Work w) {
  __shared__ SampleLds<SM_T> lds;
  __shared__ u64 list[SM_LIST];
  __shared__ unsigned listed, first;
  const int row = blockIdx.x / w.parts, part = blockIdx.x % w.parts, tid = threadIdx.x;
  Row r = row_of(a, row);
  const Kind kind = kind_of(r);
  if (kind == CUT_SLOWLY) return;
  r.top = top_of(w, row);
  if (r.top == -INFINITY) return;
  RowWork& rw = w.rows[row];
  int at = SM_BINS;
  u64 want;
  if (tid == 0) listed = 0;
  if (kind != CUT_NONE) at = cut_at(lds, r, kind, rw, want);
  __syncthreads();
  each_run<X>(a, w, row, part, [&](const float (&x)[8], int i, int run) {
    u64 sum = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int d = kind == CUT_NONE ? 0 : distance(r, x[e]);
      if (kind == CUT_COUNT ? d <= at && x[e] > -INFINITY : kind == CUT_WEIGHT && d == at && x[e] > -INFINITY) {
        const unsigned n = atomicAdd(&listed, 1u);
        if (n < SM_LIST) list[n] = place(x[e], i + e);
      }
      if (kind != CUT_COUNT && d < at) sum += r.steps(r.kept(x[e], i + e));
    }
    if (kind != CUT_COUNT) {
      sum = sum_of_wave(sum);
      if ((tid & 63) == 0) w.runs[(long)row * w.n_runs + run] = sum;
    }
  });
  __syncthreads();
  if (tid == 0 && listed) first = atomicAdd(&rw.listed, listed);
  __syncthreads();
  if (listed && first < SM_LIST)
    for (unsigned n = tid; n < listed && first + n < SM_LIST; n += SM_T) rw.list[first + n] = list[n];
}

template <class X>
__global__ __launch_bounds__(SM_FINAL) void sample_draw_kernel(const SampleArgs a, const Work w) {
  constexpr int N = SM_LIST / SM_FINAL;
  __shared__ SampleLds<SM_FINAL> lds;
  const int tid = threadIdx.x, row = blockIdx.x;
  const X* logits = (const X*)a.logits + row * a.stride;
  RowWork& rw = w.rows[row];
  Row r = row_of(a, row);
  const Kind kind = kind_of(r);
  r.top = top_of(w, row);
  if (r.top == -INFINITY) {                                          // nothing to draw from
    if (tid == 0) {
      a.tokens[row] = -1;
      rw.cut = 0;
      rw.share = 0.0;
    }
    return;
  }
  u64 total;
  int token;
  const unsigned m = kind == CUT_COUNT || kind == CUT_WEIGHT ? rw.listed : 0;
  if (kind == CUT_SLOWLY || m > SM_LIST) {
    const auto each = [&](const auto& f) {
      for (int i = tid; i < a.V; i += SM_FINAL) f(taken(logit(logits, i)), i);
    };
    cut_row(lds, r, each);
    token = draw_row(lds, a, row, r, total, each);
  } else {
    float x[N];
    int at[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const bool is = j * SM_FINAL + tid < m;
      const u64 p = is ? rw.list[j * SM_FINAL + tid] : 0;
      x[j] = is ? of_falling((unsigned)(p >> 32)) : -INFINITY;
      at[j] = (int)p;
    }
    const auto each = [&](const auto& f) {
#pragma unroll
      for (int j = 0; j < N; ++j) f(x[j], at[j]);
    };
    if (kind == CUT_COUNT) {
      cut_row(lds, r, each);
      token = draw_row(lds, a, row, r, total, each);
    } else {
      if (kind == CUT_WEIGHT) {
        u64 want;
        cut_at(lds, r, kind, rw, want);
        r.cut = select(lds, 64, want, [&](const auto& f) { each([&](float y, int i) { f(place(y, i), r.weight_of(y)); }); });
      }
      // the runs' sums with what is kept of the list; then the run that the draw falls into
      __syncthreads();
      for (int i = tid; i < SM_BINS; i += SM_FINAL) lds.sums[i] = i < w.n_runs ? w.runs[(long)row * w.n_runs + i] : 0;
      __syncthreads();
      each([&](float y, int i) {
        const u64 s = r.steps(r.kept(y, i));
        if (s) atomicAdd(&lds.sums[i / SM_RUN], s);
      });
      __syncthreads();
      total = 0;
      for (int i = tid; i < SM_BINS; i += SM_FINAL) total += lds.sums[i];
      total = sum_of_block(lds, total);
      const u64 want = drawn_at(a, row, total);
      u64 before;
      const int run = crossing(lds, want, before), i = run * SM_RUN + tid;
      const u64 s = tid < SM_RUN && i < a.V ? r.steps(r.kept(taken(logit(logits, i)), i)) : 0;
      token = run * SM_RUN + (int)select(lds, 9, want - before, [&](const auto& f) { f((u64)tid, s); });
    }
  }
  if (tid == 0) {
    a.tokens[row] = token;
    rw.cut = r.cut;
    rw.share = share_of(a, total);
  }
}

template <class X>
__global__ __launch_bounds__(SM_T) void sample_probs_kernel(const SampleArgs a, const Work w) {
  const int row = blockIdx.x / w.parts, part = blockIdx.x % w.parts;
  Row r = row_of(a, row);
  r.top = top_of(w, row);
  r.cut = w.rows[row].cut;
  const double f = w.rows[row].share;
  float* out = a.probs + row * a.p_stride;
  each_run<X>(a, w, row, part, [&](const float (&x)[8], int i, int) {
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = f > 0.0 ? (float)(r.kept(x[e], i + e) * f) : 0.f;
    if (i + 8 <= a.V) {
      typedef Eight<float>::v4 v4;
      *(v4*)(out + i) = v4{p[0], p[1], p[2], p[3]};
      *(v4*)(out + i + 4) = v4{p[4], p[5], p[6], p[7]};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (i + e < a.V) out[i + e] = p[e];
    }
  });
}

// Blocks of a row: as many as make 512 of all rows, two on a CU, with 8 turns of a wave or more each
static Work work_of(int n, int V, void* at) {
  Work w = {};
  const long want = ((long)n * V + 511) / 512, turn = SM_T / 64 * SM_RUN;
  w.len = (int)(std::min(std::max((want + turn - 1) / turn, 1l), (V + turn - 1) / turn) * turn);
  w.parts = (V + w.len - 1) / w.len;
  w.n_runs = (V + SM_RUN - 1) / SM_RUN;
  w.rows = (RowWork*)at;
  w.runs = (u64*)(w.rows + n);
  w.tops = (float*)(w.runs + (long)n * w.n_runs);
  return w;
}
size_t sample_workspace(int n, int vocab, int) {
  if (vocab <= SM_SMALL) return 0;
  const Work w = work_of(n, vocab, nullptr);
  return n * (sizeof(RowWork) + w.n_runs * sizeof(u64) + w.parts * sizeof(float));
}

template <class X>
static hipError_t sample_of(const SampleArgs& a, hipStream_t s) {
  if (a.V <= SM_SMALL) {
    if (!fits_a_launch(a.n, 1024)) return hipErrorInvalidConfiguration;
    if (a.V <= 1024) hipLaunchKernelGGL((sample_small_kernel<X, 256>), dim3(a.n), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((sample_small_kernel<X, 1024>), dim3(a.n), dim3(1024), 0, s, a);
    return hipGetLastError();
  }
  const Work w = work_of(a.n, a.V, a.work);
  const long blocks = (long)a.n * w.parts;
  if (!fits_a_launch(blocks, SM_T) || !fits_a_launch(a.n, SM_FINAL)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)blocks), block(SM_T);
  hipLaunchKernelGGL(sample_top_kernel<X>, grid, block, 0, s, a, w);
  if (a.top_k_of || a.top_p_of || a.temperature_of || a.top_k || a.top_p < 1.f || a.temperature == 0.f) hipLaunchKernelGGL(sample_sums_kernel<X>, grid, block, 0, s, a, w);
  hipLaunchKernelGGL(sample_list_kernel<X>, grid, block, 0, s, a, w);
  hipLaunchKernelGGL(sample_draw_kernel<X>, dim3(a.n), dim3(SM_FINAL), 0, s, a, w);
  if (a.probs) hipLaunchKernelGGL(sample_probs_kernel<X>, grid, block, 0, s, a, w);
  return hipGetLastError();
}
hipError_t launch_sample(SampleArgs a, int dtype, hipStream_t s) {
  int bits = 0;
  while (1 << bits < a.V) ++bits;
  a.scale_bits = 62 - bits < 51 ? 62 - bits : 51;
  return dtype == SNA_DTYPE_FP32 ? sample_of<float>(a, s) : dtype == SNA_DTYPE_BF16 ? sample_of<__bf16>(a, s) : sample_of<_Float16>(a, s);
}

}  // namespace sna
