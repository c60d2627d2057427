// A token of each row of logits, from a given random number.
//   w_i = exp((l_i - max) / temperature);  in the order of falling l (then rising i):  the first top_k;  of these the fewest whose
//   weights make top_p of theirs;  of these the ones with w_i >= min_p.  The token is the smallest i for which the weights of the
//   ones that are left, up to i in the vocabulary's order, make more than u of all of them.
// Weights are formed in 64 bits and summed as whole numbers, steps of 2^-scale_bits of the largest (2^-44 for 2^18 logits): the sums
// of many do not depend on their order, so that they can come together through atomics, and are as exact as 64-bit floats would be.
// Nothing is sorted.  Where the order is cut, and where the draw falls, is found digit by digit of the logits' bit patterns (or of
// the index): sums by digit in LDS, the digit that the wanted sum falls into, then the same among what has that digit.
// Rows of up to 4096 logits take one launch, a block a row with its logits in registers: 1000 of them, top_k 50 and top_p 0.9, 8.5 us,
// which a dozen barriers in a row make, and the launch.  Longer ones are read three times, by as many blocks as fill the chip: for the
// largest; for counts or weights by distance from it (where a row is cut); and for what lies at the cut, a list, mostly short, and the
// sums of what is kept for certain, by runs of 512.  Then one block a row has the list and the sums.  128 rows of 131072 fp32, top_p 0.95 (a third
// of each is kept): 12, 20, 27 and 11 us, 66 in a loop of calls.  The first is bound by memory (5.5 TB/s); the next two by vector
// instructions, 32 and 38 a logit, at work 84 and 71 % of the cycles, of which a weight is 20; the last by its round trips.  Where one
// logit is kept, the first reading finds it: 15 us, and 44 by the others.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "paged.h"

namespace sna {

typedef unsigned long long u64;
constexpr int SM_BINS = 2048;      // values of a digit; distances told apart; runs of a row, at most
constexpr int SM_SMALL = 4096;     // logits of a row that one block takes in one launch
constexpr int SM_LIST = 8192;      // logits at a row's cut
constexpr int SM_HELD = 2048;      // of them that are held in registers
constexpr int SM_MOST = SM_LIST / 2;             // top_k up to which a row's list is to hold all that it keeps
constexpr int SM_RUN = 512;        // logits of a wave's turn, and of a sum
constexpr int SM_STAGE = 2048;     // logits at the cut that a block writes out at once
constexpr int SM_T = 512;          // threads of the blocks that share a row
constexpr int SM_FINAL = 512;      // of the one that ends it

__device__ __forceinline__ float logit(const float* p, long i) { return p[i]; }
__device__ __forceinline__ float logit(const __bf16* p, long i) { return (float)p[i]; }
__device__ __forceinline__ float logit(const _Float16* p, long i) { return (float)p[i]; }
// What a row's logit counts as: no number as none
__device__ __forceinline__ float taken(float x) { return x == x ? x : -INFINITY; }
// Rises as the logit falls; an order of all floats, both zeros as one
__device__ __forceinline__ unsigned falling(float x) {
  const unsigned u = __float_as_uint(x + 0.f);
  return ~(u ^ (unsigned)((int)u >> 31 | (int)0x80000000));
}
// Bits that are the same for all logits of a type and sign: below the last place of its numbers, as fp32
template <class X> constexpr int kSpare = 0;
template <> constexpr int kSpare<__bf16> = 16;
template <> constexpr int kSpare<_Float16> = 13;

// 2^y for -1000 <= y <= 0, off by 7e-16 of itself: y's fraction f within 1/2, and 1 + f times the polynomial through (2^f - 1) / f at
// ten Chebyshev points, so that 2^0 is 1.  The whole number comes off by adding a power of two whose last place is 1, and goes into
// the exponent as it is.  With the library's exp, which takes any argument, the sums of 128 rows of 131072 took 36 us, not 21
struct Power {
  double c[10];
  __device__ __forceinline__ void begin() {
    const double v[10] = {0x1.62e42fefa39f7p-1, 0x1.ebfbdff82c590p-3, 0x1.c6b08d7044119p-5, 0x1.3b2ab6fba385fp-7, 0x1.5d87fe908f88ap-10,
                              0x1.4309130378460p-13, 0x1.ffcb76789860fp-17, 0x1.62bfe46117445p-20, 0x1.b6571de2f2351p-24, 0x1.e5e9f548e5725p-28};
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      c[i] = v[i];
#if defined(__HIP_DEVICE_COMPILE__)
      asm("" : "+s"(c[i]));                                          // in scalar registers: moved into vector ones, they took as long as the products
#endif
    }
  }
  __device__ __forceinline__ double of_2(double y) const {
    const double t = y + 0x1.8p52, f = y - (t - 0x1.8p52);
    double p = c[9];
#pragma unroll
    for (int i = 8; i >= 0; --i) p = fma(p, f, c[i]);
    p = fma(p, f, 1.0);
    return __hiloint2double(__double2hiint(p) + (__double2loint(t) << 20), __double2loint(p));
  }
};

struct Row {                       // of logits, and what is wanted of it
  Power power;
  double top, per, magic, min_p;   // per: powers of two to one of a logit
  u64 cut;                         // place of the last one kept
  float top_p, top32, near;        // near: see distance()
  int top_k;                       // 0: all
  int spare, bits;                 // of a logit's order, of an index
  bool infinite;                   // the largest is +inf: only such have weight
  __device__ __forceinline__ bool begin(float x) {                   // with the largest; false: nothing to draw from
    infinite = x == INFINITY;
    top32 = infinite ? 0.f : x;
    top = top32;
    return x > -INFINITY;
  }
  // and the smallest, of some: a row that spans less than 4 temperatures has its 256 even steps over that
  __device__ __forceinline__ bool begin(float2 ends) {
    const bool some = begin(ends.x);
    near = fmaxf(near, fminf(2.f / (ends.x - ends.y), 1e38f));       // where all are the same, any will do
    return some;
  }
  __device__ __forceinline__ float seen(float x) const { return infinite ? x == INFINITY ? 0.f : -INFINITY : taken(x); }
  // Where it stands among the row's
  __device__ __forceinline__ u64 place(float x, int i) const { return (u64)(falling(x) >> spare) << bits | (unsigned)i; }
  __device__ __forceinline__ double weight(float x) const { return power.of_2(fmax(((double)x - top) * per, -1000.0)); }      // NaN has none
  // In steps: the sum with a power of two whose last place is a step
  __device__ __forceinline__ u64 steps(double w) const { return (u64)__double_as_longlong(w + magic) & 0xfffffffffffffull; }
  __device__ __forceinline__ double left(double w) const { return w >= min_p ? w : 0.0; }
  __device__ __forceinline__ double kept(float x, int i) const {       // the weight of one that is left
    return x > -INFINITY && place(x, i) <= cut ? left(weight(x)) : 0.0;
  }
  // Rises as x falls, in SM_BINS steps: 256 even ones of 1 / 64 of the temperature (see begin), then twice as wide from 4 temperatures on, and
  // again from 12, 28, .. on: what a number from 2 on has of bits behind the leading ones
  __device__ __forceinline__ int distance(float x) const { return (int)min(far(x) >> 15, (unsigned)SM_BINS - 1); }
  __device__ __forceinline__ unsigned far(float x) const { return __float_as_uint(fmaf(top32 - x, near, 2.f)) & 0x3fffffff; }        // from 2 on: the exponent begins with zeros
};
template <class X>
__device__ __forceinline__ Row row_of(const SampleArgs& a, int row) {
  Row r;
  r.power.begin();
  const float t = a.temperature_of ? a.temperature_of[row] : a.temperature;
  const int k = a.top_k_of ? a.top_k_of[row] : a.top_k;
  const double inv = t > 0.f ? 1.0 / (double)fminf(t, 1e33f) : 1.0;
  r.per = inv * 1.44269504088896340736;
  r.near = fmaxf((float)fmin(inv * 0.5, 1e38), 1e-38f);
  r.min_p = fmin(fmax((double)(a.min_p_of ? a.min_p_of[row] : a.min_p), 0.0), 1.0);       // what is no number cuts nothing, and the largest stays
  r.magic = __longlong_as_double((long long)(1023 + 52 - a.scale_bits) << 52);
  r.top_p = a.top_p_of ? a.top_p_of[row] : a.top_p;
  r.top_k = t > 0.f ? k > 0 && k < a.V ? k : 0 : 1;
  r.cut = ~0ull;
  r.spare = kSpare<X>;
  r.bits = 32 - __builtin_clz(a.V);
  r.infinite = false;
  return r;
}

// Over a wave, in vector registers: a shuffle through LDS takes 50 cycles and more a step
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned moved(unsigned none, unsigned v) {
#if defined(__HIP_DEVICE_COMPILE__)
  return (unsigned)__builtin_amdgcn_update_dpp((int)none, (int)v, CTRL, ROWS, 0xf, false);
#else
  return v + none;
#endif
}
template <class F>
__device__ __forceinline__ u64 scan_of(u64 v, u64 none, const F& f) {                  // inclusive; lanes without a neighbour get `none`
  const auto step = [&](auto ctrl, auto rows) {
    const unsigned lo = moved<decltype(ctrl)::value, decltype(rows)::value>((unsigned)none, (unsigned)v), hi = moved<decltype(ctrl)::value, decltype(rows)::value>((unsigned)(none >> 32), (unsigned)(v >> 32));
    v = f(v, (u64)hi << 32 | lo);
  };
  step(std::integral_constant<int, 0x111>(), std::integral_constant<int, 0xf>());      // within 16 lanes: 1, 2, 4, 8 to the right
  step(std::integral_constant<int, 0x112>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x114>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x118>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>());      // the last of 16 to the 16 behind, in rows 1 and 3
  step(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>());      // the last of 32 to the 32 behind
  return v;
}
__device__ __forceinline__ u64 last_lane(u64 v) {
#if defined(__HIP_DEVICE_COMPILE__)
  v = (u64)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), 63) << 32 | (unsigned)__builtin_amdgcn_readlane((int)v, 63);
#endif
  return v;
}
struct Add { __device__ __forceinline__ u64 operator()(u64 a, u64 b) const { return a + b; } };
struct Or { __device__ __forceinline__ u64 operator()(u64 a, u64 b) const { return a | b; } };
struct Most { __device__ __forceinline__ u64 operator()(u64 a, u64 b) const { return a > b ? a : b; } };
struct And { __device__ __forceinline__ u64 operator()(u64 a, u64 b) const { return a & b; } };
__device__ __forceinline__ u64 scan_up(u64 v) { return scan_of(v, 0, Add()); }
__device__ __forceinline__ u64 sum_of_wave(u64 v) { return last_lane(scan_up(v)); }
__device__ __forceinline__ float max_of_wave(float v) {
  const auto step = [&](auto ctrl, auto rows) { v = fmaxf(v, __uint_as_float(moved<decltype(ctrl)::value, decltype(rows)::value>(0xff800000u, __float_as_uint(v)))); };
  step(std::integral_constant<int, 0x111>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x112>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x114>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x118>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>());
  step(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>());
  return __uint_as_float((unsigned)last_lane(__float_as_uint(v)));
}

// What lanes of a wave leave in LDS for each other: all of it is written before any of it is read behind this, and read before it is
// written anew.  The wave's accesses are in order anyway, so this keeps the compiler from moving them, and is no instruction
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr int SM_FEW = 128;        // logits that one wave ends a row with
template <int NT>
struct SampleLds {
  u64 sums[SM_BINS], waves[NT / 64], ups[NT / 64], before, found;
  u64 place[SM_FEW], steps[SM_FEW];
  double weight[SM_FEW];
  int digit, n, few;
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

// The bin of lds.sums at which their running sum reaches want(the sum of all), which is 1 .. that, and what comes before it and is
// wanted of it.  All threads get them; the sums are complete when it is called, and zero when it returns.
struct Crossing { int bin; u64 want, total; };
template <int NT, class Want>
__device__ __forceinline__ Crossing crossing(SampleLds<NT>& lds, const Want& want_of) {
  constexpr int N = SM_BINS / NT;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  u64 v[N], mine = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    mine += v[i] = lds.sums[N * tid + i];
    lds.sums[N * tid + i] = 0;
  }
  const u64 up = scan_up(mine);
  if (lane == 63) lds.ups[wave] = up;
  __syncthreads();
  if (tid == 0) lds.n = 0;
  Crossing c;
  c.total = 0;
  u64 at = up - mine;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    at += w < wave ? lds.ups[w] : 0;
    c.total += lds.ups[w];
  }
  const u64 want = want_of(c.total);
  if (at < want && want <= at + mine)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (at < want && want <= at + v[i]) { lds.digit = N * tid + i; lds.before = at; }
      at += v[i];
    }
  __syncthreads();
  c.bin = lds.digit;
  c.want = want - lds.before;
  return c;
}
// The thread at whose value the running sum of the threads' reaches `want`, which is 1 .. the sum of all
template <int NT>
__device__ __forceinline__ int reached_at(SampleLds<NT>& lds, u64 v, u64 want) {
  const int tid = threadIdx.x, wave = tid >> 6;
  u64 up = scan_up(v);
  if ((tid & 63) == 63) lds.ups[wave] = up;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) up += w < wave ? lds.ups[w] : 0;
  if (up >= want && up - v < want) lds.digit = tid;
  __syncthreads();
  return lds.digit;
}

// Of all (order, weight) that `each` visits, in rising order: the order at which the running sum of weights reaches `want`, which is
// 1 .. the sum of all.  Orders differ in their last `bits` bits only.  All threads; lds.sums is zero before and after.
template <int NT, class Each>
__device__ __forceinline__ u64 select(SampleLds<NT>& lds, int bits, u64 want, const Each& each) {
  u64 lo = 0, known = 0;                                             // of the order's bits, those found so far
  for (int left = bits; left > 0;) {
    const int shift = max(left - 11, 0);
    const u64 mask = (left == 64 ? ~0ull : (1ull << left) - 1);
    each([&](u64 order, u64 w) {
      if (w && ((order ^ lo) & known) == 0) atomicAdd(&lds.sums[(order & mask) >> shift], w);
    });
    __syncthreads();
    const Crossing c = crossing(lds, [&](u64) { return want; });
    const u64 digit = c.bin;
    want = c.want;
    known |= mask & ~((1ull << shift) - 1);
    lo |= digit << shift;
    each([&](u64 order, u64 w) {
      if (w && ((order ^ lo) & known) == 0) {
        atomicAdd(&lds.n, 1);
        lds.found = order;
      }
    });
    __syncthreads();
    if (lds.n == 1 || shift == 0) break;
    left = shift;
  }
  return lds.found;
}
// The same for what the threads have in registers; the bits that all of them share are left out
template <int NT, int N>
__device__ __forceinline__ u64 select_held(SampleLds<NT>& lds, u64 want, const u64 (&order)[N], const u64 (&w)[N]) {
  u64 any = 0, all = ~0ull;
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (w[j]) { any |= order[j]; all &= order[j]; }
  any = last_lane(scan_of(any, 0, Or()));
  all = last_lane(scan_of(all, ~0ull, And()));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) { lds.waves[threadIdx.x >> 6] = any; lds.ups[threadIdx.x >> 6] = all; }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) { any |= lds.waves[i]; all &= lds.ups[i]; }
  if (any == all) return any;
  return select(lds, 64 - __builtin_clzll(any ^ all), want, [&](const auto& f) {
#pragma unroll
    for (int j = 0; j < N; ++j) f(order[j], w[j]);
  });
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

// The cuts of logits that `each` visits (logit, index) into r.cut, top_k and then top_p
template <int NT, class Each>
__device__ __forceinline__ void cut_row(SampleLds<NT>& lds, Row& r, const Each& each) {
  const int bits = 32 - r.spare + r.bits;
  if (r.top_k) {
    u64 n = 0;
    each([&](float x, int) { n += x > -INFINITY; });
    n = sum_of_block(lds, n);
    if (n >= (u64)r.top_k) r.cut = select(lds, bits, (u64)r.top_k, [&](const auto& f) { each([&](float x, int i) { f(r.place(x, i), x > -INFINITY ? 1 : 0); }); });
  }
  if (r.top_p < 1.f) {
    const u64 cut = r.cut;
    const auto weight = [&](float x, int i) { return x > -INFINITY && r.place(x, i) <= cut ? r.steps(r.weight(x)) : 0; };
    u64 n = 0;
    each([&](float x, int i) { n += weight(x, i); });
    n = sum_of_block(lds, n);
    r.cut = select(lds, bits, part_of(r.top_p, n), [&](const auto& f) { each([&](float x, int i) { f(r.place(x, i), weight(x, i)); }); });
  }
}
// The draw among those of them that are left, and the sum of these
template <int NT, class Each>
__device__ __forceinline__ int draw_row(SampleLds<NT>& lds, const SampleArgs& a, int row, const Row& r, u64& total, const Each& each) {
  total = 0;
  each([&](float x, int i) { total += r.steps(r.kept(x, i)); });
  total = sum_of_block(lds, total);
  return (int)select(lds, r.bits, drawn_at(a, row, total), [&](const auto& f) { each([&](float x, int i) { f((u64)i, r.steps(r.kept(x, i))); }); });
}

// Both for what the threads have in registers: logits, their numbers, and which of them there are by x > -inf.  What is left of each
// comes back in w
template <int NT, int N>
__device__ __forceinline__ int draw_held(SampleLds<NT>& lds, const SampleArgs& a, int row, Row& r, u64& total, const float (&x)[N], const int (&at)[N], double (&w)[N]) {
  u64 p[N], s[N];
#pragma unroll
  for (int j = 0; j < N; ++j) p[j] = r.place(x[j], at[j]);
  if (r.top_k) {
    u64 n = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) n += s[j] = x[j] > -INFINITY;
    n = sum_of_block(lds, n);
    if (n >= (u64)r.top_k) r.cut = select_held(lds, (u64)r.top_k, p, s);               // also where there are no more than these
  }
#pragma unroll
  for (int j = 0; j < N; ++j) w[j] = x[j] > -INFINITY && p[j] <= r.cut ? r.weight(x[j]) : 0.0;
  if (r.top_p < 1.f) {
    u64 n = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) n += s[j] = r.steps(w[j]);
    n = sum_of_block(lds, n);
    r.cut = select_held(lds, part_of(r.top_p, n), p, s);
  }
  total = 0;
  u64 i[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    w[j] = p[j] <= r.cut ? r.left(w[j]) : 0.0;
    total += s[j] = r.steps(w[j]);
    i[j] = (unsigned)at[j];
  }
  total = sum_of_block(lds, total);
  return (int)select_held(lds, drawn_at(a, row, total), i, s);
}

// The same for up to SM_FEW of them, whose places and weights are in LDS, by the first wave alone, two a lane: each adds up what
// stands before it in the order of falling logits, and then what of the kept ones stands before it in the vocabulary's
template <int NT>
__device__ __forceinline__ int draw_few(SampleLds<NT>& lds, const SampleArgs& a, int row, Row& r, int n, u64& total) {
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    const u64 index = (1ull << r.bits) - 1;
    u64 p[2], s[2], before[2] = {}, last = 0;
    double w[2];
    int rank[2] = {};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int i = lane + 64 * j;
      p[j] = i < n ? lds.place[i] : ~0ull;
      w[j] = i < n ? lds.weight[i] : 0.0;
      s[j] = r.steps(w[j]);
      lds.steps[i] = s[j];
    }
    wave_sync();
    for (int i = 0; i < n; ++i) {
      const u64 pi = lds.place[i], si = lds.steps[i];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        rank[j] += pi < p[j];
        before[j] += pi < p[j] ? si : 0;
      }
    }
    bool kept[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) kept[j] = lane + 64 * j < n && (!r.top_k || rank[j] < r.top_k);
    if (r.top_p < 1.f) {
      const u64 want = part_of(r.top_p, sum_of_wave((kept[0] ? s[0] : 0) + (kept[1] ? s[1] : 0)));
#pragma unroll
      for (int j = 0; j < 2; ++j) kept[j] = kept[j] && before[j] < want;
    }
    u64 up[2] = {};
    wave_sync();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      last = kept[j] && p[j] > last ? p[j] : last;
      s[j] = kept[j] ? r.steps(r.left(w[j])) : 0;
      lds.steps[lane + 64 * j] = s[j];
    }
    wave_sync();
    last = last_lane(scan_of(last, 0, Most()));
    const u64 sum = sum_of_wave(s[0] + s[1]), want = drawn_at(a, row, sum);
    for (int i = 0; i < n; ++i) {
      const u64 pi = lds.place[i] & index, si = lds.steps[i];
#pragma unroll
      for (int j = 0; j < 2; ++j) up[j] += pi <= (p[j] & index) ? si : 0;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (up[j] >= want && up[j] - s[j] < want) lds.digit = (int)(p[j] & index);
    if (lane == 0) {
      lds.before = sum;
      lds.found = last;
    }
  }
  __syncthreads();
  total = lds.before;
  r.cut = lds.found;
  return lds.digit;
}

// ---- rows of a block -----------------------------------------------------------------------------------------------------------
template <class X, int NT>
__global__ __launch_bounds__(NT) void sample_small_kernel(const SampleArgs a) {
  constexpr int N = 4;
  __shared__ SampleLds<NT> lds;
  const int tid = threadIdx.x, row = blockIdx.x, V = a.V;
  const X* logits = (const X*)a.logits + row * a.stride;
  for (int i = tid; i < SM_BINS; i += NT) lds.sums[i] = 0;
  if (tid == 0) lds.few = 0;
  float x[N], top = -INFINITY;
  int at[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    at[j] = j * NT + tid;
    x[j] = at[j] < V ? taken(logit(logits, at[j])) : -INFINITY;
  }
  Row r = row_of<X>(a, row);
#pragma unroll
  for (int j = 0; j < N; ++j) top = fmaxf(top, x[j]);
  const bool some = r.begin(max_of_block(lds, top));
  u64 total = 0;
  double w[N] = {};
  int token = -1;                                                    // nothing to draw from
  if (some) {
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = r.seen(x[j]);
    // what may be kept, where that is little: all of a small row, or what is no further from the largest than the last of top_k
    int at_most = -1;
    if (V <= SM_FEW) at_most = SM_BINS;
    else if (r.top_k && r.top_k < SM_FEW) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (x[j] > -INFINITY) atomicAdd(&lds.sums[r.distance(x[j])], 1ull);
      __syncthreads();
      at_most = crossing(lds, [&](u64 n) { return n < (u64)r.top_k ? n : (u64)r.top_k; }).bin;
    }
    if (at_most >= 0) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (x[j] > -INFINITY && r.distance(x[j]) <= at_most) {
          const int n = atomicAdd(&lds.few, 1);
          if (n < SM_FEW) {
            lds.place[n] = r.place(x[j], at[j]);
            lds.weight[n] = r.weight(x[j]);
          }
        }
      __syncthreads();
    }
    if (at_most >= 0 && lds.few <= SM_FEW) {
      token = draw_few(lds, a, row, r, lds.few, total);
      if (a.probs)
#pragma unroll
        for (int j = 0; j < N; ++j) w[j] = r.kept(x[j], at[j]);
    } else {
      token = draw_held(lds, a, row, r, total, x, at, w);
    }
  }
  if (tid == 0) a.tokens[row] = token;
  if (a.probs) {
    const double f = some ? share_of(a, total) : 0.0;
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (at[j] < V) a.probs[row * a.p_stride + at[j]] = (float)(w[j] * f);
  }
}

// ---- rows of several blocks ------------------------------------------------------------------------------------------------------
// What a row needs between launches where it may be cut
struct RowWork {
  u64 weights[SM_BINS];            // by distance from the largest
  unsigned counts[SM_BINS];
  u64 list[SM_LIST];               // logits and, behind them, their indexes
  unsigned listed, pad;            // more than SM_LIST: not all of them are there
};
struct RowEnd { u64 cut; double share; };        // what it comes to
// How a row is cut
enum Kind { CUT_NONE, CUT_BEST, CUT_COUNT, CUT_WEIGHT, CUT_SLOWLY }; // to the first of the largest; all that is kept in the list; the list at the cut; digit by digit of the whole row
__device__ __forceinline__ Kind kind_of(const Row& r) {
  if (r.top_k == 1) return CUT_BEST;
  if (r.top_k) return r.top_k <= SM_MOST ? CUT_COUNT : CUT_SLOWLY;
  return r.top_p < 1.f ? CUT_WEIGHT : CUT_NONE;
}
struct Work {                      // of a call
  RowWork* rows;                   // [n], or nullptr: none is cut
  RowEnd* done;                    // [n]
  float2* ends;                    // [n][parts]: the largest, and of every eighth the smallest but -inf
  u64* runs;                       // [n][runs]
  int* best;                       // [n][parts]: the first of the largest, for rows of which no other is kept
  int parts, len, n_runs;          // blocks of a row, logits of one, sums of a row
};

// f(logits, which may be NaN, index of the first, run) for a block's part of a row, run by run, eight logits a lane, the next run's on their way; what
// lies behind the row is -inf
template <class X, class F>
__device__ __forceinline__ void each_run(const SampleArgs& a, const Work& w, int row, int part, const Row& r, const F& f) {
  typedef __attribute__((ext_vector_type(8), aligned(sizeof(X)))) X X8;                // rows of odd vocabularies start anywhere
  const X* logits = (const X*)a.logits + row * a.stride;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, end = min((part + 1) * w.len, a.V);
  const auto load = [&](int i) {
    X8 x;
    if (i + 8 <= a.V) return *(const X8*)(logits + i);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = i + e < a.V ? logits[i + e] : (X)-INFINITY;
    return x;
  };
  const int first = part * w.len + wave * SM_RUN;
  X8 now = {};
  if (first < end) now = load(first + 8 * lane);
  for (int i0 = first; i0 < end;) {
    const X8 this_one = now;
    const int i1 = i0 + SM_T / 64 * SM_RUN;
    if (i1 < end) now = load(i1 + 8 * lane);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)this_one[e];
    if (r.infinite)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = r.seen(x[e]);
    f(x, i0 + 8 * lane, i0 / SM_RUN);
    i0 = i1;
  }
}
__device__ __forceinline__ float2 ends_of(const Work& w, int row) {
  float2 ends = {-INFINITY, INFINITY};
  for (int p = threadIdx.x & 63; p < w.parts; p += 64) {
    const float2 x = w.ends[row * w.parts + p];
    ends = float2{fmaxf(ends.x, x.x), fminf(ends.y, x.y)};
  }
  return float2{max_of_wave(ends.x), -max_of_wave(-ends.y)};
}

template <class X>
__global__ __launch_bounds__(SM_T) void sample_top_kernel(const SampleArgs a, const Work w) {
  __shared__ SampleLds<SM_T> lds;
  const int row = blockIdx.x / w.parts, part = blockIdx.x % w.parts;
  if (part == 0 && w.rows) {
    RowWork& rw = w.rows[row];
    for (int i = threadIdx.x; i < SM_BINS; i += SM_T) {
      rw.weights[i] = 0;
      rw.counts[i] = 0;
    }
    if (threadIdx.x == 0) rw.listed = 0;
  }
  float top = -INFINITY, low = INFINITY;
  int at = INT_MAX;                                                  // the first of the lane's largest
  const Row r = row_of<X>(a, row);
  const bool best = kind_of(r) == CUT_BEST;
  each_run<X>(a, w, row, part, r, [&](const float (&x)[8], int i, int) {
    float most = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = fmaxf(most, x[e]);
    low = fminf(low, x[0] > -INFINITY ? x[0] : INFINITY);
    if (best && most > top)
#pragma unroll
      for (int e = 7; e >= 0; --e) at = x[e] == most ? i + e : at;
    top = fmaxf(top, most);
  });
  const float mine = top;
  if (threadIdx.x == 0) lds.digit = INT_MAX;
  top = max_of_block(lds, top);
  __syncthreads();
  if (best && mine == top) atomicMin(&lds.digit, at);
  low = -max_of_block(lds, -low);
  if (threadIdx.x == 0) {
    w.ends[blockIdx.x] = float2{top, low};
    if (best) w.best[blockIdx.x] = lds.digit;
  }
}

template <class X>
__global__ __launch_bounds__(SM_T) void sample_sums_kernel(const SampleArgs a, const Work w) {
  __shared__ u64 weights[SM_BINS];
  __shared__ unsigned counts[SM_BINS];
  const int row = blockIdx.x / w.parts, part = blockIdx.x % w.parts;
  Row r = row_of<X>(a, row);
  const Kind kind = kind_of(r);
  if (kind != CUT_COUNT && kind != CUT_WEIGHT) return;
  if (!r.begin(ends_of(w, row))) return;
  RowWork& rw = w.rows[row];
  for (int i = threadIdx.x; i < SM_BINS; i += SM_T) {
    if (kind == CUT_COUNT) counts[i] = 0;
    else weights[i] = 0;
  }
  __syncthreads();
  if (kind == CUT_COUNT)
    each_run<X>(a, w, row, part, r, [&](const float (&x)[8], int, int) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (x[e] > -INFINITY) atomicAdd(&counts[r.distance(x[e])], 1u);
    });
  else
    each_run<X>(a, w, row, part, r, [&](const float (&x)[8], int, int) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const u64 s = r.steps(r.weight(x[e]));
        if (s) atomicAdd(&weights[r.distance(x[e])], s);
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

// The distance that the row's cut lies at, and what is wanted of it there; SM_BINS: it is not cut.  of(j): sum j of the thread's
template <int NT, class Of>
__device__ __forceinline__ int cut_at(SampleLds<NT>& lds, const Row& r, Kind kind, u64& want, const Of& of) {
#pragma unroll
  for (int i = 0; i < SM_BINS / NT; ++i) lds.sums[i * NT + threadIdx.x] = of(i);
  __syncthreads();
  const Crossing c = crossing(lds, [&](u64 all) { return kind == CUT_WEIGHT ? part_of(r.top_p, all) : all < (u64)r.top_k ? all : (u64)r.top_k; });
  want = c.want;
  return kind == CUT_COUNT && c.total <= (u64)r.top_k ? SM_BINS : c.bin;
}

template <class X>
__global__ __launch_bounds__(SM_T) void sample_list_kernel(const SampleArgs a, const Work w) {
  __shared__ SampleLds<SM_T> lds;
  __shared__ u64 list[SM_STAGE];
  __shared__ unsigned listed, first;
  const int row = blockIdx.x / w.parts, part = blockIdx.x % w.parts, tid = threadIdx.x, lane = tid & 63;
  Row r = row_of<X>(a, row);
  const Kind kind = kind_of(r);
  if (kind == CUT_SLOWLY || kind == CUT_BEST) return;
  if (!r.begin(ends_of(w, row))) return;
  RowWork* const rw = w.rows + row;                                  // looked at only where the row is cut
  int at = SM_BINS;
  u64 want;
  if (tid == 0) listed = 0;
  if (kind != CUT_NONE) at = cut_at(lds, r, kind, want, [&](int j) { return kind == CUT_COUNT ? (u64)rw->counts[j * SM_T + tid] : rw->weights[j * SM_T + tid]; });
  __syncthreads();
  const auto add = [&](float x, int i) {
    const u64 v = (u64)__float_as_uint(x) << 32 | (unsigned)i;
    const unsigned n = atomicAdd(&listed, 1u);
    if (n < SM_STAGE) list[n] = v;
    else {                                                           // more than are written out together
      const unsigned m = atomicAdd(&rw->listed, 1u);
      if (m < SM_LIST) rw->list[m] = v;
    }
  };
  const auto end_run = [&](u64 sum, int run) {
    sum = sum_of_wave(sum);
    if (lane == 0) w.runs[(long)row * w.n_runs + run] = sum;
  };
  // of n logits, a lane's
  const auto sum_of = [&](int n, const auto& logit_at) {
    u64 sum = 0;
    int adds = 0;
    if (r.min_p > 0.0)
      for (int j = lane; j < n; j += 64) sum += r.steps(r.left(r.weight(logit_at(j))));
    else
      for (int j = lane; j < n; j += 64, ++adds) sum += (u64)__double_as_longlong(r.weight(logit_at(j)) + r.magic);       // the power of two that carries the steps comes off together
    return sum - (u64)adds * (u64)__double_as_longlong(r.magic);
  };
  if (kind == CUT_COUNT) {
    each_run<X>(a, w, row, part, r, [&](const float (&x)[8], int i, int) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (r.distance(x[e]) <= at && x[e] > -INFINITY) add(x[e], i + e);
    });
  } else if (kind == CUT_WEIGHT) {
    // The ones above the cut move together first: of 512 logits they are fewer than half as a rule, and the weights are what takes time
    float* above = (float*)lds.sums + (tid >> 6) * SM_RUN;
    static_assert(sizeof(lds.sums) >= SM_T / 64 * SM_RUN * sizeof(float), "a wave's run");
    const unsigned from = (unsigned)at << 15, width = at < SM_BINS - 1 ? 1u << 15 : ~0u - from;
    each_run<X>(a, w, row, part, r, [&](const float (&x)[8], int i, int run) {
      int n = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const unsigned d = r.far(x[e]);
        const u64 yes = __ballot(d < from);
        if (d < from) above[n + __builtin_amdgcn_mbcnt_hi((unsigned)(yes >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)yes, 0))] = x[e];
        n += __popcll(yes);
        if (d - from < width && x[e] > -INFINITY) add(x[e], i + e);
      }
      wave_sync();                                                   // a wave's own
      end_run(sum_of(n, [&](int j) { return above[j]; }), run);
      wave_sync();
    });
  } else {
    each_run<X>(a, w, row, part, r, [&](const float (&x)[8], int, int run) {
      u64 sum = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += r.steps(r.left(r.weight(x[e])));
      end_run(sum, run);
    });
  }
  __syncthreads();
  const unsigned n = min(listed, (unsigned)SM_STAGE);
  if (tid == 0 && n) first = atomicAdd(&rw->listed, n);               // none without a cut
  __syncthreads();
  for (unsigned j = tid; j < n && first + j < SM_LIST; j += SM_T) rw->list[first + j] = list[j];
}

template <class X>
__global__ __launch_bounds__(SM_FINAL) void sample_draw_kernel(const SampleArgs a, const Work w) {
  constexpr int N = SM_HELD / SM_FINAL;
  __shared__ SampleLds<SM_FINAL> lds;
  const int tid = threadIdx.x, row = blockIdx.x;
  const X* logits = (const X*)a.logits + row * a.stride;
  RowWork* const rw = w.rows + row;                                  // looked at only where there are any
  Row r = row_of<X>(a, row);
  const Kind kind = kind_of(r);
  // everything that the launches before have left, in one round trip
  u64 held[N] = {}, sums[SM_BINS / SM_FINAL] = {}, runs[SM_BINS / SM_FINAL];
  unsigned listed = 0;
  if (w.rows) {
#pragma unroll
    for (int j = 0; j < N; ++j) held[j] = rw->list[j * SM_FINAL + tid];
#pragma unroll
    for (int j = 0; j < SM_BINS / SM_FINAL; ++j) sums[j] = rw->weights[j * SM_FINAL + tid];
    listed = rw->listed;
  }
#pragma unroll
  for (int j = 0; j < SM_BINS / SM_FINAL; ++j) {
    const int i = j * SM_FINAL + tid;
    runs[j] = i < w.n_runs ? w.runs[(long)row * w.n_runs + i] : 0;
    lds.sums[i] = 0;
  }
  __syncthreads();
  const float2 ends = ends_of(w, row);
  if (!r.begin(ends)) {                                              // nothing to draw from
    if (tid == 0) {
      a.tokens[row] = -1;
      w.done[row] = RowEnd{0, 0.0};
    }
    return;
  }
  u64 total;
  int token;
  const unsigned m = kind == CUT_COUNT || kind == CUT_WEIGHT ? listed : 0;
  if (kind == CUT_BEST) {
    u64 first = INT_MAX;                                             // the complement of the largest is the smallest
    for (int p = tid & 63; p < w.parts; p += 64)
      if (w.ends[row * w.parts + p].x == ends.x) first = min(first, (u64)w.best[row * w.parts + p]);
    token = (int)~last_lane(scan_of(~first, 0, Most()));
    r.cut = r.place(r.top32, token);
    total = r.steps(1.0);
  } else if (kind == CUT_SLOWLY || m > SM_LIST) {
    const auto each = [&](const auto& f) {
      for (int i = tid; i < a.V; i += SM_FINAL) f(r.seen(logit(logits, i)), i);
    };
    cut_row(lds, r, each);
    token = draw_row(lds, a, row, r, total, each);
  } else if (kind == CUT_COUNT && m > SM_HELD) {
    const auto each = [&](const auto& f) {
      for (unsigned i = tid; i < m; i += SM_FINAL) f(__uint_as_float((unsigned)(rw->list[i] >> 32)), (int)rw->list[i]);
    };
    cut_row(lds, r, each);
    token = draw_row(lds, a, row, r, total, each);
  } else {
    float x[N];
    int at[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const bool is = j * SM_FINAL + tid < m;
      x[j] = is ? __uint_as_float((unsigned)(held[j] >> 32)) : -INFINITY;
      at[j] = is ? (int)held[j] : 0;
    }
    if (kind == CUT_COUNT && m <= SM_FEW) {
      if (tid < (int)m) {
        lds.place[tid] = r.place(x[0], at[0]);
        lds.weight[tid] = r.weight(x[0]);
      }
      __syncthreads();
      token = draw_few(lds, a, row, r, (int)m, total);
    } else if (kind == CUT_COUNT) {
      double left[N];
      token = draw_held(lds, a, row, r, total, x, at, left);
    } else {
      if (kind == CUT_WEIGHT) {
        u64 want, p[N], s[N];
        cut_at(lds, r, kind, want, [&](int j) { return sums[j]; });
        if (m > SM_HELD) {
          r.cut = select(lds, 32 - r.spare + r.bits, want, [&](const auto& f) {
            for (unsigned i = tid; i < m; i += SM_FINAL) {
              const float l = __uint_as_float((unsigned)(rw->list[i] >> 32));
              f(r.place(l, (int)rw->list[i]), r.steps(r.weight(l)));
            }
          });
        } else {
#pragma unroll
          for (int j = 0; j < N; ++j) {
            p[j] = r.place(x[j], at[j]);
            s[j] = x[j] > -INFINITY ? r.steps(r.weight(x[j])) : 0;
          }
          r.cut = select_held(lds, want, p, s);
        }
      }
      // the runs' sums with what is kept of the list; then the run that the draw falls into
      __syncthreads();
#pragma unroll
      for (int j = 0; j < SM_BINS / SM_FINAL; ++j) lds.sums[j * SM_FINAL + tid] = runs[j];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const u64 s = r.steps(r.kept(x[j], at[j]));
        if (s) atomicAdd(&lds.sums[at[j] / SM_RUN], s);
      }
      for (unsigned i = SM_HELD + tid; i < m; i += SM_FINAL) {
        const u64 s = r.steps(r.kept(__uint_as_float((unsigned)(rw->list[i] >> 32)), (int)rw->list[i]));
        if (s) atomicAdd(&lds.sums[(int)rw->list[i] / SM_RUN], s);
      }
      __syncthreads();
      const Crossing c = crossing(lds, [&](u64 all) { return drawn_at(a, row, all); });
      total = c.total;
      static_assert(SM_FINAL == SM_RUN, "a logit of the run a thread");
      const int i = c.bin * SM_RUN + tid;
      token = c.bin * SM_RUN + reached_at(lds, i < a.V ? r.steps(r.kept(r.seen(logit(logits, i)), i)) : 0, c.want);
    }
  }
  if (tid == 0) {
    a.tokens[row] = token;
    w.done[row] = RowEnd{r.cut, share_of(a, total)};
  }
}

template <class X>
__global__ __launch_bounds__(SM_T) void sample_probs_kernel(const SampleArgs a, const Work w) {
  const int row = blockIdx.x / w.parts, part = blockIdx.x % w.parts;
  Row r = row_of<X>(a, row);
  r.begin(ends_of(w, row));
  r.cut = w.done[row].cut;
  const double f = w.done[row].share;
  float* out = a.probs + row * a.p_stride;
  each_run<X>(a, w, row, part, r, [&](const float (&x)[8], int i, int) {
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = f > 0.0 ? (float)(r.kept(x[e], i + e) * f) : 0.f;
    if (i + 8 <= a.V) {
      typedef __attribute__((ext_vector_type(4), aligned(4))) float v4;
      *(v4*)(out + i) = v4{p[0], p[1], p[2], p[3]};
      *(v4*)(out + i + 4) = v4{p[4], p[5], p[6], p[7]};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (i + e < a.V) out[i + e] = p[e];
    }
  });
}

// What is known of all rows: that one logit is kept of each (temperature 0, top_k 1), which the first reading finds; that none is cut
static bool keeps_one(const SampleArgs& a) { return (!a.temperature_of && a.temperature == 0.f) || (!a.top_k_of && a.top_k == 1); }
static bool cuts_none(const SampleArgs& a) { return keeps_one(a) || (!a.top_k_of && !a.top_p_of && !a.top_k && !(a.top_p < 1.f)); }

// Rows of long logits that are worked on at a time, in the same memory: 90 KB and 1 / 64 byte a logit each, which for all rows of a large
// batch would be more than its logits (65536 of 4097: 5.9 GB beside 1.1).  A turn more costs 12 us, of the 260 that so many rows of 5000 take
// (with turns of 1024, 4096 rows of 5000 took 169 us instead of 131)
constexpr int SM_ROWS = 8192;

// Blocks of a row: as many as make 512 of all rows, two on a CU, with 8 turns of a wave or more each.  The memory goes by rows and
// vocabulary alone, so that a workspace serves calls of other settings, too
static Work work_of(int n, int V, void* work) {
  Work w = {};
  const long want = ((long)n * V + 511) / 512, turn = SM_T / 64 * SM_RUN;
  w.len = (int)(std::min(std::max((want + turn - 1) / turn, 1l), (V + turn - 1) / turn) * turn);
  w.parts = (V + w.len - 1) / w.len;
  w.n_runs = (V + SM_RUN - 1) / SM_RUN;
  w.rows = (RowWork*)work;
  w.done = (RowEnd*)(w.rows + n);
  w.runs = (u64*)(w.done + n);
  w.ends = (float2*)(w.runs + (long)n * w.n_runs);
  w.best = (int*)(w.ends + (long)n * w.parts);
  return w;
}
size_t sample_workspace(int n, int vocab) {
  if (vocab <= SM_SMALL) return 0;
  n = std::min(n, SM_ROWS);
  const Work w = work_of(n, vocab, nullptr);
  return n * (sizeof(RowWork) + sizeof(RowEnd) + w.n_runs * sizeof(u64) + w.parts * (sizeof(float2) + sizeof(int)));
}

template <class X>
static hipError_t sample_of(SampleArgs a, hipStream_t s) {
  if (a.V <= SM_SMALL) {
    if (!fits_a_launch(a.n, 1024)) return hipErrorInvalidConfiguration;
    if (a.V <= 1024) hipLaunchKernelGGL((sample_small_kernel<X, 256>), dim3(a.n), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((sample_small_kernel<X, 1024>), dim3(a.n), dim3(1024), 0, s, a);
    return hipGetLastError();
  }
  Work w = work_of(std::min(a.n, SM_ROWS), a.V, a.work);
  const bool one = keeps_one(a);
  if (cuts_none(a)) w.rows = nullptr;
  for (int left = a.n;;) {
    a.n = std::min(left, SM_ROWS);
    const dim3 grid(a.n * w.parts), block(SM_T);
    hipLaunchKernelGGL(sample_top_kernel<X>, grid, block, 0, s, a, w);
    if (w.rows) hipLaunchKernelGGL(sample_sums_kernel<X>, grid, block, 0, s, a, w);
    if (!one) hipLaunchKernelGGL(sample_list_kernel<X>, grid, block, 0, s, a, w);
    hipLaunchKernelGGL(sample_draw_kernel<X>, dim3(a.n), dim3(SM_FINAL), 0, s, a, w);
    if (a.probs) hipLaunchKernelGGL(sample_probs_kernel<X>, grid, block, 0, s, a, w);
    if ((left -= a.n) == 0) return hipGetLastError();
    a.logits = (const X*)a.logits + a.n * a.stride;
    a.u += a.n;
    a.tokens += a.n;
    if (a.probs) a.probs += a.n * a.p_stride;
    if (a.temperature_of) a.temperature_of += a.n;
    if (a.top_p_of) a.top_p_of += a.n;
    if (a.min_p_of) a.min_p_of += a.n;
    if (a.top_k_of) a.top_k_of += a.n;
  }
}
hipError_t launch_sample(SampleArgs a, int dtype, hipStream_t s) {
  int bits = 0;
  while (1 << bits < a.V) ++bits;
  a.scale_bits = 62 - bits < 51 ? 62 - bits : 51;
  return dtype == SNA_DTYPE_FP32 ? sample_of<float>(a, s) : dtype == SNA_DTYPE_BF16 ? sample_of<__bf16>(a, s) : sample_of<_Float16>(a, s);
}

}  // namespace sna
