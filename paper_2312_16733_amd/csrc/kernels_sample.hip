// A token of each row of logits, from a given random number.
//   w_i = exp((l_i - max) / temperature);  in the order of falling l (then rising i):  the first top_k;  of these the fewest whose
//   weights make top_p of theirs;  of these the ones with w_i >= min_p.  The token is the smallest i for which the weights of the
//   ones that are left, up to i in the vocabulary's order, make more than u of all of them.
// Weights are formed in 64 bits and summed as whole numbers, steps of 2^-scale_bits of the largest (2^-44 for 2^18 logits): the sums
// of many do not depend on their order, so that they can come together through atomics, and are as exact as 64-bit floats would be.
// Nothing is sorted.  Where the order is cut, and where the draw falls, is found digit by digit of the logits' bit patterns (or of
// the index): sums by digit in LDS, the digit that the wanted sum falls into, then the same among what has that digit.
#include "paged.h"

namespace sna {

typedef unsigned long long u64;
constexpr int SM_T = 1024;         // threads of a block
constexpr int SM_BINS = 2048;      // values of a digit

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

struct Row {                       // of logits, and what is wanted of it
  float top;
  double inv_t, magic, min_p;
  u64 cut;                         // (falling, index) of the last one kept
  __device__ __forceinline__ double weight(float x) const { return x == top ? 1.0 : exp(((double)x - (double)top) * inv_t); }
  // In steps: the sum with a power of two whose last place is a step
  __device__ __forceinline__ u64 steps(double w) const { return (u64)__double_as_longlong(w + magic) & 0xfffffffffffffull; }
};
__device__ __forceinline__ u64 place(float x, int i) { return (u64)falling(x) << 32 | (unsigned)i; }

struct SampleLds {
  u64 sums[SM_BINS], waves[SM_T / 64], before;
  int digit;
  float top[SM_T / 64];
};

__device__ __forceinline__ u64 scan_up(u64 v) {                      // inclusive, of a wave
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const u64 x = __shfl_up(v, m, 64);
    if (lane >= m) v += x;
  }
  return v;
}

// The digit at which the running sum of lds.sums reaches `want` (1 or more, at most the sum of all), and what comes before it.
// All threads get both.
__device__ __forceinline__ void crossing(SampleLds& lds, u64 want, int& digit, u64& before) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const u64 a = lds.sums[2 * tid], b = lds.sums[2 * tid + 1], up = scan_up(a + b);
  if (lane == 63) lds.waves[wave] = up;
  __syncthreads();
  u64 base = 0;
  for (int w = 0; w < wave; ++w) base += lds.waves[w];
  const u64 at = base + up - a - b;
  if (at < want && want <= at + a) { lds.digit = 2 * tid; lds.before = at; }
  else if (at + a < want && want <= at + a + b) { lds.digit = 2 * tid + 1; lds.before = at + a; }
  __syncthreads();
  digit = lds.digit;
  before = lds.before;
}

// All items x = (order, weight) that `each` visits, in rising order: that at which the running sum of weights reaches `want`, which
// is 1 .. the sum of all.  Returns its order, and in `before` the sum of what comes before it.  All threads.
template <class Each>
__device__ u64 select(SampleLds& lds, int bits, u64 want, u64& before, const Each& each) {
  u64 lo = 0;
  before = 0;
  for (int left = bits; left > 0;) {
    const int width = min(left, 11), shift = left - width;
    for (int i = threadIdx.x; i < SM_BINS; i += SM_T) lds.sums[i] = 0;
    __syncthreads();
    each([&](u64 order, u64 w) {
      if ((left == 64 || order >> left == lo >> left) && w) atomicAdd(&lds.sums[order >> shift & ((1 << width) - 1)], w);
    });
    __syncthreads();
    int digit;
    u64 b;
    crossing(lds, want - before, digit, b);
    lo |= (u64)digit << shift;
    before += b;
    left = shift;
    __syncthreads();
  }
  return lo;
}
__device__ __forceinline__ u64 sum_of_block(SampleLds& lds, u64 v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds.waves[threadIdx.x >> 6] = v;
  __syncthreads();
  u64 s = 0;
  for (int w = 0; w < SM_T / 64; ++w) s += lds.waves[w];
  return s;
}
// A fraction f of a sum of s steps, upwards, as a sum that can be reached
__device__ __forceinline__ u64 part_of(double f, u64 s) {
  const u64 want = (u64)ceil(fmax(f, 0.0) * (double)s);
  return want < 1 ? 1 : want > s ? s : want;
}

template <class X>
__global__ __launch_bounds__(SM_T) void sample_row_kernel(const SampleArgs a) {
  __shared__ SampleLds lds;
  const int tid = threadIdx.x, row = blockIdx.x, V = a.V;
  const X* logits = (const X*)a.logits + row * a.stride;
  const float t = a.temperature_of ? a.temperature_of[row] : a.temperature, top_p = a.top_p_of ? a.top_p_of[row] : a.top_p;
  int top_k = a.top_k_of ? a.top_k_of[row] : a.top_k;
  if (!(t > 0.f)) top_k = 1;
  Row r;
  r.inv_t = t > 0.f ? 1.0 / (double)fminf(t, 3.4028235e38f) : 0.0;
  r.min_p = fmin(fmax((double)(a.min_p_of ? a.min_p_of[row] : a.min_p), 0.0), 1.0);       // what is no number cuts nothing, and the largest stays
  r.magic = __longlong_as_double((long long)(1023 + 52 - a.scale_bits) << 52);
  float top = -INFINITY;
  for (int i = tid; i < V; i += SM_T) top = fmaxf(top, taken(logit(logits, i)));
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) top = fmaxf(top, __shfl_xor(top, m, 64));
  if ((tid & 63) == 0) lds.top[tid >> 6] = top;
  __syncthreads();
  for (int w = 0; w < SM_T / 64; ++w) top = fmaxf(top, lds.top[w]);
  r.top = top;
  r.cut = ~0ull;
  if (top == -INFINITY) {                                            // nothing to draw from
    if (tid == 0) a.tokens[row] = -1;
    if (a.probs)
      for (int i = tid; i < V; i += SM_T) a.probs[row * a.p_stride + i] = 0.f;
    return;
  }
  u64 before;
  if (top_k > 0 && top_k < V) {
    u64 n = 0;
    for (int i = tid; i < V; i += SM_T) n += taken(logit(logits, i)) > -INFINITY;
    n = sum_of_block(lds, n);
    if (n > (u64)top_k)
      r.cut = select(lds, 64, (u64)top_k, before, [&](const auto& f) {
        for (int i = tid; i < V; i += SM_T) {
          const float x = taken(logit(logits, i));
          f(place(x, i), x > -INFINITY ? 1 : 0);
        }
      });
  }
  const auto kept = [&](float x, int i) { return x > -INFINITY && place(x, i) <= r.cut; };
  if (top_p < 1.f) {
    const u64 cut = r.cut;
    u64 n = 0;
    for (int i = tid; i < V; i += SM_T) {
      const float x = taken(logit(logits, i));
      if (kept(x, i)) n += r.steps(r.weight(x));
    }
    n = sum_of_block(lds, n);
    r.cut = select(lds, 64, part_of(top_p, n), before, [&](const auto& f) {
      for (int i = tid; i < V; i += SM_T) {
        const float x = taken(logit(logits, i));
        f(place(x, i), x > -INFINITY && place(x, i) <= cut ? r.steps(r.weight(x)) : 0);
      }
    });
  }
  const auto weight = [&](float x, int i) {
    if (!kept(x, i)) return 0.0;
    const double w = r.weight(x);
    return w >= r.min_p ? w : 0.0;
  };
  u64 total = 0;
  for (int i = tid; i < V; i += SM_T) total += r.steps(weight(taken(logit(logits, i)), i));
  total = sum_of_block(lds, total);
  const double u = fmin(fmax((double)a.u[row], 0.0), 1.0);
  u64 want = (u64)(u * (double)total) + 1;
  if (want > total) want = total;
  const u64 token = select(lds, 32 - __builtin_clz(V), want, before, [&](const auto& f) {
    for (int i = tid; i < V; i += SM_T) f((u64)i, r.steps(weight(taken(logit(logits, i)), i)));
  });
  if (tid == 0) a.tokens[row] = (int)token;
  if (a.probs) {
    const double f = 1.0 / ((double)total * __longlong_as_double((long long)(1023 - a.scale_bits) << 52));
    for (int i = tid; i < V; i += SM_T) a.probs[row * a.p_stride + i] = (float)(weight(taken(logit(logits, i)), i) * f);
  }
}

size_t sample_workspace(int, int, int) { return 0; }

template <class X>
static hipError_t sample_of(const SampleArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(sample_row_kernel<X>, dim3(a.n), dim3(SM_T), 0, s, a);
  return hipGetLastError();
}
hipError_t launch_sample(SampleArgs a, int dtype, hipStream_t s) {
  int bits = 0;
  while (1 << bits < a.V) ++bits;
  a.scale_bits = 62 - bits < 51 ? 62 - bits : 51;
  if (!fits_a_launch(a.n, SM_T)) return hipErrorInvalidConfiguration;
  return dtype == SNA_DTYPE_FP32 ? sample_of<float>(a, s) : dtype == SNA_DTYPE_BF16 ? sample_of<__bf16>(a, s) : sample_of<_Float16>(a, s);
}

}  // namespace sna
