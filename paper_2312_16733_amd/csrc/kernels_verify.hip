// Verification of drafted tokens against the target's probabilities, from given random numbers.
//   drafted token i is taken while u_i q_i(x_i) < p_i(x_i) (and all before it are);  at the first that is not, a:
//   the next token is drawn from w = max(p_a - q_a, 0), or from p_a where nothing is left of it or all drafts are taken:
//   the smallest x with w_0 + .. + w_x > u_K (w_0 + .. + w_{V - 1})
// Products, differences, sums and the comparison are in 64 bits: u q is exact, and 10^5 probabilities summed in 32 bits would
// move the borders between tokens by more than many of them are worth.
// Bound by memory: two rows of the vocabulary a sequence, read once.  A block has a sequence; each of its waves sums a run of
// the row, then the run that holds the draw (V / 16 values, cached by now) is shared out over the waves, and the run of that
// over the lanes of one.  128 sequences of 131072: 19.2 us, 3.5 TB/s; 64 of 50257 with the draft's rows: 11.9 us, of which 4.5 are
// the round trips that follow each other (drafts, their probabilities, the rows, the draw), and one CU a sequence reads 0.4 MB.
#include "paged.h"

namespace sna {

constexpr int VD_W = 16;           // waves of a block
constexpr int VD_S = 8;            // values of a lane, where one wave looks for the draw

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, 64);
  return v;
}
__device__ __forceinline__ double wave_scan(double v) {              // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const double x = __shfl_up(v, m, 64);
    if (lane >= m) v += x;
  }
  return v;
}

typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4u;  // rows of odd vocabularies start anywhere

// The weights of one sequence's draw: a row of the target, less a row of the draft, or less one token, or all of it
enum Less { LESS_NOTHING, LESS_ROW, LESS_TOKEN };
struct Weights {
  const float* p; const float* q;
  int out;                         // the token taken out
};
template <Less L>
__device__ __forceinline__ double weight(const Weights& w, int x, float p, float q) {
  if (L == LESS_ROW) return fmax((double)p - (double)q, 0.0);        // NaN counts as nothing
  return L == LESS_TOKEN && x == w.out ? 0.0 : fmax((double)p, 0.0);
}

// Sum over [x0, x1) by one wave.  A wave asks for VD_U kilobytes of either row before it waits: with one at a time it waited
// out a round trip to memory for each.
constexpr int VD_U = 4;
template <Less L>
__device__ __forceinline__ double run_sum(const Weights& w, int x0, int x1) {
  const int lane = threadIdx.x & 63;
  double s[VD_U] = {};
  int x = x0 + 4 * lane;
  for (; x + 256 * (VD_U - 1) + 3 < x1; x += 256 * VD_U) {
    f32x4u p[VD_U], q[VD_U];
#pragma unroll
    for (int i = 0; i < VD_U; ++i) {
      p[i] = *(const f32x4u*)(w.p + x + 256 * i);
      if (L == LESS_ROW) q[i] = *(const f32x4u*)(w.q + x + 256 * i);
    }
#pragma unroll
    for (int i = 0; i < VD_U; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i] += weight<L>(w, x + 256 * i + e, p[i][e], L == LESS_ROW ? q[i][e] : 0.f);
  }
  // what is left: less than VD_U fours a lane, the last of one lane partial
  f32x4u p[VD_U], q[VD_U];
#pragma unroll
  for (int i = 0; i < VD_U; ++i)
    if (x + 256 * i + 3 < x1) {
      p[i] = *(const f32x4u*)(w.p + x + 256 * i);
      if (L == LESS_ROW) q[i] = *(const f32x4u*)(w.q + x + 256 * i);
    }
#pragma unroll
  for (int i = 0; i < VD_U; ++i) {
    const int y = x + 256 * i;
    if (y + 3 < x1) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i] += weight<L>(w, y + e, p[i][e], L == LESS_ROW ? q[i][e] : 0.f);
    } else {
      for (int z = y; z < x1; ++z) s[i] += weight<L>(w, z, w.p[z], L == LESS_ROW ? w.q[z] : 0.f);
    }
  }
  double t = 0.0;
#pragma unroll
  for (int i = 0; i < VD_U; ++i) t += s[i];
  return wave_sum(t);
}

// The run that a draw of `at` falls into, of VD_W with the given sums, `up` before the first of them: the first whose end lies
// beyond it, or the last with any weight where rounding leaves none.  `up` becomes what lies before that run.
__device__ __forceinline__ int run_of(const double* sums, double at, double& up) {
  int r = 0;
  bool found = false;
  double end = up;
#pragma unroll
  for (int i = 0; i < VD_W; ++i) {
    const double v = sums[i];
    if (!found && v > 0.0) { r = i; up = end; }
    end += v;
    found = found || end > at;
  }
  return uniform(r);
}

// The token that a draw with u falls on; -1 in `token` and a total of zero where there is nothing to draw from.  All waves.
template <Less L>
__device__ __forceinline__ double draw(const Weights& w, int V, double u, double* sums, int& token) {
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
  const int len1 = (((V + VD_W - 1) / VD_W) + 3) & ~3;               // values of a wave's run
  {
    const int x0 = min(V, wave * len1);
    const double s = run_sum<L>(w, x0, min(V, x0 + len1));
    if (lane == 0) sums[wave] = s;
  }
  __syncthreads();
  double total = 0.0, before = 0.0;
#pragma unroll
  for (int i = 0; i < VD_W; ++i) total += sums[i];
  if (!(total > 0.0)) return 0.0;
  const double at = u * total;
  int r = run_of(sums, at, before), s0 = min(V, r * len1), s1 = min(V, s0 + len1);
  if (len1 > 64 * VD_S) {                                            // too long for one wave's registers
    const int len2 = (((s1 - s0 + VD_W - 1) / VD_W) + 3) & ~3, x0 = min(s1, s0 + wave * len2);
    const double s = run_sum<L>(w, x0, min(s1, x0 + len2));
    if (lane == 0) sums[VD_W + wave] = s;
    __syncthreads();
    r = run_of(sums + VD_W, at, before);
    s0 = min(s1, s0 + r * len2);
    s1 = min(s1, s0 + len2);
  }
  if (wave != 0) return total;
  // VD_S values a lane at a time, in order (two turns and more for vocabularies of 131072 and more)
  for (int base = s0; base < s1; base += 64 * VD_S) {
    double v[VD_S], mine = 0.0;
    const int z0 = base + lane * VD_S;
    float p[VD_S], q[VD_S];
#pragma unroll
    for (int i = 0; i < VD_S; ++i)
      if (z0 + i < s1) {
        p[i] = w.p[z0 + i];
        if (L == LESS_ROW) q[i] = w.q[z0 + i];
      }
#pragma unroll
    for (int i = 0; i < VD_S; ++i) {
      v[i] = z0 + i < s1 ? weight<L>(w, z0 + i, p[i], L == LESS_ROW ? q[i] : 0.f) : 0.0;
      mine += v[i];
    }
    const double up = wave_scan(mine);
    double c = before + up - mine;
    int hit = -1, any = -1;
#pragma unroll
    for (int i = 0; i < VD_S; ++i) {
      c += v[i];
      if (v[i] > 0.0) {
        any = z0 + i;
        if (hit < 0 && c > at) hit = z0 + i;
      }
    }
    const unsigned long long hits = __ballot(hit >= 0), anys = __ballot(any >= 0);
    if (hits) {
      token = __shfl(hit, __ffsll((long long)hits) - 1, 64);
      break;
    }
    if (anys) token = __shfl(any, 63 - __clzll((long long)anys), 64);
    before += __shfl(up, 63, 64);
  }
  return total;
}

template <class Tok>
__global__ __launch_bounds__(64 * VD_W) void verify_kernel(const VerifyArgs a) {
  __shared__ double sums[2 * VD_W];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), K = a.K, V = a.V;
  const Tok* tokens = (const Tok*)a.tokens + (long)b * K;
  const float* u = a.uniforms + (long)b * (K + 1);
  const double u_draw = fmin(fmax((double)u[K], 0.0), 1.0);
  // the first draft that is not taken: every wave finds it for itself, 64 at a time; a place beyond the sequence's drafts is
  // looked at, too, so that its loads need not wait for their number
  const int count = a.counts ? clamped(a.counts[b], 0, K) : K;
  int acc = 0;
  for (int i0 = 0; i0 < K; i0 += 64) {
    const int i = i0 + lane;
    bool taken = false;
    if (i < K) {
      const float ui = u[i];
      const long x = (long)tokens[i];
      if (x >= 0 && x < V) {
        const double p = a.target[b * a.t_seq + i * a.t_row + x];
        const double q = a.draft ? a.draft[b * a.d_seq + i * a.d_row + x] : 1.f;
        taken = (double)ui * q < p;
      }
    }
    const unsigned long long no = ~__ballot(taken);
    const int run = no ? __ffsll((long long)no) - 1 : 64;
    acc = i0 + run;
    if (run < 64) break;
  }
  acc = uniform(min(acc, count));
  Weights w = {a.target + b * a.t_seq + acc * a.t_row, nullptr, -1};
  int token = -1;
  double total = 0.0;
  if (acc < count) {
    if (a.draft) {
      w.q = a.draft + b * a.d_seq + acc * a.d_row;
      total = draw<LESS_ROW>(w, V, u_draw, sums, token);
    } else {
      const long x = (long)tokens[acc];
      w.out = x >= 0 && x < V ? (int)x : -1;
      total = draw<LESS_TOKEN>(w, V, u_draw, sums, token);
    }
    __syncthreads();
  }
  if (!(total > 0.0)) draw<LESS_NOTHING>(w, V, u_draw, sums, token);  // all taken, or nothing left: the target's row itself
  if (wave == 0) {
    for (int i = lane; i <= K; i += 64) a.out[(long)b * (K + 1) + i] = i < acc ? (int)tokens[i] : i == acc ? token : -1;
    if (lane == 0) a.accepted[b] = acc;
  }
}

hipError_t launch_verify(const VerifyArgs& a, int token_bytes, int n_seqs, hipStream_t s) {
  if (!fits_a_launch(n_seqs, 64 * VD_W)) return hipErrorInvalidConfiguration;
  if (token_bytes == 8) hipLaunchKernelGGL(verify_kernel<long>, dim3(n_seqs), dim3(64 * VD_W), 0, s, a);
  else hipLaunchKernelGGL(verify_kernel<int>, dim3(n_seqs), dim3(64 * VD_W), 0, s, a);
  return hipGetLastError();
}

}  // namespace sna
