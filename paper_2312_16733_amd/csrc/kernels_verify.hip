// Verification of drafted tokens against the target's probabilities, from given random numbers.
//   drafted token i is taken while u_i q_i(x_i) < p_i(x_i) (and all before it are);  at the first that is not, a:
//   the next token is drawn from w = max(p_a - q_a, 0), or from p_a where nothing is left of it or all drafts are taken:
//   the smallest x with w_0 + .. + w_x > u_K (w_0 + .. + w_{V - 1})
// Products, differences, sums and the comparison are in 64 bits: u q is exact, and 10^5 probabilities summed in 32 bits would
// move the borders between tokens by more than many of them are worth.
// Bound by memory: two rows of the vocabulary a sequence, read once.  A block has a sequence; each of its waves sums a run of
// the row, then the run that holds the draw (V / 16 values, cached by now) is shared out over the waves, and the run of that
// over the lanes of one.
#include "paged.h"

namespace sna {

constexpr int VD_W = 16;           // waves of a block

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

struct Weights {                   // of one sequence's draw
  const float* p; const float* q;  // q: nullptr where the draft's token alone is taken out, or nothing
  int out;                         // that token, or -1
  __device__ __forceinline__ double of(int x, float px, float qx) const {
    double w = q ? (double)px - (double)qx : (double)px;
    if (x == out) w = 0.0;
    return w > 0.0 ? w : 0.0;                                        // NaN counts as nothing
  }
};
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4u;  // rows of odd vocabularies start anywhere

// Sum over [x0, x1) by one wave
__device__ __forceinline__ double run_sum(const Weights& w, int x0, int x1) {
  const int lane = threadIdx.x & 63;
  double s = 0.0;
  int x = x0 + 4 * lane;
  for (; x + 3 < x1; x += 256) {
    const f32x4u p = *(const f32x4u*)(w.p + x), q = w.q ? *(const f32x4u*)(w.q + x) : f32x4u{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e) s += w.of(x + e, p[e], q[e]);
  }
  for (; x < x1; ++x) s += w.of(x, w.p[x], w.q ? w.q[x] : 0.f);       // one lane's, up to three
  return wave_sum(s);
}

template <class Tok>
__global__ __launch_bounds__(64 * VD_W) void verify_kernel(const VerifyArgs a) {
  __shared__ double sums[VD_W];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), K = a.K, V = a.V;
  const Tok* tokens = (const Tok*)a.tokens + (long)b * K;
  const float* u = a.uniforms + (long)b * (K + 1);
  const int count = a.counts ? clamped(a.counts[b], 0, K) : K;
  // the first draft that is not taken: every wave finds it for itself, 64 at a time
  int acc = 0;
  for (int i0 = 0; i0 < count; i0 += 64) {
    const int i = i0 + lane;
    bool taken = false;
    if (i < count) {
      const long x = (long)tokens[i];
      if (x >= 0 && x < V) {
        const double p = a.target[b * a.t_seq + i * a.t_row + x];
        const double q = a.draft ? a.draft[b * a.d_seq + i * a.d_row + x] : 1.f;
        taken = (double)u[i] * q < p;
      }
    }
    const unsigned long long no = ~__ballot(taken);
    const int run = no ? __ffsll((long long)no) - 1 : 64;
    acc = i0 + run;
    if (run < 64) break;
  }
  acc = __builtin_amdgcn_readfirstlane(min(acc, count));
  Weights w = {a.target + b * a.t_seq + acc * a.t_row, nullptr, -1};
  if (acc < count) {
    if (a.draft) w.q = a.draft + b * a.d_seq + acc * a.d_row;
    else {
      const long x = (long)tokens[acc];
      w.out = x >= 0 && x < V ? (int)x : -1;
    }
  }
  double total = 0.0, before = 0.0, run0[VD_W];
  const int len1 = (((V + VD_W - 1) / VD_W) + 3) & ~3;               // values of a wave's run
  for (int turn = 0; turn < 2; ++turn) {
    const int x0 = min(V, wave * len1), x1 = min(V, x0 + len1);
    const double s = run_sum(w, x0, x1);
    if (turn) __syncthreads();
    if (lane == 0) sums[wave] = s;
    __syncthreads();
    total = 0.0;
#pragma unroll
    for (int i = 0; i < VD_W; ++i) {
      run0[i] = sums[i];
      total += run0[i];
    }
    if (total > 0.0 || (!w.q && w.out < 0)) break;
    w.q = nullptr;                                                   // nothing left of the difference: the target's row itself
    w.out = -1;
  }
  int token = -1;
  if (total > 0.0) {
    const double at = fmin(fmax((double)u[K], 0.0), 1.0) * total;
    // the first run whose end lies beyond the draw; the last with any weight where rounding leaves none
    int r1 = 0;
    bool found = false;
    double up = 0.0;
#pragma unroll
    for (int i = 0; i < VD_W; ++i) {
      if (!found && run0[i] > 0.0) { r1 = i; before = up; }
      up += run0[i];
      found = found || up > at;
    }
    const int s0 = min(V, r1 * len1), s1 = min(V, s0 + len1), len2 = (((s1 - s0 + VD_W - 1) / VD_W) + 3) & ~3;
    const int x0 = min(s1, s0 + wave * len2), x1 = min(s1, x0 + len2);
    const double s = run_sum(w, x0, x1);
    __syncthreads();
    if (lane == 0) sums[wave] = s;
    __syncthreads();
    if (wave == 0) {
      int r2 = 0;
      found = false;
      up = before;
#pragma unroll
      for (int i = 0; i < VD_W; ++i) {
        const double v = sums[i];
        if (!found && v > 0.0) { r2 = i; before = up; }
        up += v;
        found = found || up > at;
      }
      // that run: a stretch of it a lane
      const int y0 = min(s1, s0 + r2 * len2), y1 = min(s1, y0 + len2), len3 = (y1 - y0 + 63) / 64;
      const int z0 = min(y1, y0 + lane * len3), z1 = min(y1, z0 + len3);
      double mine = 0.0;
      for (int x = z0; x < z1; ++x) mine += w.of(x, w.p[x], w.q ? w.q[x] : 0.f);
      double c = before + wave_scan(mine) - mine;
      int hit = -1, any = -1;
      for (int x = z0; x < z1; ++x) {
        const double v = w.of(x, w.p[x], w.q ? w.q[x] : 0.f);
        c += v;
        if (v > 0.0) {
          any = x;
          if (hit < 0 && c > at) hit = x;
        }
      }
      const unsigned long long hits = __ballot(hit >= 0), anys = __ballot(any >= 0);
      if (hits) token = __shfl(hit, __ffsll((long long)hits) - 1, 64);
      else if (anys) token = __shfl(any, 63 - __clzll((long long)anys), 64);
    }
  }
  if (wave == 0) {
    for (int i = lane; i <= K; i += 64) a.out[(long)b * (K + 1) + i] = i < acc ? (int)tokens[i] : i == acc ? token : -1;
    if (lane == 0) a.accepted[b] = acc;
  }
}

hipError_t launch_verify(const VerifyArgs& a, int token_bytes, int n_seqs, hipStream_t s) {
  if (token_bytes == 8) hipLaunchKernelGGL(verify_kernel<long>, dim3(n_seqs), dim3(64 * VD_W), 0, s, a);
  else hipLaunchKernelGGL(verify_kernel<int>, dim3(n_seqs), dim3(64 * VD_W), 0, s, a);
  return hipGetLastError();
}

}  // namespace sna
