// Attention of a step's new tokens over the paged cache, few rows of queries per key / value head.
//   out = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale q.k_j - m),   m the running maximum
// All query heads of a key / value head (and a sequence's new tokens) are rows of one product, so that the cache is read once:
// its bytes bound these launches.  A wave takes 64 keys at a time, straight from the pages into the operands of the matrix
// instruction: 16 rows of K (or of V^T, which is what the value pages hold) are 16 lanes, four lanes share a row's 32 columns.
// The scores are formed transposed (keys x rows): a lane then has one row of queries and the softmax statistics are its own
// but for two exchanges.  The keys of a product's 16 rows are chosen so (row 4 h + c of product a is key 8 h + 4 a + c of 32)
// that a lane's scores are the eight keys that the second product wants of it, without a trip through LDS.
#include "paged.h"

namespace sna {

constexpr int PA_W = 4;            // waves of a block: they take tiles of keys in turn and are joined in LDS
constexpr int PA_K = 64;           // keys of a tile

// One wave's statistics of MB x 16 rows: row of queries 16 m + lane % 16, element of o[m][j][c]: dim 16 j + 4 (lane / 16) + c
template <int D, int MB>
struct RowState {
  f32x4 o[MB][D / 16];
  float top[MB], sum[MB];          // maximum that o and sum are relative to (base 2); sum over this lane's keys
};
struct Span { int lo, hi; };       // keys lo .. hi - 1

template <class T, int D, int MB>
struct Attend {
  static constexpr int S = D / 32, J = D / 16;
  const PagedKV kv;
  const int* table;                // the sequence's
  int c_lo, c_hi, h, l16, hi;
  int ids[4];                      // pages of the next tile: keys of both halves (K), value octets of both halves

  __device__ __forceinline__ int page(int key) const {
    const int id = table[clamped(key >> kv.lps, c_lo, c_hi)];
    return clamped(id, 0, kv.n_pages - 1);
  }
  __device__ __forceinline__ void find(int t) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      ids[u] = page(t * PA_K + 32 * u + 8 * (l16 >> 2));
      ids[2 + u] = page(t * PA_K + 32 * u + 8 * hi);
    }
  }
  __device__ __forceinline__ void load_k(int t, const int (&id)[4], u32x4 (&k)[2][2][S]) const {
    const int ps = 1 << kv.lps;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int slot = (t * PA_K + 32 * u + 8 * (l16 >> 2) + (l16 & 3)) & (ps - 1);
      const char* p = kv.k + id[u] * kv.kstride + ((long)h * ps + slot) * (2 * D) + hi * 16;
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int s = 0; s < S; ++s) k[u][a][s] = *(const u32x4*)(p + a * (8 * D) + s * 64);
    }
  }
  __device__ __forceinline__ void load_v(int t, const int (&id)[4], u32x4 (&v)[2][J]) const {
    const int ps = 1 << kv.lps;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int slot = (t * PA_K + 32 * u + 8 * hi) & (ps - 1);
      const char* p = kv.v + id[2 + u] * kv.vstride + (((long)h * D + l16) * ps + slot) * 2;
#pragma unroll
      for (int j = 0; j < J; ++j) v[u][j] = *(const u32x4*)(p + (long)j * 32 * ps);
    }
  }

  // Tiles t0, t0 + step, .. below t1.  lim / low: the last and first key that the lane's row of each m sees; all of them
  // see the keys from `clear.lo` to `clear.hi - 1`, none sees any outside `keys`.
  __device__ __forceinline__ void run(int t0, int t1, int step, Span keys, Span clear, const int (&lim)[MB], const int (&low)[MB],
                                      const u32x4 (&q)[MB][S], float scale2, RowState<D, MB>& st) {
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      st.top[m] = -INFINITY;
      st.sum[m] = 0.f;
#pragma unroll
      for (int j = 0; j < J; ++j) st.o[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (t0 >= t1) return;
    u32x4 k[2][2][S], v[2][J];
    int now[4];
    find(t0);
#pragma unroll
    for (int i = 0; i < 4; ++i) now[i] = ids[i];
    load_k(t0, now, k);
    load_v(t0, now, v);
    find(t0 + step);
    for (int t = t0; t < t1; t += step) {
      f32x4 sc[MB][2][2];
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int a = 0; a < 2; ++a) {
            sc[m][u][a] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < S; ++s) sc[m][u][a] = T::mma16(k[u][a][s], q[m][s], sc[m][u][a]);
          }
      const bool more = t + step < t1;
      if (more) {
#pragma unroll
        for (int i = 0; i < 4; ++i) now[i] = ids[i];
        load_k(t + step, now, k);
        find(t + 2 * step);
      }
      u32x4 p[MB][2];
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        const int key0 = t * PA_K + 8 * hi;
        if (t * PA_K < clear.lo || t * PA_K + PA_K > clear.hi) {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                const int key = key0 + 32 * u + 4 * a + c;
                sc[m][u][a][c] = key <= lim[m] && key >= low[m] ? sc[m][u][a][c] * scale2 : -INFINITY;
              }
        } else {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
              for (int c = 0; c < 4; ++c) sc[m][u][a][c] *= scale2;
        }
        float x = sc[m][0][0][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) x = fmaxf(x, sc[m][i >> 3][(i >> 2) & 1][i & 3]);
        const float top = fmaxf(st.top[m], max_of_4(x));
        const float ref = top == -INFINITY ? 0.f : top;              // nothing seen so far
        const float keep = __builtin_amdgcn_exp2f(st.top[m] - ref);
        st.top[m] = top;
        st.sum[m] *= keep;
#pragma unroll
        for (int j = 0; j < J; ++j) st.o[m][j] *= keep;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          f32x8 e;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            e[i] = __builtin_amdgcn_exp2f(sc[m][u][i >> 2][i & 3] - ref);
            st.sum[m] += e[i];
          }
          p[m][u] = to_16<T>(e);                                     // the operand type: p is at most 1, off by half a step of it
        }
      }
      if (t * PA_K < keys.lo || t * PA_K + PA_K > keys.hi) {         // slots that hold no key may hold anything: 0 * NaN is not 0
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int key0 = t * PA_K + 32 * u + 8 * hi;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const int key = key0 + 2 * w;
            const unsigned ok = (key >= keys.lo && key < keys.hi ? 0xffffu : 0u) | (key + 1 >= keys.lo && key + 1 < keys.hi ? 0xffff0000u : 0u);
#pragma unroll
            for (int j = 0; j < J; ++j) v[u][j][w] &= ok;
          }
        }
      }
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int u = 0; u < 2; ++u) st.o[m][j] = T::mma16(v[u][j], p[m][u], st.o[m][j]);
      if (more) load_v(t + step, now, v);
    }
  }
};

template <class T, int D, int MB>
__global__ __launch_bounds__(64 * PA_W) void paged_rows_kernel(const PagedAttnArgs a) {
  constexpr int S = D / 32, J = D / 16, LD = D + 4;
  __shared__ __attribute__((aligned(16))) float so[PA_W][16][LD];
  __shared__ float sm[PA_W][MB][16], sl[PA_W][MB][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, hi = lane >> 4;
  const int h = blockIdx.y, tile = blockIdx.x;
  int b = tile, i0 = 0;
  if (a.max_new > a.tpt) {
    const auto tile0 = [&](int i) { return a.by_tpt.div(clamped(a.s.starts[i], 0, a.s.T)) + i; };
    b = last_at_most(a.s.B, tile, tile0);
    i0 = (tile - tile0(b)) * a.tpt;
  }
  const Seq sq = sequence(a.s, b);
  const int n = min(sq.n - i0, a.tpt);                               // tokens of this tile
  if (n <= 0 || i0 < 0) return;
  const int row0 = sq.row0 + i0, pos0 = sq.len - sq.n + i0, rows = n * a.G;
  const unsigned inv = 65536u / a.G + 1;                             // r / G for r * G < 65536
  int lim[MB], low[MB];
  u32x4 q[MB][S];
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    const int r = min(16 * m + l16, rows - 1), i = (r * inv) >> 16;
    lim[m] = pos0 + i;
    low[m] = a.window <= lim[m] ? lim[m] - a.window + 1 : 0;
    const char* x = a.q + (row0 + i) * a.q_t + (h * a.G + r - i * a.G) * a.q_h + hi * 16;
#pragma unroll
    for (int s = 0; s < S; ++s) q[m][s] = *(const u32x4*)(x + s * 64);
  }
  const int last = min(pos0 + n - 1, (a.s.width << a.kv.lps) - 1);   // of the keys that some row sees
  const Span keys = {max(a.window <= pos0 ? pos0 - a.window + 1 : 0, 0), last + 1};
  const Span clear = {a.window <= last ? last - a.window + 1 : 0, pos0 + 1};
  RowState<D, MB> st;
  Attend<T, D, MB> at = {a.kv, a.s.table + (long)b * a.s.tstride, keys.lo >> a.kv.lps, max(last, 0) >> a.kv.lps, h, l16, hi, {}};
  at.run(keys.lo / PA_K + wave, (keys.hi + PA_K - 1) / PA_K, PA_W, keys, clear, lim, low, q, a.scale2, st);

  // join the waves: o and sum relative to the largest maximum
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    st.sum[m] = sum_of_4(st.sum[m]);
    if (hi == 0) { sm[wave][m][l16] = st.top[m]; sl[wave][m][l16] = st.sum[m]; }
  }
  __syncthreads();
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    if (16 * m >= rows) break;
    float top = sm[0][m][l16];
#pragma unroll
    for (int w = 1; w < PA_W; ++w) top = fmaxf(top, sm[w][m][l16]);
    const float keep = st.top[m] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.top[m] - top);
    if (m) __syncthreads();
#pragma unroll
    for (int j = 0; j < J; ++j) *(f32x4*)&so[wave][l16][16 * j + 4 * hi] = st.o[m][j] * keep;
    __syncthreads();
    const int r16 = tid / (D / 8), oct = tid % (D / 8), r = 16 * m + r16;
    if (r16 < 16 && r < rows) {
      float t = sm[0][m][r16], sum = 0.f;
#pragma unroll
      for (int w = 1; w < PA_W; ++w) t = fmaxf(t, sm[w][m][r16]);
      f32x8 x = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < PA_W; ++w) {
        const float tw = sm[w][m][r16];
        sum += tw == -INFINITY ? 0.f : sl[w][m][r16] * __builtin_amdgcn_exp2f(tw - t);
        const f32x4 y0 = *(const f32x4*)&so[w][r16][oct * 8], y1 = *(const f32x4*)&so[w][r16][oct * 8 + 4];
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[e] += y0[e]; x[4 + e] += y1[e]; }
      }
      const float f = sum == 0.f ? 0.f : 1.f / sum;                  // a row that sees no key is zero
      const int i = (r * inv) >> 16;
      *(u32x4*)(a.o + (row0 + i) * a.o_t + (h * a.G + r - i * a.G) * a.o_h + oct * 16) = to_16<T>(x * f);
    }
  }
}

template <class T, int D, int MB>
static void rows_grid(PagedAttnArgs a, hipStream_t s) {
  a.tpt = 16 * MB / a.G;
  a.by_tpt = FastDiv::by(a.tpt);
  const int tiles = a.max_new > a.tpt ? a.s.T / a.tpt + a.s.B : a.s.B;
  hipLaunchKernelGGL((paged_rows_kernel<T, D, MB>), dim3(tiles, a.kv.heads), dim3(64 * PA_W), 0, s, a);
}
template <class T, int D>
static void rows_of(const PagedAttnArgs& a, hipStream_t s) {
  const long rows = (long)a.max_new * a.G;
  if (rows <= 16) rows_grid<T, D, 1>(a, s);
  else if (rows <= 32) rows_grid<T, D, 2>(a, s);
  else rows_grid<T, D, 4>(a, s);
}

hipError_t launch_paged_attention(const PagedAttnArgs& a, int dtype, int head_dim, hipStream_t s) {
  if (dtype == SNA_DTYPE_FP16) head_dim == 64 ? rows_of<Fp16, 64>(a, s) : rows_of<Fp16, 128>(a, s);
  else head_dim == 64 ? rows_of<Bf16, 64>(a, s) : rows_of<Bf16, 128>(a, s);
  return hipGetLastError();
}

}  // namespace sna
