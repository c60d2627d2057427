// Attention of a step's new tokens over the paged cache, few rows of queries per key / value head.
//   out = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale q.k_j - m),   m near the running maximum (see Reference)
// All query heads of a key / value head (and a sequence's new tokens) are rows of one product, so that the cache is read once:
// its bytes bound these launches (32 heads over 8 of 128: one sequence of 131071 keys 97 us, 5.5 TB/s; 64 of up to 8192 195 us,
// 5.6 TB/s; 16 of up to 4096 with five tokens each 47 us, 3.6 TB/s; a plain read of gigabytes reaches 6.4).  A wave takes 64 keys
// at a time, straight from the pages into the operands of the matrix
// instruction: 16 rows of K (or of V^T, which is what the value pages hold) are 16 lanes, four lanes share a row's 32 columns.
// The next tile's keys are asked for when the scores are done, its values after the second product, and its pages a tile ahead
// of both, so that a wave has 16 to 32 KB under way without a ring in LDS.
// The scores are formed transposed (keys x rows): a lane then has one row of queries and the softmax statistics are its own
// but for two exchanges.  The keys of a product's 16 rows are chosen so (row 4 h + c of product a is key 8 h + 4 a + c of 32)
// that a lane's scores are the eight keys that the second product wants of it, without a trip through LDS.
#include <algorithm>
#include <climits>

#include "paged.h"

namespace sna {

// One wave's statistics of MB x 16 rows: row of queries 16 m + lane % 16, element of o[m][j][c]: dim 16 j + 4 (lane / 16) + c
template <class T, int D, int MB>
struct RowState {
  f32x4 o[MB][D / 16];
  Reference<T> ref[MB];            // of o and sum
  float sum[MB];                   // over this lane's keys
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      ref[m].clear();
      sum[m] = 0.f;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) o[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  __device__ __forceinline__ bool is_odd() const {                   // for some row of the wave: 0 x is 0 for a number, and only then
    float x = 0.f;
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int i = 0; i < D / 4; ++i) x = fmaf(o[m][i >> 2][i & 3], 0.f, x);
    return __any(x != 0.f);
  }
};
struct Span { int lo, hi; };       // keys lo .. hi - 1

// All ones for those of key .. key + 7 that lie in the span
__device__ __forceinline__ u32x4 slots_of(int key, Span keys) {
  u32x4 v;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int k = key + 2 * w;
    v[w] = (k >= keys.lo && k < keys.hi ? 0xffffu : 0u) | (k + 1 >= keys.lo && k + 1 < keys.hi ? 0xffff0000u : 0u);
  }
  return v;
}

// Queries are in registers, or in LDS where they would take those of a second block on the CU; every wave of a block has the same
constexpr bool queries_in_lds(int D, int MB) { return MB * D > 128; }
template <class T, int D, int MB>
struct Attend {
  static constexpr int S = D / 32, J = D / 16, KT = tile_keys(D, MB), U = KT / 32;
  // What rounding to the element type leaves of a probability goes through a second product, so that the result is off by its own
  // rounding alone (rounded once, the probabilities add as much again: 2.3e-3 of the norm in bf16, not 1.7e-3).  Up to 32 rows, single
  // and drafted tokens, the cache's bytes bound a launch, and this costs little: 16 sequences of up to 4096 keys with five tokens 46.5
  // us with and without, 64 of up to 2048 with eight and heads of 64 18.7 and 17.9.  Blocks of 64 rows are chunks, bound by their
  // products and exponentials (a mixed step 17.3 and 15.0 us), or groups of more than 32 heads, and round once.
  static constexpr bool PRECISE = MB <= 2;
  const PagedKV kv;
  const int* table;                // the sequence's
  int c_lo, c_hi, h, l16, hi;
  int ids[2 * U];                  // pages of the next tile: keys of each 32, value octets of each 32

  __device__ __forceinline__ int page(int key) const { return table[clamped(key >> kv.lps, c_lo, c_hi)]; }
  // where the page is used: a look at it any earlier would wait for the keys and values that were asked for before it, too
  __device__ __forceinline__ long in_pool(int id) const { return clamped(id, 0, kv.n_pages - 1); }
  __device__ __forceinline__ void find(int t) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      ids[u] = page(t * KT + 32 * u + 8 * (l16 >> 2));
      ids[U + u] = page(t * KT + 32 * u + 8 * hi);
    }
  }
  __device__ __forceinline__ void load_k(int t, const int (&id)[2 * U], u32x4 (&k)[U][2][S]) const {
    const int ps = 1 << kv.lps;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int slot = (t * KT + 32 * u + 8 * (l16 >> 2) + (l16 & 3)) & (ps - 1);
      const char* p = kv.k + in_pool(id[u]) * kv.kstride + ((long)h * ps + slot) * (2 * D) + hi * 16;
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int s = 0; s < S; ++s) k[u][a][s] = *(const u32x4*)(p + a * (8 * D) + s * 64);
    }
  }
  __device__ __forceinline__ void load_v(int t, const int (&id)[2 * U], u32x4 (&v)[U][J]) const {
    const int ps = 1 << kv.lps;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int slot = (t * KT + 32 * u + 8 * hi) & (ps - 1);
      const char* p = kv.v + in_pool(id[U + u]) * kv.vstride + (((long)h * D + l16) * ps + slot) * 2;
#pragma unroll
      for (int j = 0; j < J; ++j) v[u][j] = *(const u32x4*)(p + (long)j * 32 * ps);
    }
  }

  // What run() does, at leisure, for a wave whose sums came out as no numbers: in tiles whose rows differ in the keys they see, a
  // value that is none would have reached the rows that do not see its key, too.  Operation by operation the same, so that those
  // rows get what they would get without that value.
  __device__ __forceinline__ void run_carefully(int t0, int t1, int step, Span keys, Span clear, const int (&lim)[MB], const int (&low)[MB],
                                                const u32x4 (&q)[MB][S], const u32x4 (*q_lds)[64], float scale2, RowState<T, D, MB>& st) const {
    st.clear();
#pragma unroll 1
    for (int t = t0; t < t1; t += step) {
      int id[2 * U];
      const char* at[U];
      u32x4 ok[U], k[U][2][S];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int key = t * KT + 32 * u + 8 * hi;
        id[u] = page(t * KT + 32 * u + 8 * (l16 >> 2));
        at[u] = kv.v + in_pool(page(key)) * kv.vstride + ((((long)h * D + l16) << kv.lps) + (key & ((1 << kv.lps) - 1))) * 2;
        ok[u] = slots_of(key, keys);
      }
      load_k(t, id, k);
      const bool differ = t * KT < clear.lo || t * KT + KT > clear.hi;
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        f32x4 sc[U][2];
#pragma unroll
        for (int i = 0; i < 2 * U; ++i) sc[i >> 1][i & 1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < S; ++s) {
          const u32x4 x = queries_in_lds(D, MB) ? q_lds[m * S + s][hi * 16 + l16] : q[m][s];
#pragma unroll
          for (int i = 0; i < 2 * U; ++i) sc[i >> 1][i & 1] = T::mma16(k[i >> 1][i & 1][s], x, sc[i >> 1][i & 1]);
        }
        float x = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8 * U; ++i) {
          const int key = t * KT + 8 * hi + 32 * (i >> 3) + (i & 7);
          const float y = key <= lim[m] && key >= low[m] ? sc[i >> 3][(i >> 2) & 1][i & 3] : -INFINITY;
          sc[i >> 3][(i >> 2) & 1][i & 3] = y;
          x = fmaxf(x, y);
        }
        x = max_of_4(x) * scale2;
        const float keep = __any(st.ref[m].moves(x)) ? st.ref[m].move(x) : 1.f, ref = st.ref[m].from();
        st.sum[m] *= keep;
        u32x4 p[U], p_rest[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          f32x8 e;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            e[i] = __builtin_amdgcn_exp2f(fmaf(sc[u][i >> 2][i & 3], scale2, -ref));
            st.sum[m] += e[i];
          }
          p[u] = to_16<T>(e);
          if (PRECISE) p_rest[u] = to_16<T>(e - to_f32<T>(p[u]));
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
          u32x4 v[U];
          st.o[m][j] *= keep;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            v[u] = *(const u32x4*)(at[u] + ((long)j * 32 << kv.lps));
#pragma unroll
            for (int w = 0; w < 4; ++w) v[u][w] &= ok[u][w];
            const u32x4 x = differ ? without_odd<T>(v[u]) : v[u];
            st.o[m][j] = T::mma16(x, p[u], st.o[m][j]);
            if (PRECISE) st.o[m][j] = T::mma16(x, p_rest[u], st.o[m][j]);
          }
          if (differ)
#pragma unroll
            for (int kind = 0; kind < ODD_KINDS; ++kind) {
              f32x4 n = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int u = 0; u < U; ++u) n = T::mma16(ones_where_odd<T>(v[u], kind), ones_where_seen<T>(t * KT + 32 * u + 8 * hi, low[m], lim[m]), n);
#pragma unroll
              for (int c = 0; c < 4; ++c) st.o[m][j][c] += odd_sum(n[c] > 0.f, kind);
            }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }

  // Tiles t0, t0 + step, .. below t1.  lim / low: the last and first key that the lane's row of each m sees; all of them
  // see the keys from `clear.lo` to `clear.hi - 1`, none sees any outside `keys`.
  __device__ __forceinline__ void run(int t0, int t1, int step, Span keys, Span clear, const int (&lim)[MB], const int (&low)[MB],
                                      const u32x4 (&q)[MB][S], const u32x4 (*q_lds)[64], float scale2, RowState<T, D, MB>& st) {
    st.clear();
    if (t0 >= t1) return;
    u32x4 k[U][2][S], v[U][J];
    int now[2 * U];
    find(t0);
#pragma unroll
    for (int i = 0; i < 2 * U; ++i) now[i] = ids[i];
    load_k(t0, now, k);
    load_v(t0, now, v);
    find(t0 + step);
    for (int t = t0; t < t1; t += step) {
      const bool more = t + step < t1;
      u32x4 p[MB][U], p_rest[MB][U];
      int lane = hi * 16 + l16;
#if defined(__HIP_DEVICE_COMPILE__)
      if (queries_in_lds(D, MB)) asm volatile("" : "+v"(lane));        // read anew for each tile, not kept in registers
#endif
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        f32x4 sc[U][2];
#pragma unroll
        for (int i = 0; i < 2 * U; ++i) sc[i >> 1][i & 1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < S; ++s) {
          const u32x4 x = queries_in_lds(D, MB) ? q_lds[m * S + s][lane] : q[m][s];
#pragma unroll
          for (int i = 0; i < 2 * U; ++i) sc[i >> 1][i & 1] = T::mma16(k[i >> 1][i & 1][s], x, sc[i >> 1][i & 1]);
        }
        if (m == MB - 1 && more) {                                   // the next keys come in under the softmax and the second product
#pragma unroll
          for (int i = 0; i < 2 * U; ++i) now[i] = ids[i];
          load_k(t + step, now, k);
          find(t + 2 * step);
        }
        if (t * KT < clear.lo || t * KT + KT > clear.hi) {
#pragma unroll
          for (int i = 0; i < 8 * U; ++i) {
            const int key = t * KT + 8 * hi + 32 * (i >> 3) + (i & 7);
            sc[i >> 3][(i >> 2) & 1][i & 3] = key <= lim[m] && key >= low[m] ? sc[i >> 3][(i >> 2) & 1][i & 3] : -INFINITY;
          }
        }
        float x = sc[0][0][0];
#pragma unroll
        for (int i = 1; i < 8 * U; ++i) x = fmaxf(x, sc[i >> 3][(i >> 2) & 1][i & 3]);
        x = max_of_4(x) * scale2;
        if (__any(st.ref[m].moves(x))) {
          const float keep = st.ref[m].move(x);
          st.sum[m] *= keep;
#pragma unroll
          for (int j = 0; j < J; ++j) st.o[m][j] *= keep;
        }
        const float ref = st.ref[m].from();
#pragma unroll
        for (int u = 0; u < U; ++u) {
          f32x8 e;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            e[i] = __builtin_amdgcn_exp2f(fmaf(sc[u][i >> 2][i & 3], scale2, -ref));
            st.sum[m] += e[i];
          }
          p[m][u] = to_16<T>(e);
          if (PRECISE) p_rest[m][u] = to_16<T>(e - to_f32<T>(p[m][u]));
        }
      }
      if (t * KT < keys.lo || t * KT + KT > keys.hi) {               // slots that hold no key may hold anything: 0 * NaN is not 0
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const u32x4 ok = slots_of(t * KT + 32 * u + 8 * hi, keys);
#pragma unroll
          for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int j = 0; j < J; ++j) v[u][j][w] &= ok[w];
        }
      }
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int u = 0; u < U; ++u) {
            st.o[m][j] = T::mma16(v[u][j], p[m][u], st.o[m][j]);
            if (PRECISE) st.o[m][j] = T::mma16(v[u][j], p_rest[m][u], st.o[m][j]);
          }
      if (more) load_v(t + step, now, v);
    }
  }
};

// Where a block's rows are: tokens i0 .. i0 + n - 1 of a sequence, all heads of one key / value head
struct RowTile {
  int b, row0, n, pos0;            // first row, tokens, position of the first
  Span keys, clear;                // keys that some row sees, keys that all see
  int t0, tiles;                   // tiles of keys; at least one, so that rows without keys are written too
};
template <int KT>
__device__ __forceinline__ RowTile rows_of_sequence(const PagedAttnArgs& a, const Seq& sq, int b, int i0, int most) {
  RowTile r;
  r.b = b;
  r.n = i0 < 0 ? 0 : min(sq.n - i0, most);
  r.row0 = sq.row0 + i0;
  r.pos0 = sq.len - sq.n + i0;
  const int last = min(r.pos0 + r.n - 1, (a.s.width << a.kv.lps) - 1);
  r.keys = Span{max(a.window <= r.pos0 ? r.pos0 - a.window + 1 : 0, 0), last + 1};
  r.clear = Span{a.window <= last ? last - a.window + 1 : 0, r.pos0 + 1};
  r.t0 = r.keys.lo / KT;
  r.tiles = r.n > 0 ? max((max(r.keys.hi, 0) + KT - 1) / KT - r.t0, 1) : 0;
  return r;
}

template <int D, int MB, int W>
struct JoinLds {                   // of the W waves of a block: they take tiles of keys in turn
  __attribute__((aligned(16))) u32x4 q[queries_in_lds(D, MB) ? MB * (D / 32) : 1][64];
  __attribute__((aligned(16))) float o[W][16][D + 4];
  float top[W][MB][16], sum[W][MB][16];
};

// Keys of tiles t0 .. t1 - 1 for the rows of `r` and head h; the waves' parts are joined and leave as results, or as a part of
// them (part != nullptr): [rows_cap][D] sums, then [rows_cap][2] reference and sum.
template <class T, int D, int MB, int W, bool ONE>
__device__ __forceinline__ void attend_rows(const PagedAttnArgs& a, const RowTile& r, int h, int t0, int t1, float* part, int rows_cap, JoinLds<D, MB, W>& lds) {
  constexpr int S = D / 32, J = D / 16;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, hi = lane >> 4;
  const int rows = r.n * a.G;
  const unsigned inv = 65536u / a.G + 1;                             // row / G for row * G < 65536
  RowState<T, D, MB> st;
  {
    int lim[MB], low[MB];
    u32x4 q[MB][S];
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      const int row = min(16 * m + l16, rows - 1), i = (row * inv) >> 16;
      lim[m] = r.pos0 + i;
      low[m] = a.window <= lim[m] ? lim[m] - a.window + 1 : 0;
      const char* x = a.q + (r.row0 + i) * a.q_t + (h * a.G + row - i * a.G) * a.q_h + hi * 16;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        if (!queries_in_lds(D, MB)) q[m][s] = *(const u32x4*)(x + s * 64);
        else if ((m * S + s) % W == wave) lds.q[m * S + s][lane] = *(const u32x4*)(x + s * 64);
      }
    }
    if (queries_in_lds(D, MB)) __syncthreads();
    Attend<T, D, MB> at = {a.kv, a.s.table + (long)r.b * a.s.tstride, r.keys.lo >> a.kv.lps, max(r.keys.hi - 1, 0) >> a.kv.lps, h, l16, hi, {}};
    at.run(t0 + wave, t1, W, r.keys, r.clear, lim, low, q, lds.q, a.scale2, st);
    if (!ONE && __builtin_expect(r.n > 1 && st.is_odd(), 0)) at.run_carefully(t0 + wave, t1, W, r.keys, r.clear, lim, low, q, lds.q, a.scale2, st);
  }
  // o and sum relative to the largest reference of the waves
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    st.sum[m] = sum_of_4(st.sum[m]);
    if (hi == 0) { lds.top[wave][m][l16] = st.ref[m].at; lds.sum[wave][m][l16] = st.sum[m]; }
  }
  __syncthreads();
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    if (16 * m >= rows) break;
    float top = lds.top[0][m][l16];
#pragma unroll
    for (int w = 1; w < W; ++w) top = fmaxf(top, lds.top[w][m][l16]);
    const float keep = __builtin_amdgcn_exp2f(st.ref[m].at - (top == -INFINITY ? 0.f : top));
    if (m) __syncthreads();
#pragma unroll
    for (int j = 0; j < J; ++j) *(f32x4*)&lds.o[wave][l16][16 * j + 4 * hi] = st.o[m][j] * keep;
    __syncthreads();
    const int r16 = tid / (D / 8), oct = tid % (D / 8), row = 16 * m + r16;
    if (r16 < 16 && row < rows) {
      float t = lds.top[0][m][r16], sum = 0.f;
#pragma unroll
      for (int w = 1; w < W; ++w) t = fmaxf(t, lds.top[w][m][r16]);
      f32x8 x = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < W; ++w) {
        sum += lds.sum[w][m][r16] * __builtin_amdgcn_exp2f(lds.top[w][m][r16] - (t == -INFINITY ? 0.f : t));
        const f32x4 y0 = *(const f32x4*)&lds.o[w][r16][oct * 8], y1 = *(const f32x4*)&lds.o[w][r16][oct * 8 + 4];
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[e] += y0[e]; x[4 + e] += y1[e]; }
      }
      if (part) {
        *(f32x8*)(part + row * D + oct * 8) = x;
        if (oct == 0) { part[rows_cap * D + 2 * row] = t; part[rows_cap * D + 2 * row + 1] = sum; }
      } else {
        const int i = (row * inv) >> 16;
        const float f = sum == 0.f ? 0.f : 1.f / sum;                // a row that sees no key is zero
        *(u32x4*)(a.o + (r.row0 + i) * a.o_t + (h * a.G + row - i * a.G) * a.o_h + oct * 16) = to_16<T>(x * f);
      }
    }
  }
}

// A block for each tile of rows and key / value head.  ONE: no sequence brings more than one token, and the rows of a tile see the
// same keys
template <class T, int D, int MB, int W, bool ONE>
__global__ __launch_bounds__(64 * W, blocks_of(D, MB)) void paged_rows_kernel(const PagedAttnArgs a) {
  __shared__ JoinLds<D, MB, W> lds;
  const int tile = blockIdx.x;
  int b = tile, i0 = 0;
  if (a.max_new > a.tpt) {
    const auto tile0 = [&](int i) { return a.by_tpt.div(clamped(a.s.starts[i], 0, a.s.T)) + i; };
    b = last_at_most(a.s.B, tile, tile0);
    i0 = (tile - tile0(b)) * a.tpt;
  }
  const RowTile r = rows_of_sequence<tile_keys(D, MB)>(a, sequence(a.s, b), b, i0, a.tpt);
  if (r.n > 0) attend_rows<T, D, MB, W, ONE>(a, r, blockIdx.y, r.t0, r.t0 + r.tiles, nullptr, 0, lds);
}

// Tiles of keys of all tiles of a sequence's rows, for one head; none where the sequence has more rows than are taken here
template <int KT>
__device__ __forceinline__ int tiles_of_sequence(const PagedAttnArgs& a, int b) {
  const Seq sq = sequence(a.s, b);
  if (sq.n > a.most) return 0;
  int n = 0;
  for (int i0 = 0; i0 < sq.n; i0 += a.tpt) n += rows_of_sequence<KT>(a, sq, b, i0, a.tpt).tiles;
  return n;
}
// The keys of all tiles of rows and heads, laid end to end, in equal shares over the blocks: what a share cuts off of a
// (tile of rows, head) leaves as a part.  Part 2 p of block p continues what an earlier block began, part 2 p + 1 begins what
// a later one continues; whoever begins one writes down in first[p] what it was and which block ends it.
template <class T, int D, int MB, bool ONE>
__global__ __launch_bounds__(64 * kSplitW, blocks_of(D, MB)) void paged_split_kernel(const PagedAttnArgs a) {
  __shared__ JoinLds<D, MB, kSplitW> lds;
  constexpr int KT = tile_keys(D, MB);
  const int p = blockIdx.x, lane = threadIdx.x & 63, heads = a.kv.heads;
  First* first = (First*)a.parts;
  float* parts = (float*)(first + a.blocks);
  const long part_size = part_floats(a.rows_cap, D);
  // this share's first sequence: every wave sums the tiles of all, 64 runs of sequences at a time
  // (the host has seen to it that all of them fit 31 bits)
  int lo = 0, count = a.s.B, before = 0, share = 0, x = 0;
  for (bool top = true;; top = false) {
    const int per = (count + 63) >> 6, b0 = lo + lane * per, b1 = min(lo + count, b0 + per);
    int mine = 0;
    for (int b = b0; b < b1; ++b) mine += tiles_of_sequence<KT>(a, b);
    int up = mine;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      const int y = __shfl_up(up, m, 64);
      if (lane >= m) up += y;
    }
    if (top) {
      const int all = uniform(__shfl(up, 63, 64)) * heads;
      share = max((all + a.blocks - 1) / a.blocks, a.least);          // blocks: a power of two
      x = p * share;
      if (x >= all) {
        if (threadIdx.x == 0) first[p].n = 0;
        return;
      }
    }
    const int k = max(__ffsll((long long)__ballot((before + up) * heads > x)) - 1, 0);
    before += uniform(__shfl(up - mine, k, 64));
    lo = min(lo + k * per, a.s.B - 1);
    if (per == 1) break;
    count = clamped(count - k * per, 1, per);
  }
  // its first tile of rows, head and tile of keys
  int b = uniform(lo), i0 = 0;
  Seq sq = uniform(sequence(a.s, b));
  RowTile r = rows_of_sequence<KT>(a, sq, b, 0, a.tpt);
  int rel = x - before * heads;
  while (rel >= r.tiles * heads && i0 + a.tpt < sq.n) {
    rel -= r.tiles * heads;
    i0 += a.tpt;
    r = rows_of_sequence<KT>(a, sq, b, i0, a.tpt);
  }
  int h = clamped(rel / max(r.tiles, 1), 0, heads - 1), t = clamped(rel - h * r.tiles, 0, max(r.tiles - 1, 0)), left = share, at = 0;     // at: tiles done, of this share
  bool begun = false;
  while (true) {
    const int n = min(left, r.tiles - t);
    const bool whole = n == r.tiles;
    if (!whole && t == 0) {
      begun = true;
      if (threadIdx.x == 0) first[p] = First{r.row0, r.n, h, min((x + at + r.tiles - 1) / share, a.blocks - 1)};
    }
    if (r.n > 0) attend_rows<T, D, MB, kSplitW, ONE>(a, r, h, r.t0 + t, r.t0 + t + n, whole ? nullptr : parts + (2 * p + (t == 0)) * part_size, a.rows_cap, lds);
    left -= n;
    at += n;
    t = 0;
    if (left == 0) break;
    if (++h == heads) {
      h = 0;
      i0 += a.tpt;
      if (i0 >= sq.n) {
        i0 = 0;
        do {
          if (++b >= a.s.B) break;
          sq = uniform(sequence(a.s, b));
        } while (sq.n <= 0 || sq.n > a.most);
        if (b >= a.s.B) break;
      }
      r = rows_of_sequence<KT>(a, sq, b, i0, a.tpt);
    }
    __syncthreads();                                                 // the next part's joining
  }
  if (!begun && threadIdx.x == 0) first[p].n = 0;
}

// Parts joined: JN_Y blocks for each (tile of rows, head) that was cut.  A thread has four dims of a row; the 256 / (D / 4)
// groups of a row's threads take that many rows at a time where the parts are few, or share a row's parts where they are many.
// Sums, maximum and statistics of a part are asked for together: with the statistics first, a row of 64 parts took 5 us.
constexpr int JN_Y = 8;
template <class T, int D>
__global__ __launch_bounds__(256) void paged_join_kernel(const PagedAttnArgs a) {
  constexpr int W = D / 4, N = 256 / W, U = 8;                       // threads of a row; groups; parts under way
  __shared__ __attribute__((aligned(16))) float so[N][D];
  __shared__ float2 ss[N];
  const int p = blockIdx.x, g = threadIdx.x / W, d = threadIdx.x % W * 4;
  const First f = ((const First*)a.parts)[p];
  if (f.n == 0) return;
  const int n = f.last - p + 1, rows = f.n * a.G;
  int share = 1;                                                     // groups that share a row
  while (share < N && n > U * share) share *= 2;
  const int at_once = N / share;
  const long part_size = part_floats(a.rows_cap, D);
  const float* parts = (const float*)((const First*)a.parts + a.blocks) + (2 * p + 1) * part_size;       // part 0; part j > 0 lies 2 j - 1 further on
  for (int row0 = blockIdx.y * at_once; row0 < rows; row0 += gridDim.y * at_once) {       // the same turns for the block
    const int row = row0 + g / share, row_in = min(row, rows - 1);
    float top = -INFINITY, sum = 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = g % share; j0 < n; j0 += share * U) {
      f32x4 y[U];
      float2 st[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int j = min(j0 + u * share, n - 1);
        const float* q = parts + max(2 * j - 1, 0) * part_size;
        y[u] = *(const f32x4*)(q + row_in * D + d);
        st[u] = *(const float2*)(q + a.rows_cap * D + 2 * row_in);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (j0 + u * share < n) {
          const float now = fmaxf(top, st[u].x), ref = now == -INFINITY ? 0.f : now;
          const float keep = __builtin_amdgcn_exp2f(top - ref), w = __builtin_amdgcn_exp2f(st[u].x - ref);
          x = x * keep + y[u] * w;
          sum = sum * keep + st[u].y * w;
          top = now;
        }
    }
    if (share > 1) {                                                 // the same for the block
      __syncthreads();
      *(f32x4*)&so[g][d] = x;
      if (d == 0) ss[g] = make_float2(top, sum);
      __syncthreads();
      if (g % share) continue;
      for (int i = 1; i < share; ++i) {
        const float2 st = ss[g + i];
        const float now = fmaxf(top, st.x), ref = now == -INFINITY ? 0.f : now;
        const float keep = __builtin_amdgcn_exp2f(top - ref), w = __builtin_amdgcn_exp2f(st.x - ref);
        x = x * keep + *(const f32x4*)&so[g + i][d] * w;
        sum = sum * keep + st.y * w;
        top = now;
      }
    }
    if (row >= rows) continue;
    x *= sum == 0.f ? 0.f : 1.f / sum;
    const int i = row / a.G;
    *(uint2*)(a.o + (f.row0 + i) * a.o_t + (f.h * a.G + row - i * a.G) * a.o_h + d * 2) = __builtin_bit_cast(uint2, __builtin_convertvector(x, typename T::v4));
  }
}

constexpr int kSplitLeast = 4;     // tiles of a share: one for each wave

template <class T, int D, int MB, bool ONE>
static hipError_t rows_grid(PagedAttnArgs a, hipStream_t s) {
  a.tpt = 16 * MB / a.G;
  if (a.parts) {
    if (a.tpt > a.max_new) a.tpt = a.max_new;                        // of rows_cap rows
    a.rows_cap = a.tpt * a.G;
    a.least = kSplitLeast;
    hipLaunchKernelGGL((paged_split_kernel<T, D, MB, ONE>), dim3(a.blocks), dim3(64 * kSplitW), 0, s, a);
    hipLaunchKernelGGL((paged_join_kernel<T, D>), dim3(a.blocks, std::min(a.rows_cap, JN_Y)), dim3(256), 0, s, a);
    return hipGetLastError();
  }
  a.by_tpt = FastDiv::by(a.tpt);
  const int tiles = a.max_new > a.tpt ? a.s.T / a.tpt + a.s.B : a.s.B;
  const dim3 grid(tiles, a.kv.heads);
  if (!fits_a_launch(tiles, a.waves * 64)) return hipErrorInvalidConfiguration;
  if constexpr (blocks_of(D, MB) == 2)
    if (a.waves == 8) {
      hipLaunchKernelGGL((paged_rows_kernel<T, D, MB, 8, ONE>), grid, dim3(512), 0, s, a);
      return hipGetLastError();
    }
  hipLaunchKernelGGL((paged_rows_kernel<T, D, MB, 4, ONE>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}
template <class T, int D>
static hipError_t rows_of(const PagedAttnArgs& a, int mb, hipStream_t s) {
  if (mb == 1 && a.max_new == 1) return rows_grid<T, D, 1, true>(a, s);
  if (mb == 1) return rows_grid<T, D, 1, false>(a, s);
  return mb == 2 ? rows_grid<T, D, 2, false>(a, s) : rows_grid<T, D, 4, false>(a, s);
}

size_t paged_attention_workspace(int n_seqs, int n_tokens, int kv_heads, int group, int max_new, int max_len, int window, int head_dim) {
  const AttnPlan p = plan_of(n_seqs, n_tokens, kv_heads, group, max_new, max_len, window, head_dim);
  return p.parts + p.chunk_parts;
}

hipError_t launch_paged_attention(PagedAttnArgs a, int dtype, int head_dim, int max_len, void* workspace, hipStream_t s) {
  const AttnPlan p = plan_of(a.s.B, a.s.T, a.kv.heads, a.G, a.max_new, max_len, a.window == INT_MAX ? 0 : a.window, head_dim);
  a.most = p.most;
  a.waves = p.chunk.waves;
  a.splits = p.chunk.splits;
  if (p.chunks && !chunks_fit_a_launch(a)) return hipErrorInvalidConfiguration;        // before anything is launched
  if (p.mb) {
    PagedAttnArgs r = a;
    r.parts = p.blocks ? workspace : nullptr;
    r.blocks = p.blocks;
    r.waves = p.waves;
    hipError_t e;
    if (dtype == SNA_DTYPE_FP16) e = head_dim == 64 ? rows_of<Fp16, 64>(r, p.mb, s) : rows_of<Fp16, 128>(r, p.mb, s);
    else e = head_dim == 64 ? rows_of<Bf16, 64>(r, p.mb, s) : rows_of<Bf16, 128>(r, p.mb, s);
    if (e != hipSuccess || !p.chunks) return e;
  }
  a.parts = (char*)workspace + p.parts;
  return launch_paged_chunks(a, dtype, head_dim, s);
}

}  // namespace sna
