// Attention of a step's new tokens over the paged cache, many rows of queries per key / value head (chunks of prompts).
// Bound by the matrix pipe and, nearly as much, by the vector pipe's exponentials.  A block holds 32 rows a wave (tokens times
// the query heads of one key / value head) and walks its keys in tiles of 64, fetched from the pages straight into LDS, one
// tile ahead (4096 tokens over 8192 keys, 32 heads over 8 of 128: 386 to 402 us by card, 1.02 to 1.07 PFLOP/s, once the chip has
// settled, 26 ms into a burst, and up to 534 before; the library's plain bf16 product of 8192^3 reaches 1.20; the matrix pipe is at work
// 49 % of the cycles, the vector pipe 48 %).  A page id is looked at a tile after it was asked for: looked at once it waited for the tile's fetches, too (523 us).
// Forming the next tile's scores among this one's exponentials was worth under 1 % (393 us), forced interleaving of products,
// reads and vector instructions cost 2 %, four waves a block instead of eight 4 %.  As where rows are few, the scores are formed transposed: a lane has one row, and the keys of a product's 32
// rows are chosen so (row 16 s + 8 a + 4 h + c is key 16 s + 8 h + 4 a + c) that its scores are what the second product wants.
#include "paged.h"

namespace sna {

typedef __attribute__((address_space(3))) char lds_char;

template <int D>
struct PrefillLds {                // two tiles
  char k[2][PF_K * D * 2];         // [key][octet]
  char v[2][D * PF_K * 2];         // [dim][octet of keys]
};
// Octet o of a row lies at place o ^ swizzle(row): eight (and sixteen) lanes that read one octet of the rows of a product
// then touch different banks.
template <int D>
__device__ __forceinline__ int k_swizzle(int key) {
  const int low = (key & 3) | ((key >> 3) & 1) << 2, a = (key >> 2) & 1;
  return D == 128 ? low | a << 3 : low ^ a;
}
__device__ __forceinline__ int v_swizzle(int d) { return (d ^ (d >> 3)) & 7; }

__device__ __forceinline__ void fetch16(const char* from, lds_char* to) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) unsigned*)from, (__attribute__((address_space(3))) unsigned*)to, 16, 0, 0);
#endif
}

template <class T, int D, int W>
__global__ __launch_bounds__(64 * W, 2) void paged_chunk_kernel(const PagedAttnArgs a) {
  constexpr int S = D / 16, J = D / 32, KI = PF_K * D * 2 / 1024 / W, VI = KI;   // fetches of a wave and tile, 1 KB each
  __shared__ __attribute__((aligned(1024))) PrefillLds<D> lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hi = lane >> 5;
  // heads change fastest: where there are 8 of them, each XCD reads one and keeps it in its L2; the last tiles of rows, which
  // see the most keys, first
  const int h = blockIdx.x % a.kv.heads, rest = blockIdx.x / a.kv.heads, part = rest % a.splits, tile = gridDim.x / (a.kv.heads * a.splits) - 1 - rest / a.splits;
  const auto tile0 = [&](int i) { return a.by_tpt.div(clamped(a.s.starts[i], 0, a.s.T)) + i; };
  const int b = last_at_most(a.s.B, tile, tile0);
  const Seq sq = sequence(a.s, b);
  const int i0 = (tile - tile0(b)) * a.tpt, n = i0 < 0 ? 0 : min(sq.n - i0, a.tpt);
  if (n <= 0 || sq.n <= a.most) return;                              // few rows: not taken here
  const int row0 = sq.row0 + i0, pos0 = sq.len - sq.n + i0, rows = n * a.G;
  const int last = min(pos0 + n - 1, (a.s.width << a.kv.lps) - 1);
  const int first = max(a.window <= pos0 ? pos0 - a.window + 1 : 0, 0);
  int t0 = first / PF_K, t1 = last < 0 ? t0 : last / PF_K + 1;
  if (a.splits > 1) {                                                // this block's share of the keys
    const int per = (t1 - t0 + a.splits - 1) / a.splits;
    t0 = min(t0 + part * per, t1);
    t1 = min(t0 + per, t1);
  }
  const int* table = a.s.table + (long)b * a.s.tstride;
  const int c_lo = first >> a.kv.lps, c_hi = max(last, 0) >> a.kv.lps, ps = 1 << a.kv.lps;
  const auto page = [&](int key) { return table[clamped(key >> a.kv.lps, c_lo, c_hi)]; };
  const auto in_pool = [&](int id) { return clamped(id, 0, a.kv.n_pages - 1); };   // where the page is used: a look at it any earlier would wait for the fetches, too

  // this lane's row of queries
  const unsigned inv = 65536u / a.G + 1;
  const int row = min(32 * wave + l32, rows - 1), tok = (row * inv) >> 16;
  const bool mine = 32 * wave + l32 < rows;
  const int lim = pos0 + tok, low = a.window <= lim ? lim - a.window + 1 : 0;
  const long qi = (long)(row0 + tok), qh = h * a.G + row - tok * a.G;
  u32x4 q[S];
#pragma unroll
  for (int s = 0; s < S; ++s) q[s] = *(const u32x4*)(a.q + qi * a.q_t + qh * a.q_h + s * 32 + hi * 16);
  // of the wave's rows: the last and first key that some of them sees, the last and first that all see
  const int w_tok0 = (min(32 * wave, rows - 1) * inv) >> 16, w_tok1 = (min(32 * wave + 31, rows - 1) * inv) >> 16;
  const int w_last = 32 * wave < rows ? pos0 + w_tok1 : -1, w_all = pos0 + w_tok0;
  const int w_low = a.window <= w_all ? w_all - a.window + 1 : 0, w_first = a.window <= pos0 + w_tok1 ? pos0 + w_tok1 - a.window + 1 : 0;

  // fetches: K tile rows of 16 D / 8 bytes, 1 KB an instruction; V tile rows of 128 bytes
  constexpr int KR = 1024 / (D * 2);                                 // keys of a fetch
  const int k_row = lane / (D / 8), k_pos = lane % (D / 8), v_row = lane >> 3, v_pos = lane & 7;
  int kid, vid[VI > 1 && W < 8 ? 2 : 1];
  const auto find = [&](int t) {
    kid = page(t * PF_K + KI * KR * wave);                           // KI * KR keys of a wave: within 16 aligned ones
#pragma unroll
    for (int i = 0; i < (VI > 1 && W < 8 ? 2 : 1); ++i) vid[i] = page(t * PF_K + 8 * (v_pos ^ v_row ^ ((wave + W * i) & 7)));
  };
  int k_off[KI];                                                     // within the tile's keys, and of their octets
#pragma unroll
  for (int i = 0; i < KI; ++i) {
    const int r = (wave * KI + i) * KR + k_row;
    k_off[i] = (r & (ps - 1)) * (D * 2) + (k_pos ^ k_swizzle<D>(r)) * 16;
  }
  const auto fetch = [&](int t, int buf) {
    const int slot = (t * PF_K) & (ps - 1);
    const char* kp = a.kv.k + in_pool(__builtin_amdgcn_readfirstlane(kid)) * a.kv.kstride + ((long)h * ps + slot) * (D * 2);
#pragma unroll
    for (int i = 0; i < KI; ++i) fetch16(kp + k_off[i], (lds_char*)lds.k[buf] + (wave * KI + i) * 1024);
    const char* vp[VI > 1 && W < 8 ? 2 : 1];
#pragma unroll
    for (int i = 0; i < (VI > 1 && W < 8 ? 2 : 1); ++i)
      vp[i] = a.kv.v + in_pool(vid[i]) * a.kv.vstride + (((long)h * D + (wave + W * i) * 8 + v_row) * ps + ((t * PF_K + 8 * (v_pos ^ v_row ^ ((wave + W * i) & 7))) & (ps - 1))) * 2;
#pragma unroll
    for (int i = 0; i < VI; ++i) {
      if (W == 8) fetch16(vp[0] + i * (W * 16) * ps, (lds_char*)lds.v[buf] + (wave + W * i) * 1024);
      else fetch16(vp[i & 1] + (i >> 1) * (2 * W * 16) * ps, (lds_char*)lds.v[buf] + (wave + W * i) * 1024);
    }
  };

  f32x16 o[J];
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[j][i] = 0.f;
  Reference<T> ref;
  ref.clear();
  float sum = 0.f;
  const int key_of = (l32 & 19) | (l32 & 4) << 1 | (l32 & 8) >> 1;   // of the product's row l32
  int k_at[S], v_at[4];                                              // octets of the lane's rows; dims 32 and more further on differ by constants
#pragma unroll
  for (int s = 0; s < S; ++s) k_at[s] = key_of * (D * 2) + ((2 * s + hi) ^ k_swizzle<D>(key_of)) * 16;
#pragma unroll
  for (int s = 0; s < 4; ++s) v_at[s] = l32 * 128 + ((2 * s + hi) ^ v_swizzle(l32)) * 16;

  if (t0 < t1) {
    find(t0);
    fetch(t0, 0);
    find(t0 + 1);
  }
  for (int t = t0, buf = 0; t < t1; ++t, buf ^= 1) {
    __builtin_amdgcn_s_waitcnt(0x0F70);                              // vmcnt(0): this wave's part of the tile has arrived
    __syncthreads();
    const int key0 = t * PF_K;
    if (key0 < first || key0 + PF_K > last + 1) {                    // slots of keys that no row sees may hold anything: 0 * NaN is not 0
      for (int i = tid; i < D * 8; i += 64 * W) {
        u32x4* x = (u32x4*)lds.v[buf] + i;
        const int key = key0 + 8 * ((i & 7) ^ v_swizzle(i >> 3));
        u32x4 y = *x;
#pragma unroll
        for (int w = 0; w < 4; ++w)
          y[w] &= (key + 2 * w >= first && key + 2 * w <= last ? 0xffffu : 0u) | (key + 2 * w + 1 >= first && key + 2 * w + 1 <= last ? 0xffff0000u : 0u);
        *x = y;
      }
      __syncthreads();
    }
    if (t + 1 < t1) {
      fetch(t + 1, buf ^ 1);
      find(t + 2);
    }
    if (key0 > w_last || key0 + PF_K <= w_low) continue;             // no row of the wave sees any of it
    const char *kt = lds.k[buf], *vt = lds.v[buf];
    f32x16 sc[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[u][i] = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int u = 0; u < 2; ++u) sc[u] = T::mma32(*(const u32x4*)(kt + u * (32 * D * 2) + k_at[s]), q[s], sc[u]);
    // sc[u][4 (2 s + a) + c]: key 32 u + 16 s + 8 hi + 4 a + c of the tile
    if (key0 + PF_K - 1 > w_all || key0 < w_first) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = key0 + 32 * u + 16 * (i >> 3) + 8 * hi + (i & 7);
          sc[u][i] = key <= lim && key >= low ? sc[u][i] : -INFINITY;
        }
    }
    float x = sc[0][0];
#pragma unroll
    for (int i = 1; i < 32; ++i) x = fmaxf(x, sc[i >> 4][i & 15]);
    x = max_of_2(x) * a.scale2;
    if (__any(ref.moves(x))) {
      const float keep = ref.move(x);
      sum *= keep;
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[j][i] *= keep;
    }
    const float from = -ref.from();
    u32x4 p[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      f32x8 e;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        e[i] = __builtin_amdgcn_exp2f(fmaf(sc[s >> 1][8 * (s & 1) + i], a.scale2, from));
        sum += e[i];
      }
      // off by half a step of the operand type, which adds as much to the result as its own rounding (2.3e-3 of the norm in bf16
      // instead of 1.7e-3); a second product with what the rounding leaves took 542 us instead of 396 for 4096 tokens over 8192
      p[s] = to_16<T>(e);
    }
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int j = 0; j < J; ++j) o[j] = T::mma32(*(const u32x4*)(vt + j * (32 * 128) + v_at[s ^ 2 * (j & 1)]), p[s], o[j]);
  }
  // The same again, at leisure and straight from the pages, for a wave whose sums are no numbers: see `Odd`
  float left = 0.f;                                                  // 0 x is 0 for a number, and only then
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int i = 0; i < 16; ++i) left = fmaf(o[j][i], 0.f, left);
  if (__builtin_expect(__any(left != 0.f), 0)) {
    ref.clear();
    sum = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[j][i] = 0.f;
#pragma unroll 1
    for (int key0 = t0 * PF_K; key0 < t1 * PF_K; key0 += 32) {
      const int row = key0 + key_of;
      const char* k = a.kv.k + in_pool(page(row)) * a.kv.kstride + ((long)h * ps + (row & (ps - 1))) * (D * 2) + hi * 16;
      f32x16 sc;
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
      for (int s = 0; s < S; ++s) sc = T::mma32(*(const u32x4*)(k + s * 32), q[s], sc);
      float x = -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = key0 + 16 * (i >> 3) + 8 * hi + (i & 7);
        sc[i] = key <= lim && key >= low ? sc[i] : -INFINITY;
        x = fmaxf(x, sc[i]);
      }
      x = max_of_2(x) * a.scale2;
      const float keep = __any(ref.moves(x)) ? ref.move(x) : 1.f, from = -ref.from();
      sum *= keep;
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[j][i] *= keep;
#pragma unroll 1
      for (int s = 0; s < 2; ++s) {
        f32x8 e;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          e[i] = __builtin_amdgcn_exp2f(fmaf(s ? sc[8 + i] : sc[i], a.scale2, from));
          sum += e[i];
        }
        const u32x4 p = to_16<T>(e);
        const int key = key0 + 16 * s + 8 * hi;
        const char* vp = a.kv.v + in_pool(page(key)) * a.kv.vstride + (((long)h * D + l32) * ps + (key & (ps - 1))) * 2;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          u32x4 v = *(const u32x4*)(vp + (long)j * 64 * ps);
#pragma unroll
          for (int w = 0; w < 4; ++w)
            v[w] &= (key + 2 * w >= first && key + 2 * w <= last ? 0xffffu : 0u) | (key + 2 * w + 1 >= first && key + 2 * w + 1 <= last ? 0xffff0000u : 0u);
          o[j] = T::mma32(without_odd<T>(v), p, o[j]);
#pragma unroll 1
          for (int kind = 0; kind < ODD_KINDS; ++kind) {
            f32x16 n;
#pragma unroll
            for (int i = 0; i < 16; ++i) n[i] = 0.f;
            n = T::mma32(ones_where_odd<T>(v, kind), ones_where_seen<T>(key, low, lim), n);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[j][i] += odd_sum(n[i] > 0.f, kind);
          }
        }
      }
    }
  }
  sum = sum_of_2(sum);
  if (!mine) return;
  if (a.splits > 1) {                                                // a part: sums, then reference and sum
    const long r = ((long)part * a.s.T + qi) * (a.kv.heads * a.G) + qh;
    float* out = (float*)a.parts + r * D + hi * 4;
    if (sum != 0.f)
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) *(f32x4*)(out + 32 * j + 8 * i) = f32x4{o[j][4 * i], o[j][4 * i + 1], o[j][4 * i + 2], o[j][4 * i + 3]};
    if (hi == 0) ((float2*)((float*)a.parts + (long)a.splits * a.s.T * a.kv.heads * a.G * D))[r] = make_float2(ref.at, sum);
    return;
  }
  const float f = sum == 0.f ? 0.f : 1.f / sum;                      // a row that sees no key is zero
  char* out = a.o + qi * a.o_t + qh * a.o_h + hi * 8;
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 y = f32x4{o[j][4 * i], o[j][4 * i + 1], o[j][4 * i + 2], o[j][4 * i + 3]} * f;
      *(uint2*)(out + 64 * j + 16 * i) = __builtin_bit_cast(uint2, __builtin_convertvector(y, typename T::v4));
    }
}

// The parts of a token's rows joined: four dims a thread, all of a token's over gridDim.y blocks, four parts under way
template <class T, int D>
__global__ __launch_bounds__(256) void paged_chunk_join_kernel(const PagedAttnArgs a) {
  constexpr int U = 4;
  const int t = blockIdx.x, heads = a.kv.heads * a.G, i = blockIdx.y * 256 + threadIdx.x, h = i / (D / 4), d = i % (D / 4) * 4;
  const int b = last_at_most(a.s.B, t, [&](int k) { return clamped(a.s.starts[k], 0, a.s.T); });
  const Seq sq = sequence(a.s, b);
  if (t >= sq.row0 + sq.n || sq.n <= a.most || h >= heads) return;   // nobody's row, or one that the other kernel has written
  const long step = (long)a.s.T * heads, r = (long)t * heads + h;
  const float* parts = (const float*)a.parts;
  const float2* stats = (const float2*)(parts + a.splits * step * D);
  float top = -INFINITY, sum = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < a.splits; p0 += U) {
    f32x4 y[U];
    float2 st[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long at = min(p0 + u, a.splits - 1) * step + r;
      st[u] = stats[at];
      y[u] = *(const f32x4*)(parts + at * D + d);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (p0 + u < a.splits && st[u].y != 0.f) {                     // 0: no key of the part is seen, and its sums are not written
        const float now = fmaxf(top, st[u].x), ref = now == -INFINITY ? 0.f : now;
        const float keep = __builtin_amdgcn_exp2f(top - ref), w = __builtin_amdgcn_exp2f(st[u].x - ref);
        x = x * keep + y[u] * w;
        sum = sum * keep + st[u].y * w;
        top = now;
      }
  }
  x *= sum == 0.f ? 0.f : 1.f / sum;
  *(uint2*)(a.o + t * a.o_t + h * a.o_h + d * 2) = __builtin_bit_cast(uint2, __builtin_convertvector(x, typename T::v4));
}

static long chunk_blocks(const PagedAttnArgs& a) { return (a.s.T / (32 * a.waves / a.G) + a.s.B) * (long)a.kv.heads * a.splits; }
bool chunks_fit_a_launch(const PagedAttnArgs& a) {
  return fits_a_launch(chunk_blocks(a), 64 * a.waves) && (a.splits == 1 || fits_a_launch(a.s.T, 256));
}

template <class T, int D, int W>
static void chunk_grid(PagedAttnArgs a, hipStream_t s) {
  a.tpt = 32 * W / a.G;
  a.by_tpt = FastDiv::by(a.tpt);
  hipLaunchKernelGGL((paged_chunk_kernel<T, D, W>), dim3((unsigned)chunk_blocks(a)), dim3(64 * W), 0, s, a);
  if (a.splits > 1) hipLaunchKernelGGL((paged_chunk_join_kernel<T, D>), dim3(a.s.T, (a.kv.heads * a.G * (D / 4) + 255) / 256), dim3(256), 0, s, a);
}
template <class T, int D>
static void chunk_of(const PagedAttnArgs& a, hipStream_t s) {
  a.waves == 4 ? chunk_grid<T, D, 4>(a, s) : chunk_grid<T, D, 8>(a, s);
}

hipError_t launch_paged_chunks(const PagedAttnArgs& a, int dtype, int head_dim, hipStream_t s) {
  if (dtype == SNA_DTYPE_FP16) head_dim == 64 ? chunk_of<Fp16, 64>(a, s) : chunk_of<Fp16, 128>(a, s);
  else head_dim == 64 ? chunk_of<Bf16, 64>(a, s) : chunk_of<Bf16, 128>(a, s);
  return hipGetLastError();
}

}  // namespace sna
