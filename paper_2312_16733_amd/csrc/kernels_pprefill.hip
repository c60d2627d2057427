// Attention of a step's new tokens over the paged cache, many rows of queries per key / value head (chunks of prompts).
// Bound by the matrix pipe and, nearly as much, by the vector pipe's exponentials.  A block holds 32 rows a wave (tokens times
// the query heads of one key / value head) and walks its keys in tiles of 64, fetched from the pages straight into LDS, one
// tile ahead.  As where rows are few, the scores are formed transposed: a lane has one row, and the keys of a product's 32
// rows are chosen so (row 16 s + 8 a + 4 h + c is key 16 s + 8 h + 4 a + c) that its scores are what the second product wants.
#include <algorithm>

#include "paged.h"

namespace sna {

typedef __attribute__((address_space(3))) char lds_char;
constexpr int PF_K = 64;           // keys of a tile

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
  const int h = blockIdx.x % a.kv.heads, tile = gridDim.x / a.kv.heads - 1 - blockIdx.x / a.kv.heads;
  const auto tile0 = [&](int i) { return a.by_tpt.div(clamped(a.s.starts[i], 0, a.s.T)) + i; };
  const int b = last_at_most(a.s.B, tile, tile0);
  const Seq sq = sequence(a.s, b);
  const int i0 = (tile - tile0(b)) * a.tpt, n = i0 < 0 ? 0 : min(sq.n - i0, a.tpt);
  if (n <= 0) return;
  const int row0 = sq.row0 + i0, pos0 = sq.len - sq.n + i0, rows = n * a.G;
  const int last = min(pos0 + n - 1, (a.s.width << a.kv.lps) - 1);
  const int first = max(a.window <= pos0 ? pos0 - a.window + 1 : 0, 0);
  int t0 = first / PF_K, t1 = last < 0 ? t0 : last / PF_K + 1;
  const int* table = a.s.table + (long)b * a.s.tstride;
  const int c_lo = first >> a.kv.lps, c_hi = max(last, 0) >> a.kv.lps, ps = 1 << a.kv.lps;
  const auto page = [&](int key) { return clamped(table[clamped(key >> a.kv.lps, c_lo, c_hi)], 0, a.kv.n_pages - 1); };

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
  int kid, vid[VI > 1 ? 2 : 1];
  const auto find = [&](int t) {
    kid = page(t * PF_K + KI * KR * wave);                           // KI * KR keys of a wave: within 16 aligned ones
#pragma unroll
    for (int i = 0; i < (VI > 1 && W < 8 ? 2 : 1); ++i) vid[i] = page(t * PF_K + 8 * (v_pos ^ v_row ^ ((wave + W * i) & 7)));
  };
  const auto fetch = [&](int t, int buf) {
    const char* kp = a.kv.k + kid * a.kv.kstride + (long)h * ps * (D * 2);
#pragma unroll
    for (int i = 0; i < KI; ++i) {
      const int r = (wave * KI + i) * KR + k_row, slot = (t * PF_K + r) & (ps - 1);
      fetch16(kp + slot * (D * 2) + (k_pos ^ k_swizzle<D>(r)) * 16, (lds_char*)lds.k[buf] + (wave * KI + i) * 1024);
    }
#pragma unroll
    for (int i = 0; i < VI; ++i) {
      const int f = wave + W * i, d = f * 8 + v_row, o = v_pos ^ v_row ^ (f & 7), slot = (t * PF_K + 8 * o) & (ps - 1);
      fetch16(a.kv.v + vid[W < 8 ? i & 1 : 0] * a.kv.vstride + (((long)h * D + d) * ps + slot) * 2, (lds_char*)lds.v[buf] + f * 1024);
    }
  };

  f32x16 o[J];
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[j][i] = 0.f;
  float top = -INFINITY, sum = 0.f;                                  // top: of the scores before the scale
  const int key_of = (l32 & 19) | (l32 & 4) << 1 | (l32 & 8) >> 1;   // of the product's row l32
  const int k_at = key_of * (D * 2), k_sw = k_swizzle<D>(key_of), v_at = l32 * 128;

  if (t0 < t1) {
    find(t0);
    fetch(t0, 0);
    find(t0 + 1);
  }
  for (int t = t0, buf = 0; t < t1; ++t, buf ^= 1) {
    __builtin_amdgcn_s_waitcnt(0x0F70);                              // vmcnt(0): this wave's part of the tile has arrived
    __syncthreads();
    if (t + 1 < t1) {
      fetch(t + 1, buf ^ 1);
      find(t + 2);
    }
    const int key0 = t * PF_K;
    if (key0 > w_last || key0 + PF_K <= w_low) continue;             // no row of the wave sees any of it
    f32x16 sc[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[u][i] = 0.f;
#pragma unroll
      for (int s = 0; s < S; ++s)
        sc[u] = T::mma32(*(const u32x4*)(lds.k[buf] + u * (32 * D * 2) + k_at + ((2 * s + hi) ^ k_sw) * 16), q[s], sc[u]);
    }
    // sc[u][4 (2 s + a) + c]: key 32 u + 16 s + 8 hi + 4 a + c of the tile
    const bool edge = key0 + PF_K - 1 > w_all || key0 < w_first;
    if (edge) {
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
    x = max_of_2(x);
    // the reference is raised only where a score exceeds it by a factor of 2^8 and more: below that the exponentials, their
    // sums and the products are exact enough as they are (p up to 2^8 in the operand type, fp32 sums), and o stays untouched
    if (__any((x - top) * a.scale2 > 8.f)) {
      const float now = fmaxf(top, x), keep = __builtin_amdgcn_exp2f((top - (now == -INFINITY ? 0.f : now)) * a.scale2);
      top = now;
      sum *= keep;
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[j][i] *= keep;
    }
    const float ref = top == -INFINITY ? 0.f : -top * a.scale2;
    u32x4 p[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      f32x8 e;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        e[i] = __builtin_amdgcn_exp2f(fmaf(sc[s >> 1][8 * (s & 1) + i], a.scale2, ref));
        sum += e[i];
      }
      p[s] = to_16<T>(e);                                            // off by half a step of the operand type
    }
    const bool partial = key0 < first || key0 + PF_K > last + 1;     // slots that hold no key may hold anything: 0 * NaN is not 0
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int d = 32 * j + l32;
        u32x4 v = *(const u32x4*)(lds.v[buf] + j * (32 * 128) + v_at + ((2 * s + hi) ^ v_swizzle(d)) * 16);
        if (partial) {
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const int key = key0 + 16 * s + 8 * hi + 2 * w;
            v[w] &= (key >= first && key <= last ? 0xffffu : 0u) | (key + 1 >= first && key + 1 <= last ? 0xffff0000u : 0u);
          }
        }
        o[j] = T::mma32(v, p[s], o[j]);
      }
  }
  sum = sum_of_2(sum);
  if (!mine) return;
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

template <class T, int D>
static void chunk_grid(PagedAttnArgs a, hipStream_t s) {
  constexpr int W = 8;
  a.tpt = 32 * W / a.G;
  a.by_tpt = FastDiv::by(a.tpt);
  hipLaunchKernelGGL((paged_chunk_kernel<T, D, W>), dim3((a.s.T / a.tpt + a.s.B) * a.kv.heads), dim3(64 * W), 0, s, a);
}

hipError_t launch_paged_chunks(const PagedAttnArgs& a, int dtype, int head_dim, hipStream_t s) {
  if (dtype == SNA_DTYPE_FP16) head_dim == 64 ? chunk_grid<Fp16, 64>(a, s) : chunk_grid<Fp16, 128>(a, s);
  else head_dim == 64 ? chunk_grid<Bf16, 64>(a, s) : chunk_grid<Bf16, 128>(a, s);
  return hipGetLastError();
}

}  // namespace sna
