// New tokens enter the paged cache: per-head RMS norm and position rotation of q and k, k and v into their pages.
//   x' = x * rsqrt(mean(x^2) + eps) * w            (with a norm)
//   (x'_a, x'_b) -> (x'_a cos - x'_b sin, x'_a sin + x'_b cos),   angle = position * inv_freq[pair]
// Bound by memory: every element is read once and written once.  A block takes up to 16 tokens that share 16 aligned slots of
// a page, for some heads of q, k or v: then v, which the cache keeps transposed, leaves as whole runs of 16 slots (32 bytes,
// all of a page of 16), and an angle is evaluated once a block instead of once a head.  It is formed in 64 bits, in turns,
// and only its fraction goes on in 32: at position 10^5 a 32-bit product would be off by 6e-3 radians.
#include "paged.h"

namespace sna {

constexpr int AP_TOK = 16;         // aligned slots of a block: the smallest page
constexpr int AP_IT = 4;           // loads of 32 bytes (q, k) or 16 (v) that a thread has under way

// Tiles of the sequences before b, or more: sequence b's new tokens touch at most (n + 14) / 16 + 1 runs of 16 slots.
__device__ __forceinline__ int append_tile0(const PagedSeqs& s, int b) { return (clamped(s.starts[b], 0, s.T) >> 4) + 2 * b; }

template <class T, int D>
__device__ __forceinline__ void append_v(const AppendArgs& a, int part, int row0, int cnt, int off, char* page, int slot, char* lds) {
  constexpr int O = D / 8, LD = D + 8;                               // octets of a head, LDS row
  const int nt = blockDim.x, tid = threadIdx.x, ps2 = 2 << a.kv.lps;
  if (a.one) {
    const int u = part * 64 + tid, h = u / O, o = u % O;
    if (h >= a.kv.heads) return;
    const u32x4 x = *(const u32x4*)(a.v + row0 * a.v_t + h * a.v_h + o * 16);
    char* y = page + ((long)(h * D + o * 8) * ps2) + 2 * slot;
#pragma unroll
    for (int e = 0; e < 8; ++e) *(unsigned short*)(y + e * ps2) = (unsigned short)(x[e >> 1] >> (16 * (e & 1)));
    return;
  }
  constexpr int VH = AP_IT * 256 / (O * AP_TOK);                     // heads of a block
  const int h0 = part * VH;
  u32x4 x[AP_IT];
#pragma unroll
  for (int i = 0; i < AP_IT; ++i) {
    const int u = i * nt + tid, tok = (u / O) % AP_TOK, h = h0 + u / (O * AP_TOK);
    if (tok < cnt && h < a.kv.heads) x[i] = *(const u32x4*)(a.v + (row0 + tok) * a.v_t + h * a.v_h + (u % O) * 16);
  }
#pragma unroll
  for (int i = 0; i < AP_IT; ++i) {
    const int u = i * nt + tid, tok = (u / O) % AP_TOK, h = u / (O * AP_TOK);
    if (tok < cnt && h0 + h < a.kv.heads) *(u32x4*)(lds + ((h * AP_TOK + tok + off) * LD + (u % O) * 8) * 2) = x[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < AP_IT; ++i) {
    const int u = i * nt + tid, so = u & 1, d = (u >> 1) % D, h = (u >> 1) / D;
    if (h0 + h >= a.kv.heads) continue;
    const unsigned short* col = (const unsigned short*)lds + (h * AP_TOK + 8 * so) * LD + d;
    char* y = page + (long)((h0 + h) * D + d) * ps2 + 2 * (slot - off + 8 * so);
    if (off <= 8 * so && off + cnt >= 8 * so + 8) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = col[2 * e * LD] | (unsigned)col[(2 * e + 1) * LD] << 16;
      *(u32x4*)y = w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (8 * so + e >= off && 8 * so + e < off + cnt) *(unsigned short*)(y + 2 * e) = col[e * LD];
    }
  }
}

// A row of D is D / 16 lanes' two octets, partners of the rotation in one lane: octets l and l + half / 8 of the rotated
// elements, then two of what is left over.  Interleaved pairs lie within an octet wherever it is.
template <class T, int D, bool NORM>
__device__ __forceinline__ void append_qk(const AppendArgs& a, const bool is_k, int h0, int row0, int first, int cnt, char* page, int slot, float2* cs) {
  constexpr int L = D / 16, HP = AP_IT * 256 / (L * AP_TOK);         // lanes of a row; heads of a block (of 64 threads: 64 / L)
  const int nt = blockDim.x, tid = threadIdx.x, l = tid % L, half = a.half, ho = half >> 3;
  const int heads = is_k ? a.kv.heads : a.Hq, nh = min(a.one ? 64 / L : HP, heads - h0), rows = cnt * nh;
  const int oa = l < ho ? l : 2 * ho + 2 * (l - ho), ob = l < ho ? l + ho : oa + 1;
  const unsigned inv = 65536u / nh + 1;                              // r / nh for r * nh < 65536
  const char* src = is_k ? a.k : a.q;
  const long st = is_k ? a.k_t : a.q_t, sh = is_k ? a.k_h : a.q_h;
  u32x4 u[AP_IT][2];
#pragma unroll
  for (int i = 0; i < AP_IT; ++i) {
    const int r = (i * nt + tid) / L;
    if (r < rows) {
      const int tok = (r * inv) >> 16, h = h0 + r - tok * nh;
      const char* x = src + (row0 + tok) * st + h * sh;
      u[i][0] = *(const u32x4*)(x + oa * 16);
      u[i][1] = *(const u32x4*)(x + ob * 16);
    }
  }
  f32x8 w[2];
  if (NORM) {
    const float* g = is_k ? a.k_norm : a.q_norm;
#pragma unroll
    for (int e = 0; e < 8; ++e) { w[0][e] = g[oa * 8 + e]; w[1][e] = g[ob * 8 + e]; }
  }
  for (int i = tid; i < cnt * half; i += nt) {
    const int tok = i / half;
    double turns = (double)(first + tok) * (double)a.inv_freq[i - tok * half] * 0.15915494309189533577;
    turns -= rint(turns);
    float sn, co;
    sincospif(2.f * (float)turns, &sn, &co);
    cs[i] = make_float2(co, sn);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < AP_IT; ++i) {
    const int r = (i * nt + tid) / L;
    if (r >= rows) continue;                                         // the same for a row's lanes
    const int tok = (r * inv) >> 16, h = h0 + r - tok * nh;
    f32x8 x = to_f32<T>(u[i][0]), y = to_f32<T>(u[i][1]);
    if (NORM) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], fmaf(y[e], y[e], ss));
#pragma unroll
      for (int m = 1; m < L; m *= 2) ss += __shfl_xor(ss, m, 64);
      const float rs = 1.f / sqrtf(ss * (1.f / D) + a.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) { x[e] *= rs * w[0][e]; y[e] *= rs * w[1][e]; }
    }
    const float2* c = cs + tok * half;
    if (a.interleaved) {
      if (oa < 2 * ho)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 t = c[oa * 4 + e];
          const float p = x[2 * e], q = x[2 * e + 1];
          x[2 * e] = p * t.x - q * t.y;
          x[2 * e + 1] = p * t.y + q * t.x;
        }
      if (ob < 2 * ho)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 t = c[ob * 4 + e];
          const float p = y[2 * e], q = y[2 * e + 1];
          y[2 * e] = p * t.x - q * t.y;
          y[2 * e + 1] = p * t.y + q * t.x;
        }
    } else if (l < ho) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 t = c[l * 8 + e];
        const float p = x[e], q = y[e];
        x[e] = p * t.x - q * t.y;
        y[e] = p * t.y + q * t.x;
      }
    }
    char* dst;
    if (is_k) {
      if (!page) continue;
      dst = page + ((long)(h << a.kv.lps) + slot + tok) * (D * 2);
    } else {
      dst = a.qo + (row0 + tok) * a.o_t + h * a.o_h;
    }
    *(u32x4*)(dst + oa * 16) = to_16<T>(x);
    *(u32x4*)(dst + ob * 16) = to_16<T>(y);
  }
}

// Grid: runs of 16 slots x (parts of q's heads, of k's, of v's).  A step of single tokens, where only latency counts, gets a
// wave for each token and part instead.
template <class T, int D, bool NORM>
__global__ __launch_bounds__(256) void append_kernel(const AppendArgs a) {
  constexpr int L = D / 16, HP = AP_IT * 256 / (L * AP_TOK), VH = AP_IT * 256 / (D / 8 * AP_TOK);
  __shared__ __attribute__((aligned(16))) char lds[VH * AP_TOK * (D + 8) * 2];
  static_assert(sizeof(lds) >= AP_TOK * D / 2 * sizeof(float2), "the angles of 16 tokens");
  int b, row0, first, cnt, off;
  if (a.one) {
    b = blockIdx.x;
    row0 = b;
    first = clamped(a.s.lens[b], 0, 1 << 30) - 1;
    cnt = 1;
    off = 0;
  } else {
    const int tile = blockIdx.x;
    b = last_at_most(a.s.B, tile, [&](int i) { return append_tile0(a.s, i); });
    const Seq q = sequence(a.s, b);
    const int p0 = q.len - q.n, base = (p0 & ~(AP_TOK - 1)) + (tile - append_tile0(a.s, b)) * AP_TOK;
    first = max(p0, base);
    cnt = min(q.len, base + AP_TOK) - first;
    if (cnt <= 0) return;
    row0 = q.row0 + first - p0;
    off = first - base;
  }
  const int col = first >> a.kv.lps, slot = first & ((1 << a.kv.lps) - 1);
  int page = -1;
  if (first >= 0 && col < a.s.width) page = a.s.table[(long)b * a.s.tstride + col];
  const bool ok = page >= 0 && page < a.kv.n_pages;                  // a token without a page of the pool is not stored
  int part = blockIdx.y;
  const int hp = a.one ? 64 / L : HP;
  if (part < a.q_parts) return append_qk<T, D, NORM>(a, false, part * hp, row0, first, cnt, nullptr, 0, (float2*)lds);
  part -= a.q_parts;
  if (part < a.k_parts) return append_qk<T, D, NORM>(a, true, part * hp, row0, first, cnt, ok ? a.kv.k + page * a.kv.kstride : nullptr, slot, (float2*)lds);
  if (ok) append_v<T, D>(a, part - a.k_parts, row0, cnt, off, a.kv.v + page * a.kv.vstride, slot, lds);
}

template <class T, int D>
static void append_grid(AppendArgs a, hipStream_t s) {
  constexpr int L = D / 16;
  const int hp = a.one ? 64 / L : AP_IT * 256 / (L * AP_TOK), vh = a.one ? 64 / (D / 8) : AP_IT * 256 / (D / 8 * AP_TOK);
  a.q_parts = (a.Hq + hp - 1) / hp;
  a.k_parts = (a.kv.heads + hp - 1) / hp;
  const dim3 grid(a.one ? a.s.B : a.s.T / AP_TOK + 2 * a.s.B, a.q_parts + a.k_parts + (a.kv.heads + vh - 1) / vh), block(a.one ? 64 : 256);
  if (a.q_norm) hipLaunchKernelGGL((append_kernel<T, D, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((append_kernel<T, D, false>), grid, block, 0, s, a);
}

hipError_t launch_append(const AppendArgs& a, int dtype, int head_dim, hipStream_t s) {
  if (dtype == SNA_DTYPE_FP16) head_dim == 64 ? append_grid<Fp16, 64>(a, s) : append_grid<Fp16, 128>(a, s);
  else head_dim == 64 ? append_grid<Bf16, 64>(a, s) : append_grid<Bf16, 128>(a, s);
  return hipGetLastError();
}

}  // namespace sna
