// New tokens enter the paged cache: per-head RMS norm and position rotation of q and k, k and v into their pages.
//   x' = x * rsqrt(mean(x^2) + eps) * w            (with a norm)
//   (x'_a, x'_b) -> (x'_a cos - x'_b sin, x'_a sin + x'_b cos),   angle = position * inv_freq[pair]
// Bound by memory: every element is read once and written once (13551 tokens of 32 + 8 + 8 heads of 128: 69.6 to 71.3 us by card,
// 4.7 TB/s; a large copy reaches 4.9 to 5.0).  A block takes the new tokens of 16 aligned slots of a page and some heads of q or k, so that an
// angle is evaluated once a block instead of once a head, or of 64 slots and some heads of v: the cache keeps v transposed, and
// 64 slots are a line of 128 bytes (runs of 16 slots, written by four blocks, made it 85 to 97 us).  Two rows' loads a thread
// are under way: four took the registers of the fifth wave of a SIMD (85 us).  An angle is formed in 64 bits, in turns, and
// only its fraction goes on in 32: at position 10^5 a 32-bit product would be off by 6e-3 radians.
#include "paged.h"

namespace sna {

constexpr int AP_TOK = 16;         // aligned slots of a block of q or k: the smallest page
constexpr int AP_VT = 64;          // of v: 128 bytes of a row of the transposed page, a whole line of the cache
constexpr int AP_IT = 4;           // pieces of 32 bytes (q, k) or 16 (v) a thread

// Tiles of the sequences before b, or more: n new tokens touch at most (n + TOK - 2) / TOK + 1 runs of TOK slots
template <int TOK>
__device__ __forceinline__ int append_tile0(const PagedSeqs& s, int b) { return clamped(s.starts[b], 0, s.T) / TOK + 2 * b; }
// The new tokens of one of those runs
struct Run { int b, row0, first, cnt, off; };    // sequence, first row, its position, tokens, slots before it in the run
template <int TOK>
__device__ __forceinline__ Run append_run(const AppendArgs& a, int tile) {
  Run r;
  if (a.one) return Run{tile, tile, clamped(a.s.lens[tile], 0, a.s.max_len) - 1, 1, 0};
  r.b = last_at_most(a.s.B, tile, [&](int i) { return append_tile0<TOK>(a.s, i); });
  const Seq q = uniform(sequence(a.s, r.b));
  const int p0 = q.len - q.n, base = (p0 & ~(TOK - 1)) + (tile - append_tile0<TOK>(a.s, r.b)) * TOK;
  r.first = max(p0, base);
  r.cnt = min(q.len, base + TOK) - r.first;
  r.row0 = q.row0 + r.first - p0;
  r.off = r.first - base;
  return r;
}
__device__ __forceinline__ int page_of(const AppendArgs& a, int b, int pos) {            // -1: none of the pool's
  const int col = pos >> a.kv.lps;
  const int page = pos >= 0 && col < a.s.width ? a.s.table[(long)b * a.s.tstride + col] : -1;
  return page < a.kv.n_pages ? page : -1;
}

// Values: VT aligned slots of VH heads, through LDS
template <class T, int D>
__device__ __forceinline__ void append_v(const AppendArgs& a, int tile, int part, char* lds) {
  constexpr int O = D / 8, LD = D + 8, VH = AP_IT * 256 / (O * AP_VT);     // octets of a head, LDS row; heads of a block
  const int tid = threadIdx.x, ps2 = 2 << a.kv.lps, mask = (1 << a.kv.lps) - 1;
  const Run r = append_run<AP_VT>(a, tile);
  if (a.one) {
    const int page = page_of(a, r.b, r.first), u = part * 64 + tid, h = u / O, o = u % O;
    if (h >= a.kv.heads || page < 0) return;
    const u32x4 x = *(const u32x4*)(a.v + r.row0 * a.v_t + h * a.v_h + o * 16);
    char* y = a.kv.v + page * a.kv.vstride + ((long)(h * D + o * 8) * ps2) + 2 * (r.first & mask);
#pragma unroll
    for (int e = 0; e < 8; ++e) *(unsigned short*)(y + e * ps2) = (unsigned short)(x[e >> 1] >> (16 * (e & 1)));
    return;
  }
  if (r.cnt <= 0) return;
  const int h0 = part * VH;
  u32x4 x[AP_IT];
#pragma unroll
  for (int i = 0; i < AP_IT; ++i) {
    const int u = i * 256 + tid, tok = min((u / O) % AP_VT, r.cnt - 1), h = min(h0 + u / (O * AP_VT), a.kv.heads - 1);
    x[i] = *(const u32x4*)(a.v + (r.row0 + tok) * a.v_t + h * a.v_h + (u % O) * 16);
  }
  // a thread writes runs of 8 slots: so-th of the tile, the same for all of its runs
  constexpr int SO = AP_VT / 8;
  const int so = tid % SO, first = r.first - r.off + 8 * so, page = page_of(a, r.b, first);
#pragma unroll
  for (int i = 0; i < AP_IT; ++i) {
    const int u = i * 256 + tid, tok = (u / O) % AP_VT, h = u / (O * AP_VT);
    if (tok < r.cnt && h0 + h < a.kv.heads) *(u32x4*)(lds + ((h * AP_VT + tok + r.off) * LD + (u % O) * 8) * 2) = x[i];
  }
  __syncthreads();
  if (page < 0) return;
#pragma unroll
  for (int i = 0; i < AP_IT; ++i) {
    const int u = i * 256 + tid, d = (u / SO) % D, h = u / SO / D;
    if (h0 + h >= a.kv.heads) continue;
    const unsigned short* col = (const unsigned short*)lds + (h * AP_VT + 8 * so) * LD + d;
    char* y = a.kv.v + page * a.kv.vstride + (long)((h0 + h) * D + d) * ps2 + 2 * (first & mask);
    if (r.off <= 8 * so && r.off + r.cnt >= 8 * so + 8) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = col[2 * e * LD] | (unsigned)col[(2 * e + 1) * LD] << 16;
      *(u32x4*)y = w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (8 * so + e >= r.off && 8 * so + e < r.off + r.cnt) *(unsigned short*)(y + 2 * e) = col[e * LD];
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
  // rows beyond the last read it again: a guarded load would be waited for before the next guard
  u32x4 u[2][2];
  const auto load = [&](int i) {
    const int r = min((i * nt + tid) / L, rows - 1), tok = (r * inv) >> 16, h = h0 + r - tok * nh;
    const char* x = src + (row0 + tok) * st + h * sh;
    u[i & 1][0] = *(const u32x4*)(x + oa * 16);
    u[i & 1][1] = *(const u32x4*)(x + ob * 16);
  };
  load(0);
  if (nt / L < rows) load(1);
  f32x8 w[2];
  if (NORM) {
    const float* g = is_k ? a.k_norm : a.q_norm;
#pragma unroll
    for (int e = 0; e < 8; ++e) { w[0][e] = g[oa * 8 + e]; w[1][e] = g[ob * 8 + e]; }
  }
  for (int i = tid; i < cnt * half; i += nt) {
    const int tok = i / half;
    double turns = (double)(a.positions ? a.positions[row0 + tok] : first + tok) * (double)a.inv_freq[i - tok * half] * 0.15915494309189533577;
    turns -= rint(turns);
    float sn, co;
    sincospif(2.f * (float)turns, &sn, &co);
    cs[i] = make_float2(co, sn);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < AP_IT; ++i) {
    const int r = (i * nt + tid) / L;
    f32x8 x = to_f32<T>(u[i & 1][0]), y = to_f32<T>(u[i & 1][1]);
    if (i + 2 < AP_IT && (i + 2) * nt / L < rows) load(i + 2);
    if (r >= rows) continue;                                         // the same for a row's lanes
    const int tok = (r * inv) >> 16, h = h0 + r - tok * nh;
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

// Blocks: (runs of AP_TOK slots) x (parts of q's heads, of k's), then (runs of AP_VT) x (parts of v's).  A step of single tokens,
// where only latency counts, gets a wave for each token and part instead.
template <class T, int D, bool NORM>
__global__ __launch_bounds__(256) void append_kernel(const AppendArgs a) {
  constexpr int L = D / 16, HP = AP_IT * 256 / (L * AP_TOK), VH = AP_IT * 256 / (D / 8 * AP_VT);
  __shared__ __attribute__((aligned(16))) char lds[VH * AP_VT * (D + 8) * 2];
  static_assert(sizeof(lds) >= AP_TOK * D / 2 * sizeof(float2), "the angles of 16 tokens");
  const int x = blockIdx.x, qk = a.q_parts + a.k_parts;
  if (x >= a.qk_tiles * qk) return append_v<T, D>(a, (x - a.qk_tiles * qk) / a.v_parts, (x - a.qk_tiles * qk) % a.v_parts, lds);
  const int part = x % qk, hp = a.one ? 64 / L : HP;
  const Run r = append_run<AP_TOK>(a, x / qk);
  if (r.cnt <= 0) return;
  const bool is_k = part >= a.q_parts;
  const int page = is_k ? page_of(a, r.b, r.first) : -1;             // a token without a page of the pool is not stored
  append_qk<T, D, NORM>(a, is_k, (part - (is_k ? a.q_parts : 0)) * hp, r.row0, r.first, r.cnt, page < 0 ? nullptr : a.kv.k + page * a.kv.kstride,
                        r.first & ((1 << a.kv.lps) - 1), (float2*)lds);
}

template <class T, int D>
static hipError_t append_grid(AppendArgs a, hipStream_t s) {
  constexpr int L = D / 16;
  const int hp = a.one ? 64 / L : AP_IT * 256 / (L * AP_TOK), vh = a.one ? 64 / (D / 8) : AP_IT * 256 / (D / 8 * AP_VT);
  a.q_parts = (a.Hq + hp - 1) / hp;
  a.k_parts = (a.kv.heads + hp - 1) / hp;
  a.v_parts = (a.kv.heads + vh - 1) / vh;
  a.qk_tiles = a.one ? a.s.B : a.s.T / AP_TOK + 2 * a.s.B;
  const int v_tiles = a.one ? a.s.B : a.s.T / AP_VT + 2 * a.s.B;
  const long blocks = (long)a.qk_tiles * (a.q_parts + a.k_parts) + (long)v_tiles * a.v_parts;
  const dim3 grid((unsigned)blocks), block(a.one ? 64 : 256);
  if (!fits_a_launch(blocks, block.x)) return hipErrorInvalidConfiguration;
  if (a.q_norm) hipLaunchKernelGGL((append_kernel<T, D, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((append_kernel<T, D, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_append(const AppendArgs& a, int dtype, int head_dim, hipStream_t s) {
  if (dtype == SNA_DTYPE_FP16) return head_dim == 64 ? append_grid<Fp16, 64>(a, s) : append_grid<Fp16, 128>(a, s);
  return head_dim == 64 ? append_grid<Bf16, 64>(a, s) : append_grid<Bf16, 128>(a, s);
}

}  // namespace sna
