// Attention of chunks of prompts over the paged cache: the kernel in pprefill_kernel.h, and the join of what its shares leave.
#include "pprefill_kernel.h"

namespace sna {

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

bool chunks_fit_a_launch(const PagedAttnArgs& a) {
  return fits_a_launch(chunk_blocks(a), 64 * a.waves) && (a.splits == 1 || fits_a_launch(a.s.T, 256));
}

template <class T, int D, int W>
static void chunk_grid(PagedAttnArgs a, hipStream_t s) {
  a.tpt = 32 * W / a.G;
  a.by_tpt = FastDiv::by(a.tpt);
  hipLaunchKernelGGL((paged_chunk_kernel<T, D, W, false>), dim3((unsigned)chunk_blocks(a)), dim3(64 * W), 0, s, a);
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
