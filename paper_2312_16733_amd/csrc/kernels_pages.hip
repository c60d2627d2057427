// Moving what a paged cache holds: the accepted tokens of a drafted tree up behind the ones before, and whole pages to others.
// Bound by memory.  A slot is a row of a key page, 2 head_dim bytes in one piece, and a column of a value page, 2 bytes in each of
// head_dim rows: a value that moves costs the lines around it at both ends (64 sequences, up to 7 moves each, 256 heads of 128, pages of
// 16: 59 MB move, 100 are read and 80 written in 36 us, 5.0 TB/s).  Four pieces a thread, for fewer look-ups, took 51 us.
#include "paged.h"

namespace sna {

constexpr int CP_MOVES = 256;      // moves that a block looks up at a time, one a thread
constexpr int CP_U = 8;            // of them under way
struct Move { long from, to; };    // bytes from the page's first head

// Kept token i of a sequence goes from slot base + kept[i] to slot base + i.  The kept ones rise, so kept[i] >= i, and a slot that
// is written has been read by then if it is read at all: one thread does all moves of its 16 bytes of a key row, or of its row of
// a value page, in order, and needs no other.
__global__ __launch_bounds__(256) void kv_compact_kernel(const CompactArgs a) {
  __shared__ Move mk[CP_MOVES], mv[CP_MOVES];
  const int tid = threadIdx.x, b = blockIdx.x / a.blocks, part = blockIdx.x % a.blocks;
  const Seq q = uniform(sequence(a.s, b));
  const int n = min(q.n, a.max_new), base = q.len - n, count = min(clamped(a.counts[b], 0, a.width), n);
  if (part == 0 && tid == 0) a.lens[b] = max(base + count, 0);
  const bool keys = part < a.k_blocks;
  const int t = (keys ? part : part - a.k_blocks) * 256 + tid, D = a.dim, ps = 1 << a.kv.lps;
  const bool mine = t < (keys ? a.kv.heads * (D / 8) : a.kv.heads * D);
  // of the page's keys: head, row 0, octet; of its values: row (head, dim)
  const long at = keys ? ((long)(t / (D / 8)) * ps) * (2 * D) + t % (D / 8) * 16 : (long)t * ps * 2;
  const auto page = [&](int slot) {
    const int col = slot >> a.kv.lps, id = slot >= 0 && col < a.s.width ? a.s.table[(long)b * a.s.tstride + col] : -1;
    return id < a.kv.n_pages ? id : -1;
  };
  for (int i0 = 0; i0 < count; i0 += CP_MOVES) {
    const int left = min(count - i0, CP_MOVES);
    if (tid < left) {
      const int i = i0 + tid, j = a.kept[(long)b * a.width + i];
      Move k = {-1, -1}, v = {-1, -1};
      if (j > i && j < n) {                                          // one that stays, or is none of the step's, does not move
        const int from = base + j, to = base + i, p0 = page(from), p1 = page(to);
        if (p0 >= 0 && p1 >= 0) {
          k = Move{p0 * a.kv.kstride + (long)(from & (ps - 1)) * (2 * D), p1 * a.kv.kstride + (long)(to & (ps - 1)) * (2 * D)};
          v = Move{p0 * a.kv.vstride + 2 * (from & (ps - 1)), p1 * a.kv.vstride + 2 * (to & (ps - 1))};
        }
      }
      mk[tid] = k;
      mv[tid] = v;
    }
    __syncthreads();
    if (mine)
      for (int i = 0; i < left; i += CP_U) {
        if (keys) {
          u32x4 x[CP_U];
#pragma unroll
          for (int u = 0; u < CP_U; ++u)
            if (i + u < left && mk[i + u].from >= 0) x[u] = *(const u32x4*)(a.kv.k + at + mk[i + u].from);
#pragma unroll
          for (int u = 0; u < CP_U; ++u)
            if (i + u < left && mk[i + u].from >= 0) *(u32x4*)(a.kv.k + at + mk[i + u].to) = x[u];
        } else {
          unsigned short x[CP_U];
#pragma unroll
          for (int u = 0; u < CP_U; ++u)
            if (i + u < left && mv[i + u].from >= 0) x[u] = *(const unsigned short*)(a.kv.v + at + mv[i + u].from);
#pragma unroll
          for (int u = 0; u < CP_U; ++u)
            if (i + u < left && mv[i + u].from >= 0) *(unsigned short*)(a.kv.v + at + mv[i + u].to) = x[u];
        }
      }
    __syncthreads();
  }
}

hipError_t launch_compact(CompactArgs a, hipStream_t s) {
  a.k_blocks = (a.kv.heads * (a.dim / 8) + 255) / 256;
  a.blocks = a.k_blocks + (a.kv.heads * a.dim + 255) / 256;
  const long blocks = (long)a.s.B * a.blocks;
  if (!fits_a_launch(blocks, 256)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(kv_compact_kernel, dim3((unsigned)blocks), dim3(256), 0, s, a);
  return hipGetLastError();
}

// A block has 16 KB of the keys or values of one page, 16 bytes a thread and four of them under way (192 pages of 2 MB, each source
// three times: 117 us, 0.81 GB at 6.9 TB/s; a large copy of distinct memory reaches 4.9)
constexpr int PC_U = 4, PC_BYTES = PC_U * 256 * 16;
__global__ __launch_bounds__(256) void copy_pages_kernel(const PageCopyArgs a) {
  const int x = blockIdx.x / a.blocks, part = blockIdx.x % a.blocks;
  const int from = a.source[x], to = a.target[x];
  if ((unsigned)from >= (unsigned)a.kv.n_pages || (unsigned)to >= (unsigned)a.kv.n_pages || from == to) return;
  const bool values = part >= a.blocks / 2;
  const long stride = values ? a.kv.vstride : a.kv.kstride, at = (long)(values ? part - a.blocks / 2 : part) * PC_BYTES + threadIdx.x * 16;
  char* pages = values ? a.kv.v : a.kv.k;
  const char* src = pages + from * stride + at;
  char* dst = pages + to * stride + at;
  u32x4 v[PC_U];
#pragma unroll
  for (int u = 0; u < PC_U; ++u)
    if (at + u * 4096 < a.bytes) v[u] = *(const u32x4*)(src + u * 4096);
#pragma unroll
  for (int u = 0; u < PC_U; ++u)
    if (at + u * 4096 < a.bytes) *(u32x4*)(dst + u * 4096) = v[u];
}

hipError_t launch_copy_pages(PageCopyArgs a, int n, hipStream_t s) {
  a.blocks = 2 * (int)((a.bytes + PC_BYTES - 1) / PC_BYTES);
  const long blocks = (long)n * a.blocks;
  if (!fits_a_launch(blocks, 256)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(copy_pages_kernel, dim3((unsigned)blocks), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace sna
