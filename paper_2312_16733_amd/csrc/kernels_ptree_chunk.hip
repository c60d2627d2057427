// Attention of the tokens of drafted trees over the paged cache, many rows of queries per key / value head: pprefill_kernel.h's walk,
// 128 rows a block.
//   A turn of a tile, 2 blocks of 4 waves on a CU, takes 6200 cycles, of which products are 3070, vector instructions as much and LDS 2500
// (77 tokens over 65519 keys, 32 heads over 8 of 128: 149 to 153 us once the chip has settled).
// What was tried and brought nothing, when the probabilities had one product (4500 cycles, 127 to 130 us with the join): keys asked for two
// tiles ahead and values one and a half (three and two buffers, explicit counts; 137 to 143), operands read in fours before their
// products (129).
#include "pprefill_kernel.h"

namespace sna {

// The keys of all sequences and heads, laid end to end, in equal shares, as where rows are few: trees of a step differ in length and
// size, and shares of each would not fill the last round of blocks (16 trees of up to 32 tokens over up to 4096 keys, 32 heads over
// 8 of 128, with one product of the probabilities: 66 us in five shares each, 58 in equal ones).  A tree of more than 128 rows has a block for each 128 of them on every
// share: they walk the same keys side by side on one XCD, whose L2 reads them once.  Block j of a share is one of plane j, which has parts of
// its own, plane after plane.
template <class T, int D>
struct TreeRows {
  typedef PrefillLds<D> Lds;
  static constexpr int W = 4, kBlocks = 2, kAlign = 1024, kDim = D;
  static constexpr bool PLANES = true;
  static __device__ __forceinline__ int tpt(const PagedAttnArgs& a) { return a.max_new; }
  static __device__ __forceinline__ int tiles(const PagedAttnArgs& a, const Seq& sq, int b) { return sq.n > a.most ? 0 : rows_of_sequence<PF_K, true>(a, sq, b, 0, a.max_new).tiles; }
  static __device__ __forceinline__ RowTile rows(const PagedAttnArgs& a, const Seq& sq, int b, int, int plane) {
    RowTile r = rows_of_sequence<PF_K, true>(a, sq, b, plane * a.tpt, a.tpt);
    r.tiles = tiles(a, sq, b);                                       // also where the tree has no rows here
    r.n = max(r.n, 0);
    return r;
  }
  static __device__ __forceinline__ void attend(const PagedAttnArgs& a, Lds& lds, const RowTile& r, int h, int t0, int t1, float* part) {
    chunk_rows<T, D, W, true>(a, lds, r, h, t0, t1, 0, part);
  }
};

template <class T, int D>
static hipError_t tree_grid(PagedAttnArgs a, hipStream_t s) {
  constexpr int W = TreeRows<T, D>::W;
  a.tpt = 32 * W / a.G;
  if (a.parts) {
    if (a.tpt > a.max_new) a.tpt = a.max_new;                        // of rows_cap rows
    a.rows_cap = a.tpt * a.G;
    a.least = kTreeLeast;
    const int planes = tree_planes(a.max_new, a.G);
    const long pairs = (long)a.s.B * a.kv.heads;                     // (tree, head)s
    hipLaunchKernelGGL((paged_split_kernel<TreeRows<T, D>>), dim3(a.blocks * planes), dim3(64 * W), 0, s, a);
    // rows of a (sequence, head) that a block of the join takes at once, as many as its parts allow
    const int per = std::max(1, (int)(a.blocks / pairs)), at_once = std::max(1, 1024 / D / std::max(1, (per + 7) / 8));
    a.cut = 8 * pairs <= a.blocks ? (int)pairs : a.blocks;           // see paged_join_kernel
    hipLaunchKernelGGL((paged_join_kernel<T, D, true>), dim3(a.cut * planes, (a.rows_cap + at_once - 1) / at_once), dim3(256), 0, s, a);
    return hipGetLastError();
  }
  a.waves = W;
  a.splits = 1;
  a.by_tpt = FastDiv::by(a.tpt);
  const long blocks = chunk_blocks(a);
  if (!fits_a_launch(blocks, 64 * W)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((paged_chunk_kernel<T, D, W, true>), dim3((unsigned)blocks), dim3(64 * W), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_tree_chunks(const PagedAttnArgs& a, int dtype, int head_dim, hipStream_t s) {
  if (dtype == SNA_DTYPE_FP16) return head_dim == 64 ? tree_grid<Fp16, 64>(a, s) : tree_grid<Fp16, 128>(a, s);
  return head_dim == 64 ? tree_grid<Bf16, 64>(a, s) : tree_grid<Bf16, 128>(a, s);
}

}  // namespace sna
