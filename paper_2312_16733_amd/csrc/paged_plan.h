// How a step of paged attention is launched, from what the host knows of it: plain host code, but for the sizes that the kernels
// share with it.
#pragma once
#include <algorithm>
#include <cstddef>

namespace sna {

// ---- few rows of queries per key / value head (kernels_pattn.hip) ----
// Keys of a wave's tile: 64, or 32 where more rows of sums would leave room in the registers for one block on a CU only
constexpr int tile_keys(int D, int MB) { return MB * D > 128 ? 32 : 64; }
// Scores of a step (rows, all heads, times keys) up to which the few-rows kernel is used for chunks, too, in us there and with the
// many-rows kernel.  Heads of 64: 500 tokens over 2000 keys, 12 heads (12 M) 16.8 and 20.7; 32 x 40 over 1000, 16 heads (20 M)
// 19.7 and 26.3.  Beside single tokens, which the many-rows kernel leaves to launches of their own: 200 over 2000, 32 heads, and
// seven tokens (13 M) 39.7 and 46.0.  Chunks of one length of 128-wide heads: 60 over 4096, 32 heads (8 M) 27.2 and 24.2; 250 over
// 2000, 40 heads (19 M) 41.5 and 30.9.
constexpr long kFewScores = 24l << 20, kFewScoresEqual = 7l << 20;
// Two blocks on a CU where the registers allow it: 8 waves with 16 KB and more under way each
constexpr int blocks_of(int D, int MB) { return MB * D <= 256 ? 2 : 1; }

// Whoever begins a part that a later block continues writes down what it is
struct First { int row0, n, h, last; };                              // first row, tokens (0: none was begun), head, block
constexpr int kSplitW = 4;         // waves of a block
constexpr long part_floats(long rows, int D) { return (rows * (D + 2) + 3) & ~3l; }    // 16-byte aligned

// ---- many rows (kernels_pprefill.hip) ----
constexpr int PF_K = 64;           // keys of a tile
struct ChunkPlan { int waves, splits; };         // waves of a block, shares of the keys
// Waves of a block, of 32 rows each, and shares of the keys.  The time of a launch is taken to be its rounds of blocks times a
// block's tiles times a tile, 2 us on a full CU (one block of 8 waves, or two of 4) and 1.5 for a lone block of 4, 1.24 and 1.18 with
// heads of 64, and where the keys are shared a second launch and the parts, written and read at 4.5 TB/s.  A share has 4 tiles or
// more.  Measured, 32 heads over 8 of 128: 512 tokens over 8192 keys in shares 81 us (162 by blocks of few rows), 300 in shares 57 (113),
// 100 in shares 32 (68); four chunks of up to 500 over 2000 whole 68, in 4 shares 128.
inline ChunkPlan plan_of_chunks(int n_tokens, int kv_heads, int group, int max_new, long keys, int head_dim) {
  const long tiles = (keys + PF_K - 1) / PF_K, like = (n_tokens + max_new - 1) / max_new;                // sequences, if all were as long
  const double tile_us = head_dim == 128 ? 2.0 : 1.24, lone_us = head_dim == 128 ? 1.5 : 1.18, part_us = (double)n_tokens * kv_heads * group * (head_dim + 2) * 8 / 4.5e6;
  ChunkPlan best = {};
  double least = 1e30;
  for (int waves = 8; waves >= 4; waves -= 4) {
    const long tpt = 32 * waves / group, blocks = like * ((max_new + tpt - 1) / tpt) * kv_heads, room = 256 * (8 / waves);
    for (int s = 1; s <= 16 && (s == 1 || tiles >= 4 * s); ++s) {
      const double one = waves == 4 && blocks * s <= 256 ? lone_us : tile_us;
      const double us = (double)((blocks * s + room - 1) / room * ((tiles + s - 1) / s)) * one + (s > 1 ? 8 + s * part_us : 0.0);
      if (us < least) {
        least = us;
        best = ChunkPlan{waves, s};
      }
    }
  }
  return best;
}

// ---- which of them ----
// Blocks of whole (tile of rows, head)s walk the longest sequence, which a CU reads at 60 to 70 GB/s; shared out, the keys take
// what the chip reads at, but their parts are written and joined in a second launch, 6 us.  One tile of rows a sequence (decoding):
// shared from 1024 keys of 128 on (8 sequences of up to 2048, 8 heads: 18.1 us shared, 23.7 whole; 32 of up to 1000: 21.9 and
// 16.5), from half of that where most of the chip would be idle (one of 1000: 11.0 and 13.3).
// Several: where sharing saves kSplitGain turns of a tile for each wave, with sequences of 0.6 of the longest on average (60
// tokens over 4096 keys, 32 heads: 26.6 us shared, 55 whole; 512 over their own 512: 60 and 22.6, since there every block has to
// find its way through many short rows of tiles).
constexpr long kSplitKeys = 1024 * 128, kSplitGain = 6;

// Blocks that share the keys.  One on each CU keeps 128 KB under way (heads of 128) and cuts fewer parts off than two: one sequence
// of 131071 keys 97 us and 104, 64 of up to 8192 193 and 195; two where (tile of rows, head)s are many and few of them are cut
// (200 sequences of up to 2500: 219 and 228), or half as long (64 of up to 8192, heads of 64: 61.7 and 63.7).
inline int split_blocks(int head_dim, int mb, long units) { return 256 * (head_dim == 128 && units <= 512 ? 1 : blocks_of(head_dim, mb)); }

// How a step is launched, from what the host knows of it.
struct AttnPlan {
  int mb;                          // 16 rows of a block of the few-rows kernel, of which there are 1, 2 or 4; 0: not launched
  int blocks;                      // that its keys are shared out over; 0: a block walks all of its rows' keys
  int waves;                       // of a block that walks all keys of its rows
  int most;                        // tokens of a sequence up to which it takes it
  bool chunks;                     // the many-rows kernel takes the other sequences
  ChunkPlan chunk;
  size_t parts, chunk_parts;       // bytes of the workspace, for either
};
inline size_t parts_of(int blocks, int rows, int head_dim) { return (blocks * (sizeof(First) + 2 * part_floats(rows, head_dim) * sizeof(float)) + 255) & ~(size_t)255; }
inline AttnPlan plan_of(int n_seqs, int n_tokens, int kv_heads, int group, int max_new, int max_len, int window, int head_dim, bool few_of_tree = false) {
  const long rows = (long)max_new * group, keys = window ? std::min((long)max_len, (long)window + max_new) : max_len;
  const bool equal = (long)n_seqs * max_new == n_tokens;               // all sequences bring max_new tokens
  AttnPlan p = {};
  if (few_of_tree || rows <= 64 || (long)n_tokens * group * kv_heads * keys <= (equal && head_dim == 128 ? kFewScoresEqual : kFewScores)) {
    const auto units_of = [&](int mb) { return (n_tokens / std::max(16 * mb / group, 1) + n_seqs) * (long)kv_heads; };
    p.mb = rows <= 16 ? 1 : group <= 32 ? 2 : 4;
    // Chunks with heads of 64: 64 rows a block instead of 32, which takes 1.45 times as long, where that saves rounds of a block on
    // each CU (500 tokens and 7 single ones, 4 heads: 15.6 and 17.4 us; 600 of 8 sequences and 56: 31 and 44; 500 of 12 heads: 20.4
    // and 16.9).  With heads of 128 there is no second block on a CU then, and 32 rows are faster throughout.
    if (!few_of_tree && head_dim == 64 && rows > 64 && p.mb == 2 && (units_of(4) + 255) / 256 * 145 < (units_of(2) + 255) / 256 * 100) p.mb = 4;
    p.most = max_new;
    const long units = units_of(p.mb), room = 256 * blocks_of(head_dim, p.mb), kt = tile_keys(head_dim, p.mb), tiles = (keys + kt - 1) / kt;
    p.waves = blocks_of(head_dim, p.mb) == 2 && units <= 256 && tiles * kt > 512 ? 8 : 4;
    const long whole = (units + room - 1) / room * ((tiles + p.waves - 1) / p.waves), shared = units * tiles * 6 / (10 * kSplitW * room);
    const bool split = (max_new * group <= 16 * p.mb ? keys * head_dim > (units <= 32 ? kSplitKeys / 2 : kSplitKeys) : whole - shared > kSplitGain * 64 / kt) && units * (tiles + 2) < 1l << 30;
    if (split) p.blocks = split_blocks(head_dim, p.mb, units);
  } else {
    p.chunks = true;
    p.chunk = plan_of_chunks(n_tokens, kv_heads, group, max_new, keys, head_dim);
    if (p.chunk.splits > 1) p.chunk_parts = (size_t)p.chunk.splits * n_tokens * kv_heads * group * (head_dim + 2) * sizeof(float);
    if (!equal && group <= 16 && n_seqs * (long)kv_heads * ((keys >> 5) + 2) < 1l << 30) {    // there may be sequences of few rows
      p.mb = 1;
      p.blocks = split_blocks(head_dim, 1, n_seqs * (long)kv_heads);
      p.most = 16 / group;
    }
  }
  if (p.blocks) p.parts = parts_of(p.blocks, std::min(16 * p.mb / group, max_new) * group, head_dim);
  return p;
}

// ---- trees of drafted tokens ----
// Up to kTreeFew rows a key / value head the few-rows kernel takes them in one tile of rows, and up to twice that in two where the keys
// are few: the many-rows kernel has 20 us before and behind its turns, if its keys are shared out.  In us, 32 heads over 8 of 128: 16
// tokens over 8192 keys 23 (few rows) and 30; 16 trees of up to 12 over up to 4096 56 and 49, 64 of up to 13 over up to 2048 109 and 99.
// So are more rows where the step has few scores (kTreeScores, as for chunks): 32 tokens over 600 keys, 28 heads over 4, 12 (few rows)
// and 23.5; 64 x 32 over 600, 8 heads over 1 of 64 (10 M), 26 and 20.  Not everywhere is that border the best: 500 tokens over 1500 keys,
// 12 heads of 64 (9 M), would take 18 and take 44; 300 over 2000, 16 of 128, 29 and 37.
// The rest is walked by blocks of kTreeRows, whole, or their keys shared out over kTreeBlocks (two on a CU; 256 took 73 us for 68, 198
// for 161; one tree of 128 tokens over 30000 keys, 32 heads over 1, shared 113 and whole 725), whichever a count of the turns says is sooner,
// a turn being 2 us, 1.75 with heads of 64, and three quarters where most CUs have one block; whole where blocks come in many rounds anyway.
// Of 44 steps about that border 38 get the sooner one, or one within 10 %, and six take 1.15 to 1.47 times as long; with the 1.24 us that a turn
// had with one product of the probabilities it was ten (16 x 48 tokens over 1350 keys, 16 heads of 64: shared 31 us, whole 43).
// Two things that the count leaves out: what a plane has of rows (33 tokens, 32 heads over 8, are one plane of 128 rows and one of 4, with half
// of the blocks each: 65 us over 30000 keys, and 32 tokens 52), and the parts' bytes (512 over 4000 keys: 95 us, of which it expects 51).
constexpr int kTreeFew = 32, kTreeRows = 128, kTreeBlocks = 512, kTreeLeast = 6, kTreeTurns = 2048;
constexpr long kTreeScores = 8l << 20;
inline int tree_planes(int max_new, int group) { return (max_new + kTreeRows / group - 1) / (kTreeRows / group); }
// Blocks that share the keys, of each plane: eights, which go to the XCDs by turns, where there are as many
inline int tree_shares(int planes) { return kTreeBlocks / planes < 8 ? kTreeBlocks / planes : kTreeBlocks / planes & ~7; }
inline AttnPlan plan_of_tree(int n_seqs, int n_tokens, int kv_heads, int group, int max_new, int max_len, int window, int head_dim) {
  const long rows = (long)max_new * group, keys = window ? std::min((long)max_len, (long)window + max_new) : max_len, tiles = (keys + PF_K - 1) / PF_K;
  const long turns = (long)n_seqs * kv_heads * tiles * (n_seqs == 1 ? 10 : 7) / 10;    // sequences of 0.7 of the longest on average
  const long scores = (long)n_tokens * group * kv_heads * keys;
  if (group <= kTreeFew && (rows <= kTreeFew || (rows <= 2 * kTreeFew && turns < kTreeTurns) || scores <= kTreeScores))
    return plan_of(n_seqs, n_tokens, kv_heads, group, max_new, max_len, window, head_dim, true);
  AttnPlan p = {};
  p.most = max_new;
  const int planes = tree_planes(max_new, group), shares = tree_shares(planes);
  const long units = (n_tokens / (kTreeRows / group) + n_seqs) * (long)kv_heads;
  const double turn = head_dim == 128 ? 2.0 : 1.75;
  const double whole = (double)((units + kTreeBlocks - 1) / kTreeBlocks * tiles) * turn * (units <= 256 ? 0.75 : 1.0);
  const double shared = shares ? std::max((double)turns / shares, (double)kTreeLeast) * turn + 20.0 : 1e30;
  if (shares > 1 && units < 8 * kTreeBlocks && shared < whole && (long)n_seqs * kv_heads * (tiles + 2) < 1l << 30) {
    p.blocks = shares;
    p.parts = parts_of(shares * planes, std::min(kTreeRows / group, max_new) * group, head_dim);
  }
  return p;
}

}  // namespace sna
