// Packed documents on the device: which document a row, or a block of rows,
// belongs to.  starts[0 .. n_seqs] is read as it is on every call; values outside
// [0, tokens] are clamped, so that no access leaves the arrays whatever it holds.
#pragma once
#include "kernels.h"

namespace l4d {

__device__ __forceinline__ int seq_start(const Packing& p, int i) {
  const int64_t v = p.starts[i];
  return static_cast<int>(v < 0 ? 0 : v > p.tokens ? p.tokens : v);
}

// The last i in [0, n_seqs) with key(i) <= x, or -1; key is nondecreasing.  The
// lanes of a wave probe 64 places at once: one load latency up to 64 documents,
// two up to 4096.  Every lane must call it; the result is the same in all.
template <class Key>
__device__ __forceinline__ int last_not_above(int n_seqs, int x, int lane, Key key) {
  int base = 0, len = n_seqs, found = -1;
  while (len > 0) {
    const int step = (len + 63) / 64, i = base + lane * step;
    const bool le = lane * step < len && key(i) <= x;
    const int c = __builtin_popcountll(__builtin_amdgcn_ballot_w64(le));
    if (c == 0) break;
    found = base + (c - 1) * step;          // key(found) <= x: the rest of its stride is left to search
    len = min(step, len - (c - 1) * step) - 1;
    base = found + 1;
  }
  return __builtin_amdgcn_readfirstlane(found);
}

struct SeqRows {
  int lo, hi;      // the document's rows; lo == hi: none
  int i;           // its index, -1: none
};
// The last document i with key(starts[i], i) <= x, key nondecreasing in i.  Up to 63
// documents one load brings all starts, and the lanes that hold its rows hand them out.
template <class Key>
__device__ __forceinline__ SeqRows last_seq(const Packing& p, int x, int lane, Key key) {
  if (p.n_seqs < 64) {
    const int v = seq_start(p, min(lane, p.n_seqs));
    const int c = __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < p.n_seqs && key(v, lane) <= x));
    if (c == 0) return SeqRows{0, 0, -1};
    const int lo = __builtin_amdgcn_readlane(v, c - 1), hi = __builtin_amdgcn_readlane(v, c);
    return SeqRows{lo, max(lo, hi), c - 1};
  }
  const int i = last_not_above(p.n_seqs, x, lane, [&](int j) { return key(seq_start(p, j), j); });
  if (i < 0) return SeqRows{0, 0, -1};
  const int lo = __builtin_amdgcn_readfirstlane(seq_start(p, i)), hi = __builtin_amdgcn_readfirstlane(seq_start(p, i + 1));
  return SeqRows{lo, max(lo, hi), i};
}
// The document of a row; hi <= row: none.
__device__ __forceinline__ SeqRows seq_of_row(const Packing& p, int row, int lane) {
  return last_seq(p, row, lane, [](int v, int) { return v; });
}

// Blocks of `rows` rows that never cross a document: document i owns the slots
// from starts[i]/rows + i on.  It has ceil(len/rows) blocks and the next one's
// first slot is floor((start + len)/rows) - floor(start/rows) + 1 >= ceil(len/rows)
// further, so slots never meet, and a block finds its place without a table:
// tokens/rows + n_seqs slots cover every packing, the unused ones return at once.
struct SeqBlock {
  int lo, hi;      // the document's rows
  int row0;        // the block's first row; hi <= row0: no block in this slot
};
__device__ __forceinline__ SeqBlock seq_block(const Packing& p, int slot, int rows, int lane) {
  const SeqRows s = last_seq(p, slot, lane, [rows](int v, int j) { return v / rows + j; });
  if (s.i < 0) return SeqBlock{0, 0, 0};
  const int t = slot - (s.lo / rows + s.i);
  if (t >= (s.hi - s.lo + rows - 1) / rows) return SeqBlock{0, 0, 0};
  return SeqBlock{s.lo, s.hi, s.lo + t * rows};
}

__device__ __forceinline__ int wave_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);      // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // row_bcast 15, 31
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return __builtin_amdgcn_readlane(x, 63);
}
// The block of rank `rank` when the blocks of up to 63 documents stand by their place in
// the document, the last places first.  sum_i max(n_i - t, 0) of them, n_i the blocks of
// document i, stand at place t or behind it: a search over t.
__device__ __forceinline__ SeqBlock ranked_block(const Packing& p, int rank, int rows, int lane) {
  const int v = seq_start(p, min(lane, p.n_seqs)), next = __shfl_down(v, 1, 64);
  const int n = lane < p.n_seqs ? (max(next - v, 0) + rows - 1) / rows : 0;
  if (wave_sum(n) <= rank) return SeqBlock{0, 0, 0};
  int t = 0;
  for (int step = 1 << (31 - __builtin_clz(p.tokens / rows + 1)); step > 0; step /= 2)
    if (wave_sum(max(n - t - step, 0)) > rank) t += step;
  const uint64_t at = __builtin_amdgcn_ballot_w64(n > t);
  const int before = __builtin_popcountll(at & ((uint64_t{1} << lane) - 1)), k = rank - wave_sum(max(n - t - 1, 0));
  const int i = __builtin_ctzll(__builtin_amdgcn_ballot_w64(n > t && before == k) | uint64_t{1} << 62);
  const int lo = __builtin_amdgcn_readlane(v, i), hi = __builtin_amdgcn_readlane(v, i + 1);
  return SeqBlock{lo, max(lo, hi), lo + t * rows};
}

// The block of 128 rows that holds `row`.
__device__ __forceinline__ SeqBlock block_at(const Packing& p, int row, int lane) {
  const SeqRows s = seq_of_row(p, row, lane);
  return row < s.hi ? SeqBlock{s.lo, s.hi, s.lo + (row - s.lo) / 128 * 128} : SeqBlock{0, 0, 0};
}

}  // namespace l4d
