// The line of tiles that the decoding kernels share out: the tiles of all sequences of all KV heads, head after head and
// sequence after sequence.  Block i of nb takes the tiles [i*T/nb, (i+1)*T/nb), whatever the sequences' lengths are.
#pragma once
#include <cuda_runtime.h>

namespace line {

// (32-bit division where the product fits: a 64-bit one costs some hundred cycles before the first load.)
__device__ __forceinline__ long long muldiv(long long a, int m, long long d) {
  const unsigned long long x = (unsigned long long)a * (unsigned)m;
  return (x >> 32) == 0 && ((unsigned long long)d >> 32) == 0 ? (long long)((unsigned)x / (unsigned)d) : (long long)(x / (unsigned long long)d);
}
__device__ __forceinline__ long long share_start(int i, long long T, int nb) { return muldiv(T, i, nb); }
__device__ __forceinline__ int share_of(long long t, long long T, int nb) {
  const unsigned long long x = (unsigned long long)(t + 1) * (unsigned)nb - 1;
  return (x >> 32) == 0 && ((unsigned long long)T >> 32) == 0 ? (int)((unsigned)x / (unsigned)T) : (int)(x / (unsigned long long)T);
}

// A block's share of the line: tiles [lo, hi), the first of them in sequence b of head h, whose tiles start at `line`.
struct Share {
  long long lo, hi, line, line_len;
  int h, b, nb;                                // nb: blocks that have tiles
};
// Tiles of all sequences, 32 at a time, in every warp for itself (no barrier before the first load): the sum, then
// the sequence that holds the first tile of this block's share.  tiles(i): tiles of sequence i.
template <typename F>
__device__ __forceinline__ Share find_share(int B, int H, int blocks, int blk, int lane, F tiles) {
  Share r;
  auto tiles_of = [&](int i) { return i < B ? tiles(i) : 0; };
  const int first32 = tiles_of(lane);
  long long total = __reduce_add_sync(0xffffffffu, first32);
  for (int b0 = 32; b0 < B; b0 += 32) total += __reduce_add_sync(0xffffffffu, tiles_of(b0 + lane));
  r.line_len = total * H;                      // every head has the same tiles
  r.nb = r.line_len < blocks ? (int)r.line_len : blocks;
  r.lo = blk < r.nb ? share_start(blk, r.line_len, r.nb) : 0;
  r.hi = blk < r.nb ? share_start(blk + 1, r.line_len, r.nb) : 0;
  r.h = r.lo > 0 ? (int)muldiv(r.lo, 1, total) : 0;
  const long long lo_head = r.lo - r.h * total;              // within the head
  r.b = 0;
  r.line = 0;
  long long at = 0;
  for (int b0 = 0; b0 < B; b0 += 32) {
    const int mine = b0 == 0 ? first32 : tiles_of(b0 + lane);
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    const unsigned past = __ballot_sync(0xffffffffu, at + incl > lo_head);
    if (past) {
      const int first = __ffs(past) - 1;
      r.b = b0 + first;
      r.line = r.h * total + at + __shfl_sync(0xffffffffu, incl - mine, first);
      break;
    }
    at += __shfl_sync(0xffffffffu, incl, 31);
  }
  return r;
}

}  // namespace line
