// How the packed weight gradient cuts a group's rows into chunks: at most `most` of them (a multiple of `unit`) in each,
// equally long but for the last, in whole units; a group without rows has one empty chunk.  Plain arithmetic that the
// host can run as well.
#pragma once

namespace janus {

struct ChunkCut {
  int each, count;   // rows of a chunk, chunks
};
__host__ __device__ inline ChunkCut chunk_cut(int rows, int most, int unit) {
  const unsigned size = rows, n = (size + most - 1) / most;   // unsigned: rows up to 2^31 - 1 and a chunk more
  if (n == 0) return ChunkCut{0, 1};
  const unsigned each = ((size + n - 1) / n + unit - 1) / unit * unit;
  return ChunkCut{(int)each, (int)((size + each - 1) / each)};
}

}  // namespace janus
