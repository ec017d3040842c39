// How the blocks of a grid share a long array: block b of `blocks` takes the pieces b, b + blocks, b + 2 blocks ..
// Device code and plain C++ alike, so that the arithmetic can be run on the host at lengths that are not launched.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define GNNCO_BOTH __host__ __device__ __forceinline__
#else
#define GNNCO_BOTH inline
#endif

// for (PieceWalk w(count, block, blocks, piece); w.more(); w.next()) ... elements w.at .. w.at + piece - 1 that are below w.count
// (64 bits: a walk ends past its length by up to blocks * piece, which leaves 32 bits where the length nearly fills them)
struct PieceWalk {
  int64_t count, at, step;
  GNNCO_BOTH PieceWalk(int64_t count_, int64_t block, int64_t blocks, int64_t piece)
      : count(count_), at(block * piece), step(blocks * piece) {}
  GNNCO_BOTH bool more() const { return at < count; }
  GNNCO_BOTH void next() { at += step; }
};
