// Copies of blocks inside a pool (kvr_pages.cu).
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

namespace kvr {

// A pool as the copies see it: tiles of block_size rows, one for each block and plane.
struct PoolView {
  char *base;
  long long plane_stride, block_stride;
  int planes, num_blocks, block_size, row_bytes;
};

// Pairs (source, destination) that go to the kernel by value: nothing is uploaded or kept, whatever the stream does meanwhile.
constexpr int kInlinePairs = 1024;
struct InlinePairs {
  int2 pair[kInlinePairs];
};

// The first `rows` tokens of each pair's source to its destination, in all planes.  The pairs have been checked by the caller; their destinations
// are distinct and no sources.
cudaError_t copy_blocks(const PoolView &v, const int2 *pairs, int n, int rows, cudaStream_t s);

}  // namespace kvr
