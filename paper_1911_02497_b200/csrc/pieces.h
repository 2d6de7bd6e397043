// Which aligned 16 bytes hold the values of a row of 16-bit values that begins anywhere. Plain arithmetic, for host and device.
#pragma once

#ifdef __CUDACC__
#define CS_BOTH __host__ __device__ __forceinline__
#else
#define CS_BOTH inline
#endif

namespace cs {

constexpr int PIECE = 8;                // values of 16 bytes

// Whether the values c .. c+7 of a row of `cols`, c < cols, reach into a second piece, where value c lies `by` values behind the start of the
// first. A piece without a value of the row may lie between two rows, where there need be no memory: it is not loaded.
CS_BOTH bool second_piece(int by, int c, int cols) { return by > 0 && c - by + PIECE < cols; }

}  // namespace cs
