// Which kernel computes an 8-bit product.  Plain C++ with no HIP, so that the
// tests can ask on the host which kernels their shapes reach.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace bmlp {

// Which kernel.  Up to 32 rows the weights' bytes count and the direct kernel
// streams them (us; 16 rows, 8192 x 8192: 12.6 in 32 x 32 tiles, 13.3 in 16 x 16
// ones, 26 through LDS; 4096 x 4096, where 16 x 16 tiles find every compute unit: 7.3 and
// 7.8, 14.4).  Above, the tile whose rounds over the 256 compute units cost
// least: 256 x 256 tiles run the matrix cores at their highest rate, smaller
// ones find more compute units.  Measured, us, 256 x 256 / 128 x 256 / 128 x 128
// / 64 x 128 / 64 x 64: 4096 x 4096 x 4096 66, 70, 82, 103, 114; 2048 x 4096 x 4096
// 44, 36, 42, 52, 57; 1024 x 4096 x 4096 42, 25, 22, 26, 31; 512 x 4096 x 4096 41,
// 24, 19, 14.5, 17.4; 256 x 4096 x 4096 41, 24, 18, 13, 10; 8192 x 1024 x 1024 20,
// 14.5, 18, 22, 22; 3000 x 8192 x 3000 82, 103, 104, 114, 130.
enum QLinearKernel { kTile256x256, kTile128x256, kTile128x128, kTile64x128, kTile64x64, kDirect16, kDirect32 };
struct TileCost {
  int rows, cols, units;   // units: tiles that run at a time
  int full, least;         // ns per step of 64 inputs: all units busy (the clock falls then), and few of them
};
constexpr TileCost kTileCost[5] = {   // in the enumeration's order
    {256, 256, 256, 1000, 640}, {128, 256, 256, 560, 385}, {128, 128, 256, 344, 295}, {64, 128, 256, 226, 200}, {64, 64, 512, 270, 145}};
inline QLinearKernel best_tile(int n, int N) {
  int best = 0;
  int64_t lowest = INT64_MAX;
  for (int i = 0; i < 5; ++i) {
    const TileCost &c = kTileCost[i];
    const int64_t t = (int64_t)((n - 1) / c.rows + 1) * ((N - 1) / c.cols + 1), rest = t % c.units;
    const int64_t cost = t / c.units * c.full + (rest ? std::max((int64_t)c.least, c.full * rest / c.units) : 0);
    if (cost < lowest) {
      lowest = cost;
      best = i;
    }
  }
  return (QLinearKernel)best;
}
// ldq: elements from one row of q to the next
inline QLinearKernel qlinear_kernel(int n, int N, int64_t ldq) {
  if (n <= 16 && N < 8192) return kDirect16;
  // (rows too far apart for a tile's 32-bit offsets: the direct kernel's are 64)
  if (n <= 32 || ldq > 1 << 21) return kDirect32;
  return best_tile(n, N);
}

// Rows of q that do not start (or, for the last one, end) at 16-byte boundaries.
inline bool qlinear_ragged(uintptr_t q, int n, int64_t ldq, int K) {
  return ((q | (n > 1 ? (uintptr_t)ldq : 0) | (uintptr_t)K) & 15) != 0;
}

}  // namespace bmlp
