// Threads per row of the kernels that walk rows of vectors, 256 threads to a block.
#pragma once
#include <stdint.h>

namespace asx {

// log2 of them: one per vector up to a block's 256, and fewer where those of all rows would be more than 2^31, since a launch takes
// less than 2^32 along a dimension (2^24 rows of 256; what a caller adds in further blocks has the other half).
inline int row_threads_log(int64_t rows, int64_t vecs) {
  int b = 0;
  while (b < 8 && ((int64_t)1 << b) < vecs && rows << (b + 1) <= (int64_t)1 << 31) ++b;
  return b;
}

}  // namespace asx
