// Who waits for whom where the chunk kernel's row tiles hand probabilities to the tensor core.
#pragma once

namespace lv {

// Whether the issuer of a row tile waits for the probabilities of stream `other` before it issues stream `c`'s product with V of a
// piece's j-th key tile.  For the stream's own always.  Before the piece's first product for both: that product writes over the columns
// of O in which a row's two threads tell each other their maxima, and only their probabilities say that both have read them.
#ifdef __CUDACC__
__host__ __device__
#endif
constexpr bool kv_awaits(int j, int c, int other) { return other == c || (j == 0 && c == 0); }

}  // namespace lv
