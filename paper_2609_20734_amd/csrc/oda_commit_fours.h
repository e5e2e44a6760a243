// How the tokens of one request's commit fall into aligned fours of slots
// (commit.hip, the values of oda_commit_drafts).  Used by the kernel and, without
// a GPU, by its test: nothing here is HIP's but the function qualifiers.
#ifndef ODA_COMMIT_FOURS_H_
#define ODA_COMMIT_FOURS_H_

#include <stdint.h>

#if defined(__HIPCC__)
#define ODA_FOURS_FN __host__ __device__ __forceinline__
#else
#define ODA_FOURS_FN inline
#endif

namespace oda {

// The token in the first slot of the first four, of `count` tokens whose first
// goes to position pos0: 0 to -3; 0 where there are none, so that no four (each
// reads at least one token) comes before the count.
ODA_FOURS_FN int first_four(int64_t pos0, int count) { return count > 0 ? -(int)(pos0 & 3) : 0; }

// The token that slot k of the four at t0 < count is read from: its own, or the
// nearest one where the slot holds none (its value is not stored).
ODA_FOURS_FN int token_read(int t0, int k, int count) {
  const int t = t0 + k < 0 ? 0 : t0 + k;
  return t < count ? t : count - 1;
}

}  // namespace oda

#endif  // ODA_COMMIT_FOURS_H_
