// eql_slices.h -- calls over more workgroups than a launch takes: the slices that they are cut into, and the sequence that a
// workgroup of a slice works on.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace eqk {

// Numbers of workgroups from a slice's first sequence on stay below 2^31.
constexpr int64_t kSliceReach = ((int64_t)1 << 31) - 1;

// go(a sequence, a workgroup from it on, workgroups) for each launch of a call of `seqs` sequences of `per` workgroups, at most
// `most` a launch, as long as it gives true; `per` is at most `reach`.
template <typename F>
void slices(int64_t seqs, int64_t per, int64_t most, int64_t reach, F&& go) {
  const int64_t step = reach / per;
  for (int64_t seq = 0; seq < seqs; seq += step) {
    const int64_t n = (seqs - seq < step ? seqs - seq : step) * per;
    for (int64_t first = 0; first < n; first += most)
      if (!go(seq, (unsigned)first, (unsigned)(n - first < most ? n - first : most))) return;
  }
}

// Sequence of workgroup `block` of such a launch, and its number among the sequence's.
struct SlicePlace {
  int64_t seq;
  unsigned at;
};
__host__ __device__ __forceinline__ SlicePlace slice_place(int64_t seq, unsigned first, unsigned block, unsigned per) {
  const unsigned id = first + block;
  return {seq + id / per, id % per};
}

}  // namespace eqk
