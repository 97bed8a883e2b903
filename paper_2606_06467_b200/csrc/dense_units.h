// Where a unit of the dense attention (a sequence's rows for the KV heads of a block) lies in the list's stretches: what its fetching warps note
// and the joining kernel reads. Plain C++, so that the host can check it too.
#pragma once
#ifdef __CUDACC__
#define CLSA_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define CLSA_HOST_DEVICE inline
#endif

namespace clsa {

enum class Noted { kWhole, kCut, kNever };  // in one stretch, which finished it; in several, to be joined; not written by the launch before

// begin: 2 x the first stretch + whether another unit is in front of this one there; last: the last stretch. The scratch that they lie in is not
// cleared: where a launch gave up, they may be anything. Only what kCut comes with may be used as numbers of records, of which there are `spans`.
CLSA_HOST_DEVICE Noted noted_unit(int begin, int last, int spans) {
  if (begin < 0 || last < begin >> 1 || last >= spans) return Noted::kNever;
  return last > begin >> 1 ? Noted::kCut : Noted::kWhole;
}

}  // namespace clsa
