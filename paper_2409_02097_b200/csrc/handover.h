// The word by which one block tells another that the sums of a cut tile are there, also where the other no longer waits for them.
//
// A flag is `mark` while sums wait to be fetched.  The marks of different calls differ, but a captured call has the same one every time it
// is replayed, so whatever happens no flag may be left up: whoever fetches takes it down; one whose wait has expired leaves the mark's
// even neighbour instead, and of the two, who come in either order, the second puts the flag down.
//
// exchange(v): v into the flag, what it held back, in one step.
#pragma once

#ifdef __CUDACC__
#define LF_HANDOVER __device__ __forceinline__
#else
#define LF_HANDOVER inline
#endif

namespace lf {

typedef unsigned long long Handover;  // a mark is odd

LF_HANDOVER Handover handover_gone(Handover mark) { return mark ^ 1ull; }

// The sums are there.
template <typename Exchange>
LF_HANDOVER void handover_raise(const Exchange& exchange, Handover mark)
{
    if (exchange(mark) == handover_gone(mark)) exchange(0ull);
}
// Nobody will fetch them.
template <typename Exchange>
LF_HANDOVER void handover_leave(const Exchange& exchange, Handover mark)
{
    if (exchange(handover_gone(mark)) == mark) exchange(0ull);
}

}  // namespace lf
