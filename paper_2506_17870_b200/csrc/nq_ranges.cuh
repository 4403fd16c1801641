// Integer arithmetic of the attention kernels at the ends of what they accept, where 32 bits are short.  Plain C++ too: a test compiles it
// by itself and goes to sizes that no GPU has room for.
#pragma once

#ifdef __CUDACC__
#define NQ_BOTH __host__ __device__ __forceinline__
#else
#define NQ_BOTH inline
#endif

namespace nq {

// The first of `reach` keys that a window of the last `window` of them leaves (0: no window).  `reach` is as low as minus the number of
// queries where a sequence has fewer keys than those, and a window may be 2^31 - 1: their difference is taken only where it is positive.
NQ_BOTH int window_start(int window, int reach) { return window > 0 && reach > window ? reach - window : 0; }

}  // namespace nq
