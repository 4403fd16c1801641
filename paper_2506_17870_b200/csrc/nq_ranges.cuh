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

// Whether group `n` of 16 tokens has any of a sequence's `length`, for groups that may lie behind all that a table can name (whose
// first token's number, 16 n, does not fit 32 bits).
NQ_BOTH bool group_in(int n, int length) { return length > 0 && n <= (length - 1) >> 4; }

// How long (SM cycles) to wait for something that comes only when another role is through with `steps` steps of its own, where one step's limit
// is `one`: 2^14 cycles for each beside it, ten times what a step of the prompt kernel takes (some 1650).
NQ_BOTH long long wait_limit(long long one, int steps) { return steps > 0 ? one + ((long long)steps << 14) : one; }

}  // namespace nq
