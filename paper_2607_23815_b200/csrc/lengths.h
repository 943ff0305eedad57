// Pages of so many tokens.  A length has 31 bits (its sums with a page's size have not), so they are formed without a sign.
#pragma once

namespace kvattn {

#ifdef __CUDACC__
#define KVATTN_BOTH __host__ __device__ __forceinline__
#else
#define KVATTN_BOTH inline
#endif

constexpr int kPageSize = 16;

KVATTN_BOTH int pages_of(int tokens) { return (int)(((unsigned)tokens + (kPageSize - 1)) / kPageSize); }  // (tokens: 0 or more)

}  // namespace kvattn
