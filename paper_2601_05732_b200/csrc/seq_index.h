// Token indices of the sequences' losses are 32-bit and T may be as large as 2^31 - 257, so an index that lies a few steps behind
// the last token need not be one: what is asked of it is asked of differences, which stay between 0 and T.
#pragma once

#ifdef __CUDACC__
#define MHCL_INDEX __host__ __device__ constexpr
#else
#define MHCL_INDEX constexpr
#endif

namespace mhcl {

// Whether token base + ahead lies before `end` (0 <= base <= end, 0 <= ahead).
MHCL_INDEX bool seq_before(int base, int ahead, int end) { return ahead < end - base; }
// Whether all of the n tokens from lo on are there (0 <= lo <= T).
MHCL_INDEX bool seq_whole(int lo, int n, int T) { return T - lo >= n; }

}  // namespace mhcl
