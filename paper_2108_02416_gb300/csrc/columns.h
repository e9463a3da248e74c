// Which columns of a row a lane may load, as plain C++.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define ASPIS_BOTH __host__ __device__ __forceinline__
#else
#define ASPIS_BOTH inline
#endif

namespace aspis {

// The columns lo .. hi - 1 that a row has, counted from the first one of a share of it (`first`, which lies up to seven before the row's
// own where a share begins at a group's boundary).  Eight before a share are as many as anything needs, `most` behind.
struct Columns {
    int lo, hi;
};

ASPIS_BOTH Columns columns_from(int64_t first, int64_t cols, int most)
{
    return {first > 0 ? -8 : (int)-first, (int)(cols - first < most ? cols - first : most)};
}

// How columns c .. c + 7 are loaded: not at all where the row has none of them; whole, neighbouring rows' elements with them, where
// no element of the group lies outside the matrix, as it may where the row is the first or last (`end`); else element by
// element.  (Two conditions: as an enumeration of three the unaligned dropout of 20,001 x 1001 took 30.0 us, 28.8 so.)
ASPIS_BOTH bool load_nothing(int c, Columns row) { return c + 8 <= row.lo || c >= row.hi; }
ASPIS_BOTH bool load_whole(int c, Columns row, bool end) { return !end || (c >= row.lo && c + 8 <= row.hi); }

}  // namespace aspis
