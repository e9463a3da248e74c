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

// How columns c .. c + 7 are loaded: not at all where the row has none of them; element by element where the row is the
// matrix's first or last (`end`) and the group reaches out of it; else whole, neighbouring rows' elements with them.
enum class Load { none, elements, whole };

ASPIS_BOTH Load load_of(int c, Columns row, bool end)
{
    if (c + 8 <= row.lo || c >= row.hi) return Load::none;
    return !end || (c >= row.lo && c + 8 <= row.hi) ? Load::whole : Load::elements;
}

}  // namespace aspis
