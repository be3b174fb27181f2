// Where a token of a paged cache lies.  Plain C++, so that the walk through a
// table is checked on the host too.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#define IM2WIN_BOTH __host__ __device__
#else
#define IM2WIN_BOTH
#endif

namespace im2win {

// Position `pos` of a sequence whose table row is `row`: page row[index], place
// `within` it, index = pos / page and within = pos % page.  -1 for positions
// outside 0 .. max_pages*page - 1 and for entries that name no page of the
// pool: nothing is read or written there.
IM2WIN_BOTH inline int32_t page_of(const int32_t *row, int64_t index, int64_t max_pages, int64_t pages)
{
    if (index < 0 || index >= max_pages)
        return -1;
    const int32_t id = row[index];
    return id >= 0 && id < pages ? id : -1;
}

// Tokens of a sequence that its table can hold, of the `n` that the caller names.
IM2WIN_BOTH inline int32_t held_tokens(int32_t n, int64_t max_pages, int64_t page)
{
    const int64_t most = max_pages * page;
    return n < 0 ? 0 : n < most ? n : (int32_t)most;
}

}  // namespace im2win
