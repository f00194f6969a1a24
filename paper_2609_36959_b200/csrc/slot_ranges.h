// The rows of the slots when dest_offsets are not in order (also compiled by a host compiler).
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define COBALT_HOST_DEVICE __host__ __device__
#else
#define COBALT_HOST_DEVICE
#endif

namespace cobalt {

// Row tiles of at most `tile` rows that slots of P rows in all can need: holds for disjoint ranges only.
COBALT_HOST_DEVICE inline int64_t most_row_tiles(int64_t P, int D, int tile) { return P / tile + D; }

// Offsets that decrease are read as their running maximum m: slot d gets rows m[d] .. m[d + 1], so that no row belongs to
// two slots.  In: first[d] = min(offsets[d], P), last_end = min(offsets[D], P), rows[d] what the two offsets of slot d give
// by themselves (0 for a slot whose rows are skipped), expert[d].  Out: first and rows by m, expert -1 where no rows are left.
COBALT_HOST_DEVICE inline void make_slots_disjoint(int D, int32_t last_end, int32_t* first, int32_t* rows, int32_t* expert)
{
    int32_t taken = first[0];
    for (int d = 0; d < D; ++d) {
        const int32_t end = d + 1 < D ? first[d + 1] : last_end, left = end > taken ? end - taken : 0;
        first[d] = taken;
        if (rows[d] > left) rows[d] = left;
        if (rows[d] == 0) expert[d] = -1;
        if (end > taken) taken = end;
    }
}

}  // namespace cobalt
