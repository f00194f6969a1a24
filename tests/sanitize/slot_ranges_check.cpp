// Reads P, D and D + 1 offsets and D experts (-1: none), prints first, rows and expert of every slot and the tile bound.
#include <cstdio>
#include <vector>

#include "slot_ranges.h"

int main()
{
    long long P;
    int D;
    while (std::scanf("%lld %d", &P, &D) == 2) {
        std::vector<unsigned> offsets(D + 1);
        std::vector<int32_t> first(D), rows(D), expert(D);
        for (unsigned& o : offsets)
            if (std::scanf("%u", &o) != 1) return 1;
        for (int32_t& e : expert)
            if (std::scanf("%d", &e) != 1) return 1;
        const auto clamp = [P](unsigned o) { return static_cast<int32_t>(o < P ? o : P); };
        for (int d = 0; d < D; ++d) {
            first[d] = clamp(offsets[d]);
            const int32_t end = clamp(offsets[d + 1]);
            rows[d] = end > first[d] && expert[d] >= 0 ? end - first[d] : 0;
            if (rows[d] == 0) expert[d] = -1;
        }
        cobalt::make_slots_disjoint(D, clamp(offsets[D]), first.data(), rows.data(), expert.data());
        std::printf("%lld", static_cast<long long>(cobalt::most_row_tiles(P, D, 256)));
        for (int d = 0; d < D; ++d) std::printf(" %d %d %d", first[d], rows[d], expert[d]);
        std::printf("\n");
    }
    return 0;
}
