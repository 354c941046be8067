// Tiles of the gated projection's three products: for M, D, F and 1 phase or 6, side, rows and columns of tiles and splits of each.
#include <cstdio>
#include <initializer_list>

#include "gated_plan.hpp"

int main()
{
    long M, D, F;
    int phases;
    while (scanf("%ld %ld %ld %d", &M, &D, &F, &phases) == 4)
        for (const auto &s : {ucd::gated::forward_shape(M, D, F, phases), ucd::gated::dx_shape(M, D, F, phases), ucd::gated::dw_shape(M, D, F, phases)})
            printf("%d %d %d %d\n", s.side, s.tiles_m, s.tiles_n, s.splits);
    return 0;
}
