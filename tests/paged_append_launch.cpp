// Prints the rows of a tile and the units of a workgroup that ll_paged_append takes for: rows, units, rows of a whole tile.
#include <cstdio>
#include <cstdlib>

#include "../paper_2509_22622_amd/csrc/paged.h"

int main(int argc, char** argv) {
    if (argc != 4) return 1;
    const int tokens = std::atoi(argv[1]), units = std::atoi(argv[2]), rows = ll::paged_tile_rows(tokens, units, std::atoi(argv[3]));
    std::printf("%d %d\n", rows, ll::paged_units_per_group((tokens + rows - 1) / rows, units));
    return 0;
}
