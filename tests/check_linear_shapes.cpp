// Which block of outputs a linear layer's sizes select (csrc/linear.h), over their whole range.  Exit status 0 = all hold.
#include <cstdio>
#include <set>

#include "../paper_2509_22622_amd/csrc/linear.h"

int main() {
    std::set<int> seen;
    for (int m : {1, 2, 16, 17, 32, 33, 48, 49, 63, 64, 65, 100, 127, 128, 200, 255, 256, 257, 500, 1000, 2400, 4680, 8192, 100000, 1 << 24})
        for (int n : {1, 16, 33, 64, 300, 512, 1536, 2000, 4096, 6144, 8192, 65536, 1 << 20})
            for (int k : {8, 64, 72, 512, 1024, 1536, 4096, 6144, 65536, 1 << 20}) {
                const int i = ll::linear_choose(m, n, k);
                const ll::LinearShape& s = ll::LINEAR_SHAPES[i];
                if (m < (i >= ll::LINEAR_FEW ? s.rows : s.rows - 15)) {
                    std::printf("%d x %d x %d: a tile of %d rows\n", m, n, k, s.rows);
                    return 1;
                }
                if (m <= 1 << 20 && n <= 1 << 16 && ll::linear_blocks(s, m, n) > ll::LINEAR_MAX_BLOCKS - 7) {
                    std::printf("%d x %d x %d: %lld workgroups\n", m, n, k, static_cast<long long>(ll::linear_blocks(s, m, n)));
                    return 1;
                }
                seen.insert(i);
            }
    const int shapes = int(sizeof(ll::LINEAR_SHAPES) / sizeof(ll::LINEAR_SHAPES[0]));
    for (int i = 0; i < shapes; ++i)
        if (!seen.count(i)) {
            std::printf("nothing selects %d x %d\n", ll::LINEAR_SHAPES[i].rows, ll::LINEAR_SHAPES[i].cols);
            return 1;
        }
    std::printf("linear shapes ok\n");
    return 0;
}
