// Whether tensors share memory (csrc/overlap.h), against every byte of theirs.  Exit status 0 = all hold.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../paper_2509_22622_amd/csrc/overlap.h"

using namespace ll_api;

static bool shared(const Extent& a, const Extent& b) {
    std::vector<char> seen(4000, 0);
    for (int64_t r = 0; r < a.rows; ++r)
        for (int64_t i = 0; i < a.row; ++i) seen[reinterpret_cast<uintptr_t>(a.at) + r * a.stride + i] = 1;
    for (int64_t r = 0; r < b.rows; ++r)
        for (int64_t i = 0; i < b.row; ++i)
            if (seen[reinterpret_cast<uintptr_t>(b.at) + r * b.stride + i]) return true;
    return false;
}

int main() {
    std::srand(3);
    int yes = 0, no = 0;
    for (int i = 0; i < 400000; ++i) {
        const int kind = i % 4, stride = 1 + std::rand() % 30;
        Extent e[2];
        for (int k = 0; k < 2; ++k) {
            const int s = kind == 0 ? stride : 1 + std::rand() % 30, row = 1 + std::rand() % s;
            e[k] = Extent{reinterpret_cast<const void*>(uintptr_t(1 + std::rand() % 300)), std::rand() % 8, s, kind == 1 && k == 0 ? s : row};
            if (kind == 2 && k == 0) e[k].rows = 1;
        }
        const bool want = shared(e[0], e[1]);
        (want ? yes : no)++;
        for (int k = 0; k < 2; ++k) {
            const bool got = overlap(e[k], e[1 - k]);
            if (kind < 3 ? got != want : got && !want) {
                std::printf("kind %d: rows %lld stride %lld row %lld, rows %lld stride %lld row %lld: %d\n", kind, (long long)e[0].rows, (long long)e[0].stride, (long long)e[0].row,
                            (long long)e[1].rows, (long long)e[1].stride, (long long)e[1].row, int(got));
                return 1;
            }
            if (kind == 3 && e[0].at == e[1].at && want != got) return 1;
        }
    }
    const void* const p = reinterpret_cast<const void*>(uintptr_t(64));
    if (yes < 10000 || no < 10000 || overlap(extent(nullptr, 8), extent(p, 8)) || overlap(extent(p, 0), extent(p, 8)) || !overlap(extent(p, 1), extent(p, 8))) return 1;
    // far apart and long: 2^24 rows of 2^23 bytes' stride, columns side by side
    const Extent far{p, 1 << 24, 1 << 23, 256}, beside{reinterpret_cast<const void*>(uintptr_t(64 + 256)), 1 << 24, 1 << 23, 256};
    if (overlap(far, beside) || !overlap(far, far) || !overlap(far, extent(reinterpret_cast<const void*>(uintptr_t(64) + (uintptr_t(1) << 46)), 512))) return 1;
    const Extent three[] = {extent(p, 8), extent(reinterpret_cast<const void*>(uintptr_t(72)), 8), extent(reinterpret_cast<const void*>(uintptr_t(76)), 8)};
    if (any_overlap(three, 3, 1) || !any_overlap(three, 3, 2)) return 1;
    std::printf("overlaps ok\n");
    return 0;
}
