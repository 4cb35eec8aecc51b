// The integer rules of the paged cache (csrc/paged.h), checked on the host.  Exit status 0 = all hold.
#include <algorithm>
#include <cstdio>
#include <random>
#include <vector>

#include "../paper_2509_22622_amd/csrc/paged.h"

using namespace ll;

#define REQUIRE(x)                                                      \
    do {                                                                \
        if (!(x)) {                                                     \
            std::printf("line %d: %s\n", __LINE__, #x);                 \
            return 1;                                                   \
        }                                                               \
    } while (0)

// A granule's images hold each of its numbers once; a quad of V's tokens and the bytes a lane loads lie together.
static int layout() {
    for (int fmt : {0, 1})
        for (int D : {64, 128}) {
            std::vector<int> k(16 * D, 0), v(16 * D, 0);
            for (int t = 0; t < 16; ++t)
                for (int d = 0; d < D; ++d) {
                    const int a = paged_k_at(fmt, t, d), b = paged_v_at(fmt, t, d);
                    REQUIRE(a >= 0 && a < 16 * D && b >= 0 && b < 16 * D);
                    ++k[a];
                    ++v[b];
                    if (d % 8) REQUIRE(a == paged_k_at(fmt, t, d - d % 8) + d % 8);
                    if (t % 4) REQUIRE(b == paged_v_at(fmt, t - t % 4, d) + t % 4);
                }
            for (int i = 0; i < 16 * D; ++i) REQUIRE(k[i] == 1 && v[i] == 1);
            REQUIRE(paged_page_bytes(3, 48, D, fmt) == 3 * 2 * 48 * D * paged_number_bytes(fmt));
            REQUIRE(paged_step_keys(D) % (2 * PAGED_GRANULE) == 0);
        }
    return 0;
}

// The steps of a tile name every key that one of its rows sees, once, ascending, and no key that is not stored at all; steps come in
// runs that the workgroups and their waves deal out whole.
static int steps() {
    std::mt19937 rng(7);
    auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
    for (int trial = 0; trial < 20000; ++trial) {
        const int step = pick(0, 1) ? 32 : 64, len = pick(0, 700), tokens = pick(1, 20);
        const int i_hi = len - 1 - pick(0, 3), i_lo = i_hi - tokens + 1;                    // may be negative: no key
        const int window = pick(0, 2) ? pick(1, 400) : 0, sink = window ? pick(0, 300) : 0;
        const PagedSteps s = paged_steps(i_lo, i_hi, len, sink, window, step);
        REQUIRE(s.total >= 0);
        std::vector<int> visits((len + step - 1) / step + 1, 0);
        int last = -1;
        for (int v = 0; v < s.total; ++v) {
            const int at = s.at(v);
            REQUIRE(at > last && at >= 0 && at < int(visits.size()) - 1 && int64_t(at) * step <= i_hi);
            last = at;
            ++visits[at];
        }
        for (int j = 0; j < len; ++j)
            for (int i = i_lo; i <= i_hi; ++i)
                if (paged_sees(i, j, sink, window)) REQUIRE(visits[j / step] == 1);
        REQUIRE(s.total <= paged_most_steps(std::max(len, 1), tokens, sink, window, step));
        const int chunk = pick(1, 20), splits = pick(1, 12), run = paged_run(s.total, chunk, splits);
        REQUIRE(run >= chunk && int64_t(run) * splits >= s.total);
        std::vector<int> dealt(s.total, 0);
        for (int w = 0; w < splits; ++w) {
            const int begin = w * run, end = std::min(s.total, begin + run);
            const int per_wave = (std::max(end - begin, 0) + PAGED_WAVES - 1) / PAGED_WAVES;
            for (int k = 0; k < PAGED_WAVES; ++k)
                for (int v = begin + k * per_wave; v < std::min(end, begin + (k + 1) * per_wave); ++v) ++dealt[v];
        }
        for (int v : dealt) REQUIRE(v == 1);
    }
    // the far end of the range
    const int64_t top = PAGED_MAX_KEYS;
    REQUIRE(paged_steps(top - 1, top - 1, top, 0, 0, 32).total == top / 32);
    REQUIRE(paged_steps(top - 1, top - 1, top, 5, 1 << 30, 32).total == top / 32);
    REQUIRE(paged_steps(top - 1, top - 1, top, 5, 33, 32).total == 3 && paged_sees(top - 1, top - 33, 0, 33) && !paged_sees(top - 1, top - 34, 0, 33));
    return 0;
}

// What a call's sizes select: every tile's steps fit into its workgroups' runs, the join holds as many weights, and keys are not dealt out where
// there are workgroups enough without.
static int plans() {
    for (int64_t units : {1, 2, 7, 32, 128, 250, 256, 257, 512, 513, 1000, 2048, 2049, 100000})
        for (int64_t steps : {0, 1, 2, 8, 9, 24, 63, 64, 96, 256, 500, 4096, 40000, 1 << 24}) {
            const PagedPlan p = paged_plan(units, steps);
            const int64_t all = steps < 1 ? 1 : steps;
            REQUIRE(p.chunk >= 1 && p.splits >= 1 && int64_t(p.chunk) * p.splits >= all && int64_t(p.chunk) * (p.splits - 1) < all);
            REQUIRE(p.splits <= PAGED_MAX_SPLITS && (p.splits <= 5 || units * p.splits <= PAGED_CUS));
            if (units > PAGED_CUS / 3 && units <= PAGED_CUS && steps < 200) REQUIRE(units * p.splits <= PAGED_CUS);
            REQUIRE(paged_run(int(steps), p.chunk, p.splits) == p.chunk);
            if (units > 2048 || steps <= 24) REQUIRE(p.splits == 1);
            if (units <= 8 && steps >= 500) REQUIRE(p.splits >= 32);
        }
    for (int tokens : {1, 7, 8, 9, 96, 128, 500, 4680, 1 << 24})
        for (int units : {1, 6, 24, 1536})
            for (int most : {32, 64}) {
                const int rows = paged_tile_rows(tokens, units, most);
                REQUIRE(rows >= 8 && rows <= most && rows % 4 == 0);
                REQUIRE(rows == most || int64_t(tokens + rows - 1) / rows * units <= 512);
            }
    for (int tiles : {1, 2, 100, 147, 391, 512, 513, 1024, 1 << 19})
        for (int units : {1, 2, 18, 24, 1024 + 512}) {
            const int each = paged_units_per_group(tiles, units), groups = (units + each - 1) / each;
            REQUIRE(each >= 1 && each <= units && groups <= 1024);
            REQUIRE(tiles > 512 || tiles * groups <= 1024);
        }
    REQUIRE(paged_row_tiles(1, 1) == 1 && paged_row_tiles(16, 1) == 1 && paged_row_tiles(17, 1) == 2 && paged_row_tiles(5, 64) == 20 && paged_row_tiles(1024, PAGED_MAX_NEW) == 1 << 22);
    return 0;
}

static int division() {
    std::mt19937 rng(3);
    for (int64_t d : {1, 2, 3, 4, 5, 7, 12, 16, 17, 48, 63, 64, 65, 255, 256, 1000, 1023, 1024, 65520, 65536, 1 << 22, (1 << 26) - 1, 1 << 26}) {
        const PagedDiv by = paged_div(d);
        REQUIRE(by.d == d);
        for (int64_t q : {0, 1, 2, 3, 1000, 100000, 0x7FFFFFFF})
            for (int64_t n : {q * d - 1, q * d, q * d + 1, int64_t(0x7FFFFFFF) / d * d - 1, int64_t(0x7FFFFFFF) / d * d, int64_t(0x7FFFFFFF)})
                if (n >= 0 && n <= 0x7FFFFFFF) REQUIRE(by.of(uint32_t(n)) == uint32_t(n / d));
        for (int i = 0; i < 20000; ++i) {
            const uint32_t n = rng() & 0x7FFFFFFF;
            REQUIRE(by.of(n) == n / uint32_t(d));
        }
    }
    return 0;
}

int main() {
    if (division() || layout() || steps() || plans()) return 1;
    std::printf("paged rules ok\n");
    return 0;
}
