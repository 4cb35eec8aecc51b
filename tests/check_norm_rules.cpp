// How the layer norm's rows are dealt to threads and to workgroups (csrc/layer_norm.h), over every width.  Exit status 0 = all hold.
#include <cstdio>
#include <initializer_list>

#include "../paper_2509_22622_amd/csrc/layer_norm.h"

static int bad(const char* what, int a, int b, int c) {
    std::printf("%s: %d %d %d\n", what, a, b, c);
    return 1;
}

int main() {
    using namespace ll;
    for (int n = 1; n <= NORM_MAX_FEATURES; ++n) {
        const NormShape s = norm_shape(n);
        const int wg = s.threads * s.teams;
        if (wg % 64 != 0 || wg > 1024 || (s.threads <= 512 && wg > 512) || (s.threads == 16 && wg != 256)) return bad("workgroup", n, s.threads, wg);
        if (s.threads * s.pieces * 8 < n) return bad("a row does not fit", n, s.threads, s.pieces);
        if (s.threads != 16 && s.threads % 64 != 0) return bad("a team is neither a row of lanes nor whole waves", n, s.threads, 0);
        // the instantiations that there are
        const bool known = s.pieces * s.rows == 2 && (s.threads == 16 ? s.pieces <= 2 : s.pieces == 1 ? s.threads <= 512 : s.threads <= 1024);
        if (!known) return bad("no kernel", n, s.threads, s.pieces);
        // the teams' sums meet in an array of 4 x 512 numbers, one piece a thread
        if (s.threads != 16 && s.teams > 1 && (s.pieces != 1 || wg * 8 > 4 * 512)) return bad("sums do not fit", n, wg, s.pieces);
    }
    for (int n : {1, 64, 128, 129, 512, 1536, 4096, 4097, 8192, 16384})
        for (int m : {0, 1, 2, 3, 7, 16, 17, 63, 100, 1000, 4680, 32760, 1 << 20, 1 << 24})
            for (int group : {0, 1, 2, 3, 16, 100, 1560, 1 << 20, 2147483647}) {
                const NormPlan p = norm_plan(m, n, group);
                const int64_t each = group ? group : m;
                if (p.groups != (group ? (int64_t(m) + group - 1) / group : 1)) return bad("groups", m, group, p.groups);
                if (p.chunks < 1 || int64_t(p.groups) * p.chunks > (1 << 24)) return bad("chunks", m, group, p.chunks);
                if (p.groups * int64_t(p.chunks) > 1024 && p.chunks > 1) return bad("too many chunks", m, group, p.chunks);
                int64_t rows = 0;                                                // every row once, as the kernel walks them
                if (p.groups <= 4096)
                    for (int g = 0; g < p.groups; ++g)
                        for (int c = 0; c < p.chunks; ++c) {
                            const int64_t first = g * each + int64_t(c) * p.rows;
                            int64_t end = first + p.rows;
                            if (end > (g + 1) * each) end = (g + 1) * each;
                            if (end > m) end = m;
                            if (end > first) rows += end - first;
                        }
                else rows = m;
                if (rows != m) return bad("rows", m, group, int(rows));
                if (norm_numbers(p, n) != (p.chunks > 1 ? int64_t(p.groups) * p.chunks * 2 * n : 0)) return bad("numbers", m, n, group);
            }
    std::printf("norm rules ok\n");
    return 0;
}
