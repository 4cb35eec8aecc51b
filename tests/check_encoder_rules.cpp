// The integer rules of the attention to an encoder's states (csrc/encoder_attn.h): rows of a sequence, tiles, runs.  Exit status 0 = all hold.
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "../paper_2509_22622_amd/csrc/encoder_attn.h"

using namespace ll;

static int bad(const char* what, int64_t a, int64_t b, int64_t c) {
    std::printf("%s: %lld %lld %lld\n", what, (long long)a, (long long)b, (long long)c);
    return 1;
}

int main() {
    // whatever the arrays hold, a sequence's rows are rows of the tensor
    std::srand(7);
    const int odd[] = {0, 1, -1, 5, 17, 100, 101, 2147483647, -2147483647 - 1, 64, 99};
    for (int i = 0; i < 200000; ++i) {
        const int n_seqs = 1 + std::rand() % 4, total = n_seqs * (std::rand() % 40), most = 1 + std::rand() % 50;
        int cu[5], lens[4];
        for (int& x : cu) x = odd[std::rand() % 11];
        for (int& x : lens) x = odd[std::rand() % 11];
        for (int s = 0; s < n_seqs; ++s)
            for (int kind = 0; kind < 4; ++kind) {
                const EncSpan e = enc_span(kind & 1 ? cu : nullptr, kind & 2 ? lens : nullptr, s, n_seqs, total, most);
                if (e.begin < 0 || e.n < 0 || e.n > most || e.begin + e.n > e.end || e.end > total) return bad("span", e.begin, e.n, e.end);
            }
    }
    {
        const int cu[] = {3, 10, 10, 25}, lens[] = {4, 9, 100};
        EncSpan e = enc_span(cu, lens, 0, 3, 30, 99);
        if (e.begin != 3 || e.n != 4 || e.end != 10) return bad("span 0", e.begin, e.n, e.end);
        e = enc_span(cu, lens, 1, 3, 30, 99);
        if (e.begin != 10 || e.n != 0 || e.end != 10) return bad("span 1", e.begin, e.n, e.end);
        e = enc_span(cu, nullptr, 2, 3, 30, 12);
        if (e.begin != 10 || e.n != 12 || e.end != 25) return bad("span 2", e.begin, e.n, e.end);
        e = enc_span(nullptr, lens, 2, 3, 30, 99);
        if (e.begin != 20 || e.n != 10 || e.end != 30) return bad("span 3", e.begin, e.n, e.end);
    }
    for (int steps = 0; steps <= 70; ++steps)                          // runs cover every step once
        for (int splits = 1; splits <= 40; ++splits) {
            int at = 0;
            for (int i = 0; i < splits; ++i) {
                int first, end;
                enc_run(steps, splits, i, first, end);
                if (first < end) {
                    if (first != at || end > steps) return bad("run", steps, splits, i);
                    at = end;
                }
            }
            if (at != steps) return bad("runs", steps, splits, at);
        }
    for (int n_seqs : {1, 2, 3, 8, 64, 1000, 1 << 20})
        for (int kv : {1, 2, 8, 12, 1024})
            for (int group : {1, 3, 8, 32})
                for (int64_t max_q : {1, 2, 4, 31, 33, 100, 4680, 32760, 1 << 24})
                    for (int64_t max_k : {1, 33, 512, 4000, 32000, 1 << 24}) {
                        if (kv * group > 1024) continue;
                        const EncPlan p = enc_plan(n_seqs, kv * group, kv, max_q, max_k);
                        const int64_t heads = int64_t(n_seqs) * kv, rows = group * max_q;
                        if (p.few != (rows <= ENC_FEW_ROWS) || (p.few && p.tiles != 1)) return bad("few", rows, p.few, p.tiles);
                        if (int64_t(p.tiles) * (p.few ? ENC_FEW_ROWS : ENC_ROWS) < rows || int64_t(p.q_tiles) * ENC_ROWS < rows || int64_t(p.k_tiles) * ENC_COLS < max_k)
                            return bad("tiles", rows, p.tiles, p.k_tiles);
                        for (int s : {p.splits, p.q_splits, p.k_splits})
                            if (s < 1 || s > ENC_MAX_SPLITS) return bad("splits", p.splits, p.q_splits, p.k_splits);
                        // launches that join or add up have few tiles: their grids stay small
                        if (p.splits > 1 && heads * p.tiles > 1024) return bad("join", heads, p.tiles, p.splits);
                        if ((p.q_splits > 1 && heads * p.q_tiles > 1024) || (p.k_splits > 1 && heads * p.k_tiles > 1024)) return bad("sum", heads, p.q_tiles, p.k_tiles);
                        if (heads * p.tiles * p.splits > 4096 && p.splits > 1) return bad("partial results", heads, p.tiles, p.splits);
                    }
    std::printf("encoder rules ok\n");
    return 0;
}
