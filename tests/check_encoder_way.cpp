// How a call of the encoder attention's backward pass is launched (csrc/encoder_attn.h).  Arguments: sequences, query heads, kv heads, n_q, n_k, max_q, max_k.  Prints the way, the runs
// of dQ, and up to how many keys a sequence's delta comes first.
#include <cstdio>
#include <cstdlib>

#include "../paper_2509_22622_amd/csrc/encoder_attn.h"

int main(int argc, char** argv) {
    using namespace ll;
    if (argc != 8) return 1;
    int a[7];
    for (int i = 0; i < 7; ++i) a[i] = std::atoi(argv[i + 1]);
    const EncPlan p = enc_plan(a[0], a[1], a[2], a[5], a[6]);
    const char* const ways[] = {"small", "together", "in turn"};
    std::printf("%s\n%d\n%d\n", ways[enc_backward_way(p, int64_t(a[0]) * a[2], a[3], a[4])], p.q_splits, ENC_DELTA_FIRST);
    return 0;
}
