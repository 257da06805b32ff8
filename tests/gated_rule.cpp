// The gated linear map's choice of kernels, for tests on the host.
#include "gdn_gated_rule.h"

extern "C" {

// 0: few rows are streamed, by 16 * n of them; 1: tiles
int rule_tiles(int kind, int M, int C, int F, int bf16) {
    return kind != gdn::kGatedFwd || !gdn::gated_streams(M, C, F, bf16 != 0);
}

// BM, BN, depth, splits and the fewest stages of a part
void rule_cut(int kind, int M, int C, int F, int bf16, int *out) {
    const gdn::GatedCut g = gdn::gated_cut(kind, M, C, F, bf16 != 0);
    const int KB = bf16 ? 64 : 32;
    const int stages = kind <= gdn::kGatedD ? (C - 1) / KB + 1 : kind == gdn::kGatedDx ? 2 * ((F - 1) / KB + 1) : (M - 1) / KB + 1;
    out[0] = g.BM, out[1] = g.BN, out[2] = g.depth, out[3] = g.splits, out[4] = stages / g.splits;
}

}
