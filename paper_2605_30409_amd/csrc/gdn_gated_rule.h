// How the gated linear map's products are cut into tiles and parts, and which sizes it takes.  Host code without a
// GPU's headers.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstddef>

namespace gdn {

// The four products: h; dg and du; dx; the weights' gradients.
enum GatedKind { kGatedFwd, kGatedD, kGatedDx, kGatedDw };

constexpr int kSkinnyRows = 64;      // rows up to which the weights may be streamed

inline bool gated_shape_ok(int M, int C, int F) {
    return M >= 1 && C >= 1 && F >= 1 && C < (1 << 21) && F < (1 << 20) &&
           // a launch has fewer than 2^32 threads: the small tiles have 256, the large ones, which all larger sizes take, 512
           (M / 64 + 1LL) * (F / 64 + 1LL) < (1LL << 23) && (M / 64 + 1LL) * (C / 64 + 1LL) < (1LL << 23) &&
           (F / 128 + 1LL) * (C / 256 + 1LL) < (1LL << 22);
}

// How one of the products is cut: tiles of BM x BN, whose stages have `depth` buffers, and parts of the contraction.
struct GatedCut {
    int BM, BN, depth, splits;
    int rows, pitch;             // of a part's sums
    long long tiles;
    float us;
};

inline GatedCut gated_cut(int kind, int M, int C, int F, bool bf16) {
    const bool fwd = kind == kGatedFwd || kind == kGatedD;
    const int Fp = (F + 63) / 64 * 64, KB = bf16 ? 64 : 32;
    const long long cols = fwd ? 2LL * F : C;
    GatedCut g;
    g.rows = kind == kGatedDw ? 2 * Fp : M;
    g.pitch = fwd ? 2 * Fp : (C + 7) / 8 * 8;
    const int stages = fwd ? (C - 1) / KB + 1 : kind == kGatedDx ? 2 * ((F - 1) / KB + 1) : (M - 1) / KB + 1;
    // The cheapest by what stages were measured to take, us: of a tile that has its CU to itself, and of the one or two that a
    // CU holds on a full chip.
    const struct {
        int BM, BN, slots;
        float one, full;
    } size[] = {{256, 256, 1, bf16 ? 1.35f : 4.2f, bf16 ? 1.6f : 4.6f},
                {128, 128, 2, bf16 ? .62f : 1.65f, bf16 ? 1.2f : 3.f},
                {64, 128, 2, bf16 ? .45f : 1.25f, bf16 ? .8f : 1.95f},
                {64, 64, 2, .36f, .6f}};
    g.us = INFINITY;
    for (const auto &t : size) {
        // (decoding batches in bf16: 64 rows of 2048 x 8192 19.0 us, with 64 x 128 tiles 21.1; nothing gained elsewhere)
        if (t.BN == 64 && !(bf16 && kind == kGatedFwd && M <= kSkinnyRows)) continue;
        const long long tiles = ((long long)g.rows + t.BM - 1) / t.BM * ((cols + t.BN - 1) / t.BN);
        for (int splits = 1; splits <= 16 && splits * 4 <= stages + 3; ++splits) {
            const long long n = tiles * splits, rounds = n / (256 * t.slots), left = n % (256 * t.slots);
            if (splits > 1 && n > 256 * t.slots) break;
            float us = (rounds * t.full + (left == 0 ? 0 : left <= 256 ? t.one : t.full)) * ((stages + splits - 1) / splits + 3);
            if (splits > 1) us += 4 + 1.5e-6f * splits * g.rows * g.pitch;        // a launch, and the sums out and in at 5 TB/s
            if (us < g.us) {
                g.us = us;
                g.BM = t.BM;
                g.BN = t.BN;
                g.tiles = tiles;
                g.splits = splits;
            }
        }
    }
    // (more than 256 tiles of 64 x 64 are never the cheapest, nor of 64 x 128 for the weights' gradients, whose 2 Fp rows
    // half as many of 128 x 128 cover)
    const bool alone = g.tiles * g.splits <= 256;      // a CU each, and its LDS
    g.depth = g.BM == 256 ? 2 : g.BM == 128 ? (alone ? 4 : 2) : g.BN == 64 ? 8 : alone || kind == kGatedDw ? 6 : 3;
    return g;
}

// Whether a decoding batch streams the weights (every workgroup of 16 hidden units reads all rows of x) or goes through
// tiles.  Streams reach 6 TB/s (fp32 5) of what they read, x from the caches, and 39 (24) GB/s a workgroup where there are few.
// us, streams and tiles, bf16, 2048 x 8192: 1 row 16.3, 17.3; 16 rows 20.2, 18.3; 32 23.4, 19.0; 64 32.1, 19.0 (floor 14.2);
// 4096 x 1024: 1 row 10.4, 15.8; 32 17.0, 17.8; 64 24.4, 14.8; fp32, 2048 x 8192: 1 row 32, 42; 16 38, 43; 64 82, 47.
inline bool gated_streams(int M, int C, int F, bool bf16) {
    if (M > kSkinnyRows) return false;
    const size_t esz = bf16 ? 2 : 4;
    if (C * esz % 16) return true;                 // tiles would have the weights copied first
    const float row = (2 + M / 16.f) * (float)(C * esz), groups = (F + 15) / 16, turns = (F + 4095) / 4096;
    const float weights = 2e-6f * C * F * esz / 4.7f;
    const float stream = std::max({weights, row * 16 * groups / (bf16 ? 6e6f : 5e6f), row * 16 * turns / (bf16 ? 39e3f : 24e3f)});
    return 3 + stream <= 5 + std::max(weights, gated_cut(kGatedFwd, M, C, F, bf16).us);
}

}  // namespace gdn
