// Host side of the operators in gdn_block.h: argument validation, the choice of kernel variants, launches, and the
// extern "C" entry points.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <mutex>
#include <new>
#include <type_traits>
#include <utility>
#include <vector>

#include "gdn_block.h"
#include "gdn_clip.h"
#include "gdn_conv.h"
#include "gdn_gated.h"
#include "gdn_gated_rule.h"
#include "gdn_host.h"

namespace {

bool act_ok(int act) { return act >= GDN_ACT_NONE && act <= GDN_ACT_GELU_TANH; }

bool ws_ok(const void *ws, size_t have, size_t need) { return need == 0 || (ws && !misaligned(ws, 256) && have >= need); }

// ---------------------------------------------------------------------------
// Gated linear map.

// What a tensor with rows of n elements is aligned to: 16 bytes, or an element where its rows are not either (those are
// copied, streamed and written at any element).
uintptr_t row_alignment(int n, int is_bf16) {
    const uintptr_t esz = is_bf16 ? 2 : 4;
    return n * esz % 16 ? esz : 16;
}

// Where the parts of the workspace begin.
struct GatedLayout {
    size_t x, d, part, total;     // x: x, Wg and Wu at whole rows' pitch
    bool streams, pack;
    int ld, Fp;
};
GatedLayout gated_layout(int M, int C, int F, bool bf16, bool backward) {
    GatedLayout L{};
    const size_t esz = bf16 ? 2 : 4;
    L.Fp = (F + 63) / 64 * 64;
    L.ld = C;
    L.streams = !backward && gdn::gated_streams(M, C, F, bf16);
    if (L.streams) return L;
    L.pack = C * esz % 16 != 0;
    if (L.pack) L.ld = (C + 63) / 64 * 64;
    size_t off = 0;
    auto take = [&](size_t n) {
        const size_t at = off;
        off += align256(n);
        return at;
    };
    if (L.pack) {
        L.x = take(((size_t)M + 2 * (size_t)F) * L.ld * esz);
    }
    if (backward) L.d = take((size_t)M * 2 * L.Fp * esz);
    size_t part = 0;
    for (int kind = backward ? gdn::kGatedD : gdn::kGatedFwd; kind <= (backward ? gdn::kGatedDw : gdn::kGatedFwd); ++kind) {
        const gdn::GatedCut g = gdn::gated_cut(kind, M, C, F, bf16);
        if (g.splits > 1) part = std::max(part, (size_t)g.splits * g.rows * g.pitch * 4);
    }
    L.part = take(part);
    L.total = off;
    return L;
}

// Workgroups of the launch that copies rows, 8 elements a thread, and whether it has room for them: 2^24 of 256 threads.
long long gated_copy_groups(const GatedLayout &L, int M, int F) { return ((M + 2LL * F) * (L.ld / 8) + 255) / 256; }
bool gated_fits(const GatedLayout &L, int M, int F) { return !L.pack || gated_copy_groups(L, M, F) < (1LL << 24); }

template <class E, int KIND, int BM, int BN, int WM, int WN, int DEPTH> int launch_tiles(const gdn::GatedParams<E> &p, hipStream_t s) {
    constexpr size_t lds = DEPTH * (BM + BN) * 128;
    const auto fn = gdn::gdn_gated_tile_kernel<E, KIND, BM, BN, WM, WN, DEPTH>;
    static std::once_flag once;
    static hipError_t attr = hipSuccess;
    std::call_once(once, [&] {
        attr = hipFuncSetAttribute((const void *)fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    });
    if (attr != hipSuccess) return GDN_ERR_HIP;
    return launch(fn, dim3((unsigned)(p.tiles_m * p.tiles_n * p.splits)), dim3(64 * WM * WN), lds, s, p);
}

template <class E, int KIND> int run_tiles(gdn::GatedParams<E> p, hipStream_t s) {
    constexpr bool FWD = KIND == gdn::kGatedFwd || KIND == gdn::kGatedD;
    const gdn::GatedCut g = gdn::gated_cut(KIND, p.M, p.C, p.F, sizeof(E) == 2);
    const int cols = FWD ? p.F : p.C, wide = FWD ? g.BN / 2 : g.BN;
    p.rows = g.rows;
    p.pitch = g.pitch;
    p.splits = g.splits;
    p.tiles_m = (g.rows + g.BM - 1) / g.BM;
    p.tiles_n = (cols + wide - 1) / wide;
    int st = GDN_ERR_UNSUPPORTED;
    if constexpr (KIND == gdn::kGatedFwd && sizeof(E) == 2)
        if (g.BN == 64) st = launch_tiles<E, KIND, 64, 64, 2, 1, 8>(p, s);
    if constexpr (KIND != gdn::kGatedDw)
        if (g.BM == 64 && g.depth == 3) st = launch_tiles<E, KIND, 64, 128, 2, 2, 3>(p, s);
    if (g.BM == 64 && g.depth == 6) st = launch_tiles<E, KIND, 64, 128, 2, 2, 6>(p, s);
    if (g.BM == 128) st = g.depth == 4 ? launch_tiles<E, KIND, 128, 128, 2, 2, 4>(p, s) : launch_tiles<E, KIND, 128, 128, 2, 2, 2>(p, s);
    if (g.BM == 256) st = launch_tiles<E, KIND, 256, 256, 2, 4, 2>(p, s);
    if (st != GDN_OK || g.splits == 1) return st;
    const long long units = (long long)g.rows * ((FWD ? p.Fp : g.pitch) / 8);
    return launch(gdn::gdn_gated_join_kernel<E, KIND>, dim3((unsigned)((units + 255) / 256)), dim3(256), 0, s, p);
}

template <class E> int run_gated(gdn::GatedParams<E> p, const GatedLayout &L, unsigned char *ws, bool backward, hipStream_t s) {
    p.Fp = L.Fp;
    p.ldx = p.ldw = L.ld;
    if (L.streams) {
        const dim3 grid((unsigned)((p.F + 15) / 16)), block(64 * gdn::kSkinnyWaves);
        if (p.M <= 16) return launch(gdn::gdn_gated_skinny_kernel<E, 1>, grid, block, 0, s, p);
        if (p.M <= 32) return launch(gdn::gdn_gated_skinny_kernel<E, 2>, grid, block, 0, s, p);
        return launch(gdn::gdn_gated_skinny_kernel<E, 4>, grid, block, 0, s, p);
    }
    int st = GDN_OK;
    if (L.pack) {
        const gdn::PackParams<E> q{{p.x, p.wg, p.wu}, (E *)(ws + L.x), p.M, p.F, p.C, L.ld};
        st = launch(gdn::gdn_gated_pack_kernel<E>, dim3((unsigned)gated_copy_groups(L, p.M, p.F)), dim3(256), 0, s, q);
        p.x = (const E *)(ws + L.x);
        p.wg = p.x + (size_t)p.M * L.ld;
        p.wu = p.wg + (size_t)p.F * L.ld;
    }
    if (st != GDN_OK) return st;
    p.part = (float *)(ws + L.part);
    if (!backward) return run_tiles<E, gdn::kGatedFwd>(p, s);
    p.d = (E *)(ws + L.d);
    st = run_tiles<E, gdn::kGatedD>(p, s);
    if (st == GDN_OK) st = run_tiles<E, gdn::kGatedDx>(p, s);
    if (st == GDN_OK) st = run_tiles<E, gdn::kGatedDw>(p, s);
    return st;
}

// ---------------------------------------------------------------------------
// Short convolution.

constexpr int kMinTaps = 2, kMaxTaps = 4;

template <class P, class F> int with_taps(int W, const P &p, F f) {
    switch (W) {
    case 2: return f(p, std::integral_constant<int, 2>{});
    case 3: return f(p, std::integral_constant<int, 3>{});
    default: return f(p, std::integral_constant<int, 4>{});
    }
}

int conv_shape(int B, int T, int C, int W, long long xb, long long xt) {
    if (B < 1 || T < 1 || C < 1 || xb < 0 || xt < 0) return GDN_ERR_SHAPE;
    if (W < kMinTaps || W > kMaxTaps) return GDN_ERR_UNSUPPORTED;
    const long long G = (C + 7LL) / 8;
    if ((long long)B * T >= (1LL << 33) / G || T >= (1 << 30)) return GDN_ERR_SHAPE;
    return GDN_OK;
}

// Elements from the first to behind the last of a [B][T][C] with these strides.
size_t span(int B, int T, int C, long long xb, long long xt) { return (size_t)((B - 1) * xb + (T - 1) * xt + C); }

// Whether no two elements of such a tensor are the same: its sequences lie one behind the other, or all sequences of a
// token before the next token.
bool conv_apart(int B, int T, int C, long long xb, long long xt) {
    const bool by_sequence = (T == 1 || xt >= C) && (B == 1 || xb >= (T - 1) * xt + C);
    const bool by_token = (B == 1 || xb >= C) && (T == 1 || xt >= (B - 1) * xb + C);
    return by_sequence || by_token;
}

// Tokens of a thread's strip: many threads first, then fewer rows read twice (10560 x 2048 bf16 19.3 us, 10560 x 6144 46.5).
int conv_strip(int B, int T, int C) {
    const long long turns = (long long)B * T * ((C + 7) / 8) / 65536;
    return (int)std::max(4LL, std::min(16LL, turns / 4 * 4));
}

// Workgroups of the forward call's launch, and whether it has room for them: 2^24 of 256 threads.
long long conv_groups(int B, int T, int C) {
    const long long strips = (T - 1) / conv_strip(B, T, C) + 1;
    return (B * strips * ((C + 7) / 8) + 255) / 256;
}
bool conv_fits(int B, int T, int C) { return conv_groups(B, T, C) < (1LL << 24); }

struct ConvGrad {
    int TX, strip, strips, blocks;
    long long gx;
    size_t part;
};
ConvGrad conv_grad(int B, int T, int C, int W) {
    ConvGrad g;
    const int G = (C + 3) / 4;
    g.TX = 1;
    while (g.TX < G && g.TX < 64) g.TX *= 2;
    // Strips as long as leave 131072 threads, up to 32.  us at 16, 24, 32 and 48 tokens, bf16: 10560 x 2048 38.5, 36.6, 36.1, 35.9;
    // 10560 x 6144 92, 87, 84, 90; 3520 x 2048 18.9, 21.6, 21.6, 21.6; fp32, 10560 x 2048 62, 58, 59, 55; 10560 x 6144 162,
    // 162, 164, 180.
    const long long turns = (long long)B * T * G / 131072;
    g.strip = (int)std::max(4LL, std::min(32LL, turns / 4 * 4));
    g.strips = (T - 1) / g.strip + 1;
    const int TY = gdn::kConvGradThreads / g.TX;
    g.blocks = (g.strips - 1) / TY + 1;
    g.gx = (G - 1) / g.TX + 1;
    g.part = (size_t)B * g.blocks * (W + 1) * C * 4;
    return g;
}

// Workgroups of the second launch, 64 sums each.
long long conv_sums_groups(int C, int W) { return ((W + 1LL) * C + 63) / 64; }

// Whether both of the gradient's launches have room for their workgroups: 2^23 of 256 threads, 2^22 of 1024.
bool conv_grad_fits(int B, int T, int C, int W) {
    const ConvGrad g = conv_grad(B, T, C, W);
    return g.gx * B * g.blocks < (1LL << 23) && conv_sums_groups(C, W) < (1LL << 22);
}

// ---------------------------------------------------------------------------
// Gradient norm and clipping.

int clip_groups(long long chunks) { return (int)std::min<long long>(chunks, gdn::kClipGroups); }

int clip_launches(int count) { return (count + gdn::kClipTensors - 1) / gdn::kClipTensors; }

// Tables of the non-empty tensors, kClipTensors of them each, given to f in turn.
template <class F> int clip_tables(const void *const *in, void *const *out, const int64_t *sizes, const int *is_bf16, int count, F f) {
    gdn::ClipTable t{};
    long long chunks = 0;
    auto flush = [&] {
        t.groups = clip_groups(chunks);
        const int st = t.count ? f(t) : GDN_OK;
        t.count = 0;
        chunks = 0;
        return st;
    };
    for (int i = 0; i < count; ++i) {
        if (!sizes[i]) continue;
        const long long n = (sizes[i] - 1) / gdn::kClipChunk + 1;
        t.in[t.count] = in[i];
        t.out[t.count] = out ? out[i] : nullptr;
        chunks += n;
        t.end[t.count] = 2 * chunks + (is_bf16[i] ? 1 : 0);
        t.tail[t.count] = (unsigned)(sizes[i] - (n - 1) * gdn::kClipChunk);
        if (++t.count == gdn::kClipTensors) {
            const int st = flush();
            if (st != GDN_OK) return st;
        }
    }
    return flush();
}

// Room for all launches' sums; a norm stands behind it.
size_t clip_sums_bytes(int count) {
    return align256((size_t)std::max(1, clip_launches(count)) * gdn::kClipGroups * sizeof(double));
}

// Sums up to which every workgroup of the scaling adds them up for itself (64 KB from the caches); more are added once, by
// a launch of their own.
constexpr int kClipOwnSums = 4 * gdn::kClipGroups;

int clip_check(const void *const *in, const int64_t *sizes, const int *is_bf16, int count) {
    if (count < 0) return GDN_ERR_SHAPE;
    if (count && (!in || !sizes || !is_bf16)) return GDN_ERR_NULL;
    for (int i = 0; i < count; ++i) {
        if (sizes[i] < 0 || sizes[i] >= (1LL << 50)) return GDN_ERR_SHAPE;
        if (sizes[i] && !in[i]) return GDN_ERR_NULL;
        if (sizes[i] && misaligned(in[i], is_bf16[i] ? 2 : 4)) return GDN_ERR_ALIGN;
    }
    return GDN_OK;
}

// Squares of all tensors, a sum a workgroup; how many sums there are in `parts`.
int clip_squares(const void *const *in, const int64_t *sizes, const int *is_bf16, int count, double *part, int &parts, hipStream_t s) {
    parts = 0;
    return clip_tables(in, nullptr, sizes, is_bf16, count, [&](gdn::ClipTable &t) {
        t.part = part + parts;
        parts += t.groups;
        return launch(gdn::gdn_grad_squares_kernel, dim3((unsigned)t.groups), dim3(gdn::kClipThreads), 0, s, t);
    });
}

}  // namespace

extern "C" {

size_t gdn_gated_linear_workspace_bytes(int M, int C, int F, int is_bf16, int backward) {
    if (!gdn::gated_shape_ok(M, C, F)) return 0;
    const GatedLayout L = gated_layout(M, C, F, is_bf16 != 0, backward != 0);
    return gated_fits(L, M, F) ? L.total : 0;
}

int gdn_gated_linear_forward(const void *x, const void *w_gate, const void *w_up, void *h, int M, int C, int F,
                             int act, int is_bf16, void *ws, size_t ws_bytes, void *stream) {
    if (!x || !w_gate || !w_up || !h) return GDN_ERR_NULL;
    if (!gdn::gated_shape_ok(M, C, F)) return GDN_ERR_SHAPE;
    const GatedLayout L = gated_layout(M, C, F, is_bf16 != 0, false);
    if (!gated_fits(L, M, F)) return GDN_ERR_SHAPE;
    if (!act_ok(act)) return GDN_ERR_UNSUPPORTED;
    for (const void *p : {x, w_gate, w_up})
        if (misaligned(p, row_alignment(C, is_bf16))) return GDN_ERR_ALIGN;
    if (misaligned(h, row_alignment(F, is_bf16))) return GDN_ERR_ALIGN;
    if (!ws_ok(ws, ws_bytes, L.total)) return GDN_ERR_WORKSPACE;
    const size_t esz = is_bf16 ? 2 : 4, wb = (size_t)F * C * esz;
    const Range rh(h, (size_t)M * F * esz), rws(L.total ? ws : nullptr, L.total);
    for (const Range &r : {Range(x, (size_t)M * C * esz), Range(w_gate, wb), Range(w_up, wb)})
        if (rh.overlaps(r) || rws.overlaps(r)) return GDN_ERR_ALIAS;
    if (rh.overlaps(rws)) return GDN_ERR_ALIAS;
    auto run = [&](auto *e) {
        using E = std::remove_pointer_t<decltype(e)>;
        gdn::GatedParams<E> p{};
        p.x = (const E *)x;
        p.wg = (const E *)w_gate;
        p.wu = (const E *)w_up;
        p.h = (E *)h;
        p.M = M;
        p.C = C;
        p.F = F;
        p.act = act;
        return run_gated<E>(p, L, (unsigned char *)ws, false, (hipStream_t)stream);
    };
    return is_bf16 ? run((uint16_t *)nullptr) : run((float *)nullptr);
}

int gdn_gated_linear_backward(const void *x, const void *w_gate, const void *w_up, const void *dh, void *dx,
                              void *dw_gate, void *dw_up, int M, int C, int F, int act, int is_bf16, void *ws,
                              size_t ws_bytes, void *stream) {
    if (!x || !w_gate || !w_up || !dh || !dx || !dw_gate || !dw_up) return GDN_ERR_NULL;
    if (!gdn::gated_shape_ok(M, C, F)) return GDN_ERR_SHAPE;
    const GatedLayout L = gated_layout(M, C, F, is_bf16 != 0, true);
    if (!gated_fits(L, M, F)) return GDN_ERR_SHAPE;
    if (!act_ok(act)) return GDN_ERR_UNSUPPORTED;
    for (const void *p : {x, w_gate, w_up, (const void *)dx, (const void *)dw_gate, (const void *)dw_up})
        if (misaligned(p, row_alignment(C, is_bf16))) return GDN_ERR_ALIGN;
    if (misaligned(dh, row_alignment(F, is_bf16))) return GDN_ERR_ALIGN;
    if (!ws_ok(ws, ws_bytes, L.total)) return GDN_ERR_WORKSPACE;
    const size_t esz = is_bf16 ? 2 : 4, xb = (size_t)M * C * esz, wb = (size_t)F * C * esz;
    const Range in[] = {Range(x, xb), Range(w_gate, wb), Range(w_up, wb), Range(dh, (size_t)M * F * esz)};
    const Range outs[] = {Range(dx, xb), Range(dw_gate, wb), Range(dw_up, wb), Range(ws, L.total)};
    for (int i = 0; i < 4; ++i) {
        for (const Range &r : in)
            if (outs[i].overlaps(r)) return GDN_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (outs[i].overlaps(outs[j])) return GDN_ERR_ALIAS;
    }
    auto run = [&](auto *e) {
        using E = std::remove_pointer_t<decltype(e)>;
        gdn::GatedParams<E> p{};
        p.x = (const E *)x;
        p.wg = (const E *)w_gate;
        p.wu = (const E *)w_up;
        p.dh = (const E *)dh;
        p.dx = (E *)dx;
        p.dwg = (E *)dw_gate;
        p.dwu = (E *)dw_up;
        p.M = M;
        p.C = C;
        p.F = F;
        p.act = act;
        return run_gated<E>(p, L, (unsigned char *)ws, true, (hipStream_t)stream);
    };
    return is_bf16 ? run((uint16_t *)nullptr) : run((float *)nullptr);
}

int gdn_short_conv_forward(const void *x, int64_t x_batch, int64_t x_token, const float *w, const float *bias,
                           const void *state_in, void *y, void *state_out, int B, int T, int C, int W, int act,
                           int is_bf16, void *stream) {
    if (!x || !w || !y) return GDN_ERR_NULL;
    const int st = conv_shape(B, T, C, W, x_batch, x_token);
    if (st != GDN_OK) return st;
    if (!conv_fits(B, T, C)) return GDN_ERR_SHAPE;
    if (!act_ok(act)) return GDN_ERR_UNSUPPORTED;
    const size_t esz = is_bf16 ? 2 : 4;
    if (misaligned(x, esz)) return GDN_ERR_ALIGN;
    for (const void *p : {(const void *)w, (const void *)bias, state_in, (const void *)y, (const void *)state_out})
        if (misaligned(p)) return GDN_ERR_ALIGN;
    const size_t sb = (size_t)B * (W - 1) * C * esz;
    const Range ry(y, (size_t)B * T * C * esz), ro(state_out, sb), ri(state_in, sb);
    for (const Range &r : {Range(x, span(B, T, C, x_batch, x_token) * esz), Range(w, (size_t)C * W * 4), Range(bias, (size_t)C * 4)})
        if (ry.overlaps(r) || ro.overlaps(r)) return GDN_ERR_ALIAS;
    if (ry.overlaps(ri) || ry.overlaps(ro) || (ro.overlaps(ri) && !ro.same(ri))) return GDN_ERR_ALIAS;
    auto run = [&](auto *e) {
        using E = std::remove_pointer_t<decltype(e)>;
        gdn::ConvParams<E> p{};
        p.x = (const E *)x;
        p.state = (const E *)state_in;
        p.w = w;
        p.bias = bias;
        p.y = (E *)y;
        p.state_out = (E *)state_out;
        p.xb = x_batch;
        p.xt = x_token;
        p.ob = (long long)T * C;
        p.ot = C;
        p.B = B;
        p.T = T;
        p.C = C;
        p.act = act;
        p.strip = conv_strip(B, T, C);
        p.strips = (T - 1) / p.strip + 1;
        return with_taps(W, p, [&](const auto &q, auto taps) {
            return launch(gdn::gdn_short_conv_kernel<E, decltype(taps)::value>, dim3((unsigned)conv_groups(B, T, C)), dim3(256), 0,
                          (hipStream_t)stream, q);
        });
    };
    return is_bf16 ? run((uint16_t *)nullptr) : run((float *)nullptr);
}

size_t gdn_short_conv_workspace_bytes(int B, int T, int C, int W) {
    if (conv_shape(B, T, C, W, 0, 0) != GDN_OK || !conv_grad_fits(B, T, C, W)) return 0;
    return align256(conv_grad(B, T, C, W).part);
}

int gdn_short_conv_backward(const void *x, int64_t x_batch, int64_t x_token, const float *w, const float *bias,
                            const void *state_in, const void *dy, const void *dstate_out, void *dx, int64_t dx_batch,
                            int64_t dx_token, float *dw, float *dbias, void *dstate_in, int B, int T, int C, int W,
                            int act, int is_bf16, void *ws, size_t ws_bytes, void *stream) {
    if (!x || !w || !dy || !dx || !dw) return GDN_ERR_NULL;
    const int st = conv_shape(B, T, C, W, x_batch, x_token);
    if (st != GDN_OK) return st;
    if (!conv_grad_fits(B, T, C, W)) return GDN_ERR_SHAPE;
    if (dx_token < 0 || dx_batch < 0 || !conv_apart(B, T, C, dx_batch, dx_token)) return GDN_ERR_SHAPE;
    if (!act_ok(act)) return GDN_ERR_UNSUPPORTED;
    const size_t esz = is_bf16 ? 2 : 4;
    if (misaligned(x, esz) || misaligned(dx, esz)) return GDN_ERR_ALIGN;
    for (const void *p : {(const void *)w, (const void *)bias, state_in, dy, dstate_out, (const void *)dw, (const void *)dbias, (const void *)dstate_in})
        if (misaligned(p)) return GDN_ERR_ALIGN;
    const ConvGrad g = conv_grad(B, T, C, W);
    if (!ws_ok(ws, ws_bytes, align256(g.part))) return GDN_ERR_WORKSPACE;
    const size_t sb = (size_t)B * (W - 1) * C * esz;
    const Range in[] = {Range(x, span(B, T, C, x_batch, x_token) * esz), Range(w, (size_t)C * W * 4), Range(bias, (size_t)C * 4),
                        Range(state_in, sb), Range(dy, (size_t)B * T * C * esz), Range(dstate_out, sb)};
    const Range outs[] = {Range(dx, span(B, T, C, dx_batch, dx_token) * esz), Range(dw, (size_t)C * W * 4), Range(dbias, (size_t)C * 4),
                          Range(dstate_in, sb), Range(ws, g.part)};
    for (int i = 0; i < 5; ++i) {
        for (const Range &r : in)
            if (outs[i].overlaps(r)) return GDN_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (outs[i].overlaps(outs[j])) return GDN_ERR_ALIAS;
    }
    auto run = [&](auto *e) {
        using E = std::remove_pointer_t<decltype(e)>;
        gdn::ConvParams<E> p{};
        p.x = (const E *)x;
        p.state = (const E *)state_in;
        p.dy = (const E *)dy;
        p.dstate_out = (const E *)dstate_out;
        p.w = w;
        p.bias = bias;
        p.dx = (E *)dx;
        p.dstate = (E *)dstate_in;
        p.part = (float *)ws;
        p.dw = dw;
        p.dbias = dbias;
        p.xb = x_batch;
        p.xt = x_token;
        p.ob = dx_batch;
        p.ot = dx_token;
        p.yb = (long long)T * C;
        p.yt = C;
        p.B = B;
        p.T = T;
        p.C = C;
        p.act = act;
        p.strip = g.strip;
        p.strips = g.strips;
        const int rows = B * g.blocks;
        return with_taps(W, p, [&](const auto &q, auto taps) {
            constexpr int N = decltype(taps)::value;
            auto grad = [&](gdn::ConvParams<E> a, int tx) {
                const void *fn[] = {(const void *)gdn::gdn_short_conv_grad_kernel<E, N, GDN_ACT_NONE>,
                                    (const void *)gdn::gdn_short_conv_grad_kernel<E, N, GDN_ACT_SILU>,
                                    (const void *)gdn::gdn_short_conv_grad_kernel<E, N, GDN_ACT_GELU>,
                                    (const void *)gdn::gdn_short_conv_grad_kernel<E, N, GDN_ACT_GELU_TANH>,
                                    (const void *)gdn::gdn_short_conv_grad_kernel<E, N, -1>};
                void *args[] = {&a, &tx};
                return hipLaunchKernel(fn[C < 4 ? 4 : act], dim3((unsigned)(g.gx * rows)), dim3(gdn::kConvGradThreads), args, 0,
                                       (hipStream_t)stream);
            };
            auto sums = [&](gdn::ConvParams<E> a, int taps_, int n) {
                void *args[] = {&a, &taps_, &n};
                return hipLaunchKernel((const void *)gdn::gdn_short_conv_reduce_kernel<E>, dim3((unsigned)conv_sums_groups(C, N)),
                                       dim3(64 * gdn::kConvReduceWaves), args, 0, (hipStream_t)stream);
            };
            if (grad(q, g.TX) != hipSuccess || sums(q, N, rows) != hipSuccess) return (int)GDN_ERR_HIP;
            return (int)GDN_OK;
        });
    };
    return is_bf16 ? run((uint16_t *)nullptr) : run((float *)nullptr);
}

int gdn_short_conv_step(const void *x, int64_t x_row, int64_t x_token, const float *w, const float *bias,
                        const void *state_in, const int *slots, const int *lengths, void *y, void *state_out, int N,
                        int L, int P, int C, int W, int act, int is_bf16, void *stream) {
    if (!x || !w || !state_in || !y || !state_out) return GDN_ERR_NULL;
    const int st = conv_shape(N, L, C, W, x_row, x_token);
    if (st != GDN_OK) return st;
    const long long waves = ((C + 7) / 8 + 63) / 64;
    if (P < 1 || (!slots && N > P) || N * waves >= (1LL << 24)) return GDN_ERR_SHAPE;
    if (!act_ok(act)) return GDN_ERR_UNSUPPORTED;
    const size_t esz = is_bf16 ? 2 : 4;
    if (misaligned(x, esz) || misaligned(slots, 4) || misaligned(lengths, 4)) return GDN_ERR_ALIGN;
    for (const void *p : {(const void *)w, (const void *)bias, state_in, (const void *)y, (const void *)state_out})
        if (misaligned(p)) return GDN_ERR_ALIGN;
    const size_t sb = (size_t)P * (W - 1) * C * esz;
    const Range ry(y, (size_t)N * L * C * esz), ro(state_out, sb), ri(state_in, sb);
    for (const Range &r : {Range(x, span(N, L, C, x_row, x_token) * esz), Range(w, (size_t)C * W * 4), Range(bias, (size_t)C * 4),
                           Range(slots, (size_t)N * 4), Range(lengths, (size_t)N * 4)})
        if (ry.overlaps(r) || ro.overlaps(r)) return GDN_ERR_ALIAS;
    if (ry.overlaps(ri) || ry.overlaps(ro) || (ro.overlaps(ri) && !ro.same(ri))) return GDN_ERR_ALIAS;
    auto run = [&](auto *e) {
        using E = std::remove_pointer_t<decltype(e)>;
        gdn::ConvParams<E> p{};
        p.x = (const E *)x;
        p.state = (const E *)state_in;
        p.w = w;
        p.bias = bias;
        p.y = (E *)y;
        p.state_out = (E *)state_out;
        p.slots = slots;
        p.lengths = lengths;
        p.xb = x_row;
        p.xt = x_token;
        p.B = N;
        p.T = L;
        p.C = C;
        p.P = P;
        p.act = act;
        return with_taps(W, p, [&](const auto &q, auto taps) {
            return launch(gdn::gdn_short_conv_step_kernel<E, decltype(taps)::value>, dim3((unsigned)((N * waves + 3) / 4)), dim3(256), 0,
                          (hipStream_t)stream, q);
        });
    };
    return is_bf16 ? run((uint16_t *)nullptr) : run((float *)nullptr);
}

size_t gdn_grad_workspace_bytes(int count) {
    if (count < 0) return 0;
    return clip_sums_bytes(count) + 256;
}

int gdn_grad_norm(const void *const *tensors, const int64_t *sizes, const int *is_bf16, int count, float *norm, void *ws,
                  size_t ws_bytes, void *stream) {
    if (!norm) return GDN_ERR_NULL;
    int st = clip_check(tensors, sizes, is_bf16, count);
    if (st != GDN_OK) return st;
    if (misaligned(norm, 4)) return GDN_ERR_ALIGN;
    if (!ws_ok(ws, ws_bytes, gdn_grad_workspace_bytes(count))) return GDN_ERR_WORKSPACE;
    const Range rn(norm, 4), rws(ws, gdn_grad_workspace_bytes(count));
    if (rn.overlaps(rws)) return GDN_ERR_ALIAS;
    for (int i = 0; i < count; ++i) {
        const Range r(sizes[i] ? tensors[i] : nullptr, (size_t)sizes[i] * (is_bf16[i] ? 2 : 4));
        if (r.overlaps(rn) || r.overlaps(rws)) return GDN_ERR_ALIAS;
    }
    gdn::ClipTable t{};
    st = clip_squares(tensors, sizes, is_bf16, count, (double *)ws, t.all_parts, (hipStream_t)stream);
    if (st != GDN_OK) return st;
    t.parts = (const double *)ws;
    t.norm_out = norm;
    return launch(gdn::gdn_grad_norm_kernel, dim3(1), dim3(gdn::kClipThreads), 0, (hipStream_t)stream, t);
}

int gdn_grad_clip(const void *const *tensors, void *const *out, const int64_t *sizes, const int *is_bf16, int count,
                  const float *norm_in, float *norm, float max_norm, float eps, void *ws, size_t ws_bytes, void *stream) {
    int st = clip_check(tensors, sizes, is_bf16, count);
    if (st != GDN_OK) return st;
    if (count && !out) return GDN_ERR_NULL;
    if (!(max_norm >= 0.f) || !(eps >= 0.f)) return GDN_ERR_SHAPE;
    if (misaligned(norm_in, 4) || misaligned(norm, 4)) return GDN_ERR_ALIGN;
    const size_t need = norm_in ? 0 : gdn_grad_workspace_bytes(count);
    if (!ws_ok(ws, ws_bytes, need)) return GDN_ERR_WORKSPACE;
    const Range rws(need ? ws : nullptr, need), rn(norm, 4), ri(norm_in, 4);
    if (rn.overlaps(rws) || (rn.overlaps(ri) && !rn.same(ri))) return GDN_ERR_ALIAS;
    // Written ranges in the order of their addresses, each with the tensor it may coincide with: neighbours tell of
    // any overlap.
    try {
        struct Piece {
            uintptr_t lo, hi;
            int owner;
            bool written;
        };
        std::vector<Piece> all;
        all.reserve(2 * (size_t)count + 2);
        for (int i = 0; i < count; ++i) {
            if (!sizes[i]) continue;
            if (!out[i]) return GDN_ERR_NULL;
            if (misaligned(out[i], is_bf16[i] ? 2 : 4)) return GDN_ERR_ALIGN;
            const size_t bytes = (size_t)sizes[i] * (is_bf16[i] ? 2 : 4);
            const uintptr_t a = (uintptr_t)tensors[i], b = (uintptr_t)out[i];
            all.push_back({b, b + bytes, i, true});
            if (a != b) all.push_back({a, a + bytes, i, false});
        }
        if (norm) all.push_back({(uintptr_t)norm, (uintptr_t)norm + 4, -1, true});
        else if (norm_in) all.push_back({(uintptr_t)norm_in, (uintptr_t)norm_in + 4, -1, false});
        if (norm && norm_in && norm != norm_in) all.push_back({(uintptr_t)norm_in, (uintptr_t)norm_in + 4, -2, false});
        if (need) all.push_back({(uintptr_t)ws, (uintptr_t)ws + need, -3, true});
        std::sort(all.begin(), all.end(), [](const Piece &a, const Piece &b) { return a.lo < b.lo; });
        uintptr_t read_to = 0, write_to = 0;
        for (const Piece &p : all) {
            if (p.lo < write_to || (p.written && p.lo < read_to)) return GDN_ERR_ALIAS;
            (p.written ? write_to : read_to) = std::max(p.written ? write_to : read_to, p.hi);
        }
    } catch (const std::bad_alloc &) {
        return GDN_ERR_WORKSPACE;
    }
    int parts = 0;
    if (!norm_in) {
        st = clip_squares(tensors, sizes, is_bf16, count, (double *)ws, parts, (hipStream_t)stream);
        if (st != GDN_OK) return st;
    }
    if (parts > kClipOwnSums) {
        gdn::ClipTable t{};
        t.parts = (const double *)ws;
        t.all_parts = parts;
        t.norm_out = (float *)((unsigned char *)ws + clip_sums_bytes(count));
        st = launch(gdn::gdn_grad_norm_kernel, dim3(1), dim3(gdn::kClipThreads), 0, (hipStream_t)stream, t);
        if (st != GDN_OK) return st;
        norm_in = t.norm_out;
    }
    auto fill = [&](gdn::ClipTable &t) {
        t.parts = norm_in ? nullptr : (const double *)ws;
        t.all_parts = parts;
        t.norm_in = norm_in;
        t.max_norm = max_norm;
        t.eps = eps;
    };
    bool first = true;
    // (a norm that is norm_in stays as it is)
    st = clip_tables(tensors, out, sizes, is_bf16, count, [&](gdn::ClipTable &t) {
        fill(t);
        t.norm_out = first && norm != norm_in ? norm : nullptr;
        first = false;
        return launch(gdn::gdn_grad_scale_kernel, dim3((unsigned)t.groups), dim3(gdn::kClipThreads), 0, (hipStream_t)stream, t);
    });
    if (st == GDN_OK && first && norm && norm != norm_in) {          // nothing but empty tensors
        gdn::ClipTable t{};
        fill(t);
        t.norm_out = norm;
        st = launch(gdn::gdn_grad_norm_kernel, dim3(1), dim3(gdn::kClipThreads), 0, (hipStream_t)stream, t);
    }
    return st;
}

}  // extern "C"
