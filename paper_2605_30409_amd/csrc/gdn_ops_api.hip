// Host side of the operators in gdn_ops.h: argument validation, the choice of
// kernel variants, launches, and the extern "C" entry points.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <initializer_list>
#include <mutex>
#include <type_traits>

#include "gdn_backward.h"
#include "gdn_host.h"
#include "gdn_norm.h"
#include "gdn_ops.h"
#include "gdn_step.h"

namespace {

bool dims_ok(int Dk, int Dv) { return (Dk == 64 || Dk == 128) && (Dv == 64 || Dv == 128); }

// ---------------------------------------------------------------------------
// Recurrent step.

template <class E, int DK, int DV> int launch_step(const gdn::StepParams<E> &p, hipStream_t s) {
    const long long units = (long long)p.N * p.H * (DV / gdn::kStepCols);
    return launch(gdn::gdn_step_kernel<E, DK, DV>, dim3((unsigned)((units + gdn::kStepWaves - 1) / gdn::kStepWaves)),
                  dim3(64 * gdn::kStepWaves), 0, s, p);
}

template <class E>
int run_step(const void *q, const void *k, const void *v, const float *alpha, const float *beta, const float *state_in,
             const int *slots, const int *lengths, void *out, float *state_out, int N, int L, int P, int Hk, int H,
             int Dk, int Dv, hipStream_t s) {
    gdn::StepParams<E> p;
    p.q = (const E *)q;
    p.k = (const E *)k;
    p.v = (const E *)v;
    p.alpha = alpha;
    p.beta = beta;
    p.state_in = state_in;
    p.slots = slots;
    p.lengths = lengths;
    p.out = (E *)out;
    p.state_out = state_out;
    p.N = N;
    p.L = L;
    p.P = P;
    p.Hk = Hk;
    p.H = H;
    if (Dk == 128) return Dv == 128 ? launch_step<E, 128, 128>(p, s) : launch_step<E, 128, 64>(p, s);
    return Dv == 128 ? launch_step<E, 64, 128>(p, s) : launch_step<E, 64, 64>(p, s);
}

// ---------------------------------------------------------------------------
// Block norm.

constexpr int kNormMaxC = 8192;

// Threads that share a row: 8 channels each.
int norm_team(int C) {
    int t = 64;
    while (t * 8 < C) t *= 2;
    return t;
}

// How the gradient's rows are cut into strips (runs of consecutive rows whose
// sums one team keeps): as many as two workgroups of 256 threads a CU, and 512 of wider teams.
// Twice as many have twice the partial sums to write and add up: 54 + 5.7 us (kernel + sums)
// against 59.7 + 7.8 at 10560 x 2048 bf16, 335 + 14 against 370 + 35 at 200000 x 512; half
// as many 65.5 + 4.6 at 10560 x 2048, and 512 strips of narrow rows 721 + 5 at 200000 x 512.
struct Strips {
    int strips, strip_rows, per_unit, unit_rows;
};

Strips norm_strips(int R, int C, int gate_tokens) {
    const int rows = (R - 1) / std::max(512, (1 << 17) / norm_team(C)) + 1;
    Strips t;
    if (gate_tokens > rows) {             // a gate row spans strips: partial sums for dgate
        t.per_unit = (gate_tokens - 1) / rows + 1;
        t.strip_rows = (gate_tokens - 1) / t.per_unit + 1;
        t.per_unit = (gate_tokens - 1) / t.strip_rows + 1;
        t.unit_rows = gate_tokens;
        t.strips = R / gate_tokens * t.per_unit;
    } else {                              // strips of whole gate rows
        t.per_unit = 1;
        t.strip_rows = t.unit_rows = rows / gate_tokens * gate_tokens;
        t.strips = (R - 1) / t.strip_rows + 1;
    }
    return t;
}

bool norm_shape_ok(int R, int C, int gate_tokens) {
    return R >= 1 && C >= 1 && gate_tokens >= 1 && R % gate_tokens == 0;
}

template <class E, int TPR, bool SHORT = false> int launch_norm(const gdn::NormParams<E> &p, bool grad, hipStream_t s) {
    constexpr int threads = gdn::norm_threads<TPR>(), teams = threads / TPR;
    const dim3 grid((unsigned)((p.strips + teams - 1) / teams));
    if (!grad) return launch(gdn::gdn_block_norm_kernel<E, TPR, SHORT>, grid, dim3(threads), 0, s, p);
    const int st = launch(gdn::gdn_block_norm_grad_kernel<E, TPR, SHORT>, grid, dim3(threads), 0, s, p);
    if (st != GDN_OK) return st;
    const unsigned gates = p.gate && p.per_unit > 1 ? (unsigned)(p.R / p.gate_tokens) : 0u;
    return launch(gdn::gdn_block_norm_reduce_kernel<E>, dim3((unsigned)((2 * p.C + 63) / 64), 1 + gates),
                  dim3(64 * gdn::kNormReduceWaves), 0, s, p);
}

template <class E> int dispatch_norm(const gdn::NormParams<E> &p, bool grad, hipStream_t s) {
    if (p.C < 8) return launch_norm<E, 64, true>(p, grad, s);
    switch (norm_team(p.C)) {
    case 64: return launch_norm<E, 64>(p, grad, s);
    case 128: return launch_norm<E, 128>(p, grad, s);
    case 256: return launch_norm<E, 256>(p, grad, s);
    case 512: return launch_norm<E, 512>(p, grad, s);
    default: return launch_norm<E, 1024>(p, grad, s);
    }
}

// ---------------------------------------------------------------------------
// Gradient of the chunk forward.

// Byte offsets of the workspace regions (the records of gdn_backward.h).
struct BackWs {
    size_t gates, Tf, Tt, N0, C0, Hs, Gs, eT, vT, total;
};

BackWs back_layout(int B, int H, int T, int Dk, int Dv, size_t esz) {
    using gdn::kChunk;
    const size_t full = esz == 2 ? 6 : 4;     // bytes of an element in planes
    const size_t n = (size_t)B * H * (((size_t)T + kChunk - 1) / kChunk);
    BackWs L;
    size_t off = 0;
    auto region = [&](size_t bytes) {
        const size_t at = off;
        off = align256(off + n * bytes);
        return at;
    };
    L.gates = region(4 * gdn::kBackGateRec);
    L.Tf = region(full * kChunk * kChunk);
    L.Tt = region(full * kChunk * kChunk);
    L.N0 = region(4 * kChunk * Dv);
    L.C0 = region(4 * (size_t)Dk * Dv);
    L.Hs = region(4 * (size_t)Dk * Dv);
    L.Gs = region(4 * (size_t)Dk * Dv);
    L.eT = region(4 * kChunk * Dv);
    L.vT = region(4 * kChunk * Dv);
    L.total = off;
    return L;
}

bool back_shape_ok(int B, int H, int T) {
    // a launch has fewer than 2^32 threads; prep has 512 a chunk and head, the scan 6144 a head
    return B >= 1 && H >= 1 && T >= 1 && (long long)B * H <= 65535 &&
           (long long)B * H * ((T + (long long)gdn::kChunk - 1) / gdn::kChunk) < (1LL << 23);
}

template <class E, int DK, int DV> int launch_backward(const gdn::BackParams<E> &p, hipStream_t s) {
    using P = gdn::PrepLds<E, DK, DV>;
    // bf16, Dk = Dv = 128: a workgroup of the scan that brings all its operands through LDS has a CU
    // to itself; with first and add loaded directly two share one.  us at T = 3520, the ring's
    // first: 16 heads (one a CU) 103 and 109; 17 heads 175 and 152, 24 heads 196 and 194, 32 heads
    // 221 and 210; 4 x 31 heads of T = 1320 332 and 326.  Whole call: T = 1320, 17 heads 118 and 108, 24
    // 131 and 131, 32 169 and 172, 48 252 and 247, 64 333 and 345; T = 3520, 17 heads 293 and 276, 32 432
    // and 426.  Dv = 64 keeps the ring: T = 1320, 32 heads 118 and 120, 33 140 and 136, 40 153 and 154;
    // T = 3520, 32 heads 274 and 279, 33 334 and 338, 48 433 and 436.
    constexpr bool SHARE = sizeof(E) == 2 && DK == 128 && DV == 128;
    using S = gdn::BackScanLds<E, DK, false>;
    using D = gdn::BackScanLds<E, DK, SHARE>;
    using G = gdn::GradLds<E>;
    static std::once_flag once;
    static hipError_t attr = hipSuccess;
    std::call_once(once, [] {
        const struct {
            const void *fn;
            size_t bytes;
        } dyn[] = {{(const void *)gdn::gdn_back_prep_kernel<E, DK, DV>, P::bytes},
                   {(const void *)gdn::gdn_back_scan_kernel<E, DK, DV, false>, S::bytes},
                   {(const void *)gdn::gdn_back_scan_kernel<E, DK, DV, SHARE>, D::bytes},
                   {(const void *)gdn::gdn_back_grad_kernel<E, DK, DV, 1>, G::bytes},
                   {(const void *)gdn::gdn_back_grad_kernel<E, DK, DV, 2>, G::bytes}};
        for (const auto &d : dyn)
            if (attr == hipSuccess)
                attr = hipFuncSetAttribute(d.fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)d.bytes);
    });
    if (attr != hipSuccess) return GDN_ERR_HIP;
    const unsigned bh = (unsigned)(p.B * p.H), n = bh * (unsigned)p.NC;
    int st = launch(gdn::gdn_back_prep_kernel<E, DK, DV>, dim3(n), dim3(64 * gdn::kPrepWaves), P::bytes, s, p);
    const dim3 tiles((bh + 7) / 8 * 8 * (DV / 16), 2);
    if (st == GDN_OK && SHARE && 2LL * bh * (DV / 16) > 256)
        st = launch(gdn::gdn_back_scan_kernel<E, DK, DV, SHARE>, tiles, dim3(D::threads), D::bytes, s, p);
    else if (st == GDN_OK)
        st = launch(gdn::gdn_back_scan_kernel<E, DK, DV, false>, tiles, dim3(S::threads), S::bytes, s, p);
    // Up to a workgroup a CU they have eight waves; where CUs get a second one, four.  us with 8 and
    // 4: 256 workgroups
    // of bf16, D = 64 16.2, 18.4; D = 128 27.1, 30.8; fp32, D = 64 25.1, 27.8; 512 of them
    // 31.8, 26.1; 55.7, 46.9; 48.3, 40.8.  Whole call at 192, 256, 264, 320, 384 workgroups, bf16, D = 128: 72, 83,
    // 107, 116, 129 and 75, 86, 98, 108, 121; fp32, D = 64: 78, 93, 117, 129, 142 and 81, 95, 109, 121, 135.
    if (st == GDN_OK)
        st = n <= 256 ? launch(gdn::gdn_back_grad_kernel<E, DK, DV, 2>, dim3(n), dim3(512), G::bytes, s, p)
                      : launch(gdn::gdn_back_grad_kernel<E, DK, DV, 1>, dim3(n), dim3(256), G::bytes, s, p);
    return st;
}

template <class E> int dispatch_backward(const gdn::BackParams<E> &p, int Dk, int Dv, hipStream_t s) {
    if (Dk == 128) return Dv == 128 ? launch_backward<E, 128, 128>(p, s) : launch_backward<E, 128, 64>(p, s);
    return Dv == 128 ? launch_backward<E, 64, 128>(p, s) : launch_backward<E, 64, 64>(p, s);
}

}  // namespace

extern "C" {

size_t gdn_chunk_backward_workspace_bytes(int B, int H, int T, int Dk, int Dv, int chunk, int is_bf16) {
    if (!back_shape_ok(B, H, T) || !dims_ok(Dk, Dv) || chunk != gdn::kChunk) return 0;
    return back_layout(B, H, T, Dk, Dv, is_bf16 ? 2 : 4).total;
}

int gdn_chunk_backward(const void *q, const void *k, const void *v, const float *alpha, const float *beta,
                       const float *state_in, const void *dout, const float *dstate_out, void *dq,
                       void *dk, void *dv, float *dalpha, float *dbeta, float *dstate_in, int B, int H,
                       int T, int Dk, int Dv, int chunk, int is_bf16, void *ws, size_t ws_bytes,
                       void *stream) {
    if (!q || !k || !v || !alpha || !beta || !dout || !dq || !dk || !dv || !dalpha || !dbeta) return GDN_ERR_NULL;
    if (!back_shape_ok(B, H, T)) return GDN_ERR_SHAPE;
    if (!dims_ok(Dk, Dv) || chunk != gdn::kChunk) return GDN_ERR_UNSUPPORTED;
    for (const void *p : {q, k, v, (const void *)alpha, (const void *)beta, (const void *)state_in, dout,
                          (const void *)dstate_out, (const void *)dq, (const void *)dk, (const void *)dv,
                          (const void *)dalpha, (const void *)dbeta, (const void *)dstate_in})
        if (misaligned(p)) return GDN_ERR_ALIGN;
    const size_t esz = is_bf16 ? 2 : 4, n = (size_t)B * T * H, sb = (size_t)B * H * Dk * Dv * 4;
    const BackWs L = back_layout(B, H, T, Dk, Dv, esz);
    if (!ws || misaligned(ws, 256) || ws_bytes < L.total) return GDN_ERR_WORKSPACE;
    const Range in[] = {Range(q, n * Dk * esz), Range(k, n * Dk * esz), Range(v, n * Dv * esz), Range(alpha, n * 4),
                        Range(beta, n * 4), Range(state_in, sb), Range(dout, n * Dv * esz), Range(dstate_out, sb)};
    const Range outs[] = {Range(dq, n * Dk * esz), Range(dk, n * Dk * esz), Range(dv, n * Dv * esz), Range(dalpha, n * 4),
                          Range(dbeta, n * 4), Range(dstate_in, sb), Range(ws, L.total)};
    for (int i = 0; i < 7; ++i) {
        for (int j = 0; j < 8; ++j)
            if (outs[i].overlaps(in[j]) && !(i == 5 && j == 7 && outs[i].same(in[j]))) return GDN_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (outs[i].overlaps(outs[j])) return GDN_ERR_ALIAS;
    }
    auto run = [&](auto *e) {
        using E = std::remove_pointer_t<decltype(e)>;
        unsigned char *base = (unsigned char *)ws;
        gdn::BackParams<E> p;
        p.q = (const E *)q;
        p.k = (const E *)k;
        p.v = (const E *)v;
        p.dout = (const E *)dout;
        p.alpha = alpha;
        p.beta = beta;
        p.state_in = state_in;
        p.dstate_out = dstate_out;
        p.dq = (E *)dq;
        p.dk = (E *)dk;
        p.dv = (E *)dv;
        p.dalpha = dalpha;
        p.dbeta = dbeta;
        p.dstate_in = dstate_in;
        p.B = B;
        p.H = H;
        p.T = T;
        p.NC = (int)((T + (long long)gdn::kChunk - 1) / gdn::kChunk);
        p.gates = (float *)(base + L.gates);
        p.N0 = (float *)(base + L.N0);
        p.C0 = (float *)(base + L.C0);
        p.Tf = (E *)(base + L.Tf);
        p.Tt = (E *)(base + L.Tt);
        p.Hs = (float *)(base + L.Hs);
        p.Gs = (float *)(base + L.Gs);
        p.eT = (float *)(base + L.eT);
        p.vT = (float *)(base + L.vT);
        return dispatch_backward<E>(p, Dk, Dv, (hipStream_t)stream);
    };
    return is_bf16 ? run((uint16_t *)nullptr) : run((float *)nullptr);
}

int gdn_step_forward(const void *q, const void *k, const void *v, const float *alpha, const float *beta,
                     const float *state_in, const int *slots, const int *lengths, void *out,
                     float *state_out, int N, int L, int P, int Hk, int H, int Dk, int Dv, int is_bf16,
                     void *stream) {
    if (!q || !k || !v || !alpha || !beta || !state_in || !out || !state_out) return GDN_ERR_NULL;
    if (N < 1 || L < 1 || P < 1 || Hk < 1 || H < 1 || H % Hk || (!slots && N > P)) return GDN_ERR_SHAPE;
    if ((long long)N * H >= (1LL << 24)) return GDN_ERR_SHAPE;      // 256 threads each, below 2^32 a launch
    if (!dims_ok(Dk, Dv)) return GDN_ERR_UNSUPPORTED;
    for (const void *p : {q, k, v, (const void *)alpha, (const void *)beta, (const void *)state_in, (const void *)out,
                          (const void *)state_out})
        if (misaligned(p)) return GDN_ERR_ALIGN;
    if (misaligned(slots, 4) || misaligned(lengths, 4)) return GDN_ERR_ALIGN;
    const size_t esz = is_bf16 ? 2 : 4, nt = (size_t)N * L;
    const Range ro(out, nt * H * Dv * esz), rs(state_out, (size_t)P * H * Dk * Dv * 4),
        ri(state_in, (size_t)P * H * Dk * Dv * 4);
    for (const Range &r : {Range(q, nt * Hk * Dk * esz), Range(k, nt * Hk * Dk * esz), Range(v, nt * H * Dv * esz),
                           Range(alpha, nt * H * 4), Range(beta, nt * H * 4), Range(slots, (size_t)N * 4),
                           Range(lengths, (size_t)N * 4)})
        if (ro.overlaps(r) || rs.overlaps(r)) return GDN_ERR_ALIAS;
    if (ro.overlaps(rs) || ro.overlaps(ri) || (rs.overlaps(ri) && !rs.same(ri))) return GDN_ERR_ALIAS;
    const auto run = is_bf16 ? run_step<uint16_t> : run_step<float>;
    return run(q, k, v, alpha, beta, state_in, slots, lengths, out, state_out, N, L, P, Hk, H, Dk, Dv,
               (hipStream_t)stream);
}

int gdn_block_norm_forward(const void *x, const void *y, const void *gate, const float *w_post,
                           const float *w_pre, void *r, void *u, int R, int C, int gate_tokens,
                           float res_scale, float eps, int is_bf16, void *stream) {
    if (!x || !y || !w_post || !w_pre || !r || !u) return GDN_ERR_NULL;
    if (!norm_shape_ok(R, C, gate_tokens)) return GDN_ERR_SHAPE;
    if (C > kNormMaxC) return GDN_ERR_UNSUPPORTED;
    for (const void *p : {x, y, gate, (const void *)w_post, (const void *)w_pre, (const void *)r, (const void *)u})
        if (misaligned(p)) return GDN_ERR_ALIGN;
    const size_t bytes = (size_t)R * C * (is_bf16 ? 2 : 4);
    const Range rx(x, bytes), ry(y, bytes), rr(r, bytes), ru(u, bytes);
    for (const Range &o : {Range(gate, bytes / gate_tokens), Range(w_post, (size_t)C * 4), Range(w_pre, (size_t)C * 4)})
        if (rr.overlaps(o) || ru.overlaps(o)) return GDN_ERR_ALIAS;
    if (rr.overlaps(ru) || ru.overlaps(rx) || (ru.overlaps(ry) && !ru.same(ry)) ||
        (rr.overlaps(rx) && !rr.same(rx)) || (rr.overlaps(ry) && !rr.same(ry)))
        return GDN_ERR_ALIAS;
    auto run = [&](auto *e) {
        using E = std::remove_pointer_t<decltype(e)>;
        gdn::NormParams<E> p{};
        p.x = (const E *)x;
        p.y = (const E *)y;
        p.gate = (const E *)gate;
        p.w_post = w_post;
        p.w_pre = w_pre;
        p.r = (E *)r;
        p.u = (E *)u;
        p.R = R;
        p.C = C;
        p.gate_tokens = gate_tokens;
        // Up to 2048 teams a row each; then longer strips, for the next row's loads to be on their way, but
        // short ones: a new team's loads run beside an old one's stores.  us at 10560 x 2048 bf16 with
        // 1, 2, 3, 4 and 6 rows: 40, 33, 31, 30.5, 33; 100000 x 2048 with 3, 4, 6, 8 and 49: 364, 373, 386,
        // 383, 428; 30000 x 8192 (teams of 1024) with 1, 2, 4, 6, 8 and 15: 566, 437, 381, 363, 366, 377.
        // Past 2^31 threads (rows of up to 512 channels from 2^27 on) strips grow with the rows: a launch
        // has fewer than 2^32.
        p.strip_rows = std::min((R - 1) / 2048 + 1, norm_team(C) < 1024 ? 4 : 8);
        p.strip_rows = std::max(p.strip_rows, (R - 1) / (INT32_MAX / norm_team(C)) + 1);
        p.strips = (R - 1) / p.strip_rows + 1;
        p.res_scale = res_scale;
        p.eps = eps;
        return dispatch_norm<E>(p, false, (hipStream_t)stream);
    };
    return is_bf16 ? run((uint16_t *)nullptr) : run((float *)nullptr);
}

size_t gdn_block_norm_workspace_bytes(int R, int C, int gate_tokens) {
    if (!norm_shape_ok(R, C, gate_tokens) || C > kNormMaxC) return 0;
    const Strips t = norm_strips(R, C, gate_tokens);
    return align256((size_t)t.strips * 2 * C * 4) + align256(t.per_unit > 1 ? (size_t)t.strips * C * 4 : 0);
}

int gdn_block_norm_backward(const void *x, const void *y, const void *gate, const float *w_post,
                            const float *w_pre, const void *du, const void *dr, void *dx, void *dy,
                            void *dgate, float *dw_post, float *dw_pre, int R, int C, int gate_tokens,
                            float res_scale, float eps, int is_bf16, void *ws, size_t ws_bytes,
                            void *stream) {
    if (!x || !y || !w_post || !w_pre || !du || !dx || !dy || !dw_post || !dw_pre || !gate != !dgate) return GDN_ERR_NULL;
    if (!norm_shape_ok(R, C, gate_tokens)) return GDN_ERR_SHAPE;
    if (C > kNormMaxC) return GDN_ERR_UNSUPPORTED;
    for (const void *p : {x, y, gate, (const void *)w_post, (const void *)w_pre, du, dr, (const void *)dx,
                          (const void *)dy, (const void *)dgate, (const void *)dw_post, (const void *)dw_pre})
        if (misaligned(p)) return GDN_ERR_ALIGN;
    if (!ws || misaligned(ws, 256) || ws_bytes < gdn_block_norm_workspace_bytes(R, C, gate_tokens))
        return GDN_ERR_WORKSPACE;
    const size_t bytes = (size_t)R * C * (is_bf16 ? 2 : 4), wb = (size_t)C * 4;
    const Range in[] = {Range(x, bytes), Range(gate, bytes / gate_tokens), Range(w_post, wb), Range(w_pre, wb),
                        Range(y, bytes), Range(du, bytes), Range(dr, bytes)};
    const Range outs[] = {Range(dx, bytes), Range(dy, bytes), Range(dgate, bytes / gate_tokens), Range(dw_post, wb),
                          Range(dw_pre, wb), Range(ws, gdn_block_norm_workspace_bytes(R, C, gate_tokens))};
    for (int i = 0; i < 6; ++i) {
        for (int j = 0; j < 7; ++j) {
            // a row's y, du and dr are in registers before its dx and dy are written
            const bool shared = (i == 0 && j >= 5) || (i == 1 && j >= 4);
            if (outs[i].overlaps(in[j]) && !(shared && outs[i].same(in[j]))) return GDN_ERR_ALIAS;
        }
        for (int j = 0; j < i; ++j)
            if (outs[i].overlaps(outs[j])) return GDN_ERR_ALIAS;
    }
    auto run = [&](auto *e) {
        using E = std::remove_pointer_t<decltype(e)>;
        const Strips t = norm_strips(R, C, gate_tokens);
        gdn::NormParams<E> p{};
        p.x = (const E *)x;
        p.y = (const E *)y;
        p.gate = (const E *)gate;
        p.w_post = w_post;
        p.w_pre = w_pre;
        p.du = (const E *)du;
        p.dr = (const E *)dr;
        p.dx = (E *)dx;
        p.dy = (E *)dy;
        p.dgate = (E *)dgate;
        p.dw_post = dw_post;
        p.dw_pre = dw_pre;
        p.part_w = (float *)ws;
        p.part_g = (float *)((unsigned char *)ws + align256((size_t)t.strips * 2 * C * 4));
        p.R = R;
        p.C = C;
        p.gate_tokens = gate_tokens;
        p.strips = t.strips;
        p.strip_rows = t.strip_rows;
        p.per_unit = t.per_unit;
        p.unit_rows = t.unit_rows;
        p.res_scale = res_scale;
        p.eps = eps;
        return dispatch_norm<E>(p, true, (hipStream_t)stream);
    };
    return is_bf16 ? run((uint16_t *)nullptr) : run((float *)nullptr);
}

}  // extern "C"
