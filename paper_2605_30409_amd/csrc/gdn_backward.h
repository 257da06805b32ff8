// Gradient of the token-wise chunk forward (gdn_chunk_backward in gdn_ops.h).
//
// Notation, per batch and head and for a chunk of C = 64 tokens with entry
// state H (= S^T, [Dk][Dv]) and G = dL/d(exit state): g_i the running sum of
// log alpha in the chunk, D_ij = e^{g_i - g_j} (j <= i), gam_i = e^{g_i}, tail_i =
// e^{g_C - g_i}, and "strict" the part below the diagonal.  The forward is
//   N  = strict(D o K K^T) diag(beta),   T = (I + N)^{-1}
//   e  = T (V - gam K H)                 (what a token writes, before beta)
//   H' = e^{g_C} H + K^T (tail beta e),  O = gam Q H + (D o Q K^T) (beta e)
// and its gradient, with A = D o Q K^T:
//   dV = T^T (beta (A^T dO + tail K G))
//   G  <- e^{g_C} G + Q^T (gam dO) - K^T (gam dV)                (dL/dH)
//   Z  = dO e^T,  F = dV e^T,  G1 = D o Z diag(beta),  G2 = strict(D o F) diag(beta)
//   PQ = dO H^T,  PV = dV H^T,  PE = e G^T
//   dQ = gam PQ + G1 K
//   dK = G1^T Q + tail beta PE - gam PV - (G2 + G2^T) K
//   dbeta_j  = sum_{i >= j} D_ij (q_i.k_j) Z_ij - sum_{i > j} D_ij (k_i.k_j) F_ij + tail_j k_j.PE_j
//   dalpha_t = sum_{i >= t} D_it sum_{j < t} D_{t-1,j} X_ij
// where X_ij = beta_j ((q_i.k_j) Z_ij - (k_i.k_j) F_ij) is what the pair (i, j)
// adds to the loss per unit of decay between them; j = -1 is the entry state
// (X_i,-1 = q_i.PQ_i - k_i.PV_i, decay gam_{t-1}) and a last row i = C the exit state
// (X_C,j = beta_j k_j.PE_j, X_C,-1 = <G, H>, decay tail_t).  With the decays on
// either side of alpha_t as two factors nothing is divided by alpha, so alpha = 0 has
// its gradient too, and nothing by beta.
//
// Three launches: per chunk the gates, T and the operands of the scans
// (gdn_back_prep_kernel); the scans over chunks, states forward and their gradients
// backward side by side (gdn_back_scan_kernel); per chunk all that remains
// (gdn_back_grad_kernel).
//
// Precision: gate gradients and states are fp32 results, and so every operand
// that is not itself an input keeps 16 bits of mantissa or more.  On the bf16
// path such a "wide" operand is a pair of bf16 planes, x = hi + lo with hi = bf16(x)
// and lo = bf16(x - hi) (off by at most 2^-18 |x|); a product with an input takes two bf16
// MFMAs and one of two wide operands three (the fourth, lo lo, is below what lo
// was rounded by).  On the fp32 path it is fp32 and all products are fp32 MFMAs.
#pragma once

#include "gdn_device.h"

namespace gdn {

// A wide operand fragment: 8 consecutive k per lane, like Tr<E>::frag.
template <class E> struct Wide;
template <> struct Wide<uint16_t> {
    using T = Tr<uint16_t>;
    struct frag {
        u32x4 hi, lo;
    };
    static constexpr int planes = 2;
    static __device__ __forceinline__ f32x4 hi_of(u32x2 h) { return T::to_f32(h); }
    static __device__ __forceinline__ void store4(uint16_t *p, size_t plane, f32x4 x) {
        const u32x2 h = T::from_f32(x);
        T::store(p, h);
        T::store(p + plane, T::from_f32(x - T::to_f32(h)));
    }
    static __device__ __forceinline__ void store1(uint16_t *p, size_t plane, float x) {
        const uint32_t h = pack_bf16x2(x, 0.f);
        p[0] = (uint16_t)h;
        p[plane] = (uint16_t)pack_bf16x2(x - __uint_as_float(h << 16), 0.f);
    }
    static __device__ __forceinline__ frag split(f32x4 a, f32x4 b) {
        const u32x2 ha = T::from_f32(a), hb = T::from_f32(b);
        return frag{T::cat(ha, hb), T::cat(T::from_f32(a - T::to_f32(ha)), T::from_f32(b - T::to_f32(hb)))};
    }
    static __device__ __forceinline__ frag load8(const uint16_t *p, size_t plane) {
        return frag{T::load8(p), T::load8(p + plane)};
    }
    static __device__ __forceinline__ void store8(uint16_t *p, size_t plane, frag f) {
        T::store8(p, f.hi);
        T::store8(p + plane, f.lo);
    }
    static __device__ __forceinline__ frag tr(const uint16_t *M, size_t plane, int ld, int row0, int col, int li, int lg) {
        return frag{tr_frag<uint16_t>(M, ld, row0, col, false, 0, li, lg),
                    tr_frag<uint16_t>(M + plane, ld, row0, col, false, 0, li, lg)};
    }
    static __device__ __forceinline__ void values(frag f, f32x4 &a, f32x4 &b) {
        a = T::to_f32(T::lo(f.hi)) + T::to_f32(T::lo(f.lo));
        b = T::to_f32(T::hi(f.hi)) + T::to_f32(T::hi(f.lo));
    }
    static __device__ __forceinline__ f32x4 ew(u32x4 a, frag b, f32x4 c) { return T::mma(a, b.hi, T::mma(a, b.lo, c)); }
    static __device__ __forceinline__ f32x4 we(frag a, u32x4 b, f32x4 c) { return T::mma(a.hi, b, T::mma(a.lo, b, c)); }
    static __device__ __forceinline__ f32x4 ww(frag a, frag b, f32x4 c) {
        return T::mma(a.hi, b.hi, T::mma(a.hi, b.lo, T::mma(a.lo, b.hi, c)));
    }
    // the value rounded to the storage type, as an output fragment
    static __device__ __forceinline__ u32x4 rounded(frag f) { return f.hi; }
};
template <> struct Wide<float> {
    using T = Tr<float>;
    using frag = f32x8;
    static constexpr int planes = 1;
    static __device__ __forceinline__ void store4(float *p, size_t, f32x4 x) { T::store(p, x); }
    static __device__ __forceinline__ void store1(float *p, size_t, float x) { *p = x; }
    static __device__ __forceinline__ frag split(f32x4 a, f32x4 b) { return T::cat(a, b); }
    static __device__ __forceinline__ frag load8(const float *p, size_t) { return T::load8(p); }
    static __device__ __forceinline__ void store8(float *p, size_t, frag f) { T::store8(p, f); }
    static __device__ __forceinline__ frag tr(const float *M, size_t, int ld, int row0, int col, int li, int lg) {
        return tr_frag<float>(M, ld, row0, col, false, 0, li, lg);
    }
    static __device__ __forceinline__ void values(frag f, f32x4 &a, f32x4 &b) { a = T::lo(f), b = T::hi(f); }
    static __device__ __forceinline__ f32x4 ew(frag a, frag b, f32x4 c) { return T::mma(a, b, c); }
    static __device__ __forceinline__ f32x4 we(frag a, frag b, f32x4 c) { return T::mma(a, b, c); }
    static __device__ __forceinline__ f32x4 ww(frag a, frag b, f32x4 c) { return T::mma(a, b, c); }
    static __device__ __forceinline__ frag rounded(frag f) { return f; }
};

// Gate record of a chunk, in floats: g as 64 doubles, gam, tail and beta, e^{g_C}.
constexpr int kBackGam = 128, kBackTail = 192, kBackBeta = 256, kBackGC = 320, kBackGateRec = 336;

// Workspace records per (b*H + h, chunk).  "Wide" regions take 4 bytes an element on
// either path (two planes of bf16, the second n elements behind the first, or fp32).
//   gates [336] fp32
//   Tf, Tt  64 x 64   wide, fragments: [4 row tile][2 k block][64 lane][8] of T and T^T
//   Kt, Qt  Dk x 64   E, fragments [Dk/16][2][64][8] of K^T and Q^T
//   N0      64 x Dv   fp32, beta A^T dO as accumulator tiles [Dv/16][4][64 lane][4]
//   Gd      64 x Dv   wide, gam dO as fragments [Dv/16][2][64][8] (k = token)
//   Hs, Gs  Dk x Dv   wide, row-major: H and G of the chunk
//   eT, vT  Dv x 64   wide, row-major: e^T and dV^T
template <class E> struct BackParams {
    const E *q, *k, *v, *dout;
    const float *alpha, *beta, *state_in, *dstate_out;
    E *dq, *dk, *dv;
    float *dalpha, *dbeta, *dstate_in;
    int B, H, T, NC;
    float *gates, *N0;
    E *Tf, *Tt, *Kt, *Qt, *Gd, *Hs, *Gs, *eT, *vT;
};

template <class E> constexpr int wide_elems(int n) { return n * Wide<E>::planes; }

// Padded leading dimension of an LDS tile with rows of n elements of E.
template <class E> constexpr int lds_ld(int n) { return n + 16 / (int)sizeof(E); }

// --------------------------------------------------------------------------
// Stage 1, per chunk and head: gates, T, and the operands of the scans.
// --------------------------------------------------------------------------
template <class E, int DK, int DV> struct PrepLds {
    static constexpr int LDK = lds_ld<E>(DK), LDV = lds_ld<E>(DV), LDA = kChunk + 4, LDT = lds_ld<E>(kChunk);
    static constexpr size_t oK = 0;
    static constexpr size_t oQ = oK + sizeof(E) * kChunk * LDK;
    static constexpr size_t oO = oQ + sizeof(E) * kChunk * LDK;
    static constexpr size_t oN = oO + sizeof(E) * kChunk * LDV;    // N, fp32
    static constexpr size_t oT = oN + 4 * kChunk * LDA;            // T, fp32
    static constexpr size_t oA = oT + 4 * kChunk * LDA;            // A^T, wide
    static constexpr size_t oG = oA + sizeof(E) * Wide<E>::planes * kChunk * LDT;
    static constexpr size_t bytes = oG + 8 * kChunk + 2 * 4 * kChunk;
};

constexpr int kPrepWaves = 8;

// Lower tile t = 0..9 of a 4 x 4 grid of tiles: row and column tile.
__device__ __forceinline__ void lower_tile(int t, int &bi, int &bj) {
    bi = (t >= 6) ? 3 : (t >= 3) ? 2 : (t >= 1) ? 1 : 0;
    bj = t - bi * (bi + 1) / 2;
}

// 16-byte vectors of a [64][D] tile of token rows into LDS, rows past nvalid as zeros.
template <class E, int D, int NT>
__device__ __forceinline__ void stage_rows(const E *src, size_t rstride, int nvalid, E *dst, int ld, int tid) {
    constexpr int VE = 16 / (int)sizeof(E), NVEC = kChunk * (D / VE);
#pragma unroll
    for (int i0 = 0; i0 < NVEC; i0 += NT) {
        const int idx = tid + i0, r = idx / (D / VE), cv = idx % (D / VE);
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (r < nvalid) x = *(const uint4 *)(src + r * rstride + cv * VE);
        *(uint4 *)(dst + r * ld + cv * VE) = x;
    }
}

template <class E, int DK, int DV>
__global__ __launch_bounds__(64 * kPrepWaves) void gdn_back_prep_kernel(BackParams<E> p) {
    using L = PrepLds<E, DK, DV>;
    using TR = Tr<E>;
    using WD = Wide<E>;
    constexpr int NT = 64 * kPrepWaves;
    constexpr size_t PA = (size_t)kChunk * L::LDT;      // plane of A^T
    extern __shared__ __align__(16) unsigned char smem[];
    E *sK = (E *)(smem + L::oK), *sQ = (E *)(smem + L::oQ), *sO = (E *)(smem + L::oO), *sA = (E *)(smem + L::oA);
    float *sN = (float *)(smem + L::oN), *sT = (float *)(smem + L::oT);
    double *sg = (double *)(smem + L::oG);
    float *sb = (float *)(sg + kChunk), *sgam = sb + kChunk;
    const int c = blockIdx.x / (p.B * p.H), bh = blockIdx.x - c * (p.B * p.H);
    const int b = bh / p.H, h = bh - b * p.H;
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, li = l & 15, lg = l >> 4;
    const int t0 = c * kChunk, nvalid = min(kChunk, p.T - t0);
    const size_t cidx = (size_t)bh * p.NC + c;
    const size_t row0 = ((size_t)b * p.T + t0) * p.H + h;
    float *gate = p.gates + cidx * kBackGateRec;

    if (w == 0) {
        float a = 1.f, be = 0.f;
        if (l < nvalid) {
            a = p.alpha[row0 + (size_t)l * p.H];
            be = p.beta[row0 + (size_t)l * p.H];
        }
        float la = logf(a);
        la = (la < kLogAlphaMin) ? kLogAlphaMin : la;   // keeps NaN
        double g = (double)la;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const double o = __shfl_up(g, d);
            if (l >= d) g += o;
        }
        const double gC = __shfl(g, kChunk - 1);
        const float gam = expf((float)g);
        sg[l] = g;
        sb[l] = be;
        sgam[l] = gam;
        ((double *)gate)[l] = g;
        gate[kBackGam + l] = gam;
        gate[kBackTail + l] = expf((float)(gC - g));
        gate[kBackBeta + l] = be;
        if (l == 0) gate[kBackGC] = expf((float)gC);
    }
    stage_rows<E, DK, NT>(p.k + row0 * DK, (size_t)p.H * DK, nvalid, sK, L::LDK, tid);
    stage_rows<E, DK, NT>(p.q + row0 * DK, (size_t)p.H * DK, nvalid, sQ, L::LDK, tid);
    stage_rows<E, DV, NT>(p.dout + row0 * DV, (size_t)p.H * DV, nvalid, sO, L::LDV, tid);
    // the tiles of A^T and T that stay empty are read as zeros
    for (int i = tid; i < (int)(L::oG - L::oT) / 4; i += NT) ((float *)(smem + L::oT))[i] = 0.f;
    lds_barrier();

    // N and A^T: ten lower tiles each
    for (int t = w; t < 20; t += kPrepWaves) {
        int bi, bj;
        lower_tile(t % 10, bi, bj);
        const E *rows = t < 10 ? sK : sQ;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb)
            acc = TR::mma(load_frag<E>(rows + (16 * bi + li) * L::LDK + 32 * kb, lg),
                          load_frag<E>(sK + (16 * bj + li) * L::LDK + 32 * kb, lg), acc);
        const int j = 16 * bj + li, i0 = 16 * bi + 4 * lg;
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[q] = j <= i0 + q ? acc[q] * expf((float)(sg[i0 + q] - sg[j])) : 0.f;
        if (t < 10) {
#pragma unroll
            for (int q = 0; q < 4; ++q) sN[(i0 + q) * L::LDA + j] = j < i0 + q ? acc[q] * sb[j] : 0.f;
        } else {
            WD::store4(sA + j * L::LDT + i0, PA, acc);
        }
    }
    lds_barrier();

    // T = (I + N)^{-1}: the diagonal blocks by substitution (lane = block * 16 +
    // column) on wave 0, while the others write the operands that do not need T.
    if (w == 0) {
        const int base = 16 * lg;
        float x[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float acc = (r == li) ? 1.f : 0.f;
#pragma unroll
            for (int s = 0; s < r; ++s) acc -= sN[(base + r) * L::LDA + base + s] * x[s];
            x[r] = acc;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) sT[(base + r) * L::LDA + base + li] = x[r];
    } else {
        E *Kt = p.Kt + cidx * (size_t)DK * kChunk, *Qt = p.Qt + cidx * (size_t)DK * kChunk;
        for (int f = w - 1; f < 2 * (DK / 16) * 2; f += kPrepWaves - 1) {
            const int which = f & 1, kb = (f >> 1) & 1, t = f >> 2;
            TR::store8((which ? Qt : Kt) + (size_t)(t * 2 + kb) * 512 + l * 8,
                       tr_frag<E>(which ? sQ : sK, L::LDK, 32 * kb, 16 * t, false, 0, li, lg));
        }
        E *Gd = p.Gd + cidx * (size_t)wide_elems<E>(kChunk * DV);
        for (int f = w - 1; f < (DV / 16) * 2; f += kPrepWaves - 1) {
            const int kb = f & 1, jt = f >> 1;
            const typename TR::frag o = tr_frag<E>(sO, L::LDV, 32 * kb, 16 * jt, false, 0, li, lg);
            const float *gm = sgam + 32 * kb + 8 * lg;
            WD::store8(Gd + (size_t)(jt * 2 + kb) * 512 + l * 8, (size_t)kChunk * DV,
                       WD::split(TR::to_f32(TR::lo(o)) * *(const f32x4 *)gm, TR::to_f32(TR::hi(o)) * *(const f32x4 *)(gm + 4)));
        }
        float *N0 = p.N0 + cidx * (size_t)kChunk * DV;
        for (int f = w - 1; f < (DV / 16) * 4; f += kPrepWaves - 1) {
            const int rt = f & 3, jt = f >> 2;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
                if (kb >= rt / 2)                        // rows i >= j only
                    acc = WD::we(WD::load8(sA + (16 * rt + li) * L::LDT + 32 * kb + 8 * lg, PA),
                                 tr_frag<E>(sO, L::LDV, 32 * kb, 16 * jt, false, 0, li, lg), acc);
            const f32x4 bq = *(const f32x4 *)(sb + 16 * rt + 4 * lg);
            *(f32x4 *)(N0 + (size_t)(jt * 4 + rt) * 256 + l * 4) = acc * bq;
        }
    }
    lds_barrier();
    // Off-diagonal blocks by block distance: T_ij = -T_ii sum_{m=j}^{i-1} N_im T_mj.
    for (int dist = 1; dist < 4; ++dist) {
        if (w < 4 - dist) {
            const int j = w, i = w + dist;
            f32x4 X = {0.f, 0.f, 0.f, 0.f};
            for (int m = j; m < i; ++m) {
                const f32x4 a = *(const f32x4 *)(sN + (16 * i + li) * L::LDA + 16 * m + 4 * lg);
#pragma unroll
                for (int q = 0; q < 4; ++q) X = mma_f32_k4(a[q], sT[(16 * m + 4 * lg + q) * L::LDA + 16 * j + li], X);
            }
            const f32x4 a = *(const f32x4 *)(sT + (16 * i + li) * L::LDA + 16 * i + 4 * lg);
            f32x4 Y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int q = 0; q < 4; ++q) Y = mma_f32_k4(a[q], X[q], Y);
#pragma unroll
            for (int q = 0; q < 4; ++q) sT[(16 * i + 4 * lg + q) * L::LDA + 16 * j + li] = -Y[q];
        }
        lds_barrier();
    }
    // T and T^T as fragments: one of 16 per wave and turn
    for (int f = w; f < 16; f += kPrepWaves) {
        const int kb = f & 1, rt = (f >> 1) & 3;
        f32x4 x[2];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int k = 32 * kb + 8 * lg + e, r = 16 * rt + li;
            x[e >> 2][e & 3] = f < 8 ? sT[r * L::LDA + k] : sT[k * L::LDA + r];
        }
        E *dst = (f < 8 ? p.Tf : p.Tt) + cidx * (size_t)wide_elems<E>(kChunk * kChunk);
        WD::store8(dst + (size_t)(rt * 2 + kb) * 512 + l * 8, (size_t)kChunk * kChunk, WD::split(x[0], x[1]));
    }
}

// --------------------------------------------------------------------------
// Stage 2: the scans.  A workgroup of four waves carries 16 columns of one
// state through the chunks: blockIdx.y = 0 the states forward, 1 their gradients
// backward.  Each product's rows are split over the waves, and its result goes
// to all of them through LDS (as [column][row], so a result tile is stored in
// quads and read back as operand rows).
// --------------------------------------------------------------------------
constexpr int kBackScanWaves = 4;

template <class E, int DK> struct BackScanLds {
    static constexpr int LDH = lds_ld<E>(DK), LDC = lds_ld<E>(kChunk);
    static constexpr size_t PH = 16 * (size_t)LDH, PC = 16 * (size_t)LDC;     // planes
    static constexpr size_t oX = sizeof(E) * Wide<E>::planes * PH;            // first exchange
    static constexpr size_t oY = oX + sizeof(E) * Wide<E>::planes * PC;       // second
    static constexpr size_t bytes = oY + sizeof(E) * Wide<E>::planes * PC;
};

// Operands of one chunk, loaded ahead of their use.
template <class E, int DK, bool REV> struct BackOps {
    static constexpr int NT = DK / 64;                  // state row tiles per wave
    typename Tr<E>::frag K[DK / 32], Kt[NT][2], Qt[REV ? NT : 1][2];
    typename Wide<E>::frag T[2], Gd[REV ? 2 : 1];
    f32x4 first, scale, out;                            // V or N0; per-token factors
    float gC;
};

template <class E, int DK, int DV, bool REV>
__device__ __forceinline__ void back_load(const BackParams<E> &p, BackOps<E, DK, REV> &o, int b, int h, int bh, int jt,
                                          int c, int w, int l) {
    using TR = Tr<E>;
    using WD = Wide<E>;
    const int li = l & 15, lg = l >> 4;
    const size_t cidx = (size_t)bh * p.NC + c;
    const int t0 = c * kChunk, nvalid = min(kChunk, p.T - t0);
    const size_t row0 = ((size_t)b * p.T + t0) * p.H + h;
    const int r = 16 * w + li;
#pragma unroll
    for (int kb = 0; kb < DK / 32; ++kb)
        o.K[kb] = r < nvalid ? load_frag<E>(p.k + (row0 + (size_t)r * p.H) * DK + 32 * kb, lg)
                             : TR::cat(TR::zero(), TR::zero());
    const E *Tm = (REV ? p.Tt : p.Tf) + cidx * (size_t)wide_elems<E>(kChunk * kChunk);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) o.T[kb] = WD::load8(Tm + (size_t)(w * 2 + kb) * 512 + l * 8, (size_t)kChunk * kChunk);
    const E *Kt = p.Kt + cidx * (size_t)DK * kChunk, *Qt = p.Qt + cidx * (size_t)DK * kChunk;
#pragma unroll
    for (int t = 0; t < DK / 64; ++t)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const size_t at = (size_t)((w * (DK / 64) + t) * 2 + kb) * 512 + l * 8;
            o.Kt[t][kb] = TR::load8(Kt + at);
            if (REV) o.Qt[t][kb] = TR::load8(Qt + at);
        }
    const float *gate = p.gates + cidx * kBackGateRec + 16 * w + 4 * lg;
    const f32x4 gam = *(const f32x4 *)(gate + kBackGam), tail = *(const f32x4 *)(gate + kBackTail),
                be = *(const f32x4 *)(gate + kBackBeta);
    o.gC = p.gates[cidx * kBackGateRec + kBackGC];
    if constexpr (REV) {
        const E *Gd = p.Gd + cidx * (size_t)wide_elems<E>(kChunk * DV);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) o.Gd[kb] = WD::load8(Gd + (size_t)(jt * 2 + kb) * 512 + l * 8, (size_t)kChunk * DV);
        o.first = *(const f32x4 *)(p.N0 + cidx * (size_t)kChunk * DV + (size_t)(jt * 4 + w) * 256 + l * 4);
        o.scale = be * tail;
        o.out = -gam;
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int t = 16 * w + 4 * lg + q;
            float x = 0.f;
            if (t < nvalid) {
                const E e = p.v[(row0 + (size_t)t * p.H) * DV + 16 * jt + li];
                if constexpr (sizeof(E) == 2) x = __uint_as_float((uint32_t)e << 16);
                else x = e;
            }
            o.first[q] = x;
        }
        o.scale = -gam;
        o.out = be * tail;
    }
}

// A 16 x 16 tile of LDS matrix X [column][row] (row tile at row0) into memory as
// [row][column] with row stride ld.
template <class E>
__device__ __forceinline__ void store_transposed(const E *X, size_t xplane, int xld, int row0, E *dst, size_t dplane,
                                                 int ld, int li, int lg) {
    if constexpr (sizeof(E) == 2) {
        typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
#pragma unroll
        for (int pl = 0; pl < 2; ++pl) {
            // lane li of a 16-lane group receives column li of rows 4 lg .. 4 lg + 3 of X
            const i16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_i16x4 *)(X + pl * xplane + (4 * lg + (li >> 2)) * xld + row0 + 4 * (li & 3)));
            *(u32x2 *)(dst + pl * dplane + (size_t)(row0 + li) * ld + 4 * lg) = __builtin_bit_cast(u32x2, v);
        }
    } else {
        f32x4 v;
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = X[(4 * lg + q) * xld + row0 + li];
        *(f32x4 *)(dst + (size_t)(row0 + li) * ld + 4 * lg) = v;
    }
}

template <class E, int DK, int DV, bool REV>
__device__ __forceinline__ void back_scan(const BackParams<E> &p, unsigned char *smem, int bh, int jt) {
    using L = BackScanLds<E, DK>;
    using WD = Wide<E>;
    constexpr int NT = DK / 64;
    E *sH = (E *)smem, *sX = (E *)(smem + L::oX), *sY = (E *)(smem + L::oY);
    const int b = bh / p.H, h = bh - b * p.H;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, li = l & 15, lg = l >> 4;
    const float *init = REV ? p.dstate_out : p.state_in;
    const size_t sbase = (size_t)bh * DK * DV + 16 * jt + li;
    f32x4 st[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            st[t][q] = init ? init[sbase + (size_t)(16 * (w * NT + t) + 4 * lg + q) * DV] : 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t) WD::store4(sH + li * L::LDH + 16 * (w * NT + t) + 4 * lg, L::PH, st[t]);

    auto step = [&](const BackOps<E, DK, REV> &o, int c) {
        const size_t cidx = (size_t)bh * p.NC + c;
        lds_barrier();
        // the state that enters this step, for stage 3
        E *keep = (REV ? p.Gs : p.Hs) + cidx * (size_t)wide_elems<E>(DK * DV) + 16 * jt;
#pragma unroll
        for (int t = 0; t < NT; ++t)
            store_transposed<E>(sH, L::PH, L::LDH, 16 * (w * NT + t), keep, (size_t)DK * DV, DV, li, lg);
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb)
            x = WD::ew(o.K[kb], WD::load8(sH + li * L::LDH + 32 * kb + 8 * lg, L::PH), x);
        WD::store4(sX + li * L::LDC + 16 * w + 4 * lg, L::PC, o.first + o.scale * x);
        lds_barrier();
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
            if (REV ? kb >= w / 2 : kb <= w / 2)         // T is lower triangular
                y = WD::ww(o.T[kb], WD::load8(sX + li * L::LDC + 32 * kb + 8 * lg, L::PC), y);
        WD::store4(sY + li * L::LDC + 16 * w + 4 * lg, L::PC, o.out * y);
        E *res = (REV ? p.vT : p.eT) + cidx * (size_t)wide_elems<E>(kChunk * DV);
        WD::store4(res + (size_t)(16 * jt + li) * kChunk + 16 * w + 4 * lg, (size_t)kChunk * DV, y);
        lds_barrier();
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            st[t] *= o.gC;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                if constexpr (REV) st[t] = WD::ew(o.Qt[t][kb], o.Gd[kb], st[t]);
                st[t] = WD::ew(o.Kt[t][kb], WD::load8(sY + li * L::LDC + 32 * kb + 8 * lg, L::PC), st[t]);
            }
            WD::store4(sH + li * L::LDH + 16 * (w * NT + t) + 4 * lg, L::PH, st[t]);
        }
    };
    auto chunk = [&](int i) { return REV ? p.NC - 1 - i : i; };
    BackOps<E, DK, REV> o0, o1;
    back_load<E, DK, DV, REV>(p, o0, b, h, bh, jt, chunk(0), w, l);
    for (int i = 0; i < p.NC; i += 2) {
        if (i + 1 < p.NC) back_load<E, DK, DV, REV>(p, o1, b, h, bh, jt, chunk(i + 1), w, l);
        step(o0, chunk(i));
        if (i + 1 == p.NC) break;
        if (i + 2 < p.NC) back_load<E, DK, DV, REV>(p, o0, b, h, bh, jt, chunk(i + 2), w, l);
        step(o1, chunk(i + 1));
    }
    if (REV && p.dstate_in) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                p.dstate_in[sbase + (size_t)(16 * (w * NT + t) + 4 * lg + q) * DV] = st[t][q];
    }
}

template <class E, int DK, int DV>
__global__ __launch_bounds__(64 * kBackScanWaves) __attribute__((amdgpu_waves_per_eu(1, 1)))
void gdn_back_scan_kernel(BackParams<E> p) {
    __shared__ __align__(16) unsigned char smem[BackScanLds<E, DK>::bytes];
    // the column tiles of a head share its operands: they get the same XCD
    constexpr int NJ = DV / 16;
    const int u = blockIdx.x >> 3, jt = u % NJ, bh = (u / NJ) * 8 + (blockIdx.x & 7);
    if (bh >= p.B * p.H) return;
    if (blockIdx.y == 0) back_scan<E, DK, DV, false>(p, smem, bh, jt);
    else back_scan<E, DK, DV, true>(p, smem, bh, jt);
}

// --------------------------------------------------------------------------
// Stage 3, per chunk and head: dQ, dK, dV, dalpha and dbeta.  Wave w has the 16
// key channels from 16 w on in the products over Dk; the 64 x 64 products are
// dealt out as tiles.
// --------------------------------------------------------------------------
template <class E, int DK, int DV> struct GradLds {
    static constexpr int LDC = lds_ld<E>(kChunk);
    static constexpr size_t PV = (size_t)DV * LDC, PC = (size_t)kChunk * LDC;
    static constexpr int NW = DK / 16;
    static constexpr size_t szV = sizeof(E) * Wide<E>::planes * PV, szC = sizeof(E) * Wide<E>::planes * PC;
    static constexpr size_t oE = 0;                     // e^T
    static constexpr size_t oV = oE + szV;              // dV^T
    static constexpr size_t oG1 = oV + szV;             // G1^T
    static constexpr size_t oX = oG1 + szC;             // X^T, its row 0 the exit state's
    static constexpr size_t oG2 = oX + szC;             // G2 + G2^T
    static constexpr size_t oD = oG2 + szC;             // D_{t-1,j}
    static constexpr size_t oGate = oD + szC;           // the gate record
    static constexpr size_t oRed = oGate + 4 * kBackGateRec;
    // floats behind oRed: [NW][64] X_i,-1, [NW][64] k.PE, [4][64] column sums of dbeta, [4][64] of
    // dalpha, [64] X_i,-1 summed, [64] exit-state part of dalpha, [NW] parts of <G, H>
    static constexpr size_t bytes = oRed + 4 * (2 * NW * 64 + 10 * 64 + 16);
};

template <class E, int DK, int DV>
__global__ __launch_bounds__(64 * (DK / 16)) void gdn_back_grad_kernel(BackParams<E> p) {
    using L = GradLds<E, DK, DV>;
    using TR = Tr<E>;
    using WD = Wide<E>;
    using frag = typename TR::frag;
    using wfrag = typename WD::frag;
    constexpr int NW = L::NW, NT = 64 * NW;
    extern __shared__ __align__(16) unsigned char smem[];
    E *sE = (E *)(smem + L::oE), *sV = (E *)(smem + L::oV), *sG1 = (E *)(smem + L::oG1), *sX = (E *)(smem + L::oX),
      *sG2 = (E *)(smem + L::oG2), *sD = (E *)(smem + L::oD);
    const double *sg = (const double *)(smem + L::oGate);
    const float *gate = (const float *)(smem + L::oGate);
    const float *gam = gate + kBackGam, *tail = gate + kBackTail, *beta = gate + kBackBeta;
    float *rX = (float *)(smem + L::oRed), *rE = rX + NW * 64, *cb = rE + NW * 64, *ca = cb + 4 * 64, *xm = ca + 4 * 64,
          *cC = xm + 64, *gh = cC + 64;
    const int c = blockIdx.x / (p.B * p.H), bh = blockIdx.x - c * (p.B * p.H);
    const int b = bh / p.H, h = bh - b * p.H;
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, li = l & 15, lg = l >> 4;
    const int t0 = c * kChunk, nvalid = min(kChunk, p.T - t0);
    const size_t cidx = (size_t)bh * p.NC + c;
    const size_t row0 = ((size_t)b * p.T + t0) * p.H + h;
    auto rows = [&](const E *base, int D, int r, int kb) {          // row fragment of an input
        return r < nvalid ? load_frag<E>(base + (row0 + (size_t)r * p.H) * D + 32 * kb, lg) : TR::cat(TR::zero(), TR::zero());
    };

    // e^T and dV^T, gates; G1^T and X^T are zero where no tile writes them
    {
        constexpr int VE = 16 / (int)sizeof(E), NV = wide_elems<E>(kChunk * DV) / VE;
        const E *ge = p.eT + cidx * (size_t)wide_elems<E>(kChunk * DV), *gv = p.vT + cidx * (size_t)wide_elems<E>(kChunk * DV);
#pragma unroll 4
        for (int i = tid; i < NV; i += NT) {
            const int r = i / (kChunk / VE), cv = i % (kChunk / VE), pl = r / DV;    // rows of plane 0, then 1
            const size_t at = (size_t)pl * L::PV + (size_t)(r - pl * DV) * L::LDC + cv * VE;
            *(uint4 *)(sE + at) = *(const uint4 *)(ge + (size_t)i * VE);
            *(uint4 *)(sV + at) = *(const uint4 *)(gv + (size_t)i * VE);
        }
        for (int i = tid; i < kBackGateRec; i += NT) ((float *)(smem + L::oGate))[i] = p.gates[cidx * kBackGateRec + i];
        for (int i = tid; i < (int)(2 * L::szC / 4); i += NT) ((float *)(smem + L::oG1))[i] = 0.f;
    }
    lds_barrier();

    // D_{t-1,j}: thread (t, 8 j)
    for (int i = tid; i < 64 * 8; i += NT) {
        const int t = i >> 3, j0 = 8 * (i & 7);
        f32x4 x[2];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e >> 2][e & 3] = j0 + e < t ? expf((float)(sg[t > 0 ? t - 1 : 0] - sg[j0 + e])) : 0.f;
        WD::store8(sD + t * L::LDC + j0, L::PC, WD::split(x[0], x[1]));
    }

    // PQ, PV, PE transposed: tiles [16 key channels][16 tokens]
    f32x4 pq[4], pv[4], pe[4];
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) pq[rt] = pv[rt] = pe[rt] = f32x4{0.f, 0.f, 0.f, 0.f};
    {
        const size_t sb = cidx * (size_t)wide_elems<E>(DK * DV) + (size_t)(16 * w + li) * DV + 8 * lg;
        f32x4 dot = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < DV / 32; ++kb) {
            const wfrag H = WD::load8(p.Hs + sb + 32 * kb, (size_t)DK * DV), G = WD::load8(p.Gs + sb + 32 * kb, (size_t)DK * DV);
            f32x4 ha, hb, ga, gb;
            WD::values(H, ha, hb);
            WD::values(G, ga, gb);
            dot += ha * ga + hb * gb;
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) {
                pq[rt] = WD::we(H, rows(p.dout, DV, 16 * rt + li, kb), pq[rt]);
                pv[rt] = WD::ww(H, WD::tr(sV, L::PV, L::LDC, 32 * kb, 16 * rt, li, lg), pv[rt]);
                pe[rt] = WD::ww(G, WD::tr(sE, L::PV, L::LDC, 32 * kb, 16 * rt, li, lg), pe[rt]);
            }
        }
        float s = dot[0] + dot[1] + dot[2] + dot[3];
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d);
        if (l == 0) gh[w] = s;
    }
    // q.PQ - k.PV and k.PE of this wave's channels; then the parts of dQ and dK that
    // come from the states
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) {
        const int t = 16 * rt + li;
        f32x4 q4 = {0.f, 0.f, 0.f, 0.f}, k4 = q4;
        if (t < nvalid) {
            const size_t at = (row0 + (size_t)t * p.H) * DK + 16 * w + 4 * lg;
            q4 = TR::to_f32(TR::load(p.q + at));
            k4 = TR::to_f32(TR::load(p.k + at));
        }
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            x += q4[q] * pq[rt][q] - k4[q] * pv[rt][q];
            y += k4[q] * pe[rt][q];
        }
        x += __shfl_xor(x, 16);
        x += __shfl_xor(x, 32);
        y += __shfl_xor(y, 16);
        y += __shfl_xor(y, 32);
        if (lg == 0) {
            rX[w * 64 + t] = x;
            rE[w * 64 + t] = y;
        }
        pq[rt] *= gam[t];
        pe[rt] = pe[rt] * (tail[t] * beta[t]) - pv[rt] * gam[t];
    }
    // The 64 x 64 products, lower tiles: element (i, j) with i = 16 bi + 4 lg + q, j = 16 bj + li.
    for (int t = w; t < 10; t += NW) {
        int bi, bj;
        lower_tile(t, bi, bj);
        f32x4 sqk = {0.f, 0.f, 0.f, 0.f}, skk = sqk, z = sqk, f = sqk;
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb) {
            const frag kj = rows(p.k, DK, 16 * bj + li, kb);
            sqk = TR::mma(rows(p.q, DK, 16 * bi + li, kb), kj, sqk);
            skk = TR::mma(rows(p.k, DK, 16 * bi + li, kb), kj, skk);
        }
#pragma unroll
        for (int kb = 0; kb < DV / 32; ++kb) {
            const wfrag ej = WD::tr(sE, L::PV, L::LDC, 32 * kb, 16 * bj, li, lg);
            z = WD::ew(rows(p.dout, DV, 16 * bi + li, kb), ej, z);
            f = WD::ww(WD::tr(sV, L::PV, L::LDC, 32 * kb, 16 * bi, li, lg), ej, f);
        }
        const int j = 16 * bj + li, i0 = 16 * bi + 4 * lg;
        const float bj_ = beta[j];
        f32x4 g1, g2, xx;
        float cs = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int i = i0 + q;
            const float d = i >= j ? expf((float)(sg[i] - sg[j])) : 0.f;
            const float dz = d * z[q], df = i > j ? d * f[q] : 0.f;
            g1[q] = dz * bj_;
            g2[q] = df * bj_;
            xx[q] = i > j ? bj_ * (sqk[q] * z[q] - skk[q] * f[q]) : 0.f;
            cs += sqk[q] * dz - skk[q] * df;
        }
        WD::store4(sG1 + j * L::LDC + i0, L::PC, g1);
        WD::store4(sX + j * L::LDC + i0, L::PC, xx);
        if (bi != bj) {
            WD::store4(sG2 + j * L::LDC + i0, L::PC, g2);
#pragma unroll
            for (int q = 0; q < 4; ++q) WD::store1(sG2 + (i0 + q) * L::LDC + j, L::PC, g2[q]);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (i0 + q < j) continue;                // written from below the diagonal
                WD::store1(sG2 + (i0 + q) * L::LDC + j, L::PC, g2[q]);
                if (i0 + q > j) WD::store1(sG2 + j * L::LDC + i0 + q, L::PC, g2[q]);
            }
        }
        cs += __shfl_xor(cs, 16);
        cs += __shfl_xor(cs, 32);
        if (lg == 0) cb[bi * 64 + j] = cs;
    }
    lds_barrier();

    // Sums over the waves: dbeta, X's border row and column
    if (tid < 64) {
        float y = 0.f, x = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            x += rX[i * 64 + tid];
            y += rE[i * 64 + tid];
        }
        xm[tid] = x;
        float d = tail[tid] * y;
        for (int bi = tid >> 4; bi < 4; ++bi) d += cb[bi * 64 + tid];
        if (tid < nvalid) p.dbeta[row0 + (size_t)tid * p.H] = d;
        WD::store1(sX + tid * L::LDC, L::PC, beta[tid] * y);
    }
    // dQ += G1 K;  dK += G1^T Q - (G2 + G2^T) K
    {
        const E *Kt = p.Kt + cidx * (size_t)DK * kChunk + l * 8, *Qt = p.Qt + cidx * (size_t)DK * kChunk + l * 8;
        frag kt[2], qt[2], km[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            kt[kb] = TR::load8(Kt + (size_t)(w * 2 + kb) * 512);
            qt[kb] = TR::load8(Qt + (size_t)(w * 2 + kb) * 512);
            if constexpr (sizeof(E) == 2) km[kb] = kt[kb] ^ 0x80008000u;     // -K^T
            else km[kb] = -kt[kb];
        }
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) {
            f32x4 dq = pq[rt], dk = pe[rt];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                if (kb <= rt / 2) dq = WD::ew(kt[kb], WD::tr(sG1, L::PC, L::LDC, 32 * kb, 16 * rt, li, lg), dq);
                if (kb >= rt / 2) dk = WD::ew(qt[kb], WD::load8(sG1 + (16 * rt + li) * L::LDC + 32 * kb + 8 * lg, L::PC), dk);
                dk = WD::ew(km[kb], WD::load8(sG2 + (16 * rt + li) * L::LDC + 32 * kb + 8 * lg, L::PC), dk);
            }
            const int t = 16 * rt + li;
            if (t < nvalid) {
                const size_t at = (row0 + (size_t)t * p.H) * DK + 16 * w + 4 * lg;
                TR::store(p.dq + at, TR::from_f32(dq));
                TR::store(p.dk + at, TR::from_f32(dk));
            }
        }
    }
    // dV from its transpose
    for (int f = w; f < 4 * (DV / 32); f += NW) {
        const int rt = f & 3, kb = f >> 2, t = 16 * rt + li;
        const frag x = WD::rounded(WD::tr(sV, L::PV, L::LDC, 32 * kb, 16 * rt, li, lg));
        if (t < nvalid) TR::store8(p.dv + (row0 + (size_t)t * p.H) * DV + 32 * kb + 8 * lg, x);
    }
    lds_barrier();
    // dalpha: M_it = sum_j X_ij D_{t-1,j}, then D_it M_it summed over rows; row 0 of X is the
    // exit state's (its own has no j < 0), so row tile 0 is needed for every t
    for (int f = w; f < 16; f += NW) {
        const int bi = f >> 2, bt = f & 3;
        if (bt > bi && bi != 0) continue;
        f32x4 m = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
            if (kb <= bt / 2)
                m = WD::ww(WD::tr(sX, L::PC, L::LDC, 32 * kb, 16 * bi, li, lg),
                           WD::load8(sD + (16 * bt + li) * L::LDC + 32 * kb + 8 * lg, L::PC), m);
        const int t = 16 * bt + li, i0 = 16 * bi + 4 * lg;
        const float gb = t > 0 ? gam[t - 1] : 1.f;
        if (bi == 0 && lg == 0) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < NW; ++i) s += gh[i];
            cC[t] = tail[t] * (m[0] + s * gb);
        }
        float cs = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int i = i0 + q;
            if (i == 0) m[q] = 0.f;
            if (i >= t) cs += expf((float)(sg[i] - sg[t])) * (m[q] + xm[i] * gb);
        }
        cs += __shfl_xor(cs, 16);
        cs += __shfl_xor(cs, 32);
        if (lg == 0 && bt <= bi) ca[bi * 64 + t] = cs;
    }
    lds_barrier();
    if (tid < nvalid) {
        float d = cC[tid];
        for (int bi = tid >> 4; bi < 4; ++bi) d += ca[bi * 64 + tid];
        p.dalpha[row0 + (size_t)tid * p.H] = d;
    }
}

}  // namespace gdn
