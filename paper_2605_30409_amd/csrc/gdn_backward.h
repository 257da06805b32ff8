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
// (gdn_back_grad_kernel).  bf16, Dk = Dv = 128, us and MB between the L2 caches and memory:
//                      prep         scan          grad
//   T = 3520,  H = 16   42, 175     103, 338       90, 278
//   T = 10560, H = 16  108, 523     319, 1011     255, 833
// A large copy reaches 4.7 TB/s: prep is there, the last launch and the scan, at 3.2, are not: the scan waits for
// its exchanges (its arithmetic alone, without loads and stores, takes 79 us of the 100).
//
// Precision: gate gradients and states are fp32 results, and dQ and dK sums whose terms
// may cancel, so what leads to them
// keeps fp32's mantissa.  On the bf16 path an operand that is not itself an input
// is cut into three bf16 planes, x = hi + mid + lo exactly (8 bits of mantissa
// each, denormals aside); a product with an input takes three bf16 MFMAs and one of two
// such operands six (the terms left out are below 2^-25).  That is 48 and 96 cycles where
// fp32 MFMAs take 256.  Two planes, tried first, left 2e-6 to 4e-6 of error in
// the fp32 results; fp32 evaluation has 2e-7 to 3e-7.  On the fp32 path
// operands are fp32 and all products fp32 MFMAs.
#pragma once

#include <type_traits>

#include "gdn_device.h"

namespace gdn {

// An operand fragment in P planes (8 consecutive k per lane, like Tr<E>::frag).
template <class E, int P> struct Wide;
template <int P> struct Wide<uint16_t, P> {
    using T = Tr<uint16_t>;
    static constexpr int planes = P;
    struct frag {
        u32x4 pl[P];
    };
    static __device__ __forceinline__ void store4(uint16_t *p, int plane, f32x4 x) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const u32x2 h = T::from_f32(x);
            T::store(p + i * plane, h);
            x -= T::to_f32(h);
        }
    }
    static __device__ __forceinline__ void store1(uint16_t *p, int plane, float x) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const uint32_t h = pack_bf16x2(x, 0.f);
            p[i * plane] = (uint16_t)h;
            x -= __uint_as_float(h << 16);
        }
    }
    static __device__ __forceinline__ frag split(f32x4 a, f32x4 b) {
        frag f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const u32x2 ha = T::from_f32(a), hb = T::from_f32(b);
            f.pl[i] = T::cat(ha, hb);
            a -= T::to_f32(ha);
            b -= T::to_f32(hb);
        }
        return f;
    }
    template <class I> static __device__ __forceinline__ frag load8(const uint16_t *p, I plane) {
        frag f;
#pragma unroll
        for (int i = 0; i < P; ++i) f.pl[i] = T::load8(p + i * plane);
        return f;
    }
    template <class I> static __device__ __forceinline__ void store8(uint16_t *p, I plane, frag f) {
#pragma unroll
        for (int i = 0; i < P; ++i) T::store8(p + i * plane, f.pl[i]);
    }
    static __device__ __forceinline__ frag tr(const uint16_t *M, int plane, int ld, int row0, int col, int li, int lg) {
        frag f;
#pragma unroll
        for (int i = 0; i < P; ++i) f.pl[i] = tr_frag<uint16_t>(M + i * plane, ld, row0, col, false, 0, li, lg);
        return f;
    }
    // products, the smallest terms first: e an input's fragment, w one in planes
    static __device__ __forceinline__ f32x4 ew(u32x4 a, const frag &b, f32x4 c) {
#pragma unroll
        for (int i = P - 1; i >= 0; --i) c = T::mma(a, b.pl[i], c);
        return c;
    }
    static __device__ __forceinline__ f32x4 we(const frag &a, u32x4 b, f32x4 c) {
#pragma unroll
        for (int i = P - 1; i >= 0; --i) c = T::mma(a.pl[i], b, c);
        return c;
    }
    static __device__ __forceinline__ f32x4 ww(const frag &a, const frag &b, f32x4 c) {
#pragma unroll
        for (int s = P - 1; s >= 0; --s)
#pragma unroll
            for (int i = 0; i <= s; ++i) c = T::mma(a.pl[i], b.pl[s - i], c);
        return c;
    }
    // the value rounded to the storage type
    static __device__ __forceinline__ u32x4 rounded(const frag &f) { return f.pl[0]; }
};
template <int P> struct Wide<float, P> {
    using T = Tr<float>;
    using frag = f32x8;
    static constexpr int planes = 1;
    static __device__ __forceinline__ void store4(float *p, int, f32x4 x) { T::store(p, x); }
    static __device__ __forceinline__ void store1(float *p, int, float x) { *p = x; }
    static __device__ __forceinline__ frag split(f32x4 a, f32x4 b) { return T::cat(a, b); }
    template <class I> static __device__ __forceinline__ frag load8(const float *p, I) { return T::load8(p); }
    template <class I> static __device__ __forceinline__ void store8(float *p, I, frag f) { T::store8(p, f); }
    static __device__ __forceinline__ frag tr(const float *M, int, int ld, int row0, int col, int li, int lg) {
        return tr_frag<float>(M, ld, row0, col, false, 0, li, lg);
    }
    static __device__ __forceinline__ f32x4 ew(frag a, frag b, f32x4 c) { return T::mma(a, b, c); }
    static __device__ __forceinline__ f32x4 we(frag a, frag b, f32x4 c) { return T::mma(a, b, c); }
    static __device__ __forceinline__ f32x4 ww(frag a, frag b, f32x4 c) { return T::mma(a, b, c); }
    static __device__ __forceinline__ frag rounded(frag f) { return f; }
};
// One contraction block of R = 32 or 16 state rows per wave: an input's operand (R / 4
// consecutive k per lane) and the state's accumulator tiles as the other one in planes.
template <class E, int R> struct RowBlock;
template <class E> struct RowBlock<E, 32> {            // tiles in P32 order
    using in = typename Tr<E>::frag;
    using planes = typename Wide<E, 3>::frag;
    static __device__ __forceinline__ planes split(const f32x4 *st) { return Wide<E, 3>::split(st[0], st[1]); }
    static __device__ __forceinline__ f32x4 product(const planes &a, in b) {
        return Wide<E, 3>::we(a, b, f32x4{0.f, 0.f, 0.f, 0.f});
    }
};
template <> struct RowBlock<uint16_t, 16> {
    using T = Tr<uint16_t>;
    using in = u32x2;
    struct planes {
        u32x2 pl[3];
    };
    static __device__ __forceinline__ planes split(const f32x4 *st) {
        planes f;
        f32x4 x = st[0];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            f.pl[i] = T::from_f32(x);
            x -= T::to_f32(f.pl[i]);
        }
        return f;
    }
    static __device__ __forceinline__ f32x4 product(const planes &a, in b) {
        f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 2; i >= 0; --i)
            c = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(i16x4, a.pl[i]), __builtin_bit_cast(i16x4, b), c, 0, 0, 0);
        return c;
    }
};
template <> struct RowBlock<float, 16> {
    using in = f32x4;
    using planes = f32x4;
    static __device__ __forceinline__ planes split(const f32x4 *st) { return st[0]; }
    static __device__ __forceinline__ f32x4 product(const planes &a, in b) {
        f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; ++i) c = mma_f32_k4(a[i], b[i], c);
        return c;
    }
};

// Transposes the 4 x 4 values that 4 neighbouring lanes hold in 4 elements each.
__device__ __forceinline__ f32x4 quad_transpose(f32x4 x, int l) {
    auto other = [](float v, auto sel) {                   // the value of lane ^ 1 (0xb1) or lane ^ 2 (0x4e)
        return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), decltype(sel)::value, 0xf, 0xf, true));
    };
    const std::integral_constant<int, 0xb1> one{};
    const std::integral_constant<int, 0x4e> two{};
    const bool o = l & 1, h = l & 2;
#pragma unroll
    for (int r = 0; r < 4; r += 2) {
        const float t = other(o ? x[r] : x[r + 1], one);
        x[r] = o ? t : x[r];
        x[r + 1] = o ? x[r + 1] : t;
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const float t = other(h ? x[r] : x[r + 2], two);
        x[r] = h ? t : x[r];
        x[r + 2] = h ? x[r + 2] : t;
    }
    return x;
}

template <class E> using Full = Wide<E, 3>;    // fp32's mantissa

__device__ __forceinline__ float elem_f32(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float elem_f32(float x) { return x; }

// Gate record of a chunk, in floats: g log2(e) as a sum of two, tail, beta; then, what the scans
// take, gam, beta tail and e^{g_C}.
constexpr int kBackGHi = 0, kBackGLo = 64, kBackTail = 128, kBackBeta = 192, kBackGam = 256, kBackBt = 320, kBackGC = 384, kBackGateRec = 400;
constexpr int kBackScanGates = 132;    // floats of it from kBackGam on that the scans copy

// Workspace records per (b*H + h, chunk); "planes": three of bf16, each behind the
// whole of the one before, on the bf16 path, fp32 on the other.
//   gates [400] fp32
//   Tf, Tt  64 x 64   planes, fragments [4 row tile][2 k block][64 lane][8] of T and T^T (those
//                     that are all zeros are neither written nor read)
//   N0      64 x Dv   fp32, beta A^T dO as transposed accumulator tiles [Dv/16][4 token tile][64 lane][4]
//   C0      Dk x Dv   fp32, Q^T gam dO as accumulator tiles [Dv/16][4 wave][Dk/64][64 lane][4]
//   Hs, Gs  Dk x Dv   fp32: H and G of the chunk, [Dv/16][Dk rows][16], the rows of each wave's 32 (Dk =
//                     128) in P32 order, tile after tile
//   eT, vT  Dv x 64   fp32, row-major: e^T and dV^T
template <class E> struct BackParams {
    const E *q, *k, *v, *dout;
    const float *alpha, *beta, *state_in, *dstate_out;
    E *dq, *dk, *dv;
    float *dalpha, *dbeta, *dstate_in;
    int B, H, T, NC;
    float *gates, *N0, *C0, *Hs, *Gs, *eT, *vT;
    E *Tf, *Tt;
};

template <class E> constexpr int full_elems(int n) { return n * Full<E>::planes; }

// D_ij = e^{g_i - g_j} from g log2(e) in two floats: the difference is as exact as its own rounding,
// where one float would have that of g (5600 after a chunk of alpha ~ 0).
__device__ __forceinline__ float back_decay(const float *gate, int i, int j) {
    return __builtin_amdgcn_exp2f((gate[kBackGHi + i] - gate[kBackGHi + j]) + (gate[kBackGLo + i] - gate[kBackGLo + j]));
}

// Padded leading dimension of an LDS tile with rows of n elements of E.
template <class E> constexpr int lds_ld(int n) { return n + 16 / (int)sizeof(E); }

// --------------------------------------------------------------------------
// Stage 1, per chunk and head: gates, T, and the operands of the scans.
// --------------------------------------------------------------------------
// LDS: K rows (dO takes their place once N and A are formed), Q rows, N below the diagonal and T^T
// on and above it in one fp32 square, A^T: 79 KB on the bf16 path at D = 128, two
// workgroups a CU.
template <class E, int DK, int DV> struct PrepLds {
    static constexpr int LDK = lds_ld<E>(DK), LDV = lds_ld<E>(DV), LDA = kChunk + 4, LDT = lds_ld<E>(kChunk);
    static constexpr size_t oK = 0;                                // K, then dO
    static constexpr size_t oQ = oK + sizeof(E) * kChunk * (LDK > LDV ? LDK : LDV);
    static constexpr size_t oN = oQ + sizeof(E) * kChunk * LDK;
    static constexpr size_t oA = oN + 4 * kChunk * LDA;            // A^T, planes
    static constexpr size_t oG = oA + sizeof(E) * Full<E>::planes * kChunk * LDT;
    static constexpr size_t bytes = oG + 8 * kChunk + 2 * 4 * kChunk;
    // waves per SIMD of the eight-wave workgroups that fit a CU
    static constexpr int waves_per_simd = bytes * 2 <= 160 * 1024 ? 4 : 2;
};

// (Four waves a SIMD have 128 registers; one or two more are spilled in bf16 and at fp32 heads of 64.)
constexpr int kPrepWaves = 8;

// Lower tile t = 0..9 of a 4 x 4 grid of tiles: row and column tile.
__device__ __forceinline__ void lower_tile(int t, int &bi, int &bj) {
    bi = (t >= 6) ? 3 : (t >= 3) ? 2 : (t >= 1) ? 1 : 0;
    bj = t - bi * (bi + 1) / 2;
}

// A [64][D] tile of token rows in 16-byte vectors: NT threads read it into registers (rows
// past nvalid as the last one) and write it to LDS (those rows as zeros).
template <class E, int D, int NT> struct RowTile {
    static constexpr int VE = 16 / (int)sizeof(E), N = kChunk * (D / VE) / NT;
    static_assert(N * NT == kChunk * (D / VE), "whole vectors per thread");
    uint4 x[N];
    __device__ __forceinline__ void load(const E *src, size_t rstride, int nvalid, int tid) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int idx = tid + i * NT, r = min(idx / (D / VE), nvalid - 1);
            x[i] = *(const uint4 *)(src + r * rstride + idx % (D / VE) * VE);
        }
    }
    __device__ __forceinline__ void store(E *dst, int ld, int nvalid, int tid) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int idx = tid + i * NT, r = idx / (D / VE);
            *(uint4 *)(dst + r * ld + idx % (D / VE) * VE) = r < nvalid ? x[i] : make_uint4(0u, 0u, 0u, 0u);
        }
    }
};

template <class E, int DK, int DV>
__global__ __launch_bounds__(64 * kPrepWaves)
__attribute__((amdgpu_waves_per_eu(PrepLds<E, DK, DV>::waves_per_simd)))
void gdn_back_prep_kernel(BackParams<E> p) {
    using L = PrepLds<E, DK, DV>;
    using TR = Tr<E>;
    using WD = Full<E>;
    constexpr int NT = 64 * kPrepWaves;
    constexpr int PA = kChunk * L::LDT;      // plane of A^T
    extern __shared__ __align__(16) unsigned char smem[];
    E *sK = (E *)(smem + L::oK), *sQ = (E *)(smem + L::oQ), *sO = sK, *sA = (E *)(smem + L::oA);
    float *sN = (float *)(smem + L::oN);     // N[r][c] at [r][c] (c < r), T[r][c] at [c][r] (c <= r)
    float *sg = (float *)(smem + L::oG), *sb = sg + 2 * kChunk, *sgam = sb + kChunk;
    const int c = blockIdx.x / (p.B * p.H), bh = blockIdx.x - c * (p.B * p.H);
    const int b = bh / p.H, h = bh - b * p.H;
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, li = l & 15, lg = l >> 4;
    const int t0 = c * kChunk, nvalid = min(kChunk, p.T - t0);
    const size_t cidx = (size_t)bh * p.NC + c;
    const size_t row0 = ((size_t)b * p.T + t0) * p.H + h;

    float a = 1.f, be = 0.f;
    if (w == 0 && l < nvalid) {
        a = p.alpha[row0 + (size_t)l * p.H];
        be = p.beta[row0 + (size_t)l * p.H];
    }
    RowTile<E, DK, NT> kr, qr;
    RowTile<E, DV, NT> orr;
    kr.load(p.k + row0 * DK, (size_t)p.H * DK, nvalid, tid);
    qr.load(p.q + row0 * DK, (size_t)p.H * DK, nvalid, tid);
    orr.load(p.dout + row0 * DV, (size_t)p.H * DV, nvalid, tid);
    if (w == 0) {
        float *gate = p.gates + cidx * kBackGateRec;
        float la = logf(a);
        la = (la < kLogAlphaMin) ? kLogAlphaMin : la;   // keeps NaN
        double g = (double)la;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const double o = __shfl_up(g, d);
            if (l >= d) g += o;
        }
        const double gC = __shfl(g, kChunk - 1);
        const double g2 = g * 1.4426950408889634;
        const float ghi = (float)g2, glo = (float)(g2 - (double)ghi);
        sg[kBackGHi + l] = gate[kBackGHi + l] = ghi;
        sg[kBackGLo + l] = gate[kBackGLo + l] = glo;
        sb[l] = be;
        const float gam = expf((float)g), tail = expf((float)(gC - g));
        sgam[l] = gam;
        gate[kBackGam + l] = gam;
        gate[kBackTail + l] = tail;
        gate[kBackBeta + l] = be;
        gate[kBackBt + l] = be * tail;
        if (l == 0) gate[kBackGC] = expf((float)gC);
    }
    kr.store(sK, L::LDK, nvalid, tid);
    qr.store(sQ, L::LDK, nvalid, tid);
    // the tiles of A^T that stay empty are read as zeros
    for (int i = tid; i < (int)(L::oG - L::oA) / 16; i += NT) ((uint4 *)(smem + L::oA))[i] = make_uint4(0u, 0u, 0u, 0u);
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
        for (int q = 0; q < 4; ++q) acc[q] = j <= i0 + q ? acc[q] * back_decay(sg, i0 + q, j) : 0.f;
        if (t < 10) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (j < i0 + q) sN[(i0 + q) * L::LDA + j] = acc[q] * sb[j];
        } else {
            WD::store4(sA + j * L::LDT + i0, PA, acc);
        }
    }
    lds_barrier();
    orr.store(sO, L::LDV, nvalid, tid);
    lds_barrier();

    // T = (I + N)^{-1}: the diagonal blocks by substitution (lane = block * 16 +
    // column) on wave 0, while the others form beta A^T dO.
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
        for (int r = 0; r < 16; ++r)
            if (r >= li) sN[(base + li) * L::LDA + base + r] = x[r];
    } else {
        float *N0 = p.N0 + cidx * (size_t)kChunk * DV;
        for (int f = w - 1; f < (DV / 16) * 4; f += kPrepWaves - 1) {
            const int rt = f & 3, jt = f >> 2;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
                if (kb >= rt / 2)                        // rows i >= j only
                    acc = WD::ew(tr_frag<E>(sO, L::LDV, 32 * kb, 16 * jt, false, 0, li, lg),
                                 WD::load8(sA + (16 * rt + li) * L::LDT + 32 * kb + 8 * lg, PA), acc);
            *(f32x4 *)(N0 + (jt * 4 + rt) * 256 + l * 4) = acc * sb[16 * rt + li];
        }
    }
    // Q^T gam dO: a column tile and every second (or each) row tile per wave
    {
        constexpr int NK = DK / 64, NJ = DV / 16, PER = kPrepWaves / NJ;
        float *C0 = p.C0 + cidx * (size_t)(DK * DV);
        const int jt = w / PER;
        typename WD::frag gd[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const typename TR::frag o = tr_frag<E>(sO, L::LDV, 32 * kb, 16 * jt, false, 0, li, lg);
            const float *gm = sgam + 32 * kb + 8 * lg;
            gd[kb] = WD::split(TR::to_f32(TR::lo(o)) * *(const f32x4 *)gm, TR::to_f32(TR::hi(o)) * *(const f32x4 *)(gm + 4));
        }
        for (int t = w % PER; t < 4 * NK; t += PER) {    // tile a = t % NK of scan wave t / NK
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
                acc = WD::ew(tr_frag<E>(sQ, L::LDK, 32 * kb, 16 * NK * (t / NK), NK == 2, t % NK, li, lg), gd[kb], acc);
            *(f32x4 *)(C0 + (jt * 4 * NK + t) * 256 + l * 4) = acc;
        }
    }
    lds_barrier();
    // Off-diagonal blocks by block distance: T_ij = -T_ii sum_{m=j}^{i-1} N_im T_mj.
    for (int dist = 1; dist < 4; ++dist) {
        if (w < 4 - dist) {
            const int j = w, i = w + dist;
            f32x4 X = {0.f, 0.f, 0.f, 0.f};
            for (int m = j; m < i; ++m) {
                const f32x4 n = *(const f32x4 *)(sN + (16 * i + li) * L::LDA + 16 * m + 4 * lg);
                f32x4 t = *(const f32x4 *)(sN + (16 * j + li) * L::LDA + 16 * m + 4 * lg);
#pragma unroll
                for (int q = 0; q < 4; ++q) X = mma_f32_k4(n[q], m > j || 4 * lg + q >= li ? t[q] : 0.f, X);
            }
            f32x4 Y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int q = 0; q < 4; ++q)
                Y = mma_f32_k4(li >= 4 * lg + q ? sN[(16 * i + 4 * lg + q) * L::LDA + 16 * i + li] : 0.f, X[q], Y);
            *(f32x4 *)(sN + (16 * j + li) * L::LDA + 16 * i + 4 * lg) = -Y;
        }
        lds_barrier();
    }
    // T and T^T as fragments
    for (int f = w; f < 16; f += kPrepWaves) {
        const int kb = f & 1, rt = (f >> 1) & 3, r = 16 * rt + li, k0 = 32 * kb + 8 * lg;
        if (f < 8 ? kb > rt / 2 : kb < rt / 2) continue;
        f32x4 x[2];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e >> 2][e & 3] = f < 8 ? (k0 + e <= r ? sN[(k0 + e) * L::LDA + r] : 0.f)
                                     : (k0 + e >= r ? sN[r * L::LDA + k0 + e] : 0.f);
        E *dst = (f < 8 ? p.Tf : p.Tt) + cidx * (size_t)full_elems<E>(kChunk * kChunk);
        WD::store8(dst + (rt * 2 + kb) * 512 + l * 8, kChunk * kChunk, WD::split(x[0], x[1]));
    }
}

// --------------------------------------------------------------------------
// Stage 2: the scans.  A workgroup carries 16 columns of one state through the
// chunks: blockIdx.y = 0 the states forward, 1 their gradients backward.  With X the
// state and first, before, after, add as in the table, a chunk is
//   y = T (first + before K X),   X <- e^{g_C} X + add + K^T (after y)
//                 T    first   before       after       add
//   forward       T    V       -gam         beta tail   -            y = e
//   backward      T^T  N0      beta tail    -gam        C0           y = dV
// Four compute waves; wave w holds rows R w .. R w + R - 1 of the state, R = Dk / 4 (32 of
// them in P32 order), so that its planes are a product's operand as they stand.  A
// chunk takes three exchanges through LDS, each ended by a barrier:
//   1  every wave multiplies its rows into K X for all 64 tokens; wave r adds up the
//      partial sums of token tile r and forms T's operand there;
//   2  wave r forms rows 16 r .. of y;
//   3  every wave adds K^T (after y) to its rows.
// Two loader waves bring K, first, add and the gates of a chunk into a ring of three
// slots by asynchronous copies, two chunks ahead, a share of them in each phase (a wave
// needs some 50 cycles to issue one, and compute waves that load for themselves were
// held up by that: 2.5 us a chunk); T, which is no LDS operand, goes to registers one
// chunk ahead.  No load of the compute waves is under a condition: a wait
// behind a branch that may have loaded waits for everything.  Rows past the end
// of the sequence are read as its last row: their beta is 0, and so is their part in
// the states and in dV.
// --------------------------------------------------------------------------
constexpr int kBackScanWaves = 4, kBackLoadWaves = 2;

// DIRECT: the compute waves load first and add themselves, with T.  Four more waves that formed them
// here from Q, dO and beta A^T in place of the prep stage saved 192 KB of traffic a chunk and head
// and lost by it: prep 27 in place of 39 us at T = 3520, but the scan 123 in place of 102, and 419 in
// place of 325 at T = 10560 (Q's rows, eight times over, and their products, in every workgroup).
template <class E, int DK, bool DIRECT> struct BackScanLds {
    static constexpr int R = DK / 4, NK = R / 16;                             // state rows and row tiles per wave
    static constexpr int LDC = sizeof(E) == 2 ? kChunk : lds_ld<E>(kChunk);
    static constexpr int PT = 16 * kChunk, PC = 16 * LDC;                     // planes
    static constexpr int szK = (int)sizeof(E) * kChunk * DK, szF = DIRECT ? 0 : 4096, szA = DIRECT ? 0 : 4096 * NK;
    static constexpr int oF = szK, oA = oF + szF, oG = oA + szA;              // in a slot: K, first, add, gates
    static constexpr int SLOT = oG + 4 * kBackScanGates + 16, DEPTH = 3;
    static constexpr int oP = DEPTH * SLOT;                                   // partial sums of K X
    static constexpr int oX = oP + 4 * 4 * 4 * 256;                           // T's operand, [token][column]
    static constexpr int oY = oX + (int)sizeof(E) * Full<E>::planes * PT;     // after y, [column][token]
    static constexpr size_t bytes = oY + sizeof(E) * Full<E>::planes * PC;
    static constexpr int threads = 64 * (kBackScanWaves + kBackLoadWaves);
    // Waves per SIMD: six waves are two on one of the SIMDs, and each workgroup of a CU puts them on
    // the same one.
    static constexpr bool shares = bytes * 2 <= 160 * 1024;
    static constexpr int waves_per_simd = shares ? 4 : 2;
    static_assert(SLOT % 16 == 0 && bytes <= 160 * 1024, "the ring fits the LDS");
};

// LDS layouts of the bf16 path.  A 16-byte read is served in 4 cycles, lanes 0-3, 12-15 and 20-27 in one
// (the other lanes of the half in the next), if those 16 lanes take different 16-byte places of 256 bytes; an
// 8-byte read, transposing or not, in 2, the lanes of each half in different 8-byte places; an
// 8-byte store in 4, 16 lanes each, in different places of 128 bytes.  So the granules of a row are
// permuted, granule g stored at g ^ perm(row); rows padded by 16 bytes cost twice that, and a
// store of 32-byte rows four times (the scan: 102 -> 98.5 us at T = 3520, 16 heads of 128, 227 -> 220 at
// 80 heads of 64).
//
// Rows of 128 bytes: 16-byte reads of 16 rows and transposing reads of 8 (r .. r + 3, r + 8 .. r + 11) at
// full rate, 8-byte stores of one granule in 16 rows at half.
__device__ __forceinline__ int perm128(int r) { return ((r >> 2) & 1) + (r & 2) + 4 * (((r >> 2) ^ (r >> 3)) & 1); }

// K rows in the ring (of 256 bytes at Dk = 128: transposing reads at half rate, which they are in P32 order
// in any case).
template <class E, int DK> __device__ __forceinline__ int kperm(int r) {
    if constexpr (sizeof(E) == 4) return r & 15;
    else if constexpr (DK == 128) return 2 * (r & 3) + (r & 8);
    else return perm128(r);
}

// T's operand, [token][16 columns]: 8-byte granule g of a token, and its planes with transposing reads.
template <class E> __device__ __forceinline__ int xaddr(int row, int g) {
    if constexpr (sizeof(E) == 2) return (row ^ ((row & 8) >> 1)) * 16 + ((g ^ (row >> 2)) & 3) * 4;
    else return row * 16 + 4 * g;
}
template <class E> __device__ __forceinline__ typename Full<E>::frag xcols(const E *X, int plane, int row0, int li, int lg) {
    if constexpr (sizeof(E) == 2) {
        typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
        const int row = row0 + 8 * lg + (li >> 2);
        const E *lo = X + xaddr<E>(row, li & 3), *hi = X + xaddr<E>(row + 4, li & 3);
        typename Full<E>::frag f;
#pragma unroll
        for (int i = 0; i < Full<E>::planes; ++i)
            f.pl[i] = Tr<E>::cat(__builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(lo + i * plane))),
                                 __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(hi + i * plane))));
        return f;
    } else {
        return Full<E>::tr(X, plane, 16, row0, 0, li, lg);
    }
}
// after y, [column][token]: the place of token t's group of 4 or 8 (t a multiple of it)
template <class E> __device__ __forceinline__ int yaddr(int col, int t) {
    if constexpr (sizeof(E) == 2) return col * kChunk + (((t >> 3) ^ perm128(col)) << 3) + (t & 4);
    else return col * lds_ld<E>(kChunk) + t;
}
template <class E, int DK> __device__ __forceinline__ const E *kaddr(const E *K, int row, int col) {
    constexpr int VE = 16 / (int)sizeof(E);
    return K + row * DK + ((col / VE) ^ kperm<E, DK>(row)) * VE + col % VE;
}
// R / 4 consecutive channels of a row
template <class E, int DK, int R> __device__ __forceinline__ typename RowBlock<E, R>::in krow(const E *K, int row, int col) {
    if constexpr (sizeof(E) == 4 && R == 32)
        return Tr<E>::cat(*(const f32x4 *)kaddr<E, DK>(K, row, col), *(const f32x4 *)kaddr<E, DK>(K, row, col + 4));
    else
        return *(const typename RowBlock<E, R>::in *)kaddr<E, DK>(K, row, col);
}
// tr_frag through the permutation
template <class E, int DK, int NK>
__device__ __forceinline__ typename Tr<E>::frag kcols(const E *K, int row0, int colbase, int a, int li, int lg) {
    if constexpr (sizeof(E) == 2) {
        typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
        const int row = row0 + 8 * lg + (li >> 2);
        const int col = NK == 2 ? colbase + 8 * (li & 3) + 4 * a : colbase + 4 * (li & 3);
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)kaddr<E, DK>(K, row, col));
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)kaddr<E, DK>(K, row + 4, col));
        return Tr<E>::cat(__builtin_bit_cast(u32x2, lo), __builtin_bit_cast(u32x2, hi));
    } else {
        const int col = NK == 2 ? colbase + p32_row(a, li) : colbase + li;
        typename Tr<E>::frag f;
#pragma unroll
        for (int q = 0; q < 8; ++q) f[q] = *kaddr<E, DK>(K, row0 + 8 * lg + q, col);
        return f;
    }
}

// The loader waves (part = 0, 1).
template <class E, int DK, int DV, bool REV, bool DIRECT>
__device__ __forceinline__ void back_loader(const BackParams<E> &p, unsigned char *smem, int bh, int jt, int part, int l) {
    using L = BackScanLds<E, DK, DIRECT>;
    constexpr int sz = (int)sizeof(E), GPR = DK * sz / 16, RPC = 64 / GPR;   // granules per K row, rows per copy
    constexpr int NKC = L::szK / 2048;                                       // copies of K per wave
    constexpr int GPV = sz, RPV = 64 / GPV;                                  // granules per row of 16 columns of V
    constexpr int NF = DIRECT ? 0 : REV ? 2 : sz / 2, NA = REV ? L::szA / 2048 : 0;   // of first and add per wave
    constexpr int ALL = NKC + NF + NA + 1;
    const int b = bh / p.H, h = bh - b * p.H;
    const size_t head = (size_t)b * p.T * p.H + h;
    typedef __attribute__((address_space(3))) void lds_void;
    auto copy = [](const void *src, unsigned char *dst) { __builtin_amdgcn_global_load_lds(src, (lds_void *)dst, 16, 0, 0); };
    // chunks in the order of this direction; past the last one the last one again
    auto chunk = [&](int i) { return REV ? max(p.NC - 1 - i, 0) : min(i, p.NC - 1); };
    auto rows = [&](int i, int n0, int n1) {                                 // copies n0 .. n1 - 1 of K
        const int c = chunk(i), last = min(kChunk, p.T - c * kChunk) - 1;
        const E *k = p.k + (head + (size_t)c * kChunk * p.H) * DK;
        unsigned char *slot = smem + i % L::DEPTH * L::SLOT;
#pragma unroll
        for (int n = n0; n < n1; ++n) {
            const int r = RPC * (2 * n + part) + l / GPR, g = (l % GPR) ^ kperm<E, DK>(r);
            copy(k + (size_t)min(r, last) * p.H * DK + g * (16 / sz), slot + 1024 * (2 * n + part));
        }
    };
    auto rest = [&](int i) {
        const int c = chunk(i), last = min(kChunk, p.T - c * kChunk) - 1;
        const size_t cidx = (size_t)bh * p.NC + c;
        unsigned char *slot = smem + i % L::DEPTH * L::SLOT;
        if constexpr (REV) {
            const float *n0 = p.N0 + cidx * (size_t)(kChunk * DV) + jt * 1024 + l * 4;
            const float *c0 = p.C0 + cidx * (size_t)(DK * DV) + jt * (1024 * L::NK) + l * 4;
#pragma unroll
            for (int n = 0; n < NF; ++n) copy(n0 + 256 * (2 * n + part), slot + L::oF + 1024 * (2 * n + part));
#pragma unroll
            for (int n = 0; n < NA; ++n) copy(c0 + 256 * (2 * n + part), slot + L::oA + 1024 * (2 * n + part));
        } else {
            const E *v = p.v + (head + (size_t)c * kChunk * p.H) * DV + 16 * jt;
#pragma unroll
            for (int n = 0; n < NF; ++n) {
                const int r = RPV * (2 * n + part) + l / GPV;
                copy(v + (size_t)min(r, last) * p.H * DV + l % GPV * (16 / sz), slot + L::oF + 1024 * (2 * n + part));
            }
        }
        // (by both waves, so that their counts agree)
        if (l < kBackScanGates / 4) copy(p.gates + cidx * kBackGateRec + kBackGam + 4 * l, slot + L::oG);
    };
    rows(0, 0, NKC);
    rest(0);
    rows(1, 0, NKC);
    rest(1);
    wait_vmcnt<ALL>();
    lds_only_barrier();                                // chunk 0 is there
    for (int i = 0; i < p.NC; ++i) {
        // slot of chunk i + 2: that of chunk i - 1, which no wave reads any more
        rows(i + 2, 0, NKC / 2);
        lds_only_barrier();
        rows(i + 2, NKC / 2, NKC);
        wait_vmcnt<NKC>();                             // chunk i + 1 is there
        lds_only_barrier();
        rest(i + 2);
        lds_only_barrier();
    }
    wait_vmcnt<0>();
}

template <class E, int DK, int DV, bool REV, bool DIRECT>
__device__ __forceinline__ void back_scan(const BackParams<E> &p, unsigned char *smem, int bh, int jt, int w, int l) {
    using L = BackScanLds<E, DK, DIRECT>;
    using TR = Tr<E>;
    using WD = Full<E>;
    using wfrag = typename WD::frag;
    constexpr int R = L::R, NK = L::NK;
    using RB = RowBlock<E, R>;
    struct Ahead {
        wfrag T[2];
        typename RB::in k[4];
        f32x4 n0, add[NK];
        typename TR::quad v;
    };
    const int li = l & 15, lg = l >> 4;
    float *sP = (float *)(smem + L::oP);                          // [wave][token tile][lane][4]
    E *sX = (E *)(smem + L::oX), *sY = (E *)(smem + L::oY);
    const float *init = REV ? p.dstate_out : p.state_in;
    const size_t head = (size_t)(bh / p.H) * p.T * p.H + bh % p.H;
    // element (R w + R / 4 lg + 4 a + q, 16 jt + li) is st[a][q]
    const size_t sbase = (size_t)bh * DK * DV;
    const unsigned soff = (R * w + R / 4 * lg) * DV + 16 * jt + li;
    f32x4 st[NK];
#pragma unroll
    for (int a = 0; a < NK; ++a)
#pragma unroll
        for (int q = 0; q < 4; ++q) st[a][q] = init ? init[sbase + soff + (4 * a + q) * DV] : 0.f;
    auto chunk = [&](int i) { return REV ? max(p.NC - 1 - i, 0) : min(i, p.NC - 1); };
    // (for a zero block of T, which is not used, the other one again)
    Ahead o;
    auto load = [&](int c) {
        const E *T = (REV ? p.Tt : p.Tf) + ((size_t)bh * p.NC + c) * (size_t)full_elems<E>(kChunk * kChunk);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
            o.T[kb] = WD::load8(T + (unsigned)((w * 2 + (REV ? max(kb, w / 2) : min(kb, w / 2))) * 512 + l * 8), kChunk * kChunk);
        if constexpr (DIRECT && REV) {
            const size_t cidx = (size_t)bh * p.NC + c;
            o.n0 = *(const f32x4 *)(p.N0 + cidx * (size_t)(kChunk * DV) + (unsigned)((jt * 4 + w) * 256 + l * 4));
#pragma unroll
            for (int a = 0; a < NK; ++a)
                o.add[a] = *(const f32x4 *)(p.C0 + cidx * (size_t)(DK * DV) + (unsigned)(((jt * 4 + w) * NK + a) * 256 + l * 4));
        } else if constexpr (DIRECT) {
            const int last = min(kChunk, p.T - c * kChunk) - 1;
            o.v = TR::load(p.v + (head + (size_t)c * kChunk * p.H) * DV +
                           (unsigned)(min(16 * w + li, last) * p.H * DV + 16 * jt + 4 * lg));
        }
    };
    // K's rows for the next chunk, which is in the ring since the barrier before the last, are read
    // where this chunk's y is on its way, if the workgroup has the CU to itself (103 against 111
    // us at T = 3520, H = 16, D = 128); where two share it (D = 64) the other one uses that time (253
    // against 232 us at T = 3520, 80 heads).
    constexpr bool KAHEAD = !L::shares;
    auto rows_of = [&](const E *K, int rt) { return krow<E, DK, R>(K, 16 * rt + li, R * w + R / 4 * lg); };
    // the i-th chunk of this direction
    auto step = [&](int i) {
        const size_t cidx = (size_t)bh * p.NC + chunk(i);
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        const unsigned char *slot = smem + i % L::DEPTH * L::SLOT;
        const E *K = (const E *)slot;
        const float *gate = (const float *)(slot + L::oG) - kBackGam;
        // K X transposed, [column][token]
        {
            typename RB::in k[4];
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) k[rt] = KAHEAD ? o.k[rt] : rows_of(K, rt);
            const typename RB::planes H = RB::split(st);
            f32x4 part[4];
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) part[rt] = RB::product(H, k[rt]);
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) *(f32x4 *)(sP + (w * 4 + rt) * 256 + l * 4) = part[rt];
        }
        f32x4 first;
        if constexpr (DIRECT && REV) first = o.n0;
        else if constexpr (DIRECT) first = TR::to_f32(o.v);
        else if constexpr (REV) first = *(const f32x4 *)(slot + L::oF + (w * 64 + l) * 16);
        else first = TR::to_f32(TR::load((const E *)(slot + L::oF) + (16 * w + li) * 16 + 4 * lg));
        const float before = REV ? gate[kBackBt + 16 * w + li] : -gate[kBackGam + 16 * w + li];
        lds_only_barrier();
        f32x4 xs[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) xs[j] = *(const f32x4 *)(sP + (j * 4 + w) * 256 + l * 4);
        // The state that entered this chunk, for stage 3: lane (li, lg) stores 4 columns of row
        // 4 lg + li % 4 of a tile, 1 KB in a row from a wave (a store of 4 bytes a lane takes as
        // long to issue, and eight of them held up the wave for 700 cycles).
        float *keep = (REV ? p.Gs : p.Hs) + cidx * (size_t)(DK * DV) +
                      (unsigned)((jt * DK + R * w + 4 * lg + (li & 3)) * 16 + (li & 12));
#pragma unroll
        for (int a = 0; a < NK; ++a) *(f32x4 *)(keep + 256 * a) = quad_transpose(st[a], li);
        const f32x4 x = (xs[0] + xs[1]) + (xs[2] + xs[3]);
        WD::store4(sX + xaddr<E>(16 * w + li, lg), L::PT, first + before * x);
        typename TR::frag kt[NK][2];
#pragma unroll
        for (int a = 0; a < NK; ++a)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) kt[a][kb] = kcols<E, DK, NK>(K, 32 * kb, R * w, a, li, lg);
        const f32x4 after = REV ? -*(const f32x4 *)(gate + kBackGam + 16 * w + 4 * lg) : *(const f32x4 *)(gate + kBackBt + 16 * w + 4 * lg);
        const float gC = gate[kBackGC];
        lds_only_barrier();
        f32x4 y[2] = {zero, zero};
#pragma unroll
        for (int a = 0; a < NK; ++a) {
            st[a] *= gC;
            if constexpr (DIRECT && REV) st[a] += o.add[a];
            else if constexpr (REV) st[a] += *(const f32x4 *)(slot + L::oA + ((w * NK + a) * 64 + l) * 16);
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
            if (REV ? kb >= w / 2 : kb <= w / 2)                  // T is lower triangular
                y[kb] = WD::ww(o.T[kb], xcols<E>(sX, L::PT, 32 * kb, li, lg), y[kb]);
        load(chunk(i + 1));
        y[0] += y[1];
        WD::store4(sY + yaddr<E>(li, 16 * w + 4 * lg), L::PC, after * y[0]);
        *(f32x4 *)((REV ? p.vT : p.eT) + cidx * (size_t)(kChunk * DV) + (unsigned)((16 * jt + li) * kChunk + 16 * w + 4 * lg)) = y[0];
        if constexpr (KAHEAD) {
            const E *Kn = (const E *)(smem + (i + 1) % L::DEPTH * L::SLOT);
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) o.k[rt] = rows_of(Kn, rt);
        }
        lds_only_barrier();
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const wfrag u = WD::load8(sY + yaddr<E>(li, 32 * kb + 8 * lg), L::PC);
#pragma unroll
            for (int a = 0; a < NK; ++a) st[a] = WD::ew(kt[a][kb], u, st[a]);
        }
    };
    load(chunk(0));
    // (vmcnt(0): loads pending from before the loop would be taken for pending at
    // the start of every turn, and the waits there for all loads of the turn before)
    __builtin_amdgcn_s_waitcnt(0x0f70);
    lds_only_barrier();
    if constexpr (KAHEAD) {
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) o.k[rt] = rows_of((const E *)smem, rt);
    }
    for (int i = 0; i < p.NC; ++i) step(i);
    if (REV && p.dstate_in) {
#pragma unroll
        for (int a = 0; a < NK; ++a)
#pragma unroll
            for (int q = 0; q < 4; ++q) p.dstate_in[sbase + soff + (4 * a + q) * DV] = st[a][q];
    }
}

template <class E, int DK, int DV, bool DIRECT>
__global__ __launch_bounds__((BackScanLds<E, DK, DIRECT>::threads))
__attribute__((amdgpu_waves_per_eu(BackScanLds<E, DK, DIRECT>::waves_per_simd)))
void gdn_back_scan_kernel(BackParams<E> p) {
    extern __shared__ __align__(16) unsigned char smem[];
    // the column tiles of a head share its operands: they get the same XCD
    constexpr int NJ = DV / 16;
    const int u = blockIdx.x >> 3, jt = u % NJ, bh = (u / NJ) * 8 + (blockIdx.x & 7);
    if (bh >= p.B * p.H) return;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
    if (w >= kBackScanWaves) {
        if (blockIdx.y == 0) back_loader<E, DK, DV, false, DIRECT>(p, smem, bh, jt, w - kBackScanWaves, l);
        else back_loader<E, DK, DV, true, DIRECT>(p, smem, bh, jt, w - kBackScanWaves, l);
    } else {
        if (blockIdx.y == 0) back_scan<E, DK, DV, false, DIRECT>(p, smem, bh, jt, w, l);
        else back_scan<E, DK, DV, true, DIRECT>(p, smem, bh, jt, w, l);
    }
}

// --------------------------------------------------------------------------
// Stage 3, per chunk and head: dQ, dK, dV, dalpha and dbeta.  Four waves, two
// workgroups to a CU (or eight, see NH).  Wave w has the Dk / 4 key channels from (Dk / 4) w on in the
// products over Dk; the 64 x 64 products are dealt out as lower tiles.  The value
// channels go through LDS 64 at a time; once they are done, X and G1, then G2, take their
// place there (all three at once are more than two workgroups a CU leave room for;
// G1 and G2 side by side in two planes of bf16 took 1 % less of the whole call at heads of 128, 2 % at
// 64, and lost what their sums cancel down to).
// --------------------------------------------------------------------------

template <class E> struct GradLds {
    static constexpr int LDC = lds_ld<E>(kChunk), PC = kChunk * LDC;
    static constexpr size_t szF = sizeof(E) * Full<E>::planes * PC;
    static constexpr size_t oE = 0;                     // e^T, 64 value channels
    static constexpr size_t oV = oE + szF;              // dV^T
    static constexpr size_t oO = oV + szF;              // dO, [token][value channel]
    static constexpr size_t endA = oO + sizeof(E) * PC;
    static constexpr size_t oX = 0;                     // X^T, its column 0 the exit state's
    static constexpr size_t oG1 = oX + szF;             // G1^T, then G2 + G2^T
    static constexpr size_t oG2 = oG1 + szF;            // G2's ten lower tiles, fp32, as their lanes have them
    static constexpr size_t endB = oG2 + 10 * 1024;
    static constexpr size_t oGate = endA > endB ? endA : endB;
    static constexpr size_t oRed = oGate + 4 * kBackGateRec;
    // floats behind oRed: [4 wave][4 lg][64] parts of X_i,-1, the same of k.PE, [4 row tile][4 lg][64] of
    // dbeta, [64] X_i,-1, [4] parts of <G, H>
    static constexpr size_t bytes = oRed + 4 * (48 * 64 + 64 + 4);
};

// NH = 2: eight waves, four for each half of the tokens in the products over Dk, for launches that
// leave every workgroup a CU of its own.
// Registers: all 256 of two waves a SIMD at Dk = 128 and NH = 1, in bf16 five more than that (spilled to
// scratch memory, 24 bytes a lane).
template <class E, int DK, int DV, int NH>
__global__ __launch_bounds__(256 * NH) __attribute__((amdgpu_waves_per_eu(2, 2)))
void gdn_back_grad_kernel(BackParams<E> p) {
    using L = GradLds<E>;
    using TR = Tr<E>;
    using WD = Full<E>;
    using frag = typename TR::frag;
    using wfrag = typename WD::frag;
    constexpr int NW = 4 * NH, NT = 64 * NW;
    constexpr int NK = DK / 64, RT = 4 / NH;                       // channel and token tiles per wave
    constexpr int VE = 16 / (int)sizeof(E);
    constexpr int NST = kChunk * 64 / 4 / NT, NSO = kChunk * 64 / VE / NT;   // staged quads / vectors per thread
    extern __shared__ __align__(16) unsigned char smem[];
    E *sE = (E *)(smem + L::oE), *sV = (E *)(smem + L::oV), *sO = (E *)(smem + L::oO), *sX = (E *)(smem + L::oX),
      *sG = (E *)(smem + L::oG1);
    float *sG2 = (float *)(smem + L::oG2);
    const float *gate = (const float *)(smem + L::oGate);
    const float *gam = gate + kBackGam, *tail = gate + kBackTail, *beta = gate + kBackBeta;
    float *rX = (float *)(smem + L::oRed), *rE = rX + 16 * 64, *cb = rE + 16 * 64, *xm = cb + 16 * 64, *gh = xm + 64;
    const int c = blockIdx.x / (p.B * p.H), bh = blockIdx.x - c * (p.B * p.H);
    const int b = bh / p.H, h = bh - b * p.H;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
    const int w = wave & 3, rt0 = wave / 4 * RT;                   // its channels, its first token tile
    int tid = threadIdx.x, li = l & 15, lg = l >> 4;
    // What follows computes its addresses anew: kept from the front on, they would take the
    // registers of the products between.
    auto forget = [&] { asm volatile("" : "+v"(tid), "+v"(li), "+v"(lg)); };
    const int t0 = c * kChunk, nvalid = min(kChunk, p.T - t0);
    const size_t cidx = (size_t)bh * p.NC + c;
    const size_t row0 = ((size_t)b * p.T + t0) * p.H + h;
    // row fragments of K and Q; rows past the end read the last one, whose products
    // with them meet beta = 0, dO = 0 or dV = 0
    auto rows = [&](const E *base, int r, int kb) {
        return load_frag<E>(base + (row0 + (size_t)min(r, nvalid - 1) * p.H) * DK + 32 * kb, lg);
    };
    const float *ge = p.eT + cidx * (size_t)(kChunk * DV), *gv = p.vT + cidx * (size_t)(kChunk * DV);
    for (int i = tid; i < kBackGateRec; i += NT) ((float *)(smem + L::oGate))[i] = p.gates[cidx * kBackGateRec + i];

    // PQ, PV, PE transposed, tiles [16 key channels][16 tokens]; Z and F
    constexpr int NTI = (9 + NW) / NW;                             // lower tiles wave, wave + NW, .. of ten
    f32x4 pq[NK][RT], pv[NK][RT], pe[NK][RT], z[NTI], f[NTI], dot = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < NTI; ++n) z[n] = f[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < NK; ++n)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) pq[n][rt] = pv[n][rt] = pe[n][rt] = f32x4{0.f, 0.f, 0.f, 0.f};
    // row li of tile n stands for channel 32 w + p32_row(n, li) (Dk = 64: 16 w + li): a lane gets
    // 4 NK consecutive channels in its NK results
    auto channel = [&](int n) { return NK == 2 ? 32 * w + p32_row(n, li) : 16 * w + li; };
    auto ch0 = [&] { return NK == 2 ? 32 * w + 8 * lg : 16 * w + 4 * lg; };
    auto quads = [&](const float *m, int j0, f32x4 (&x)[NK][2]) {  // 8 columns from j0 on of the rows of NK tiles
        const float *at = m + cidx * (size_t)(DK * DV) + (j0 >> 4) * (DK * 16) +
                          (unsigned)(((lg >> 1) * DK + 16 * NK * w + li) * 16 + 8 * (lg & 1));
#pragma unroll
        for (int n = 0; n < NK; ++n) {
            x[n][0] = *(const f32x4 *)(at + 256 * n);
            x[n][1] = *(const f32x4 *)(at + 256 * n + 4);
        }
    };
    // The scheduling barriers keep each group of loads where it is, a product ahead of its
    // use: all at the front they do not fit the registers, at their uses every one is waited for.
    f32x4 hs[NK][2];
    quads(p.Hs, 0, hs);
#pragma unroll 1
    for (int j0 = 0; j0 < DV; j0 += 32) {                          // 32 value channels a turn
        const int dv0 = j0 & ~63, kb = (j0 >> 5) & 1;
        forget();
        if (kb == 0) {
            if (j0) lds_barrier();
            f32x4 re[NST], rv[NST];
            uint4 ro[NSO];
#pragma unroll
            for (int i = 0; i < NST; ++i) {
                re[i] = *(const f32x4 *)(ge + dv0 * kChunk + (tid + i * NT) * 4);
                rv[i] = *(const f32x4 *)(gv + dv0 * kChunk + (tid + i * NT) * 4);
            }
#pragma unroll
            for (int i = 0; i < NSO; ++i) {
                const int idx = tid + i * NT, r = idx / (64 / VE), cv = idx % (64 / VE);
                ro[i] = *(const uint4 *)(p.dout + (row0 + (size_t)min(r, nvalid - 1) * p.H) * DV + dv0 + cv * VE);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < NST; ++i) {
                const int idx = tid + i * NT, at = (idx >> 4) * L::LDC + (idx & 15) * 4;
                WD::store4(sE + at, L::PC, re[i]);
                WD::store4(sV + at, L::PC, rv[i]);
            }
#pragma unroll
            for (int i = 0; i < NSO; ++i) {
                const int idx = tid + i * NT, r = idx / (64 / VE), cv = idx % (64 / VE);
                *(uint4 *)(sO + r * L::LDC + cv * VE) = r < nvalid ? ro[i] : make_uint4(0u, 0u, 0u, 0u);
            }
            lds_barrier();
        }
        {
            f32x4 g[NK][2];
            wfrag S[NK];
            quads(p.Gs, j0, g);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < NK; ++n) S[n] = WD::split(hs[n][0], hs[n][1]);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const int tt = rt0 + rt;
                const frag o = load_frag<E>(sO + (16 * tt + li) * L::LDC + 32 * kb, lg);
                const wfrag dv = WD::tr(sV, L::PC, L::LDC, 32 * kb, 16 * tt, li, lg);
#pragma unroll
                for (int n = 0; n < NK; ++n) {
                    pq[n][rt] = WD::we(S[n], o, pq[n][rt]);
                    pv[n][rt] = WD::ww(S[n], dv, pv[n][rt]);
                }
                // dV: one wave stores the rows it has at hand
                if (w == tt && 16 * tt + li < nvalid)
                    TR::store8(p.dv + (row0 + (size_t)(16 * tt + li) * p.H) * DV + dv0 + 32 * kb + 8 * lg, WD::rounded(dv));
                if (rt & 1) __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int n = 0; n < NTI; ++n) {
                if (wave + NW * n >= 10) continue;
                int bi, bj;
                lower_tile(wave + NW * n, bi, bj);
                const wfrag ej = WD::tr(sE, L::PC, L::LDC, 32 * kb, 16 * bj, li, lg);
                z[n] = WD::ew(load_frag<E>(sO + (16 * bi + li) * L::LDC + 32 * kb, lg), ej, z[n]);
                f[n] = WD::ww(WD::tr(sV, L::PC, L::LDC, 32 * kb, 16 * bi, li, lg), ej, f[n]);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int n = 0; n < NK; ++n) {
                dot += hs[n][0] * g[n][0] + hs[n][1] * g[n][1];
                S[n] = WD::split(g[n][0], g[n][1]);
            }
            quads(p.Hs, min(j0 + 32, DV - 32), hs);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const wfrag e = WD::tr(sE, L::PC, L::LDC, 32 * kb, 16 * (rt0 + rt), li, lg);
#pragma unroll
                for (int n = 0; n < NK; ++n) pe[n][rt] = WD::ww(S[n], e, pe[n][rt]);
                if (rt & 1) __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    forget();
    // Row fragments of K and Q for tile n of this wave, and its channels of all tokens, asked
    // for before they are used (fp32: the second and third tile's where they are used, for want
    // of registers).
    constexpr bool AHEAD = sizeof(E) == 2;
    struct Rows {
        frag q[DK / 32], k[DK / 32], kj[DK / 32];
    } ra, rb;
    auto tile_rows = [&](int n, Rows &x) {
        int bi, bj;
        lower_tile(min(wave + NW * n, 9), bi, bj);
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb) {
            x.q[kb] = rows(p.q, 16 * bi + li, kb);
            x.k[kb] = rows(p.k, 16 * bi + li, kb);
            x.kj[kb] = rows(p.k, 16 * bj + li, kb);
        }
    };
    using own = std::conditional_t<NK == 2, frag, typename TR::quad>;
    own qo[RT], ko[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const size_t at = (row0 + (size_t)min(16 * (rt0 + rt) + li, nvalid - 1) * p.H) * DK + ch0();
        if constexpr (NK == 2) qo[rt] = TR::load8(p.q + at), ko[rt] = TR::load8(p.k + at);
        else qo[rt] = TR::load(p.q + at), ko[rt] = TR::load(p.k + at);
    }
    if (AHEAD) tile_rows(0, ra);
    __builtin_amdgcn_sched_barrier(0);
    {
        float s = dot[0] + dot[1] + dot[2] + dot[3];
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d);
        if (l == 0 && rt0 == 0) gh[w] = s;
    }
    // q.PQ - k.PV and k.PE of this wave's channels; then the parts of dQ and dK that
    // come from the states
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int t = 16 * (rt0 + rt) + li;
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int n = 0; n < NK; ++n) {
            f32x4 q4, k4;
            if constexpr (NK == 2) {
                q4 = TR::to_f32(n ? TR::hi(qo[rt]) : TR::lo(qo[rt]));
                k4 = TR::to_f32(n ? TR::hi(ko[rt]) : TR::lo(ko[rt]));
            } else {
                q4 = TR::to_f32(qo[rt]);
                k4 = TR::to_f32(ko[rt]);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                x += q4[q] * pq[n][rt][q] - k4[q] * pv[n][rt][q];
                y += k4[q] * pe[n][rt][q];
            }
            pq[n][rt] *= gam[t];
            pe[n][rt] = pe[n][rt] * (tail[t] * beta[t]) - pv[n][rt] * gam[t];
        }
        rX[(w * 4 + lg) * 64 + t] = x;
        rE[(w * 4 + lg) * 64 + t] = y;
    }
    if (AHEAD && wave + NW < 10) tile_rows(1, rb);
    lds_barrier();
    // The 64 x 64 matrices: element (i, j) with i = 16 bi + 4 lg + q, j = 16 bj + li.  The six
    // tiles above the diagonal of G1 and X are zero.  G2 waits as it is until G1 has been read.
    auto matrices = [&](int n, const Rows &r) {
        if (wave + NW * n >= 10) return;
        int bi, bj;
        lower_tile(wave + NW * n, bi, bj);
        const int j = 16 * bj + li, i0 = 16 * bi + 4 * lg;
        const float bj_ = beta[j];
        f32x4 sqk = {0.f, 0.f, 0.f, 0.f}, skk = sqk, g1, g2, xx;
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb) {
            sqk = TR::mma(r.q[kb], r.kj[kb], sqk);
            skk = TR::mma(r.k[kb], r.kj[kb], skk);
        }
        float cs = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int i = i0 + q;
            const float d = i >= j ? back_decay(gate, i, j) : 0.f;
            const float dz = d * z[n][q], df = i > j ? d * f[n][q] : 0.f;
            g1[q] = dz * bj_;
            g2[q] = df * bj_;
            xx[q] = i > j ? bj_ * (sqk[q] * z[n][q] - skk[q] * f[n][q]) : 0.f;
            cs += sqk[q] * dz - skk[q] * df;
        }
        *(f32x4 *)(sG2 + (wave + NW * n) * 256 + l * 4) = g2;
        WD::store4(sG + j * L::LDC + i0, L::PC, g1);
        WD::store4(sX + j * L::LDC + i0, L::PC, xx);
        if (bi != bj) {
            const f32x4 none = {0.f, 0.f, 0.f, 0.f};
            WD::store4(sG + (16 * bi + li) * L::LDC + 16 * bj + 4 * lg, L::PC, none);
            WD::store4(sX + (16 * bi + li) * L::LDC + 16 * bj + 4 * lg, L::PC, none);
        }
        cb[(bi * 4 + lg) * 64 + j] = cs;
    };
    auto symmetric = [&](int n) {                                  // G2 + G2^T
        if (wave + NW * n >= 10) return;
        int bi, bj;
        lower_tile(wave + NW * n, bi, bj);
        const int j = 16 * bj + li, i0 = 16 * bi + 4 * lg;
        const f32x4 g2 = *(const f32x4 *)(sG2 + (wave + NW * n) * 256 + l * 4);
        if (bi != bj) WD::store4(sG + j * L::LDC + i0, L::PC, g2);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (i0 + q < j) continue;                              // written from below the diagonal
            WD::store1(sG + (i0 + q) * L::LDC + j, L::PC, g2[q]);
            if (bi == bj && i0 + q > j) WD::store1(sG + j * L::LDC + i0 + q, L::PC, g2[q]);
        }
    };
    if (!AHEAD) tile_rows(0, ra);
    matrices(0, ra);
    __builtin_amdgcn_sched_barrier(0);
    if (!AHEAD) tile_rows(1, rb);
    else if (NTI == 3) tile_rows(2, ra);
    __builtin_amdgcn_sched_barrier(0);
    matrices(1, rb);
    __builtin_amdgcn_sched_barrier(0);
    // K^T and Q^T, as they are, for dQ and dK
    E kt_[NK][2][8], qt_[NK][2][8];
    auto columns = [&](const E *base, E (&x)[NK][2][8]) {          // channel of tokens 32 kb + 8 lg .. + 7
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[n][kb][e] = base[(row0 + (size_t)min(32 * kb + 8 * lg + e, nvalid - 1) * p.H) * DK + channel(n)];
    };
    if (AHEAD) {
        columns(p.k, kt_);
        columns(p.q, qt_);
    } else if (NTI == 3) {
        tile_rows(2, ra);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (NTI == 3) matrices(2, ra);
    __builtin_amdgcn_sched_barrier(0);
    if (!AHEAD) {
        columns(p.k, kt_);
        columns(p.q, qt_);
    }
    lds_barrier();
    forget();

    // Sums over the waves: X's border row and column, dbeta
    if (wave == 0) {
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) x += rX[i * 64 + l];
        xm[l] = x;
    } else if (wave == 1) {
        float y = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) y += rE[i * 64 + l];
        WD::store1(sX + l * L::LDC, L::PC, beta[l] * y);
        float d = tail[l] * y;
        for (int i = l >> 4 << 2; i < 16; ++i) d += cb[i * 64 + l];
        if (l < nvalid) p.dbeta[row0 + (size_t)l * p.H] = d;
    }
    // dQ += G1 K;  dK += G1^T Q, then, with G2 in the place of G1, dK -= (G2 + G2^T) K
    {
        frag kt[NK][2], qt[NK][2];
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                kt[n][kb] = __builtin_bit_cast(frag, kt_[n][kb]);
                qt[n][kb] = __builtin_bit_cast(frag, qt_[n][kb]);
            }
        auto put = [&](E *dst, int tt, const f32x4 (&x)[NK]) {
            const int t = 16 * tt + li;
            if (t >= nvalid) return;
            dst += (row0 + (size_t)t * p.H) * DK + ch0();
            if constexpr (NK == 2) TR::store8(dst, TR::cat(TR::from_f32(x[0]), TR::from_f32(x[1])));
            else TR::store(dst, TR::from_f32(x[0]));
        };
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int tt = rt0 + rt;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                if (kb <= tt / 2) {
                    const wfrag g1 = WD::tr(sG, L::PC, L::LDC, 32 * kb, 16 * tt, li, lg);
#pragma unroll
                    for (int n = 0; n < NK; ++n) pq[n][rt] = WD::ew(kt[n][kb], g1, pq[n][rt]);
                }
                if (kb >= tt / 2) {
                    const wfrag g1 = WD::load8(sG + (16 * tt + li) * L::LDC + 32 * kb + 8 * lg, L::PC);
#pragma unroll
                    for (int n = 0; n < NK; ++n) pe[n][rt] = WD::ew(qt[n][kb], g1, pe[n][rt]);
                }
            }
            f32x4 x[NK];
#pragma unroll
            for (int n = 0; n < NK; ++n) x[n] = pq[n][rt];
            put(p.dq, tt, x);
        }
        lds_barrier();
#pragma unroll
        for (int n = 0; n < NTI; ++n) symmetric(n);
        lds_barrier();
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int tt = rt0 + rt;
            f32x4 x[NK];
#pragma unroll
            for (int n = 0; n < NK; ++n) x[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const wfrag g2 = WD::load8(sG + (16 * tt + li) * L::LDC + 32 * kb + 8 * lg, L::PC);
#pragma unroll
                for (int n = 0; n < NK; ++n) x[n] = WD::ew(kt[n][kb], g2, x[n]);
            }
#pragma unroll
            for (int n = 0; n < NK; ++n) x[n] = pe[n][rt] - x[n];
            put(p.dk, tt, x);
        }
    }
    if (wave >= 4) return;
    // dalpha: M_it = sum_j X_ij D_{t-1,j}, then D_it M_it summed over rows; row 0 of X is the
    // exit state's (its own has no j < 0), so row tile 0 is needed for every t.  Wave w has the
    // tokens t of tile w.
    {
        const int t = 16 * w + li;
        const float g1hi = t > 0 ? gate[kBackGHi + t - 1] : 0.f, g1lo = t > 0 ? gate[kBackGLo + t - 1] : 0.f;
        wfrag D[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            if (kb > w / 2) continue;
            f32x4 x[2];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int j = 32 * kb + 8 * lg + e;
                x[e >> 2][e & 3] =
                    j < t ? __builtin_amdgcn_exp2f((g1hi - gate[kBackGHi + j]) + (g1lo - gate[kBackGLo + j])) : 0.f;
            }
            D[kb] = WD::split(x[0], x[1]);
        }
        const float gb = t > 0 ? gam[t - 1] : 1.f, s = gh[0] + gh[1] + gh[2] + gh[3];
        float cs = 0.f;
        for (int bi = 0; bi < 4; ++bi) {
            if (bi < w && bi != 0) continue;
            f32x4 m = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
                if (kb <= w / 2) m = WD::ww(WD::tr(sX, L::PC, L::LDC, 32 * kb, 16 * bi, li, lg), D[kb], m);
            const int i0 = 16 * bi + 4 * lg;
            if (i0 == 0) {
                cs += tail[t] * (m[0] + s * gb);
                m[0] = 0.f;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (i0 + q >= t) cs += back_decay(gate, i0 + q, t) * (m[q] + xm[i0 + q] * gb);
        }
        cs += __shfl_xor(cs, 16);
        cs += __shfl_xor(cs, 32);
        if (lg == 0 && t < nvalid) p.dalpha[row0 + (size_t)t * p.H] = cs;
    }
}

}  // namespace gdn
