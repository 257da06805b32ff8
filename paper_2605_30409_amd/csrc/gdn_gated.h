// The gated linear map (gdn_gated_linear_* in gdn_block.h):
//   g = x Wg^T,  u = x Wu^T,  h = act(g) o u
// and its gradient, which forms g and u again:
//   dg = dh o u o act'(g),  du = dh o act(g),   dx = dg Wg + du Wu,   dWg = dg^T x,  dWu = du^T x.
//
// Three products of one tiled kernel, and a kernel of their own for few rows (bound by memory: the weights).
// With d = [dg | du] in the workspace (pitch 2 Fp, Fp = F up to a multiple of 64, zeros between):
//   kGatedFwd   N side: rows of Wg and Wu, 32 of each in turn; M side: rows of x;   contraction over C
//   kGatedD     the same; the epilogue forms dg and du
//   kGatedDx    N side: columns of W; M side: rows of d;       contraction over 2 Fp (W: Wg, then Wu)
//   kGatedDw    N side: columns of x; M side: columns of d;    contraction over the rows
// The N side is the MFMA's A operand, so a lane has consecutive columns of a result's row: a pair of tiles in P32
// order (see gdn_device.h) gives it 8 of them.
//
// Tiles go to LDS by asynchronous 16-byte copies, 128 bytes of the contraction a stage ("granule": 16 bytes).
// An operand whose contraction runs along memory rows is stored as rows of 8 granules, granule g of row r at place
// g ^ (r & 7); one whose contraction runs down the rows is stored as it is in memory and read transposed
// (bf16: ds_read_b64_tr_b16, fp32: element by element).
#pragma once

#include "gdn_act.h"
#include "gdn_norm.h"

namespace gdn {

template <class E> struct GatedParams {
    const E *x, *wg, *wu, *dh;
    E *h, *d, *dx, *dwg, *dwu;
    long long ldx, ldw;          // elements from row to row of x and the weights
    int M, C, F, Fp;
    int act;
    int tiles_m, tiles_n;
};

enum GatedKind { kGatedFwd, kGatedD, kGatedDx, kGatedDw };

// Products of a 16-byte granule of each operand: k = 8 (bf16) or 4 (fp32) a lane.
__device__ __forceinline__ f32x4 mma_granule(uint16_t *, u32x4 a, u32x4 b, f32x4 c) {
    return Tr<uint16_t>::mma(a, b, c);
}
__device__ __forceinline__ f32x4 mma_granule(float *, u32x4 a, u32x4 b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = mma_f32_k4(__uint_as_float(a[i]), __uint_as_float(b[i]), c);
    return c;
}

// ---------------------------------------------------------------------------
// Few rows.  A workgroup has 16 hidden units (their rows of both weights), its waves every WAVES-th block of 128
// bytes of the contraction; rows are read straight into MFMA operands, two 64-byte halves of a line
// one after the other, and the waves' sums joined through LDS.

constexpr int kSkinnyWaves = 8;

template <class E, int MT> __global__ __launch_bounds__(64 * kSkinnyWaves) void gdn_gated_skinny_kernel(GatedParams<E> p) {
    constexpr int EG = 16 / (int)sizeof(E), KB = 8 * EG;       // elements of a granule, of a block
    __shared__ f32x4 sm[kSkinnyWaves][2 * MT][64];
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, li = l & 15, lg = l >> 4;
    const int n0 = 16 * blockIdx.x;
    const E *rg = p.wg + (size_t)min(n0 + li, p.F - 1) * p.ldw, *ru = p.wu + (size_t)min(n0 + li, p.F - 1) * p.ldw;
    const E *rx[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) rx[m] = p.x + (size_t)min(16 * m + li, p.M - 1) * p.ldx;
    f32x4 acc[2 * MT];
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int blocks = (p.C + KB - 1) / KB;
    typedef typename Vec8<E>::loose loose;
    // (columns past the end read as zeros, on both sides)
    auto granule = [&](const E *row, int k) {
        if (k + EG <= p.C) return __builtin_bit_cast(u32x4, *(const loose *)(row + k));
        E e[EG];
#pragma unroll
        for (int i = 0; i < EG; ++i) e[i] = k + i < p.C ? row[k + i] : E(0);
        return __builtin_bit_cast(u32x4, e);
    };
    auto turn = [&](int kb, auto n) {
        constexpr int NB = decltype(n)::value;
        u32x4 a[NB][2], b[NB][2], x[NB][2][MT];
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int k = (kb + j * kSkinnyWaves) * KB + (lg + 4 * i) * EG;
                a[j][i] = granule(rg, k);
                b[j][i] = granule(ru, k);
#pragma unroll
                for (int m = 0; m < MT; ++m) x[j][i][m] = granule(rx[m], k);
            }
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    acc[m] = mma_granule((E *)nullptr, a[j][i], x[j][i][m], acc[m]);
                    acc[MT + m] = mma_granule((E *)nullptr, b[j][i], x[j][i][m], acc[MT + m]);
                }
    };
    constexpr int NB = MT > 2 ? 2 : 4;
    int kb = w;
    for (; kb + (NB - 1) * kSkinnyWaves < blocks; kb += NB * kSkinnyWaves) turn(kb, std::integral_constant<int, NB>{});
    for (; kb < blocks; kb += kSkinnyWaves) turn(kb, std::integral_constant<int, 1>{});
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) sm[w][i][l] = acc[i];
    lds_barrier();
    if (w >= MT) return;
    f32x4 g = sm[0][w][l], u = sm[0][MT + w][l];
#pragma unroll
    for (int i = 1; i < kSkinnyWaves; ++i) g += sm[i][w][l], u += sm[i][MT + w][l];
    float v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = g[q];
    act_all<4>(v, p.act);
    const int m = 16 * w + li, n = n0 + 4 * lg;
    if (m >= p.M) return;
    E *out = p.h + (size_t)m * p.F + n;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (n + q < p.F) out[q] = Vec8<E>::cvt(v[q] * u[q]);
}

// ---------------------------------------------------------------------------
// Tiles.

// One asynchronous copy: lane l's 16 bytes to LDS at `lds` + 16 l.  (As assembly, so that the compiler does
// not wait for it before every read of LDS; it has no output register.  M0 holds the LDS address.)
__device__ __forceinline__ void copy_tile(const void *base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void copy_lane(const void *src, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(src) : "memory");
}

__device__ const u32x4 kZeroGranule = {0u, 0u, 0u, 0u};

// An operand of R rows (or columns) of the tile, staged by NW waves.
//   ROWS: rows of memory along the contraction.  COLS: contraction down the rows.
template <class E, bool COLS, int R, int NW> struct Operand {
    static constexpr int EG = 16 / (int)sizeof(E), KB = 8 * EG;     // elements of a granule, of a stage
    static constexpr int BYTES = R * 128, COPIES = BYTES / 1024 / NW;
    static constexpr int GR = R / EG;                               // COLS: granules of a row
    static_assert(BYTES % (1024 * NW) == 0, "whole copies");
    uint32_t off[COPIES];
    int l, w;

    // COLS: place of granule g of row k.  Four rows that a transposed read takes at once, 16 bytes apart, lie 64
    // bytes apart after it (bf16); fp32 reads 4 rows k, k + 4, .. of 64 bytes each.
    static __device__ __forceinline__ int place(int k, int g) {
        if (sizeof(E) == 2) return g ^ ((k & 3) << 2) ;
        return g ^ (((k >> 2) & 3) << 2);
    }
    // row(r): memory row of the tile's row r, or for COLS granule(g): first column of granule g
    template <class Row> __device__ __forceinline__ void init(int wave, int lane, long long ld, Row row) {
        w = wave, l = lane;
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            const int at = (w + i * NW) * 64 + l;                   // granule's place in the tile
            if (COLS) {
                const int k = at / GR, g = place(k, at % GR);
                off[i] = (uint32_t)(((long long)k * ld + row(g)) * (long long)sizeof(E));
            } else {
                const int r = at / 8, g = (at & 7) ^ (r & 7);
                off[i] = (uint32_t)((row(r) * ld + g * EG) * (long long)sizeof(E));
            }
        }
    }
    __device__ __forceinline__ void stage(const E *base, uint32_t lds) const {
#pragma unroll
        for (int i = 0; i < COPIES; ++i) copy_tile(base, off[i], lds + (w + i * NW) * 1024);
    }
    // A stage with `k` < KB valid elements of the contraction: zeros behind them.
    __device__ __forceinline__ void stage_tail(const E *base, uint32_t lds, int k) const {
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            const int at = (w + i * NW) * 64 + l;
            const int e = COLS ? at / GR : ((at & 7) ^ ((at / 8) & 7)) * EG;
            copy_lane(e < k ? (const char *)base + off[i] : (const char *)&kZeroGranule, lds + (w + i * NW) * 1024);
        }
    }
    // Granule kk (of two 64-byte halves) of tile t's 16 rows; P32: tiles 2 j, 2 j + 1 stand for 32 columns in
    // P32 order (for ROWS the order is in the staged rows).
    template <bool P32> static __device__ __forceinline__ u32x4 frag(const unsigned char *tile, int r0, int t, int kk, int li, int lg) {
        if constexpr (!COLS) {
            const int r = r0 + 16 * t + li;
            return *(const u32x4 *)(tile + r * 128 + (((lg + 4 * kk) ^ (li & 7)) << 4));
        } else if constexpr (sizeof(E) == 2) {
            typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
            const int k = 32 * kk + 8 * lg + (li >> 2);
            const int c = P32 ? r0 + 32 * (t >> 1) + 8 * (li & 3) + 4 * (t & 1) : r0 + 16 * t + 4 * (li & 3);
            auto at = [&](int kr) { return (lds_i16x4 *)(tile + kr * (2 * R) + place(kr, c >> 3) * 16 + (c & 7) * 2); };
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(k));
            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(k + 4));
            return Tr<uint16_t>::cat(__builtin_bit_cast(u32x2, lo), __builtin_bit_cast(u32x2, hi));
        } else {
            const int c = P32 ? r0 + 32 * (t >> 1) + p32_row(t & 1, li) : r0 + 16 * t + li;
            u32x4 f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = 16 * kk + 4 * lg + j;
                f[j] = *(const uint32_t *)(tile + k * (4 * R) + place(k, c >> 2) * 16 + (c & 3) * 4);
            }
            return f;
        }
    }
};

// 8 consecutive results of a row from column n on, of which those before `end` are there.
template <class E> __device__ __forceinline__ void store_row(E *row, int n, int end, const float *v) {
    if (n + 8 <= end) {
        Vec8<E>::store(row + n, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (n + i < end) row[n + i] = Vec8<E>::cvt(v[i]);
    }
}

template <class E, int KIND, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 2) void gdn_gated_tile_kernel(GatedParams<E> p) {
    constexpr bool FWD = KIND == kGatedFwd || KIND == kGatedD;
    constexpr int NW = WM * WN, MT = BM / WM / 16, NT = BN / WN / 16;
    using OpN = Operand<E, !FWD, BN, NW>;
    using OpM = Operand<E, KIND == kGatedDw, BM, NW>;
    constexpr int KB = OpN::KB, EG = OpN::EG, STAGE = (BM + BN) * 128;
    extern __shared__ __align__(1024) unsigned char smem[];
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, li = l & 15, lg = l >> 4;
    const int wm = w / WN, wn = w % WN;

    // Tiles of an XCD (workgroups go to the 8 of them in turn) are neighbours: runs of 8 rows of tiles, column by
    // column, so that what its CUs read together fits its L2.
    int tm, tn;
    {
        const int total = p.tiles_m * p.tiles_n, per = total / 8, more = total % 8;
        const int xcd = blockIdx.x % 8;
        const int id = xcd * per + min(xcd, more) + blockIdx.x / 8;
        constexpr int RUN = 8;
        const int run = id / (RUN * p.tiles_n), in = id - run * RUN * p.tiles_n;
        const int height = min(RUN, p.tiles_m - run * RUN);
        tm = run * RUN + in % height;
        tn = in / height;
    }
    const int m0 = tm * BM, n0 = tn * (FWD ? BN / 2 : BN);

    OpN on;
    OpM om;
    const E *bn, *bn2 = nullptr, *bm;
    long long step_n = KB, step_m = KB;        // elements from stage to stage
    int stages, half = 0, tail;                // kGatedDx: stages of Wg
    if constexpr (FWD) {
        // rows 64 j + 32 s + 16 a + i of the tile: hidden unit 32 j + p32_row(a, i) of Wg (s = 0) or Wu (s = 1); the
        // two weights' distance goes into the offset of the second half of the copies
        bn = p.wg;
        bm = p.x + (long long)m0 * p.ldx;
        om.init(w, l, p.ldx, [&](int r) { return (long long)min(r, p.M - 1 - m0); });
        stages = (p.C + KB - 1) / KB;
        tail = p.C - (stages - 1) * KB;
    } else if constexpr (KIND == kGatedDx) {
        bn = p.wg;
        bn2 = p.wu;
        bm = p.d + (long long)m0 * 2 * p.Fp;
        on.init(w, l, p.ldw, [&](int g) { return (long long)min(n0 + g * EG, (p.C - 1) / EG * EG); });
        om.init(w, l, 2 * p.Fp, [&](int r) { return (long long)min(r, p.M - 1 - m0); });
        half = p.Fp / KB;
        stages = 2 * half;
        tail = 0;
        step_n = (long long)KB * p.ldw;
    } else {
        bn = p.x;
        bm = p.d;
        on.init(w, l, p.ldx, [&](int g) { return (long long)min(n0 + g * EG, (p.C - 1) / EG * EG); });
        om.init(w, l, 2 * p.Fp, [&](int g) { return (long long)min(m0 + g * EG, 2 * p.Fp - EG); });
        stages = (p.M + KB - 1) / KB;
        tail = p.M - (stages - 1) * KB;
        step_n = (long long)KB * p.ldx;
        step_m = (long long)KB * 2 * p.Fp;
    }
    // FWD: Wg's rows and Wu's through bases of their own
    const E *wrow[2];
    if constexpr (FWD) {
        wrow[0] = p.wg + (long long)n0 * p.ldw;
        wrow[1] = p.wu + (long long)n0 * p.ldw;
        on.init(w, l, p.ldw, [&](int r) {
            return (long long)min(32 * (r >> 6) + p32_row((r >> 4) & 1, r & 15), p.F - 1 - n0);
        });
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;

    auto stage = [&](int s) {
        const uint32_t lds = lds0 + (s & 1) * STAGE;
        if constexpr (FWD) {
            const bool end = s == stages - 1 && tail < KB;
            // a copy holds 8 rows: all of Wg or all of Wu
#pragma unroll
            for (int i = 0; i < OpN::COPIES; ++i) {
                const int c = w + i * NW;
                const E *base = wrow[(c >> 2) & 1] + (long long)s * KB;
                const uint32_t to = lds + BM * 128 + c * 1024;
                if (!end) copy_tile(base, on.off[i], to);
                else copy_lane(((l & 7) ^ ((l >> 3) & 7)) * EG < tail ? (const char *)base + on.off[i] : (const char *)&kZeroGranule, to);
            }
            const E *xb = bm + (long long)s * KB;
            if (!end) om.stage(xb, lds);
            else om.stage_tail(xb, lds, tail);
        } else if constexpr (KIND == kGatedDx) {
            const int f = (s < half ? s : s - half) * KB;
            const E *base = (s < half ? bn : bn2) + (long long)f * p.ldw;
            if (f + KB <= p.F) on.stage(base, lds + BM * 128);
            else on.stage_tail(base, lds + BM * 128, p.F - f);
            om.stage(bm + (long long)s * KB, lds);
        } else {
            const bool end = s == stages - 1 && tail < KB;
            if (!end) {
                on.stage(bn + s * step_n, lds + BM * 128);
                om.stage(bm + s * step_m, lds);
            } else {
                on.stage_tail(bn + s * step_n, lds + BM * 128, tail);
                om.stage_tail(bm + s * step_m, lds, tail);
            }
        }
    };

    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    stage(0);
    for (int s = 0; s < stages; ++s) {
        asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        if (s + 1 < stages) stage(s + 1);
        const unsigned char *tm_ = smem + (s & 1) * STAGE, *tn_ = tm_ + BM * 128;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            u32x4 a[NT], b[MT];
#pragma unroll
            for (int j = 0; j < NT; ++j) a[j] = OpN::template frag<true>(tn_, wn * (BN / WN), j, kk, li, lg);
#pragma unroll
            for (int i = 0; i < MT; ++i) b[i] = OpM::template frag<false>(tm_, wm * (BM / WM), i, kk, li, lg);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = mma_granule((E *)nullptr, a[j], b[i], acc[i][j]);
        }
    }

    // Results.  Lane (li, lg): row 16 i + li, columns 8 lg .. 8 lg + 7 of a pair of tiles.
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int m = m0 + wm * (BM / WM) + 16 * i + li;
        if constexpr (FWD) {
            if (m >= p.M) continue;
#pragma unroll
            for (int j = 0; j < NT; j += 4) {
                const int n = n0 + (wn * (BN / WN) + 16 * j) / 2 + 8 * lg;
                float g[8], u[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) g[q] = acc[i][j + (q >> 2)][q & 3], u[q] = acc[i][j + 2 + (q >> 2)][q & 3];
                if constexpr (KIND == kGatedFwd) {
                    act_all<8>(g, p.act);
#pragma unroll
                    for (int q = 0; q < 8; ++q) g[q] *= u[q];
                    store_row(p.h + (size_t)m * p.F, n, p.F, g);
                } else {
                    float dh[8];
                    Vec8<E> v;
                    const E *row = p.dh + (size_t)m * p.F;
                    if (n >= p.Fp) continue;
                    if (n + 8 <= p.F) v.load(row + n);
                    else v.load_some(row + n, max(p.F - n, 0));
                    v.values(dh);
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        float a, s;
                        act_and_slope(g[q], p.act, a, s);
                        const bool on = n + q < p.F;
                        g[q] = on ? dh[q] * u[q] * s : 0.f;
                        u[q] = on ? dh[q] * a : 0.f;
                    }
                    E *d = p.d + (size_t)m * 2 * p.Fp + n;
                    Vec8<E>::store(d, g);
                    Vec8<E>::store(d + p.Fp, u);
                }
            }
        } else {
            E *row;
            if constexpr (KIND == kGatedDx) {
                if (m >= p.M) continue;
                row = p.dx + (size_t)m * p.C;
            } else {
                const int f = m < p.Fp ? m : m - p.Fp;
                if (f >= p.F) continue;
                row = (m < p.Fp ? p.dwg : p.dwu) + (size_t)f * p.C;
            }
#pragma unroll
            for (int j = 0; j < NT; j += 2) {
                const int n = n0 + wn * (BN / WN) + 16 * j + 8 * lg;
                float v[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] = acc[i][j + (q >> 2)][q & 3];
                store_row(row, n, p.C, v);
            }
        }
    }
}

// Rows copied to a pitch that is a multiple of 64 elements, zeros behind them: operands whose rows do not start
// at 16 bytes.
template <class E> struct PackParams {
    const E *src;
    E *dst;
    long long rows;
    int C, ld;
};
template <class E> __global__ __launch_bounds__(256) void gdn_gated_pack_kernel(PackParams<E> p) {
    const int G = p.ld / 8;
    const long long unit = (long long)blockIdx.x * 256 + threadIdx.x, r = unit / G;
    const int c = (int)(unit % G) * 8;
    if (r >= p.rows) return;
    const E *row = p.src + r * p.C;
    Vec8<E> v;
    if (c + 8 <= p.C) v.load(row + c);
    else v.load_some(row + min(c, p.C - 1), max(p.C - c, 0));
    float f[8];
    v.values(f);
    Vec8<E>::store(p.dst + r * p.ld + c, f);
}

}  // namespace gdn
