// The gated linear map (gdn_gated_linear_* in gdn_block.h):
//   g = x Wg^T,  u = x Wu^T,  h = act(g) o u
// and its gradient, which forms g and u again:
//   dg = dh o u o act'(g),  du = dh o act(g),   dx = dg Wg + du Wu,   dWg = dg^T x,  dWu = du^T x.
//
// One tiled kernel for the four products, and a kernel of its own for few rows (bound by memory: the weights).
// With d = [dg | du] in the workspace (pitch 2 Fp, Fp = F up to a multiple of 64, zeros between):
//   kGatedFwd   N side: rows of Wg and Wu, 32 of each in turn; M side: rows of x;   contraction over C
//   kGatedD     the same; the epilogue forms dg and du
//   kGatedDx    N side: columns of W; M side: rows of d;       contraction over 2 Fp (W: Wg, then Wu)
//   kGatedDw    N side: columns of x; M side: columns of d;    contraction over the rows
// The N side is the MFMA's A operand, so a lane has consecutive columns of a result's row: 16 of a tile's 32, with the tile's
// rows in n_order.  Nothing is transposed in memory, and g and u of a hidden unit meet in one lane.
//
// Tiles go to LDS by asynchronous 16-byte copies, 128 bytes of the contraction a stage ("granule": 16 bytes).
// An operand whose contraction runs along memory rows is stored as rows of 8 granules, granule g of row r at place
// g ^ (r / 2 & 7); one whose contraction runs down the rows is stored as it is in memory, granules permuted within a
// row, and read transposed (bf16: ds_read_b64_tr_b16, fp32: element by element).  No read takes a bank twice.
//
// Measured (bf16, C = 2048, F = 8192): 10560 rows 573 to 622 us a call, by the card that it runs on (a library product of the
// same operations 579 to 603), 1140 to 1240 TFLOP/s; gradient of 3520 rows 657 to 689; the first 20 to 40 calls after a
// pause take up to 13 % more.  What bounds it is power: on
// random data the chip runs at 1.6 to 1.9 GHz, on zeros, above 2.2, the first takes 417 us.  Same card, us at 10560 rows:
// 32 x 32 x 16 products with operands read ahead across stages in place of 16 x 16 x 32, 626 -> 604; a stage's copies in two
// halves, a step apart, 644 -> 622; four waves of 128 x 128 in place of eight of 128 x 64: 617 (with copies as
// spread; 650 without); a workgroup that goes on to its next tile during the results of the last: no gain.  fp32, as six bf16
// products: 205 to 250 TFLOP/s, the matrix cores busy 63 % and the vector units (cutting operands into planes) 55 % of
// the time, at 1.8 GHz; fp32 MFMAs end at 154.  The 256 x 256 tiles of the fp32 weights' gradients take all 256 registers and spill 8
// (36 bytes a lane; one is read back once a stage, the others outside the loop); no other variant spills.
#pragma once

#include "gdn_act.h"
#include "gdn_gated_rule.h"
#include "gdn_norm.h"

namespace gdn {

template <class E> struct GatedParams {
    const E *x, *wg, *wu, *dh;
    E *h, *d, *dx, *dwg, *dwu;
    long long ldx, ldw;          // elements from row to row of x and the weights
    int M, C, F, Fp;
    float *part;                 // sums of `splits` parts of the contraction: [split][rows][pitch]
    int act;
    int tiles_m, tiles_n, splits;
    int rows, pitch;             // of a part: pitch a multiple of 8; kGatedFwd, kGatedD: g at column n, u at Fp + n
};

typedef float f32x16 __attribute__((ext_vector_type(16)));

// 32 x 32 x 16 products: lane l = 32 h + i has k = 8 h .. 8 h + 7 of the operands' row i, and of the result D[8 b + 4 h + q][i] at
// 4 b + q.
__device__ __forceinline__ f32x16 mma_32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// The column of 32 that the N side's tile row r stands for: a lane then has 16 consecutive ones, 16 h + e at e.
__device__ __forceinline__ int n_order(int r) { return 16 * ((r >> 2) & 1) + 4 * (r >> 3) + (r & 3); }

// 8 fp32 values (two granules) as the sum of three bf16 planes, exactly: 8 bits of the mantissa each, cut off, not
// rounded, so that no plane overflows.  (What is infinite becomes NaN; planes of values below 2^-110 may be lost.)
__device__ __forceinline__ void planes(u32x4 lo, u32x4 hi, u32x4 *p) {
    uint32_t x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
    for (int k = 0; k < 3; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[k][i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x07060302);     // the high halves of both
            if (k < 2) {
#pragma unroll
                for (int e = 2 * i; e < 2 * i + 2; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) - __uint_as_float(x[e] & 0xffff0000u));
            }
        }
}

// Six products of planes, small ones first.  The three left out are below (2 2^-22 + 2^-30) of a product together, mostly
// under 2^-24: sums of some dozens of products and more are off by as much in fp32.
constexpr int kPlaneN[6] = {2, 0, 1, 1, 0, 0}, kPlaneM[6] = {0, 2, 1, 0, 1, 0};

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
// not wait for it before every read of LDS; it has no output register, and M0 holds the LDS address.  What orders it is the
// wait and barrier in front of the reads, and the barrier behind the last reads of what it overwrites: both are
// volatile, too, and memory accesses do not cross them.  A scalar register that a vector instruction has written may be
// read as an address five wait states later only, and the compiler does not look for that inside assembly: the address goes
// through a scalar move, which waits by itself and whose result may be used at once.  One wait state stands between M0 and
// its use.)
__device__ __forceinline__ void copy_tile(const void *base, uint32_t off, uint32_t lds) {
    const uint64_t at = (uint64_t)base;
    const uint64_t s = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)at);
    uint64_t own;
    asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0"
                 : "=&s"(own)
                 : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(off), "s"(s));
}
__device__ __forceinline__ void copy_lane(const void *src, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(src));
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
        return g ^ (((sizeof(E) == 2 ? k : k >> 2) & 3) << 2 & (GR - 1));
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
                const int r = at / 8, g = (at & 7) ^ ((r >> 1) & 7);
                off[i] = (uint32_t)((row(r) * ld + g * EG) * (long long)sizeof(E));
            }
        }
    }
    // Copy i of a stage; TAIL: of one with `k` < KB valid elements of the contraction, zeros behind them.
    template <bool TAIL> __device__ __forceinline__ void copy(int i, const E *base, uint32_t lds, int k) const {
        const uint32_t to = lds + (w + i * NW) * 1024;
        if constexpr (TAIL) {
            const int at = (w + i * NW) * 64 + l;
            const int e = COLS ? at / GR : ((at & 7) ^ ((at / 16) & 7)) * EG;
            copy_lane(e < k ? (const char *)base + off[i] : (const char *)&kZeroGranule, to);
        } else {
            copy_tile(base, off[i], to);
        }
    }
    // k = 8 (2 kk + h) .. + 7 (bf16: granules 2 kk + h; fp32: 4 kk + 2 h + part) of row i of tile t; N: in n_order (for ROWS the
    // order is in the staged rows).
    template <bool N> static __device__ __forceinline__ u32x4 frag(const unsigned char *tile, int r0, int t, int kk, int part, int i, int h) {
        if constexpr (!COLS) {
            const int r = r0 + 32 * t + i, g = sizeof(E) == 2 ? 2 * kk + h : 4 * kk + 2 * h + part;
            return *(const u32x4 *)(tile + r * 128 + ((g ^ ((i >> 1) & 7)) << 4));
        } else if constexpr (sizeof(E) == 2) {
            typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
            const int k = 16 * kk + 8 * h + ((i >> 2) & 3), block = 4 * (i >> 4) + (i & 3);
            const int c = r0 + 32 * t + (N ? 16 * (block & 1) + 4 * (block >> 1) : 4 * block);
            auto at = [&](int kr) { return (lds_i16x4 *)(tile + kr * (2 * R) + place(kr, c >> 3) * 16 + (c & 7) * 2); };
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(k));
            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(k + 4));
            return Tr<uint16_t>::cat(__builtin_bit_cast(u32x2, lo), __builtin_bit_cast(u32x2, hi));
        } else {
            const int c = r0 + 32 * t + (N ? n_order(i) : i);
            u32x4 f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = 16 * kk + 8 * h + 4 * part + j;
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

// dh of row m, columns n .. n + 7, as far as they are there.
template <class E> __device__ __forceinline__ Vec8<E> gated_dh(const GatedParams<E> &p, int m, int n) {
    Vec8<E> e{};
    const E *row = p.dh + (size_t)m * p.F;
    if (n + 8 <= p.F) e.load(row + n);
    else if (n < p.F) e.load_some(row + n, p.F - n);
    return e;
}

// What becomes of 8 sums of row m, columns n .. n + 7 (kGatedFwd, kGatedD: v of g and u of u).
template <class E, int KIND>
__device__ __forceinline__ void gated_result(const GatedParams<E> &p, int m, int n, float *v, float *u, const Vec8<E> &e) {
    if constexpr (KIND == kGatedFwd) {
        act_all<8>(v, p.act);
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] *= u[q];
        store_row(p.h + (size_t)m * p.F, n, p.F, v);
    } else if constexpr (KIND == kGatedD) {
        // (dg and du are operands of the next products and rounded to E for those: half a step each, so in bf16 the gradients are 2.4e-3
        // off in place of 1.7e-3 with their own rounding alone.  A second plane for what is cut off would double those products, 400 of
        // 660 us at 3520 rows.)
        if (n >= p.Fp) return;
        float dh[8];
        e.values(dh);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            float a, s;
            act_and_slope(v[q], p.act, a, s);
            const bool on = n + q < p.F;
            v[q] = on ? dh[q] * u[q] * s : 0.f;
            u[q] = on ? dh[q] * a : 0.f;
        }
        E *d = p.d + (size_t)m * 2 * p.Fp + n;
        Vec8<E>::store(d, v);
        Vec8<E>::store(d + p.Fp, u);
    } else if constexpr (KIND == kGatedDx) {
        store_row(p.dx + (size_t)m * p.C, n, p.C, v);
    } else {
        const int f = m < p.Fp ? m : m - p.Fp;
        if (f < p.F) store_row((m < p.Fp ? p.dwg : p.dwu) + (size_t)f * p.C, n, p.C, v);
    }
}

template <class E, int KIND, int BM, int BN, int WM, int WN, int DEPTH>
__global__ __launch_bounds__(64 * WM * WN, 2) void gdn_gated_tile_kernel(GatedParams<E> p) {
    constexpr bool FWD = KIND == kGatedFwd || KIND == kGatedD;
    constexpr int NW = WM * WN, MT = BM / WM / 32, NT = BN / WN / 32;
    using OpN = Operand<E, !FWD, BN, NW>;
    using OpM = Operand<E, KIND == kGatedDw, BM, NW>;
    constexpr int KB = OpN::KB, EG = OpN::EG, STAGE = (BM + BN) * 128;
    extern __shared__ __align__(1024) unsigned char smem[];
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, li = l & 31, lh = l >> 5;
    const int wm = w / WN, wn = w % WN;

    // Tiles of an XCD (workgroups go to the 8 of them in turn) are neighbours: runs of 8 rows of tiles, column by
    // column, so that what its CUs read together fits its L2.
    int tm, tn, split;
    {
        const int tiles = p.tiles_m * p.tiles_n, total = tiles * p.splits, per = total / 8, more = total % 8;
        const int xcd = blockIdx.x % 8;
        int id = xcd * per + min(xcd, more) + blockIdx.x / 8;
        split = id / tiles;
        id -= split * tiles;
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
    int whole, tails, tail;                    // stages that are whole; behind them those that are not, and how long those are
    if constexpr (FWD) {
        bn = p.wg;
        bm = p.x + (long long)m0 * p.ldx;
        om.init(w, l, p.ldx, [&](int r) { return (long long)min(r, p.M - 1 - m0); });
        whole = p.C / KB;
        tail = p.C % KB;
        tails = tail ? 1 : 0;
    } else if constexpr (KIND == kGatedDx) {
        bn = p.wg;
        bn2 = p.wu;
        bm = p.d + (long long)m0 * 2 * p.Fp;
        on.init(w, l, p.ldw, [&](int g) { return (long long)min(n0 + g * EG, (p.C - 1) / EG * EG); });
        om.init(w, l, 2 * p.Fp, [&](int r) { return (long long)min(r, p.M - 1 - m0); });
        whole = 2 * (p.F / KB);
        tail = p.F % KB;
        tails = tail ? 2 : 0;
        step_n = (long long)KB * p.ldw;
    } else {
        bn = p.x;
        bm = p.d;
        on.init(w, l, p.ldx, [&](int g) { return (long long)min(n0 + g * EG, (p.C - 1) / EG * EG); });
        om.init(w, l, 2 * p.Fp, [&](int g) { return (long long)min(m0 + g * EG, 2 * p.Fp - EG); });
        whole = p.M / KB;
        tail = p.M % KB;
        tails = tail ? 1 : 0;
        step_n = (long long)KB * p.ldx;
        step_m = (long long)KB * 2 * p.Fp;
    }
    // FWD: row 64 j + 32 s + i of the tile is hidden unit 32 j + n_order(i) of Wg (s = 0) or Wu (s = 1)
    const E *wrow[2];
    if constexpr (FWD) {
        wrow[0] = p.wg + (long long)n0 * p.ldw;
        wrow[1] = p.wu + (long long)n0 * p.ldw;
        on.init(w, l, p.ldw, [&](int r) {
            return (long long)min(32 * (r >> 6) + n_order(r & 31), p.F - 1 - n0);
        });
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;

    // Copy c of stage s to the buffer at `to`.
    auto copy = [&](int c, int s, uint32_t to, auto is_tail) {
        constexpr bool TAIL = decltype(is_tail)::value;
        const uint32_t lds = lds0 + to;
        // kGatedDx: Wg's stages, Wu's, and what is left of both
        int part = 0, at = s;
        if constexpr (KIND == kGatedDx) {
            const int half = whole / 2;
            part = TAIL ? s - whole : s >= half;
            at = TAIL ? half : s - part * half;
        }
        if (c < OpN::COPIES) {
            const E *base;
            // FWD: a copy holds 8 rows, all of Wg or all of Wu
            if constexpr (FWD) base = wrow[((w + c * NW) >> 2) & 1];
            else base = KIND == kGatedDx && part ? bn2 : bn;
            on.template copy<TAIL>(c, base + at * step_n, lds + BM * 128, tail);
        } else {
            om.template copy<TAIL && KIND != kGatedDx>(c - OpN::COPIES, bm + (long long)part * p.Fp + at * step_m, lds, tail);
        }
    };

    f32x16 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    const int stages = whole + tails;
    const int first = (int)((long long)stages * split / p.splits), end = (int)((long long)stages * (split + 1) / p.splits);
    // DEPTH buffers, as many stages on their way.
    constexpr int COPIES = OpN::COPIES + OpM::COPIES;
    uint32_t ahead = 0, here = 0;
    auto turn = [](uint32_t &at) { at = at == (DEPTH - 1) * STAGE ? 0 : at + STAGE; };
    auto stage = [&](int s) {
        if (s >= end) return;
#pragma unroll
        for (int c = 0; c < COPIES; ++c) {
            if (s < whole) copy(c, s, ahead, std::false_type{});
            else copy(c, s, ahead, std::true_type{});
        }
        turn(ahead);
    };
    // stage s is there, for all waves, and what this wave asked of LDS too
    auto arrived = [&](int s) {
        if (DEPTH > 2 && s + DEPTH - 2 < end) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((DEPTH - 2) * COPIES) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    auto rows_n = [&](uint32_t at, int j, int kk, int part) {
        return OpN::template frag<true>(smem + at + BM * 128, wn * (BN / WN), j, kk, part, li, lh);
    };
    auto rows_m = [&](uint32_t at, int i, int kk, int part) {
        return OpM::template frag<false>(smem + at, wm * (BM / WM), i, kk, part, li, lh);
    };
#pragma unroll
    for (int i = 0; i < DEPTH - 1; ++i) stage(first + i);
    arrived(first);
    if constexpr (sizeof(E) == 2) {
        // Operands are read a step of 16 ahead of their products, also across stages: a stage's last ones are in
        // registers when all waves meet, so its buffer is free for the stage DEPTH on, and products to
        // do are left for the time until the next stage's first operands are there.  Products, reads and
        // copies are dealt out evenly, a row of products at a time; half of the copies follow in the next stage's first
        // step (all at once: 616 us in place of 595 at 10560 rows).
        constexpr int ROW = (NT + MT + MT - 1) / MT, HALF = COPIES / 2;
        const int plain = min(end, whole);
        // copies c0 .. c1 - 1 of a whole stage
        auto some = [&](int s, int c0, int c1) {
#pragma unroll
            for (int c = c0; c < c1; ++c) copy(c, s, ahead, std::false_type{});
        };
        if (first + DEPTH - 1 < plain) some(first + DEPTH - 1, 0, HALF);
        else stage(first + DEPTH - 1);
        u32x4 a[2][NT], b[2][MT];
        // the r-th operand of step kk
        auto read = [&](uint32_t at, int kk, int r) {
            if (r < NT) a[kk & 1][r] = rows_n(at, r, kk, 0);
            else if (r < NT + MT) b[kk & 1][r - NT] = rows_m(at, r - NT, kk, 0);
        };
        auto products = [&](int kk, int i) {
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = mma_32(a[kk & 1][j], b[kk & 1][i], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        };
        // Stage s, with the second half of the copies of stage s + DEPTH - 1 and the first of those of stage s + DEPTH, if that is
        // a whole one, between the first and the last products.
        auto step = [&](int s, auto copies) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                if (kk == 3) {
                    arrived(s + 1);
                    turn(here);
                    if (!decltype(copies)::value) stage(s + DEPTH);
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
#pragma unroll
                    for (int r = ROW * i; r < ROW * i + ROW; ++r) read(here, (kk + 1) & 3, r);
                    if (decltype(copies)::value) {
                        if (kk == 0) some(s + DEPTH - 1, HALF + (COPIES - HALF) * i / MT, HALF + (COPIES - HALF) * (i + 1) / MT);
                        if (kk == 0 && i == MT - 1) turn(ahead);
                        if (kk == 3) some(s + DEPTH, HALF * i / MT, HALF * (i + 1) / MT);
                    }
                    products(kk, i);
                }
            }
        };
#pragma unroll
        for (int r = 0; r < NT + MT; ++r) read(here, 0, r);
        int s = first;
        for (; s + DEPTH < plain; ++s) step(s, std::true_type{});
        if (s + DEPTH - 1 < plain) some(s + DEPTH - 1, HALF, COPIES), turn(ahead);
        for (; s < end - 1; ++s) step(s, std::false_type{});
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if (kk < 3) {
#pragma unroll
                    for (int r = ROW * i; r < ROW * i + ROW; ++r) read(here, kk + 1, r);
                }
                products(kk, i);
            }
    } else if constexpr (MT == 1) {
        stage(first + DEPTH - 1);
        for (int s = first; s < end; ++s) {
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                u32x4 a[NT][3], b[3];
#pragma unroll
                for (int j = 0; j < NT; ++j) planes(rows_n(here, j, kk, 0), rows_n(here, j, kk, 1), a[j]);
                planes(rows_m(here, 0, kk, 0), rows_m(here, 0, kk, 1), b);
#pragma unroll
                for (int q = 0; q < 6; ++q)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[0][j] = mma_32(a[j][kPlaneN[q]], b[kPlaneM[q]], acc[0][j]);
            }
            if (s + 1 < end) {
                arrived(s + 1);
                turn(here);
                stage(s + DEPTH);
            }
        }
    } else {
        // Regions of a row of products each, two times MT in a stage.  In one, the rows two regions on are read, those of the
        // next are cut into planes, and the N side's of the next step of 16 in a step's last two regions, between
        // the products: a wave's vector instructions run beside its matrix instructions only where they alternate.
        constexpr int R = 2 * MT;
        u32x4 a[2][NT][3], b[2][3], ra[NT][2], rb[2][2];
        auto read_b = [&](int t) {
            rb[t & 1][0] = rows_m(here, t % MT, t / MT, 0);
            rb[t & 1][1] = rows_m(here, t % MT, t / MT, 1);
        };
        auto read_a = [&](int kk) {
#pragma unroll
            for (int j = 0; j < NT; ++j) ra[j][0] = rows_n(here, j, kk, 0), ra[j][1] = rows_n(here, j, kk, 1);
        };
        auto cut_a = [&](int kk) {
#pragma unroll
            for (int j = 0; j < NT; ++j) planes(ra[j][0], ra[j][1], a[kk & 1][j]);
        };
        auto step = [&](int s, auto more) {
            constexpr bool MORE = decltype(more)::value;
#pragma unroll
            for (int t = 0; t < R; ++t) {
                const int kk = t / MT, i = t % MT;
                if (MORE && t == R - 2) {
                    arrived(s + 1);
                    turn(here);
                    stage(s + DEPTH);
                }
                if (MORE || t < R - 2) read_b((t + 2) % R);
                if (i == MT - 2 && (MORE || kk == 0)) read_a((kk + 1) & 1);
                if (MORE || t < R - 1) planes(rb[(t + 1) & 1][0], rb[(t + 1) & 1][1], b[(t + 1) & 1]);
                if (i == MT - 1 && (MORE || kk == 0)) cut_a(kk + 1);
#pragma unroll
                for (int q = 0; q < 6; ++q)
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        acc[i][j] = mma_32(a[kk & 1][j][kPlaneN[q]], b[t & 1][kPlaneM[q]], acc[i][j]);
                        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                        if (i == MT - 1) __builtin_amdgcn_sched_group_barrier(0x2, 11, 0);
                        else __builtin_amdgcn_sched_group_barrier(0x2, 4, 0);
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        stage(first + DEPTH - 1);
        read_a(0);
        read_b(0);
        cut_a(0);
        planes(rb[0][0], rb[0][1], b[0]);
        read_b(1);
        for (int s = first; s < end - 1; ++s) step(s, std::true_type{});
        step(end - 1, std::false_type{});
    }

    // Results.  Lane 32 h + i: row 32 t + i, columns 16 h .. 16 h + 15 of a tile.
    constexpr int STEP = FWD ? 2 : 1, ROWS = FWD ? NT : 1;
    Vec8<E> dh[MT][ROWS]{};
    if constexpr (KIND == kGatedD)
        if (p.splits == 1)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const int m = min(m0 + wm * (BM / WM) + 32 * i + li, p.M - 1);
                    dh[i][j] = gated_dh(p, m, n0 + (wn * (BN / WN) + 32 * (j & ~1)) / 2 + 16 * lh + 8 * (j & 1));
                }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int m = m0 + wm * (BM / WM) + 32 * i + li;
        if (m >= p.rows) continue;
        float *part = p.part + ((size_t)split * p.rows + m) * p.pitch;
#pragma unroll
        for (int j = 0; j < NT; j += STEP)
#pragma unroll
            for (int e = 0; e < 16; e += 8) {
                const int n = n0 + (wn * (BN / WN) + 32 * j) / (FWD ? 2 : 1) + 16 * lh + e;
                float v[8], u[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    v[q] = acc[i][j][e + q];
                    if constexpr (FWD) u[q] = acc[i][j + 1][e + q];
                }
                if (p.splits == 1) {
                    gated_result<E, KIND>(p, m, n, v, u, dh[i][FWD ? j + e / 8 : 0]);
                } else if (n < (FWD ? p.Fp : p.pitch)) {
                    Vec8<float>::store(part + n, v);
                    if constexpr (FWD) Vec8<float>::store(part + p.Fp + n, u);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
    }
}

// The parts of a contraction that was split, added up in a fixed order.
template <class E, int KIND> __global__ __launch_bounds__(256) void gdn_gated_join_kernel(GatedParams<E> p) {
    constexpr bool FWD = KIND == kGatedFwd || KIND == kGatedD;
    const int G = (FWD ? p.Fp : p.pitch) / 8;
    const long long unit = (long long)blockIdx.x * 256 + threadIdx.x;
    const int m = (int)min(unit / G, (long long)p.rows), n = (int)(unit % G) * 8;
    if (m >= p.rows) return;
    float v[8] = {}, u[8] = {};
    const size_t step = (size_t)p.rows * p.pitch;
    const float *at = p.part + (size_t)m * p.pitch + n;
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s) {
        const f32x4 a = *(const f32x4 *)(at + s * step), b = *(const f32x4 *)(at + s * step + 4);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] += a[q], v[4 + q] += b[q];
        if constexpr (FWD) {
            const f32x4 c = *(const f32x4 *)(at + p.Fp + s * step), d = *(const f32x4 *)(at + p.Fp + s * step + 4);
#pragma unroll
            for (int q = 0; q < 4; ++q) u[q] += c[q], u[4 + q] += d[q];
        }
    }
    Vec8<E> e{};
    if constexpr (KIND == kGatedD) e = gated_dh(p, m, n);
    gated_result<E, KIND>(p, m, n, v, u, e);
}

// x, Wg and Wu copied to rows of a multiple of 64 elements, zeros behind them: operands whose rows do not start
// at 16 bytes.
template <class E> struct PackParams {
    const E *src[3];
    E *dst;
    int M, F, C, ld;
};
template <class E> __global__ __launch_bounds__(256) void gdn_gated_pack_kernel(PackParams<E> p) {
    const int G = p.ld / 8;
    const long long unit = (long long)blockIdx.x * 256 + threadIdx.x, r = unit / G;
    const int c = (int)(unit % G) * 8;
    if (r >= p.M + 2LL * p.F) return;
    const E *row = r < p.M ? p.src[0] + r * p.C : r < p.M + (long long)p.F ? p.src[1] + (r - p.M) * p.C : p.src[2] + (r - p.M - p.F) * p.C;
    Vec8<E> v{};
    if (c + 8 <= p.C) v.load(row + c);
    else if (c < p.C) v.load_some(row + c, p.C - c);
    float f[8];
    v.values(f);
    Vec8<E>::store(p.dst + r * p.ld + c, f);
}

}  // namespace gdn
