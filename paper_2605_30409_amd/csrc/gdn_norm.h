// The border between two blocks (gdn_block_norm_* in gdn_ops.h):
//   n = w_post o y iy,  iy = 1 / sqrt(mean y^2 + eps)
//   r = res_scale x + gate o n
//   u = w_pre o r ir,   ir = 1 / sqrt(mean r^2 + eps)
// and its gradient, with h = r ir, yh = y iy, d = w_pre o du:
//   g  = dr + ir (d - h mean(d o h))             dL/dr
//   dx = res_scale g,   dgate = sum_rows n o g
//   d2 = w_post o gate o g,   dy = iy (d2 - yh mean(d2 o yh))
//   dw_pre = sum_rows du o h,   dw_post = sum_rows gate o g o yh
//
// Both are bound by memory.  A team of TPR threads takes a row at a time and
// holds it in registers, 8 consecutive channels per thread, so every element is
// read and written once; the means are wave reductions joined through LDS, and the
// next row's loads are issued before this row's means are formed.  A team's
// rows are consecutive (a strip): the weights stay in registers, the gate row is
// read again only where it changes, and the sums over rows are kept in registers
// until the strip ends.  10560 rows of 2048 channels, bf16: forward 31 to 35 us (173 MB at 4.9 to
// 5.6 TB/s), gradient 54 to 57 us (272 MB at 4.7 to 5.0) and 5 us for its sums.
// Whole calls at other widths, TB/s of what must move (172 MB forward, 258 MB gradient in bf16, twice that
// in fp32):
//   channels             32     64    128    256    512   1024   4096   5120   8192
//   bf16 forward       0.78   1.47   2.72   4.75   5.18   4.85   4.95   3.42   3.82
//        gradient      0.51   0.97   1.77   3.07   3.80   4.11   4.10   2.23   2.58
//   fp32 forward       1.45   2.51   4.15   4.85   4.62   4.85   5.03   4.04   4.08
//        gradient      1.04   1.90   3.25   4.34   4.26   4.46   4.44   2.64   2.84
// Rows under 512 channels leave lanes of their wave without any (8 channels each).  Rows over 4096 take 1024
// threads: at 5120 channels 3 in 8 of them have none, and in the gradient 128 registers a thread are too
// few (16 spilled in bf16, 30 in fp32).
#pragma once

#include <type_traits>

#include "gdn_device.h"

namespace gdn {

template <class E> struct NormParams {
    const E *x, *y, *gate;
    const float *w_post, *w_pre;
    E *r, *u;               // forward
    const E *du, *dr;       // backward
    E *dx, *dy, *dgate;
    float *part_w;          // [strips][2][C]: sums for dw_post and dw_pre
    float *part_g;          // [strips][C]: sums for dgate, where a gate row spans strips
    float *dw_post, *dw_pre;
    int R, C, gate_tokens;
    int strips, strip_rows; // strips start at multiples of strip_rows inside a unit
    int per_unit;           // strips per gate row (> 1), or 1: strips hold whole gate rows
    int unit_rows;          // rows that per_unit strips cover
    float res_scale, eps;
};

// 8 consecutive elements at any element alignment (a row of odd length starts
// at any element): whole 16-byte accesses either way.
template <class E> struct Vec8;
template <> struct Vec8<uint16_t> {
    typedef u32x4 loose __attribute__((aligned(2)));
    u32x4 v;
    __device__ __forceinline__ void load(const uint16_t *p) { v = *(const loose *)p; }
    __device__ __forceinline__ void load_some(const uint16_t *p, int n) {
        uint16_t x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < n ? p[i] : 0;
        v = __builtin_bit_cast(u32x4, x);
    }
    __device__ __forceinline__ void values(float *x) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(v[i] << 16);
            x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ void store(uint16_t *p, const float *x) {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
        *(loose *)p = v;
    }
    static __device__ __forceinline__ uint16_t cvt(float v) { return (uint16_t)pack_bf16x2(v, 0.f); }
};
template <> struct Vec8<float> {
    typedef f32x4 loose __attribute__((aligned(4)));
    f32x4 a, b;
    __device__ __forceinline__ void load(const float *p) { a = *(const loose *)p, b = *(const loose *)(p + 4); }
    __device__ __forceinline__ void load_some(const float *p, int n) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < n ? p[i] : 0.f;
        a = f32x4{x[0], x[1], x[2], x[3]}, b = f32x4{x[4], x[5], x[6], x[7]};
    }
    __device__ __forceinline__ void values(float *x) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
    }
    static __device__ __forceinline__ void store(float *p, const float *x) {
        *(loose *)p = f32x4{x[0], x[1], x[2], x[3]};
        *(loose *)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
    }
    static __device__ __forceinline__ float cvt(float v) { return v; }
};

// The 8 channels of a thread.  Rows of 8 channels or more: the last ones of the row where
// its own would reach past the end, so that every access is a whole vector; what
// another thread has too is left out of the sums (`own`) and written twice, with
// the same bits.  Shorter rows (SHORT) are thread 0's, element by element.
template <bool SHORT> struct Channels {
    int c, n;           // first channel, elements (SHORT)
    bool own[8];
    __device__ __forceinline__ Channels(int t, int C) {
        const int c0 = 8 * t;
        c = SHORT ? 0 : min(c0, C - 8);
        n = SHORT && t == 0 ? C : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) own[i] = SHORT ? i < n : c + i >= c0;
    }
    template <class E> __device__ __forceinline__ Vec8<E> load(const E *row) const {
        Vec8<E> v;
        if constexpr (SHORT) v.load_some(row, n);
        else v.load(row + c);
        return v;
    }
    template <class E> __device__ __forceinline__ void load(const E *row, float *x) const { load(row).values(x); }
    template <class E> __device__ __forceinline__ void store(E *row, const float *x) const {
        if constexpr (SHORT) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) row[i] = Vec8<E>::cvt(x[i]);
        } else {
            Vec8<E>::store(row + c, x);
        }
    }
};

// Sum over the lanes of a wave, in every lane: 16 lanes by cross-lane adds, the four
// groups of 16 by reading a lane of each.
__device__ __forceinline__ float wave_sum(float v) {
    auto add = [&](auto sel) {
        v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), decltype(sel)::value, 0xf, 0xf, true));
    };
    add(std::integral_constant<int, 0xb1>{});      // lane ^ 1
    add(std::integral_constant<int, 0x4e>{});      // lane ^ 2
    add(std::integral_constant<int, 0x141>{});     // the other 4 of 8
    add(std::integral_constant<int, 0x140>{});     // the other 8 of 16
    auto lane = [&](int l) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l)); };
    return (lane(0) + lane(16)) + (lane(32) + lane(48));
}

// Sums of NS values over the TPR threads of a team, in every thread.  `buf`: two
// halves used in turn (`turn`), so one barrier a sum is enough.
template <int NS, int TPR>
__device__ __forceinline__ void team_sum(float *v, float *buf, int &turn) {
#pragma unroll
    for (int s = 0; s < NS; ++s) v[s] = wave_sum(v[s]);
    if constexpr (TPR > 64) {
        constexpr int NW = TPR / 64;
        float *b = buf + turn * 32;
        const int w = threadIdx.x >> 6, w0 = w / NW * NW;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int s = 0; s < NS; ++s) b[s * 16 + w] = v[s];
        lds_barrier();
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            float t = 0.f;
#pragma unroll
            for (int i = 0; i < NW; ++i) t += b[s * 16 + w0 + i];
            v[s] = t;
        }
        turn ^= 1;
    }
}

template <int TPR> constexpr int norm_threads() { return TPR > 256 ? TPR : 256; }

// Rows of strip s: first row and count (0: none).
template <class E> __device__ __forceinline__ int strip_begin(const NormParams<E> &p, int s, int &rows) {
    const int unit = s / p.per_unit, part = s - unit * p.per_unit;
    const long long r0 = (long long)unit * p.unit_rows + (long long)part * p.strip_rows;
    const long long end = min((long long)(unit + 1) * p.unit_rows, (long long)p.R);
    rows = (int)max(0LL, min((long long)p.strip_rows, end - r0));
    return (int)r0;
}

template <class E, int TPR, bool SHORT>
__global__ __launch_bounds__(norm_threads<TPR>()) void gdn_block_norm_kernel(NormParams<E> p) {
    constexpr int TEAMS = norm_threads<TPR>() / TPR;
    __shared__ float buf[64];
    int turn = 0;
    const Channels<SHORT> ch(threadIdx.x % TPR, p.C);
    const long long r0 = ((long long)blockIdx.x * TEAMS + threadIdx.x / TPR) * p.strip_rows;
    const float rc = 1.f / (float)p.C;
    float wa[8], wb[8], ga[8];
    ch.load(p.w_post, wa);
    ch.load(p.w_pre, wb);
#pragma unroll
    for (int i = 0; i < 8; ++i) ga[i] = 1.f;
    int grow = -1;
    // rows past the end (of the last teams) read the last row again and write nothing
    auto at = [&](int i) { return (size_t)min(r0 + min(i, p.strip_rows - 1), (long long)p.R - 1) * p.C; };
    Vec8<E> yn = ch.load(p.y + at(0)), xn = ch.load(p.x + at(0));
    // every team of a workgroup makes the same number of turns (barriers)
    for (int i0 = 0; i0 < p.strip_rows; ++i0) {
        const bool on = r0 + i0 < p.R;
        const size_t base = at(i0);
        float x[8], y[8], s[1] = {0.f};
        yn.values(y);
        xn.values(x);
        if (p.gate) {
            const int gr = (int)(min(r0 + i0, (long long)p.R - 1) / p.gate_tokens);
            if (gr != grow) {
                grow = gr;
                ch.load(p.gate + (size_t)gr * p.C, ga);
            }
        }
        yn = ch.load(p.y + at(i0 + 1));
        xn = ch.load(p.x + at(i0 + 1));
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] += ch.own[i] ? y[i] * y[i] : 0.f;
        team_sum<1, TPR>(s, buf, turn);
        const float iy = 1.f / sqrtf(s[0] * rc + p.eps);
        s[0] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = p.res_scale * x[i] + ga[i] * (y[i] * iy * wa[i]);
            s[0] += ch.own[i] ? x[i] * x[i] : 0.f;
        }
        team_sum<1, TPR>(s, buf, turn);
        const float ir = 1.f / sqrtf(s[0] * rc + p.eps);
        if (!on) continue;
        ch.store(p.r + base, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= ir * wb[i];
        ch.store(p.u + base, x);
    }
}

template <class E, int TPR, bool SHORT>
__global__ __launch_bounds__(norm_threads<TPR>()) void gdn_block_norm_grad_kernel(NormParams<E> p) {
    constexpr int TEAMS = norm_threads<TPR>() / TPR;
    __shared__ float buf[64];
    int turn = 0;
    const Channels<SHORT> ch(threadIdx.x % TPR, p.C);
    const int strip = blockIdx.x * TEAMS + threadIdx.x / TPR;
    const int C = p.C;
    const float rc = 1.f / (float)C;
    int rows = 0, r0 = 0;
    if (strip < p.strips) r0 = strip_begin(p, strip, rows);
    float wa[8], wb[8], ga[8], sa[8], sb[8], sg[8];
    ch.load(p.w_post, wa);
    ch.load(p.w_pre, wb);
#pragma unroll
    for (int i = 0; i < 8; ++i) ga[i] = 1.f, sa[i] = sb[i] = sg[i] = 0.f;
    int left = 0;                                         // rows until the gate row changes
    // turns past the strip's last row read it again and write nothing
    auto at = [&](int i) { return (size_t)(r0 + min(i, max(rows - 1, 0))) * C; };
    Vec8<E> xn, yn, dn, en{};
    auto fetch = [&](int i) {
        const size_t base = at(i);
        yn = ch.load(p.y + base);
        xn = ch.load(p.x + base);
        dn = ch.load(p.du + base);
        if (p.dr) en = ch.load(p.dr + base);
    };
    // (1024 threads have no registers for a row ahead)
    constexpr bool AHEAD = TPR < 1024;
    if (AHEAD) fetch(0);
    for (int i0 = 0; i0 < p.strip_rows; ++i0) {
        const bool on = i0 < rows;
        const int row = r0 + i0;
        const size_t base = at(i0);
        float x[8], y[8], d[8], e[8];
        if (!AHEAD) fetch(i0);
        yn.values(y);
        xn.values(x);
        dn.values(d);
        en.values(e);
        if (p.gate && on && left == 0) {
            const int gr = row / p.gate_tokens;
            left = p.gate_tokens - (row - gr * p.gate_tokens);
            ch.load(p.gate + (size_t)gr * C, ga);
#pragma unroll
            for (int i = 0; i < 8; ++i) sg[i] = 0.f;
        }
        if (AHEAD) fetch(i0 + 1);
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] += ch.own[i] ? y[i] * y[i] : 0.f;
        team_sum<1, TPR>(s, buf, turn);
        const float iy = 1.f / sqrtf(s[0] * rc + p.eps);
        s[0] = s[1] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[i] *= iy;                                            // yh
            x[i] = p.res_scale * x[i] + ga[i] * (y[i] * wa[i]);    // r
            s[0] += ch.own[i] ? x[i] * x[i] : 0.f;
            s[1] += ch.own[i] ? x[i] * (d[i] * wb[i]) : 0.f;
        }
        team_sum<2, TPR>(s, buf, turn);
        const float ir = 1.f / sqrtf(s[0] * rc + p.eps);
        const float m1 = s[1] * rc * ir;                           // mean(d o h)
        s[0] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float hh = x[i] * ir;
            const float g = e[i] + ir * (d[i] * wb[i] - hh * m1);
            x[i] = p.res_scale * g;
            const float gg = ga[i] * g;
            if (on) {
                sb[i] += d[i] * hh;
                sa[i] += gg * y[i];
                sg[i] += y[i] * wa[i] * g;
            }
            d[i] = gg * wa[i];                                     // d2
            s[0] += ch.own[i] ? d[i] * y[i] : 0.f;
        }
        team_sum<1, TPR>(s, buf, turn);
        const float m2 = s[0] * rc;
        if (!on) continue;
        ch.store(p.dx + base, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = iy * (d[i] - y[i] * m2);
        ch.store(p.dy + base, d);
        if (p.gate && --left == 0 && p.per_unit == 1) ch.store(p.dgate + (size_t)(row / p.gate_tokens) * C, sg);
    }
    if (strip < p.strips) {
        ch.store(p.part_w + (size_t)strip * 2 * C, sa);
        ch.store(p.part_w + (size_t)strip * 2 * C + C, sb);
        if (p.gate && p.per_unit > 1) ch.store(p.part_g + (size_t)strip * C, sg);
    }
}

// Sums of the strips' partial sums, in a fixed order.  Workgroup (x, 0): 64
// channels of [dw_post | dw_pre]; (x, 1 + g): 64 channels of gate row g.  16
// waves take every 16th strip each, joined through LDS.
constexpr int kNormReduceWaves = 16;

template <class E>
__global__ __launch_bounds__(64 * kNormReduceWaves) void gdn_block_norm_reduce_kernel(NormParams<E> p) {
    __shared__ float sm[kNormReduceWaves][64];
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
    const bool weights = blockIdx.y == 0;
    const long long width = weights ? 2LL * p.C : p.C;
    const long long c = (long long)blockIdx.x * 64 + l;
    const int g = (int)blockIdx.y - 1;
    const int s0 = weights ? 0 : g * p.per_unit, n = weights ? p.strips : p.per_unit;
    const float *src = (weights ? p.part_w : p.part_g) + (size_t)s0 * width + c;
    float a = 0.f;
    if (c < width)
#pragma unroll 4
        for (int s = w; s < n; s += kNormReduceWaves) a += src[(size_t)s * width];
    sm[w][l] = a;
    lds_barrier();
    if (w != 0 || c >= width) return;
#pragma unroll
    for (int i = 1; i < kNormReduceWaves; ++i) a += sm[i][l];
    if (weights) {
        (c < p.C ? p.dw_post[c] : p.dw_pre[c - p.C]) = a;
    } else {
        p.dgate[(size_t)g * p.C + c] = Vec8<E>::cvt(a);
    }
}

}  // namespace gdn
