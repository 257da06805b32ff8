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
// read and written once; the means are wave reductions joined
// through LDS.  A team's rows are consecutive (a strip): the weights stay in
// registers, the gate row is read again only where it changes, and the sums
// over rows are kept in registers until the strip ends.
#pragma once

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

// Vectors of 8 elements at any element alignment (a row of odd length starts
// at any element): one access per 16 bytes either way.
template <class E> struct Vec8;
template <> struct Vec8<uint16_t> {
    typedef u32x4 raw __attribute__((aligned(2)));
    static __device__ __forceinline__ void load(const uint16_t *p, float *x) {
        const u32x4 v = *(const raw *)p;
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
        *(raw *)p = v;
    }
    static __device__ __forceinline__ float one(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
    static __device__ __forceinline__ uint16_t cvt(float v) { return (uint16_t)pack_bf16x2(v, 0.f); }
};
template <> struct Vec8<float> {
    typedef f32x4 raw __attribute__((aligned(4)));
    static __device__ __forceinline__ void load(const float *p, float *x) {
        const f32x4 a = *(const raw *)p, b = *(const raw *)(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
    }
    static __device__ __forceinline__ void store(float *p, const float *x) {
        *(raw *)p = f32x4{x[0], x[1], x[2], x[3]};
        *(raw *)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
    }
    static __device__ __forceinline__ float one(float v) { return v; }
    static __device__ __forceinline__ float cvt(float v) { return v; }
};

// 8 channels from c of a row of C; channels past the row's end read as 0 and
// are not written.
template <class E> __device__ __forceinline__ void load_row(const E *row, int c, int C, float *x) {
    if (c + 8 <= C) {
        Vec8<E>::load(row + c, x);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = c + i < C ? Vec8<E>::one(row[c + i]) : 0.f;
    }
}
template <class E> __device__ __forceinline__ void store_row(E *row, int c, int C, const float *x) {
    if (c + 8 <= C) {
        Vec8<E>::store(row + c, x);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < C) row[c + i] = Vec8<E>::cvt(x[i]);
    }
}

// Sums of NS values over the TPR threads of a team, in every thread.  `buf`: two
// halves used in turn (`turn`), so one barrier a sum is enough.
template <int NS, int TPR>
__device__ __forceinline__ void team_sum(float *v, float *buf, int &turn) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
#pragma unroll
        for (int s = 0; s < NS; ++s) v[s] += __shfl_xor(v[s], d);
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

template <class E, int TPR>
__global__ __launch_bounds__(norm_threads<TPR>()) void gdn_block_norm_kernel(NormParams<E> p) {
    constexpr int TEAMS = norm_threads<TPR>() / TPR;
    __shared__ float buf[64];
    int turn = 0;
    const int team = threadIdx.x / TPR, c = threadIdx.x % TPR * 8;
    const int strip = blockIdx.x * TEAMS + team;
    const long long r0 = (long long)strip * p.strip_rows; // forward strips are plain runs of rows
    const int C = p.C;
    const float rc = 1.f / (float)C;
    float wa[8], wb[8], ga[8];
    load_row<float>(p.w_post, c, C, wa);
    load_row<float>(p.w_pre, c, C, wb);
#pragma unroll
    for (int i = 0; i < 8; ++i) ga[i] = 1.f;
    int grow = -1;
    // every team of a workgroup makes the same number of turns (barriers)
    for (int i0 = 0; i0 < p.strip_rows; ++i0) {
        const long long row = r0 + i0;
        const bool on = row < p.R;
        const size_t base = (size_t)(on ? row : 0) * C;
        float x[8], y[8];
        float s[1] = {0.f};
        load_row<E>(p.y + base, c, C, y);
        load_row<E>(p.x + base, c, C, x);
        if (p.gate) {
            const int gr = (int)((on ? row : 0) / p.gate_tokens);
            if (gr != grow) {
                grow = gr;
                load_row<E>(p.gate + (size_t)gr * C, c, C, ga);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] += y[i] * y[i];
        team_sum<1, TPR>(s, buf, turn);
        const float iy = 1.f / sqrtf(s[0] * rc + p.eps);
        s[0] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = p.res_scale * x[i] + ga[i] * (y[i] * iy * wa[i]);
            // channels past the row's end stay out of the sum whatever res_scale and iy are
            if (c + i < C) s[0] += x[i] * x[i];
        }
        team_sum<1, TPR>(s, buf, turn);
        const float ir = 1.f / sqrtf(s[0] * rc + p.eps);
        if (!on) continue;
        store_row<E>(p.r + base, c, C, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= ir * wb[i];
        store_row<E>(p.u + base, c, C, x);
    }
}

template <class E, int TPR>
__global__ __launch_bounds__(norm_threads<TPR>()) void gdn_block_norm_grad_kernel(NormParams<E> p) {
    constexpr int TEAMS = norm_threads<TPR>() / TPR;
    __shared__ float buf[64];
    int turn = 0;
    const int team = threadIdx.x / TPR, c = threadIdx.x % TPR * 8;
    const int strip = blockIdx.x * TEAMS + team;
    const int C = p.C;
    const float rc = 1.f / (float)C;
    int rows = 0, r0 = 0;
    if (strip < p.strips) r0 = strip_begin(p, strip, rows);
    float wa[8], wb[8], ga[8], sa[8], sb[8], sg[8];
    load_row<float>(p.w_post, c, C, wa);
    load_row<float>(p.w_pre, c, C, wb);
#pragma unroll
    for (int i = 0; i < 8; ++i) ga[i] = 1.f, sa[i] = sb[i] = sg[i] = 0.f;
    int left = 0;                                         // rows until the gate row changes
    for (int i0 = 0; i0 < p.strip_rows; ++i0) {
        const bool on = i0 < rows;
        const int row = on ? r0 + i0 : 0;
        const size_t base = (size_t)row * C;
        float x[8], y[8], d[8], e[8];
        load_row<E>(p.y + base, c, C, y);
        load_row<E>(p.x + base, c, C, x);
        load_row<E>(p.du + base, c, C, d);
        if (p.dr) {
            load_row<E>(p.dr + base, c, C, e);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = 0.f;
        }
        if (p.gate && on && left == 0) {
            const int gr = row / p.gate_tokens;
            left = p.gate_tokens - (row - gr * p.gate_tokens);
            load_row<E>(p.gate + (size_t)gr * C, c, C, ga);
#pragma unroll
            for (int i = 0; i < 8; ++i) sg[i] = 0.f;
        }
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] += y[i] * y[i];
        team_sum<1, TPR>(s, buf, turn);
        const float iy = 1.f / sqrtf(s[0] * rc + p.eps);
        s[0] = s[1] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[i] *= iy;                                            // yh
            x[i] = p.res_scale * x[i] + ga[i] * (y[i] * wa[i]);    // r
            if (c + i < C) {
                s[0] += x[i] * x[i];
                s[1] += x[i] * (d[i] * wb[i]);
            }
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
            if (c + i < C) s[0] += d[i] * y[i];
        }
        team_sum<1, TPR>(s, buf, turn);
        const float m2 = s[0] * rc;
        if (!on) continue;
        store_row<E>(p.dx + base, c, C, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = iy * (d[i] - y[i] * m2);
        store_row<E>(p.dy + base, c, C, d);
        if (p.gate && --left == 0 && p.per_unit == 1) {
            store_row<E>(p.dgate + (size_t)(row / p.gate_tokens) * C, c, C, sg);
        }
    }
    if (strip < p.strips) {
        store_row<float>(p.part_w + (size_t)strip * 2 * C, c, C, sa);
        store_row<float>(p.part_w + (size_t)strip * 2 * C + C, c, C, sb);
        if (p.gate && p.per_unit > 1) store_row<float>(p.part_g + (size_t)strip * C, c, C, sg);
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
