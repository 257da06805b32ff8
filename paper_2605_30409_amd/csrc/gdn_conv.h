// The short causal convolution in front of the recurrence (gdn_short_conv_* in gdn_block.h), with the W - 1
// inputs before the first token as state: xe = [state; x],
//   z_t = bias + sum_i w_i xe_{t+i},   y_t = act(z_t),   state_out = xe[T .. T+W-2]
// and its gradient,
//   dz_t = dy_t act'(z_t),   dxe_p = sum_i w_i dz_{p-i} (+ dstate_out),   dw_i = sum_t dz_t xe_{t+i},
//   dbias = sum_t dz_t.
//
// Both are bound by memory.  A thread has 8 (gradient: 4) consecutive channels of a strip of consecutive tokens, so a wave
// reads a row's whole lines, every input is read once (W - 1 rows of the neighbouring strip again) and
// the window stays in registers.  10560 tokens of 2048 channels, bf16: 19.4 us (86 MB at 4.5 TB/s), gradient 33 and 4 for its
// sums (130 MB at 3.6; the vector units are busy 53 % of the time); of 6144
// channels 46.5 (5.6 TB/s) and 84 (4.6).  A step of one token: 4.4 us, a launch and two round trips.
#pragma once

#include "gdn_act.h"
#include "gdn_norm.h"

namespace gdn {

template <class E> struct ConvParams {
    const E *x, *state, *dy, *dstate_out;
    const float *w, *bias;
    E *y, *state_out, *dx, *dstate;
    const int *slots, *lengths;      // step
    float *part;                     // [blocks][W + 1][C]: sums for dw and dbias
    float *dw, *dbias;
    long long xb, xt, ob, ot;        // elements from batch to batch and from token to token: x; y, or dx
    long long yb, yt;                // dy
    int B, T, C, P;                  // step: B rows of up to T tokens, P slots
    int strip, strips;               // tokens of a strip, strips of a sequence
    int act;
};

// The n <= 8 channels of a thread from c on.  Nothing is shared with another thread, so that states may be
// updated in place; a row's last thread goes element by element.
struct Chan {
    int c, n;
    template <class E> __device__ __forceinline__ Vec8<E> fetch(const E *row) const {
        Vec8<E> v;
        if (n == 8) v.load(row + c);
        else v.load_some(row + c, n);
        return v;
    }
    template <class E> __device__ __forceinline__ void load(const E *row, float *x) const { fetch(row).values(x); }
    template <class E> __device__ __forceinline__ void store(E *row, const float *x) const {
        if (n == 8) {
            Vec8<E>::store(row + c, x);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) row[c + i] = Vec8<E>::cvt(x[i]);
        }
    }
};

template <int W> __device__ __forceinline__ void conv_weights(const float *w, const float *bias, const Chan &ch,
                                                              float (&wt)[W][8], float (&b)[8]) {
    if (ch.n == 8) {
        float v[8 * W];
#pragma unroll
        for (int i = 0; i < 2 * W; ++i) {
            const f32x4 q = *(const f32x4 *)(w + (size_t)ch.c * W + 4 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * i + e] = q[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int i = 0; i < W; ++i) wt[i][e] = v[e * W + i];
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        const f32x4 b0 = bias ? *(const f32x4 *)(bias + ch.c) : zero, b1 = bias ? *(const f32x4 *)(bias + ch.c + 4) : zero;
#pragma unroll
        for (int e = 0; e < 4; ++e) b[e] = b0[e], b[4 + e] = b1[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = ch.c + min(e, ch.n - 1);
#pragma unroll
            for (int i = 0; i < W; ++i) wt[i][e] = w[(size_t)c * W + i];
            b[e] = bias ? bias[c] : 0.f;
        }
    }
}

// Row p of xe: state before x; zero without a state and past the end.
template <class E, int W>
__device__ __forceinline__ Vec8<E> conv_row(const ConvParams<E> &p, const Chan &ch, int b, int at) {
    if (at >= W - 1) return ch.fetch(p.x + b * p.xb + (long long)(at - (W - 1)) * p.xt);
    if (p.state) return ch.fetch(p.state + ((size_t)b * (W - 1) + at) * p.C);
    return Vec8<E>{};
}

template <class E, int W> __global__ __launch_bounds__(256) void gdn_short_conv_kernel(ConvParams<E> p) {
    const int G = (p.C + 7) / 8;
    const long long unit = (long long)blockIdx.x * 256 + threadIdx.x;
    const int g = (int)(unit % G);
    const long long rest = unit / G;
    const int s = (int)(rest % p.strips);
    const long long bl = rest / p.strips;
    if (bl >= p.B) return;
    const int b = (int)bl;
    const Chan ch{8 * g, min(8, p.C - 8 * g)};
    const int t0 = s * p.strip, t1 = min(t0 + p.strip, p.T);
    float wt[W][8], bias[8], win[W][8];
#pragma unroll
    for (int i = 1; i < W; ++i) conv_row<E, W>(p, ch, b, t0 + i - 1).values(win[i]);
    constexpr int AHEAD = 4;                       // rows asked for at once
    Vec8<E> nx[AHEAD];
    auto ask = [&](int t) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) nx[j] = ch.fetch(p.x + b * p.xb + (long long)min(t + j, p.T - 1) * p.xt);
    };
    ask(t0);
    conv_weights<W>(p.w, p.bias, ch, wt, bias);
    if (s == 0 && p.state_out) {
        // (by the threads that read the state, so that it may be the same buffer: all rows before the first store)
        Vec8<E> last[W - 1];
#pragma unroll
        for (int i = 0; i < W - 1; ++i) last[i] = conv_row<E, W>(p, ch, b, p.T + i);
#pragma unroll
        for (int i = 0; i < W - 1; ++i) {
            float v[8];
            last[i].values(v);
            ch.store(p.state_out + ((size_t)b * (W - 1) + i) * p.C, v);
        }
    }
    for (int t = t0; t < t1; t += AHEAD) {
        Vec8<E> cur[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) cur[j] = nx[j];
        if (t + AHEAD < t1) ask(t + AHEAD);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            float z[8];
#pragma unroll
            for (int i = 0; i + 1 < W; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) win[i][e] = win[i + 1][e];
            cur[j].values(win[W - 1]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                z[e] = bias[e];
#pragma unroll
                for (int i = 0; i < W; ++i) z[e] += wt[i][e] * win[i][e];
            }
            act_all<8>(z, p.act);
            if (t + j < t1) ch.store(p.y + b * p.ob + (long long)(t + j) * p.ot, z);
        }
    }
}

// 4 consecutive elements at any element alignment.
template <class E> struct Vec4;
template <> struct Vec4<uint16_t> {
    typedef u32x2 loose __attribute__((aligned(2)));
    u32x2 v;
    __device__ __forceinline__ void load(const uint16_t *p) { v = *(const loose *)p; }
    __device__ __forceinline__ void load_some(const uint16_t *p, int n) {
        v = u32x2{p[0] | (n > 1 ? (uint32_t)p[1] << 16 : 0u), n > 2 ? (uint32_t)p[2] : 0u};
    }
    __device__ __forceinline__ void values(float *x) const {
        const f32x4 f = Tr<uint16_t>::to_f32(v);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = f[i];
    }
    static __device__ __forceinline__ void store(uint16_t *p, const float *x) {
        *(loose *)p = Tr<uint16_t>::from_f32(f32x4{x[0], x[1], x[2], x[3]});
    }
};
template <> struct Vec4<float> {
    typedef f32x4 loose __attribute__((aligned(4)));
    f32x4 v;
    __device__ __forceinline__ void load(const float *p) { v = *(const loose *)p; }
    __device__ __forceinline__ void load_some(const float *p, int n) { v = f32x4{p[0], n > 1 ? p[1] : 0.f, n > 2 ? p[2] : 0.f, 0.f}; }
    __device__ __forceinline__ void values(float *x) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = v[i];
    }
    static __device__ __forceinline__ void store(float *p, const float *x) { *(loose *)p = f32x4{x[0], x[1], x[2], x[3]}; }
};

// The gradient.  A thread has 4 channels (8 leave registers for two waves a SIMD only) and forms dz for its strip and the
// W - 1 tokens behind it; with the last W of them it has dxe of its own tokens (the first strip: of the state too).  A
// row's last thread takes its last 4 channels, what another has too among them: those are written twice, with the
// same bits, and left out of the sums.  The sums of a strip go through LDS to those of the workgroup (TY strips of one
// sequence) and from there to the second launch, in a fixed order.  ACT: the activation, or -1: p.act, rows of fewer than
// 4 channels.
constexpr int kConvGradThreads = 256;

template <class E, int W, int ACT> __global__ __launch_bounds__(kConvGradThreads) void gdn_short_conv_grad_kernel(ConvParams<E> p, int TX) {
    constexpr bool SHORT = ACT < 0;
    __shared__ float sm[2][kConvGradThreads][5];
    const int G = (p.C + 3) / 4, TY = kConvGradThreads / TX;
    const int tx = threadIdx.x % TX, ty = threadIdx.x / TX;
    const int gx = (G + TX - 1) / TX;
    const int bx = blockIdx.x % gx, by = blockIdx.x / gx;
    const int g = bx * TX + tx;
    const int blocks = (p.strips + TY - 1) / TY;               // of a sequence
    const int b = by / blocks, s = (by % blocks) * TY + ty;
    float sw[W][4], sb[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        sb[e] = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) sw[i][e] = 0.f;
    }
    if (g < G && s < p.strips) {
        const int c0 = SHORT ? 0 : min(4 * g, p.C - 4);
        auto fetch = [&](const E *row) {
            Vec4<E> v;
            if constexpr (SHORT) v.load_some(row, p.C);
            else v.load(row + c0);
            return v;
        };
        auto store = [&](E *row, const float *x) {
            if constexpr (SHORT) {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < p.C) row[e] = Vec8<E>::cvt(x[e]);
            } else {
                Vec4<E>::store(row + c0, x);
            }
        };
        const int t0 = s * p.strip, t1 = min(t0 + p.strip, p.T);
        float wt[W][4], bias[4], win[W][4], dz[W][4];
        constexpr int AHEAD = 4;
        Vec4<E> nx[AHEAD], nd[AHEAD];
        const E *x = p.x + b * p.xb, *dy = p.dy + b * p.yb;
        E *dx = p.dx + b * p.ob - (W - 1) * p.ot;
        auto ask = [&](int t) {
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int r = min(t + j, p.T - 1);
                nx[j] = fetch(x + (long long)r * p.xt);
                nd[j] = fetch(dy + (long long)r * p.yt);
            }
        };
        ask(t0);
#pragma unroll
        for (int i = 0; i < W; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) dz[i][e] = 0.f;
#pragma unroll
        for (int i = 1; i < W; ++i) {
            const int at = t0 + i - 1;
            Vec4<E> v{};
            if (at >= W - 1) v = fetch(x + (long long)(at - (W - 1)) * p.xt);
            else if (p.state) v = fetch(p.state + ((size_t)b * (W - 1) + at) * p.C);
            v.values(win[i]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = SHORT ? min(e, p.C - 1) : c0 + e;
#pragma unroll
            for (int i = 0; i < W; ++i) wt[i][e] = p.w[(size_t)c * W + i];
            bias[e] = p.bias ? p.bias[c] : 0.f;
        }
        // the next token: its inputs into the window, its dz (zero behind the end) in front of the others, and dxe_tt
        auto shift = [&] {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
#pragma unroll
                for (int i = 0; i + 1 < W; ++i) win[i][e] = win[i + 1][e];
#pragma unroll
                for (int i = W - 1; i > 0; --i) dz[i][e] = dz[i - 1][e];
            }
        };
        auto token = [&](const Vec4<E> &vx, const Vec4<E> &vd) {
            float z[4], d[4];
            vx.values(win[W - 1]);
            vd.values(d);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                z[e] = bias[e];
#pragma unroll
                for (int i = 0; i < W; ++i) z[e] += wt[i][e] * win[i][e];
            }
            slope_all<4>(z, SHORT ? p.act : ACT);
#pragma unroll
            for (int e = 0; e < 4; ++e) dz[0][e] = d[e] * z[e];
        };
        auto result = [&](float *o) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                o[e] = 0.f;
#pragma unroll
                for (int i = 0; i < W; ++i) o[e] += wt[i][e] * dz[i][e];
            }
        };
        auto sums = [&] {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sb[e] += dz[0][e];
#pragma unroll
                for (int i = 0; i < W; ++i) sw[i][e] += dz[0][e] * win[i][e];
            }
        };
        // the strip's whole runs of AHEAD tokens; of the first run, some results belong elsewhere
        int t = t0;
        for (; t + AHEAD <= t1; t += AHEAD) {
            Vec4<E> cx[AHEAD], cd[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) cx[j] = nx[j], cd[j] = nd[j];
            ask(t + AHEAD);
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                float o[4];
                shift();
                token(cx[j], cd[j]);
                sums();
                result(o);
                if (j >= W - 1 || t > t0) store(dx + (long long)(t + j) * p.ot, o);
                else if (s == 0 && p.dstate) store(p.dstate + ((size_t)b * (W - 1) + t + j) * p.C, o);
            }
        }
        // what is left of it, and the tokens behind it
        const int end = t1 + W - 1;
        for (; t < end; ++t) {
            float o[4];
            shift();
            token(nx[0], nd[0]);
            const bool in = t < p.T;
#pragma unroll
            for (int e = 0; e < 4; ++e) dz[0][e] = in ? dz[0][e] : 0.f;
            if (t < t1) sums();
            result(o);
            if (!in && p.dstate_out) {
                float d[4];
                fetch(p.dstate_out + ((size_t)b * (W - 1) + t - p.T) * p.C).values(d);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] += d[e];
            }
            if (t >= t0 + W - 1) store(dx + (long long)t * p.ot, o);
            else if (s == 0 && p.dstate) store(p.dstate + ((size_t)b * (W - 1) + t) * p.C, o);
#pragma unroll
            for (int j = 0; j + 1 < AHEAD; ++j) nx[j] = nx[j + 1], nd[j] = nd[j + 1];
            if (t + AHEAD < end) {
                const int r = min(t + AHEAD, p.T - 1);
                nx[AHEAD - 1] = fetch(x + (long long)r * p.xt);
                nd[AHEAD - 1] = fetch(dy + (long long)r * p.yt);
            }
        }
    }
    // sums of the TY strips, one tap at a time, through two buffers in turn
    float *part = p.part + (size_t)by * (W + 1) * p.C;
#pragma unroll
    for (int i = 0; i <= W; ++i) {
        float (*buf)[5] = sm[i & 1];
#pragma unroll
        for (int e = 0; e < 4; ++e) buf[threadIdx.x][e] = i < W ? sw[i < W ? i : 0][e] : sb[e];
        lds_barrier();
        const int c = threadIdx.x, col = 4 * TX * bx + c;
        if (c < 4 * TX && col < p.C) {
            const int e = SHORT ? col : col - min(col / 4 * 4, p.C - 4);
            float a = 0.f;
            for (int y = 0; y < TY; ++y) a += buf[y * TX + c / 4][e];
            part[(size_t)i * p.C + col] = a;
        }
    }
}

// Sums of the workgroups' sums: 64 columns of [W + 1][C] a workgroup, 16 waves taking every 16th row.
constexpr int kConvReduceWaves = 16;

template <class E> __global__ __launch_bounds__(64 * kConvReduceWaves) void gdn_short_conv_reduce_kernel(ConvParams<E> p, int W, int rows) {
    __shared__ float sm[kConvReduceWaves][64];
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
    const long long width = (long long)(W + 1) * p.C, c = (long long)blockIdx.x * 64 + l;
    float a = 0.f;
    if (c < width)
#pragma unroll 4
        for (int s = w; s < rows; s += kConvReduceWaves) a += p.part[(size_t)s * width + c];
    sm[w][l] = a;
    lds_barrier();
    if (w != 0 || c >= width) return;
#pragma unroll
    for (int i = 1; i < kConvReduceWaves; ++i) a += sm[i][l];
    const int tap = (int)(c / p.C), ch = (int)(c % p.C);
    if (tap < W) p.dw[(size_t)ch * W + tap] = a;
    else if (p.dbias) p.dbias[ch] = a;
}

// One or a few tokens of many sequences, windows in a pool of slots.  A wave has 512 channels of one row.
template <class E, int W> __global__ __launch_bounds__(256) void gdn_short_conv_step_kernel(ConvParams<E> p) {
    const int G = (p.C + 7) / 8, WG = (G + 63) / 64;             // waves of a row
    const long long unit = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l = threadIdx.x & 63;
    const long long nl = unit / WG;
    if (nl >= p.B) return;
    const int n = (int)nl, g = (int)(unit % WG) * 64 + l;
    const int slot = p.slots ? p.slots[n] : n;
    if (slot < 0) return;
    int len = p.T;
    if (p.lengths) len = max(0, min(p.lengths[n], p.T));
    const Chan ch{8 * min(g, G - 1), min(8, p.C - 8 * min(g, G - 1))};
    bool bad = slot >= p.P;
    const size_t at = (size_t)slot * (W - 1) * p.C;
    const E *x = p.x + n * p.xb;
    float wt[W][8], bias[8], win[W][8];
    Vec8<E> nx = ch.fetch(x);
#pragma unroll
    for (int i = 1; i < W; ++i) {
        if (!bad) ch.load(p.state + at + (size_t)(i - 1) * p.C, win[i]);
    }
    conv_weights<W>(p.w, p.bias, ch, wt, bias);
    // a slot belongs to the first row that names it
    if (p.slots) {
        bool taken = false;
        for (int m = l; m < n; m += 64) taken |= p.slots[m] == slot;
        bad |= __any(taken);
    }
    if (g >= G) return;
    E *y = p.y + (size_t)n * p.T * p.C;
    if (bad) {
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = __builtin_nanf("");
        for (int t = 0; t < len; ++t) ch.store(y + (size_t)t * p.C, z);
        return;
    }
    for (int t = 0; t < len; ++t) {
        float z[8];
#pragma unroll
        for (int i = 0; i + 1 < W; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) win[i][e] = win[i + 1][e];
        nx.values(win[W - 1]);
        nx = ch.fetch(x + (long long)min(t + 1, p.T - 1) * p.xt);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            z[e] = bias[e];
#pragma unroll
            for (int i = 0; i < W; ++i) z[e] += wt[i][e] * win[i][e];
        }
        act_all<8>(z, p.act);
        ch.store(y + (size_t)t * p.C, z);
    }
#pragma unroll
    for (int i = 1; i < W; ++i) ch.store(p.state_out + at + (size_t)(i - 1) * p.C, win[i]);
}

}  // namespace gdn
