// The norm over all elements of many tensors, and their scaling by min(1, max_norm / (norm + eps))
// (gdn_grad_* in gdn_block.h).
//
// Bound by memory: one pass to read, one to read and write.  The tensors' addresses and sizes go along in the
// launch itself, kClipTensors at a time, so nothing has to be copied to the device first.  A workgroup takes
// chunks of kClipChunk elements, wherever tensors begin and end; squares are exact in fp64 and summed there, so
// no value a tensor may hold overflows, and partial sums are added in a fixed order.  268 M elements in 40 bf16 tensors:
// squares 125 us (4.3 TB/s), scaling into others 183 (5.9); in one tensor 95 for the norm (5.7 TB/s).
#pragma once

#include "gdn_norm.h"

namespace gdn {

constexpr int kClipTensors = 128;     // of one launch: 3.7 KB of its arguments
constexpr int kClipChunk = 16384;     // elements of a workgroup's turn
constexpr int kClipThreads = 256;
constexpr int kClipGroups = 2048;     // workgroups of one launch at most

struct ClipTable {
    const void *in[kClipTensors];
    void *out[kClipTensors];
    long long end[kClipTensors];      // chunks up to this tensor's last, doubled, plus 1 where it holds bf16
    unsigned tail[kClipTensors];      // elements of its last chunk
    double *part;                     // sums of squares of this launch's workgroups (norm)
    const double *parts;              // all launches' sums (scale: NULL where the norm is given)
    const float *norm_in;
    float *norm_out;
    int count, groups, all_parts;
    float max_norm, eps;
};

// The tensor that chunk c is in, its first element there and the elements of the chunk.
struct ClipPiece {
    int i, n;
    long long first;
    bool bf16;
};
__device__ __forceinline__ ClipPiece clip_piece(const ClipTable &t, long long c) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if ((t.end[mid] >> 1) > c) hi = mid;
        else lo = mid + 1;
    }
    const long long begin = lo ? t.end[lo - 1] >> 1 : 0, last = (t.end[lo] >> 1) - 1;
    return {lo, c == last ? (int)t.tail[lo] : kClipChunk, (c - begin) * kClipChunk, (t.end[lo] & 1) != 0};
}

__device__ __forceinline__ double block_sum(double v, double *buf) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < kClipThreads / 64; ++i) v += buf[i];
    __syncthreads();
    return v;
}

template <class E> __device__ __forceinline__ double clip_squares(const E *x, int n) {
    double a = 0.0;
    auto add = [&](const Vec8<E> &v) {
        float f[8];
        v.values(f);
#pragma unroll
        for (int i = 0; i < 8; ++i) a = fma((double)f[i], (double)f[i], a);
    };
    constexpr int ROW = 8 * kClipThreads;
    int at = 8 * threadIdx.x;
    for (; at + 3 * ROW + 8 <= n; at += 4 * ROW) {
        Vec8<E> v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j].load(x + at + j * ROW);
#pragma unroll
        for (int j = 0; j < 4; ++j) add(v[j]);
    }
    for (; at < n; at += ROW) {
        Vec8<E> v;
        if (at + 8 <= n) v.load(x + at);
        else v.load_some(x + at, n - at);
        add(v);
    }
    return a;
}

template <class E> __device__ __forceinline__ void clip_scale(const E *x, E *y, int n, float scale) {
    constexpr int ROW = 8 * kClipThreads;
    auto put = [&](E *o, const Vec8<E> &v) {
        float f[8];
        v.values(f);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= scale;
        Vec8<E>::store(o, f);
    };
    int at = 8 * threadIdx.x;
    for (; at + 3 * ROW + 8 <= n; at += 4 * ROW) {
        Vec8<E> v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j].load(x + at + j * ROW);
#pragma unroll
        for (int j = 0; j < 4; ++j) put(y + at + j * ROW, v[j]);
    }
    for (; at < n; at += ROW) {
        Vec8<E> v;
        if (at + 8 <= n) {
            v.load(x + at);
            put(y + at, v);
        } else {
            float f[8];
            v.load_some(x + at, n - at);
            v.values(f);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (at + i < n) y[at + i] = Vec8<E>::cvt(f[i] * scale);
        }
    }
}

__global__ __launch_bounds__(kClipThreads) void gdn_grad_squares_kernel(ClipTable t) {
    __shared__ double buf[kClipThreads / 64];
    const long long chunks = t.end[t.count - 1] >> 1;
    double a = 0.0;
    for (long long c = blockIdx.x; c < chunks; c += t.groups) {
        const ClipPiece p = clip_piece(t, c);
        a += p.bf16 ? clip_squares((const uint16_t *)t.in[p.i] + p.first, p.n) : clip_squares((const float *)t.in[p.i] + p.first, p.n);
    }
    a = block_sum(a, buf);
    if (threadIdx.x == 0) t.part[blockIdx.x] = a;
}

__device__ __forceinline__ float clip_norm(const ClipTable &t, double *buf) {
    if (!t.parts) return *t.norm_in;
    double a = 0.0;
    for (int i = threadIdx.x; i < t.all_parts; i += kClipThreads) a += t.parts[i];
    return (float)sqrt(block_sum(a, buf));
}

// The norm alone, one workgroup.
__global__ __launch_bounds__(kClipThreads) void gdn_grad_norm_kernel(ClipTable t) {
    __shared__ double buf[kClipThreads / 64];
    const float norm = clip_norm(t, buf);
    if (threadIdx.x == 0) *t.norm_out = norm;
}

// Every workgroup adds up the sums for itself; the first one also writes the norm.
__global__ __launch_bounds__(kClipThreads) void gdn_grad_scale_kernel(ClipTable t) {
    __shared__ double buf[kClipThreads / 64];
    const float norm = clip_norm(t, buf);
    if (t.norm_out && blockIdx.x == 0 && threadIdx.x == 0) *t.norm_out = norm;
    // (a norm of NaN makes a NaN of it; zeros, and what no bound is set for, stay as they are: not 0 / 0, inf / inf)
    const double want = (double)t.max_norm / ((double)norm + (double)t.eps);
    const bool whole = want >= 1.0 || norm == 0.f || (t.max_norm == __builtin_inff() && norm == norm);
    const float scale = whole ? 1.f : (float)want;
    const long long chunks = t.count ? t.end[t.count - 1] >> 1 : 0;
    // (from the end: what was read last for the norm may still be in the caches)
    for (long long c = chunks - 1 - blockIdx.x; c >= 0; c -= t.groups) {
        const ClipPiece p = clip_piece(t, c);
        const void *x = t.in[p.i];
        void *y = t.out[p.i];
        if (scale == 1.f && x == y) continue;
        if (p.bf16) clip_scale((const uint16_t *)x + p.first, (uint16_t *)y + p.first, p.n, scale);
        else clip_scale((const float *)x + p.first, (float *)y + p.first, p.n, scale);
    }
}

}  // namespace gdn
