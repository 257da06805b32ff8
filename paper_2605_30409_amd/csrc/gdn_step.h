// The recurrent step of a decoding batch (gdn_step_forward in gdn_ops.h).
//
// Per row, head and token, with the state S [Dk][Dv] in fp32:
//   u = beta (v - alpha S^T k),   S <- alpha S + k u^T,
//   o = S^T q = alpha S_old^T q + (k . q) u,
// so S^T k, S^T q and k . q come from one pass over the state and the output
// does not wait for the update.
//
// One wave holds kStepCols columns of one state in registers: lane (rg, cl)
// has rows RPL rg .. RPL rg + RPL - 1 of four columns, a load instruction reads whole
// 128-byte lines, and the columns of a state are independent, so waves share
// nothing and there is no LDS and no barrier.  The state goes through once
// whatever the number of tokens.
//
// Bound by memory, the state read and written: 256 rows of 32 heads (Dk = Dv = 128) 208 us,
// 5.2 TB/s; a large plain copy reaches 4.7.  One row, one token: 4.8 us, a launch and one
// round trip to memory.
#pragma once

#include "gdn_device.h"

namespace gdn {

template <class E> struct StepParams {
    const E *q, *k, *v;
    const float *alpha, *beta, *state_in;
    const int *slots, *lengths;
    E *out;
    float *state_out;
    int N, L, P, Hk, H;
};

// State columns per wave: a row of 32 is a whole line of 128 bytes.  us with 16, 32, 64: one row of 16
// heads 4.4, 4.9, 6.4; 64 rows 59, 53, 57; 256 rows of 32 heads 247, 206, 205.
constexpr int kStepCols = 32;
constexpr int kStepWaves = 4;    // waves per workgroup

// n consecutive elements as fp32 (n a multiple of 4).
template <int n, class E> __device__ __forceinline__ void load_f32(const E *p, float *x) {
#pragma unroll
    for (int i = 0; i < n; i += 4) {
        const f32x4 y = Tr<E>::to_f32(Tr<E>::load(p + i));
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i + e] = y[e];
    }
}

template <class E, int DK, int DV>
__global__ __launch_bounds__(64 * kStepWaves) void gdn_step_kernel(StepParams<E> p) {
    constexpr int CL = kStepCols / 4;      // lanes across the columns
    constexpr int RPL = DK / (64 / CL);    // rows per lane
    constexpr int NT = DV / kStepCols;     // waves per state
    const long long unit = (long long)blockIdx.x * kStepWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l = threadIdx.x & 63, cl = l % CL, rg = l / CL;
    const int tile = (int)(unit % NT);
    const long long nh = unit / NT;
    const int h = (int)(nh % p.H);
    const int n = (int)(nh / p.H);
    if (n >= p.N) return;
    const int slot = p.slots ? p.slots[n] : n;
    if (slot < 0) return;
    int len = p.L;
    if (p.lengths) len = max(0, min(p.lengths[n], p.L));
    const int col = kStepCols * tile + 4 * cl;
    E *out = p.out + ((size_t)n * p.L * p.H + h) * DV + col;
    const size_t ostep = (size_t)p.H * DV;
    bool bad = slot >= p.P;
    f32x4 s[RPL];
    const size_t at = ((size_t)slot * p.H + h) * DK * DV + (size_t)(RPL * rg) * DV + col;
    if (!bad) {
#pragma unroll
        for (int i = 0; i < RPL; ++i) s[i] = *(const f32x4 *)(p.state_in + at + (size_t)i * DV);
    }
    // A slot belongs to the first row that names it: a row looks at those before it, 64 at a time (N^2 / 128
    // loads a head and column tile; hidden behind the state's load up to some thousand rows, see gdn_ops.h).
    if (p.slots) {
        bool taken = false;
        for (int m = l; m < n; m += 64) taken |= p.slots[m] == slot;
        bad |= __any(taken);
    }
    if (bad) {
        const float nan = __builtin_nanf("");
        if (rg == 0)
            for (int t = 0; t < len; ++t) Tr<E>::store(out + t * ostep, Tr<E>::from_f32(f32x4{nan, nan, nan, nan}));
        return;
    }
    const int hk = h / (p.H / p.Hk);
    const E *qp = p.q + ((size_t)n * p.L * p.Hk + hk) * DK + RPL * rg;
    const E *kp = p.k + ((size_t)n * p.L * p.Hk + hk) * DK + RPL * rg;
    const E *vp = p.v + ((size_t)n * p.L * p.H + h) * DV + col;
    const size_t kstep = (size_t)p.Hk * DK;
    const size_t g0 = (size_t)n * p.L * p.H + h;
    for (int t = 0; t < len; ++t) {
        float kv[RPL], qv[RPL];
        load_f32<RPL>(kp + t * kstep, kv);
        load_f32<RPL>(qp + t * kstep, qv);
        const f32x4 v = Tr<E>::to_f32(Tr<E>::load(vp + t * ostep));
        const float a = p.alpha[g0 + (size_t)t * p.H], b = p.beta[g0 + (size_t)t * p.H];
        f32x4 sk = {0.f, 0.f, 0.f, 0.f}, sq = sk;
        float kq = 0.f;
#pragma unroll
        for (int i = 0; i < RPL; ++i) {
            sk += s[i] * kv[i];
            sq += s[i] * qv[i];
            kq += kv[i] * qv[i];
        }
#pragma unroll
        for (int d = CL; d < 64; d <<= 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sk[e] += __shfl_xor(sk[e], d);
                sq[e] += __shfl_xor(sq[e], d);
            }
            kq += __shfl_xor(kq, d);
        }
        const f32x4 u = b * (v - a * sk);
#pragma unroll
        for (int i = 0; i < RPL; ++i) s[i] = a * s[i] + kv[i] * u;
        if (rg == 0) Tr<E>::store(out + t * ostep, Tr<E>::from_f32(a * sq + kq * u));
    }
#pragma unroll
    for (int i = 0; i < RPL; ++i) *(f32x4 *)(p.state_out + at + (size_t)i * DV) = s[i];
}

}  // namespace gdn
