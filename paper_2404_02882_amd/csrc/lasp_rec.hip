// HIP kernels (gfx950 / CDNA4) for the gated linear recurrence h_s = a_s h_{s-1} + b_s x_s, a_s = exp(log_a_s), elementwise
// over channels: the vector-state member of the recurrences of LASP (arxiv 2404.02882) App. A.4, Table 6.
#include <hip/hip_runtime.h>

#include "lasp_block.h"

namespace lasp {

// The gate of one element. A step of the recurrence is y -> a y + u.
template <typename T>
struct Gate;
// bfloat16 data: a in one float. Its rounding, 2^-25 of a, is a relative 2^-25 / (1 - a) of what the state converges to;
// log_a itself comes rounded to 2^-9, which weighs more for any a that a memory of fewer than 2^16 tokens has.
template <>
struct Gate<bf16_t> {
    float a;
    DEVI explicit Gate(float log_a) : a(__builtin_amdgcn_exp2f(log_a * 1.44269504f)) {}
    DEVI float step(float y, float u) const { return __builtin_fmaf(a, y, u); }
    DEVI float times(float y) const { return a * y; }
    DEVI float b() const { return 1.0f - a; }
};
// Float data: a = hi + lo. For |log_a| < 1/2 from m = a - 1 by its power series (log_a^9 / 9! < 2^-26 of log_a is left
// out), so that 1 - a has 24 bits however near to 1 a is; beyond, lo = 0.
template <>
struct Gate<float> {
    float hi, lo, m;
    DEVI explicit Gate(float l) {
        if (__builtin_fabsf(l) < 0.5f) {
            float q = 1.0f / 40320;
            q = __builtin_fmaf(q, l, 1.0f / 5040);
            q = __builtin_fmaf(q, l, 1.0f / 720);
            q = __builtin_fmaf(q, l, 1.0f / 120);
            q = __builtin_fmaf(q, l, 1.0f / 24);
            q = __builtin_fmaf(q, l, 1.0f / 6);
            q = __builtin_fmaf(q, l, 0.5f);
            m = __builtin_fmaf(l * l, q, l);
            hi = 1.0f + m;
            lo = m - (hi - 1.0f);
        } else {
            // log_a log2(e) in two floats: the product's rounding would be |log_a| 2^-24 of a
            const float t = l * 1.44269504f, rest = __builtin_fmaf(l, 1.44269504f, -t) + l * 1.92596303e-8f;
            const float e = __builtin_amdgcn_exp2f(t);
            hi = e > 0.0f ? __builtin_fmaf(e, rest * 0.693147181f, e) : e;   // (log_a = -inf: rest is NaN)
            lo = 0.0f;
            m = hi - 1.0f;
        }
    }
    DEVI float step(float y, float u) const { return __builtin_fmaf(hi, y, __builtin_fmaf(lo, y, u)); }
    DEVI float times(float y) const { return __builtin_fmaf(hi, y, lo * y); }
    DEVI float b() const { return -m; }
};

// Where a column lies: its sequence, first channel, tokens that exist.
template <typename T>
struct Column {
    int seq, ch, n;
    DEVI Column(int col, int N, int D, const int *len) {
        const int per = D / Piece<T>::W;
        seq = col / per;
        ch = (col - seq * per) * Piece<T>::W;
        n = len ? min(max(len[seq], 0), N) : N;
    }
};

// ---------------------------------------------------------------------------
// k_rec_step_fwd / k_rec_step_bwd: a thread carries a column's state over all tokens, AHEAD tokens requested ahead.
// ---------------------------------------------------------------------------
constexpr int kStepThreads = 64, kAhead = 4;

template <typename T, bool COUPLED>
__global__ __launch_bounds__(kStepThreads) void k_rec_step_fwd(const T *__restrict__ X, const T *__restrict__ L, const float *h_in,
                                                               const int *__restrict__ len, T *__restrict__ out, float *h_out,
                                                               int cols, int N, int D, long long ld) {
    using P = Piece<T>;
    constexpr int W = P::W;
    const int col = blockIdx.x * kStepThreads + threadIdx.x;
    if (col >= cols) return;
    const Column<T> c(col, N, D, len);
    const size_t state = (size_t)c.seq * D + c.ch, row0 = (size_t)c.seq * N;
    float y[W] = {};
    if (h_in) load_floats<W>(h_in + state, y);
    const T *x = X + row0 * ld + c.ch, *l = L + row0 * ld + c.ch;
    T *o = out + row0 * D + c.ch;
    for (int s0 = 0; s0 < c.n; s0 += kAhead) {
        u32x4 vx[kAhead], vl[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const size_t at = (size_t)min(s0 + k, c.n - 1) * ld;
            vx[k] = *(const u32x4 *)(x + at);
            vl[k] = *(const u32x4 *)(l + at);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (s0 + k < c.n) {
                float fx[W], fl[W];
                P::unpack(vx[k], fx);
                P::unpack(vl[k], fl);
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const Gate<T> g(fl[i]);
                    y[i] = g.step(y[i], COUPLED ? g.b() * fx[i] : fx[i]);
                }
                *(u32x4 *)(o + (size_t)(s0 + k) * D) = P::pack(y);
            }
    }
    for (int s = c.n; s < N; ++s) *(u32x4 *)(o + (size_t)s * D) = u32x4{0, 0, 0, 0};
    if (h_out) store_floats<W>(h_out + state, y);
}

template <typename T, bool COUPLED>
__global__ __launch_bounds__(kStepThreads) void k_rec_step_bwd(const T *__restrict__ X, const T *__restrict__ L, const T *__restrict__ out,
                                                               const T *__restrict__ dout, const float *h_in, const float *dh_out,
                                                               const int *__restrict__ len, T *__restrict__ dx, T *__restrict__ dl,
                                                               float *dh_in, int cols, int N, int D, long long ld) {
    using P = Piece<T>;
    constexpr int W = P::W;
    const int col = blockIdx.x * kStepThreads + threadIdx.x;
    if (col >= cols) return;
    const Column<T> c(col, N, D, len);
    const size_t state = (size_t)c.seq * D + c.ch, row0 = (size_t)c.seq * N;
    float y[W] = {};   // a_s e_s, the gradient that reaches h_{s-1}
    if (dh_out) load_floats<W>(dh_out + state, y);
    const size_t p0 = row0 * ld + c.ch, t0 = row0 * D + c.ch;
    for (int s = N - 1; s >= c.n; --s) {
        *(u32x4 *)(dx + p0 + (size_t)s * ld) = u32x4{0, 0, 0, 0};
        *(u32x4 *)(dl + p0 + (size_t)s * ld) = u32x4{0, 0, 0, 0};
    }
    for (int s0 = c.n - 1; s0 >= 0; s0 -= kAhead) {
        u32x4 vx[kAhead], vl[kAhead], vo[kAhead], vd[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int s = max(s0 - k, 0);
            if constexpr (COUPLED) vx[k] = *(const u32x4 *)(X + p0 + (size_t)s * ld);
            vl[k] = *(const u32x4 *)(L + p0 + (size_t)s * ld);
            vd[k] = *(const u32x4 *)(dout + t0 + (size_t)s * D);
            vo[k] = *(const u32x4 *)(out + t0 + (size_t)max(s - 1, 0) * D);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int s = s0 - k;
            if (s >= 0) {
                float fx[W], fl[W], fd[W], fo[W], ox[W], ol[W];
                if constexpr (COUPLED) P::unpack(vx[k], fx);
                P::unpack(vl[k], fl);
                P::unpack(vd[k], fd);
                P::unpack(vo[k], fo);
                if (s == 0) {
#pragma unroll
                    for (int i = 0; i < W; ++i) fo[i] = 0.0f;
                    if (h_in) load_floats<W>(h_in + state, fo);
                }
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const Gate<T> g(fl[i]);
                    const float e = fd[i] + y[i];
                    y[i] = g.times(e);
                    ox[i] = COUPLED ? g.b() * e : e;
                    ol[i] = y[i] * (COUPLED ? fo[i] - fx[i] : fo[i]);
                }
                *(u32x4 *)(dx + p0 + (size_t)s * ld) = P::pack(ox);
                *(u32x4 *)(dl + p0 + (size_t)s * ld) = P::pack(ol);
            }
        }
    }
    if (dh_in) store_floats<W>(dh_in + state, y);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
size_t rec_scratch(const RecPlan &) { return 256; }

template <typename T, bool C>
static hipError_t rec_fwd(const RecPlan &p, const RecArgs &a, hipStream_t s) {
    const int cols = p.B * (p.D / Piece<T>::W);
    k_rec_step_fwd<T, C><<<dim3((cols + kStepThreads - 1) / kStepThreads), dim3(kStepThreads), 0, s>>>(
        (const T *)a.x, (const T *)a.log_a, a.h_in, a.len, (T *)a.out, a.h_out, cols, p.N, p.D, p.ld);
    return hipGetLastError();
}
template <typename T, bool C>
static hipError_t rec_bwd(const RecPlan &p, const RecArgs &a, hipStream_t s) {
    const int cols = p.B * (p.D / Piece<T>::W);
    k_rec_step_bwd<T, C><<<dim3((cols + kStepThreads - 1) / kStepThreads), dim3(kStepThreads), 0, s>>>(
        (const T *)a.x, (const T *)a.log_a, (const T *)a.out_in, (const T *)a.dout, a.h_in, a.dh_out, a.len, (T *)a.dx, (T *)a.dlog_a,
        a.dh_in, cols, p.N, p.D, p.ld);
    return hipGetLastError();
}
hipError_t launch_rec_fwd(const RecPlan &p, const RecArgs &a, hipStream_t s) {
    if (p.dtype == 0) return p.coupled ? rec_fwd<float, true>(p, a, s) : rec_fwd<float, false>(p, a, s);
    return p.coupled ? rec_fwd<bf16_t, true>(p, a, s) : rec_fwd<bf16_t, false>(p, a, s);
}
hipError_t launch_rec_bwd(const RecPlan &p, const RecArgs &a, hipStream_t s) {
    if (p.dtype == 0) return p.coupled ? rec_bwd<float, true>(p, a, s) : rec_bwd<float, false>(p, a, s);
    return p.coupled ? rec_bwd<bf16_t, true>(p, a, s) : rec_bwd<bf16_t, false>(p, a, s);
}

}  // namespace lasp
