// HIP kernels (gfx950 / CDNA4) for what stands before and behind a mixer in its block:
//   k_addnorm_fwd / k_addnorm_bwd : residual add with a scale per channel, root-mean-square norm with a weight
//   k_gate_fwd / k_gate_bwd       : norm of a mixer's output (heads first), times weight and gate, tokens first
// All of them stream: a row is read once, kept in registers while its sums are formed, and written once. `LANES` threads
// take a row, `PIECES` pieces of 16 bytes each; a workgroup takes several rows where one does not need it whole, and goes
// on to further rows, so that weights are loaded once and the gradients of weights are summed in registers.
// Bound by memory (bfloat16, a copy reaches 4.9 TB/s): k_addnorm_bwd 32768 x 2048 with scale and weight 805 MB in 132 us, 6.1 TB/s; 16 heads x 32768 x 128
// k_gate_fwd 403 MB in 74 us, 5.4, k_gate_bwd 671 MB in 123 us, 5.5. Small calls are one launch: 64 rows of 2048 3.2 us.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "lasp_block.h"

namespace lasp {

// Threads of a workgroup, and the rows it takes at a time.
template <int LANES>
struct Group {
    static constexpr int NT = LANES > 256 ? LANES : 256, ROWS = NT / LANES, WAVES = LANES / 64;
};

// Sums over the threads of a row, in every one of them, in a fixed order.
template <int LANES, int K>
DEVI void row_sums(float (&v)[K], float *lds) {
#pragma unroll
    for (int d = LANES < 64 ? LANES / 2 : 32; d > 0; d >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor(v[k], d);
    if constexpr (LANES > 64) {   // over the waves of the row
        constexpr int WAVES = LANES / 64;
        lds += threadIdx.x / LANES * (K * WAVES);
        __syncthreads();          // the sums of the turn before have been read
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) lds[k * WAVES + (threadIdx.x % LANES >> 6)] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) v[k] += lds[k * WAVES + w];
        }
    }
}
DEVI float rstd_of(float squares, int C, float eps) { return 1.0f / __builtin_sqrtf(squares / (float)C + eps); }

// The pieces of a row a thread takes: piece k is number lane + k LANES of C / W.
template <typename T, int LANES, int PIECES>
struct Mine {
    static constexpr int W = Piece<T>::W;
    int lane, n;
    DEVI explicit Mine(int C) : lane(threadIdx.x % LANES), n(C / W) {}
    DEVI bool has(int k) const { return lane + k * LANES < n; }
    DEVI int at(int k) const { return min(lane + k * LANES, n - 1) * W; }   // (one that exists, whatever k)
};
template <int PIECES>
struct Places {
    int t[PIECES];
};
template <typename T, int LANES, int PIECES>
DEVI Places<PIECES> places(const Mine<T, LANES, PIECES> &my) {
    Places<PIECES> p;
#pragma unroll
    for (int k = 0; k < PIECES; ++k) p.t[k] = my.at(k);
    return p;
}
template <int W>
DEVI void load_weight(const float *w, int at, float (&f)[W]) {
    if (w) {
        load_floats<W>(w + at, f);
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) f[i] = 1.0f;
    }
}

// The weights of a thread's pieces: in registers for all rows it takes, or (rows of a 1024-thread workgroup, whose threads have
// 128 registers) loaded for every row.
template <typename T, int LANES, int PIECES>
struct Weights {
    static constexpr int W = Piece<T>::W;
    static constexpr bool KEEP = LANES <= 256;
    const float *p;
    float f[KEEP ? PIECES : 1][W];
    DEVI Weights(const float *vec, const int (&at)[PIECES]) : p(vec) {
        if constexpr (KEEP)
#pragma unroll
            for (int k = 0; k < PIECES; ++k) load_weight<W>(p, at[k], f[k]);
    }
    DEVI void get(int k, int at, float (&w)[W]) const {
        if constexpr (KEEP) {
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = f[k][i];
        } else {
            load_weight<W>(p, at, w);
        }
    }
};

// A workgroup's sums for a vector of C floats, one partial row: the row groups of a wave are added by shuffles, those of several
// waves (or rows of two waves) one after the other in LDS.
template <typename T, int LANES, int PIECES>
DEVI void write_partial(const Mine<T, LANES, PIECES> &my, float (&acc)[PIECES][Piece<T>::W], float *dst, float *lds) {
    constexpr int W = Piece<T>::W, SPAN = LANES < 64 ? 64 : LANES, PARTS = Group<LANES>::NT / SPAN;
#pragma unroll
    for (int d = LANES; d < 64; d *= 2)
#pragma unroll
        for (int k = 0; k < PIECES; ++k)
#pragma unroll
            for (int i = 0; i < W; ++i) acc[k][i] += __shfl_xor(acc[k][i], d);
    const bool writes = threadIdx.x % SPAN < LANES;
    for (int r = 0; r < PARTS; ++r) {
        if (r > 0) __syncthreads();
        if (writes && threadIdx.x / SPAN == r)
#pragma unroll
            for (int k = 0; k < PIECES; ++k)
                if (my.has(k)) {
                    float *p = lds + my.at(k);
                    if (r > 0) {
                        float g[W];
                        load_floats<W>(p, g);
#pragma unroll
                        for (int i = 0; i < W; ++i) acc[k][i] += g[i];
                    }
                    store_floats<W>(r == PARTS - 1 ? dst + my.at(k) : p, acc[k]);
                }
    }
    if (PARTS > 1) __syncthreads();   // (LDS is free again)
}

// ---------------------------------------------------------------------------
// Before a block.
// ---------------------------------------------------------------------------
template <typename T, int LANES, int PIECES, bool STREAM>
__global__ __launch_bounds__(Group<LANES>::NT) void k_addnorm_fwd(const T *r, const T *__restrict__ x, const float *__restrict__ scale,
                                                                  const float *__restrict__ weight, float eps, T *r_out,
                                                                  T *__restrict__ y, int rows, int C) {
    using P = Piece<T>;
    constexpr int W = P::W, ROWS = Group<LANES>::ROWS;
    __shared__ float lds[Group<LANES>::NT / 64];
    const Mine<T, LANES, PIECES> my(C);
    const Weights<T, LANES, PIECES> ws(weight, places(my).t), scs(scale, places(my).t);
    for (long long row0 = (long long)blockIdx.x * ROWS; row0 < rows; row0 += (long long)gridDim.x * ROWS) {
        const long long row = row0 + threadIdx.x / LANES;
        const bool there = row < rows;
        const size_t base = (size_t)(there ? row : row0) * C;
        u32x4 vr[PIECES], vx[PIECES];
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            vr[k] = gload<u32x4, STREAM>(r + base + my.at(k), 0);
            if (x) vx[k] = gload<u32x4, STREAM>(x + base + my.at(k), 0);
        }
        float f[PIECES][W], sums[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            P::unpack(vr[k], f[k]);
            if (x) {
                float g[W], sc[W];
                P::unpack(vx[k], g);
                scs.get(k, my.at(k), sc);
#pragma unroll
                for (int i = 0; i < W; ++i) f[k][i] = __builtin_fmaf(sc[i], g[i], f[k][i]);
            }
            if (my.has(k))
#pragma unroll
                for (int i = 0; i < W; ++i) sums[0] = __builtin_fmaf(f[k][i], f[k][i], sums[0]);
        }
        row_sums<LANES>(sums, lds);
        const float rstd = rstd_of(sums[0], C, eps);
        if (there)
#pragma unroll
            for (int k = 0; k < PIECES; ++k)
                if (my.has(k)) {
                    if (r_out) put<STREAM>(r_out + base + my.at(k), P::pack(f[k]));
                    float o[W], w[W];
                    ws.get(k, my.at(k), w);
#pragma unroll
                    for (int i = 0; i < W; ++i) o[i] = f[k][i] * rstd * w[i];
                    put<STREAM>(y + base + my.at(k), P::pack(o));
                }
    }
}

template <typename T, int LANES, int PIECES, bool STREAM>
__global__ __launch_bounds__(Group<LANES>::NT) void k_addnorm_bwd(const T *__restrict__ r, const T *__restrict__ x,
                                                                  const float *__restrict__ scale, const float *__restrict__ weight,
                                                                  float eps, const T *__restrict__ dy, const T *dr_out, T *dr,
                                                                  T *__restrict__ dx, float *__restrict__ pw, float *__restrict__ ps,
                                                                  int rows, int C) {
    using P = Piece<T>;
    constexpr int W = P::W, ROWS = Group<LANES>::ROWS;
    constexpr bool LATE = LANES == 1024;   // (128 registers a thread: what the sums do not need is loaded behind them)
    __shared__ float lds[2 * Group<LANES>::NT / 64];
    __shared__ __attribute__((aligned(16))) float part[ROWS > 1 ? LANES * PIECES * W : 4];
    const Mine<T, LANES, PIECES> my(C);
    const Weights<T, LANES, PIECES> ws(weight, places(my).t), scs(scale, places(my).t);
    float aw[PIECES][W] = {}, as[PIECES][W] = {};
    for (long long row0 = (long long)blockIdx.x * ROWS; row0 < rows; row0 += (long long)gridDim.x * ROWS) {
        const long long row = row0 + threadIdx.x / LANES;
        const bool there = row < rows;
        const size_t base = (size_t)(there ? row : row0) * C;
        u32x4 vr[PIECES], vy[PIECES], vx[PIECES], vd[PIECES];
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            const size_t at = base + my.at(k);
            vr[k] = gload<u32x4, STREAM>(r + at, 0);
            vy[k] = gload<u32x4, STREAM>(dy + at, 0);
            if constexpr (!LATE) {
                if (ps) vx[k] = gload<u32x4, STREAM>(x + at, 0);
                if (dr_out) vd[k] = gload<u32x4, STREAM>(dr_out + at, 0);
            }
        }
        float sums[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < PIECES; ++k)
            if (my.has(k)) {
                float f[W], g[W], w[W];
                P::unpack(vr[k], f);
                P::unpack(vy[k], g);
                ws.get(k, my.at(k), w);
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    sums[0] = __builtin_fmaf(f[i], f[i], sums[0]);
                    sums[1] = __builtin_fmaf(w[i] * g[i], f[i], sums[1]);
                }
            }
        row_sums<LANES>(sums, lds);
        const float rstd = rstd_of(sums[0], C, eps), c = sums[1] / (float)C * rstd * rstd;
        if (there)
#pragma unroll
            for (int k = 0; k < PIECES; ++k)
                if (my.has(k)) {
                    float f[W], g[W], d[W], o[W], w[W], sc[W];
                    if constexpr (LATE) {
                        if (ps) vx[k] = gload<u32x4, STREAM>(x + base + my.at(k), 0);
                        if (dr_out) vd[k] = gload<u32x4, STREAM>(dr_out + base + my.at(k), 0);
                    }
                    P::unpack(vr[k], f);
                    P::unpack(vy[k], g);
                    ws.get(k, my.at(k), w);
                    scs.get(k, my.at(k), sc);
                    if (dr_out) P::unpack(vd[k], d);
                    else
#pragma unroll
                        for (int i = 0; i < W; ++i) d[i] = 0.0f;
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        d[i] = __builtin_fmaf(rstd, w[i] * g[i] - f[i] * c, d[i]);
                        aw[k][i] = __builtin_fmaf(g[i] * f[i], rstd, aw[k][i]);
                        o[i] = sc[i] * d[i];
                    }
                    put<STREAM>(dr + base + my.at(k), P::pack(d));
                    if (dx) put<STREAM>(dx + base + my.at(k), P::pack(o));
                    if (ps) {
                        P::unpack(vx[k], f);
#pragma unroll
                        for (int i = 0; i < W; ++i) as[k][i] = __builtin_fmaf(f[i], d[i], as[k][i]);
                    }
                }
    }
    if (pw) write_partial<T, LANES, PIECES>(my, aw, pw + (size_t)blockIdx.x * C, part);
    if (ps) write_partial<T, LANES, PIECES>(my, as, ps + (size_t)blockIdx.x * C, part);
}

// ---------------------------------------------------------------------------
// Behind a block. A row is a head of a token (its C = D features) or a whole token (C = H D); `per` rows make a token, and
// a thread stays with the same head of every token it comes to, so that its weights and their gradients stay in registers.
// ---------------------------------------------------------------------------
// act(u) and its derivative.
DEVI void activate(int gate, float u, float &act, float &slope) {
    if (gate == 1) {
        act = u;
        slope = 1.0f;
    } else {
        // s = 1 / (1 + e^-u): 0 and 1 at the ends, where the power is infinite or 0. Its complement s(-u) where s is near 1, e^-u s, has the
        // precision that 1 - s loses there (at u = 16 6 %, from 17 on everything).
        const float e = __builtin_amdgcn_exp2f(u * -1.44269504f), s = __builtin_amdgcn_rcpf(1.0f + e), c = u > 0.0f ? e * s : 1.0f - s;
        act = gate == 2 ? s : u * s;
        slope = s * (gate == 2 ? c : __builtin_fmaf(u, c, 1.0f));
    }
}

// Where a thread's pieces lie: o(k) in a token's part of o, t(k) in its row of u, y.
template <typename T, int LANES, int PIECES>
struct GatePlace {
    Mine<T, LANES, PIECES> my;
    long long slot, token0, step;   // this thread's row group, its first token, tokens from one turn to the next
    size_t o[PIECES];
    int t[PIECES];
    DEVI GatePlace(int C, int per, int H, int N, int D) : my(C) {
        constexpr int ROWS = Group<LANES>::ROWS;
        slot = (long long)blockIdx.x * ROWS + threadIdx.x / LANES;
        step = (long long)gridDim.x * ROWS / per;
        token0 = slot / per;
        const int head = (int)(slot - token0 * per);
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            t[k] = head * C + my.at(k);
            const int h = t[k] / D;
            o[k] = (size_t)h * N * D + (t[k] - h * D);
        }
    }
};

template <typename T, int LANES, int PIECES, bool STREAM>
__global__ __launch_bounds__(Group<LANES>::NT) void k_gate_fwd(const T *__restrict__ O, const T *__restrict__ U,
                                                               const float *__restrict__ weight, float eps, T *__restrict__ Y, int gate,
                                                               int tokens, int per, int C, int H, int N, int D, long long ld) {
    using P = Piece<T>;
    constexpr int W = P::W;
    __shared__ float lds[Group<LANES>::NT / 64];
    const GatePlace<T, LANES, PIECES> at(C, per, H, N, D);
    const auto &my = at.my;
    const size_t wide = (size_t)H * D;
    const Weights<T, LANES, PIECES> ws(weight, at.t);
    // (every thread takes as many turns as the first of its workgroup: the sums may need all of them)
    const long long first = (long long)blockIdx.x * Group<LANES>::ROWS / per;
    for (long long turn = 0; first + turn * at.step < tokens; ++turn) {
        const long long want = at.token0 + turn * at.step;
        const bool there = want < tokens && at.token0 < at.step;
        const size_t tok = there ? want : 0, seq = tok / N;
        const T *o = O + (tok + seq * (H - 1) * N) * D;
        u32x4 vo[PIECES], vu[PIECES];
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            vo[k] = gload<u32x4, STREAM>(o + at.o[k], 0);
            if (gate) vu[k] = gload<u32x4, STREAM>(U + tok * ld + at.t[k], 0);
        }
        float f[PIECES][W], sums[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            P::unpack(vo[k], f[k]);
            if (my.has(k))
#pragma unroll
                for (int i = 0; i < W; ++i) sums[0] = __builtin_fmaf(f[k][i], f[k][i], sums[0]);
        }
        row_sums<LANES>(sums, lds);
        const float rstd = rstd_of(sums[0], C, eps);
        if (there)
#pragma unroll
            for (int k = 0; k < PIECES; ++k)
                if (my.has(k)) {
                    float u[W], w[W];
                    if (gate) P::unpack(vu[k], u);
                    ws.get(k, at.t[k], w);
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        f[k][i] *= rstd * w[i];
                        if (gate) {
                            float act, slope;
                            activate(gate, u[i], act, slope);
                            f[k][i] *= act;
                        }
                    }
                    put<STREAM>(Y + tok * wide + at.t[k], P::pack(f[k]));
                }
    }
}

template <typename T, int LANES, int PIECES, bool STREAM>
__global__ __launch_bounds__(Group<LANES>::NT) void k_gate_bwd(const T *__restrict__ O, const T *__restrict__ U,
                                                               const float *__restrict__ weight, float eps, const T *__restrict__ dY,
                                                               T *__restrict__ dO, T *__restrict__ dU, float *__restrict__ pw, int gate,
                                                               int tokens, int per, int C, int H, int N, int D, long long ld) {
    using P = Piece<T>;
    constexpr int W = P::W, ROWS = Group<LANES>::ROWS;
    __shared__ float lds[2 * Group<LANES>::NT / 64];
    __shared__ __attribute__((aligned(16))) float part[ROWS > 1 ? LANES * PIECES * W : 4];
    const GatePlace<T, LANES, PIECES> at(C, per, H, N, D);
    const auto &my = at.my;
    const size_t wide = (size_t)H * D;
    const Weights<T, LANES, PIECES> ws(weight, at.t);
    float aw[PIECES][W] = {};
    const long long first = (long long)blockIdx.x * ROWS / per;
    for (long long turn = 0; first + turn * at.step < tokens; ++turn) {
        const long long want = at.token0 + turn * at.step;
        const bool there = want < tokens && at.token0 < at.step;
        const size_t tok = there ? want : 0, seq = tok / N, head0 = (tok + seq * (H - 1) * N) * D;
        u32x4 vo[PIECES], vu[PIECES], vy[PIECES];
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            vo[k] = gload<u32x4, STREAM>(O + head0 + at.o[k], 0);
            vy[k] = gload<u32x4, STREAM>(dY + tok * wide + at.t[k], 0);
            if (gate) vu[k] = gload<u32x4, STREAM>(U + tok * ld + at.t[k], 0);
        }
        float sums[2] = {0.0f, 0.0f};
        float g[PIECES][W], du[PIECES][W];   // dy act(u), dy weight act'(u)
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            float f[W], u[W], w[W];
            P::unpack(vo[k], f);
            P::unpack(vy[k], g[k]);
            ws.get(k, at.t[k], w);
            if (gate) {
                P::unpack(vu[k], u);
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    float act, slope;
                    activate(gate, u[i], act, slope);
                    du[k][i] = g[k][i] * w[i] * slope;
                    g[k][i] *= act;
                }
            }
            if (my.has(k))
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    sums[0] = __builtin_fmaf(f[i], f[i], sums[0]);
                    sums[1] = __builtin_fmaf(w[i] * g[k][i], f[i], sums[1]);
                }
        }
        row_sums<LANES>(sums, lds);
        const float rstd = rstd_of(sums[0], C, eps), c = sums[1] / (float)C * rstd * rstd;
        if (there)
#pragma unroll
            for (int k = 0; k < PIECES; ++k)
                if (my.has(k)) {
                    float f[W], d[W], w[W];
                    P::unpack(vo[k], f);
                    ws.get(k, at.t[k], w);
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        d[i] = rstd * (w[i] * g[k][i] - f[i] * c);
                        aw[k][i] = __builtin_fmaf(g[k][i] * f[i], rstd, aw[k][i]);
                    }
                    put<STREAM>(dO + head0 + at.o[k], P::pack(d));
                    if (gate) {
#pragma unroll
                        for (int i = 0; i < W; ++i) d[i] = du[k][i] * f[i] * rstd;
                        put<STREAM>(dU + tok * ld + at.t[k], P::pack(d));
                    }
                }
    }
    if (!pw) return;
    if (per == 1) {
        write_partial<T, LANES, PIECES>(my, aw, pw + (size_t)blockIdx.x * C, part);
    } else if (at.token0 < at.step) {   // a partial row per token of a turn; every head's part from its own threads
#pragma unroll
        for (int k = 0; k < PIECES; ++k)
            if (my.has(k)) store_floats<W>(pw + at.token0 * wide + at.t[k], aw[k]);
    }
}

// ---------------------------------------------------------------------------
// k_column_sums: out[c] = part[0][c] + part[1][c] + ..., blockIdx.y one of two such sums. A workgroup takes 32 columns, eight
// threads by 32 groups of rows; fixed order.
// ---------------------------------------------------------------------------
constexpr int kSumColumns = 32, kSumGroups = 32;
__global__ __launch_bounds__(kSumColumns * kSumGroups / 4) void k_column_sums(const float *__restrict__ part0, float *__restrict__ out0,
                                                                              const float *__restrict__ part1, float *__restrict__ out1,
                                                                              int n, int C) {
    __shared__ f32x4 lds[kSumGroups][kSumColumns / 4];
    const float *part = blockIdx.y ? part1 : part0;
    float *out = blockIdx.y ? out1 : out0;
    const int c4 = threadIdx.x % (kSumColumns / 4), g = threadIdx.x / (kSumColumns / 4);
    const int c = blockIdx.x * kSumColumns + 4 * c4;
    f32x4 sum{0, 0, 0, 0};
    if (c < C)
#pragma unroll 8
        for (int r = g; r < n; r += kSumGroups) sum += *(const f32x4 *)(part + (size_t)r * C + c);
    lds[g][c4] = sum;
    __syncthreads();
    if (g != 0 || c >= C) return;
    for (int i = 1; i < kSumGroups; ++i) sum += lds[i][c4];
    *(f32x4 *)(out + c) = sum;
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
// A row over as many threads as it has pieces, up to 256; a wave with four pieces a thread needs no barrier, but keeps fewer rows on
// their way (addnorm bfloat16 32768 x 2048, a wave / four: forward 91 / 90 us, backward 143 / 132; float 20011 x 1000 forward 62.5 / 57.4). Wider rows in
// two and four pieces (16384 x 4096 backward, 256 threads / 512 148 / 151 us; 8192 x 8192, 256 / 512 / 1024 148 / 156 / 174; 4096 x 16384, 512 / 1024 182 / 204).
RowPlan row_plan(int tokens, int heads, int C, int dtype) {
    RowPlan p{tokens, heads, C, dtype, 64, 1};
    const int n = C / (dtype == 0 ? 4 : 8);
    p.lanes = 2;
    while (p.lanes < n && p.lanes < 256) p.lanes *= 2;
    if (n > 1024) p.lanes = n <= 2048 ? 512 : 1024;
    p.pieces = n <= p.lanes ? 1 : n <= 2 * p.lanes ? 2 : 4;
    return p;
}
namespace {
constexpr int kCus = 256, kForward = 4 * kCus;
int rows_at_a_time(const RowPlan &p) { return std::max(p.lanes, 256) / p.lanes; }
// Workgroups: no more than there are rows for, and (rows that are heads) at least one row group for every head of a token.
int workgroups(const RowPlan &p, int most) {
    const long long rows = (long long)p.tokens * p.heads, at = rows_at_a_time(p);
    return (int)std::max<long long>(std::min<long long>((rows + at - 1) / at, most), (p.heads + at - 1) / at);
}
// Workgroups of a backward pass that reads `loads` tensors. Rows of one piece a thread: as many on a CU (every CU the same) as keep
// about the same number of bytes on their way, and no more, since each writes a partial row (addnorm bfloat16 32768 x 2048, four tensors
// read, 512 / 576 / 768 / 1024 workgroups: 132 / 148 / 144 / 153 us; three: 109 / - / 92 / 97; float 65536 x 1024, four: 324 / - / 270 / 277);
// more where a row leaves half of its threads without a piece (129055 x 520, 512 / 1024: 212 / 166; float 768 / 1536: 419 / 305). Small
// calls: four turns or more each (8192 x 512 16.3 -> 14.8). Rows of more pieces have enough with two.
int backward_workgroups(const RowPlan &p, int loads) {
    const long long turns = ((long long)p.tokens * p.heads + rows_at_a_time(p) - 1) / rows_at_a_time(p);
    int a_cu = 2;
    if (p.pieces == 1) {
        const int n = p.C / (p.dtype == 0 ? 4 : 8), full = (p.dtype == 0 ? 7 : 6) - loads;
        a_cu = std::min((full * p.lanes + n / 2) / n, p.dtype == 0 ? 2 * full : 4);
    }
    return workgroups(p, (int)std::max<long long>(std::min<long long>(a_cu * kCus, turns / 4), kCus));
}
// A partial row of the weights' gradients for every workgroup (rows that are tokens), or for every token of a turn.
int partial_rows(const RowPlan &p, int loads) {
    const int n = backward_workgroups(p, loads);
    return p.heads == 1 ? n : (int)((long long)n * rows_at_a_time(p) / p.heads);
}
constexpr int kLeastLoads = 2;   // (o or r, and dy)
// f.template operator()<T, LANES, PIECES, STREAM>() for the plan's.
template <typename T, bool STREAM, typename F>
void by_lanes(const RowPlan &p, F f) {
    const int key = p.lanes * 8 + p.pieces;
    switch (key) {
#define LASP_ROWS(LANES, PIECES) \
    case LANES * 8 + PIECES: return f.template operator()<T, LANES, PIECES, STREAM>();
        LASP_ROWS(2, 1) LASP_ROWS(4, 1) LASP_ROWS(8, 1) LASP_ROWS(16, 1) LASP_ROWS(32, 1) LASP_ROWS(64, 1) LASP_ROWS(128, 1) LASP_ROWS(256, 1)
        LASP_ROWS(256, 2) LASP_ROWS(256, 4) LASP_ROWS(512, 4)
#undef LASP_ROWS
        default:
            if constexpr (sizeof(T) == 4) return f.template operator()<T, 1024, 4, STREAM>();   // (two-byte rows have 2048 pieces at most)
    }
}
// tensors: of the rows' size that the call reads and writes
template <typename F>
void by_plan(const RowPlan &p, int tensors, F f) {
    const bool stream = past_cache((size_t)tensors * p.tokens * p.heads * p.C * (p.dtype == 0 ? 4 : 2));
    if (p.dtype == 0) stream ? by_lanes<float, true>(p, f) : by_lanes<float, false>(p, f);
    else stream ? by_lanes<bf16_t, true>(p, f) : by_lanes<bf16_t, false>(p, f);
}
struct AddNormFwd {
    const RowPlan &p;
    const AddNormArgs &a;
    hipStream_t s;
    template <typename T, int LANES, int PIECES, bool STREAM>
    void operator()() const {
        k_addnorm_fwd<T, LANES, PIECES, STREAM><<<dim3(workgroups(p, kForward)), dim3(Group<LANES>::NT), 0, s>>>(
            (const T *)a.r, (const T *)a.x, a.scale, a.weight, a.eps, (T *)a.r_out, (T *)a.y, p.tokens, p.C);
    }
};
struct AddNormBwd {
    const RowPlan &p;
    const AddNormArgs &a;
    hipStream_t s;
    template <typename T, int LANES, int PIECES, bool STREAM>
    void operator()() const {
        const int n = backward_workgroups(p, a.loads());
        k_addnorm_bwd<T, LANES, PIECES, STREAM><<<dim3(n), dim3(Group<LANES>::NT), 0, s>>>(
            (const T *)a.r, (const T *)a.x, a.scale, a.weight, a.eps, (const T *)a.dy, (const T *)a.dr_out, (T *)a.dr, (T *)a.dx,
            a.dweight ? a.scratch : nullptr, a.dscale ? a.scratch + (size_t)n * p.C : nullptr, p.tokens, p.C);
    }
};
struct GateFwd {
    const RowPlan &p;
    const GateArgs &a;
    hipStream_t s;
    template <typename T, int LANES, int PIECES, bool STREAM>
    void operator()() const {
        k_gate_fwd<T, LANES, PIECES, STREAM><<<dim3(workgroups(p, kForward)), dim3(Group<LANES>::NT), 0, s>>>(
            (const T *)a.o, (const T *)a.u, a.weight, a.eps, (T *)a.y, a.gate, p.tokens, p.heads, p.C, a.H, a.N, a.D, a.ld);
    }
};
struct GateBwd {
    const RowPlan &p;
    const GateArgs &a;
    hipStream_t s;
    template <typename T, int LANES, int PIECES, bool STREAM>
    void operator()() const {
        k_gate_bwd<T, LANES, PIECES, STREAM><<<dim3(backward_workgroups(p, a.loads())), dim3(Group<LANES>::NT), 0, s>>>(
            (const T *)a.o, (const T *)a.u, a.weight, a.eps, (const T *)a.dy, (T *)a.d_o, (T *)a.du, a.dweight ? a.scratch : nullptr,
            a.gate, p.tokens, p.heads, p.C, a.H, a.N, a.D, a.ld);
    }
};
}  // namespace

hipError_t launch_column_sums(const float *p0, float *o0, const float *p1, float *o1, int n, int C, hipStream_t s) {
    if (!o0) {
        p0 = p1;
        o0 = o1;
        o1 = nullptr;
    }
    if (o0) k_column_sums<<<dim3((C + kSumColumns - 1) / kSumColumns, o1 ? 2 : 1), dim3(kSumColumns * kSumGroups / 4), 0, s>>>(p0, o0, p1, o1, n, C);
    return hipGetLastError();
}
size_t addnorm_scratch(const RowPlan &p) { return 2 * (size_t)partial_rows(p, kLeastLoads) * p.C * sizeof(float); }
size_t gatenorm_scratch(const RowPlan &p) { return (size_t)partial_rows(p, kLeastLoads) * p.heads * p.C * sizeof(float); }

hipError_t launch_addnorm_fwd(const RowPlan &p, const AddNormArgs &a, hipStream_t s) {
    by_plan(p, a.x ? 4 : 2, AddNormFwd{p, a, s});
    return hipGetLastError();
}
hipError_t launch_addnorm_bwd(const RowPlan &p, const AddNormArgs &a, hipStream_t s) {
    by_plan(p, 3 + !!a.dscale + !!a.dr_out + !!a.dx, AddNormBwd{p, a, s});
    const int n = partial_rows(p, a.loads());
    return launch_column_sums(a.scratch, a.dweight, a.scratch + (size_t)n * p.C, a.dscale, n, p.C, s);
}
hipError_t launch_gatenorm_fwd(const RowPlan &p, const GateArgs &a, hipStream_t s) {
    by_plan(p, 2 + !!a.gate, GateFwd{p, a, s});
    return hipGetLastError();
}
hipError_t launch_gatenorm_bwd(const RowPlan &p, const GateArgs &a, hipStream_t s) {
    by_plan(p, 3 + 2 * !!a.gate, GateBwd{p, a, s});
    return launch_column_sums(a.scratch, a.dweight, nullptr, nullptr, partial_rows(p, a.loads()), p.heads * p.C, s);
}

}  // namespace lasp
