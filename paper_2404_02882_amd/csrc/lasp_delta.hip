// HIP kernels (gfx950 / CDNA4) of the gated delta rule,
//     S_s = a_s S_{s-1} + k_s u_s^T,   u_s = beta_s w_s,   w_s = v_s - a_s S_{s-1}^T k_s,   out_s = S_s^T q_s.
// Over a tile of C tokens that starts from S, with G_s = log a_1 + .. + log a_s, W_ij = exp(G_i - G_j) and M_ij = W_ij k_i . k_j (i > j):
//     (I + M beta) w = r,   r_i = v_i - exp(G_i) S^T k_i,
//     out_i = exp(G_i) S^T q_i + sum_{j <= i} W_ij (q_i . k_j) u_j,   S' = exp(G_C) S + sum_j exp(G_C - G_j) k_j u_j^T.
// With N the sums over paths, N_ij = -M_ij - sum_{j<k<i} M_ik beta_k N_kj, the inverse is I + N beta and that of (I + beta M) is I + beta N:
// neither divides by a beta, so beta = 0 needs no case of its own, and with keys of length 1 no |N_ij| exceeds 1.
//   k_delta_prep : N of every tile (tiles are independent)
//   k_delta_walk : the walk over the tiles of a segment, 64 value features a workgroup (columns of S do not meet)
//   k_delta_scan : states between segments: a segment takes S to T S + S_local, T the product of its tiles' matrices
//   k_delta_step : token by token, for calls of a few tokens: state in registers, read and written once
// Backward, with dS the gradient of the state behind the tile:
//     dU = P^T dO + exp(G_C - G) K dS,   dR = dU + N^T (beta dU),   dV = beta dR,   dbeta_i = dR_i . w_i,
//     dS' = exp(G_C) dS + Q^T (exp(G) dO) - K^T (exp(G) dV),   P_ij = W_ij q_i . k_j
//     dQ = exp(G) dO S^T + Ep K,   dK = Ep^T Q + Em K + Em^T K - exp(G) dV S^T + exp(G_C - G) U dS^T,
//     Ep = W (dO U^T),   Em = -W (dV U^T) below the diagonal,
//     dlog_a_i = <dS, S'> + sum_{t >= i} (q_t . dq_t - v_t . dv_t)   (sums within the tile, so that they stay short).
//   k_delta_back : the walk in reverse: dV, and dS and dR of every tile
//   k_delta_grad : dQ, dK, dbeta, dlog_a of every tile (tiles are independent)
//   k_delta_group: sums over the states that share a head of q and k
// Products run on bfloat16 MFMA with fp32 sums. A factor that is no input is kept in parts, x = hi + lo with bfloat16 data (16 significant
// bits, 2^-18 of x: gradients and states come out in float and are held to its precision, which one part, 2^-9, would not reach), and in three
// parts with float data, whose inputs are split too; products of parts below the last kept bit are left out.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "lasp_delta.h"
#include "lasp_device.h"

namespace lasp {
namespace {

typedef Elem<bf16_t> E;
template <typename T>
struct Parts;
template <>
struct Parts<bf16_t> {
    static constexpr int DATA = 1, MADE = 2, C = 64;   // parts of an input and of what is computed; tokens of a tile
};
template <>
struct Parts<float> {
    static constexpr int DATA = 3, MADE = 3, C = 32;
};
constexpr int kThreads = 256, kWaves = 4;

template <int NP>
struct Frags {
    bf16x8 p[NP];
};
// c + a b, smallest terms first; parts (i, j) with i + j < KEEP
template <int KEEP, int NA, int NB>
DEVI f32x16 mm(const Frags<NA> &a, const Frags<NB> &b, f32x16 c) {
#pragma unroll
    for (int s = KEEP - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (s - i >= 0 && s - i < NB) c = E::mfma(a.p[i], b.p[s - i], c);
    return c;
}

constexpr int ld_of(int width) { return width == 128 ? kSwzLd : width + E::PAD; }

// A tile in LDS: NP parts of ROWS rows of WIDTH bfloat16.
template <int NP, int ROWS, int WIDTH>
struct Tile {
    static constexpr int LD = ld_of(WIDTH), PS = ROWS * LD, BYTES = NP * PS * 2;
    bf16_t *p;
    // contraction along a row / down the rows
    DEVI Frags<NP> kc(const Lane &ln, int row0, int k0) const {
        Frags<NP> f;
#pragma unroll
        for (int i = 0; i < NP; ++i) f.p[i] = E::ld_kc(ln, p + i * PS, LD, row0, k0);
        return f;
    }
    DEVI Frags<NP> ks(const Lane &ln, int k0, int col0) const {
        Frags<NP> f;
#pragma unroll
        for (int i = 0; i < NP; ++i) f.p[i] = E::ld_ks(ln, p + i * PS, LD, k0, col0);
        return f;
    }
    DEVI void st4(int row, int col, f32x4 v) const {
        bf16_t *at = p + lds_off(LD, row, col);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const bf16x4 b = __builtin_convertvector(v, bf16x4);
            *(bf16x4 *)(at + i * PS) = b;
            if (i + 1 < NP) v -= __builtin_convertvector(b, f32x4);
        }
    }
    DEVI f32x4 get4(int row, int col) const {
        const bf16_t *at = p + lds_off(LD, row, col);
        f32x4 v{0, 0, 0, 0};
#pragma unroll
        for (int i = NP - 1; i >= 0; --i) v += __builtin_convertvector(*(const bf16x4 *)(at + i * PS), f32x4);
        return v;
    }
    // an accumulator tile, transposed: its column r is row row0 + r here, its rows are columns col0 ..
    DEVI void st_acc(const Lane &ln, int row0, int col0, const f32x16 &t) const {
#pragma unroll
        for (int g = 0; g < 4; ++g) st4(row0 + ln.r, col0 + 8 * g + 4 * ln.h, f32x4{t[4 * g], t[4 * g + 1], t[4 * g + 2], t[4 * g + 3]});
    }
};

// Rows of a global tensor on their way to a tile: 16 bytes a thread and piece. Rows from `valid` on are zeros.
template <typename T, int ROWS, int WIDTH>
struct Fetch {
    static constexpr int EPC = 16 / sizeof(T), CPR = WIDTH / EPC, N = ROWS * CPR / kThreads;
    static_assert(N * kThreads == ROWS * CPR, "whole pieces");
    u32x4 v[N];
    DEVI void load(const T *base, size_t ld, int valid) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = threadIdx.x + n * kThreads, row = c / CPR, col = (c % CPR) * EPC;
            v[n] = u32x4{0, 0, 0, 0};
            if (row < valid) v[n] = *(const u32x4 *)(base + row * ld + col);
        }
    }
    template <typename F>
    DEVI void each(F f) const {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = threadIdx.x + n * kThreads;
            f(c / CPR, (c % CPR) * EPC, v[n]);
        }
    }
    template <typename Tl>
    DEVI void store(const Tl &t) const {
        each([&](int row, int col, u32x4 x) {
            if constexpr (sizeof(T) == 2) *(u32x4 *)(t.p + lds_off(Tl::LD, row, col)) = x;
            else t.st4(row, col, __builtin_bit_cast(f32x4, x));
        });
    }
    // every row times its weight
    template <typename Tl>
    DEVI void store_scaled(const Tl &t, const float *w) const {
        each([&](int row, int col, u32x4 x) {
            if constexpr (sizeof(T) == 2) {
                const f32x8 f = __builtin_convertvector(__builtin_bit_cast(bf16x8, x), f32x8) * w[row];
                t.st4(row, col, __builtin_shufflevector(f, f, 0, 1, 2, 3));
                t.st4(row, col + 4, __builtin_shufflevector(f, f, 4, 5, 6, 7));
            } else {
                t.st4(row, col, __builtin_bit_cast(f32x4, x) * w[row]);
            }
        });
    }
};
// N of a tile, as k_delta_prep leaves it: its parts one after the other.
template <int NP, int C>
struct FetchParts {
    static constexpr int PIECES = NP * C * C / 8, N = (PIECES + kThreads - 1) / kThreads;
    u32x4 v[N];
    DEVI void load(const bf16_t *base) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = threadIdx.x + n * kThreads;
            if (c < PIECES) v[n] = *(const u32x4 *)(base + c * 8);
        }
    }
    DEVI void store(const Tile<NP, C, C> &t) const {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = threadIdx.x + n * kThreads;
            if (c < PIECES) *(u32x4 *)(t.p + c / (C * C / 8) * Tile<NP, C, C>::PS + c / (C / 8) % C * Tile<NP, C, C>::LD + c % (C / 8) * 8) = v[n];
        }
    }
};

// 16 features of the lane's token in the order of an accumulator tile (p: the token's row at the tile's first feature).
template <typename T>
DEVI f32x16 load_acc(const T *p, const Lane &ln, bool there) {
    f32x16 x = {};
    if (there)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f32x4 v;
            if constexpr (sizeof(T) == 2) v = __builtin_convertvector(*(const bf16x4 *)(p + 8 * g + 4 * ln.h), f32x4);
            else v = *(const f32x4 *)(p + 8 * g + 4 * ln.h);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * g + e] = v[e];
        }
    return x;
}
template <typename T>
DEVI void store_acc(T *p, const Lane &ln, const f32x16 &x) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const f32x4 v{x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]};
        if constexpr (sizeof(T) == 2) *(bf16x4 *)(p + 8 * g + 4 * ln.h) = __builtin_convertvector(v, bf16x4);
        else *(f32x4 *)(p + 8 * g + 4 * ln.h) = v;
    }
}

// The gates of a tile. Logarithms are summed in 64 bits and to base 2: the sum over a tile may be large where a difference is small.
// From 2^-300 on (-infinity among them: the state starts anew) a gate counts as 2^-300, whose power is 0 as a float, so that
// differences of sums stay numbers.
template <int C>
struct Gates {
    double sum[C];
    float start[C], rest[C], beta[C];   // exp(G_i), exp(G_C - G_i)
    float whole;
};
struct GateIn {
    float log_g, beta;
    DEVI void load(const float *lg, const float *b, int valid, int lane) {
        log_g = lg && lane < valid ? lg[lane] : 0.0f;
        beta = lane < valid ? b[lane] : 0.0f;
    }
};
DEVI double to_base2(float log_g) {
    const double x = (double)log_g * 1.4426950408889634;
    return x < -300.0 ? -300.0 : x;   // (NaN stays)
}
template <int C>
DEVI void make_gates(Gates<C> &g, const GateIn &in, int lane) {   // one wave
    double x = to_base2(in.log_g);
#pragma unroll
    for (int d = 1; d < C; d *= 2) {
        const double y = __shfl_up(x, d, C);
        if ((lane & (C - 1)) >= d) x += y;
    }
    const double all = __shfl(x, C - 1, C);
    if (lane < C) {
        g.sum[lane] = x;
        g.start[lane] = __builtin_amdgcn_exp2f((float)x);
        g.rest[lane] = __builtin_amdgcn_exp2f((float)(all - x));
        g.beta[lane] = in.beta;
    }
    if (lane == 0) g.whole = __builtin_amdgcn_exp2f((float)all);
}
DEVI float power(double d) { return __builtin_amdgcn_exp2f((float)d); }

struct DeltaCall {
    int B, H, Hk, N, Dv, tiles, segments, seg_tiles;
    const float *log_g, *beta;
    const int *len;
    // tokens of sequence b from token0 on, 0 .. most
    DEVI int valid(int b, int token0, int most) const {
        const int n = len ? min(max(len[b], 0), N) : N;
        return min(max(n - token0, 0), most);
    }
    DEVI size_t key_row(int b, int h) const { return ((size_t)b * Hk + h / (H / Hk)) * N; }   // first row of a head of q, k
};

// ---------------------------------------------------------------------------
// k_delta_prep: N of a tile. Blocks of 16 by substitution, a thread per column; then joined to twice the size,
//     N21 = -(I + N22 beta) M21 (I + beta N11).
// ---------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void k_delta_prep(const T *__restrict__ K, bf16_t *__restrict__ inv, DeltaCall a) {
    using P = Parts<T>;
    constexpr int C = P::C, LDM = C + 4;
    typedef Tile<P::DATA, C, D> KTile;
    __shared__ __attribute__((aligned(16))) unsigned char lds_k[KTile::BYTES];
    __shared__ __attribute__((aligned(16))) float M[C * LDM], Nn[C * LDM];
    __shared__ Gates<C> g;
    const KTile kt{(bf16_t *)lds_k};
    const Lane ln(threadIdx.x);
    const int wave = threadIdx.x >> 6, tile = blockIdx.x, bh = blockIdx.y, b = bh / a.H, h = bh - b * a.H, token0 = tile * C;
    const int valid = a.valid(b, token0, C);
    Fetch<T, C, D> fk;
    fk.load(K + (a.key_row(b, h) + token0) * D, D, valid);
    if (wave == 0) {
        GateIn in;
        in.load(a.log_g ? a.log_g + (size_t)bh * a.N + token0 : nullptr, a.beta + (size_t)bh * a.N + token0, valid, ln.id);
        make_gates<C>(g, in, ln.id);
    }
    fk.store(kt);
    __syncthreads();
    constexpr int NT = C / 32;
    if (wave < NT * NT && wave % NT <= wave / NT) {
        const int it = wave / NT, jt = wave % NT;
        f32x16 m = {};
#pragma unroll
        for (int k0 = 0; k0 < D; k0 += 16) m = mm<P::MADE>(kt.kc(ln, 32 * it, k0), kt.kc(ln, 32 * jt, k0), m);
        const int j = 32 * jt + ln.r;
        const double gj = g.sum[j];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int i = 32 * it + ln.acc_row(e);
            M[i * LDM + j] = i > j ? m[e] * power(g.sum[i] - gj) : 0.0f;
        }
    }
    for (int c = threadIdx.x; c < C * C; c += kThreads) Nn[c / C * LDM + c % C] = 0.0f;
    __syncthreads();
    if (threadIdx.x < C) {
        const int j = threadIdx.x, b0 = j & ~15, jj = j & 15;
        float n[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float s = M[(b0 + i) * LDM + j];
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if (k < i) s = __builtin_fmaf(M[(b0 + i) * LDM + b0 + k], n[k], s);
            s = i > jj ? -s : 0.0f;
            Nn[(b0 + i) * LDM + j] = s;
            n[i] = s * g.beta[b0 + i];
        }
    }
    __syncthreads();
#pragma unroll
    for (int s = 16; s < C; s *= 2) {
        // pairs of blocks of s rows; 4 columns of a row a thread. First M21 (I + beta N11), in place of N21, then the other factor.
        const int quads = s / 4, jobs = C / (2 * s) * s * quads;
        const int job = threadIdx.x, pair = job / (s * quads), i = job / quads % s, j = 4 * (job % quads), r0 = 2 * s * pair;
        static_assert(C / 2 * C / 8 <= kThreads, "a job a thread");
        f32x4 y = {};
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (job < jobs) {
                const float *m = half ? Nn + (r0 + s + i) * LDM + r0 + s : M + (r0 + s + i) * LDM + r0;
                const float *n0 = half ? Nn + (r0 + s) * LDM + r0 + j : Nn + r0 * LDM + r0 + j;
                const float *bt = g.beta + r0 + (half ? s : 0);
                y = half ? *(const f32x4 *)(n0 + i * LDM) : *(const f32x4 *)(m + j);
#pragma unroll 8
                for (int k = 0; k < s; ++k) y += (m[k] * bt[k]) * *(const f32x4 *)(n0 + k * LDM);
                if (half) y = -y;
            }
            __syncthreads();
            if (job < jobs) *(f32x4 *)(Nn + (r0 + s + i) * LDM + r0 + j) = y;
            __syncthreads();
        }
    }
    bf16_t *to = inv + ((size_t)bh * a.tiles + tile) * (P::MADE * C * C);
    for (int c = threadIdx.x; c < C * C / 4; c += kThreads) {
        const int i = c / (C / 4), j = c % (C / 4) * 4;
        f32x4 v = *(const f32x4 *)(Nn + i * LDM + j);
#pragma unroll
        for (int part = 0; part < P::MADE; ++part) {
            const bf16x4 x = __builtin_convertvector(v, bf16x4);
            *(bf16x4 *)(to + part * C * C + i * C + j) = x;
            v -= __builtin_convertvector(x, f32x4);
        }
    }
}

// Where a wave's accumulator tiles of the state lie: D / 32 by 2 tiles of 32 features of the key by 32 of the value.
template <int D>
struct StatePlace {
    static constexpr int N = D == 128 ? 2 : 1;
    int wave;
    DEVI int key0(int s) const { return 32 * (N == 2 ? wave : wave >> 1); }
    DEVI int col0(int s) const { return 32 * (N == 2 ? s : wave & 1); }
};
template <int D>
DEVI void load_state(f32x16 (&S)[StatePlace<D>::N], const StatePlace<D> &at, const Lane &ln, const float *src, int ld) {
#pragma unroll
    for (int s = 0; s < StatePlace<D>::N; ++s)
#pragma unroll
        for (int e = 0; e < 16; ++e) S[s][e] = src ? src[(size_t)(at.key0(s) + ln.acc_row(e)) * ld + at.col0(s) + ln.r] : 0.0f;
}
template <int D>
DEVI void save_state(const f32x16 (&S)[StatePlace<D>::N], const StatePlace<D> &at, const Lane &ln, float *dst, int ld) {
#pragma unroll
    for (int s = 0; s < StatePlace<D>::N; ++s)
#pragma unroll
        for (int e = 0; e < 16; ++e) dst[(size_t)(at.key0(s) + ln.acc_row(e)) * ld + at.col0(s) + ln.r] = S[s][e];
}

// ---------------------------------------------------------------------------
// k_delta_walk. LOCAL: no outputs; the state a segment reaches from zero, and (column blocks behind those of the values) its
// matrix T, which is the state reached from the identity without values.
// ---------------------------------------------------------------------------
template <typename T, int D>
struct WalkLds {
    using P = Parts<T>;
    static constexpr int C = P::C;
    typedef Tile<P::DATA, C, D> Data;
    typedef Tile<P::MADE, kDeltaCols, D> State;   // transposed: a row per column
    typedef Tile<P::MADE, C, C> Square;
    typedef Tile<P::MADE, C, kDeltaCols> Rows;
    static constexpr int K = 0, S = K + Data::BYTES, NN = S + State::BYTES, X = NN + Square::BYTES, Z = X + Rows::BYTES, G = Z + Rows::BYTES,
                         Q = G + (int)((sizeof(Gates<C>) + 15) / 16 * 16), PP = Q + Data::BYTES, Y = PP + Square::BYTES, ALL = Y + Rows::BYTES;
    static constexpr int bytes(bool local) { return local ? Q : ALL; }
};
struct WalkStates {
    const float *first;   // states that segments start from ([head][segment], or kv_in where there is one segment); null = zeros
    float *last;          // kv_out
    float *local, *trans; // LOCAL
    float *cache;         // the state in front of every tile; may be null
    int all_trans;        // T is wanted of the last segment too
};
template <typename T, int D, bool LOCAL>
__global__ __launch_bounds__(kThreads, 1) void k_delta_walk(const T *__restrict__ Q, const T *__restrict__ K, const T *__restrict__ V,
                                                            const bf16_t *__restrict__ inv, T *__restrict__ O, WalkStates st, DeltaCall a) {
    using P = Parts<T>;
    using L = WalkLds<T, D>;
    constexpr int C = P::C;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const typename L::Data kt{(bf16_t *)(lds + L::K)}, qt{(bf16_t *)(lds + L::Q)};
    const typename L::State stt{(bf16_t *)(lds + L::S)};
    const typename L::Square nt{(bf16_t *)(lds + L::NN)}, pt{(bf16_t *)(lds + L::PP)};
    const typename L::Rows xt{(bf16_t *)(lds + L::X)}, yt{(bf16_t *)(lds + L::Y)}, zt{(bf16_t *)(lds + L::Z)};
    Gates<C> &g = *(Gates<C> *)(lds + L::G);
    const Lane ln(threadIdx.x);
    const int wave = threadIdx.x >> 6;
    const int blocks = a.Dv / kDeltaCols + (LOCAL ? D / kDeltaCols : 0);
    const int cb = blockIdx.x % blocks, seg = blockIdx.x / blocks % a.segments, bh = blockIdx.x / (blocks * a.segments);
    const int b = bh / a.H, h = bh - b * a.H;
    const bool trans = LOCAL && cb >= a.Dv / kDeltaCols;
    const int c0 = trans ? (cb - a.Dv / kDeltaCols) * kDeltaCols : cb * kDeltaCols;
    if (LOCAL && seg == a.segments - 1 && !(trans && st.all_trans)) return;
    const int t0 = seg * a.seg_tiles, t1 = min(a.tiles, t0 + a.seg_tiles);
    const size_t key_row = a.key_row(b, h), row = (size_t)bh * a.N;
    const int ct = wave & 1, tt = wave >> 1;          // this wave's block of 32 columns and 32 tokens
    const bool active = tt < C / 32;
    const StatePlace<D> at{wave};
    f32x16 S[StatePlace<D>::N];
    if (trans) {
#pragma unroll
        for (int s = 0; s < StatePlace<D>::N; ++s)
#pragma unroll
            for (int e = 0; e < 16; ++e) S[s][e] = at.key0(s) + ln.acc_row(e) == c0 + at.col0(s) + ln.r ? 1.0f : 0.0f;
    } else {
        const float *from = LOCAL || !st.first ? nullptr : st.first + ((size_t)bh * a.segments + seg) * D * a.Dv + c0;
        load_state<D>(S, at, ln, from, a.Dv);
    }
#pragma unroll
    for (int s = 0; s < StatePlace<D>::N; ++s) stt.st_acc(ln, at.col0(s), at.key0(s), S[s]);

    Fetch<T, C, D> fk, fq;
    FetchParts<P::MADE, C> fn;
    f32x16 v = {};
    GateIn gi{0.0f, 0.0f};
    auto fetch = [&](int t) {
        const int token0 = t * C, valid = a.valid(b, token0, C);
        fk.load(K + (key_row + token0) * D, D, valid);
        if constexpr (!LOCAL) fq.load(Q + (key_row + token0) * D, D, valid);
        fn.load(inv + ((size_t)bh * a.tiles + t) * (P::MADE * C * C));
        const int i = 32 * tt + ln.r;
        if (active && !trans) v = load_acc(V + (row + token0 + i) * a.Dv + c0 + 32 * ct, ln, i < valid);
        if (wave == 0) gi.load(a.log_g ? a.log_g + row + token0 : nullptr, a.beta + row + token0, valid, ln.id);
    };
    fetch(t0);
    for (int t = t0; t < t1; ++t) {
        const int token0 = t * C, i = 32 * tt + ln.r;
        fk.store(kt);
        if constexpr (!LOCAL) fq.store(qt);
        fn.store(nt);
        if (wave == 0) make_gates<C>(g, gi, ln.id);
        const f32x16 vt = v;
        __syncthreads();
        if (t + 1 < t1) fetch(t + 1);
        if (!LOCAL && st.cache) save_state<D>(S, at, ln, st.cache + ((size_t)bh * a.tiles + t) * D * a.Dv + c0, a.Dv);
        f32x16 r = {}, o = {};
        float beta = 0.0f, start = 0.0f, rest = 0.0f;
        if (active) {
            beta = g.beta[i];
            start = g.start[i];
            rest = g.rest[i];
#pragma unroll
            for (int k0 = 0; k0 < D; k0 += 16) {
                const auto s = stt.kc(ln, 32 * ct, k0);
                r = mm<P::MADE>(s, kt.kc(ln, 32 * tt, k0), r);
                if constexpr (!LOCAL) o = mm<P::MADE>(s, qt.kc(ln, 32 * tt, k0), o);
            }
            f32x16 x;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                r[e] = vt[e] - start * r[e];
                x[e] = beta * r[e];
            }
            xt.st_acc(ln, 32 * tt, 32 * ct, x);
            if constexpr (!LOCAL) {
                o *= start;
                if (ct <= tt) {   // scores of the tokens of block ct with this one's
                    f32x16 p = {};
#pragma unroll
                    for (int k0 = 0; k0 < D; k0 += 16) p = mm<P::MADE>(kt.kc(ln, 32 * ct, k0), qt.kc(ln, 32 * tt, k0), p);
                    const double gs = g.sum[i];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int j = 32 * ct + ln.acc_row(e);
                        p[e] = j <= i ? p[e] * power(gs - g.sum[j]) : 0.0f;
                    }
                    pt.st_acc(ln, 32 * tt, 32 * ct, p);
                }
            }
        }
        __syncthreads();
        if (active) {
            for (int k0 = 0; k0 < 32 * (tt + 1); k0 += 16) r = mm<P::MADE>(xt.ks(ln, k0, 32 * ct), nt.kc(ln, 32 * tt, k0), r);
            r *= beta;
            if constexpr (!LOCAL) yt.st_acc(ln, 32 * tt, 32 * ct, r);
            r *= rest;
            zt.st_acc(ln, 32 * tt, 32 * ct, r);
        }
        __syncthreads();
        if constexpr (!LOCAL)
            if (active) {
                for (int k0 = 0; k0 < 32 * (tt + 1); k0 += 16) o = mm<P::MADE>(yt.ks(ln, k0, 32 * ct), pt.kc(ln, 32 * tt, k0), o);
                if (token0 + i < a.N) store_acc(O + (row + token0 + i) * a.Dv + c0 + 32 * ct, ln, o);
            }
        const float whole = g.whole;
#pragma unroll
        for (int s = 0; s < StatePlace<D>::N; ++s) {
            S[s] *= whole;
#pragma unroll
            for (int k0 = 0; k0 < C; k0 += 16) S[s] = mm<P::MADE>(kt.ks(ln, k0, at.key0(s)), zt.ks(ln, k0, at.col0(s)), S[s]);
            stt.st_acc(ln, at.col0(s), at.key0(s), S[s]);
        }
        __syncthreads();
    }
    if constexpr (LOCAL) {
        if (trans) save_state<D>(S, at, ln, st.trans + ((size_t)bh * a.segments + seg) * D * D + c0, D);
        else save_state<D>(S, at, ln, st.local + ((size_t)bh * a.segments + seg) * D * a.Dv + c0, a.Dv);
    } else if (seg == a.segments - 1) {
        save_state<D>(S, at, ln, st.last + (size_t)bh * D * a.Dv + c0, a.Dv);
    }
}

// ---------------------------------------------------------------------------
// k_delta_scan: first[0] = in, first[p + 1] = T_p first[p] + local[p]; BACK: last[P - 1] = in, last[p - 1] = T_p^T last[p] + local[p].
// 16 columns a workgroup, in float.
// ---------------------------------------------------------------------------
constexpr int kScanCols = 16;
template <int D, bool BACK>
__global__ __launch_bounds__(kThreads) void k_delta_scan(const float *__restrict__ in, const float *__restrict__ trans, const float *__restrict__ local,
                                                         float *__restrict__ states, int Dv, int segments) {
    __shared__ __attribute__((aligned(16))) float S[D][kScanCols];
    constexpr int PER = D * kScanCols / kThreads, TPR = kScanCols / PER;   // columns a thread takes of one row
    const int bh = blockIdx.y, c0 = blockIdx.x * kScanCols, d = threadIdx.x / TPR, c = threadIdx.x % TPR * PER;
    float x[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) x[e] = in ? in[((size_t)bh * D + d) * Dv + c0 + c + e] : 0.0f;
    for (int step = 0; step < segments; ++step) {
        const int p = BACK ? segments - 1 - step : step;
        const size_t at = (((size_t)bh * segments + p) * D + d) * Dv + c0 + c;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            states[at + e] = x[e];
            S[d][c + e] = x[e];
        }
        if (step + 1 == segments) break;
        __syncthreads();
        const float *m = trans + ((size_t)bh * segments + p) * D * D;
#pragma unroll
        for (int e = 0; e < PER; ++e) x[e] = local[at + e];
#pragma unroll 8
        for (int k = 0; k < D; ++k) {
            const float w = BACK ? m[(size_t)k * D + d] : m[(size_t)d * D + k];
#pragma unroll
            for (int e = 0; e < PER; ++e) x[e] = __builtin_fmaf(w, S[k][c + e], x[e]);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// k_delta_step: COLS columns of a head's state in the registers of 256 threads, four columns by some rows apiece. One reduction a token:
//     S^T k, S^T q and q . k of the state as it was give u = beta (v - a S^T k) and out = a S^T q + (q . k) u.
// ---------------------------------------------------------------------------
template <typename T, int D, int COLS>
__global__ __launch_bounds__(kThreads) void k_delta_step(const T *__restrict__ Q, const T *__restrict__ K, const T *__restrict__ V, const float *kv_in,
                                                         T *__restrict__ O, float *kv_out, DeltaCall a) {
    constexpr int QUADS = COLS / 4, GROUPS = kThreads / QUADS, ROWS = D / GROUPS;   // row groups; rows of a thread: d = group + GROUPS n
    __shared__ float red[2][kWaves][QUADS][9];
    const int quad = threadIdx.x % QUADS, group = threadIdx.x / QUADS, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int blocks = a.Dv / COLS, cb = blockIdx.x % blocks, bh = blockIdx.x / blocks, b = bh / a.H, h = bh - b * a.H;
    const int c = cb * COLS + 4 * quad;
    const size_t state = (size_t)bh * D * a.Dv + c, row = (size_t)bh * a.N;
    const T *q = Q + a.key_row(b, h) * D, *k = K + a.key_row(b, h) * D, *v = V + row * a.Dv + c;
    T *o = O + row * a.Dv + c;
    const int n = a.valid(b, 0, a.N);
    f32x4 S[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) S[r] = kv_in ? *(const f32x4 *)(kv_in + state + (size_t)(group + GROUPS * r) * a.Dv) : f32x4{0, 0, 0, 0};
    auto four = [](const T *p) {
        if constexpr (sizeof(T) == 2) return __builtin_convertvector(*(const bf16x4 *)p, f32x4);
        else return *(const f32x4 *)p;
    };
    auto put4 = [](T *p, f32x4 x) {
        if constexpr (sizeof(T) == 2) *(bf16x4 *)p = __builtin_convertvector(x, bf16x4);
        else *(f32x4 *)p = x;
    };
    for (int s = 0; s < n; ++s) {
        float kd[ROWS], qd[ROWS], sums[9] = {};
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            kd[r] = Elem<T>::ld1(k + (size_t)s * D + group + GROUPS * r);
            qd[r] = Elem<T>::ld1(q + (size_t)s * D + group + GROUPS * r);
        }
        const f32x4 vs = four(v + (size_t)s * a.Dv);
        const float beta = a.beta[row + s], lg = a.log_g ? a.log_g[row + s] : 0.0f;
        const float gate = power(to_base2(lg));
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sums[e] = __builtin_fmaf(kd[r], S[r][e], sums[e]);
                sums[4 + e] = __builtin_fmaf(qd[r], S[r][e], sums[4 + e]);
            }
            sums[8] = __builtin_fmaf(kd[r], qd[r], sums[8]);
        }
#pragma unroll
        for (int d = QUADS; d < 64; d *= 2)
#pragma unroll
            for (int e = 0; e < 9; ++e) sums[e] += __shfl_xor(sums[e], d);
        auto &to = red[s & 1];
        if (lane < QUADS)
#pragma unroll
            for (int e = 0; e < 9; ++e) to[wave][lane][e] = sums[e];
        __syncthreads();   // (one a token: the next one writes the other half)
#pragma unroll
        for (int e = 0; e < 9; ++e) sums[e] = (to[0][quad][e] + to[1][quad][e]) + (to[2][quad][e] + to[3][quad][e]);
        f32x4 u, out;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            u[e] = beta * __builtin_fmaf(-gate, sums[e], vs[e]);
            out[e] = __builtin_fmaf(sums[8], u[e], gate * sums[4 + e]);
        }
        if (group == 0) put4(o + (size_t)s * a.Dv, out);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) S[r] = gate * S[r] + kd[r] * u;
    }
    for (int s = n + group; s < a.N; s += GROUPS) put4(o + (size_t)s * a.Dv, f32x4{0, 0, 0, 0});
#pragma unroll
    for (int r = 0; r < ROWS; ++r) *(f32x4 *)(kv_out + state + (size_t)(group + GROUPS * r) * a.Dv) = S[r];
}

// ---------------------------------------------------------------------------
// k_delta_back: the walk in reverse. LOCAL: the gradient that reaches a segment's front from its own tokens.
// ---------------------------------------------------------------------------
template <typename T, int D>
struct BackLds {
    using P = Parts<T>;
    static constexpr int C = P::C;
    typedef Tile<P::DATA, C, D> Data;
    typedef Tile<P::MADE, kDeltaCols, D> State;   // transposed
    typedef Tile<P::MADE, C, C> Square;
    typedef Tile<P::MADE, C, kDeltaCols> Rows;
    typedef Tile<P::DATA, C, kDeltaCols> Grad;
    static constexpr int GATES = (int)((sizeof(Gates<C>) + 15) / 16 * 16);
    static constexpr int K = 0, Q = K + Data::BYTES, S = Q + Data::BYTES, DO = S + State::BYTES, GO = DO + Grad::BYTES, NN = GO + Rows::BYTES,
                         X = NN + Square::BYTES, PP = X + Rows::BYTES, G = PP + (Rows::BYTES > Square::BYTES ? Rows::BYTES : Square::BYTES),
                         ALL = G + 2 * GATES;
    static_assert(ALL <= 163840, "LDS of a CU");
};
struct BackStates {
    const float *last;   // gradients of the states segments end with ([head][segment], or dkv_out where there is one segment); null = zeros
    float *first;        // dkv_in
    float *local;        // LOCAL
    float *grads;        // the gradient of the state behind every tile
    float *dr;           // [B][H][N][Dv]
};
template <typename T, int D, bool LOCAL>
__global__ __launch_bounds__(kThreads, 1) void k_delta_back(const T *__restrict__ Q, const T *__restrict__ K, const T *__restrict__ dO,
                                                            const bf16_t *__restrict__ inv, T *__restrict__ dV, BackStates st, DeltaCall a) {
    using P = Parts<T>;
    using L = BackLds<T, D>;
    constexpr int C = P::C;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const typename L::Data kt{(bf16_t *)(lds + L::K)}, qt{(bf16_t *)(lds + L::Q)};
    const typename L::State stt{(bf16_t *)(lds + L::S)};
    const typename L::Square nt{(bf16_t *)(lds + L::NN)}, pt{(bf16_t *)(lds + L::PP)};   // pt: [key token][query token]
    const typename L::Rows xt{(bf16_t *)(lds + L::X)}, gt{(bf16_t *)(lds + L::GO)}, zt{(bf16_t *)(lds + L::PP)};
    const typename L::Grad dot{(bf16_t *)(lds + L::DO)};
    auto gates = [&](int t) -> Gates<C> & { return *(Gates<C> *)(lds + L::G + (t & 1) * L::GATES); };
    const Lane ln(threadIdx.x);
    const int wave = threadIdx.x >> 6;
    const int blocks = a.Dv / kDeltaCols, c0 = blockIdx.x % blocks * kDeltaCols, seg = blockIdx.x / blocks % a.segments;
    const int bh = blockIdx.x / (blocks * a.segments), b = bh / a.H, h = bh - b * a.H;
    if (LOCAL && seg == 0) return;
    const int t0 = seg * a.seg_tiles, t1 = min(a.tiles, t0 + a.seg_tiles);
    const size_t key_row = a.key_row(b, h), row = (size_t)bh * a.N;
    const int ct = wave & 1, jt = wave >> 1;   // this wave's block of 32 columns and 32 tokens
    const bool active = jt < C / 32;
    const StatePlace<D> at{wave};
    f32x16 S[StatePlace<D>::N];
    load_state<D>(S, at, ln, LOCAL || !st.last ? nullptr : st.last + ((size_t)bh * a.segments + seg) * D * a.Dv + c0, a.Dv);
#pragma unroll
    for (int s = 0; s < StatePlace<D>::N; ++s) stt.st_acc(ln, at.col0(s), at.key0(s), S[s]);

    Fetch<T, C, D> fk, fq;
    Fetch<T, C, kDeltaCols> fo;
    FetchParts<P::MADE, C> fn;
    GateIn gi{0.0f, 0.0f};
    auto fetch = [&](int t) {
        const int token0 = t * C, valid = a.valid(b, token0, C);
        fk.load(K + (key_row + token0) * D, D, valid);
        fq.load(Q + (key_row + token0) * D, D, valid);
        fo.load(dO + (row + token0) * a.Dv + c0, a.Dv, valid);
        fn.load(inv + ((size_t)bh * a.tiles + t) * (P::MADE * C * C));
        if (wave == 0) gi.load(a.log_g ? a.log_g + row + token0 : nullptr, a.beta + row + token0, valid, ln.id);
    };
    fetch(t1 - 1);
    if (wave == 0) make_gates<C>(gates(t1 - 1), gi, ln.id);
    __syncthreads();
    for (int t = t1 - 1; t >= t0; --t) {
        const int token0 = t * C, j = 32 * jt + ln.r;
        const Gates<C> &g = gates(t);
        fk.store(kt);
        fq.store(qt);
        fo.store(dot);
        fo.store_scaled(gt, g.start);
        fn.store(nt);
        __syncthreads();
        if (t > t0) fetch(t - 1);
        if (!LOCAL) save_state<D>(S, at, ln, st.grads + ((size_t)bh * a.tiles + t) * D * a.Dv + c0, a.Dv);
        f32x16 du = {};
        float beta = 0.0f, start = 0.0f;
        if (active) {
            beta = g.beta[j];
            start = g.start[j];
#pragma unroll
            for (int k0 = 0; k0 < D; k0 += 16) du = mm<P::MADE>(stt.kc(ln, 32 * ct, k0), kt.kc(ln, 32 * jt, k0), du);
            du *= g.rest[j];
            // scores of block `qb` of queries with this block of keys: the two waves of a block of keys take one each
            const int qb = C == 32 ? 0 : ct;
            if (qb >= jt && (C > 32 || ct == 0)) {
                f32x16 p = {};
#pragma unroll
                for (int k0 = 0; k0 < D; k0 += 16) p = mm<P::MADE>(qt.kc(ln, 32 * qb, k0), kt.kc(ln, 32 * jt, k0), p);
                const double gj = g.sum[j];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int i = 32 * qb + ln.acc_row(e);
                    p[e] = i >= j ? p[e] * power(g.sum[i] - gj) : 0.0f;
                }
                pt.st_acc(ln, 32 * jt, 32 * qb, p);
            }
        }
        __syncthreads();
        if (active) {
            for (int k0 = 32 * jt; k0 < C; k0 += 16) du = mm<P::MADE>(dot.ks(ln, k0, 32 * ct), pt.kc(ln, 32 * jt, k0), du);
            xt.st_acc(ln, 32 * jt, 32 * ct, du * beta);
        }
        __syncthreads();
        if (active) {
            for (int k0 = 32 * jt; k0 < C; k0 += 16) du = mm<P::MADE>(xt.ks(ln, k0, 32 * ct), nt.ks(ln, k0, 32 * jt), du);
            const f32x16 dv = du * beta;
            if (!LOCAL && token0 + j < a.N) {
                store_acc(st.dr + (row + token0 + j) * a.Dv + c0 + 32 * ct, ln, du);
                store_acc(dV + (row + token0 + j) * a.Dv + c0 + 32 * ct, ln, dv);
            }
            zt.st_acc(ln, 32 * jt, 32 * ct, dv * -start);   // (in the scores' place: every wave is past them)
        }
        const float whole = g.whole;
        if (t > t0 && wave == 0) make_gates<C>(gates(t - 1), gi, ln.id);
        __syncthreads();
#pragma unroll
        for (int s = 0; s < StatePlace<D>::N; ++s) {
            S[s] *= whole;
#pragma unroll
            for (int k0 = 0; k0 < C; k0 += 16) {
                S[s] = mm<P::MADE>(qt.ks(ln, k0, at.key0(s)), gt.ks(ln, k0, at.col0(s)), S[s]);
                S[s] = mm<P::MADE>(kt.ks(ln, k0, at.key0(s)), zt.ks(ln, k0, at.col0(s)), S[s]);
            }
            stt.st_acc(ln, at.col0(s), at.key0(s), S[s]);
        }
        __syncthreads();
    }
    if (LOCAL) save_state<D>(S, at, ln, st.local + ((size_t)bh * a.segments + seg) * D * a.Dv + c0, a.Dv);
    else if (seg == 0) save_state<D>(S, at, ln, st.first + (size_t)bh * D * a.Dv + c0, a.Dv);
}

// ---------------------------------------------------------------------------
// k_delta_grad: a tile's gradients, from the state in front of it and the gradient of the one behind it, 64 value features at a time.
// ---------------------------------------------------------------------------
template <typename T, int D>
struct GradLds {
    using P = Parts<T>;
    static constexpr int C = P::C;
    typedef Tile<P::DATA, C, D> Data;
    typedef Tile<P::MADE, D, kDeltaCols> State;
    typedef Tile<P::MADE, C, C> Square;
    typedef Tile<P::MADE, C, kDeltaCols> Rows;
    typedef Tile<P::DATA, C, kDeltaCols> Grad;
    static_assert(Square::BYTES <= Rows::BYTES, "Ep and Em take the places of rows");
    static constexpr int K = 0, Q = K + Data::BYTES, S = Q + Data::BYTES, DO = S + State::BYTES, NN = DO + Grad::BYTES, X = NN + Square::BYTES,
                         Y = X + Rows::BYTES, G = Y + Rows::BYTES, RED = G + (int)((sizeof(Gates<C>) + 15) / 16 * 16),
                         ALL = RED + kWaves * (3 * C + 4) * 4;
    static_assert(ALL <= 163840, "LDS of a CU");
};
template <typename T, int D, typename TO>
__global__ __launch_bounds__(kThreads, 1) void k_delta_grad(const T *__restrict__ Q, const T *__restrict__ K, const T *__restrict__ V,
                                                            const T *__restrict__ dO, const bf16_t *__restrict__ inv, const float *__restrict__ states,
                                                            const float *__restrict__ grads, const float *__restrict__ dR, TO *__restrict__ dQ,
                                                            TO *__restrict__ dK, float *__restrict__ dbeta, float *__restrict__ dlog_g, DeltaCall a) {
    using P = Parts<T>;
    using L = GradLds<T, D>;
    constexpr int C = P::C, KEY_BLOCKS = D / 32, BLOCKS = KEY_BLOCKS * (C / 32), PER = BLOCKS > kWaves ? BLOCKS / kWaves : 1;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const typename L::Data kt{(bf16_t *)(lds + L::K)}, qt{(bf16_t *)(lds + L::Q)};
    const typename L::State stt{(bf16_t *)(lds + L::S)};
    const typename L::Square nt{(bf16_t *)(lds + L::NN)}, ep{(bf16_t *)(lds + L::X)}, em{(bf16_t *)(lds + L::Y)};
    const typename L::Rows xt{(bf16_t *)(lds + L::X)}, yt{(bf16_t *)(lds + L::Y)};
    const typename L::Grad dot{(bf16_t *)(lds + L::DO)};
    Gates<C> &g = *(Gates<C> *)(lds + L::G);
    float(*red)[3 * C + 4] = (float(*)[3 * C + 4])(lds + L::RED);
    const Lane ln(threadIdx.x);
    const int wave = threadIdx.x >> 6, tile = blockIdx.x, bh = blockIdx.y, b = bh / a.H, h = bh - b * a.H, token0 = tile * C;
    const int valid = a.valid(b, token0, C);
    const size_t key_row = a.key_row(b, h), row = (size_t)bh * a.N;
    const int ct = wave & 1, tt = wave >> 1, i = 32 * tt + ln.r;     // block of 32 columns and 32 tokens
    const bool active = tt < C / 32;
    const int tk = wave * PER / KEY_BLOCKS, m = 32 * tk + ln.r;      // token block of the accumulators of dQ and dK
    auto key0 = [&](int s) { return (wave * PER + s) % KEY_BLOCKS * 32; };
    const bool active_k = wave * PER < BLOCKS;

    Fetch<T, C, D> fk, fq;
    fk.load(K + (key_row + token0) * D, D, valid);
    fq.load(Q + (key_row + token0) * D, D, valid);
    if (wave == 0) {
        GateIn gi;
        gi.load(a.log_g ? a.log_g + row + token0 : nullptr, a.beta + row + token0, valid, ln.id);
        make_gates<C>(g, gi, ln.id);
    }
    fk.store(kt);
    fq.store(qt);
    for (int e = threadIdx.x; e < kWaves * (3 * C + 4); e += kThreads) ((float *)red)[e] = 0.0f;

    f32x16 ap = {}, am = {};                          // dO U^T, dV U^T
    f32x16 aq[PER] = {}, a1[PER] = {}, a2[PER] = {};  // S dO, S dV, dS U (a row per key feature)
    float sum_b = 0.0f, sum_v = 0.0f, both = 0.0f;    // dR . w and V . dV of the lane's token, <dS, S>
    for (int c0 = 0; c0 < a.Dv; c0 += kDeltaCols) {
        const size_t state = ((size_t)bh * a.tiles + tile) * D * a.Dv + c0;
        Fetch<float, D, kDeltaCols> fs, fd;
        Fetch<T, C, kDeltaCols> fo;
        FetchParts<P::MADE, C> fn;
        fs.load(states + state, a.Dv, D);
        fo.load(dO + (row + token0) * a.Dv + c0, a.Dv, valid);
        fn.load(inv + ((size_t)bh * a.tiles + tile) * (P::MADE * C * C));
        f32x16 v = {}, dr = {};
        if (active) {
            v = load_acc(V + (row + token0 + i) * a.Dv + c0 + 32 * ct, ln, i < valid);
            dr = load_acc(dR + (row + token0 + i) * a.Dv + c0 + 32 * ct, ln, i < valid);
        }
        if (c0 > 0) __syncthreads();
        fs.store(stt);
        fo.store(dot);
        fn.store(nt);
        __syncthreads();
        fd.load(grads + state, a.Dv, D);
        f32x16 r = {};
        float beta = 0.0f;
        if (active) {
            beta = g.beta[i];
            const float start = g.start[i];
#pragma unroll
            for (int k0 = 0; k0 < D; k0 += 16) r = mm<P::MADE>(stt.ks(ln, k0, 32 * ct), kt.kc(ln, 32 * tt, k0), r);
            r = v - start * r;
            xt.st_acc(ln, 32 * tt, 32 * ct, r * beta);
        }
        __syncthreads();
        f32x16 dv = {};
        if (active) {
            for (int k0 = 0; k0 < 32 * (tt + 1); k0 += 16) r = mm<P::MADE>(xt.ks(ln, k0, 32 * ct), nt.kc(ln, 32 * tt, k0), r);
            dv = dr * beta;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                sum_b = __builtin_fmaf(dr[e], r[e], sum_b);
                sum_v = __builtin_fmaf(dv[e], v[e], sum_v);
            }
        }
        __syncthreads();
        if (active) {
            xt.st_acc(ln, 32 * tt, 32 * ct, dv);
            yt.st_acc(ln, 32 * tt, 32 * ct, r * beta);
        }
        __syncthreads();
        if (active && ct <= tt && ct < C / 32)   // (as block of key tokens here)
#pragma unroll
            for (int k0 = 0; k0 < kDeltaCols; k0 += 16) {
                const auto u = yt.kc(ln, 32 * ct, k0);
                ap = mm<P::MADE>(u, dot.kc(ln, 32 * tt, k0), ap);
                am = mm<P::MADE>(u, xt.kc(ln, 32 * tt, k0), am);
            }
        if (active_k)
#pragma unroll
            for (int s = 0; s < PER; ++s)
#pragma unroll
                for (int k0 = 0; k0 < kDeltaCols; k0 += 16) {
                    const auto x = stt.kc(ln, key0(s), k0);
                    aq[s] = mm<P::MADE>(x, dot.kc(ln, 32 * tk, k0), aq[s]);
                    a1[s] = mm<P::MADE>(x, xt.kc(ln, 32 * tk, k0), a1[s]);
                }
        __syncthreads();
        fd.store(stt);
#pragma unroll
        for (int n = 0; n < Fetch<float, D, kDeltaCols>::N; ++n) {
            const f32x4 x = __builtin_bit_cast(f32x4, fs.v[n]), y = __builtin_bit_cast(f32x4, fd.v[n]);
#pragma unroll
            for (int e = 0; e < 4; ++e) both = __builtin_fmaf(x[e], y[e], both);
        }
        __syncthreads();
        if (active_k)
#pragma unroll
            for (int s = 0; s < PER; ++s)
#pragma unroll
                for (int k0 = 0; k0 < kDeltaCols; k0 += 16) a2[s] = mm<P::MADE>(stt.kc(ln, key0(s), k0), yt.kc(ln, 32 * tk, k0), a2[s]);
    }
    __syncthreads();
    if (active && ct <= tt && ct < C / 32) {
        const double gi = g.sum[i];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int j = 32 * ct + ln.acc_row(e);
            const float w = j <= i ? power(gi - g.sum[j]) : 0.0f;
            ap[e] *= w;
            am[e] *= j < i ? -w : 0.0f;
        }
        ep.st_acc(ln, 32 * tt, 32 * ct, ap);
        em.st_acc(ln, 32 * tt, 32 * ct, am);
    }
    __syncthreads();
    float sum_q = 0.0f, phi = g.whole * both;
    if (active_k) {
        const float start = g.start[m], rest = g.rest[m];
        const bool there = token0 + m < a.N;
        const size_t to = (row + token0 + m) * D;   // (shared heads: a partial sum for every state, in float)
#pragma unroll
        for (int s = 0; s < PER; ++s) {
            const int d0 = key0(s);
            f32x16 x = aq[s] * start;
            for (int k0 = 0; k0 < 32 * (tk + 1); k0 += 16) x = mm<P::MADE>(kt.ks(ln, k0, d0), ep.kc(ln, 32 * tk, k0), x);
            f32x16 y = a2[s] * rest;
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const f32x4 q4 = qt.get4(m, d0 + 8 * f + 4 * ln.h), k4 = kt.get4(m, d0 + 8 * f + 4 * ln.h);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    sum_q = __builtin_fmaf(q4[e], x[4 * f + e], sum_q);
                    phi = __builtin_fmaf(k4[e], y[4 * f + e], phi);
                }
            }
            if (there) store_acc(dQ + to + d0, ln, x);
            y -= a1[s] * start;
            for (int k0 = 32 * tk; k0 < C; k0 += 16) {
                y = mm<P::MADE>(qt.ks(ln, k0, d0), ep.ks(ln, k0, 32 * tk), y);
                y = mm<P::MADE>(kt.ks(ln, k0, d0), em.ks(ln, k0, 32 * tk), y);
            }
            for (int k0 = 0; k0 < 32 * (tk + 1); k0 += 16) y = mm<P::MADE>(kt.ks(ln, k0, d0), em.kc(ln, 32 * tk, k0), y);
            if (there) store_acc(dK + to + d0, ln, y);
        }
    }
    sum_b += __shfl_xor(sum_b, 32);
    sum_v += __shfl_xor(sum_v, 32);
    sum_q += __shfl_xor(sum_q, 32);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) phi += __shfl_xor(phi, d);
    if (ln.h == 0) {
        if (active) {
            red[wave][i] = sum_b;
            red[wave][C + i] = sum_v;
        }
        if (active_k) red[wave][2 * C + m] = sum_q;
    }
    if (ln.id == 0) red[wave][3 * C] = phi;
    __syncthreads();
    if (wave != 0) return;
    double x = 0.0, all = 0.0;
    float db = 0.0f;
    if (ln.id < C)
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            db += red[w][ln.id];
            x += (double)red[w][2 * C + ln.id] - (double)red[w][C + ln.id];
        }
#pragma unroll
    for (int w = 0; w < kWaves; ++w) all += red[w][3 * C];
#pragma unroll
    for (int d = 1; d < C; d *= 2) {
        const double y = __shfl_down(x, d, C);
        if ((ln.id & (C - 1)) + d < C) x += y;
    }
    if (ln.id < C && token0 + ln.id < a.N) {
        dbeta[row + token0 + ln.id] = db;
        if (dlog_g) {
            const bool none = ln.id >= valid || to_base2(a.log_g[row + token0 + ln.id]) <= -150.0;   // (a gate of 0 has no slope)
            dlog_g[row + token0 + ln.id] = none ? 0.0f : (float)(all + x);
        }
    }
}

// k_delta_group: dq and dk of a head that several states share, from a partial sum of each. 16 bytes of floats a thread.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void k_delta_group(const float *__restrict__ part, T *__restrict__ dQ, T *__restrict__ dK, size_t per_tensor,
                                                          int share, int N) {
    const size_t n4 = per_tensor / share / 4, at = (size_t)blockIdx.x * kThreads + threadIdx.x, head = (size_t)N * D / 4;
    if (at >= n4) return;
    const float *p = part + (blockIdx.y ? per_tensor : 0);
    const size_t hk = at / head, in = at - hk * head;
    f32x4 s{0, 0, 0, 0};
    for (int e = 0; e < share; ++e) s += *(const f32x4 *)(p + ((hk * share + e) * head + in) * 4);
    T *to = (blockIdx.y ? dK : dQ) + at * 4;
    if constexpr (sizeof(T) == 2) *(bf16x4 *)to = __builtin_convertvector(s, bf16x4);
    else *(f32x4 *)to = s;
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
constexpr int kCus = 256;

size_t up(size_t n) { return (n + 255) / 256 * 256; }

struct Layout {   // byte offsets
    size_t states, inv, trans, cache;                               // cache
    size_t own_inv, own_trans, local, first, scratch;               // forward scratch
    size_t grads, dr, back_local, last, part, back_scratch;         // backward scratch
};
Layout layout(const DeltaPlan &p) {
    Layout l{};
    const size_t bh = (size_t)p.B * p.H, state = (size_t)p.D * p.Dv * 4, made = p.dtype == 0 ? Parts<float>::MADE : Parts<bf16_t>::MADE;
    const size_t inv = bh * p.tiles * made * p.tile * p.tile * 2, between = p.segments > 1 ? bh * p.segments * state : 0;
    const size_t trans = p.segments > 1 ? bh * p.segments * p.D * p.D * 4 : 0;
    l.inv = up(bh * p.tiles * state);
    l.trans = l.inv + up(inv);
    l.cache = l.trans + up(trans);
    l.own_trans = up(inv);
    l.local = l.own_trans + up(trans);
    l.first = l.local + up(between);
    l.scratch = l.first + up(between);
    l.dr = up(bh * p.tiles * state);
    l.back_local = l.dr + up(bh * p.N * p.Dv * 4);
    l.last = l.back_local + up(between);
    l.part = l.last + up(between);
    l.back_scratch = l.part + (p.key_heads < p.H ? 2 * up(bh * p.N * p.D * 4) : 0);
    return l;
}
DeltaCall call_of(const DeltaPlan &p, const DeltaArgs &a) {
    return {p.B, p.H, p.key_heads, p.N, p.Dv, p.tiles, p.segments, p.seg_tiles, a.log_g, a.beta, a.len};
}
// f.template operator()<T, D>()
template <typename F>
hipError_t by_type(const DeltaPlan &p, F f) {
    if (p.dtype == 0) return p.D == 128 ? f.template operator()<float, 128>() : f.template operator()<float, 64>();
    return p.D == 128 ? f.template operator()<bf16_t, 128>() : f.template operator()<bf16_t, 64>();
}
template <typename K>
hipError_t room(K kernel, size_t bytes) { return allow_dynamic_lds((const void *)kernel, bytes); }

struct Forward {
    const DeltaPlan &p;
    const DeltaArgs &a;
    hipStream_t s;
    template <typename T, int D>
    hipError_t operator()() const {
        const DeltaCall c = call_of(p, a);
        const int bh = p.B * p.H;
        const T *q = (const T *)a.q, *k = (const T *)a.k, *v = (const T *)a.v;
        if (!a.cache && p.N <= kDeltaStepTokens) {
            // narrower blocks of columns where 32 would not give every CU two workgroups
            if (bh * (p.Dv / 32) >= 2 * kCus)
                k_delta_step<T, D, 32><<<dim3(bh * (p.Dv / 32)), dim3(kThreads), 0, s>>>(q, k, v, a.kv_in, (T *)a.out, a.kv_out, c);
            else
                k_delta_step<T, D, 16><<<dim3(bh * (p.Dv / 16)), dim3(kThreads), 0, s>>>(q, k, v, a.kv_in, (T *)a.out, a.kv_out, c);
            return hipGetLastError();
        }
        const Layout l = layout(p);
        char *sc = (char *)a.scratch, *ca = (char *)a.cache;
        bf16_t *inv = (bf16_t *)(ca ? ca + l.inv : sc);
        float *trans = (float *)(ca ? ca + l.trans : sc + l.own_trans), *local = (float *)(sc + l.local), *first = (float *)(sc + l.first);
        k_delta_prep<T, D><<<dim3(p.tiles, bh), dim3(kThreads), 0, s>>>(k, inv, c);
        const int blocks = p.Dv / kDeltaCols;
        typedef WalkLds<T, D> L;
        WalkStates st{a.kv_in, a.kv_out, local, trans, (float *)ca, ca != nullptr};
        if (p.segments > 1) {
            if (hipError_t e = room(k_delta_walk<T, D, true>, L::bytes(true)); e != hipSuccess) return e;
            k_delta_walk<T, D, true><<<dim3((blocks + D / kDeltaCols) * p.segments * bh), dim3(kThreads), L::bytes(true), s>>>(
                nullptr, k, v, inv, nullptr, st, c);
            k_delta_scan<D, false><<<dim3(p.Dv / kScanCols, bh), dim3(kThreads), 0, s>>>(a.kv_in, trans, local, first, p.Dv, p.segments);
            st.first = first;
        }
        if (hipError_t e = room(k_delta_walk<T, D, false>, L::bytes(false)); e != hipSuccess) return e;
        k_delta_walk<T, D, false><<<dim3(blocks * p.segments * bh), dim3(kThreads), L::bytes(false), s>>>(q, k, v, inv, (T *)a.out, st, c);
        return hipGetLastError();
    }
};

struct Backward {
    const DeltaPlan &p;
    const DeltaArgs &a;
    hipStream_t s;
    template <typename T, int D>
    hipError_t operator()() const {
        const DeltaCall c = call_of(p, a);
        const int bh = p.B * p.H, blocks = p.Dv / kDeltaCols;
        const T *q = (const T *)a.q, *k = (const T *)a.k, *v = (const T *)a.v, *dout = (const T *)a.dout;
        const Layout l = layout(p);
        char *sc = (char *)a.scratch, *ca = (char *)a.cache;
        const bf16_t *inv = (const bf16_t *)(ca + l.inv);
        typedef BackLds<T, D> L;
        float *last = (float *)(sc + l.last);
        BackStates st{a.dkv_out, a.dkv_in, (float *)(sc + l.back_local), (float *)sc, (float *)(sc + l.dr)};
        const dim3 grid(blocks * p.segments * bh);
        if (p.segments > 1) {
            if (hipError_t e = room(k_delta_back<T, D, true>, L::ALL); e != hipSuccess) return e;
            k_delta_back<T, D, true><<<grid, dim3(kThreads), L::ALL, s>>>(q, k, dout, inv, nullptr, st, c);
            k_delta_scan<D, true><<<dim3(p.Dv / kScanCols, bh), dim3(kThreads), 0, s>>>(a.dkv_out, (const float *)(ca + l.trans), st.local, last, p.Dv,
                                                                                     p.segments);
            st.last = last;
        }
        if (hipError_t e = room(k_delta_back<T, D, false>, L::ALL); e != hipSuccess) return e;
        k_delta_back<T, D, false><<<grid, dim3(kThreads), L::ALL, s>>>(q, k, dout, inv, (T *)a.dv, st, c);
        const dim3 tiles(p.tiles, bh);
        if (p.key_heads == p.H) {
            if (hipError_t e = room(k_delta_grad<T, D, T>, GradLds<T, D>::ALL); e != hipSuccess) return e;
            k_delta_grad<T, D, T><<<tiles, dim3(kThreads), GradLds<T, D>::ALL, s>>>(q, k, v, dout, inv, (const float *)ca, st.grads, st.dr, (T *)a.dq,
                                                                                 (T *)a.dk, a.dbeta, a.dlog_g, c);
        } else {
            const size_t n = (size_t)bh * p.N * D;
            float *part = (float *)(sc + l.part);
            if (hipError_t e = room(k_delta_grad<T, D, float>, GradLds<T, D>::ALL); e != hipSuccess) return e;
            k_delta_grad<T, D, float><<<tiles, dim3(kThreads), GradLds<T, D>::ALL, s>>>(q, k, v, dout, inv, (const float *)ca, st.grads, st.dr, part,
                                                                                     part + n, a.dbeta, a.dlog_g, c);
            const int share = p.H / p.key_heads;
            k_delta_group<T, D><<<dim3((unsigned)((n / share / 4 + kThreads - 1) / kThreads), 2), dim3(kThreads), 0, s>>>(part, (T *)a.dq, (T *)a.dk, n,
                                                                                                                 share, p.N);
        }
        return hipGetLastError();
    }
};

}  // namespace

// Segments: a walk takes the longer the fewer workgroups it has. Cutting a sequence costs a second walk (the local one, over twice the
// columns) and a chain of one step a segment, so it is cut where that leaves a third of the tiles or less.
DeltaPlan delta_plan(int B, int H, int N, int D, int Dv, int dtype, int key_heads) {
    DeltaPlan p{B, H, N, D, Dv, dtype, key_heads};
    p.tile = dtype == 0 ? Parts<float>::C : Parts<bf16_t>::C;
    p.tiles = (int)(((long long)N + p.tile - 1) / p.tile);
    const long long walks = (long long)B * H * (Dv / kDeltaCols);
    int cut = (int)std::min<long long>(kCus / std::min<long long>(walks, kCus), p.tiles / 4);
    while (cut > 1 && (long long)cut * cut > 2LL * p.tiles) --cut;
    if (cut < 3) cut = 1;
    p.seg_tiles = (p.tiles + cut - 1) / cut;
    p.segments = (p.tiles + p.seg_tiles - 1) / p.seg_tiles;
    return p;
}
size_t delta_cache(const DeltaPlan &p) { return layout(p).cache; }
size_t delta_scratch(const DeltaPlan &p) { return layout(p).scratch; }
size_t delta_bwd_scratch(const DeltaPlan &p) { return layout(p).back_scratch; }
hipError_t launch_delta_fwd(const DeltaPlan &p, const DeltaArgs &a, hipStream_t s) { return by_type(p, Forward{p, a, s}); }
hipError_t launch_delta_bwd(const DeltaPlan &p, const DeltaArgs &a, hipStream_t s) { return by_type(p, Backward{p, a, s}); }

}  // namespace lasp
