// HIP kernels (gfx950 / CDNA4) of the gated delta rule,
//     S_s = a_s S_{s-1} + k_s u_s^T,   u_s = beta_s w_s,   w_s = v_s - a_s S_{s-1}^T k_s,   out_s = S_s^T q_s.
// Over a tile of C tokens that starts from S, with G_s = log a_1 + .. + log a_s, W_ij = exp(G_i - G_j) and M_ij = W_ij k_i . k_j (i > j):
//     (I + M beta) w = r,   r_i = v_i - exp(G_i) S^T k_i,
//     out_i = exp(G_i) S^T q_i + sum_{j <= i} W_ij (q_i . k_j) u_j,   S' = exp(G_C) S + sum_j exp(G_C - G_j) k_j u_j^T.
// With N the sums over paths, N_ij = -M_ij - sum_{j<k<i} M_ik beta_k N_kj, the inverse is I + N beta and that of (I + beta M) is I + beta N:
// neither divides by a beta, so beta = 0 needs no case of its own, and with keys of length 1 no |N_ij| exceeds 1.
//   k_delta_prep : N, P and the gates of every tile of 32 tokens (tiles are independent)
//   k_delta_walk : the walk over the tiles of a segment (columns of S do not meet)
//   k_delta_scan : states between segments: a segment takes S to T S + S_local, T the product of its tiles' matrices
//   k_delta_step : token by token, for calls of a few tokens: state in registers, read and written once
// Backward, with dS the gradient of the state behind the tile:
//     dU = P^T dO + exp(G_C - G) K dS,   dR = dU + N^T (beta dU),   dV = beta dR,   dbeta_i = dR_i . w_i,
//     dS' = exp(G_C) dS + Q^T (exp(G) dO) - K^T (exp(G) dV),   P_ij = W_ij q_i . k_j
//     dQ = exp(G) dO S^T + Ep K,   dK = Ep^T Q + Em K + Em^T K - exp(G) dV S^T + exp(G_C - G) U dS^T,
//     Ep = W (dO U^T),   Em = -W (dV U^T) below the diagonal,
//     and dlog_a_i = a_i <dS_i - beta_i k_i (dS_i^T k_i)^T, S_{i-1}>, by what goes through gate i (k_delta_grad).
//   k_delta_back : the walk in reverse: dV, and dS and dR of every tile
//   k_delta_grad : dQ, dK, dbeta, dlog_a of every tile (tiles are independent)
//   k_delta_group: sums over the states that share a head of q and k
// Products run on bfloat16 MFMA with fp32 sums. A factor that is no input is kept in three bfloat16 parts (8 significant bits each: a float's
// 24), as states and the gradients of gates and betas come out in float and a state passes every tile: two parts (off by up to 2^-17)
// leave them further off than float sums do. Two where all that follows is rounded to bfloat16, by up to 2^-8: one output in 300 then differs by a step from what float
// products round to, and the distance from the definition is the same in four digits (three: 8 prompts up to 1777 tokens 206 us instead of 197). Float data is
// split in three as well. Products of parts i + j >= 3 (of two: 2) are left out, less than 2^-23 (at most 2^-16) of a product of two such factors.
// 32768 tokens x 16 heads of 128, bfloat16, forward and backward: 1.99 ms, 12 KB of memory a token and head (6.3 GB, 3.2 TB/s over all):
// outputs and inputs are 2.8 KB of it, the rest states and their gradients every 64 tokens (4 KB), w and dR in float (2 KB), N, P and gates
// (1.9 KB), and keys, queries and values read again. k_delta_walk and k_delta_back run at 4.4 TB/s of it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "lasp_delta.h"
#include "lasp_device.h"

namespace lasp {
namespace {

typedef Elem<bf16_t> E;
template <typename T>
struct Parts;
template <>
struct Parts<bf16_t> {
    // parts of an input, of what is computed, and of what only ends in outputs of the data's type; tiles of the walks that k_delta_grad takes at a time
    static constexpr int DATA = 1, MADE = 3, ROUNDED = 2, GRAD_TILES = 2;
};
template <>
struct Parts<float> {
    static constexpr int DATA = 3, MADE = 3, ROUNDED = 3, GRAD_TILES = 1;
};
constexpr int kThreads = 256, kWaves = 4;
constexpr int kTile = kDeltaTile;   // tokens of a walk's tile: one block of an MFMA

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

// The wave's number, as the scalar that it is: what is addressed by it then takes scalar registers.
DEVI int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

constexpr int ld_of(int width) { return width == 128 ? kSwzLd : width + E::PAD; }

// Two transposing reads: lane i of 16 gets column i of the four rows that the lanes point to in pieces of four.
DEVI bf16x8 transposed(const bf16_t *lo, const bf16_t *hi) {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    union {
        struct {
            s16x4 a, b;
        } s;
        bf16x8 v;
    } u;
    u.s.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)lo);
    u.s.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)hi);
    return u.v;
}
// Eight values in parts, by pairs: element by element the compiler converts every one of them twice.
template <int NP>
DEVI Frags<NP> split(const f32x8 &x) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    u32x4 d[NP];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f32x2 y{x[2 * e], x[2 * e + 1]};
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const unsigned u = __builtin_bit_cast(unsigned, __builtin_convertvector(y, bf16x2));
            d[i][e] = u;
            if (i + 1 < NP) y -= f32x2{__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)};
        }
    }
    Frags<NP> f;
#pragma unroll
    for (int i = 0; i < NP; ++i) f.p[i] = __builtin_bit_cast(bf16x8, d[i]);
    return f;
}
// Rows 16 m .. 16 m + 15 of an accumulator tile as the fragment of sub-step m (contraction along the rows).
template <int NP>
DEVI Frags<NP> split(const f32x16 &t, int m) {
    f32x8 x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = t[8 * m + e];
    return split<NP>(x);
}
// Four values in parts, to LDS or memory: part i at `at` + i PS.
template <int NP, int PS>
DEVI void store_parts(bf16_t *at, f32x4 v) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    f32x2 y[2] = {{v[0], v[1]}, {v[2], v[3]}};
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        u32x2 d;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            d[e] = __builtin_bit_cast(unsigned, __builtin_convertvector(y[e], bf16x2));
            if (i + 1 < NP) y[e] -= f32x2{__uint_as_float(d[e] << 16), __uint_as_float(d[e] & 0xffff0000u)};
        }
        *(u32x2 *)(at + i * PS) = d;
    }
}

// Infinities and NaN. A tile's squares hold zeros where a token does not reach another, and 0 x infinity is NaN: a broken value would spoil tokens of its tile
// that it does not reach. So N and P are made without broken values, the other operands of their products go without them, which leaves every product as it is for
// the other tokens, and what a broken value does reach is set to NaN. A state that is broken spoils its whole column, as it should.
DEVI bool is_broken(float x) { return !(__builtin_fabsf(x) < 0x1.ffp127f); }   // (floats from there on are infinite as bfloat16)
DEVI bool any_broken(const f32x16 &x) {   // in any lane of the wave (or values so large that their sum is)
    float s[2] = {x[0], x[1]};
#pragma unroll
    for (int e = 2; e < 16; ++e) s[e & 1] += x[e];
    return __builtin_expect(__builtin_amdgcn_ballot_w64(is_broken(s[0] + s[1])) != 0, 0);
}
// The first broken row of the lane's column (32: none).
DEVI int first_broken(const f32x16 &x, const Lane &ln) {
    int n = 32;
#pragma unroll
    for (int e = 0; e < 16; ++e) n = is_broken(x[e]) ? min(n, ln.acc_row(e)) : n;
    return min(n, __shfl_xor(n, 32));
}
// Zeros in place of broken bfloat16 elements.
DEVI u32x4 drop_broken(u32x4 x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = (x[e] & 0x7f80u) == 0x7f80u ? x[e] & 0xffff0000u : x[e];
        x[e] = (x[e] & 0x7f800000u) == 0x7f800000u ? x[e] & 0xffffu : x[e];
    }
    return x;
}
template <int NP>
DEVI void drop_broken(Frags<NP> &f) {
#pragma unroll
    for (int i = 0; i < NP; ++i) f.p[i] = __builtin_bit_cast(bf16x8, drop_broken(__builtin_bit_cast(u32x4, f.p[i])));
}
// How far what is broken in a tile reaches: of even and odd tiles the greatest of 32 times a number that grows from tile to tile, plus a number of rows: up to 32
// from the tile's end the walk goes to.
template <int COLS>
struct Marks {
    int any[2], keys[2], cols[2][COLS];   // (any: the tile's number)
    DEVI void clear() {
        for (int e = threadIdx.x; e < (int)(sizeof(*this) / 4); e += blockDim.x) ((int *)this)[e] = -1;
    }
    DEVI void mark(int &to, int tile, int rows) {
        any[tile & 1] = tile;
        atomicMax(&to, 32 * tile + rows - 1);
    }
    DEVI bool at(int tile) const { return __builtin_expect(__builtin_amdgcn_readfirstlane(any[tile & 1]) == tile, 0); }
    DEVI int rows(int tile, int col) const { return max(max(keys[tile & 1], cols[tile & 1][col]) - 32 * tile + 1, 0); }
};

// What the lanes of a wave wrote to LDS is there for its other lanes.
DEVI void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A square of 32 by 32: NP parts, PS elements apart.
template <int NP, int PART = 1024>
struct Block {
    static constexpr int PS = PART, BYTES = NP * PS * 2;
    bf16_t *p;
    DEVI Frags<NP> kc(const Lane &ln, int k0) const {
        Frags<NP> f;
#pragma unroll
        for (int i = 0; i < NP; ++i) f.p[i] = E::ld_kc(ln, p + i * PS, kBlockLd, 0, k0);
        return f;
    }
    DEVI Frags<NP> ks(const Lane &ln, int k0) const {
        Frags<NP> f;
#pragma unroll
        for (int i = 0; i < NP; ++i) f.p[i] = E::ld_ks(ln, p + i * PS, kBlockLd, k0, 0);
        return f;
    }
    // contraction in the order in which an accumulator tile enumerates its rows, sub-step m
    DEVI Frags<NP> kp(const Lane &ln, int m) const {
        const bf16_t *at = p + ln.r * 32 + 4 * ln.h;
        const int sw = swz4(ln.r);
        Frags<NP> f;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            union {
                struct {
                    bf16x4 a, b;
                } s;
                bf16x8 v;
            } u;
            u.s.a = *(const bf16x4 *)(at + i * PS + (((2 * m) ^ sw) << 3));
            u.s.b = *(const bf16x4 *)(at + i * PS + (((2 * m + 1) ^ sw) << 3));
            f.p[i] = u.v;
        }
        return f;
    }
    DEVI Frags<NP> ksp(const Lane &ln, int m) const {
        const int l16 = ln.id & 15, row = 16 * m + 4 * ln.h + (l16 >> 2), col = (ln.id & 16) + 4 * (l16 & 3);
        const bf16_t *lo = p + lds_off(kBlockLd, row, col), *hi = p + lds_off(kBlockLd, row + 8, col);
        Frags<NP> f;
#pragma unroll
        for (int i = 0; i < NP; ++i) f.p[i] = transposed(lo + i * PS, hi + i * PS);
        return f;
    }
    DEVI void st4(int row, int col, f32x4 v) const { store_parts<NP, PS>(p + lds_off(kBlockLd, row, col), v); }
    DEVI void st_acc(const Lane &ln, const f32x16 &t) const {   // (transposed, as Tile's)
#pragma unroll
        for (int g = 0; g < 4; ++g) st4(ln.r, 8 * g + 4 * ln.h, f32x4{t[4 * g], t[4 * g + 1], t[4 * g + 2], t[4 * g + 3]});
    }
};
// A lower triangular square of C tokens: its blocks (0,0), (1,0), (1,1).
template <int NP, int C>
struct Lower {
    static constexpr int NB = C / 32, BLOCKS = NB * (NB + 1) / 2, PS = BLOCKS * 1024, BYTES = NP * PS * 2;
    bf16_t *p;
    DEVI Block<NP, PS> at(int it, int jt) const { return {p + (it * (it + 1) / 2 + jt) * 1024}; }
};

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
        store_parts<NP, PS>(p + lds_off(LD, row, col), v);
    }
    DEVI f32x4 get4(int row, int col) const {
        const bf16_t *at = p + lds_off(LD, row, col);
        f32x4 v{0, 0, 0, 0};
#pragma unroll
        for (int i = NP - 1; i >= 0; --i) v += __builtin_convertvector(*(const bf16x4 *)(at + i * PS), f32x4);
        return v;
    }
    // contraction in the order in which an accumulator tile enumerates its rows: sub-step m of the 32 from k0
    DEVI Frags<NP> kp(const Lane &ln, int row0, int k0, int m) const {
        Frags<NP> f;
#pragma unroll
        for (int i = 0; i < NP; ++i) f.p[i] = E::ld_kp(ln, p + i * PS, LD, row0, k0, m);
        return f;
    }
    DEVI Frags<NP> ksp(const Lane &ln, int k0, int col0, int m) const {
        const int l16 = ln.id & 15, row = k0 + 16 * m + 4 * ln.h + (l16 >> 2), col = col0 + (ln.id & 16) + 4 * (l16 & 3);
        const bf16_t *lo = p + lds_off(LD, row, col), *hi = p + lds_off(LD, row + 8, col);
        Frags<NP> f;
#pragma unroll
        for (int i = 0; i < NP; ++i) f.p[i] = transposed(lo + i * PS, hi + i * PS);
        return f;
    }
    // the 32 rows of a tile in the order of an accumulator's, a lane per column (one part)
    DEVI f32x16 rows(const Lane &ln, int col0) const {
        f32x16 x;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const f32x8 y = __builtin_convertvector(ksp(ln, 0, col0, m).p[0], f32x8);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[8 * m + e] = y[e];
        }
        return x;
    }
    // an accumulator tile, transposed: its column r is row row0 + r here, its rows are columns col0 ..
    DEVI void st_acc(const Lane &ln, int row0, int col0, const f32x16 &t) const {
#pragma unroll
        for (int g = 0; g < 4; ++g) st4(row0 + ln.r, col0 + 8 * g + 4 * ln.h, f32x4{t[4 * g], t[4 * g + 1], t[4 * g + 2], t[4 * g + 3]});
    }
};

// Rows of a global tensor on their way to a tile: 16 bytes a thread (of NT) and piece. Rows from `valid` (at least 1) on are zeros, but the last of the
// others is read in their place: behind a load that may not have been issued no other one could be waited for by itself.
template <typename T, int ROWS, int WIDTH, int NT>
struct Fetch {
    static constexpr int EPC = 16 / sizeof(T), CPR = WIDTH / EPC, PIECES = ROWS * CPR, N = (PIECES + NT - 1) / NT;
    u32x4 v[N];
    int rows;
    DEVI void load(const T *base, size_t ld, int valid) {
        rows = valid;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = threadIdx.x + n * NT, row = c / CPR, col = (c % CPR) * EPC;
            v[n] = gload<u32x4>(base, (min(row, valid - 1) * (unsigned)ld + col) * sizeof(T));
        }
    }
    template <typename F>
    DEVI void each(F f) const {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = threadIdx.x + n * NT;
            const u32x4 x = c / CPR < rows ? v[n] : u32x4{0, 0, 0, 0};
            if (PIECES % NT == 0 || c < PIECES) f(n, c / CPR, (c % CPR) * EPC, x);
        }
    }
    // Whether this thread's pieces hold a broken value; those are handed to f(row, column) and become zeros.
    DEVI bool looks_broken() const {
        if constexpr (sizeof(T) == 2) {   // (by their sum, two elements an instruction)
            typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
            float y = 0.0f;
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned two = v[n][e];   // (a cast of the element itself would take the vector's first)
                    y = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), bf16x2{1, 1}, y, false);
                }
            return __builtin_expect(is_broken(y), 0);
        } else {
            bool y = false;
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) y |= is_broken(__uint_as_float(v[n][e]));
            return __builtin_expect(y, 0);
        }
    }
    template <typename F>
    DEVI void drop(F f) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = threadIdx.x + n * NT, row = c / CPR, col = c % CPR * EPC;
            const bool there = (PIECES % NT == 0 || c < PIECES) && row < rows;
#pragma unroll
            for (int e = 0; e < EPC; ++e) {
                const unsigned x = sizeof(T) == 4 ? v[n][e & 3] : e & 1 ? v[n][e / 2] & 0xffff0000u : v[n][e / 2] << 16;
                if (!is_broken(__uint_as_float(x))) continue;
                if (there) f(row, col + e);
                if constexpr (sizeof(T) == 4) v[n][e & 3] = 0;
                else v[n][e / 2] &= e & 1 ? 0xffffu : 0xffff0000u;
            }
        }
    }
    template <typename Tl>
    DEVI void store(const Tl &t) const {
        each([&](int, int row, int col, u32x4 x) {
            if constexpr (sizeof(T) == 2) *(u32x4 *)(t.p + lds_off(Tl::LD, row, col)) = x;
            else t.st4(row, col, __builtin_bit_cast(f32x4, x));
        });
    }
};
// BYTES that lie in LDS as they do in global memory.
template <int BYTES, int NT>
struct Copy {
    static constexpr int PIECES = BYTES / 16, N = (PIECES + NT - 1) / NT;
    u32x4 v[N];
    DEVI void load(const void *base) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = threadIdx.x + n * NT;
            v[n] = gload<u32x4>((const u32x4 *)base, min(c, PIECES - 1) * 16u);
        }
    }
    DEVI void store(void *to) const {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = threadIdx.x + n * NT;
            if (PIECES % NT == 0 || c < PIECES) ((u32x4 *)to)[c] = v[n];
        }
    }
};

// 16 features of the lane's token, as an accumulator tile has them (p: the token's row at the tile's first feature).
template <typename T>
DEVI void store_acc(T *p, const Lane &ln, const f32x16 &x) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const f32x4 v{x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]};
        if constexpr (sizeof(T) == 2) *(bf16x4 *)(p + 8 * g + 4 * ln.h) = __builtin_convertvector(v, bf16x4);
        else *(f32x4 *)(p + 8 * g + 4 * ln.h) = v;
    }
}

// The gates of C tokens. Logarithms are summed in 64 bits and to base 2: the sum over a tile may be large where a difference is small.
// From 2^-300 on (-infinity among them: the state starts anew) a gate counts as 2^-300, whose power is 0 as a float, so that
// differences of sums stay numbers.
DEVI double to_base2(float log_g) {
    const double x = (double)log_g * 1.4426950408889634;
    return x < -300.0 ? -300.0 : x;   // (NaN stays)
}
constexpr double kLeastGate = -126.0;   // (the power of less is 0)
DEVI float power(double d) { return __builtin_amdgcn_exp2f((float)d); }
// Sums over the lanes of C up to this one.
template <int C>
DEVI double sum_up(double x, int lane) {
#pragma unroll
    for (int d = 1; d < C; d *= 2) {
        const double y = __shfl_up(x, d, C);
        if ((lane & (C - 1)) >= d) x += y;
    }
    return x;
}

// Values of a tile's rows in the order of an accumulator tile's rows, from LDS.
DEVI f32x16 by_row(const float *w, const Lane &ln) {
    f32x16 x;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const f32x4 v = *(const f32x4 *)(w + 8 * g + 4 * ln.h);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * g + e] = v[e];
    }
    return x;
}
// exp(G_i - G_j) for this lane's token and an accumulator's rows (of the one as i, or with NEGATIVE as j), whatever their order. Computed for all: a choice in front
// of it would be compiled as sixteen branches, each with its own wait.
template <bool NEGATIVE>
DEVI f32x16 weights_by_row(const double *sums, double own, const Lane &ln) {
    typedef __attribute__((ext_vector_type(2))) double f64x2;
    f64x2 s[8];
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int i = 0; i < 2; ++i) s[2 * g + i] = *(const f64x2 *)(sums + 8 * g + 4 * ln.h + 2 * i);
    f32x16 x;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = power(NEGATIVE ? s[e / 2][e & 1] - own : own - s[e / 2][e & 1]);
    return x;
}

struct DeltaCall {
    int B, H, Hk, N, Dv, tiles, segments, seg_tiles, grad_tiles;
    const float *log_g, *beta;
    const int *len;
    // tokens of sequence b from token0 on, 0 .. most
    DEVI int valid(int b, int token0, int most) const {
        const int n = len ? min(max(len[b], 0), N) : N;
        return min(max(n - token0, 0), most);
    }
    DEVI size_t key_row(int b, int h) const { return ((size_t)b * Hk + h / (H / Hk)) * N; }   // first row of a head of q, k
};

// What k_delta_prep leaves of a tile: N, by token exp(G_i), exp(G_C - G_i), beta_i and (every one the same) exp(G_C), and (last, as a walk without
// outputs has no use for them) the scores P, a row per query.
template <typename T>
struct Prepared {
    typedef Block<Parts<T>::MADE> Square;
    static constexpr int N = 0, START = Square::BYTES, REST = START + 4 * kTile, BETA = REST + 4 * kTile, WHOLE = BETA + 4 * kTile, P = WHOLE + 4 * kTile,
                         BYTES = P + Square::BYTES;
};

// ---------------------------------------------------------------------------
// k_delta_prep: a wave per tile, keys and queries straight into operands. N in blocks of 16 by substitution, a lane per column; then joined,
//     N21 = -(I + N22 beta) M21 (I + beta N11).
// 16384 tiles of 128 features: 99 us, 4.8 TB/s: bound by memory.
// ---------------------------------------------------------------------------
template <typename T, int D>
DEVI void operands(Frags<Parts<T>::DATA> (&f)[D / 16], const T *row, const Lane &ln, bool there) {
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
        if constexpr (sizeof(T) == 2) {
            u32x4 x{0, 0, 0, 0};
            if (there) x = *(const u32x4 *)(row + 16 * k + 8 * ln.h);
            f[k].p[0] = __builtin_bit_cast(bf16x8, x);
        } else {
            f32x4 x{0, 0, 0, 0}, y{0, 0, 0, 0};
            if (there) {
                x = *(const f32x4 *)(row + 16 * k + 8 * ln.h);
                y = *(const f32x4 *)(row + 16 * k + 8 * ln.h + 4);
            }
            f[k] = split<3>(__builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
}
template <typename T, int D>
__global__ __launch_bounds__(kThreads, 2) void k_delta_prep(const T *__restrict__ Q, const T *__restrict__ K, char *__restrict__ prepared, DeltaCall a) {
    using P = Parts<T>;
    using Pr = Prepared<T>;
    constexpr int LDM = kTile + 4;
    __shared__ __attribute__((aligned(16))) float lds_m[kWaves][kTile * LDM], lds_n[kWaves][kTile * LDM], lds_beta[kWaves][kTile];
    __shared__ __attribute__((aligned(16))) double lds_sum[kWaves][kTile];
    const Lane ln(threadIdx.x);
    const int wave = wave_id(), tile = blockIdx.x * kWaves + wave, bh = blockIdx.y, b = bh / a.H, h = bh - b * a.H, token0 = tile * kTile;
    float *M = lds_m[wave], *N = lds_n[wave], *beta = lds_beta[wave];
    double *sum = lds_sum[wave];
    const int valid = tile < a.tiles ? a.valid(b, token0, kTile) : 0;
    if (valid == 0) return;   // (no walk reads it; the waves share nothing)
    const size_t key_row = a.key_row(b, h) + token0 + ln.r, gate = (size_t)bh * a.N + token0 + ln.r;
    const bool there = ln.r < valid;
    Frags<P::DATA> fk[D / 16], fq[D / 16];
    auto load = [&]() {
        operands<T, D>(fk, K + key_row * D, ln, there);
        operands<T, D>(fq, Q + key_row * D, ln, there);
    };
    load();
    const float bt = there ? a.beta[gate] : 0.0f;
    const double x = sum_up<kTile>(a.log_g && there ? to_base2(a.log_g[gate]) : 0.0, ln.id), all = __shfl(x, kTile - 1, kTile);
    char *to = prepared + ((size_t)bh * a.tiles + tile) * Pr::BYTES;
    if (ln.h == 0) {
        beta[ln.r] = bt;
        sum[ln.r] = x;
        ((float *)(to + Pr::START))[ln.r] = power(x);
        ((float *)(to + Pr::REST))[ln.r] = power(all - x);
        ((float *)(to + Pr::BETA))[ln.r] = bt;
        ((float *)(to + Pr::WHOLE))[ln.r] = power(all);
    }
    f32x16 m, p;   // k_i . k_j, a row per i;  q_i . k_j, a row per j
    auto products = [&]() {
        m = p = f32x16{};
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            m = mm<P::MADE>(fk[k], fk[k], m);
            p = mm<P::MADE>(fk[k], fq[k], p);
        }
    };
    products();
    if (any_broken(p)) {   // (a broken key shows there, too; loaded again, as operands that are kept would spill)
        load();
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            drop_broken(fk[k]);
            drop_broken(fq[k]);
        }
        products();
    }
    wave_sync();
    const f32x16 below = weights_by_row<true>(sum, x, ln), above = weights_by_row<false>(sum, x, ln);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int o = ln.acc_row(e);
        const float v = m[e] * below[e], y = p[e] * above[e];
        M[o * LDM + ln.r] = o > ln.r ? v : 0.0f;
        p[e] = o <= ln.r ? y : 0.0f;
    }
    const typename Pr::Square pt{(bf16_t *)(to + Pr::P)}, nt{(bf16_t *)(to + Pr::N)};
    pt.st_acc(ln, p);
    wave_sync();
    if (ln.h == 0) {
        const int j = ln.r, b0 = j & ~15, jj = j & 15;
        float n[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float s = M[(b0 + i) * LDM + j];
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if (k < i) s = __builtin_fmaf(M[(b0 + i) * LDM + b0 + k], n[k], s);
            s = i > jj ? -s : 0.0f;
            N[(b0 + i) * LDM + j] = s;
            N[((b0 ^ 16) + i) * LDM + j] = 0.0f;   // (below the blocks: in place of what is joined next)
            n[i] = s * beta[b0 + i];
        }
    }
    wave_sync();
    {
        const int i = ln.id >> 2, j = 4 * (ln.id & 3);   // four columns of a row
        f32x4 y = *(const f32x4 *)(M + (16 + i) * LDM + j);
#pragma unroll
        for (int k = 0; k < 16; ++k) y += (M[(16 + i) * LDM + k] * beta[k]) * *(const f32x4 *)(N + k * LDM + j);
        *(f32x4 *)(N + (16 + i) * LDM + j) = y;
        wave_sync();
#pragma unroll
        for (int k = 0; k < 16; ++k) y += (N[(16 + i) * LDM + 16 + k] * beta[16 + k]) * *(const f32x4 *)(N + (16 + k) * LDM + j);
        wave_sync();
        *(f32x4 *)(N + (16 + i) * LDM + j) = -y;
        wave_sync();
    }
#pragma unroll
    for (int c = ln.id; c < kTile * kTile / 4; c += 64) nt.st4(c / 8, c % 8 * 4, *(const f32x4 *)(N + c / 8 * LDM + c % 8 * 4));
}

// Waves a SIMD that a walk is compiled for: two, so that one computes while the other waits, where 256 registers are enough.
template <typename T, int D, int DV, int SPLIT>
constexpr int waves_of() { return SPLIT == 1 && D == 128 && (sizeof(T) == 4 || DV == 64) ? 1 : 2; }
// Two waves that have half a sum each: a square of accumulators through LDS, a lane's values as they lie.
constexpr int kSplitCols = 64, kSquareBytes = 4096;
DEVI void put_tile(float *to, const Lane &ln, const f32x16 &x) {
#pragma unroll
    for (int g = 0; g < 4; ++g) *(f32x4 *)(to + 256 * g + 4 * ln.id) = f32x4{x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]};
}
DEVI f32x16 get_tile(const float *from, const Lane &ln) {
    f32x16 x;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const f32x4 v = *(const f32x4 *)(from + 256 * g + 4 * ln.id);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * g + e] = v[e];
    }
    return x;
}

// Values of the lane's column in rows of LD elements, in the order of an accumulator tile's rows; `there`: rows that exist. A scalar base every
// eight rows, so that a row is at most an instruction's own offset away from it.
template <int LD, typename T>
DEVI f32x16 load_rows(const T *p, const Lane &ln, int there) {
    f32x16 x = {};
    const unsigned at = (4 * ln.h * LD + ln.r) * sizeof(T);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const T *row = p + (8 * (e >> 2)) * LD;
        if (there >= 32 || ln.acc_row(e) < there) {
            const T v = gload<T>(row, at + (e & 3) * LD * sizeof(T));
            x[e] = Elem<T>::ld1(&v);
        }
    }
    return x;
}
template <int LD, typename T>
DEVI void store_rows(T *p, const Lane &ln, int there, const f32x16 &x) {
    const unsigned at = (4 * ln.h * LD + ln.r) * sizeof(T);
    if (there >= 32)
#pragma unroll
        for (int e = 0; e < 16; ++e) Elem<T>::gst1(p + (8 * (e >> 2)) * LD, at + (e & 3) * LD * sizeof(T), x[e]);
    else
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (ln.acc_row(e) < there) Elem<T>::gst1(p + (8 * (e >> 2)) * LD, at + (e & 3) * LD * sizeof(T), x[e]);
}
// Zeros in the rows behind a sequence's end, from row `first` on: what the products leave there is 0 times the state, which need not be a number.
template <int LD, typename T>
DEVI void zero_rows(T *p, const Lane &ln, int first, int there) {
    const unsigned at = (4 * ln.h * LD + ln.r) * sizeof(T);
#pragma unroll
    for (int e = 0; e < 16; ++e)
        if (ln.acc_row(e) >= first && ln.acc_row(e) < there) Elem<T>::gst1(p + (8 * (e >> 2)) * LD, at + (e & 3) * LD * sizeof(T), 0.0f);
}
// A wave's part of a state: KB blocks of 32 key features (rows) by its 32 columns (a lane each).
template <int KB, int LD>
DEVI void load_state(f32x16 (&S)[KB], const Lane &ln, const float *src) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) S[kb] = src ? load_rows<LD>(src + 32 * kb * LD, ln, 32) : f32x16{};
}
template <int KB, int LD>
DEVI void save_state(const f32x16 (&S)[KB], const Lane &ln, float *dst) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) store_rows<LD>(dst + 32 * kb * LD, ln, 32, S[kb]);
}

// A matrix as k_delta_scan's waves load it, sixteen bytes a lane and a kilobyte an instruction: of rows 16 tile + l16 the columns 16 step + 4 l4 .. + 3.
// (Row by row, neighbouring lanes are rows apart, and the loads of a step take longer than its products: 109 us for 32 segments x 16 heads.)
template <int D>
DEVI unsigned matrix_piece(int tile, int step, int l16, int l4) { return ((tile * (D / 16) + step) * 64 + 16 * l4 + l16) * 4; }
// A wave's part of T, rows from d0 on of the lane's column c, and of T^T (may be null).
template <int KB, int D>
DEVI void save_matrix(const f32x16 (&S)[KB], const Lane &ln, int d0, int c, float *T, float *back, size_t at) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int r = d0 + 32 * kb + 8 * g + 4 * ln.h;
            const f32x4 v{S[kb][4 * g], S[kb][4 * g + 1], S[kb][4 * g + 2], S[kb][4 * g + 3]};
            if (back) *(f32x4 *)(back + at + matrix_piece<D>(c / 16, r / 16, c % 16, r % 16 / 4)) = v;
#pragma unroll
            for (int e = 0; e < 4; ++e) T[at + matrix_piece<D>(r / 16, c / 16, r % 16 + e, c % 16 / 4) + c % 4] = v[e];
        }
}

// ---------------------------------------------------------------------------
// k_delta_walk: a wave carries 32 columns of the state in its accumulators and meets no other wave's: what a product leaves in an
// accumulator tile (a row per token or key feature, a lane per column) is the next one's operand as it lies there, with the contraction in the
// order of the accumulator's rows; the waves share the tile's keys, queries, N and scores in LDS. SPLIT = 2: two waves have half of the key
// features of 32 columns each, and add up S^T k and S^T q once a tile. LOCAL: no outputs; the state a segment reaches
// from zero, and (waves behind those of the values) its matrix T, which is the state reached from the identity without values.
// 32768 tokens x 16 heads of 128, bfloat16, with a cache: 349 us, 4.4 TB/s, memory (2 % of it the look for broken values); LOCAL: 350 us over twice the columns, 1.4 TB/s, bound by what
// a wave issues (a tile takes 3.6 us of matrix products, parts of accumulators and waits for LDS, one after the other).
// ---------------------------------------------------------------------------
template <typename T, int D, int DV, bool LOCAL, int SPLIT>
struct Walk {
    using P = Parts<T>;
    static constexpr int ALL = DV + (LOCAL ? D : 0), COLS = SPLIT == 1 ? ALL : kSplitCols, GROUPS = ALL / COLS;
    static constexpr int CW = COLS / 32, WAVES = CW * SPLIT, NT = 64 * WAVES, KB = D / 32 / SPLIT;   // (KB: blocks of key features of a wave)
    typedef Tile<P::DATA, kTile, D> Data;
    static constexpr int VALUES = COLS < DV ? COLS : DV;
    typedef Tile<1, kTile, VALUES> Value;
    static constexpr bool STAGED = sizeof(T) == 2;   // two-byte values go through LDS, which hands a lane four tokens of its column at a time
    static constexpr int PREP = LOCAL ? Prepared<T>::P : Prepared<T>::BYTES;   // what is taken of a prepared tile
    static constexpr int K = PREP, V = K + Data::BYTES, Q = V + (STAGED ? Value::BYTES : 0),
                         STAGE = LOCAL ? Q : Q + Data::BYTES, XCH = 2 * STAGE, LDS = XCH + (SPLIT == 1 ? 0 : CW * (LOCAL ? 2 : 3) * kSquareBytes);
};
struct WalkStates {
    const float *first;   // states that segments start from ([head][segment], or kv_in where there is one segment); null = zeros
    float *last;          // kv_out
    float *local, *trans, *back;   // LOCAL: state, T and (goes with the cache) T^T, as k_delta_scan takes them
    float *cache;         // the state in front of every tile that k_delta_grad takes; may be null
    float *w;             // w of every token; goes with the cache
    int all_trans;        // T is wanted of the last segment too
};
template <typename T, int D, int DV, bool LOCAL, int SPLIT>
__global__ __launch_bounds__((Walk<T, D, DV, LOCAL, SPLIT>::NT), (waves_of<T, D, DV, SPLIT>())) void k_delta_walk(const T *__restrict__ Q, const T *__restrict__ K,
                                                                              const T *__restrict__ V, const char *__restrict__ prepared,
                                                                              T *__restrict__ O, WalkStates st, DeltaCall a) {
    using L = Walk<T, D, DV, LOCAL, SPLIT>;
    using P = typename L::P;
    using Pr = Prepared<T>;
    constexpr int KB = L::KB, MADE = P::MADE;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const Lane ln(threadIdx.x);
    const int wave = wave_id(), seg = blockIdx.x % a.segments, bh = blockIdx.x / a.segments, b = bh / a.H, h = bh - b * a.H;
    if (LOCAL && seg == a.segments - 1 && !st.all_trans) return;
    const int part = SPLIT == 1 ? 0 : wave / L::CW, cw = wave - part * L::CW, v0 = L::GROUPS == 1 ? 0 : blockIdx.y * L::COLS;
    const bool trans = LOCAL && v0 + 32 * cw >= DV;
    const int c0 = v0 + 32 * cw - (trans ? DV : 0), d0 = 32 * KB * part;
    const int tokens = a.valid(b, 0, a.N), end = min(a.tiles, (seg + 1) * a.seg_tiles);
    const int t0 = seg * a.seg_tiles, t1 = min(end, (tokens + kTile - 1) / kTile);   // (tiles behind a sequence's end leave the state as it is)
    const size_t key_row = a.key_row(b, h), row = (size_t)bh * a.N;
    f32x16 S[KB];
    if (trans) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) S[kb][e] = d0 + 32 * kb + ln.acc_row(e) == c0 + ln.r ? 1.0f : 0.0f;
    } else {
        load_state<KB, DV>(S, ln, LOCAL || !st.first ? nullptr : st.first + (((size_t)bh * a.segments + seg) * D + d0) * DV + c0);
    }
    Fetch<T, kTile, D, L::NT> fk, fq;
    Copy<L::PREP, L::NT> fp;
    Fetch<T, kTile, L::VALUES, L::NT> fv;   // (STAGED)
    f32x16 v = {};                   // (else)
    auto fetch = [&](int t) {
        const int token0 = t * kTile, valid = min(tokens - token0, kTile);
        fp.load(prepared + ((size_t)bh * a.tiles + t) * Pr::BYTES);
        fk.load(K + (key_row + token0) * D, D, valid);
        if constexpr (!LOCAL) fq.load(Q + (key_row + token0) * D, D, valid);
        if constexpr (L::STAGED) fv.load(V + (row + token0) * DV + (v0 < DV ? v0 : 0), DV, valid);
        else if (!trans) v = load_rows<DV>(V + (row + token0) * DV + c0, ln, valid);
    };
    if (t0 < t1) fetch(t0);
    for (int t = t0; t < t1; ++t) {
        const int token0 = t * kTile, valid = min(tokens - token0, kTile);
        unsigned char *at = lds + (t & 1) * L::STAGE;   // (the waves that still read the tile before have the other half)
        const typename L::Data kt{(bf16_t *)(at + L::K)}, qt{(bf16_t *)(at + L::Q)};
        const typename Pr::Square nt{(bf16_t *)(at + Pr::N)}, pt{(bf16_t *)(at + Pr::P)};
        fp.store(at);
        fk.store(kt);
        if constexpr (!LOCAL) fq.store(qt);
        const typename L::Value vt{(bf16_t *)(at + L::V)};
        if constexpr (L::STAGED) fv.store(vt);
        f32x16 r = v;
        __syncthreads();
        if (t + 1 < t1) fetch(t + 1);
        if constexpr (!LOCAL)
            if (st.cache && t % P::GRAD_TILES == 0)
                save_state<KB, DV>(S, ln, st.cache + (((size_t)bh * a.grad_tiles + t / P::GRAD_TILES) * D + d0) * DV + c0);
        bool spoilt = false;   // (LOCAL: the state that is left is NaN either way)
        f32x16 o = {};   // r: a row per token;  o: a lane per token, a row per column
        {
            f32x16 x = {};
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const auto s = split<MADE>(S[kb], m);
                    x = mm<MADE>(kt.kp(ln, 0, d0 + 32 * kb, m), s, x);
                    if constexpr (!LOCAL) o = mm<P::ROUNDED>(s, qt.kp(ln, 0, d0 + 32 * kb, m), o);
                }
            if constexpr (SPLIT == 2) {
                float *mine = (float *)(lds + L::XCH + (part * L::CW + cw) * kSquareBytes), *other = (float *)(lds + L::XCH + ((1 - part) * L::CW + cw) * kSquareBytes),
                      *out = (float *)(lds + L::XCH + (2 * L::CW + cw) * kSquareBytes);
                put_tile(mine, ln, x);
                if constexpr (!LOCAL)
                    if (part == 0) put_tile(out, ln, o);
                __syncthreads();
                x += get_tile(other, ln);
                if constexpr (!LOCAL)
                    if (part == 1) o += get_tile(out, ln);
            }
            if constexpr (L::STAGED)
                if (!trans) r = vt.rows(ln, c0 - v0);
            r -= by_row((const float *)(at + Pr::START), ln) * x;
            x = by_row((const float *)(at + Pr::BETA), ln) * r;
            if (!LOCAL && any_broken(x)) {
                spoilt = true;
                const int first = first_broken(x, ln);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (ln.acc_row(e) >= first) {
                        x[e] = 0.0f;
                        r[e] = __builtin_nanf("");
                    }
            }
#pragma unroll
            for (int m = 0; m < 2; ++m) r = mm<MADE>(nt.kp(ln, m), split<MADE>(x, m), r);
        }
        if constexpr (!LOCAL)
            if (st.cache && part == 0) store_rows<DV>(st.w + (row + token0) * DV + c0, ln, valid, r);
        r *= by_row((const float *)(at + Pr::BETA), ln);
        if (!LOCAL && part == SPLIT - 1) {
            o *= ((const float *)(at + Pr::START))[ln.r];
            if (spoilt) {
                const int first = first_broken(r, ln);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    if (ln.acc_row(e) >= first) r[e] = 0.0f;
                    if (ln.r >= __shfl(first, ln.acc_row(e))) o[e] = __builtin_nanf("");
                }
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) S[kb] = first < kTile ? f32x16(__builtin_nanf("")) : S[kb];
            }
#pragma unroll
            for (int m = 0; m < 2; ++m) o = mm<P::ROUNDED>(split<P::ROUNDED>(r, m), pt.kp(ln, m), o);
            if (ln.r < valid) store_acc(O + (row + token0 + ln.r) * DV + c0, ln, o);
        }
        r *= by_row((const float *)(at + Pr::REST), ln);
        const float whole = *(const float *)(at + Pr::WHOLE);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) S[kb] *= whole;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const auto f = split<MADE>(r, m);
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) S[kb] = mm<MADE>(kt.ksp(ln, 0, d0 + 32 * kb, m), f, S[kb]);
        }
    }
    if constexpr (LOCAL) {
        if (trans) save_matrix<KB, D>(S, ln, d0, c0 + ln.r, st.trans, st.back, ((size_t)bh * a.segments + seg) * D * D);
        else save_state<KB, DV>(S, ln, st.local + (((size_t)bh * a.segments + seg) * D + d0) * DV + c0);
    } else {
        if (part == 0)
            for (int t = max(t0, tokens / kTile); t < end; ++t)
                zero_rows<DV>(O + (row + t * kTile) * DV + c0, ln, tokens - t * kTile, min(a.N - t * kTile, kTile));
        if (seg == a.segments - 1) save_state<KB, DV>(S, ln, st.last + ((size_t)bh * D + d0) * DV + c0);
    }
}

// ---------------------------------------------------------------------------
// k_delta_scan: first[0] = in, first[p + 1] = T_p first[p] + local[p]; BACK: last[P - 1] = in, last[p - 1] = T_p^T last[p] + local[p].
// 16 columns a workgroup, 16 rows a wave, in float. 32 segments x 16 heads of 128: 82 us in either direction, 2.5 us a step, a chain of barrier, LDS and 32
// matrix products on top of each other; more matrices on their way change nothing. (Fewer segments cost the walks what they save here.)
// ---------------------------------------------------------------------------
// (v_mfma_f32_16x16x4_f32: lane l supplies row or column l & 15 and contraction index l >> 4; accumulator rows 4 (l >> 4) .. + 3, column l & 15.)
constexpr int kScanCols = 16;
template <int D, bool BACK>
__global__ __launch_bounds__(4 * D) void k_delta_scan(const float *__restrict__ in, const float *__restrict__ trans, const float *__restrict__ local,
                                                         float *__restrict__ states, int Dv, int segments) {
    __shared__ __attribute__((aligned(16))) float S[2][kScanCols][D + 4];   // a row per column
    const int bh = blockIdx.x, c = blockIdx.y * kScanCols + (threadIdx.x & 15), wave = threadIdx.x >> 6, l16 = threadIdx.x & 15, l4 = threadIdx.x >> 4 & 3;
    struct Step {
        f32x4 add;
        float m[D / 4];   // contraction 16 s + 4 l4 + i at 4 s + i
    };
    f32x4 x;
    auto at = [&](size_t segment, int i) { return (segment * D + 16 * wave + 4 * l4 + i) * Dv + c; };
    auto fetch = [&](Step &to, int step) {
        step = min(step, segments - 2);   // (without a branch, behind which no load could be waited for apart from those that follow it)
        const int p = BACK ? segments - 1 - step : step;
        const float *t = trans + ((size_t)bh * segments + p) * D * D;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            const f32x4 y = *(const f32x4 *)(t + matrix_piece<D>(wave, s, l16, l4));
#pragma unroll
            for (int i = 0; i < 4; ++i) to.m[4 * s + i] = y[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) to.add[i] = local[at((size_t)bh * segments + p, i)];
    };
    auto go = [&](const Step &now, int step) {   // the state in front of this step's segment is written, and taken through it
        const int p = BACK ? segments - 1 - step : step;
        auto &lds = S[step & 1];   // (read by the other waves until the barrier of the next step)
        *(f32x4 *)(&lds[l16][16 * wave + 4 * l4]) = x;
#pragma unroll
        for (int i = 0; i < 4; ++i) states[at((size_t)bh * segments + p, i)] = x[i];
        if (step + 1 == segments) return;
        __syncthreads();
        f32x4 y[D / 16], z = {};
#pragma unroll
        for (int s = 0; s < D / 16; ++s) y[s] = *(const f32x4 *)(&lds[l16][16 * s + 4 * l4]);
        x = now.add;
        __builtin_amdgcn_sched_barrier(0);   // (all reads are on their way before the first product waits for one)
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) {   // (two chains)
                auto &sum = i & 1 ? z : x;
                sum = __builtin_amdgcn_mfma_f32_16x16x4f32(now.m[4 * s + i], y[s][i], sum, 0, 0, 0);
            }
        x += z;
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = in ? in[at(bh, i)] : 0.0f;
    constexpr int AHEAD = 2;   // (a matrix is on its way while the one before is used)
    Step ring[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD - 1; ++i) fetch(ring[i], i);
    for (int step = 0; step < segments; step += AHEAD)
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (step + i < segments) {
                fetch(ring[(i + AHEAD - 1) % AHEAD], step + i + AHEAD - 1);
                go(ring[i], step + i);
            }
}

// ---------------------------------------------------------------------------
// k_delta_step: COLS columns of a head's state in the registers of 256 threads, four columns by some rows apiece. One reduction a token:
//     S^T k, S^T q and q . k of the state as it was give u = beta (v - a S^T k) and out = a S^T q + (q . k) u.
// One token of 64 x 16 heads of 128: 28 us, 4.8 TB/s, memory; of 1 x 16 heads 3.8 us, the launch.
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
// k_delta_back: the walk in reverse (SPLIT as there; the sum is dU's). LOCAL: the gradient that reaches a segment's front from its own tokens.
// What a thread stages is looked at for broken values on its way, which costs no register behind it (a look at dU and dO where they are used: 34 registers spilt, 78 us more).
// Sizes as above: 355 us, 4.3 TB/s; LOCAL 250 us.
// ---------------------------------------------------------------------------
template <typename T, int D, int DV, int SPLIT>
struct Back {
    using P = Parts<T>;
    static constexpr int COLS = SPLIT == 1 ? DV : kSplitCols, GROUPS = DV / COLS, CW = COLS / 32, WAVES = CW * SPLIT, NT = 64 * WAVES, KB = D / 32 / SPLIT;
    typedef Tile<P::DATA, kTile, D> Data;
    typedef Tile<P::DATA, kTile, COLS> Grad;
    static constexpr int PREP = 0, K = Prepared<T>::BYTES, Q = K + Data::BYTES, DO = Q + Data::BYTES, STAGE = DO + Grad::BYTES,
                         XBYTES = SPLIT == 1 ? 0 : 2 * CW * kSquareBytes,
                         MBYTES = (int)sizeof(Marks<COLS>), STAGES = 2 * STAGE + XBYTES + MBYTES <= 163840 ? 2 : 1, XCH = STAGES * STAGE, MARKS = XCH + XBYTES,
                         LDS = MARKS + MBYTES;
};
struct BackStates {
    const float *last;   // gradients of the states segments end with ([head][segment], or dkv_out where there is one segment); null = zeros
    float *first;        // dkv_in
    float *local;        // LOCAL
    float *grads;        // the gradient of the state behind every tile that k_delta_grad takes
    float *dr;           // [B][H][N][Dv]
};
template <typename T, int D, int DV, bool LOCAL, int SPLIT>
__global__ __launch_bounds__((Back<T, D, DV, SPLIT>::NT), (waves_of<T, D, DV, SPLIT>())) void k_delta_back(const T *__restrict__ Q, const T *__restrict__ K, const T *__restrict__ dO,
                                                                       const char *__restrict__ prepared, T *__restrict__ dV, BackStates st,
                                                                       DeltaCall a) {
    using L = Back<T, D, DV, SPLIT>;
    using P = typename L::P;
    using Pr = Prepared<T>;
    constexpr int KB = L::KB, MADE = P::MADE, GT = P::GRAD_TILES;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const Lane ln(threadIdx.x);
    const int wave = wave_id(), part = SPLIT == 1 ? 0 : wave / L::CW, cw = wave - part * L::CW, v0 = L::GROUPS == 1 ? 0 : blockIdx.y * L::COLS, c0 = v0 + 32 * cw,
              d0 = 32 * KB * part, seg = blockIdx.x % a.segments, bh = blockIdx.x / a.segments, b = bh / a.H, h = bh - b * a.H;
    if (LOCAL && seg == 0) return;
    const int tokens = a.valid(b, 0, a.N), end = min(a.tiles, (seg + 1) * a.seg_tiles);
    const int t0 = seg * a.seg_tiles, t1 = min(end, (tokens + kTile - 1) / kTile);
    const size_t key_row = a.key_row(b, h), row = (size_t)bh * a.N;
    f32x16 S[KB];
    load_state<KB, DV>(S, ln, LOCAL || !st.last ? nullptr : st.last + (((size_t)bh * a.segments + seg) * D + d0) * DV + c0);
    if (!LOCAL && part == 0)
        for (int t = max(t0, tokens / kTile); t < end; ++t)
            zero_rows<DV>(dV + (row + t * kTile) * DV + c0, ln, tokens - t * kTile, min(a.N - t * kTile, kTile));
    Fetch<T, kTile, D, L::NT> fk, fq;
    Fetch<T, kTile, L::COLS, L::NT> fo;
    Copy<Pr::BYTES, L::NT> fp;
    auto fetch = [&](int t) {
        const int token0 = t * kTile, valid = min(tokens - token0, kTile);
        fp.load(prepared + ((size_t)bh * a.tiles + t) * Pr::BYTES);
        fk.load(K + (key_row + token0) * D, D, valid);
        fq.load(Q + (key_row + token0) * D, D, valid);
        fo.load(dO + (row + token0) * DV + v0, DV, valid);
    };
    if (t0 < t1) fetch(t1 - 1);
    Marks<L::COLS> &marks = *(Marks<L::COLS> *)(lds + L::MARKS);   // (LOCAL needs none)
    if constexpr (!LOCAL) {
        marks.clear();
        __syncthreads();
    }
    for (int t = t1 - 1; t >= t0; --t) {
        const int token0 = t * kTile, valid = min(tokens - token0, kTile);
        unsigned char *at = lds + t % L::STAGES * L::STAGE;
        const typename L::Data kt{(bf16_t *)(at + L::K)}, qt{(bf16_t *)(at + L::Q)};
        const typename L::Grad dot{(bf16_t *)(at + L::DO)};
        const typename Pr::Square nt{(bf16_t *)(at + Pr::N)}, pt{(bf16_t *)(at + Pr::P)};
        if (L::STAGES == 1) __syncthreads();
        const int number = a.tiles - t;
        if constexpr (!LOCAL) {   // what is broken reaches the tokens up to it
            auto token = [&](int row, int) { marks.mark(marks.keys[number & 1], number, row + 1); };
            if (fk.looks_broken()) fk.drop(token);
            if (fq.looks_broken()) fq.drop(token);
            if (fo.looks_broken()) fo.drop([&](int row, int col) { marks.mark(marks.cols[number & 1][col], number, row + 1); });
        }
        fp.store(at);
        fk.store(kt);
        fq.store(qt);
        fo.store(dot);
        __syncthreads();
        if (t > t0) fetch(t - 1);
        if constexpr (!LOCAL)
            if (t % GT == GT - 1 || t == t1 - 1) save_state<KB, DV>(S, ln, st.grads + (((size_t)bh * a.grad_tiles + t / GT) * D + d0) * DV + c0);
        f32x16 du = {};   // a row per token
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int m = 0; m < 2; ++m) du = mm<MADE>(kt.kp(ln, 0, d0 + 32 * kb, m), split<MADE>(S[kb], m), du);
        du *= by_row((const float *)(at + Pr::REST), ln);
        const float whole = *(const float *)(at + Pr::WHOLE);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) S[kb] *= whole;
#pragma unroll
        for (int f = 0; f < kTile / 16; ++f) {
            const auto go = dot.ks(ln, 16 * f, c0 - v0);
            if (SPLIT == 1 || part == f) du = mm<MADE>(pt.ks(ln, 16 * f), go, du);
            f32x8 y = {};   // Q^T (exp(G) dO)
#pragma unroll
            for (int i = P::DATA - 1; i >= 0; --i) y += __builtin_convertvector(go.p[i], f32x8);
            const float *start = (const float *)(at + Pr::START) + 16 * f + 8 * ln.h;
            y *= __builtin_shufflevector(*(const f32x4 *)start, *(const f32x4 *)(start + 4), 0, 1, 2, 3, 4, 5, 6, 7);
            const auto s = split<MADE>(y);
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) S[kb] = mm<MADE>(qt.ks(ln, 16 * f, d0 + 32 * kb), s, S[kb]);
        }
        if constexpr (SPLIT == 2) {
            put_tile((float *)(lds + L::XCH + wave * kSquareBytes), ln, du);
            __syncthreads();
            du += get_tile((const float *)(lds + L::XCH + ((1 - part) * L::CW + cw) * kSquareBytes), ln);
        }
        const f32x16 beta = by_row((const float *)(at + Pr::BETA), ln);
        {
            const f32x16 x = beta * du;
#pragma unroll
            for (int m = 0; m < 2; ++m) du = mm<MADE>(nt.ksp(ln, m), split<MADE>(x, m), du);
        }
        if (!LOCAL && marks.at(number)) {
            const int rows = marks.rows(number, c0 - v0 + ln.r);
#pragma unroll
            for (int e = 0; e < 16; ++e) du[e] = ln.acc_row(e) < rows ? __builtin_nanf("") : du[e];
        }
        const f32x16 dv = beta * du;
        if constexpr (!LOCAL) {
            const size_t to = (row + token0) * DV + c0;
            if (part == 0) store_rows<DV>(st.dr + to, ln, valid, du);
            if (part == SPLIT - 1) store_rows<DV>(dV + to, ln, valid, dv);
        }
        const f32x16 z = -dv * by_row((const float *)(at + Pr::START), ln);
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const auto f = split<MADE>(z, m);
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) S[kb] = mm<MADE>(kt.ksp(ln, 0, d0 + 32 * kb, m), f, S[kb]);
        }
    }
    if (LOCAL) save_state<KB, DV>(S, ln, st.local + (((size_t)bh * a.segments + seg) * D + d0) * DV + c0);
    else if (seg == 0) save_state<KB, DV>(S, ln, st.first + ((size_t)bh * D + d0) * DV + c0);
}

// ---------------------------------------------------------------------------
// k_delta_grad: a tile's gradients, from the state in front of it, the gradient of the one behind it, w and dR, 64 value features at a time. A wave
// has 32 key features of dQ and dK; its rows of both states come from memory straight into its registers, as they are read once.
// 32768 tokens x 16 heads of 128, bfloat16: 608 us, 4.6 KB a token and head (3.9 TB/s), two workgroups of four waves a CU, as LDS has room for. (With
// loads that a branch may leave out, every wait was one for all of them: 640; keys of 64, 8 x 4096 x 8 heads, 257 us against 235.)
// ---------------------------------------------------------------------------
template <int C>
struct Gates {
    double sum[C];
    float start[C], rest[C], beta[C];   // exp(G_i), exp(G_C - G_i)
    float whole;
    int spoilt;   // something in the tile is broken
};
template <typename T, int D>
struct Grad {
    using P = Parts<T>;
    static constexpr int NB = P::GRAD_TILES, C = NB * kTile, COLS = NB == 2 ? 32 : 64, SLICES = D / 32;
    static constexpr int PER = SLICES * NB > 4 ? NB : 1, WAVES = SLICES * NB / PER, NT = 64 * WAVES;   // PER: token blocks of a wave
    typedef Tile<P::DATA, C, D> Data;
    typedef Lower<P::ROUNDED, C> Square;
    typedef Tile<P::MADE, C, COLS> Rows;
    typedef Tile<P::DATA, C, COLS> Out;
    static constexpr int JOBS = 2 * Square::BLOCKS, MINE = (JOBS + WAVES - 1) / WAVES;   // blocks of Ep and of Em; of a wave
    struct Sums {   // by token: dbeta, sums of Z (of a block), x and y (of a wave's key features); <dS, S>
        float beta[C], row[JOBS][32], col[JOBS][32], up[SLICES][C], on[SLICES][C], both[SLICES];
    };
    static constexpr int PAIR = Rows::BYTES > Square::BYTES ? Rows::BYTES : Square::BYTES;   // (Ep and Em take the places of w and dR)
    static constexpr int K = 0, Q = K + Data::BYTES, W = Q + Data::BYTES, DR = W + PAIR, DO = DR + PAIR, G = DO + Out::BYTES,
                         LDS = G + (int)((sizeof(Gates<C>) + 15) / 16 * 16);
    static_assert(sizeof(Sums) <= Out::BYTES, "the sums take the place of dO");
    // waves a SIMD: as many workgroups a CU as LDS has room for
    static constexpr int PER_SIMD = NB == 2 ? (163840 / LDS * WAVES) / 4 : 1;
};
// Sums over the 32 lanes of a half wave of 16 values: lane r gets that of value r / 2 (two lanes each). By halves: 16 exchanges. (By masks: a
// choice between elements of a vector would be compiled as an index into it.)
DEVI float choose(unsigned mask, float a, float b) { return __uint_as_float((__float_as_uint(a) & mask) | (__float_as_uint(b) & ~mask)); }
DEVI float sum_lanes(const f32x16 &z, const Lane &ln) {
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = z[i];
#pragma unroll
    for (int n = 8; n > 0; n /= 2) {   // lanes 2 n apart keep n values each
        const unsigned up = ln.r & 2 * n ? ~0u : 0u;
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = choose(up, v[n + i], v[i]) + __shfl_xor(choose(up, v[i], v[n + i]), 2 * n);
    }
    return v[0] + __shfl_xor(v[0], 1);
}
// Row i: the sum of the rows in front of it, of a tile with a row per register.
DEVI f32x16 rows_before(const f32x16 &z, const Lane &ln) {
    f32x16 x;
    float all = 0.0f;   // of both halves' rows in front of the four
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const float two = z[4 * g] + z[4 * g + 1], three = two + z[4 * g + 2], four = three + z[4 * g + 3], other = __shfl_xor(four, 32);
        const float from = ln.h ? all + other : all;
        x[4 * g] = from;
        x[4 * g + 1] = from + z[4 * g];
        x[4 * g + 2] = from + two;
        x[4 * g + 3] = from + three;
        all += four + other;
    }
    return x;
}
template <typename T, int D, typename TO>
__global__ __launch_bounds__((Grad<T, D>::NT), (Grad<T, D>::PER_SIMD)) void k_delta_grad(const T *__restrict__ Q, const T *__restrict__ K,
                                                                                   const T *__restrict__ dO, const float *__restrict__ states,
                                                                                   const float *__restrict__ grads, const float *__restrict__ w,
                                                                                   const float *__restrict__ dR, TO *__restrict__ dQ,
                                                                                   TO *__restrict__ dK, float *__restrict__ dbeta,
                                                                                   float *__restrict__ dlog_g, DeltaCall a) {
    using L = Grad<T, D>;
    using P = typename L::P;
    constexpr int C = L::C, NB = L::NB, COLS = L::COLS, MADE = P::MADE, NT = L::NT, MINE = L::MINE, PER = L::PER;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const typename L::Data kt{(bf16_t *)(lds + L::K)}, qt{(bf16_t *)(lds + L::Q)};
    const typename L::Rows wt{(bf16_t *)(lds + L::W)}, rt{(bf16_t *)(lds + L::DR)};
    const typename L::Out dot{(bf16_t *)(lds + L::DO)};
    const typename L::Square ep{wt.p}, em{rt.p};
    Gates<C> &g = *(Gates<C> *)(lds + L::G);
    typename L::Sums &red = *(typename L::Sums *)(lds + L::DO);
    const Lane ln(threadIdx.x);
    const int wave = wave_id(), tile = blockIdx.x, bh = blockIdx.y, b = bh / a.H, h = bh - b * a.H, token0 = tile * C;
    const int valid = a.valid(b, token0, C), there = min(a.N - token0, C);
    const size_t key_row = a.key_row(b, h), row = (size_t)bh * a.N + token0;
    if (valid == 0) {
        for (int e = threadIdx.x; e < there * D; e += NT) {
            Elem<TO>::st1(dQ + row * D + e, 0.0f);
            Elem<TO>::st1(dK + row * D + e, 0.0f);
        }
        if ((int)threadIdx.x < there) {
            dbeta[row + threadIdx.x] = 0.0f;
            if (dlog_g) dlog_g[row + threadIdx.x] = 0.0f;
        }
        return;
    }
    const int slice = wave % L::SLICES, d0 = 32 * slice, tk0 = wave / L::SLICES * PER;   // a wave's 32 key features and first block of tokens
    // a wave's blocks of Ep (even) and Em (odd)
    auto job = [&](int n) { return wave + n * L::WAVES; };
    auto token_block = [](int j) { return j >= 2 ? 1 : 0; };
    auto key_block = [](int j) { return j >= 4 ? 1 : 0; };
    // What is read once is on its way before it is needed: the next columns' rows while these are used, a state's next piece as soon as the one
    // before has been split.
    Fetch<float, C, COLS, NT> fw, fr;
    Fetch<T, C, COLS, NT> fo;
    f32x4 s4[COLS / 16][2], d4[COLS / 16][2];
    auto fetch_rows = [&](int c0) {
        fw.load(w + row * a.Dv + c0, a.Dv, valid);
        fr.load(dR + row * a.Dv + c0, a.Dv, valid);
        fo.load(dO + row * a.Dv + c0, a.Dv, valid);
    };
    const size_t state = (((size_t)bh * a.grad_tiles + tile) * D + d0) * a.Dv;
    const unsigned piece = (ln.r * a.Dv + 8 * ln.h) * 4;
    auto fetch_states = [&](int c0, int k) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s4[k][i] = gload<f32x4>(states + state + c0, piece + 64 * k + 16 * i);
            d4[k][i] = gload<f32x4>(grads + state + c0, piece + 64 * k + 16 * i);
        }
    };
    {
        Fetch<T, C, D, NT> fk, fq;
        fk.load(K + (key_row + token0) * D, D, valid);
        fq.load(Q + (key_row + token0) * D, D, valid);
        const bool in = wave == 0 && ln.id < valid;
        const float lg = a.log_g && in ? a.log_g[row + ln.id] : 0.0f, bt = in ? a.beta[row + ln.id] : 0.0f;
        fetch_rows(0);
#pragma unroll
        for (int k = 0; k < COLS / 16; ++k) fetch_states(0, k);
        if (wave == 0) {
            const double x = sum_up<C>(to_base2(lg), ln.id), all = __shfl(x, C - 1, C);
            if (ln.id < C) {
                g.sum[ln.id] = x;
                g.start[ln.id] = power(x);
                g.rest[ln.id] = power(all - x);
                g.beta[ln.id] = bt;
            }
            if (ln.id == 0) {
                g.whole = power(all);
                g.spoilt = 0;
            }
        }
        fk.store(kt);
        fq.store(qt);
    }
    f32x16 pr[MINE] = {};                              // w dO^T or w dR^T, a row per key token
    f32x16 aq[PER] = {}, a1[PER] = {}, a2[PER] = {};   // S dO^T, S dR^T, dS w^T, a row per key feature
    float both = 0.0f;                                 // <dS, S>
    auto columns = [&](int c0, auto next) {
        constexpr bool more = next;
        const Lane ln = fresh_lane();   // (offsets that all rounds share take the registers of what is on its way, and are reloaded from memory behind it)
        int c1 = c0 + COLS;
        asm volatile("" : "+s"(c1));   // (not seen through: addresses then stay a scalar base and 32 bits a lane, where pointers that are counted up spill)
        if (c0 > 0) __syncthreads();   // the tiles have been read
        fo.store(dot);
        fw.store(wt);
        fr.store(rt);
        __syncthreads();
        if constexpr (more) fetch_rows(c1);
#pragma unroll
        for (int k = 0; k < COLS / 16; ++k) {
            const auto fs = split<MADE>(__builtin_shufflevector(s4[k][0], s4[k][1], 0, 1, 2, 3, 4, 5, 6, 7));
            const auto fd = split<MADE>(__builtin_shufflevector(d4[k][0], d4[k][1], 0, 1, 2, 3, 4, 5, 6, 7));
            if (tk0 == 0)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) both = __builtin_fmaf(s4[k][i][e], d4[k][i][e], both);
            if constexpr (more) fetch_states(c1, k);
#pragma unroll
            for (int n = 0; n < PER; ++n) {
                aq[n] = mm<MADE>(fs, dot.kc(ln, 32 * (tk0 + n), 16 * k), aq[n]);
                a1[n] = mm<MADE>(fs, rt.kc(ln, 32 * (tk0 + n), 16 * k), a1[n]);
                a2[n] = mm<MADE>(fd, wt.kc(ln, 32 * (tk0 + n), 16 * k), a2[n]);
            }
        }
#pragma unroll
        for (int n = 0; n < MINE; ++n)
            if (job(n) < L::JOBS) {
                const int j = job(n), tb = token_block(j), jb = key_block(j);
                if (j & 1)
#pragma unroll
                    for (int k0 = 0; k0 < COLS; k0 += 16) pr[n] = mm<MADE>(wt.kc(ln, 32 * jb, k0), rt.kc(ln, 32 * tb, k0), pr[n]);
                else
#pragma unroll
                    for (int k0 = 0; k0 < COLS; k0 += 16) pr[n] = mm<MADE>(wt.kc(ln, 32 * jb, k0), dot.kc(ln, 32 * tb, k0), pr[n]);
            }
    };
    for (int c0 = 0; c0 < a.Dv - COLS; c0 += COLS) columns(c0, std::true_type{});
    columns(a.Dv - COLS, std::false_type{});
    __syncthreads();
    // dlog_a_i = exp(G_C) <dS, S> + sum_{t >= i} x_t + sum_{j < i} y_j + sum_{t >= i > j} Z_tj: what goes through gate i and nothing else, with
    // x_t = exp(G_t) (q_t . S dO_t - k_t . S dV_t), y_j = exp(G_C - G_j) k_j . dS u_j and Z = Ep q.k + Em k.k. The last one without a difference of sums: of a block on the
    // diagonal a sum for every gate; of the one below it, its columns in front of the gate for the first 32 tokens, its rows from the gate on for the others.
#pragma unroll
    for (int n = 0; n < MINE; ++n)
        if (job(n) < L::JOBS) {
            const int jo = job(n), tb = token_block(jo), jb = key_block(jo), i = 32 * tb + ln.r;
            const bool is_em = jo & 1;
            if (any_broken(pr[n])) g.spoilt = 1;   // (a broken key has spoilt its w, a broken query its dR)
            f32x16 z = {};   // k_j . q_i or k_j . k_i
            if (dlog_g) {
                const typename L::Data other{is_em ? kt.p : qt.p};
#pragma unroll
                for (int k0 = 0; k0 < D; k0 += 16) z = mm<MADE>(kt.kc(ln, 32 * jb, k0), other.kc(ln, 32 * tb, k0), z);
            }
            float diagonal = 0.0f;
            const float bi = is_em ? -g.beta[i] : 1.0f;
            const f32x16 x = weights_by_row<false>(g.sum + 32 * jb, g.sum[i], ln) * by_row(g.beta + 32 * jb, ln) * bi;
            const int last = 32 * (tb - jb) + ln.r - is_em;   // rows up to here are keys that the token sees
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int o = ln.acc_row(e);
                diagonal = o == ln.r ? pr[n][e] : diagonal;
                const float v = pr[n][e] * x[e];
                pr[n][e] = o <= last ? v : 0.0f;
                z[e] = o < 32 * (tb - jb) + ln.r ? v * z[e] : 0.0f;
            }
            if (is_em && tb == jb && ln.h == (ln.r >> 2 & 1)) red.beta[i] = diagonal;   // dbeta_i = w_i . dR_i
            if (dlog_g) {
                if (tb == jb) {
                    z = rows_before(z, ln);
#pragma unroll
                    for (int e = 0; e < 16; ++e) z[e] = ln.r >= ln.acc_row(e) ? z[e] : 0.0f;
                } else {
                    float along = 0.0f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) along += z[e];
                    along += __shfl_xor(along, 32);
                    if (ln.h == 0) red.row[jo][ln.r] = along;
                }
                const float down = sum_lanes(z, ln);
                if ((ln.r & 1) == 0) red.col[jo][ln.acc_row(ln.r >> 1)] = down;
            }
            const auto to = is_em ? em.at(tb, jb) : ep.at(tb, jb);
            to.st_acc(ln, pr[n]);
        }
    __syncthreads();
    if (__builtin_expect(g.spoilt, 0)) {   // Ep and Em hold zeros for tokens that a broken one does not reach, NaN for those that it does
        for (int e = threadIdx.x; e < 2 * L::Data::BYTES / 16; e += NT) ((u32x4 *)(lds + L::K))[e] = drop_broken(((const u32x4 *)(lds + L::K))[e]);
        __syncthreads();
    }
#pragma unroll
    for (int n = 0; n < PER; ++n) {
        const int tk = tk0 + n, m = 32 * tk + ln.r;
        const float start = g.start[m], rest = g.rest[m];
        const size_t to = (row + m) * D + d0;   // (shared heads: a partial sum for every state, in float)
        f32x16 x = aq[n] * start, z = a1[n] * (start * g.beta[m]), y = a2[n] * (rest * g.beta[m]);
        if (dlog_g) {
            float up = 0.0f, on = 0.0f;
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const f32x4 q4 = qt.get4(m, d0 + 8 * f + 4 * ln.h), k4 = kt.get4(m, d0 + 8 * f + 4 * ln.h);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    up = __builtin_fmaf(q4[e], x[4 * f + e], __builtin_fmaf(-k4[e], z[4 * f + e], up));
                    on = __builtin_fmaf(k4[e], y[4 * f + e], on);
                }
            }
            up += __shfl_xor(up, 32);
            on += __shfl_xor(on, 32);
            if (ln.h == 0) {
                red.up[slice][m] = up;
                red.on[slice][m] = on;
            }
        }
        for (int jb = 0; jb <= tk; ++jb)
#pragma unroll
            for (int k0 = 0; k0 < 32; k0 += 16) x = mm<P::ROUNDED>(kt.ks(ln, 32 * jb + k0, d0), ep.at(tk, jb).kc(ln, k0), x);
        if (m < valid) store_acc(dQ + to, ln, x);
        else if (m < there) store_acc(dQ + to, ln, f32x16{});
        y -= z;
        for (int it = tk; it < NB; ++it)
#pragma unroll
            for (int k0 = 0; k0 < 32; k0 += 16) {
                y = mm<P::ROUNDED>(qt.ks(ln, 32 * it + k0, d0), ep.at(it, tk).ks(ln, k0), y);
                y = mm<P::ROUNDED>(kt.ks(ln, 32 * it + k0, d0), em.at(it, tk).ks(ln, k0), y);
            }
        for (int jb = 0; jb <= tk; ++jb)
#pragma unroll
            for (int k0 = 0; k0 < 32; k0 += 16) y = mm<P::ROUNDED>(kt.ks(ln, 32 * jb + k0, d0), em.at(tk, jb).kc(ln, k0), y);
        if (m < valid) store_acc(dK + to, ln, y);
        else if (m < there) store_acc(dK + to, ln, f32x16{});
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) both += __shfl_xor(both, d);
    if (ln.id == 0 && tk0 == 0) red.both[slice] = both;
    __syncthreads();
    if (wave != 0) return;
    if (ln.id < there) dbeta[row + ln.id] = ln.id < valid ? red.beta[ln.id] : 0.0f;
    if (!dlog_g) return;
    const bool in = ln.id < C, first = ln.id < 32;
    double up = 0.0, on = 0.0, across = 0.0, all = 0.0, z = 0.0;   // x_t; y of the token in front; sums of Z below the diagonal
    if (in) {
#pragma unroll
        for (int v = 0; v < L::SLICES; ++v) {
            up += red.up[v][ln.id];
            on += ln.id > 0 ? red.on[v][ln.id - 1] : 0.0f;
        }
#pragma unroll
        for (int v = 0; v < L::JOBS; ++v) {
            if (token_block(v) != key_block(v)) across += !first ? red.row[v][31 - ln.r] : ln.r > 0 ? red.col[v][ln.r - 1] : 0.0f;   // (rows from the last one on)
            else if (key_block(v) == ln.id / 32) z += red.col[v][ln.r];
        }
    }
#pragma unroll
    for (int v = 0; v < L::SLICES; ++v) all += red.both[v];
    on = sum_up<C>(on, ln.id);
    if constexpr (NB == 2) {
        across = sum_up<32>(across, ln.id);
        const double back = __shfl_xor(across, 31);
        z += first ? across : back;
    }
#pragma unroll
    for (int d = 1; d < C; d *= 2) {
        const double y = __shfl_down(up, d, C);
        if ((ln.id & (C - 1)) + d < C) up += y;
    }
    if (ln.id < there) {
        const bool none = ln.id >= valid || to_base2(a.log_g[row + ln.id]) < kLeastGate;   // (a gate of 0 has no slope)
        dlog_g[row + ln.id] = none ? 0.0f : (float)(g.whole * all + up + on + z);
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
    size_t states, inv, trans, back, w, cache;                // cache
    size_t own_inv, own_trans, local, first, scratch;         // forward scratch
    size_t grads, dr, back_local, last, part, back_scratch;   // backward scratch
};
Layout layout(const DeltaPlan &p) {
    Layout l{};
    const size_t bh = (size_t)p.B * p.H, state = (size_t)p.D * p.Dv * 4, rows = bh * p.N * p.Dv * 4;
    const size_t inv = bh * p.tiles * (p.dtype == 0 ? Prepared<float>::BYTES : Prepared<bf16_t>::BYTES), between = p.segments > 1 ? bh * p.segments * state : 0;
    const size_t trans = p.segments > 1 ? bh * p.segments * p.D * p.D * 4 : 0;
    l.inv = up(bh * p.grad_tiles * state);
    l.trans = l.inv + up(inv);
    l.back = l.trans + up(trans);
    l.w = l.back + up(trans);
    l.cache = l.w + up(rows);
    l.own_trans = up(inv);
    l.local = l.own_trans + up(trans);
    l.first = l.local + up(between);
    l.scratch = l.first + up(between);
    l.dr = up(bh * p.grad_tiles * state);
    l.back_local = l.dr + up(rows);
    l.last = l.back_local + up(between);
    l.part = l.last + up(between);
    l.back_scratch = l.part + (p.key_heads < p.H ? 2 * up(bh * p.N * p.D * 4) : 0);
    return l;
}
DeltaCall call_of(const DeltaPlan &p, const DeltaArgs &a) {
    return {p.B, p.H, p.key_heads, p.N, p.Dv, p.tiles, p.segments, p.seg_tiles, p.grad_tiles, a.log_g, a.beta, a.len};
}
// f.template operator()<T, D, DV>()
template <typename T, typename F>
hipError_t by_dims(const DeltaPlan &p, F f) {
    if (p.D == 128) return p.Dv == 128 ? f.template operator()<T, 128, 128>() : f.template operator()<T, 128, 64>();
    return p.Dv == 128 ? f.template operator()<T, 64, 128>() : f.template operator()<T, 64, 64>();
}
template <typename F>
hipError_t by_type(const DeltaPlan &p, F f) { return p.dtype == 0 ? by_dims<float>(p, f) : by_dims<bf16_t>(p, f); }
template <typename K>
hipError_t room(K kernel, size_t bytes) { return allow_dynamic_lds((const void *)kernel, bytes); }

struct Forward {
    const DeltaPlan &p;
    const DeltaArgs &a;
    hipStream_t s;
    template <typename T, int D, int DV>
    hipError_t operator()() const {
        const DeltaCall c = call_of(p, a);
        const int bh = p.B * p.H;
        const T *q = (const T *)a.q, *k = (const T *)a.k, *v = (const T *)a.v;
        // Token by token (16 heads of 128): bf16, 1 sequence 11 us for 4 tokens, 19 for 16, in a tile 13; 64 sequences 36 for 4, 63 for 8,
        // 115 for 16, in a tile 42. Float: 11 for 8 and 62 for 8, in a tile 17 and 67.
        if (!a.cache && p.N <= delta_step_tokens(p)) {
            // narrower blocks of columns where 32 would not give every CU two workgroups (64 sequences: 23 us with 32, 33 with 16;
            // one: 13 and 10)
            if (bh * (DV / 32) >= 2 * kCus)
                k_delta_step<T, D, 32><<<dim3(bh * (DV / 32)), dim3(kThreads), 0, s>>>(q, k, v, a.kv_in, (T *)a.out, a.kv_out, c);
            else
                k_delta_step<T, D, 16><<<dim3(bh * (DV / 16)), dim3(kThreads), 0, s>>>(q, k, v, a.kv_in, (T *)a.out, a.kv_out, c);
            return hipGetLastError();
        }
        const Layout l = layout(p);
        char *sc = (char *)a.scratch, *ca = (char *)a.cache;
        char *inv = ca ? ca + l.inv : sc;
        float *trans = (float *)(ca ? ca + l.trans : sc + l.own_trans), *back = (float *)(ca ? ca + l.back : nullptr), *local = (float *)(sc + l.local), *first = (float *)(sc + l.first);
        k_delta_prep<T, D><<<dim3((p.tiles + kWaves - 1) / kWaves, bh), dim3(kThreads), 0, s>>>(q, k, inv, c);
        WalkStates st{a.kv_in, a.kv_out, local, trans, back, (float *)ca, (float *)(ca ? ca + l.w : nullptr), ca != nullptr};
        if (p.segments > 1) {
            if (hipError_t e = walk<T, D, DV, true>(nullptr, k, v, inv, nullptr, st, c); e != hipSuccess) return e;
            k_delta_scan<D, false><<<dim3(bh, DV / kScanCols), dim3(4 * D), 0, s>>>(a.kv_in, trans, local, first, DV, p.segments);
            st.first = first;
        }
        return walk<T, D, DV, false>(q, k, v, inv, (T *)a.out, st, c);
    }
    template <typename T, int D, int DV, bool LOCAL>
    hipError_t walk(const T *q, const T *k, const T *v, const char *inv, T *out, const WalkStates &st, const DeltaCall &c) const {
        return p.split ? walk<T, D, DV, LOCAL, 2>(q, k, v, inv, out, st, c) : walk<T, D, DV, LOCAL, 1>(q, k, v, inv, out, st, c);
    }
    template <typename T, int D, int DV, bool LOCAL, int SPLIT>
    hipError_t walk(const T *q, const T *k, const T *v, const char *inv, T *out, const WalkStates &st, const DeltaCall &c) const {
        typedef Walk<T, D, DV, LOCAL, SPLIT> L;
        if (hipError_t e = room(k_delta_walk<T, D, DV, LOCAL, SPLIT>, L::LDS); e != hipSuccess) return e;
        k_delta_walk<T, D, DV, LOCAL, SPLIT><<<dim3(p.segments * p.B * p.H, L::GROUPS), dim3(L::NT), L::LDS, s>>>(q, k, v, inv, out, st, c);
        return hipGetLastError();
    }
};

struct Backward {
    const DeltaPlan &p;
    const DeltaArgs &a;
    hipStream_t s;
    template <typename T, int D, int DV>
    hipError_t operator()() const {
        const DeltaCall c = call_of(p, a);
        const int bh = p.B * p.H;
        const T *q = (const T *)a.q, *k = (const T *)a.k, *v = (const T *)a.v, *dout = (const T *)a.dout;
        const Layout l = layout(p);
        char *sc = (char *)a.scratch, *ca = (char *)a.cache;
        const char *inv = ca + l.inv;
        float *last = (float *)(sc + l.last);
        BackStates st{a.dkv_out, a.dkv_in, (float *)(sc + l.back_local), (float *)sc, (float *)(sc + l.dr)};
        if (p.segments > 1) {
            if (hipError_t e = back<T, D, DV, true>(q, k, dout, inv, nullptr, st, c); e != hipSuccess) return e;
            k_delta_scan<D, true><<<dim3(bh, DV / kScanCols), dim3(4 * D), 0, s>>>(a.dkv_out, (const float *)(ca + l.back), st.local, last, DV,
                                                                                   p.segments);
            st.last = last;
        }
        if (hipError_t e = back<T, D, DV, false>(q, k, dout, inv, (T *)a.dv, st, c); e != hipSuccess) return e;
        if (p.key_heads == p.H) return grad<T, D>(c, (T *)a.dq, (T *)a.dk, st, l);
        const size_t n = (size_t)bh * p.N * D;
        float *part = (float *)(sc + l.part);
        if (hipError_t e = grad<T, D>(c, part, part + n, st, l); e != hipSuccess) return e;
        const int share = p.H / p.key_heads;
        k_delta_group<T, D><<<dim3((unsigned)((n / share / 4 + kThreads - 1) / kThreads), 2), dim3(kThreads), 0, s>>>(part, (T *)a.dq, (T *)a.dk, n, share,
                                                                                                             p.N);
        return hipGetLastError();
    }
    template <typename T, int D, int DV, bool LOCAL>
    hipError_t back(const T *q, const T *k, const T *dout, const char *inv, T *dv, const BackStates &st, const DeltaCall &c) const {
        return p.split ? back<T, D, DV, LOCAL, 2>(q, k, dout, inv, dv, st, c) : back<T, D, DV, LOCAL, 1>(q, k, dout, inv, dv, st, c);
    }
    template <typename T, int D, int DV, bool LOCAL, int SPLIT>
    hipError_t back(const T *q, const T *k, const T *dout, const char *inv, T *dv, const BackStates &st, const DeltaCall &c) const {
        typedef Back<T, D, DV, SPLIT> L;
        if (hipError_t e = room(k_delta_back<T, D, DV, LOCAL, SPLIT>, L::LDS); e != hipSuccess) return e;
        k_delta_back<T, D, DV, LOCAL, SPLIT><<<dim3(p.segments * p.B * p.H, L::GROUPS), dim3(L::NT), L::LDS, s>>>(q, k, dout, inv, dv, st, c);
        return hipGetLastError();
    }
    template <typename T, int D, typename TO>
    hipError_t grad(const DeltaCall &c, TO *dq, TO *dk, const BackStates &st, const Layout &l) const {
        if (hipError_t e = room(k_delta_grad<T, D, TO>, Grad<T, D>::LDS); e != hipSuccess) return e;
        k_delta_grad<T, D, TO><<<dim3(p.grad_tiles, p.B * p.H), dim3(Grad<T, D>::NT), Grad<T, D>::LDS, s>>>(
            (const T *)a.q, (const T *)a.k, (const T *)a.dout, (const float *)a.cache, st.grads,
            (const float *)((const char *)a.cache + l.w), st.dr, dq, dk, a.dbeta, a.dlog_g, c);
        return hipGetLastError();
    }
};

}  // namespace

// Segments: a walk takes the longer the fewer workgroups it has. Cutting a sequence costs a second walk (the local one, over twice the
// columns) and a chain of one step a segment: two workgroups a CU are looked for, a segment has two tiles or more, the chain is kept to a
// part of the walk, and fewer than five segments do not pay, also where that leaves CUs without a workgroup. (Forward, bf16, heads of 128: 8 x 1777 tokens
// x 16 heads 234 us uncut, 327 in four; 7 x 4096 x 16 474 and 581, values of 64 477 and 505, 7 x 16384 x 16 1880 and 2170; 16384 x 8 heads 230 us in 32
// segments, 1570 uncut. Forward and backward: 32768 x 16 heads 2.0 ms in 32 segments, 7.7 uncut; 8 x 4096 x 8 heads with keys of 64 672 us in eight, 921 uncut. The
// chain's part, on an earlier state of these kernels: 32768 x 16 heads 2.03 ms in 32 as in 16, 2.2 in 48; 4096 x 16 heads 372 us in 16, 424 in 26, 396 in 11.)
// split: a second wave to every 32 columns, which takes half of the key features, as long as every such workgroup has a CU to itself. (The
// two meet once a tile: 8 x 1777 x 16 heads 234 us with it and 277 without, 7 x 4096 x 16 474 and 606, float, 2 x 1001 x 4 heads, forward and backward 149 and 197;
// beyond that it costs: 12 x 1777 x 16 heads 407 us with it, 298 without.)
DeltaPlan delta_plan(int B, int H, int N, int D, int Dv, int dtype, int key_heads) {
    DeltaPlan p{B, H, N, D, Dv, dtype, key_heads};
    p.tiles = (int)(((long long)N + kTile - 1) / kTile);
    const int together = dtype == 0 ? Parts<float>::GRAD_TILES : Parts<bf16_t>::GRAD_TILES;
    p.grad_tiles = (p.tiles + together - 1) / together;
    const long long walks = (long long)B * H;
    int cut = (int)std::min<long long>(2 * kCus / std::min<long long>(walks, 2 * kCus), p.tiles / 2);
    while (cut > 1 && (long long)cut * cut > 2LL * p.tiles) --cut;
    if (cut < 5) cut = 1;
    p.seg_tiles = ((p.tiles + cut - 1) / cut + together - 1) / together * together;
    p.segments = (p.tiles + p.seg_tiles - 1) / p.seg_tiles;
    p.split = walks * p.segments * (Dv / kSplitCols) <= kCus;
    return p;
}
size_t delta_cache(const DeltaPlan &p) { return layout(p).cache; }
size_t delta_scratch(const DeltaPlan &p) { return layout(p).scratch; }
size_t delta_bwd_scratch(const DeltaPlan &p) { return layout(p).back_scratch; }
hipError_t launch_delta_fwd(const DeltaPlan &p, const DeltaArgs &a, hipStream_t s) { return by_type(p, Forward{p, a, s}); }
hipError_t launch_delta_bwd(const DeltaPlan &p, const DeltaArgs &a, hipStream_t s) { return by_type(p, Backward{p, a, s}); }

}  // namespace lasp
