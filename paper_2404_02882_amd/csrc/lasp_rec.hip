// HIP kernels (gfx950 / CDNA4) for the gated linear recurrence h_s = a_s h_{s-1} + b_s x_s, a_s = exp(log_a_s), elementwise
// over channels: the vector-state member of the recurrences of LASP (arxiv 2404.02882) App. A.4, Table 6.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>

#include "lasp_block.h"

namespace lasp {

// The gate of one token, or the product of several (log_a summed, up to 88): a step of the recurrence is y -> a y + u.
template <typename T>
struct Gate;
// bfloat16 data: a as a float, off by at most a step of 2^-24, which is at most N 2^-24 of a state after N tokens. 1 - a to a relative 2^-12, an
// eighth of what rounding to bfloat16 does at most, however near to 1 a is: from -2^-11 on as -log_a (what is left out is log_a / 2 of it),
// elsewhere from the power (off by a step of 2^-24 of 1). Gates near 1 held as float data's are: 32768 x 2048 forward + backward 211 -> 242 us.
template <>
struct Gate<bf16_t> {
    float w, l;
    DEVI explicit Gate(float log_a) : w(__builtin_amdgcn_exp2f(log_a * 1.44269504f)), l(log_a) {}
    static DEVI Gate of_word(float w) { return Gate(w, 0); }
    DEVI float step(float y, float u) const { return __builtin_fmaf(w, y, u); }
    DEVI float times(float y) const { return w * y; }
    DEVI float b() const { return __builtin_fabsf(l) < 1.0f / 2048 ? -l : 1.0f - w; }

private:
    DEVI Gate(float word, int) : w(word), l(0) {}
};
// Float data: for -1/4 < log_a < 0 the distance a - 1 from 1, by its power series (what is left out, log_a^6 / 7! < 2^-24 of it,
// rounds away), so that 1 - a has 24 bits however near to 1 a is: with a itself 20000 tokens of a = 1 - 1e-6 are 1.4e-4 off, as
// every rounding of a goes the same way. The sign bit tells the two apart. Elsewhere the power: the exponent's rounding,
// |log_a| 2^-24 of a, is at most 2^-25 of 1.
template <>
struct Gate<float> {
    float w;
    DEVI explicit Gate(float l) {
        float q = 1.0f / 720;
        q = __builtin_fmaf(q, l, 1.0f / 120);
        q = __builtin_fmaf(q, l, 1.0f / 24);
        q = __builtin_fmaf(q, l, 1.0f / 6);
        q = __builtin_fmaf(q, l, 0.5f);
        const float m = __builtin_fmaf(l * l, q, l), a = __builtin_amdgcn_exp2f(l * 1.44269504f);
        w = l > -0.25f && l < 0.0f ? m : a;
    }
    static DEVI Gate of_word(float w) { return Gate(w, 0); }
    DEVI bool near() const { return __builtin_bit_cast(int, w) < 0; }
    DEVI float step(float y, float u) const { return __builtin_fmaf(w, y, u) + (near() ? y : 0.0f); }
    DEVI float times(float y) const { return __builtin_fmaf(w, y, near() ? y : 0.0f); }
    DEVI float b() const { return near() ? -w : 1.0f - w; }

private:
    DEVI Gate(float word, int) : w(word) {}
};

// The product of several gates, given their log_a summed, as one word, and a step by that word. Small: sums of up to kMostLog.
constexpr float kMostLog = 88.0f;
template <typename T>
struct SmallProduct {
    static DEVI float word(float l) { return Gate<T>(l).w; }
    static DEVI float step(float w, float y, float u) { return Gate<T>::of_word(w).step(y, u); }
};
// Any: above e^88, which is near the largest float, the word is minus the sum (those of gates lie above -1). Such a product of a state
// of 0 is 0, and that of a tiny state need not be infinite.
template <typename T>
struct AnyProduct {
    static DEVI float word(float l) { return l > kMostLog ? -l : Gate<T>(l).w; }
    static DEVI float step(float w, float y, float u) {
        if (w < -1.0f) {   // e^-w y as 2^n (2^rest y), the rest up to 1/2; from 2^300 on anything but 0 is infinite
            const float e = fminf(w * -1.44269504f, 300.0f), n = __builtin_rintf(e);
            return __builtin_ldexpf(y * __builtin_amdgcn_exp2f(e - n), (int)n) + u;
        }
        return Gate<T>::of_word(w).step(y, u);
    }
};
template <typename T, typename F>
DEVI auto by_product(bool small, F f) {
    if (__all(small)) return f(SmallProduct<T>{});
    return f(AnyProduct<T>{});
}

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
// k_rec_step_fwd / k_rec_step_bwd: a thread carries a column's state over all tokens, kAhead tokens requested together. One token for
// 64 sequences x 2048: 3.2 us, all of it launch and one trip to memory.
// ---------------------------------------------------------------------------
constexpr int kStepThreads = 64, kAhead = 8;

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
// k_rec_tiles: the sequence in tiles, one workgroup each. A thread takes ROWS consecutive rows of a column (in the order of the
// scan: from the first token on, backward from the last one), which it keeps in registers as they were loaded:
//   1. its rows as one step y -> A y + X, joined over the rows of the wave and the waves of the workgroup,
//   2. the tile's step is published, and the state that enters the tile found: the nearest tile in front whose end state
//      is published, and the steps of those between, applied in order,
//   3. its rows again, from the state that enters them, to the outputs.
// So every input is read once and every output written once, which is what bounds it: bfloat16 4 x 16384 x 4096, coupled, 1.6 GB in 291 us,
// backward 3.2 GB in 562, 5.5 and 5.7 TB/s (a copy 4.9). States are applied one tile after the other whatever is
// published when: the same results on every run.
// Workgroups take their tiles from counters, in the order of the scan: a tile waits only for tiles whose workgroups have
// started, and those for none behind them, so every wait ends. Each counter serves a quarter of the column blocks: a single one
// passes a workgroup every 13 ns, which is all the time of short tiles (8 x 1777 x 2048, half of it padding: 40.2 us, with four 35.0).
// One for every block 33.6, but then the blocks drift apart, and rows of memory are opened more than once: 4 x 16384 x 4096
// forward / backward 314 / 608 us, with four 306 / 596. Values carry their own flag: a word that is kEmpty has not
// been published (NaN are published as another one), so no fence is needed.
// ---------------------------------------------------------------------------
constexpr unsigned kEmpty = 0xffffffffu;
DEVI unsigned published(float f) { return f != f ? 0x7fc00000u : __builtin_bit_cast(unsigned, f); }

constexpr int kGroups = 4, kTicketStride = 32;
struct RecLook {                 // in the scratch
    unsigned *tickets;           // [kGroups], a line of 128 bytes each
    unsigned long long *steps;   // [tile][column block][channel]: the gate's word, X
    unsigned *ends;              // [tile][column block][channel]: the state behind the tile
};
template <typename V>
DEVI V look(const V *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename V>
DEVI void show(V *p, V v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// The state that enters a tile for one channel, whose slots in consecutive tiles are `stride` apart, `slot` that of this one. The
// channel's first tile, `back` tiles in front, publishes no step, and nothing in front of it is looked at. NaN after kMostLooks, some
// seconds: only where a call that overlaps in time has cleared the scratch, and the words never come.
constexpr int kMostLooks = 1 << 22;
template <typename T, int BACK>
DEVI float entering(const RecLook &lk, int back, size_t slot, size_t stride) {
    auto at = [&](int k) { return slot - (size_t)min(k + 1, back) * stride; };
    unsigned long long step[BACK];
#pragma unroll
    for (int k = 0; k < BACK; ++k) step[k] = look(lk.steps + at(k));
    for (int looks = 0; looks < kMostLooks; ++looks) {
        unsigned end[BACK];
#pragma unroll
        for (int k = 0; k < BACK; ++k) end[k] = look(lk.ends + at(k));
        float least = 0.0f;               // (a word below -1: a product above e^88)
#pragma unroll
        for (int k = 0; k < BACK; ++k) least = fminf(least, __builtin_bit_cast(float, (unsigned)step[k]));
        int found = -1, missing = BACK;   // nearest end; nearest tile without a step
#pragma unroll
        for (int k = BACK - 1; k >= 0; --k) {
            if (end[k] != kEmpty) found = k;
            if ((unsigned)step[k] == kEmpty) missing = k;
        }
        if (found >= 0 && found <= missing) {
            return by_product<T>(least >= -1.0f, [&](auto p) {
                float y = 0.0f;
#pragma unroll
                for (int k = BACK - 1; k >= 0; --k) {
                    if (k == found) y = __builtin_bit_cast(float, end[k]);
                    else if (k < found) y = p.step(__builtin_bit_cast(float, (unsigned)step[k]), y, __builtin_bit_cast(float, (unsigned)(step[k] >> 32)));
                }
                return y;
            });
        }
        // (a published step stays: asked for again only where one is missing)
        if (missing < BACK) {
#pragma unroll
            for (int k = 0; k < BACK; ++k)
                if ((unsigned)step[k] == kEmpty) step[k] = look(lk.steps + at(k));
        }
        __builtin_amdgcn_s_sleep(1);
    }
    return __builtin_nanf("");
}

// LANES threads side by side along the columns; the others of a wave are further rows. Eight, a line of 128 bytes of every row:
// the fewer columns, the longer the tile and the fewer there are to pass the state on through (bfloat16 32768 x 2048, tiles of
// 4 waves, one counter, no streaming: 64 / 16 / 8 lanes forward 214 / 92 / 88 us, backward 216 / 137 / 134). Rows that are no whole lines: two column blocks
// share the lines between them, so those are wider (see rec_cut).
constexpr int kBack = 8;
template <typename T, bool COUPLED, bool BWD, int LANES, int WAVES, int ROWS, bool STREAM>
__global__ __launch_bounds__(64 * WAVES, WAVES <= 4 && !BWD ? 3 : 2) void k_rec_tiles(const T *__restrict__ X, const T *__restrict__ L, const T *__restrict__ out_in,
                                                         const T *__restrict__ dout, const float *h_in, const float *enter,
                                                         const int *__restrict__ len, T *__restrict__ out, T *__restrict__ dx,
                                                         T *__restrict__ dl, float *leave, RecLook lk, int cols, int N, int D,
                                                         long long ld, int ntiles, int nblocks) {
    using P = Piece<T>;
    constexpr int W = P::W, NT = 64 * WAVES, PARTS = 64 / LANES, NCH = LANES * W;
    static_assert(NCH <= NT, "a thread per channel");
    constexpr bool kKeepGates = sizeof(T) == 4;   // the rows' gates, once computed, in the place of their log_a
    __shared__ __attribute__((aligned(16))) float sL[WAVES][NCH], sX[WAVES][NCH];   // (moved in pieces)
    __shared__ unsigned sTicket;
    // (moved on by one from tile to tile: a block's tiles then go to all XCDs in turn)
    const unsigned turn = (nblocks % 8 == 0 ? blockIdx.x + blockIdx.x / nblocks : blockIdx.x) % nblocks;
    const int group = turn % kGroups, per = (nblocks - group + kGroups - 1) / kGroups;   // column blocks group, group + kGroups, ...
    unsigned ticket = turn / kGroups;
    if (ntiles > 1) {
        if (threadIdx.x == 0) sTicket = __hip_atomic_fetch_add(lk.tickets + group * kTicketStride, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        ticket = sTicket;
    }
    const int tile = __builtin_amdgcn_readfirstlane(ticket / per), block = group + kGroups * __builtin_amdgcn_readfirstlane(ticket % per);
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, part = lane / LANES, cl = lane % LANES;
    const int col = block * LANES + cl;
    const bool mine = col < cols;
    const Column<T> c(min(col, cols - 1), N, D, len);
    const size_t row0 = (size_t)c.seq * N;
    const size_t pbase = row0 * ld + c.ch, tbase = row0 * D + c.ch;
    // row r of the thread is token at(r)
    const long long p0 = ((long long)tile * WAVES * PARTS + w * PARTS + part) * ROWS, first = BWD ? N - 1 - p0 : p0;
    constexpr int dir = BWD ? -1 : 1;
    auto at = [&](int r) { return first + dir * r; };
    auto there = [&](int r) { return at(r) >= 0 && at(r) < c.n; };
    const bool whole = __all(there(0) && there(ROWS - 1));
    // A tile behind the last tokens of all its sequences (every wave has the same columns): zeros, and nobody waits for it.
    constexpr int TOKENS = WAVES * PARTS * ROWS;
    if (len && (BWD ? tile + 1 < ntiles : tile > 0) && __all((BWD ? N - (long long)(tile + 1) * TOKENS : (long long)tile * TOKENS) >= c.n)) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
            if (mine && at(r) < N) {
                if constexpr (BWD) {
                    put<STREAM>(dx + pbase + at(r) * ld, u32x4{0, 0, 0, 0});
                    put<STREAM>(dl + pbase + at(r) * ld, u32x4{0, 0, 0, 0});
                } else {
                    put<STREAM>(out + tbase + at(r) * D, u32x4{0, 0, 0, 0});
                }
            }
        return;
    }

    u32x4 vu[ROWS], vl[ROWS];   // x, or the gradient of out
    [[maybe_unused]] u32x4 vo[BWD ? ROWS : 1], vx[BWD && COUPLED ? ROWS : 1];
    auto load_all = [&](auto token) {   // of row r, one that exists
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            vl[r] = gload<u32x4, STREAM>(L + pbase + token(r) * ld, 0);
            if constexpr (BWD) vu[r] = gload<u32x4, STREAM>(dout + tbase + token(r) * D, 0);
            else vu[r] = gload<u32x4, STREAM>(X + pbase + token(r) * ld, 0);
        }
        if constexpr (BWD)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const long long t = token(r);
                vo[r] = gload<u32x4, STREAM>(out_in + tbase + (t > 0 ? t - 1 : 0) * D, 0);
                if constexpr (COUPLED) vx[r] = gload<u32x4, STREAM>(X + pbase + t * ld, 0);
            }
    };
    if (whole) {
        load_all(at);
    } else {
        load_all([&](int r) { return min(max(at(r), 0ll), (long long)max(c.n - 1, 0)); });
#pragma unroll
        for (int r = 0; r < ROWS; ++r)   // a row that does not exist leaves the state as it is
            if (!there(r)) vl[r] = vu[r] = u32x4{0, 0, 0, 0};
    }
    // 1.
    float S[W] = {}, Y[W] = {};   // the gates' product as its logarithm: a sum near 0 keeps the bits that a product near 1 would lose
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        float fl[W], fu[W], fw[W];
        P::unpack(vl[r], fl);
        P::unpack(vu[r], fu);
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const Gate<T> g(fl[i]);
            if constexpr (BWD) Y[i] = g.times(fu[i] + Y[i]);
            else Y[i] = g.step(Y[i], COUPLED ? g.b() * fu[i] : fu[i]);
            S[i] += fl[i];
            fw[i] = g.w;
        }
        if constexpr (kKeepGates) vl[r] = P::pack(fw);
    }
    float most = S[0];   // (of PARTS sums of up to 88 / PARTS none adds up to more than 88)
#pragma unroll
    for (int i = 1; i < W; ++i) most = fmaxf(most, S[i]);
    const bool small = __all(most <= kMostLog / PARTS);
    if constexpr (PARTS > 1)   // joined with those in front, along the wave
        by_product<T>(small, [&](auto p) {
#pragma unroll
            for (int d = LANES; d < 64; d *= 2)
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const float l = __shfl_up(S[i], d), y = __shfl_up(Y[i], d);
                    if (lane >= d) {
                        Y[i] = p.step(p.word(S[i]), y, Y[i]);
                        S[i] += l;
                    }
                }
        });
    if (part == PARTS - 1) {
        store_floats<W>(&sX[w][cl * W], Y);
        store_floats<W>(&sL[w][cl * W], S);
    }
    // (the rows opaque from here on: the compiler would keep their gates as floats, twice the registers, for the second time)
#pragma unroll
    for (int r = 0; r < ROWS; ++r) asm volatile("" : "+v"(vl[r]), "+v"(vu[r]));
    __syncthreads();
    // 2. a thread per channel
    const size_t nstate = (size_t)cols * W, stride = (size_t)nblocks * NCH;
    if (const int ch = threadIdx.x; ch < NCH) {
        const size_t state = (size_t)block * NCH + ch, slot = tile * stride + state;
        float tl = 0.0f, tx = 0.0f, y, gate[WAVES], whole_tile, end, most = 0.0f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) most = fmaxf(most, sL[i][ch]);
        const bool small = __all(most <= kMostLog / WAVES);
        by_product<T>(small, [&](auto p) {
#pragma unroll
            for (int i = 0; i < WAVES; ++i) {
                gate[i] = p.word(sL[i][ch]);
                tx = p.step(gate[i], tx, sX[i][ch]);
                tl += sL[i][ch];
            }
            whole_tile = p.word(tl);
        });
        // The channel's tiles, from that of its sequence's first token in the order of the scan to that of its last.
        int begin = 0, last = ntiles - 1;
        if (len) {
            const Column<T> cc(min(block * LANES + ch / W, cols - 1), N, D, len);
            if constexpr (BWD) begin = cc.n > 0 ? (N - cc.n) / TOKENS : last;
            else last = cc.n > 0 ? (cc.n - 1) / TOKENS : 0;
        }
        if (tile < begin || tile > last) {
            y = 0.0f;   // none of its tokens here: nothing uses the state, and nobody waits for it
        } else if (tile == begin) {
            y = enter && state < nstate ? enter[state] : 0.0f;
        } else {
            if (tile < last) show(lk.steps + slot, (unsigned long long)published(whole_tile) | (unsigned long long)published(tx) << 32);
            y = entering<T, kBack>(lk, tile - begin, slot, stride);
        }
        by_product<T>(small, [&](auto p) { end = p.step(whole_tile, y, tx); });   // (as the tiles behind form it)
        if (begin <= tile && tile < last) show(lk.ends + slot, published(end));
        if (tile == last && leave && state < nstate) leave[state] = end;
        by_product<T>(small, [&](auto p) {
#pragma unroll
            for (int i = 0; i < WAVES; ++i) {
                const float x = sX[i][ch];
                sX[i][ch] = y;
                y = p.step(gate[i], y, x);
            }
        });
    }
    __syncthreads();
    // 3.
    float y[W];
    load_floats<W>(&sX[w][cl * W], y);
    if constexpr (PARTS > 1)
        by_product<T>(small, [&](auto p) {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float l = __shfl_up(S[i], LANES), x = __shfl_up(Y[i], LANES);
                if (part > 0) y[i] = p.step(p.word(l), y[i], x);
            }
        });
    auto again = [](float f) {
        if constexpr (kKeepGates) return Gate<T>::of_word(f);
        else return Gate<T>(f);
    };
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        float fl[W], fu[W];
        P::unpack(vl[r], fl);
        P::unpack(vu[r], fu);
        if constexpr (!BWD) {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const Gate<T> g = again(fl[i]);
                y[i] = g.step(y[i], COUPLED ? g.b() * fu[i] : fu[i]);
            }
            if (mine && (whole || at(r) < N))
                put<STREAM>(out + tbase + at(r) * D, whole || there(r) ? P::pack(y) : u32x4{0, 0, 0, 0});
        } else {
            float fo[W], fx[W], ox[W], ol[W];
            P::unpack(vo[r], fo);
            if constexpr (COUPLED) P::unpack(vx[r], fx);
            if (at(r) == 0) {
                if (h_in) load_floats<W>(h_in + (size_t)c.seq * D + c.ch, fo);
                else
#pragma unroll
                    for (int i = 0; i < W; ++i) fo[i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const Gate<T> g = again(fl[i]);
                const float e = fu[i] + y[i];
                y[i] = g.times(e);
                ox[i] = COUPLED ? g.b() * e : e;
                // (h_{s-1} as it was stored: bfloat16 rounds it to 2^-8, as it will round the gradient; to form it again would take x and log_a twice)
                ol[i] = y[i] * (COUPLED ? fo[i] - fx[i] : fo[i]);
            }
            if (mine && (whole || at(r) >= 0)) {
                const size_t to = pbase + at(r) * ld;
                put<STREAM>(dx + to, whole || there(r) ? P::pack(ox) : u32x4{0, 0, 0, 0});
                put<STREAM>(dl + to, whole || there(r) ? P::pack(ol) : u32x4{0, 0, 0, 0});
            }
        }
    }
}

// The scratch of k_rec_tiles as its workgroups expect it: the counters 0 (they come first), nothing published.
__global__ __launch_bounds__(256) void k_rec_clear(u32x4 *scratch, size_t counters, size_t n) {
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256)
        scratch[i] = i < counters ? u32x4{0, 0, 0, 0} : u32x4{kEmpty, kEmpty, kEmpty, kEmpty};
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
// How a call is cut (bfloat16, forward / backward in us, from a graph):
//   a thread per column    up to kShort tokens, where all is latency (8 x 16 x 2048 5.3 / 6.9, as a tile 7.0 / 8.6; 24 tokens 6.7 / 9.1
//                          and 7.0 / 8.6), and up to 128 where the columns alone fill the device: of 65536 columns 24 tokens
//                          16 / 25, 64 34 / 66, 128 81 / 132, as tiles 27 / 41, 38 / 82, 88 / 149; of 131072 26 / 42, 81 / 133, 155 / 265
//                          and 47 / 73, 90 / 147, 169 / 285; of 32768 9 / 16, 25 / 33, 40 / 72 and 17 / 24, 23 / 32, 37 / 82
//   one tile               of as few waves as cover the tokens (64 x 64 x 2048 12.6 / 17.5, in four waves 22.8 / 37.8), up to 512 tokens if that
//                          needs no more than two workgroups a CU (8 x 512 x 2048 with the host's time 11.9 / 17.3, as two tiles with what they
//                          need cleared first 16.0 / 21.1; 64 x 512 x 2048 87.7 / 136 and 77.0 / 124)
//   tiles of 8 waves       of few columns and many tokens, where the state's way from tile to tile takes the time, 1 us per kBack tiles
//                          (131072 x 128 33 / 49, in four waves 73 / 75; 16384 x 128 16.2 / 16.6 and 15.2 / 18.2; 8192 x 128
//                          15.1 / 14.3 and 11.7 / 14.8; 131072 tokens of 8 column blocks 92 / 137 and 96 / 139, of 16 162 / 255 and 155 / 246,
//                          32768 of 8 28 / 42 and 34 / 46, of 16 47 / 79 and 48 / 78, of 32 96 / 136 and 83 / 128)
//   tiles of 4 waves       otherwise
// Rows that are no whole lines, in blocks of 8 / 16 / 32 / 64 lanes: 4 x 16384 x 1000 forward 119 / 108 / 109 / 105, backward 205 / 178 / 167 / 166;
// float 32768 x 296 42 / 36.5 / 38.5 / 50 and 58 / 51 / 51 / 75; of 37 columns 22 / 25 / 34 / 44 and 34 / 36 / 46 / 70. (With non-temporal accesses in
// blocks of 8 163 / 300: a line goes before the other workgroup's half has come.)
constexpr int kShort = 16, kLongForward = 16384, kLongBackward = 8192, kFewBlocks = 8, kManyColumns = 1 << 16, kCus = 256;
namespace {
struct RecCut {
    int lanes;                       // of a column block
    bool lines;                      // rows are whole lines of 128 bytes
    int waves, rows;                 // of a workgroup of k_rec_tiles, of a thread; 0: a thread per column
    int nblocks, ntiles;
    size_t counters, slots, bytes;   // of the scratch: of the counters, slots, bytes of everything
};
RecCut rec_cut(const RecPlan &p, bool bwd) {
    const int w = p.dtype == 0 ? 4 : 8, cols = p.B * (p.D / w);
    RecCut c{};
    const int line = 128 / (p.dtype == 0 ? 4 : 2);   // elements
    c.lines = p.D % line == 0 && p.ld % line == 0;
    const bool one = p.N <= 512 && (cols + 7) / 8 <= (c.lines || p.N <= 256 ? 2 * kCus : kCus);   // tile of eight waves, at most
    c.lanes = c.lines || p.N <= 128 || cols < 64 || one ? 8 : cols < 512 ? 16 : 32;
    c.nblocks = (cols + c.lanes - 1) / c.lanes;
    const bool long_tiles = c.nblocks <= kFewBlocks && p.N >= (bwd ? kLongBackward : kLongForward);
    if (p.N <= kShort || (p.N <= 128 && cols >= kManyColumns)) c.waves = 0;
    else if (p.N <= 64) c.waves = 1;
    else if (p.N <= 128) c.waves = 2;
    else c.waves = long_tiles || (one && p.N > 256) ? 8 : 4;
    c.rows = long_tiles && !bwd ? 16 : 8;
    const int tokens = std::max(c.waves, 1) * (64 / c.lanes) * c.rows;
    c.ntiles = c.waves ? (int)(((long long)p.N + tokens - 1) / tokens) : 1;
    c.slots = c.ntiles > 1 ? (size_t)c.ntiles * c.nblocks * c.lanes * w : 0;
    c.counters = (size_t)kGroups * kTicketStride * sizeof(unsigned);
    c.bytes = c.counters + (c.slots * 12 + 15) / 16 * 16;
    return c;
}
bool on_lines(std::initializer_list<const void *> buffers) {
    for (const void *b : buffers)
        if ((uintptr_t)b % 128 != 0) return false;
    return true;
}
template <typename T, bool C, bool BWD, int LANES, int WAVES, int ROWS = 8>
void rec_tiles(const RecPlan &p, const RecArgs &a, const RecCut &c, hipStream_t s) {
    char *base = (char *)a.scratch;
    RecLook lk{(unsigned *)base, (unsigned long long *)(base + c.counters), (unsigned *)(base + c.counters + c.slots * 8)};
    if (c.ntiles > 1) {
        const size_t n = c.bytes / 16;
        k_rec_clear<<<dim3((unsigned)std::min<size_t>((n + 255) / 256, 2048)), dim3(256), 0, s>>>((u32x4 *)base, c.counters / 16, n);
    }
    auto kernel = k_rec_tiles<T, C, BWD, LANES, WAVES, ROWS, false>;
    // (lines that two workgroups share have to stay in the cache; forward, 8 waves of 8 rows take one tile of 100 MB at most)
    if constexpr (LANES == 8 && (WAVES == 4 || (WAVES == 8 && (BWD || ROWS == 16))))
        if (c.lines && on_lines({a.x, a.log_a, a.out_in, a.dout, a.out, a.dx, a.dlog_a}) && past_cache((size_t)(BWD ? (C ? 6 : 5) : 3) * p.B * p.N * p.D * sizeof(T)))
            kernel = k_rec_tiles<T, C, BWD, LANES, WAVES, ROWS, true>;
    kernel<<<dim3((unsigned)c.ntiles * c.nblocks), dim3(64 * WAVES), 0, s>>>(
        (const T *)a.x, (const T *)a.log_a, (const T *)a.out_in, (const T *)a.dout, a.h_in, BWD ? a.dh_out : a.h_in, a.len, (T *)a.out, (T *)a.dx,
        (T *)a.dlog_a, BWD ? a.dh_in : a.h_out, lk, p.B * (p.D / Piece<T>::W), p.N, p.D, p.ld, c.ntiles, c.nblocks);
}
template <typename T, bool C, bool BWD>
hipError_t rec(const RecPlan &p, const RecArgs &a, hipStream_t s) {
    const RecCut c = rec_cut(p, BWD);
    const int cols = p.B * (p.D / Piece<T>::W);
    const dim3 grid((cols + kStepThreads - 1) / kStepThreads), block(kStepThreads);
    switch (c.waves) {
        case 1: rec_tiles<T, C, BWD, 8, 1>(p, a, c, s); break;
        case 2: rec_tiles<T, C, BWD, 8, 2>(p, a, c, s); break;
        case 4:
            if (c.lanes == 8) rec_tiles<T, C, BWD, 8, 4>(p, a, c, s);
            else if (c.lanes == 16) rec_tiles<T, C, BWD, 16, 4>(p, a, c, s);
            else rec_tiles<T, C, BWD, 32, 4>(p, a, c, s);
            break;
        case 8:   // (of 8 column blocks at most: not 32 lanes)
            if (c.rows == 8 && c.lanes == 8) rec_tiles<T, C, BWD, 8, 8>(p, a, c, s);
            else if constexpr (BWD) rec_tiles<T, C, BWD, 16, 8>(p, a, c, s);
            else if (c.lanes == 8) rec_tiles<T, C, BWD, 8, 8, 16>(p, a, c, s);
            else rec_tiles<T, C, BWD, 16, 8, 16>(p, a, c, s);
            break;
        default:
            if constexpr (BWD)
                k_rec_step_bwd<T, C><<<grid, block, 0, s>>>((const T *)a.x, (const T *)a.log_a, (const T *)a.out_in, (const T *)a.dout, a.h_in,
                                                            a.dh_out, a.len, (T *)a.dx, (T *)a.dlog_a, a.dh_in, cols, p.N, p.D, p.ld);
            else
                k_rec_step_fwd<T, C><<<grid, block, 0, s>>>((const T *)a.x, (const T *)a.log_a, a.h_in, a.len, (T *)a.out, a.h_out, cols, p.N, p.D, p.ld);
    }
    return hipGetLastError();
}
template <bool BWD>
hipError_t by_type(const RecPlan &p, const RecArgs &a, hipStream_t s) {
    if (p.dtype == 0) return p.coupled ? rec<float, true, BWD>(p, a, s) : rec<float, false, BWD>(p, a, s);
    return p.coupled ? rec<bf16_t, true, BWD>(p, a, s) : rec<bf16_t, false, BWD>(p, a, s);
}
}  // namespace

size_t rec_scratch(const RecPlan &p) { return std::max(rec_cut(p, false).bytes, rec_cut(p, true).bytes); }
hipError_t launch_rec_fwd(const RecPlan &p, const RecArgs &a, hipStream_t s) { return by_type<false>(p, a, s); }
hipError_t launch_rec_bwd(const RecPlan &p, const RecArgs &a, hipStream_t s) { return by_type<true>(p, a, s); }

}  // namespace lasp
