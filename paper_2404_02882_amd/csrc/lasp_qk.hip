// HIP kernels (gfx950 / CDNA4) for what stands between a projection and a mixer: queries and keys normalised by head, rotated by
// position and laid out heads first, in one pass over them.
//     y = amplitude R(pos) n  on the first `rot` features, y = n on the others;   n = w * x * r,   r = (mean x^2 + eps)^(-1/2), (sum x^2 + eps)^(-1/2) or 1
//     backward: dn = amplitude R(pos)^T dy,   dw = sum dn * x * r,   dx = r (w dn - x r^2 mean(w dn * x))   (sum for the second r, none for 1)
// A head of a token is a row: LANES threads with one piece of 16 bytes each. The workgroup first makes the table of cosines and
// sines of the tokens it takes, each angle once for all heads (an angle costs about as much as ten rows' pieces: position times frequency in 64 bits, whole turns
// taken off there, so that far positions keep the float's precision), then its threads go over the rows of these tokens, queries and keys.
// Bound by memory: 32768 tokens x 16 + 16 heads of 128, bfloat16: forward 112 us (4.8 TB/s), backward 155 (5.2 TB/s). A row's next piece is
// loaded before this one is used. A few tokens (64 x 16 + 4 heads): 5.2 us, launch, table and one row one after the other. Where a group's tokens have fewer heads than the
// workgroup takes rows at a time, threads are idle and the table and its barriers bound it: 65536 tokens, heads of 128, 8 + 8 of them 4.5 TB/s forward and 5.0 backward,
// 4 + 4 4.3 and 4.2, 4 + 1 2.4 and 2.9, 1 + 1 0.8 and 1.0.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "lasp_block.h"

namespace lasp {
namespace {

constexpr int kThreads = 256, kTable = 512;   // entries of the table: tokens times pairs

struct QkCall {
    int B, N, H, Hk, D, rot, half, norm, tokens, group;   // tokens of the call; of a group (one table)
    long long ldq, ldk;                                    // elements between rows of the projections
    float eps, amplitude, share;   // share: of a row's squares (1 / D or 1)
    const double *freq;
    const int *pos;
};

// The rows (heads of tokens) that a thread comes to in a group, one after the other; counted up, as a division takes as long as the row itself (one subtraction a row
// with 16 heads of 128; with one head sixteen of them).
struct Walk {
    int slot, head, b, s;    // token of the group, its head, sequence and place there
    int left;                // rows left up to the last of the group, less than 1: none
    DEVI Walk(const QkCall &c, int token0, int count, int heads, int first) {
        b = token0 / c.N;
        s = token0 - b * c.N;
        slot = 0;
        head = first;
        left = count * heads - first;
        settle(c, heads);
    }
    DEVI void settle(const QkCall &c, int heads) {
        while (head >= heads) {
            head -= heads;
            ++slot;
            if (++s == c.N) s = 0, ++b;
        }
    }
    DEVI void next(const QkCall &c, int heads, int rows) {
        head += rows;
        left -= rows;
        settle(c, heads);
    }
};
DEVI void make_table(const QkCall &c, float2 *table, int token0, int count) {
    const int pairs = c.rot / 2;
    for (int e = threadIdx.x; e < count * pairs; e += kThreads) {
        const int slot = e / pairs, i = e - slot * pairs, token = token0 + slot;
        const int p = c.pos ? c.pos[token] : token % c.N;
        double turns = (double)p * c.freq[i] * 0.15915494309189533577;
        turns -= rint(turns);
        float s, co;
        sincospif(2.0f * (float)turns, &s, &co);
        table[e] = float2{co * c.amplitude, s * c.amplitude};
    }
}

// Sum over the threads of a row, in every one of them.
template <int LANES>
DEVI float row_sum(float v) {
#pragma unroll
    for (int d = LANES / 2; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// What a thread does to its piece of a row: features at .. at + W - 1.
template <typename T, int LANES>
struct Turn {
    static constexpr int W = Piece<T>::W;
    int at, other;   // first feature; lane of the piece that holds the pairs' other features (layout by halves)
    int first;       // first pair of the piece, -1: it is not rotated
    bool low;        // the piece holds the pairs' first features
    DEVI Turn(const QkCall &c, int lane) {
        at = lane * W;
        const int pairs = c.rot / 2;
        first = at >= c.rot ? -1 : !c.half ? at / 2 : at < pairs ? at : at - pairs;
        low = at < pairs;
        other = c.half && first >= 0 ? lane + (low ? pairs / W : -(pairs / W)) : lane;
        other += (int)(threadIdx.x & 63) - lane;
    }
    DEVI u32x4 partner(const QkCall &c, u32x4 v) const {   // every lane of the wave calls it
        if (!c.half || c.rot == 0) return v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __shfl((int)v[i], other);
        return v;
    }
    // own (and, by halves, the partner's) features turned; BACK: the other way
    template <bool BACK>
    DEVI void turn(const QkCall &c, const float2 *t, float (&own)[W], const float (&oth)[W]) const {
        if (first < 0) return;
        if (c.half) {
#pragma unroll
            for (int i = 0; i < W; i += 2) {
                const f32x4 cs = *(const f32x4 *)(t + first + i);
                const float sign = low != BACK ? -1.0f : 1.0f;
                own[i] = own[i] * cs[0] + sign * (oth[i] * cs[1]);
                own[i + 1] = own[i + 1] * cs[2] + sign * (oth[i + 1] * cs[3]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < W; i += 4) {
                const f32x4 cs = *(const f32x4 *)(t + first + i / 2);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float co = cs[2 * j], si = BACK ? -cs[2 * j + 1] : cs[2 * j + 1], a = own[i + 2 * j], b = own[i + 2 * j + 1];
                    own[i + 2 * j] = a * co - b * si;
                    own[i + 2 * j + 1] = a * si + b * co;
                }
            }
        }
    }
};
// x^(-1/2): the instruction is good to one step, but takes numbers below the smallest normal one as 0.
DEVI float rsqrt_of(float x) {
    const bool tiny = x < 0x1p-96f;
    const float y = __builtin_amdgcn_rsqf(tiny ? x * 0x1p64f : x);
    return tiny ? y * 0x1p32f : y;
}
DEVI float scale_of(const QkCall &c, float squares) { return c.norm == 0 ? 1.0f : rsqrt_of(__builtin_fmaf(squares, c.share, c.eps)); }
template <int W>
DEVI void weights_of(const float *w, int at, bool has, float (&f)[W]) {
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = 1.0f;
    if (w && has) load_floats<W>(w + at, f);
}

// The weights of a thread's piece and of its partner's.
template <int W>
struct Weighted {
    float own[W], other[W];
};
template <typename T, int LANES>
DEVI Weighted<Piece<T>::W> weighted(const float *w, const Turn<T, LANES> &my) {
    constexpr int W = Piece<T>::W;
    Weighted<W> f;
    load_floats<W>(w + my.at, f.own);
    load_floats<W>(w + (my.other & (LANES - 1)) * W, f.other);
    return f;
}

template <typename T, int LANES, bool STREAM>
__global__ __launch_bounds__(kThreads) void k_qk_fwd(const T *__restrict__ xq, const T *__restrict__ xk, const float *__restrict__ wq,
                                                     const float *__restrict__ wk, T *__restrict__ yq, T *__restrict__ yk, QkCall c) {
    using P = Piece<T>;
    constexpr int W = P::W, ROWS = kThreads / LANES;
    __shared__ __attribute__((aligned(16))) float2 table[kTable];
    const int lane = threadIdx.x % LANES;
    const bool has = lane * W < c.D;
    const Turn<T, LANES> my(c, lane);
    const int at = has ? my.at : 0;
    __shared__ __attribute__((aligned(16))) float weights[2][LANES * W];   // (read once a group: in registers they leave room for four waves a SIMD, not five)
    for (int e = threadIdx.x; e < 2 * LANES * W; e += kThreads) {
        const int n = e / (LANES * W), d = e - n * LANES * W;
        const float *w = n ? wk : wq;
        weights[n][d] = w && d < c.D ? w[d] : 1.0f;
    }
    if (!c.rot) __syncthreads();
    for (int token0 = blockIdx.x * c.group; token0 < c.tokens; token0 += gridDim.x * c.group) {
        const int count = min(c.group, c.tokens - token0);
        if (c.rot) {
            __syncthreads();   // the table has been read
            make_table(c, table, token0, count);
            __syncthreads();
        }
        auto part = [&](const T *x, T *y, const float *ws, int heads, long long ld) {
            const auto w = weighted<T, LANES>(ws, my);
            Walk r(c, token0, count, heads, threadIdx.x / LANES);
            const T *rows = x + (size_t)token0 * ld + at;
            auto load = [&]() { return gload<u32x4, STREAM>(r.left > 0 ? rows + r.slot * ld + r.head * c.D : rows, 0); };
            u32x4 next = load();
            for (int turn = count * heads; turn > 0; turn -= ROWS) {   // (all threads take part in every turn: the sums want whole waves)
                const u32x4 v = next;
                const Walk now = r;
                r.next(c, heads, ROWS);
                if (turn > ROWS) next = load();
                float f[W], g[W], s = 0.0f;
                P::unpack(v, f);
#pragma unroll
                for (int i = 0; i < W; ++i) s = __builtin_fmaf(f[i], f[i], s);
                const float k = scale_of(c, c.norm == 0 ? 0.0f : row_sum<LANES>(has ? s : 0.0f));
                P::unpack(my.partner(c, v), g);
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    f[i] *= k * w.own[i];
                    g[i] *= k * w.other[i];
                }
                my.template turn<false>(c, table + (now.left > 0 ? now.slot : 0) * (c.rot / 2), f, g);
                if (now.left > 0 && has) put<STREAM>(y + (((size_t)now.b * heads + now.head) * c.N + now.s) * c.D + at, P::pack(f));
            }
        };
        part(xq, yq, weights[0], c.H, c.ldq);
        if (c.Hk) part(xk, yk, weights[1], c.Hk, c.ldk);
    }
}

template <typename T, int LANES, bool STREAM>
__global__ __launch_bounds__(kThreads) void k_qk_bwd(const T *__restrict__ xq, const T *__restrict__ xk, const float *__restrict__ wq,
                                                     const float *__restrict__ wk, const T *__restrict__ dyq, const T *__restrict__ dyk,
                                                     T *__restrict__ dxq, T *__restrict__ dxk, float *__restrict__ pq, float *__restrict__ pk, QkCall c) {
    using P = Piece<T>;
    constexpr int W = P::W, ROWS = kThreads / LANES;
    __shared__ __attribute__((aligned(16))) float2 table[kTable];
    __shared__ __attribute__((aligned(16))) float part_sums[kThreads / 64][LANES * W];
    const int lane = threadIdx.x % LANES;
    const bool has = lane * W < c.D, sums = pq || pk, reads = c.norm != 0 || sums;
    const Turn<T, LANES> my(c, lane);
    const int at = has ? my.at : 0;
    float w[2][W], acc[2][W] = {};
    weights_of<W>(wq, at, has, w[0]);
    weights_of<W>(wk, at, has, w[1]);
    for (int token0 = blockIdx.x * c.group; token0 < c.tokens; token0 += gridDim.x * c.group) {
        const int count = min(c.group, c.tokens - token0);
        if (c.rot) {
            __syncthreads();
            make_table(c, table, token0, count);
            __syncthreads();
        }
        auto part = [&](const T *x, const T *dy, T *dx, const float (&w)[W], float (&acc)[W], int heads, long long ld) {
            Walk r(c, token0, count, heads, threadIdx.x / LANES);
            const T *rows = x + (size_t)token0 * ld + at;
            T *to = dx + (size_t)token0 * ld + at;
            u32x4 nx{0, 0, 0, 0}, ny;
            auto load = [&]() {
                const bool there = r.left > 0;
                ny = gload<u32x4, STREAM>(dy + (there ? (((size_t)r.b * heads + r.head) * c.N + r.s) * c.D : 0) + at, 0);
                if (reads) nx = gload<u32x4, STREAM>(there ? rows + r.slot * ld + r.head * c.D : rows, 0);
            };
            load();
            for (int turn = count * heads; turn > 0; turn -= ROWS) {
                const u32x4 vx = nx, vy = ny;
                const Walk now = r;
                r.next(c, heads, ROWS);
                if (turn > ROWS) load();
                float f[W], d[W], o[W], s = 0.0f, t = 0.0f;
                P::unpack(vy, d);
                P::unpack(my.partner(c, vy), o);
                P::unpack(vx, f);
                my.template turn<true>(c, table + (now.left > 0 ? now.slot : 0) * (c.rot / 2), d, o);
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    o[i] = d[i] * w[i];
                    s = __builtin_fmaf(f[i], f[i], s);
                    t = __builtin_fmaf(o[i], f[i], t);
                }
                float k = 1.0f, mean = 0.0f;
                if (c.norm != 0) {
                    k = scale_of(c, row_sum<LANES>(has ? s : 0.0f));
                    mean = row_sum<LANES>(has ? t : 0.0f) * c.share * k * k;
                }
                if (now.left > 0 && has) {
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        acc[i] = __builtin_fmaf(d[i] * k, f[i], acc[i]);
                        o[i] = k * (o[i] - f[i] * mean);
                    }
                    put<STREAM>(to + now.slot * ld + now.head * c.D, P::pack(o));
                }
            }
        };
        part(xq, dyq, dxq, w[0], acc[0], c.H, c.ldq);
        if (c.Hk) part(xk, dyk, dxk, w[1], acc[1], c.Hk, c.ldk);
    }
    // a partial row per workgroup: the rows of a wave by shuffles, the waves in LDS, in a fixed order
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        float *to = n ? pk : pq;
        if (!to) continue;
#pragma unroll
        for (int i = 0; i < W; ++i)
#pragma unroll
            for (int d = LANES; d < 64; d *= 2) acc[n][i] += __shfl_xor(acc[n][i], d);
        __syncthreads();
        if ((threadIdx.x & 63) < LANES) store_floats<W>(&part_sums[threadIdx.x >> 6][lane * W], acc[n]);
        __syncthreads();
        for (int e = threadIdx.x; e < c.D; e += kThreads) to[(size_t)blockIdx.x * c.D + e] = (part_sums[0][e] + part_sums[1][e]) + (part_sums[2][e] + part_sums[3][e]);
    }
}

constexpr int kCus = 256;
// Tokens of a group: four, and no more than the table holds or than leave four workgroups a CU something to do (bf16, 32768 tokens x 16 + 16
// heads of 128, with eight workgroups a CU: forward 122 us with four, 126 with eight, 128 with 16; backward 155, 162, 163). Measured with many heads; with few
// of them four tokens are too few rows for a workgroup (rates at the top).
int group_of(const QkPlan &p) {
    const long long tokens = (long long)p.B * p.N;
    const long long room = p.rot ? std::min(4, kTable / (p.rot / 2)) : 4;
    return (int)std::max<long long>(1, std::min<long long>(room, tokens / (4 * kCus)));
}
int workgroups(const QkPlan &p, int a_cu) {
    const long long tokens = (long long)p.B * p.N, g = group_of(p);
    return (int)std::min<long long>((tokens + g - 1) / g, (long long)a_cu * kCus);
}
// Workgroups a CU. Forward 64, which is one a group up to 65536 tokens (same sizes: 112 us, 120 with eight; 20012 tokens x 12 + 12 heads of 96: 45.6,
// 49.6); backward each leaves a row of partial sums (185 us with two a CU, 162 with four, 161 with eight, 165 with sixteen; float, 7503 tokens x
// 8 + 2 heads of 64: 20, 15.7, 13.2, 13.2).
constexpr int kForwardACu = 64, kBackwardACu = 8;
QkCall call_of(const QkPlan &p, const QkArgs &a) {
    return {p.B, p.N, p.H, p.Hk, p.D, p.rot, p.half, p.norm, p.B * p.N, group_of(p), p.ldq, p.ldk, a.eps, a.amplitude, p.norm == 1 ? 1.0f / p.D : 1.0f, a.freq, a.pos};
}
// f.template operator()<T, LANES, STREAM>()
template <typename T, bool STREAM, typename F>
void by_lanes(int n, F f) {
    if (n <= 1) f.template operator()<T, 1, STREAM>();
    else if (n <= 2) f.template operator()<T, 2, STREAM>();
    else if (n <= 4) f.template operator()<T, 4, STREAM>();
    else if (n <= 8) f.template operator()<T, 8, STREAM>();
    else if (n <= 16) f.template operator()<T, 16, STREAM>();
    else if (n <= 32) f.template operator()<T, 32, STREAM>();
    else if constexpr (sizeof(T) == 4) f.template operator()<T, 64, STREAM>();   // (two-byte rows have 32 pieces at most)
}
template <typename F>
hipError_t by_plan(const QkPlan &p, int tensors, F f) {
    const size_t bytes = (size_t)tensors * p.B * p.N * (p.H + p.Hk) * p.D * (p.dtype == 0 ? 4 : 2);
    if (p.dtype == 0) past_cache(bytes) ? by_lanes<float, true>(p.D / 4, f) : by_lanes<float, false>(p.D / 4, f);
    else past_cache(bytes) ? by_lanes<bf16_t, true>(p.D / 8, f) : by_lanes<bf16_t, false>(p.D / 8, f);
    return hipGetLastError();
}
struct QkFwd {
    const QkPlan &p;
    const QkArgs &a;
    hipStream_t s;
    template <typename T, int LANES, bool STREAM>
    void operator()() const {
        k_qk_fwd<T, LANES, STREAM><<<dim3(workgroups(p, kForwardACu)), dim3(kThreads), 0, s>>>(
            (const T *)a.xq, (const T *)a.xk, a.wq, a.wk, (T *)a.q, (T *)a.k, call_of(p, a));
    }
};
struct QkBwd {
    const QkPlan &p;
    const QkArgs &a;
    hipStream_t s;
    template <typename T, int LANES, bool STREAM>
    void operator()() const {
        const int n = workgroups(p, kBackwardACu);
        k_qk_bwd<T, LANES, STREAM><<<dim3(n), dim3(kThreads), 0, s>>>(
            (const T *)a.xq, (const T *)a.xk, a.wq, a.wk, (const T *)a.dq, (const T *)a.dk, (T *)a.dxq, (T *)a.dxk,
            a.dwq ? a.scratch : nullptr, a.dwk ? a.scratch + (size_t)n * p.D : nullptr, call_of(p, a));
    }
};

}  // namespace

size_t qk_scratch(const QkPlan &p) { return 2 * (size_t)workgroups(p, kBackwardACu) * p.D * sizeof(float); }

hipError_t launch_qk_fwd(const QkPlan &p, const QkArgs &a, hipStream_t s) { return by_plan(p, 2, QkFwd{p, a, s}); }
hipError_t launch_qk_bwd(const QkPlan &p, const QkArgs &a, hipStream_t s) {
    if (hipError_t e = by_plan(p, 3, QkBwd{p, a, s}); e != hipSuccess) return e;
    const int n = workgroups(p, kBackwardACu);
    return launch_column_sums(a.scratch, a.dwq, a.scratch + (size_t)n * p.D, a.dwk, n, p.D, s);
}

}  // namespace lasp
