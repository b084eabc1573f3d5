// What the kernels around the mixers share (lasp_rec.hip, lasp_norms.hip): pieces of 16 bytes as floats, and the
// arguments the host layer (lasp_block_api.cpp) hands them, already validated.
#ifndef LASP_BLOCK_H
#define LASP_BLOCK_H

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

namespace lasp {

// Gated recurrence. Channels go in pieces of 16 bytes (a column: W channels of one sequence).
struct RecPlan {
    int B, N, D, dtype;
    int coupled;
    long long ld;        // elements between the rows of x, log_a, dx, dlog_a
};
struct RecArgs {         // forward: x, log_a -> out;  backward: log_a, out, dout (x) -> dx, dlog_a
    const void *x, *log_a, *out_in, *dout;
    const float *h_in;   // may be null
    const int *len;      // may be null
    const float *dh_out; // may be null
    void *out, *dx, *dlog_a;
    float *h_out, *dh_in;   // may be null
    void *scratch;
};
size_t rec_scratch(const RecPlan &p);
hipError_t launch_rec_fwd(const RecPlan &p, const RecArgs &a, hipStream_t s);
hipError_t launch_rec_bwd(const RecPlan &p, const RecArgs &a, hipStream_t s);

// Whether a call moves more bytes than the last-level cache holds: its loads and stores then leave the cache to what is used
// again (non-temporal). bfloat16 32768 x 2048: recurrence forward / backward 87 / 135 -> 83 / 129 us, 4 x 16384 x 4096 coupled 311 / 589 -> 292 / 557,
// norm before a block forward / backward 94 / 145 -> 87 / 130; smaller calls find their inputs there (float 2 x 4099 x 1000, 30 / 61 us as they are, 41 / 72 so).
constexpr bool past_cache(size_t bytes) { return bytes > ((size_t)256 << 20); }

// Norms: rows of C elements, each handled by `lanes` threads with `pieces` 16-byte pieces apiece. A token of `heads` rows.
struct RowPlan {
    int tokens, heads, C;
    int dtype;
    int lanes, pieces;
};
struct AddNormArgs {
    const void *r, *x, *dy, *dr_out;
    const float *scale, *weight;
    float eps;
    void *r_out, *y, *dr, *dx;
    float *dweight, *dscale, *scratch;
    int loads() const { return 2 + (dscale ? 1 : 0) + (dr_out ? 1 : 0); }   // tensors the backward pass reads
};
struct GateArgs {
    int H, N, D;         // of the tensors (the rows normalised: RowPlan)
    int gate;
    long long ld;        // elements between the rows of u, du
    const void *o, *u, *dy;
    const float *weight;
    float eps;
    void *y, *d_o, *du;
    float *dweight, *scratch;
    int loads() const { return gate ? 3 : 2; }
};
RowPlan row_plan(int tokens, int heads, int C, int dtype);
size_t addnorm_scratch(const RowPlan &p);
size_t gatenorm_scratch(const RowPlan &p);
hipError_t launch_addnorm_fwd(const RowPlan &p, const AddNormArgs &a, hipStream_t s);
hipError_t launch_addnorm_bwd(const RowPlan &p, const AddNormArgs &a, hipStream_t s);
hipError_t launch_gatenorm_fwd(const RowPlan &p, const GateArgs &a, hipStream_t s);
hipError_t launch_gatenorm_bwd(const RowPlan &p, const GateArgs &a, hipStream_t s);

// out0 = the sum of n rows of C floats at part0, in a fixed order; the same for part1 and out1. An out may be null.
hipError_t launch_column_sums(const float *part0, float *out0, const float *part1, float *out1, int n, int C, hipStream_t s);

// Queries and keys by head: norm and position rotation, from rows of projections to heads-first tensors.
struct QkPlan {
    int B, N, H, Hk, D, dtype;
    int norm;               // 0 none, 1 over the mean of squares, 2 over their sum
    int rot, half;          // features rotated; pairs by halves (else neighbours)
    long long ldq, ldk;     // elements between the rows of the projections
};
struct QkArgs {
    const void *xq, *xk, *dq, *dk;
    const float *wq, *wk;   // may be null
    float eps, amplitude;
    const double *freq;
    const int *pos;         // may be null
    void *q, *k, *dxq, *dxk;
    float *dwq, *dwk, *scratch;   // may be null
};
size_t qk_scratch(const QkPlan &p);
hipError_t launch_qk_fwd(const QkPlan &p, const QkArgs &a, hipStream_t s);
hipError_t launch_qk_bwd(const QkPlan &p, const QkArgs &a, hipStream_t s);

}  // namespace lasp

#ifdef __HIPCC__
#include "lasp_device.h"
namespace lasp {

// 16 bytes of data as W floats.
template <typename T>
struct Piece;
template <>
struct Piece<float> {
    static constexpr int W = 4;
    static DEVI void unpack(u32x4 v, float (&f)[W]) {
        const f32x4 x = __builtin_bit_cast(f32x4, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = x[i];
    }
    static DEVI u32x4 pack(const float (&f)[W]) { return __builtin_bit_cast(u32x4, f32x4{f[0], f[1], f[2], f[3]}); }
};
template <>
struct Piece<bf16_t> {
    static constexpr int W = 8;
    static DEVI void unpack(u32x4 v, float (&f)[W]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __builtin_bit_cast(float, v[i] << 16);
            f[2 * i + 1] = __builtin_bit_cast(float, v[i] & 0xffff0000u);
        }
    }
    static DEVI u32x4 pack(const float (&f)[W]) {
        f32x8 x;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = f[i];
        return __builtin_bit_cast(u32x4, __builtin_convertvector(x, bf16x8));
    }
};
template <bool STREAM, typename T>
DEVI void put(T *p, u32x4 v) {
    if constexpr (STREAM) __builtin_nontemporal_store(v, (u32x4 *)p);
    else *(u32x4 *)p = v;
}
// W floats of a float array (16-byte aligned).
template <int W>
DEVI void load_floats(const float *p, float (&f)[W]) {
#pragma unroll
    for (int i = 0; i < W; i += 4) {
        const f32x4 v = *(const f32x4 *)(p + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[i + j] = v[j];
    }
}
template <int W>
DEVI void store_floats(float *p, const float (&f)[W]) {
#pragma unroll
    for (int i = 0; i < W; i += 4) *(f32x4 *)(p + i) = f32x4{f[i], f[i + 1], f[i + 2], f[i + 3]};
}

}  // namespace lasp
#endif
#endif
