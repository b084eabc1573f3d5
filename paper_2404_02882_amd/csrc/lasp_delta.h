// The gated delta rule's plan and arguments, as the host layer (lasp_delta_api.cpp) hands them to the kernels (lasp_delta.hip),
// already validated.
#ifndef LASP_DELTA_H
#define LASP_DELTA_H

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

namespace lasp {

constexpr int kDeltaTile = 32;         // tokens of a walk's tile

struct DeltaPlan {
    int B, H, N, D, Dv, dtype, key_heads;
    int tiles, grad_tiles;    // tiles of a sequence; those that the gradients are computed in
    int segments, seg_tiles;  // segments a sequence is cut into, tiles of one
    bool split;               // the walks: a state's key features shared by two waves
};
// Forward calls without a cache run token by token up to this length.
inline int delta_step_tokens(const DeltaPlan &p) { return p.dtype == 0 ? 8 : 4; }
DeltaPlan delta_plan(int B, int H, int N, int D, int Dv, int dtype, int key_heads);

struct DeltaArgs {
    const void *q, *k, *v, *dout;
    const float *log_g, *beta;       // log_g: may be null
    const int *len;                  // may be null
    const float *kv_in, *dkv_out;    // may be null
    void *out, *dq, *dk, *dv;
    float *kv_out, *dlog_g, *dbeta, *dkv_in;   // dlog_g: may be null
    void *cache;                     // forward: may be null
    void *scratch;
};
size_t delta_cache(const DeltaPlan &p);
size_t delta_scratch(const DeltaPlan &p);
size_t delta_bwd_scratch(const DeltaPlan &p);
hipError_t launch_delta_fwd(const DeltaPlan &p, const DeltaArgs &a, hipStream_t s);
hipError_t launch_delta_bwd(const DeltaPlan &p, const DeltaArgs &a, hipStream_t s);

}  // namespace lasp
#endif
