// C-ABI host layer of the gated delta rule (lasp_delta_*): argument checks and dispatch. No device memory is allocated or freed
// here and nothing synchronises.
#include "../../include/lasp.h"

#include "lasp_checks.h"
#include "lasp_delta.h"

namespace {

using lasp::elem_bytes;
using lasp::Span;

constexpr int64_t kMostHeads = 65535;   // (a dimension of a launch)

int make(const lasp_delta_shape *s, lasp::DeltaPlan *p) {
    if (!s) return LASP_ERR_NULL;
    if (s->dtype != LASP_F32 && s->dtype != LASP_BF16) return LASP_ERR_DTYPE;
    if (s->B < 1 || s->H < 1 || s->N < 1 || (int64_t)s->B * s->H > kMostHeads) return LASP_ERR_SHAPE;
    const int dv = s->Dv ? s->Dv : s->D, hk = s->key_heads ? s->key_heads : s->H;
    if ((s->D != 64 && s->D != 128) || (dv != 64 && dv != 128)) return LASP_ERR_SHAPE;
    if (hk < 1 || hk > s->H || s->H % hk != 0) return LASP_ERR_SHAPE;
    *p = lasp::delta_plan(s->B, s->H, s->N, s->D, dv, s->dtype, hk);
    return LASP_OK;
}

struct Sizes {   // bytes of a call's buffers
    size_t keys, values, state, gate, len;
    explicit Sizes(const lasp::DeltaPlan &p) {
        const size_t e = elem_bytes(p.dtype), tokens = (size_t)p.B * p.N;
        keys = tokens * p.key_heads * p.D * e;
        values = tokens * p.H * p.Dv * e;
        state = (size_t)p.B * p.H * p.D * p.Dv * sizeof(float);
        gate = tokens * p.H * sizeof(float);
        len = p.B * sizeof(int32_t);
    }
};

// As lasp::check_buffers; `to` may be `from` (the same pointer): a state updated in place.
int check(std::initializer_list<Span> ins, Span from, std::initializer_list<Span> outs, Span to) {
    if (int rc = lasp::check_buffers(ins, outs); rc != LASP_OK) return rc;
    if ((uintptr_t)from.p % 16 != 0 || (uintptr_t)to.p % 16 != 0) return LASP_ERR_ALIGN;
    if (lasp::overlap_any(to, ins) || lasp::overlap_any(to, outs) || lasp::overlap_any(from, outs)) return LASP_ERR_ALIAS;
    return to.p != from.p && lasp::overlap(to, from) ? LASP_ERR_ALIAS : LASP_OK;
}

int status(hipError_t e) { return e == hipSuccess ? LASP_OK : LASP_ERR_HIP; }

}  // namespace

extern "C" {

int lasp_check_delta(const lasp_delta_shape *shape) {
    lasp::DeltaPlan p;
    return make(shape, &p);
}

size_t lasp_delta_cache_bytes(const lasp_delta_shape *shape) {
    lasp::DeltaPlan p;
    return make(shape, &p) == LASP_OK ? lasp::delta_cache(p) : 0;
}

size_t lasp_delta_scratch_bytes(const lasp_delta_shape *shape) {
    lasp::DeltaPlan p;
    return make(shape, &p) == LASP_OK ? lasp::delta_scratch(p) : 0;
}

size_t lasp_delta_bwd_scratch_bytes(const lasp_delta_shape *shape) {
    lasp::DeltaPlan p;
    return make(shape, &p) == LASP_OK ? lasp::delta_bwd_scratch(p) : 0;
}

int lasp_delta_fwd(const lasp_delta_shape *shape, const void *q, const void *k, const void *v, const float *log_g, const float *beta,
                   const float *kv_in, const int32_t *len, void *out, float *kv_out, void *state_cache, void *scratch,
                   size_t scratch_bytes, void *hip_stream) {
    lasp::DeltaPlan p;
    if (int rc = make(shape, &p); rc != LASP_OK) return rc;
    if (!q || !k || !v || !beta || !out || !kv_out) return LASP_ERR_NULL;
    const size_t need = !state_cache && p.N <= lasp::delta_step_tokens(p) ? 0 : lasp::delta_scratch(p);
    if (need > 0 && (!scratch || scratch_bytes < need)) return LASP_ERR_WORKSPACE;
    if (need == 0) scratch = nullptr;
    const Sizes b(p);
    if (int rc = check({{q, b.keys}, {k, b.keys}, {v, b.values}, {log_g, b.gate}, {beta, b.gate}, {len, b.len}}, {kv_in, b.state},
                       {{out, b.values}, {state_cache, state_cache ? lasp::delta_cache(p) : 0}, {scratch, need}}, {kv_out, b.state});
        rc != LASP_OK)
        return rc;
    lasp::DeltaArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.log_g = log_g;
    a.beta = beta;
    a.kv_in = kv_in;
    a.len = len;
    a.out = out;
    a.kv_out = kv_out;
    a.cache = state_cache;
    a.scratch = scratch;
    return status(lasp::launch_delta_fwd(p, a, (hipStream_t)hip_stream));
}

int lasp_delta_bwd(const lasp_delta_shape *shape, const void *q, const void *k, const void *v, const float *log_g, const float *beta,
                   const int32_t *len, const void *dout, const float *dkv_out, const void *state_cache, void *dq, void *dk, void *dv,
                   float *dlog_g, float *dbeta, float *dkv_in, void *scratch, size_t scratch_bytes, void *hip_stream) {
    lasp::DeltaPlan p;
    if (int rc = make(shape, &p); rc != LASP_OK) return rc;
    if (!q || !k || !v || !beta || !dout || !state_cache || !dq || !dk || !dv || !dbeta || !dkv_in) return LASP_ERR_NULL;
    if ((log_g == nullptr) != (dlog_g == nullptr)) return LASP_ERR_NULL;   // a gate and its gradient, or neither
    const size_t need = lasp::delta_bwd_scratch(p);
    if (!scratch || scratch_bytes < need) return LASP_ERR_WORKSPACE;
    const Sizes b(p);
    if (int rc = check({{q, b.keys}, {k, b.keys}, {v, b.values}, {log_g, b.gate}, {beta, b.gate}, {len, b.len}, {dout, b.values},
                        {state_cache, lasp::delta_cache(p)}},
                       {dkv_out, b.state}, {{dq, b.keys}, {dk, b.keys}, {dv, b.values}, {dlog_g, b.gate}, {dbeta, b.gate}, {scratch, need}},
                       {dkv_in, b.state});
        rc != LASP_OK)
        return rc;
    lasp::DeltaArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.log_g = log_g;
    a.beta = beta;
    a.len = len;
    a.dout = dout;
    a.dkv_out = dkv_out;
    a.cache = const_cast<void *>(state_cache);
    a.dq = dq;
    a.dk = dk;
    a.dv = dv;
    a.dlog_g = dlog_g;
    a.dbeta = dbeta;
    a.dkv_in = dkv_in;
    a.scratch = scratch;
    return status(lasp::launch_delta_bwd(p, a, (hipStream_t)hip_stream));
}

}  // extern "C"
