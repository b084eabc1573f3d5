// C-ABI host layer of the gated recurrence and of the norms around a mixer (lasp_rec_*, lasp_addnorm_*, lasp_gatenorm_*, lasp_qk_*):
// argument checks and dispatch. No device memory is allocated or freed here and nothing synchronises.
#include "../../include/lasp.h"

#include <algorithm>
#include <cmath>

#include "lasp_block.h"
#include "lasp_checks.h"

namespace {

using lasp::check_buffers;
using lasp::elem_bytes;
using lasp::Span;

constexpr int64_t kMost = 0x7fffffff;

bool known(int dtype) { return dtype == LASP_F32 || dtype == LASP_BF16; }
bool eighths(int64_t n) { return n > 0 && n % 8 == 0; }
// A row stride: 0 stands for `width`, which rows have at least; rows begin at 16 bytes.
bool valid_ld(int ld, int64_t width) { return ld == 0 || (ld >= width && ld % 8 == 0); }

int make_rec(const lasp_rec_shape *s, lasp::RecPlan *p) {
    if (!s) return LASP_ERR_NULL;
    if (!known(s->dtype)) return LASP_ERR_DTYPE;
    if (s->B < 1 || s->N < 1 || !eighths(s->D) || !valid_ld(s->ld, s->D)) return LASP_ERR_SHAPE;
    if ((int64_t)s->B * s->N > kMost || (int64_t)s->B * s->D > kMost) return LASP_ERR_SHAPE;
    *p = {s->B, s->N, s->D, s->dtype, s->coupled != 0, s->ld ? s->ld : s->D};
    return LASP_OK;
}
int make_rows(const lasp_rows *s, lasp::RowPlan *p) {
    if (!s) return LASP_ERR_NULL;
    if (!known(s->dtype)) return LASP_ERR_DTYPE;
    if (s->rows < 1 || !eighths(s->C) || s->C > 16384) return LASP_ERR_SHAPE;
    *p = lasp::row_plan(s->rows, 1, s->C, s->dtype);
    return LASP_OK;
}
int make_gate(const lasp_gate_shape *s, lasp::RowPlan *p) {
    if (!s) return LASP_ERR_NULL;
    if (!known(s->dtype)) return LASP_ERR_DTYPE;
    if (s->B < 1 || s->H < 1 || s->N < 1 || !eighths(s->D)) return LASP_ERR_SHAPE;
    const int64_t wide = (int64_t)s->H * s->D, tokens = (int64_t)s->B * s->N;
    if (wide > 16384 || tokens > kMost || tokens * s->H > kMost || !valid_ld(s->ld, wide)) return LASP_ERR_SHAPE;
    if (s->gate < LASP_GATE_NONE || s->gate > LASP_GATE_SILU) return LASP_ERR_SHAPE;
    if (s->over != LASP_OVER_HEAD && s->over != LASP_OVER_TOKEN) return LASP_ERR_SHAPE;
    const bool heads = s->over == LASP_OVER_HEAD;
    *p = lasp::row_plan((int)tokens, heads ? s->H : 1, heads ? s->D : (int)wide, s->dtype);
    return LASP_OK;
}

int make_qk(const lasp_qk_shape *s, lasp::QkPlan *p) {
    if (!s) return LASP_ERR_NULL;
    if (!known(s->dtype)) return LASP_ERR_DTYPE;
    if (s->B < 1 || s->N < 1 || s->H < 1 || s->key_heads < 0 || !eighths(s->D) || s->D > 256) return LASP_ERR_SHAPE;
    const int64_t tokens = (int64_t)s->B * s->N, heads = (int64_t)s->H + s->key_heads, q = (int64_t)s->H * s->D, k = (int64_t)s->key_heads * s->D;
    // (a group's rows are counted in 32 bits, tokens on their way past the last one too)
    if (heads > 65536 || tokens > kMost / 2 || tokens * heads > kMost || !valid_ld(s->ld, std::max(q, k))) return LASP_ERR_SHAPE;
    if (s->norm < LASP_NORM_NONE || s->norm > LASP_NORM_L2) return LASP_ERR_SHAPE;
    if (s->rot < 0 || s->rot > s->D || s->rot % 16 != 0) return LASP_ERR_SHAPE;
    if (s->layout != LASP_ROT_HALF && s->layout != LASP_ROT_INTERLEAVED) return LASP_ERR_SHAPE;
    *p = {s->B, s->N, s->H, s->key_heads, s->D, s->dtype, s->norm, s->rot, s->layout == LASP_ROT_HALF, s->ld ? s->ld : q, s->ld ? s->ld : k};
    return LASP_OK;
}

// A tensor of rows: `width` of the `ld` bytes from row to row are its own. Two of the same row stride may lie in each other's gaps.
struct Rows {
    const void *p;
    size_t n, width, ld;   // rows, bytes
    Span span() const { return {p, (n - 1) * ld + width}; }
};
bool overlap(const Rows &a, const Rows &b) {
    if (!lasp::overlap(a.span(), b.span())) return false;
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    const size_t apart = (x < y ? y - x : x - y) % a.ld;   // from a row of the one to the next row of the other
    return a.ld != b.ld || apart < (x < y ? a.width : b.width) || apart + (x < y ? b.width : a.width) > a.ld;
}
// As check_buffers, for tensors of rows. in_place[i] (may be null): an input that output i may coincide with.
int check_rows(std::initializer_list<Rows> ins, std::initializer_list<Rows> outs, std::initializer_list<const void *> in_place = {}) {
    for (const Rows &x : ins)
        if ((uintptr_t)x.p % 16 != 0) return LASP_ERR_ALIGN;
    for (const Rows &x : outs)
        if ((uintptr_t)x.p % 16 != 0) return LASP_ERR_ALIGN;
    size_t i = 0;
    for (const Rows &o : outs) {
        const void *same = i < in_place.size() ? in_place.begin()[i] : nullptr;
        ++i;
        if (!o.p) continue;
        for (const Rows &x : ins)
            if (x.p && !(o.p == same && x.p == same) && overlap(o, x)) return LASP_ERR_ALIAS;
        for (const Rows &o2 : outs)
            if (&o != &o2 && o2.p && overlap(o, o2)) return LASP_ERR_ALIAS;
    }
    return LASP_OK;
}
Rows whole(const void *p, size_t bytes) { return {p, 1, bytes, bytes}; }

// What the buffers of a recurrence's call take.
struct RecSizes {
    size_t rows, width, ld, state, len;
    explicit RecSizes(const lasp::RecPlan &p)
        : rows((size_t)p.B * p.N), width(p.D * lasp::elem_bytes(p.dtype)), ld(p.ld * lasp::elem_bytes(p.dtype)),
          state((size_t)p.B * p.D * sizeof(float)), len(p.B * sizeof(int32_t)) {}
    Rows gate(const void *p) const { return {p, rows, width, ld}; }
    Rows token(const void *p) const { return whole(p, rows * width); }
};

// What the buffers of a call on queries and keys take.
struct QkSizes {
    size_t e, tokens, q, k, ldq, ldk, weight, freq, pos;
    explicit QkSizes(const lasp::QkPlan &p)
        : e(lasp::elem_bytes(p.dtype)), tokens((size_t)p.B * p.N), q((size_t)p.H * p.D * e), k((size_t)p.Hk * p.D * e), ldq(p.ldq * e), ldk(p.ldk * e),
          weight(p.D * sizeof(float)), freq(p.rot / 2 * sizeof(double)), pos(tokens * sizeof(int32_t)) {}
    Rows xq(const void *p) const { return {p, tokens, q, ldq}; }
    Rows xk(const void *p) const { return k ? Rows{p, tokens, k, ldk} : whole(nullptr, 0); }
    Rows yq(const void *p) const { return whole(p, tokens * q); }
    Rows yk(const void *p) const { return whole(p, tokens * k); }
};
// What both calls are refused for beside their shape and buffers.
int check_qk(const lasp::QkPlan &p, float eps, float amplitude, const double *freq) {
    if (!(eps >= 0.0f) || !std::isfinite(eps) || !std::isfinite(amplitude)) return LASP_ERR_SHAPE;
    return p.rot > 0 && !freq ? LASP_ERR_NULL : LASP_OK;
}

bool bad_eps(float eps) { return !(eps >= 0.0f) || !std::isfinite(eps); }
int status(hipError_t e) { return e == hipSuccess ? LASP_OK : LASP_ERR_HIP; }

}  // namespace

extern "C" {

int lasp_check_rec(const lasp_rec_shape *shape) {
    lasp::RecPlan p;
    return make_rec(shape, &p);
}

size_t lasp_rec_scratch_bytes(const lasp_rec_shape *shape) {
    lasp::RecPlan p;
    return make_rec(shape, &p) == LASP_OK ? lasp::rec_scratch(p) : 0;
}

int lasp_rec_fwd(const lasp_rec_shape *shape, const void *x, const void *log_a, const float *h_in, const int32_t *len, void *out,
                 float *h_out, void *scratch, size_t scratch_bytes, void *hip_stream) {
    lasp::RecPlan p;
    if (int rc = make_rec(shape, &p); rc != LASP_OK) return rc;
    if (!x || !log_a || !out) return LASP_ERR_NULL;
    const size_t need = lasp::rec_scratch(p);
    if (!scratch || scratch_bytes < need) return LASP_ERR_WORKSPACE;
    const RecSizes b(p);
    if (int rc = check_rows({b.gate(x), b.gate(log_a), whole(h_in, b.state), whole(len, b.len)},
                            {b.token(out), whole(h_out, b.state), whole(scratch, need)}, {nullptr, h_in});
        rc != LASP_OK)
        return rc;
    lasp::RecArgs a{};
    a.x = x;
    a.log_a = log_a;
    a.h_in = h_in;
    a.len = len;
    a.out = out;
    a.h_out = h_out;
    a.scratch = scratch;
    return status(lasp::launch_rec_fwd(p, a, (hipStream_t)hip_stream));
}

int lasp_rec_bwd(const lasp_rec_shape *shape, const void *x, const void *log_a, const void *out, const float *h_in, const int32_t *len,
                 const void *dout, const float *dh_out, void *dx, void *dlog_a, float *dh_in, void *scratch, size_t scratch_bytes,
                 void *hip_stream) {
    lasp::RecPlan p;
    if (int rc = make_rec(shape, &p); rc != LASP_OK) return rc;
    if (!p.coupled) x = nullptr;
    if ((p.coupled && !x) || !log_a || !out || !dout || !dx || !dlog_a) return LASP_ERR_NULL;
    const size_t need = lasp::rec_scratch(p);
    if (!scratch || scratch_bytes < need) return LASP_ERR_WORKSPACE;
    const RecSizes b(p);
    if (int rc = check_rows({b.gate(x), b.gate(log_a), b.token(out), whole(h_in, b.state), whole(len, b.len), b.token(dout), whole(dh_out, b.state)},
                            {b.gate(dx), b.gate(dlog_a), whole(dh_in, b.state), whole(scratch, need)}, {nullptr, nullptr, dh_out});
        rc != LASP_OK)
        return rc;
    lasp::RecArgs a{};
    a.x = x;
    a.log_a = log_a;
    a.out_in = out;
    a.h_in = h_in;
    a.len = len;
    a.dout = dout;
    a.dh_out = dh_out;
    a.dx = dx;
    a.dlog_a = dlog_a;
    a.dh_in = dh_in;
    a.scratch = scratch;
    return status(lasp::launch_rec_bwd(p, a, (hipStream_t)hip_stream));
}

int lasp_check_rows(const lasp_rows *shape) {
    lasp::RowPlan p;
    return make_rows(shape, &p);
}

size_t lasp_addnorm_scratch_bytes(const lasp_rows *shape) {
    lasp::RowPlan p;
    return make_rows(shape, &p) == LASP_OK ? lasp::addnorm_scratch(p) : 0;
}

int lasp_addnorm_fwd(const lasp_rows *shape, const void *r, const void *x, const float *scale, const float *weight, float eps,
                     void *r_out, void *y, void *hip_stream) {
    lasp::RowPlan p;
    if (int rc = make_rows(shape, &p); rc != LASP_OK) return rc;
    if (bad_eps(eps)) return LASP_ERR_SHAPE;
    // a sum, and what goes into it, or neither
    if (!r || !y || (x && !r_out)) return LASP_ERR_NULL;
    if (!x && (r_out || scale)) return LASP_ERR_NULL;
    const size_t t = (size_t)p.tokens * p.C * elem_bytes(p.dtype), v = p.C * sizeof(float);
    if (int rc = check_rows({whole(r, t), whole(x, t), whole(scale, v), whole(weight, v)}, {whole(r_out, t), whole(y, t)}, {r}); rc != LASP_OK)
        return rc;
    lasp::AddNormArgs a{};
    a.r = r;
    a.x = x;
    a.scale = scale;
    a.weight = weight;
    a.eps = eps;
    a.r_out = r_out;
    a.y = y;
    return status(lasp::launch_addnorm_fwd(p, a, (hipStream_t)hip_stream));
}

int lasp_addnorm_bwd(const lasp_rows *shape, const void *r_out, const void *x, const float *scale, const float *weight, float eps,
                     const void *dy, const void *dr_out, void *dr, void *dx, float *dweight, float *dscale, void *scratch,
                     size_t scratch_bytes, void *hip_stream) {
    lasp::RowPlan p;
    if (int rc = make_rows(shape, &p); rc != LASP_OK) return rc;
    if (bad_eps(eps)) return LASP_ERR_SHAPE;
    if (!r_out || !dy || !dr || (dscale && !x)) return LASP_ERR_NULL;
    const bool sums = dweight || dscale;
    const size_t need = sums ? lasp::addnorm_scratch(p) : 0;
    if (sums && (!scratch || scratch_bytes < need)) return LASP_ERR_WORKSPACE;
    if (!sums) scratch = nullptr;
    if (!dscale) x = nullptr;
    const size_t t = (size_t)p.tokens * p.C * elem_bytes(p.dtype), v = p.C * sizeof(float);
    if (int rc = check_rows({whole(r_out, t), whole(x, t), whole(scale, v), whole(weight, v), whole(dy, t), whole(dr_out, t)},
                            {whole(dr, t), whole(dx, t), whole(dweight, v), whole(dscale, v), whole(scratch, need)}, {dr_out});
        rc != LASP_OK)
        return rc;
    lasp::AddNormArgs a{};
    a.r = r_out;
    a.x = x;
    a.scale = scale;
    a.weight = weight;
    a.eps = eps;
    a.dy = dy;
    a.dr_out = dr_out;
    a.dr = dr;
    a.dx = dx;
    a.dweight = dweight;
    a.dscale = dscale;
    a.scratch = (float *)scratch;
    return status(lasp::launch_addnorm_bwd(p, a, (hipStream_t)hip_stream));
}

int lasp_check_gate(const lasp_gate_shape *shape) {
    lasp::RowPlan p;
    return make_gate(shape, &p);
}

size_t lasp_gatenorm_scratch_bytes(const lasp_gate_shape *shape) {
    lasp::RowPlan p;
    return make_gate(shape, &p) == LASP_OK ? lasp::gatenorm_scratch(p) : 0;
}

int lasp_gatenorm_fwd(const lasp_gate_shape *shape, const void *o, const void *u, const float *weight, float eps, void *y,
                      void *hip_stream) {
    lasp::RowPlan p;
    if (int rc = make_gate(shape, &p); rc != LASP_OK) return rc;
    if (bad_eps(eps)) return LASP_ERR_SHAPE;
    if (shape->gate == LASP_GATE_NONE) u = nullptr;
    if (!o || !y || (shape->gate != LASP_GATE_NONE && !u)) return LASP_ERR_NULL;
    const size_t e = elem_bytes(p.dtype), wide = (size_t)shape->H * shape->D, n = (size_t)p.tokens;
    const size_t ld = shape->ld ? shape->ld : wide;
    if (int rc = check_rows({whole(o, n * wide * e), {u, n, wide * e, ld * e}, whole(weight, wide * sizeof(float))}, {whole(y, n * wide * e)});
        rc != LASP_OK)
        return rc;
    lasp::GateArgs a{};
    a.H = shape->H;
    a.N = shape->N;
    a.D = shape->D;
    a.gate = shape->gate;
    a.ld = (long long)ld;
    a.o = o;
    a.u = u;
    a.weight = weight;
    a.eps = eps;
    a.y = y;
    return status(lasp::launch_gatenorm_fwd(p, a, (hipStream_t)hip_stream));
}

int lasp_gatenorm_bwd(const lasp_gate_shape *shape, const void *o, const void *u, const float *weight, float eps, const void *dy,
                      void *d_o, void *du, float *dweight, void *scratch, size_t scratch_bytes, void *hip_stream) {
    lasp::RowPlan p;
    if (int rc = make_gate(shape, &p); rc != LASP_OK) return rc;
    if (bad_eps(eps)) return LASP_ERR_SHAPE;
    if (shape->gate == LASP_GATE_NONE) u = du = nullptr;
    if (!o || !dy || !d_o || (shape->gate != LASP_GATE_NONE && (!u || !du))) return LASP_ERR_NULL;
    const size_t need = dweight ? lasp::gatenorm_scratch(p) : 0;
    if (dweight && (!scratch || scratch_bytes < need)) return LASP_ERR_WORKSPACE;
    if (!dweight) scratch = nullptr;
    const size_t e = elem_bytes(p.dtype), wide = (size_t)shape->H * shape->D, n = (size_t)p.tokens;
    const size_t ld = shape->ld ? shape->ld : wide, v = wide * sizeof(float);
    if (int rc = check_rows({whole(o, n * wide * e), {u, n, wide * e, ld * e}, whole(weight, v), whole(dy, n * wide * e)},
                            {whole(d_o, n * wide * e), {du, n, wide * e, ld * e}, whole(dweight, v), whole(scratch, need)});
        rc != LASP_OK)
        return rc;
    lasp::GateArgs a{};
    a.H = shape->H;
    a.N = shape->N;
    a.D = shape->D;
    a.gate = shape->gate;
    a.ld = (long long)ld;
    a.o = o;
    a.u = u;
    a.weight = weight;
    a.eps = eps;
    a.dy = dy;
    a.d_o = d_o;
    a.du = du;
    a.dweight = dweight;
    a.scratch = (float *)scratch;
    return status(lasp::launch_gatenorm_bwd(p, a, (hipStream_t)hip_stream));
}

int lasp_check_qk(const lasp_qk_shape *shape) {
    lasp::QkPlan p;
    return make_qk(shape, &p);
}

size_t lasp_qk_scratch_bytes(const lasp_qk_shape *shape) {
    lasp::QkPlan p;
    return make_qk(shape, &p) == LASP_OK ? lasp::qk_scratch(p) : 0;
}

int lasp_qk_fwd(const lasp_qk_shape *shape, const void *xq, const void *xk, const float *wq, const float *wk, float eps, const double *freq,
                const int32_t *pos, float amplitude, void *q, void *k, void *hip_stream) {
    lasp::QkPlan p;
    if (int rc = make_qk(shape, &p); rc != LASP_OK) return rc;
    if (int rc = check_qk(p, eps, amplitude, freq); rc != LASP_OK) return rc;
    if (p.Hk == 0) xk = wk = nullptr, k = nullptr;
    if (p.rot == 0) freq = nullptr, pos = nullptr;
    if (!xq || !q || (p.Hk > 0 && (!xk || !k))) return LASP_ERR_NULL;
    const QkSizes b(p);
    if (int rc = check_rows({b.xq(xq), b.xk(xk), whole(wq, b.weight), whole(wk, b.weight), whole(freq, b.freq), whole(pos, b.pos)}, {b.yq(q), b.yk(k)});
        rc != LASP_OK)
        return rc;
    lasp::QkArgs a{};
    a.xq = xq;
    a.xk = xk;
    a.wq = wq;
    a.wk = wk;
    a.eps = eps;
    a.amplitude = amplitude;
    a.freq = freq;
    a.pos = pos;
    a.q = q;
    a.k = k;
    return status(lasp::launch_qk_fwd(p, a, (hipStream_t)hip_stream));
}

int lasp_qk_bwd(const lasp_qk_shape *shape, const void *xq, const void *xk, const float *wq, const float *wk, float eps, const double *freq,
                const int32_t *pos, float amplitude, const void *dq, const void *dk, void *dxq, void *dxk, float *dwq, float *dwk, void *scratch,
                size_t scratch_bytes, void *hip_stream) {
    lasp::QkPlan p;
    if (int rc = make_qk(shape, &p); rc != LASP_OK) return rc;
    if (int rc = check_qk(p, eps, amplitude, freq); rc != LASP_OK) return rc;
    if (p.Hk == 0) xk = wk = nullptr, dk = nullptr, dxk = nullptr, dwk = nullptr;
    if (p.rot == 0) freq = nullptr, pos = nullptr;
    const bool sums = dwq || dwk;
    if (p.norm == LASP_NORM_NONE && !sums) xq = xk = nullptr;
    else if (!xq || (p.Hk > 0 && !xk)) return LASP_ERR_NULL;
    if (!dq || !dxq || (p.Hk > 0 && (!dk || !dxk))) return LASP_ERR_NULL;
    const size_t need = sums ? lasp::qk_scratch(p) : 0;
    if (sums && (!scratch || scratch_bytes < need)) return LASP_ERR_WORKSPACE;
    if (!sums) scratch = nullptr;
    const QkSizes b(p);
    if (int rc = check_rows({b.xq(xq), b.xk(xk), whole(wq, b.weight), whole(wk, b.weight), whole(freq, b.freq), whole(pos, b.pos), b.yq(dq), b.yk(dk)},
                            {b.xq(dxq), b.xk(dxk), whole(dwq, b.weight), whole(dwk, b.weight), whole(scratch, need)});
        rc != LASP_OK)
        return rc;
    lasp::QkArgs a{};
    a.xq = xq;
    a.xk = xk;
    a.wq = wq;
    a.wk = wk;
    a.eps = eps;
    a.amplitude = amplitude;
    a.freq = freq;
    a.pos = pos;
    a.dq = dq;
    a.dk = dk;
    a.dxq = dxq;
    a.dxk = dxk;
    a.dwq = dwq;
    a.dwk = dwk;
    a.scratch = (float *)scratch;
    return status(lasp::launch_qk_bwd(p, a, (hipStream_t)hip_stream));
}

int lasp_rope_frequencies(int32_t rot, double base, int32_t scaling, double factor, double trained, double few_turns, double many_turns,
                          double *freq_host) {
    if (!freq_host) return LASP_ERR_NULL;
    const auto good = [](double x) { return std::isfinite(x) && x > 0.0; };
    if (rot < 4 || rot % 2 != 0 || !good(base) || scaling < LASP_ROPE_PLAIN || scaling > LASP_ROPE_BANDS) return LASP_ERR_SHAPE;
    if (scaling != LASP_ROPE_PLAIN && !good(factor)) return LASP_ERR_SHAPE;
    if (scaling == LASP_ROPE_BANDS && (!good(trained) || !std::isfinite(few_turns) || !std::isfinite(many_turns) || few_turns >= many_turns))
        return LASP_ERR_SHAPE;
    if (scaling == LASP_ROPE_BASE) base *= std::pow(factor, (double)rot / (rot - 2));
    for (int i = 0; i < rot / 2; ++i) {
        double f = std::pow(base, -2.0 * i / rot);
        if (scaling == LASP_ROPE_LINEAR) f /= factor;
        if (scaling == LASP_ROPE_BANDS) {
            const double turns = trained * f / 6.283185307179586477;
            const double keep = std::min(1.0, std::max(0.0, (turns - few_turns) / (many_turns - few_turns)));
            f = keep * f + (1.0 - keep) * f / factor;
        }
        freq_host[i] = f;
    }
    return LASP_OK;
}

}  // extern "C"
