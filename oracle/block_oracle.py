"""64-bit CPU oracle of the gated recurrence and of the norms around a mixer (test infrastructure only): the
definitions of include/lasp.h token by token, in numpy, beside the bounds that the GPU results are held to."""
import numpy as np

# half a step of the storage type, relative to the value
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def rec_fwd(x, log_a, h_in=None, lens=None, coupled=False):
    """(out [B,N,D], h_out [B,D]); rows past a sequence's length are 0."""
    B, N, D = x.shape
    h = np.zeros((B, D)) if h_in is None else np.array(h_in, dtype=np.float64)
    lens = np.full(B, N) if lens is None else np.clip(lens, 0, N)
    out = np.zeros((B, N, D))
    with np.errstate(over="ignore"):
        for b in range(B):
            for s in range(lens[b]):
                la = log_a[b, s]
                h[b] = np.exp(la) * h[b] + (-np.expm1(la) * x[b, s] if coupled else x[b, s])
                out[b, s] = h[b]
    return out, h


def rec_bwd(x, log_a, dout, h_in=None, lens=None, dh_out=None, coupled=False):
    """(dx, dlog_a, dh_in) of sum(out * dout) + sum(h_out * dh_out)."""
    B, N, D = x.shape
    out, _ = rec_fwd(x, log_a, h_in, lens, coupled)
    lens = np.full(B, N) if lens is None else np.clip(lens, 0, N)
    g = np.zeros((B, D)) if dh_out is None else np.array(dh_out, dtype=np.float64)
    dx, dl = np.zeros((B, N, D)), np.zeros((B, N, D))
    for b in range(B):
        for s in range(lens[b] - 1, -1, -1):
            a, e = np.exp(log_a[b, s]), dout[b, s] + g[b]
            before = out[b, s - 1] if s > 0 else (np.zeros(D) if h_in is None else h_in[b])
            dx[b, s] = -np.expm1(log_a[b, s]) * e if coupled else e
            g[b] = a * e
            dl[b, s] = g[b] * (before - x[b, s] if coupled else before)
    return dx, dl, g


def rec_bounds(dtype, x, log_a, dout=None, h_in=None, lens=None, dh_out=None, coupled=False):
    """What rounding may do to every output, element by element.

    A step rounds its result (2^-24), its gate (a relative (|log_a| + 4) 2^-24: the exponent's product and the power) and b x
    (2^-23); joining segments rounds as often again. With H the sum of the absolute terms, the state's error E follows
    E_s = a_s E_{s-1} + (|log_a_s| + 16) 2^-24 H_s, and an output is off by E and half a step of its type. dlog_a takes h_{s-1}
    as it was stored."""
    B, N, D = x.shape
    half = HALF[dtype]
    zero = np.zeros((B, D))
    with np.errstate(invalid="ignore"):
        delta = (np.minimum(np.abs(log_a), 100.0) + 16) * 2.0 ** -24
    a = np.exp(log_a)
    n = np.full(B, N) if lens is None else np.clip(lens, 0, N)

    def carry(terms, order, gates, start, extra=0.0):
        """Absolute sums and errors along `order` of rows; gates[s] multiplies what enters row s."""
        S, E = np.zeros((B, N, D)), np.zeros((B, N, D))
        end_s, end_e = np.abs(start), np.zeros((B, D))
        for b in range(B):
            for s in order(n[b]):
                end_e[b] = gates[b, s] * end_e[b]
                end_s[b] = gates[b, s] * end_s[b] + terms[b, s]
                end_e[b] += delta[b, s] * end_s[b] + (extra if np.isscalar(extra) else extra[b, s])
                S[b, s], E[b, s] = end_s[b], end_e[b]
        return S, E, end_s, end_e

    b_abs = np.abs(np.expm1(log_a)) if coupled else np.ones_like(a)
    # 1 - a from a as a single float, as bfloat16 calls and float ones with log_a > 0 form it: the power is off by at most 2^-24 of its
    # exponent's rounding and 2^-23 of its own for a <= 2, and the difference rounds once more, 2^-24: below 2^-22 of 1. bfloat16 calls take
    # -log_a within 2^-11 of 0, which is off by at most 2^-12 of 1 - a: below 2^-11 of it everywhere up to log_a = 0
    b_err = np.where((log_a > 0) | (dtype == "bf16"), 2.0 ** -22, 0.0) if coupled else np.zeros_like(a)
    b_err = np.where(log_a > 0, b_err, np.minimum(b_err, 2.0 ** -11 * b_abs))
    H, E, _, E_out = carry(b_abs * np.abs(x), range, a, zero if h_in is None else h_in, b_err * np.abs(x))
    out, h_out = rec_fwd(x, log_a, h_in, lens, coupled)
    got = {"out": half * np.abs(out) + E, "h_out": E_out + 2.0 ** -24 * np.abs(h_out)}
    if dout is None:
        return got
    # the gradient in front of row s, g_s = a_s (dout_s + g_{s+1})
    G, Eg, _, E_in = carry(a * np.abs(dout), lambda m: range(m - 1, -1, -1), a, zero if dh_out is None else dh_out)
    dx, dl, dh_in = rec_bwd(x, log_a, dout, h_in, lens, dh_out, coupled)
    first = zero if h_in is None else np.asarray(h_in, dtype=np.float64)
    before = np.concatenate([first[:, None], out[:, :-1]], axis=1)
    before_err = np.concatenate([np.zeros((B, 1, D)), E[:, :-1] + half * np.abs(out[:, :-1])], axis=1)
    other = before - x if coupled else before
    there = np.arange(N)[None, :, None] < n[:, None, None]
    # e_s = dout_s + g_{s+1}
    e_err = np.zeros((B, N, D))
    for b in range(B):
        for s in range(n[b]):
            e_err[b, s] = (Eg[b, s + 1] if s + 1 < n[b] else 0.0) + 2.0 ** -23 * (np.abs(dout[b, s]) + (G[b, s + 1] if s + 1 < n[b] else
                           np.abs(dh_out[b]) if dh_out is not None else 0.0))
    e_abs = np.where(there, np.abs(dx) / np.maximum(b_abs, 1e-30) if coupled else np.abs(dx), 0.0)
    got["dx"] = half * np.abs(dx) + b_abs * e_err + (delta * np.abs(dx) if coupled else 0.0) + b_err * e_abs
    got["dlog_a"] = half * np.abs(dl) + (Eg + delta * G) * np.abs(other) + G * (before_err + 2.0 ** -22 * (np.abs(before) + np.abs(x)))
    got["dlog_a"] = np.where(there, got["dlog_a"], 0.0)
    got["dh_in"] = E_in + 2.0 ** -24 * np.abs(dh_in)
    return got


# ---------------------------------------------------------------------------
# norms; KAPPA: rows are summed by at most 32 elements a lane and 26 partial sums, columns by at most 100 additions: fewer than 128
# roundings of 2^-24
# ---------------------------------------------------------------------------
KAPPA = 2.0 ** -17


def addnorm_fwd(r, x, scale, weight, eps):
    r_out = r if x is None else r + (1.0 if scale is None else scale) * x
    rstd = 1.0 / np.sqrt((r_out ** 2).mean(-1, keepdims=True) + eps)
    return r_out, (1.0 if weight is None else weight) * r_out * rstd


def addnorm_fwd_bounds(dtype, r, x, scale, weight, eps):
    half = HALF[dtype]
    r_out, y = addnorm_fwd(r, x, scale, weight, eps)
    parts = np.abs(r) + (0.0 if x is None else np.abs((1.0 if scale is None else scale) * x))
    off = 2.0 ** -22 * parts
    rstd = 1.0 / np.sqrt((r_out ** 2).mean(-1, keepdims=True) + eps)
    w = 1.0 if weight is None else np.abs(weight)
    # rstd moves with the errors of r_out as r_out . off / mean r_out^2, at most sqrt(mean off^2) rstd
    moved = np.sqrt((off ** 2).mean(-1, keepdims=True)) * rstd
    return {"r_out": half * np.abs(r_out) + off, "y": half * np.abs(y) + w * rstd * off + (KAPPA + moved) * np.abs(y)}


def addnorm_bwd(r, x, scale, weight, eps, dy, dr_out):
    """r: the sum as stored. (dr, dx, dscale, dweight)."""
    w, sc = 1.0 if weight is None else weight, 1.0 if scale is None else scale
    rstd = 1.0 / np.sqrt((r ** 2).mean(-1, keepdims=True) + eps)
    c = (w * dy * r).mean(-1, keepdims=True) * rstd ** 2
    dr = (0.0 if dr_out is None else dr_out) + rstd * (w * dy - r * c)
    return {"dr": dr, "dx": sc * dr, "dscale": None if x is None else (x * dr).sum(0), "dweight": (dy * r * rstd).sum(0)}


def addnorm_bwd_bounds(dtype, r, x, scale, weight, eps, dy, dr_out):
    half = HALF[dtype]
    ref = addnorm_bwd(r, x, scale, weight, eps, dy, dr_out)
    w, sc = 1.0 if weight is None else np.abs(weight), 1.0 if scale is None else np.abs(scale)
    rstd = 1.0 / np.sqrt((r ** 2).mean(-1, keepdims=True) + eps)
    c = (w * np.abs(dy * r)).mean(-1, keepdims=True) * rstd ** 2
    off = KAPPA * 4 * ((0.0 if dr_out is None else np.abs(dr_out)) + rstd * (w * np.abs(dy) + np.abs(r) * c))
    got = {"dr": half * np.abs(ref["dr"]) + off, "dx": half * np.abs(ref["dx"]) + sc * off + 2.0 ** -23 * np.abs(ref["dx"])}
    got["dweight"] = 4 * KAPPA * np.abs(dy * r * rstd).sum(0)
    if x is not None:
        got["dscale"] = (np.abs(x) * off).sum(0) + 4 * KAPPA * np.abs(x * ref["dr"]).sum(0)
    return got


def _act(u, gate):
    s = 1.0 / (1.0 + np.exp(-u))
    if gate == "identity":
        return u, np.ones_like(u)
    return (s, s * (1 - s)) if gate == "sigmoid" else (u * s, s * (1 + u * (1 - s)))


def _rows(o, over):
    """o [B,H,N,D] as [B,N,rows,C], tokens first."""
    B, H, N, D = o.shape
    t = o.transpose(0, 2, 1, 3)
    return t if over == "head" else t.reshape(B, N, 1, H * D)


def gatenorm(o, u, weight, eps, gate, over, dy=None):
    """{"y"} and, given dy, {"do", "du", "dweight"} and {"bound": the same names}, bounds without the output type's half step."""
    B, H, N, D = o.shape
    rows = _rows(o, over)
    shape = rows.shape
    rstd = 1.0 / np.sqrt((rows ** 2).mean(-1, keepdims=True) + eps)
    n = rows * rstd
    w = (np.ones(H * D) if weight is None else np.asarray(weight)).reshape((1, 1) + shape[2:])
    act, slope = (np.ones(shape), np.zeros(shape)) if gate == "none" else [v.reshape(shape) for v in _act(u, gate)]
    # the sigmoid and its complement: a relative (|u| + 4) 2^-23 each; the slope: twice that of s (1 - s), or of s (1 + |u| (1 - s))
    au = np.zeros(shape) if gate == "none" else np.abs(u).reshape(shape)
    act_off = 2.0 ** -21 * (1 + au) ** 2 * (np.abs(act) + (0 if gate in ("none", "identity") else 2.0 ** -6))
    slope_off = 0
    if gate not in ("none", "identity"):
        s, c = 1.0 / (1.0 + np.exp(-u.reshape(shape))), 1.0 / (1.0 + np.exp(u.reshape(shape)))
        slope_off = 2.0 ** -21 * (1 + au) ** 2 * s * (c if gate == "sigmoid" else 1.0 + au * c)
    flat = lambda t: t.reshape(B, N, H * D)   # noqa: E731
    y = w * n * act
    got = {"y": flat(y)}
    bound = {"y": flat(np.abs(w * n) * act_off + 2 * KAPPA * np.abs(y))}
    if dy is not None:
        g = dy.reshape(shape)
        t = g * act
        c = (w * t * n).mean(-1, keepdims=True)
        heads = lambda v: v.reshape(B, N, H, D).transpose(0, 2, 1, 3)   # noqa: E731
        got["do"] = heads(rstd * (w * t - n * c))
        t_off = np.abs(w * g) * act_off
        size = np.abs(w * t) + np.abs(n) * np.abs(w * t * n).mean(-1, keepdims=True)
        bound["do"] = heads(rstd * (t_off + np.abs(n) * (t_off * np.abs(n)).mean(-1, keepdims=True) + 4 * KAPPA * size))
        got["du"] = flat(g * w * n * slope)
        bound["du"] = flat(np.abs(g * w * n) * slope_off + 2 * KAPPA * np.abs(g * w * n * slope))
        got["dweight"] = (t * n).sum((0, 1)).reshape(H * D)
        bound["dweight"] = (4 * KAPPA * np.abs(t * n) + np.abs(g * n) * act_off).sum((0, 1)).reshape(H * D)
    got["bound"] = bound
    return got
