"""64-bit CPU oracle of the gated delta rule and of the norm and rotation of queries and keys (test infrastructure only):
the definitions of include/lasp.h in numpy, token by token, beside the bounds that the GPU results are held to."""
import numpy as np

# half a step of the storage type, relative to the value
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}

# A float result of the delta rule comes out of at most 8 products one after the other (w, u, a state, an output; back through a state's gradient, dR, a
# gradient), each a sum of at most D + 64 <= 192 terms in float. Roundings of random sign add up to sqrt(192) 2^-24 of a sum's 2-norm, and by the definition no step
# makes an error grow (keys of length 1, 0 <= beta <= 2: I - beta k k^T has no value beyond 1). Eight of them, four times that for
# terms that partly cancel: 4 * 8 * sqrt(192) * 2^-24 = 2.6e-5 of the result's 2-norm.
DELTA = 4 * 8 * 192 ** 0.5 * 2.0 ** -24
# What float sums come to, as roundings of random sign spread evenly over half a step do: 2^-24 / sqrt(3) of a partial sum each, and partial sums of n terms grow to the
# whole one like sqrt(n), so that n roundings have sqrt(n / 2) of the last one's: sqrt(n / 6) 2^-24 of the sum, n at most D + 32 = 160 (a tile has 32 tokens). Eight of
# them independent of one another, twice that for terms that partly cancel: 2 sqrt(8 * 160 / 6) 2^-24 = 1.7e-6 of the 2-norm of a result of thousands of elements.
# Products whose computed factors are cut to two bfloat16 parts (2^-17) are off by more.
FLOAT = 2 * (8 * 160 / 6) ** 0.5 * 2.0 ** -24


def delta_fwd(q, k, v, log_g, beta, kv_in=None, lens=None):
    """(out [B,H,N,Dv], kv_out [B,H,D,Dv], the state in front of every token); q, k [B,key_heads,N,D]."""
    B, H, N, Dv = v.shape
    D, share = q.shape[-1], H // q.shape[1]
    S = np.zeros((B, H, D, Dv)) if kv_in is None else np.array(kv_in, dtype=np.float64)
    lens = np.full(B, N) if lens is None else np.clip(lens, 0, N)
    out, before = np.zeros((B, H, N, Dv)), np.zeros((N, B, H, D, Dv))
    a = np.ones((B, H, N)) if log_g is None else np.exp(log_g)
    for s in range(N):
        before[s] = S
        for b in range(B):
            if s >= lens[b]:
                continue
            ks, qs = (np.repeat(t[b, :, s], share, axis=0) for t in (k, q))
            S[b] *= a[b, :, s, None, None]
            w = v[b, :, s] - np.einsum("hd,hdc->hc", ks, S[b])
            S[b] += np.einsum("hd,hc->hdc", ks, beta[b, :, s, None] * w)
            out[b, :, s] = np.einsum("hd,hdc->hc", qs, S[b])
    return out, S, before


def delta_bwd(q, k, v, log_g, beta, dout, kv_in=None, lens=None, dkv_out=None):
    """dict of dq, dk, dv, dlog_g (with a gate), dbeta, dkv_in of sum(out * dout) + sum(kv_out * dkv_out)."""
    B, H, N, Dv = v.shape
    D, share = q.shape[-1], H // q.shape[1]
    _, _, before = delta_fwd(q, k, v, log_g, beta, kv_in, lens)
    lens = np.full(B, N) if lens is None else np.clip(lens, 0, N)
    a = np.ones((B, H, N)) if log_g is None else np.exp(log_g)
    dS = np.zeros((B, H, D, Dv)) if dkv_out is None else np.array(dkv_out, dtype=np.float64)
    g = {"dq": np.zeros_like(q, dtype=np.float64), "dk": np.zeros_like(k, dtype=np.float64), "dv": np.zeros((B, H, N, Dv)),
         "dbeta": np.zeros((B, H, N)), "dlog_g": np.zeros((B, H, N))}
    sums = lambda t: t.reshape(-1, share, D).sum(1)   # noqa: E731
    for b in range(B):
        for s in range(lens[b] - 1, -1, -1):
            ks, qs = (np.repeat(t[b, :, s], share, axis=0) for t in (k, q))
            aS, bt, do = a[b, :, s, None, None] * before[s, b], beta[b, :, s, None], dout[b, :, s]
            w = v[b, :, s] - np.einsum("hd,hdc->hc", ks, aS)
            S = aS + np.einsum("hd,hc->hdc", ks, bt * w)
            dS[b] += np.einsum("hd,hc->hdc", qs, do)
            g["dq"][b, :, s] = sums(np.einsum("hdc,hc->hd", S, do))
            du = np.einsum("hdc,hd->hc", dS[b], ks)
            g["dbeta"][b, :, s], g["dv"][b, :, s] = (du * w).sum(-1), bt * du
            g["dk"][b, :, s] = sums(np.einsum("hdc,hc->hd", dS[b], bt * w) - np.einsum("hdc,hc->hd", aS, bt * du))
            dS[b] -= np.einsum("hd,hc->hdc", ks, bt * du)
            g["dlog_g"][b, :, s] = (dS[b] * aS).sum((-1, -2))
            dS[b] *= a[b, :, s, None, None]
    g["dkv_in"] = dS
    if log_g is None:
        del g["dlog_g"]
    return g


def off(got, want, dtype, float_part=DELTA, floor=0.0):
    """How far `got` is from `want` in units of what rounding may do: in the 2-norm half a step of the storage type and `float_part` of the whole, and element
    by element half a step and 16 times that part of the values' root mean square. At most 1 is right. `floor`: a size of the terms that
    a small result is the difference of."""
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64)
    if not np.isfinite(got).all():
        return np.inf
    norm = max(np.linalg.norm(want), floor * want.size ** 0.5)
    err = np.abs(got - want)
    if norm == 0:
        return 0.0 if err.max(initial=0.0) == 0 else np.inf
    half = HALF[dtype]
    by_norm = np.linalg.norm(err) / ((half + float_part) * norm)
    rms = norm / want.size ** 0.5
    return max(by_norm, (err / (half * np.abs(want) + 16 * float_part * np.maximum(rms, np.abs(want)))).max())


def off_in_norm(got, want, floor=0.0):
    """The 2-norm of the difference in units of FLOAT times that of `want` (or of the size `floor` of its elements)."""
    want = np.asarray(want, dtype=np.float64)
    return np.linalg.norm(np.asarray(got, dtype=np.float64) - want) / (FLOAT * max(np.linalg.norm(want), floor * want.size ** 0.5))


# ---------------------------------------------------------------------------
# queries and keys
# ---------------------------------------------------------------------------
# Squares are summed over at most 8 elements a thread and 6 steps of a wave, a root, a quotient and 8 more operations follow, and a sine is good to 2 steps: below 32
# roundings of 2^-24. Sums over tokens (dw) take at most 2^16 / 1024 rows a thread and 16 partial sums one after the other: below 128.
QK = 32 * 2.0 ** -24
QK_SUM = 128 * 2.0 ** -24


def pairs_of(rot, layout):
    i = np.arange(rot // 2)
    return (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)


def rotate(n, pos, freq, rot, layout, amplitude, back=False):
    """amplitude R(pos) n of [..., N, D] (pos broadcastable to [..., N]); back: its transpose."""
    y = np.array(n, dtype=np.float64)
    if rot == 0:
        return y
    a, b = pairs_of(rot, layout)
    t = np.asarray(pos, dtype=np.float64)[..., None] * freq
    c, s = amplitude * np.cos(t), amplitude * np.sin(t) * (-1.0 if back else 1.0)
    y[..., a], y[..., b] = c * n[..., a] - s * n[..., b], s * n[..., a] + c * n[..., b]
    return y


def _scale(x, norm, eps):
    if norm == "none":
        return np.ones(x.shape[:-1] + (1,))
    sq = (x ** 2).sum(-1, keepdims=True)
    return 1.0 / np.sqrt((sq / x.shape[-1] if norm == "rms" else sq) + eps)


def heads_first(x, heads):
    B, N, C = x.shape
    return x.reshape(B, N, heads, C // heads).transpose(0, 2, 1, 3)


def qk_fwd(x, heads, w, norm, eps, pos, freq, rot, layout, amplitude):
    """[B,heads,N,D] of rows [B,N,heads*D]; pos [B,N]."""
    h = heads_first(np.asarray(x, dtype=np.float64), heads)
    return rotate(h * _scale(h, norm, eps) * (1.0 if w is None else w), pos[:, None], freq, rot, layout, amplitude)


def qk_bwd(x, heads, w, norm, eps, pos, freq, rot, layout, amplitude, dy):
    """(dx [B,N,heads*D], dw [D])."""
    h = heads_first(np.asarray(x, dtype=np.float64), heads)
    r = _scale(h, norm, eps)
    n = h * r
    dn = rotate(np.asarray(dy, dtype=np.float64), pos[:, None], freq, rot, layout, amplitude, back=True)
    dw = (dn * n).sum((0, 1, 2))
    dn = dn * (1.0 if w is None else w)
    if norm != "none":
        dn = r * (dn - n * (dn * n).sum(-1, keepdims=True) / (h.shape[-1] if norm == "rms" else 1))
    B, H, N, D = h.shape
    return dn.transpose(0, 2, 1, 3).reshape(B, N, H * D), dw
