"""Timing cases of the operators around and beside the attention: the gated linear recurrence, the residual add with
the norm before a block, and the norm with the gate behind it.

A case is a dict of plain values. `prepare` makes what a caller's program holds before the call, `run` is one pass (in
plain torch, or with `own` through the library), `work` the bytes and flops a pass cannot do without, `exact` the same
results in 64 bits from the definitions.

Keys of a case (missing = 0 / False):
    op          "rec" h_s = a_s h_{s-1} + b_s x_s, "addnorm" r' = r + scale x and y = w Norm(r'),
                "gatenorm" y = w Norm(o) act(u)
    kind        "forward", "backward" (addnorm: from the sum that the forward pass stored), "train" both
    dtype       "bf16" or "f32"
    B, N, D     rec: sequences, tokens, channels;  gatenorm: with H, heads of D features
    rows, C     addnorm: tokens and channels
    coupled     rec: b = 1 - a instead of 1
    states      rec: a state enters from the left (training: a gradient from the right)
    lens        rec: a batch of sequences of several lengths, padded to N
    packed      rec: several documents in one sequence, a = 0 at the first token of each
    fused       the inputs that come out of one projection lie side by side in its rows (so do their gradients)
    scale, weight, carry    addnorm: residual scale, norm weight, gradient that enters past the norm
    gate, over  gatenorm: "none", "identity", "sigmoid", "silu";  rows normalised over a "head" or a whole "token"
"""
import math

import torch

own = False

EPS = 1e-5
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # generation: one new token for a batch of sequences, each continuing its own state; all launch and latency
        {"name": "rec_one_token", "op": "rec", "kind": "forward", "dtype": "bf16", "B": 64, "N": 1, "D": 2048, "states": True},
        # prompts of several lengths as one padded batch, before generation
        {"name": "rec_prompts", "op": "rec", "kind": "forward", "dtype": "bf16", "B": 8, "N": 1777, "D": 2048, "coupled": True,
         "states": True, "lens": True},
        # training on one long sequence, value and gate from one projection
        {"name": "rec_long_train", "op": "rec", "kind": "train", "dtype": "bf16", "B": 1, "N": 32768, "D": 2048, "fused": True},
        # full precision, odd sizes, documents packed into the sequences, continued from left and right
        {"name": "rec_packed_train_f32", "op": "rec", "kind": "train", "dtype": "f32", "B": 2, "N": 4099, "D": 1000, "coupled": True,
         "states": True, "packed": True},
        # few channels, very long
        {"name": "rec_narrow_train", "op": "rec", "kind": "train", "dtype": "bf16", "B": 1, "N": 131072, "D": 128},
        # the largest: a training batch of long sequences at a width of 4096
        {"name": "rec_batch_train", "op": "rec", "kind": "train", "dtype": "bf16", "B": 4, "N": 16384, "D": 4096, "coupled": True},
        # generation again: the add and norm in front of the next block
        {"name": "addnorm_one_token", "op": "addnorm", "kind": "forward", "dtype": "bf16", "rows": 64, "C": 2048, "weight": True},
        # a residual stream kept in full precision, width that is no power of two
        {"name": "addnorm_forward_f32", "op": "addnorm", "kind": "forward", "dtype": "f32", "rows": 20011, "C": 1000, "weight": True,
         "scale": True},
        # training at the width and length of the attention benchmark: 32768 tokens of 16 x 128 features
        {"name": "addnorm_backward", "op": "addnorm", "kind": "backward", "dtype": "bf16", "rows": 32768, "C": 2048, "weight": True,
         "scale": True, "carry": True},
        # generation: the attention's output of one token, gated
        {"name": "gatenorm_one_token", "op": "gatenorm", "kind": "forward", "dtype": "bf16", "B": 64, "H": 16, "N": 1, "D": 128,
         "gate": "silu", "weight": True, "over": "head"},
        # training: the attention's output heads first, gate and result tokens first
        {"name": "gatenorm_heads_train", "op": "gatenorm", "kind": "train", "dtype": "bf16", "B": 1, "H": 16, "N": 32768, "D": 128,
         "gate": "silu", "weight": True, "over": "head"},
        # full precision, normalised over all heads of a token, odd length
        {"name": "gatenorm_token_train_f32", "op": "gatenorm", "kind": "train", "dtype": "f32", "B": 2, "H": 8, "N": 5001, "D": 64,
         "gate": "sigmoid", "weight": True, "over": "token"},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = {"op": rng.choice(["rec", "rec", "addnorm", "gatenorm"]), "dtype": "f32" if rng.random() < 0.25 else "bf16"}
    most = 1 << 26
    if c["op"] == "rec":
        c["kind"] = "forward" if rng.random() < 0.3 else "train"
        c["D"] = 8 * _log_uniform(rng, 1, 1024)
        c["B"] = _log_uniform(rng, 1, min(64, most // c["D"]))
        c["N"] = _log_uniform(rng, 1, min(131072, most // (c["D"] * c["B"])))
        c["coupled"], c["states"], c["fused"] = rng.random() < 0.4, rng.random() < 0.5, rng.random() < 0.3
        c["lens"], c["packed"] = rng.random() < 0.3, rng.random() < 0.2
    elif c["op"] == "addnorm":
        c["kind"] = rng.choice(["forward", "backward"])
        c["C"] = 8 * _log_uniform(rng, 1, 2048)
        c["rows"] = _log_uniform(rng, 1, min(65536, most // c["C"]))
        c["scale"], c["weight"], c["carry"] = rng.random() < 0.5, rng.random() < 0.8, rng.random() < 0.7
    else:
        c["kind"] = "forward" if rng.random() < 0.3 else "train"
        c["gate"], c["weight"] = rng.choice(["none", "identity", "sigmoid", "silu", "silu"]), rng.random() < 0.8
        c["over"] = rng.choice(["head", "head", "token"])
        if rng.random() < 0.25:     # behind a recurrence: one head as wide as the model
            c["H"], c["D"] = 1, 8 * _log_uniform(rng, 1, 1024)
        else:
            c["H"], c["D"] = rng.choice([1, 2, 3, 5, 8, 12, 16, 24, 32]), rng.choice([64, 128, 128, 96])
        c["B"] = _log_uniform(rng, 1, 32)
        c["N"] = _log_uniform(rng, 1, min(65536, most // (c["B"] * c["H"] * c["D"])))
        c["fused"] = rng.random() < 0.3
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _inputs(case, seed):
    """Made from the seed alone. rec: x ~ N(0,1); log a = log sigmoid of a logit around 4, other for every channel, as
    a gate's projection gives it (a between about 0.8 and 0.999); norms: rows ~ N(0,1) times a spread per channel."""
    dt, dev = DTYPES[case["dtype"]], "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device=dev, dtype=torch.float32)

    train, x = case["kind"] != "forward", {}
    if case["op"] == "rec":
        B, N, D = case["B"], case["N"], case["D"]
        value = normal(B, N, D)
        log_a = -torch.nn.functional.softplus(-(4.0 + normal(D) + 0.7 * normal(B, N, D)))
        if case.get("packed"):
            log_a[uniform(B, N) < 4.0 / N] = -math.inf
        if case.get("fused"):
            x["proj"] = torch.cat([value, log_a], dim=-1).to(dt)
        else:
            x["x"], x["log_a"] = value.to(dt), log_a.to(dt)
        if case.get("states"):
            x["h_in"] = 4.0 * normal(B, D)
        if case.get("lens"):
            n = (1.0 + uniform(B) * N).int().clamp(max=N)
            x["lens"] = n
        if train:
            x["dout"] = normal(B, N, D).to(dt)
            if case.get("states"):
                x["dh_out"] = normal(B, D)
        return x
    if case["op"] == "addnorm":
        R, C = case["rows"], case["C"]
        x["r"] = (2.0 * normal(R, C) * (0.5 + uniform(C))).to(dt)     # backward: the sum that the forward pass stored
        if not train or case.get("scale"):
            x["x"] = normal(R, C).to(dt)
        if case.get("scale"):
            x["scale"] = 0.1 + uniform(C)
        if case.get("weight"):
            x["weight"] = 1.0 + 0.2 * normal(C)
        if train:
            x["dy"] = normal(R, C).to(dt)
            if case.get("carry"):
                x["dr_out"] = normal(R, C).to(dt)
        return x
    B, H, N, D = (case[k] for k in ("B", "H", "N", "D"))
    x["o"] = (normal(B, H, N, D) * (0.2 + 2.0 * uniform(B, H, N, 1))).to(dt)
    if case["gate"] != "none":
        x["u"] = normal(B, N, (4 if case.get("fused") else 1) * H * D).to(dt)   # fused: behind q, k, v of one projection
    if case.get("weight"):
        x["weight"] = 1.0 + 0.2 * normal(H * D)
    if train:
        x["dy"] = normal(B, N, H * D).to(dt)
    return x


def prepare(case, seed):
    s = {"case": case, "in": _inputs(case, seed)}
    if own:
        s["plan"] = _plan(case, s["in"])
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _f(t):
    return None if t is None else t.float()


def _scan(a, u):
    """y_s = a_s y_{s-1} + u_s along dim 1 from y_{-1} = 0, by doubling: after a step, u_s is the part of y_s that comes from the
    last k tokens and a_s the product of their gates."""
    k = 1
    while k < u.shape[1]:
        u = torch.cat([u[:, :k], u[:, k:] + a[:, k:] * u[:, :-k]], dim=1)
        a = torch.cat([a[:, :k], a[:, k:] * a[:, :-k]], dim=1)
        k *= 2
    return u


def _rec_plain(case, i):
    B, N, D = case["B"], case["N"], case["D"]
    dt, dev, train = DTYPES[case["dtype"]], (i.get("proj") if "proj" in i else i["x"]).device, case["kind"] == "train"
    x, log_a = i["proj"].float().split(D, dim=-1) if case.get("fused") else (i["x"].float(), i["log_a"].float())
    n = i["lens"] if "lens" in i else torch.full((B,), N, device=dev)
    there = torch.arange(N, device=dev)[None, :, None] < n[:, None, None]
    a = torch.where(there, log_a.exp(), 1.0)
    b = torch.where(there, -torch.expm1(log_a) if case.get("coupled") else torch.ones_like(log_a), 0.0)
    h_in = i["h_in"] if "h_in" in i else torch.zeros(B, D, device=dev)
    u = b * x
    u[:, 0] += a[:, 0] * h_in
    h = _scan(a, u)
    got = {"out": torch.where(there, h, 0.0).to(dt), "h_out": h[:, -1].clone()}
    if not train:
        return got
    e = torch.where(there, i["dout"].float(), 0.0)
    if "dh_out" in i:
        e[:, -1] += i["dh_out"]
    after = torch.cat([a[:, 1:], torch.ones(B, 1, D, device=dev)], dim=1)
    e = _scan(after.flip(1), e.flip(1)).flip(1)
    before = torch.cat([h_in[:, None], h[:, :-1]], dim=1)
    dlog_a = torch.where(there, a * e * (before - x if case.get("coupled") else before), 0.0).to(dt)
    dx = (b * e).to(dt)
    got["dh_in"] = a[:, 0] * e[:, 0]
    if case.get("fused"):
        got["dproj"] = torch.cat([dx, dlog_a], dim=-1)
    else:
        got.update(dx=dx, dlog_a=dlog_a)
    return got


def _addnorm_plain(case, i):
    dt = DTYPES[case["dtype"]]
    r, x, scale, w = _f(i["r"]), _f(i.get("x")), i.get("scale"), i.get("weight")
    if case["kind"] == "forward":
        r = r + (x if scale is None else scale * x)
    rstd = (r.square().mean(-1, keepdim=True) + EPS).rsqrt()
    if case["kind"] == "forward":
        y = r * rstd
        return {"r_out": r.to(dt), "y": (y if w is None else y * w).to(dt)}
    dy = i["dy"].float()
    wdy = dy if w is None else dy * w
    dr = rstd * (wdy - r * rstd.square() * (wdy * r).mean(-1, keepdim=True))
    if "dr_out" in i:
        dr = dr + i["dr_out"].float()
    got = {"dr": dr.to(dt)}
    if scale is not None:
        got["dx"], got["dscale"] = (scale * dr).to(dt), (x * dr).sum(0)
    if w is not None:
        got["dweight"] = (dy * r * rstd).sum(0)
    return got


def _act(u, gate):
    """act(u) and its derivative."""
    if gate == "identity":
        return u, torch.ones_like(u)
    s = 1.0 / (1.0 + torch.exp(-u))
    return (s, s * (1.0 - s)) if gate == "sigmoid" else (u * s, s * (1.0 + u * (1.0 - s)))


def _gatenorm_plain(case, i):
    B, H, N, D = (case[k] for k in ("B", "H", "N", "D"))
    dt, gate = DTYPES[case["dtype"]], case["gate"]
    o = i["o"].float().transpose(1, 2)                      # [B][N][H][D]
    dims = (-1,) if case["over"] == "head" else (-2, -1)
    rstd = (o.square().mean(dims, keepdim=True) + EPS).rsqrt()
    n = o * rstd
    w = i["weight"].view(H, D) if case.get("weight") else torch.ones(H, D, device=o.device)
    if gate == "none":
        act, slope = torch.ones_like(o), torch.zeros_like(o)
    else:
        act, slope = _act(i["u"][..., -H * D:].float().reshape(B, N, H, D), gate)
    got = {"y": (w * n * act).to(dt).reshape(B, N, H * D)}
    if case["kind"] == "forward":
        return got
    dy = i["dy"].float().view(B, N, H, D)
    dt_ = dy * act
    wdt = w * dt_
    got["do"] = (rstd * (wdt - n * (wdt * n).mean(dims, keepdim=True))).to(dt).transpose(1, 2).contiguous()
    if gate != "none":
        got["du"] = (dy * w * n * slope).to(dt).reshape(B, N, H * D)
    if case.get("weight"):
        got["dweight"] = (dt_ * n).sum((0, 1)).reshape(H * D)
    return got


# ---------------------------------------------------------------------------
# through the library
# ---------------------------------------------------------------------------
def _plan(case, i):
    """What a caller's program keeps: shape, workspace and output buffers."""
    from paper_2404_02882_amd import lasp
    dt, train = DTYPES[case["dtype"]], case["kind"] != "forward"

    def like(t):
        return torch.empty_like(t)

    def f32(*shape):
        return torch.empty(*shape, dtype=torch.float32, device="cuda")

    def scratch(n):
        return torch.empty(n, dtype=torch.uint8, device="cuda")

    p = {"lasp": lasp}
    if case["op"] == "rec":
        B, N, D = case["B"], case["N"], case["D"]
        p["shape"] = lasp.make_rec_shape(B, N, D, dt, coupled=bool(case.get("coupled")), ld=2 * D if case.get("fused") else 0)
        p["scratch"] = scratch(lasp.rec_scratch_bytes(p["shape"]))
        p.update(out=torch.empty(B, N, D, dtype=dt, device="cuda"), h_out=f32(B, D))
        if train:
            p["dh_in"] = f32(B, D)
            if case.get("fused"):
                p["dproj"] = like(i["proj"])
            else:
                p.update(dx=like(i["x"]), dlog_a=like(i["log_a"]))
    elif case["op"] == "addnorm":
        p["shape"] = lasp.make_rows(case["rows"], case["C"], dt)
        if train:
            p["scratch"] = scratch(lasp.addnorm_scratch_bytes(p["shape"]))
            p["dr"] = like(i["r"])
            if case.get("scale"):
                p.update(dx=like(i["r"]), dscale=f32(case["C"]))
            if case.get("weight"):
                p["dweight"] = f32(case["C"])
        else:
            p.update(r_out=like(i["r"]), y=like(i["r"]))
    else:
        B, H, N, D = (case[k] for k in ("B", "H", "N", "D"))
        fused = case.get("fused") and case["gate"] != "none"
        p["shape"] = lasp.make_gate_shape(B, H, N, D, dt, gate=case["gate"], over=case["over"], ld=4 * H * D if fused else 0)
        p["y"] = torch.empty(B, N, H * D, dtype=dt, device="cuda")
        if train:
            p["scratch"] = scratch(lasp.gatenorm_scratch_bytes(p["shape"]))
            p["do"] = like(i["o"])
            if case["gate"] != "none":      # fused: the gate's part of the projection's gradient
                p["du"] = torch.empty_like(i["u"])[..., -H * D:]
            if case.get("weight"):
                p["dweight"] = f32(H * D)
    return p


def _rec_own(case, i, p):
    D, lasp = case["D"], p["lasp"]
    x, log_a = (i["proj"][..., :D], i["proj"][..., D:]) if case.get("fused") else (i["x"], i["log_a"])
    h_in, lens = i.get("h_in"), i.get("lens")
    lasp.lasp_rec_fwd(p["shape"], x, log_a, h_in, lens, p["out"], p["h_out"], p["scratch"])
    got = {"out": p["out"], "h_out": p["h_out"]}
    if case["kind"] == "train":
        dx, dlog_a = (p["dproj"][..., :D], p["dproj"][..., D:]) if case.get("fused") else (p["dx"], p["dlog_a"])
        lasp.lasp_rec_bwd(p["shape"], x, log_a, p["out"], h_in, lens, i["dout"], i.get("dh_out"), dx, dlog_a, p["dh_in"],
                          p["scratch"])
        got["dh_in"] = p["dh_in"]
        if case.get("fused"):
            got["dproj"] = p["dproj"]
        else:
            got.update(dx=dx, dlog_a=dlog_a)
    return got


def _addnorm_own(case, i, p):
    lasp = p["lasp"]
    if case["kind"] == "forward":
        lasp.lasp_addnorm_fwd(p["shape"], i["r"], i["x"], i.get("scale"), i.get("weight"), EPS, p["r_out"], p["y"])
        return {"r_out": p["r_out"], "y": p["y"]}
    lasp.lasp_addnorm_bwd(p["shape"], i["r"], i.get("x"), i.get("scale"), i.get("weight"), EPS, i["dy"], i.get("dr_out"), p["dr"],
                          p.get("dx"), p.get("dweight"), p.get("dscale"), p["scratch"])
    return {k: p[k] for k in ("dr", "dx", "dscale", "dweight") if k in p}


def _gatenorm_own(case, i, p):
    lasp, HD = p["lasp"], case["H"] * case["D"]
    u = i["u"][..., -HD:] if "u" in i else None
    lasp.lasp_gatenorm_fwd(p["shape"], i["o"], u, i.get("weight"), EPS, p["y"])
    got = {"y": p["y"]}
    if case["kind"] == "train":
        lasp.lasp_gatenorm_bwd(p["shape"], i["o"], u, i.get("weight"), EPS, i["dy"], p["do"], p.get("du"), p.get("dweight"),
                               p["scratch"])
        got.update({k: p[k] for k in ("do", "du", "dweight") if k in p})
    return got


def run(state):
    case, i = state["case"], state["in"]
    if own:
        return {"rec": _rec_own, "addnorm": _addnorm_own, "gatenorm": _gatenorm_own}[case["op"]](case, i, state["plan"])
    return {"rec": _rec_plain, "addnorm": _addnorm_plain, "gatenorm": _gatenorm_plain}[case["op"]](case, i)


def work(case):
    e, train = 2 if case["dtype"] == "bf16" else 4, case["kind"] != "forward"
    if case["op"] == "rec":
        t, state = case["B"] * case["N"] * case["D"], 4 * case["B"] * case["D"]
        nbytes, flops = 3 * e * t + state, (5 if case.get("coupled") else 3) * t
        if case.get("states"):
            nbytes += state
        if train:       # the forward pass, then log a, out, dout (coupled: x) -> dx, dlog a
            nbytes += (6 if case.get("coupled") else 5) * e * t + state * (3 if case.get("states") else 1)
            flops += (9 if case.get("coupled") else 6) * t
        return {"bytes": nbytes, "flops": flops}
    if case["op"] == "addnorm":
        t, vec = case["rows"] * case["C"], 4 * case["C"]
        vecs = int(bool(case.get("scale"))) + int(bool(case.get("weight")))
        if not train:
            return {"bytes": 4 * e * t + vecs * vec, "flops": 6 * t}
        return {"bytes": e * t * (3 + (2 if case.get("scale") else 0) + int(bool(case.get("carry")))) + 2 * vecs * vec, "flops": 12 * t}
    t, vec, gated = case["B"] * case["H"] * case["N"] * case["D"], 4 * case["H"] * case["D"], case["gate"] != "none"
    nbytes, flops = e * t * (3 if gated else 2), 8 * t
    if train:
        nbytes += e * t * (5 if gated else 3)
        flops += 20 * t
    return {"bytes": nbytes + (vec * (3 if train else 1) if case.get("weight") else 0), "flops": flops}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _rec_exact(case, i):
    """Token by token, tokens first in memory."""
    B, N, D = case["B"], case["N"], case["D"]
    d = lambda t: t.double().transpose(0, 1).contiguous()   # noqa: E731
    x, log_a = (d(t) for t in ((i["proj"][..., :D], i["proj"][..., D:]) if case.get("fused") else (i["x"], i["log_a"])))
    dev = x.device
    a = log_a.exp()
    b = 1.0 - a if not case.get("coupled") else -torch.expm1(log_a)
    if not case.get("coupled"):
        b = torch.ones_like(a)
    lens = i["lens"].long() if "lens" in i else torch.full((B,), N, dtype=torch.long, device=dev)
    gone = torch.arange(N, device=dev)[:, None] >= lens[None, :]
    a[gone], b[gone], x[gone] = 1.0, 0.0, 0.0
    h = i["h_in"].double() if "h_in" in i else torch.zeros(B, D, dtype=torch.float64, device=dev)
    hs = torch.empty(N + 1, B, D, dtype=torch.float64, device=dev)
    hs[0] = h
    bx = b * x
    for s in range(N):
        torch.addcmul(bx[s], a[s], hs[s], out=hs[s + 1])
    back = lambda t: t.transpose(0, 1).contiguous()   # noqa: E731
    out = hs[1:].clone()
    out[gone] = 0.0
    got = {"out": back(out), "h_out": hs[N].clone()}
    if case["kind"] != "train":
        return got
    do = d(i["dout"])
    do[gone] = 0.0
    g = i["dh_out"].double() if "dh_out" in i else torch.zeros(B, D, dtype=torch.float64, device=dev)
    for s in range(N - 1, -1, -1):      # do becomes the gradient with respect to h_s
        do[s] += g
        g = a[s] * do[s]
    dlog_a = a * do * (hs[:N] - x if case.get("coupled") else hs[:N])
    dlog_a[gone] = 0.0
    dx, dlog_a = back(b * do), back(dlog_a)
    got["dh_in"] = g
    if case.get("fused"):
        got["dproj"] = torch.cat([dx, dlog_a], dim=-1)
    else:
        got.update(dx=dx, dlog_a=dlog_a)
    return got


def _by_autograd(outputs, grads, wrt):
    return torch.autograd.grad(outputs, wrt, grads, allow_unused=True)


def _addnorm_exact(case, i):
    d = {k: t.double() for k, t in i.items()}
    if case["kind"] == "forward":
        r = d["r"] + d["x"] * d.get("scale", 1.0)
        return {"r_out": r, "y": d.get("weight", 1.0) * r / (r.pow(2).sum(-1, keepdim=True) / case["C"] + EPS).sqrt()}
    # gradients of <y, dy> + <r, dr_out> through r = r0 + scale x
    scale, w, x = d.get("scale"), d.get("weight"), d.get("x")
    r0 = d["r"].requires_grad_()
    leaves = {"dr": r0}
    if w is not None:
        leaves["dweight"] = w.requires_grad_()
    y = r0 / (r0.pow(2).sum(-1, keepdim=True) / case["C"] + EPS).sqrt()
    y = y if w is None else w * y
    loss = (y * d["dy"]).sum() + ((r0 * d["dr_out"]).sum() if "dr_out" in d else 0.0)
    got = dict(zip(leaves, _by_autograd(loss, None, list(leaves.values()))))
    if scale is not None:
        got["dx"], got["dscale"] = scale * got["dr"], (x * got["dr"]).sum(0)
    return {k: got[k] for k in ("dr", "dx", "dscale", "dweight") if k in got}


def _gatenorm_exact(case, i):
    B, H, N, D = (case[k] for k in ("B", "H", "N", "D"))
    train = case["kind"] == "train"
    leaves = {"do": i["o"].double().requires_grad_(train)}
    t = leaves["do"].permute(0, 2, 1, 3).reshape(B, N, H * D)
    rows = t.reshape(B, N, H, D) if case["over"] == "head" else t.reshape(B, N, 1, H * D)
    y = (rows / (rows.pow(2).sum(-1, keepdim=True) / rows.shape[-1] + EPS).sqrt()).reshape(B, N, H * D)
    if case["gate"] != "none":
        u = leaves["du"] = i["u"][..., -H * D:].double().clone().requires_grad_(train)
        y = y * {"identity": lambda v: v, "sigmoid": torch.sigmoid, "silu": lambda v: v * torch.sigmoid(v)}[case["gate"]](u)
    if case.get("weight"):
        leaves["dweight"] = i["weight"].double().requires_grad_(train)
        y = y * leaves["dweight"]
    got = {"y": y.detach()}
    if train:
        got.update(zip(leaves, _by_autograd(y, i["dy"].double(), list(leaves.values()))))
    return {k: got[k] for k in ("y", "do", "du", "dweight") if k in got}


def exact(case, seed):
    return {"rec": _rec_exact, "addnorm": _addnorm_exact, "gatenorm": _gatenorm_exact}[case["op"]](case, _inputs(case, seed))
