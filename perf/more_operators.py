"""Timing cases of the gated delta rule and of what stands in front of a mixer: norms of queries and keys by head with the
position rotation, from the rows of a projection to the heads-first tensors that the mixers read.

A case is a dict of plain values. `prepare` makes what a caller's program holds before the call, `run` is one pass (in
plain torch, or with `own` through the library), `work` the bytes and flops a pass cannot do without, `exact` the same
results in 64 bits from the definitions.

Keys of a case (missing = 0 / False / ""):
    op          "delta"  S_s = a_s S_{s-1} + beta_s k_s (v_s - a_s S_{s-1}^T k_s)^T,  out_s = S_s^T q_s,  a_s = exp(log_g_s)
                "qk"     q, k = amplitude R(pos) (weight * Norm(x)), heads first, from rows that hold all heads of a token
    kind        "forward" or "train" (forward and backward)
    dtype       "bf16" or "f32"
    B, H, N, D  sequences, heads (qk: of queries), tokens, features of a query and key
    Dv          delta: features of a value (0 = D)
    key_heads   delta: heads of q and k, each shared by H / key_heads states (0 = H);  qk: heads of k (0 = no k)
    decay       delta: with a gate a_s (else a_s = 1)
    states      delta: a state enters (training: and a gradient of the last one)
    lens        delta: a batch of sequences of several lengths, padded to N
    packed      delta: several documents in one sequence, a = 0 at the first token of each
    norm        qk: "none", "rms", "l2"
    weight      qk: a weight per feature, shared by the heads
    rot         qk: features that are rotated (0 = none), `layout` "half" (i, i + rot / 2) or "interleaved" (2 i, 2 i + 1)
    scaling     qk: "none", "linear", "base" or "bands": how angles are scaled for contexts longer than the trained one
    far         qk: positions given per token, at the end of a long context (else 0 .. N - 1)
    fused       qk: q and k lie side by side, with values behind them, in the rows of one projection
"""
import math

import torch

own = False

EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # generation for a single user: one new token, each head's state read and written once; all launch and latency
        {"name": "delta_one_token", "op": "delta", "kind": "forward", "dtype": "bf16", "B": 1, "H": 16, "N": 1, "D": 128, "decay": True,
         "states": True},
        # generation for a batch of users
        {"name": "delta_batch_token", "op": "delta", "kind": "forward", "dtype": "bf16", "B": 64, "H": 16, "N": 1, "D": 128,
         "key_heads": 8, "decay": True, "states": True},
        # prompts of several lengths as one padded batch, before generation
        {"name": "delta_prompts", "op": "delta", "kind": "forward", "dtype": "bf16", "B": 8, "H": 16, "N": 1777, "D": 128, "decay": True,
         "lens": True},
        # training on one long sequence, at the sizes of the attention benchmark
        {"name": "delta_long_train", "op": "delta", "kind": "train", "dtype": "bf16", "B": 1, "H": 16, "N": 32768, "D": 128, "decay": True},
        # training on a batch, documents packed into the sequences, keys narrower than values, continued from left and right
        {"name": "delta_batch_train", "op": "delta", "kind": "train", "dtype": "bf16", "B": 8, "H": 8, "N": 4096, "D": 64, "Dv": 128,
         "key_heads": 4, "decay": True, "states": True, "packed": True},
        # full precision, odd length, without a gate
        {"name": "delta_train_f32", "op": "delta", "kind": "train", "dtype": "f32", "B": 2, "H": 4, "N": 1001, "D": 128, "Dv": 64},
        # generation: the queries and keys of one token a user, each at its own far position
        {"name": "qk_one_token", "op": "qk", "kind": "forward", "dtype": "bf16", "B": 64, "H": 16, "N": 1, "D": 128, "key_heads": 4,
         "norm": "rms", "weight": True, "rot": 128, "layout": "half", "scaling": "bands", "far": True, "fused": True},
        # a prompt of a model that rotates part of each head, interleaved, without norms
        {"name": "qk_part_prompt", "op": "qk", "kind": "forward", "dtype": "bf16", "B": 4, "H": 12, "N": 5003, "D": 96, "key_heads": 12,
         "norm": "none", "rot": 32, "layout": "interleaved", "scaling": "linear", "fused": True},
        # training at the width and length of the attention benchmark: 32768 tokens of 16 x 128 features
        {"name": "qk_long_train", "op": "qk", "kind": "train", "dtype": "bf16", "B": 1, "H": 16, "N": 32768, "D": 128, "key_heads": 16,
         "norm": "rms", "weight": True, "rot": 128, "layout": "half", "scaling": "base", "fused": True},
        # full precision, normalised as the delta rule takes its keys, few heads of keys, odd length
        {"name": "qk_train_f32", "op": "qk", "kind": "train", "dtype": "f32", "B": 3, "H": 8, "N": 2501, "D": 64, "key_heads": 2,
         "norm": "l2", "rot": 32, "layout": "half", "far": True},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    c = {"op": rng.choice(["delta", "delta", "qk"]), "dtype": "f32" if rng.random() < 0.25 else "bf16"}
    c["kind"] = "forward" if rng.random() < 0.4 else "train"
    c["H"] = _log_uniform(rng, 1, 32)
    if c["op"] == "delta":
        most = 1 << (25 if c["dtype"] == "f32" else 26)
        c["D"], c["Dv"] = rng.choice([64, 128, 128]), rng.choice([64, 128, 128])
        c["key_heads"] = rng.choice([n for n in range(1, c["H"] + 1) if c["H"] % n == 0]) if rng.random() < 0.4 else c["H"]
        wide = c["H"] * 128
        c["B"] = _log_uniform(rng, 1, min(64, most // (wide * 64)))
        c["N"] = _log_uniform(rng, 1, min(32768, most // (wide * c["B"])))
        if c["kind"] == "forward" and rng.random() < 0.3:
            c["N"] = rng.choice([1, 1, 2, 3])
        c["decay"], c["states"], c["lens"], c["packed"] = rng.random() < 0.8, rng.random() < 0.6, rng.random() < 0.3, rng.random() < 0.2
        return c
    c["D"] = rng.choice([64, 128, 128, 96, 80, 256])
    c["key_heads"] = rng.choice([n for n in range(0, c["H"] + 1) if n == 0 or c["H"] % n == 0])
    c["norm"], c["weight"] = rng.choice(["none", "rms", "rms", "l2"]), rng.random() < 0.6
    c["rot"] = 16 * rng.randint(0, c["D"] // 16) if rng.random() < 0.5 else c["D"]
    c["layout"], c["scaling"] = rng.choice(["half", "interleaved"]), rng.choice(["none", "linear", "base", "bands"])
    c["far"], c["fused"] = rng.random() < 0.5, rng.random() < 0.6
    most = 1 << (25 if c["dtype"] == "f32" else 26)
    c["B"] = _log_uniform(rng, 1, 64)
    c["N"] = _log_uniform(rng, 1, min(65536, most // (c["B"] * c["H"] * c["D"])))
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _sizes(case):
    """Key heads and value features of a delta case."""
    return case.get("key_heads") or case["H"], case.get("Dv") or case["D"]


def _frequencies(case):
    """Radians a position for every rotated pair, in 64 bits: 10000^(-2 i / rot), for a context 8 times as long as the trained one
    of 4096: all divided by 8 ("linear"), a larger base, so that the slowest is divided by 8 ("base"), or pairs that turn more than
    32 times within the trained context kept, less than once divided, and linear between ("bands")."""
    rot, factor, trained = case["rot"], 8.0, 4096.0
    i = torch.arange(0, rot, 2, dtype=torch.float64)
    base = 10000.0
    if case["scaling"] == "base":
        base *= factor ** (rot / (rot - 2))
    f = base ** (-i / rot)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "bands":
        turns = trained * f / (2 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        f = keep * f + (1.0 - keep) * f / factor
    return f.to("cuda")


def _inputs(case, seed):
    """Made from the seed alone. delta: keys and queries as a norm leaves them, of length 1 (queries over sqrt(D)), with a part that all of
    a head's have in common; memory of between 2 and 1000 tokens, another for every head; beta = sigmoid(N(0,1)). qk: rows ~ N(0,1)
    times a spread per feature."""
    dt, dev = DTYPES[case["dtype"]], "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device=dev, dtype=torch.float32)

    B, H, N, D = (case[k] for k in ("B", "H", "N", "D"))
    train, x = case["kind"] == "train", {}
    if case["op"] == "delta":
        Hk, Dv = _sizes(case)
        unit = lambda t: t / t.square().sum(-1, keepdim=True).sqrt()   # noqa: E731
        x["q"] = (unit(normal(B, Hk, N, D) + 0.3 * normal(Hk, 1, D)) / math.sqrt(D)).to(dt)
        x["k"] = unit(normal(B, Hk, N, D) + 0.3 * normal(Hk, 1, D)).to(dt)
        x["v"] = normal(B, H, N, Dv).to(dt)
        x["beta"] = 1.0 / (1.0 + torch.exp(-normal(B, H, N)))
        if case.get("decay"):
            memory = torch.exp(math.log(2.0) + uniform(H, 1) * math.log(500.0))
            x["log_g"] = -torch.exp(0.5 * normal(B, H, N)) / memory
            if case.get("packed"):
                x["log_g"] = torch.where(uniform(B, 1, N) < 5.0 / N, -math.inf, x["log_g"])
        if case.get("states"):
            x["kv_in"] = 0.3 * normal(B, H, D, Dv)
        if case.get("lens"):
            x["lens"] = (1.0 + uniform(B) * N).int().clamp(max=N)
        if train:
            x["dout"] = normal(B, H, N, Dv).to(dt)
            if case.get("states"):
                x["dkv_out"] = 0.1 * normal(B, H, D, Dv)
        return x
    Hk = case["key_heads"]
    wide = (H + 2 * Hk) * D
    if case.get("fused"):
        x["proj"] = (normal(B, N, wide) * (0.5 + uniform(wide))).to(dt)
    else:
        x["xq"] = (normal(B, N, H * D) * (0.5 + uniform(H * D))).to(dt)
        if Hk:
            x["xk"] = (normal(B, N, Hk * D) * (0.5 + uniform(Hk * D))).to(dt)
    if case.get("weight"):
        x["wq"] = 1.0 + 0.2 * normal(D)
        if Hk:
            x["wk"] = 1.0 + 0.2 * normal(D)
    if case["rot"]:
        x["freq"] = _frequencies(case)
        if case.get("far"):
            x["pos"] = ((uniform(B, 1) * 131072).long() + torch.arange(N, device=dev)).int()
    if train:
        x["dq"] = normal(B, H, N, D).to(dt)
        if Hk:
            x["dk"] = normal(B, Hk, N, D).to(dt)
    return x


def _amplitude(case):
    return 0.1 * math.log(8.0) + 1.0 if case["rot"] and case["scaling"] == "bands" else 1.0


def prepare(case, seed):
    if case["op"] == "qk":
        case = {"rot": 0, "layout": "half", "scaling": "none", **case}
    s = {"case": case, "in": _inputs(case, seed)}
    if own:
        s["plan"] = _plan(case, s["in"])
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
CHUNK = 64


def _strict_inverse(A):
    """(I + A)^-1 of strictly lower triangular A, joining inverses of diagonal blocks of twice the size each time."""
    n = A.shape[-1]
    i = torch.arange(n, device=A.device)
    T = torch.eye(n, device=A.device).expand_as(A)
    s = 1
    while s < n:
        below = (i[:, None] // (2 * s) == i[None, :] // (2 * s)) & (i[:, None] // s > i[None, :] // s)
        T = T - T @ (A * below) @ T
        s *= 2
    return T


def _chain(A, b):
    """All S_{c+1} = A_c S_c + b_c from S_0 = 0 along dim 2, by doubling."""
    k = 1
    while k < A.shape[2]:
        b = torch.cat([b[:, :, :k], b[:, :, k:] + A[:, :, k:] @ b[:, :, :-k]], dim=2)
        A = torch.cat([A[:, :, :k], A[:, :, k:] @ A[:, :, :-k]], dim=2)
        k *= 2
    return b


def _delta_chunks(case, q, k, v, log_g, beta, kv_in, lens):
    """out and kv_out in 32 bits, chunk by chunk: within a chunk the corrections u solve a triangular system, across chunks the
    states follow a chain of matrices."""
    B, H, N, D = (case[x] for x in ("B", "H", "N", "D"))
    Hk, Dv = _sizes(case)
    dev, C = v.device, CHUNK
    nc = -(-N // C)
    there = torch.arange(nc * C, device=dev)[None, :] < (lens[:, None] if lens is not None else N)

    def cut(t, heads):
        pad = torch.zeros(*t.shape[:2], nc * C - N, *t.shape[3:], device=dev)
        t = torch.cat([t, pad], dim=2)
        t = torch.where(there.view(-1, 1, nc * C, *([1] * (t.dim() - 3))), t, 0.0)
        return t.repeat_interleave(heads, dim=1).reshape(B, H, nc, C, *t.shape[3:])

    q, k, v, beta = cut(q, H // Hk), cut(k, H // Hk), cut(v, 1), cut(beta, 1)[..., None]
    G = cut(log_g.clamp(min=-200.0), 1).double().cumsum(-1) if log_g is not None else torch.zeros(B, H, nc, C, dtype=torch.float64, device=dev)
    i = torch.arange(C, device=dev)
    apart = G[..., :, None] - G[..., None, :]
    W = torch.where(i[:, None] >= i[None, :], apart, -math.inf).float().exp()
    strict = (i[:, None] > i[None, :])
    start, rest, whole = G.float().exp()[..., None], (G[..., -1:] - G).float().exp()[..., None], G[..., -1].float().exp()[..., None, None]
    T = _strict_inverse(beta * W * (k @ k.transpose(-1, -2)) * strict)
    u0, w0 = T @ (beta * v), T @ (beta * start * k)
    kr = (rest * k).transpose(-1, -2)
    A, b = whole * torch.eye(D, device=dev) - kr @ w0, kr @ u0
    b = torch.cat([b[:, :, :1] + A[:, :, :1] @ kv_in[:, :, None], b[:, :, 1:]], dim=2)
    S = _chain(A, b)
    S0 = torch.cat([kv_in[:, :, None], S[:, :, :-1]], dim=2)
    u = u0 - w0 @ S0
    out = start * (q @ S0) + (W * (q @ k.transpose(-1, -2))) @ u
    out = torch.where(there[:, None, :, None], out.reshape(B, H, nc * C, Dv), 0.0)
    return out[:, :, :N], S[:, :, -1]


def _delta_plain(case, i):
    B, H, D = (case[x] for x in ("B", "H", "D"))
    dt, train = DTYPES[case["dtype"]], case["kind"] == "train"
    x = {n: i[n].float() for n in ("q", "k", "v", "log_g", "beta") if n in i}
    x["kv_in"] = i["kv_in"] if "kv_in" in i else torch.zeros(B, H, D, _sizes(case)[1], device=i["v"].device)
    if not train:
        out, kv_out = _delta_chunks(case, x["q"], x["k"], x["v"], x.get("log_g"), x["beta"], x["kv_in"], i.get("lens"))
        return {"out": out.to(dt), "kv_out": kv_out}
    x = {n: t.detach().requires_grad_() for n, t in x.items()}
    out, kv_out = _delta_chunks(case, x["q"], x["k"], x["v"], x.get("log_g"), x["beta"], x["kv_in"], i.get("lens"))
    dkv_out = i["dkv_out"] if "dkv_out" in i else torch.zeros_like(kv_out)
    grads = torch.autograd.grad([out, kv_out], list(x.values()), [i["dout"].float(), dkv_out])
    got = {"out": out.detach().to(dt), "kv_out": kv_out.detach()}
    for n, g in zip(x, grads):
        got["d" + n] = g.to(dt) if n in ("q", "k", "v") else g
    return got


def _rotate(case, i, n, back):
    """amplitude R n of [B][H][N][D], or with `back` amplitude R^T n."""
    B, N, rot = case["B"], case["N"], case["rot"]
    if not rot:
        return n
    pos = i["pos"] if "pos" in i else torch.arange(N, device=n.device).expand(B, N)
    angle = pos.double()[:, None, :, None] * i["freq"]
    cos, sin = (angle.cos() * _amplitude(case)).float(), (angle.sin() * _amplitude(case)).float()
    sin = -sin if back else sin
    head, tail = n[..., :rot], n[..., rot:]
    if case["layout"] == "half":
        a, b = head[..., :rot // 2], head[..., rot // 2:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, tail], dim=-1)
    a, b = head[..., 0::2], head[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2), tail], dim=-1)


def _rows(case, i):
    """(name, rows, heads, weight) of the queries and keys."""
    H, Hk, D = case["H"], case["key_heads"], case["D"]
    if "proj" in i:
        parts = [("q", i["proj"][..., :H * D], H)] + ([("k", i["proj"][..., H * D:(H + Hk) * D], Hk)] if Hk else [])
    else:
        parts = [("q", i["xq"], H)] + ([("k", i["xk"], Hk)] if Hk else [])
    return [(n, x, h, i.get("w" + n)) for n, x, h in parts]


def _qk_plain(case, i):
    B, N, D = (case[x] for x in ("B", "N", "D"))
    dt, got, dproj = DTYPES[case["dtype"]], {}, []
    for name, x, h, w in _rows(case, i):
        x = x.float().reshape(B, N, h, D).transpose(1, 2)
        squares = x.square().sum(-1, keepdim=True)
        r = {"none": torch.ones_like(squares), "rms": (squares / D + EPS).rsqrt(), "l2": (squares + EPS).rsqrt()}[case["norm"]]
        n = x * r
        got[name] = _rotate(case, i, n if w is None else n * w, False).to(dt)
        if case["kind"] != "train":
            continue
        dn = _rotate(case, i, i["d" + name].float(), True)
        if w is not None:
            got["dw" + name] = (dn * n).sum((0, 1, 2))
            dn = dn * w
        if case["norm"] != "none":
            mean = (dn * n).sum(-1, keepdim=True) / (D if case["norm"] == "rms" else 1)
            dn = r * (dn - n * mean)
        dx = dn.to(dt).transpose(1, 2).reshape(B, N, h * D)
        if "proj" in i:
            dproj.append(dx)
        else:
            got["dx" + name] = dx
    if dproj:
        got["dproj"] = torch.cat(dproj, dim=-1)
    return got


# ---------------------------------------------------------------------------
# through the library
# ---------------------------------------------------------------------------
def _plan(case, i):
    """What a caller's program keeps: shape, workspaces and output buffers."""
    from paper_2404_02882_amd import lasp
    B, H, N, D = (case[k] for k in ("B", "H", "N", "D"))
    dt, train, p = DTYPES[case["dtype"]], case["kind"] == "train", {"lasp": lasp}

    def scratch(n):
        return torch.empty(n, dtype=torch.uint8, device="cuda")

    if case["op"] == "delta":
        Hk, Dv = _sizes(case)
        p["shape"] = lasp.make_delta_shape(B, H, N, D, dt, Dv=Dv, key_heads=Hk)
        need = lasp.delta_scratch_bytes(p["shape"])
        state = torch.empty(B, H, D, Dv, device="cuda")
        p.update(out=torch.empty_like(i["v"]), kv_out=state, cache=None)
        if train:
            need = max(need, lasp.delta_bwd_scratch_bytes(p["shape"]))
            p["cache"] = scratch(lasp.delta_cache_bytes(p["shape"]))
            p.update({"d" + n: torch.empty_like(i[n]) for n in ("q", "k", "v", "beta", "log_g") if n in i}, dkv_in=torch.empty_like(state))
        p["scratch"] = scratch(need)
        return p
    Hk = case["key_heads"]
    ld = (H + 2 * Hk) * D if case.get("fused") else 0
    p["shape"] = lasp.make_qk_shape(B, N, H, Hk, D, dt, norm=case["norm"], rot=case["rot"], layout=case["layout"], ld=ld)
    p["q"] = torch.empty(B, H, N, D, dtype=dt, device="cuda")
    p["k"] = torch.empty(B, Hk, N, D, dtype=dt, device="cuda") if Hk else None
    if train:
        p["scratch"] = scratch(lasp.qk_scratch_bytes(p["shape"]))
        p["grads"] = {"proj": torch.empty_like(i["proj"])} if "proj" in i else {n: torch.empty_like(i[n]) for n in ("xq", "xk") if n in i}
        p.update({"d" + n: torch.empty_like(i[n]) for n in ("wq", "wk") if n in i})
    return p


def _delta_own(case, i, p):
    lasp, log_g, lens = p["lasp"], i.get("log_g"), i.get("lens")
    lasp.lasp_delta_fwd(p["shape"], i["q"], i["k"], i["v"], log_g, i["beta"], i.get("kv_in"), lens, p["out"], p["kv_out"], p["cache"],
                        p["scratch"])
    got = {"out": p["out"], "kv_out": p["kv_out"]}
    if case["kind"] == "train":
        lasp.lasp_delta_bwd(p["shape"], i["q"], i["k"], i["v"], log_g, i["beta"], lens, i["dout"], i.get("dkv_out"), p["cache"], p["dq"],
                            p["dk"], p["dv"], p.get("dlog_g"), p["dbeta"], p["dkv_in"], p["scratch"])
        got.update({n: p[n] for n in ("dq", "dk", "dv", "dlog_g", "dbeta", "dkv_in") if n in p})
    return got


def _qk_own(case, i, p):
    lasp, parts = p["lasp"], _rows(case, i)
    xq, xk = parts[0][1], parts[1][1] if len(parts) > 1 else None
    wq, wk, freq, pos, amplitude = i.get("wq"), i.get("wk"), i.get("freq"), i.get("pos"), _amplitude(case)
    lasp.lasp_qk_fwd(p["shape"], xq, xk, wq, wk, EPS, freq, pos, amplitude, p["q"], p["k"])
    got = {"q": p["q"]}
    if p["k"] is not None:
        got["k"] = p["k"]
    if case["kind"] == "train":
        grads = _rows(case, p["grads"])
        lasp.lasp_qk_bwd(p["shape"], xq, xk, wq, wk, EPS, freq, pos, amplitude, i["dq"], i.get("dk"), grads[0][1],
                         grads[1][1] if len(grads) > 1 else None, p.get("dwq"), p.get("dwk"), p["scratch"])
        got.update({n: p[n] for n in ("dwq", "dwk") if n in p})
        if "proj" in p["grads"]:    # the rows' part that is q and k
            got["dproj"] = p["grads"]["proj"][..., :(case["H"] + case["key_heads"]) * case["D"]]
        else:
            got.update({"d" + n: t for n, t in p["grads"].items()})
    return got


def run(state):
    case, i = state["case"], state["in"]
    if own:
        return {"delta": _delta_own, "qk": _qk_own}[case["op"]](case, i, state["plan"])
    return {"delta": _delta_plain, "qk": _qk_plain}[case["op"]](case, i)


def work(case):
    e, train = 2 if case["dtype"] == "bf16" else 4, case["kind"] == "train"
    B, H, N, D = (case[k] for k in ("B", "H", "N", "D"))
    if case["op"] == "delta":
        Hk, Dv = _sizes(case)
        tokens, state, gates = B * N, 4 * B * H * D * Dv, 4 * (2 if case.get("decay") else 1)
        qkv = tokens * e * (2 * Hk * D + H * Dv)
        nbytes = qkv + tokens * H * (e * Dv + gates) + state * (2 if case.get("states") else 1)
        flops = 6 * tokens * H * D * Dv         # S^T k, k u^T, S^T q
        if train:                               # q, k, v, dout, gates again; their gradients; dkv_out and dkv_in
            nbytes += 2 * qkv + tokens * H * (e * Dv + 2 * gates) + state * (2 if case.get("states") else 1)
            flops += 14 * tokens * H * D * Dv   # q do^T, dS^T k, dS u, k de^T, S de, S do, and the states once more
        return {"bytes": nbytes, "flops": flops}
    Hk = case["key_heads"]
    t = B * N * (H + Hk) * D
    nbytes, flops = 2 * e * t, 8 * t
    if case.get("far") and case.get("rot"):
        nbytes += 4 * B * N * (2 if train else 1)
    if train:
        nbytes += (3 if case["norm"] != "none" or case.get("weight") else 2) * e * t
        flops += 16 * t
    return {"bytes": nbytes, "flops": flops}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _delta_exact(case, i):
    """Token by token, with one state kept for every 64."""
    B, H, N, D = (case[x] for x in ("B", "H", "N", "D"))
    Hk, Dv = _sizes(case)
    share, dev, f = H // Hk, i["v"].device, torch.float64
    lens = i["lens"].long() if "lens" in i else torch.full((B,), N, device=dev)

    def tokens_first(t, heads):
        t = t.to(f).repeat_interleave(heads, dim=1).transpose(0, 2).transpose(1, 2).contiguous()     # [N][B][H]...
        t[torch.arange(N, device=dev)[:, None] >= lens[None, :]] = 0.0
        return t

    q, k, v, beta = (tokens_first(i[n], share if n in "qk" else 1) for n in ("q", "k", "v", "beta"))
    a = tokens_first(i["log_g"], 1).exp() if "log_g" in i else torch.ones(N, B, H, dtype=f, device=dev)
    S = i["kv_in"].to(f).clone() if "kv_in" in i else torch.zeros(B, H, D, Dv, dtype=f, device=dev)

    def step(S, s):
        aS = a[s][..., None, None] * S
        e = v[s] - (aS * k[s][..., None]).sum(-2)
        return aS, e, torch.addcmul(aS, k[s][..., None], (beta[s][..., None] * e)[..., None, :])

    out, kept = torch.zeros(N, B, H, Dv, dtype=f, device=dev), []
    for s in range(N):
        if s % 64 == 0:
            kept.append(S)
        S = step(S, s)[2]
        out[s] = (S * q[s][..., None]).sum(-2)
    back = lambda t: t.transpose(1, 2).transpose(0, 2).contiguous()   # noqa: E731
    got = {"out": back(out), "kv_out": S}
    if case["kind"] != "train":
        return got
    do = tokens_first(i["dout"], 1)
    dS = i["dkv_out"].to(f).clone() if "dkv_out" in i else torch.zeros_like(S)
    dq, dk, dv, dbeta, dlog_g = (torch.zeros_like(t) for t in (q, k, v, beta, a))
    for c in reversed(range(len(kept))):
        first, states = 64 * c, [kept[c]]
        for s in range(first, min(N, first + 64)):
            states.append(step(states[-1], s)[2])
        for s in reversed(range(first, min(N, first + 64))):
            aS, e, S = step(states[s - first], s)
            dS = torch.addcmul(dS, q[s][..., None], do[s][..., None, :])
            dq[s] = (S * do[s][..., None, :]).sum(-1)
            du = (dS * k[s][..., None]).sum(-2)
            de = beta[s][..., None] * du
            dbeta[s], dv[s] = (du * e).sum(-1), de
            dk[s] = (dS * (beta[s][..., None] * e)[..., None, :]).sum(-1) - (aS * de[..., None, :]).sum(-1)
            dS = dS - k[s][..., None] * de[..., None, :]
            dlog_g[s] = (dS * aS).sum((-1, -2))
            dS = a[s][..., None, None] * dS
    gone = torch.arange(N, device=dev)[:, None] >= lens[None, :]
    for t in (dbeta, dlog_g):
        t[gone] = 0.0
    shared = lambda t: back(t).reshape(B, Hk, share, N, D).sum(2)   # noqa: E731
    got.update(dq=shared(dq), dk=shared(dk), dv=back(dv), dbeta=back(dbeta), dkv_in=dS)
    if "log_g" in i:
        got["dlog_g"] = back(dlog_g)
    return got


def _qk_exact(case, i):
    """Pairs as complex numbers, gradients by autograd."""
    B, N, D, rot, train = case["B"], case["N"], case["D"], case["rot"], case["kind"] == "train"
    got, dproj = {}, []
    for name, x, h, w in _rows(case, i):
        x = x.double().detach().clone().requires_grad_(train)
        leaves = {"dx" + name: x}
        y = x.view(B, N, h, D).permute(0, 2, 1, 3)
        if case["norm"] != "none":
            y = y / (y.pow(2).sum(-1, keepdim=True) / (D if case["norm"] == "rms" else 1) + EPS).sqrt()
        if w is not None:
            leaves["dw" + name] = w.double().detach().clone().requires_grad_(train)
            y = y * leaves["dw" + name]
        if rot:
            pos = i["pos"].double() if "pos" in i else torch.arange(N, device=x.device, dtype=torch.float64).expand(B, N)
            turn = torch.polar(torch.full((), _amplitude(case), dtype=torch.float64, device=x.device), pos[:, None, :, None] * i["freq"])
            pairs = y[..., :rot].reshape(B, h, N, 2, rot // 2).transpose(-1, -2) if case["layout"] == "half" else y[..., :rot].reshape(B, h, N, rot // 2, 2)
            turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            turned = (turned.transpose(-1, -2) if case["layout"] == "half" else turned).reshape(B, h, N, rot)
            y = torch.cat([turned, y[..., rot:]], dim=-1)
        got[name] = y.detach()
        if train:
            grads = dict(zip(leaves, torch.autograd.grad(y, list(leaves.values()), i["d" + name].double())))
            dx = grads.pop("dx" + name)
            got.update(grads)
            if "proj" in i:
                dproj.append(dx)
            else:
                got["dx" + name] = dx
    if dproj:
        got["dproj"] = torch.cat(dproj, dim=-1)
    return got


def exact(case, seed):
    if case["op"] == "qk":
        case = {"rot": 0, "layout": "half", "scaling": "none", **case}
    return {"delta": _delta_exact, "qk": _qk_exact}[case["op"]](case, _inputs(case, seed))
