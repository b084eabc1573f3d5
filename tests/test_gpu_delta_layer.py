"""The gated delta rule as a layer uses it: norm before the block, one projection to queries, keys, values and gate, queries and keys normalised by head
and rotated, the delta rule over two sub-sequences, norm and gate behind it, projection back, residual add; then the attention with decay behind
the same norms and rotation. Forward and backward in float against 64-bit autograd of the same formulas, then captured and replayed.

Tolerance: every value passes at most 12 operators between an input and an output, each with a relative error of at most about 2^-16
of its terms: 1e-3 in the 2-norm leaves room for their growth through norms with factors of order 1."""
import pytest
import torch

pytestmark = pytest.mark.gpu

B, H, HK, N, D = 2, 4, 2, 150, 64
C, WIDE, EPS = H * D, (2 * HK + 2 * H) * D, 1e-5
SPLIT = [HK * D, HK * D, H * D, H * D]


@pytest.fixture(scope="module")
def gpu():
    assert torch.cuda.is_available(), "needs a GPU"
    from paper_2404_02882_amd import lasp, sequence
    return lasp, sequence


def parameters():
    g = torch.Generator().manual_seed(21)
    r = lambda *s: torch.randn(*s, generator=g)   # noqa: E731
    return {"x": r(B, N, C), "dout": r(B, N, C), "w1": 1 + 0.1 * r(C), "wq": 1 + 0.1 * r(D), "wk": 1 + 0.1 * r(D), "w2": 1 + 0.1 * r(C),
            "P": r(C, WIDE) / C ** 0.5, "PB": r(C, H) / C ** 0.5, "PG": r(C, H) / C ** 0.5, "Q": r(C, C) / C ** 0.5}


def norm(x, w):
    return w * x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt()


def reference(p, freq, mixer, lam):
    """64 bits, by autograd."""
    p = {k: v.double().requires_grad_(k != "dout") for k, v in p.items()}
    n = norm(p["x"], p["w1"])
    q, k, v, u = (n @ p["P"]).split(SPLIT, dim=-1)
    beta, log_g = torch.sigmoid(n @ p["PB"]).transpose(1, 2), -torch.nn.functional.softplus(n @ p["PG"] - 2.0).transpose(1, 2)

    def heads(t, w, h):
        t = t.reshape(B, N, h, D).transpose(1, 2)
        t = w * t * (t.square().sum(-1, keepdim=True) + EPS).rsqrt()
        a, b = t[..., :16], t[..., 16:32]
        ang = torch.arange(N, dtype=torch.float64)[:, None] * freq
        return torch.cat([a * ang.cos() - b * ang.sin(), a * ang.sin() + b * ang.cos(), t[..., 32:]], dim=-1).repeat_interleave(H // h, dim=1)
    q, k = heads(q, p["wq"], HK), heads(k, p["wk"], HK)
    v = v.reshape(B, N, H, D).transpose(1, 2)
    if mixer == "delta":
        S, o = torch.zeros(B, H, D, D, dtype=torch.float64), []
        for s in range(N):
            aS = log_g[:, :, s, None, None].exp() * S
            w = v[:, :, s] - (aS * k[:, :, s, :, None]).sum(-2)
            S = aS + k[:, :, s, :, None] * (beta[:, :, s, None] * w)[..., None, :]
            o.append((S * q[:, :, s, :, None]).sum(-2))
        o = torch.stack(o, 2)
    else:
        i = torch.arange(N)
        M = torch.where(i[:, None] >= i[None, :], lam.double().view(H, 1, 1) ** (i[:, None] - i[None, :]).clamp(min=0),
                        torch.zeros((), dtype=torch.float64))
        o = ((q @ k.transpose(-1, -2)) * M) @ v
    o = o * (o.square().mean(-1, keepdim=True) + EPS).rsqrt()
    y = p["w2"] * o.transpose(1, 2).reshape(B, N, C) * torch.nn.functional.silu(u)
    out = p["x"] + y @ p["Q"]
    wrt = [k for k in p if k != "dout" and (mixer == "delta" or k not in ("PB", "PG"))]
    grads = torch.autograd.grad((out * p["dout"]).sum(), [p[k] for k in wrt])
    return out.detach(), dict(zip(wrt, grads))


class Layer:
    """Everything between the torch products through the library, forward and backward."""

    def __init__(self, lasp, sequence, p, freq, mixer, lam):
        self.L, self.p, self.freq, self.mixer, self.lam = lasp, {k: v.cuda() for k, v in p.items()}, freq.cuda(), mixer, lam.cuda()
        f = torch.float32
        self.T = 2 if mixer == "delta" else 1
        self.mix = sequence.DeltaSequence(B, H, N, D, f, self.T, key_heads=HK) if mixer == "delta" else sequence.LaspSequence(B, H, N, D, 64, f)
        self.rows = lasp.make_rows(B * N, C, f)
        self.qk = lasp.make_qk_shape(B, N, HK, HK, D, f, "l2", 32, "half", WIDE)
        self.gate = lasp.make_gate_shape(B, H, N, D, f, "silu", "head", WIDE)
        need = max(lasp.addnorm_scratch_bytes(self.rows), lasp.qk_scratch_bytes(self.qk), lasp.gatenorm_scratch_bytes(self.gate))
        self.scratch = torch.empty(need, dtype=torch.uint8, device="cuda")
        self.grads = {k: torch.zeros_like(v) for k, v in self.p.items() if k != "dout"}
        self.out = torch.empty(B, N, C, device="cuda")

    def run(self):
        L, p, g = self.L, self.p, self.grads
        new = lambda *s: torch.empty(*s, device="cuda")   # noqa: E731
        cut = lambda t: [c.contiguous() for c in t.chunk(self.T, dim=2)]   # noqa: E731
        share = 1 if self.mixer == "delta" else H // HK
        n = new(B, N, C)
        L.lasp_addnorm_fwd(self.rows, p["x"], None, None, p["w1"], EPS, None, n)
        proj = n @ p["P"]
        parts = proj.split(SPLIT, dim=-1)
        q, k = new(B, HK, N, D), new(B, HK, N, D)
        L.lasp_qk_fwd(self.qk, parts[0], parts[1], p["wq"], p["wk"], EPS, self.freq, None, 1.0, q, k)
        v = parts[2].reshape(B, N, H, D).transpose(1, 2).contiguous()
        qs, ks, vs = cut(q.repeat_interleave(share, dim=1)), cut(k.repeat_interleave(share, dim=1)), cut(v)
        o = [torch.empty_like(t) for t in vs]
        if self.mixer == "delta":
            zb, zg = n @ p["PB"], n @ p["PG"] - 2.0
            beta, log_g = torch.sigmoid(zb).transpose(1, 2), -torch.nn.functional.softplus(zg).transpose(1, 2)
            bs, gs = cut(beta), cut(log_g)
            self.mix.forward(qs, ks, vs, gs, bs, o)
        else:
            self.mix.forward(qs, ks, vs, self.lam, o)
        whole = torch.cat(o, dim=2)
        y = new(B, N, C)
        L.lasp_gatenorm_fwd(self.gate, whole, parts[3], p["w2"], EPS, y)
        self.out.copy_(p["x"] + y @ p["Q"])
        # backward
        dy = p["dout"] @ p["Q"].t()
        g["Q"].copy_(y.reshape(-1, C).t() @ p["dout"].reshape(-1, C))
        do, dproj = torch.empty_like(whole), new(B, N, WIDE)
        dparts = dproj.split(SPLIT, dim=-1)
        L.lasp_gatenorm_bwd(self.gate, whole, parts[3], p["w2"], EPS, dy, do, dparts[3], g["w2"], self.scratch)
        dq, dk, dv = ([torch.empty_like(t) for t in x] for x in (qs, ks, vs))
        dn = torch.zeros(B, N, C, device="cuda")
        if self.mixer == "delta":
            dg, db = [torch.empty_like(t) for t in gs], [torch.empty_like(t) for t in bs]
            self.mix.backward(qs, ks, vs, gs, bs, cut(do), dq, dk, dv, dg, db)
            db, dg = torch.cat(db, dim=2).transpose(1, 2), torch.cat(dg, dim=2).transpose(1, 2)
            dzb, dzg = db * torch.sigmoid(zb) * torch.sigmoid(-zb), -dg * torch.sigmoid(zg)
            for z, name in ((dzb, "PB"), (dzg, "PG")):
                g[name].copy_(n.reshape(-1, C).t() @ z.reshape(-1, H))
                dn += z @ p[name].t()
        else:
            self.mix.backward(qs, ks, vs, [do], self.lam, dq, dk, dv)
        sums = lambda t: torch.cat(t, dim=2).view(B, HK, share, N, D).sum(2)   # noqa: E731
        dq, dk = sums(dq), sums(dk)
        dparts[2].copy_(torch.cat(dv, dim=2).transpose(1, 2).reshape(B, N, C))
        L.lasp_qk_bwd(self.qk, parts[0], parts[1], p["wq"], p["wk"], EPS, self.freq, None, 1.0, dq, dk, dparts[0], dparts[1], g["wq"], g["wk"], self.scratch)
        g["P"].copy_(n.reshape(-1, C).t() @ dproj.reshape(-1, WIDE))
        dn += dproj @ p["P"].t()
        L.lasp_addnorm_bwd(self.rows, p["x"], None, None, p["w1"], EPS, dn, p["dout"], g["x"], None, g["w1"], None, self.scratch)


@pytest.mark.parametrize("mixer", ["delta", "attention"])
def test_layer(gpu, mixer):
    lasp, sequence = gpu
    p, lam = parameters(), torch.tensor([0.9, 0.99, 0.95, 1.0])
    freq = lasp.rope_frequencies(32, scaling="bands", factor=4, trained=64, device="cpu")
    layer = Layer(lasp, sequence, p, freq, mixer, lam)
    out, grads = reference(p, freq, mixer, lam)
    off = lambda a, b: ((a.cpu().double() - b).norm() / b.norm()).item()   # noqa: E731
    layer.run()
    torch.cuda.synchronize()
    for name, got, want in [("out", layer.out, out)] + [(k, layer.grads[k], v) for k, v in grads.items()]:
        print(f"  {name}: {off(got, want):.2e}", flush=True)
        assert off(got, want) <= 1e-3, name
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.run()
    for k in range(3):
        fresh = parameters()
        layer.p["x"].copy_(fresh["x"] * (1.0 + 0.5 * k))
        layer.run()
        torch.cuda.synchronize()
        eager = [layer.out.clone()] + [layer.grads[n].clone() for n in grads]
        layer.out.zero_()
        for n in grads:
            layer.grads[n].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, [layer.out] + [layer.grads[n] for n in grads]):
            assert off(a, b.cpu().double()) <= 1e-5
