"""The operators as a layer uses them: norm before the block, one projection, a mixer that carries a state, norm and gate
behind it, projection back, residual add; first with linear attention (LaspSequence), then with the gated recurrence. Forward and
backward in float against 64-bit autograd of the same formulas, then captured and replayed.

Tolerance: every value passes at most 12 operators between an input and an output, each with a relative error of at most about 2^-16
of its terms (sums of up to 256 products in float, LASP's stated 1e-4 at most): 1e-3 in the 2-norm leaves room for their growth
through norms with factors of order 1."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

B, H, N, D = 2, 2, 200, 64
C, EPS = H * D, 1e-5


@pytest.fixture(scope="module")
def gpu():
    assert torch.cuda.is_available(), "needs a GPU"
    from paper_2404_02882_amd import lasp, sequence
    return lasp, sequence


def parameters():
    g = torch.Generator().manual_seed(11)
    r = lambda *s: torch.randn(*s, generator=g)   # noqa: E731
    p = {"x": r(B, N, C), "dout": r(B, N, C), "w1": 1 + 0.1 * r(C), "w2": 1 + 0.1 * r(C), "w3": 1 + 0.1 * r(C), "w4": 1 + 0.1 * r(C),
         "s1": 0.5 + 0.1 * r(C), "s2": 0.5 + 0.1 * r(C), "P1": r(C, 4 * C) / C ** 0.5, "O1": r(C, C) / C ** 0.5,
         "P2": r(C, 3 * C) / C ** 0.5, "O2": r(C, C) / C ** 0.5}
    return p, torch.tensor([0.9, 0.99])


def norm(x, w):
    return w * x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt()


def reference(p, lam):
    """64 bits, by autograd."""
    p = {k: v.double().requires_grad_(k != "dout") for k, v in p.items()}
    lam = lam.double()
    q, k, v, u = (norm(p["x"], p["w1"]) @ p["P1"]).split(C, dim=-1)
    heads = lambda t: t.reshape(B, N, H, D).transpose(1, 2)   # noqa: E731
    q, k, v = heads(q) / D ** 0.5, heads(k), heads(v)
    i = torch.arange(N)
    M = torch.where(i[:, None] >= i[None, :], lam.view(H, 1, 1) ** (i[:, None] - i[None, :]).clamp(min=0), torch.zeros((), dtype=torch.float64))
    o = ((q @ k.transpose(-1, -2)) * M) @ v
    o = o * (o.square().mean(-1, keepdim=True) + EPS).rsqrt()
    y = p["w2"] * o.transpose(1, 2).reshape(B, N, C) * torch.nn.functional.silu(u)
    r = p["x"] + p["s1"] * (y @ p["O1"])
    c, z, u = (norm(r, p["w3"]) @ p["P2"]).split(C, dim=-1)
    a, h, hs = torch.sigmoid(z + 2.0), torch.zeros(B, C, dtype=torch.float64), []
    for s in range(N):
        h = a[:, s] * h + (1 - a[:, s]) * c[:, s]
        hs.append(h)
    y = norm(torch.stack(hs, 1), p["w4"]) * torch.sigmoid(u)
    out = r + p["s2"] * (y @ p["O2"])
    (out * p["dout"]).sum().backward()
    return out.detach(), {k: t.grad for k, t in p.items() if k != "dout"}


class Layer:
    def __init__(self, lasp, sequence, p, lam):
        self.L, self.p, self.lam = lasp, {k: v.cuda() for k, v in p.items()}, lam.cuda()
        f = torch.float32
        self.att = sequence.LaspSequence(B, H, N, D, 64, f)
        self.rec = sequence.RecurrenceSequence(B, N, C, f, coupled=True)
        self.rows = lasp.make_rows(B * N, C, f)
        self.gate1 = lasp.make_gate_shape(B, H, N, D, f, "silu", "head", 4 * C)
        self.gate2 = lasp.make_gate_shape(B, 1, N, C, f, "sigmoid", "head", 3 * C)
        need = max(lasp.addnorm_scratch_bytes(self.rows), lasp.gatenorm_scratch_bytes(self.gate1), lasp.gatenorm_scratch_bytes(self.gate2))
        self.scratch = torch.empty(need, dtype=torch.uint8, device="cuda")
        self.out = torch.empty(B, N, C, device="cuda")
        self.grads = {k: torch.empty_like(v) for k, v in self.p.items() if k != "dout"}

    def run(self):
        L, p, g = self.L, self.p, self.grads
        new = lambda *s: torch.empty(*s, device="cuda")   # noqa: E731
        tok = lambda: new(B, N, C)   # noqa: E731
        heads = lambda t: t.reshape(B, N, H, D).transpose(1, 2).contiguous()   # noqa: E731
        tokens = lambda t: t.transpose(1, 2).reshape(B, N, C)   # noqa: E731
        # forward
        n1, r, n3, y1, y2, end = tok(), tok(), tok(), tok(), tok(), tok()
        L.lasp_addnorm_fwd(self.rows, p["x"], None, None, p["w1"], EPS, None, n1)
        proj1 = n1 @ p["P1"]
        q, k, v = heads(proj1[..., :C]) / D ** 0.5, heads(proj1[..., C:2 * C]), heads(proj1[..., 2 * C:3 * C])
        o = torch.empty_like(q)
        self.att.forward([q], [k], [v], self.lam, [o])
        L.lasp_gatenorm_fwd(self.gate1, o, proj1[..., 3 * C:], p["w2"], EPS, y1)
        b1 = y1 @ p["O1"]
        L.lasp_addnorm_fwd(self.rows, p["x"], b1, p["s1"], p["w3"], EPS, r, n3)
        proj2 = n3 @ p["P2"]
        c, log_a = proj2[..., :C].contiguous(), torch.nn.functional.logsigmoid(proj2[..., C:2 * C] + 2.0)
        h = tok()
        self.rec.forward([c], [log_a], [h])
        L.lasp_gatenorm_fwd(self.gate2, h, proj2[..., 2 * C:], p["w4"], EPS, y2)
        b2 = y2 @ p["O2"]
        L.lasp_addnorm_fwd(self.rows, r, b2, p["s2"], None, EPS, self.out, end)     # (the norm of the next block)
        # backward: nothing behind the last norm, so its dy is 0
        flat = lambda t: t.reshape(-1, t.shape[-1])   # noqa: E731
        zero, dr, db2 = torch.zeros(B, N, C, device="cuda"), tok(), tok()
        L.lasp_addnorm_bwd(self.rows, self.out, b2, p["s2"], None, EPS, zero, p["dout"], dr, db2, None, g["s2"], self.scratch)
        g["O2"].copy_(flat(y2).T @ flat(db2))
        dproj2, dh = new(B, N, 3 * C), tok()
        L.lasp_gatenorm_bwd(self.gate2, h, proj2[..., 2 * C:], p["w4"], EPS, db2 @ p["O2"].T, dh, dproj2[..., 2 * C:], g["w4"], self.scratch)
        dc, dl = tok(), tok()
        self.rec.backward([c], [log_a], [h], [dh], [dc], [dl])
        dproj2[..., :C] = dc
        dproj2[..., C:2 * C] = dl * (1.0 - log_a.exp())
        g["P2"].copy_(flat(n3).T @ flat(dproj2))
        db1 = tok()
        L.lasp_addnorm_bwd(self.rows, r, b1, p["s1"], p["w3"], EPS, dproj2 @ p["P2"].T, dr, dr, db1, g["w3"], g["s1"], self.scratch)
        g["O1"].copy_(flat(y1).T @ flat(db1))
        dproj1, do = new(B, N, 4 * C), torch.empty_like(o)
        L.lasp_gatenorm_bwd(self.gate1, o, proj1[..., 3 * C:], p["w2"], EPS, db1 @ p["O1"].T, do, dproj1[..., 3 * C:], g["w2"], self.scratch)
        dq, dk, dv = (torch.empty_like(q) for _ in range(3))
        self.att.backward([q], [k], [v], [do], self.lam, [dq], [dk], [dv])
        for j, t in enumerate((dq / D ** 0.5, dk, dv)):
            dproj1[..., j * C:(j + 1) * C] = tokens(t)
        g["P1"].copy_(flat(n1).T @ flat(dproj1))
        L.lasp_addnorm_bwd(self.rows, p["x"], None, None, p["w1"], EPS, dproj1 @ p["P1"].T, dr, g["x"], None, g["w1"], None, self.scratch)


def near(got, ref, name):
    rel = float((got.double().cpu() - ref).norm() / ref.norm())
    print(f"  {name}: {rel:.2e}", flush=True)
    assert rel < 1e-3 and math.isfinite(rel), (name, rel)


def test_a_layer_and_its_gradients(gpu):
    p, lam = parameters()
    out, grads = reference(p, lam)
    layer = Layer(*gpu, p, lam)
    layer.run()
    torch.cuda.synchronize()
    near(layer.out, out, "out")
    for k, ref in grads.items():
        near(layer.grads[k], ref, k)


def test_the_layer_captured_and_replayed(gpu):
    p, lam = parameters()
    layer = Layer(*gpu, p, lam)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    want = [layer.out.clone()] + [t.clone() for t in layer.grads.values()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.run()
    for _ in range(3):
        for t in [layer.out] + list(layer.grads.values()):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, [layer.out] + list(layer.grads.values())):
            torch.testing.assert_close(a, b, rtol=1e-5, atol=1e-5)     # (the library's products may be cut in another order)
        layer.run()
        torch.cuda.synchronize()


@pytest.mark.parametrize("T", [1, 4])
def test_recurrence_over_sub_sequences(gpu, T):
    """RecurrenceSequence with the states handed on, the whole step also captured, against one call over the whole sequence."""
    lasp, sequence = gpu
    g = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")   # noqa: E731
    B_, N_, D_ = 3, 1200, 72
    x, la, do, h, dh = r(B_, N_, D_), -r(B_, N_, D_).abs(), r(B_, N_, D_), r(B_, D_), r(B_, D_)
    results = []
    for parts in (1, T):
        seq = sequence.RecurrenceSequence(B_, N_, D_, torch.float32, T=parts, coupled=True)
        cut = lambda t: [c.contiguous() for c in t.chunk(parts, dim=1)]   # noqa: E731
        xs, ls, ds = cut(x), cut(la), cut(do)
        out, dx, dl = ([torch.empty_like(t) for t in xs] for _ in range(3))
        fwd = dict(x=xs, log_a=ls, out=out, h_in=h)
        bwd = dict(x=xs, log_a=ls, out=out, dout=ds, dx=dx, dlog_a=dl, dh_out=dh)
        seq.forward(**fwd)
        seq.backward(**bwd)
        torch.cuda.synchronize()
        got = lambda: [torch.cat(t, dim=1) for t in (out, dx, dl)] + [seq.h[parts].clone(), seq.dh[0].clone()]   # noqa: E731
        eager = got()
        step = sequence.GraphedStep(seq, fwd, bwd)
        for _ in range(3):
            for t in out + dx + dl:
                t.fill_(float("nan"))
            step.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(eager, got()))
        results.append(eager)
    for a, b in zip(*results):   # sums in another order: roundings of 2^-24 of terms that add up to a few units
        torch.testing.assert_close(a, b, rtol=2e-5, atol=2e-5)
