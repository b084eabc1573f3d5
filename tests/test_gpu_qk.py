"""Norm and rotation of queries and keys on the GPU against the 64-bit oracle."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def L():
    assert torch.cuda.is_available(), "needs a GPU"
    from paper_2404_02882_amd import lasp
    return lasp


@pytest.fixture(scope="module")
def O():
    from oracle import delta_oracle
    return delta_oracle


class Call:
    """Rows of a projection with a gap of 24 elements behind queries, keys and a part that is neither; outputs are filled with NaN first."""

    def __init__(self, L, dtype, B=2, N=9, H=3, Hk=2, D=64, norm="rms", rot=64, layout="half", weight=True, fused=True, pos=None, amplitude=1.0, eps=1e-5,
                 seed=0, scale=1.0):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g)   # noqa: E731
        t = DT[dtype]
        self.L, self.dtype, self.k = L, dtype, (norm, rot, layout, amplitude, eps)
        self.dims = (B, N, H, Hk, D)
        ld = (H + 2 * Hk) * D + 24 if fused else 0
        self.shape = L.make_qk_shape(B, N, H, Hk, D, t, norm, rot, layout, ld)
        self.wide = torch.full((B, N, ld), 7.0, dtype=t).cuda() if fused else None

        def rows(heads, first):
            x = (scale * r(B, N, heads * D) * (0.2 + torch.rand(B, N, 1, generator=g))).to(t).cuda()
            if not fused:
                return x
            part = self.wide[..., first:first + heads * D]
            part.copy_(x)
            return part
        self.xq, self.xk = rows(H, 0), rows(Hk, H * D) if Hk else None
        w = lambda: (1 + 0.3 * r(D)).cuda() if weight else None   # noqa: E731
        self.wq, self.wk = w(), w() if Hk else None
        self.freq = L.rope_frequencies(rot) if rot else None
        self.pos = None if pos is None else torch.as_tensor(pos, dtype=torch.int32).expand(B, N).contiguous().cuda()
        nan = lambda *s, dt=t: torch.full(s, float("nan"), dtype=dt, device="cuda")   # noqa: E731
        self.q, self.key = nan(B, H, N, D), nan(B, Hk, N, D) if Hk else None
        self.dq, self.dk = r(B, H, N, D).to(t).cuda(), r(B, Hk, N, D).to(t).cuda() if Hk else None
        self.dwide = torch.full((B, N, ld), 7.0, dtype=t).cuda() if fused else None
        self.dxq = self.dwide[..., :H * D] if fused else nan(B, N, H * D)
        self.dxk = (self.dwide[..., H * D:(H + Hk) * D] if fused else nan(B, N, Hk * D)) if Hk else None
        self.dwq, self.dwk = nan(D, dt=torch.float32), nan(D, dt=torch.float32) if Hk else None
        self.scratch = torch.full((L.qk_scratch_bytes(self.shape),), 0xff, dtype=torch.uint8, device="cuda")

    def forward(self, stream=None):
        norm, rot, layout, amplitude, eps = self.k
        self.L.lasp_qk_fwd(self.shape, self.xq, self.xk, self.wq, self.wk, eps, self.freq, self.pos, amplitude, self.q, self.key, stream=stream)

    def backward(self, stream=None, sums=True):
        norm, rot, layout, amplitude, eps = self.k
        self.L.lasp_qk_bwd(self.shape, self.xq, self.xk, self.wq, self.wk, eps, self.freq, self.pos, amplitude, self.dq, self.dk, self.dxq, self.dxk,
                           self.dwq if sums else None, self.dwk if sums else None, self.scratch if sums else None, stream=stream)

    def run(self):
        self.forward()
        self.backward()
        torch.cuda.synchronize()
        return self

    def check(self, O):
        B, N, H, Hk, D = self.dims
        norm, rot, layout, amplitude, eps = self.k
        n = lambda t: None if t is None else t.double().cpu().numpy()   # noqa: E731
        pos = n(self.pos) if self.pos is not None else np.broadcast_to(np.arange(N), (B, N))
        f = n(self.freq) if rot else None
        for name, x, h, w, y, dy, dx, dw in (("q", self.xq, H, self.wq, self.q, self.dq, self.dxq, self.dwq),
                                             ("k", self.xk, Hk, self.wk, self.key, self.dk, self.dxk, self.dwk)):
            if h == 0:
                continue
            want = O.qk_fwd(n(x), h, n(w), norm, eps, pos, f, rot, layout, amplitude)
            wdx, wdw = O.qk_bwd(n(x), h, n(w), norm, eps, pos, f, rot, layout, amplitude, n(dy))
            # a sum over few rows is small against its terms: held to their size, dy times a normed feature times sqrt(rows)
            size = {"none": np.abs(n(x)).mean(), "rms": 1.0, "l2": D ** -0.5}[norm] * amplitude * (B * N * h) ** 0.5
            for what, got, ref, part, kind, floor in (("", y, want, O.QK, self.dtype, 0.0), ("dx", dx, wdx, O.QK, self.dtype, 0.0),
                                                      ("dw", dw, wdw, O.QK_SUM, "f32", size)):
                off = O.off(n(got), ref, kind, part, floor)
                print(f"  {what}{name}: {off:.3f}", flush=True)
                assert off <= 1.0, (what, name, off)
        if self.dwide is not None:
            assert (self.wide[..., (H + Hk) * D:] == 7).all() and (self.dwide[..., (H + Hk) * D:] == 7).all()


CASES = [dict(), dict(layout="interleaved"), dict(norm="l2"), dict(norm="none"), dict(norm="none", weight=False), dict(weight=False, fused=False), dict(rot=0),
         dict(rot=0, norm="none"), dict(rot=16), dict(rot=32, layout="interleaved"), dict(rot=48), dict(Hk=0), dict(Hk=0, fused=False, norm="l2"), dict(N=1), dict(N=1, B=1, H=1, Hk=1),
         dict(D=8, rot=0), dict(D=16, rot=16), dict(D=24, rot=16, layout="interleaved"), dict(D=80, rot=80), dict(D=96, rot=32), dict(D=128, rot=128),
         dict(D=256, rot=256), dict(D=256, rot=240, layout="interleaved"), dict(H=16, Hk=16, N=77, D=128, rot=128), dict(H=1, Hk=5, N=40), dict(amplitude=1.3), dict(amplitude=-0.5, rot=32),
         dict(N=700, B=3, H=2, Hk=1), dict(N=3000, B=1, H=5, Hk=1, D=96, rot=96)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", CASES, ids=lambda kw: "-".join(f"{k}{v}" for k, v in kw.items()) or "plain")
def test_forward_and_backward(L, O, dtype, kw):
    Call(L, dtype, seed=len(str(kw)), **kw).run().check(O)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_positions(L, O, layout):
    """Angles of positions up to the last int32 keep the float's precision, and positions may be negative."""
    pos = [0, 1, 4095, 131071, 2 ** 24 + 1, 2 ** 31 - 1, -1, -(2 ** 31), 10 ** 9 + 7]
    Call(L, "f32", layout=layout, pos=pos).run().check(O)
    Call(L, "bf16", layout=layout, pos=pos, D=128, rot=128).run().check(O)


def test_positions_by_sequence(L, O):
    """One token each, at its own place: as the token of a sequence that stands there."""
    c = Call(L, "f32", B=5, N=1, pos=[[3], [0], [17], [4], [9]]).run()
    c.check(O)
    whole = Call(L, "f32", B=1, N=18, fused=False)
    whole.xq[0, [3, 0, 17, 4, 9]] = c.xq[:, 0]
    whole.wq = c.wq
    whole.forward()
    assert torch.equal(whole.q[0][:, [3, 0, 17, 4, 9]].transpose(0, 1), c.q[:, :, 0])


@pytest.mark.parametrize("norm", ["rms", "l2"])
def test_rows_of_zeros_and_extremes(L, O, norm):
    for dtype, scale in (("f32", 0.0), ("bf16", 0.0), ("f32", 1e-15), ("f32", 1e15), ("bf16", 1e15)):
        c = Call(L, dtype, norm=norm, scale=scale, eps=1e-6)
        c.run()
        if scale > 1:      # (dx and dw of rows this large: eps is nothing)
            c.check(O)
        else:
            c.check(O)
            assert torch.isfinite(c.dxq.float()).all()


def test_a_broken_row_stays_alone(L):
    for bad in (float("nan"), float("inf")):
        a, b = Call(L, "bf16").run(), Call(L, "bf16")
        b.xq[1, 4, 64 + 5] = bad
        b.run()
        same = torch.ones_like(a.q[..., 0], dtype=torch.bool)
        same[1, 1, 4] = False
        assert torch.equal(a.q[same], b.q[same]) and torch.isnan(b.q[1, 1, 4]).any() and torch.equal(a.key, b.key)
        assert torch.equal(a.dxk, b.dxk) and torch.equal(a.dwk, b.dwk) and torch.equal(a.dxq[0], b.dxq[0])


def test_gradient_without_sums_and_without_inputs(L):
    a, b = Call(L, "bf16").run(), Call(L, "bf16")
    b.forward()
    b.backward(sums=False)
    torch.cuda.synchronize()
    assert torch.equal(a.dxq, b.dxq) and torch.equal(a.dxk, b.dxk)
    a, b = Call(L, "bf16", norm="none").run(), Call(L, "bf16", norm="none")
    b.xq = b.xk = None      # neither a norm nor a weight's gradient: they are not read
    b.backward(sums=False)
    torch.cuda.synchronize()
    assert torch.equal(a.dxq, b.dxq) and torch.equal(a.dxk, b.dxk)


def test_repeats_streams_and_graphs(L):
    args = dict(dtype="bf16", B=2, N=2500, H=8, Hk=2, D=128, rot=128)
    a, b = Call(L, **args).run(), Call(L, **args)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    b.forward(stream=side)
    b.backward(stream=side)
    side.synchronize()
    got = lambda c: (c.q, c.key, c.dxq, c.dxk, c.dwq, c.dwk)   # noqa: E731
    for s, t in zip(got(a), got(b)):
        assert torch.equal(s, t)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.forward()
        b.backward()
    for k in range(4):
        for c in (a, b):
            c.xq.copy_(torch.randn(c.xq.shape, generator=torch.Generator().manual_seed(k)).to(c.xq.dtype))
            c.pos is None or c.pos.add_(1)
        a.run()
        for t in got(b):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for s, t in zip(got(a), got(b)):
            assert torch.equal(s, t), k
        torch.zeros(1000, device="cuda").sum()


def test_offsets_past_32_bits(L, O):
    """More than 2^31 elements in the rows; the last token against a call of it alone."""
    B, N, H, D = 1, 70000, 250, 128
    shape, one = L.make_qk_shape(B, N, H, 0, D, torch.bfloat16, rot=128), L.make_qk_shape(1, 1, H, 0, D, torch.bfloat16, rot=128)
    x = torch.ones(B, N, H * D, dtype=torch.bfloat16, device="cuda")
    x[0, -1] = torch.randn(H * D, device="cuda").to(torch.bfloat16)
    assert x.numel() > 2 ** 31
    f, q = L.rope_frequencies(128), torch.empty(B, H, N, D, dtype=torch.bfloat16, device="cuda")
    L.lasp_qk_fwd(shape, x, None, None, None, 1e-5, f, None, 1.0, q, None)
    few = torch.empty(1, H, 1, D, dtype=torch.bfloat16, device="cuda")
    L.lasp_qk_fwd(one, x[:, -1:].contiguous(), None, None, None, 1e-5, f, torch.tensor([[N - 1]], dtype=torch.int32, device="cuda"), 1.0, few, None)
    assert torch.equal(q[:, :, -1:], few)
    dx = torch.empty_like(x)
    L.lasp_qk_bwd(shape, x, None, None, None, 1e-5, f, None, 1.0, q, None, dx, None, None, None, None)
    dfew = torch.empty(1, 1, H * D, dtype=torch.bfloat16, device="cuda")
    L.lasp_qk_bwd(one, x[:, -1:].contiguous(), None, None, None, 1e-5, f, torch.tensor([[N - 1]], dtype=torch.int32, device="cuda"), 1.0, few, None, dfew,
                  None, None, None, None)
    assert torch.equal(dx[:, -1:], dfew)
