"""Norm and rotation of queries and keys at the sizes of training: workgroups that take groups of four tokens, several of them one after the other, with a remainder and
with sequences that end inside a group, and calls beyond the last-level cache, all by value; positions that change under a captured call."""
import numpy as np
import pytest
import torch

from test_gpu_qk import Call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    assert torch.cuda.is_available(), "needs a GPU"
    from paper_2404_02882_amd import lasp
    return lasp


@pytest.fixture(scope="module")
def O():
    from oracle import delta_oracle
    return delta_oracle


# groups of four tokens from 4096 tokens on; backward 2048 workgroups at most, so that some take a second group from 8193 tokens on
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", [dict(B=3, N=3001, H=2, Hk=1), dict(B=3, N=3001, H=2, Hk=1, layout="interleaved", rot=48), dict(B=1, N=4096, H=3, Hk=0),
                                dict(B=1, N=9001, H=1, Hk=1, D=256, rot=256, fused=False), dict(B=7, N=1301, H=1, Hk=2, D=24, rot=16, norm="l2"),
                                dict(B=9001, N=1, H=2, Hk=1, D=128, rot=128), dict(B=2, N=8503, H=2, Hk=2, norm="none", rot=32)],
                         ids=lambda kw: "-".join(f"{k}{v}" for k, v in kw.items()))
def test_groups_of_tokens(L, O, dtype, kw):
    Call(L, dtype, seed=len(str(kw)), **kw).run().check(O)


def test_many_positions(L, O):
    """Positions given for every token, another order in each sequence, in groups of four."""
    pos = torch.stack([torch.randperm(3001, generator=torch.Generator().manual_seed(s)) + 1000 * s for s in range(3)])
    Call(L, "bf16", B=3, N=3001, H=2, Hk=1, pos=pos).run().check(O)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_beyond_the_cache(L, O, dtype):
    """More than 256 MB in and out, forward and backward, with keys, weights and their gradients: by parts of the sequence against the oracle, the sums over all
    tokens from the oracle's sums of the parts."""
    N = 21001 if dtype == "bf16" else 10501
    c = Call(L, dtype, B=1, N=N, H=16, Hk=10, D=128, rot=128, layout="interleaved")
    assert 2 * (c.xq.numel() + c.xk.numel()) * c.q.element_size() > 256 << 20
    c.run()
    norm, rot, layout, amplitude, eps = c.k
    n = lambda t: t.double().cpu().numpy()   # noqa: E731
    f, D = n(c.freq), 128
    for name, x, h, w, y, dy, dx, dw in (("q", c.xq, 16, c.wq, c.q, c.dq, c.dxq, c.dwq), ("k", c.xk, 10, c.wk, c.key, c.dk, c.dxk, c.dwk)):
        sums = 0.0
        for a in range(0, N, 1500):
            b = min(N, a + 1500)
            pos = np.arange(a, b)[None]
            want = O.qk_fwd(n(x[:, a:b]), h, n(w), norm, eps, pos, f, rot, layout, amplitude)
            wdx, part = O.qk_bwd(n(x[:, a:b]), h, n(w), norm, eps, pos, f, rot, layout, amplitude, n(dy[:, :, a:b]))
            sums = sums + part
            for what, got, ref in (("", y[:, :, a:b], want), ("dx", dx[:, a:b], wdx)):
                off = O.off(n(got), ref, dtype, O.QK, 0.0)
                assert off <= 1.0, (what, name, a, off)
        off = O.off(n(dw), sums, "f32", O.QK_SUM, (N * h) ** 0.5)
        print(f"  dw{name}: {off:.3f}", flush=True)
        assert off <= 1.0, (name, off)
    assert (c.dwide[..., 26 * D:] == 7).all()


def test_positions_that_change_under_a_graph(L, O):
    """A captured call reads its positions and rows when it is replayed."""
    call = Call(L, "bf16", B=5, N=7, H=4, Hk=2, D=128, rot=128, pos=torch.arange(7))
    call.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.forward()
        call.backward()
    outputs = lambda: (call.q, call.key, call.dxq, call.dxk, call.dwq, call.dwk)   # noqa: E731
    for k in range(4):
        call.pos.add_(torch.arange(35, device="cuda", dtype=torch.int32).view(5, 7) * 100 + 1)
        call.xq.copy_(torch.randn(call.xq.shape, generator=torch.Generator().manual_seed(k)).to(call.xq.dtype))
        for t in outputs():
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        call.check(O)
        replayed = [t.clone() for t in outputs()]
        call.run()
        for a, b in zip(replayed, outputs()):
            assert torch.equal(a, b), k
        torch.zeros(1000, device="cuda").sum()
