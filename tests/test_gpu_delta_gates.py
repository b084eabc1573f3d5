"""Slopes of the gated delta rule's gates where neighbours differ by orders of magnitude, and float results held to what sums in float come to."""
import numpy as np
import pytest
import torch

from test_gpu_delta import Call, make, np64, want

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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", [dict(D=64), dict(D=128, Dv=64), dict(D=64, Dv=128, H=4, Hk=2), dict(D=128, N=64)], ids=str)
@pytest.mark.parametrize("down", [-20.0, -45.0])
def test_slopes_of_gates_that_let_little_pass(L, O, dtype, kw, down):
    """dlog_g_i = <dS_{i-1}, S_{i-1}>, the gradient of the state in front of token i times that state. Both come with a relative error of at most
    DELTA in the 2-norm, and the product with both: 2 DELTA of the product of their norms, whatever the slopes of the tokens around are."""
    x = make(dtype, seed=4, **{"N": 150, **kw})
    N = x["v"].shape[2]
    places = [p for p in (0, 9, 31, 40, 63, 64, 75, 96, 127, 149) if p < N]
    x["log_g"][..., places] = down
    call = Call(L, x, dtype).run()
    got = np64(call.g["dlog_g"])
    n = {k: np64(t) for k, t in x.items()}
    w = want(O, x)["dlog_g"]
    before = O.delta_fwd(*[n[k] for k in ("q", "k", "v", "log_g", "beta")], n["kv_in"])[2]
    for p in places:
        rest = {k: (t if k in ("kv_in", "dkv_out") else t[:, :, p:]) for k, t in n.items()}
        rest["kv_in"] = before[p]
        dS = O.delta_bwd(*[rest[k] for k in ("q", "k", "v", "log_g", "beta")], rest["dout"], rest["kv_in"], None, rest["dkv_out"])["dkv_in"]
        size = np.sqrt((dS ** 2).sum((-1, -2)) * (before[p] ** 2).sum((-1, -2)))
        off = np.abs(got[:, :, p] - w[:, :, p]) / (2 * O.DELTA * size)
        print(f"  token {p}: {off.max():.3f} of the bound, slope {np.abs(w[:, :, p]).max():.2e}", flush=True)
        assert off.max() <= 1.0, (p, off.max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("train,N", [(True, 130), (False, 70), (False, 3)])
def test_gates_below_the_least_are_none(L, dtype, train, N):
    """A gate below 2^-126 counts as 0: all results are those of -infinity, bit for bit."""
    results = []
    for down in (-np.log(2.0) * 126.5, -100.0, -float("inf")):
        x = make(dtype, N=N, seed=5)
        x["log_g"][..., [p for p in (0, 2, 31, 32, 50, 64) if p < N]] = down
        results.append(Call(L, x, dtype, train=train).run().got())
    for got in results[:2]:
        for name, t in got.items():
            assert torch.equal(t, results[2][name]), name
    if train:
        assert (results[0]["dlog_g"][..., [0, 2, 31, 32, 50, 64]] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", [dict(N=200, D=64), dict(N=200, D=128), dict(N=200, D=64, Dv=128, H=4, Hk=2), dict(N=1100, D=128, Dv=64), dict(N=1100, D=64),
                                dict(N=67, D=64, B=9, H=32, Hk=16), dict(N=67, D=128, B=9, H=32)], ids=lambda kw: "-".join(f"{k}{v}" for k, v in kw.items()))
def test_float_results_are_as_good_as_float_sums(L, O, dtype, kw):
    """States and the slopes of gates and betas, of either data type, in the 2-norm over all of them. (A slope is a sum of terms of either sign: held to 0.05 a token at least.)"""
    x = make(dtype, seed=6, **kw)
    call, w = Call(L, x, dtype).run(), want(O, x)
    for name, floor in (("kv_out", 0.0), ("dkv_in", 0.0), ("dlog_g", 0.05), ("dbeta", 0.05)):
        off = O.off_in_norm(np64(call.got()[name]), w[name], floor)
        print(f"  {name}: {off:.3f}", flush=True)
        assert off <= 1.0, (name, off)
