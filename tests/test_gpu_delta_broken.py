"""The gated delta rule with values that are no numbers, on the GPU: what lies behind a sequence's end is 0 whatever its state holds."""
import pytest
import torch

from test_gpu_delta import Call, make

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")
SIZES = [dict(D=64), dict(D=128), dict(D=64, Dv=128, H=4, Hk=2), dict(D=128, Dv=64)]
MANY = dict(B=9, H=32, D=64)      # (a wave then has all key features of its columns)


@pytest.fixture(scope="module")
def L():
    assert torch.cuda.is_available(), "needs a GPU"
    from paper_2404_02882_amd import lasp
    return lasp


def ids(x):
    return "-".join(f"{k}{v}" for k, v in x.items()) if isinstance(x, dict) else None


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", SIZES + [dict(D=128, N=700), dict(MANY, N=50)], ids=ids)
@pytest.mark.parametrize("bad", [NAN, INF])
def test_zeros_behind_a_length(L, dtype, kw, bad):
    """A state, a gradient and a value that are no numbers: out and all gradients are 0 behind a sequence's end, inside its last tile as behind it."""
    N = kw.get("N", 100)
    x = make(dtype, seed=1, **{"B": 4, "N": N, **kw})
    lens = [N - 1, 33, 1, N // 2, 0, 31, N, 17, 2][:x["v"].shape[0]]
    x["kv_in"][:, 0, 3, 5] = bad
    x["dkv_out"][:, 0, 7, 2] = -bad
    x["v"][:, 0, 0, 9] = bad
    for train in (True, False):
        got = Call(L, x, dtype, lens, train).run().got()
        assert not torch.isfinite(got["out"][0, 0, 0]).all()
        for name, t in got.items():
            if name not in ("kv_out", "dkv_in"):
                for b, n in enumerate(lens):
                    assert (t[b, :, n:] == 0).all(), (name, b, n)
