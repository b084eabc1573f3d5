"""The gated delta rule with values that are no numbers, on the GPU: what lies behind a sequence's end is 0 whatever its state holds, and
an infinite or NaN value reaches exactly what the definition makes of it: everything else is, bit for bit, as without it. N, P and the weights of a tile hold zeros where
a token does not reach another, and 0 x infinity is NaN, so that rows of the same tile are where this can go wrong."""
import pytest
import torch

from test_gpu_delta import Call, make

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")
SIZES = [dict(D=64), dict(D=128), dict(D=64, Dv=128, H=4, Hk=2), dict(D=128, Dv=64)]
MANY = dict(B=9, H=32, D=64)      # (a wave then has all key features of its columns)
WIDE = [dict(MANY, D=128), dict(MANY, D=128, Dv=64), dict(MANY, Dv=128)]


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


def same(name, got, want, where=""):
    assert torch.equal(got, want), (name, where, int((got != want).sum()), got.numel())


def broken(name, got, where=""):
    assert not torch.isfinite(got.float()).any(), (name, where)


def spoil(x, what, j, bad):
    """One value of one token of the second sequence; the states that it enters and its column."""
    share = x["v"].shape[1] // x["q"].shape[1]
    states, head, c = ([1], 1, 11) if what in ("v", "dout") else (list(range(share)), 0, 5)
    x[what][1, head, j, c] = bad
    return states, c


CASES = [pytest.mark.parametrize("dtype", ["f32", "bf16"]), pytest.mark.parametrize("kw", SIZES + [dict(D=128, N=700), MANY] + WIDE, ids=ids),
         pytest.mark.parametrize("j,bad", [(0, NAN), (45, INF), (77, NAN), (90, -INF)])]   # (tokens of the same tile in front of and behind it)


def cases(fn):
    for mark in CASES:
        fn = mark(fn)
    return fn


@cases
@pytest.mark.parametrize("what", ["v", "q", "k"])
def test_a_broken_token(L, dtype, kw, j, bad, what):
    x = make(dtype, seed=2, **{"B": 2, "N": 100, **kw})
    B, H, N, Dv = x["v"].shape
    good = Call(L, x, dtype, train=False).run().got()
    states, c = spoil(x, what, j, bad)
    for train in (False, True):
        got = Call(L, x, dtype, train=train).run().got()
        for b in range(B):
            for h in range(H):
                if b != 1 or h not in states:
                    for name in ("out", "kv_out"):
                        same(name, got[name][b, h], good[name][b, h], (b, h))
        (out, was), (state, state_was) = ((got[n][1, states], good[n][1, states]) for n in ("out", "kv_out"))
        same("out", out[:, :j], was[:, :j], "in front")
        if what == "v":        # its column of the state, from it on
            other = [e for e in range(Dv) if e != c]
            same("out", out[..., other], was[..., other], "other columns")
            same("kv_out", state[..., other], state_was[..., other], "other columns")
            broken("out", out[:, j:, c])
            broken("kv_out", state[..., c])
        elif what == "q":      # its own output
            same("out", out[:, j + 1:], was[:, j + 1:], "behind")
            same("kv_out", state, state_was)
            broken("out", out[:, j])
        else:                  # the state from it on
            broken("out", out[:, j:])
            broken("kv_out", state)


@cases
@pytest.mark.parametrize("what", ["v", "q", "k", "dout"])
def test_gradients_around_a_broken_token(L, dtype, kw, j, bad, what):
    x = make(dtype, seed=2, **{"B": 2, "N": 100, **kw})
    B, H, N, Dv = x["v"].shape
    share = H // x["q"].shape[1]
    good = Call(L, x, dtype).run().got()
    states, c = spoil(x, what, j, bad)
    got = Call(L, x, dtype).run().got()
    grads = [n for n in got if n not in ("out", "kv_out")]
    heads = {n: sorted({s // share for s in states}) if n in ("dq", "dk") else states for n in grads}
    for n in grads:      # other sequences and heads
        for b in range(B):
            for h in range(got[n].shape[1]):
                if b != 1 or h not in heads[n]:
                    same(n, got[n][b, h], good[n][b, h], (b, h))
    of, was = ({n: t[n][1, heads[n]] for n in grads} for t in (got, good))
    other = [e for e in range(Dv) if e != c]

    def unchanged(names, a, b):
        for n in names:
            same(n, of[n][:, a:b], was[n][:, a:b], (a, b))

    def spoilt(names, a, b):
        for n in names:
            broken(n, of[n][:, a:b], (a, b))

    if what == "v":        # the state's column from it on; gradients of v and of the state do not depend on it, nor does its own gate's (which stands in front of it)
        unchanged(["dv", "dkv_in"], 0, None)
        unchanged(["dq", "dk", "dbeta"], 0, j)
        unchanged(["dlog_g"], 0, j + 1)
        spoilt(["dq", "dk", "dbeta"], j, N)
        spoilt(["dlog_g"], j + 1, N)
    elif what == "q":      # the state's gradient up to it
        unchanged(["dq"], 0, N)
        unchanged(["dv", "dk", "dbeta", "dlog_g"], j + 1, N)
        spoilt(["dv", "dk", "dbeta", "dlog_g"], 0, j + 1)
        spoilt(["dkv_in"], 0, None)
    elif what == "k":      # both
        unchanged(["dq"], 0, j)
        unchanged(["dv"], j + 1, N)
        spoilt(["dq"], j, N)
        spoilt(["dv"], 0, j + 1)
        spoilt(["dk", "dbeta", "dlog_g", "dkv_in"], 0, None)
    else:                  # a column of the state's gradient up to it
        unchanged(["dq"], 0, j)
        unchanged(["dq", "dv", "dk", "dbeta", "dlog_g"], j + 1, N)
        for n in ("dv", "dkv_in"):
            same(n, of[n][..., other], was[n][..., other], "other columns")
        broken("dv", of["dv"][:, :j + 1, c])
        broken("dkv_in", of["dkv_in"][..., c])
        spoilt(["dq"], j, j + 1)
        spoilt(["dk", "dbeta", "dlog_g"], 0, j + 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", SIZES + [dict(D=128, N=700), MANY], ids=ids)
@pytest.mark.parametrize("bad", [NAN, -INF])
@pytest.mark.parametrize("what", ["kv_in", "dkv_out"])
def test_a_broken_state(L, dtype, kw, bad, what):
    """One element of a head's state, or of its gradient: its column, whatever the tokens are."""
    x = make(dtype, seed=4, **{"B": 2, "N": 100, **kw})
    Dv, share = x["v"].shape[-1], x["v"].shape[1] // x["q"].shape[1]
    good = Call(L, x, dtype).run().got()
    x[what][1, 1, 7, 11] = bad
    got = Call(L, x, dtype).run().got()
    other = [e for e in range(Dv) if e != 11]
    forward, columns = what == "kv_in", ("out", "kv_out") if what == "kv_in" else ("dv", "dkv_in")
    for n, t in got.items():
        head = 1 // share if n in ("dq", "dk") else 1
        for b in range(t.shape[0]):
            for h in range(t.shape[1]):
                if (b, h) != (1, head):
                    same(n, t[b, h], good[n][b, h], (b, h))
        if n in columns:
            same(n, t[1, 1][..., other], good[n][1, 1][..., other], "other columns")
            broken(n, t[1, 1][..., 11])
        elif n in (("dv", "dkv_in") if forward else ("out", "kv_out", "dq")):
            same(n, t[1, head], good[n][1, head])
        else:
            broken(n, t[1, head])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", ["q", "k", "v"])
def test_tokens_in_front_do_not_depend_on_the_length_of_the_call(L, dtype, what):
    """A few tokens go one by one, more in tiles: in front of the broken one both give what they gave."""
    for N in (3, 30):
        x = make(dtype, N=N, D=128, seed=3)
        good = Call(L, x, dtype, train=False).run().got()
        x[what][0, 1, 2, 4] = NAN
        got = Call(L, x, dtype, train=False).run().got()
        same("out", got["out"][0, 1, :2], good["out"][0, 1, :2], N)
        same("out", got["out"][0, 0], good["out"][0, 0], N)
        assert torch.isnan(got["out"][0, 1, 2].float()).any()


@pytest.mark.parametrize("what", ["q", "k", "dout"])
@pytest.mark.parametrize("kw", [dict(D=64), dict(D=128)], ids=ids)
def test_floats_that_round_to_infinity(L, what, kw):
    """Finite, but infinite as bfloat16: as an infinity."""
    if what != "dout":
        test_a_broken_token(L, "f32", kw, 45, 3.4e38, what)
    test_gradients_around_a_broken_token(L, "f32", kw, 45, 3.4e38, what)
