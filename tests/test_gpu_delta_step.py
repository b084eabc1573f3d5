"""The gated delta rule token by token, as generation calls it without a cache: every kernel of it by value, with lengths, gates of 0, without gates or states, in
place, around the length up to which it is taken, and captured."""
import pytest
import torch

from test_gpu_delta import Call, check, make, want

pytestmark = pytest.mark.gpu

MOST = {"bf16": 4, "f32": 8}      # tokens of a call that goes token by token
STATES = {"narrow": dict(B=4, H=2), "wide": dict(B=8, H=64)}      # blocks of 16 columns; of 32 (512 blocks or more)


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
@pytest.mark.parametrize("states", list(STATES))
@pytest.mark.parametrize("D,Dv", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("more", [0, 1])
def test_up_to_the_last_length_and_past_it(L, O, dtype, states, D, Dv, more):
    """Scratch is not looked at where a call goes token by token, and asked for one token later."""
    x = make(dtype, N=MOST[dtype] + more, D=D, Dv=Dv, Hk=2, seed=1, **STATES[states])
    call = Call(L, x, dtype, train=False)
    scratch, call.scratch = call.scratch, None
    if more:
        with pytest.raises(L.LaspError) as e:
            call.forward()
        assert e.value.status == 5
        call.scratch = scratch
    check(O, call.run(), want(O, x, train=False), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("states", list(STATES))
@pytest.mark.parametrize("kw", [dict(D=64, Dv=128), dict(D=128, Dv=64), dict(D=128, Hk=1)], ids=str)
def test_lengths(L, O, dtype, states, kw):
    """NaN behind a sequence's end is not looked at, out is 0 there, and an empty sequence hands its state on."""
    N, sizes = MOST[dtype], STATES[states]
    lens = ([0, N, 1, N + 5, -1, N - 1, 2, 0] * 2)[:sizes["B"]]
    x = make(dtype, N=N, seed=2, **sizes, **kw)
    w = want(O, x, lens, train=False)
    for b, n in enumerate(lens):
        for name in ("q", "k", "v", "beta", "log_g"):
            x[name][b, :, max(0, n):] = float("nan")
    call = Call(L, x, dtype, lens, train=False).run()
    check(O, call, w, dtype)
    for b, n in enumerate(lens):
        assert (call.out[b, :, max(0, n):] == 0).all()
        if n <= 0:
            assert torch.equal(call.kv_out[b], call.x["kv_in"][b])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("states", list(STATES))
@pytest.mark.parametrize("down", [-float("inf"), -2000.0])
def test_gates_of_zero(L, O, dtype, states, down):
    """At the first token, at one behind another, and at the last; the state in front of it leaves no trace."""
    N = MOST[dtype]
    x = make(dtype, N=N, D=128, Dv=64, seed=3, **STATES[states])
    for b, places in enumerate(([0], [1, 2], [N - 1], [])):
        x["log_g"][b, :, places] = down
    call = Call(L, x, dtype, train=False).run()
    check(O, call, want(O, x, train=False), dtype)
    x["kv_in"][:3] = 5.0
    again = Call(L, x, dtype, train=False).run()
    assert torch.equal(again.kv_out[:3], call.kv_out[:3]) and torch.equal(again.out[0], call.out[0])
    assert not torch.equal(again.out[2], call.out[2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", [dict(gate=False), dict(states=False), dict(gate=False, states=False), dict(beta=0.0), dict(beta=2.0)], ids=str)
@pytest.mark.parametrize("N", [1, 4])
def test_without_gates_or_states(L, O, dtype, kw, N):
    x = make(dtype, B=3, H=4, Hk=2, N=N, D=64, Dv=128, seed=4, **kw)
    check(O, Call(L, x, dtype, train=False).run(), want(O, x, train=False), dtype)


@pytest.mark.parametrize("dtype,N", [("bf16", 1), ("bf16", 4), ("f32", 1), ("f32", 8)])
@pytest.mark.parametrize("states", list(STATES))
def test_in_place(L, dtype, N, states):
    x = make(dtype, N=N, D=128, seed=5, **STATES[states])
    a, b = Call(L, x, dtype, train=False).run(), Call(L, x, dtype, train=False)
    b.kv_out = b.x["kv_in"]
    b.run()
    assert torch.equal(a.out, b.out) and torch.equal(a.kv_out, b.kv_out)


@pytest.mark.parametrize("dtype,N", [("bf16", 1), ("bf16", 4), ("f32", 3), ("bf16", 100), ("bf16", 2000)])
@pytest.mark.parametrize("place", ["apart", "in place"])
def test_captured(L, dtype, N, place):
    """Forward calls without a cache, replayed on changing inputs: each replay is what the same call gives outside of the graph."""
    xs = [make(dtype, B=2, H=4, Hk=2, N=N, D=128, seed=s) for s in (6, 7)]
    call = Call(L, xs[0], dtype, train=False)
    if place == "in place":
        call.kv_out = call.x["kv_in"]
    call.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.forward()
    for k in range(4):
        eager = Call(L, xs[k % 2], dtype, train=False).run()
        call.kv_out.fill_(float("nan"))
        call.out.fill_(float("nan"))
        for name, t in xs[k % 2].items():
            call.x[name].copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(call.out, eager.out) and torch.equal(call.kv_out, eager.kv_out), k
        torch.zeros(1000, device="cuda").sum()
