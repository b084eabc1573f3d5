"""The gated delta rule on the GPU against the 64-bit oracle: every type, head layout and dimension, lengths around tiles and segments, gates
of 0, empty sequences, states handed on, and the ways a caller's program uses it."""
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


def make(dtype, B=1, H=2, N=64, D=64, Dv=0, Hk=0, gate=True, states=True, seed=0, beta=None):
    """Tensors on the CPU, already of the type that the call takes; keys of length 1 that have a part in common."""
    g = torch.Generator().manual_seed(seed)
    Dv, Hk = Dv or D, Hk or H
    r = lambda *s: torch.randn(*s, generator=g)   # noqa: E731
    unit = lambda t: t / t.norm(dim=-1, keepdim=True)   # noqa: E731
    x = {"q": (unit(r(B, Hk, N, D) + 0.3) * 0.3).to(DT[dtype]), "k": unit(r(B, Hk, N, D) + 0.3).to(DT[dtype]), "v": r(B, H, N, Dv).to(DT[dtype]),
         "beta": torch.rand(B, H, N, generator=g) if beta is None else torch.full((B, H, N), beta)}
    x["log_g"] = -0.2 * torch.rand(B, H, N, generator=g) ** 3 if gate else None
    x["kv_in"] = 0.5 * r(B, H, D, Dv) if states else None
    x["dout"] = r(B, H, N, Dv).to(DT[dtype])
    x["dkv_out"] = 0.5 * r(B, H, D, Dv) if states else None
    return x


def dev(t):
    return None if t is None else t.cuda()


def np64(t):
    return None if t is None else t.double().cpu().numpy()


class Call:
    """A call's buffers; outputs are filled with NaN first."""

    def __init__(self, L, x, dtype, lens=None, train=True):
        B, H, N, Dv = x["v"].shape
        self.L, self.train, d = L, train, x["q"].shape[-1]
        self.shape = L.make_delta_shape(B, H, N, d, DT[dtype], Dv, x["q"].shape[1])
        self.x = {k: dev(t) for k, t in x.items()}
        self.lens = None if lens is None else torch.tensor(lens, dtype=torch.int32).cuda()
        nan = lambda t, *s: torch.full(s or t.shape, float("nan"), dtype=t.dtype, device="cuda")   # noqa: E731
        f = torch.zeros((), dtype=torch.float32)
        room = lambda n: torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")   # noqa: E731
        self.out, self.kv_out = nan(x["v"]), nan(f, B, H, d, Dv)
        self.cache = room(L.delta_cache_bytes(self.shape)) if train else None
        self.scratch = room(max(L.delta_scratch_bytes(self.shape), L.delta_bwd_scratch_bytes(self.shape) if train else 0))
        self.g = {"dq": nan(x["q"]), "dk": nan(x["k"]), "dv": nan(x["v"]), "dbeta": nan(x["beta"]), "dkv_in": nan(self.kv_out)}
        if x["log_g"] is not None:
            self.g["dlog_g"] = nan(x["log_g"])

    def forward(self, stream=None):
        x = self.x
        self.L.lasp_delta_fwd(self.shape, x["q"], x["k"], x["v"], x["log_g"], x["beta"], x["kv_in"], self.lens, self.out, self.kv_out, self.cache,
                              self.scratch, stream=stream)

    def backward(self, stream=None):
        x, g = self.x, self.g
        self.L.lasp_delta_bwd(self.shape, x["q"], x["k"], x["v"], x["log_g"], x["beta"], self.lens, x["dout"], x["dkv_out"], self.cache, g["dq"],
                              g["dk"], g["dv"], g.get("dlog_g"), g["dbeta"], g["dkv_in"], self.scratch, stream=stream)

    def run(self):
        self.forward()
        if self.train:
            self.backward()
        torch.cuda.synchronize()
        return self

    def got(self):
        return {"out": self.out, "kv_out": self.kv_out, **(self.g if self.train else {})}


def want(O, x, lens=None, train=True):
    n = {k: np64(t) for k, t in x.items()}
    args = [n[k] for k in ("q", "k", "v", "log_g", "beta")]
    lens = None if lens is None else np.array(lens)
    out, kv_out, _ = O.delta_fwd(*args, n["kv_in"], lens)
    w = {"out": out, "kv_out": kv_out}
    if train:
        w.update(O.delta_bwd(*args, n["dout"], n["kv_in"], lens, n["dkv_out"]))
    return w


def check(O, call, w, dtype):
    """A gradient of a gate or of beta is a sum of products of either sign, and in a short sequence one of few: it is held to the size of its terms, which that
    of the state's gradient and of the state make (`floor`)."""
    for name, t in call.got().items():
        kind = dtype if name in ("out", "dq", "dk", "dv") else "f32"
        floor = 0.05 if name in ("dlog_g", "dbeta") else 0.0
        off = O.off(t.double().cpu().numpy(), w[name], kind, floor=floor)
        print(f"  {name}: {off:.3f}", flush=True)
        assert off <= 1.0, (name, off)


CASES = [dict(N=n) for n in (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 96, 97, 200)] + [
    dict(N=70, D=128), dict(N=70, D=64, Dv=128), dict(N=70, D=128, Dv=64), dict(N=40, H=6, Hk=2), dict(N=100, H=4, Hk=1, D=128), dict(N=50, B=3, H=3),
    dict(N=130, gate=False), dict(N=130, states=False), dict(N=66, gate=False, states=False, D=128), dict(N=33, beta=0.0), dict(N=90, beta=1.0),
    dict(N=90, beta=2.0, gate=False), dict(N=700, H=1), dict(N=1100, H=2, D=128, Dv=64)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", CASES, ids=lambda kw: "-".join(f"{k}{v}" for k, v in kw.items()))
def test_forward_and_backward(L, O, dtype, kw):
    x = make(dtype, seed=len(str(kw)), **kw)
    check(O, Call(L, x, dtype).run(), want(O, x), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,Dv", [(64, 64), (64, 128), (128, 64), (128, 128)])
def test_many_states(L, O, dtype, D, Dv):
    """As many states as fill the card (a wave then has all key features of its columns), uncut and in segments; fewer in segments."""
    x = make(dtype, B=9, H=32, N=67, D=D, Dv=Dv, Hk=16, seed=3)
    lens = [67, 0, 1, 64, 65, 33, 32, 31, 66]
    check(O, Call(L, x, dtype, lens).run(), want(O, x, lens), dtype)
    for H in (52 if Dv == 64 else 28, 3):
        x = make(dtype, H=H, N=550, D=D, Dv=Dv, seed=4)
        check(O, Call(L, x, dtype).run(), want(O, x), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", [dict(N=1), dict(N=3, D=128), dict(N=16, Dv=128), dict(N=7, B=5, H=4, Hk=2, D=128), dict(N=9, gate=False, states=False),
                                dict(N=2, B=40, H=8, D=128), dict(N=17), dict(N=600, D=128)], ids=str)
def test_forward_without_a_cache(L, O, dtype, kw):
    x = make(dtype, seed=5, **kw)
    check(O, Call(L, x, dtype, train=False).run(), want(O, x, train=False), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,lens", [(100, [0, 100, 64, 37]), (100, [1, 33, 32, 99]), (10, [0, 10, 3, 200]), (70, [-5, 71, 65, 2]), (700, [0, 650, 300, 32])])
def test_lengths(L, O, dtype, N, lens):
    """What the inputs hold past a sequence's end is not looked at, and everything is 0 there; an empty sequence hands its state on."""
    x = make(dtype, B=4, N=N, seed=1)
    w = want(O, x, lens)
    for b, n in enumerate(lens):
        for name in ("q", "k", "v", "beta", "log_g", "dout"):
            x[name][b, :, max(0, n):] = float("nan")
    for train in (True, False):
        call = Call(L, x, dtype, lens, train).run()
        check(O, call, w, dtype)
        for name, t in call.got().items():
            if name not in ("kv_out", "dkv_in"):
                for b, n in enumerate(lens):
                    assert (t[b, :, max(0, n):] == 0).all(), name
    for b, n in enumerate(lens):
        if n <= 0:
            assert torch.equal(call.kv_out[b], call.x["kv_in"][b])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("train", [True, False])
def test_documents_packed_into_one_sequence(L, O, dtype, train):
    """A gate of 0 (-infinity, and so far down that its power is 0) starts the state anew: at the first token, next to one another, at a tile's ends."""
    N = 130 if train else 14
    x = make(dtype, H=3, N=N, seed=2)
    for h, places in enumerate(([0, 1, 2, 40], [31, 32, 63, 64, 129], [5, 6, 13])):
        x["log_g"][0, h, [p for p in places if p < N]] = -float("inf") if h else -2000.0
    call = Call(L, x, dtype, train=train).run()
    check(O, call, want(O, x, train=train), dtype)
    if train:
        assert (call.g["dlog_g"][x["log_g"].cuda() < -1000] == 0).all()
        assert (call.g["dkv_in"][0, 0] == 0).all()
    # the documents apart give the same
    cut = 40 if train else 2
    second = {k: (t if t is None or k in ("kv_in", "dkv_out") else t[:, :1, cut:].contiguous()) for k, t in x.items()}
    second["kv_in"], second["dkv_out"] = None, x["dkv_out"][:, :1].contiguous()
    alone = Call(L, second, dtype, train=train).run()
    assert O.off(alone.out.double().cpu().numpy(), call.out[:, :1, cut:].double().cpu().numpy(), dtype) <= 2.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strong_decay(L, O, dtype):
    """Gates whose product over a tile is far below the smallest float, and ones that differ by 30 orders of magnitude."""
    x = make(dtype, N=150, seed=3)
    x["log_g"] = -torch.rand(1, 2, 150, generator=torch.Generator().manual_seed(1)) * torch.tensor([8.0, 70.0])[None, :, None]
    check(O, Call(L, x, dtype).run(), want(O, x), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_key_for_all_tokens(L, O, dtype):
    """The triangular system at its worst: all products of keys are 1."""
    x = make(dtype, N=128, gate=False, seed=4, beta=1.0)
    x["k"] = torch.zeros_like(x["k"])
    x["k"][..., 3] = 1.0
    call = Call(L, x, dtype).run()
    check(O, call, want(O, x), dtype)


def test_a_broken_head_stays_alone(L):
    for bad in (float("nan"), float("inf")):
        x = make("bf16", B=2, H=2, N=100, seed=6)
        good = Call(L, x, "bf16").run().got()
        x["v"][1, 0, 50] = bad
        broken = Call(L, x, "bf16").run().got()
        assert torch.isnan(broken["out"][1, 0, 64:]).any()
        for name, t in broken.items():
            for b, h in ((0, 0), (0, 1), (1, 1)):
                assert torch.equal(t[b, h], good[name][b, h]), name


def test_states_updated_in_place_and_runs_repeat(L):
    for dtype, N in (("bf16", 1), ("bf16", 100), ("f32", 13), ("bf16", 1500)):
        x = make(dtype, N=N, seed=7)
        for train in (True, False):
            a, b = Call(L, x, dtype, train=train).run(), Call(L, x, dtype, train=train)
            b.kv_out, b.g["dkv_in"] = b.x["kv_in"], b.x["dkv_out"]
            b.run()
            for (name, s), t in zip(a.got().items(), b.got().values()):
                assert torch.equal(s, t), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N", [(3, 120), (2, 2000), (5, 5)])
def test_sequence(L, O, dtype, T, N):
    from paper_2404_02882_amd import sequence
    x = make(dtype, H=4, Hk=2, N=N, Dv=128, seed=8)
    seq = sequence.DeltaSequence(1, 4, N, 64, DT[dtype], T, Dv=128, key_heads=2)
    cut = lambda t: [p.contiguous().cuda() for p in t.chunk(T, dim=2)]   # noqa: E731
    t = {k: cut(x[k]) for k in ("q", "k", "v", "log_g", "beta", "dout")}
    new = lambda name: [torch.full_like(p, float("nan")) for p in t[name]]   # noqa: E731
    out, g = new("v"), {n: new(n) for n in ("q", "k", "v", "log_g", "beta")}
    args = [t[k] for k in ("q", "k", "v", "log_g", "beta")]
    kv = seq.forward(*args, out, kv_in=x["kv_in"].cuda())
    dkv = seq.backward(*args, t["dout"], *[g[n] for n in ("q", "k", "v", "log_g", "beta")], dkv_out=x["dkv_out"].cuda())

    class Whole:
        @staticmethod
        def got():
            join = lambda p: torch.cat(p, dim=2)   # noqa: E731
            return {"out": join(out), "kv_out": kv, "dkv_in": dkv, **{"d" + n: join(p) for n, p in g.items()}}
    check(O, Whole, want(O, x), dtype)


def test_tokens_one_by_one_are_the_sequence(L, O):
    """Serving: a prompt, then single tokens, the state in place."""
    x = make("bf16", B=2, H=4, Hk=2, N=80, D=128, seed=9, states=False)
    state = torch.zeros(2, 4, 128, 128, device="cuda")
    outs = []
    for a, b in [(0, 60)] + [(s, s + 1) for s in range(60, 80)]:
        part = {k: (t if t is None else t[:, :, a:b].contiguous()) for k, t in x.items()}
        part["kv_in"] = part["dkv_out"] = None
        call = Call(L, part, "bf16", train=False)
        call.x["kv_in"] = call.kv_out = state
        call.run()
        outs.append(call.out)
    w = want(O, x, train=False)
    assert O.off(torch.cat(outs, dim=2).double().cpu().numpy(), w["out"], "bf16") <= 1.0
    assert O.off(state.cpu().numpy(), w["kv_out"], "f32") <= 1.0


def test_on_another_stream(L):
    x = make("bf16", N=300, seed=10)
    a, b = Call(L, x, "bf16").run(), Call(L, x, "bf16")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    b.forward(stream=side)
    b.backward(stream=side)
    with torch.cuda.stream(side):       # as the current stream
        b.forward()
        b.backward()
    side.synchronize()
    for (name, s), t in zip(a.got().items(), b.got().values()):
        assert torch.equal(s, t), name


def test_two_calls_at_once(L):
    """On two streams, each with its own scratch and cache."""
    xs = [make("bf16", B=2, N=2000, seed=s) for s in (11, 12)]
    alone = [Call(L, x, "bf16").run().got() for x in xs]
    calls, streams = [Call(L, x, "bf16") for x in xs], [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, s in zip(calls, streams):
            c.forward(stream=s)
            c.backward(stream=s)
    torch.cuda.synchronize()
    for c, a in zip(calls, alone):
        for name, t in c.got().items():
            assert torch.equal(t, a[name]), name


@pytest.mark.parametrize("N", [1, 100, 2000])
def test_captured(L, N):
    x, y = make("bf16", N=N, seed=13), make("bf16", N=N, seed=14)
    eager = Call(L, x, "bf16").run()
    call = Call(L, x, "bf16").run()
    serve = Call(L, x, "bf16", train=False).run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.forward()
        call.backward()
        serve.forward()
    for k in range(4):
        for name, t in (x if k % 2 else y).items():
            for c in (eager, call, serve):
                c.x[name].copy_(t)
        eager.run()
        for c in (call, serve):
            for t in c.got().values():
                t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for (name, s), t in zip(eager.got().items(), call.got().values()):
            assert torch.equal(s, t), (k, name)
        assert torch.equal(serve.kv_out, eager.kv_out) or N <= 16
        torch.zeros(1000, device="cuda").sum()


def test_offsets_past_32_bits(L, O):
    """More than 2^31 elements in q, k and v; the last head against the oracle."""
    B, H, N, D = 2, 560, 16384, 128
    shape = L.make_delta_shape(B, H, N, D, torch.bfloat16)
    last = make("bf16", H=1, N=N, D=D, seed=15, states=False)
    t = {n: torch.zeros(B, H, N, D, dtype=torch.bfloat16, device="cuda") for n in ("q", "k", "v")}
    for n in t:
        t[n][-1, -1] = last[n][0, 0].cuda()
    gates = {n: torch.zeros(B, H, N, device="cuda") for n in ("log_g", "beta")}
    for n in gates:
        gates[n][-1, -1] = last[n][0, 0].cuda()
    assert t["q"].numel() > 2 ** 31
    out, kv_out = torch.full_like(t["v"], float("nan")), torch.full((B, H, D, D), float("nan"), device="cuda")
    scratch = torch.empty(L.delta_scratch_bytes(shape), dtype=torch.uint8, device="cuda")
    L.lasp_delta_fwd(shape, t["q"], t["k"], t["v"], gates["log_g"], gates["beta"], None, None, out, kv_out, None, scratch)
    torch.cuda.synchronize()
    few = 300     # (the oracle on the first tokens, and a call of the head alone for the others)
    head = Call(L, last, "bf16", train=False).run()
    w = want(O, {k: (v if v is None or k in ("kv_in", "dkv_out") else v[:, :, :few]) for k, v in last.items()}, train=False)
    assert O.off(out[-1, -1, :few].double().cpu().numpy(), w["out"][0, 0], "bf16") <= 1.0
    assert O.off(out[-1, -1].double().cpu().numpy(), head.out[0, 0].double().cpu().numpy(), "bf16") <= 2.0
    assert O.off(kv_out[-1, -1].cpu().numpy(), head.kv_out[0, 0].cpu().numpy(), "f32") <= 2.0
    assert (out[0, 0] == 0).all() and (kv_out[0] == 0).all() and (out[-1, -2] == 0).all()
