"""GPU parity of the gated recurrence (lasp_rec_fwd / lasp_rec_bwd) against the 64-bit oracle, element by element within the
bounds that the oracle derives from the roundings. Outputs are pre-filled with NaN, and so is what lies past a sequence's
length in the inputs."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def L():
    assert torch.cuda.is_available(), "needs a GPU"
    from paper_2404_02882_amd import lasp
    return lasp


def make(dtype, B, N, D, seed, states=True, lens=None, packed=False, low=0.5):
    """x ~ N(0,1), log a of a sigmoid gate (a between about `low` and 1), rounded to the type; 64-bit copies."""
    rng = np.random.default_rng(seed)
    raw = {"x": rng.normal(size=(B, N, D)), "log_a": -np.log1p(np.exp(-(3.0 + 2.0 * rng.normal(size=(B, N, D))))),
           "dout": rng.normal(size=(B, N, D))}
    if packed:
        raw["log_a"][rng.random((B, N)) < 0.2] = -np.inf
    inp = {k: torch.tensor(v, dtype=torch.float32).to(DT[dtype]) for k, v in raw.items()}
    if states:
        inp["h_in"] = torch.tensor(rng.normal(size=(B, D)), dtype=torch.float32)
        inp["dh_out"] = torch.tensor(rng.normal(size=(B, D)), dtype=torch.float32)
    if lens is not None:
        inp["lens"] = torch.tensor(lens, dtype=torch.int32)
    return inp


def run(L, inp, dtype, coupled, fused=False, in_place=False, stream=None, backward=True):
    B, N, D = inp["x"].shape
    shape = L.make_rec_shape(B, N, D, DT[dtype], coupled, 2 * D if fused else 0)
    g = {k: v.cuda() for k, v in inp.items()}
    if "lens" in g:   # what lies past the lengths must not matter
        gone = torch.arange(N, device="cuda")[None, :] >= g["lens"].clamp(0, N)[:, None]
        for k in ("x", "log_a", "dout"):
            g[k] = torch.where(gone[..., None], torch.full_like(g[k], float("nan")), g[k])

    def pair(a, b):
        if not fused:
            return a.contiguous(), b.contiguous()
        both = torch.cat([a, b], dim=-1).contiguous()
        return both[..., :D], both[..., D:]

    nan = lambda *size, dt=torch.float32: torch.full(size, float("nan"), dtype=dt, device="cuda")   # noqa: E731
    x, la = pair(g["x"], g["log_a"])
    dx, dl = pair(nan(B, N, D, dt=DT[dtype]), nan(B, N, D, dt=DT[dtype]))
    out, scratch = nan(B, N, D, dt=DT[dtype]), torch.full((L.rec_scratch_bytes(shape),), 0x5a, dtype=torch.uint8, device="cuda")
    h_in, dh_out = g.get("h_in"), g.get("dh_out")
    h_out, dh_in = nan(B, D), nan(B, D)
    h_keep = h_in
    if in_place and h_in is not None:
        h_keep, h_out, dh_in = h_in.clone(), h_in, dh_out
    L.lasp_rec_fwd(shape, x, la, h_in, g.get("lens"), out, h_out, scratch, stream=stream)
    got = {"out": out, "h_out": h_out}
    if backward:
        saved = out
        if "lens" in g:
            saved = torch.where(gone[..., None], torch.full_like(out, float("nan")), out)
        scratch.fill_(0x5a)
        L.lasp_rec_bwd(shape, x if coupled else None, la, saved, h_keep, g.get("lens"), g["dout"], dh_out, dx, dl, dh_in, scratch, stream=stream)
        got.update(dx=dx, dlog_a=dl, dh_in=dh_in)
    if stream is not None:
        stream.synchronize()
    return {k: v.detach().cpu() for k, v in got.items()}


def check(got, inp, dtype, coupled, label):
    d = {k: v.double().numpy() if v.dtype != torch.int32 else v.numpy() for k, v in inp.items()}
    x, la, do = d["x"], d["log_a"], d["dout"]
    lens, h_in, dh_out = d.get("lens"), d.get("h_in"), d.get("dh_out")
    ref = dict(zip(("out", "h_out"), bo.rec_fwd(x, la, h_in, lens, coupled)))
    ref.update(zip(("dx", "dlog_a", "dh_in"), bo.rec_bwd(x, la, do, h_in, lens, dh_out, coupled)))
    bounds = bo.rec_bounds(dtype, x, la, do, h_in, lens, dh_out, coupled)
    for k, t in got.items():
        err, room = np.abs(t.double().numpy() - ref[k]), bounds[k] + 1e-37
        worst = np.unravel_index(np.argmax(np.where(np.isfinite(err), err / room, np.inf)), err.shape)
        print(f"  {label} {k}: {err[worst] / room[worst]:.3f} of the bound", flush=True)
        assert np.isfinite(err).all() and (err <= room).all(), (label, k, worst, err[worst], room[worst])


CASES = [  # B, N, D, lens, packed, fused
    (1, 1, 8, None, False, False),
    (64, 1, 64, None, False, False),
    (2, 2, 64, None, False, True),
    (3, 5, 40, [5, 0, 3], False, False),
    (2, 7, 1000, None, True, False),
    (1, 17, 520, None, False, True),
    (4, 33, 136, [33, 1, 40, -2], False, True),
    (2, 63, 24, None, True, False),
    (1, 64, 512, None, False, False),
    (1, 65, 512, None, False, False),
    (3, 129, 64, [64, 65, 129], False, False),
    (2, 300, 72, None, True, True),
    (1, 700, 256, [511], False, False),
    (5, 257, 8, [257, 128, 0, 200, 3], True, False),
    (2, 1500, 16, None, False, False),
    (1, 4100, 8, None, True, False),
    (1, 2111, 1040, None, False, False),
    (17, 600, 64, None, False, False),
    (9, 3000, 8, [3000, 0, 1, 256, 257, 2999, 512, 1000, 40], True, False),     # sequences of one column block end in different tiles
    (4, 1500, 72, [1500, 300, 0, 700], False, True),
    (3, 700, 64, [1, 0, 256], False, False),                                    # and none of them in the last
    (3, 5000, 8, [700, 4600, 0], False, False),
    (1, 8200, 600, None, False, False),        # rows that are no whole lines: blocks of 16 columns, backward in tiles of 8 waves
    (1, 16400, 520, None, True, False),        # forward too
    (2, 1300, 1000, [900, 1300], True, False), # and in tiles of 4
    (2, 16500, 8, [16500, 9000], False, False),
    (1, 16384, 64, None, False, True),
    (1, 400, 4104, None, False, False),        # blocks of 32
    (1, 400, 4096, None, False, True),
    (2, 512, 72, [257, 512], True, False),     # one tile of 8 waves, and one token more
    (2, 513, 64, [513, 100], False, False),
    (33, 300, 1024, None, False, False),       # too many columns for it
]


@pytest.mark.parametrize("coupled", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,N,D,lens,packed,fused", CASES)
def test_against_the_definition(L, B, N, D, lens, packed, fused, dtype, coupled):
    inp = make(dtype, B, N, D, seed=B * N + D, states=(N + D // 8) % 2 == 0, lens=lens, packed=packed)
    print(f"case rec {dtype} B={B} N={N} D={D} lens={lens} packed={packed} fused={fused} coupled={coupled}", flush=True)
    check(run(L, inp, dtype, coupled, fused=fused), inp, dtype, coupled, "rec")


@pytest.mark.parametrize("N,lens", [(1, None), (3, [1, 0, 3]), (200, None), (2500, None), (2500, [2500, 0, 900])])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_states_updated_in_place(L, dtype, N, lens):
    inp = make(dtype, 3, N, 128, seed=N, lens=lens)
    a, b = run(L, inp, dtype, False), run(L, inp, dtype, False, in_place=True)
    for k in a:
        assert torch.equal(a[k], b[k]), k


def test_only_a_length_of_zero(L):
    inp = make("bf16", 2, 300, 64, seed=9, lens=[0, 0])
    got = run(L, inp, "bf16", True)
    assert torch.equal(got["h_out"], inp["h_in"]) and torch.equal(got["dh_in"], inp["dh_out"])
    assert not got["out"].any() and not got["dx"].any() and not got["dlog_a"].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_outputs_that_are_not_wanted(L, dtype):
    inp = make(dtype, 2, 700, 64, seed=10)
    ref = run(L, inp, dtype, False)
    shape = L.make_rec_shape(2, 700, 64, DT[dtype])
    g = {k: v.cuda() for k, v in inp.items()}
    out, dx, dl = (torch.empty_like(g["x"]) for _ in range(3))
    scratch = torch.empty(L.rec_scratch_bytes(shape), dtype=torch.uint8, device="cuda")
    L.lasp_rec_fwd(shape, g["x"], g["log_a"], g["h_in"], None, out, None, scratch)
    L.lasp_rec_bwd(shape, None, g["log_a"], out, g["h_in"], None, g["dout"], g["dh_out"], dx, dl, None, scratch)
    for k, t in (("out", out), ("dx", dx), ("dlog_a", dl)):
        assert torch.equal(ref[k], t.cpu()), k


def test_memory_of_a_million_tokens_in_float(L):
    """a = 1 - 1e-6: 32-bit floats step by 6e-8 there, 6 % of 1 - a. Over 20000 tokens that would be 1e-4 of the state; roundings of
    the state alone are a random walk of about sqrt(20000) 2^-25 = 4e-6."""
    N = 20000
    rng = np.random.default_rng(3)
    x = torch.tensor(rng.normal(loc=1.0, size=(1, N, 8)), dtype=torch.float32)
    la = torch.full((1, N, 8), -1e-6, dtype=torch.float32)
    shape = L.make_rec_shape(1, N, 8, torch.float32)
    out, h_out = torch.empty(1, N, 8, device="cuda"), torch.empty(1, 8, device="cuda")
    scratch = torch.empty(L.rec_scratch_bytes(shape), dtype=torch.uint8, device="cuda")
    L.lasp_rec_fwd(shape, x.cuda(), la.cuda(), None, None, out, h_out, scratch)
    weights = np.exp(float(la[0, 0, 0].double()) * np.arange(N - 1, -1, -1))
    ref = (weights[:, None] * x[0].double().numpy()).sum(0)
    err = np.abs(h_out[0].cpu().double().numpy() / ref - 1).max()
    print(f"relative error {err:.2e}", flush=True)
    assert err < 3e-5


@pytest.mark.parametrize("B,N,D", [(2, 50, 64), (1, 3000, 128)])
def test_gradients_against_differences(L, B, N, D):
    """Float data, along one random direction of (x, log_a, h_in): the loss is nearly linear over a step of 2^-7, whose third
    derivative leaves about 2^-14 of the slope; the sums in 64 bits carry the outputs' 2^-20."""
    inp = make("f32", B, N, D, seed=77)
    got = run(L, inp, "f32", True)
    rng = np.random.default_rng(1)
    way = {k: torch.tensor(rng.normal(size=inp[k].shape), dtype=torch.float32) for k in ("x", "log_a", "h_in")}
    way["log_a"] = way["log_a"] * inp["log_a"].abs()      # (log a stays below 0)
    loss = lambda r: float((r["out"].double() * inp["dout"].double()).sum() + (r["h_out"].double() * inp["dh_out"].double()).sum())   # noqa: E731
    step = 2.0 ** -7
    sides = [loss(run(L, {**inp, **{k: inp[k] + s * step * way[k] for k in way}}, "f32", True, backward=False)) for s in (1, -1)]
    slope = (sides[0] - sides[1]) / (2 * step)
    want = sum(float((got[g].double() * way[k].double()).sum()) for g, k in (("dx", "x"), ("dlog_a", "log_a"), ("dh_in", "h_in")))
    size = sum(float((got[g].double() * way[k].double()).norm()) for g, k in (("dx", "x"), ("dlog_a", "log_a"), ("dh_in", "h_in")))
    print(f"slope {slope:.6f} gradient {want:.6f} size {size:.3f}", flush=True)
    assert abs(slope - want) <= 2.0 ** -10 * size


@pytest.mark.parametrize("dtype,B,N,D", [("bf16", 2, 3000, 256), ("f32", 1, 900, 1024), ("bf16", 1, 9000, 32)])
def test_runs_are_bit_reproducible(L, dtype, B, N, D):
    inp = make(dtype, B, N, D, seed=4)
    a = run(L, inp, dtype, True)
    for _ in range(3):
        b = run(L, inp, dtype, True)
        for k in a:
            assert torch.equal(a[k], b[k]), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_sequence_in_parts(L, dtype):
    """h_out of one part is h_in of the next, dh_in the dh_out of the part before: within the whole sequence's bounds."""
    N, cuts = 1300, [0, 1, 400, 1299, 1300]
    inp = make(dtype, 2, N, 64, seed=12)
    parts, h, fwd = [], inp["h_in"], []
    for a, b in zip(cuts, cuts[1:]):
        p = {k: inp[k][:, a:b].contiguous() for k in ("x", "log_a", "dout")}
        p["h_in"], p["dh_out"] = h, inp["dh_out"]
        fwd.append(run(L, p, dtype, True, backward=False))
        h = fwd[-1]["h_out"]
        parts.append(p)
    got, dh = {}, inp["dh_out"]
    pieces = []
    for p in reversed(parts):
        p["dh_out"] = dh
        r = run(L, p, dtype, True)
        dh = r["dh_in"]
        pieces.insert(0, r)
    for k in ("out", "dx", "dlog_a"):
        got[k] = torch.cat([r[k] for r in pieces], dim=1)
    got["h_out"], got["dh_in"] = pieces[-1]["h_out"], pieces[0]["dh_in"]
    check(got, inp, dtype, True, "parts")


def test_another_stream(L):
    inp = make("bf16", 2, 2000, 512, seed=21)
    a = run(L, inp, "bf16", True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = run(L, inp, "bf16", True)
    for k in a:
        assert torch.equal(a[k], b[k]), k
    c = run_on(L, inp, s)
    for k in c:
        assert torch.equal(a[k], c[k]), k


def run_on(L, inp, s):
    """The forward call with `stream=`, everything it reads ready before."""
    B, N, D = inp["x"].shape
    shape = L.make_rec_shape(B, N, D, torch.bfloat16, True)
    g = {k: v.cuda() for k, v in inp.items()}
    out, h_out = torch.empty_like(g["x"]), torch.empty_like(g["h_in"])
    scratch = torch.empty(L.rec_scratch_bytes(shape), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    L.lasp_rec_fwd(shape, g["x"], g["log_a"], g["h_in"], None, out, h_out, scratch, stream=s)
    s.synchronize()
    return {"out": out.cpu(), "h_out": h_out.cpu()}


def test_captured_and_replayed(L):
    """Both passes of two sequences of other lengths in one graph, with a workspace that they share, replayed with eager work between."""
    sets = []
    for N, dtype in ((3000, "bf16"), (40, "bf16")):
        inp = make(dtype, 2, N, 256, seed=N)
        shape = L.make_rec_shape(2, N, 256, DT[dtype], True)
        g = {k: v.cuda() for k, v in inp.items()}
        o = {k: torch.empty_like(g["x"]) for k in ("out", "dx", "dl")}
        o.update(h=torch.empty_like(g["h_in"]), dh=torch.empty_like(g["h_in"]))
        sets.append((shape, g, o))
    scratch = torch.empty(max(L.rec_scratch_bytes(s[0]) for s in sets), dtype=torch.uint8, device="cuda")

    def both():
        for shape, g, o in sets:
            L.lasp_rec_fwd(shape, g["x"], g["log_a"], g["h_in"], None, o["out"], o["h"], scratch)
            L.lasp_rec_bwd(shape, g["x"], g["log_a"], o["out"], g["h_in"], None, g["dout"], g["dh_out"], o["dx"], o["dl"], o["dh"], scratch)

    both()
    torch.cuda.synchronize()
    want = [{k: v.clone() for k, v in o.items()} for _, _, o in sets]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(4):
        for _, _, o in sets:
            for t in o.values():
                t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for w, (_, _, o) in zip(want, sets):
            for k in w:
                assert torch.equal(w[k], o[k]), k
        both()
        torch.cuda.synchronize()


@pytest.mark.parametrize("N", [5, 60, 1500])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gates_at_the_ends(L, dtype, N):
    """Gates that are open (log a = 0: sums), shut (-inf: the inputs themselves), nearly shut, and above 1."""
    inp = make(dtype, 2, N, 64, seed=31)
    la = inp["log_a"]
    la[:, :, :16] = 0.0
    la[:, :, 16:32] = -float("inf")
    la[:, :, 32:40] = -60.0
    la[:, :, 40:48] = torch.tensor(0.004).to(la.dtype)      # 1.004^1500 = 400
    got = run(L, inp, dtype, False)
    check(got, inp, dtype, False, "ends")
    assert torch.equal(got["out"][:, :, 16:32], inp["x"][:, :, 16:32]) and not got["dlog_a"][:, :, 16:32].any()
    check(run(L, inp, dtype, True), inp, dtype, True, "ends, coupled")


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_broken_stays_in_its_channel(L, dtype, bad):
    """A NaN or infinity in x spoils its channel of its sequence from its token on, and nothing else, in any direction."""
    N, at = 1300, 700
    inp = make(dtype, 2, N, 64, seed=32)
    clean = run(L, inp, dtype, False)
    inp["x"] = inp["x"].clone()
    inp["x"][1, at, 5] = bad
    got = run(L, inp, dtype, False)
    spoilt = torch.zeros(2, N, 64, dtype=torch.bool)
    spoilt[1, at:, 5] = True
    assert torch.equal(got["out"][~spoilt], clean["out"][~spoilt]) and not got["out"][spoilt].isfinite().any()
    after = torch.zeros(2, N, 64, dtype=torch.bool)
    after[1, at + 1:, 5] = True          # dlog_a takes the state in front of a token
    assert torch.equal(got["dx"], clean["dx"]) and torch.equal(got["dlog_a"][~after], clean["dlog_a"][~after])


def test_two_calls_at_once(L):
    """Calls on two streams, each with a workspace of its own."""
    sets = []
    for seed, (B, N, D) in enumerate(((1, 20000, 512), (4, 3000, 1000))):
        inp = {k: v.cuda() for k, v in make("bf16", B, N, D, seed=seed).items()}
        shape = L.make_rec_shape(B, N, D, torch.bfloat16, True)
        new = lambda: [torch.empty_like(inp["x"]) for _ in range(3)] + [torch.empty_like(inp["h_in"]) for _ in range(2)]   # noqa: E731
        sets.append((shape, inp, new(), new(), torch.empty(L.rec_scratch_bytes(shape), dtype=torch.uint8, device="cuda"), torch.cuda.Stream()))

    def both_passes(shape, i, o, scratch, stream):
        L.lasp_rec_fwd(shape, i["x"], i["log_a"], i["h_in"], None, o[0], o[3], scratch, stream=stream)
        L.lasp_rec_bwd(shape, i["x"], i["log_a"], o[0], i["h_in"], None, i["dout"], i["dh_out"], o[1], o[2], o[4], scratch, stream=stream)

    for shape, inp, want, _, scratch, _ in sets:
        both_passes(shape, inp, want, scratch, None)
    torch.cuda.synchronize()
    for _ in range(5):
        for shape, inp, _, got, scratch, stream in sets:
            both_passes(shape, inp, got, scratch, stream)
    torch.cuda.synchronize()
    for _, _, want, got, _, _ in sets:
        assert all(torch.equal(a, b) for a, b in zip(want, got))
