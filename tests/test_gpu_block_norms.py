"""GPU parity of the norms before and behind a mixer (lasp_addnorm_*, lasp_gatenorm_*) against the 64-bit oracle, element by
element within the bounds that the oracle derives from the roundings. Outputs are pre-filled with NaN."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


@pytest.fixture(scope="module")
def L():
    assert torch.cuda.is_available(), "needs a GPU"
    from paper_2404_02882_amd import lasp
    return lasp


def rounded(rng, dtype, *size, scale=1.0):
    t = torch.tensor(scale * rng.normal(size=size), dtype=torch.float32).to(DT[dtype])
    return t, t.double().numpy()


def nan(dtype, *size):
    return torch.full(size, float("nan"), dtype=dtype, device="cuda")


def held(got, ref, room, label):
    err = np.abs(got.detach().cpu().double().numpy() - ref)
    room = np.broadcast_to(room, err.shape) + 1e-37
    worst = np.unravel_index(np.argmax(np.where(np.isfinite(err), err / room, np.inf)), err.shape)
    print(f"  {label}: {err[worst] / room[worst]:.3f} of the bound", flush=True)
    assert np.isfinite(err).all() and (err <= room).all(), (label, worst, err[worst], room[worst])


# one row and many, widths of every way a row is spread over threads, on both sides of each
WIDTHS = [8, 16, 32, 64, 72, 128, 136, 256, 264, 512, 520, 1000, 1024, 1032, 2048, 2056, 4096, 4104, 8192, 8200, 16384]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", WIDTHS)
def test_addnorm_widths(L, dtype, C):
    rng = np.random.default_rng(C)
    rows = 5 if C > 2048 else 77
    (r, r64), (x, x64), (dy, dy64), (dro, dro64) = (rounded(rng, dtype, rows, C) for _ in range(4))
    scale, w = (torch.tensor(rng.normal(size=C), dtype=torch.float32) for _ in range(2))
    s64, w64 = scale.double().numpy(), w.double().numpy()
    print(f"case addnorm {dtype} rows={rows} C={C}", flush=True)
    shape = L.make_rows(rows, C, DT[dtype])
    r_out, y = nan(DT[dtype], rows, C), nan(DT[dtype], rows, C)
    L.lasp_addnorm_fwd(shape, r.cuda(), x.cuda(), scale.cuda(), w.cuda(), EPS, r_out, y)
    ref, room = bo.addnorm_fwd(r64, x64, s64, w64, EPS), bo.addnorm_fwd_bounds(dtype, r64, x64, s64, w64, EPS)
    held(r_out, ref[0], room["r_out"], "r_out")
    held(y, ref[1], room["y"], "y")
    saved = r_out.cpu().double().numpy()
    dr, dx, dw, ds = nan(DT[dtype], rows, C), nan(DT[dtype], rows, C), nan(torch.float32, C), nan(torch.float32, C)
    scratch = torch.full((L.addnorm_scratch_bytes(shape),), 0x5a, dtype=torch.uint8, device="cuda")
    L.lasp_addnorm_bwd(shape, r_out, x.cuda(), scale.cuda(), w.cuda(), EPS, dy.cuda(), dro.cuda(), dr, dx, dw, ds, scratch)
    ref = bo.addnorm_bwd(saved, x64, s64, w64, EPS, dy64, dro64)
    room = bo.addnorm_bwd_bounds(dtype, saved, x64, s64, w64, EPS, dy64, dro64)
    for name, t in (("dr", dr), ("dx", dx), ("dweight", dw), ("dscale", ds)):
        held(t, ref[name], room[name], name)


def addnorm_of(L, dtype, rows, C):
    rng = np.random.default_rng(rows)
    (r, r64), (dy, dy64) = (rounded(rng, dtype, rows, C) for _ in range(2))
    shape = L.make_rows(rows, C, DT[dtype])
    dr, dw = nan(DT[dtype], rows, C), nan(torch.float32, C)
    scratch = torch.empty(L.addnorm_scratch_bytes(shape), dtype=torch.uint8, device="cuda")
    L.lasp_addnorm_bwd(shape, r.cuda(), None, None, None, EPS, dy.cuda(), None, dr, None, dw, None, scratch)
    ref, room = bo.addnorm_bwd(r64, None, None, None, EPS, dy64, None), bo.addnorm_bwd_bounds(dtype, r64, None, None, None, EPS, dy64, None)
    held(dr, ref["dr"], room["dr"], "dr")
    held(dw, ref["dweight"], room["dweight"], "dweight")


@pytest.mark.parametrize("rows", [1, 2, 3, 64, 513, 4097])
def test_addnorm_rows(L, rows):
    addnorm_of(L, "bf16", rows, 264)
    addnorm_of(L, "f32", rows, 40)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_addnorm_options(L, dtype):
    """The norm alone; without weight, scale; sums updated in place; gradients that are not wanted; a row of zeros."""
    rng = np.random.default_rng(2)
    rows, C = 130, 520
    (r, r64), (x, x64), (dy, dy64), (dro, dro64) = (rounded(rng, dtype, rows, C) for _ in range(4))
    r[7] = 0
    r64[7] = 0
    x[7] = 0
    x64[7] = 0
    w = torch.tensor(rng.normal(size=C), dtype=torch.float32)
    shape = L.make_rows(rows, C, DT[dtype])
    y = nan(DT[dtype], rows, C)
    L.lasp_addnorm_fwd(shape, r.cuda(), None, None, w.cuda(), EPS, None, y)
    held(y, bo.addnorm_fwd(r64, None, None, w.double().numpy(), EPS)[1],
         bo.addnorm_fwd_bounds(dtype, r64, None, None, w.double().numpy(), EPS)["y"], "norm alone")
    assert not y[7].any()
    both, y2, apart = r.cuda(), nan(DT[dtype], rows, C), nan(DT[dtype], rows, C)
    L.lasp_addnorm_fwd(shape, both.clone(), x.cuda(), None, None, EPS, apart, y)
    L.lasp_addnorm_fwd(shape, both, x.cuda(), None, None, EPS, both, y2)
    assert torch.equal(both, apart) and torch.equal(y, y2)
    held(y, bo.addnorm_fwd(r64, x64, None, None, EPS)[1], bo.addnorm_fwd_bounds(dtype, r64, x64, None, None, EPS)["y"], "no scale, no weight")
    s64 = both.cpu().double().numpy()
    dr, grad = nan(DT[dtype], rows, C), dro.cuda()
    L.lasp_addnorm_bwd(shape, both, None, None, w.cuda(), EPS, dy.cuda(), dro.cuda(), dr, None, None, None, None)
    L.lasp_addnorm_bwd(shape, both, None, None, w.cuda(), EPS, dy.cuda(), grad, grad, None, None, None, None)
    assert torch.equal(dr, grad)
    held(dr, bo.addnorm_bwd(s64, None, None, w.double().numpy(), EPS, dy64, dro64)["dr"],
         bo.addnorm_bwd_bounds(dtype, s64, None, None, w.double().numpy(), EPS, dy64, dro64)["dr"], "dr alone")
    # the scale's gradient alone
    ds = nan(torch.float32, C)
    scratch = torch.empty(L.addnorm_scratch_bytes(shape), dtype=torch.uint8, device="cuda")
    L.lasp_addnorm_bwd(shape, both, x.cuda(), None, w.cuda(), EPS, dy.cuda(), None, dr, None, None, ds, scratch)
    held(ds, bo.addnorm_bwd(s64, x64, None, w.double().numpy(), EPS, dy64, None)["dscale"],
         bo.addnorm_bwd_bounds(dtype, s64, x64, None, w.double().numpy(), EPS, dy64, None)["dscale"], "dscale alone")


def test_addnorm_keeps_large_and_broken_rows_apart(L):
    """A row with an infinity or NaN spoils itself only."""
    rng = np.random.default_rng(3)
    rows, C = 33, 128
    (r, r64), (x, x64) = (rounded(rng, "bf16", rows, C) for _ in range(2))
    clean = nan(torch.bfloat16, rows, C)
    shape = L.make_rows(rows, C, torch.bfloat16)
    L.lasp_addnorm_fwd(shape, r.cuda(), None, None, None, EPS, None, clean)
    r[4, 3], r[9, 100] = float("inf"), float("nan")
    y = nan(torch.bfloat16, rows, C)
    L.lasp_addnorm_fwd(shape, r.cuda(), None, None, None, EPS, None, y)
    keep = [i for i in range(rows) if i not in (4, 9)]
    assert torch.equal(clean[keep], y[keep]) and y[9].isnan().all() and y[4, 3].isnan()


GATE_CASES = [  # B, H, N, D, over, fused
    (1, 1, 1, 8, "head", False),
    (64, 2, 1, 64, "head", False),
    (1, 16, 33, 128, "head", False),
    (3, 5, 17, 64, "head", True),
    (2, 3, 40, 96, "token", False),
    (1, 12, 7, 64, "token", True),
    (2, 1, 50, 1040, "head", True),
    (1, 1, 700, 24, "token", False),
    (1, 33, 9, 32, "head", False),
    (2, 7, 300, 128, "head", False),
    (1, 128, 3, 128, "token", False),
    (1, 2, 5, 8192, "head", False),
    (1, 2000, 3, 8, "head", False),
    (5, 2, 3, 256, "head", True),
]


@pytest.mark.parametrize("gate", ["none", "identity", "sigmoid", "silu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,N,D,over,fused", GATE_CASES)
def test_gatenorm(L, B, H, N, D, over, fused, dtype, gate):
    rng = np.random.default_rng(H * N + D)
    wide, ld = H * D, 3 * H * D if fused else 0
    (o, o64), (dy, dy64) = rounded(rng, dtype, B, H, N, D), rounded(rng, dtype, B, N, wide)
    u_all, _ = rounded(rng, dtype, B, N, ld or wide, scale=3.0)
    u64 = u_all[..., -wide:].double().numpy()
    w = torch.tensor(rng.normal(size=wide), dtype=torch.float32) if (H + N) % 3 else None
    w64 = None if w is None else w.double().numpy()
    print(f"case gatenorm {dtype} {gate} B={B} H={H} N={N} D={D} over={over} fused={fused}", flush=True)
    shape = L.make_gate_shape(B, H, N, D, DT[dtype], gate, over, ld)
    u = u_all.cuda()[..., -wide:] if gate != "none" else None
    du_all = nan(DT[dtype], B, N, ld or wide)
    du = du_all[..., -wide:] if gate != "none" else None
    y, do, dw = nan(DT[dtype], B, N, wide), nan(DT[dtype], B, H, N, D), nan(torch.float32, wide)
    wg = None if w is None else w.cuda()
    L.lasp_gatenorm_fwd(shape, o.cuda(), u, wg, EPS, y)
    scratch = torch.full((L.gatenorm_scratch_bytes(shape),), 0x5a, dtype=torch.uint8, device="cuda")
    L.lasp_gatenorm_bwd(shape, o.cuda(), u, wg, EPS, dy.cuda(), do, du, dw, scratch)
    ref = bo.gatenorm(o64, u64, w64, EPS, gate, over, dy64)
    for name, t in (("y", y), ("do", do), ("du", du), ("dweight", dw)):
        if t is not None:
            half = 0.0 if name == "dweight" else bo.HALF[dtype]
            held(t, ref[name], half * np.abs(ref[name]) + ref["bound"][name], name)
    if fused and gate != "none":
        assert du_all[..., :-wide].isnan().all()          # what lies beside the gate's gradient is not touched
    do2, du2 = nan(DT[dtype], B, H, N, D), None if du is None else nan(DT[dtype], B, N, ld or wide)[..., -wide:]
    L.lasp_gatenorm_bwd(shape, o.cuda(), u, wg, EPS, dy.cuda(), do2, du2, None, None)
    assert torch.equal(do, do2) and (du is None or torch.equal(du, du2))


def test_gates_at_the_ends(L):
    """Gates far out: sigmoid and silu reach 0, 1 and u without NaN."""
    far = torch.tensor([-1e30, -1e4, -200.0, -90.0, 90.0, 200.0, 1e4, 1e30], dtype=torch.float32)
    o = torch.ones(1, 1, 1, 8, dtype=torch.float32, device="cuda")
    u = far.view(1, 1, 8).cuda()
    for gate, want in (("sigmoid", (far > 0).float()), ("silu", torch.where(far > 0, far, torch.zeros(8)))):
        shape = L.make_gate_shape(1, 1, 1, 8, torch.float32, gate)
        y, do, du = nan(torch.float32, 1, 1, 8), nan(torch.float32, 1, 1, 1, 8), nan(torch.float32, 1, 1, 8)
        L.lasp_gatenorm_fwd(shape, o, u, None, 0.0, y)
        torch.testing.assert_close(y.cpu().flatten(), want, rtol=1e-6, atol=1e-30)
        L.lasp_gatenorm_bwd(shape, o, u, None, 0.0, torch.ones(1, 1, 8, device="cuda"), do, du, None, None)
        assert du.isfinite().all()
        torch.testing.assert_close(du.cpu().flatten(), torch.zeros(8) if gate == "sigmoid" else (far > 0).float(), rtol=1e-6, atol=1e-30)


@pytest.mark.parametrize("over", ["head", "token"])
def test_runs_are_bit_reproducible_and_capturable(L, over):
    rng = np.random.default_rng(8)
    B, H, N, D = 2, 6, 1500, 128
    (o, _), (dy, _), (u, _) = rounded(rng, "bf16", B, H, N, D), rounded(rng, "bf16", B, N, H * D), rounded(rng, "bf16", B, N, H * D)
    o, dy, u = o.cuda(), dy.cuda(), u.cuda()
    w, scale = (torch.tensor(rng.normal(size=H * D), dtype=torch.float32, device="cuda") for _ in range(2))
    shape, rows = L.make_gate_shape(B, H, N, D, torch.bfloat16, "silu", over), L.make_rows(B * N, H * D, torch.bfloat16)
    y, r_out, z, dr, dx, du = (torch.empty(B, N, H * D, dtype=torch.bfloat16, device="cuda") for _ in range(6))
    do = torch.empty_like(o)
    grads = [torch.empty(H * D, device="cuda") for _ in range(3)]
    scratch = torch.empty(max(L.gatenorm_scratch_bytes(shape), L.addnorm_scratch_bytes(rows)), dtype=torch.uint8, device="cuda")

    def step():
        L.lasp_gatenorm_fwd(shape, o, u, w, EPS, y)
        L.lasp_addnorm_fwd(rows, dy, y, scale, w, EPS, r_out, z)
        L.lasp_addnorm_bwd(rows, r_out, y, scale, w, EPS, z, dy, dr, dx, grads[0], grads[1], scratch)
        L.lasp_gatenorm_bwd(shape, o, u, w, EPS, dx, do, du, grads[2], scratch)

    outs = [y, r_out, z, dr, dx, du, do] + grads
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in outs:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))
