"""Norms over many rows: the weights' gradients by value where many workgroups each leave a partial row, and calls past the last-level
cache (non-temporal loads and stores) at every way a row is spread over threads, against the formulas in 64 bits.

Bounds as in the oracle (KAPPA: fewer than 128 roundings of 2^-24 in any sum): rows 4 KAPPA of their absolute terms and half a step of the
type, columns 4 KAPPA of the sum of absolute terms. Here a column's sum is of at most 48 rows in a thread, 7 additions over a wave
and a workgroup, and 16 + 32 partial rows."""
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


def held(got, ref, room, label):
    share = float(((got.double() - ref).abs() / (room + 1e-37)).nan_to_num(nan=float("inf")).max())
    assert share <= 1.0, (label, share)
    return share


WIDTHS = [8, 16, 32, 64, 128, 256, 512, 1024, 2048, 4096, 8192, 16384]


def normal(g, dtype, *size):
    return torch.randn(*size, generator=g, device="cuda").to(DT[dtype])


@pytest.mark.parametrize("dtype,rows,C,carry", [
    ("bf16", 8192, 264, True), ("f32", 8192, 136, False), ("bf16", 5000, 2048, False), ("f32", 9001, 520, True),
    ("bf16", 12000, 2048, True), ("f32", 6000, 2048, True),        # past the cache
    ("bf16", 1500, 16384, True), ("f32", 1400, 8192, False), ("f32", 720, 16384, True),
])
def test_addnorm_backward(L, dtype, rows, C, carry):
    addnorm_backward(L, dtype, rows, C, carry)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", WIDTHS)
def test_addnorm_past_the_cache(L, dtype, C):
    rows = (35 if dtype == "bf16" else 18) * 10 ** 6 // C
    addnorm_backward(L, dtype, rows, C, True)
    g = torch.Generator(device="cuda").manual_seed(C)
    r, x = (normal(g, dtype, rows, C) for _ in range(2))
    scale, w = (torch.randn(C, generator=g, device="cuda") for _ in range(2))
    r_out, y = torch.full_like(r, float("nan")), torch.full_like(r, float("nan"))
    L.lasp_addnorm_fwd(L.make_rows(rows, C, DT[dtype]), r, x, scale, w, EPS, r_out, y)
    half, step = bo.HALF[dtype], max(512, (1 << 20) // C)
    for i in range(0, rows, step):
        s = slice(i, min(rows, i + step))
        R, X = r[s].double(), x[s].double()
        ref, off = R + scale.double() * X, 2.0 ** -22 * (R.abs() + (scale.double() * X).abs())
        rstd = 1.0 / (ref.square().mean(-1, keepdim=True) + EPS).sqrt()
        moved = off.square().mean(-1, keepdim=True).sqrt() * rstd          # as rstd moves with the errors of the row
        held(r_out[s], ref, half * ref.abs() + off, "r_out")
        ref = w.double() * ref * rstd
        held(y[s], ref, half * ref.abs() + w.double().abs() * rstd * off + (bo.KAPPA + moved) * ref.abs(), "y")


def addnorm_backward(L, dtype, rows, C, carry):
    g = torch.Generator(device="cuda").manual_seed(rows + C)
    r, x, dy, dro = (normal(g, dtype, rows, C) for _ in range(4))
    scale, w = (torch.randn(C, generator=g, device="cuda") for _ in range(2))
    dr, dx, dw, ds = torch.full_like(r, float("nan")), torch.full_like(r, float("nan")), *(torch.full_like(w, float("nan")) for _ in range(2))
    shape = L.make_rows(rows, C, DT[dtype])
    scratch = torch.full((L.addnorm_scratch_bytes(shape),), 0x5a, dtype=torch.uint8, device="cuda")
    print(f"case addnorm {dtype} rows={rows} C={C} carry={carry}", flush=True)
    L.lasp_addnorm_bwd(shape, r, x, scale, w, EPS, dy, dro if carry else None, dr, dx, dw, ds, scratch)
    half, k = bo.HALF[dtype], 4 * bo.KAPPA
    sums = {n: torch.zeros(2, C, dtype=torch.float64, device="cuda") for n in ("dweight", "dscale")}     # values, bounds
    worst = {}
    sc, wt = scale.double(), w.double()
    step = max(512, (1 << 20) // C)
    for i in range(0, rows, step):
        s = slice(i, min(rows, i + step))
        R, X, Y, O = (t[s].double() for t in (r, x, dy, dro if carry else torch.zeros_like(dro)))
        rstd = 1.0 / (R.square().mean(-1, keepdim=True) + EPS).sqrt()
        ref = O + rstd * (wt * Y - R * rstd.square() * (wt * Y * R).mean(-1, keepdim=True))
        off = k * (O.abs() + rstd * ((wt * Y).abs() + R.abs() * rstd.square() * (wt * Y * R).abs().mean(-1, keepdim=True)))
        worst["dr"] = max(worst.get("dr", 0.0), held(dr[s], ref, half * ref.abs() + off, "dr"))
        worst["dx"] = max(worst.get("dx", 0.0), held(dx[s], sc * ref, (half + 2.0 ** -23) * (sc * ref).abs() + sc.abs() * off, "dx"))
        t = Y * R * rstd
        sums["dweight"] += torch.stack([t.sum(0), k * t.abs().sum(0)])
        sums["dscale"] += torch.stack([(X * ref).sum(0), (X.abs() * off).sum(0) + k * (X * ref).abs().sum(0)])
    for name, got in (("dweight", dw), ("dscale", ds)):
        worst[name] = held(got, sums[name][0], sums[name][1], name)
    print("  ", {n: round(v, 3) for n, v in worst.items()}, flush=True)


@pytest.mark.parametrize("dtype,B,H,N,D,over,gate", [
    ("bf16", 1, 16, 4100, 128, "head", "silu"), ("f32", 2, 3, 5001, 64, "head", "sigmoid"), ("f32", 2, 8, 2500, 64, "token", "silu"),
    ("bf16", 3, 5, 3000, 96, "token", "identity"),
    ("bf16", 1, 16, 13500, 128, "head", "silu"), ("f32", 2, 16, 3400, 128, "head", "sigmoid"),      # past the cache
    ("bf16", 2, 8, 13500, 128, "token", "sigmoid"), ("f32", 1, 128, 840, 128, "token", "silu"), ("bf16", 1, 1, 1700, 16384, "head", "silu"),
    ("f32", 1, 5, 21000, 128, "head", "silu"),
])
def test_gatenorm_both_passes(L, dtype, B, H, N, D, over, gate):
    gatenorm_both_passes(L, dtype, B, H, N, D, over, gate)


@pytest.mark.parametrize("past", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", WIDTHS)
def test_gatenorm_heads_of_every_width(L, dtype, D, past):
    H = max(1, 1024 // D)
    most = (46 if dtype == "bf16" else 23) * 10 ** 6 if past else 10 ** 6
    gatenorm_both_passes(L, dtype, 1, H, most // (H * D), D, "head", "silu")


def gatenorm_both_passes(L, dtype, B, H, N, D, over, gate):
    g = torch.Generator(device="cuda").manual_seed(H * N + D)
    o, u, dy = normal(g, dtype, B, H, N, D), normal(g, dtype, B, N, H * D), normal(g, dtype, B, N, H * D)
    w = torch.randn(H * D, generator=g, device="cuda")
    y, do, du, dw = (torch.full_like(t, float("nan")) for t in (u, o, u, w))
    shape = L.make_gate_shape(B, H, N, D, DT[dtype], gate, over)
    scratch = torch.full((L.gatenorm_scratch_bytes(shape),), 0x5a, dtype=torch.uint8, device="cuda")
    print(f"case gatenorm {dtype} B={B} H={H} N={N} D={D} over={over} gate={gate}", flush=True)
    L.lasp_gatenorm_fwd(shape, o, u, w, EPS, y)
    L.lasp_gatenorm_bwd(shape, o, u, w, EPS, dy, do, du, dw, scratch)
    half, k = bo.HALF[dtype], 4 * bo.KAPPA
    sums, worst = torch.zeros(2, H * D, dtype=torch.float64, device="cuda"), {}
    rows = (lambda t: t.reshape(-1, H, D)) if over == "head" else (lambda t: t.reshape(-1, 1, H * D))
    W = rows(w.double())
    for b in range(B):
        for i in range(0, N, 2048):
            s = slice(i, min(N, i + 2048))
            O, U, Y = rows(o[b, :, s].transpose(0, 1).double()), rows(u[b, s].double()), rows(dy[b, s].double())
            rstd = 1.0 / (O.square().mean(-1, keepdim=True) + EPS).sqrt()
            n = O * rstd
            if gate == "identity":
                act, slope, loose, size = U, torch.ones_like(U), 0.0, 1.0
            else:
                sg = torch.sigmoid(U)
                act, slope = (sg, sg * (1 - sg)) if gate == "sigmoid" else (U * sg, sg * (1 + U * (1 - sg)))
                size = slope if gate == "sigmoid" else sg * (1 + U.abs() * (1 - sg))
                loose = 2.0 ** -21 * (1 + U.abs()) ** 2       # (a sigmoid and its complement: a relative (|u| + 4) 2^-23, the slope twice that)
            # (rows of one token again)
            flat = lambda t: t.reshape(-1, H * D)   # noqa: E731
            ref, t = flat(W * n * act), Y * act
            parts = {"y": (y[b, s], ref, half * ref.abs() + flat((W * n).abs() * loose * act.abs()) + k * ref.abs())}
            ref = flat(Y * W * n * slope)
            parts["du"] = (du[b, s], ref, half * ref.abs() + flat((Y * W * n).abs() * loose * size) + k * ref.abs())
            wt, off = W * t, (W * t).abs() * loose
            ref = flat(rstd * (wt - n * (wt * n).mean(-1, keepdim=True)))
            room = half * ref.abs() + flat(rstd * (off + n.abs() * (off * n.abs()).mean(-1, keepdim=True)
                                                   + k * (wt.abs() + n.abs() * (wt * n).abs().mean(-1, keepdim=True))))
            parts["do"] = (flat(do[b, :, s].transpose(0, 1)), ref, room)
            for name, part in parts.items():
                worst[name] = max(worst.get(name, 0.0), held(*part, name))
            sums += torch.stack([flat(t * n).sum(0), flat((k + loose) * (t * n).abs()).sum(0)])
    worst["dweight"] = held(dw, sums[0], sums[1], "dweight")
    print("  ", {m: round(v, 3) for m, v in worst.items()}, flush=True)
