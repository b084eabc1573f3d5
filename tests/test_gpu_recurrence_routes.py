"""The recurrence's kernels that no other size is handed to, against the 64-bit oracle: a thread per column over more tokens than it requests
together, and where columns alone fill the device; rows that are no whole lines in blocks of 32 columns and, float, in tiles of 8 waves;
calls past the last-level cache, whose loads and stores leave it (non-temporal)."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
W = 464     # gates up to e^-0.11: what lies so far away weighs less than 2^-73


@pytest.fixture(scope="module")
def L():
    assert torch.cuda.is_available(), "needs a GPU"
    from paper_2404_02882_amd import lasp
    return lasp


def windows(N):
    """Token ranges to look at: the ends, across the borders of tiles, the middle."""
    if N <= 600:
        return [(0, N)]
    return sorted({(max(0, t - 24), min(N, t + 24)) for t in (0, 256, 512, min(N, 1024), N // 2, N)})


def some(D):
    """Channels to look at: the first and last column blocks', and some between."""
    return np.unique(np.concatenate([np.arange(min(D, 40)), np.arange(max(0, D - 40), D), np.arange(0, D, max(1, D // 37))]))


def check(L, dtype, B, N, D, coupled, lens=None, fused=False, seqs=None):
    g = torch.Generator(device="cuda").manual_seed(N + D)
    dt = DT[dtype]
    both = torch.empty(B, N, 2 * D if fused else D, dtype=dt, device="cuda")
    if fused:
        x, la = both[..., :D], both[..., D:]
        dboth = torch.full_like(both, float("nan"))
        dx, dl = dboth[..., :D], dboth[..., D:]
    else:
        x, la, dx, dl = both, torch.empty_like(both), torch.full_like(both, float("nan")), torch.full_like(both, float("nan"))
    x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
    la.copy_(torch.rand(x.shape, generator=g, device="cuda") * -0.89 - 0.11)
    dout = torch.randn(B, N, D, generator=g, device="cuda").to(dt)
    h_in, dh_out = (torch.randn(B, D, generator=g, device="cuda") for _ in range(2))
    n = torch.tensor(lens if lens else [N] * B, dtype=torch.int32, device="cuda")
    shape = L.make_rec_shape(B, N, D, dt, coupled, 2 * D if fused else 0)
    out, h_out, dh_in = torch.full((B, N, D), float("nan"), dtype=dt, device="cuda"), torch.full_like(h_in, float("nan")), torch.full_like(h_in, float("nan"))
    scratch = torch.full((L.rec_scratch_bytes(shape),), 0x5a, dtype=torch.uint8, device="cuda")
    print(f"case rec {dtype} B={B} N={N} D={D} lens={lens} fused={fused} coupled={coupled}", flush=True)
    L.lasp_rec_fwd(shape, x, la, h_in, n if lens else None, out, h_out, scratch)
    L.lasp_rec_bwd(shape, x if coupled else None, la, out, h_in, n if lens else None, dout, dh_out, dx, dl, dh_in, scratch)
    assert not bool(out.isnan().any()) and not bool(dx.isnan().any()) and not bool(dl.isnan().any())
    seqs, chans = list(range(B)) if seqs is None else seqs, some(D)
    at = torch.tensor(chans, device="cuda")
    pick = lambda t, a, b: t[seqs, a:b][..., at].cpu().double().numpy()   # noqa: E731
    state = lambda t: t[seqs][:, at].cpu().double().numpy()   # noqa: E731
    length = n[seqs].cpu().numpy()
    for t0, t1 in windows(N):
        a, b = max(0, t0 - W), min(N, t1 + W)
        there = np.clip(length - a, 0, b - a)
        args = dict(h_in=state(h_in) if a == 0 else np.zeros((len(seqs), len(chans))), lens=there, coupled=coupled)
        ends = np.where((length <= b)[:, None], state(dh_out), 0.0)
        vx, vl, vd = pick(x, a, b), pick(la, a, b), pick(dout, a, b)
        ref = dict(zip(("out", "h_out"), bo.rec_fwd(vx, vl, **args)))
        ref.update(zip(("dx", "dlog_a", "dh_in"), bo.rec_bwd(vx, vl, vd, dh_out=ends, **args)))
        room = bo.rec_bounds(dtype, vx, vl, vd, dh_out=ends, **args)
        for name, t in (("out", out), ("dx", dx), ("dlog_a", dl)):
            sl = slice(t0 - a, t1 - a)
            held(pick(t, t0, t1), ref[name][:, sl], room[name][:, sl], f"{name} {t0}..{t1}")
        mine = (length > a + (W if a else -1)) & (length <= b)     # sequences that end here
        if mine.any():
            held(state(h_out)[mine], ref["h_out"][mine], room["h_out"][mine], "h_out")
        if a == 0:
            held(state(dh_in), ref["dh_in"], room["dh_in"], "dh_in")


def held(got, ref, room, label):
    err, room = np.abs(got - ref), room + 1e-37
    worst = np.unravel_index(np.argmax(np.where(np.isfinite(err), err / room, np.inf)), err.shape)
    print(f"  {label}: {err[worst] / room[worst]:.3f} of the bound", flush=True)
    assert np.isfinite(err).all() and (err <= room).all(), (label, worst, got[worst], ref[worst], room[worst])


@pytest.mark.parametrize("coupled", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,N,D,lens", [(2, 8, 72, None), (2, 9, 64, None), (3, 13, 40, [13, 9, 2]), (5, 16, 1000, [16, 0, 8, 15, 1])])
def test_a_thread_per_column(L, B, N, D, lens, dtype, coupled):
    check(L, dtype, B, N, D, coupled, lens)


@pytest.mark.parametrize("dtype,B,N,D,lens", [
    ("bf16", 64, 17, 8192, None),                           # 65536 columns
    ("bf16", 128, 17, 8192, None),
    ("bf16", 128, 128, 8192, [128, 1, 0, 77] * 32),
    ("f32", 64, 41, 8192, [41, 40, 0, 9] * 16),
    ("f32", 131072, 33, 8, None),                           # two columns each
])
def test_columns_that_fill_the_device(L, dtype, B, N, D, lens):
    check(L, dtype, B, N, D, True, lens, seqs=[0, 1, 2, 3, B - 2, B - 1])


@pytest.mark.parametrize("coupled", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,N,D,lens,fused", [
    (1, 700, 4104, None, False),                            # 513 columns (float 1026)
    (1, 1300, 4104, None, True),
    (5, 900, 1000, [900, 0, 513, 899, 64], False),          # sequences that begin inside a block
    (2, 513, 2104, [513, 300], False),
])
def test_rows_that_are_no_lines_in_blocks_of_32(L, B, N, D, lens, fused, dtype, coupled):
    check(L, dtype, B, N, D, coupled, lens, fused)


@pytest.mark.parametrize("coupled", [False, True])
@pytest.mark.parametrize("dtype,D", [("f32", 264), ("bf16", 520)])
@pytest.mark.parametrize("N", [8200, 16400])
def test_few_rows_that_are_no_lines_in_tiles_of_8_waves(L, N, dtype, D, coupled):
    check(L, dtype, 1, N, D, coupled)


@pytest.mark.parametrize("coupled", [False, True])
@pytest.mark.parametrize("dtype,B,N,D,lens,fused", [
    ("bf16", 2, 11200, 2048, [11200, 9001], False),
    ("f32", 2, 5600, 2048, [3000, 5600], False),
    ("bf16", 1, 45000, 1024, None, True),
    ("bf16", 1, 90000, 512, None, False),                   # backward in tiles of 8 waves
    ("f32", 1, 90000, 256, None, False),
])
def test_past_the_last_level_cache(L, dtype, B, N, D, lens, fused, coupled):
    check(L, dtype, B, N, D, coupled, lens, fused)
