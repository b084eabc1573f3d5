"""Gates above 1 whose products pass the largest float, against the definition in 64 bits, in every kernel that a call may be handed to."""
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


def both_passes(L, dtype, coupled, x, la, dout, h_in=None, dh_out=None):
    """64-bit copies of what the calls write, inputs as they come."""
    B, N, D = x.shape
    shape = L.make_rec_shape(B, N, D, DT[dtype], coupled)
    g = [None if t is None else t.cuda() for t in (x, la, dout, h_in, dh_out)]
    out, dx, dl = (torch.full_like(g[0], float("nan")) for _ in range(3))
    h_out, dh_in = (torch.full((B, D), float("nan"), device="cuda") for _ in range(2))
    scratch = torch.full((L.rec_scratch_bytes(shape),), 0x5a, dtype=torch.uint8, device="cuda")
    L.lasp_rec_fwd(shape, g[0], g[1], g[3], None, out, h_out, scratch)
    L.lasp_rec_bwd(shape, g[0], g[1], out, g[3], None, g[2], g[4], dx, dl, dh_in, scratch)
    return {k: t.cpu().double().numpy() for k, t in (("out", out), ("h_out", h_out), ("dx", dx), ("dlog_a", dl), ("dh_in", dh_in))}


def held(got, ref, room, label):
    err = np.abs(got - ref)
    room = np.broadcast_to(room, err.shape) + 1e-37
    worst = np.unravel_index(np.argmax(np.where(np.isfinite(err), err / room, np.inf)), err.shape)
    print(f"  {label}: {err[worst] / room[worst]:.3f} of the bound", flush=True)
    assert np.isfinite(err).all() and (err <= room).all(), (label, worst, got[worst], ref[worst], room[worst])


LENGTHS = [(1, 12, 64), (1, 60, 64), (2, 120, 64), (1, 300, 64), (2, 500, 64), (2, 2500, 64), (1, 1500, 1032), (1, 700, 4104), (1, 16500, 64), (1, 9000, 520)]


@pytest.mark.parametrize("coupled", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,N,D", LENGTHS)
def test_growing_gates_of_a_state_of_zero(L, B, N, D, dtype, coupled):
    """log a = 1 at every token: products of 89 gates and more pass the largest float. While nothing has entered the state it is 0 and
    stays 0; from the first x that is not 0 it grows, as far as it is followed here, by 2^29. The gradient likewise from the right."""
    x, la, dout = torch.zeros(B, N, D), torch.ones(B, N, D), torch.zeros(B, N, D)
    last = min(20, N)
    rng = np.random.default_rng(N + D)
    x[:, N - last:] = torch.tensor(rng.normal(size=(B, last, D)))
    dout[:, :last] = torch.tensor(rng.normal(size=(B, last, D)))
    x, la, dout = (t.to(DT[dtype]) for t in (x, la, dout))
    got = both_passes(L, dtype, coupled, x, la, dout)
    print(f"case {dtype} B={B} N={N} D={D} coupled={coupled}", flush=True)
    d = [t.double().numpy() for t in (x, la, dout)]
    # what is not 0 is in the last (backward the first) tokens, so that the definition's loops can stay short
    k = min(N, 2 * last)
    out, h_out = bo.rec_fwd(d[0][:, N - k:], d[1][:, :k], coupled=coupled)
    dx, _, dh_in = bo.rec_bwd(d[0][:, :k] * 0, d[1][:, :k], d[2][:, :k], coupled=coupled)
    tail = bo.rec_bounds(dtype, d[0][:, N - k:], d[1][:, :k], d[2][:, :k] * 0, coupled=coupled)
    head = bo.rec_bounds(dtype, d[0][:, :k] * 0, d[1][:, :k], d[2][:, :k], coupled=coupled)
    held(got["out"][:, N - k:], out, tail["out"], "out")
    held(got["h_out"], h_out, tail["h_out"], "h_out")
    held(got["dx"][:, :k], dx, head["dx"], "dx")
    held(got["dh_in"], dh_in, head["dh_in"], "dh_in")
    assert not got["out"][:, :N - k].any() and not got["dx"][:, k:].any()
    if N > 2 * k:   # dlog_a: the state in front is 0 where the gradient is not, and the gradient 0 where the state is not
        assert np.isfinite(got["dlog_a"]).all() and not got["dlog_a"][:, k:N - k].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [60, 128, 300, 700])
def test_growth_beyond_the_largest_float_from_a_tiny_state(L, N, dtype):
    """The state enters as 2^-120 and grows by e^150 over the sequence, of which e^130 lie between tokens 10 and 40: a product that no float
    holds times a state that is far below 1. Every step's gate is rounded to (|log a| + 16) 2^-24, 150 + 16 N of them."""
    x = torch.zeros(1, N, 8, dtype=DT[dtype])
    la = torch.full((1, N, 8), 20.0 / (N - 30)).to(DT[dtype])
    la[:, 10:40] = torch.tensor(4.34375).to(DT[dtype])
    h_in = torch.full((1, 8), 2.0 ** -120)
    got = both_passes(L, dtype, False, x, la, x, h_in, h_in)
    ref = 2.0 ** -120 * np.exp(np.cumsum(la.double().numpy(), axis=1))
    off = (200 + 16 * N) * 2.0 ** -24
    held(got["out"], ref, (bo.HALF[dtype] + off) * ref, "out")
    held(got["h_out"], ref[:, -1], off * ref[:, -1], "h_out")
    held(got["dh_in"], ref[:, -1], off * ref[:, -1], "dh_in")
