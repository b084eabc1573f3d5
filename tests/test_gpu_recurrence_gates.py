"""Gates of the recurrence at their limits, against the definition in 64 bits, in every kernel that a call may be handed to."""
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


CLOSE = [-2.0 ** -5, -2.0 ** -6, -2.0 ** -7 * 1.25, -1e-3, -2.0 ** -12, -1e-4, -1e-5, -1e-6, -1e-7, -3e-8, -1e-8, -1e-12, -1e-20, -1e-30, -2.0 ** -4, 0.0]
APART = [-2.0 ** -13, -2.0 ** -13 * 1.5, -2.0 ** -12, -2.0 ** -11 * 1.25, -2.0 ** -10, -2.0 ** -9, -2.0 ** -8, -2.0 ** -7] * 2


@pytest.mark.parametrize("logs", [CLOSE, APART])
@pytest.mark.parametrize("N", [1, 12, 60, 300, 2500])
def test_bfloat16_gates_close_to_one(L, N, logs):
    """Coupled: b = 1 - a to a relative 2^-12 however near to 1 a is: -log_a up to 2^-11, which leaves out log_a / 2 of it; beyond, the
    power's distance from 1, of which a step, 2^-24 of 1, is at most 2^-13.

    All x and dout are positive, so every sum is of terms of one sign, and a relative error of b is at most the same of out; the N
    roundings of a sum and of its joins add N 2^-23 (steps of a float, 2^-24 each, and the gates' own). What the type rounds: half
    a step 2^-8. dlog_a = a e (h_{s-1} - x): h as stored, half a step of h more."""
    rng = np.random.default_rng(N)
    la = torch.tensor(logs, dtype=torch.float32).to(torch.bfloat16).expand(2, N, 16).contiguous()
    x, dout = (torch.tensor(0.5 + rng.random((2, N, 16)), dtype=torch.float32).to(torch.bfloat16) for _ in range(2))
    got = both_passes(L, "bf16", True, x, la, dout)
    d = [t.double().numpy() for t in (x, la, dout)]
    out, h_out = bo.rec_fwd(d[0], d[1], coupled=True)
    dx, dl, dh_in = bo.rec_bwd(d[0], d[1], d[2], coupled=True)
    off, half = 2.0 ** -12 + (N + 8) * 2.0 ** -23, bo.HALF["bf16"]
    held(got["out"], out, (half + off) * out, "out")
    held(got["h_out"], h_out, off * h_out, "h_out")
    held(got["dx"], dx, (half + 2 * off) * dx, "dx")
    held(got["dh_in"], dh_in, off * dh_in, "dh_in")
    a = np.exp(d[1])
    e = np.divide(dx, -np.expm1(d[1]), out=np.zeros_like(dx), where=d[1] < 0)
    before = np.concatenate([np.zeros((2, 1, 16)), out[:, :-1]], axis=1)
    held(got["dlog_a"], dl, half * np.abs(dl) + a * e * ((half + 2 * off) * before + 3 * off * (before + d[0])) + (d[1] == 0) * 1e30, "dlog_a")
