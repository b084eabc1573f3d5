"""Gradients of the gates of lasp_gatenorm_bwd where a sigmoid is nearly 0 or 1, relative to their size.

Rows of ones with eps = 0 have a root mean square of exactly 1, so du = dy act'(u). With e = exp(-|u|): the exponent is rounded to
2^-24 |u| log2 e in two steps, and the power, the sum and the reciprocal add 2^-23 each: s and 1 - s are off by at most a relative
(|u| + 4) 2^-23. sigmoid' = s (1 - s): twice that. silu' = s (1 + u (1 - s)): the same of s (1 + |u| (1 - s)). Every product rounds
once more (2^-24), the stored value by half a step of its type."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = [0.0, 0.5, 1.25, 3.0, 6.0, 8.0, 10.0, 11.0, 12.0, 13.5, 15.0, 16.0, 16.5, 17.0, 18.0, 20.0, 24.0, 30.0, 40.0, 60.0, 80.0]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["sigmoid", "silu"])
def test_slopes(dtype, gate):
    assert torch.cuda.is_available(), "needs a GPU"
    from paper_2404_02882_amd import lasp as L
    u = torch.tensor([s * v for v in U for s in (1.0, -1.0)] + [0.25] * 6, dtype=torch.float32).to(DT[dtype]).view(1, 1, -1)
    n = u.numel()
    dy = torch.linspace(0.5, 2.0, n).to(DT[dtype]).view(1, 1, n)
    shape = L.make_gate_shape(1, 1, 1, n, DT[dtype], gate)
    o = torch.ones(1, 1, 1, n, dtype=DT[dtype], device="cuda")
    do, du = torch.full_like(o, float("nan")), torch.full((1, 1, n), float("nan"), dtype=DT[dtype], device="cuda")
    L.lasp_gatenorm_bwd(shape, o, u.cuda(), None, 0.0, dy.cuda(), do, du, None, None)
    v, d = u.double().numpy().ravel(), dy.double().numpy().ravel()
    s, c = 1.0 / (1.0 + np.exp(-v)), 1.0 / (1.0 + np.exp(v))      # c: 1 - s
    ref, size = (s * c, s * c) if gate == "sigmoid" else (s * (1.0 + v * c), s * (1.0 + np.abs(v) * c))
    room = bo.HALF[dtype] * np.abs(d * ref) + (2 * np.abs(v) + 12) * 2.0 ** -23 * d * size
    err = np.abs(du.cpu().double().numpy().ravel() - d * ref)
    worst = int(np.argmax(err / room))
    print(f"{gate} {dtype}: {err[worst] / room[worst]:.3f} of the bound at u = {v[worst]}", flush=True)
    assert (err <= room).all(), (v[err > room], err[err > room] / np.abs(d * ref)[err > room])
