"""The bound that float results of the delta rule are held to tells products with factors in three bfloat16 parts (all of a float's bits) from products with two:
the mistake is planted in the oracle's recurrence here, on the CPU."""
import numpy as np
import pytest
import torch


def cut(x, parts):
    """x as the sum of its first bfloat16 parts."""
    x = torch.as_tensor(np.ascontiguousarray(x))
    whole, rest = torch.zeros_like(x), x.clone()
    for _ in range(parts):
        p = rest.float().to(torch.bfloat16).double()
        whole, rest = whole + p, rest - p
    return whole.numpy()


def float_results(x, parts):
    """kv_out, dkv_in, dlog_g and dbeta [H]... of one sequence, with states, their gradients, u and dV cut to parts where they enter products with keys."""
    q, k, v, log_g, beta, S, dout, dS = (x[n] for n in ("q", "k", "v", "log_g", "beta", "kv_in", "dout", "dkv_out"))
    a, before, (H, N, _) = np.exp(log_g), [], v.shape

    def residual(s):
        aS = a[:, s, None, None] * before[s]
        return aS, v[:, s] - np.einsum("hd,hdc->hc", k[:, s], cut(aS, parts))

    for s in range(N):
        before.append(S)
        aS, w = residual(s)
        S = aS + np.einsum("hd,hc->hdc", k[:, s], cut(beta[:, s, None] * w, parts))
    got = {"kv_out": S, "dlog_g": np.zeros((H, N)), "dbeta": np.zeros((H, N))}
    for s in range(N - 1, -1, -1):
        aS, w = residual(s)
        dS = dS + np.einsum("hd,hc->hdc", q[:, s], dout[:, s])
        du = np.einsum("hdc,hd->hc", cut(dS, parts), k[:, s])
        got["dbeta"][:, s] = (du * w).sum(-1)
        dS = dS - np.einsum("hd,hc->hdc", k[:, s], cut(beta[:, s, None] * du, parts))
        got["dlog_g"][:, s] = (dS * aS).sum((-1, -2))
        dS = a[:, s, None, None] * dS
    return {**got, "dkv_in": dS}


@pytest.mark.parametrize("D,N", [(64, 200), (128, 200), (128, 400)])
def test_two_parts_are_told_from_three(D, N):
    from oracle import delta_oracle as O
    r = np.random.RandomState(D + N)
    H, Dv = 2, 64
    unit = lambda t: t / np.linalg.norm(t, axis=-1, keepdims=True)   # noqa: E731
    x = {"q": 0.3 * unit(r.randn(H, N, D) + 0.3), "k": unit(r.randn(H, N, D) + 0.3), "v": r.randn(H, N, Dv), "log_g": -0.2 * r.rand(H, N) ** 3,
         "beta": r.rand(H, N), "kv_in": 0.5 * r.randn(H, D, Dv), "dout": r.randn(H, N, Dv), "dkv_out": 0.5 * r.randn(H, D, Dv)}
    one = {n: t[None] for n, t in x.items()}
    args = [one[n] for n in ("q", "k", "v", "log_g", "beta")]
    want = O.delta_bwd(*args, one["dout"], one["kv_in"], None, one["dkv_out"])
    want["kv_out"] = O.delta_fwd(*args, one["kv_in"])[1]
    for parts in (3, 2):
        off = {n: O.off_in_norm(t, want[n][0]) for n, t in float_results(x, parts).items()}
        print(parts, off)
        if parts == 3:
            assert max(off.values()) < 0.01
        else:
            assert max(off.values()) > 1.0 and min(off.values()) > 0.1     # (one result past the bound fails the comparison)
