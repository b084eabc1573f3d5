"""Host-side checks of the gated delta rule and of the norm and rotation of queries and keys that need no GPU: the oracle against
differences and closed forms, shapes, sizes, and the refusals of bad arguments before any launch (no compute call is made here)."""
import ctypes
import math

import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def L():
    from paper_2404_02882_amd import lasp
    return lasp


def fake(n):
    """Distinct non-null addresses that are never dereferenced (validation fails first)."""
    return ctypes.c_void_p(0x100000000 + n * 0x40000000)


def refused(fn, args, changes):
    for i, value, status in changes:
        a = list(args)
        a[i] = value
        assert fn(*a) == status, (i, value)


# ---- oracle ---------------------------------------------------------------------
def case(seed=3, B=2, H=2, Hk=1, N=5, D=4, Dv=3):
    r = np.random.RandomState(seed)
    k = r.randn(B, Hk, N, D)
    x = {"q": r.randn(B, Hk, N, D), "k": k / np.linalg.norm(k, axis=-1, keepdims=True), "v": r.randn(B, H, N, Dv), "log_g": -r.rand(B, H, N),
         "beta": r.rand(B, H, N), "kv_in": r.randn(B, H, D, Dv)}
    return x, r.randn(B, H, N, Dv), r.randn(B, H, D, Dv)


def test_oracle_gradients_are_differences():
    from oracle import delta_oracle as O
    x, dout, dkv = case()
    lens = np.array([5, 3])
    loss = lambda **y: (lambda o, s, _: (o * dout).sum() + (s * dkv).sum())(*O.delta_fwd(lens=lens, **{**x, **y}))   # noqa: E731
    g = O.delta_bwd(dout=dout, dkv_out=dkv, lens=lens, **x)
    r = np.random.RandomState(1)
    for name in ("q", "k", "v", "log_g", "beta", "kv_in"):
        d, h = r.randn(*x[name].shape), 1e-5
        diff = (loss(**{name: x[name] + h * d}) - loss(**{name: x[name] - h * d})) / (2 * h)
        assert abs(diff - (g["d" + name] * d).sum()) <= 1e-7 * max(1.0, abs(diff)), name


def test_oracle_closed_forms():
    """beta = 1 and one key for all tokens: the state returns the last value. Orthonormal keys: it is plain attention with decay."""
    from oracle import delta_oracle as O
    r = np.random.RandomState(0)
    k, v = np.zeros((1, 1, 6, 4)), r.randn(1, 1, 6, 3)
    k[..., 1] = 1.0
    out, S, _ = O.delta_fwd(k, k, v, None, np.ones((1, 1, 6)))
    assert np.allclose(out, v, atol=1e-15) and np.allclose(S[0, 0, 1], v[0, 0, -1], atol=1e-15)
    k = np.eye(4)[None, None]
    v, q, lg, bt = r.randn(1, 1, 4, 3), r.randn(1, 1, 4, 4), -r.rand(1, 1, 4), r.rand(1, 1, 4)
    out, _, _ = O.delta_fwd(q, k, v, lg, bt)
    G = np.cumsum(lg[0, 0])
    want = [sum(math.exp(G[s] - G[i]) * bt[0, 0, i] * q[0, 0, s, i] * v[0, 0, i] for i in range(s + 1)) for s in range(4)]
    assert np.allclose(out[0, 0], want, atol=1e-14)


def test_oracle_rotation():
    """Pairs turn as complex numbers do, lengths stay, and the products of two rotated vectors go by their distance."""
    from oracle import delta_oracle as O
    r = np.random.RandomState(0)
    x, y, f = r.randn(7, 12), r.randn(7, 12), np.array([0.7, 0.1, 1e-3])
    for layout in ("half", "interleaved"):
        a, b = O.pairs_of(6, layout)
        z = (x[:, a] + 1j * x[:, b]) * np.exp(1j * np.arange(7)[:, None] * f)
        got = O.rotate(x, np.arange(7), f, 6, layout, 1.0)
        assert np.allclose(got[:, a], z.real) and np.allclose(got[:, b], z.imag) and (got[:, 6:] == x[:, 6:]).all()
        p = np.arange(7)
        one = (O.rotate(x, p + 5, f, 6, layout, 1.0) * O.rotate(y, p, f, 6, layout, 1.0)).sum(-1)
        two = (O.rotate(x, p * 0 + 5, f, 6, layout, 1.0) * y).sum(-1)
        assert np.allclose(one, two)


@pytest.mark.parametrize("norm", ["none", "rms", "l2"])
def test_oracle_qk_gradients_are_differences(norm):
    from oracle import delta_oracle as O
    r = np.random.RandomState(2)
    x, w, dy, pos, f = r.randn(2, 3, 2 * 8), r.randn(8), r.randn(2, 2, 3, 8), r.randint(0, 50, (2, 3)), np.array([1.0, 0.1])
    fn = lambda x, w: (O.qk_fwd(x, 2, w, norm, 1e-3, pos, f, 4, "half", 1.3) * dy).sum()   # noqa: E731
    dx, dw = O.qk_bwd(x, 2, w, norm, 1e-3, pos, f, 4, "half", 1.3, dy)
    for i, (t, g) in enumerate(((x, dx), (w, dw))):
        d, h = r.randn(*t.shape), 1e-5
        up, down = [x, w], [x, w]
        up[i], down[i] = t + h * d, t - h * d
        diff = (fn(*up) - fn(*down)) / (2 * h)
        assert abs(diff - (g * d).sum()) <= 1e-7 * max(1.0, abs(diff))


# ---- delta rule -------------------------------------------------------------------
@pytest.mark.parametrize("kw,expect", [
    (dict(), 0), (dict(B=1, H=1, N=1), 0), (dict(D=64), 0), (dict(D=96), 2), (dict(D=0), 2), (dict(Dv=64), 0), (dict(Dv=128), 0), (dict(Dv=32), 2),
    (dict(Dv=-64), 2), (dict(N=0), 2), (dict(B=0), 2), (dict(H=0), 2), (dict(key_heads=2), 0), (dict(key_heads=4), 0), (dict(key_heads=3), 2),
    (dict(key_heads=8), 2), (dict(key_heads=-1), 2), (dict(dtype=2), 3), (dict(dtype=-1), 3), (dict(B=1 << 14, H=4), 2), (dict(B=65535, H=1), 0),
    (dict(B=1 << 20, H=1 << 20), 2), (dict(N=2 ** 31 - 1), 0),
])
def test_delta_shapes(L, kw, expect):
    s = L.make_delta_shape(**{**dict(B=2, H=4, N=100, D=128, dtype=1), **kw})
    assert L.check_delta(s) == expect
    for size in (L.delta_cache_bytes, L.delta_scratch_bytes, L.delta_bwd_scratch_bytes):
        assert (size(s) > 0) == (expect == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_delta_sizes_grow_with_the_length(L, dtype):
    """A longer sequence is never given less room, from one token to the longest, and the cache holds a state for every 64 tokens (float data: 32)."""
    lengths = [1, 16, 17, 32, 33, 64, 65, 100, 1000, 32768, 32769, 1 << 20, 1 << 30, 2 ** 31 - 1]
    cache = [L.delta_cache_bytes(L.make_delta_shape(1, 2, n, 128, dtype)) for n in lengths]
    assert all(a <= b for a, b in zip(cache, cache[1:]))
    assert all(c >= -(-n // (64 if dtype == "bf16" else 32)) * 2 * 128 * 128 * 4 for n, c in zip(lengths, cache))
    back = [L.delta_bwd_scratch_bytes(L.make_delta_shape(1, 2, n, 128, dtype)) for n in lengths]
    assert all(b >= n * 2 * 128 * 4 for n, b in zip(lengths, back))


def test_delta_rejects_before_launch(L):
    s = L.make_delta_shape(2, 4, 100, 128, "bf16", 64, 2)
    sb, bb = L.delta_scratch_bytes(s), L.delta_bwd_scratch_bytes(s)
    q, k, v, lg, bt, kin, ln, out, kout, cache, scr = [fake(i) for i in range(1, 12)]
    dout, dkout, dq, dk, dv, dlg, dbt, dkin = [fake(i) for i in range(12, 20)]
    odd = lambda p: ctypes.c_void_p(p.value + 8)   # noqa: E731
    inside = lambda p: ctypes.c_void_p(p.value + 64)   # noqa: E731
    fwd = [ctypes.byref(s), q, k, v, lg, bt, kin, ln, out, kout, cache, scr, sb, None]
    refused(L.lib.lasp_delta_fwd, fwd, [
        (0, None, 1), (1, None, 1), (2, None, 1), (3, None, 1), (5, None, 1), (8, None, 1), (9, None, 1), (11, None, 5), (12, sb - 1, 5),
        (8, q, 6), (8, v, 6), (8, lg, 6), (9, v, 6), (9, inside(kin), 6), (8, kin, 6), (10, kin, 6), (11, kin, 6), (10, out, 6), (11, cache, 6), (9, cache, 6),
        (8, ln, 6)] + [(i, odd(p), 8) for i, p in ((1, q), (2, k), (3, v), (4, lg), (5, bt), (6, kin), (7, ln), (8, out), (9, kout), (10, cache),
                                                  (11, scr))])
    bwd = [ctypes.byref(s), q, k, v, lg, bt, ln, dout, dkout, cache, dq, dk, dv, dlg, dbt, dkin, scr, bb, None]
    refused(L.lib.lasp_delta_bwd, bwd, [(i, None, 1) for i in (0, 1, 2, 3, 5, 7, 9, 10, 11, 12, 14, 15)] + [
        (4, None, 1), (13, None, 1),                          # a gate without its gradient's place, a place without a gate
        (16, None, 5), (17, bb - 1, 5), (10, q, 6), (11, dq, 6), (12, v, 6), (12, dout, 6), (13, lg, 6), (14, dlg, 6), (15, cache, 6), (16, cache, 6),
        (15, inside(dkout), 6), (16, dkout, 6), (10, odd(dq), 8), (9, odd(cache), 8), (8, odd(dkout), 8), (15, odd(dkin), 8)])
    for bad, status in ((L.make_delta_shape(2, 4, 100, 80, "bf16"), 2), (L.make_delta_shape(2, 4, 100, 64, 7), 3)):
        assert L.lib.lasp_delta_fwd(*([ctypes.byref(bad)] + fwd[1:])) == status
        assert L.lib.lasp_delta_bwd(*([ctypes.byref(bad)] + bwd[1:])) == status
    # a few tokens with a cache need the scratch, too
    few = L.make_delta_shape(2, 4, 16, 128, "bf16", 64, 2)
    assert L.lib.lasp_delta_fwd(*([ctypes.byref(few)] + fwd[1:11] + [None, 0, None])) == 5


def test_delta_binding_refuses_tensors_that_do_not_fit(L):
    s = L.make_delta_shape(2, 4, 3, 64, torch.float32, 128, 2)
    t = lambda *size, dt=torch.float32: torch.zeros(size, dtype=dt)   # noqa: E731
    ok = [t(2, 2, 3, 64), t(2, 2, 3, 64), t(2, 4, 3, 128), None, t(2, 4, 3), None, None, t(2, 4, 3, 128), t(2, 4, 64, 128), None,
          torch.zeros(L.delta_scratch_bytes(s), dtype=torch.uint8)]
    with pytest.raises(ValueError, match="GPU"):
        L.lasp_delta_fwd(s, *ok)
    for i, bad in ((0, t(2, 4, 3, 64)), (1, t(2, 2, 3, 64, dt=torch.bfloat16)), (2, t(2, 4, 3, 64)), (3, t(2, 4)), (4, t(2, 4, 3, dt=torch.float64)),
                   (5, t(2, 4, 128, 128)), (6, t(3, dt=torch.int32)), (6, t(2, dt=torch.int64)), (7, t(2, 4, 6, 128)[:, :, ::2]), (8, t(2, 4, 64, 64))):
        a = list(ok)
        a[i] = bad
        with pytest.raises(ValueError):
            L.lasp_delta_fwd(s, *a)
    with pytest.raises(L.LaspError) as e:
        L.lasp_delta_fwd(L.make_delta_shape(2, 4, 3, 64, torch.float16), *ok)
    assert e.value.status == 3
    with pytest.raises(L.LaspError) as e:
        L.lasp_delta_fwd(s, *([None] + ok[1:]))
    assert e.value.status == 1


def test_delta_sequence_refuses_short_lists_first():
    from paper_2404_02882_amd import sequence
    seq = sequence.DeltaSequence(1, 2, 16, 64, torch.float32, T=2, device="cpu")
    full, short = [torch.zeros(1, 2, 8, 64)] * 2, [torch.zeros(1, 2, 8, 64)]
    for i in range(6):
        args = [full] * 6
        args[i] = short
        with pytest.raises(ValueError, match="1 tensors for 2 sub-sequences"):
            seq.forward(*args)
    for i in range(11):
        args = [full] * 11
        args[i] = short
        with pytest.raises(ValueError, match="1 tensors for 2 sub-sequences"):
            seq.backward(*args)
    with pytest.raises(ValueError, match="lens: 1 tensors"):
        seq.forward(full, full, full, None, full, full, lens=[torch.zeros(1, dtype=torch.int32)])
    with pytest.raises(ValueError, match="multiple"):
        sequence.DeltaSequence(1, 2, 15, 64, torch.float32, T=2, device="cpu")
    with pytest.raises(Exception, match="LASP_ERR_SHAPE"):
        sequence.DeltaSequence(1, 2, 16, 48, torch.float32, device="cpu")


# ---- queries and keys -------------------------------------------------------------
@pytest.mark.parametrize("kw,expect", [
    (dict(), 0), (dict(B=1, N=1, H=1, key_heads=0, D=8, rot=0), 0), (dict(D=256, rot=256), 0), (dict(D=264), 2), (dict(D=20), 2), (dict(D=0), 2),
    (dict(rot=8), 2), (dict(rot=-16), 2), (dict(rot=144), 2), (dict(rot=0), 0), (dict(rot=48), 0), (dict(norm="layer"), 2), (dict(layout="x"), 2),
    (dict(key_heads=-1), 2), (dict(key_heads=7), 0), (dict(H=0), 2), (dict(N=0), 2), (dict(ld=512), 0), (dict(ld=504), 2), (dict(ld=516), 2),
    (dict(ld=768), 0), (dict(key_heads=8, ld=512), 2), (dict(dtype=2), 3), (dict(B=1 << 15, N=1 << 15), 2), (dict(B=1 << 13, N=1 << 15, H=8), 2),
    (dict(H=65536, key_heads=1, N=1, B=1), 2),
])
def test_qk_shapes(L, kw, expect):
    s = L.make_qk_shape(**{**dict(B=2, N=10, H=4, key_heads=2, D=128, dtype=1, rot=128), **kw})
    assert L.check_qk(s) == expect
    assert (L.qk_scratch_bytes(s) > 0) == (expect == 0)


def test_qk_rejects_before_launch(L):
    s = L.make_qk_shape(2, 10, 4, 2, 128, "bf16", rot=64, ld=1024)
    sb = L.qk_scratch_bytes(s)
    xq, xk, wq, wk, fr, pos, q, k, dq, dk, dxq, dxk, dwq, dwk, scr = [fake(i) for i in range(1, 16)]
    odd = lambda p: ctypes.c_void_p(p.value + 8)   # noqa: E731
    nan, inf = float("nan"), float("inf")
    fwd = [ctypes.byref(s), xq, xk, wq, wk, 1e-5, fr, pos, 1.0, q, k, None]
    refused(L.lib.lasp_qk_fwd, fwd, [
        (0, None, 1), (1, None, 1), (2, None, 1), (6, None, 1), (9, None, 1), (10, None, 1), (5, -1.0, 2), (5, nan, 2), (8, inf, 2), (8, nan, 2),
        (9, xq, 6), (9, xk, 6), (10, q, 6), (10, wk, 6), (9, fr, 6), (9, pos, 6)] + [(i, odd(p), 8) for i, p in (
            (1, xq), (2, xk), (3, wq), (4, wk), (6, fr), (7, pos), (9, q), (10, k))])
    bwd = [ctypes.byref(s), xq, xk, wq, wk, 1e-5, fr, pos, 1.0, dq, dk, dxq, dxk, dwq, dwk, scr, sb, None]
    refused(L.lib.lasp_qk_bwd, bwd, [
        (0, None, 1), (1, None, 1), (2, None, 1), (9, None, 1), (10, None, 1), (11, None, 1), (12, None, 1), (15, None, 5), (16, sb - 1, 5), (11, xq, 6),
        (12, dxq, 6), (12, dk, 6), (13, wq, 6), (14, dwq, 6), (15, dxk, 6), (11, odd(dxq), 8), (14, odd(dwk), 8), (5, inf, 2)])
    # gradients of queries and keys in one projection's rows: side by side, but not sharing elements
    base = fake(20).value
    at = lambda e: ctypes.c_void_p(base + 2 * e)   # noqa: E731
    for a, b, status in ((0, 504, 6), (128, 0, 6), (0, 776, 6)):   # (the last across a row's end)
        args = list(bwd)
        args[11], args[12] = at(a), at(b)
        assert L.lib.lasp_qk_bwd(*args) == status, (a, b)


def test_qk_binding_refuses_tensors_that_do_not_fit(L):
    s = L.make_qk_shape(2, 3, 2, 1, 32, torch.float32, rot=32)
    t = lambda *size, dt=torch.float32: torch.zeros(size, dtype=dt)   # noqa: E731
    f = torch.zeros(16, dtype=torch.float64)
    ok = [t(2, 3, 64), t(2, 3, 32), None, None, 1e-5, f, None, 1.0, t(2, 2, 3, 32), t(2, 1, 3, 32)]
    with pytest.raises(ValueError, match="GPU"):
        L.lasp_qk_fwd(s, *ok)
    for i, bad in ((0, t(2, 3, 32)), (1, t(2, 3, 64)), (1, t(2, 3, 64)[..., :32]), (2, t(64)), (5, f.float()), (5, f[:8]), (6, t(2, 3)), (8, t(2, 3, 32)),
                   (9, t(2, 2, 3, 32))):
        a = list(ok)
        a[i] = bad
        with pytest.raises(ValueError):
            L.lasp_qk_fwd(s, *a)


def test_frequencies(L):
    i = np.arange(32)
    plain = 10000.0 ** (-2.0 * i / 64)
    get = lambda *a, **k: L.rope_frequencies(*a, device="cpu", **k).numpy()   # noqa: E731
    assert np.allclose(get(64), plain, rtol=1e-14)
    assert np.allclose(get(64, scaling="linear", factor=4), plain / 4, rtol=1e-14)
    base = get(64, scaling="base", factor=4)
    assert base[0] == 1.0 and math.isclose(base[-1], plain[-1] / 4, rel_tol=1e-13)
    assert np.allclose(base, (10000.0 * 4 ** (64 / 62)) ** (-2.0 * i / 64), rtol=1e-13)
    bands = get(64, scaling="bands", factor=4, trained=4096, few_turns=1, many_turns=32)
    turns = 4096 * plain / (2 * math.pi)
    assert np.allclose(bands[turns >= 32], plain[turns >= 32], rtol=1e-14) and np.allclose(bands[turns <= 1], plain[turns <= 1] / 4, rtol=1e-14)
    between = (turns > 1) & (turns < 32)
    keep = (turns[between] - 1) / 31
    assert between.any() and np.allclose(bands[between], plain[between] * (keep + (1 - keep) / 4), rtol=1e-13)
    for bad in (dict(rot=3), dict(rot=2), dict(rot=0), dict(rot=-4), dict(base=0.0), dict(base=float("inf")), dict(scaling="x"), dict(scaling="linear", factor=0),
                dict(scaling="bands", factor=2, few_turns=32, many_turns=32), dict(scaling="bands", factor=2, trained=-1)):
        with pytest.raises(L.LaspError):
            get(**{**dict(rot=64), **bad})
