"""Host-side checks of the gated recurrence and of the norms around a mixer that need no GPU: shapes, sizes and the refusals of
bad arguments before any launch (no compute call is made here)."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def L():
    from paper_2404_02882_amd import lasp
    return lasp


def fake(n):
    """Distinct non-null addresses that are never dereferenced (validation fails first)."""
    return ctypes.c_void_p(0x10000000 + n * 0x10000000)


@pytest.mark.parametrize("kw,expect", [
    (dict(), 0), (dict(B=1, N=1, D=8), 0), (dict(D=12), 2), (dict(D=0), 2), (dict(D=-8), 2), (dict(N=0), 2), (dict(B=0), 2),
    (dict(ld=128), 0), (dict(ld=64), 0), (dict(ld=56), 2), (dict(ld=68), 2), (dict(ld=-64), 2), (dict(dtype=2), 3), (dict(dtype=-1), 3),
    (dict(B=1 << 16, N=1 << 16), 2), (dict(B=1 << 20, N=1, D=1 << 12), 2), (dict(coupled=True), 0),
])
def test_recurrence_shapes(L, kw, expect):
    s = L.make_rec_shape(**{**dict(B=2, N=100, D=64, dtype=1), **kw})
    assert L.check_rec(s) == expect
    assert (L.rec_scratch_bytes(s) > 0) == (expect == 0)


@pytest.mark.parametrize("kw,expect", [
    (dict(), 0), (dict(rows=1, C=8), 0), (dict(C=16384), 0), (dict(C=16392), 2), (dict(C=20), 2), (dict(C=0), 2), (dict(rows=0), 2),
    (dict(dtype=5), 3),
])
def test_row_shapes(L, kw, expect):
    s = L.make_rows(**{**dict(rows=10, C=64, dtype=0), **kw})
    assert L.check_rows(s) == expect
    assert (L.addnorm_scratch_bytes(s) > 0) == (expect == 0)


@pytest.mark.parametrize("kw,expect", [
    (dict(), 0), (dict(gate="none"), 0), (dict(gate="relu"), 2), (dict(over="batch"), 2), (dict(D=20), 2), (dict(H=0), 2),
    (dict(H=256, D=64), 0), (dict(H=256, D=72), 2), (dict(N=0), 2), (dict(ld=256), 0), (dict(ld=248), 2), (dict(ld=260), 2),
    (dict(dtype=2), 3), (dict(B=1 << 15, N=1 << 15, H=4), 2), (dict(over="token"), 0),
])
def test_gate_shapes(L, kw, expect):
    s = L.make_gate_shape(**{**dict(B=2, H=4, N=10, D=64, dtype=1), **kw})
    assert L.check_gate(s) == expect
    assert (L.gatenorm_scratch_bytes(s) > 0) == (expect == 0)


def refused(fn, args, changes):
    for i, value, status in changes:
        a = list(args)
        a[i] = value
        assert fn(*a) == status, (i, value)


def test_recurrence_rejects_before_launch(L):
    s = L.make_rec_shape(2, 100, 64, "bf16")
    sb = L.rec_scratch_bytes(s)
    x, la, hin, lens, out, hout, scr, dout, dhout, dx, dl, dhin = [fake(i) for i in range(1, 13)]
    odd = lambda p: ctypes.c_void_p(p.value + 8)   # noqa: E731
    fwd = [ctypes.byref(s), x, la, hin, lens, out, hout, scr, sb, None]
    refused(L.lib.lasp_rec_fwd, fwd, [
        (0, None, 1), (1, None, 1), (2, None, 1), (5, None, 1), (7, None, 5), (8, sb - 1, 5),
        (5, x, 6), (5, la, 6), (6, out, 6), (7, x, 6), (6, ctypes.c_void_p(hin.value + 16), 6), (5, lens, 6), (7, hin, 6),
        (1, odd(x), 8), (2, odd(la), 8), (3, odd(hin), 8), (4, odd(lens), 8), (5, odd(out), 8), (6, odd(hout), 8), (7, odd(scr), 8)])
    bwd = [ctypes.byref(s), None, la, out, hin, lens, dout, dhout, dx, dl, dhin, scr, sb, None]
    refused(L.lib.lasp_rec_bwd, bwd, [
        (0, None, 1), (2, None, 1), (3, None, 1), (6, None, 1), (8, None, 1), (9, None, 1), (11, None, 5), (12, 0, 5),
        (8, la, 6), (8, out, 6), (9, dx, 6), (9, dout, 6), (10, hin, 6), (10, ctypes.c_void_p(dhout.value + 32), 6), (11, dx, 6), (8, odd(dx), 8),
        (10, odd(dhin), 8)])
    c = L.make_rec_shape(2, 100, 64, "bf16", coupled=True)
    assert L.lib.lasp_rec_bwd(*([ctypes.byref(c)] + bwd[1:])) == 1      # x is read then
    refused(L.lib.lasp_rec_bwd, [ctypes.byref(c), x] + bwd[2:], [(8, x, 6)])
    bad = L.make_rec_shape(2, 100, 60, "bf16")
    assert L.lib.lasp_rec_fwd(*([ctypes.byref(bad)] + fwd[1:])) == 2
    bad = L.make_rec_shape(2, 100, 64, 9)
    assert L.lib.lasp_rec_bwd(*([ctypes.byref(bad)] + bwd[1:])) == 3


def test_rows_that_share_elements_are_refused(L):
    """Rows 160 elements apart hold two halves of 64 (which the GPU tests run); halves that share elements are refused, also
    across the row's end, and so are halves of contiguous rows."""
    s = L.make_rec_shape(2, 100, 64, "bf16", ld=160)
    tight = L.make_rec_shape(2, 100, 64, "bf16")
    la, out, dout, scr, base = fake(1), fake(2), fake(3), fake(4), fake(5).value
    at = lambda elements: ctypes.c_void_p(base + 2 * elements)   # noqa: E731
    for shape, dx, dl in [(tight, 0, 64), (tight, 64, 0)] + [(s, *p) for p in ((0, 56), (56, 0), (0, 0), (104, 160), (0, 104))]:
        assert L.lib.lasp_rec_bwd(ctypes.byref(shape), None, la, out, None, None, dout, None, at(dx), at(dl), None, scr,
                                  L.rec_scratch_bytes(shape), None) == 6, (dx, dl)


def test_addnorm_rejects_before_launch(L):
    s = L.make_rows(10, 64, "f32")
    sb = L.addnorm_scratch_bytes(s)
    r, x, sc, w, ro, y, dy, dro, dr, dx, dw, ds, scr = [fake(i) for i in range(1, 14)]
    odd = lambda p: ctypes.c_void_p(p.value + 4)   # noqa: E731
    fwd = [ctypes.byref(s), r, x, sc, w, 1e-5, ro, y, None]
    nan = float("nan")
    refused(L.lib.lasp_addnorm_fwd, fwd, [
        (0, None, 1), (1, None, 1), (6, None, 1), (7, None, 1), (2, None, 1),        # (a sum's buffer or scale without what is added)
        (5, -1e-5, 2), (5, nan, 2), (5, float("inf"), 2),
        (6, x, 6), (7, r, 6), (7, ro, 6), (7, w, 6), (6, ctypes.c_void_p(r.value + 256), 6),
        (1, odd(r), 8), (2, odd(x), 8), (3, odd(sc), 8), (4, odd(w), 8), (6, odd(ro), 8), (7, odd(y), 8)])
    alone = [ctypes.byref(s), r, None, None, w, 1e-5, None, y, None]
    refused(L.lib.lasp_addnorm_fwd, alone, [(6, ro, 1), (3, sc, 1), (7, r, 6)])
    bwd = [ctypes.byref(s), ro, x, sc, w, 1e-5, dy, dro, dr, dx, dw, ds, scr, sb, None]
    refused(L.lib.lasp_addnorm_bwd, bwd, [
        (0, None, 1), (1, None, 1), (6, None, 1), (8, None, 1), (2, None, 1), (12, None, 5), (13, sb - 1, 5), (5, nan, 2),
        (8, ro, 6), (8, dy, 6), (9, dr, 6), (9, x, 6), (10, w, 6), (11, dw, 6), (12, dx, 6), (8, ctypes.c_void_p(dro.value + 16), 6),
        (10, odd(dw), 8), (12, odd(scr), 8)])
    bad = L.make_rows(10, 63, "f32")
    assert L.lib.lasp_addnorm_fwd(*([ctypes.byref(bad)] + fwd[1:])) == 2


def test_gatenorm_rejects_before_launch(L):
    s = L.make_gate_shape(2, 4, 10, 64, "bf16", ld=512)
    sb = L.gatenorm_scratch_bytes(s)
    o, u, w, y, dy, do, du, dw, scr = [fake(i) for i in range(1, 10)]
    odd = lambda p: ctypes.c_void_p(p.value + 4)   # noqa: E731
    fwd = [ctypes.byref(s), o, u, w, 1e-5, y, None]
    refused(L.lib.lasp_gatenorm_fwd, fwd, [
        (0, None, 1), (1, None, 1), (2, None, 1), (5, None, 1), (4, -1.0, 2), (5, o, 6), (5, u, 6), (5, w, 6), (1, odd(o), 8), (2, odd(u), 8),
        (3, odd(w), 8), (5, odd(y), 8)])
    bwd = [ctypes.byref(s), o, u, w, 1e-5, dy, do, du, dw, scr, sb, None]
    refused(L.lib.lasp_gatenorm_bwd, bwd, [
        (1, None, 1), (2, None, 1), (5, None, 1), (6, None, 1), (7, None, 1), (9, None, 5), (10, sb - 1, 5), (4, float("inf"), 2),
        (6, o, 6), (7, u, 6), (7, dy, 6), (8, w, 6), (9, do, 6), (7, odd(du), 8), (7, ctypes.c_void_p(u.value + 2 * 128), 6)])
    for kw in (dict(gate="tanh"), dict(over="row")):
        bad = L.make_gate_shape(2, 4, 10, 64, "bf16", **kw)
        assert L.lib.lasp_gatenorm_fwd(*([ctypes.byref(bad)] + fwd[1:])) == 2


def test_binding_refuses_tensors_that_do_not_fit(L):
    s = L.make_rec_shape(2, 3, 8, torch.float32)
    t = lambda *size, dt=torch.float32: torch.zeros(size, dtype=dt)   # noqa: E731
    scratch = torch.zeros(L.rec_scratch_bytes(s), dtype=torch.uint8)
    ok = [t(2, 3, 8), t(2, 3, 8), None, None, t(2, 3, 8), t(2, 8), scratch]
    with pytest.raises(ValueError, match="GPU"):
        L.lasp_rec_fwd(s, *ok)
    for i, bad in ((0, t(2, 3, 9)), (0, t(2, 3, 8, dt=torch.float64)), (1, t(2, 3, 16)[..., ::2]), (1, t(2, 3, 16)[..., :8]), (2, t(8)),
                   (3, t(2)), (4, t(2, 4, 8)), (5, t(2, 16)[:, :8])):
        a = list(ok)
        a[i] = bad
        with pytest.raises(ValueError):
            L.lasp_rec_fwd(s, *a)
    g = L.make_gate_shape(1, 2, 3, 8, torch.bfloat16)
    b = lambda *size: torch.zeros(size, dtype=torch.bfloat16)   # noqa: E731
    with pytest.raises(ValueError):
        L.lasp_gatenorm_fwd(g, b(1, 2, 3, 8), b(1, 3, 32)[..., 16:], None, 1e-5, b(1, 3, 16))
    r = L.make_rows(4, 16, torch.float32)
    with pytest.raises(ValueError):
        L.lasp_addnorm_fwd(r, t(4, 16), t(4, 16), t(8), None, 1e-5, t(4, 16), t(4, 16))
