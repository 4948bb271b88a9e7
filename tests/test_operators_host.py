"""The host side of the layer norm, orthogonalisation and Muon calls: every refusal, and the workspace sizes
(no kernel is launched)."""

import ctypes
import math

import pytest

from paper_1409_6070_amd import sscn

FAKE = 1 << 20  # never dereferenced: every call below fails its host checks first
COEF = (ctypes.c_float * 15)(*(sscn.MUON_COEF * 5))
INVALID, BAD_STATE, WORKSPACE = 1, 5, 7


def _fwd(dtype=0, x=FAKE, xs=8, rows=4, cols=8, eps=1e-5, y=FAKE, ys=8):
    return sscn.load_library().sscn_layer_norm_forward(dtype, x, xs, rows, cols, None, None, eps, y, ys, None)


def _bwd(dtype=0, dy=FAKE, ds=8, x=FAKE, xs=8, rows=4, cols=8, eps=1e-5, dx=FAKE, os=8, dg=FAKE, ws=FAKE, nb=1 << 20):
    return sscn.load_library().sscn_layer_norm_backward(dtype, dy, ds, x, xs, rows, cols, None, eps, dx, os, dg, None,
                                                        ws, nb, None)


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(dtype=-1), dict(x=None), dict(y=None), dict(rows=-1), dict(rows=1 << 31), dict(cols=0),
    dict(cols=-3), dict(cols=sscn.NORM_MAX_COLS + 1, xs=1 << 21, ys=1 << 21), dict(xs=7), dict(ys=7), dict(xs=-8),
    dict(eps=0.0), dict(eps=-1e-5), dict(eps=math.nan), dict(eps=math.inf)])
def test_norm_forward_refuses(bad):
    assert _fwd(**bad) == INVALID


def test_norm_of_no_rows_is_nothing():
    assert _fwd(rows=0, x=None, y=None) == 0


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=2), INVALID), (dict(dy=None), INVALID), (dict(x=None), INVALID), (dict(dx=None), INVALID),
    (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(ds=7), INVALID), (dict(xs=7), INVALID),
    (dict(os=7), INVALID), (dict(eps=0.0), INVALID), (dict(ws=None), WORKSPACE), (dict(nb=63), WORKSPACE),
    (dict(ws=FAKE + 128), WORKSPACE)])
def test_norm_backward_refuses(bad, status):
    assert _bwd(**bad) == status


def test_norm_workspace_holds_two_rows_per_part_and_grows():
    last = 0
    for rows in (0, 1, 31, 32, 33, 1000, 10 ** 5, 10 ** 6):
        n = sscn.sscn_layer_norm_workspace_bytes(1, rows, 100)
        assert n >= 800 and n % 800 == 0 and n >= last
        last = n
    assert sscn.sscn_layer_norm_workspace_bytes(0, 2 ** 31 - 1, sscn.NORM_MAX_COLS) <= 1 << 28
    for bad in ((2, 1, 1), (0, -1, 1), (0, 1, 0), (0, 1, sscn.NORM_MAX_COLS + 1)):
        with pytest.raises(sscn.SSCNError):
            sscn.sscn_layer_norm_workspace_bytes(*bad)


def _mats(*shapes, **kw):
    return (sscn.OrthoMatrix * max(len(shapes), 1))(*[
        sscn.OrthoMatrix(r, c, kw.get("d_in", FAKE), kw.get("si", c), kw.get("d_out", FAKE), kw.get("so", c))
        for r, c in shapes])


def _ortho(mats, n=None, dtype=0, steps=5, coef=COEF, ws=FAKE, nb=1 << 40):
    return sscn.load_library().sscn_orthogonalize(dtype, len(mats) if n is None else n, mats, steps, coef, ws, nb, None)


def test_orthogonalize_refuses():
    good = _mats((5, 7), (9, 3))
    need = sscn.sscn_orthogonalize_workspace_bytes(good)
    assert need > 0
    assert _ortho(good, dtype=2) == INVALID
    assert _ortho(good, n=-1) == INVALID
    assert _ortho(None, n=1) == INVALID
    assert _ortho(good, steps=0) == INVALID
    assert _ortho(good, steps=33, coef=(ctypes.c_float * 99)(*([1.5, -0.5, 0.0] * 33))) == INVALID
    assert _ortho(good, coef=None) == INVALID
    assert _ortho(good, ws=None) == WORKSPACE
    assert _ortho(good, nb=need - 1) == WORKSPACE
    assert _ortho(good, ws=FAKE + 64) == WORKSPACE
    for shape in ((0, 4), (4, 0), (-1, 4), (16385, 16385), (1, (1 << 20) + 1), ((1 << 20) + 1, 1)):
        assert _ortho(_mats(shape)) == INVALID, shape
    for kw in (dict(d_in=None), dict(d_out=None), dict(si=6), dict(so=6), dict(si=-7)):
        assert _ortho(_mats((5, 7), **kw)) == INVALID, kw
    assert _ortho(good, n=0, ws=None, nb=0) == 0  # nothing to do


@pytest.mark.parametrize("row,ok", [
    ((3.4445, -4.7750, 2.0315), True), ((1.5, -0.5, 0.0), True), ((1.0, 0.0, 0.0), True), ((15 / 8, -10 / 8, 3 / 8), True),
    ((3.6, 0.0, 0.0), False),        # singular values up to 3.6
    ((1.0, 3.0, 0.0), False),        # 1 + 3
    ((0.0, 250.0, -250.0), False),   # b s^2 + c s^4 stays below 200, the singular value does not
    ((20.0, -75.0, 55.5), False),    # zero at the end of the range, 2.7 .. inside it
    ((math.nan, 0.0, 0.0), False), ((1.0, math.inf, 0.0), False)])
def test_coefficients_are_followed_over_the_whole_range(row, ok):
    """The largest |p(s)| of each step over [0, hi], against a dense scan here."""
    coef = (ctypes.c_float * 3)(*row)
    want = WORKSPACE if ok else INVALID  # good coefficients get as far as the missing workspace
    assert _ortho(_mats((5, 7)), steps=1, coef=coef, ws=None) == want
    if all(math.isfinite(v) for v in row):
        a, b, c = list(coef)
        s = [i / 20000 for i in range(20001)]
        worst = max(abs(a * x + b * x ** 3 + c * x ** 5) for x in s)
        assert ok == (worst <= 3.5 and max(abs(b * x ** 2 + c * x ** 4) for x in s) <= 200)


def test_coefficients_are_followed_through_the_steps():
    grow = (1.5, 0.0, 0.0)  # 1.5^3 < 3.5 < 1.5^4
    for steps, ok in ((3, True), (4, False)):
        coef = (ctypes.c_float * (3 * steps))(*(grow * steps))
        assert _ortho(_mats((5, 7)), steps=steps, coef=coef, ws=None) == (WORKSPACE if ok else INVALID)


def _param(rows=6, cols=4, orthogonal=1, w=FAKE, g=FAKE, v=FAKE, lr=0.1, wd=0.0, scale=1.0):
    return sscn.MuonParam(rows, cols, w, None, g, v, lr, wd, scale, orthogonal)


def _update(*params, n=None, dtype=0, momentum=0.9, steps=5, coef=COEF, ws=FAKE, nb=1 << 40):
    arr = (sscn.MuonParam * max(len(params), 1))(*params)
    return sscn.load_library().sscn_muon_update(dtype, len(params) if n is None else n, arr, momentum, 1, steps, coef, ws,
                                                nb, None)


def test_muon_update_refuses():
    for kw in (dict(w=None), dict(g=None), dict(v=None), dict(lr=-0.1), dict(lr=math.nan), dict(wd=-1.0),
               dict(wd=math.inf), dict(scale=math.nan), dict(rows=0), dict(cols=0), dict(rows=16385, cols=16385),
               dict(rows=-1, orthogonal=0), dict(cols=1 << 31, orthogonal=0)):
        assert _update(_param(**kw)) == INVALID, kw
    for kw in (dict(dtype=2), dict(momentum=-0.1), dict(momentum=math.nan), dict(steps=0), dict(coef=None), dict(n=-1)):
        assert _update(_param(), **kw) == INVALID, kw
    need = sscn.sscn_muon_workspace_bytes((sscn.MuonParam * 1)(_param()))
    assert _update(_param(), nb=need - 1) == WORKSPACE
    assert _update(_param(), ws=None) == WORKSPACE
    assert _update(_param(), ws=FAKE + 8) == WORKSPACE
    assert _update(n=0, ws=None, nb=0, steps=0, coef=None) == 0


def test_muon_workspace_covers_its_largest_group():
    """Matrices go 24 at a time, vectors need none, a permutation of equal matrices changes nothing."""
    def need(*params):
        return sscn.sscn_muon_workspace_bytes((sscn.MuonParam * len(params))(*params))

    one, vec = _param(64, 32), _param(1, 500, 0)
    assert need(vec, vec) == 0
    assert need(one, vec) == need(one)
    assert need(*([one] * 24)) == need(*([one] * 25)) == need(*([one] * 70))
    assert need(one) < need(*([one] * 24)) <= 24 * need(one)  # a group shares its counters
    mats = _mats(*([(64, 32)] * 30))
    assert sscn.sscn_orthogonalize_workspace_bytes(mats) == need(*([one] * 30))


def test_net_calls_refuse():
    lib = sscn.load_library()
    h = sscn.sscn_net_create(sscn.NetDesc(2, 3, 9, 4, 4, 100, sscn.SSCN_BF16))
    try:
        opt = sscn.MuonOptions(0.1, 0.1, 0.9, 0.0, 1, 0, 5, ctypes.addressof(COEF))
        need = sscn.sscn_net_muon_workspace_bytes(h, opt)
        assert need > 0
        opt.softmax = 1
        assert sscn.sscn_net_muon_workspace_bytes(h, opt) > need
        ptrs = (ctypes.c_void_p * 4)(*([FAKE] * 4))
        args = [h, ptrs, ptrs, ptrs, ptrs, ptrs, ctypes.byref(opt), FAKE, 1 << 40, None]
        assert lib.sscn_muon_step(*args) == BAD_STATE  # no backward yet
        for i in (0, 1, 3, 4, 5, 6):
            assert lib.sscn_muon_step(*args[:i], None, *args[i + 1:]) == INVALID, i
        for field in ("lr", "lr_rest", "momentum", "weight_decay"):
            for bad in (-1.0, math.nan, math.inf):
                keep = getattr(opt, field)
                setattr(opt, field, bad)
                assert lib.sscn_muon_step(*args) == INVALID, field
                setattr(opt, field, keep)
        n = sscn.sscn_head_norm_workspace_bytes(h)
        assert n >= 4 * 3 * 9  # batch_max rows of the top layer's nine channels
        good = [h, FAKE, FAKE, FAKE, FAKE, 1e-5, FAKE, n]
        for i in (1, 2, 3, 4):
            assert lib.sscn_set_head_norm(*good[:i], None, *good[i + 1:]) == INVALID
        for eps in (0.0, -1.0, math.nan, math.inf):
            assert lib.sscn_set_head_norm(*good[:5], eps, FAKE, n) == INVALID
        assert lib.sscn_set_head_norm(*good[:6], None, n) == WORKSPACE
        assert lib.sscn_set_head_norm(*good[:6], FAKE, n - 1) == WORKSPACE
        assert lib.sscn_set_head_norm(*good[:6], FAKE + 4, n) == WORKSPACE
        assert lib.sscn_set_head_norm(None, *good[1:]) == INVALID
        assert lib.sscn_set_head_norm(*good) == 0
        assert lib.sscn_set_head_norm(h, None, None, None, None, 0.0, None, 0) == 0
    finally:
        sscn.sscn_net_destroy(h)


def _dense(rows):
    """(largest singular value after a step, largest |b s^2 + c s^4|) over the steps, on a dense scan of [0, hi]."""
    hi, most, inner = 1.0, 0.0, 0.0
    for a, b, c in rows:
        s = [hi * i / 20000 for i in range(20001)]
        inner = max(inner, max(abs(b * x ** 2 + c * x ** 4) for x in s))
        hi = max(abs(a * x + b * x ** 3 + c * x ** 5) for x in s)
        most = max(most, hi)
    return most, inner


@pytest.mark.parametrize("rows", [
    [(100.0, -100.0, 1e-20)], [(100.0, -100.0, 1e-14)], [(10.0, -10.0, 1e-18)], [(9.5, -9.5, 1e-17)], [(9.5, -9.5, -1e-17)],
    [(9.0, -9.0, 1e-17)], [(9.0, -9.0, -1e-17)], [(9.0, -9.0, 1e-30)],
    [(100.0, -100.0, 1e-20), (1.0, 0.0, 0.0)], [(1.0, 0.0, 0.0), (100.0, -100.0, 1e-20)],
    [(9.0, -9.0, 1e-17), (1.05, 0.0, 0.0)], [(9.0, -9.0, 1e-17), (1.0, 0.0, 0.0)],
    [(-100.0, 100.0, 1e-20)], [(1e-20, -3.0, 1e-20)], [(0.0, 0.0, 1e-20)], [(0.0, 0.0, 0.0), (2.0, 0.0, 0.0)]], ids=str)
def test_an_extremum_inside_the_range_is_found_for_any_coefficients(rows):
    """A fifth-power coefficient too small to matter must not hide where the cubic turns."""
    coef = (ctypes.c_float * (3 * len(rows)))(*[x for r in rows for x in r])
    most, inner = _dense([list(coef)[3 * k: 3 * k + 3] for k in range(len(rows))])
    want = WORKSPACE if most <= 3.5 and inner <= 200 else INVALID
    assert _ortho(_mats((5, 7)), steps=len(rows), coef=coef, ws=None) == want


def test_arrays_past_the_address_space_are_refused():
    """2^31 rows 2^31 elements apart: byte offsets would pass 63 bits."""
    top, far = (1 << 31) - 1, 1 << 31
    assert _fwd(rows=top, xs=far) == INVALID and _fwd(rows=top, ys=far) == INVALID
    for kw in (dict(ds=far), dict(xs=far), dict(os=far)):
        assert _bwd(rows=top, nb=0, **kw) == INVALID, kw  # (fewer bytes than any workspace: nothing is launched)
        assert _bwd(rows=1 << 28, nb=0, **kw) == WORKSPACE, kw  # 2^61 bytes
    assert _update(_param(top, top, 0)) == INVALID


def _apart(n, rows=6, cols=4):
    """n parameters whose masters, gradients and velocities are all apart (addresses that nothing reads)."""
    at = iter(range(FAKE, FAKE + 4096 * 4 * n, 4096))
    return [_param(rows, cols, i % 2, next(at), next(at), next(at)) for i in range(n)]


@pytest.mark.parametrize("n", [2, 3, 40])
def test_muon_update_refuses_arrays_that_overlap(n):
    """One velocity or copy for two parameters, a gradient that is also a velocity, ...: two sets of workgroups would
    write, or read and write, the same memory.  (Refused before anything is launched.)"""
    ws = FAKE + (1 << 24)
    size = 6 * 4 * 4
    for i, j in ((0, 1), (0, n - 1), (n - 1, 0)):
        for x in ("d_w", "d_v", "d_w_store"):
            for y in ("d_w", "d_v", "d_g", "d_w_store"):
                for off in (0, size - 4, 4 - size):  # the same array, its last and first element
                    p = _apart(n)
                    for q in p:
                        q.d_w_store = q.d_w + 2048
                    setattr(p[i], x, getattr(p[j], y) + off)
                    assert _update(*p, ws=ws) == INVALID, (i, j, x, y, off)
    for x, y in (("d_w", "d_v"), ("d_w", "d_g"), ("d_v", "d_g"), ("d_w_store", "d_v"), ("d_w_store", "d_g")):
        p = _apart(n)
        setattr(p[0], x, getattr(p[0], y))
        assert _update(*p, ws=ws) == INVALID, (x, y)
    p = _apart(n)
    p[0].d_w_store = p[0].d_w + 4  # not the master itself, which means no copy
    assert _update(*p, ws=ws) == INVALID
    for name in ("d_w", "d_g", "d_v"):
        p = _apart(n)
        assert _update(*p, ws=(getattr(p[0], name) - 512) // 256 * 256) == INVALID  # in the workspace


def test_orthogonalize_refuses_outputs_that_overlap():
    """Views of one buffer whose rows share elements."""
    def call(*mats, ws=FAKE + (1 << 24), nb=1 << 40, dtype=0):
        arr = (sscn.OrthoMatrix * len(mats))(*[sscn.OrthoMatrix(r, c, i, si, o, so) for r, c, i, si, o, so in mats])
        return _ortho(arr, ws=ws, nb=nb, dtype=dtype)

    A, B, C, D = (FAKE + 65536 * k for k in range(4))
    for dtype, e in ((0, 4), (1, 2)):
        one = lambda i, o, si=16, so=16: (8, 16, i, si, o, so)  # noqa: E731
        for bad in ([one(A, C), one(B, C)],                       # an output twice
                    [one(A, C), one(B, C + 7 * 16 * e + 15 * e)],  # its last element
                    [one(A, B), one(B, A)], [one(A, C), one(C, D)],  # another's input
                    [one(A, A), one(A, B)],                       # in place, and read by another
                    [one(A, A + 4 * 16 * e)],                     # its own input, rows further on
                    [one(A, A, 16, 20)], [one(A, A, 20, 16)],     # its own input in other strides
                    [one(A, C, 40, 40), one(B, C + 15 * e, 40, 40)],  # columns that share one
                    [one(A, C, 40, 40), one(B, C + 30 * e, 40, 40)],  # that wrap into the next row
                    [one(A, C), (1, 5, B, 5, C + 100 * e, 5)]):
            assert call(*bad, dtype=dtype) == INVALID, bad
        ws = FAKE + (1 << 24)
        assert call(one(A, ws), dtype=dtype) == INVALID and call(one(ws + 256, A), dtype=dtype) == INVALID


def test_norm_refuses_outputs_that_overlap():
    """Other than x's (dy's) own array with the same stride; gain, shift, the parameters' gradients and the workspace."""
    lib = sscn.load_library()
    A, B, C, D, G, S = (FAKE + 65536 * k for k in range(6))
    for dtype, e in ((0, 4), (1, 2)):
        def fwd(x=A, xs=16, y=B, ys=16, gain=G, shift=S):
            return lib.sscn_layer_norm_forward(dtype, x, xs, 8, 16, gain, shift, 1e-5, y, ys, None)
        for bad in (dict(y=A, ys=20), dict(y=A, xs=20), dict(y=A + e), dict(y=A + 16 * e), dict(y=A - 7 * 16 * e),
                    dict(y=A + 15 * e, xs=40, ys=40), dict(y=A + 30 * e, xs=40, ys=40), dict(y=G), dict(y=S), dict(y=G + 60),
                    dict(y=S - 7 * 16 * e)):
            assert fwd(**bad) == INVALID, bad
        need = sscn.sscn_layer_norm_workspace_bytes(dtype, 8, 16)
        W = FAKE + (1 << 20)

        def bwd(dy=A, ds=16, x=B, xs=16, dx=C, os=16, gain=G, dg=D, dh=D + 64, ws=W):
            return lib.sscn_layer_norm_backward(dtype, dy, ds, x, xs, 8, 16, gain, 1e-5, dx, os, dg, dh, ws, need, None)
        for bad in (dict(dx=A, os=20), dict(dx=B, os=20), dict(dx=A, ds=20), dict(dx=A + e), dict(dx=B - e), dict(dx=G),
                    dict(dx=D), dict(dx=W), dict(dh=D), dict(dh=D + 60), dict(dg=G), dict(dg=A), dict(dg=B), dict(dh=W + need - 4),
                    dict(ws=A), dict(ws=C), dict(ws=G), dict(gain=W), dict(gain=C + 8)):
            assert bwd(**bad) == INVALID, bad


def test_muon_step_wrapper_wants_every_array():
    """A list that is too short, or an array that is too small or lies elsewhere, would be read where nothing is."""
    import torch
    net = sscn.SparseDeepCNet(2, 3, 9, 4, 4, 100, "bf16", device="cpu")  # (buffers only: nothing runs)
    W32 = [torch.zeros(s) for s in net.param_shapes]
    W = [w.bfloat16() for w in W32]
    b = [torch.zeros(s[1]) for s in net.param_shapes]
    good = [W32, W, b, [w.clone() for w in W32], [v.clone() for v in b]]
    for i in range(5):
        for bad in (good[i][:-1], good[i] + good[i][:1], good[i][:-1] + [good[i][-1][:-1]], good[i][::-1],
                    good[i][:-1] + [good[i][-1].to("meta")]):  # (of another device)
            with pytest.raises(ValueError):
                net.muon_step(*good[:i], bad, *good[i + 1:], 0.1, 0.1)
