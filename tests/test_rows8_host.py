"""The host side of the group norm, 8-bit row and product calls: every refusal, strides and workspace sizes (no
kernel is launched)."""

import ctypes
import math

import pytest
import torch

from paper_1409_6070_amd import sscn

FAKE = 1 << 20  # never dereferenced: every call below fails its host checks first
INVALID, WORKSPACE = 1, 7
BIG = 1 << 40


def _far(i):
    return FAKE + (i << 32)


def _norm(**kw):
    d = dict(dtype=0, act=0, rows=12, cols=8, groups=2, batch=3, eps=1e-5, d_begin=_far(1), d_x=_far(2), x_stride=8,
             d_stats=_far(3))
    d.update(kw)
    return sscn.GroupNormCall(**d)


def _fwd(norm, y=_far(4), ys=8, ws=_far(5), nb=BIG):
    return sscn.load_library().sscn_group_norm_forward(norm, y, ys, ws, nb, None)


def _bwd(norm, dy=_far(6), ds=8, dx=_far(7), os=8, dg=_far(8), db=_far(9), ws=_far(5), nb=BIG):
    return sscn.load_library().sscn_group_norm_backward(norm, dy, ds, dx, os, dg, db, ws, nb, None)


BAD_NORM = [dict(dtype=2), dict(dtype=-1), dict(act=4), dict(act=-1), dict(rows=-1), dict(rows=1 << 31), dict(cols=0),
            dict(cols=4097, groups=1, x_stride=4097), dict(groups=0), dict(groups=3), dict(groups=-2), dict(batch=-1),
            dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(x_stride=7), dict(x_stride=-8),
            dict(d_stats=None), dict(d_begin=None, batch=5), dict(d_begin=None, batch=0)]


@pytest.mark.parametrize("bad", BAD_NORM + [dict(d_x=None), dict(d_x=None, d_codes=_far(10), d_scales=_far(11))])
def test_group_norm_forward_refuses(bad):
    assert _fwd(_norm(**bad)) == INVALID


@pytest.mark.parametrize("bad", BAD_NORM + [dict(d_x=None), dict(d_x=None, d_codes=_far(10)),
                                            dict(d_x=None, d_codes=_far(10) + 8, d_scales=_far(11)),
                                            dict(d_x=None, d_codes=_far(10), d_scales=_far(11) + 2)])
def test_group_norm_backward_refuses(bad):
    assert _bwd(_norm(**bad)) == INVALID


@pytest.mark.parametrize("batch", [(1 << 30) + 1, (1 << 31) - 1024, (1 << 31) - 1])
def test_group_norm_sample_numbers_stay_in_32_bits(batch):
    """More samples than the kernels' counters, which go on by a grid's step, can pass."""
    for backward in (0, 1):
        with pytest.raises(sscn.SSCNError):
            sscn.sscn_group_norm_workspace_bytes(1, 12, 8, 2, batch, backward)
        assert sscn.sscn_group_norm_workspace_bytes(1, 12, 8, 2, 1 << 30, backward) > 0
    assert _fwd(_norm(batch=batch)) == INVALID and _bwd(_norm(batch=batch)) == INVALID


def test_group_norm_results_and_workspace():
    n = _norm()
    assert _fwd(None) == INVALID and _bwd(None) == INVALID
    assert _fwd(n, y=None) == INVALID and _fwd(n, ys=7) == INVALID
    assert _bwd(n, dy=None) == INVALID and _bwd(n, dx=None) == INVALID and _bwd(n, ds=7) == INVALID and _bwd(n, os=7) == INVALID
    for call, backward in ((_fwd, 0), (_bwd, 1)):
        need = sscn.sscn_group_norm_workspace_bytes(0, 12, 8, 2, 3, backward)
        assert need > 0
        assert call(n, ws=None) == WORKSPACE and call(n, nb=need - 1) == WORKSPACE and call(n, ws=FAKE + 128) == WORKSPACE


def test_group_norm_arrays_that_overlap_are_refused():
    """Every array that is written against every other one; y on x and dx on dy or x in the same stride are allowed (these
    get as far as the missing workspace of the next check only where it is missing, so the check is made with one)."""
    spread = dict(y=_far(4), ws=_far(5))
    for at in (_far(1), _far(3), _far(2) + 4):  # begin, stats, x one element further
        assert _fwd(_norm(), **dict(spread, y=at)) == INVALID
    assert _fwd(_norm(), **dict(spread, y=_far(2)), ys=9) == INVALID  # x, another stride
    assert _fwd(_norm(d_gain=_far(4))) == INVALID and _fwd(_norm(d_shift=_far(4) + 256)) == INVALID
    assert _fwd(_norm(d_stats=_far(2))) == INVALID and _fwd(_norm(), ws=_far(2)) == INVALID
    x8 = dict(d_x=None, d_codes=_far(10), d_scales=_far(11))
    for kw in (dict(dx=_far(1)), dict(dx=_far(3)), dict(dx=_far(6) + 4), dict(dg=_far(9)), dict(dg=_far(6)), dict(db=_far(2)),
               dict(ws=_far(6)), dict(dx=_far(6), os=9), dict(dg=_far(3))):
        assert _bwd(_norm(), **kw) == INVALID, kw
    for kw in (dict(dx=_far(10)), dict(dx=_far(11)), dict(dg=_far(10)), dict(ws=_far(11) - 256)):
        assert _bwd(_norm(**x8), **kw) == INVALID, kw


def test_group_norm_workspace_grows():
    for backward in (0, 1):
        last = 0
        for rows in (0, 1, 31, 1000, 10 ** 4, 10 ** 5, 10 ** 5 + 1, 10 ** 6, 2 ** 31 - 1):
            n = sscn.sscn_group_norm_workspace_bytes(1, rows, 100, 10, 50, backward)
            assert n >= last
            last = n
        assert last < 1 << 26
        assert sscn.sscn_group_norm_workspace_bytes(1, 1000, 100, 10, 51, backward) > \
            sscn.sscn_group_norm_workspace_bytes(1, 1000, 100, 10, 50, backward)
    for bad in ((2, 1, 8, 2, 1, 0), (0, -1, 8, 2, 1, 0), (0, 1, 0, 1, 1, 0), (0, 1, 8, 3, 1, 0), (0, 1, 4098, 2, 1, 1),
                (0, 1, 8, 2, -1, 0)):
        with pytest.raises(sscn.SSCNError):
            sscn.sscn_group_norm_workspace_bytes(*bad)


def _rows8(rows=4, cols=50, codes=_far(1), scales=_far(2)):
    return sscn.Rows8Call(rows, cols, codes, scales)


BAD_ROWS8 = [dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=(1 << 20) + 1), dict(codes=None), dict(scales=None),
             dict(codes=_far(1) + 8), dict(scales=_far(2) + 2)]


@pytest.mark.parametrize("bad", BAD_ROWS8)
def test_rows8_refuses(bad):
    lib = sscn.load_library()
    r = _rows8(**bad)
    assert lib.sscn_rows8_store(0, _far(3), 1 << 21, r, None) == INVALID
    assert lib.sscn_rows8_load(0, r, _far(3), 1 << 21, None) == INVALID
    good = _rows8(4, 30, _far(5), _far(6))
    assert lib.sscn_product8_weight_grad(r, good, _far(7), 30, None, _far(8), BIG, None) == INVALID
    assert lib.sscn_product8_weight_grad(good, r, _far(7), 1 << 21, None, _far(8), BIG, None) == INVALID
    assert lib.sscn_product8_forward(0, r, _far(9), BIG, 30, None, _far(7), 30, None) == INVALID
    assert lib.sscn_product8_input_grad(0, r, _far(9), BIG, 30, _far(7), 30, None) == INVALID


def test_rows8_store_and_load_refuse():
    lib = sscn.load_library()
    r = _rows8()
    for args in ((2, _far(3), 50, r), (-1, _far(3), 50, r), (0, None, 50, r), (0, _far(3), 49, r), (0, _far(3), 50, None),
                 (0, _far(1), 50, r), (0, _far(2), 50, r), (1, _far(1) - 299, 50, r)):
        assert lib.sscn_rows8_store(*args, None) == INVALID, args
    for args in ((2, r, _far(3), 50), (0, None, _far(3), 50), (0, r, None, 50), (0, r, _far(3), 49), (0, r, _far(1), 50),
                 (0, r, _far(2) + 15, 50)):
        assert lib.sscn_rows8_load(*args, None) == INVALID, args
    assert lib.sscn_rows8_store(0, None, 50, _rows8(rows=0, codes=None, scales=None), None) == 0


def test_rows8_strides():
    for cols, want in ((1, (16, 4)), (16, (16, 4)), (17, (32, 4)), (128, (128, 4)), (129, (144, 4)), (512, (512, 4)),
                       (513, (528, 8)), (1 << 20, (1 << 20, 1 << 13))):
        assert sscn.sscn_rows8_strides(cols) == want
    for bad in (0, -1, (1 << 20) + 1):
        with pytest.raises(sscn.SSCNError):
            sscn.sscn_rows8_strides(bad)
    assert sscn.load_library().sscn_rows8_strides(5, None, None) == INVALID


def test_weight8_refuses():
    lib = sscn.load_library()
    need = sscn.sscn_weight8_bytes(50, 30)
    store = lambda dtype=0, w=_far(1), stride=30, k=50, n=30, w8=_far(2), nb=need: lib.sscn_weight8_store(  # noqa: E731
        dtype, w, stride, k, n, w8, nb, None)
    for kw in (dict(dtype=2), dict(w=None), dict(stride=29), dict(k=0), dict(n=0), dict(k=65537), dict(n=65537, stride=65537),
               dict(w=_far(2)), dict(w=_far(2) + need - 1)):
        assert store(**kw) == INVALID, kw
    for kw in (dict(w8=None), dict(nb=need - 1), dict(w8=_far(2) + 64)):
        assert store(**kw) == WORKSPACE, kw
    for bad in ((0, 1), (1, 0), (-1, 5), (65537, 1), (1, 65537)):
        with pytest.raises(sscn.SSCNError):
            sscn.sscn_weight8_bytes(*bad)
    assert lib.sscn_weight8_bytes(1, 1, None) == INVALID


def test_products_refuse():
    lib = sscn.load_library()
    need = sscn.sscn_weight8_bytes(50, 30)
    fwd = lambda dtype=0, x=_rows8(), w8=_far(3), nb=need, n=30, bias=_far(4), y=_far(5), ys=30: lib.sscn_product8_forward(  # noqa: E731
        dtype, x, w8, nb, n, bias, y, ys, None)
    for kw in (dict(dtype=2), dict(x=None), dict(n=0), dict(n=65537, ys=65537), dict(y=None), dict(ys=29), dict(y=_far(1)),
               dict(y=_far(2)), dict(y=_far(3)), dict(y=_far(4)), dict(x=_rows8(cols=65537))):
        assert fwd(**dict(dict(nb=BIG), **kw)) == INVALID, kw
    for kw in (dict(w8=None), dict(nb=need - 1), dict(w8=_far(3) + 16)):
        assert fwd(**kw) == WORKSPACE, kw
    dx = lambda dtype=0, dy=_rows8(cols=30), w8=_far(3), nb=need, k=50, y=_far(5), ys=50: lib.sscn_product8_input_grad(  # noqa: E731
        dtype, dy, w8, nb, k, y, ys, None)
    for kw in (dict(dtype=2), dict(dy=None), dict(k=0), dict(y=None), dict(ys=49), dict(y=_far(1)), dict(y=_far(3))):
        assert dx(**kw) == INVALID, kw
    assert dx(nb=need - 1) == WORKSPACE
    dw = lambda x=_rows8(1000), dy=_rows8(1000, 30, _far(3), _far(4)), out=_far(5), s=30, db=_far(6), ws=_far(7), nb=BIG: (  # noqa: E731
        lib.sscn_product8_weight_grad(x, dy, out, s, db, ws, nb, None))
    for kw in (dict(x=None), dict(dy=None), dict(dy=_rows8(999, 30, _far(3), _far(4))), dict(out=None), dict(s=29),
               dict(out=_far(1)), dict(out=_far(4)), dict(db=_far(5)), dict(db=_far(3)), dict(ws=_far(5)), dict(ws=_far(2))):
        assert dw(**kw) == INVALID, kw
    need = sscn.sscn_product8_weight_grad_workspace_bytes(1000, 50, 30)
    assert need > 0
    for kw in (dict(ws=None), dict(nb=need - 1), dict(ws=_far(7) + 8)):
        assert dw(**kw) == WORKSPACE, kw


def test_weight_grad_workspace_grows():
    for k, n in ((1, 1), (300, 3755), (4096, 4096), (65536, 65536)):
        last = 0
        for rows in (0, 1, 63, 64, 1000, 5000, 10 ** 5, 2 ** 31 - 1):
            b = sscn.sscn_product8_weight_grad_workspace_bytes(rows, k, n)
            assert b >= last
            last = b
        assert last <= 1 << 27
    for bad in ((-1, 1, 1), (1 << 31, 1, 1), (1, 0, 1), (1, 1, 65537)):
        with pytest.raises(sscn.SSCNError):
            sscn.sscn_product8_weight_grad_workspace_bytes(*bad)


def test_structures_match_the_header():
    """Field offsets as the C compiler lays them out."""
    c = sscn.GroupNormCall
    assert [getattr(c, f).offset for f, _ in c._fields_] == [0, 4, 8, 16, 20, 24, 28, 32, 40, 48, 56, 64, 72, 80, 88]
    assert ctypes.sizeof(c) == 96
    r = sscn.Rows8Call
    assert [getattr(r, f).offset for f, _ in r._fields_] == [0, 8, 16, 24] and ctypes.sizeof(r) == 32


@pytest.mark.parametrize("device", ["cpu", "cpu:0"])
def test_classes_refuse_the_host(device):
    from paper_1409_6070_amd.sscn import GroupNorm, Product8, Rows8
    codes, scales = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8)
    for make in (lambda: Rows8(4, 50, device), lambda: Rows8(4, 50, codes=codes, scales=scales),
                 lambda: GroupNorm(10, 2, 4, 1, device=device), lambda: Product8(10, 2, 4, device=device)):
        with pytest.raises(ValueError):
            make()
