"""Group norm with an activation on the GPU against its formula in 64 bits: samples of no rows, one row and many, groups
of one channel and of all, odd lengths, strides and alignments, rows outside the samples, 8-bit rows in the backward
pass, infinities and NaN; and a stage of 8-bit product, group norm and network as they are used together.

Bounds.  u = 2^-24.  A term passes at most D additions in a sum: a thread's rows of a chunk (8, or its share of
1024 chunks) or of a small sample (16 in registers), the row lanes of a workgroup (1024 at most where rows are short, and
as many in the channels of a group), the pieces of a sample by 64 lanes: D = 32 + rows / 1024 + lanes + channels +
pieces / 64, lanes <= 1024 / vectors of a row.  A sample of more than three times the mean length may be read in a loop
by one workgroup of 256 threads or more: its rows times the vectors of a row, over 256, besides.  e = D u mean|x| for the mean.  The variance sums deviations from one of a thread's own n values, whose squares sum
to at most 2 (1 + n) times those from the mean: D u (3 + 2 n) relative, and (e r)^2 for the mean's error; r half of that
plus 3 u.  The rest counts one u per operation; the result's rounding is half a step of its type.  The exponential's
argument is rounded once more and its result by 2 u: a sigmoid is off by (6 + |z|) u relative, SiLU's derivative by
(16 + 3 |z|) u absolute, and by at most half of z's own error.  Rectifiers take the branch of the float32 z, which is
followed here operation by operation."""

import numpy as np
import pytest
import torch

from tests.gpu_harness import log

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
ACTS = ["none", "relu", "leaky", "silu"]
SLOPE = {"none": 1.0, "relu": 0.0, "leaky": 1.0 / 3.0}


@pytest.fixture(autouse=True, scope="module")
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1409_6070_amd import sscn
    sscn.load_library()


def _np(t):
    return t.double().cpu().numpy()


def _depth(rows, cols, per, dtype, mean=None):
    """D, rows of a thread (mean: rows of a sample on average, where there are several)"""
    v = 8 if dtype == "bf16" else 4
    vecs = -(-cols // v)
    lanes = max(1, 1024 // vecs)
    loop = rows * 2 * vecs / 256 if mean is not None and rows > 3 * mean else 0
    return 32 + rows / 1024 + lanes + per + (rows / 8 + 2) / 64 + loop, 16 + rows / 1024


def _act(z, act):
    """(act(z), act'(z))"""
    if act == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return z * s, s * (1 + z * (1 - s))
    slope = np.where(z > 0 if act == "relu" else z >= 0, 1.0, SLOPE[act])
    return z * slope, slope


def _spans(begin, rows):
    return [(b, e) for b, e in zip(begin[:-1], begin[1:])]


def _want_forward(x, begin, gain, shift, groups, act, dtype):
    """(y, its bound, means, r, their bounds); rows outside the samples are NaN."""
    rows, cols = x.shape
    per, batch = cols // groups, len(begin) - 1
    y, tol = np.full_like(x, np.nan), np.zeros_like(x)
    means, rs, te, tr = (np.zeros((batch, groups)) for _ in range(4))
    rs[:] = EPS ** -0.5
    tr[:] = 3 * U * EPS ** -0.5
    for b, (lo, hi) in enumerate(_spans(begin, rows)):
        if lo == hi:
            continue
        p = x[lo:hi].reshape(hi - lo, groups, per)
        D, n = _depth(hi - lo, cols, per, dtype, rows / batch)
        m = p.mean((0, 2))
        d = p - m[:, None]
        r = 1.0 / np.sqrt((d * d).mean((0, 2)) + EPS)
        e = (D + 4) * U * np.abs(p).mean((0, 2))
        rel = 0.5 * ((D + 6) * U * (3 + 2 * n) + (e * r) ** 2) + 3 * U
        means[b], rs[b], te[b], tr[b] = m, r, e + U * np.abs(m), rel * r
        dh = (r * e)[:, None] + np.abs(d) * (r * (rel + 3 * U))[:, None] + 2 * U * (np.abs(p) * r[:, None])
        h, dh = (d * r[:, None]).reshape(hi - lo, cols), dh.reshape(hi - lo, cols)
        z = h * gain + shift
        dz = np.abs(gain) * dh + 3 * U * (np.abs(h * gain) + np.abs(shift))
        y[lo:hi], _ = _act(z, act)
        # (no activation is steeper than 1.1)
        tol[lo:hi] = 1.1 * dz + (np.abs(z) * (8 + np.abs(z)) * U if act == "silu" else U * np.abs(y[lo:hi]))
    tol = tol * 1.01 + HALF[dtype] * (np.nan_to_num(np.abs(y)) + tol) + 1e-38
    return y, tol, means, rs, te + 1e-38, tr


def _float_z(x, mean, r, gain, shift):
    """z and h as float32 operations leave them."""
    f = np.float32
    h = (x.astype(f) - mean.astype(f)) * r.astype(f)
    return (h * gain.astype(f)) + shift.astype(f), h


def _want_backward(dy, x, stats, begin, gain, shift, groups, act, dtype):
    rows, cols = x.shape
    per = cols // groups
    dx, tol = np.full_like(x, np.nan), np.zeros_like(x)
    dg, ds, tg, ts = (np.zeros(cols) for _ in range(4))
    D_all, _ = _depth(rows, cols, per, dtype)
    D_all += 1024 / 16 + 16
    for b, (lo, hi) in enumerate(_spans(begin, rows)):
        if lo == hi:
            continue
        m, r = (np.repeat(stats[i, b], per) for i in range(2))
        zf, _ = _float_z(x[lo:hi], m, r, gain, shift)
        h = (x[lo:hi] - m) * r
        dh = 2 * U * np.abs(h) + 1e-300
        z = h * gain + shift
        ez = np.abs(gain) * dh + 2 * U * (np.abs(h * gain) + np.abs(shift))
        slope = _act(z if act == "silu" else zf.astype(np.float64), act)[1]
        eslope = 0.5 * ez + (16 + 3 * np.abs(z)) * U if act == "silu" else U * slope
        d = dy[lo:hi]
        dz = d * slope
        edz = np.abs(d) * eslope + U * np.abs(dz)
        t, et = dz * gain, np.abs(gain) * edz + U * np.abs(dz * gain)
        D, _ = _depth(hi - lo, cols, per, dtype, rows / (len(begin) - 1))

        def mean(v):
            return np.repeat(v.sum(0).reshape(groups, per).sum(1) / ((hi - lo) * per), per)
        m1, m2 = mean(t), mean(t * h)
        em1 = mean(et) + (D + 4) * U * mean(np.abs(t))
        em2 = mean(et * np.abs(h) + np.abs(t) * dh) + (D + 5) * U * mean(np.abs(t * h))
        dx[lo:hi] = r * (t - m1 - h * m2)
        tol[lo:hi] = r * (et + em1 + np.abs(h) * em2 + dh * np.abs(m2) + 4 * U * (np.abs(t) + np.abs(m1) + np.abs(h * m2)))
        dg += (dz * h).sum(0)
        ds += dz.sum(0)
        tg += (edz * np.abs(h) + np.abs(dz) * dh).sum(0) + (D_all + 2) * U * np.abs(dz * h).sum(0)
        ts += edz.sum(0) + D_all * U * np.abs(dz).sum(0)
    tol = tol * 1.01 + HALF[dtype] * (np.nan_to_num(np.abs(dx)) + tol) + 1e-38
    return (dx, tol), (dg, tg * 1.01 + 1e-37), (ds, ts * 1.01 + 1e-37)


def _within(got, want, tol, what):
    got = _np(got)
    assert got.shape == want.shape
    live = ~np.isnan(want)
    worst = float((np.abs(got - want) / tol)[live].max()) if live.any() else 0.0
    log(f"  {what}: at most {worst:.3f} of the bound")
    assert np.isfinite(got[live]).all() and worst <= 1.0, what


def _wide(t, pad, fill=7.0):
    rows, cols = t.shape
    buf = torch.full((rows, cols + 2 * pad), fill, dtype=t.dtype, device="cuda")
    buf[:, pad: pad + cols] = t.cuda()
    return buf, buf[:, pad: pad + cols]


def _make(rows, cols, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(0.5 * torch.randn(cols, generator=g)) + torch.randn(cols, generator=g)
    dy = 0.3 * torch.randn(rows, cols, generator=g)
    gain, shift = 1 + 0.3 * torch.randn(cols, generator=g), 0.3 * torch.randn(cols, generator=g)
    return x.to(TORCH[dtype]), dy.to(TORCH[dtype]), gain, shift


def _check(rows, cols, groups, begin, dtype, act, pad=0, seed=0, x8=False, params=True):
    from paper_1409_6070_amd.sscn import GroupNorm, Rows8
    log(f"[group norm] {rows} x {cols} in {groups}, {len(begin) - 1} samples, {dtype} {act} pad {pad}{' 8 bits' if x8 else ''}")
    x, dy, gain, shift = _make(rows, cols, dtype, seed)
    plan = GroupNorm(cols, groups, rows, len(begin) - 1, dtype, act, EPS)
    b = torch.tensor(begin, dtype=torch.int32, device="cuda")
    g, s = (gain.cuda(), shift.cuda()) if params else (None, None)
    gn, sn = (gain.double().numpy(), shift.double().numpy()) if params else (np.ones(cols), np.zeros(cols))
    xd = _wide(x, pad)[1]
    out, y = _wide(torch.full_like(x, 3.0), pad)
    _, stats = plan.forward(xd, b, g, s, out=y)
    want, tol, means, rs, te, tr = _want_forward(_np(x), begin, gn, sn, groups, act, dtype)
    _within(y, want, tol, "y")
    _within(stats[0], means, te + U * np.abs(means), "mean")
    _within(stats[1], rs, tr, "r")
    outside = np.isnan(want[:, 0])
    assert (_np(y)[outside] == 3).all() and (out[:, :pad] == 7).all() and (out[:, pad + cols:] == 7).all()
    held = x
    if x8:
        held8 = Rows8(rows, cols).store(xd)
        held = held8.load("f32")
    out, dx = _wide(torch.full_like(dy, 3.0), pad + 1)
    _, dg, ds = plan.backward(_wide(dy, pad)[1], held8 if x8 else xd, stats, b, g, s, dx=dx)
    bx, bg, bs = _want_backward(_np(dy), _np(held), _np(stats), begin, gn, sn, groups, act, dtype)
    _within(dx, *bx, "dx")
    _within(dg, *bg, "dgain")
    _within(ds, *bs, "dshift")
    assert (_np(dx)[outside] == 3).all() and (out[:, :pad + 1] == 7).all() and (out[:, pad + 1 + cols:] == 7).all()


def _begins(rows, batch, seed, front=0, behind=0):
    g = np.random.default_rng(seed)
    return [front] + sorted(g.integers(front, rows - behind + 1, size=batch - 1).tolist()) + [rows - behind]


# groups of one channel, of all, of odd and even numbers; rows of less than a vector to the longest
SHAPES = [(1, 1), (2, 1), (3, 3), (5, 1), (7, 7), (8, 2), (9, 3), (10, 2), (12, 4), (20, 5), (31, 1), (33, 11), (50, 10), (64, 8),
          (100, 10), (100, 100), (129, 3), (256, 32), (300, 20), (300, 1), (512, 32), (1000, 8), (1023, 11), (2049, 3),
          (2056, 8), (4096, 32), (4095, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols,groups", SHAPES)
def test_channels_and_groups(cols, groups, dtype):
    for i, (rows, batch, pad) in enumerate(((1, 1, 0), (7, 3, 1), (90, 4, 0), (333, 2, 3))):
        _check(rows, cols, groups, _begins(rows, batch, i), dtype, ACTS[(cols + i) % 4], pad, seed=cols + i, x8=i % 2 == 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
def test_activations(act, dtype):
    for x8 in (False, True):
        _check(500, 60, 4, _begins(500, 6, 3), dtype, act, 2, x8=x8)
    _check(200, 24, 3, [0, 200], dtype, act, params=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_samples(dtype):
    """Samples without rows at either end and between, of one row, many small ones, rows before and behind them."""
    _check(40, 30, 3, [0, 0, 0, 13, 13, 14, 40, 40], dtype, "leaky")
    _check(40, 30, 3, [5, 5, 17, 33], dtype, "relu", 1, x8=True)
    _check(40, 30, 3, [40, 40], dtype, "silu")
    _check(700, 18, 2, list(range(0, 701)), dtype, "silu")        # one row each
    _check(3000, 18, 2, _begins(3000, 1500, 1, 7, 11), dtype, "leaky", x8=True)
    _check(3000, 100, 10, [0, 2990, 2991, 3000], dtype, "silu")   # very different lengths
    _check(70000, 9, 3, _begins(70000, 5, 2), dtype, "leaky")


@pytest.mark.parametrize("rows,cols,groups,batch,dtype", [(200001, 20, 2, 1, "bf16"), (60001, 100, 10, 100, "bf16"),
                                                          (20011, 300, 20, 40, "f32"), (33333, 64, 64, 3, "f32"),
                                                          (9000, 1024, 32, 9, "bf16")])
def test_many_rows(rows, cols, groups, batch, dtype):
    _check(rows, cols, groups, _begins(rows, batch, 5), dtype, "leaky", x8=batch % 2 == 1)


@pytest.mark.parametrize("rows,cols,groups,batch,dtype", [(24001, 288, 32, 60, "f32"), (24001, 288, 32, 60, "bf16"),
                                                          (1100, 3709, 3709, 8, "f32")])
def test_joined_slices_of_unequal_width(rows, cols, groups, batch, dtype):
    """One sample of nearly all rows among short ones, its pieces joined by a launch of their own in slices of groups
    of which the last is narrower."""
    _check(rows, cols, groups, [0] + list(range(rows - batch + 1, rows + 1)), dtype, "silu")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_small_samples(dtype):
    """One launch: slices of groups of unequal number, samples that fill the registers and ones that outgrow them."""
    for cols, groups, lengths, act in ((100, 10, [600] * 3 + [0, 3, 2500], "silu"), (60, 12, [30] * 40, "leaky"), (100, 100, [1, 5, 2], "none"),
                                       (24, 3, [200] * 9 + [4000], "relu"), (7, 7, [100, 3], "silu"), (300, 20, [64, 1, 190], "leaky"),
                                       (2048, 16, [9, 7], "silu"), (34, 17, [20] * 1100, "leaky"), (4096, 4, [3, 1, 2], "none")):
        begin = [0] + np.cumsum(lengths).tolist()
        for x8 in (False, True):
            _check(begin[-1], cols, groups, begin, dtype, act, 1, seed=cols, x8=x8)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_samples_by_number(dtype):
    from paper_1409_6070_amd.sscn import GroupNorm, SSCNError
    x, dy, gain, shift = _make(60, 40, dtype, 1)
    plan = GroupNorm(40, 4, 60, 60, dtype, "silu")
    x, dy, gain, shift = x.cuda(), dy.cuda(), gain.cuda(), shift.cuda()
    for batch in (1, 5, 60):
        b = torch.arange(batch + 1, dtype=torch.int32, device="cuda") * (60 // batch)
        y, stats = plan.forward(x, batch, gain, shift)
        y2, stats2 = plan.forward(x, b, gain, shift)
        assert torch.equal(y, y2) and torch.equal(stats, stats2)
        for p, q in zip(plan.backward(dy, x, stats, batch, gain, shift), plan.backward(dy, x, stats, b, gain, shift)):
            assert torch.equal(p, q)
    with pytest.raises(SSCNError):
        plan.forward(x, 7, gain, shift)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [5, 8, 100, 300, 77])
def test_in_place(cols, dtype):
    from paper_1409_6070_amd.sscn import GroupNorm
    x, dy, gain, shift = (t.cuda() for t in _make(1500, cols, dtype, 2))
    plan = GroupNorm(cols, 1, 1500, 3, dtype, "leaky")
    b = torch.tensor([0, 700, 701, 1490], dtype=torch.int32, device="cuda")
    y, stats = plan.forward(x, b, gain, shift, out=x.clone())
    x1 = x.clone()
    plan.forward(x1, b, gain, shift, out=x1)
    assert torch.equal(x1, y)
    dx, dg, ds = plan.backward(dy, x, stats, b, gain, shift, dx=dy.clone())
    for over in ("dy", "x"):
        d1, x1 = dy.clone(), x.clone()
        got = plan.backward(d1, x1, stats, b, gain, shift, dx=d1 if over == "dy" else x1)
        assert torch.equal(got[0][:1490], dx[:1490]) and torch.equal(got[1], dg) and torch.equal(got[2], ds)


def test_bad_values_stay_in_their_sample_and_group():
    from paper_1409_6070_amd.sscn import GroupNorm
    for act in ACTS:
        x, dy, gain, shift = (t.cuda() for t in _make(300, 24, "f32", 3))
        b = torch.tensor([0, 100, 200, 300], dtype=torch.int32, device="cuda")
        plan = GroupNorm(24, 3, 300, 3, "f32", act)
        clean, cstats = plan.forward(x, b, gain, shift)
        cdx = plan.backward(dy, x, cstats, b, gain, shift)[0]
        x[150, 9], x[299, 23] = float("nan"), float("inf")
        y, stats = plan.forward(x, b, gain, shift)
        dx = plan.backward(dy, x, stats, b, gain, shift)[0]
        bad = torch.zeros(300, 24, dtype=torch.bool, device="cuda")
        bad[100:200, 8:16] = bad[200:, 16:] = True
        assert y[bad].isnan().all() and torch.equal(y[~bad], clean[~bad])
        assert dx[bad].isnan().all() and torch.equal(dx[~bad], cdx[~bad])


# samples in registers, pieces joined by the last launch and by a launch of their own, the longest rows
PATHS = [(400, 60, 4, [0, 100, 100, 370]), (1500, 34, 17, list(range(0, 1501))), (30000, 100, 10, [0, 20000, 30000]),
         (200001, 20, 2, [0, 200001]), (24001, 288, 32, [0] + list(range(24001 - 59, 24002))), (9, 4096, 8, [0, 9])]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,groups,begin", PATHS)
def test_workspaces_are_as_large_as_they_say(rows, cols, groups, begin, dtype):
    """Exactly the bytes asked for, between bytes that have to stay as they were; results as from a plan, and as from
    one for more rows and samples."""
    from paper_1409_6070_amd import sscn
    from paper_1409_6070_amd.sscn import GroupNorm
    x, dy, gain, shift = (t.cuda() for t in _make(rows, cols, dtype, 7))
    b = torch.tensor(begin, dtype=torch.int32, device="cuda")
    batch, code = len(begin) - 1, int(dtype == "bf16")
    want = None
    for more in (0, 1, 5000):
        plan = GroupNorm(cols, groups, rows + more, batch + more, dtype, "leaky", EPS)
        y, stats = plan.forward(x, b, gain, shift, out=torch.zeros_like(x))
        got = (y, stats) + plan.backward(dy, x, stats, b, gain, shift, dx=torch.zeros_like(x))
        want = got if want is None else want
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    call = sscn.GroupNormCall(dtype=code, act=2, rows=rows, cols=cols, groups=groups, batch=batch, eps=EPS,
                              d_begin=b.data_ptr(), d_gain=gain.data_ptr(), d_shift=shift.data_ptr(), d_x=x.data_ptr(),
                              x_stride=cols)
    y, dx, stats = torch.zeros_like(x), torch.zeros_like(x), torch.zeros(2, batch, groups, device="cuda")
    dgain, dshift = torch.empty(2, cols, device="cuda").unbind(0)
    call.d_stats = stats.data_ptr()
    stream = torch.cuda.current_stream().cuda_stream
    for backward in (0, 1):
        need = sscn.sscn_group_norm_workspace_bytes(code, rows, cols, groups, batch, backward)
        ws = torch.full((need + 8192,), 0x5A, dtype=torch.uint8, device="cuda")
        at = ws.data_ptr() + 4096
        if backward:
            sscn.sscn_group_norm_backward(call, dy.data_ptr(), cols, dx.data_ptr(), cols, dgain.data_ptr(), dshift.data_ptr(),
                                          at, need, stream)
        else:
            sscn.sscn_group_norm_forward(call, y.data_ptr(), cols, at, need, stream)
        assert (ws[:4096] == 0x5A).all() and (ws[4096 + need:] == 0x5A).all()
    assert all(torch.equal(p, q) for p, q in zip((y, stats, dx, dgain, dshift), want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,begin", [(300, 60, [40, 100, 100, 250]), (30000, 100, [5000, 5001, 28000]),
                                             (5000, 12, [2000, 4000]), (40000, 16, [30000, 30000, 30001, 39999])])
def test_rows_outside_the_samples_do_not_matter(rows, cols, begin, dtype):
    """NaN, infinities and large values there: the samples' results are the same to the bit, and nothing is written."""
    from paper_1409_6070_amd.sscn import GroupNorm, Rows8
    x, dy, gain, shift = (t.cuda() for t in _make(rows, cols, dtype, 5))
    b = torch.tensor(begin, dtype=torch.int32, device="cuda")
    plan = GroupNorm(cols, 2, rows, len(begin) - 1, dtype, "leaky")
    inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
    inside[begin[0]: begin[-1]] = True

    def results():
        y, stats = plan.forward(x, b, gain, shift, out=torch.full_like(x, 3.0))
        got = [y, stats]
        for held in (x, Rows8(rows, cols).store(x)):
            got += plan.backward(dy, held, stats, b, gain, shift, dx=torch.full_like(x, 3.0))
        return got

    want = results()
    assert all((want[i][~inside] == 3).all() and want[i][inside].isfinite().all() for i in (0, 2, 5))
    for value in (float("nan"), float("inf"), 1e30):
        x[~inside], dy[~inside] = value, value
        assert all(torch.equal(p, q) for p, q in zip(results(), want))


def test_constant_groups():
    """No variance: r = 1 / sqrt(eps), h is zero or a rounding of the mean."""
    from paper_1409_6070_amd.sscn import GroupNorm
    for v in (0.0, 3.25, -1e4):
        x = torch.full((200, 16), v, device="cuda")
        y, stats = GroupNorm(16, 2, 200, 2, "f32").forward(x, 2)
        assert (y == 0).all() and (stats[0] == v).all() and torch.allclose(stats[1], torch.tensor(EPS ** -0.5).cuda(), rtol=3e-7)


def test_large_means_and_outliers():
    """A mean of a thousand deviations, and a first row far from all others: what the variance's own sums can lose."""
    from paper_1409_6070_amd.sscn import GroupNorm
    x, _, gain, shift = _make(5000, 16, "f32", 4)
    for change in (lambda t: t + 1000.0, lambda t: torch.cat([t[:1] + 1e4, t[1:]])):
        xs = change(x)
        plan = GroupNorm(16, 2, 5000, 1, "f32")
        y, stats = plan.forward(xs.cuda(), 1, gain.cuda(), shift.cuda())
        want, tol, means, rs, te, tr = _want_forward(_np(xs), [0, 5000], gain.double().numpy(), shift.double().numpy(), 2, "none", "f32")
        _within(y, want, tol, "y")
        _within(stats[1], rs, tr, "r")


def test_offsets_past_32_bits():
    from paper_1409_6070_amd.sscn import GroupNorm, Rows8
    rows, cols = (1 << 20) + 500, 4096
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    tail, dyt, gain, shift = _make(400, cols, "bf16", 6)
    x[-400:] = tail.cuda()
    begin = [0, rows - 400, rows]
    b = torch.tensor(begin, dtype=torch.int32, device="cuda")
    plan = GroupNorm(cols, 32, rows, 2, "bf16", "leaky")
    y, stats = plan.forward(x, b, gain.cuda(), shift.cuda())
    gn, sn = gain.double().numpy(), shift.double().numpy()
    want, tol, *_ = _want_forward(_np(tail), [0, 400], gn, sn, 32, "leaky", "bf16")
    _within(y[-400:], want, tol, "y")
    first = _act(sn, "leaky")[0]
    assert (np.abs(_np(y[:1000]) - first) <= 2.0 ** -8 * np.abs(first) + 1e-30).all()
    dy = torch.zeros_like(x)
    dy[-400:] = dyt.cuda()
    bx, bg, bs = _want_backward(_np(dyt), _np(tail), _np(stats)[:, 1:], [0, 400], gn, sn, 32, "leaky", "bf16")
    dx, dg, ds = plan.backward(dy, x, stats, b, gain.cuda(), shift.cuda(), dx=y)
    _within(dx[-400:], *bx, "dx")
    assert (dx[:rows - 400] == 0).all()
    _within(ds, *bs, "dshift")
    x8 = Rows8(rows, cols).store(x)
    held = x8.rows_from(rows - 400, rows).load("f32")
    bx, bg, bs = _want_backward(_np(dyt), _np(held), _np(stats)[:, 1:], [0, 400], gn, sn, 32, "leaky", "bf16")
    dx, dg, ds = plan.backward(dy, x8, stats, b, gain.cuda(), shift.cuda(), dx=dy)
    _within(dx[-400:], *bx, "dx, 8 bits")
    _within(dg, *bg, "dgain, 8 bits")


def test_no_rows_and_no_samples():
    from paper_1409_6070_amd.sscn import GroupNorm
    plan = GroupNorm(12, 3, 50, 4, "f32", "relu")
    none = torch.empty(0, 12, device="cuda")
    for begin in (torch.zeros(3, dtype=torch.int32, device="cuda"), 2, 0, torch.zeros(1, dtype=torch.int32, device="cuda")):
        y, stats = plan.forward(none, begin)
        batch = stats.shape[1]
        assert y.shape == (0, 12) and (stats[0] == 0).all() and torch.allclose(stats[1], torch.tensor(EPS ** -0.5).cuda())
        dx, dg, ds = plan.backward(none, none, stats, begin)
        assert dx.shape == (0, 12) and (dg == 0).all() and (ds == 0).all() and batch in (0, 2)
    x = torch.randn(50, 12, device="cuda")
    out = torch.full_like(x, 3.0)
    y, stats = plan.forward(x, torch.tensor([7], dtype=torch.int32, device="cuda"), out=out)  # rows, but no sample
    assert (out == 3).all()
    dx, dg, ds = plan.backward(x, x, stats, torch.tensor([7], dtype=torch.int32, device="cuda"), dx=out)
    assert (out == 3).all() and (dg == 0).all() and (ds == 0).all()


def test_streams_and_graphs():
    from paper_1409_6070_amd.sscn import GroupNorm, Rows8
    for rows, cols, groups, begin in ((400, 60, 4, [0, 100, 100, 370]), (30000, 100, 10, [0, 20000, 30000])):
        plan = GroupNorm(cols, groups, rows, 3, "bf16", "leaky")
        sets = [[t.cuda() for t in _make(rows, cols, "bf16", i)] for i in range(3)]
        b = torch.tensor(begin, dtype=torch.int32, device="cuda")
        x, dy, gain, shift = (t.clone() for t in sets[0])
        x8, y, dx = Rows8(rows, cols), torch.zeros_like(x), torch.zeros_like(x)

        def step():
            _, stats = plan.forward(x, b, gain, shift, out=y)
            return (stats,) + plan.backward(dy, x8.store(x), stats, b, gain, shift, dx=dx)[1:]

        def values(i):
            for t, v in zip((x, dy, gain, shift), sets[i]):
                t.copy_(v)

        want = []
        for i in range(3):
            values(i)
            want.append([t.clone() for t in step() + (y, dx)])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            values(1)
            assert all(torch.equal(p, q) for p, q in zip(step() + (y, dx), want[1]))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step()
        for i in (0, 2, 1, 0):
            values(i)
            y.zero_(), dx.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got + (y, dx), want[i]))
            values((i + 1) % 3)
            step()
            torch.cuda.synchronize()


def test_two_plans_at_once():
    """Each with its own workspaces, on a stream of its own, over the same rows and parameters."""
    from paper_1409_6070_amd.sscn import GroupNorm
    rows, cols = 60001, 100
    x, dy, gain, shift = (t.cuda() for t in _make(rows, cols, "bf16", 1))
    b = torch.tensor(_begins(rows, 9, 2), dtype=torch.int32, device="cuda")
    plans = [GroupNorm(cols, g, rows, 9, "bf16", a) for g, a in ((10, "leaky"), (4, "silu"))]

    def step(plan):
        y, stats = plan.forward(x, b, gain, shift, out=torch.zeros_like(x))
        dx, dgain, dshift = plan.backward(dy, x, stats, b, gain, shift, dx=torch.zeros_like(x))
        return y, stats, dx, dgain, dshift

    want = [step(p) for p in plans]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in plans]
    got = []
    for _ in range(3):
        for p, s in zip(plans, streams):
            with torch.cuda.stream(s):
                got.append(step(p))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert all(torch.equal(p, q) for p, q in zip(g, want[i % 2]))


def test_gradients_against_differences():
    """Central differences of sum(w * y) in float32 values nudged by 2^-7, against the formula's derivative."""
    from paper_1409_6070_amd.sscn import GroupNorm
    g = torch.Generator().manual_seed(1)
    x, w = torch.randn(40, 12, generator=g), torch.randn(40, 12, generator=g)
    gain, shift = 1 + 0.2 * torch.randn(12, generator=g), 0.2 * torch.randn(12, generator=g)
    b = torch.tensor([0, 15, 40], dtype=torch.int32, device="cuda")
    plan = GroupNorm(12, 3, 40, 2, "f32", "silu")

    def loss():
        return float((plan.forward(x.cuda(), b, gain.cuda(), shift.cuda())[0].double().cpu() * w).sum())

    _, stats = plan.forward(x.cuda(), b, gain.cuda(), shift.cuda())
    dx, dg, ds = (t.cpu() for t in plan.backward(w.cuda(), x.cuda(), stats, b, gain.cuda(), shift.cuda()))
    step = 2.0 ** -7
    for t, d, spots in ((x, dx, [(0, 0), (14, 5), (15, 11), (39, 3)]), (gain, dg, [(0,), (7,), (11,)]), (shift, ds, [(2,), (11,)])):
        for i in spots:
            old = float(t[i])
            t[i] = old + step
            up = loss()
            t[i] = old - step
            down = loss()
            t[i] = old
            # third derivatives of a few units times step^2 / 6, and float32 roundings of 480 terms over the step
            assert abs((up - down) / (2 * step) - float(d[i])) < 20 * step ** 2 / 6 + 480 * 4 * U / step + 1e-3


def test_a_stage_in_front_of_the_network():
    """A 1x1 layer in 8 bits and a group norm on the input sites, whose gradient comes from the network's backward pass:
    every step against the same formulas in 64 bits, on what the step before it left."""
    from paper_1409_6070_amd.sscn import GroupNorm, Product8, Rows8, SparseDeepCNet
    from tests.test_gpu_rows8 import _held, _held_matrix, _product_bound
    from workloads import he_params
    ell, k, c_raw, c_in, classes, batch = 3, 12, 37, 24, 10, 6
    rng = np.random.default_rng(2)
    side = 3 * 2 ** ell
    per = [40, 0, 7, 90, 1, 33]  # sites of each sample
    coords = np.concatenate([np.stack([np.full(n, b), *np.divmod(rng.permutation(side * side)[:n], side)], 1)
                             for b, n in enumerate(per)]).astype(np.int32)
    begin = np.concatenate([[0], np.cumsum(per)]).astype(np.int32)
    n = len(coords)
    for dtype in ("f32", "bf16"):
        to = TORCH[dtype]
        raw = torch.tensor(rng.normal(size=(n, c_raw))).to(to).cuda()
        w = torch.tensor(rng.normal(size=(c_raw, c_in)) * c_raw ** -0.5).float().cuda()
        gain, shift = torch.ones(c_in, device="cuda"), torch.zeros(c_in, device="cuda")
        Ws, bs = he_params(ell, k, c_in, classes, 1)
        Ws = [torch.tensor(v, dtype=torch.float32).to(to).cuda().contiguous() for v in Ws]
        bs = [torch.tensor(v, dtype=torch.float32).cuda() for v in bs]
        labels = torch.tensor(rng.integers(0, classes, batch), dtype=torch.int32, device="cuda")
        net = SparseDeepCNet(ell, k, c_in, classes, batch, n, dtype)
        b_dev = torch.tensor(begin, device="cuda")
        net.rulebook_build(torch.tensor(coords, device="cuda"), batch, b_dev)
        layer, norm = Product8(c_raw, c_in, n, dtype).set_weights(w), GroupNorm(c_in, 4, n, batch, dtype, "leaky")
        raw8 = Rows8(n, c_raw).store(raw)
        u = layer.forward(raw8)
        feats, stats = norm.forward(u, b_dev, gain, shift)
        u8 = Rows8(n, c_in).store(u)  # kept for the backward pass
        net.forward(feats, Ws, bs, labels)
        _, _, dfeats = net.backward(want_dfeats=True)
        du, dgain, dshift = norm.backward(dfeats, u8, stats, b_dev, gain, shift)
        du8 = Rows8(n, c_in).store(du)
        dw, _ = layer.weight_grad(raw8, du8)
        draw = layer.input_grad(du8)

        rawq, wq = _held(_np(raw))[0], _held_matrix(_np(w))
        want, tol = _product_bound(rawq, wq, dtype)
        _within(u, want, tol, "u")
        one, zero = np.ones(c_in), np.zeros(c_in)
        want, tol, *_ = _want_forward(_np(u), begin.tolist(), one, zero, 4, "leaky", dtype)
        _within(feats, want, tol, "features")
        held = _held(_np(u))[0]
        bx, bg, bs_ = _want_backward(_np(dfeats), held, _np(stats), begin.tolist(), one, zero, 4, "leaky", dtype)
        _within(du, *bx, "du")
        _within(dgain, *bg, "dgain")
        duq = _held(_np(du))[0]
        _within(dw, rawq.T @ duq, (32 + n / 32 + 520) * U * (np.abs(rawq).T @ np.abs(duq)) + 1e-300, "dw")
        want, tol = _product_bound(duq, wq.T, dtype)
        _within(draw, want, tol, "draw")
        assert float(dw.abs().max()) > 0 and dfeats.isfinite().all()


def test_binding_refuses():
    from paper_1409_6070_amd.sscn import GroupNorm, Rows8, SSCNError
    for args in ((12, 5, 10, 1), (0, 1, 10, 1), (4097, 1, 10, 1), (12, 3, -1, 1), (12, 3, 10, -1)):
        with pytest.raises(SSCNError):
            GroupNorm(*args)
    for kw in (dict(dtype="f16"), dict(act="gelu")):
        with pytest.raises(ValueError):
            GroupNorm(12, 3, 10, 1, **kw)
    plan = GroupNorm(12, 3, 10, 2, "f32")
    x = torch.randn(10, 12, device="cuda")
    y, stats = plan.forward(x, 2)
    one = torch.ones(12, device="cuda")
    for call in (lambda: plan.forward(x.bfloat16(), 2), lambda: plan.forward(x[:, :11], 2), lambda: plan.forward(x.cpu(), 2),
                 lambda: plan.forward(torch.randn(11, 12, device="cuda"), 1), lambda: plan.forward(x, 5),
                 lambda: plan.forward(x, torch.zeros(3, device="cuda")), lambda: plan.forward(x, torch.zeros(3, dtype=torch.int32)),
                 lambda: plan.forward(x, 2, gain=one[:11]), lambda: plan.forward(x, 2, gain=one.double()),
                 lambda: plan.forward(x, 2, out=x[:9]), lambda: plan.backward(x, x[:9], stats, 2),
                 lambda: plan.backward(x, x, stats[:1], 2), lambda: plan.backward(x, x, stats, 1),
                 lambda: plan.backward(x, Rows8(9, 12), stats, 2), lambda: plan.backward(x, Rows8(10, 13), stats, 2),
                 lambda: plan.forward(torch.randn(12, 10, device="cuda").t(), 2)):
        with pytest.raises(ValueError):
            call()
