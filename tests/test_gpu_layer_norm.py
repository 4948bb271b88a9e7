"""Layer norm on the GPU against its formula in 64 bits: rows of one column to rows that outgrow a workgroup,
odd lengths, strides and alignments, rows without variance, infinities and NaN; the norm in front of the softmax
layer inside a network's passes.

Bounds.  u = 2^-24.  A sum of n terms in a thread's chain of at most k additions, then a tree, is off by at most
D u sum|terms| with D = k + 16.  With e = D u mean|x| for the mean: x - mean is off by e + u |d|; the variance by
(D + 4) u + (e r)^2 relative (the deviations sum to zero, so e enters squared); r by half that plus 3 u.  The rest
counts one u per operation, and the result's rounding is half a step of its type."""

import numpy as np
import pytest
import torch

from tests.gpu_harness import log

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
EPS = 1e-5


@pytest.fixture(autouse=True, scope="module")
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1409_6070_amd import sscn
    sscn.load_library()


def _chain(cols, dtype):
    """Additions in a thread's chain: its elements of a row (16 in registers), or a looping row's share, and the
    sixteen waves' sums."""
    return 16 + 16 + -(-cols // 1024)


def _stats(x, eps=EPS):
    c = x.shape[1]
    mean = x.mean(1, keepdims=True)
    d = x - mean
    r = 1.0 / np.sqrt((d * d).mean(1, keepdims=True) + eps)
    D = _chain(c, None) + 16
    e = D * U * np.abs(x).mean(1, keepdims=True)
    rel_r = 0.5 * ((D + 4) * U + (e * r) ** 2) + 3 * U
    return d, r, d * r, e, rel_r, D


def _want_forward(x, gain, shift, dtype):
    d, r, h, e, rel_r, _ = _stats(x)
    y = h * gain + shift
    err = np.abs(gain) * (r * (e + U * np.abs(d)) + np.abs(h) * (rel_r + 3 * U)) + U * (np.abs(h * gain) + np.abs(shift))
    return y, err * 1.01 + HALF[dtype] * (np.abs(y) + err) + 1e-38


def _want_backward(dy, x, gain, dtype, parts, rpb):
    d, r, h, e, rel_r, D = _stats(x)
    t = dy * gain
    m1, m2 = t.mean(1, keepdims=True), (t * h).mean(1, keepdims=True)
    a1, a2 = np.abs(t).mean(1, keepdims=True), np.abs(t * h).mean(1, keepdims=True)
    dx = r * (t - m1 - h * m2)
    dh = r * (e + U * np.abs(d)) + np.abs(h) * (rel_r + 2 * U)   # error of h
    dm1 = (D + 2) * U * a1
    dm2 = (D + 6) * U * a2 + (np.abs(t) * dh).mean(1, keepdims=True)
    err = r * (2 * U * np.abs(t) + dm1 + dh * np.abs(m2) + np.abs(h) * dm2 + 4 * U * (np.abs(t) + a1 + np.abs(h) * a2))
    err += (rel_r + 2 * U) * r * (np.abs(t) + np.abs(m1) + np.abs(h * m2))
    # parameter sums: a thread's rows, the rows of its workgroup, sixteen slices of the parts
    n = -(-dy.shape[0] // (parts * rpb)) + rpb + -(-parts // 16) + 16 + 4
    dg, ds = (dy * h).sum(0), dy.sum(0)
    eg = (np.abs(dy) * dh).sum(0) + n * U * np.abs(dy * h).sum(0)
    es = n * U * np.abs(dy).sum(0)
    return (dx, err * 1.01 + HALF[dtype] * (np.abs(dx) + err) + 1e-38), (dg, eg * 1.01 + 1e-38), (ds, es * 1.01 + 1e-38)


def _within(got, want, tol, what):
    got = got.double().cpu().numpy()
    assert got.shape == want.shape
    off = np.abs(got - want) - tol
    worst = float((np.abs(got - want) / tol).max()) if got.size else 0.0
    log(f"  {what}: at most {worst:.3f} of the bound")
    assert np.isfinite(got).all() and (off <= 0).all(), what


def _make(rows, cols, dtype, pad, seed, offset=0.5):
    """x, dy as [rows, cols] views of buffers `pad` elements wider (a width of its own for each), gain, shift."""
    g = torch.Generator().manual_seed(seed)
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = (torch.randn(rows, cols + pad, generator=g) * 0.8 + offset).to(tdt).cuda()[:, pad // 2: pad // 2 + cols]
    dy = (torch.randn(rows, cols + 2 * pad, generator=g) * 0.3).to(tdt).cuda()[:, pad: pad + cols]
    gain = (1 + 0.3 * torch.randn(cols, generator=g)).cuda()
    shift = (0.2 * torch.randn(cols, generator=g)).cuda()
    return x, dy, gain, shift


def _np(t):
    return t.double().cpu().numpy()


def _parts(code, rows, cols):
    from paper_1409_6070_amd import sscn
    return sscn.sscn_layer_norm_workspace_bytes(code, rows, cols) // (8 * cols)


def _check(rows, cols, dtype, pad, seed=0, x=None):
    from paper_1409_6070_amd.sscn import LayerNorm
    x0, dy, gain, shift = _make(rows, cols, dtype, pad, seed)
    x = x0 if x is None else x
    log(f"[layer norm] {rows} x {cols} {dtype} pad {pad}")
    ln = LayerNorm(cols, rows, dtype, EPS)
    y = ln.forward(x, gain, shift)
    dx, dg, ds = ln.backward(dy, x, gain)
    torch.cuda.synchronize()
    xs, gs = _np(x), _np(gain)
    _within(y, *_want_forward(xs, gs, _np(shift), dtype), "y")
    bx, bg, bs = _want_backward(_np(dy), xs, gs, dtype, _parts(ln.code, rows, cols), 1)
    _within(dx, *bx, "dx")
    _within(dg, *bg, "dgain")
    _within(ds, *bs, "dshift")


# every row shape of the kernels: fewer columns than a vector, 8 .. 64 lanes, one and two vectors, workgroups of
# 256 .. 1024, rows that loop; lengths on both sides of each border, odd ones
COLS = [1, 2, 3, 7, 8, 9, 31, 32, 33, 50, 63, 64, 65, 100, 127, 129, 255, 257, 300, 511, 513, 1000, 1025, 2047, 2049, 4097,
        8191, 8193]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_columns(cols, dtype):
    for rows, pad in ((1, 0), (5, 0), (37, 3), (70, 8)):
        _check(rows, cols, dtype, pad, seed=cols)


@pytest.mark.parametrize("cols,dtype", [(16383, "bf16"), (16385, "bf16"), (20001, "f32"), (70001, "bf16")])
def test_long_rows(cols, dtype):
    _check(3, cols, dtype, 1)
    _check(300 if cols < 20000 else 5, cols, dtype, 0)


@pytest.mark.parametrize("rows,cols,dtype", [(1000, 9, "f32"), (40000, 50, "bf16"), (20000, 100, "bf16"), (8193, 61, "f32"),
                                             (8192, 511, "bf16"), (33001, 100, "f32"), (9001, 300, "bf16"),
                                             (5000, 1024, "f32"), (2500, 4099, "f32"), (1500, 8192, "bf16")])
def test_many_rows(rows, cols, dtype):
    _check(rows, cols, dtype, 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_misaligned_bases_and_everything_around_the_rows_stays(dtype):
    """Arrays that start at odd elements, with guards before, between and behind their rows."""
    from paper_1409_6070_amd.sscn import LayerNorm
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    for rows, cols, stride, start in ((6, 100, 107, 1), (9, 53, 53, 3), (4, 1030, 1031, 5), (3, 9000, 9003, 7), (5, 5, 6, 1)):
        log(f"[layer norm] guards {rows} x {cols} stride {stride} start {start} {dtype}")
        x, dy, gain, shift = _make(rows, cols, dtype, 0, 3)
        def place(t):
            buf = torch.full((start + rows * stride + 8,), 7.5, dtype=tdt, device="cuda")
            v = torch.as_strided(buf, (rows, cols), (stride, 1), start)
            if t is not None:
                v.copy_(t)
            return buf, v
        (bx, vx), (bd, vd), (by, vy), (bo, vo) = place(x), place(dy), place(None), place(None)
        keep = bx.clone(), bd.clone()
        ln = LayerNorm(cols, rows, dtype, EPS)
        ln.forward(vx, gain, shift, out=vy)
        _, dg, ds = ln.backward(vd, vx, gain, dx=vo)
        want_y = ln.forward(x, gain, shift)
        want = ln.backward(dy, x, gain)
        torch.cuda.synchronize()
        assert torch.equal(vy, want_y) and torch.equal(vo, want[0])  # placement changes no bit
        assert torch.equal(dg, want[1]) and torch.equal(ds, want[2])
        assert torch.equal(bx, keep[0]) and torch.equal(bd, keep[1])
        for buf in (by, bo):
            mask = torch.ones_like(buf, dtype=torch.bool)
            torch.as_strided(mask, (rows, cols), (stride, 1), start).fill_(False)
            assert (buf[mask] == 7.5).all()


@pytest.mark.parametrize("cols", [100, 20000])
def test_offsets_past_32_bits(cols):
    """Rows 2^30 and some elements apart, the last beyond 2^32 elements: the bits of packed rows."""
    from paper_1409_6070_amd.sscn import LayerNorm
    rows, stride = 5, (1 << 30) + 3
    x, dy, gain, shift = _make(rows, cols, "bf16", 0, 3)
    far = [torch.as_strided(torch.empty((rows - 1) * stride + cols, dtype=torch.bfloat16, device="cuda"), (rows, cols),
                            (stride, 1)) for _ in range(2)]
    far[0].copy_(x)
    far[1].copy_(dy)
    ln = LayerNorm(cols, rows, "bf16", EPS)
    want_y, want = ln.forward(x, gain, shift), ln.backward(dy, x, gain)
    got = ln.backward(far[1], far[0], gain, dx=far[1])
    ln.forward(far[0], gain, shift, out=far[0])
    assert torch.equal(far[0], want_y) and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [1, 5, 100, 1025, 4096, 20000])
def test_in_place(cols, dtype):
    from paper_1409_6070_amd.sscn import LayerNorm
    x, dy, gain, shift = _make(40, cols, dtype, 0, 5)
    ln = LayerNorm(cols, 40, dtype, EPS)
    y = ln.forward(x, gain, shift)
    dx, dg, ds = ln.backward(dy, x, gain)
    a, b, c, d = x.clone(), dy.clone(), x.clone(), dy.clone()
    ln.forward(a, gain, shift, out=a)
    r1 = ln.backward(b, x, gain, dx=b)
    r2 = ln.backward(d, c, gain, dx=c)
    torch.cuda.synchronize()
    assert torch.equal(a, y) and torch.equal(b, dx) and torch.equal(c, dx)
    for r in (r1, r2):
        assert torch.equal(r[1], dg) and torch.equal(r[2], ds)


@pytest.mark.parametrize("cols", [1, 6, 100, 3001])
def test_without_gain_and_shift(cols):
    from paper_1409_6070_amd.sscn import LayerNorm
    x, dy, _, _ = _make(11, cols, "f32", 0, 6)
    one, zero = torch.ones(cols, device="cuda"), torch.zeros(cols, device="cuda")
    ln = LayerNorm(cols, 11, "f32", EPS)
    assert torch.equal(ln.forward(x), ln.forward(x, one, zero))
    for p, q in zip(ln.backward(dy, x), ln.backward(dy, x, one)):
        assert torch.equal(p, q)


def test_rows_without_variance():
    """Equal values: h is 0 up to the mean's rounding, y is the shift, and nothing is NaN."""
    from paper_1409_6070_amd.sscn import LayerNorm
    for cols in (1, 3, 64, 1000, 9000):
        for value in (0.0, 1.0, -3.0, 2.0 ** 20):
            x = torch.full((3, cols), value, device="cuda")
            gain, shift = torch.full((cols,), 2.0, device="cuda"), torch.full((cols,), 0.25, device="cuda")
            ln = LayerNorm(cols, 3, "f32", EPS)
            y = ln.forward(x, gain, shift)
            # the mean's error, times r = 1 / sqrt(eps) at most, times the gain
            tol = 2.0 * (_chain(cols, None) + 16) * U * abs(value) / EPS ** 0.5 + 1e-7
            assert (y - 0.25).abs().max().item() <= tol
            assert all(torch.isfinite(t).all() for t in ln.backward(torch.ones_like(x), x, gain))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [6, 100, 700, 5000, 40000])
def test_bad_rows_stay_alone(cols, dtype):
    """A NaN or an infinity makes its own row NaN; the rows beside it keep their bits."""
    from paper_1409_6070_amd.sscn import LayerNorm
    x, dy, gain, shift = _make(9, cols, dtype, 0, 8)
    ln = LayerNorm(cols, 9, dtype, EPS)
    y, (dx, _, _) = ln.forward(x, gain, shift), ln.backward(dy, x, gain)
    bad = x.clone()
    bad[2, cols - 1], bad[4, 0], bad[7, cols // 2] = float("nan"), float("inf"), float("-inf")
    y2, (dx2, dg2, _) = ln.forward(bad, gain, shift), ln.backward(dy, bad, gain)
    torch.cuda.synchronize()
    hit = torch.zeros(9, dtype=torch.bool, device="cuda")
    hit[[2, 4, 7]] = True
    for a, b in ((y, y2), (dx, dx2)):
        assert torch.equal(a[~hit], b[~hit]) and torch.isnan(b[hit]).all()
    assert torch.isnan(dg2).all()


def test_no_rows():
    from paper_1409_6070_amd.sscn import LayerNorm
    ln = LayerNorm(10, 4, "f32", EPS)
    e = torch.empty(0, 10, device="cuda")
    assert ln.forward(e).shape == (0, 10)
    dx, dg, ds = ln.backward(e, e)
    assert dx.shape == (0, 10) and (dg == 0).all() and (ds == 0).all()


def test_gradient_against_differences():
    """d/de sum(w norm(x + e v)) by central differences of the forward kernel, for x, gain and shift."""
    from paper_1409_6070_amd.sscn import LayerNorm
    rows, cols = 20, 257
    x, w, gain, shift = _make(rows, cols, "f32", 0, 11)
    g = torch.Generator().manual_seed(12)
    v = torch.randn(rows, cols, generator=g).cuda()
    p = torch.randn(cols, generator=g).cuda()
    ln = LayerNorm(cols, rows, "f32", EPS)
    dx, dg, ds = ln.backward(w, x, gain)
    f = lambda x, a, b: (ln.forward(x, a, b).double() * w.double()).sum().item()  # noqa: E731
    h = 2.0 ** -6
    # the difference's own error: h^2 / 6 of a third derivative of the order of the value's scale, and forward
    # roundings (about 4 u of each |w y|, independent) over 2 h
    scale = (w.double().abs() * ln.forward(x, gain, shift).double().abs()).sum().item()
    for got, hi, lo in (((dx.double() * v.double()).sum().item(), f(x + h * v, gain, shift), f(x - h * v, gain, shift)),
                        ((dg.double() * p.double()).sum().item(), f(x, gain + h * p, shift), f(x, gain - h * p, shift)),
                        ((ds.double() * p.double()).sum().item(), f(x, gain, shift + h * p), f(x, gain, shift - h * p))):
        want = (hi - lo) / (2 * h)
        log(f"  differences {want:.6g}, gradient {got:.6g}")
        assert abs(got - want) <= h * h * scale + 8 * U * scale / (2 * h)


def test_repeats_streams_and_graphs():
    """The same bits every time: on another stream, and replayed from a graph with eager work between."""
    from paper_1409_6070_amd.sscn import LayerNorm
    x, dy, gain, shift = _make(3000, 300, "bf16", 4, 13)
    ln = LayerNorm(300, 3000, "bf16", EPS)
    want = (ln.forward(x, gain, shift), *ln.backward(dy, x, gain))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = (ln.forward(x, gain, shift), *ln.backward(dy, x, gain))
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    out, dx = torch.empty_like(want[0]), torch.empty_like(want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ln.forward(x, gain, shift, out=out)
        _, dg, ds = ln.backward(dy, x, gain, dx=dx)
    for i in range(4):
        x.add_(0.25 * i)
        out.zero_(), dx.zero_(), dg.zero_(), ds.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want = (ln.forward(x, gain, shift), *ln.backward(dy, x, gain))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, dx, dg, ds), want)), i


def test_wrapper_refuses():
    from paper_1409_6070_amd.sscn import LayerNorm
    ln = LayerNorm(16, 8, "f32")
    x = torch.randn(8, 16, device="cuda")
    g = torch.ones(16, device="cuda")
    for bad in (x.bfloat16(), x.cpu(), x[:, :15], x.t(), x[0], x[:1].expand(8, 16)):
        with pytest.raises(ValueError):
            ln.forward(bad, g, g)
    for p in (g[:15], g.double(), g.cpu(), torch.ones(32, device="cuda")[::2]):
        with pytest.raises(ValueError):
            ln.forward(x, p, g)
        with pytest.raises(ValueError):
            ln.backward(x, x, p)
    for out in (x[:7], x.bfloat16(), torch.empty(16, 8, device="cuda").t()):
        with pytest.raises(ValueError):
            ln.forward(x, g, g, out=out)
        with pytest.raises(ValueError):
            ln.backward(x, x, g, dx=out)
    big = torch.randn(9, 16, device="cuda")
    with pytest.raises(ValueError):
        ln.backward(big, big, g)


# ---------------------------------------------------------------------------------------------------------
# the norm in front of the softmax layer

HEADS = [("f32", 10, None), ("f32", 3755, None), ("bf16", 10, None), ("bf16", 3755, None), ("f32", 10, 0.5), ("bf16", 3755, 0.4)]


def _net(dtype, classes, drop, seed=0):
    from paper_1409_6070_amd.sscn import SparseDeepCNet
    from workloads import he_params, random_labels
    rng = np.random.default_rng(seed)
    ell, k, c_in, batch = 3, 13, 2, 21
    N = 3 * 2 ** ell
    coords = np.concatenate([np.stack([np.full(9, b), *np.divmod(rng.choice(N * N, 9, replace=False), N)], 1)
                             for b in range(batch) if b != 4])  # sample 4 is empty: its top row is the ground row
    net = SparseDeepCNet(ell, k, c_in, classes, batch + 3, len(coords) + 5, dtype, dropout=drop is not None)
    tdt = net.tdtype
    coords = torch.tensor(coords, dtype=torch.int32, device="cuda")
    feats = torch.tensor(rng.normal(size=(len(coords), c_in))).to(tdt).cuda()
    Ws, bs = he_params(ell, k, c_in, classes, 1)
    W32 = [torch.tensor(w, dtype=torch.float32, device="cuda") for w in Ws]
    b = [torch.tensor(v, dtype=torch.float32, device="cuda") for v in bs]
    labels = torch.tensor(random_labels(batch, classes, 2), dtype=torch.int32, device="cuda")
    if drop is not None:
        net.set_dropout([0.0] * (ell + 1) + [drop], 77)
    net.rulebook_build(coords, batch)
    return net, feats, W32, [w.to(tdt) for w in W32], b, labels, batch


def _keep(batch, channels, level, p, seed):
    from paper_1409_6070_amd import sscn
    f = np.zeros((batch, channels))
    thr = int(np.floor(p * 2 ** 32))
    for b in range(batch):
        for c4 in range(-(-channels // 4)):
            w = sscn.sscn_philox4x32_10([b, c4, level, 0], [seed & 0xffffffff, seed >> 32])
            for e in range(min(4, channels - 4 * c4)):
                f[b, 4 * c4 + e] = np.float32(1.0 / (1.0 - p)) if w[e] >= thr else 0.0
    return f


@pytest.mark.parametrize("dtype,classes,drop", HEADS)
def test_head_norm_in_a_network(dtype, classes, drop):
    """Logits, loss gradient, the norm's gradients and the top layer's, from the network's own top features."""
    net, feats, _, Ws, bs, labels, batch = _net(dtype, classes, drop)
    C = net.param_shapes[-1][0]
    g = torch.Generator().manual_seed(3)
    gain, shift = (1 + 0.3 * torch.randn(C, generator=g)).cuda(), (0.2 * torch.randn(C, generator=g)).cuda()
    dgain, dshift = net.set_head_norm(gain, shift, EPS)
    logits, loss = net.forward(feats, Ws, bs, labels)
    logits = _np(logits)
    dW, db, dfeats = net.backward(want_dfeats=True)
    torch.cuda.synchronize()
    top = net.nlayers - 1
    view = net.layer_view(top)
    X, G = _np(view["features"])[:, :C], _np(view["grad"])[:, :C]
    side = view["side"]
    rows = np.zeros(batch, dtype=int)
    assert side == 1
    rows[_np(view["sites"]).astype(int)] = np.arange(1, view["n"] + 1)
    assert rows[4] == 0 and (rows > 0).sum() == batch - 1
    x = X[rows]
    y, tol_y = _want_forward(x, _np(gain), _np(shift), dtype)
    # the stored norm is y within tol_y (its rounding included); products and sums of C terms in float32
    keep = np.ones((batch, C)) if drop is None else _keep(batch, C, net.ell + 1, drop, 77)
    hin = y * keep
    tol_h = tol_y * keep + (0 if drop is None else (HALF[dtype] + U) * np.abs(hin) * 1.01)
    W = _np(Ws[-1])
    want = hin @ W + _np(bs[-1])
    tol = tol_h @ np.abs(W) + (C + 4) * U * (np.abs(hin) @ np.abs(W) + np.abs(_np(bs[-1])))
    off = np.abs(logits - want) / (1.01 * tol)
    log(f"[head norm] {dtype} {classes} classes dropout {drop}: logits at most {off.max():.3f} of the bound")
    assert (off <= 1).all()
    # from the network's logits on: softmax, its gradient (stored in the storage type), dh
    z = logits - logits.max(1, keepdims=True)
    p = np.exp(z) / np.exp(z).sum(1, keepdims=True)
    want_loss = -np.mean(np.log(p[np.arange(batch), labels.cpu().numpy()]))
    assert abs(float(loss) - want_loss) <= 1e-5 * max(1.0, abs(want_loss))
    dl = p.copy()
    dl[np.arange(batch), labels.cpu().numpy()] -= 1
    dl /= batch
    # exp and the sum of the softmax: a few u per unit of |z|, and the sum's chain
    tol_dl = np.abs(dl) * HALF[dtype] + (40 + 2 * np.abs(z)) * U * p / batch + 4 * U / batch * (np.abs(dl) > 0)
    dh = (dl @ W.T) * keep
    tol_dh = (tol_dl @ np.abs(W.T) + (classes + 8) * U * (np.abs(dl) @ np.abs(W.T))) * keep
    (dx, tol_dx), (dg, tol_dg), (ds, tol_ds) = _want_backward(dh, x, _np(gain), "f32", 1, 32)
    _, r, h, e, _, _ = _stats(x)
    t = tol_dh * np.abs(_np(gain))  # dx is linear in dy: its coefficients' magnitudes
    tol_dx = tol_dx + r * (t + t.mean(1, keepdims=True) + np.abs(h) * (t * np.abs(h)).mean(1, keepdims=True))
    tol_dg, tol_ds = tol_dg + (tol_dh * np.abs(h)).sum(0) * 1.01, tol_ds + tol_dh.sum(0)
    for got, want, tol, what in ((dgain, dg, tol_dg, "dgain"), (dshift, ds, tol_ds, "dshift")):
        _within(got, want, tol * 1.01, what)
    live = rows > 0
    mask = X[rows[live]] > 0
    got = G[rows[live]]
    want = dx[live] * mask
    tol = tol_dx[live] * mask * 1.01 + HALF[dtype] * np.abs(want) * 1.01
    assert (np.abs(got - want) <= tol + 1e-38).all()
    # the softmax layer's weight gradient reads the stored input
    want, tol = hin.T @ dl, (np.abs(hin).T @ tol_dl + tol_h.T @ (np.abs(dl) + tol_dl)) * 1.01
    tol += (batch + 4) * U * (np.abs(hin).T @ np.abs(dl))
    _within(dW[-1], want, tol * 1.01 + 1e-38, "softmax dW")
    assert torch.isfinite(dfeats).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_head_norm_inference_and_switching_off(dtype):
    from paper_1409_6070_amd.sscn import SSCNError
    net, feats, _, Ws, bs, labels, batch = _net(dtype, 10, None)
    C = net.param_shapes[-1][0]
    plain, _ = net.forward(feats, Ws, bs, labels)
    plain = plain.clone()
    plain_dW = [t.clone() for t in net.backward()[0]]
    gain, shift = torch.full((C,), 1.5, device="cuda"), torch.full((C,), 0.1, device="cuda")
    net.set_head_norm(gain, shift)
    with pytest.raises(SSCNError) as e:
        net.backward()
    assert e.value.name == "SSCN_ERR_BAD_STATE"  # the pass before it is over
    train, _ = net.forward(feats, Ws, bs, labels)
    train = train.clone()
    infer, none = net.forward(feats, Ws, bs, None)
    assert none is None and torch.equal(train, infer) and not torch.equal(train, plain)
    net.set_head_norm(None)
    again, _ = net.forward(feats, Ws, bs, labels)
    assert torch.equal(again, plain)
    assert all(torch.equal(a, b) for a, b in zip(net.backward()[0], plain_dW))


def test_head_norm_gradients_against_differences():
    """dgain and dshift against central differences of the loss."""
    net, feats, _, Ws, bs, labels, batch = _net("f32", 10, None)
    C = net.param_shapes[-1][0]
    g = torch.Generator().manual_seed(3)
    gain, shift = (1 + 0.3 * torch.randn(C, generator=g)).cuda(), (0.2 * torch.randn(C, generator=g)).cuda()
    dgain, dshift = net.set_head_norm(gain, shift)
    net.forward(feats, Ws, bs, labels)
    net.backward()
    dirs = torch.randn(C, generator=g).cuda()
    dg, ds = float((dgain.double() * dirs.double()).sum()), float((dshift.double() * dirs.double()).sum())

    def loss(p, h):
        keep = p.clone()
        p.add_(dirs, alpha=h)
        v = float(net.forward(feats, Ws, bs, labels)[1])
        p.copy_(keep)
        return v

    h = 2.0 ** -6
    for p, got in ((gain, dg), (shift, ds)):
        want = (loss(p, h) - loss(p, -h)) / (2 * h)
        log(f"  differences {want:.6g}, gradient {got:.6g}")
        # h^2/6 of a third derivative that logits changing by |dirs| |W| (a few units) bound by their cube, and the
        # loss's rounding (some u of values near 3) over 2 h
        assert abs(got - want) <= h * h * 30.0 / 6 + 16 * U * 3 / h


@pytest.mark.parametrize("dtype,k", [("f32", 300), ("f32", 512), ("bf16", 600), ("bf16", 1001), ("bf16", 1024)])
def test_head_norm_of_wide_networks(dtype, k):
    """Up to 256 vectors a row in front of the softmax layer (1024 float32 or 2048 bfloat16 channels), the most that
    a network may have. The norm's gradients from the network's own top features, logits and weights."""
    from paper_1409_6070_amd.sscn import SparseDeepCNet
    rng = np.random.default_rng(k)
    ell, c_in, classes, batch, C = 1, 2, 7, 5, 2 * k
    coords = np.concatenate([np.stack([np.full(4, b), *np.divmod(rng.choice(36, 4, replace=False), 6)], 1)
                             for b in range(batch)])
    net = SparseDeepCNet(ell, k, c_in, classes, batch, len(coords), dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    Ws = [(torch.randn(r, c, generator=g, device="cuda") * (2 / r) ** 0.5).to(net.tdtype) for r, c in net.param_shapes]
    bs = [0.1 * torch.randn(c, generator=g, device="cuda") for _, c in net.param_shapes]
    labels = torch.arange(batch, dtype=torch.int32, device="cuda") % classes
    feats = torch.tensor(rng.normal(size=(len(coords), c_in))).to(net.tdtype).cuda()
    net.rulebook_build(torch.tensor(coords, dtype=torch.int32, device="cuda"), batch)
    gain = 1 + 0.3 * torch.randn(C, generator=g, device="cuda")
    shift = 0.2 * torch.randn(C, generator=g, device="cuda")
    dgain, dshift = net.set_head_norm(gain, shift, EPS)
    logits, _ = net.forward(feats, Ws, bs, labels)
    logits = _np(logits)
    net.backward()
    torch.cuda.synchronize()
    view = net.layer_view(net.nlayers - 1)
    rows = np.zeros(batch, dtype=int)
    rows[_np(view["sites"]).astype(int)] = np.arange(1, view["n"] + 1)
    X, G, W = _np(view["features"])[rows, :C], _np(view["grad"])[rows, :C], _np(Ws[-1])
    y, tol = _want_forward(X, _np(gain), _np(shift), dtype)
    want = y @ W + _np(bs[-1])
    tol = tol @ np.abs(W) + (C + 4) * U * (np.abs(y) @ np.abs(W) + np.abs(_np(bs[-1])))
    assert (np.abs(logits - want) <= 1.01 * tol).all()
    z = logits - logits.max(1, keepdims=True)
    p = np.exp(z) / np.exp(z).sum(1, keepdims=True)
    dl = p.copy()
    dl[np.arange(batch), labels.cpu().numpy()] -= 1
    dl /= batch
    tol_dl = np.abs(dl) * HALF[dtype] + (40 + 2 * np.abs(z)) * U * p / batch + 4 * U / batch
    dh, tol_dh = dl @ W.T, tol_dl @ np.abs(W.T) + (classes + 8) * U * (np.abs(dl) @ np.abs(W.T))
    (dx, tol_dx), (dg, tol_dg), (ds, tol_ds) = _want_backward(dh, X, _np(gain), "f32", 1, 32)
    _, r, h, _, _, _ = _stats(X)
    t = tol_dh * np.abs(_np(gain))
    tol_dx = tol_dx + r * (t + t.mean(1, keepdims=True) + np.abs(h) * (t * np.abs(h)).mean(1, keepdims=True))
    _within(dgain, dg, 1.01 * (tol_dg + (tol_dh * np.abs(h)).sum(0)), "dgain")
    _within(dshift, ds, 1.01 * (tol_ds + tol_dh.sum(0)), "dshift")
    mask = X > 0
    assert (np.abs(G - dx * mask) <= 1.01 * (tol_dx * mask + HALF[dtype] * np.abs(dx * mask)) + 1e-38).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [5, 100, 9000])
def test_outputs_side_by_side_and_overlapping(cols, dtype):
    """Columns of one buffer and every other row take part in one call; rows that share elements are refused."""
    from paper_1409_6070_amd.sscn import LayerNorm, SSCNError
    rows = 40
    x, dy, gain, shift = _make(rows, cols, dtype, 0, 4)
    ln = LayerNorm(cols, rows, dtype, EPS)
    want = (ln.forward(x, gain, shift), *ln.backward(dy, x, gain))
    buf = torch.zeros(3 * rows, 3 * cols + 7, dtype=x.dtype, device="cuda")
    side = [buf[:rows, k * cols: (k + 1) * cols] for k in range(3)]
    turn = [buf[k: 3 * rows: 3, 1: cols + 1] for k in range(3)]
    for vx, vy, vd in (side, turn):
        buf.zero_()
        vx.copy_(x), vd.copy_(dy)
        ln.forward(vx, gain, shift, out=vy)
        got = [vy.clone(), *ln.backward(vd, vx, gain, dx=vy)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        vx.zero_(), vy.zero_(), vd.zero_()
        assert (buf == 0).all()
    flat = buf.view(-1)
    for out in (buf[1: rows + 1, :cols], buf[:rows, 1: cols + 1], torch.as_strided(flat, (rows, cols), (cols, 1)),
                buf[:rows, buf.shape[1] - 1:].as_strided((rows, cols), (buf.shape[1], 1), buf.shape[1] - 1)):
        with pytest.raises(SSCNError) as e:
            ln.forward(side[0], gain, shift, out=out)
        assert e.value.name == "SSCN_ERR_INVALID_ARGUMENT"
        for d, v in ((side[0], x), (dy, side[0])):
            with pytest.raises(SSCNError):
                ln.backward(d, v, gain, dx=out)
    assert (buf == 0).all()
    for i in range(2):  # in place in rows with gaps, and x as its own gradient
        side[0].copy_(x)
        ln.forward(side[0], gain, shift, out=side[0])
        assert torch.equal(side[0], want[0])
        side[0].copy_(x)
        both = ln.backward(x, x, gain)
        again = ln.backward(side[0], side[0], gain, dx=side[0])
        assert all(torch.equal(a, b) for a, b in zip(both, again))


def test_a_forward_only_norm_holds_no_workspace():
    """The backward pass's workspace (up to 256 MiB) comes with the first backward pass, and stays."""
    from paper_1409_6070_amd.sscn import LayerNorm
    cols, rows = 100000, 500
    torch.cuda.synchronize()
    base = torch.cuda.memory_allocated()
    ln = LayerNorm(cols, rows, "bf16")
    x = torch.randn(2, cols, device="cuda", dtype=torch.bfloat16)
    own = torch.cuda.memory_allocated()
    ln.forward(x, out=x)
    assert own - base <= 2 * cols * 2 + 4096 and torch.cuda.memory_allocated() == own
    dx, dg, ds = ln.backward(x, x)
    ptr = ln.ws.data_ptr()
    assert torch.cuda.memory_allocated() - own >= ln.ws_bytes > 1 << 26
    again = ln.backward(x, x)
    assert ln.ws.data_ptr() == ptr and all(torch.equal(a, b) for a, b in zip((dx, dg, ds), again))


def test_a_first_backward_inside_a_capture():
    """The workspace that a captured pass brings with it serves the eager passes and graphs behind it."""
    from paper_1409_6070_amd.sscn import LayerNorm
    x, dy, gain, _ = _make(500, 300, "bf16", 0, 21)
    want = LayerNorm(300, 500, "bf16", EPS).backward(dy, x, gain)
    ln = LayerNorm(300, 500, "bf16", EPS)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        dx = torch.empty_like(x)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = ln.backward(dy, x, gain, dx=dx)
        graphs.append((g, got))
    for i in range(3):
        for g, got in graphs:
            for t in got:
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), i
            assert all(torch.equal(a, b) for a, b in zip(ln.backward(dy, x, gain), want)), i
    graphs.pop(0)  # its memory pool goes, the workspace stays
    torch.cuda.empty_cache()
    torch.empty(1 << 24, device="cuda").fill_(float("nan"))
    for i in range(3):
        g, got = graphs[0]
        for t in got:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        assert all(torch.equal(a, b) for a, b in zip(ln.backward(dy, x, gain), want)), i


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [5, 100, 3000, 40000])
def test_parameter_gradients_that_are_not_wanted(cols, dtype):
    """Each of dgain and dshift may be null; without both no workspace is needed. The others keep their bits."""
    from paper_1409_6070_amd import sscn
    rows = 70
    x, dy, gain, _ = _make(rows, cols, dtype, 0, 15)
    ln = sscn.LayerNorm(cols, rows, dtype, EPS)
    want = ln.backward(dy, x, gain)
    for wants in ((1, 0), (0, 1), (0, 0)):
        dx = torch.zeros_like(x)
        out = [torch.full((cols,), 7.5, device="cuda") for _ in range(2)]
        sscn.sscn_layer_norm_backward(ln.code, dy.data_ptr(), cols, x.data_ptr(), cols, rows, cols, gain.data_ptr(), EPS,
                                      dx.data_ptr(), cols, *[o.data_ptr() if w else None for o, w in zip(out, wants)],
                                      ln.ws.data_ptr() if any(wants) else None, ln.ws_bytes if any(wants) else 0,
                                      sscn._stream())
        torch.cuda.synchronize()
        assert torch.equal(dx, want[0])
        for o, w, p in zip(out, wants, want[1:]):
            assert torch.equal(o, p) if w else (o == 7.5).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("drop", [None, 0.4])
def test_head_norm_of_a_network_in_network(dtype, drop):
    """DeepCNiN: the leaky rectifier below the norm, several empty samples on one ground row. The norm's gradients and
    the top layer's from the network's own top features, logits and weights."""
    from paper_1409_6070_amd.sscn import SparseDeepCNet
    from workloads import he_params, random_labels
    rng = np.random.default_rng(5)
    ell, k, c_in, classes, batch = 2, 11, 3, 12, 19
    N, empty = 3 * 2 ** ell, (0, 4, 5, 18)
    coords = np.concatenate([np.stack([np.full(6, b), *np.divmod(rng.choice(N * N, 6, replace=False), N)], 1)
                             for b in range(batch) if b not in empty])
    net = SparseDeepCNet(ell, k, c_in, classes, batch, len(coords), dtype, arch="deepcnin", dropout=drop is not None)
    feats = torch.tensor(rng.normal(size=(len(coords), c_in))).to(net.tdtype).cuda()
    Ws, bs = he_params(ell, k, c_in, classes, 1, arch="deepcnin")
    Ws = [torch.tensor(w, dtype=torch.float32, device="cuda").to(net.tdtype) for w in Ws]
    bs = [torch.tensor(v, dtype=torch.float32, device="cuda") + 0.05 for v in bs]
    labels = torch.tensor(random_labels(batch, classes, 2), dtype=torch.int32, device="cuda")
    if drop is not None:
        net.set_dropout([0.0] * (ell + 1) + [drop], 91)
    net.rulebook_build(torch.tensor(coords, dtype=torch.int32, device="cuda"), batch)
    C = net.param_shapes[-1][0]
    g = torch.Generator().manual_seed(3)
    gain, shift = (1 + 0.3 * torch.randn(C, generator=g)).cuda(), (0.2 * torch.randn(C, generator=g)).cuda()
    dgain, dshift = net.set_head_norm(gain, shift, EPS)
    logits = _np(net.forward(feats, Ws, bs, labels)[0])
    net.backward()
    torch.cuda.synchronize()
    view = net.layer_view(net.nlayers - 1)
    rows = np.zeros(batch, dtype=int)
    rows[_np(view["sites"]).astype(int)] = np.arange(1, view["n"] + 1)
    assert set(np.flatnonzero(rows == 0)) == set(empty)
    x, W = _np(view["features"])[rows, :C], _np(Ws[-1])
    assert (x < 0).any() and (x > 0).any()
    keep = np.ones((batch, C)) if drop is None else _keep(batch, C, ell + 1, drop, 91)
    y, tol_y = _want_forward(x, _np(gain), _np(shift), dtype)
    tol_y = tol_y * keep + (0 if drop is None else (HALF[dtype] + U) * np.abs(y * keep) * 1.01)
    want = (y * keep) @ W + _np(bs[-1])
    tol = tol_y @ np.abs(W) + (C + 4) * U * (np.abs(y * keep) @ np.abs(W) + np.abs(_np(bs[-1])))
    assert (np.abs(logits - want) <= 1.01 * tol).all()
    z = logits - logits.max(1, keepdims=True)
    p = np.exp(z) / np.exp(z).sum(1, keepdims=True)
    dl = p.copy()
    dl[np.arange(batch), labels.cpu().numpy()] -= 1
    dl /= batch
    tol_dl = np.abs(dl) * HALF[dtype] + (40 + 2 * np.abs(z)) * U * p / batch + 4 * U / batch
    dh, tol_dh = (dl @ W.T) * keep, (tol_dl @ np.abs(W.T) + (classes + 8) * U * (np.abs(dl) @ np.abs(W.T))) * keep
    (dx, tol_dx), (dg, tol_dg), (ds, tol_ds) = _want_backward(dh, x, _np(gain), "f32", 1, 32)
    _, r, h, _, _, _ = _stats(x)
    t = tol_dh * np.abs(_np(gain))
    tol_dx = tol_dx + r * (t + t.mean(1, keepdims=True) + np.abs(h) * (t * np.abs(h)).mean(1, keepdims=True))
    _within(dgain, dg, 1.01 * (tol_dg + (tol_dh * np.abs(h)).sum(0)), "dgain")
    _within(dshift, ds, 1.01 * (tol_ds + tol_dh.sum(0)), "dshift")
    live = rows > 0
    slope = np.where(x[live] >= 0, 1.0, 1.0 / 3.0)
    got, want = _np(view["grad"])[rows[live], :C], dx[live] * slope
    assert (np.abs(got - want) <= 1.01 * (tol_dx[live] * slope + (HALF[dtype] + 2 * U) * np.abs(want)) + 1e-38).all()
