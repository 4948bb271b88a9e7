"""Rows and matrices held in 8 bits and their products, on the GPU.

The codes are compared exactly, with a table of e4m3's values made from its definition.  Products are compared exactly
on small whole numbers (every product and partial sum fits the instructions' narrowest sums), and on random values
against 64 bits.

Bounds.  u = 2^-24.  Results in float32: products of codes are exact, a sum in which a term passes at most D additions
is off by at most D u sum|terms|; one instruction adds 32 products, one follows the other: D = 32 + terms / 32 + 4, where
waves share a sum eight more, and the parts of a weight gradient's rows add their number.  Results in bf16: of eight products what lies under 2^-13 of
the largest may be dropped: at most 7 * 2^-13 sum|terms| beside the rounding of 2^-8; as a whole (2-norm) the roundings
alone make at most 2^-8 and 2^-9 in the root mean square over mantissas spread over an octave (half a step is between
2^-9 and 2^-8 of a value: 2^-8 / sqrt 3 times the mean of that over the octave, under 0.0018), to which errors of
random sign add in squares."""

import numpy as np
import pytest
import torch

from tests.gpu_harness import log

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True, scope="module")
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1409_6070_amd import sscn
    sscn.load_library()


def _table():
    """The values of codes 0 .. 126: three bits of fraction, four of exponent with bias 7, code 127 is NaN."""
    c = np.arange(127)
    e, f = c >> 3, c & 7
    return np.where(e == 0, f * 2.0 ** -9, (1 + f / 8) * 2.0 ** (e - 7.0))


TABLE = _table()


def _round(v):
    """|v| <= 448 to the nearest value of the table, ties to the even code."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(TABLE, a), 1, 126)
    lo = hi - 1
    dl, dh = a - TABLE[lo], TABLE[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.copysign(TABLE[code], v)


def _exponent(most):
    """The least e >= -126 with most <= 448 2^e."""
    e = -126
    while most > 448.0 * 2.0 ** e:
        e += 1
    return e


def _held(x):
    """Values and exponents of rows x (64 bits): [rows, cols], [rows, blocks]."""
    rows, cols = x.shape
    nb = -(-cols // 128)
    out, exps = np.empty_like(x), np.empty((rows, nb), int)
    for b in range(nb):
        p = x[:, b * 128: b * 128 + 128]
        ok = np.isfinite(p)
        most = np.where(ok, np.abs(p), 0).max(1)
        es = {m: _exponent(m) for m in set(most)}
        exps[:, b] = [es[m] for m in most]
        s = 2.0 ** exps[:, b, None]
        out[:, b * 128: b * 128 + 128] = np.where(ok, _round(np.where(ok, p, 0) / s) * s, np.nan)
    return out, exps


def _held_matrix(w):
    out = np.empty_like(w)
    for k in range(0, w.shape[0], 128):
        for n in range(0, w.shape[1], 128):
            p = w[k: k + 128, n: n + 128]
            s = 2.0 ** _exponent(np.abs(p).max())
            out[k: k + 128, n: n + 128] = _round(p / s) * s
    return out


def _values(rows, cols, dtype, seed):
    """Blocks of very different size, with zeros."""
    g = np.random.default_rng(seed)
    x = g.normal(size=(rows, cols)) * np.exp(3 * g.normal(size=(rows, cols))) * (g.random((rows, cols)) < 0.8)
    x *= 2.0 ** g.integers(-20, 20, size=(rows, 1))
    return torch.tensor(x, dtype=torch.float32).to(TORCH[dtype])


def _np(t):
    return t.double().cpu().numpy()


def _wide(t, pad):
    """t on the GPU as columns of a wider buffer."""
    rows, cols = t.shape
    buf = torch.full((rows, cols + 2 * pad), 7.0, dtype=t.dtype, device="cuda")
    buf[:, pad: pad + cols] = t.cuda()
    return buf, buf[:, pad: pad + cols]


COLS = [1, 2, 7, 8, 15, 16, 17, 50, 127, 128, 129, 130, 255, 257, 300, 513, 1000, 4099, 8200]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_store_and_load(cols, dtype):
    from paper_1409_6070_amd.sscn import Rows8
    for rows, pad in ((1, 0), (5, 3), (67, 1)):
        x = _values(rows, cols, dtype, cols + rows)
        r = Rows8(rows, cols)
        r.codes.fill_(255), r.scales.fill_(255)
        r.store(_wide(x, pad)[1])
        want, exps = _held(_np(x))
        nb = exps.shape[1]
        scales = r.scales.cpu().numpy()
        assert (scales[:, :nb] == exps + 127).all() and (scales[:, nb:] == 0).all()
        codes = r.codes.cpu()
        assert (codes[:, cols:] == 0).all()
        assert (np.signbit(_np(codes[:, :cols].view(torch.float8_e4m3fn))) == np.signbit(_np(x))).all()
        for to in ("f32", "bf16"):
            buf = torch.full((rows, cols + 2 * pad), 7.0, dtype=TORCH[to], device="cuda")
            y = r.load(out=buf[:, pad: pad + cols]) if pad else r.load(to)
            assert (_np(y) == want).all(), (rows, to)
            if pad:
                assert (buf[:, :pad] == 7).all() and (buf[:, pad + cols:] == 7).all()


def test_values_at_borders():
    """The largest value of a block at, below and behind 448 2^e; ties; zeros; the ends of float32's range."""
    from paper_1409_6070_amd.sscn import Rows8
    tie = [1.0625, 1.1875, 1.3125, -1.0625, -1.4375, 2.0 ** -9 * 0.5, 2.0 ** -9 * 1.5, 2.0 ** -9 * 2.5, -(2.0 ** -10), 0.0, -0.0]
    rows = []
    for e in (-120, -20, -1, 0, 1, 30, 110):
        for most in (448.0, np.nextafter(np.float32(448), np.float32(0)), np.nextafter(np.float32(448), np.float32(1e9)),
                     224.0, 225.0, 256.0, 511.0):
            rows.append([float(most) * 2.0 ** e] + [t * 2.0 ** e for t in tie])
    rows += [[0.0] * 12, [-0.0] * 12, [2.0 ** -149] + [0.0] * 11, [2.0 ** -126] + [2.0 ** -130] * 11,
             [448 * 2.0 ** -126] + [2.0 ** -135, 2.0 ** -136, 2.0 ** -137] + [0.0] * 8, [3.0e38] + [1e38, -2e38] + [1.0] * 9]
    x = torch.tensor(rows, dtype=torch.float64).float()
    r = Rows8(*x.shape).store(x.cuda())
    want, _ = _held(_np(x))
    assert (_np(r.load("f32")) == want).all()


def test_nan_and_infinities_stay_alone():
    from paper_1409_6070_amd.sscn import Rows8
    x = _values(9, 300, "f32", 5)
    bad = [(1, 0, np.nan), (1, 200, np.inf), (2, 127, -np.inf), (2, 128, np.nan), (4, 299, np.inf)]
    for r, c, v in bad:
        x[r, c] = v
    x[5] = np.nan
    for dtype in ("f32", "bf16"):
        t = x.to(TORCH[dtype])
        got = _np(Rows8(9, 300).store(t.cuda()).load("f32"))
        want, _ = _held(_np(t))
        assert (np.isnan(got) == np.isnan(want)).all() and np.isnan(got).sum() == 305
        assert (got[np.isfinite(want)] == want[np.isfinite(want)]).all()


@pytest.mark.parametrize("bits", [0x7f800001, 0x7fa55555, 0x7fbfffff, 0x7fc00000, 0x7fffffff])
def test_every_kind_of_nan_leaves_its_block_alone(bits):
    """Signalling ones too, before, at and behind the place of the block's largest value."""
    from paper_1409_6070_amd.sscn import Product8, Rows8
    at = torch.arange(24)
    for most in (0, 7, 9, 23):
        for sign in (0, 1 << 31):
            x = torch.ones(24, 130)
            x[:, most] = 300.0
            clean = _held(_np(x))[0]
            v = np.array([bits | sign], dtype=np.uint32).view(np.int32)[0]
            x.view(torch.int32)[at, at] = int(v)
            for t in (x, (x.view(torch.int32) >> 16).to(torch.int16).view(torch.bfloat16)):
                if not t.float().isnan()[at, at].all():
                    continue  # (a NaN whose upper half is an infinity's)
                got = _np(Rows8(24, 130).store(t.cuda()).load("f32"))
                assert np.isnan(got[at, at]).all() and np.isnan(got).sum() == 24
                assert (got == clean)[~np.isnan(got)].all()
            w = x[most].clone()[None].repeat(130, 1)  # a column of NaN
            w[0, 1] = 300.0                           # 288 in steps of 32
            layer = Product8(130, 130, 1, "f32").set_weights(w.cuda())
            e = torch.zeros(1, 130)
            e[0, 0] = 1.0
            y = _np(layer.forward(Rows8(1, 130).store(e.cuda())))[0]
            assert np.isnan(y[most]) and np.isnan(y).sum() == 1 and y[1] == 288.0


def test_offsets_past_32_bits():
    from paper_1409_6070_amd.sscn import Rows8
    rows, cols = (1 << 20) + 77, 4099  # codes 4.3e9 bytes, x 8.6e9
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    tail = _values(70, cols, "bf16", 3)
    x[-70:] = tail.cuda()
    r = Rows8(rows, cols).store(x)
    y = r.load("bf16", out=x)
    assert (_np(y[-70:]) == _held(_np(tail))[0]).all()
    part = r.rows_from(rows - 70, rows)
    assert (_np(part.load("f32")) == _held(_np(tail))[0]).all()


def test_no_rows():
    from paper_1409_6070_amd.sscn import Product8, Rows8
    r = Rows8(0, 50).store(torch.empty(0, 50, device="cuda"))
    assert r.load("f32").shape == (0, 50)
    p = Product8(50, 30, 100).set_weights(torch.ones(50, 30, device="cuda"))
    assert p.forward(r).shape == (0, 30) and p.input_grad(Rows8(0, 30)).shape == (0, 50)
    dw, db = p.weight_grad(r, Rows8(0, 30))
    assert (dw == 0).all() and (db == 0).all()


# ---------------------------------------------------------------------------------------------------------
# products

SHAPES = [(1, 1, 1), (1, 300, 3755), (2, 16, 17), (5, 129, 130), (16, 128, 64), (17, 127, 128), (33, 1000, 48), (100, 300, 3755),
          (127, 50, 65), (128, 256, 256), (129, 257, 255), (300, 513, 300), (1000, 64, 1000), (2049, 300, 300), (513, 1025, 129),
          (257, 4099, 33), (64, 2050, 520)]


def _ints(rows, cols, seed, most=3):
    g = np.random.default_rng(seed)
    return torch.tensor(g.integers(-most, most + 1, size=(rows, cols)), dtype=torch.float32)


@pytest.mark.parametrize("rows,k,n", SHAPES)
def test_products_of_whole_numbers_are_exact(rows, k, n):
    """Entries of -1 .. 1 (bf16) and -3 .. 3 (float32): every sum is exact, and so is its rounding here."""
    from paper_1409_6070_amd.sscn import Product8, Rows8
    for dtype, most in (("bf16", 1), ("f32", 3)):
        x, w, dy = _ints(rows, k, 1, most), _ints(k, n, 2, most), _ints(rows, n, 3, most)
        bias = _ints(1, n, 4)[0]
        p = Product8(k, n, rows, dtype).set_weights(w.cuda())
        x8, dy8 = Rows8(rows, k).store(x.cuda()), Rows8(rows, n).store(dy.cuda())
        xd, wd, dyd = x.double(), w.double(), dy.double()
        to = TORCH[dtype]
        assert torch.equal(p.forward(x8, bias.cuda()).cpu(), (xd @ wd + bias.double()).to(to)), "forward"
        assert torch.equal(p.input_grad(dy8).cpu(), (dyd @ wd.t()).to(to)), "input gradient"
        dw, db = p.weight_grad(x8, dy8)
        assert torch.equal(dw.cpu().double(), xd.t() @ dyd) and torch.equal(db.cpu().double(), dyd.sum(0)), "weight gradient"


def _inside(got, want, tol, what):
    got = _np(got)
    worst = float((np.abs(got - want) / tol).max())
    log(f"  {what}: at most {worst:.3f} of the bound")
    assert np.isfinite(got).all() and worst <= 1.0, what


def _product_bound(a, b, dtype):
    """[m, k] @ [k, n] in 64 bits, with the bound of each entry."""
    want, mag = a @ b, np.abs(a) @ np.abs(b)
    D = 32 + a.shape[1] / 32 + 4 + 8
    if dtype == "f32":
        return want, D * U * mag + 1e-300
    return want, (7 * 2.0 ** -13 + D * U) * mag + 2.0 ** -8 * np.abs(want) + 1e-300


def _norm(got, want):
    return float(np.linalg.norm(_np(got) - want) / np.linalg.norm(want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k,n", SHAPES)
def test_products(rows, k, n, dtype):
    from paper_1409_6070_amd.sscn import Product8, Rows8
    log(f"[products] {rows} x {k} x {n} {dtype}")
    x, w, dy = (torch.randn(s, generator=torch.Generator().manual_seed(i)) for i, s in enumerate(((rows, k), (k, n), (rows, n))))
    x = torch.where(x < 0, x / 3, x) * 2.0 ** torch.randint(-9, 9, (rows, 1), generator=torch.Generator().manual_seed(4))
    dy = dy * 1e-3
    bias = torch.randn(n, generator=torch.Generator().manual_seed(5))
    x, w, dy = (t.to(TORCH[dtype]) for t in (x, w, dy))
    p = Product8(k, n, rows, dtype).set_weights(_wide(w, 3)[1])
    x8, dy8 = Rows8(rows, k).store(x.cuda()), Rows8(rows, n).store(dy.cuda())
    xq, wq, dyq = _held(_np(x))[0], _held_matrix(_np(w)), _held(_np(dy))[0]
    b = bias.double().numpy()

    want, tol = _product_bound(xq, wq, dtype)
    buf, y = _wide(torch.zeros(rows, n, dtype=TORCH[dtype]), 5)
    p.forward(x8, bias.cuda(), out=y)
    half = U if dtype == "f32" else 2.0 ** -8
    _inside(y, want + b, tol + 2 * half * (np.abs(want) + np.abs(b)), "y")
    assert (buf[:, :5] == 7).all() and (buf[:, 5 + n:] == 7).all()
    if dtype == "bf16" and rows * n > 1000:
        assert _norm(p.forward(x8), want) < 0.0018 + 1e-4
    want, tol = _product_bound(dyq, wq.T, dtype)
    dx = p.input_grad(dy8)
    _inside(dx, want, tol, "dx")
    if dtype == "bf16" and rows * k > 1000:
        assert _norm(dx, want) < 0.0018 + 1e-4
    dw, db = p.weight_grad(x8, dy8)
    D = 32 + rows / 32 + 4 + 512
    _inside(dw, xq.T @ dyq, D * U * (np.abs(xq).T @ np.abs(dyq)) + 1e-300, "dw")
    _inside(db, dyq.sum(0), D * U * np.abs(dyq).sum(0) + 1e-300, "db")


@pytest.mark.parametrize("rows,k,n", [(8187, 2050, 2040), (16400, 4100, 2048), (40000, 129, 300), (3000, 520, 515), (260, 4099, 4101)])
def test_large_products_of_whole_numbers(rows, k, n):
    """The large tiles, several of them to a workgroup, results that go past the caches; sums checked in 64 bits on the
    GPU.  Entries are -1 .. 1: every sum is exact, rounded once to bf16."""
    from paper_1409_6070_amd.sscn import Product8, Rows8
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, w, dy = (torch.randint(-1, 2, s, generator=g, device="cuda").float() for s in ((rows, k), (k, n), (rows, n)))
    x8, dy8 = Rows8(rows, k).store(x), Rows8(rows, n).store(dy)
    xd, wd, dyd = x.double(), w.double(), dy.double()
    y, dx = torch.mm(xd, wd), torch.mm(dyd, wd.t().contiguous())
    for dtype in ("bf16", "f32"):
        p = Product8(k, n, rows, dtype).set_weights(w)
        assert torch.equal(p.forward(x8), y.to(TORCH[dtype])), "forward"
        assert torch.equal(p.input_grad(dy8), dx.to(TORCH[dtype])), "input gradient"
    dw, db = p.weight_grad(x8, dy8)
    assert torch.equal(dw.double(), torch.mm(xd.t().contiguous(), dyd)) and torch.equal(db.double(), dyd.sum(0))


@pytest.mark.parametrize("rows,k,n", [(0, 5, 3), (64, 128, 128), (65, 1, 1), (128, 257, 129), (129, 130, 1), (191, 1, 300),
                                      (193, 256, 256), (65600, 1, 1), (70001, 128, 127), (33000, 256, 257), (5000, 1030, 700)])
def test_rows_of_weight_gradients_are_divided(rows, k, n):
    """From one workgroup a tile to hundreds, whose runs of rows are of unequal lengths: exact sums of whole numbers (a
    column of at most 70001 x 1), nothing behind the workspace and beside the result, and the same with no bias gradient."""
    from paper_1409_6070_amd import sscn
    g = torch.Generator(device="cuda").manual_seed(rows + k)
    x, dy = (torch.randint(-1, 2, (rows, c), generator=g, device="cuda").float() for c in (k, n))
    x8, dy8 = sscn.Rows8(rows, k).store(x), sscn.Rows8(rows, n).store(dy)
    need = sscn.sscn_product8_weight_grad_workspace_bytes(rows, k, n)
    ws = torch.full((need + 4096,), 0x7f, dtype=torch.uint8, device="cuda")
    want = torch.mm(x.double().t().contiguous(), dy.double())
    st = torch.cuda.current_stream().cuda_stream
    for with_db in (True, False):
        buf = torch.full((k, n + 5), 7.0, device="cuda")
        db = torch.full((n + 5,), 7.0, device="cuda")
        sscn.sscn_product8_weight_grad(x8.call, dy8.call, buf.data_ptr(), n + 5, db.data_ptr() if with_db else None,
                                       ws.data_ptr(), need, st)
        torch.cuda.synchronize()
        assert torch.equal(buf[:, :n].double(), want) and (buf[:, n:] == 7).all() and (ws[need:] == 0x7f).all()
        assert (db[n:] == 7).all()
        assert torch.equal(db[:n].double(), dy.double().sum(0)) if with_db else (db == 7).all()


def test_two_plans_at_once():
    """Each with its own workspace, on a stream of its own, over the same 8-bit rows."""
    from paper_1409_6070_amd.sscn import Product8, Rows8
    rows, k, n = 20000, 512, 300
    g = torch.Generator(device="cuda").manual_seed(1)
    x8, dy8 = (Rows8(rows, c).store(torch.randn(rows, c, generator=g, device="cuda")) for c in (k, n))
    ps = [Product8(k, n, rows, d).set_weights(torch.randn(k, n, generator=g, device="cuda")) for d in ("bf16", "f32")]
    step = lambda p: (p.forward(x8), p.input_grad(dy8), *p.weight_grad(x8, dy8))
    want = [step(p) for p in ps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ps]
    got = []
    for _ in range(3):
        for p, s in zip(ps, streams):
            with torch.cuda.stream(s):
                got.append(step(p))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want[i % 2]))


@pytest.mark.parametrize("rows,cols", [(20000, 1024), (40001, 1000)])
def test_large_loads(rows, cols):
    """Results that go past the caches, of whole lines and not."""
    from paper_1409_6070_amd.sscn import Rows8
    r = Rows8(rows, cols).store(torch.randn(rows, cols, device="cuda"))
    a, b = r.load("f32"), r.load("bf16")
    assert torch.equal(a, b.float())
    part = r.rows_from(rows - 50, rows)
    assert torch.equal(part.load("f32"), a[-50:])


@pytest.mark.parametrize("k,n", [(1, 1), (130, 257), (300, 129), (128, 128)])
def test_matrix_is_held_in_blocks(k, n):
    """Rows of the unit matrix read it back, either way (float32: exactly)."""
    from paper_1409_6070_amd.sscn import Product8, Rows8
    w = _values(k, n, "f32", 11)
    want = _held_matrix(_np(w))
    for t in (w, w.to(torch.bfloat16)):
        if t.dtype != torch.float32:
            want = _held_matrix(_np(t))
        p = Product8(k, n, 512, "f32").set_weights(t.cuda())
        assert (_np(p.forward(Rows8(k, k).store(torch.eye(k, device="cuda")))) == want).all()
        assert (_np(p.input_grad(Rows8(n, n).store(torch.eye(n, device="cuda")))) == want.T).all()


def test_gradients_against_differences():
    """Each entry of w and x moves the loss by its gradient: products are linear, so whole steps are exact."""
    from paper_1409_6070_amd.sscn import Product8, Rows8
    rows, k, n = 7, 20, 18
    x, w, dy = _ints(rows, k, 1), _ints(k, n, 2), _ints(rows, n, 3)
    p = Product8(k, n, rows, "f32").set_weights(w.cuda())
    x8, dy8 = Rows8(rows, k).store(x.cuda()), Rows8(rows, n).store(dy.cuda())
    loss = lambda: float((p.forward(Rows8(rows, k).store(x.cuda())).cpu() * dy).double().sum())  # noqa: E731
    base, dx = loss(), p.input_grad(dy8).cpu()
    dw, db = (t.cpu() for t in p.weight_grad(x8, dy8))
    for i, j in ((0, 0), (3, 17), (6, 19)):
        x[i, j] += 1
        assert loss() - base == float(dx[i, j])
        x[i, j] -= 1
    for i, j in ((0, 0), (19, 17), (7, 3)):
        w[i, j] += 1
        p.set_weights(w.cuda())
        assert loss() - base == float(dw[i, j])
        w[i, j] -= 1
    assert torch.equal(db, dy.sum(0))


def test_products_of_the_smallest_values():
    """Held values from 2^-130 on are exact in float32 products, at every number of rows that takes another kernel; smaller
    ones are taken in steps of 2^-133, each off by half a step at most."""
    from paper_1409_6070_amd.sscn import Product8, Rows8
    k, n = 300, 200
    g = torch.Generator().manual_seed(3)
    for rows in (1, 20, 60, 3000, 9000):
        m, j, q = (torch.randint(-8, 9, s, generator=g).float() for s in ((rows, k), (k, n), (rows, n)))
        for low in (0, 5):  # (x 2^-5: values under 2^-130 too)
            x = (m.double() * 2.0 ** (-130 - low)).float()
            p = Product8(k, n, rows, "f32").set_weights((j * 2.0 ** 60).cuda())
            x8, dy8 = Rows8(rows, k).store(x.cuda()), Rows8(rows, n).store((q * 2.0 ** 60).cuda())
            held = _np(x8.load("f32"))
            assert low or (held == _np(x)).all()
            w, dy = _np(j) * 2.0 ** 60, _np(q) * 2.0 ** 60
            y, dw = _np(p.forward(x8)), _np(p.weight_grad(x8, dy8)[0])
            if low == 0:  # whole numbers up to 64 * 9000 of 2^-70
                assert (y == held @ w).all() and (dw == held.T @ dy).all()
            else:
                off = 2.0 ** -134 * (np.abs(held) < 2.0 ** -130)
                for got, a, b, terms in ((y, held, w, k), (dw, held.T, dy, rows)):
                    bound = (off if a is held else off.T) @ np.abs(b)
                    assert (np.abs(got - a @ b) <= bound + (44 + terms / 32 + 520) * U * (np.abs(a) @ np.abs(b) + bound)).all()


def test_a_nan_stays_in_its_row():
    from paper_1409_6070_amd.sscn import Product8, Rows8
    for dtype in ("f32", "bf16"):
        x, w = torch.randn(300, 200, device="cuda"), torch.randn(200, 150, device="cuda")
        p = Product8(200, 150, 300, dtype).set_weights(w)
        clean = p.forward(Rows8(300, 200).store(x))
        x[130, 199], x[7, 0] = float("nan"), float("inf")
        y = p.forward(Rows8(300, 200).store(x))
        rest = torch.ones(300, dtype=torch.bool)
        rest[[7, 130]] = False
        assert y[[7, 130]].isnan().all() and torch.equal(y[rest.cuda()], clean[rest.cuda()])


def test_many_rows_and_offsets_past_32_bits():
    """Codes and results of more than 2^32 bytes; the last rows and the sums over all of them."""
    from paper_1409_6070_amd.sscn import Product8, Rows8
    rows, k, n = (1 << 20) + 131, 4112, 20
    r = Rows8(rows, k)
    r.codes.zero_(), r.scales.fill_(127)
    tail = _ints(131, k, 1, 1)
    r.rows_from(rows - 131, rows).store(tail.cuda())
    w = _ints(k, n, 2, 1)
    for dtype in ("bf16", "f32"):
        p = Product8(k, n, rows, dtype).set_weights(w.cuda())
        y = p.forward(r)
        assert (y[:-131] == 0).all() and torch.equal(y[-131:].cpu(), (tail.double() @ w.double()).to(TORCH[dtype]))
        dy = torch.zeros(rows, n, device="cuda")
        dy[-131:] = _ints(131, n, 3, 1).cuda()
        dw, db = p.weight_grad(r, Rows8(rows, n).store(dy))
        assert torch.equal(dw.cpu().double(), tail.double().t() @ dy[-131:].cpu().double()) and torch.equal(db, dy.sum(0))


def test_streams_and_graphs():
    """The same bits on another stream and from a graph that is replayed on new values, eager calls between."""
    from paper_1409_6070_amd.sscn import Product8, Rows8
    rows, k, n = 333, 300, 210
    for dtype in ("bf16", "f32"):
        p = Product8(k, n, rows, dtype)
        xs = [torch.randn(rows, k, device="cuda") for _ in range(3)]
        dys = [torch.randn(rows, n, device="cuda") for _ in range(3)]
        ws = [torch.randn(k, n, device="cuda") for _ in range(3)]
        x, dy, w = xs[0].clone(), dys[0].clone(), ws[0].clone()
        x8, dy8 = Rows8(rows, k), Rows8(rows, n)
        y, dx, dw = (torch.empty(s, dtype=t, device="cuda") for s, t in
                     (((rows, n), TORCH[dtype]), ((rows, k), TORCH[dtype]), ((k, n), torch.float32)))

        def step():
            p.set_weights(w)
            p.forward(x8.store(x), out=y)
            p.input_grad(dy8.store(dy), out=dx)
            return p.weight_grad(x8, dy8, out=dw)[1]

        def values(i):
            x.copy_(xs[i]), dy.copy_(dys[i]), w.copy_(ws[i])

        want = []
        for i in range(3):
            values(i)
            db = step()
            want.append([t.clone() for t in (y, dx, dw, db)])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            values(1)
            db = step()
            assert all(torch.equal(a, b) for a, b in zip((y, dx, dw, db), want[1]))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            db = step()
        for i in (0, 2, 1, 0):
            values(i)
            for t in (y, dx, dw):
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((y, dx, dw, db), want[i]))
            values((i + 1) % 3)
            step()
            torch.cuda.synchronize()


def test_binding_refuses():
    from paper_1409_6070_amd.sscn import Product8, Rows8, SSCNError
    x = torch.zeros(4, 50, device="cuda")
    r = Rows8(4, 50)
    for bad in (x.half(), x[:3], x[:, :49], x.t(), x.cpu()):
        with pytest.raises(ValueError):
            r.store(bad)
        with pytest.raises(ValueError):
            r.load(out=bad)
    for kw in (dict(codes=torch.zeros(4, 50, dtype=torch.uint8, device="cuda")), dict(scales=torch.zeros(4, 1, device="cuda")),
               dict(codes=torch.zeros(4, 128, dtype=torch.uint8, device="cuda")[:, :64])):
        with pytest.raises(ValueError):
            Rows8(4, 50, **kw)
    odd = torch.zeros(4 * 64 + 8, dtype=torch.uint8, device="cuda")[8:].view(4, 64)  # 8-byte aligned
    with pytest.raises(SSCNError):
        Rows8(4, 50, codes=odd).store(x)
    p = Product8(50, 30, 4)
    with pytest.raises(ValueError):
        p.forward(r)  # no weights yet
    p.set_weights(torch.zeros(50, 30, device="cuda"))
    for call in (lambda: p.forward(Rows8(4, 51)), lambda: p.input_grad(r), lambda: p.forward(x),
                 lambda: p.forward(r, bias=torch.zeros(29, device="cuda")), lambda: p.set_weights(x),
                 lambda: p.forward(r, out=torch.zeros(4, 30, device="cuda")),
                 lambda: p.weight_grad(r, Rows8(3, 30)), lambda: p.weight_grad(Rows8(5, 50), Rows8(5, 30))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        Rows8(4, 50).rows_from(2, 5)
    for kn in ((0, 5), (5, 0), (65537, 5)):
        with pytest.raises(SSCNError):
            Product8(*kn, 4)
