"""Newton-Schulz orthogonalisation and Muon's update on the GPU, against the formula in 64 bits.

Bound of the orthogonalisation, as a 2-norm relative to the result.  Two sources of error, both propagated through
the steps for the very matrix at hand, since the steps multiply an early error by the derivatives p'(s) that its
singular values meet (up to 4 each):

* float32 sums and roundings: the distance of the same steps computed here in float32;
* operands split into two fp16 numbers: hi is off by at most 2^-11 of the entry, lo by at most 2^-11 of that, so the
  operand by 2^-22 of the entry; the dropped lo lo is at most 2^-22 of the product.  Together at most 1.5 2^-22 of
  each operand: the steps in 64 bits with every operand entry of every product off by that much, with random signs
  (the largest distance of four trials).

Three times their sum, and half a step of the result's type."""

import math

import numpy as np
import pytest
import torch

from tests.gpu_harness import log

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
MUON = (3.4445, -4.7750, 2.0315)


@pytest.fixture(autouse=True, scope="module")
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1409_6070_amd import sscn
    sscn.load_library()


def ns(u, dt, coef=MUON, steps=5, off=None):
    """The formula in dtype dt where u lies, with coefficients as float32 holds them; off: a generator of the signs
    that put every product's operands off by 1.5 2^-22."""
    def o(t):
        if off is None:
            return t
        return t * (1 + 1.5 * 2.0 ** -22 * (2 * torch.randint(0, 2, t.shape, generator=off, device=t.device) - 1))
    rows = [coef] * steps if not hasattr(coef[0], "__len__") else coef
    x = u.double()
    norm = x.norm()
    x = (x / norm if norm > 0 else x).to(dt)
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    for r in rows:
        a, b, c = (float(np.float32(v)) for v in r)
        g = o(x) @ o(x).t()
        x = a * x + o(b * g + c * (o(g) @ o(g))) @ o(x)
    return x.t() if tall else x


def _bound(u, dtype, coef=MUON, steps=5):
    # (large matrices: on the GPU, by the library's products)
    u = (u.cpu() if u.numel() < 4 * 10 ** 6 else u).float()
    want = ns(u, torch.float64, coef, steps)
    f32 = ns(u, torch.float32, coef, steps).double()
    scale = max(want.norm().item(), 1e-300)
    off32 = (f32 - want).norm().item() / scale
    off22 = max((ns(u, torch.float64, coef, steps, torch.Generator(u.device).manual_seed(k)) - want).norm().item()
                for k in range(4 if u.numel() < 10 ** 6 else 1)) / scale
    return want.cpu(), 3 * (off32 + off22) + HALF[dtype]


def _check(outs, mats, dtype, coef=MUON, steps=5):
    for o, u in zip(outs, mats):
        want, tol = _bound(u, dtype, coef, steps)
        got = o.double().cpu()
        assert torch.isfinite(got).all()
        rel = (got - want).norm().item() / max(want.norm().item(), 1e-300)
        log(f"  {tuple(u.shape)}: off {rel:.3g}, allowed {tol:.3g}")
        assert rel <= tol


def _rand(rows, cols, seed, dtype="f32", kind="gauss"):
    g = torch.Generator().manual_seed(seed)
    t = torch.randn(rows, cols, generator=g)
    if kind == "spread":  # channels of differing size, a few strong directions
        t = t * torch.exp(torch.randn(rows, 1, generator=g)) * torch.exp(torch.randn(1, cols, generator=g))
        t = t + 3 * torch.randn(rows, 2, generator=g) @ torch.randn(2, cols, generator=g)
    if kind == "rank":  # gradients of a batch of three
        t = torch.randn(rows, 3, generator=g) @ torch.randn(3, cols, generator=g)
    return t.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()


# one row, one column, edges of the 32, 64 and 128 tiles, tall and wide; the largest take the 64 and 128 tiles
SHAPES = [(1, 1), (1, 7), (7, 1), (2, 2), (9, 50), (31, 33), (32, 32), (33, 31), (64, 64), (65, 129), (100, 200), (200, 100),
          (300, 300), (128, 1000), (1000, 128), (40, 5000), (300, 3755), (777, 777), (1433, 1500), (1500, 1433)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_one_matrix(shape, dtype):
    from paper_1409_6070_amd.sscn import Orthogonalizer
    u = _rand(*shape, seed=sum(shape), dtype=dtype, kind="spread")
    log(f"[orthogonalize] {shape} {dtype}")
    _check(Orthogonalizer([shape], dtype).orthogonalize([u]), [u], dtype)


# 128-tiles in one round; tiles divided over k (X X^T and A A) and a divided last round of 256-tiles (B X), tall and
# wide; a long sum divided sixteen times
@pytest.mark.parametrize("shape", [(2900, 3011), (2100, 3900), (3900, 2100), (520, 40000)], ids=str)
def test_large_matrices(shape):
    """Against the formula, and the same bits again from a workspace full of NaN: partial sums are added in one order."""
    from paper_1409_6070_amd.sscn import Orthogonalizer
    u = _rand(*shape, 1)
    log(f"[orthogonalize] {shape}")
    plan = Orthogonalizer([shape], "f32")
    out = plan.orthogonalize([u])
    _check(out, [u], "f32")
    plan.ws.fill_(0xFF)
    assert torch.equal(plan.orthogonalize([u])[0], out[0])


def test_large_matrices_of_several_sizes_update():
    """A list whose products divide some tiles, through the update: masters, copies, velocities."""
    from paper_1409_6070_amd.sscn import Muon
    shapes = [(1200, 9000), (700, 300), (2000, 1300)]
    W = [_rand(*s, seed=i) * 0.02 for i, s in enumerate(shapes)]
    G = [_rand(*s, seed=10 + i) for i, s in enumerate(shapes)]
    V = [torch.zeros_like(w) for w in W]
    C = [torch.zeros_like(w, dtype=torch.bfloat16) for w in W]
    w0 = [w.clone() for w in W]
    Muon(shapes, "bf16").step(W, C, G, V, lr=0.02, momentum=0.9, weight_decay=0.1, nesterov=False)
    for w, c, g, v, b in zip(W, C, G, V, w0):
        assert torch.equal(v, g) and torch.equal(c, w.bfloat16())
        scale = max(1.0, w.shape[1] / w.shape[0]) ** 0.5
        want, rel = _bound(g, "f32")
        got = (b.double() * (1 - 0.02 * 0.1) - w.double()).cpu() / (0.02 * scale)
        # the update as the weights show it: rounded to half a step of weights of about 0.02 and of lr, wd and scale
        off = (got - want).norm().item() / want.norm().item()
        tol = rel + 8 * U * (b.double().norm().item() / (0.02 * scale)) / want.norm().item() + 8 * U
        log(f"[muon] {tuple(w.shape)}: off {off:.3g}, allowed {tol:.3g}")
        assert off <= tol


@pytest.mark.parametrize("kind", ["gauss", "spread", "rank"])
def test_spectra(kind):
    """Small and vanishing singular values: as exact as float32 products carry them."""
    from paper_1409_6070_amd.sscn import Orthogonalizer
    for shape in ((96, 96), (150, 400), (600, 200)):
        u = _rand(*shape, seed=3, kind=kind)
        log(f"[orthogonalize] {kind} {shape}")
        _check(Orthogonalizer([shape], "f32").orthogonalize([u]), [u], "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_matrices_equal_one_at_a_time_in_value(dtype):
    """A list of 30 shapes (two groups) against the formula, and each alone within rounding of the list's."""
    from paper_1409_6070_amd.sscn import Orthogonalizer
    shapes = [(9 * (i % 5 + 1), 20 + 13 * i) for i in range(29)] + [(500, 260)]
    mats = [_rand(*s, seed=i, dtype=dtype) for i, s in enumerate(shapes)]
    log(f"[orthogonalize] list of {len(shapes)} {dtype}")
    _check(Orthogonalizer(shapes, dtype).orthogonalize(mats), mats, dtype)


# matrices that one workgroup holds (short side to 64, 8192 padded elements), their borders, and lists of them
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(64, 128), (128, 64), (63, 127), (32, 256), (256, 31), (5, 250), (33, 97), (48, 48), (64, 129),
                                   (32, 257), (65, 65)], ids=str)
def test_small_matrices(shape, dtype):
    from paper_1409_6070_amd.sscn import Orthogonalizer
    mats = [_rand(*shape, seed=sum(shape) + i, dtype=dtype, kind=k) for i, k in enumerate(("gauss", "spread"))]
    log(f"[orthogonalize] small {shape} {dtype}")
    _check(Orthogonalizer([shape] * 2, dtype).orthogonalize(mats), mats, dtype)


def test_a_list_of_small_matrices_and_more_steps_than_one_launch_takes():
    from paper_1409_6070_amd.sscn import Orthogonalizer
    shapes = [(9, 16), (16, 9), (64, 32), (1, 200), (64, 24), (40, 60)] * 5
    mats = [_rand(*s, seed=i) for i, s in enumerate(shapes)]
    log("[orthogonalize] 30 small matrices")
    _check(Orthogonalizer(shapes, "f32").orthogonalize(mats), mats, "f32")
    for steps in (8, 9, 12):
        log(f"[orthogonalize] small, {steps} steps")
        plan = Orthogonalizer([(40, 60)], "f32", coef=(1.5, -0.5, 0.0), steps=steps)
        _check(plan.orthogonalize([mats[5]]), [mats[5]], "f32", (1.5, -0.5, 0.0), steps)


def test_other_coefficients_and_step_counts():
    from paper_1409_6070_amd.sscn import Orthogonalizer
    u = _rand(70, 90, 4)
    for coef, steps in (((1.5, -0.5, 0.0), 12), ((1.875, -1.25, 0.375), 9), (MUON, 1), (MUON, 2),
                        ([(3.4445, -4.7750, 2.0315), (2.5, -2.0, 0.6), (1.5, -0.5, 0.0)], 3)):
        log(f"[orthogonalize] {coef} x {steps}")
        _check(Orthogonalizer([(70, 90)], "f32", coef=coef, steps=steps).orthogonalize([u]), [u], "f32", coef, steps)
    o = Orthogonalizer([(70, 90)], "f32", coef=(1.5, -0.5, 0.0), steps=32).orthogonalize([u])[0].double().cpu()
    assert (o @ o.t() - torch.eye(70, dtype=torch.float64)).abs().max() < 1e-5  # the cubic has converged


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-8, 1.0, 1e18, 1e36])
def test_the_size_of_a_matrix_does_not_matter(scale):
    from paper_1409_6070_amd.sscn import Orthogonalizer
    u = _rand(40, 60, 5) * scale
    log(f"[orthogonalize] values of about {scale}")
    _check(Orthogonalizer([(40, 60)], "f32").orthogonalize([u]), [u], "f32")


def test_zero_and_bad_matrices_stay_alone():
    from paper_1409_6070_amd.sscn import Orthogonalizer
    shapes = [(40, 70)] * 4
    mats = [_rand(40, 70, i) for i in range(4)]
    plan = Orthogonalizer(shapes, "f32")
    want = [o.clone() for o in plan.orthogonalize(mats)]
    mats[1] = torch.zeros_like(mats[1])
    mats[2] = mats[2].clone()
    mats[2][39, 69] = float("nan")
    mats[3] = mats[3].clone()
    mats[3][0, 0] = float("inf")
    got = plan.orthogonalize(mats)
    assert torch.equal(got[0], want[0])
    assert (got[1] == 0).all()
    assert torch.isnan(got[2]).all() and torch.isnan(got[3]).all()


@pytest.mark.parametrize("shape", [(200, 300), (700, 650), (1600, 1700)], ids=str)
def test_zero_and_bad_matrices_of_many_tiles_stay_alone(shape):
    """The same beside each other in one launch of products, whose tiles some workgroups share."""
    from paper_1409_6070_amd.sscn import Orthogonalizer
    mats = [_rand(*shape, i) for i in range(4)]
    plan = Orthogonalizer([shape] * 4, "f32")
    want = [o.clone() for o in plan.orthogonalize(mats)]
    mats[1] = torch.zeros_like(mats[1])
    mats[2] = mats[2].clone()
    mats[2][shape[0] - 1, shape[1] - 1] = float("nan")
    mats[3] = mats[3].clone()
    mats[3][0, 0] = float("-inf")
    got = plan.orthogonalize(mats)
    assert torch.equal(got[0], want[0])
    assert (got[1] == 0).all()
    assert torch.isnan(got[2]).all() and torch.isnan(got[3]).all()
    mats = [mats[0]] * 4  # nothing of it stays in the workspace
    assert all(torch.equal(o, want[0]) for o in plan.orthogonalize(mats))


@pytest.mark.parametrize("shape", [(5, 60), (5, 2000)], ids=str)
def test_offsets_past_32_bits(shape):
    from paper_1409_6070_amd.sscn import Orthogonalizer
    stride = (1 << 30) + 3
    u = _rand(*shape, seed=1, dtype="bf16")
    far = torch.as_strided(torch.empty((shape[0] - 1) * stride + shape[1], dtype=torch.bfloat16, device="cuda"), shape,
                           (stride, 1))
    far.copy_(u)
    plan = Orthogonalizer([shape], "bf16")
    want = plan.orthogonalize([u])[0]
    assert torch.equal(plan.orthogonalize([far], out=[far])[0], want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_in_place_and_guards(dtype):
    from paper_1409_6070_amd.sscn import Orthogonalizer
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    for shape, stride, start in (((50, 33), 37, 1), ((33, 50), 51, 3), ((129, 65), 65, 5)):
        u = _rand(*shape, seed=6, dtype=dtype)
        plan = Orthogonalizer([shape], dtype)
        want = plan.orthogonalize([u])[0]
        src = torch.full((start + shape[0] * stride + 9,), 7.5, dtype=tdt, device="cuda")
        dst = src.clone()
        vs, vd = (torch.as_strided(b, shape, (stride, 1), start) for b in (src, dst))
        vs.copy_(u)
        keep = src.clone()
        plan.orthogonalize([vs], out=[vd])
        assert torch.equal(vd, want) and torch.equal(src, keep)
        mask = torch.ones_like(dst, dtype=torch.bool)
        torch.as_strided(mask, shape, (stride, 1), start).fill_(False)
        assert (dst[mask] == 7.5).all()
        plan.orthogonalize([vs], out=[vs])
        assert torch.equal(vs, want)


def test_repeats_streams_and_graphs():
    """The same bits every time: fresh and dirty workspace, another stream, a graph replayed between eager calls that
    use the same workspace."""
    from paper_1409_6070_amd.sscn import Orthogonalizer
    shapes = [(200, 100), (64, 300), (9, 50)]
    mats = [_rand(*s, seed=i) for i, s in enumerate(shapes)]
    plan = Orthogonalizer(shapes, "f32")
    want = [o.clone() for o in plan.orthogonalize(mats)]
    plan.ws.fill_(0xFF)  # NaN everywhere in the workspace
    assert all(torch.equal(a, b) for a, b in zip(plan.orthogonalize(mats), want))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = plan.orthogonalize(mats)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    out = [torch.empty_like(m) for m in mats]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.orthogonalize(mats, out=out)
    for i in range(4):
        for m in mats:
            m.add_(0.1 * i)
        graph.replay()
        torch.cuda.synchronize()
        want = plan.orthogonalize(mats)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i


def test_wrapper_refuses():
    from paper_1409_6070_amd.sscn import Muon, Orthogonalizer, SSCNError
    for bad in ([(0, 3)], [(20000, 20000)]):
        with pytest.raises(SSCNError):
            Orthogonalizer(bad)
    with pytest.raises(ValueError):
        Orthogonalizer([(3, 4)], "f16")
    with pytest.raises(ValueError):
        Orthogonalizer([(3, 4)], coef=[MUON] * 4, steps=5)
    plan = Orthogonalizer([(8, 16)], "f32")
    x = torch.randn(8, 16, device="cuda")
    for mats in ([x, x], [], [x.bfloat16()], [x.cpu()], [x[:7]], [torch.randn(16, 8, device="cuda").t()],
                 [x[:1].expand(8, 16)]):
        with pytest.raises(ValueError):
            plan.orthogonalize(mats)
    with pytest.raises(SSCNError):
        Orthogonalizer([(8, 16)], "f32", coef=(4.0, 0.0, 0.0)).orthogonalize([x])
    with pytest.raises(ValueError):
        Muon([(2, 3, 4)])
    m = Muon([(8, 16), (16,)], "f32")
    v = torch.zeros(16, device="cuda")
    good = [[x, v], None, [x.clone(), v.clone()], [x.clone(), v.clone()]]
    for i in (0, 2, 3):
        for bad in ([x], [x, v, v], [x, v.double()], [x[:, :15], v], [x.t().contiguous().t(), v], [x.cpu(), v]):
            with pytest.raises(ValueError):
                m.step(*good[:i], bad, *good[i + 1:], lr=0.1)
    with pytest.raises(ValueError):
        m.step(good[0], [x.bfloat16(), None], *good[2:], lr=0.1)
    with pytest.raises(SSCNError):
        m.step(*good, lr=-0.1)


def test_outputs_that_would_race_are_refused():
    """An output named twice, or another matrix's input; a parameter array named twice."""
    from paper_1409_6070_amd.sscn import Muon, Orthogonalizer
    plan = Orthogonalizer([(8, 16)] * 2, "f32")
    x, y, o = (torch.randn(8, 16, device="cuda") for _ in range(3))
    for mats, out in (([x, y], [o, o]), ([x, y], [y, x]), ([x, y], [o, x]), ([x, x], [x, o]), ([x, x], [x, x])):
        with pytest.raises(ValueError):
            plan.orthogonalize(mats, out=out)
    a, b = plan.orthogonalize([x, x])  # an input may be named twice
    assert torch.equal(a, b)
    plan.orthogonalize([x, y], out=[x, y])
    assert torch.equal(x, a)
    m = Muon([(8, 16)] * 2, "f32")
    with pytest.raises(ValueError):
        m.step([x, x], None, [y, y], [a, b], lr=0.1)


# ---------------------------------------------------------------------------------------------------------
# the update


def _want_step(w, g, v, orthogonal, lr, momentum, wd, nesterov, scale):
    """(w, tolerance of w, v): one update in 64 bits from float32 arrays."""
    lr, momentum, wd = (float(np.float32(x)) for x in (lr, momentum, wd))
    w, g, v = w.double().cpu(), g.double().cpu(), v.double().cpu()
    if not orthogonal:
        vn = momentum * v + (g + wd * w)
        return w - lr * vn, 4 * U * (w.abs() + lr * (momentum * v.abs() + g.abs() + wd * w.abs())), vn
    vn = momentum * v + g
    u = g + momentum * vn if nesterov else vn
    want, rel = _bound(u.float(), "f32")
    # the float32 velocity and u are off by 3 u of their terms, which the steps (|p'| up to 4 each) enlarge at most by
    # 4^5 = 1024 in norm: into the bound of the direction, as a share of its norm
    terms = (momentum * v.abs() + g.abs()) * (1 + momentum) + g.abs()
    rel = rel + 3 * U * 1024 * (terms.norm() / u.norm()).item() * (min(u.shape) ** 0.5 / want.norm().item())
    tol_o = rel * want.norm().item()  # one entry may hold all of it
    wn = w - lr * (scale * want + wd * w)
    return wn, lr * scale * tol_o + 4 * U * (w.abs() + lr * (scale * want.abs() + wd * w.abs())), vn


MIXED = [(9, 50), (50,), (200, 100), (100,), (300, 400), (1, 33), (70, 30), (1,)]
SMALL = [(9, 50), (50,), (120, 60), (100,), (60, 90), (1, 33), (70, 30), (1,)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("shapes", [MIXED, SMALL], ids=["mixed", "small"])
def test_update_of_matrices_and_vectors(shapes, dtype, nesterov):
    """Three steps of a list with tall, wide and single-row matrices, biases, and a matrix by the SGD rule."""
    from paper_1409_6070_amd.sscn import Muon
    orth = [True, False, True, False, True, True, False, False]
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    W = [_rand(s[0] if len(s) == 2 else 1, s[-1], i).reshape(s) for i, s in enumerate(shapes)]
    V = [torch.zeros_like(w) for w in W]
    C = [None if i in (3, 6) else torch.full(s, 7.0, dtype=tdt, device="cuda") for i, s in enumerate(shapes)]
    plan = Muon(shapes, dtype, orthogonal=orth)
    lr, mu, wd, rest = 0.02, 0.9, 0.1, 0.005
    for k in range(3):
        G = [_rand(s[0] if len(s) == 2 else 1, s[-1], 100 * k + i + 50).reshape(s) for i, s in enumerate(shapes)]
        w0, v0 = [w.clone() for w in W], [v.clone() for v in V]
        plan.step(W, C, G, V, lr=lr, momentum=mu, weight_decay=wd, nesterov=nesterov, lr_rest=rest)
        torch.cuda.synchronize()
        for i, s in enumerate(shapes):
            scale = float(np.float32(max(1.0, s[-1] / s[0]) ** 0.5)) if len(s) == 2 else 1.0
            want, tol, vn = _want_step(w0[i], G[i], v0[i], orth[i], lr if orth[i] else rest, mu,
                                       wd if len(s) == 2 else 0.0, nesterov, scale)
            got = W[i].double().cpu()
            log(f"[muon] step {k} {s} {dtype}: at most {((got - want).abs() / (tol + 1e-30)).max():.3f} of the bound")
            assert ((got - want).abs() <= tol + 1e-30).all()
            assert ((V[i].double().cpu() - vn).abs() <= 4 * U * (mu * v0[i].double().cpu().abs() + G[i].double().cpu().abs()
                                                                 + wd * w0[i].double().cpu().abs())).all()
            if C[i] is not None:
                assert torch.equal(C[i], W[i].to(tdt))  # the rounded master, bit for bit


def test_update_without_matrices_is_the_sgd_rule():
    """No workspace, no coefficients: a list longer than one launch holds."""
    from paper_1409_6070_amd import sscn
    n = 130
    W, G, V = ([_rand(1, 10 + i, k * n + i).reshape(-1) for i in range(n)] for k in range(3))
    W0, V0 = [w.clone() for w in W], [v.clone() for v in V]
    arr = (sscn.MuonParam * n)(*[sscn.MuonParam(1, w.numel(), w.data_ptr(), None, g.data_ptr(), v.data_ptr(),
                                                0.1 + 0.001 * i, 0.5, 0.0, 0)
                                 for i, (w, g, v) in enumerate(zip(W, G, V))])
    assert sscn.sscn_muon_workspace_bytes(arr) == 0
    sscn.sscn_muon_update(sscn.SSCN_F32, arr, 0.9, 0, 0, None, None, 0, sscn._stream())
    torch.cuda.synchronize()
    for i in range(n):
        want, tol, vn = _want_step(W0[i], G[i], V0[i], False, 0.1 + 0.001 * i, 0.9, 0.5, False, 0)
        assert ((W[i].double().cpu() - want).abs() <= tol).all()


def _net(dtype, arch="deepcnet", classes=40, seed=0):
    from paper_1409_6070_amd.sscn import SparseDeepCNet
    from workloads import he_params, random_labels
    rng = np.random.default_rng(seed)
    ell, k, c_in, batch = 3, 12, 2, 16
    N = 3 * 2 ** ell
    coords = np.concatenate([np.stack([np.full(30, b), *np.divmod(rng.choice(N * N, 30, replace=False), N)], 1)
                             for b in range(batch)])
    net = SparseDeepCNet(ell, k, c_in, classes, batch, len(coords), dtype, arch=arch)
    feats = torch.tensor(rng.normal(size=(len(coords), c_in))).to(net.tdtype).cuda()
    Ws, bs = he_params(ell, k, c_in, classes, 1, arch=arch)
    W32 = [torch.tensor(w, dtype=torch.float32, device="cuda") for w in Ws]
    b = [torch.tensor(v, dtype=torch.float32, device="cuda") for v in bs]
    labels = torch.tensor(random_labels(batch, classes, 2), dtype=torch.int32, device="cuda")
    net.rulebook_build(torch.tensor(coords, dtype=torch.int32, device="cuda"), batch)
    return net, feats, W32, [w.to(net.tdtype) for w in W32], b, labels


@pytest.mark.parametrize("dtype,arch,softmax", [("f32", "deepcnet", False), ("bf16", "deepcnet", True),
                                                ("bf16", "deepcnin", False), ("f32", "deepcnin", True)])
def test_muon_step_of_a_network(dtype, arch, softmax):
    net, feats, W32, W, b, labels = _net(dtype, arch)
    vW, vb = [torch.zeros_like(w) for w in W32], [torch.zeros_like(v) for v in b]
    lr, rest, mu, wd = 0.03, 0.01, 0.95, 0.05
    for k in range(2):
        net.forward(feats, W, b, labels)
        dW, db, _ = net.backward()
        torch.cuda.synchronize()
        keep = [[t.clone() for t in ts] for ts in (W32, dW, vW, b, db, vb)]
        net.muon_step(W32, W, b, vW, vb, lr, rest, mu, wd, softmax=softmax)
        torch.cuda.synchronize()
        for i, w in enumerate(W32):
            orth = softmax or i < len(W32) - 1
            scale = float(np.float32(math.sqrt(max(1.0, w.shape[1] / w.shape[0]))))
            want, tol, vn = _want_step(keep[0][i], keep[1][i], keep[2][i], orth, lr if orth else rest, mu, wd, True, scale)
            log(f"[muon step] {dtype} {arch} step {k} matrix {i}")
            assert ((w.double().cpu() - want).abs() <= tol + 1e-30).all()
            assert torch.equal(W[i], w.to(net.tdtype))
            want, tol, vn = _want_step(keep[3][i], keep[4][i], keep[5][i], False, rest, mu, 0.0, True, 0)
            assert ((b[i].double().cpu() - want).abs() <= tol + 1e-30).all()


def test_muon_step_needs_a_backward_and_has_its_times():
    from paper_1409_6070_amd.sscn import SSCNError
    net, feats, W32, W, b, labels = _net("bf16")
    vW, vb = [torch.zeros_like(w) for w in W32], [torch.zeros_like(v) for v in b]
    net.forward(feats, W, b, labels)
    with pytest.raises(SSCNError) as e:
        net.muon_step(W32, W, b, vW, vb, 0.02, 0.01)
    assert e.value.name == "SSCN_ERR_BAD_STATE"
    net.backward()
    with pytest.raises(SSCNError) as e:
        net.muon_step(W32, None, b, vW, vb, 0.02, 0.01)
    assert e.value.name == "SSCN_ERR_INVALID_ARGUMENT"  # the bf16 copies
    net.timing(["sgd"])
    net.muon_step(W32, W, b, vW, vb, 0.02, 0.01)
    n, ms = net.timing_collect("sgd")
    net.timing([])
    assert n == 1 and ms > 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_training_steps_with_a_head_norm_in_one_graph(dtype):
    """A whole step (forward, backward, Muon on the matrices, the SGD rule on biases and the norm's gain and shift)
    captured once and replayed gives what the eager calls give, bit for bit."""
    from paper_1409_6070_amd.sscn import Muon
    runs = []
    for graphed in (False, True):
        net, feats, W32, W, b, labels = _net(dtype)
        c = W32[-1].shape[0]
        gain, shift = torch.ones(c, device="cuda"), torch.zeros(c, device="cuda")
        dgain, dshift = net.set_head_norm(gain, shift)
        vW, vb = [torch.zeros_like(w) for w in W32], [torch.zeros_like(v) for v in b]
        vn = [torch.zeros_like(gain), torch.zeros_like(shift)]
        norms = Muon([(c,), (c,)], dtype)
        net.forward(feats, W, b, labels)  # buffers and kernels are there before the capture
        net.backward()

        def step():
            net.forward(feats, W, b, labels)
            net.backward()
            net.muon_step(W32, W, b, vW, vb, 0.02, 0.01)
            norms.step([gain, shift], None, [dgain, dshift], vn, lr=0.01)

        if graphed:
            keep = [[t.clone() for t in ts] for ts in (W32, W, b, [gain, shift])]
            step()  # the workspace of the update is allocated by the first step
            torch.cuda.synchronize()
            for ts, ks in zip((W32, W, b, [gain, shift]), keep):
                for t, k in zip(ts, ks):
                    t.copy_(k)
            for t in (*vW, *vb, *vn):
                t.zero_()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        got = []
        for _ in range(4):
            graph.replay() if graphed else step()
            torch.cuda.synchronize()
            got.append([net.loss.clone(), gain.clone(), shift.clone(), *[w.clone() for w in W32], *[v.clone() for v in vb]])
        runs.append(got)
    for k, (e, g) in enumerate(zip(*runs)):
        assert all(torch.isfinite(t).all() for t in e)
        for i, (p, q) in enumerate(zip(e, g)):
            assert torch.equal(p, q), (k, i)
    log(f"[training] {dtype}: losses {[float(r[0]) for r in runs[0]]}")


def test_buffers_of_a_captured_step_outlive_other_choices():
    """A captured step keeps its workspaces when eager steps after it choose differently: its replays give what they
    gave before."""
    net, feats, W32, W, b, labels = _net("f32")
    c = W32[-1].shape[0]
    gain, shift = torch.ones(c, device="cuda"), torch.zeros(c, device="cuda")
    grads = net.set_head_norm(gain, shift)
    vW, vb = [torch.zeros_like(w) for w in W32], [torch.zeros_like(v) for v in b]
    keep = [[t.clone() for t in ts] for ts in (W32, b)]

    def reset():
        for ts, ks in zip((W32, b), keep):
            for t, k in zip(ts, ks):
                t.copy_(k)
        for t in (*vW, *vb):
            t.zero_()

    def step(softmax):
        net.forward(feats, W, b, labels)
        net.backward()
        net.muon_step(W32, W, b, vW, vb, 0.02, 0.01, softmax=softmax)

    step(False)
    reset()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(False)
    want = None
    for i in range(3):
        reset()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*W32, *b, *grads)]
        want = got if want is None else want
        assert all(torch.equal(p, q) for p, q in zip(got, want)), i
        reset()
        ws = net._muon_ws.data_ptr()
        step(True)
        net.set_head_norm(None)
        step(True)
        again = net.set_head_norm(gain, shift)
        assert net._muon_ws.data_ptr() == ws and all(p is q for p, q in zip(again, grads))
        torch.cuda.synchronize()


def _largest(rows):
    """Largest values that X, A and B = b A + c A A may hold in each step: dense scans of [0, hi]."""
    hi, out = 1.0, []
    for a, b, c in ((float(np.float32(v)) for v in r) for r in rows):
        s = np.linspace(0.0, hi, 20001)
        out.append((hi, hi * hi, np.abs(b * s ** 2 + c * s ** 4).max()))
        hi = np.abs(a * s + b * s ** 3 + c * s ** 5).max()
    return out


def _ns_held(u, rows, gen):
    """The formula in 64 bits with every operand's entries off, in a random direction, by what the interface states:
    1.5 2^-22 of themselves (the dropped product of the lo parts included) or 2^-39 of the operand's largest value."""
    def o(t, most):
        sign = 2 * torch.randint(0, 2, t.shape, generator=gen, device=t.device) - 1
        return t + sign * torch.clamp(1.5 * 2.0 ** -22 * t.abs(), min=2.0 ** -39 * most)
    x = u.double() / u.double().norm()
    for (a, b, c), (hx, ha, hb) in zip(((float(np.float32(v)) for v in r) for r in rows), _largest(rows)):
        g = o(x, hx) @ o(x, hx).t().contiguous()
        x = a * x + o(b * o(g, ha) + c * (o(g, ha) @ o(g, ha).t().contiguous()), hb) @ o(x, hx)
    return x


# by each kernel: one workgroup, 32 and 64 wide register tiles, tiles in LDS; other coefficients: smaller and larger values
@pytest.mark.parametrize("size", [1e-3, 1e-4, 1e-5, 1e-6, 1e-8])
@pytest.mark.parametrize("axis", [0, 1], ids=["rows", "columns"])
@pytest.mark.parametrize("shape,coef", [((48, 100), MUON), ((300, 1000), MUON), ((1100, 1150), MUON), ((1433, 1500), MUON),
                                        ((300, 1000), (1.5, -0.5, 0.0)), ((300, 1000), (2.0, -0.2, 0.0))], ids=str)
def test_small_rows_and_columns_relative_to_themselves(shape, coef, axis, size):
    """Every second row or column of another size: their error, relative to themselves alone.  Bound: three times the
    distance of the steps in float32 plus that of the steps with operands held as the interface states, both taken
    over these rows or columns."""
    from paper_1409_6070_amd.sscn import Orthogonalizer
    rows = [coef] * 5
    at = [slice(None)] * 2
    at[axis] = slice(0, None, 2)
    at = tuple(at)
    u = _rand(*shape, seed=7)
    u[at] *= size
    want = ns(u, torch.float64, coef)[at]
    norm = want.norm().item()
    off32 = (ns(u, torch.float32, coef).double()[at] - want).norm().item() / norm
    held = max((_ns_held(u, rows, torch.Generator(u.device).manual_seed(k))[at] - want).norm().item()
               for k in range(3)) / norm
    got = Orthogonalizer([shape], "f32", coef=coef).orthogonalize([u])[0].double()[at]
    off = (got - want).norm().item() / norm
    log(f"[orthogonalize] {shape} {coef} {'columns' if axis else 'rows'} of {size}: off {off:.3g} (float32 {off32:.3g}), "
        f"allowed {3 * (off32 + held):.3g}")
    assert off <= 3 * (off32 + held)


# singular values that end just below where the planes' powers of two change (1.25^2 = 1.5625 = 51200 / 2^15), and at 3.5
REACH = [[(1.5624, 0.0, 0.0), (0.9, 0.0, 0.0)], [(1.2499, 0.0, 0.0), (0.9, 0.1, 0.0)], [(1.2501, 0.0, 0.0), (0.9, 0.1, 0.0)],
         [(3.499, 0.0, 0.0), (0.9, -0.05, 0.0)], [(17.4, -69.6, 55.68), (0.25, -0.02, 0.001)], [(1e-9, 0.0, 0.0), (3e4, 0.0, 0.0)],
         [(1.0, 0.7812, 0.7812), (0.5, 0.0, 0.0)], [(1.0, 0.0, 0.0)]]


@pytest.mark.parametrize("shape", [(1, 1), (40, 60), (300, 1000), (1433, 1500)], ids=str)
@pytest.mark.parametrize("rows", REACH, ids=str)
def test_values_that_reach_the_ends_of_the_planes(rows, shape):
    """One entry alone is its own singular value, 1 before the first step: what the coefficients were followed for.
    Bound: a step's relative error of s is |s p'(s) / p(s)| times the last one's, and ten roundings of the terms' sizes,
    of which those of B s hold 2^-21."""
    from paper_1409_6070_amd.sscn import Orthogonalizer
    u = torch.zeros(shape, device="cuda")
    u[shape[0] // 2, shape[1] // 3] = -7.0
    s, rel = 1.0, 2 * U
    for a, b, c in ((float(np.float32(v)) for v in r) for r in rows):
        terms = abs(a) + 2 ** 3 * (abs(b) * s ** 2 + abs(c) * s ** 4)
        p = a + b * s ** 2 + c * s ** 4
        rel = abs((a + 3 * b * s ** 2 + 5 * c * s ** 4) / p) * rel + 10 * U * terms / abs(p)
        s *= p
    got = Orthogonalizer([shape], "f32", coef=rows, steps=len(rows)).orthogonalize([u])[0].double().cpu()
    want = torch.zeros(shape, dtype=torch.float64)
    want[shape[0] // 2, shape[1] // 3] = -s
    log(f"[orthogonalize] {shape} {rows}: {got.min().item():.9g}, {-s:.9g} within {rel:.2g}")
    assert (got - want).abs().max() <= rel * abs(s)


def test_update_refuses_overlapping_arrays_and_shares_gradients():
    from paper_1409_6070_amd.sscn import Muon, SSCNError
    m = Muon([(8, 16), (8, 16), (16,)], "f32")
    mat = lambda: torch.randn(8, 16, device="cuda")  # noqa: E731
    W, G, V, C = [mat(), mat(), mat()[0]], [mat(), mat(), mat()[0]], [mat(), mat(), mat()[0]], [mat(), mat(), mat()[0]]
    keep = [t.clone() for t in W + V + C]
    pair = torch.randn(12, 16, device="cuda")
    for w, c, g, v in ((W, C, G, [V[0], V[0], V[2]]), (W, [C[0], C[0], C[2]], G, V), (W, C, [V[1], G[1], G[2]], V),
                       (W, C, G, [pair[:8], pair[4:], V[2]]), (W, [C[0], W[0], C[2]], G, V), (W, C, G, [V[0], V[1], C[0][3]])):
        with pytest.raises(SSCNError) as e:
            m.step(w, c, g, v, lr=0.1)
        assert e.value.name == "SSCN_ERR_INVALID_ARGUMENT"
    assert all(torch.equal(a, b) for a, b in zip(W + V + C, keep))
    w0, v0 = [w.clone() for w in W], [v.clone() for v in V]
    m.step(W, C, [G[0], G[0], G[0][5]], V, lr=0.1)  # one gradient for all
    m.step(w0, [w0[0], None, w0[2]], [G[0].clone(), G[0].clone(), G[0][5].clone()], v0, lr=0.1)  # the master as its own copy
    for a, b, c, p, q in zip(W, w0, C, V, v0):
        assert torch.equal(a, b) and torch.equal(c, a) and torch.equal(p, q)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_orthogonalize_outputs_side_by_side_and_overlapping(dtype):
    from paper_1409_6070_amd.sscn import Orthogonalizer, SSCNError
    shapes = [(8, 16), (8, 16), (1, 9)]
    mats = [_rand(*s, seed=i, dtype=dtype) for i, s in enumerate(shapes)]
    plan = Orthogonalizer(shapes, dtype)
    want = plan.orthogonalize(mats)
    buf = torch.zeros(17, 40, dtype=mats[0].dtype, device="cuda")
    for bad in ([buf[:8, :16], buf[:8, 15:31], buf[9:10, :9]], [buf[:8, :16], buf[:8, 30:].as_strided((8, 16), (40, 1), 30),
                buf[9:10, :9]], [buf[:8, :16], buf[7:15, :16], buf[16:, :9]], [buf[:8, :16], buf[8:16, :16], buf[3:4, 15:24]]):
        with pytest.raises(SSCNError) as e:
            plan.orthogonalize(mats, out=bad)
        assert e.value.name == "SSCN_ERR_INVALID_ARGUMENT"
    assert (buf == 0).all()
    side = [buf[:8, :16], buf[:8, 16:32], buf[3:4, 32:41].as_strided((1, 9), (9, 1), 16 * 40)]  # columns, the last row
    rows = [buf[0:16:2, 1:17], buf[1:16:2, 1:17], buf[16:, :9]]  # every other row
    for out in (side, rows):
        buf.zero_()
        plan.orthogonalize(mats, out=out)
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        for o in out:
            o.zero_()
        assert (buf == 0).all()  # nothing beside them
    for v, m in zip(side, mats):
        v.copy_(m)
    plan.orthogonalize(side, out=side)  # in place, and an input twice
    assert all(torch.equal(a, b) for a, b in zip(side, want))
    a, b, _ = plan.orthogonalize([mats[0], mats[0], mats[2]])
    assert torch.equal(a, want[0]) and torch.equal(b, want[0])


def _direction(w0, w, g, v, lr, momentum, wd, nesterov, scale):
    """(distance of the update that the weights show from the formula's, its bound), both relative to the formula's
    norm.  The bound: that of the steps on the formula's u; u as float32 holds it, which is off by at most three
    roundings of its terms' sizes, taken through the steps in random directions; and the weights' own roundings (of w,
    lr, wd and scale: eight of the terms' sizes)."""
    lr, momentum, wd = (float(np.float32(x)) for x in (lr, momentum, wd))
    w0, w, g, v = (t.double().cpu() for t in (w0, w, g, v))
    vn = momentum * v + g
    u = g + momentum * vn if nesterov else vn
    terms = g.abs() + momentum * (momentum * v.abs() + g.abs()) if nesterov else momentum * v.abs() + g.abs()
    want = ns(u, torch.float64)
    _, rel = _bound(u.float(), "f32")
    gen = torch.Generator().manual_seed(0)
    for _ in range(3):
        sign = 2 * torch.randint(0, 2, u.shape, generator=gen) - 1
        rel = max(rel, _bound(u.float(), "f32")[1] + 3 * (ns(u + 3 * U * sign * terms, torch.float64) - want).norm().item()
                  / want.norm().item())
    got = (w0 * (1 - lr * wd) - w) / (lr * scale)
    rel += 8 * U * (1 + (w0.norm() / (lr * scale * want.norm())).item())
    return (got - want).norm().item() / want.norm().item(), rel


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("shape", [(9, 50), (60, 90), (120, 33), (200, 100), (100, 300), (700, 650)], ids=str)
def test_direction_of_the_update_with_a_velocity(shape, nesterov):
    """The orthogonalised direction from a velocity that is not zero, tightly enough that another momentum, the other
    rule for u or another scale would show."""
    from paper_1409_6070_amd.sscn import Muon
    W, G, V = _rand(*shape, 1) * 0.02, _rand(*shape, 2), 2 * _rand(*shape, 3)
    w0, v0 = W.clone(), V.clone()
    scale = float(np.float32(max(1.0, shape[1] / shape[0]) ** 0.5))
    Muon([shape], "f32").step([W], None, [G], [V], lr=0.02, momentum=0.95, weight_decay=0.1, nesterov=nesterov)
    off, tol = _direction(w0, W, G, v0, 0.02, 0.95, 0.1, nesterov, scale)
    log(f"[muon] direction {shape} nesterov {nesterov}: off {off:.3g}, allowed {tol:.3g}")
    assert off <= tol
    for wrong in (dict(momentum=0.94), dict(nesterov=not nesterov), dict(scale=scale * 1.002), dict(lr=0.02005)):
        args = dict(dict(lr=0.02, momentum=0.95, wd=0.1, nesterov=nesterov, scale=scale), **wrong)
        off, tol = _direction(w0, W, G, v0, **args)
        assert off > 4 * tol, (wrong, off, tol)  # (a mistake planted in the formula)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nesterov", [True, False])
def test_direction_of_a_networks_second_step(dtype, nesterov):
    net, feats, W32, W, b, labels = _net(dtype)
    vW, vb = [torch.zeros_like(w) for w in W32], [torch.zeros_like(v) for v in b]
    for k in range(2):
        net.forward(feats, W, b, labels)
        dW, _, _ = net.backward()
        keep = [[t.clone() for t in ts] for ts in (W32, dW, vW)]
        net.muon_step(W32, W, b, vW, vb, 0.03, 0.01, 0.95, 0.05, nesterov=nesterov, softmax=True)
    for i, w in enumerate(W32):
        scale = float(np.float32(math.sqrt(max(1.0, w.shape[1] / w.shape[0]))))
        off, tol = _direction(keep[0][i], w, keep[1][i], keep[2][i], 0.03, 0.95, 0.05, nesterov, scale)
        log(f"[muon] network's matrix {i} {tuple(w.shape)} nesterov {nesterov}: off {off:.3g}, allowed {tol:.3g}")
        assert off <= tol


@pytest.mark.parametrize("shape", [(1, 1 << 20), (1 << 20, 1), (33, 1000003), (200000, 64)], ids=str)
def test_longest_matrices(shape):
    from paper_1409_6070_amd.sscn import Orthogonalizer
    u = _rand(*shape, seed=9)
    log(f"[orthogonalize] {shape}")
    plan = Orthogonalizer([shape], "f32")
    out = plan.orthogonalize([u])
    _check(out, [u], "f32")
    plan.ws.fill_(0xFF)
    assert torch.equal(plan.orthogonalize([u])[0], out[0])
