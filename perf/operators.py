"""Four operators of training, as cases that can be timed and compared: the layer norm of feature rows and its
backward pass, the orthogonalising of an update by Newton-Schulz products, and the weight update that uses it.

``run`` computes a case either in its plain form (elementary torch operations in 32 bits) or, where ``own`` is
true, with the package's calls.  Formulas, with x a row of C features, u an update matrix:

    layer norm      mean = sum x / C, r = 1 / sqrt(sum (x - mean)^2 / C + eps), h = (x - mean) r,
                    y = h * gain + shift
    its backward    t = dy * gain, dx = r (t - sum t / C - h sum (t h) / C),
                    dgain = sum over rows of dy * h, dshift = sum over rows of dy
    orthogonalise   X = u / |u|_F (transposed where u has more rows than columns), then five times
                    A = X X^T, X = a X + (b A + c A A) X
    Muon's update   v = mu v + g, u = g + mu v, w = w - lr (scale orthogonalise(u) + wd w), and the copy of
                    w in the network's storage type
"""

import math

import torch

own = False

EPS = 1e-5
COEF = (3.4445, -4.7750, 2.0315)  # the quintic commonly used with Muon
STEPS = 5
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

# ---------------------------------------------------------------------------------------------------------
# the cases


def _norm(name, op, rows, cols, dtype, padded):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "dtype": dtype, "padded": padded}


def _ortho(name, rows, cols, count, dtype):
    return {"name": name, "op": "orthogonalize", "rows": rows, "cols": cols, "count": count, "dtype": dtype}


def _muon(name, arch, ell, k, c_in, classes, head, dtype):
    return {"name": name, "op": "muon", "arch": arch, "ell": ell, "k": k, "c_in": c_in, "classes": classes,
            "head": head, "dtype": dtype}


def listed():
    return [
        # one character classified as it is drawn: a single row before the softmax layer of DeepCNet(5,50)
        _norm("norm_one_row", "norm", 1, 300, "bf16", True),
        # every active site of a wide layer at batch 1600: rows as the network lays them out, 16-byte aligned
        _norm("norm_sites_c100", "norm", 200001, 100, "bf16", True),
        # long rows in float32, an odd length packed without padding: nothing is aligned
        _norm("norm_odd_f32", "norm", 20011, 4099, "f32", False),
        # the ordinary training batch before the softmax layer
        _norm("norm_bwd_b100", "norm_bwd", 100, 300, "f32", True),
        # active sites again, few features in each: the reduction over rows is the work
        _norm("norm_bwd_sites_c100", "norm_bwd", 200001, 100, "bf16", True),
        # long rows: the features of one row outgrow a wave's registers
        _norm("norm_bwd_wide", "norm_bwd", 16384, 8192, "bf16", True),
        # one hidden matrix of DeepCNet(5,50), tall: five steps of three small dependent products
        _ortho("ortho_1000x300", 1000, 300, 1, "f32"),
        # several square matrices at once, as layers of one width give them
        _ortho("ortho_1024_x8", 1024, 1024, 8, "bf16"),
        # one large matrix
        _ortho("ortho_4096", 4096, 4096, 1, "f32"),
        # the package's headline network: its six convolutions, stored in bfloat16
        _muon("muon_5_50", "deepcnet", 5, 50, 1, 3755, False, "bf16"),
        # network-in-network layers, float32, with the wide softmax matrix
        _muon("muon_nin_5_50_head", "deepcnin", 5, 50, 8, 3755, True, "f32"),
        # the deep and wide network
        _muon("muon_6_100_head", "deepcnet", 6, 100, 1, 3755, True, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_bwd", "orthogonalize", "muon"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("norm", "norm_bwd"):
        cols = _log(rng, 9, 12000)
        rows = _log(rng, 1, min(250000, 2 ** 26 // cols))
        case = _norm("", op, rows, cols, dtype, rng.random() < 0.5)
    elif op == "orthogonalize":
        short = _log(rng, 9, 2000)
        long = max(short, int(short * rng.uniform(1, 4)))
        count = rng.choice([1, 1, 2, 3, 5]) if short < 1000 else 1
        rows, cols = (short, long) if rng.random() < 0.5 else (long, short)
        case = _ortho("", rows, cols, count, dtype)
    else:
        case = _muon("", rng.choice(["deepcnet", "deepcnin"]), rng.randint(2, 6), _log(rng, 8, 100), rng.randint(1, 9),
                     _log(rng, 10, 4000), rng.random() < 0.5, dtype)
    del case["name"]
    return case


def _matrices(case):
    """Shapes [fan in, fan out] of a case's matrices."""
    if case["op"] == "orthogonalize":
        return [(case["rows"], case["cols"])] * case["count"]
    shapes, below, nin = [], case["c_in"], case["arch"] == "deepcnin"
    for n in range(1, case["ell"] + 2):
        out = n * case["k"]
        window = 9 if n == 1 else 4
        if nin and n > 1:  # the 1x1 layer behind each pooling layer
            shapes.append((below, below))
        shapes.append((window * below, out))
        below = out
    if nin:
        shapes.append((below, below))
    if case["head"]:
        shapes.append((below, case["classes"]))
    return shapes


def _scale(rows, cols):
    return math.sqrt(max(1.0, cols / rows))


# ---------------------------------------------------------------------------------------------------------
# inputs


def _rows(g, case, scale, offset):
    """Feature rows [rows, cols]; a padded case's rows start 16-byte aligned."""
    per = 16 // (2 if case["dtype"] == "bf16" else 4)
    stride = -(-case["cols"] // per) * per if case["padded"] else case["cols"]
    t = torch.randn(case["rows"], stride, generator=g, device="cuda")
    t = t * scale + offset
    return t.to(TYPES[case["dtype"]])[:, : case["cols"]]


def _update(g, rows, cols):
    """What gradients of trained layers look like: channels of differing size, and a few directions that dominate."""
    d = torch.randn(rows, cols, generator=g, device="cuda")
    d = d * torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))
    d = d * torch.exp(0.5 * torch.randn(1, cols, generator=g, device="cuda"))
    u = torch.randn(rows, 4, generator=g, device="cuda")
    return 1e-3 * (d + 2.0 * u @ torch.randn(4, cols, generator=g, device="cuda"))


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] in ("norm", "norm_bwd"):
        # features behind a rectifier lean to one side: rows with a mean of their own
        offset = 0.5 + 0.25 * torch.randn(case["rows"], 1, generator=g, device="cuda")
        state = {"x": _rows(g, case, 0.7, offset),
                 "gain": 1.0 + 0.1 * torch.randn(case["cols"], generator=g, device="cuda"),
                 "shift": 0.1 * torch.randn(case["cols"], generator=g, device="cuda")}
        if case["op"] == "norm_bwd":
            state["dy"] = _rows(g, case, 0.01, 0.0)
        return state
    shapes = _matrices(case)
    if case["op"] == "orthogonalize":
        return {"u": [_update(g, r, c).to(TYPES[case["dtype"]]) for r, c in shapes]}
    w = [torch.randn(r, c, generator=g, device="cuda") * math.sqrt(2.0 / r) for r, c in shapes]
    return {"w": w, "store": [t.to(TYPES[case["dtype"]]) for t in w], "g": [_update(g, r, c) for r, c in shapes],
            "v": [8.0 * _update(g, r, c) for r, c in shapes]}


def prepare(case, seed):
    state = dict(_inputs(case, seed), case=case)
    if own:  # the plan and workspace that a program keeps beside its buffers
        from paper_1409_6070_amd import sscn
        if case["op"] in ("norm", "norm_bwd"):
            state["plan"] = sscn.LayerNorm(case["cols"], case["rows"], case["dtype"], eps=EPS)
        elif case["op"] == "orthogonalize":
            state["plan"] = sscn.Orthogonalizer(_matrices(case), case["dtype"], coef=COEF, steps=STEPS)
        else:
            state["plan"] = sscn.Muon(_matrices(case), case["dtype"], coef=COEF, steps=STEPS)
    return state


# ---------------------------------------------------------------------------------------------------------
# one pass


def _plain_norm(x, gain, shift):
    x32 = x.float()
    d = x32 - x32.mean(1, keepdim=True)
    r = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    return (d * r * gain + shift).to(x.dtype)


def _plain_norm_bwd(dy, x, gain):
    x32, dy32 = x.float(), dy.float()
    d = x32 - x32.mean(1, keepdim=True)
    r = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    h = d * r
    t = dy32 * gain
    dx = r * (t - t.mean(1, keepdim=True) - h * (t * h).mean(1, keepdim=True))
    return dx.to(x.dtype), (dy32 * h).sum(0), dy32.sum(0)


def _plain_ortho(u):
    """Five dependent steps of three matrix products each."""
    a, b, c = COEF
    x = u.float()
    if x.shape[0] > x.shape[1]:
        x = x.t()
    x = x / torch.sqrt((x * x).sum())
    for _ in range(STEPS):
        g = x @ x.t()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


def _plain_muon(w, store, grad, v):
    v.mul_(MOMENTUM).add_(grad)
    o = _plain_ortho(grad + MOMENTUM * v)
    w.sub_(LR * (_scale(*w.shape) * o + DECAY * w))
    store.copy_(w)


def run(state):
    op = state["case"]["op"]
    if own:
        plan = state["plan"]
        if op == "norm":
            return plan.forward(state["x"], state["gain"], state["shift"])
        if op == "norm_bwd":
            return plan.backward(state["dy"], state["x"], state["gain"])
        if op == "orthogonalize":
            return plan.orthogonalize(state["u"])
        plan.step(state["w"], state["store"], state["g"], state["v"], lr=LR, momentum=MOMENTUM, weight_decay=DECAY,
                  nesterov=True)
        return {k: state[k] for k in ("w", "store", "v")}
    if op == "norm":
        return _plain_norm(state["x"], state["gain"], state["shift"])
    if op == "norm_bwd":
        return _plain_norm_bwd(state["dy"], state["x"], state["gain"])
    if op == "orthogonalize":
        return [_plain_ortho(u).to(u.dtype) for u in state["u"]]
    for w, store, g, v in zip(state["w"], state["store"], state["g"], state["v"]):
        _plain_muon(w, store, g, v)
    return {k: state[k] for k in ("w", "store", "v")}


# ---------------------------------------------------------------------------------------------------------
# what a pass cannot do without, and its value in 64 bits


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":
        n = case["rows"] * case["cols"]
        return {"bytes": 2 * n * size + 8 * case["cols"], "flops": 7 * n}
    if case["op"] == "norm_bwd":
        n = case["rows"] * case["cols"]
        return {"bytes": 3 * n * size + 12 * case["cols"], "flops": 16 * n}
    total, flops = 0, 0
    for r, c in _matrices(case):
        m, n = min(r, c), max(r, c)
        # X X^T and A A are symmetric: half of each is computed
        flops += STEPS * (m * (m + 1) * n + m * m * (m + 1) + 2 * m * m * n)
        total += r * c
    if case["op"] == "orthogonalize":
        return {"bytes": 2 * total * size, "flops": flops}
    # w, v and g are read, w, its copy and v written
    return {"bytes": total * (20 + size), "flops": flops + 8 * total}


def _exact_ortho(u):
    x = u.double()
    tall = x.size(0) > x.size(1)
    x = x.t().contiguous() if tall else x
    x = x / torch.linalg.vector_norm(x)
    eye = torch.eye(x.size(0), dtype=torch.float64, device=x.device)
    for _ in range(STEPS):
        gram = torch.mm(x, x.t().contiguous())
        x = torch.mm(COEF[0] * eye + torch.mm(COEF[1] * eye + COEF[2] * gram, gram), x)
    return x.t() if tall else x


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] in ("norm", "norm_bwd"):
        x, gain = s["x"].double(), s["gain"].double()
        var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
        r = 1.0 / torch.sqrt(var + EPS)
        if case["op"] == "norm":
            return (x - mean) * r * gain + s["shift"].double()
        n, dy = case["cols"], s["dy"].double()
        t = dy * gain
        s1 = t.sum(1, keepdim=True)
        s2 = (t * (x - mean)).sum(1, keepdim=True)
        dx = r * t - r * s1 / n - (x - mean) * r ** 3 * s2 / n
        return dx, ((x - mean) * r * dy).sum(0), dy.sum(0)
    if case["op"] == "orthogonalize":
        return [_exact_ortho(u) for u in s["u"]]
    out = {"w": [], "store": [], "v": []}
    for w, g, v in zip(s["w"], s["g"], s["v"]):
        g, v, w = g.double(), MOMENTUM * v.double() + g.double(), w.double()
        w = (1.0 - LR * DECAY) * w - LR * _scale(*w.shape) * _exact_ortho(g + MOMENTUM * v)
        for k, t in (("w", w), ("store", w), ("v", v)):
            out[k].append(t)
    return out
