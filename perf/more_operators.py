"""Operators of a network-in-network stage on site rows whose activations are held in 8 bits, as cases that can be
timed and compared: group norm with an activation and its backward pass, rows stored in 8 bits and restored, and the
product of 8-bit rows with an 8-bit matrix, forward and backward.

``run`` computes a case either in its plain form (elementary torch operations in 32 bits) or, where ``own`` is
true, with the package's calls.  Formulas:

    8-bit rows      per row and block of 128 columns e = the least integer >= -126 with max |x| <= 448 2^e,
                    code = x 2^-e rounded to e4m3 (ties to even), xq = code 2^e
    8-bit matrix    the same with a block of 128 x 128
    product         y = xq wq + bias, dx = dyq wq^T, dw = xq^T dyq, dbias = sum over rows of dyq
    group norm      over the rows of a sample and the channels of a group:
                    mean = sum x / n, r = 1 / sqrt(sum (x - mean)^2 / n + eps),
                    h = (x - mean) r, z = h gain + shift, y = act(z)
    its backward    dz = dy act'(z), t = dz gain, dx = r (t - sum t / n - h sum (t h) / n),
                    dgain = sum over rows of dz h, dshift = sum over rows of dz;
                    x as rows, or as 8-bit rows (then h is taken from xq)
"""

import math

import torch

own = False

EPS = 1e-5
BLOCK = 128
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SLOPES = {"none": 1.0, "relu": 0.0, "leaky": 1.0 / 3.0}

# ---------------------------------------------------------------------------------------------------------
# the cases


def _norm(name, op, batch, rows, cols, groups, act, dtype, equal=False):
    return {"name": name, "op": op, "batch": batch, "rows": rows, "cols": cols, "groups": groups, "act": act,
            "dtype": dtype, "equal": equal}


def _store(name, rows, cols, dtype):
    return {"name": name, "op": "store", "rows": rows, "cols": cols, "dtype": dtype}


def _product(name, op, rows, k, n, dtype):
    return {"name": name, "op": op, "rows": rows, "k": k, "n": n, "dtype": dtype}


def listed():
    return [
        # one digit picture as it is classified: a single small sample
        _norm("norm_one_digit", "norm", 1, 150, 10, 2, "relu", "f32"),
        # an ordinary training batch: pen strokes of very different lengths, ten channels a group
        _norm("norm_strokes_c100", "norm", 100, 60001, 100, 10, "leaky", "bf16"),
        # dense planes of the 96 x 96 grid, channels last
        _norm("norm_planes_c256", "norm", 64, 64 * 96 * 96, 256, 32, "silu", "bf16", True),
        # the training batch backward: float32, fifteen channels a group
        _norm("norm_bwd_strokes_c300", "norm_bwd", 100, 20011, 300, 20, "silu", "f32"),
        # one sample of many sites: the sums go over the whole array
        _norm("norm_bwd_one_plane", "norm_bwd", 1, 200001, 100, 5, "leaky", "bf16"),
        # 32 x 32 patches whose input was kept in 8 bits
        _norm("norm_bwd8_patch_c512", "norm_bwd8", 128, 128 * 32 * 32, 512, 32, "relu", "bf16", True),
        # the softmax layer's input of a training batch, stored and restored
        _store("store_b100_c300", 100, 300, "f32"),
        # the sites of a wide layer
        _store("store_sites_c1000", 200001, 1000, "bf16"),
        # one character's scores: a single row against the softmax layer of DeepCNet(5,50)
        _product("product_one_row", "product", 1, 300, 3755, "bf16"),
        # a large product
        _product("product_wide", "product", 32768, 4096, 4096, "bf16"),
        # the sites of DeepCNiN(5,50)'s top 1x1 layers backward, behind an update of the weights
        _product("product_dx_sites_c300", "product_dx", 200001, 300, 300, "bf16"),
        # weight gradient from the rows kept in 8 bits, an odd number of them
        _product("product_dw_wide", "product_dw", 65537, 2048, 1000, "f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_bwd", "norm_bwd8", "store", "product", "product_dx", "product_dw"])
    dtype = rng.choice(["f32", "bf16"])
    if op.startswith("norm"):
        groups = rng.choice([1, 2, 3, 5, 8, 16, 32])
        cols = groups * _log(rng, 2, 1024 // groups)
        rows = _log(rng, 30, 2 ** 26 // cols)
        batch = _log(rng, 1, min(1000, max(1, rows // 20)))
        equal = rng.random() < 0.3
        case = _norm("", op, batch, rows // batch * batch if equal else rows, cols, groups,
                     rng.choice(["none", "relu", "leaky", "silu"]), dtype, equal)
    elif op == "store":
        cols = _log(rng, 9, 4096)
        case = _store("", _log(rng, 1, 2 ** 27 // cols), cols, dtype)
    else:
        k, n = _log(rng, 9, 4096), _log(rng, 9, 4096)
        case = _product("", op, _log(rng, 1, min(250000, 2 ** 38 // (k * n))), k, n, dtype)
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------------------------
# 8 bits, elementwise


def _blocks(cols):
    return -(-cols // BLOCK)


def _pow2(e):
    """2^e exactly, -126 <= e <= 127."""
    return ((e + 127) << 23).view(torch.float32)


def _exponents(largest):
    m, q = torch.frexp(largest)
    return torch.clamp(q - 9 + (m > 0.875), min=-126)


def _e4m3(v):
    """|v| <= 448 rounded to three bits behind the leading one, in steps of 2^-9 below 2^-6."""
    _, q = torch.frexp(v)
    step = torch.clamp(q - 1, min=-6) - 3
    return torch.round(v * _pow2(-step)) * _pow2(step)


def _quantized_rows(x):
    """Codes' values and exponents of rows: [rows, cols] float32, [rows, blocks] int32."""
    rows, cols = x.shape
    nb = _blocks(cols)
    padded = torch.zeros(rows, nb * BLOCK, device=x.device)
    padded[:, :cols] = x
    e = _exponents(padded.view(rows, nb, BLOCK).abs().amax(2))
    v = _e4m3(padded.view(rows, nb, BLOCK) * _pow2(-e)[:, :, None])
    return v.view(rows, -1)[:, :cols], e


def _restored(v, e):
    rows, cols = v.shape
    return v * _pow2(e).repeat_interleave(BLOCK, 1)[:, :cols]


def _plain_rows8(x):
    return _restored(*_quantized_rows(x.float()))


def _plain_matrix8(w):
    k, n = w.shape
    kb, nb = _blocks(k), _blocks(n)
    padded = torch.zeros(kb * BLOCK, nb * BLOCK, device=w.device)
    padded[:k, :n] = w
    t = padded.view(kb, BLOCK, nb, BLOCK)
    e = _exponents(t.abs().amax((1, 3)))[:, None, :, None]
    return (_e4m3(t * _pow2(-e)) * _pow2(e)).view(kb * BLOCK, nb * BLOCK)[:k, :n].contiguous()


# ---------------------------------------------------------------------------------------------------------
# inputs


def _begins(g, case):
    """Row offsets of the samples: lengths that differ severalfold, a few samples without a site."""
    batch, rows = case["batch"], case["rows"]
    if case["equal"]:
        return torch.arange(batch + 1, device="cuda", dtype=torch.int32) * (rows // batch)
    w = torch.exp(0.6 * torch.randn(batch, generator=g, device="cuda", dtype=torch.float64))
    if batch > 20:
        w = w * (torch.rand(batch, generator=g, device="cuda") > 0.03)
    ends = torch.round(torch.cumsum(w, 0) * (rows / w.sum())).to(torch.int32)
    return torch.cat([torch.zeros_like(ends[:1]), ends[:-1], torch.full_like(ends[:1], rows)])


def _features(g, rows, cols, dtype):
    """Sums before a norm: channels of differing mean and size."""
    t = torch.randn(rows, cols, generator=g, device="cuda")
    t = t * torch.exp(0.3 * torch.randn(cols, generator=g, device="cuda")) + torch.randn(cols, generator=g, device="cuda")
    return t.to(TYPES[dtype])


def _activations(g, rows, cols, dtype):
    """What a leaky rectifier leaves: mostly one sign, channels of differing size."""
    t = torch.randn(rows, cols, generator=g, device="cuda")
    t = torch.where(t < 0, t / 3, t) * torch.exp(0.7 * torch.randn(cols, generator=g, device="cuda"))
    return t.to(TYPES[dtype])


def _gradients(g, rows, cols, dtype):
    """Small, and of very different size from row to row."""
    t = torch.randn(rows, cols, generator=g, device="cuda")
    return (1e-4 * t * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))).to(TYPES[dtype])


def _stored(x):
    """The 8-bit form of rows as a program holds it: codes [rows, cols rounded up to 16], scales 2^(s - 127)
    [rows, blocks rounded up to 4], both bytes, zero behind the columns and blocks."""
    v, e = _quantized_rows(x.float())
    rows, cols = v.shape
    codes = torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.uint8, device="cuda")
    codes[:, :cols] = v.to(torch.float8_e4m3fn).view(torch.uint8)
    scales = torch.zeros(rows, -(-e.shape[1] // 4) * 4, dtype=torch.uint8, device="cuda")
    scales[:, : e.shape[1]] = (e + 127).to(torch.uint8)
    return codes, scales


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, dtype = case["op"], case["dtype"]
    if op.startswith("norm"):
        rows, cols, groups = case["rows"], case["cols"], case["groups"]
        state = {"begin": _begins(g, case), "x": _features(g, rows, cols, dtype),
                 "gain": 1.0 + 0.1 * torch.randn(cols, generator=g, device="cuda"),
                 "shift": 0.1 * torch.randn(cols, generator=g, device="cuda")}
        if op != "norm":  # the statistics that the forward pass left
            mean, r = _plain_stats(state["x"], state["begin"], groups)
            state.update(stats=torch.stack([mean, r]), dy=_gradients(g, rows, cols, dtype))
        if op == "norm_bwd8":
            state["codes"], state["scales"] = _stored(state.pop("x"))
        return state
    if op == "store":
        return {"x": _activations(g, case["rows"], case["cols"], dtype)}
    rows, k, n = case["rows"], case["k"], case["n"]
    state = {}
    if op != "product_dw":
        state["w"] = _features(g, k, n, dtype) * math.sqrt(1.0 / k)
    if op == "product":
        state["x"] = _activations(g, rows, k, dtype)
        state["bias"] = 0.1 * torch.randn(n, generator=g, device="cuda")
    elif op == "product_dx":
        state["dy"] = _gradients(g, rows, n, dtype)
    else:
        state["codes"], state["scales"] = _stored(_activations(g, rows, k, dtype))
        state["dy_codes"], state["dy_scales"] = _stored(_gradients(g, rows, n, dtype))
    return state


def prepare(case, seed):
    state = dict(_inputs(case, seed), case=case)
    op = case["op"]
    if own:  # the plan, workspace and weights that a program keeps beside its buffers
        from paper_1409_6070_amd import sscn
        if op.startswith("norm"):
            state["plan"] = sscn.GroupNorm(case["cols"], case["groups"], case["rows"], case["batch"], case["dtype"],
                                           act=case["act"], eps=EPS)
        elif op == "store":
            state["rows8"] = sscn.Rows8(case["rows"], case["cols"])
        else:
            state["plan"] = sscn.Product8(case["k"], case["n"], case["rows"], case["dtype"])
            if op == "product":
                state["plan"].set_weights(state["w"])
                state["x8"] = sscn.Rows8(case["rows"], case["k"])
            elif op == "product_dx":
                state["dy8"] = sscn.Rows8(case["rows"], case["n"])
            else:
                state["dy8"] = sscn.Rows8(case["rows"], case["n"], codes=state["dy_codes"], scales=state["dy_scales"])
        if "codes" in state:
            cols = case["cols"] if "cols" in case else case["k"]
            state["x8"] = sscn.Rows8(case["rows"], cols, codes=state["codes"], scales=state["scales"])
    elif op == "product":  # weights are laid out once
        state["wq"] = _plain_matrix8(state["w"])
    return state


# ---------------------------------------------------------------------------------------------------------
# one pass


def _samples(begin, rows):
    at = torch.arange(rows, device=begin.device, dtype=torch.int32)
    return torch.searchsorted(begin[1:], at, right=True)


def _span_means(v, begin, per):
    """Sums of rows over the samples, divided by their elements."""
    rows, groups = v.shape
    sums = torch.zeros(groups * rows + 1, dtype=torch.float64, device=v.device)
    torch.cumsum(v.t().reshape(-1), 0, dtype=torch.float64, out=sums[1:])
    at = begin.long()[:, None] + rows * torch.arange(groups, device=v.device)
    n = (begin[1:] - begin[:-1]).clamp(min=1) * per
    return (sums[at[1:]] - sums[at[:-1]]) / n[:, None]


def _plain_stats(x, begin, groups):
    rows, cols = x.shape
    per = cols // groups
    x32, ids = x.float().view(rows, groups, per), _samples(begin, rows)
    mean = _span_means(x32.sum(2), begin, per).float()
    d = x32 - mean[ids][:, :, None]
    var = _span_means((d * d).sum(2), begin, per)
    return mean, (1.0 / torch.sqrt(var + EPS)).float()


def _plain_norm(x, begin, gain, shift, groups, act):
    rows, cols = x.shape
    mean, r = _plain_stats(x, begin, groups)
    ids = _samples(begin, rows)
    h = (x.float().view(rows, groups, -1) - mean[ids][:, :, None]) * r[ids][:, :, None]
    z = h.view(rows, cols) * gain + shift
    y = z / (1.0 + torch.exp(-z)) if act == "silu" else torch.where(z < 0, z * SLOPES[act], z)
    return y.to(x.dtype), torch.stack([mean, r])


def _plain_norm_bwd(dy, x, stats, begin, gain, shift, groups, act):
    rows, cols = x.shape
    per, ids = cols // groups, _samples(begin, rows)
    mean, r = stats[0][ids][:, :, None], stats[1][ids][:, :, None]
    h = (x.float().view(rows, groups, per) - mean) * r
    z, d = h.view(rows, cols) * gain + shift, dy.float()
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        dz = d * s * (1.0 + z * (1.0 - s))
    else:
        dz = torch.where(z > 0 if act == "relu" else z >= 0, d, d * SLOPES[act])
    t = (dz * gain).view(rows, groups, per)
    m1 = _span_means(t.sum(2), begin, per).float()
    m2 = _span_means((t * h).sum(2), begin, per).float()
    dx = r * (t - m1[ids][:, :, None] - h * m2[ids][:, :, None])
    return dx.view(rows, cols).to(dy.dtype), (dz * h.view(rows, cols)).sum(0), dz.sum(0)


def _plain_held(codes, scales, cols):
    e = scales[:, : _blocks(cols)].to(torch.int32) - 127
    return _restored(codes[:, :cols].view(torch.float8_e4m3fn).float(), e)


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        if op == "norm":
            return state["plan"].forward(state["x"], state["begin"], state["gain"], state["shift"])
        if op in ("norm_bwd", "norm_bwd8"):
            x = state["x8"] if op == "norm_bwd8" else state["x"]
            return state["plan"].backward(state["dy"], x, state["stats"], state["begin"], state["gain"], state["shift"])
        if op == "store":
            return state["rows8"].store(state["x"]).load(case["dtype"])
        if op == "product":
            return state["plan"].forward(state["x8"].store(state["x"]), state["bias"])
        if op == "product_dx":
            state["plan"].set_weights(state["w"])
            return state["plan"].input_grad(state["dy8"].store(state["dy"]))
        return state["plan"].weight_grad(state["x8"], state["dy8"])
    if op == "norm":
        return _plain_norm(state["x"], state["begin"], state["gain"], state["shift"], case["groups"], case["act"])
    if op in ("norm_bwd", "norm_bwd8"):
        x = _plain_held(state["codes"], state["scales"], case["cols"]) if op == "norm_bwd8" else state["x"]
        return _plain_norm_bwd(state["dy"], x, state["stats"], state["begin"], state["gain"], state["shift"],
                               case["groups"], case["act"])
    if op == "store":
        return _plain_rows8(state["x"]).to(state["x"].dtype)
    if op == "product":
        return (_plain_rows8(state["x"]) @ state["wq"] + state["bias"]).to(state["x"].dtype)
    if op == "product_dx":
        return (_plain_rows8(state["dy"]) @ _plain_matrix8(state["w"].float()).t()).to(state["dy"].dtype)
    dy = _plain_held(state["dy_codes"], state["dy_scales"], case["n"])
    return _plain_held(state["codes"], state["scales"], case["k"]).t() @ dy, dy.sum(0)


# ---------------------------------------------------------------------------------------------------------
# what a pass cannot do without, and its value in 64 bits


def _bytes8(rows, cols):
    return rows * (cols + _blocks(cols))


def work(case):
    size, op, rows = (2 if case["dtype"] == "bf16" else 4), case["op"], case["rows"]
    if op.startswith("norm"):
        n, small = rows * case["cols"], 8 * case["cols"] + 4 * case["batch"] * (1 + 2 * case["groups"])
        if op == "norm":
            return {"bytes": 2 * n * size + small, "flops": 10 * n}
        x = _bytes8(rows, case["cols"]) if op == "norm_bwd8" else n * size
        return {"bytes": 2 * n * size + x + small + 8 * case["cols"], "flops": 22 * n}
    if op == "store":
        n = rows * case["cols"]
        return {"bytes": 2 * n * size + 2 * _bytes8(rows, case["cols"]), "flops": 4 * n}
    k, n = case["k"], case["n"]
    flops = 2 * rows * k * n
    if op == "product":
        return {"bytes": rows * (k + n) * size + k * n + 4 * n, "flops": flops}
    if op == "product_dx":
        return {"bytes": rows * (k + n) * size + k * n * size, "flops": flops}
    return {"bytes": _bytes8(rows, k) + _bytes8(rows, n) + 4 * k * n + 4 * n, "flops": flops}


def _exact_scaled(x, largest):
    """x in e4m3 under the least power of two that brings `largest` within 448."""
    e = torch.where(largest > 0, torch.ceil(torch.log2(largest / 448.0)), torch.full_like(largest, -126.0))
    e = torch.where(448.0 * torch.exp2(e - 1) >= largest, e - 1, e)  # a logarithm rounded up past a border
    e = torch.where(448.0 * torch.exp2(e) < largest, e + 1, e).clamp(min=-126.0)
    scale = torch.exp2(e)
    return (x / scale).float().to(torch.float8_e4m3fn).double() * scale


def _exact_rows8(x):
    parts = []
    for p in x.double().split(BLOCK, 1):
        parts.append(_exact_scaled(p, p.abs().amax(1, keepdim=True)))
    return torch.cat(parts, 1)


def _exact_matrix8(w):
    return torch.cat([torch.cat([_exact_scaled(p, p.abs().max()) for p in s.split(BLOCK, 1)], 1)
                      for s in w.double().split(BLOCK, 0)], 0)


def _exact_held(codes, scales, cols):
    s = torch.exp2(scales.double() - 127.0)
    v = codes.view(torch.float8_e4m3fn).double()
    return torch.cat([v[:, c: min(c + BLOCK, cols)] * s[:, c // BLOCK, None] for c in range(0, cols, BLOCK)], 1)


def _exact_act(z, act):
    """(act(z), act'(z))"""
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s)
    slope = torch.full_like(z, SLOPES[act])
    slope[z > 0 if act == "relu" else z >= 0] = 1.0
    return z * slope, slope


def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    if op == "store":
        return _exact_rows8(s["x"])
    if op == "product":
        return torch.addmm(s["bias"].double(), _exact_rows8(s["x"]), _exact_matrix8(s["w"]))
    if op == "product_dx":
        return torch.mm(_exact_rows8(s["dy"]), _exact_matrix8(s["w"]).t().contiguous())
    if op == "product_dw":
        x, dy = _exact_held(s["codes"], s["scales"], case["k"]), _exact_held(s["dy_codes"], s["dy_scales"], case["n"])
        return torch.mm(x.t().contiguous(), dy), dy.sum(0)
    groups, cols, act = case["groups"], case["cols"], case["act"]
    per, begin = cols // groups, s["begin"].tolist()
    gain, shift = s["gain"].double(), s["shift"].double()
    x = _exact_held(s["codes"], s["scales"], cols) if op == "norm_bwd8" else s["x"].double()
    out = torch.empty_like(x)
    stats = torch.zeros(2, case["batch"], groups, dtype=torch.float64, device=x.device)
    stats[1] = EPS ** -0.5
    dgain, dshift = torch.zeros_like(gain), torch.zeros_like(gain)
    for b in range(case["batch"]):
        at = slice(begin[b], begin[b + 1])
        if begin[b] == begin[b + 1]:
            continue
        if op == "norm":
            var, mean = torch.var_mean(x[at].view(-1, groups, per), dim=(0, 2), unbiased=False)
            r = (var + EPS) ** -0.5
            stats[0, b], stats[1, b] = mean, r
        else:
            mean, r = s["stats"][:, b].double()
        mean, r = mean.repeat_interleave(per), r.repeat_interleave(per)
        h = (x[at] - mean) * r
        y, slope = _exact_act(h * gain + shift, act)
        if op == "norm":
            out[at] = y
            continue
        dz = s["dy"][at].double() * slope
        t = dz * gain
        n = h.shape[0] * per
        m1 = t.sum(0).view(groups, per).sum(1).repeat_interleave(per) / n
        m2 = (t * h).sum(0).view(groups, per).sum(1).repeat_interleave(per) / n
        out[at] = r * (t - m1 - h * m2)
        dgain += (dz * h).sum(0)
        dshift += dz.sum(0)
    return (out, stats) if op == "norm" else (out, dgain, dshift)
