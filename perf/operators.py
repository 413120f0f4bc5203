"""The operators of a training step on gathered feature rows: their plain forms, the calls of the framework, and what each needs.

A model on this data path holds its features as 4-bit rows (a seventh of the bytes over the host link, in the cache and in the
gather's output), projects the gathered rows, normalises them, and updates its weights from clipped gradients:

  quantise   rg_mx4_quantize + rg_mx4_dequantize: rows of numbers to packed 4-bit rows (groups of 32 with a scale of their own) and
             back; the pass returns the values that the packed rows stand for
  product    rg_mx4_matmul: packed rows times packed weight rows, y = rows . weight^T
  gradient   rg_mx4_matmul_grad: the gradient of that product to its weight, dy^T . rows
  norm       rg_layer_norm: layer norm of rows, with each row's mean and reciprocal deviation
  norm-grad  rg_layer_norm_grad: its backward pass to the rows, the gain and the bias
  clip       rg_clip_grad_norm: the norm of all gradients together, and the gradients scaled to a largest norm

A packed row of `dim` numbers has G = ceil(dim / 32) groups: 16 bytes of codes for each (code of number 2i in the low half of
byte i), then a scale byte for each, then zeros up to a multiple of four bytes.  A code is sign and magnitude 0, 0.5, 1, 1.5, 2, 3, 4 or
6; the scale byte s stands for 2^(s - 127), s = 255 for a group that held something that is not finite.

Sizes are those of the five workloads of synth/configs.py: their feature widths, batches' input nodes, and classes.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5


def listed():
    return [
        # a graph's whole feature table to 4 bits, once before training
        dict(name="quantise-copurchase", kind="quantise", rows=2_449_029, dim=100, type="f32"),
        # the means of one dense batch's neighbours, in half precision: latency
        dict(name="quantise-seeds-f16", kind="quantise", rows=1024, dim=602, type="f16"),
        # the projection of the largest batch's input rows, whose result stays in bf16
        dict(name="product-stress-bf16", kind="product", rows=794_123, dim=256, out=256, type="bf16"),
        # one node's classes, as a server answers: latency
        dict(name="product-one-row", kind="product", rows=1, dim=602, out=41, type="f32"),
        # the weight's gradient on the largest batch
        dict(name="gradient-stress-bf16", kind="gradient", rows=794_123, dim=256, out=256, type="bf16"),
        # the same on an ordinary batch with long ragged rows, in full precision
        dict(name="gradient-dense-social", kind="gradient", rows=100_003, dim=602, out=256, type="f32"),
        # layer norm of the largest batch's outermost destinations
        dict(name="norm-stress", kind="norm", rows=270_011, dim=256, type="f32"),
        # of one batch's seeds: latency
        dict(name="norm-seeds-bf16", kind="norm", rows=1024, dim=602, type="bf16"),
        # its backward pass on the largest batch
        dict(name="norm-grad-stress-bf16", kind="norm-grad", rows=794_123, dim=256, type="bf16"),
        # and on a small batch in full precision
        dict(name="norm-grad-tiny", kind="norm-grad", rows=3961, dim=64, type="f32"),
        # the gradients of a model of a few layers, small enough that most steps are not clipped: latency
        dict(name="clip-layers", kind="clip", tensors=13, total=462_001, type="f32", std=1e-3, max_norm=1.0, layout=1),
        # of one that learns a vector for every node
        dict(name="clip-embeddings", kind="clip", tensors=40, total=245_902_903, type="f32", std=1e-2, max_norm=1.0, layout=2),
    ]


# ---------------------------------------------------------------------------- drawing
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantise", "product", "gradient", "norm", "norm-grad", "clip"])
    if kind == "clip":
        total = _log(rng, 2_000, 240_000_000)
        return dict(kind=kind, tensors=_log(rng, 1, min(60, total // 64)), total=total, type=rng.choice(["f32", "bf16", "f16", "mixed"]),
                    std=rng.choice([1e-3, 1e-2]), max_norm=rng.choice([0.1, 1.0, 10.0]), layout=rng.randrange(1 << 30))
    dim = rng.choice([64, 100, 128, 256, 602, _log(rng, 16, 1024)])
    case = dict(kind=kind, rows=1, dim=dim, type=rng.choice(["f32", "bf16", "f16"]))
    width = dim
    if kind in ("product", "gradient"):
        case["out"] = rng.choice([41, 47, 128, 256, _log(rng, 2, 512)])
        width = max(dim, case["out"])
    case["rows"] = _log(rng, 1, min(2_000_000, 180_000_000 // width))
    return case


# ---------------------------------------------------------------------------- inputs
def _sizes(case):
    """Numbers in each tensor of a clip case: one or two large ones, most of them small, as a model's."""
    rng = random.Random(case["layout"])
    weights = [math.exp(rng.uniform(0.0, 9.0)) for _ in range(case["tensors"])]
    sizes = [max(1, int(case["total"] * w / sum(weights))) for w in weights]
    sizes[0] += max(0, case["total"] - sum(sizes))
    return sizes


def _tensor_types(case):
    if case["type"] != "mixed":
        return [case["type"]] * case["tensors"]
    rng = random.Random(case["layout"] + 1)
    return [rng.choice(["f32", "bf16", "f16"]) for _ in range(case["tensors"])]


def _randn(gen, shape, type, std=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * std).to(TYPES[type])


def row_words(dim):
    groups = -(-dim // 32)
    return 4 * groups + -(-groups // 4)


def _row_stride(dim):
    return -(-row_words(dim) // 4) * 4                   # rows that start on 16 bytes


def _inputs(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind = case["kind"]
    if kind == "clip":
        return dict(grads=[_randn(gen, (n,), t, case["std"]) for n, t in zip(_sizes(case), _tensor_types(case))])
    n, dim, type = case["rows"], case["dim"], case["type"]
    if kind == "quantise":
        return dict(x=_randn(gen, (n, dim), type))
    if kind in ("product", "gradient"):
        d = dict(rows=_pack(_randn(gen, (n, dim), "f32"), _row_stride(dim)))
        if kind == "product":
            d["weight"] = _pack(_randn(gen, (case["out"], dim), "f32", dim ** -0.5), _row_stride(dim))
        else:
            d["dy"] = _randn(gen, (n, case["out"]), type, 1e-2)
        return d
    d = dict(x=_randn(gen, (n, dim), type, 1.5) + torch.randn((n, 1), generator=gen, device=DEV).to(TYPES[type]),
             gamma=1.0 + 0.2 * torch.randn((dim,), generator=gen, device=DEV),
             beta=0.2 * torch.randn((dim,), generator=gen, device=DEV))
    if kind == "norm-grad":
        x = d["x"].float()
        d["mean"] = x.mean(1)
        d["rstd"] = torch.rsqrt((x - d["mean"][:, None]).square().mean(1) + EPS)
        d["dy"] = _randn(gen, (n, dim), type, 1e-2)
    return d


_handle = None


def _context():
    """The one handle of the program."""
    global _handle
    if _handle is None:
        from paper_2505_10806_amd import binding as B
        _handle = B.Context(0)
    return _handle


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    if own:
        from paper_2505_10806_amd import binding as B
        state["ctx"] = _context()
        kind, t = case["kind"], TYPES[case["type"]] if case["type"] in TYPES else None
        empty = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=DEV)    # noqa: E731
        if kind == "clip":
            state["out"] = [torch.empty_like(g) for g in state["grads"]]
            state["list"] = B.TensorList(state["grads"], state["out"])
            state["norm"] = empty(1)
            return state
        n, dim = case["rows"], case["dim"]
        if kind == "quantise":
            state["packed"], state["values"] = empty(n, _row_stride(dim)), empty(n, dim)
        elif kind == "product":
            state["y"] = empty(n, case["out"], dtype=t)
        elif kind == "gradient":
            state["grad"] = empty(case["out"], dim)
        elif kind == "norm":
            state["y"], state["mean"], state["rstd"] = empty(n, dim, dtype=t), empty(n), empty(n)
        else:
            state["dx"], state["dgamma"], state["dbeta"] = empty(n, dim, dtype=t), empty(dim), empty(dim)
    return state


# ---------------------------------------------------------------------------- plain forms
def _pack(x, stride):
    """Packed 4-bit rows (float32 words, `stride` to a row) of a matrix."""
    n, dim = x.shape
    groups = -(-dim // 32)
    v = torch.zeros((n, groups * 32), dtype=torch.float32, device=x.device)
    v[:, :dim] = x
    v = v.view(n, groups, 32)
    top = v.abs().amax(2)
    good = torch.isfinite(v).all(2)
    exponent = torch.frexp(torch.where(good, top, torch.ones_like(top)))[1] - 3        # floor(log2(top)) - 2
    exponent = torch.where(top > 0, exponent, torch.full_like(exponent, -127)).clamp(min=-127)
    m = torch.ldexp(v.abs(), -exponent[:, :, None])
    code = torch.zeros(v.shape, dtype=torch.uint8, device=x.device)
    for line, tie_up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (m >= line) if tie_up else (m > line)                                    # halves go to the even code
    code += torch.signbit(v).to(torch.uint8) * 8
    code = torch.where(good[:, :, None], code, torch.zeros_like(code)).view(n, groups * 16, 2)
    out = torch.zeros((n, stride * 4), dtype=torch.uint8, device=x.device)
    out[:, :groups * 16] = code[:, :, 0] + code[:, :, 1] * 16
    out[:, groups * 16:groups * 17] = torch.where(good, exponent + 127, torch.full_like(exponent, 255)).to(torch.uint8)
    return out.view(torch.float32)


def _unpack(packed, dim):
    """The numbers that packed rows stand for, in 32 bits."""
    groups = -(-dim // 32)
    raw = packed.contiguous().view(torch.uint8)
    code = raw[:, :groups * 16]
    code = torch.stack((code & 15, code >> 4), 2).view(-1, groups, 32)
    low = (code & 7).float()
    m = torch.where(low < 4, low * 0.5, torch.where(low < 6, low - 2.0, low * 2.0 - 8.0))
    m = torch.where(code >= 8, -m, m)
    scale = raw[:, groups * 16:groups * 17].int()
    v = torch.ldexp(m, scale[:, :, None] - 127)
    v = torch.where((scale == 255)[:, :, None], torch.full_like(v, math.nan), v)
    return v.view(-1, groups * 32)[:, :dim]


def _plain(state):
    case, kind = state["case"], state["case"]["kind"]
    if kind == "clip":
        norm = torch.zeros((), device=DEV)
        for g in state["grads"]:
            norm = norm + g.float().square().sum()
        norm = norm.sqrt()
        scale = torch.where(torch.isfinite(norm) & (norm > case["max_norm"]), case["max_norm"] / norm, torch.ones_like(norm))
        return dict(norm=norm.view(1), out=[(g.float() * scale).to(g.dtype) for g in state["grads"]])
    dim, t = case["dim"], TYPES[case["type"]]
    if kind == "quantise":
        return dict(values=_unpack(_pack(state["x"].float(), row_words(dim)), dim))
    if kind == "product":
        return dict(y=(_unpack(state["rows"], dim) @ _unpack(state["weight"], dim).t()).to(t))
    if kind == "gradient":
        return dict(grad=state["dy"].float().t() @ _unpack(state["rows"], dim))
    x, gamma = state["x"].float(), state["gamma"]
    if kind == "norm":
        mean = x.mean(1)
        centred = x - mean[:, None]
        rstd = torch.rsqrt(centred.square().mean(1) + EPS)
        return dict(y=(centred * rstd[:, None] * gamma + state["beta"]).to(t), mean=mean, rstd=rstd)
    dy, rstd = state["dy"].float(), state["rstd"][:, None]
    xhat = (x - state["mean"][:, None]) * rstd
    g = dy * gamma
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return dict(dx=dx.to(t), dgamma=(dy * xhat).sum(0), dbeta=dy.sum(0))


# ---------------------------------------------------------------------------- the framework's calls
def _own(state):
    case, ctx, kind = state["case"], state["ctx"], state["case"]["kind"]
    if kind == "clip":
        ctx.clip_grad_norm(state["list"], case["max_norm"], state["norm"])
        return dict(norm=state["norm"], out=state["out"])
    n, dim = case["rows"], case["dim"]
    if kind == "quantise":
        ctx.mx4_quantize(state["x"], n, dim, state["packed"])
        ctx.mx4_dequantize(state["packed"], n, dim, state["values"])
        return dict(values=state["values"])
    if kind == "product":
        ctx.mx4_matmul(state["rows"], n, state["weight"], case["out"], dim, state["y"])
        return dict(y=state["y"])
    if kind == "gradient":
        ctx.mx4_matmul_grad(state["dy"], state["rows"], n, case["out"], dim, state["grad"])
        return dict(grad=state["grad"])
    if kind == "norm":
        ctx.layer_norm(state["x"], n, dim, state["gamma"], state["beta"], EPS, state["y"], state["mean"], state["rstd"])
        return dict(y=state["y"], mean=state["mean"], rstd=state["rstd"])
    ctx.layer_norm_grad(state["dy"], state["x"], n, dim, state["gamma"], state["mean"], state["rstd"], state["dx"], state["dgamma"],
                        state["dbeta"])
    return dict(dx=state["dx"], dgamma=state["dgamma"], dbeta=state["dbeta"])


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    kind = case["kind"]
    if kind == "clip":
        size = sum(n * BYTES[t] for n, t in zip(_sizes(case), _tensor_types(case)))
        return {"bytes": 2 * size + 4, "flops": 3 * sum(_sizes(case))}
    n, dim, b = case["rows"], case["dim"], BYTES[case["type"]]
    packed = 4 * row_words(dim)
    if kind == "quantise":
        return {"bytes": n * (dim * b + packed + dim * 4), "flops": 4 * n * dim}
    if kind == "product":
        return {"bytes": (n + case["out"]) * packed + n * case["out"] * b, "flops": 2 * n * dim * case["out"]}
    if kind == "gradient":
        return {"bytes": n * (packed + case["out"] * b) + case["out"] * dim * 4, "flops": 2 * n * dim * case["out"]}
    if kind == "norm":
        return {"bytes": n * (2 * dim * b + 8) + 8 * dim, "flops": 8 * n * dim}
    return {"bytes": n * (3 * dim * b + 8) + 12 * dim, "flops": 14 * n * dim}


# ---------------------------------------------------------------------------- the definitions in 64 bits
_VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _decode64(packed, dim):
    groups = -(-dim // 32)
    raw = packed.contiguous().view(torch.uint8).long()
    table = torch.tensor(_VALUES + [-v for v in _VALUES], dtype=torch.float64, device=packed.device)
    scales = torch.pow(2.0, torch.arange(256, dtype=torch.float64, device=packed.device) - 127.0)
    scales[255] = math.nan
    place = torch.arange(dim, device=packed.device)
    code = (raw[:, place // 2] >> (4 * (place % 2))) & 15
    return table[code] * scales[raw[:, groups * 16 + place // 32]]


def _nearest64(x):
    """Each group of 32 rounded to the nearest values of its scale (halves to even), in 64 bits."""
    n, dim = x.shape
    out = torch.empty((n, dim), dtype=torch.float64, device=x.device)
    for first in range(0, dim, 32):
        v = x[:, first:first + 32].double()
        top = v.abs().amax(1, keepdim=True)
        good = torch.isfinite(v).all(1, keepdim=True)
        power = torch.floor(torch.log2(torch.where(good & (top > 0), top, torch.ones_like(top))))
        power = power + (torch.pow(2.0, power + 1) <= top).double() - (torch.pow(2.0, power) > top).double() * (top > 0)
        scale = torch.pow(2.0, torch.where(top > 0, power - 2.0, torch.full_like(power, -127.0)).clamp(min=-127.0))
        m = v / scale
        step = torch.where(m.abs() < 2.0, 0.5, torch.where(m.abs() < 4.0, 1.0, 2.0)).double()
        m = (torch.round(m / step) * step).clamp(-6.0, 6.0)
        out[:, first:first + 32] = torch.where(good, m * scale, torch.full_like(m, math.nan))
    return out


def exact(case, seed):
    d, kind = _inputs(case, seed), case["kind"]
    if kind == "clip":
        norm = math.sqrt(sum(float(g.double().pow(2).sum()) for g in d["grads"]))
        scale = case["max_norm"] / norm if math.isfinite(norm) and norm > case["max_norm"] else 1.0
        return dict(norm=torch.tensor([norm], dtype=torch.float64, device=DEV), out=[g.double() * scale for g in d["grads"]])
    dim = case["dim"]
    if kind == "quantise":
        return dict(values=_nearest64(d["x"]))
    if kind == "product":
        return dict(y=torch.matmul(_decode64(d["rows"], dim), _decode64(d["weight"], dim).t().contiguous()))
    if kind == "gradient":
        return dict(grad=torch.matmul(d["dy"].double().t().contiguous(), _decode64(d["rows"], dim)))
    x, gamma = d["x"].double(), d["gamma"].double()
    if kind == "norm":
        mean = x.sum(1) / dim
        variance = (x * x).sum(1) / dim - mean * mean
        rstd = 1.0 / torch.sqrt(variance + EPS)
        return dict(y=(x - mean[:, None]) * (rstd[:, None] * gamma[None, :]) + d["beta"].double(), mean=mean, rstd=rstd)
    dy, mean, rstd = d["dy"].double(), d["mean"].double()[:, None], d["rstd"].double()[:, None]
    xhat = (x - mean) * rstd
    share = torch.matmul(dy, gamma[:, None]) / dim
    along = torch.matmul(dy * xhat, gamma[:, None]) / dim
    return dict(dx=(dy * gamma - share - xhat * along) * rstd, dgamma=(dy * xhat).sum(0), dbeta=dy.sum(0))
