"""The operators of a model that learns a vector for every node: their plain forms, the calls of the framework, and what each needs.

Where nodes have no features, or beside the ones they have, a model on this data path learns their vectors: it looks up those of a
sampled batch, and what it answers with is a class, or a node among all nodes.  The two ends of its step:

  lookup      rg_embedding: rows of a table by id, times a factor
  rows-grad   rg_embedding_grad_rows: the gradient of the looked-up rows, summed by id, as the list of the ids met (ascending) and a row for each
  table-grad  rg_embedding_grad: the same as a whole table, zeros (or what it held) where no id was met
  loss        rg_cross_entropy: softmax cross entropy of rows . weight^T against labels, with each row's log of the sum of exponentials;
              the logits are not kept
  loss-grad   rg_cross_entropy_grad: its gradients to the rows and to the weight

Ids outside [0, table rows) are padding: they read as zeros and add to no gradient.  Labels outside [0, classes) mark rows that do not
count: their loss, log-sum and gradient are 0 and they add nothing to the weight's.

Sizes are those of the workloads of synth/configs.py: their nodes, feature widths, batches (seeds and input nodes) and classes.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # the vectors of the largest batch's input nodes (all different), scaled by sqrt(dim)
        dict(name="lookup-stress-bf16", kind="lookup", n=794_123, table=10_000_000, dim=256, type="bf16", out="bf16", ids="distinct", scale=16.0),
        # one batch's seeds, 32-bit vectors into the 16-bit rows that a product takes: latency
        dict(name="lookup-seeds", kind="lookup", n=1024, table=232_965, dim=602, type="f32", out="bf16", ids="distinct", scale=1.0),
        # the gradient of that lookup, only the rows met
        dict(name="rows-grad-stress-bf16", kind="rows-grad", n=794_123, table=10_000_000, dim=256, type="bf16", ids="distinct", scale=16.0),
        # of one small batch's seeds: latency
        dict(name="rows-grad-tiny", kind="rows-grad", n=256, table=10_000, dim=64, type="f32", ids="skewed", scale=1.0),
        # of vectors for the categories of a batch's nodes: few ids, each met thousands of times
        dict(name="table-grad-categories", kind="table-grad", n=1_500_003, table=47, dim=100, type="f32", out="f32", ids="skewed", scale=1.0, add=False),
        # of the ends of sampled edges, hubs met often, as the whole table that an optimiser with momentum takes
        dict(name="table-grad-edges-f16", kind="table-grad", n=65_536, table=200_000, dim=128, type="f16", out="f32", ids="skewed", scale=1.0, add=False),
        # the loss of one batch's seeds over a data set's classes: latency
        dict(name="loss-classes", kind="loss", n=1024, classes=41, dim=256, type="f32"),
        # one row against all nodes, as a server scores an answer: the weight is read once
        dict(name="loss-one-row-bf16", kind="loss", n=1, classes=2_449_029, dim=100, type="bf16"),
        # the largest batch's seeds, each to be told from all nodes
        dict(name="loss-social-f16", kind="loss", n=4096, classes=232_965, dim=256, type="f16"),
        # the gradient over few classes of many nodes, in full precision: every row counts, with a weight of its own
        dict(name="loss-grad-classes", kind="loss-grad", n=100_003, classes=47, dim=256, type="f32", weights=True),
        # one batch's seeds among all nodes, ragged rows; the weight's gradient is the largest output
        dict(name="loss-grad-copurchase-bf16", kind="loss-grad", n=1024, classes=2_449_029, dim=100, type="bf16", weights=False),
        # the same on a smaller graph in full precision
        dict(name="loss-grad-small", kind="loss-grad", n=1024, classes=200_000, dim=128, type="f32", weights=False),
    ]


# ---------------------------------------------------------------------------- drawing
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["lookup", "rows-grad", "table-grad", "loss", "loss-grad"])
    type = rng.choice(["f32", "bf16", "f16"])
    if kind in ("loss", "loss-grad"):
        dim = rng.choice([64, 100, 128, 256, 602, _log(rng, 16, 1024)])
        classes = rng.choice([41, 47, _log(rng, 2, 2_449_029), _log(rng, 256, 400_000)])
        most = 2.4e11 if type != "f32" else 2.4e10               # numbers multiplied
        n = _log(rng, 1, max(1, min(200_000, int(most / (classes * dim)), 2_500_000_000 // classes)))
        case = dict(kind=kind, n=n, classes=classes, dim=dim, type=type)
        if kind == "loss-grad":
            case["weights"] = rng.random() < 0.5
        return case
    dim = rng.choice([64, 100, 128, 256, 602, _log(rng, 16, 1024)])
    n = _log(rng, 1, min(2_000_000, 200_000_000 // dim))
    table = rng.choice([47, _log(rng, 2, 2_449_029)])
    table = min(table, 400_000_000 // dim)
    case = dict(kind=kind, n=n, table=table, dim=dim, type=type, ids=rng.choice(["distinct", "skewed", "padded"]),
                scale=rng.choice([1.0, math.sqrt(dim), 0.125]))
    if case["ids"] == "distinct":
        case["n"] = min(n, table)
    if kind != "rows-grad":
        case["out"] = rng.choice(sorted({"f32", type}))
    if kind == "table-grad":
        case["add"] = rng.random() < 0.5
    return case


# ---------------------------------------------------------------------------- inputs
def _randn(gen, shape, type, std=1.0):
    return torch.randn(shape, generator=gen, device=DEV, dtype=TYPES[type]) * std


def _ids(case, gen):
    n, table = case["n"], case["table"]
    if case["ids"] == "distinct":
        if table <= 4 * n:
            return torch.randperm(table, generator=gen, device=DEV)[:n].int()
        step = table // n                                  # one node of every stretch of them, in no order
        at = torch.arange(n, device=DEV) * step + torch.randint(0, step, (n,), generator=gen, device=DEV)
        return at[torch.randperm(n, generator=gen, device=DEV)].int()
    u = torch.rand((n,), generator=gen, device=DEV, dtype=torch.float64)
    ids = (u.pow(3) * table).long().clamp(max=table - 1).int()               # hubs first
    if case["ids"] == "padded":
        gone = torch.rand((n,), generator=gen, device=DEV) < 0.1
        ids = torch.where(gone, torch.full_like(ids, -1), ids)
    return ids


def _inputs(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    n, dim, kind, type = case["n"], case["dim"], case["kind"], case["type"]
    if kind in ("loss", "loss-grad"):
        classes = case["classes"]
        d = dict(x=_randn(gen, (n, dim), type), weight=_randn(gen, (classes, dim), type, 2.0 * dim ** -0.5),
                 labels=torch.randint(0, classes, (n,), generator=gen, device=DEV).int())
        if n > 8:                                          # some have no label
            d["labels"] = torch.where(torch.rand((n,), generator=gen, device=DEV) < 0.05, torch.full_like(d["labels"], -1), d["labels"])
        if kind == "loss-grad":
            d["lse"] = _log_sums(d["x"].float(), d["weight"].float(), d["labels"])
            d["dloss"] = torch.rand((n,), generator=gen, device=DEV) * 2.0 if case["weights"] else None
        return d
    d = dict(ids=_ids(case, gen))
    if kind == "lookup":
        d["table"] = _randn(gen, (case["table"], dim), type)
    else:
        d["dy"] = _randn(gen, (n, dim), type)
        if kind == "table-grad" and case["add"]:
            d["before"] = _randn(gen, (case["table"], dim), case["out"])
    return d


def _log_sums(x, weight, labels):
    """Each row's log of the sum of exponentials of its logits (0 where it does not count), the weight taken in pieces."""
    top = torch.full((x.shape[0],), -math.inf, device=x.device)
    total = torch.zeros_like(top)
    piece = max(1, (1 << 28) // x.shape[0])
    for first in range(0, weight.shape[0], piece):
        z = x @ weight[first:first + piece].t()
        now = torch.maximum(top, z.amax(1))
        total = total * (top - now).exp() + (z - now[:, None]).exp().sum(1)
        top = now
    return torch.where((labels >= 0) & (labels < weight.shape[0]), top + total.log(), torch.zeros_like(top))


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
        state["ctx"] = _context()
        kind, n, dim = case["kind"], case["n"], case["dim"]
        empty = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=DEV)    # noqa: E731
        if kind == "lookup":
            state["y"] = empty(n, dim, dtype=TYPES[case["out"]])
        elif kind == "table-grad":
            state["grad"] = empty(case["table"], dim, dtype=TYPES[case["out"]])
        elif kind == "rows-grad":                          # (what lies behind the rows met is left as it was)
            most = min(n, case["table"])
            state["grad"] = torch.zeros((most, dim), device=DEV)
            state["touched"] = torch.full((most,), -1, dtype=torch.int32, device=DEV)
            state["count"] = torch.zeros((1,), dtype=torch.int32, device=DEV)
        elif kind == "loss":
            state["loss"], state["log_sum"] = empty(n), empty(n)
        else:
            state["dx"], state["dweight"] = torch.empty_like(state["x"]), torch.empty_like(state["weight"])
    return state


# ---------------------------------------------------------------------------- plain forms
def _plain(state):
    case, kind = state["case"], state["case"]["kind"]
    if kind == "lookup":
        ids, table = state["ids"].long(), state["table"]
        there = (ids >= 0) & (ids < table.shape[0])
        y = table[torch.where(there, ids, torch.zeros_like(ids))].float() * case["scale"]
        return dict(y=torch.where(there[:, None], y, torch.zeros_like(y)).to(TYPES[case["out"]]))
    if kind in ("table-grad", "rows-grad"):
        ids, rows, dim = state["ids"].long(), case["table"], case["dim"]
        there = (ids >= 0) & (ids < rows)
        dy = torch.where(there[:, None], state["dy"].float(), torch.zeros((), device=DEV))
        to = torch.where(there, ids, torch.full_like(ids, rows))             # padding: a row behind the last
        if kind == "table-grad":
            grad = torch.zeros((rows + 1, dim), device=DEV).index_add_(0, to, dy)[:rows] * case["scale"]
            if case["add"]:
                grad = grad + state["before"].float()
            return dict(grad=grad.to(TYPES[case["out"]]))
        met = torch.zeros((rows + 1,), dtype=torch.int64, device=DEV)
        met[to] = 1
        met[rows] = 0
        place = met.cumsum(0) - 1
        most = min(case["n"], rows)
        place[rows] = most
        touched = torch.full((most + 1,), -1, dtype=torch.int32, device=DEV)
        touched[place[to]] = to.int()
        touched[most] = -1
        grad = torch.zeros((most + 1, dim), device=DEV).index_add_(0, place[to], dy)[:most] * case["scale"]
        return dict(count=met.sum().int().view(1), touched=touched[:most], grad=grad)
    x, weight, labels = state["x"].float(), state["weight"].float(), state["labels"].long()
    counts = (labels >= 0) & (labels < weight.shape[0])
    at = torch.where(counts, labels, torch.zeros_like(labels))
    z = x @ weight.t()
    if kind == "loss":
        target = z.gather(1, at[:, None])[:, 0]
        top = z.amax(1)
        log_sum = top + z.sub_(top[:, None]).exp_().sum(1).log()
        nothing = torch.zeros_like(top)
        return dict(loss=torch.where(counts, log_sum - target, nothing), log_sum=torch.where(counts, log_sum, nothing))
    z = z.sub_(state["lse"][:, None]).exp_()
    z.scatter_add_(1, at[:, None], torch.full((z.shape[0], 1), -1.0, device=DEV))
    share = torch.full((z.shape[0],), 1.0 / z.shape[0], device=DEV)
    if state["dloss"] is not None:
        share = share * state["dloss"]
    z.mul_(torch.where(counts, share, torch.zeros_like(share))[:, None])
    return dict(dx=(z @ weight).to(TYPES[case["type"]]), dweight=(z.t() @ x).to(TYPES[case["type"]]))


# ---------------------------------------------------------------------------- the framework's calls
def _own(state):
    case, ctx, kind = state["case"], state["ctx"], state["case"]["kind"]
    n, dim = case["n"], case["dim"]
    if kind == "lookup":
        ctx.embedding(state["table"], case["table"], state["ids"], n, dim, state["y"], scale=case["scale"])
        return dict(y=state["y"])
    if kind == "table-grad":
        if case["add"]:
            state["grad"].copy_(state["before"])
        ctx.embedding_grad(state["dy"], state["ids"], n, dim, case["table"], state["grad"], scale=case["scale"], add=case["add"])
        return dict(grad=state["grad"])
    if kind == "rows-grad":
        ctx.embedding_grad_rows(state["dy"], state["ids"], n, dim, case["table"], state["grad"], state["touched"], state["count"],
                                scale=case["scale"])
        return dict(count=state["count"], touched=state["touched"], grad=state["grad"])
    if kind == "loss":
        ctx.cross_entropy(state["x"], n, dim, state["weight"], case["classes"], state["labels"], state["loss"], state["log_sum"])
        return dict(loss=state["loss"], log_sum=state["log_sum"])
    ctx.cross_entropy_grad(state["x"], n, dim, state["weight"], case["classes"], state["labels"], state["lse"], state["dx"], state["dweight"],
                           dloss=state["dloss"], scale=1.0 / n)
    return dict(dx=state["dx"], dweight=state["dweight"])


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    kind, n, dim, b = case["kind"], case["n"], case["dim"], BYTES[case["type"]]
    if kind in ("loss", "loss-grad"):
        classes = case["classes"]
        read, products = (n + classes) * dim * b, 2 * n * classes * dim
        if kind == "loss":
            return {"bytes": read + 12 * n, "flops": products}
        return {"bytes": 2 * read + (12 if case["weights"] else 8) * n, "flops": 3 * products}     # logits again, then both gradients
    table = case["table"]
    met = min(n, table)
    if kind == "lookup":
        return {"bytes": 4 * n + met * dim * b + n * dim * BYTES[case["out"]], "flops": n * dim}
    size = n * (4 + dim * b)
    if kind == "rows-grad":
        return {"bytes": size + met * (4 + 4 * dim) + 4, "flops": n * dim}
    return {"bytes": size + table * dim * BYTES[case["out"]] * (2 if case["add"] else 1), "flops": n * dim}


# ---------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    d, kind = _inputs(case, seed), case["kind"]
    f64 = torch.float64
    if kind == "lookup":
        ids = d["ids"].long()
        y = torch.zeros((case["n"], case["dim"]), dtype=f64, device=DEV)
        good = ((ids >= 0) & (ids < case["table"])).nonzero()[:, 0]
        y[good] = d["table"].index_select(0, ids[good]).double() * case["scale"]
        return dict(y=y)
    if kind in ("table-grad", "rows-grad"):
        ids = d["ids"].long()
        good = ((ids >= 0) & (ids < case["table"])).nonzero()[:, 0]
        met, group = torch.unique(ids[good], return_inverse=True)
        sums = torch.zeros((met.numel(), case["dim"]), dtype=f64, device=DEV)
        sums.index_add_(0, group, d["dy"][good].double())
        sums *= case["scale"]
        if kind == "table-grad":
            grad = d["before"].double() if case["add"] else torch.zeros((case["table"], case["dim"]), dtype=f64, device=DEV)
            grad[met] += sums
            return dict(grad=grad)
        most = min(case["n"], case["table"])
        touched = torch.full((most,), -1, dtype=torch.int32, device=DEV)
        touched[:met.numel()] = met.int()
        grad = torch.zeros((most, case["dim"]), dtype=f64, device=DEV)
        grad[:met.numel()] = sums
        return dict(count=torch.tensor([met.numel()], dtype=torch.int32, device=DEV), touched=touched, grad=grad)
    x, labels, classes, n = d["x"].double(), d["labels"].long(), case["classes"], case["n"]
    valid = ((labels >= 0) & (labels < classes)).double()
    piece = max(1, (1 << 28) // n)
    if kind == "loss":
        tops, sums = [], []
        target = torch.zeros((n,), dtype=f64, device=DEV)
        for first in range(0, classes, piece):
            w = d["weight"][first:first + piece].double()
            z = torch.matmul(x, w.t().contiguous())
            inside = ((labels >= first) & (labels < first + w.shape[0])).nonzero()[:, 0]
            target[inside] = z[inside, labels[inside] - first]
            tops.append(z.max(1)[0])
            sums.append(torch.exp(z - tops[-1][:, None]).sum(1))
        tops, sums = torch.stack(tops), torch.stack(sums)
        top = tops.max(0)[0]
        log_sum = top + torch.log((sums * torch.exp(tops - top)).sum(0))
        return dict(loss=(log_sum - target) * valid, log_sum=log_sum * valid)
    share = valid / n
    if d["dloss"] is not None:
        share = share * d["dloss"].double()
    dx = torch.zeros_like(x)
    dweight = torch.empty((classes, case["dim"]), dtype=f64, device=DEV)
    for first in range(0, classes, piece):
        w = d["weight"][first:first + piece].double()
        g = torch.exp(torch.matmul(x, w.t().contiguous()) - d["lse"].double()[:, None])
        inside = ((labels >= first) & (labels < first + w.shape[0])).nonzero()[:, 0]
        g[inside, labels[inside] - first] -= 1.0
        g *= share[:, None]
        dx += torch.matmul(g, w)
        dweight[first:first + piece] = torch.matmul(g.t().contiguous(), x)
    return dict(dx=dx, dweight=dweight)
