"""Training a factor model on a CSF tensor: the operators that follow the contraction, in their plain form and as calls of the library.

Two operators:
  loss  softmax cross entropy over the leaf mode of a CSF tensor, with its gradient (const_softmax_loss).  A CP model scores
        every coordinate k of the leaf mode for a stored fibre (i, j): s_k = sum_r A[i,r] B[j,r] C[k,r]; the leaves of the fibre
        are the targets, weighted with their values.  Of order 2 this is the loss of a language model's head: rows of hidden
        states, a table of the vocabulary, one target a row.
  clip  the global norm of many gradients, and the gradients scaled so that it is at most max_norm (const_clip_gradients).

Sizes are those of workloads/generators.py (200^3 at rank 8; 12000 x 9000 x 29000 at rank 16; 50000^3 at rank 32), the paper's rank 50,
or generic and ragged.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _loss(name, dims, rank, fibres, leaves, dtype="f32", grad=True):
    """dims: extents in level order; fibres: rows of the softmax; leaves: targets a row (on average, at least one)."""
    return {"name": name, "op": "loss", "dims": dims, "rank": rank, "fibres": fibres, "leaves": leaves, "dtype": dtype, "grad": grad}


def _clip(name, count, values, dtype="f32", factor=0.5):
    """count tensors of `values` values in all; max_norm is `factor` times their norm."""
    return {"name": name, "op": "clip", "count": count, "values": values, "dtype": dtype, "factor": factor}


def listed():
    return [
        # scoring one fibre: a query with one answer, against the whole leaf mode (latency)
        _loss("score_one", "12000x9000x29000", 16, 1, 1.0, grad=False),
        # a whole small tensor a step: 20 000 nonzeros of 200^3
        _loss("train_small_r8", "200x200x200", 8, 15_700, 1.27),
        # a batch of the large skewed tensor's fibres, several targets each
        _loss("train_r16", "12000x9000x29000", 16, 8_192, 4.0),
        # the uniform tensor at rank 32
        _loss("train_r32", "50000x50000x50000", 32, 16_384, 1.0),
        # the paper's rank, ragged extents, order 4
        _loss("train_o4_r50", "301x701x1501x28999", 50, 4_099, 1.5),
        # few rows and a long vocabulary: the work is split over the vocabulary
        _loss("train_few_rows", "2003x100003", 64, 77, 1.0),
        # a language model's head: hidden states in 16 bits, one target a row, the largest training step
        _loss("train_head_bf16", "16384x50000", 128, 16_000, 1.0, dtype="bf16"),
        # evaluation alone, on held-out fibres
        _loss("evaluate_r64", "50000x50000x50000", 64, 8_191, 1.0, grad=False),
        # gradients of the three factors of the 200^3 tensor (latency)
        _clip("clip_3_small", 3, 4_800),
        # gradients of the three factors of the 50 000^3 tensor at rank 32
        _clip("clip_3_r32", 3, 4_800_000),
        # many tensors of mixed sizes in 16 bits
        _clip("clip_300_bf16", 300, 60_000_007, dtype="bf16"),
        # the factors of a tensor with tens of millions of coordinates
        _clip("clip_3_large", 3, 488_640_000, factor=0.01),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["f32", "f32", "bf16"])
    if rng.random() < 0.35:
        return {k: v for k, v in _clip("", _log_uniform(rng, 1, 400), _log_uniform(rng, 1_000, 200_000_000), dtype,
                                       rng.choice([0.01, 0.5, 2.0])).items() if k != "name"}
    order = rng.choice([2, 3, 3, 4])
    fibres = _log_uniform(rng, 1, 20_000)
    vocabulary = _log_uniform(rng, 50, 100_000)
    rank = rng.choice([4, 7, 8, 16, 24, 32, 50, 64, 100, 128])
    while fibres * vocabulary * rank > 16_000 * 50_000 * 128 or fibres * vocabulary > 900_000_000:
        fibres = (fibres + 1) // 2
    dims = [_log_uniform(rng, 50, 20_000) for _ in range(order - 1)]
    dims[0] = max(dims[0], fibres if order == 2 else fibres // 50 + 1)
    if order > 2:
        dims[1] = max(dims[1], 100)
    dims.append(vocabulary)
    case = _loss("", "x".join(str(d) for d in dims), rank, fibres, rng.choice([1.0, 1.5, 4.0]), dtype, rng.random() < 0.75)
    return {k: v for k, v in case.items() if k != "name"}


def _pieces(case):
    """How many values each of the tensors of a clip case has: sizes spread over a factor of some thousands, none empty."""
    count, total = case["count"], case["values"]
    weights = [math.exp(8.0 * ((0.37 + 0.6180339887 * t) % 1.0)) for t in range(count)]
    scale = max(total - count, 0) / sum(weights)
    sizes = [1 + int(w * scale) for w in weights]
    sizes[0] += max(total - sum(sizes), 0)
    return sizes


def _inputs(case, seed):
    """The inputs as tensors: of a loss the factors in level order, the coordinates of every level above the leaves for each
    fibre (in lexicographic order), and fibre, coordinate and value of every leaf; of a clip the gradients and their largest norm."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "clip":
        flat = torch.randn(sum(_pieces(case)), device="cuda", generator=g) * 1e-3
        grads = [(t * float(10.0 ** (n % 3 - 1))).to(dtype) for n, t in enumerate(torch.split(flat, _pieces(case)))]
        norm = math.sqrt(sum(float(t.double().square().sum()) for t in grads))
        return {"grads": grads, "max_norm": case["factor"] * norm}
    dims = [int(d) for d in case["dims"].split("x")]
    upper, vocabulary, rank, fibres = dims[:-1], dims[-1], case["rank"], case["fibres"]
    cells = math.prod(upper)
    if cells <= 4_000_000:
        key = torch.randperm(cells, device="cuda", generator=g)[:fibres].sort().values
    else:                                               # slices of unequal size: the root coordinate is drawn with a skew
        lower = cells // upper[0]
        u = torch.rand(4 * fibres + 64, device="cuda", generator=g, dtype=torch.float64)
        root = (u.square() * upper[0]).long().clamp_(max=upper[0] - 1)
        key = torch.unique(root * lower + torch.randint(lower, root.shape, device="cuda", generator=g))
        key = key[torch.randperm(key.numel(), device="cuda", generator=g)[:fibres]].sort().values
    coords, rest = [], key
    for d in reversed(upper):
        coords.insert(0, rest % d)
        rest = rest // d
    more = int(round((case["leaves"] - 1.0) * fibres))
    row = torch.cat([torch.arange(fibres, device="cuda"), torch.randint(fibres, (more,), device="cuda", generator=g)])
    u = torch.rand(row.numel(), device="cuda", generator=g, dtype=torch.float64)
    leaf = torch.unique(row * vocabulary + (u.pow(3) * vocabulary).long().clamp_(max=vocabulary - 1))   # popular coordinates first
    row, col = leaf // vocabulary, leaf % vocabulary
    x = 1.0 - torch.rand(leaf.numel(), device="cuda", generator=g) if case["leaves"] > 1 else torch.ones(leaf.numel(), device="cuda")
    # scores of a standard deviation of about 3, as a model has after some training
    size = (3.0 / math.sqrt(rank)) ** (1.0 / len(dims))
    factors = [(torch.randn(d, rank, device="cuda", generator=g) * size).to(dtype) for d in dims]
    return {"dims": dims, "factors": factors, "coords": coords, "row": row, "col": col, "x": x, "scale": 1.0 / fibres}


def _side_by_side(tensors):
    """A buffer with room for all of them, each from a multiple of 16 bytes on (zeros between), and the views."""
    step = 16 // tensors[0].element_size()
    first, total = [], 0
    for t in tensors:
        first.append(total)
        total += -(-t.numel() // step) * step
    flat = torch.zeros(total, dtype=tensors[0].dtype, device="cuda")
    return flat, [flat[at:at + t.numel()] for at, t in zip(first, tensors)]


def prepare(case, seed):
    state = {"case": case, **_inputs(case, seed)}
    if case["op"] == "clip":                            # the clipped gradients side by side in one buffer
        state["norm"] = torch.empty(1, device="cuda")
        state["flat"], state["out"] = _side_by_side(state["grads"])
        return state
    state["loss"] = torch.empty(case["fibres"], device="cuda")
    state["out"] = [torch.empty_like(f) for f in state["factors"]] if case["grad"] else None
    if own:
        import paper_2401_04836_b200 as cb
        modes = [c[state["row"]].int() for c in state["coords"]] + [state["col"].int()]
        state["csf"] = cb.const_csf_build(modes, state["x"], state["dims"], list(range(len(modes))))
    return state


def _run_own(state):
    import paper_2401_04836_b200 as cb
    if state["case"]["op"] == "clip":
        cb.const_clip_gradients(state["grads"], state["max_norm"], state["norm"], out=state["out"])
        return {"norm": state["norm"], "grads": state["flat"]}
    cb.const_softmax_loss(state["csf"], state["factors"], state["loss"], grads=state["out"], scale=state["scale"])
    return {"loss": state["loss"], "grads": state["out"]}


def _product(rows):
    h = rows[0]
    for r in rows[1:]:
        h = h * r
    return h


def _clip_plain(grads, max_norm, out):
    total = torch.stack([torch.linalg.vector_norm(g.float()) for g in grads]).square().sum().sqrt()
    factor = (max_norm / total).clamp(max=1.0)
    torch._foreach_copy_(out, [g.float() * factor for g in grads])
    return total.reshape(1)


def _loss_plain(state):
    *upper, table = [f.float() for f in state["factors"]]
    row, col, x, scale = state["row"], state["col"], state["x"], state["scale"]
    rows = [f[c] for f, c in zip(upper, state["coords"])]
    h = _product(rows)
    scores = h @ table.t()
    top = scores.amax(1, keepdim=True)
    shares = torch.exp(scores - top)
    total = shares.sum(1, keepdim=True)
    weight = torch.zeros_like(h[:, 0]).index_add_(0, row, x)
    lse = (top + torch.log(total))[:, 0]
    loss = weight * lse - torch.zeros_like(lse).index_add_(0, row, x * scores[row, col])
    if not state["case"]["grad"]:
        return loss, None
    del scores
    shares *= weight[:, None] / total
    shares.index_put_((row, col), -x, accumulate=True)
    d_table = shares.t() @ h * scale
    d_h = (shares.double() @ table.double()).float() * scale        # a long sum of terms that nearly cancel
    grads = []
    for n, (f, c) in enumerate(zip(upper, state["coords"])):
        others = [r for m, r in enumerate(rows) if m != n]
        grads.append(torch.zeros_like(f).index_add_(0, c, _product([d_h] + others)))
    return loss, [g.to(f.dtype) for g, f in zip(grads + [d_table], state["factors"])]


def run(state):
    if own:
        got = _run_own(state)
    elif state["case"]["op"] == "clip":
        got = {"norm": _clip_plain(state["grads"], state["max_norm"], state["out"]), "grads": state["flat"]}
    else:
        loss, grads = _loss_plain(state)
        got = {"loss": loss, "grads": grads}
    return got


def work(case):
    wide = DTYPES[case["dtype"]].itemsize
    if case["op"] == "clip":
        return {"bytes": 2.0 * wide * case["values"], "flops": 3.0 * case["values"]}
    dims = [int(d) for d in case["dims"].split("x")]
    rank, fibres, vocabulary, leaves = case["rank"], case["fibres"], dims[-1], case["leaves"] * case["fibres"]
    gathered = sum(min(d, fibres) for d in dims[:-1])
    moved = wide * rank * (gathered + vocabulary) + 8.0 * leaves + 4.0 * fibres * len(dims)
    if case["grad"]:
        moved += wide * rank * sum(dims)
    return {"bytes": moved, "flops": (6.0 if case["grad"] else 2.0) * fibres * vocabulary * rank}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "clip":
        norm = torch.sqrt(sum((t.double() ** 2).sum() for t in s["grads"]))
        scale = torch.minimum(torch.ones_like(norm), s["max_norm"] / norm)
        flat, views = _side_by_side(s["grads"])
        whole = torch.zeros(flat.shape, dtype=torch.float64, device="cuda")
        for v, t in zip(views, s["grads"]):
            whole[v.storage_offset():v.storage_offset() + t.numel()] = t.double() * scale
        return {"norm": norm.reshape(1), "grads": whole}
    factors = [f.double() for f in s["factors"]]
    fibres, x = case["fibres"], s["x"].double()
    d_factors = [torch.zeros_like(f) for f in factors]
    loss = torch.zeros(fibres, dtype=torch.float64, device="cuda")
    for first in range(0, fibres, 1024):                # row by row the definition; 1024 rows at a time for memory
        last = min(first + 1024, fibres)
        mine = (s["row"] >= first) & (s["row"] < last)
        target = torch.zeros(last - first, factors[-1].shape[0], dtype=torch.float64, device="cuda")
        target[s["row"][mine] - first, s["col"][mine]] = x[mine]
        at = [c[first:last] for c in s["coords"]]
        hidden = torch.ones(last - first, case["rank"], dtype=torch.float64, device="cuda")
        for f, c in zip(factors, at):
            hidden = hidden * f[c]
        logits = torch.einsum("fr,kr->fk", hidden, factors[-1])
        log_p = logits - torch.logsumexp(logits, 1, keepdim=True)
        loss[first:last] = -(target * log_p).sum(1)
        if case["grad"]:
            g = (target.sum(1, keepdim=True) * torch.exp(log_p) - target) * s["scale"]
            d_factors[-1] += torch.einsum("fk,fr->kr", g, hidden)
            d_hidden = torch.einsum("fk,kr->fr", g, factors[-1])
            for n in range(len(at)):
                term = d_hidden.clone()
                for m, (f, c) in enumerate(zip(factors, at)):
                    if m != n:
                        term = term * f[c]
                d_factors[n].index_put_((at[n],), term, accumulate=True)
    return {"loss": loss, "grads": d_factors if case["grad"] else None}
