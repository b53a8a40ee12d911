"""const_softmax_loss against the definition in 64 bits, its gradient also against differences of the definition's loss."""
import numpy as np
import pytest
import torch

import paper_2401_04836_b200 as cb
from tests.gpu_util import to_dev
from tests.loss_reference import fibres_of, loss_and_gradient

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True, params=["by size", "tensor cores", "fp32 pipes"])
def path(request):
    """Which kernels make the scores (the tensor cores' take ranks up to 128): as chosen by size, and each for every size."""
    cb.const_debug_set(2, {"by size": 0, "tensor cores": 2, "fp32 pipes": 1}[request.param])
    yield request.param
    cb.const_debug_set(2, 0)


class Case:
    """A random tensor of `nnz` distinct nonzeros (at most) with factors whose scores spread by about `spread`."""

    def __init__(self, dims, rank, nnz, mode_order=None, dtype="f32", seed=0, weights="unit", spread=3.0, scale=0.37, size=1.0):
        rng = np.random.default_rng([seed, rank, nnz, *dims])
        self.dims, self.rank, self.dtype, self.scale = dims, rank, dtype, scale
        self.mode_order = tuple(mode_order or range(len(dims)))
        flat = np.unique(rng.integers(0, np.prod(dims, dtype=np.int64), nnz))
        rng.shuffle(flat)
        self.coords = [c.astype(np.int32) for c in np.unravel_index(flat, dims)]
        n = len(flat)
        self.x = {"unit": np.ones(n), "uniform": 1 - rng.random(n), "signed": rng.standard_normal(n),
                  "zeros": (rng.random(n) < 0.5) * 1.0, "wide": 10.0 ** rng.uniform(-4, 4, n)}[weights].astype(np.float32)
        each = (spread / np.sqrt(rank)) ** (1.0 / len(dims))
        factors = [(rng.standard_normal((d, rank)) * each).astype(np.float32) for d in dims]
        factors[self.mode_order[-1]] *= np.float32(size)                 # the scores stay as they are
        factors[self.mode_order[0]] *= np.float32(1.0 / size)
        self.factors = [to_dev(f).to(TYPES[dtype]) for f in factors]
        self.fibres = len(fibres_of(self.coords, self.mode_order)[0])

    def handle(self):
        return cb.const_csf_build([to_dev(c) for c in self.coords], to_dev(self.x), self.dims, self.mode_order)

    def run(self, grads=True, handle=None):
        self.loss = torch.full((self.fibres,), float("nan"), device="cuda")
        self.grads = [torch.full_like(f, float("nan")) if (grads is True or grads[m]) else None for m, f in enumerate(self.factors)] \
            if grads else None
        cb.const_softmax_loss(handle or self.handle(), self.factors, self.loss, grads=self.grads, scale=self.scale)
        return self

    def expected(self):
        return loss_and_gradient(self.coords, self.x, [f.double().cpu().numpy() for f in self.factors], self.mode_order, self.scale,
                                 self.dtype == "bf16")

    def check(self):
        (loss, bound), grads = self.expected()
        within(self.loss, loss, bound, "loss")
        for m, g in enumerate(self.grads or []):
            if g is not None:
                within(g, *grads[m], f"gradient of mode {m}")
        return self


def within(got, value, bound, what):
    got = got.double().cpu().numpy()
    assert np.all(np.isfinite(got)), f"{what}: not finite, or an element was never written"
    far = np.abs(got - value) / bound
    assert far.max(initial=0.0) <= 1.0, f"{what}: {far.max()} times its bound at {np.unravel_index(far.argmax(), far.shape)}"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rank", [1, 3, 8, 16, 17, 32, 33, 50, 64, 65, 100, 128, 129, 200])
def test_ranks(rank, dtype):
    Case((40, 30, 300), rank, 900, dtype=dtype, weights="uniform").run().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocabulary", [1, 2, 15, 63, 64, 65, 127, 128, 129, 257, 1000, 5003])
def test_extents_of_the_leaf_mode(vocabulary, dtype):
    Case((70, vocabulary), 24, 60, dtype=dtype).run().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nnz,rows", [(1, 1), (1, 500), (2, 500), (64, 64), (200, 129), (3000, 257), (4000, 3001)])
def test_numbers_of_rows(nnz, rows, dtype):
    Case((rows, 401), 40, nnz, dtype=dtype).run().check()


@pytest.mark.parametrize("dims,mode_order", [((50, 300), (1, 0)), ((20, 30, 40), (0, 1, 2)), ((20, 30, 40), (2, 0, 1)), ((20, 30, 40), (1, 2, 0)),
                                             ((9, 14, 11, 150), (0, 1, 2, 3)), ((9, 14, 11, 150), (3, 1, 0, 2)), ((1, 1, 1, 7), (0, 1, 2, 3))])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_orders_and_mode_orders(dims, mode_order, dtype):
    Case(dims, 20, 2000, mode_order=mode_order, dtype=dtype, weights="uniform").run().check()


@pytest.mark.parametrize("weights", ["unit", "uniform", "signed", "zeros", "wide"])
@pytest.mark.parametrize("rank", [12, 150])
def test_weights(weights, rank):
    Case((60, 20, 300), rank, 3000, weights=weights).run().check()


@pytest.mark.parametrize("rank", [12, 150])
@pytest.mark.parametrize("spread", [0.0, 0.01, 30.0, 300.0, 30_000.0])
def test_spread_of_the_scores(spread, rank):
    """All scores equal, and scores so far apart that one coordinate has all the probability."""
    Case((60, 20, 700), rank, 1500, spread=spread).run().check()


@pytest.mark.parametrize("rank", [12, 40, 100])
def test_scores_too_large_to_mean_anything_end(rank):
    """A base that fp32 cannot hold to a whole power of two is raised once a tile at most."""
    for spread in (1e9, 1e20, 1e37):
        c = Case((200, 700), rank, 300, spread=spread)
        c.run()
        c.run(grads=None)
    torch.cuda.synchronize()
    Case((60, 20, 700), rank, 1500).run().check()


@pytest.mark.parametrize("size", [1e-12, 1e-3, 1e4, 1e12])
def test_sizes_of_the_factors(size):
    Case((60, 20, 700), 16, 1500, size=size).run().check()


def test_fibres_with_many_leaves():
    """Fibres whose leaves lie in several runs, next to fibres of one leaf."""
    rng = np.random.default_rng(8)
    c = Case((30, 2000), 24, 10, weights="unit")
    rows = np.concatenate([np.full(1900, 3), np.full(700, 17), np.arange(30)])
    cols = np.concatenate([rng.permutation(2000)[:1900], rng.permutation(2000)[:700], rng.integers(0, 2000, 30)])
    flat = np.unique(rows * 2000 + cols)
    c.coords = [(flat // 2000).astype(np.int32), (flat % 2000).astype(np.int32)]
    c.x = (1 - rng.random(len(flat))).astype(np.float32)
    c.fibres = 30
    c.run().check()


def test_long_vocabulary_few_rows():
    Case((7, 60_001), 32, 9).run().check()
    Case((3, 50_021), 150, 4).run().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rank", [24, 50, 100])
@pytest.mark.parametrize("rows,vocabulary", [(60_001, 333), (390, 40_003)])
def test_many_groups_and_tiles(rows, vocabulary, rank, dtype, path):
    """Several groups of rows a block, groups cut between blocks, a last group with one tile of rows."""
    if path == "by size":
        pytest.skip("the tensor cores' kernels, which are tested by name")
    Case((rows, vocabulary), rank, rows, dtype=dtype).run().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rank", [12, 40, 100])
@pytest.mark.parametrize("falling", [False, True])
def test_scores_that_grow_along_the_leaf_mode(rank, dtype, falling):
    """Every tile of the leaf mode has larger scores than all before it, by more than a share may exceed its base; or smaller ones."""
    c = Case((300, 3001), rank, 400, dtype=dtype)
    ramp = torch.linspace(0.02, 25.0, 3001, device="cuda")
    c.factors[1] = (c.factors[1].float() * (ramp.flip(0) if falling else ramp)[:, None]).to(TYPES[dtype])
    c.run().check()


def test_the_same_call_gives_the_same_losses():
    c = Case((40, 30, 3000), 20, 900)
    h = c.handle()
    first = c.run(handle=h).loss.clone()
    for _ in range(3):
        assert torch.equal(c.run(handle=h).loss, first)


def test_waits_that_give_up(path):
    """The products are withheld: every wait for them runs out, losses and gradients become NaN, and the next call is unharmed."""
    for rank in (12, 40, 100):
        c = Case((200, 300), rank, 150)
        h = c.handle()
        cb.const_debug_set(0, 200)
        cb.const_debug_set(1, 1)
        try:
            for grads in (True, None):
                c.run(grads=grads, handle=h)
                torch.cuda.synchronize()
                if path == "tensor cores":
                    assert all(torch.isnan(t).all() for t in (c.loss, *(c.grads or [])))
        finally:
            cb.const_debug_set(1, 0)
            cb.const_debug_set(0, 0)
        c.run(handle=h).check()


def test_many_rows():
    Case((400, 120, 157), 16, 40_000).run().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("wanted", [(True, False, False), (False, True, False), (False, False, True), (True, True, False), (False, False, False)])
def test_gradients_of_some_modes(wanted, dtype):
    c = Case((40, 30, 300), 20, 900, dtype=dtype).run(grads=wanted).check()
    assert [g is not None for g in c.grads] == list(wanted)


def test_the_loss_alone_is_the_same_loss():
    c = Case((40, 30, 300), 20, 900).run()
    with_gradient = c.loss.clone()
    c.run(grads=None).check()
    (_, bound), _ = c.expected()
    assert np.all(np.abs(c.loss.cpu().numpy() - with_gradient.cpu().numpy()) <= 2 * bound)


def test_rows_without_a_leaf_have_no_gradient():
    c = Case((500, 300), 20, 100).run().check()
    unused = np.setdiff1d(np.arange(500), c.coords[0])
    assert len(unused) > 300 and torch.count_nonzero(c.grads[0][to_dev(unused)]) == 0


def test_values_of_rows_that_no_leaf_reaches_are_not_read():
    """Infinities and NaN in factor rows above the leaves that no fibre has."""
    c = Case((500, 40, 300), 20, 100)
    for m in (0, 1):
        unused = to_dev(np.setdiff1d(np.arange(c.dims[m]), c.coords[m]))
        c.factors[m][unused[::2]] = float("nan")
        c.factors[m][unused[1::2]] = float("inf")
    clean = [torch.nan_to_num(f, 0.0, 0.0, 0.0) for f in c.factors]
    c.run()
    c.factors = clean
    c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rank", [7, 40, 300])
@pytest.mark.parametrize("leaves", [1, 9, 63, 64, 65, 130])
@pytest.mark.parametrize("rows", [1, 60])
def test_the_loss_alone_of_few_leaves(rows, leaves, rank, dtype):
    Case((80, 400), 40, 3000).run(grads=False)                           # what it leaves in the scratch memory must not matter
    c = Case((rows, 333), rank, leaves, dtype=dtype, weights="uniform")
    for _ in range(2):
        c.run(grads=False).check()


def test_a_row_that_is_not_finite_stays_alone():
    c = Case((200, 300), 20, 150).run().check()
    loss, bound = c.loss.clone(), to_dev(c.expected()[0][1])
    bad = int(c.coords[0][0])
    c.factors[0][bad, 3] = float("nan")
    c.run()
    at = int(np.searchsorted(np.unique(c.coords[0]), bad))
    assert torch.isnan(c.loss[at])
    keep = torch.arange(c.fibres, device="cuda") != at
    assert ((c.loss[keep].double() - loss[keep].double()).abs() <= 2 * bound[keep]).all()
    rest = torch.ones(200, dtype=torch.bool, device="cuda")
    rest[bad] = False
    assert torch.isfinite(c.grads[0][rest]).all() and torch.isnan(c.grads[0][bad]).any()


def test_no_fibres():
    for dtype in (torch.float32, torch.bfloat16):
        h = cb.const_csf_build([torch.zeros(0, dtype=torch.int32, device="cuda")] * 2, torch.zeros(0, device="cuda"), (5, 9), (0, 1))
        factors = [torch.randn(5, 7, device="cuda").to(dtype), torch.randn(9, 7, device="cuda").to(dtype)]
        grads = [torch.full_like(f, float("nan")) for f in factors]
        cb.const_softmax_loss(h, factors, torch.empty(0, device="cuda"), grads=grads)
        cb.const_softmax_loss(h, factors, torch.empty(0, device="cuda"))
        for g in grads:
            assert torch.count_nonzero(g) == 0 and not torch.isnan(g).any()


@pytest.mark.parametrize("rank", [10, 140])
def test_against_differences(rank):
    """The gradient along random directions against central differences of the definition's loss, in 64 bits.

    The loss's third derivative along the direction is bounded by about the cube of the scores' change, so a step of 1e-4
    leaves an error of some 1e-8 of the terms; 1e-5 of the sum of the gradient's magnitudes covers that and the kernel's own."""
    c = Case((30, 20, 250), rank, 800, weights="uniform", scale=1.0).run()
    rng = np.random.default_rng(5)
    host = [f.double().cpu().numpy() for f in c.factors]
    for m in range(3):
        d = rng.standard_normal(host[m].shape)
        d /= np.abs(d).max()
        ends = []
        for s in (-1e-4, 1e-4):
            moved = [f + s * d if n == m else f for n, f in enumerate(host)]
            ends.append(loss_and_gradient(c.coords, c.x, moved, c.mode_order, 1.0)[0][0].sum())
        g = c.grads[m].double().cpu().numpy()
        assert abs((g * d).sum() - (ends[1] - ends[0]) / 2e-4) <= 1e-5 * np.abs(g * d).sum() + 1e-6 * np.abs(g).sum()


def test_on_another_stream_and_captured():
    c = Case((40, 30, 300), 20, 900)
    h = c.handle()
    c.run(handle=h).check()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        c.run(handle=h)
    torch.cuda.synchronize()
    c.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        cb.const_softmax_loss(h, c.factors, c.loss, grads=c.grads, scale=c.scale)
    other = torch.cuda.CUDAGraph()                                      # a second graph of the same call: its scratch is its own
    loss, grads = torch.empty_like(c.loss), [torch.empty_like(g) for g in c.grads]
    with torch.cuda.graph(other, stream=stream):
        cb.const_softmax_loss(h, c.factors, loss, grads=grads, scale=c.scale)
    for _ in range(2):
        for t in (c.loss, loss, *c.grads, *grads):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(stream):                                 # beside the first
            other.replay()
        torch.cuda.synchronize()
        c.check()
        c.loss, c.grads, loss, grads = loss, grads, c.loss, c.grads
        c.check()
    c.factors[2].mul_(0.5)                                              # new factors under the same graph
    graph.replay()
    torch.cuda.synchronize()
    other.replay()
    torch.cuda.synchronize()
    c.check()


def test_two_calls_side_by_side():
    """Calls on two streams share nothing."""
    a, b = Case((40, 30, 3000), 20, 900), Case((60, 25, 2000), 33, 1500)
    ha, hb = a.handle(), b.handle()
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(sa):
            a.run(handle=ha)
        with torch.cuda.stream(sb):
            b.run(handle=hb)
    torch.cuda.synchronize()
    a.check()
    b.check()


def test_refusals():
    c = Case((40, 30, 300), 20, 900)
    h = c.handle()
    loss, grads = torch.empty(c.fibres, device="cuda"), [torch.empty_like(f) for f in c.factors]
    with pytest.raises(ValueError):
        cb.const_softmax_loss(h, c.factors[:2], loss)
    with pytest.raises(ValueError):
        cb.const_softmax_loss(h, c.factors, loss, grads=grads[:2])
    with pytest.raises(ValueError):
        cb.const_softmax_loss(h, [f.double() for f in c.factors], loss)
    with pytest.raises(ValueError):
        cb.const_softmax_loss(h, [c.factors[0], c.factors[1], c.factors[2].bfloat16()], loss)
    with pytest.raises(ValueError):
        cb.const_softmax_loss(h, [c.factors[1], c.factors[0], c.factors[2]], loss)
    with pytest.raises(ValueError):
        cb.const_softmax_loss(h, [f.t() for f in c.factors], loss)
    with pytest.raises(ValueError):
        cb.const_softmax_loss(h, c.factors, loss[:-1])
    with pytest.raises(ValueError):
        cb.const_softmax_loss(h, c.factors, loss.double())
    with pytest.raises(ValueError):
        cb.const_softmax_loss(h, [f.cpu() for f in c.factors], loss)
    with pytest.raises(ValueError):
        cb.const_softmax_loss(h, c.factors, loss, grads=[grads[0], grads[1].cpu(), grads[2]])
    for bad in ([c.factors[0], grads[1], grads[2]], [grads[0], grads[1], c.factors[2]]):
        with pytest.raises(cb.ConstError) as e:                         # a gradient in a factor's place
            cb.const_softmax_loss(h, c.factors, loss, grads=bad)
        assert e.value.status == 1
    flat = torch.zeros(12_000, device="cuda")
    for at in (0, 4, 5996):                                             # results that overlap
        with pytest.raises(cb.ConstError) as e:
            cb.const_softmax_loss(h, c.factors, loss, grads=[None, flat[at:at + 600].view(30, 20), flat[:6000].view(300, 20)])
        assert e.value.status == 1
    cb.const_softmax_loss(h, c.factors, flat[6601:6601 + c.fibres], grads=[None, flat[6000:6600].view(30, 20), flat[:6000].view(300, 20)])
    for scale in (float("nan"), float("inf"), 1e60):
        with pytest.raises(cb.ConstError):
            cb.const_softmax_loss(h, c.factors, loss, scale=scale)
    wide = [torch.zeros(d, 1025, device="cuda") for d in c.dims]
    with pytest.raises(cb.ConstError) as e:
        cb.const_softmax_loss(h, wide, loss)
    assert e.value.status == 2
    h64 = cb.const_csf_build([to_dev(x) for x in c.coords], to_dev(c.x.astype(np.float64)), c.dims, c.mode_order)
    with pytest.raises(cb.ConstError) as e:
        cb.const_softmax_loss(h64, c.factors, loss)
    assert e.value.status == 1
    c.run(handle=h).check()


def test_without_scratch():
    c = Case((40, 30, 300), 20, 900)
    h = c.handle()
    loss, grads = torch.full((c.fibres,), 7.0, device="cuda"), [torch.full_like(f, 7.0) for f in c.factors]
    cb.const_debug_set(3, 1)
    try:
        with pytest.raises(cb.ConstError) as e:
            cb.const_softmax_loss(h, c.factors, loss, grads=grads)
        assert e.value.status == 7
    finally:
        cb.const_debug_set(3, 0)
    torch.cuda.synchronize()
    assert all((t == 7.0).all() for t in (loss, *grads))
    c.run(handle=h).check()
