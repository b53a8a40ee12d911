"""The contraction, the loss with its gradient and the clipping together, as a program uses them that trains a CP model of a CSF tensor."""
import numpy as np
import pytest
import torch

import paper_2401_04836_b200 as cb
from tests.gpu_util import to_dev
from tests.loss_reference import loss_and_gradient

pytestmark = pytest.mark.gpu


def problem(dims, rank, nnz, seed=0):
    rng = np.random.default_rng(seed)
    flat = np.unique(rng.integers(0, np.prod(dims, dtype=np.int64), nnz))
    coords = [c.astype(np.int32) for c in np.unravel_index(flat, dims)]
    x = (1 - rng.random(len(flat))).astype(np.float32)
    factors = [rng.standard_normal((d, rank)).astype(np.float32) * np.float32(0.5) for d in dims]
    return coords, x, factors


def test_the_data_term_is_mttkrp():
    """The gradient of the slices' factor is scale * (expected - stored): its second term is the MTTKRP of the same handle and factors.

    Added to the gradient, MTTKRP leaves the expectation alone, which the 64-bit definition gives without the targets: the bound is the
    gradient's own and the contraction's 1e-5 of its terms."""
    dims, rank, scale = (60, 50, 300), 16, 0.25
    coords, x, factors = problem(dims, rank, 4000)
    h = cb.const_csf_build([to_dev(c) for c in coords], to_dev(x), dims, (0, 1, 2))
    dev = [to_dev(f) for f in factors]
    plan = cb.const_plan_create("A[i,r] = X[i,j,k] * B[j,r] * C[k,r]", ["T[i,j,r] = X[i,j,k] * C[k,r]", "A[i,r] = T[i,j,r] * B[j,r]"],
                                {"X": (0, 1, 2)}, ["ijkr", "ijr"], {"i": dims[0], "j": dims[1], "k": dims[2], "r": rank}, cb.F32)
    stored = torch.empty(dims[0], rank, device="cuda")
    cb.const_execute(plan, {"X": h, "B": dev[1], "C": dev[2]}, stored)
    fibres = len(np.unique(coords[0].astype(np.int64) * dims[1] + coords[1]))
    loss, grad = torch.empty(fibres, device="cuda"), torch.empty_like(dev[0])
    cb.const_softmax_loss(h, dev, loss, grads=[grad, None, None], scale=scale)
    expected = (grad.double() + scale * stored.double()).cpu().numpy()
    _, grads = loss_and_gradient(coords, x, factors, (0, 1, 2), scale)
    exact, terms = np.zeros((dims[0], rank)), np.zeros((dims[0], rank))
    np.add.at(exact, coords[0], x[:, None].astype(np.float64) * factors[1][coords[1]] * factors[2][coords[2]])
    np.add.at(terms, coords[0], np.abs(x[:, None].astype(np.float64) * factors[1][coords[1]] * factors[2][coords[2]]))
    assert (np.abs(expected - (grads[0][0] + scale * exact)) <= grads[0][1] + 1e-5 * scale * terms).all()


def steps(h, factors, fibres, n, rate, max_norm, captured):
    """n steps of clipped gradient descent; returns the losses and norms of every step."""
    factors = [f.clone() for f in factors]
    loss, norm = torch.empty(fibres, device="cuda"), torch.empty(1, device="cuda")
    grads = [torch.empty_like(f) for f in factors]

    def step():
        cb.const_softmax_loss(h, factors, loss, grads=grads, scale=1.0 / fibres)
        cb.const_clip_gradients(grads, max_norm, norm)
        for f, g in zip(factors, grads):
            f.sub_(g, alpha=rate)

    graph, seen = None, []
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    for _ in range(n):
        graph.replay() if captured else step()
        seen.append((loss.clone(), norm.clone()))
    torch.cuda.synchronize()
    return seen, factors


@pytest.mark.parametrize("captured", [False, True])
def test_steps_of_training(captured):
    """Each step against the definition at the same factors: losses, the norm of the gradient, and the clipped update."""
    dims, rank, rate, max_norm = (60, 50, 700), 20, 0.5, 0.02
    coords, x, factors = problem(dims, rank, 3000, seed=3)
    h = cb.const_csf_build([to_dev(c) for c in coords], to_dev(x), dims, (0, 1, 2))
    fibres = len(np.unique(coords[0].astype(np.int64) * dims[1] + coords[1]))
    dev = [to_dev(f) for f in factors]
    for n in range(1, 4):
        seen, after = steps(h, dev, fibres, n, rate, max_norm, captured)
        _, before = steps(h, dev, fibres, n - 1, rate, max_norm, captured) if n > 1 else (None, dev)
        host = [f.double().cpu().numpy() for f in before]
        (loss, bound), grads = loss_and_gradient(coords, x, host, (0, 1, 2), 1.0 / fibres)
        # two runs of the same steps differ in the last bits of the factors: 2^-20 of a score's terms is allowed for that
        assert (np.abs(seen[-1][0].double().cpu().numpy() - loss) <= 4 * bound).all()
        norm = np.sqrt(sum((g ** 2).sum() for g, _ in grads))
        off = np.sqrt(sum((b ** 2).sum() for _, b in grads))
        assert norm > max_norm                                           # the clipping is at work
        assert abs(float(seen[-1][1]) - norm) <= 4 * off + 1e-6 * norm
        for f, b, (g, e) in zip(after, host, grads):
            want = b - rate * g * (max_norm / norm)
            assert (np.abs(f.double().cpu().numpy() - want) <= rate * (4 * e + np.abs(g) * (4 * off / norm + 2e-6)) + 2.0 ** -20 * np.abs(b) + 1e-7).all()
