"""The softmax loss over a CSF tensor's leaf mode and its gradient from the definition, in 64 bits on the CPU, with bounds.

The bounds count the roundings of an fp32 computation whose operands carry 22 bits (two 11-bit terms): with
A_f = max_k sum_r |h_fr c_kr|,
  a score          A_f (2^-21 for the operands + (rank + 8) 2^-23 for the additions, which may cut instead of round)
  lse              a score's error + 2^-20 (exponentials, logarithm) + |lse| 2^-22
  a share p_fk     relative, the errors of its score and of lse + 2^-20
  a sum of terms   2^-20 of the sum of their magnitudes, and a share below the smallest 11-bit number: 2^-30 of the row's largest
Factors in bf16: shares (and the rows of a product of several factors) may carry 11 bits in the gradient's sums, 2^-10 of every
term's magnitude, and a result is off by half a step, 2^-8 of its value.
"""
import numpy as np

TINY = 1e-30


def fibres_of(coords, mode_order):
    """(fibres [F, order - 1] in CSF order, row of every leaf, leaf coordinate)."""
    upper = np.stack([coords[m] for m in mode_order[:-1]], axis=1).astype(np.int64)
    fibres, row = np.unique(upper, axis=0, return_inverse=True)
    return fibres, row.reshape(-1), coords[mode_order[-1]].astype(np.int64)


def loss_and_gradient(coords, x, factors, mode_order, scale, bf16=False):
    """factors by mode, float64 arrays holding the values the kernel reads.  Returns ((loss, bound), [(grad, bound) per mode])."""
    fibres, row, col = fibres_of(coords, mode_order)
    x = x.astype(np.float64)
    by_level = [factors[m].astype(np.float64) for m in mode_order]
    upper, table = by_level[:-1], by_level[-1]
    F, (V, R) = len(fibres), table.shape
    rows = [f[fibres[:, l]] for l, f in enumerate(upper)]
    h = np.prod(rows, axis=0)
    s = h @ table.T
    top = s.max(axis=1, keepdims=True)
    lse = (top + np.log(np.exp(s - top).sum(axis=1, keepdims=True)))[:, 0]
    p = np.exp(s - lse[:, None])
    target = np.zeros((F, V))
    target[row, col] = x
    w, w_abs = target.sum(axis=1), np.abs(target).sum(axis=1)
    loss = w * lse - (target * s).sum(axis=1)
    largest = (np.abs(h) @ np.abs(table).T).max(axis=1)
    e_score = largest * (2.0 ** -21 + (R + 8) * 2.0 ** -23)
    e_lse = e_score + 2.0 ** -20 + np.abs(lse) * 2.0 ** -22
    loss_bound = w_abs * (e_lse + e_score + 2.0 ** -22 * (np.abs(lse) + largest)) + TINY
    g = scale * (w[:, None] * p - target)
    e_share = e_score + e_lse + 2.0 ** -20 + (2.0 ** -10 if bf16 else 0.0)
    share = np.abs(scale) * np.abs(w)[:, None] * p
    e_g = share * e_share[:, None] + 2.0 ** -20 * (share + np.abs(scale) * np.abs(target)) + 2.0 ** -30 * share.max(axis=1, keepdims=True)
    e_g = e_g + 2.0 ** -36 * share.max() + (2.0 ** -10 * share if bf16 else 0.0)

    def rounded(value, bound):
        return value, (bound + (2.0 ** -8 * (np.abs(value) + bound) if bf16 else 0.0)) + TINY

    grads = [None] * len(mode_order)
    grads[mode_order[-1]] = rounded(g.T @ h, e_g.T @ np.abs(h))
    dh, e_dh = g @ table, e_g @ np.abs(table)
    e_dh = e_dh + 2.0 ** -22 * np.abs(dh)
    for l in range(len(upper)):
        others = [r for m, r in enumerate(rows) if m != l]
        term, e_term = np.prod([dh] + others, axis=0), np.prod([e_dh] + [np.abs(r) for r in others], axis=0)
        value, bound = np.zeros_like(upper[l]), np.zeros_like(upper[l])
        np.add.at(value, fibres[:, l], term)
        np.add.at(bound, fibres[:, l], e_term + 2.0 ** -20 * np.abs(term))
        grads[mode_order[l]] = rounded(value, bound)
    return (loss, loss_bound), grads
