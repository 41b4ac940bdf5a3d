"""Attention of new tokens against 64 bits, with bounds of what a row's own probabilities lose to roundings: they do not grow with the context."""
import math

import torch


def row(batch, i, h, sink=None, window=None, parts=1, faint=0.0, off_reference=0.0, scale=128.0 ** -0.5):
    """(out [128], lse, bound of |out - it|, bound of |lse - it|) of packed row i, head h; window None: every earlier token.

    Counted, eta being half a step of the type: the output's rounding, eta.  Probabilities as one rounding (parts = 1): eta of each, and the quotient divides by
    the sum of them as rounded, so that an error of a probability moves it by that times the value's distance from the output.  In two
    parts (the rounding, and the rounding of the rest): eta^2 of each, but divided by the unrounded sum.  A probability that is no more than `faint` of the
    row's largest may be lost altogether, and a larger one be off by as much.  off_reference: the same relative to the sum, of all keys together.
    A logit's 128 products, summed in 32 bits, move a probability by twice their relative size; sums of n terms."""
    eta, b = torch.finfo(batch.dtype).eps / 2, next(b for b in range(len(batch.new)) if batch.off[b] <= i < batch.off[b + 1])
    m = batch.ctx[b] - batch.new[b] + i - batch.off[b]
    pos = torch.arange(min(m + 1, batch.table.shape[1] * batch.page))
    if window is not None:
        pos = pos[(pos < sink) | (pos > m - window)]
    page = batch.table[b].long()[pos // batch.page]
    there = (page >= 0) & (page < batch.n_pages)
    at = page[there] * batch.page + pos[there] % batch.page
    if at.numel() == 0:
        return torch.zeros(128, dtype=torch.float64), -math.inf, torch.zeros(128, dtype=torch.float64), 0.0
    k, v = (x.reshape(-1, 128)[at].double() for x in batch.rows[:, h // (batch.hq // batch.hkv)])
    q = batch.q[i, h].double()
    x = (k @ q) * scale
    lse = torch.logsumexp(x, 0)
    p = torch.exp(x - lse)[:, None]
    o = (p * v).sum(0)
    e_x = 128 * 2.0 ** -24 * float((k.abs() @ q.abs()).max() * scale) + 2.0 ** -21
    e_sum, off = (at.numel() + 64) * 2.0 ** -24, (v - o).abs()
    lost = torch.minimum(p, faint * p.max())
    tol = eta * o.abs() + 2 * e_x * (p * off).sum(0) + 2 * e_sum * (p * v.abs()).sum(0) + off_reference * off.amax(0) + 1e-30
    tol = tol + (1.02 * ((eta * p + lost) * off).sum(0) if parts == 1 else ((eta * eta * p + lost) * v.abs()).sum(0))
    if batch.dtype == torch.float16:
        tol = tol + 2.0 ** -25                                    # (an output below 2^-14)
    return o, float(lse), tol, e_x + e_sum + abs(float(lse)) * 2.0 ** -23 + 2.0 ** -22


def check_rows(batch, out, lse, which, **how):
    """Rows and heads [(i, h)]; the largest error in units of its bound."""
    out, worst = out.double().cpu(), 0.0
    for i, h in which:
        o, z, tol, tol_z = row(batch, i, h, **how)
        d = (out[i, h] - o).abs()
        assert (d <= tol).all(), f"row {i} head {h}: off by {float(d.max()):.3g}, {float((d / tol).max()):.3g} times its bound"
        worst = max(worst, float((d / tol).max())) if z > -math.inf else worst
        if lse is not None:
            got = float(lse[i, h])
            assert got == z if z == -math.inf else abs(got - z) <= tol_z, f"row {i} head {h}: lse {got}, {z}"
    return worst
