"""Gradients of ht_head_loss for classes that no row is likely to have: probabilities down to 2^-48, in rows of dW of their own.

A gradient of a logit is the sum of two fp16 numbers, p 2^15 rounded and what that leaves times 2^12: off by 2^-22 of itself and 2^-52 at most; a product of what is
left with what H or W leave is left out, 2^-11 of 2^-40 where the first number has few bits.  Tolerances are those of test_gpu_head with 2^-50 for its 2^-39."""
import numpy as np
import pytest
import torch

from paper_2311_14898_amd import binding as B
from tests.test_gpu_head import STEP, call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.ht_ctx_create(0)
    yield c
    B.ht_ctx_destroy(c)


# (n, d, C): few rows; all classes in one tile; sums kept, for dW that is and is not split; sums made again
@pytest.mark.parametrize("n,d,C", [(40, 32, 300), (70, 32, 90), (300, 20, 200), (2000, 64, 256), (100, 200, 1000), (300, 32, 1500), (700, 256, 9000), (2000, 64, 9000)])
@pytest.mark.parametrize("form", [B.HT_W_IN_OUT, B.HT_W_OUT_IN])
def test_classes_without_a_label(ctx, n, d, C, form):
    rng = np.random.default_rng(n + C)
    likely = C // 4
    t = np.concatenate([np.zeros(likely), np.linspace(8.0, 28.0, C - likely)])       # nats below the likely ones
    H = rng.standard_normal((n, d)).astype(np.float32)
    H[:, 0] = 1.0
    W = (rng.standard_normal((d, C)) / np.sqrt(d)).astype(np.float32)
    W[0] = -t
    y = rng.integers(0, likely, n)
    h, w = H.astype(np.float64), W.astype(np.float64)
    x = h @ w
    e = (3 * 2.0 ** -22 + (3 * np.ceil(d / 16) + 4) * STEP) * (np.abs(h) @ np.abs(w))
    lse = np.log(np.exp(x).sum(axis=1))
    b = (e * np.exp(x - lse[:, None])).sum(axis=1) + 4 * STEP * (np.abs(x).max(axis=1) + np.abs(lse) + 1) + 2.0 ** -20       # (of log sum exp: each class's by its share)
    p = np.exp(x - lse[:, None])
    assert p[:, likely:].max() < 2.0 ** -8 and 2.0 ** -60 < p.min() < 2.0 ** -40
    pe = p * (e + b[:, None] + 2.0 ** -20) + 2.0 ** -50
    pe[np.arange(n), y] += 2 * STEP
    g = p.copy()
    g[np.arange(n), y] -= 1.0
    terms = 3 * 2.0 ** -22 + (3 * max(n, C) / 16 + 64) * STEP
    out = call(ctx, H, W, y, form, mean=False)
    err, room = np.abs(out["dW"] - h.T @ g), np.abs(h).T @ pe + terms * (np.abs(h).T @ np.abs(g))
    worst = (err / (np.abs(h).T @ np.abs(g))).max(axis=0)
    assert (err <= room).all(), [(int(c), float(p[:, c].max()), float(worst[c])) for c in np.flatnonzero((err > room).any(axis=0))[:5]]
    assert (np.abs(out["dH"] - g @ w.T) <= pe @ np.abs(w).T + terms * (np.abs(g) @ np.abs(w).T)).all()
    # classes of 2^-35 to 2^-30, all of whose bits the first number had lost: to 1e-4 of their columns' sizes
    some = (p.max(axis=0) < 2.0 ** -30) & (p.max(axis=0) > 2.0 ** -35)
    assert some.sum() > 3 and worst[some].max() <= 1e-4 + e[:, some].max()
