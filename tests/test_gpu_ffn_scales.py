"""Gated blocks: where what a factor is scaled by is nothing, or at the ends of the range.  Against 64 bits, with the tolerances of test_gpu_ffn.

A reduction over rows scales X and dY by the largest value of 32 rows, and one over hidden columns the weights by that of 32 hidden columns.  Where those are all zeros they add
nothing, whatever the other factor is there, and so they may take no bits of it elsewhere: the same tolerances hold."""
import numpy as np
import pytest

from paper_2311_14898_amd import binding as B
from tests.test_gpu_ffn import _inputs, call, check, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.ht_ctx_create(0)
    yield c
    B.ht_ctx_destroy(c)


# (packed; packed with narrow widths on both sides of it; weights that are read once)
ROWS = [(140, 30, 60, 20), (330, 150, 200, 140), (100, 301, 2_405, 300)]


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("tiny", [1e-3, 1e-5, 1e-8])
@pytest.mark.parametrize("n,d,f,e", ROWS)
def test_blocks_of_rows_without_gradients(ctx, n, d, f, e, tiny, keep):
    """dY of 32 and of 64 rows beside each other is zero, as that of rows without a label is."""
    X, Wg, Wu, Wd, dY = _inputs(n, d, f, e)
    dY *= np.float32(tiny * 100)
    for first, last in ((0, 32), (32, 96)):
        masked = dY.copy()
        masked[first:last] = 0.0
        ref, tol = reference(X, Wg, Wu, Wd, "silu", masked)
        check(call(ctx, X, Wg, Wu, Wd, dY=masked, keep=keep), ref, tol)


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("tiny", [1e-3, 1e-5, 1e-8])
@pytest.mark.parametrize("n,d,f,e", ROWS)
def test_blocks_of_rows_of_zeros(ctx, n, d, f, e, tiny, keep):
    """X of such rows is zero, and their gates are open: dB of them is not zero, and adds nothing to dWu."""
    X, Wg, Wu, Wd, dY = _inputs(n, d, f, e)
    X *= np.float32(tiny)
    for first, last in ((0, 32), (32, 96)):
        padded = X.copy()
        padded[first:last] = 0.0
        ref, tol = reference(padded, Wg, Wu, Wd, "sigmoid", dY)
        check(call(ctx, padded, Wg, Wu, Wd, act="sigmoid", dY=dY, keep=keep), ref, tol)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("n,d,f,e", ROWS)
def test_what_is_not_finite_meets_blocks_of_zeros(ctx, n, d, f, e, bad):
    """A zero times what is not finite is NaN, on either side."""
    X, Wg, Wu, Wd, dY = _inputs(n, d, f, e)
    dY[32:64] = 0.0
    Xb = X.copy()
    Xb[40, 3] = bad                          # a row without gradients
    got = call(ctx, Xb, Wg, Wu, Wd, dY=dY)
    assert np.isnan(got["dWd"]).all() and np.isnan(got["dWg"]).all() and np.isnan(got["dWu"]).all()
    db = dY.copy()
    db[50, 7] = bad                          # and one whose block's other gradients are zeros: column 7 of dWd, and all that G reaches
    ref, tol = reference(X, Wg, Wu, Wd, "silu", dY)
    got = call(ctx, X, Wg, Wu, Wd, dY=db)
    assert np.isnan(got["dWd"][:, 7]).all() and np.isnan(got["dWg"]).all() and np.isnan(got["dWu"]).all() and np.isnan(got["dX"][50]).all()
    rest, rows = np.arange(e) != 7, np.arange(n) != 50
    check({"dWd": got["dWd"][:, rest]}, {"dWd": ref["dWd"][:, rest]}, {"dWd": tol["dWd"][:, rest]})
    check({"dX": got["dX"][rows]}, {"dX": ref["dX"][rows]}, {"dX": tol["dX"][rows]})


# (weights are packed from 65 rows on backward, and from 2,049 on forward)
HIDDEN = [(140, 30, 100, 20), (330, 150, 200, 140), (2_100, 40, 97, 24)]


@pytest.mark.parametrize("form", [B.HT_W_IN_OUT, B.HT_W_OUT_IN])
@pytest.mark.parametrize("tiny", [1e-2, 1e-4, 1e-7])
@pytest.mark.parametrize("n,d,f,e", HIDDEN)
def test_blocks_of_hidden_columns_without_weights(ctx, n, d, f, e, tiny, form):
    """32 hidden columns' rows of Wd, or columns of Wg and of Wu, are zeros, as pruned ones are."""
    X, Wg, Wu, Wd, dY = _inputs(n, d, f, e)
    Wz = Wd * np.float32(tiny)
    Wz[32:64] = 0.0
    ref, tol = reference(X, Wg, Wu, Wz, "silu", dY)
    check(call(ctx, X, Wg, Wu, Wz, dY=dY, form=form), ref, tol)
    gates = [w * np.float32(tiny) for w in (Wg, Wu)]
    for which in ((0,), (1,), (0, 1)):
        zeros = [w.copy() for w in gates]
        for k in which:
            zeros[k][:, 64:96] = 0.0
        ref, tol = reference(X, *zeros, Wd, "sigmoid", dY)
        check(call(ctx, X, *zeros, Wd, act="sigmoid", dY=dY, form=form), ref, tol)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("n", [140, 2_100])
def test_what_is_not_finite_meets_hidden_columns_of_zeros(ctx, n, bad):
    X, Wg, Wu, Wd, dY = _inputs(n, 30, 100, 20)
    Wd[32:64] = 0.0
    Wb = Wu.copy()
    Wb[5, 40] = bad                          # hidden column 40 is not finite, its weights behind are zeros: so is Y
    got = call(ctx, X, Wg, Wb, Wd, dY=dY)
    assert np.isnan(got["Y"]).all()
    Wb = Wd.copy()
    Wb[33, 4] = bad                          # column 4 of Y
    ref, tol = reference(X, Wg, Wu, Wd, "silu")
    got = call(ctx, X, Wg, Wu, Wb)
    assert np.isnan(got["Y"][:, 4]).all()
    rest = np.arange(20) != 4
    check({"Y": got["Y"][:, rest]}, {"Y": ref["Y"][:, rest]}, {"Y": tol["Y"][:, rest]})


@pytest.mark.parametrize("form", [B.HT_W_IN_OUT, B.HT_W_OUT_IN])
@pytest.mark.parametrize("small,large", [(-114, 16), (-116, 30), (-118, 100), (-60, 60)])
def test_small_hidden_values_and_large_weights(ctx, small, large, form):
    """Hidden values near the least of all floats, and weights that bring what is made of them back: each power of two may lie outside the range of floats, their products do not.
    (Floats have no finer step than 2^-149: half of it for each rounding on the way to hidden values, times what they meet, is added to what these may be off.)"""
    half = 2.0 ** -150
    n, d, f, e = 2_100, 40, 96, 24
    X, Wg, Wu, Wd, dY = _inputs(n, d, f, e)
    Wu, Wd = Wu * np.float32(2.0 ** small), Wd * np.float32(2.0 ** large)
    ref, tol = reference(X, Wg, Wu, Wd, "silu")
    a = np.abs(X.astype(np.float64) @ Wg)    # (H = v B, |v| <= |a|)
    tol["Y"] = tol["Y"] + 1.01 * half * ((1.0 + a) @ np.abs(Wd).astype(np.float64))
    got = call(ctx, X, Wg, Wu, Wd, form=form)
    check({"Y": got["Y"]}, ref, tol)
    n = 140
    X, Wg, Wu, Wd, dY = _inputs(n, d, f, e)
    back = np.float32(2.0 ** -large)
    X, Wg, Wu, dY = X * back, Wg / back, Wu / back, dY * np.float32(2.0 ** (small + 7))
    ref, tol = reference(X, Wg, Wu, Wd, "silu", dY)
    a, u = (np.abs(X.astype(np.float64) @ w) for w in (Wg, Wu))
    # (dA = G u s, |s| < 1.1, with roundings of G, of G u and of the whole; dB = G v)
    tol["dX"] = tol["dX"] + 1.01 * half * ((2.1 + 1.1 * u) @ np.abs(Wg).T.astype(np.float64) + (1.0 + a) @ np.abs(Wu).T.astype(np.float64))
    for keep in (False, True):
        got = call(ctx, X, Wg, Wu, Wd, dY=dY, form=form, keep=keep, only=("dX",))
        check({"dX": got["dX"]}, ref, tol)
