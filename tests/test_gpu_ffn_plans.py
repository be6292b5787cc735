"""Gated blocks by the plans of large calls, against 64 bits with the tolerances of test_gpu_ffn: reductions of several stages that end inside one, every gate, and products behind
the hidden tensors that have a launch each; pieces of rows where memory is scarce."""
import pytest
import torch

from paper_2311_14898_amd import binding as B
from tests.test_gpu_ffn import ACTS, _inputs, call, check, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.ht_ctx_create(0)
    yield c
    B.ht_ctx_destroy(c)


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("n,d,f,e", [(2_100, 301, 700, 172), (4_200, 301, 1_100, 99)])
def test_forward_of_many_rows(ctx, n, d, f, e, act):
    """Packed weights by half tiles (102 whole ones) and by whole ones (297); 301 features are five pairs of stages, the last of 45."""
    X, Wg, Wu, Wd, _ = _inputs(n, d, f, e, gate=3.0)
    ref, tol = reference(X, Wg, Wu, Wd, act)
    check(call(ctx, X, Wg, Wu, Wd, act=act), ref, tol)
    check(call(ctx, X, Wg, Wu, Wd, act=act, form=B.HT_W_OUT_IN, keep=True, add=True), ref, tol, add=True)


# (relu's slope has a border, which products that differ in their last bits may lie on either side of)
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("act", [a for a in ACTS if a != "relu"])
def test_backward_of_many_rows(ctx, act, keep):
    n, d, f, e = 2_100, 301, 700, 172
    X, Wg, Wu, Wd, dY = _inputs(n, d, f, e, gate=3.0)
    ref, tol = reference(X, Wg, Wu, Wd, act, dY)
    check(call(ctx, X, Wg, Wu, Wd, act=act, dY=dY, keep=keep, fwd=keep), ref, tol)


@pytest.mark.parametrize("n,d,f,e,form", [(270, 100, 17_005, 300, B.HT_W_OUT_IN), (270, 300, 17_005, 90, B.HT_W_IN_OUT)])
def test_last_products_by_themselves(ctx, n, d, f, e, form):
    """More than 512 tiles of dX, dWg with dWu, and dWd together: a launch each, of whole and of narrow tiles."""
    X, Wg, Wu, Wd, dY = _inputs(n, d, f, e)
    ref, tol = reference(X, Wg, Wu, Wd, "silu", dY)
    check(call(ctx, X, Wg, Wu, Wd, dY=dY, form=form, fwd=False), ref, tol)
    check(call(ctx, X, Wg, Wu, Wd, dY=dY, form=form, keep=True, add=True), ref, tol, add=True)


def test_pieces_follow_the_memory_there_is():
    """28 KB of scratch memory a row: where all rows do not fit, half of the most that a piece may take, or half of that, and so on.  Here 128 MiB of 205, in two pieces."""
    n, d, f, e = 7_500, 60, 2_020, 36
    X, Wg, Wu, Wd, dY = _inputs(n, d, f, e)
    ref, tol = reference(X, Wg, Wu, Wd, "silu", dY)
    ctx = B.ht_ctx_create(0)
    try:
        B.ht_ctx_set_hbm_budget(ctx, 200 << 20)
        check(call(ctx, X, Wg, Wu, Wd, dY=dY, fwd=False), ref, tol)      # (torch keeps what it has allocated)
        torch.cuda.synchronize()
        there = torch.cuda.mem_get_info()[0]
        B.ht_ctx_destroy(ctx)
        ctx = None
        used = torch.cuda.mem_get_info()[0] - there
        assert 128 << 20 <= used <= 200 << 20, used >> 20
    finally:
        if ctx is not None:
            B.ht_ctx_destroy(ctx)
