"""ht_head_loss of very small and very large values: gradients keep their bits, and where products of H and W are far below the smallest float logits are 0, not NaN.
Tolerances as in test_gpu_head."""
import numpy as np
import pytest

from paper_2311_14898_amd import binding as B
from tests.test_gpu_head import _inputs, call, check, ctx, reference  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("h", [1e-28, 1e-30, 1e-33])
@pytest.mark.parametrize("n,C", [(20, 64), (150, 64), (3000, 172), (150, 1001)])
def test_small_features(ctx, n, C, h):  # noqa: F811
    """Gradients of W stay above the smallest normal float (tolerances are relative): 1e-33 / 3,000 rows x 172 classes, added up, is 1e-36."""
    rng = np.random.default_rng(n + C + 1)
    H, W, y = _inputs(n, 96, C, rng, unlabelled=0.1)
    H = (H * np.float32(h)).astype(np.float32)
    ref, tol = reference(H, W, y, None, False)
    for form in (B.HT_W_IN_OUT, B.HT_W_OUT_IN):
        check(call(ctx, H, W, y, form, mean=False), ref, tol)
    if h >= 1e-30:
        ref, tol = reference(H, W, y, None, True)
        check(call(ctx, H, W, y, B.HT_W_OUT_IN), ref, tol)


@pytest.mark.parametrize("h,w", [(1e-20, 1e-18), (1e-26, 1e-12), (1e-30, 1e-9), (1e-10, 1e-25)])
@pytest.mark.parametrize("n,C", [(20, 130), (150, 64), (150, 70), (150, 200), (90, 256), (150, 400), (150, 1001)])
def test_products_below_the_smallest_float(ctx, n, C, h, w):  # noqa: F811
    rng = np.random.default_rng(n + C)
    H, W, y = _inputs(n, 96, C, rng, unlabelled=0.1)
    H, W = (H * np.float32(h)).astype(np.float32), (W * np.float32(w)).astype(np.float32)
    ref, tol = reference(H, W, y, None, True)
    for form in (B.HT_W_IN_OUT, B.HT_W_OUT_IN):
        out = call(ctx, H, W, y, form)
        check(out, ref, tol)
        assert np.abs(out["row_lse"][y >= 0] - np.log(C)).max() <= 1e-5


def test_one_small_row_among_others(ctx):  # noqa: F811
    rng = np.random.default_rng(4)
    H, W, y = _inputs(100, 40, 333, rng)
    H[17] *= np.float32(1e-30)
    W *= np.float32(1e-10)
    H[:17] *= np.float32(1e10)
    H[18:] *= np.float32(1e10)
    ref, tol = reference(H, W, y, None, True)
    check(call(ctx, H, W, y, B.HT_W_OUT_IN), ref, tol)


@pytest.mark.parametrize("n", [1, 40, 64, 65, 200])
def test_losses_are_weighted_and_added_up_in_64_bits(ctx, n):  # noqa: F811
    """u l is beyond fp32 for a row, the mean is not; and weights of both signs whose sum is small."""
    rng = np.random.default_rng(n)
    H, W, y = _inputs(n, 8, 30, rng, spread=40.0)
    u = np.zeros(n, np.float32)
    u[0], y[0] = 3e38, int((H[0].astype(np.float64) @ W).argmin())
    out = call(ctx, H, W, y, B.HT_W_IN_OUT, u=u, grad=False)
    l = float(out["row_loss"][0])
    assert l > 5
    want = float(u[0]) * l / n
    assert (abs(out["loss"] - want) <= 2.0 ** -22 * want) if want < 3.4e38 else out["loss"] == np.inf
    u = np.where(np.arange(n) % 2, -1.0, 1.0).astype(np.float32) * np.float32(1.1)
    out = call(ctx, H, W, y, B.HT_W_IN_OUT, u=u, mean=False, grad=False)
    want = (u.astype(np.float64) * out["row_loss"].astype(np.float64)).sum()
    assert abs(out["loss"] - want) <= 2.0 ** -24 * abs(want) + 1e-12 * np.abs(out["row_loss"]).sum()
