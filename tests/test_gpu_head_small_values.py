"""ht_head_loss of very small values: gradients keep their bits.
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
