"""ht_distill_loss of rows whose logits have no largest: -inf throughout is a row without a possible class, NaN stays NaN.  And temperatures at the end of their range."""
import numpy as np
import pytest
import torch

from paper_2311_14898_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.ht_ctx_create(0)
    yield c
    B.ht_ctx_destroy(c)


@pytest.mark.parametrize("n", [4, 70])
@pytest.mark.parametrize("C", [1, 3, 61, 250, 500, 1000, 4096, 5000, 9001, 30_000, 60_000, 70_001])
def test_rows_of_no_numbers(ctx, n, C):
    rng = np.random.default_rng(C)
    X = rng.standard_normal((n, C)).astype(np.float32)
    X[0] = np.nan
    X[1] = -np.inf
    X[1, C // 2] = np.nan                                  # (nothing but -inf beside it)
    X[2] = -np.inf
    ids = rng.integers(0, C, (n, 4)).astype(np.int32)
    top = rng.standard_normal((n, 4)).astype(np.float32)
    u = np.ones(n, np.float32)
    ld = (C + 3) // 4 * 4
    Xd = torch.full((n, ld), float("nan"), device="cuda")
    Xd[:, :C] = torch.from_numpy(X).cuda()
    loss, row_loss, dX = torch.zeros(1, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, ld, device="cuda")
    B.ht_distill_loss(ctx, C, Xd, torch.from_numpy(ids).cuda(), torch.from_numpy(top).cuda(), loss, row_loss=row_loss, dlogits=dX,
                      row_weight=torch.from_numpy(u).cuda(), reduction=B.HT_REDUCE_SUM)
    B.ht_sync(ctx)
    row_loss, dX = row_loss.cpu().numpy(), dX.cpu().numpy()[:, :C]
    assert np.isnan(float(loss)) and np.isnan(row_loss[:2]).all() and np.isnan(dX[:2]).all()
    assert row_loss[2] == np.inf                           # (q > 0 = p)
    q = np.exp(top[2].astype(np.float64) - top[2].max())
    want = np.zeros(C)
    np.add.at(want, ids[2], -q / q.sum())
    assert np.abs(dX[2] - want).max() <= 1e-6
    assert np.isfinite(row_loss[3:]).all() and np.isfinite(dX[3:]).all()


@pytest.mark.parametrize("n,C", [(2, 40), (3, 9001), (70, 300), (70, 70_001)])
def test_the_largest_temperature(ctx, n, C):
    rng = np.random.default_rng(1)
    T, K = 1e37, 200
    ld = (C + 3) // 4 * 4
    X = torch.randn(n, ld, device="cuda")
    ids, top = torch.from_numpy(rng.integers(0, C, (n, K)).astype(np.int32)).cuda(), torch.randn(n, K, device="cuda")
    loss, row_loss, dX = torch.zeros(1, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, ld, device="cuda")
    B.ht_distill_loss(ctx, C, X, ids, top, loss, temperature=T, row_loss=row_loss, dlogits=dX, reduction=B.HT_REDUCE_SUM)
    B.ht_sync(ctx)
    # p = 1 / C, q = 1 / K: T^2 (log C - log K) is beyond fp32, not NaN
    sign = np.sign(C - K)
    assert float(loss) == sign * np.inf and (row_loss.cpu().numpy() == sign * np.inf).all()
    want = np.full((n, C), 1.0 / C)
    np.add.at(want, (np.arange(n)[:, None], ids.cpu().numpy()), -1.0 / K)
    assert np.abs(dX.cpu().numpy()[:, :C].astype(np.float64) / T - want).max() <= 1e-6
    for t in (1.01e37, 3e38):
        with pytest.raises(B.HongtuError) as err:
            B.ht_distill_loss(ctx, C, X, ids, top, loss, temperature=t)
        assert err.value.code == B.HT_EINVAL
