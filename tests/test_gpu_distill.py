"""ht_distill_loss against the same formulas in 64 bits.

Tolerances: with z = x / T, an exponential's argument is off by a few half steps of |z| and of log sum exp, its value by as much and
two steps of its own; a row's sum by a step per 64 terms and joining; so p and q are off by r = 2^-24 (8 S + 40 + C / 64) of themselves, S the
largest |z| among the finite ones (of student and teacher, log sum exp's within it but for log C).  A loss adds r (1 + ...) of its terms."""
import numpy as np
import pytest
import torch

from paper_2311_14898_amd import binding as B

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    c = B.ht_ctx_create(0)
    yield c
    B.ht_ctx_destroy(c)


def reference(X, ids, top, T, u, mean):
    X, top = X.astype(np.float64), top.astype(np.float64)
    n, C = X.shape
    T = np.float64(np.float32(T))
    there = (ids >= 0) & (top != -np.inf)
    has = there.any(axis=1)
    N = max(1, has.sum()) if mean else 1
    u = np.ones(n) if u is None else u.astype(np.float64)
    with np.errstate(all="ignore"):
        t = np.where(there, top / T, -np.inf)
        t = t - np.where(has, t.max(axis=1), 0.0)[:, None]
        lq = t - np.log(np.where(has, np.exp(t).sum(axis=1), 1.0))[:, None]
        q = np.exp(lq)
        z = X / T
        m = z.max(axis=1)
        some = m != -np.inf
        m = np.where(some, m, 0.0)
        lse = np.where(some, np.log(np.exp(z - m[:, None]).sum(axis=1)), 0.0) + m
        lp = z - lse[:, None]
        p = np.where(some[:, None], np.exp(lp), 0.0)
        at = np.where(there, ids, 0)
        lpk = np.take_along_axis(lp, at, axis=1)
        l = np.where(q > 0, q * (lq - lpk), 0.0).sum(axis=1) * T * T
        S = np.maximum(np.where(np.isfinite(z), np.abs(z), 0.0).max(axis=1), np.where(there & np.isfinite(top), np.abs(top / T), 0.0).max(axis=1)) + np.log(C)
        r = HALF * (8 * S + 40 + C / 64)
        le = (np.where(q > 0, q * (np.abs(lq) + np.abs(lpk) + 4), 0.0).sum(axis=1) * r[:] + r) * T * T
        take = np.zeros_like(X)
        np.add.at(take, (np.repeat(np.arange(n), ids.shape[1]), at.ravel()), np.where(there, q, 0.0).ravel())
    f = np.where(has, u * T / N, 0.0)[:, None]
    out = dict(loss=(np.where(has, u * l, 0.0)).sum() / N, row_loss=np.where(has, l, 0.0), dX=(p - take) * f)
    tol = dict(loss=(np.where(has, np.abs(u) * le, 0.0)).sum() / N + 2 * HALF * np.abs(out["loss"]), row_loss=np.where(has, le, 0.0),
               dX=((p + take) * (r[:, None] + ids.shape[1] * HALF) + 2.0 ** -120) * np.abs(f))
    return out, tol


def call(ctx, X, ids, top, T, u=None, mean=True, grad=True, ld=None, inplace=False):
    n, C = X.shape
    Xd = torch.full((n + 1, ld or (C + 3) // 4 * 4), float("nan"), device="cuda")
    Xd[:n, :C] = torch.from_numpy(X).cuda()
    loss, row_loss = torch.full((1,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    dX = Xd if inplace else torch.full_like(Xd, 7.0) if grad else None
    B.ht_distill_loss(ctx, C, Xd[:n], torch.from_numpy(ids.astype(np.int32)).cuda(), torch.from_numpy(top).cuda(), loss, temperature=T,
                      row_weight=None if u is None else torch.from_numpy(u).cuda(), row_loss=row_loss, dlogits=dX[:n] if grad else None,
                      reduction=B.HT_REDUCE_MEAN if mean else B.HT_REDUCE_SUM)
    B.ht_sync(ctx)
    out = dict(loss=float(loss), row_loss=row_loss.cpu().numpy())
    if grad:
        out["dX"] = dX[:n, :C].cpu().numpy()
        assert inplace or (dX[n] == 7.0).all()
    return out


def check(out, ref, tol):
    for k in out:
        got, want = np.asarray(out[k], dtype=np.float64), np.asarray(ref[k])
        with np.errstate(over="ignore"):                   # (T^2 q 1.7e38 of the rows of lowest values can be beyond fp32's last number)
            want = np.where(np.abs(want) > np.finfo(np.float32).max, want.astype(np.float32), want)
        same = (got == want) | (np.isnan(got) & np.isnan(want))
        with np.errstate(invalid="ignore"):
            err = np.where(same, 0.0, np.abs(got - want))
        assert (err <= np.where(same, 1.0, tol[k])).all(), (k, float(np.nanmax(err)), float(np.nanmax(np.abs(want))))


def _inputs(n, C, K, rng, missing=0.1):
    X = (rng.standard_normal((n, C)) * 2).astype(np.float32)
    ids = np.stack([rng.permutation(C)[:K] if C < 5000 else rng.choice(C, K, replace=False) for _ in range(n)])
    top = (np.take_along_axis(X, ids, axis=1) + rng.standard_normal((n, K))).astype(np.float32)
    lot = rng.random(n)
    ids[lot < missing] = -1
    ids[(lot >= missing) & (lot < 3 * missing), (K + 1) // 2:] = -1
    return X, ids, top


SIZES = [(1, 1, 1), (1, 131_072, 32), (2, 5, 5), (3, 4097, 64), (5, 47, 8), (9, 300, 256), (100, 172, 8), (130, 1027, 33), (4, 20_001, 100), (17, 2048, 3),
         (6, 2049, 1), (2, 33_000, 17), (3, 70_001, 256), (2001, 41, 4), (257, 8192, 10)]


@pytest.mark.parametrize("T", [1.0, 4.0])
@pytest.mark.parametrize("n,C,K", SIZES)
def test_sizes(ctx, n, C, K, T):
    rng = np.random.default_rng(n + C + K)
    X, ids, top = _inputs(n, C, K, rng, missing=0.1 if n > 4 else 0.0)
    ref, tol = reference(X, ids, top, T, None, True)
    a = call(ctx, X, ids, top, T)
    check(a, ref, tol)
    check(call(ctx, X, ids, top, T, grad=False), ref, tol)
    b = call(ctx, X, ids, top, T, inplace=True, ld=(C + 3) // 4 * 4 + 8)
    assert all(np.array_equal(a[k], b[k]) for k in a)
    u = (rng.standard_normal(n) * 2).astype(np.float32)
    ref, tol = reference(X, ids, top, T, u, False)
    check(call(ctx, X, ids, top, T, u=u, mean=False), ref, tol)


@pytest.mark.parametrize("C", [50, 3001, 40_000])
def test_masked_and_repeated_entries(ctx, C):
    rng = np.random.default_rng(C)
    n, K = 12, 12
    X, ids, top = _inputs(n, C, K, rng, missing=0.0)
    low = np.finfo(np.float32).min
    X[0, :] = -np.inf                                      # no class is possible
    X[1, 1:] = -np.inf                                     # one is, and not the teacher's
    ids[1] = rng.integers(1, C, K)
    X[2, ::2] = low                                        # masked by the type's lowest value
    X[3] = low
    ids[4] = -1                                            # no teacher
    top[5] = -np.inf                                       # a teacher that says nothing
    top[6, 1:] = -np.inf                                   # one entry
    ids[7] = ids[7, 0]                                     # the same id in all entries
    ids[8, 3] = ids[8, 9]
    top[9, 2:] = low
    X[10, ids[10, 0]] = -np.inf                            # p = 0 where q > 0
    ref, tol = reference(X, ids, top, 2.0, None, True)
    assert np.isinf(ref["row_loss"][[0, 1, 10]]).all() and np.isinf(ref["loss"])
    for inplace in (False, True):
        check(call(ctx, X, ids, top, 2.0, inplace=inplace), ref, tol)


@pytest.mark.parametrize("C", [60, 9000])
def test_ids_beyond_the_classes_and_nan(ctx, C):
    rng = np.random.default_rng(C)
    X, ids, top = _inputs(8, C, 6, rng, missing=0.0)
    good = call(ctx, X, ids, top, 1.0)
    rest = np.arange(8) != 3
    for what in ("id", "logit", "teacher"):
        Y, i, t = X.copy(), ids.copy(), top.copy()
        if what == "id":
            i[3, 2] = C
        elif what == "logit":
            Y[3, 7] = np.nan
        else:
            t[3, 1] = np.nan
        out = call(ctx, Y, i, t, 1.0)
        assert np.isnan(out["loss"]) and np.isnan(out["row_loss"][3])
        assert (out["row_loss"][rest] == good["row_loss"][rest]).all() and (out["dX"][rest] == good["dX"][rest]).all()


def test_nothing_at_all(ctx):
    X = np.ones((3, 10), np.float32)
    out = call(ctx, X, np.full((3, 2), -1), np.zeros((3, 2), np.float32), 1.0)
    assert out["loss"] == 0 and (out["dX"] == 0).all() and (out["row_loss"] == 0).all()
    out = call(ctx, np.ones((0, 10), np.float32), np.zeros((0, 2)), np.zeros((0, 2), np.float32), 1.0)
    assert out["loss"] == 0


def test_differences(ctx):
    rng = np.random.default_rng(4)
    X, ids, top = _inputs(5, 30, 4, rng, missing=0.0)
    g = call(ctx, X, ids, top, 2.0)["dX"]
    for v, c in ((0, 0), (2, ids[2, 1]), (4, 29)):
        up, down = X.astype(np.float64).copy(), X.astype(np.float64).copy()
        up[v, c] += 1e-4
        down[v, c] -= 1e-4
        d = reference(up, ids, top, 2.0, None, True)[0]["loss"] - reference(down, ids, top, 2.0, None, True)[0]["loss"]
        assert abs(d / 2e-4 - g[v, c]) <= 1e-6             # 1e-9 by the third derivative, the rest is the gradient's own


def test_refusals(ctx):
    X, ids, top, loss = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda"), torch.zeros(1, device="cuda")

    def refused(code, C=8, X=X, ids=ids, top=top, **kw):
        with pytest.raises(B.HongtuError) as err:
            B.ht_distill_loss(ctx, C, X, ids, top, loss, **kw)
        assert err.value.code == code, err.value

    refused(B.HT_ESHAPE, C=0)
    refused(B.HT_ESHAPE, C=9)
    for T in (0.0, -1.0, float("nan"), float("inf")):
        refused(B.HT_EINVAL, temperature=T)
    refused(B.HT_EINVAL, reduction=5)
    refused(B.HT_ESHAPE, X=torch.zeros(4, 8, pin_memory=True))
    refused(B.HT_ESHAPE, dlogits=torch.zeros(3, 8, device="cuda"))
    refused(B.HT_ESHAPE, ids=torch.zeros(4, 257, dtype=torch.int32, device="cuda"), top=torch.zeros(4, 257, device="cuda"))
    refused(B.HT_ESHAPE, ids=torch.zeros(4, 0, dtype=torch.int32, device="cuda"), top=torch.zeros(4, 0, device="cuda"))
    big = torch.zeros(5, 8, device="cuda")
    refused(B.HT_EINVAL, X=big[:4], dlogits=big[1:])
    with pytest.raises(AssertionError):
        B.ht_distill_loss(ctx, 8, X, ids.long(), top, loss)


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("n,C,K", [(70, 66_003, 40), (65, 131_073, 256)])
def test_rows_past_the_registers(ctx, n, C, K, inplace):
    X, ids, top = _inputs(n, C, K, np.random.default_rng(n), missing=0.1)
    X[1, ::3] = -np.inf
    ids[1] = np.where(ids[1] % 3 == 0, -1, ids[1])
    ids[2, 1::2] = ids[2, 0]
    ref, tol = reference(X, ids, top, 2.0, None, True)
    check(call(ctx, X, ids, top, 2.0, inplace=inplace), ref, tol)


@pytest.mark.parametrize("n,C", [(3, 5), (40, 70), (5, 190), (6, 301), (3, 5_001), (66, 5_001), (65, 66_003)])
def test_what_lies_behind_the_last_class(ctx, n, C):
    X, ids, top = _inputs(n, C, 4, np.random.default_rng(C), missing=0.0)
    ids[n - 1] = -1
    u = np.full(n, np.inf, np.float32)
    u[0] = np.nan
    wide = (C + 3) // 4 * 4
    Xd = torch.full((n, wide), float("nan"), device="cuda")
    Xd[:, :C] = torch.from_numpy(X).cuda()
    dX = torch.full_like(Xd, 7.0)
    loss = torch.zeros(1, device="cuda")
    B.ht_distill_loss(ctx, C, Xd, torch.from_numpy(ids.astype(np.int32)).cuda(), torch.from_numpy(top).cuda(), loss, row_weight=torch.from_numpy(u).cuda(), dlogits=dX)
    assert (dX[:, C:] == 0).all() and dX[0, :C].isnan().all() and (dX[n - 1] == 0).all() and not dX[1:n - 1, :C].isfinite().all()


@pytest.mark.parametrize("n,C", [(0, 10), (0, 5_000), (0, 70_000), (64, 10), (64, 4_096), (64, 4_097), (65, 4_096)])
def test_few_rows(ctx, n, C):
    X, ids, top = _inputs(n, C, 5, np.random.default_rng(C), missing=0.2) if n else (np.ones((0, C), np.float32), np.zeros((0, 5), np.int64), np.zeros((0, 5), np.float32))
    for mean in (True, False):
        out = call(ctx, X, ids, top, 1.5, mean=mean)
        if n:
            ref, tol = reference(X, ids, top, 1.5, None, mean)
            check(out, ref, tol)
        else:
            assert out["loss"] == 0
