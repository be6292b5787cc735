"""ht_head_loss against the same formulas in 64 bits.

Tolerances, element by element.  A logit's products are off by 3 x 2^-22 of their size at most and its sum is rounded 3 times per 16
values and at its scaling (a step each, 2^-23 of the sum of sizes A): e = (3 x 2^-22 + (3 ceil(d / 16) + 4) 2^-23) A.  log sum exp
is off by the largest e of its row, and a few steps of itself and of the logits (their product with log2 e, its maximum, the exponential): b.  A
probability is off by (e + its row's b + 2^-20) of itself and 2^-39, the label's by a step of 1 more; gradients by what those
put in, by the products' 3 x 2^-22 and by a rounding of the sum per 16 values, per part of it and per scaling."""
import numpy as np
import pytest
import torch

from paper_2311_14898_amd import binding as B

pytestmark = pytest.mark.gpu
STEP = 2.0 ** -23


@pytest.fixture(scope="module")
def ctx():
    c = B.ht_ctx_create(0)
    yield c
    B.ht_ctx_destroy(c)


def _pad(x, ld=None, fill=float("nan")):
    ld = ld or (x.shape[1] + 3) // 4 * 4
    m = torch.full((x.shape[0], ld), fill, device="cuda")
    m[:, :x.shape[1]] = torch.from_numpy(x).cuda()
    return m


def reference(H, W, y, u, mean):
    """In 64 bits: loss, row_loss, row_lse, dH, dW of the [d x C] weights, and how far fp32 may be off each of them."""
    H, W = H.astype(np.float64), W.astype(np.float64)
    (n, d), C = H.shape, W.shape[1]
    has = y >= 0
    N = max(1, has.sum()) if mean else 1
    u = np.where(has, 1.0 if u is None else u.astype(np.float64), 0.0)
    x = H @ W
    A = np.abs(H) @ np.abs(W)
    e = (3 * 2.0 ** -22 + (3 * np.ceil(d / 16) + 4) * STEP) * A
    m = x.max(axis=1)
    lse = np.log(np.exp(x - m[:, None]).sum(axis=1)) + m
    at = np.arange(n), np.where(has, y, 0)
    size = np.abs(x).max(axis=1) + np.abs(lse)
    b = e.max(axis=1) + 4 * STEP * (size + 1) + 2.0 ** -20
    l = np.where(has, lse - x[at], 0.0)
    p = np.exp(x - lse[:, None])
    g = p.copy()
    g[at] -= 1.0
    pe = p * (e + b[:, None] + 2.0 ** -20) + 2.0 ** -39
    pe[at] += 2 * STEP
    f = (u / N)[:, None]
    g, pe = g * f, pe * np.abs(f)
    terms = 3 * 2.0 ** -22 + (3 * max(n, C) / 16 + 64) * STEP
    out = dict(loss=(u * l).sum() / N, row_loss=l, row_lse=np.where(has, lse, 0.0), dH=g @ W.T, dW=H.T @ g)
    le = np.where(has, b + e[at] + 2 * STEP * np.abs(l), 0.0)
    tol = dict(loss=(np.abs(u) * le).sum() / N + STEP * np.abs(u * l).sum() / N, row_loss=le, row_lse=np.where(has, b, 0.0),
               dH=pe @ np.abs(W).T + terms * (np.abs(g) @ np.abs(W).T), dW=np.abs(H).T @ pe + terms * (np.abs(H).T @ np.abs(g)))
    return out, tol


def call(ctx, H, W, y, form, u=None, mean=True, grad=True, dW0=None, ld_w=None):
    n, d, C = H.shape[0], H.shape[1], W.shape[1]
    stored = W if form == B.HT_W_IN_OUT else np.ascontiguousarray(W.T)
    cols = stored.shape[1]
    Hd, Wd = _pad(H), _pad(stored, ld_w or cols)
    yd = torch.from_numpy(y.astype(np.int32)).cuda()
    ud = None if u is None else torch.from_numpy(u).cuda()
    loss, row_loss, row_lse = (torch.full((k,), 7.0, device="cuda") for k in (1, n, n))
    dH = torch.full((n + 1, Hd.shape[1]), 7.0, device="cuda") if grad else None
    dW = None
    if grad:
        dW = torch.full((stored.shape[0], ld_w or cols), 7.0, device="cuda")
        if dW0 is not None:
            dW[:, :cols] = torch.from_numpy(dW0 if form == B.HT_W_IN_OUT else np.ascontiguousarray(dW0.T)).cuda()
    B.ht_head_loss(ctx, d, C, Hd, Wd, yd, loss, row_weight=ud, row_loss=row_loss, row_lse=row_lse, dH=dH[:n] if grad else None, dW=dW, w_form=form,
                   reduction=B.HT_REDUCE_MEAN if mean else B.HT_REDUCE_SUM, accumulate_dW=dW0 is not None)
    B.ht_sync(ctx)
    out = dict(loss=float(loss), row_loss=row_loss.cpu().numpy(), row_lse=row_lse.cpu().numpy())
    if grad:
        assert (dH[n] == 7.0).all()
        got = dW[:, :cols].cpu().numpy()
        out.update(dH=dH[:n, :d].cpu().numpy(), dW=got if form == B.HT_W_IN_OUT else got.T)
    return out


def check(out, ref, tol, dW0=None):
    for k in out:
        want, room = ref[k], tol[k]
        if k == "dW" and dW0 is not None:
            want, room = want + dW0, room + STEP * np.abs(dW0)
        err = np.abs(np.asarray(out[k], dtype=np.float64) - want)
        assert (err <= room).all(), (k, float((err - room).max()), float(err.max()), float(np.abs(want).max()))


def _inputs(n, d, C, rng, unlabelled=0.0, spread=2.0):
    H = rng.standard_normal((n, d)).astype(np.float32)
    W = (rng.standard_normal((d, C)) * (spread / np.sqrt(d))).astype(np.float32)
    y = rng.integers(0, C, n)
    y[rng.random(n) < unlabelled] = -1
    return H, W, y


SIZES = [(1, 1, 1), (1, 256, 5000), (2, 16, 3), (5, 33, 257), (31, 64, 1000), (32, 100, 256), (33, 7, 41), (64, 602, 300), (65, 128, 2049), (100, 1, 70),
         (127, 31, 513), (129, 256, 1024), (200, 300, 9001), (257, 47, 8192), (1000, 64, 172), (2000, 130, 777), (700, 1030, 640)]


@pytest.mark.parametrize("form", [B.HT_W_IN_OUT, B.HT_W_OUT_IN])
@pytest.mark.parametrize("n,d,C", SIZES)
def test_sizes(ctx, n, d, C, form):
    H, W, y = _inputs(n, d, C, np.random.default_rng(n + d + C), unlabelled=0.2 if n > 40 else 0.0)
    ref, tol = reference(H, W, y, None, True)
    check(call(ctx, H, W, y, form), ref, tol)
    check(call(ctx, H, W, y, form, grad=False), ref, tol)


@pytest.mark.parametrize("n", [3, 40, 300])
def test_weights_sums_and_added_gradients(ctx, n):
    rng = np.random.default_rng(n)
    H, W, y = _inputs(n, 70, 333, rng, unlabelled=0.3)
    y[0] = 5
    u = (rng.standard_normal(n) * 3).astype(np.float32)
    u[1] = 0.0
    dW0 = rng.standard_normal(W.shape).astype(np.float32)
    for form in (B.HT_W_IN_OUT, B.HT_W_OUT_IN):
        for mean in (True, False):
            ref, tol = reference(H, W, y, u, mean)
            check(call(ctx, H, W, y, form, u=u, mean=mean), ref, tol)
            check(call(ctx, H, W, y, form, u=u, mean=mean, dW0=dW0, ld_w=W.shape[1] + 3 if form == B.HT_W_IN_OUT else 77), ref, tol, dW0)


@pytest.mark.parametrize("labelled", ["none", "first", "last", "every 50th"])
def test_rows_without_labels(ctx, labelled):
    rng = np.random.default_rng(3)
    n, d, C = 1500, 40, 600
    H, W, y = _inputs(n, d, C, rng)
    keep = {"none": [], "first": [0], "last": [n - 1], "every 50th": list(range(7, n, 50))}[labelled]
    z = np.full(n, -1)
    z[keep] = y[keep]
    H[z < 0] = np.nan                                      # nothing of these rows is read
    clean = np.where((z < 0)[:, None], 0.0, H).astype(np.float32)
    ref, tol = reference(clean, W, z, None, True)
    for form in (B.HT_W_IN_OUT, B.HT_W_OUT_IN):
        out = call(ctx, H, W, z, form)
        check(out, ref, tol)
        assert (out["dH"][z < 0] == 0).all() and (out["row_loss"][z < 0] == 0).all()
        if not keep:
            assert out["loss"] == 0 and (out["dW"] == 0).all()


@pytest.mark.parametrize("h,w", [(1e-20, 1e20), (1e18, 1e-17), (1e-30, 1.0), (3e4, 1e-4)])
def test_sizes_of_values(ctx, h, w):
    """Rows and classes whose values lie many powers of two apart: each keeps its own precision."""
    rng = np.random.default_rng(8)
    n, d, C = 150, 96, 400
    H, W, y = _inputs(n, d, C, rng)
    H = (H * np.float32(h) * np.exp2(rng.integers(-8, 2, (n, 1)))).astype(np.float32)
    W = (W * np.float32(w) * np.exp2(rng.integers(-8, 2, (1, C)))).astype(np.float32)
    ref, tol = reference(H, W, y, None, True)
    check(call(ctx, H, W, y, B.HT_W_OUT_IN), ref, tol)


def test_large_logits_and_sure_rows(ctx):
    """Logits of hundreds, rows whose label has all of the probability, rows whose label has none."""
    rng = np.random.default_rng(9)
    H, W, y = _inputs(130, 64, 700, rng, spread=60.0)
    x = H.astype(np.float64) @ W
    y[:60] = x[:60].argmax(axis=1)
    y[60:90] = x[60:90].argmin(axis=1)
    ref, tol = reference(H, W, y, None, True)
    check(call(ctx, H, W, y, B.HT_W_IN_OUT), ref, tol)


def test_labels_beyond_the_classes_and_values_that_are_not_finite(ctx):
    rng = np.random.default_rng(10)
    H, W, y = _inputs(70, 32, 90, rng)
    good = call(ctx, H, W, y, B.HT_W_OUT_IN)
    z = y.copy()
    z[11] = 90
    out = call(ctx, H, W, z, B.HT_W_OUT_IN)
    assert np.isnan(out["loss"]) and np.isnan(out["row_loss"][11])
    rest = np.arange(70) != 11
    assert (out["row_loss"][rest] == good["row_loss"][rest]).all() and (out["dH"][rest] == good["dH"][rest]).all()
    for bad in (np.nan, np.inf, -np.inf):
        G = H.copy()
        G[11, 3] = bad
        out = call(ctx, G, W, y, B.HT_W_OUT_IN)
        assert np.isnan(out["loss"]) and np.isnan(out["row_loss"][11]) and np.isnan(out["dH"][11]).all()
        assert (out["row_loss"][rest] == good["row_loss"][rest]).all() and (out["dH"][rest] == good["dH"][rest]).all()


@pytest.mark.parametrize("n", [40, 70])
@pytest.mark.parametrize("first,last", [(0, 300), (300, 600), (599, 600)])
def test_weights_that_are_not_numbers_reach_every_row(ctx, n, first, last):
    """Whole tiles of classes without a largest logit, before and behind others."""
    H, W, y = _inputs(n, 32, 600, np.random.default_rng(14))
    W[5, first:last] = np.nan
    for form in (B.HT_W_IN_OUT, B.HT_W_OUT_IN):
        out = call(ctx, H, W, y, form)
        assert np.isnan(out["loss"]) and np.isnan(out["row_loss"]).all() and np.isnan(out["row_lse"]).all()
        assert np.isnan(out["dH"]).all() and np.isnan(out["dW"]).all()


@pytest.mark.parametrize("n", [8, 90])
def test_logits_of_millions(ctx, n):
    """Far from 0 the rows' own differences count: integers, whose logits are exact, so that tolerances have no part of the products' errors."""
    rng = np.random.default_rng(15)
    d, C = 4, 700
    H = rng.integers(1, 5, (n, d)).astype(np.float32)
    W = (rng.integers(-3, 4, (d, C)) + np.array([[1 << 20], [0], [0], [0]])).astype(np.float32)
    y = rng.integers(0, C, n)
    x = H.astype(np.float64) @ W.astype(np.float64)
    p = np.exp(x - x.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    g = p.copy()
    g[np.arange(n), y] -= 1.0
    out = call(ctx, H, W, y, B.HT_W_IN_OUT, mean=False)
    # p: the exponential's argument (up to 100) in half steps, two steps of its own, the sum of 700 terms; products and their sums as above
    rel = 2.0 ** -24 * (100 + 4) + 20 * STEP
    pe = p * rel + 2.0 ** -39
    pe[np.arange(n), y] += 2 * STEP
    terms = 3 * 2.0 ** -22 + (3 * C / 16 + 64) * STEP
    assert (np.abs(out["dW"] - H.T.astype(np.float64) @ g) <= H.T @ pe + terms * (H.T @ np.abs(g))).all()
    # dH = sum over classes of g W, where each row's g has the sum 0: W's common part, 2^20, multiplies what rounding leaves of it
    assert (np.abs(out["dH"] - g @ W.T.astype(np.float64)) <= pe @ np.abs(W).T + terms * (np.abs(g) @ np.abs(W).T)).all()


def test_differences(ctx):
    """Gradients against central differences of the loss in 64 bits at the same point, and of the call's own loss."""
    rng = np.random.default_rng(11)
    H, W, y = _inputs(12, 20, 50, rng)
    out = call(ctx, H, W, y, B.HT_W_IN_OUT)

    def loss(H, W):
        x = H.astype(np.float64) @ W.astype(np.float64)
        return (np.log(np.exp(x).sum(axis=1)) - x[np.arange(12), y]).mean()

    for v, j in ((0, 0), (5, 13), (11, 19)):
        for at, M, g in ((("H", v, j), H, out["dH"][v, j]), (("W", j, v), W, out["dW"][j, v])):
            up, down = M.astype(np.float64).copy(), M.astype(np.float64).copy()
            up[at[1], at[2]] += 1e-4
            down[at[1], at[2]] -= 1e-4
            d = (loss(up, W) - loss(down, W)) if at[0] == "H" else (loss(H, up) - loss(H, down))
            assert abs(d / 2e-4 - g) <= 1e-6               # 1e-8 by the third derivative, the rest is the gradient's own
    eps = 0.25
    G = H.copy()
    G[5, 13] += eps
    F = H.copy()
    F[5, 13] -= eps
    d = (call(ctx, G, W, y, B.HT_W_IN_OUT, grad=False)["loss"] - call(ctx, F, W, y, B.HT_W_IN_OUT, grad=False)["loss"]) / (2 * eps)
    assert abs(d - out["dH"][5, 13]) <= 0.02 * np.abs(out["dH"]).max() + 2e-6      # (third derivative: eps^2 / 6 of a few weights cubed / 12 rows)


def test_the_same_bits_and_one_gradient_alone(ctx):
    rng = np.random.default_rng(12)
    n, d, C = 900, 200, 3000
    H, W, y = _inputs(n, d, C, rng, unlabelled=0.1)
    a, b = call(ctx, H, W, y, B.HT_W_IN_OUT), call(ctx, H, W, y, B.HT_W_IN_OUT)
    for k in a:
        assert np.array_equal(a[k], b[k]), k
    Hd, Wd, yd = _pad(H), _pad(W), torch.from_numpy(y.astype(np.int32)).cuda()
    for which in ("dH", "dW"):
        loss, out = torch.zeros(1, device="cuda"), torch.zeros(n if which == "dH" else d, d if which == "dH" else C, device="cuda")
        B.ht_head_loss(ctx, d, C, Hd, Wd, yd, loss, **{which: out})
        B.ht_sync(ctx)
        assert float(loss) == a["loss"] and np.array_equal(out.cpu().numpy(), a[which])


def test_pieces_under_a_byte_budget():
    """With little memory rows and classes go in many pieces; other sizes of pieces, the same tolerances."""
    rng = np.random.default_rng(13)
    n, d, C = 40_000, 24, 1500
    H, W, y = _inputs(n, d, C, rng, unlabelled=0.05)
    ref, tol = reference(H, W, y, None, True)
    ctx = B.ht_ctx_create(0)
    try:
        B.ht_ctx_set_hbm_budget(ctx, 200 << 20)
        check(call(ctx, H, W, y, B.HT_W_IN_OUT), ref, tol)
        check(call(ctx, H, W, y, B.HT_W_OUT_IN), ref, tol)
    finally:
        B.ht_ctx_destroy(ctx)
    ctx = B.ht_ctx_create(0)
    try:
        B.ht_ctx_set_hbm_budget(ctx, 1 << 20)
        with pytest.raises(B.HongtuError) as err:
            call(ctx, H, W, y, B.HT_W_IN_OUT)
        assert err.value.code == B.HT_ENOMEM
    finally:
        B.ht_ctx_destroy(ctx)


def test_no_rows(ctx):
    loss = torch.full((1,), 7.0, device="cuda")
    dW = torch.full((8, 12), 7.0, device="cuda")
    B.ht_head_loss(ctx, 8, 12, torch.zeros(0, 8, device="cuda"), torch.zeros(8, 12, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"), loss, dW=dW)
    B.ht_sync(ctx)
    assert float(loss) == 0 and (dW == 0).all()


def test_refusals(ctx):
    H, W, y, loss = torch.zeros(6, 8, device="cuda"), torch.zeros(8, 5, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda")

    def refused(code, d=8, C=5, H=H, W=W, **kw):
        with pytest.raises(B.HongtuError) as err:
            B.ht_head_loss(ctx, d, C, H, W, y, loss, **kw)
        assert err.value.code == code, err.value

    refused(B.HT_ESHAPE, d=0)
    refused(B.HT_ESHAPE, C=0)
    refused(B.HT_ESHAPE, d=B.HT_HEAD_MAX_WIDTH + 1)
    refused(B.HT_ESHAPE, C=B.HT_HEAD_MAX_CLASSES + 1)
    refused(B.HT_ESHAPE, d=7)
    refused(B.HT_ESHAPE, C=6)
    refused(B.HT_ESHAPE, w_form=B.HT_W_OUT_IN)
    refused(B.HT_EINVAL, w_form=2)
    refused(B.HT_EINVAL, reduction=2)
    refused(B.HT_ESHAPE, H=torch.zeros(6, 9, device="cuda")[:, :9])
    refused(B.HT_ESHAPE, H=torch.zeros(6, 8, pin_memory=True))
    refused(B.HT_ESHAPE, W=torch.zeros(8, 5, pin_memory=True))
    refused(B.HT_EINVAL, dH=H)
    refused(B.HT_EINVAL, dW=W)
    refused(B.HT_ESHAPE, dH=torch.zeros(5, 8, device="cuda"))
    both = torch.zeros(200, device="cuda")
    refused(B.HT_EINVAL, dH=both[:48].view(6, 8), dW=both[40:80].view(8, 5))
    with pytest.raises(AssertionError):
        B.ht_head_loss(ctx, 8, 5, H, W, y.long(), loss)
    with pytest.raises(AssertionError):
        B.ht_head_loss(ctx, 8, 5, H, W, y, loss, row_weight=torch.zeros(5, device="cuda"))


@pytest.mark.parametrize("n", [16_384, 16_385, 70_001])
def test_few_labels_among_many_rows(ctx, n):
    rng = np.random.default_rng(n)
    d, C = 35, 300
    H, W, y = _inputs(n, d, C, rng)
    y[rng.random(n) < 0.98] = -1
    y[[0, n - 1]] = [-1, 7]
    H[y < 0] = np.nan                                      # nothing of these rows is read
    has = y >= 0
    ref, tol = reference(H[has], W, y[has], None, True)
    for form in (B.HT_W_IN_OUT, B.HT_W_OUT_IN):
        out = call(ctx, H, W, y, form)
        assert (out["dH"][~has] == 0).all() and (out["row_loss"][~has] == 0).all() and (out["row_lse"][~has] == 0).all()
        check({k: v[has] if k in ("dH", "row_loss", "row_lse") else v for k, v in out.items()}, ref, tol)


@pytest.mark.parametrize("n,d,C", [(2_300, 193, 262_144), (300, 256, 70_001), (66, 100, 262_145)])
def test_many_classes(ctx, n, d, C):
    """The same formulas and tolerances with the 64-bit sums on the GPU: rows in two pieces whose sums are kept, rows in one, rows whose sums are made again."""
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    H = torch.randn(n, (d + 3) // 4 * 4, generator=g, device="cuda")
    W = torch.randn(C, d, generator=g, device="cuda") * (2.0 / d ** 0.5)
    y = torch.randint(0, C, (n,), generator=g, device="cuda", dtype=torch.int32)
    y[5] = -1
    loss, row_loss, dH, dW = torch.zeros(1, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros_like(H), torch.zeros_like(W)
    B.ht_head_loss(ctx, d, C, H, W, y, loss, row_loss=row_loss, dH=dH, dW=dW, w_form=B.HT_W_OUT_IN)
    H, W, dH = H[:, :d].double(), W.double(), dH[:, :d]
    has, at, N = y >= 0, (torch.arange(n, device="cuda"), y.clamp(min=0).long()), float((y >= 0).sum())
    x = H @ W.t().contiguous()
    e = (H.abs() @ W.abs().t().contiguous()) * (3 * 2.0 ** -22 + (3 * np.ceil(d / 16) + 4) * STEP)
    lse = torch.logsumexp(x, dim=1)
    b = e.amax(dim=1) + 4 * STEP * (x.abs().amax(dim=1) + lse.abs() + 1) + 2.0 ** -20
    l = torch.where(has, lse - x[at], 0.0)
    le = b + e[at] + 2 * STEP * l.abs()
    assert ((row_loss - l).abs() <= torch.where(has, le, 0.0)).all()
    assert abs(float(loss) - float(l.sum()) / N) <= float(torch.where(has, le, 0.0).sum()) / N + STEP * float(l.sum()) / N
    p = x.sub_(lse[:, None]).exp_()
    e.add_(b[:, None] + 2.0 ** -20).mul_(p).add_(2.0 ** -39)
    e[at] += 2 * STEP
    p[at] -= 1.0
    f = torch.where(has, 1.0 / N, 0.0).double()[:, None]
    p.mul_(f), e.mul_(f)
    terms = 3 * 2.0 ** -22 + (3 * max(n, C) / 16 + 64) * STEP
    assert ((dH - p @ W).abs() <= e @ W.abs() + terms * (p.abs() @ W.abs())).all()
    p, e = p.t().contiguous(), e.t().contiguous()
    assert ((dW - p @ H).abs() <= e @ H.abs() + terms * (p.abs() @ H.abs())).all()


@pytest.mark.parametrize("d,C,budget", [(100, 200, 150 << 20), (200, 1500, 200 << 20)])
@pytest.mark.parametrize("labelled", ["most", "the first", "none"])
def test_pieces_of_rows(d, C, budget, labelled):
    """Rows in pieces whose classes are all in one tile, or whose sums are kept; the last pieces may have no rows."""
    rng = np.random.default_rng(d)
    n = 40_000
    H, W, y = _inputs(n, d, C, rng, unlabelled=0.05)
    if labelled != "most":
        y[9_000 if labelled == "the first" else 0:] = -1
    ref, tol = reference(H, W, y, None, True)
    ctx = B.ht_ctx_create(0)
    try:
        B.ht_ctx_set_hbm_budget(ctx, budget)
        check(call(ctx, H, W, y, B.HT_W_IN_OUT), ref, tol)
        check(call(ctx, H, W, y, B.HT_W_OUT_IN, grad=False), ref, tol)
    finally:
        B.ht_ctx_destroy(ctx)
