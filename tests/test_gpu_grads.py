"""ht_grad_norm and ht_grad_clip against 64-bit sums.

A norm is summed up in 64 bits and rounded once: half a step, 2^-24 of it, and 2^-40 for the sums.  What is scaled takes the rounding of the factor and that of the
product (or of the sum with what is there), half a step each."""
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


def _tensors(shapes, seed=0, scale=1.0):
    """(rows, columns, pitch, floats before it): tensors on the GPU with NaN around their data, and that data."""
    rng = np.random.default_rng(seed)
    out = []
    for k, (rows, cols, ld, off) in enumerate(shapes):
        x = (rng.standard_normal((rows, cols)) * scale * 10.0 ** (k % 4 - 2)).astype(np.float32)
        whole = torch.full((off + rows * ld + 5,), float("nan"), device="cuda")
        t = whole[off:off + rows * ld].view(rows, ld)
        t[:, :cols] = torch.from_numpy(x).cuda()
        out.append((t, x))
    return out


SETS = {
    "one": [(1, 1, 1, 0)],
    "vector": [(1, 4099, 4099, 1)],
    "unit": [(1, 16384, 16384, 0), (1, 16385, 16385, 3)],
    "pitched": [(5, 7, 9, 2), (300, 33, 64, 0), (33, 300, 301, 1), (1000, 3, 4, 0), (4, 1000, 1000, 0)],
    "some empty": [(0, 5, 8, 0), (7, 3, 3, 0), (0, 1, 1, 0)],
    "many": [(1 + i % 17, 1 + 13 * i % 70, 1 + 13 * i % 70 + i % 3, i % 4) for i in range(200)],
    "just a list": [(2, 5, 5, 0)] * 64,
    "a list and one": [(2, 5, 7, 0)] * 65,
    "large": [(3000, 701, 704, 0), (2000, 2000, 2000, 0), (1, 1_000_003, 1_000_003, 2)],
}


def _norm(data):
    return np.sqrt(sum((x.astype(np.float64) ** 2).sum() for x in data))


def _run(ctx, tensors, max_norm, **kw):
    norm = torch.full((1,), 7.0, device="cuda")
    cols = [x.shape[1] for _, x in tensors]
    B.ht_grad_clip(ctx, [t for t, _ in tensors], max_norm, norm=norm, cols=cols, **kw)
    B.ht_sync(ctx)
    return float(norm)


def _close(got, want, room):
    got, want = got.astype(np.float64), np.asarray(want, dtype=np.float64)
    assert (np.abs(got - want) <= room).all(), float((np.abs(got - want) - room).max())


@pytest.mark.parametrize("name", list(SETS))
def test_norms(ctx, name):
    tensors = _tensors(SETS[name])
    norm = torch.full((1,), 7.0, device="cuda")
    B.ht_grad_norm(ctx, [t for t, _ in tensors], norm, cols=[x.shape[1] for _, x in tensors])
    B.ht_sync(ctx)
    want = _norm([x for _, x in tensors])
    assert abs(float(norm) - want) <= (HALF + 2.0 ** -40) * want


@pytest.mark.parametrize("ratio", [0.3, 1.5])
@pytest.mark.parametrize("name", list(SETS))
def test_clipping(ctx, name, ratio):
    """In place, beside, and added with a scale; what surrounds the data is left as it was."""
    data = [x for _, x in _tensors(SETS[name])]
    want = _norm(data)
    max_norm = float(np.float32(ratio * want)) if want > 0 else 1.0
    c = min(1.0, max_norm / want) if want > 0 else 1.0
    cols = [x.shape[1] for x in data]
    # in place
    tensors = _tensors(SETS[name])
    before = [t.clone() for t, _ in tensors]
    got = _run(ctx, tensors, max_norm)
    assert abs(got - want) <= (HALF + 2.0 ** -40) * want
    for (t, x), b in zip(tensors, before):
        _close(t[:, :x.shape[1]].cpu().numpy(), c * x.astype(np.float64), 2.1 * HALF * np.abs(x))
        assert torch.equal(t[:, x.shape[1]:].nan_to_num(nan=-3.0), b[:, x.shape[1]:].nan_to_num(nan=-3.0))
        if ratio > 1:
            assert np.array_equal(t[:, :x.shape[1]].cpu().numpy(), x)
    # beside, with other pitches, scaled; then added
    tensors = _tensors(SETS[name])
    out = [torch.full((x.shape[0], x.shape[1] + 1 + k % 3), 0.25, device="cuda") for k, x in enumerate(data)]
    for add in (False, True):
        _run(ctx, tensors, max_norm, out=out, scale=-0.5, accumulate=add)
        for o, (t, x), b in zip(out, tensors, before):
            g = -0.5 * c * x.astype(np.float64)
            once = 2.1 * HALF * np.abs(g)
            _close(o[:, :x.shape[1]].cpu().numpy(), 2 * g if add else g, 2 * once + 3 * HALF * np.abs(2 * g) if add else once)
            assert (o[:, x.shape[1]:] == 0.25).all()
            assert torch.equal(t.nan_to_num(nan=-3.0), b.nan_to_num(nan=-3.0))
        assert cols == [x.shape[1] for x in data]


def test_a_step_of_gradient_descent(ctx):
    rng = np.random.default_rng(3)
    W = [rng.standard_normal(s).astype(np.float32) for s in ((40, 30), (30, 90), (1, 30))]
    G = [(rng.standard_normal(w.shape) * 10).astype(np.float32) for w in W]
    Wd, Gd = [torch.from_numpy(w).cuda() for w in W], [torch.from_numpy(g).cuda() for g in G]
    B.ht_grad_clip(ctx, Gd, 1.0, out=Wd, scale=-0.1, accumulate=True)
    B.ht_sync(ctx)
    norm = _norm(G)
    for w, g, t in zip(W, G, Wd):
        step = 0.1 / norm * g.astype(np.float64)
        _close(t.cpu().numpy(), w - step, HALF * np.abs(w - step) * 1.01 + 1.1 * HALF * np.abs(step))


def test_values_whose_squares_leave_the_range_of_floats(ctx):
    norm = torch.zeros(1, device="cuda")
    for scale in (1e-42, 1e-30, 1e25, 1e36):
        x = (np.random.default_rng(1).standard_normal((50, 40)) * scale).astype(np.float32)
        B.ht_grad_norm(ctx, [torch.from_numpy(x).cuda()], norm)
        B.ht_sync(ctx)
        assert abs(float(norm) - _norm([x])) <= (HALF + 2.0 ** -40) * _norm([x]) + 2.0 ** -150
    x = np.full((1, 100), 3e38, dtype=np.float32)
    t = torch.from_numpy(x).cuda()
    B.ht_grad_clip(ctx, [t], 1.0, norm=norm)           # a norm of 3e39: the factor is taken from it in 64 bits
    B.ht_sync(ctx)
    assert float(norm) == float("inf")
    _close(t.cpu().numpy(), np.full((1, 100), 0.1), 3 * HALF * 0.1 + 0.1 * 2.0 ** -17)      # (a factor of 3e-40 has 18 bits)


def test_what_is_not_finite(ctx):
    norm = torch.zeros(1, device="cuda")
    a, b = torch.ones(3, 5, device="cuda"), torch.ones(4, device="cuda")
    b[2] = float("inf")
    B.ht_grad_clip(ctx, [a, b], 1.0, norm=norm)
    B.ht_sync(ctx)
    assert float(norm) == float("inf") and (a == 0).all() and b.isnan().tolist() == [False, False, True, False]
    a, b = torch.ones(3, 5, device="cuda"), torch.ones(4, device="cuda")
    a[1, 1] = float("nan")
    for max_norm in (1.0, float("inf")):
        B.ht_grad_clip(ctx, [a, b], max_norm, norm=norm)
        B.ht_sync(ctx)
        assert norm.isnan().all() and a.isnan().all() and b.isnan().all()
    b = torch.full((4,), 2.0, device="cuda")
    B.ht_grad_clip(ctx, [b], float("inf"), norm=norm)  # no limit: as they are
    B.ht_sync(ctx)
    assert float(norm) == 4.0 and (b == 2.0).all()


def test_nothing_at_all(ctx):
    norm = torch.full((1,), 7.0, device="cuda")
    B.ht_grad_norm(ctx, [], norm)
    B.ht_sync(ctx)
    assert float(norm) == 0.0
    norm.fill_(7.0)
    B.ht_grad_clip(ctx, [], 1.0, norm=norm)
    B.ht_grad_clip(ctx, [], 1.0)
    B.ht_sync(ctx)
    assert float(norm) == 0.0
    z = torch.zeros(3, 3, device="cuda")
    B.ht_grad_clip(ctx, [z], 1.0, norm=norm)
    B.ht_sync(ctx)
    assert float(norm) == 0.0 and (z == 0).all()


def test_the_same_bits_from_call_to_call(ctx):
    tensors = _tensors(SETS["large"] + SETS["many"])
    norms = []
    for _ in range(3):
        norm = torch.zeros(1, device="cuda")
        B.ht_grad_norm(ctx, [t for t, _ in tensors], norm, cols=[x.shape[1] for _, x in tensors])
        B.ht_sync(ctx)
        norms.append(float(norm))
    assert len(set(norms)) == 1


def test_refusals(ctx):
    def refused(code, text, call):
        with pytest.raises(B.HongtuError) as err:
            call()
        assert err.value.code == code and text in str(err.value), str(err.value)

    EINVAL, ESHAPE = -1, -4
    a, b = torch.ones(6, 8, device="cuda"), torch.ones(6, 8, device="cuda")
    for bad in (0.0, -1.0, float("nan")):
        refused(EINVAL, "max_norm", lambda: B.ht_grad_clip(ctx, [a], bad))
    refused(ESHAPE, "gradient 1", lambda: B.ht_grad_norm(ctx, [a, b[:, :4]], torch.zeros(1, device="cuda"), cols=[8, 9]))
    refused(ESHAPE, "out 0", lambda: B.ht_grad_clip(ctx, [a], 1.0, out=[b[:5]]))
    refused(EINVAL, "shares memory", lambda: B.ht_grad_clip(ctx, [a, a], 1.0))                       # scaled twice
    refused(EINVAL, "shares memory", lambda: B.ht_grad_clip(ctx, [a, b], 1.0, out=[b, a]))
    refused(EINVAL, "shares memory", lambda: B.ht_grad_clip(ctx, [a[:5]], 1.0, out=[a[1:]]))
    refused(EINVAL, "shares memory", lambda: B.ht_grad_clip(ctx, [a, b], 1.0, out=[a, a]))
    host = torch.ones(4, 4).pin_memory()
    refused(ESHAPE, "HBM", lambda: B.ht_grad_norm(ctx, [host], torch.zeros(1, device="cuda")))
    assert (a == 1).all() and (b == 1).all()
    B.ht_grad_clip(ctx, [a[:, :4], a[:, 4:]], 1.0)                                                   # halves of one matrix share nothing
    B.ht_sync(ctx)
    assert np.allclose(a.cpu().numpy(), 1 / np.sqrt(48))
    norm = torch.zeros(1, device="cuda")
    B.ht_grad_norm(ctx, [b, b], norm)                                                                # a norm may count a tensor twice
    B.ht_sync(ctx)
    assert abs(float(norm) - np.sqrt(96)) < 1e-5


def test_a_norm_lies_in_no_tensor(ctx):
    """Written over a gradient it would be scaled with it, written over an output it would be none; between a tensor's rows it may lie."""
    whole, out = torch.ones(6, 8, device="cuda"), torch.zeros(6, 8, device="cuda")
    norm = whole.view(-1)
    for at in (0, 4, 43, 44):                                       # the first value, the first row's last, the last row's
        for call in (lambda: B.ht_grad_norm(ctx, [out, whole], norm[at:at + 1], cols=[8, 5]),
                     lambda: B.ht_grad_clip(ctx, [out, whole], 1.0, norm=norm[at:at + 1], cols=[8, 5]),
                     lambda: B.ht_grad_clip(ctx, [out], 1.0, out=[whole], norm=norm[at:at + 1], cols=[5])):
            with pytest.raises(B.HongtuError) as err:
                call()
            assert err.value.code == -1 and "norm shares memory" in str(err.value)
    assert (whole == 1).all() and (out == 0).all()
    for at in (5, 15, 45, 47):                                      # behind a row's five values
        whole.fill_(1.0)
        B.ht_grad_clip(ctx, [whole], 1.0, norm=norm[at:at + 1], cols=[5])
        B.ht_sync(ctx)
        assert float(norm[at]) == np.float32(np.sqrt(30.0))
        assert (np.abs(whole[:, :5].cpu().numpy() - 1 / np.sqrt(30.0)) <= 2 * HALF).all()
