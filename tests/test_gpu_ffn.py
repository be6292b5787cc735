"""ht_ffn_fwd and ht_ffn_bwd against the same formulas in 64 bits.

Tolerances, element by element.  A product of two matrices is off by 3 x 2^-22 of the sizes of its terms, by 2^-39 of the largest value of what either
factor is scaled by (the row, or the whole) times the other, and its sum is rounded 3 times per 16 terms and a few times behind that (a step each): `product`.
Activations are off by what their argument is off, times a slope of 1.13 at most (a curvature of 1.1), and by a few steps of themselves, more where their
argument is large and its rounding counts a^2 fold.  What a factor is off by passes through the products behind it."""
import math

import numpy as np
import pytest
import torch

from paper_2311_14898_amd import binding as B

pytestmark = pytest.mark.gpu
STEP = 2.0 ** -23
ACTS = {"silu": B.HT_GATE_SILU, "gelu": B.HT_GATE_GELU, "gelu_tanh": B.HT_GATE_GELU_TANH, "relu": B.HT_GATE_RELU, "sigmoid": B.HT_GATE_SIGMOID}
OUTS = ("dX", "dWg", "dWu", "dWd")


@pytest.fixture(scope="module")
def ctx():
    c = B.ht_ctx_create(0)
    yield c
    B.ht_ctx_destroy(c)


def activation(a, act):
    """act(a), act'(a), and how far fp32 may be off each for this very a."""
    erfc = np.vectorize(math.erfc, otypes=[np.float64])
    with np.errstate(over="ignore"):
        if act == "relu":
            return np.maximum(a, 0.0), (a > 0).astype(np.float64), 0.0 * a, 0.0 * a
        if act == "gelu":
            phi, dphi = 0.5 * erfc(-a / math.sqrt(2.0)), np.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi)
        else:
            k = 2.0 * math.sqrt(2.0 / math.pi)
            u, du = (k * (a + 0.044715 * a ** 3), k * (1.0 + 3.0 * 0.044715 * a * a)) if act == "gelu_tanh" else (a, 1.0)
            phi = 1.0 / (1.0 + np.exp(-u))
            dphi = phi / (1.0 + np.exp(u)) * du
    steps = (16.0 + 4.0 * a * a) * STEP
    if act == "sigmoid":
        return phi, dphi, steps * phi, steps * dphi
    return a * phi, phi + a * dphi, steps * np.abs(a * phi), steps * (phi + np.abs(a * dphi))


def product(x, w, xe=0.0, we=0.0, x_top=None, w_top=None):
    """x @ w, and how far it may be off where x and w are off by xe and we.  x_top, w_top: the largest values of what is scaled together (else rows of x, all of w)."""
    ax, aw = np.abs(x), np.abs(w)
    k = x.shape[1]
    x_top = ax.max(axis=1, keepdims=True) if x_top is None else x_top
    w_top = aw.max() if w_top is None else w_top
    room = (3 * 2.0 ** -22 + (3 * math.ceil(k / 16) + 8) * STEP) * (ax @ aw)
    room += 2.0 ** -39 * (np.broadcast_to(x_top, ax.shape) @ aw + ax @ np.broadcast_to(w_top, aw.shape))
    if np.ndim(xe):
        room += 1.01 * (xe @ (aw + we))
    if np.ndim(we):
        room += 1.01 * (ax @ we)
    return x @ w, room


def reference(X, Wg, Wu, Wd, act, dY=None, kept=None):
    """In 64 bits: outputs and how far fp32 may be off each of them.  kept: fp32 projections that are taken as they are."""
    X, Wg, Wu, Wd = (t.astype(np.float64) for t in (X, Wg, Wu, Wd))
    (A, ae), (U, ue) = product(X, Wg), product(X, Wu)
    out, tol = dict(gate=A, up=U), dict(gate=ae, up=ue)
    v, s, ve, se = activation(A, act)
    ve, se = ve + 1.13 * ae, se + (1.1 * ae if act != "relu" else 0.0)
    H, he = v * U, np.abs(v) * ue + np.abs(U) * ve + ve * ue + STEP * np.abs(v * U)
    out["Y"], tol["Y"] = product(H, Wd, he)
    if dY is None:
        return out, tol
    dY = dY.astype(np.float64)
    G, ge = product(dY, Wd.T)
    dU, due = G * v, ge * (np.abs(v) + ve) + np.abs(G) * ve + STEP * np.abs(G * v)
    dA = G * U * s
    dae = 1.01 * (ge * np.abs(U * s) + np.abs(G * s) * ue + np.abs(G * U) * se + ge * ue * np.abs(s)) + 2 * STEP * np.abs(dA)
    D, De, W2 = np.hstack([dA, dU]), np.hstack([dae, due]), np.hstack([Wg, Wu]).T
    out["dX"], tol["dX"] = product(D, W2, De)
    top = lambda x: np.abs(x).max(axis=0, keepdims=True)
    for name, g, e in (("dWg", dA, dae), ("dWu", dU, due)):
        out[name], tol[name] = product(X.T, g, 0.0, e, w_top=top(g))
    out["dWd"], tol["dWd"] = product(H.T, dY, he.T, 0.0, w_top=top(dY))
    return out, tol


def _matrix(x, ld=None, fill=float("nan"), extra=0):
    """On the GPU, in rows of a multiple of 4 (or ld) floats with `fill` behind the columns, and `extra` rows of it."""
    m = torch.full((x.shape[0] + extra, ld or (x.shape[1] + 3) // 4 * 4), fill, device="cuda")
    m[:x.shape[0], :x.shape[1]] = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return m


def call(ctx, X, Wg, Wu, Wd, act="silu", dY=None, form=B.HT_W_IN_OUT, keep=False, add=False, only=OUTS, fwd=True, ld_w=0):
    """All outputs as arrays, weights' gradients as [in x out]; with `add`, 0.5 lies in what is added to."""
    turn = (lambda w: w) if form == B.HT_W_IN_OUT else (lambda w: np.ascontiguousarray(w.T))
    (n, d), f, e = X.shape, Wg.shape[1], Wd.shape[1]
    Xd = _matrix(X)
    W = [_matrix(turn(w), ld=turn(w).shape[1] + ld_w) for w in (Wg, Wu, Wd)]
    first = 0.5 if add else 7.0
    room = lambda r, c: torch.full((r + 1, (c + 3) // 4 * 4), first, device="cuda")
    out, kept = {}, {}
    if keep:
        kept = dict(gate=room(n, f)[:n], up=room(n, f)[:n])
    if fwd:
        Y = room(n, e)
        B.ht_ffn_fwd(ctx, d, f, e, Xd, *W, Y[:n], act=ACTS[act], w_form=form, accumulate=add, **kept)
        B.ht_sync(ctx)
        assert (Y[n] == first).all()
        out["Y"] = Y[:n, :e].cpu().numpy()
        for k, t in kept.items():
            out[k] = t[:, :f].cpu().numpy()
    if dY is not None:
        grads = {"dX": room(n, d)}
        for k, w in zip(("dWg", "dWu", "dWd"), W):
            grads[k] = torch.full((w.shape[0] + 1, w.shape[1]), first, device="cuda")
        B.ht_ffn_bwd(ctx, d, f, e, Xd, *W, _matrix(dY), **{k: grads[k][:-1] for k in only}, act=ACTS[act], w_form=form, accumulate=add, accumulate_dW=add,
                     **kept)
        B.ht_sync(ctx)
        for k, t in grads.items():
            assert (t[-1] == first).all()
            if k not in only:
                assert (t == first).all()
            elif k == "dX":
                out[k] = t[:n, :d].cpu().numpy()
            else:
                i, o = (f, e) if k == "dWd" else (d, f)
                out[k] = t[:-1, :o].cpu().numpy() if form == B.HT_W_IN_OUT else t[:-1, :i].cpu().numpy().T
                cols = o if form == B.HT_W_IN_OUT else i
                assert (t[:-1, cols:] == first).all()
    return out


def check(out, ref, tol, add=False):
    for k in out:
        want, room = ref[k], tol[k]
        if add and k not in ("gate", "up"):
            want, room = want + 0.5, room + STEP * (np.abs(want) + 0.5)
        err = np.abs(out[k].astype(np.float64) - want)
        assert (err <= room).all(), (k, float((err - room).max()), float(err.max()), float(np.abs(want).max()))


def _inputs(n, d, f, e, seed=0, gate=1.5):
    rng = np.random.default_rng(n + 3 * d + 5 * f + 7 * e + seed)
    r = lambda a, b, s: (rng.standard_normal((a, b)) * s).astype(np.float32)
    return r(n, d, 1.0), r(d, f, gate / math.sqrt(d)), r(d, f, 1.0 / math.sqrt(d)), r(f, e, 1.0 / math.sqrt(f)), r(n, e, 1e-2)


SIZES = [(1, 1, 1, 1), (1, 64, 172, 64), (1, 1000, 2100, 1000), (2, 33, 65, 17), (3, 5, 4099, 6), (5, 256, 1024, 256), (16, 200, 300, 100), (17, 7, 41, 130), (31, 100, 37, 7),
         (33, 64, 256, 301), (64, 128, 256, 128), (65, 16, 40, 16), (100, 301, 77, 45), (127, 31, 129, 257), (128, 64, 128, 64), (129, 256, 300, 256), (257, 47, 1100, 90),
         (300, 1, 2, 3), (1000, 64, 172, 64), (700, 600, 1030, 128), (4000, 32, 48, 32)]


@pytest.mark.parametrize("form", [B.HT_W_IN_OUT, B.HT_W_OUT_IN])
@pytest.mark.parametrize("n,d,f,e", SIZES)
def test_sizes(ctx, n, d, f, e, form):
    X, Wg, Wu, Wd, dY = _inputs(n, d, f, e)
    ref, tol = reference(X, Wg, Wu, Wd, "silu", dY)
    check(call(ctx, X, Wg, Wu, Wd, dY=dY, form=form), ref, tol)
    check(call(ctx, X, Wg, Wu, Wd, dY=dY, form=form, keep=True, ld_w=3), ref, tol)


@pytest.mark.parametrize("n", [1, 20, 150])
@pytest.mark.parametrize("act", list(ACTS))
def test_activations(ctx, act, n):
    X, Wg, Wu, Wd, dY = _inputs(n, 40, 90, 50, gate=3.0)
    if act == "relu":                        # whole numbers: what is on which side of 0 is the same in any arithmetic
        X, Wg = np.rint(X * 3).astype(np.float32), np.rint(Wg * 20).astype(np.float32)
    ref, tol = reference(X, Wg, Wu, Wd, act, dY)
    if act == "relu":
        assert n == 1 or (ref["gate"] == 0).any()
    check(call(ctx, X, Wg, Wu, Wd, act=act, dY=dY, keep=True), ref, tol)
    check(call(ctx, X, Wg, Wu, Wd, act=act, dY=dY), ref, tol)


@pytest.mark.parametrize("n", [2, 40, 200])
@pytest.mark.parametrize("form", [B.HT_W_IN_OUT, B.HT_W_OUT_IN])
def test_sums_are_added_to_what_is_there(ctx, n, form):
    X, Wg, Wu, Wd, dY = _inputs(n, 70, 130, 66)
    ref, tol = reference(X, Wg, Wu, Wd, "silu", dY)
    check(call(ctx, X, Wg, Wu, Wd, dY=dY, form=form, add=True), ref, tol, add=True)


@pytest.mark.parametrize("n", [1, 50, 300])
def test_outputs_that_are_not_asked_for(ctx, n):
    """Any of them alone: the same bits as all of them together."""
    X, Wg, Wu, Wd, dY = _inputs(n, 60, 100, 80)
    whole = call(ctx, X, Wg, Wu, Wd, dY=dY)
    for only in [("dX",), ("dWg",), ("dWu",), ("dWd",), ("dWg", "dWd"), ("dX", "dWu"), ()]:
        part = call(ctx, X, Wg, Wu, Wd, dY=dY, only=only, fwd=False)
        assert set(part) == set(only)
        for k in only:
            assert np.array_equal(part[k], whole[k]), (only, k)


@pytest.mark.parametrize("n", [4, 64, 65, 1000])
def test_the_same_bits_from_call_to_call(ctx, n):
    X, Wg, Wu, Wd, dY = _inputs(n, 200, 700, 130)
    a, b = (call(ctx, X, Wg, Wu, Wd, dY=dY, keep=True) for _ in range(2))
    for k in a:
        assert np.array_equal(a[k], b[k]), k


@pytest.mark.parametrize("n", [3, 90])
def test_gradients_against_differences(ctx, n):
    """sum(Y R) along random directions, by differences in 64 bits."""
    X, Wg, Wu, Wd, R = _inputs(n, 20, 30, 10)
    for act in ("silu", "gelu", "gelu_tanh", "sigmoid"):
        got = call(ctx, X, Wg, Wu, Wd, act=act, dY=R, fwd=False)
        _, tol = reference(X, Wg, Wu, Wd, act, R)
        rng = np.random.default_rng(5)
        for k, name in enumerate(OUTS):
            args = [t.astype(np.float64) for t in (X, Wg, Wu, Wd)]
            D = rng.standard_normal(args[k].shape)
            h, at = 1e-4, args[k]
            ends = []
            for s in (h, -h):
                args[k] = at + s * D
                v = activation(args[0] @ args[1], act)[0]
                ends.append((((v * (args[0] @ args[2])) @ args[3]) * R).sum())
            want, have = (ends[0] - ends[1]) / (2 * h), (got[name].astype(np.float64) * D).sum()
            # (the third derivative of what is differenced: sums of n f terms of size |R| |Wd|, below 100 each in these ranges)
            room = (tol[name] * np.abs(D)).sum() + h * h * 100 * np.abs(R).sum()
            assert abs(want - have) <= room, (act, name, want, have, room)


@pytest.mark.parametrize("n", [7, 130])
def test_halves_of_one_matrix(ctx, n):
    """Wg and Wu, their gradients, gate and up as the halves of one matrix each."""
    d, f, e = 36, 52, 20
    X, Wg, Wu, Wd, dY = _inputs(n, d, f, e)
    ref, tol = reference(X, Wg, Wu, Wd, "silu", dY)
    W2, dW2, kept = _matrix(np.hstack([Wg, Wu])), torch.full((d, 2 * f), 7.0, device="cuda"), torch.full((n, 2 * f), 7.0, device="cuda")
    Xd, Wdd, Y, dX, dWd = _matrix(X), _matrix(Wd), torch.empty(n, e, device="cuda"), torch.empty(n, d, device="cuda"), torch.empty(f, e, device="cuda")
    halves = lambda t: (t[:, :f], t[:, f:])
    gate, up = halves(kept)
    dWg, dWu = halves(dW2)
    B.ht_ffn_fwd(ctx, d, f, e, Xd, *halves(W2), Wdd, Y, gate=gate, up=up)
    B.ht_ffn_bwd(ctx, d, f, e, Xd, *halves(W2), Wdd, _matrix(dY), dX=dX, dWg=dWg, dWu=dWu, dWd=dWd, gate=gate, up=up)
    B.ht_sync(ctx)
    got = dict(Y=Y, gate=gate, up=up, dX=dX, dWg=dWg, dWu=dWu, dWd=dWd)
    check({k: t.cpu().numpy() for k, t in got.items()}, ref, tol)


@pytest.mark.parametrize("n", [3, 100])
def test_scales_far_apart(ctx, n):
    """Rows, and weights, of very different magnitudes: each output relative to the sizes of its own terms."""
    X, Wg, Wu, Wd, dY = _inputs(n, 48, 80, 40)
    X[::3] *= np.float32(2.0 ** -40)
    X[1::3] *= np.float32(2.0 ** 10)
    Wg *= np.float32(2.0 ** -9)
    Wu *= np.float32(2.0 ** 60)
    Wd *= np.float32(2.0 ** -70)
    dY *= np.float32(2.0 ** 30)
    dY[0] *= np.float32(2.0 ** -90)
    for act in ("silu", "gelu_tanh"):
        ref, tol = reference(X, Wg, Wu, Wd, act, dY)
        check(call(ctx, X, Wg, Wu, Wd, act=act, dY=dY, keep=True), ref, tol)


@pytest.mark.parametrize("n", [5, 140])
def test_zeros(ctx, n):
    X, Wg, Wu, Wd, dY = _inputs(n, 30, 60, 20)
    X[1], dY[2] = 0.0, 0.0
    Wg[:, 7], Wu[:, 8], Wd[9] = 0.0, 0.0, 0.0
    ref, tol = reference(X, Wg, Wu, Wd, "gelu", dY)
    got = call(ctx, X, Wg, Wu, Wd, act="gelu", dY=dY)
    check(got, ref, tol)
    assert (got["Y"][1] == 0).all() and (got["dX"][2] == 0).all()
    got = call(ctx, X, 0 * Wg, 0 * Wu, 0 * Wd, dY=0 * dY)
    for k, t in got.items():
        assert (t == 0).all(), k


@pytest.mark.parametrize("n", [5, 140])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_is_not_finite_stays_where_it_reaches(ctx, n, bad):
    X, Wg, Wu, Wd, dY = _inputs(n, 30, 60, 20)
    ref, tol = reference(X, Wg, Wu, Wd, "silu", dY)
    Xb = X.copy()
    Xb[3, 4] = bad
    got = call(ctx, Xb, Wg, Wu, Wd, dY=dY)
    rest = np.arange(n) != 3
    for k in ("Y", "dX"):
        assert not np.isfinite(got[k][3]).any(), k
        check({k: got[k][rest]}, {k: ref[k][rest]}, {k: tol[k][rest]})
    Wb = Wd.copy()
    Wb[11, 6] = bad                          # reaches column 6 of Y, and in the backward pass the hidden column 11
    got = call(ctx, X, Wg, Wu, Wb, dY=dY)
    assert not np.isfinite(got["Y"][:, 6]).any() and not np.isfinite(got["dX"]).any()
    other = np.arange(20) != 6
    check({"Y": got["Y"][:, other]}, {"Y": ref["Y"][:, other]}, {"Y": tol["Y"][:, other]})
    hid = np.arange(60) != 11
    for k in ("dWg", "dWu"):
        assert not np.isfinite(got[k][:, 11]).any()
        check({k: got[k][:, hid]}, {k: ref[k][:, hid]}, {k: tol[k][:, hid]})
    check({"dWd": got["dWd"]}, ref, tol)


# (few rows, and weights that are most of what there is to read)
STREAMED = [(65, 301, 2_405, 300), (128, 300, 2_400, 300), (130, 513, 1_366, 514), (256, 130, 8_200, 47), (500, 61, 130, 37), (17, 1_001, 5_603, 1_003), (64, 1_024, 5_600, 1_000), (16, 1_001, 5_603, 1_003)]


@pytest.mark.parametrize("form", [B.HT_W_IN_OUT, B.HT_W_OUT_IN])
@pytest.mark.parametrize("n,d,f,e", STREAMED)
def test_weights_that_are_read_once(ctx, n, d, f, e, form):
    X, Wg, Wu, Wd, dY = _inputs(n, d, f, e)
    ref, tol = reference(X, Wg, Wu, Wd, "silu", dY)
    check(call(ctx, X, Wg, Wu, Wd, dY=dY, form=form, ld_w=n % 3), ref, tol)
    check(call(ctx, X, Wg, Wu, Wd, dY=dY, form=form, keep=True, add=True), ref, tol, add=True)


@pytest.mark.parametrize("only", [("dX",), ("dWg",), ("dWd",), ("dWu", "dX")])
def test_some_gradients_of_weights_that_are_read_once(ctx, only):
    X, Wg, Wu, Wd, dY = _inputs(70, 301, 2_405, 300)
    ref, tol = reference(X, Wg, Wu, Wd, "gelu", dY)
    check(call(ctx, X, Wg, Wu, Wd, act="gelu", dY=dY, only=only), ref, tol)


@pytest.mark.parametrize("form", [B.HT_W_IN_OUT, B.HT_W_OUT_IN])
def test_weights_that_grow_along_a_reduction(ctx, form):
    """Each step of a reduction meets a larger value than those before it: what was added up with a smaller scale comes with; zeros before them have no scale at all."""
    X, Wg, Wu, Wd, dY = _inputs(100, 320, 2_240, 320)
    grow = lambda n, top: np.exp2(np.linspace(-top, 0, n)).astype(np.float32)[:, None]
    Wg, Wu = Wg * grow(320, 30), Wu * grow(320, 60)
    Wg[:40] = 0.0
    Wd = Wd * grow(2_240, 50)
    ref, tol = reference(X, Wg, Wu, Wd, "silu", dY)
    check(call(ctx, X, Wg, Wu, Wd, dY=dY, form=form), ref, tol)
    Wd = np.ascontiguousarray(Wd[:, ::-1]) * grow(320, 40).T
    Wg, Wu = (w * np.float32(2.0 ** s) * grow(2_240, 20).T for w, s in ((Wg, -20), (Wu, 40)))      # (dX: two products whose factors are far apart, and whose sums are not)
    ref, tol = reference(X, Wg, Wu, Wd, "silu", dY)
    check(call(ctx, X, Wg, Wu, Wd, dY=dY, form=form, keep=True), ref, tol)
    tiny = [w * np.float32(2.0 ** -110) for w in (Wg, Wu)]
    ref, tol = reference(X, *tiny, Wd, "sigmoid", dY)
    got = call(ctx, X, *tiny, Wd, act="sigmoid", dY=dY, form=form, only=("dWu",))
    check({"dWu": got["dWu"]}, ref, tol)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_is_not_finite_in_weights_that_are_read_once(ctx, bad):
    n, d, f, e = 100, 300, 2_405, 290
    X, Wg, Wu, Wd, dY = _inputs(n, d, f, e)
    ref, tol = reference(X, Wg, Wu, Wd, "silu", dY)
    Wb = Wd.copy()
    Wb[2_401, 289] = bad                     # in the last steps of both reductions
    got = call(ctx, X, Wg, Wu, Wb, dY=dY)
    assert not np.isfinite(got["Y"][:, 289]).any() and not np.isfinite(got["dX"]).any()
    check({"Y": got["Y"][:, :289]}, {"Y": ref["Y"][:, :289]}, {"Y": tol["Y"][:, :289]})
    rest = np.arange(f) != 2_401
    for k in ("dWg", "dWu"):
        assert not np.isfinite(got[k][:, 2_401]).any()
        check({k: got[k][:, rest]}, {k: ref[k][:, rest]}, {k: tol[k][:, rest]})
    check({"dWd": got["dWd"]}, ref, tol)
    Xb = X.copy()
    Xb[77, 299] = bad
    got = call(ctx, Xb, Wg, Wu, Wd, dY=dY)
    rest = np.arange(n) != 77
    for k in ("Y", "dX"):
        assert not np.isfinite(got[k][77]).any(), k
        check({k: got[k][rest]}, {k: ref[k][rest]}, {k: tol[k][rest]})


def test_no_rows(ctx):
    d, f, e = 12, 20, 8
    z = lambda r, c: torch.zeros(r, c, device="cuda")
    W = [torch.randn(d, f, device="cuda"), torch.randn(d, f, device="cuda"), torch.randn(f, e, device="cuda")]
    B.ht_ffn_fwd(ctx, d, f, e, z(0, d), *W, z(0, e))
    for add in (False, True):
        grads = [torch.full_like(w, 3.0) for w in W]
        B.ht_ffn_bwd(ctx, d, f, e, z(0, d), *W, z(0, e), dX=z(0, d), dWg=grads[0], dWu=grads[1], dWd=grads[2], accumulate_dW=add)
        B.ht_sync(ctx)
        for g in grads:
            assert (g == (3.0 if add else 0.0)).all()


def test_refusals(ctx):
    n, d, f, e = 6, 12, 20, 8
    r = lambda a, b: torch.randn(a, b, device="cuda")
    X, Wg, Wu, Wd, Y, gate, up = r(n, d), r(d, f), r(d, f), r(f, e), r(n, e), r(n, f), r(n, f)      # (the binding takes columns from the widths, rows from the tensors)

    def refused(code, text, call):
        with pytest.raises(B.HongtuError) as err:
            call()
        assert err.value.code == code and text in str(err.value), str(err.value)

    EINVAL, ESHAPE = -1, -4
    fwd = lambda **kw: B.ht_ffn_fwd(ctx, kw.pop("d", d), kw.pop("f", f), kw.pop("e", e), kw.pop("X", X), kw.pop("Wg", Wg), kw.pop("Wu", Wu), kw.pop("Wd", Wd),
                                    kw.pop("Y", Y), **kw)
    bwd = lambda **kw: B.ht_ffn_bwd(ctx, d, f, e, X, Wg, Wu, Wd, kw.pop("dY", Y), **kw)
    refused(EINVAL, "activation", lambda: fwd(act=5))
    refused(EINVAL, "activation", lambda: fwd(act=-1))
    refused(EINVAL, "form", lambda: fwd(w_form=2))
    refused(EINVAL, "go together", lambda: fwd(gate=gate))
    refused(EINVAL, "go together", lambda: bwd(up=up))
    refused(ESHAPE, "width 0", lambda: fwd(f=0))
    refused(ESHAPE, "Wg", lambda: fwd(Wg=r(d + 1, f)))
    refused(ESHAPE, "Wd", lambda: fwd(f=f - 1))
    refused(ESHAPE, "Y", lambda: fwd(Y=r(n + 1, e)))
    refused(ESHAPE, "multiple of 4", lambda: fwd(X=r(n, d + 1)))
    refused(ESHAPE, "aligned", lambda: fwd(Y=r(n, e + 4)[:, 1:]))
    refused(EINVAL, "Y shares memory with X", lambda: fwd(d=8, Wg=r(8, f), Wu=r(8, f), X=Y))
    refused(EINVAL, "up shares memory with gate", lambda: fwd(gate=gate, up=gate))
    refused(EINVAL, "Y shares memory with Wd", lambda: fwd(Wd=(w := r(f, e)), Y=w[:n]))
    both = r(n, 2 * f)
    refused(EINVAL, "up shares memory with gate", lambda: fwd(gate=both[:, :f], up=both[:, f - 4:2 * f - 4]))
    refused(EINVAL, "dWu shares memory with dWg", lambda: bwd(dWg=(w := r(d, f)), dWu=w))
    refused(EINVAL, "dX shares memory with X", lambda: bwd(dX=X))
    refused(EINVAL, "dWd shares memory with Wd", lambda: bwd(dWd=Wd))
    refused(ESHAPE, "dWd", lambda: bwd(dWd=r(f - 1, e)))
