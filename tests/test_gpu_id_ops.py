"""The calls of models over ids as a program uses them: together with layers, on streams of its own, recorded and replayed."""
import numpy as np
import pytest
import torch

from oracle import oracle as orc
from paper_2311_14898_amd import binding as B
from paper_2311_14898_amd import inputs
from tests.util import assert_close, assert_close_grad

pytestmark = pytest.mark.gpu


def _softmax_ce(x, y):
    """Mean loss and gradient of the logits, in 64 bits, over rows with y >= 0."""
    has = y >= 0
    m = x.max(axis=1, keepdims=True)
    lse = np.log(np.exp(x - m).sum(axis=1)) + m[:, 0]
    g = np.exp(x - lse[:, None])
    g[np.arange(len(y)), np.where(has, y, 0)] -= 1.0
    return (lse - x[np.arange(len(y)), np.where(has, y, 0)])[has].mean(), np.where(has[:, None], g, 0.0) / has.sum()


def test_a_layer_between_a_table_and_its_transpose():
    """Vertices have items of a table; a layer; every vertex predicts an item.  The table's gradient comes from both of its ends."""
    V, E, items, d = 3000, 30_000, 700, 48
    src, dst = inputs.rmat_edges(V, E, seed=3)
    rng = np.random.default_rng(1)
    T = (rng.standard_normal((items, d)) * 0.3).astype(np.float32)
    W = (rng.standard_normal((d, d)) / np.sqrt(d)).astype(np.float32)
    ids, y = rng.integers(-1, items, V).astype(np.int32), rng.integers(-1, items, V).astype(np.int32)
    scale = 1.5
    # in 64 bits
    indptr, col = orc.csc_build(V, src.numpy(), dst.numpy())
    h0 = np.where((ids >= 0)[:, None], T[np.maximum(ids, 0)].astype(np.float64), 0.0) * scale
    a = orc.aggregate(indptr, col, h0)
    h1 = a @ W.astype(np.float64)
    loss, g = _softmax_ce(h1 @ T.astype(np.float64).T, y)
    dh1, dT = g @ T.astype(np.float64), g.T @ h1
    dW = a.T @ dh1
    da = dh1 @ W.astype(np.float64).T
    # the aggregation's matrix is D^-1/2 (A + I) D^-1/2: its transpose by columns
    deg = np.diff(indptr).astype(np.float64)
    dh0 = np.zeros_like(h0)
    rows = np.repeat(np.arange(V), np.diff(indptr))
    np.add.at(dh0, col, da[rows] / np.sqrt(deg[rows] * deg[col])[:, None])
    np.add.at(dT, ids[ids >= 0], dh0[ids >= 0] * scale)

    ctx = B.ht_ctx_create(0)
    try:
        graph = B.ht_partition(ctx, V, src.cuda(), dst.cuda(), 3)
        Td, Wd = B.to_matrix(torch.from_numpy(T)), torch.from_numpy(W).cuda()
        ids_d, y_d = torch.from_numpy(ids).cuda(), torch.from_numpy(y).cuda()
        H0, A, H1, dH1, dH0 = (B.alloc_matrix(V, d) for _ in range(5))
        dTd, dWd, l = torch.empty_like(Td), torch.empty_like(Wd), torch.zeros(1, device="cuda")
        B.ht_embed_fwd(ctx, d, Td, ids_d, H0, scale=scale)
        B.ht_layer_fwd(ctx, graph, d, d, B.HT_ACT_NONE, H0, Wd, H1, A)
        B.ht_head_loss(ctx, d, items, H1, Td, y_d, l, dH=dH1, dW=dTd, w_form=B.HT_W_OUT_IN)
        B.ht_layer_bwd(ctx, graph, d, d, B.HT_ACT_NONE, A, Wd, dH1, dWd, dH_in=dH0)
        B.ht_embed_bwd(ctx, d, dH0, ids_d, dTd, scale=scale, accumulate=True)
        B.ht_sync(ctx)
        assert abs(float(l) - loss) <= 1e-5 * abs(loss)
        assert_close(H1.cpu().numpy()[:, :d], h1, "h1")
        assert_close_grad(dH1.cpu().numpy()[:, :d], dh1, "dh1")
        assert_close_grad(dWd.cpu().numpy(), dW, "dW")
        assert_close_grad(dTd.cpu().numpy()[:, :d], dT, "dT")
        B.ht_graph_destroy(graph)
    finally:
        B.ht_ctx_destroy(ctx)


def test_a_student_layer_learns_from_a_teacher():
    V, E, d, C, K, temp = 2000, 20_000, 40, 61, 5, 2.0
    src, dst = inputs.rmat_edges(V, E, seed=5)
    rng = np.random.default_rng(2)
    H, W = rng.standard_normal((V, d)).astype(np.float32), (rng.standard_normal((d, C)) / np.sqrt(d)).astype(np.float32)
    ids = np.stack([rng.permutation(C)[:K] for _ in range(V)]).astype(np.int32)
    top = rng.standard_normal((V, K)).astype(np.float32)
    ids[::9] = -1
    indptr, col = orc.csc_build(V, src.numpy(), dst.numpy())
    a = orc.aggregate(indptr, col, H)
    x = a @ W.astype(np.float64)
    has = ids[:, 0] >= 0
    q = np.exp(top / np.float64(temp))
    q /= q.sum(axis=1, keepdims=True)
    z = x / temp
    p = np.exp(z - z.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    at = np.maximum(ids, 0)
    loss = ((q * (np.log(q) - np.log(np.take_along_axis(p, at, axis=1)))).sum(axis=1) * temp * temp)[has].mean()
    g = p.copy()
    np.add.at(g, (np.arange(V)[:, None], at), -q)
    g = np.where(has[:, None], g * temp / has.sum(), 0.0)

    ctx = B.ht_ctx_create(0)
    try:
        graph = B.ht_partition(ctx, V, src.cuda(), dst.cuda(), 2)
        Hd, Wd = B.to_matrix(torch.from_numpy(H)), torch.from_numpy(W).cuda()
        X, A, dW, l = B.alloc_matrix(V, C), B.alloc_matrix(V, d), torch.empty_like(Wd), torch.zeros(1, device="cuda")
        B.ht_layer_fwd(ctx, graph, d, C, B.HT_ACT_NONE, Hd, Wd, X, A)
        B.ht_distill_loss(ctx, C, X, torch.from_numpy(ids).cuda(), torch.from_numpy(top).cuda(), l, temperature=temp, dlogits=X)   # in place
        B.ht_layer_bwd(ctx, graph, d, C, B.HT_ACT_NONE, A, Wd, X, dW)
        B.ht_sync(ctx)
        assert abs(float(l) - loss) <= 1e-5 * abs(loss)
        assert_close_grad(X.cpu().numpy()[:, :C], g, "dlogits")
        assert_close_grad(dW.cpu().numpy(), a.T @ g, "dW")
        B.ht_graph_destroy(graph)
    finally:
        B.ht_ctx_destroy(ctx)


class Work:
    """One call of each kind on a context, its inputs and outputs; sizes by `big`."""

    def __init__(self, ctx, big=1, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.ctx, n, V, d, C, K = ctx, 700 * big, 300 * big, 36, 500 * big, 9
        self.n, self.V, self.d, self.C = n, V, d, C
        self.g = g
        self.table, self.dH0 = torch.randn(V, d, generator=g, device="cuda"), torch.randn(n, d, generator=g, device="cuda")
        self.ids = torch.randint(-1, V, (n,), generator=g, device="cuda", dtype=torch.int32)
        self.y = torch.randint(-1, C, (n,), generator=g, device="cuda", dtype=torch.int32)
        self.W = torch.randn(d, C, generator=g, device="cuda")
        self.few = min(n, 40)                              # rows of the call that scores few of them
        self.X = torch.randn(n, C, generator=g, device="cuda")
        self.top_ids = torch.randint(-1, C, (n, K), generator=g, device="cuda", dtype=torch.int32)
        self.top = torch.randn(n, K, generator=g, device="cuda")
        z = lambda *s: torch.zeros(*s, device="cuda")
        self.H, self.dT, self.dH, self.dW, self.loss, self.rows = z(n, d), z(V, d), z(n, d), z(d, C), z(1), z(n)
        self.dHf, self.dWf, self.lossf, self.dX, self.lossd, self.lossx, self.dX1 = z(self.few, d), z(d, C), z(1), z(n, C), z(1), z(1), z(2, C)
        torch.cuda.synchronize()

    def outputs(self):
        return [self.H, self.dT, self.dH, self.dW, self.loss, self.rows, self.dHf, self.dWf, self.lossf, self.dX, self.lossd, self.lossx, self.dX1]

    def run(self, sync=False):
        c, d, C, f = self.ctx, self.d, self.C, self.few
        B.ht_embed_fwd(c, d, self.table, self.ids, self.H, scale=2.0, sync=sync)
        B.ht_embed_bwd(c, d, self.dH0, self.ids, self.dT, scale=2.0, sync=sync)
        B.ht_head_loss(c, d, C, self.H, self.W, self.y, self.loss, row_loss=self.rows, dH=self.dH, dW=self.dW, sync=sync)
        B.ht_head_loss(c, d, C, self.H[:f], self.W, self.y[:f], self.lossf, dH=self.dHf, dW=self.dWf, sync=sync)
        B.ht_distill_loss(c, C, self.X, self.top_ids, self.top, self.lossd, dlogits=self.dX, sync=sync)
        B.ht_distill_loss(c, C, self.X[:2], self.top_ids[:2], self.top[:2], self.lossx, dlogits=self.dX1, sync=sync)

    def renew(self, seed):
        """Other values in the same places."""
        self.g.manual_seed(seed)
        for t in (self.table, self.dH0, self.W, self.X, self.top):
            t.copy_(torch.randn(t.shape, generator=self.g, device="cuda"))
        self.ids.copy_(torch.randint(-1, self.V, (self.n,), generator=self.g, device="cuda", dtype=torch.int32))
        for t in (self.y, self.top_ids):
            t.copy_(torch.randint(-1, self.C, t.shape, generator=self.g, device="cuda", dtype=torch.int32))

    def eager(self):
        """Results of an unrecorded pass on a context of its own."""
        other = Work.__new__(Work)
        other.__dict__.update(self.__dict__)
        other.__dict__.update({k: torch.zeros_like(v) for k, v in self.__dict__.items()
                               if k in ("H", "dT", "dH", "dW", "loss", "rows", "dHf", "dWf", "lossf", "dX", "lossd", "lossx", "dX1")})
        other.ctx = B.ht_ctx_create(0)
        torch.cuda.synchronize()
        other.run(sync=True)
        B.ht_sync(other.ctx)
        B.ht_ctx_destroy(other.ctx)
        return other.outputs()


@pytest.mark.parametrize("big", [1, 40])                   # lists put in order by counting and by sorting
def test_recorded_and_replayed(big):
    s = torch.cuda.Stream()
    ctx = B.ht_ctx_create(0, s.cuda_stream)
    try:
        w = Work(ctx, big)
        w.run()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            w.run()
        for k in range(4):
            w.renew(100 + k)
            want = w.eager()                               # the program's own work and synchronizations between the replays
            for o in w.outputs():
                o.fill_(float(k))
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                graph.replay()
            s.synchronize()
            for a, b in zip(w.outputs(), want):
                assert torch.equal(a, b)
        # a larger call outgrows the scratch memory; the graph keeps what it works in
        Work(ctx, big * 3, seed=9).run()
        s.synchronize()
        hog = torch.full((64 << 20,), float("nan"), device="cuda")        # (whoever gets memory that was given back writes into it)
        w.renew(200)
        want = w.eager()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            graph.replay()
        s.synchronize()
        for a, b in zip(w.outputs(), want):
            assert torch.equal(a, b)
        assert bool(torch.isnan(hog).all())
        del graph
    finally:
        B.ht_ctx_destroy(ctx)


def test_a_recorded_first_call_is_refused():
    """Nothing can be allocated while a stream is recorded: the call says so, and the recording goes on."""
    s = torch.cuda.Stream()
    ctx = B.ht_ctx_create(0, s.cuda_stream)
    try:
        w = Work(ctx)
        x = torch.zeros(8, device="cuda")
        many, many_ids = w.dH0.repeat(9, 1), w.ids.repeat(9)
        codes = []
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            x.add_(1.0)
            for call in (lambda: B.ht_embed_bwd(ctx, w.d, w.dH0, w.ids, w.dT, sync=False),
                         lambda: B.ht_head_loss(ctx, w.d, w.C, w.H, w.W, w.y, w.loss, sync=False),
                         lambda: B.ht_head_loss(ctx, w.d, w.C, w.H[:3], w.W, w.y[:3], w.loss, sync=False),
                         lambda: B.ht_distill_loss(ctx, w.C, w.X, w.top_ids, w.top, w.lossd, sync=False),
                         lambda: B.ht_embed_bwd(ctx, w.d, many, many_ids, w.dT, sync=False)):
                try:
                    call()
                    codes.append(0)
                except B.HongtuError as e:
                    codes.append(e.code)
            B.ht_embed_fwd(ctx, w.d, w.table, w.ids, w.H, sync=False)     # (needs no scratch memory)
        assert codes == [0] + [B.HT_ESTATE] * 4            # (the gradient of few entries needs no scratch memory either)
        with torch.cuda.stream(s):
            graph.replay()
            graph.replay()
        s.synchronize()
        assert float(x[0]) == 2.0
        keep = w.ids >= 0
        assert torch.equal(w.H[keep], w.table[w.ids[keep].long()])
        w.run()                                            # and the context works on
        s.synchronize()
        for a, b in zip(w.outputs(), w.eager()):
            assert torch.equal(a, b)
        del graph
    finally:
        B.ht_ctx_destroy(ctx)


def test_two_contexts_at_once():
    """Two streams, a context each, calls of both under way together."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    ctxs = [B.ht_ctx_create(0, s.cuda_stream) for s in streams]
    try:
        work = [Work(c, big=1 + 10 * i, seed=i) for i, c in enumerate(ctxs)]
        want = [w.eager() for w in work]
        for _ in range(5):
            for w in work:
                w.run()
        torch.cuda.synchronize()
        for w, e in zip(work, want):
            for a, b in zip(w.outputs(), e):
                assert torch.equal(a, b)
    finally:
        for c in ctxs:
            B.ht_ctx_destroy(c)


def test_results_wait_for_the_context_only():
    """A context of its own stream; inputs made on another, the binding's synchronization between them."""
    ctx = B.ht_ctx_create(0)
    try:
        s = torch.cuda.Stream()
        w = Work(ctx, 5)
        with torch.cuda.stream(s):
            w.renew(7)
        w.run(sync=True)
        B.ht_sync(ctx)
        for a, b in zip(w.outputs(), w.eager()):
            assert torch.equal(a, b)
    finally:
        B.ht_ctx_destroy(ctx)


def test_refused_memory_is_said_and_gone_again():
    """A byte budget too small for a call is an error, and with a larger one the same context goes on."""
    ctx = B.ht_ctx_create(0)
    try:
        B.ht_ctx_set_hbm_budget(ctx, 4096)
        w = Work(ctx)
        many, many_ids = w.dH0.repeat(9, 1), w.ids.repeat(9)      # (the gradient of few entries needs no scratch memory)
        for call in (lambda: B.ht_embed_bwd(ctx, w.d, many, many_ids, w.dT), lambda: B.ht_head_loss(ctx, w.d, w.C, w.H, w.W, w.y, w.loss),
                     lambda: B.ht_head_loss(ctx, w.d, w.C, w.H[:3], w.W, w.y[:3], w.loss), lambda: B.ht_distill_loss(ctx, w.C, w.X, w.top_ids, w.top, w.lossd)):
            with pytest.raises(B.HongtuError) as err:
                call()
            assert err.value.code == B.HT_ENOMEM
        B.ht_ctx_set_hbm_budget(ctx, 1 << 30)
        w.run(sync=True)
        B.ht_sync(ctx)
        for a, b in zip(w.outputs(), w.eager()):
            assert torch.equal(a, b)
    finally:
        B.ht_ctx_destroy(ctx)
