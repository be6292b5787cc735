"""Scratch memory of a context that has recorded something: what the recorded calls work in stays, and nothing else."""
import pytest
import torch

from paper_2311_14898_amd import binding as B
from paper_2311_14898_amd import inputs

pytestmark = pytest.mark.gpu


def _many_entries(ctx, n):
    """A call that leaves some 18 n bytes of scratch memory."""
    dH, ids, dT = torch.ones(n, 4, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(9, 4, device="cuda")
    torch.cuda.synchronize()
    return lambda: B.ht_embed_bwd(ctx, 4, dH, ids, dT, sync=False), dT


@pytest.mark.parametrize("recorded", [False, True])
def test_memory_that_no_replay_needs_comes_back(recorded):
    """1.4 GB of scratch memory under a budget of 1.6: a partition that needs more than the rest gets it, also where the context has begun a call while it was
    recorded (and refused it), or has recorded one that works in another block."""
    s = torch.cuda.Stream()
    ctx = B.ht_ctx_create(0, s.cuda_stream)
    try:
        x, loss = torch.zeros(8, device="cuda"), torch.zeros(1, device="cuda")
        X, top, ids = torch.randn(90, 64, device="cuda"), torch.randn(90, 3, device="cuda"), torch.zeros(90, 3, dtype=torch.int32, device="cuda")
        run = lambda: B.ht_distill_loss(ctx, 64, X, ids, top, loss, sync=False)
        torch.cuda.synchronize()
        if recorded:
            run()
            s.synchronize()
        want = loss.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            x.add_(1.0)
            try:
                run()
                assert recorded
            except B.HongtuError as e:
                assert e.code == B.HT_ESTATE and not recorded
        many, dT = _many_entries(ctx, 80_000_000)
        many()
        s.synchronize()
        assert float(dT[0, 0]) > 1e7
        B.ht_ctx_set_hbm_budget(ctx, 1600 << 20)
        src, dst = inputs.rmat_edges(1_000_000, 20_000_000, seed=1)
        g = B.ht_partition(ctx, 1_000_000, src.cuda(), dst.cuda(), 2)
        B.ht_graph_destroy(g)
        for k in range(3):
            if recorded:
                loss.fill_(7.0)
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                graph.replay()
            s.synchronize()
            assert float(x[0]) == k + 1 and torch.equal(loss, want)
        del graph
    finally:
        B.ht_ctx_destroy(ctx)


def test_what_replays_work_in_stays_when_memory_is_given_back():
    """A partition that makes the context give back what it can, between two replays of a call in scratch memory."""
    s = torch.cuda.Stream()
    ctx = B.ht_ctx_create(0, s.cuda_stream)
    try:
        run, dT = _many_entries(ctx, 2_000_000)
        run()
        s.synchronize()
        want = dT.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            run()
        B.ht_ctx_set_hbm_budget(ctx, 64 << 20)
        src, dst = inputs.rmat_edges(500_000, 10_000_000, seed=1)
        with pytest.raises(B.HongtuError) as err:
            B.ht_partition(ctx, 500_000, src.cuda(), dst.cuda(), 2)
        assert err.value.code == B.HT_ENOMEM
        hog = torch.full((64 << 20,), float("nan"), device="cuda")        # (whoever gets memory that was given back writes into it)
        for _ in range(3):
            dT.fill_(7.0)
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                graph.replay()
            s.synchronize()
            assert torch.equal(dT, want)
        assert bool(torch.isnan(hog).all())
        run()
        s.synchronize()
        assert torch.equal(dT, want)
        del graph
    finally:
        B.ht_ctx_destroy(ctx)


@pytest.mark.parametrize("n,V", [(262_144, 5000), (262_145, 131_072), (3_000_001, 70_000)])
def test_long_sorts_recorded_and_replayed(n, V):
    """Beyond 262,144 entries the sort scans its counts in memory of its own; other ids in the same place before each replay."""
    s = torch.cuda.Stream()
    ctx = B.ht_ctx_create(0, s.cuda_stream)
    other = B.ht_ctx_create(0)
    try:
        g = torch.Generator(device="cuda")
        g.manual_seed(n)
        dH, ids = torch.randn(n, 8, generator=g, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
        dT, want = torch.zeros(V, 8, device="cuda"), torch.zeros(V, 8, device="cuda")

        def renew():
            ids.copy_(torch.randint(-1, V, (n,), generator=g, device="cuda", dtype=torch.int32))
            ids[: n // 3] = V // 2
            B.ht_embed_bwd(other, 8, dH, ids, want)
            B.ht_sync(other)
            dT.fill_(7.0)
            torch.cuda.synchronize()

        renew()
        B.ht_embed_bwd(ctx, 8, dH, ids, dT, sync=False)
        s.synchronize()
        assert torch.equal(dT, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            B.ht_embed_bwd(ctx, 8, dH, ids, dT, sync=False)
        for _ in range(4):
            renew()
            with torch.cuda.stream(s):
                graph.replay()
            s.synchronize()
            assert torch.equal(dT, want)
        src, dst = inputs.rmat_edges(50_000, 1_000_000, seed=2)          # (a partition sorts in the same memory)
        B.ht_graph_destroy(B.ht_partition(ctx, 50_000, src.cuda(), dst.cuda(), 2))
        renew()
        with torch.cuda.stream(s):
            graph.replay()
        s.synchronize()
        assert torch.equal(dT, want)
        del graph
    finally:
        B.ht_ctx_destroy(ctx)
        B.ht_ctx_destroy(other)
