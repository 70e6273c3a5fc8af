"""Captured calls of a worker and what happens to the handle afterwards (needs a GPU)."""
import pytest
import torch

from paper_2205_11048_gb300 import binding as B
from tests.test_gpu_worker import gen, rand, tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("n,more", [(300, 9000), (9000, 40_000)])
def test_a_graph_outlives_the_growth_of_the_workspace(n, more):
    """A batch captured, a larger one run (and memory of the old workspace's size used by others),
    the first replayed: the same bits as from direct calls."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        w = B.Worker()
        g = gen(n)
        V, d = 900, 72
        ids, G = tokens(g, n, V, "skew", 0.1), rand(g, n, d)
        x, gamma = rand(g, n, d), rand(g, d)

        def step(ids, G, x):
            _, mean, rstd = w.layer_norm(x, gamma)
            dx, dgamma, dbeta = w.layer_norm_grad(G, x, gamma, mean, rstd)
            i, r, c = w.embed_grad(ids, dx, V, pad_id=-1)
            dense = w.embed_grad_dense(ids, dx, torch.empty(V, d, device="cuda"), pad_id=-1)
            norm = w.clip_grads([r, dgamma, dbeta], 0.5)
            return i, r, c, dense, dgamma, dbeta, norm

        step(ids, G, x)
        w.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = step(ids, G, x)
        step(tokens(g, more, V, "skew", 0.1), rand(g, more, d), rand(g, more, d))
        w.sync()
        others = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(64)]
        for seed in (1, 2):
            ids.copy_(tokens(gen(seed), n, V, "skew", 0.1))
            G.copy_(rand(gen(seed), n, d))
            graph.replay()
            got = [t.clone() for t in out]
            for a, b in zip(got, step(ids, G, x)):
                assert torch.equal(a, b)
        assert all(bool(t.isnan().all()) for t in others)
        w.sync()
        del graph
    w.close()


@pytest.mark.parametrize("dim", [20, 33])
def test_a_captured_lookup_follows_a_hash_table_that_grows(dim):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        w = B.Worker()
        srv = B.GBA([(64, dim, B.HASH, 4096, B.opt_desc(B.ADAGRAD, 0.05))], 0, None, 1, 4, seed=11)
        none = torch.empty(0, device="cuda")
        ids = torch.arange(3000, device="cuda") * 7_777_777_777 - 2**40
        asked = torch.cat([ids[::7], ids[:1] + 1])
        first = ids[:20].clone()
        srv.push(0, [first], [torch.ones(20, dim, device="cuda")], none, 1)
        assert srv.try_apply() == 1
        w.embed_table(srv, 0, asked, scale=3.0)
        srv.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            y = w.embed_table(srv, 0, asked, scale=3.0)
        for step in (1, 2):
            srv.push(step, [ids], [torch.ones(3000, dim, device="cuda")], none, 1)
            assert srv.try_apply() == 1
            graph.replay()
            got = y.clone()
            assert torch.equal(got, w.embed_table(srv, 0, asked, scale=3.0))
            assert torch.equal(got, (srv.pull(0, asked).double() * 3.0).float())
        w.sync()
        srv.sync()
        del graph
        srv.close()
    w.close()
