"""Trees where their kernels change course: step, run and row-tile borders, lengths the host does not know yet, vocabularies and batches around the
sizes at which a call takes another form."""
import numpy as np
import pytest
import torch

import test_gpu_accept_tree as accept
import test_gpu_evict as evict
from paper_2506_09397_amd import sled
from test_gpu_tree_attention import HEADS, Batch
from tree_common import attention_bounds, generator, pool

pytestmark = pytest.mark.gpu

# a step is 32 (float32: 16) tokens, a turn up to four steps, a round of turns 128 (64) tokens
BORDERS = [0, 1, 15, 16, 17, 31, 33, 48, 63, 64, 65, 80, 95, 96, 97, 127, 128, 129, 143, 160, 191, 192, 255, 256, 257, 384, 385, 511, 513]


@pytest.mark.parametrize("heads,nodes", [("8b", 3), ("8b", 14), ("8b", 30), ("8b", 64), ("70b", 5), ("g1", 33), ("f32_64", 5), ("f32_64", 40), ("f32_64", 64),
                                         ("f32_128", 9)])
def test_lengths_around_every_border(heads, nodes):
    with pool(*HEADS[heads], n_pages=600, max_requests=32) as p:
        b = Batch(p, BORDERS, [nodes] * len(BORDERS), seed=41)
        b.run()
        b.check()


def mass_of(b, i, l=0):
    """(exact mass of request i's tokens and nodes [Hkv, L + n], how far a result may lie from it)."""
    (out, lse, w, big, vmax), at = b.plain(i, l)
    s = b.p.shape
    n, hq, t = w.shape
    m = w.reshape(n, s.n_kv_heads, hq // s.n_kv_heads, t).sum(dim=(0, 2))
    # a weight as in the attention, against a lse that is itself off by as much; each of the n G additions by half a step of the sum
    score = (s.head_dim + 8) * 2.0**-24 * big + 2.0**-20 + 2.0**-22 * lse.abs()
    off = (w * (3.0 * score)[:, :, None]).reshape(n, s.n_kv_heads, hq // s.n_kv_heads, t).sum(dim=(0, 2)) + n * (hq // s.n_kv_heads) * 2.0**-24 * m
    return m, off + 1e-30


@pytest.mark.parametrize("heads", ["70b", "8b", "f32_128"])
def test_every_number_of_row_tiles(heads):
    """Groups of two, four and eight tiles in one batch, several groups for one request; the mass of the same rows."""
    nodes = [1, 2, 3, 4, 5, 7, 8, 9, 12, 16, 17, 18, 20, 24, 25, 32, 33, 34, 40, 48, 49, 63, 64]
    ctx = [170 + 13 * i for i in range(len(nodes))]
    with pool(*HEADS[heads], n_pages=800, max_requests=32) as p:
        b = Batch(p, ctx, nodes, seed=42)
        b.run()
        b.check()
        mass = torch.zeros(32, 1, p.shape.n_kv_heads, 600, device="cuda")
        sled.sled_tree_mass(p.pool, 0, b.q[0], b.lse[0], mass, b.ws)
        torch.cuda.synchronize()
        for i, (L, n) in enumerate(zip(ctx, nodes)):
            m, off = mass_of(b, i)
            got = mass[b.reqs[i], 0].double()
            err = (got[:, :L + n] - m).abs()
            assert bool((err <= off).all()), f"request {i} ({n} nodes): {float((err / off).max())} of what is allowed"
            assert bool((got[:, L + n:] == 0).all())


def test_contexts_longer_than_a_work_item_holds():
    """So many heads that nothing is split for balance, and more than 1024 pages each."""
    n, L = 97, 16500
    with pool(*HEADS["8b"], n_pages=n * ((L + 15) // 16 + 1), max_requests=n) as p:
        b = Batch(p, [L] * n, [1] * n, seed=43)
        b.run()
        for i in (0, 50, 96):
            (out, lse, _, big, vmax), at = b.plain(i)
            tol, tol_lse = attention_bounds(out, lse, big, vmax, 128, True)
            assert bool(((b.out[0, at].double() - out).abs() <= tol).all()) and bool(((b.lse[0, at].double() - lse).abs() <= tol_lse).all())


@pytest.mark.parametrize("invariant", [True, False])
def test_the_workspace_asked_for_holds_one_large_tree_on_all_the_context(invariant):
    """Several row groups on a long context, beside requests of one node: more items than an even share of groups would make."""
    ctx, nodes = [31000] + [5] * 15, [64] + [1] * 15
    with pool(*HEADS["70b"], n_pages=2000, invariant=invariant) as p:
        b = Batch(p, ctx, nodes, seed=46)
        b.run()
        (out, lse, _, big, vmax), at = b.plain(0)
        tol, tol_lse = attention_bounds(out, lse, big, vmax, 128, True)
        assert bool(((b.out[0, at].double() - out).abs() <= tol).all()) and bool(((b.lse[0, at].double() - lse).abs() <= tol_lse).all())


@pytest.mark.parametrize("heads", ["8b", "f32_64"])
def test_lengths_that_the_host_does_not_know_yet(heads):
    """Trees begun right behind a commit: the host's bound counts every node as accepted, the length only those that were."""
    ctx, nodes, accepted = [0, 10, 31, 100, 200, 515], [64, 64, 33, 64, 5, 64], [0, 63, 1, 0, 4, 2]
    with pool(*HEADS[heads], n_pages=200) as p:
        b = Batch(p, ctx, nodes, seed=44, kind="chain")
        b.run()
        path = torch.full((len(ctx), sled.TREE_MAX), -1, dtype=torch.int32)
        for i, a in enumerate(accepted):
            path[i, :a] = torch.arange(1, a + 1)
        at = 0
        for i, (n, a) in enumerate(zip(nodes, accepted)):
            b.K[i] = torch.cat([b.K[i], b.k[:, at:at + a + 1]], dim=1)
            b.V[i] = torch.cat([b.V[i], b.v[:, at:at + a + 1]], dim=1)
            at += n
        lens, path = torch.tensor(accepted, dtype=torch.int32).cuda(), path.cuda()
        b.ws = p.workspace(len(ctx), sum(nodes), sum(ctx) + 2 * sum(nodes) + 16 * len(ctx))
        g = generator(45)
        q, k, v = (torch.randn(x.shape, generator=g, device="cuda").to(x.dtype) for x in (b.q, b.k, b.v))
        torch.cuda.synchronize()
        sled.sled_tree_commit(p.pool, b.reqs, lens, path)
        b.q, b.k, b.v = q, k, v
        b.run()   # begins before the commit's lengths have been read back
        b.ctx = [L + a + 1 for L, a in zip(ctx, accepted)]
        b.check()


VOCABS = [2, 3, 4, 5, 7, 255, 4095, 4096, 4097, 16385, 65535, 65536, 65537, 131073]


@pytest.mark.parametrize("mode", [sled.GREEDY, sled.SAMPLE], ids=["greedy", "sample"])
@pytest.mark.parametrize("vocab", VOCABS)
def test_vocabularies_around_a_threads_share(mode, vocab):
    trees = [accept.random_tree(np.random.default_rng(vocab + i), n) for i, n in enumerate([1, 9, 30])]
    logits, tokens, u = accept.case(trees, vocab, seed=vocab)
    accept.check(mode, trees, logits, tokens, u, temperature=0.8)
    # the largest logit in the last place, and nothing but it
    logits[:, -1] = 30.0
    accept.check(mode, trees, logits, tokens, u)
    logits[:, :-1] = -float("inf")
    _, _, o = accept.run(mode, trees, logits, tokens, u)
    assert o.tolist() == [vocab - 1] * 3


@pytest.mark.parametrize("mode", [sled.GREEDY, sled.SAMPLE], ids=["greedy", "sample"])
@pytest.mark.parametrize("sizes", [[4] * 64, [4] * 63 + [5], [1] * 65, [16] * 64, [16] * 64 + [1], [32] * 48, [32] * 48 + [1], [16] * 128, [16] * 128 + [1], [64] * 64 + [3]],
                         ids=lambda s: f"{len(s)}x{sum(s)}")
def test_batches_around_the_sizes_that_travel_with_a_launch(mode, sizes):
    trees = [accept.random_tree(np.random.default_rng(i), n) for i, n in enumerate(sizes)]
    logits, tokens, u = accept.case(trees, 300, seed=len(sizes))
    accept.check(mode, trees, logits, tokens, u, temperature=1.25)


@pytest.mark.parametrize("hq,D,dtype", [(32, 128, "bf16"), (16, 64, "f32")])
def test_all_query_heads_on_one_kv_head(hq, D, dtype):
    with pool(hq, 1, D, dtype, n_pages=200) as p:
        b = Batch(p, [0, 77, 1000, 18], [1, 64, 9, 33], seed=47)
        b.run()
        b.check()
        mass = torch.zeros(16, 1, 1, 1100, device="cuda")
        sled.sled_tree_mass(p.pool, 0, b.q[0], b.lse[0], mass, b.ws)
        torch.cuda.synchronize()
        for i, (L, n) in enumerate(zip(b.ctx, b.n)):
            m, off = mass_of(b, i)
            assert bool(((mass[b.reqs[i], 0, :, :L + n].double() - m).abs() <= off).all())


def test_two_pools_at_once():
    """Attention, mass and acceptance of two pools on two streams, nothing waiting for anything: the same bits as one after the other."""
    with pool(32, 8, 128, "bf16", layers=2, n_pages=600) as p0, pool(8, 2, 128, "f32", layers=2, n_pages=600) as p1:
        batches = [Batch(p0, [900, 33, 2000], [40, 64, 7], seed=48, layers=2), Batch(p1, [1500, 0, 260], [9, 30, 64], seed=49, layers=2)]
        walks = []
        for k, vocab in enumerate((50000, 3001)):
            trees = batches[k].trees
            logits, tokens, u = accept.case(trees, vocab, seed=50 + k)
            B, T = len(trees), sum(batches[k].n)
            walks.append((trees, vocab, logits, tokens, u, sled.workspace(sled.sled_accept_tree_workspace_bytes(B, T, vocab)),
                          *(torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2)), torch.zeros(B, sled.TREE_MAX, dtype=torch.int32, device="cuda")))
        mass = [torch.zeros(16, 2, b.p.shape.n_kv_heads, 2100, device="cuda") for b in batches]

        def step(k):
            b, (trees, vocab, logits, tokens, u, ws, a, o, path) = batches[k], walks[k]
            sled.sled_tree_begin(b.p.pool, b.reqs, b.n, b.trees, b.ws)
            for l in range(2):
                sled.sled_tree_attention(b.p.pool, l, b.q[l], b.k[l], b.v[l], b.out[l], b.lse[l], b.ws)
                sled.sled_tree_mass(b.p.pool, l, b.q[l], b.lse[l], mass[k], b.ws)
            sled.sled_accept_tree(sled.SAMPLE if k else sled.GREEDY, b.n, trees, vocab, 0.9, logits, tokens, u, a, path, o, ws)

        def results(k):
            return [x.clone() for x in (batches[k].out, batches[k].lse, mass[k], *walks[k][6:])]

        for k in range(2):
            step(k)
        torch.cuda.synchronize()
        want = [results(k) for k in range(2)]
        streams = [torch.cuda.Stream() for _ in range(2)]
        for _ in range(4):
            for k in range(2):
                batches[k].out.zero_(), batches[k].lse.zero_(), mass[k].zero_(), walks[k][8].zero_()
            torch.cuda.synchronize()
            for k in range(2):
                with torch.cuda.stream(streams[k]):
                    step(k)
            torch.cuda.synchronize()
            for k in range(2):
                assert all(torch.equal(x, y) for x, y in zip(results(k), want[k]))


@pytest.mark.parametrize("fork", [False, True], ids=["in_place", "fork"])
@pytest.mark.parametrize("kind", ["random", "ties"])
def test_evictions_around_what_a_workgroup_holds(kind, fork):
    """Up to 8192 masses stay in registers while the kept ones are chosen; nothing to choose between the first and the last."""
    with pool(2, 2, 128, "bf16", n_pages=4500) as p:
        evict.check_eviction(p, [8191, 8192, 8193, 9000], [4000, 8191, 200, 8999], 5, 100, kind, fork, seed=51)
    with pool(2, 2, 128, "bf16", n_pages=2500) as p:
        evict.check_eviction(p, [8192, 8195, 600], [300, 300, 300], 100, 200, kind, fork, seed=52)
