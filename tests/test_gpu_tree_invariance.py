"""Batch-invariant pools: the bits of a tree's attention do not depend on how closely the host knows the context's length."""
import numpy as np
import pytest
import torch

from paper_2506_09397_amd import sled
from tree_common import attention_bounds, generator, plain_attention, pool, random_tree

pytestmark = pytest.mark.gpu

HEADS = {"8b": (32, 8, 128, "bf16"), "70b": (64, 8, 128, "bf16"), "f32_64": (4, 4, 64, "f32")}


def busy(ms=60):
    """Work in front of what follows on the stream, so that a commit's lengths are not back when the next call looks for them."""
    x = torch.randn(4096, 4096, device="cuda")
    for _ in range(int(ms)):
        x = torch.mm(x, x) * 1e-2
    return x


# a chain of 64 nodes on `ctx` tokens, so many accepted: the bound is ctx + 64, the length ctx + accepted + 1.  Contexts are summed in runs of 768 tokens.
@pytest.mark.parametrize("ctx,accepted", [(720, 39), (720, 0), (704, 63), (704, 62), (1500, 20), (1500, 35), (0, 0), (0, 12), (768, 0), (2290, 3)])
@pytest.mark.parametrize("heads,nodes", [("8b", 5), ("8b", 64), ("70b", 40), ("f32_64", 9)])
def test_same_bits_before_and_after_the_lengths_have_arrived(heads, nodes, ctx, accepted):
    with pool(*HEADS[heads], n_pages=600, invariant=True) as p:
        s, g = p.shape, generator(ctx + accepted)
        r, K, V = p.open(ctx, g)
        rnd = lambda n, h: torch.randn(n, h, s.head_dim, generator=g, device="cuda").to(p.dt)
        q, k, v = rnd(64, s.n_q_heads), rnd(64, s.n_kv_heads), rnd(64, s.n_kv_heads)
        out, lse = torch.empty_like(q), torch.empty(64, s.n_q_heads, device="cuda")
        ws = p.workspace(1, 64, ctx + 200)
        sled.sled_tree_begin(p.pool, [r], [64], [random_tree(None, 64, "chain")], ws)
        sled.sled_tree_attention(p.pool, 0, q, k, v, out, lse, ws)
        path = torch.full((1, sled.TREE_MAX), -1, dtype=torch.int32)
        path[0, :accepted] = torch.arange(1, accepted + 1)
        path, length = path.cuda(), torch.tensor([accepted], dtype=torch.int32, device="cuda")
        tree = random_tree(np.random.default_rng(nodes), nodes)
        q2, k2, v2 = rnd(nodes, s.n_q_heads), rnd(nodes, s.n_kv_heads), rnd(nodes, s.n_kv_heads)

        def attend():
            o, l = torch.full_like(q2, 7.0), torch.full((nodes, s.n_q_heads), 7.0, device="cuda")
            sled.sled_tree_begin(p.pool, [r], [nodes], [tree], ws)
            sled.sled_tree_attention(p.pool, 0, q2, k2, v2, o, l, ws)
            return o, l

        torch.cuda.synchronize()
        keep = busy()
        sled.sled_tree_commit(p.pool, [r], length, path)
        loose = attend()
        assert sled.sled_kvpool_lengths(p.pool, [r]) == [ctx + accepted + 1]
        exact = attend()
        torch.cuda.synchronize()
        assert torch.equal(loose[0], exact[0]) and torch.equal(loose[1], exact[1])
        a = accepted + 1
        o, l, _, big, vmax = plain_attention(q2, torch.cat([K[0], k[:a]]), torch.cat([V[0], v[:a]]), k2, v2, tree)
        tol, tol_lse = attention_bounds(o, l, big, vmax, s.head_dim, s.dtype == "bf16")
        assert bool(((exact[0].double() - o).abs() <= tol).all()) and bool(((exact[1].double() - l).abs() <= tol_lse).all())
        del keep
