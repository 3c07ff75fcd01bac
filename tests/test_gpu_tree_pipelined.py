"""Rounds over trees that nothing waits for: steps, acceptance, commits and evictions issued one behind the other, while the host knows lengths only by
their bounds; and plans of more requests than a launch takes by value."""
import numpy as np
import pytest
import torch

import test_gpu_evict as evict
from paper_2506_09397_amd import sled, synth
from paper_2506_09397_amd.runtime import Verifier
from test_gpu_tree_invariance import busy
from tree_common import generator, plain_attention, pool, random_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["tiny", "tiny_bf16"])
@pytest.mark.parametrize("with_mass", [False, True], ids=["plain", "mass"])
def test_pipelined_rounds_give_the_same_bits_as_rounds_that_are_waited_for(kind, with_mass):
    """A batch-invariant model, contexts around a border of its runs of 768 tokens: logits, paths, caches and mass."""
    shape, rounds, nodes = synth.SHAPES[kind], 6, [40, 9, 64]
    w = synth.SynthWeights(shape, seed=3, device="cuda", gain_jitter=0.1, std=0.08)
    ctx = [700, 5, 1490]
    results = []
    for wait in (True, False):
        v = Verifier(shape, w, 400, 3, 3, 4000, batch_invariant=True)
        v.enable_trees(64, 4000, mass_cap=2600 if with_mass else 0)
        reqs = [v.open_bounded() if with_mass else v.open() for _ in ctx]
        KV = [synth.context_kv(shape, L, seed=2, req=i, device="cuda") for i, L in enumerate(ctx)]
        v.append_context(reqs, [a for a, _ in KV], [b for _, b in KV])
        rng = np.random.default_rng(1)
        # everything that comes from the host is there before the first round (a copy from it would wait for the stream)
        plan = [[random_tree(rng, n) for n in nodes] for _ in range(rounds)]
        tokens = torch.from_numpy(rng.integers(0, 6, size=(rounds, sum(nodes))).astype(np.int32)).cuda()      # few tokens, so that ...
        at = torch.tensor([0, nodes[0], nodes[0] + nodes[1]], device="cuda")
        pend, out = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda"), []
        v.lengths(reqs)
        keep = busy(100)
        for trees, tok in zip(plan, tokens):
            tok[at] = pend
            logits = v.verify_tree(reqs, trees, tok).clone()
            logits[:, 6:] = -1e4                                                                              # ... walks go on for a while
            a, path, t = v.accept_tree(sled.GREEDY, trees, logits, tok)
            v.commit_tree(reqs, a, path)
            pend = t.clone()
            out += [logits, a.clone(), path.clone(), pend]
            if wait:
                v.lengths(reqs)
        lens = v.lengths(reqs)
        out.append(torch.tensor(lens))
        for r, L in zip(reqs, lens):
            out += list(v.read_kv(r, 0, L))
            if with_mass:
                out.append(v.mass[r].clone())
                assert bool((v.mass[r, :, :, L:] == 0).all())
        results.append(out)
        assert sum(int(x.sum()) for x in out[1::4][:rounds]) >= 2      # something was accepted
        v.destroy()
        del keep
    assert len(results[0]) == len(results[1])
    for x, y in zip(*results):
        assert torch.equal(x, y)


@pytest.mark.parametrize("fork", [False, True], ids=["in_place", "fork"])
@pytest.mark.parametrize("keep", [10, 101, 120, 163, 200])
def test_evictions_behind_a_commit_whose_lengths_are_not_known(keep, fork):
    """100 tokens, a chain of 64 nodes of which 20 are accepted: the host knows 164, there are 121."""
    with pool(32, 8, 128, "bf16", layers=2) as p:
        s, g = p.shape, generator(keep)
        r, K, V = p.open(100, g)
        rnd = lambda h: torch.randn(2, 64, h, 128, generator=g, device="cuda").to(p.dt)
        q, k, v = rnd(32), rnd(8), rnd(8)
        ws, out = p.workspace(1, 64, 164), torch.empty_like(q[0])
        sled.sled_tree_begin(p.pool, [r], [64], [random_tree(None, 64, "chain")], ws)
        for l in range(2):
            sled.sled_tree_attention(p.pool, l, q[l], k[l], v[l], out, None, ws)
        path = torch.full((1, sled.TREE_MAX), -1, dtype=torch.int32)
        path[0, :20] = torch.arange(1, 21)
        path, length = path.cuda(), torch.tensor([20], dtype=torch.int32, device="cuda")
        mass = torch.zeros(16, 2, 8, 170, device="cuda")
        mass[r, :, :, :121] = torch.rand(2, 8, 121, generator=g, device="cuda")
        want_mass = mass.cpu().numpy()
        dst = [sled.sled_kvpool_open(p.pool)] if fork else None
        ev = sled.workspace(sled.sled_kv_evict_workspace_bytes(p.model, 1, keep))
        torch.cuda.synchronize()
        hold = busy()
        sled.sled_tree_commit(p.pool, [r], length, path)
        sled.sled_kv_evict(p.pool, [r], [keep], 2, 5, mass, ev, dst_ids=dst)
        to, n = (dst[0] if fork else r), min(keep, 121)
        # a step behind it, which nothing has been waited for either
        sled.sled_tree_begin(p.pool, [to], [5], [random_tree(None, 5, "chain")], p.workspace(1, 5, 300))
        assert sled.sled_kvpool_lengths(p.pool, [to]) == [n] and sled.sled_kvpool_positions(p.pool, [to]) == [121]
        del hold
        Ka, Va = torch.cat([K, k[:, :21]], dim=1), torch.cat([V, v[:, :21]], dim=1)
        gotK, gotV = p.read(to, 0, n)
        for l in range(2):
            for h in range(8):
                idx = torch.tensor(evict.kept_tokens(want_mass[r, l, h], 121, keep, 2, 5), device="cuda")
                assert torch.equal(gotK[l, :, h], Ka[l, idx, h]) and torch.equal(gotV[l, :, h], Va[l, idx, h])
                assert torch.equal(mass[to, l, h, :n], torch.from_numpy(want_mass).cuda()[r, l, h, idx]) and bool((mass[to, l, h, n:] == 0).all())


@pytest.mark.parametrize("requests", [129, 300])
def test_mass_of_more_requests_than_a_launch_takes_by_value(requests):
    with pool(4, 4, 64, "f32", n_pages=requests * 4, max_requests=requests) as p:
        s, g, rng = p.shape, generator(requests), np.random.default_rng(requests)
        ctx = [int(x) for x in rng.integers(0, 24, size=requests)]
        opened = [p.open(L, g) for L in ctx]
        reqs = [o[0] for o in opened]
        mass = torch.zeros(requests, 1, 4, 64, device="cuda")
        want = torch.zeros(requests, 4, 64, dtype=torch.float64, device="cuda")
        for most in (17, 4):       # the second trees take the place of the first
            nodes = [int(x) for x in rng.integers(1, most, size=requests)]
            trees, T = [random_tree(rng, n) for n in nodes], sum(nodes)
            q, k, v = (torch.randn(T, 4, 64, generator=g, device="cuda") for _ in range(3))
            lse, ws = torch.empty(T, 4, device="cuda"), p.workspace(requests, T, sum(ctx) + T)
            sled.sled_tree_begin(p.pool, reqs, nodes, trees, ws)
            sled.sled_tree_attention(p.pool, 0, q, k, v, torch.empty_like(q), lse, ws)
            sled.sled_tree_mass(p.pool, 0, q, lse, mass, ws)
            at = 0
            for i, (n, L) in enumerate(zip(nodes, ctx)):
                _, _, w, _, _ = plain_attention(q[at:at + n], opened[i][1][0], opened[i][2][0], k[at:at + n], v[at:at + n], trees[i])
                m = w.sum(dim=0)
                want[reqs[i], :, :L] += m[:, :L]
                want[reqs[i], :, L:] = 0
                want[reqs[i], :, L:L + n] = m[:, L:]
                at += n
        assert bool(((mass[:, 0].double() - want).abs() <= 3e-4 * want).all())      # scores of |q||k| up to 12 in float32: 1e-4, twice, and sums of 17
