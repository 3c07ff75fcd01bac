"""sled_tree_begin / sled_tree_attention / sled_tree_mass on given projections, against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2506_09397_amd import sled
from tree_common import BF16_HALF_STEP, attention_bounds, generator, plain_attention, pool, random_tree

pytestmark = pytest.mark.gpu

HEADS = {"8b": (32, 8, 128, "bf16"), "70b": (64, 8, 128, "bf16"), "g1": (2, 2, 128, "bf16"), "g3": (6, 2, 128, "bf16"), "f32_64": (4, 4, 64, "f32"),
         "f32_128": (8, 2, 128, "f32")}


class Batch:
    """Requests with contexts of the given lengths and trees of the given sizes, on one layer or several."""

    def __init__(self, p, ctx, nodes, seed, kind="mixed", layers=1, q_scale=2.0):
        s = p.shape
        g, rng = generator(seed), np.random.default_rng(seed)
        self.p, self.ctx, self.n, self.layers = p, ctx, nodes, layers
        self.trees = [random_tree(rng, n, kind) for n in nodes]
        opened = [p.open(L, g) for L in ctx]
        self.reqs, self.K, self.V = [o[0] for o in opened], [o[1] for o in opened], [o[2] for o in opened]
        T = sum(nodes)
        self.q = (q_scale * torch.randn(layers, T, s.n_q_heads, s.head_dim, generator=g, device="cuda")).to(p.dt)
        self.k = torch.randn(layers, T, s.n_kv_heads, s.head_dim, generator=g, device="cuda").to(p.dt)
        self.v = torch.randn(layers, T, s.n_kv_heads, s.head_dim, generator=g, device="cuda").to(p.dt)
        self.out, self.lse = torch.full_like(self.q, 7.0), torch.full((layers, T, s.n_q_heads), 7.0, device="cuda")
        self.ws = p.workspace(len(ctx), T, sum(ctx) + T)

    def run(self):
        sled.sled_tree_begin(self.p.pool, self.reqs, self.n, self.trees, self.ws)
        for l in range(self.layers):
            sled.sled_tree_attention(self.p.pool, l, self.q[l], self.k[l], self.v[l], self.out[l], self.lse[l], self.ws)
        torch.cuda.synchronize()

    def plain(self, i, l=0):
        a = sum(self.n[:i])
        b = a + self.n[i]
        return plain_attention(self.q[l, a:b], self.K[i][l], self.V[i][l], self.k[l, a:b], self.v[l, a:b], self.trees[i]), slice(a, b)

    def check(self):
        D, bf = self.p.shape.head_dim, self.p.shape.dtype == "bf16"
        for l in range(self.layers):
            for i in range(len(self.n)):
                (out, lse, _, big, vmax), at = self.plain(i, l)
                tol, tol_lse = attention_bounds(out, lse, big, vmax, D, bf)
                err, err_lse = (self.out[l, at].double() - out).abs(), (self.lse[l, at].double() - lse).abs()
                where = f"layer {l} request {i} (L {self.ctx[i]}, {self.n[i]} nodes)"
                assert bool((err <= tol).all()), f"{where}: out off by {float(err.max())}, {float((err / tol).max())} of what is allowed"
                assert bool((err_lse <= tol_lse).all()), f"{where}: lse off by {float(err_lse.max())}"


# contexts around page and step borders, trees around row-tile borders; every number of row tiles and several row groups
CASES = [
    ("8b", [300], [1]), ("8b", [0], [1]), ("8b", [0, 1, 15, 16, 17, 31, 32, 33], [4, 5, 1, 2, 3, 8, 9, 16]), ("8b", [47, 48, 49, 63, 64, 65, 127, 129], [16, 17, 15, 33, 32, 31, 64, 63]),
    ("8b", [2000, 5], [12, 64]), ("70b", [700, 90, 0], [3, 64, 40]), ("g1", [100, 333], [64, 17]), ("g3", [250, 16], [11, 43]),
    ("f32_64", [0, 1, 16, 17, 100], [1, 64, 16, 33, 7]), ("f32_128", [700, 31, 0], [5, 64, 40]), ("f32_128", [64], [1]),
]


@pytest.mark.parametrize("heads,ctx,nodes", CASES, ids=[f"{h}-{'_'.join(map(str, c))}-{'_'.join(map(str, n))}" for h, c, n in CASES])
def test_attention_of_trees_against_the_formula(heads, ctx, nodes):
    with pool(*HEADS[heads]) as p:
        b = Batch(p, ctx, nodes, seed=len(ctx) * 100 + nodes[0])
        b.run()
        b.check()
        # the nodes' keys and values lie in the tail slots, as given
        at = 0
        for i, n in enumerate(nodes):
            K, V = p.read(b.reqs[i], ctx[i], n)
            assert torch.equal(K[0], b.k[0, at:at + n]) and torch.equal(V[0], b.v[0, at:at + n])
            if ctx[i]:
                K, V = p.read(b.reqs[i], 0, ctx[i])
                assert torch.equal(K, b.K[i]) and torch.equal(V, b.V[i])
            at += n


@pytest.mark.parametrize("kind", ["chain", "star"])
def test_chains_and_stars(kind):
    with pool(32, 8, 128, "bf16") as p:
        b = Batch(p, [40, 200], [64, 21], seed=5, kind=kind)
        b.run()
        b.check()


@pytest.mark.parametrize("heads,L", [("8b", 6000), ("70b", 4111), ("f32_64", 3001)])
def test_long_contexts_are_split_and_joined(heads, L):
    with pool(*HEADS[heads], n_pages=600) as p:
        b = Batch(p, [L, 20], [9, 2], seed=11)
        b.run()
        b.check()
        first = b.out.clone(), b.lse.clone()
        for _ in range(3):   # the joining order is fixed
            b.out.zero_(), b.lse.zero_()
            b.run()
            assert torch.equal(b.out, first[0]) and torch.equal(b.lse, first[1])


@pytest.mark.parametrize("heads,requests,L", [("g1", 256, 4200), ("f32_64", 128, 4801)])
def test_more_than_one_block_of_page_numbers(heads, requests, L):
    """So many requests that a context is one work item or a few, of hundreds of pages."""
    with pool(*HEADS[heads], n_pages=requests * ((L + 15) // 16 + 1), max_requests=requests) as p:
        b = Batch(p, [L] * requests, [1] * requests, seed=12)
        b.n, b.trees = [1] * requests, [[-1]] * requests
        b.run()
        D, bf = p.shape.head_dim, p.shape.dtype == "bf16"
        for i in range(0, requests, 37):
            (out, lse, _, big, vmax), at = b.plain(i)
            tol, tol_lse = attention_bounds(out, lse, big, vmax, D, bf)
            assert bool(((b.out[0, at].double() - out).abs() <= tol).all()) and bool(((b.lse[0, at].double() - lse).abs() <= tol_lse).all())


def test_peaked_and_shifted_scores():
    """Scores of hundreds, and keys that all point away from the query: the running reference moves a long way, up and from far below."""
    with pool(32, 8, 128, "bf16") as p:
        b = Batch(p, [500], [10], seed=13, q_scale=60.0)
        b.run()
        b.check()
        b.q[:] = -30.0
        b.k[:] = 4.0
        K = torch.full_like(b.K[0], 4.0)
        r = sled.sled_kvpool_open(p.pool)
        sled.sled_kv_append(p.pool, [r], [500], [K], [b.V[0]])
        b.K[0], b.reqs[0] = K, r
        b.run()
        b.check()


def test_parts_of_one_matrix():
    """q, k and v as slices of one [T, (Hq + 2 Hkv) D] matrix, and a lse that nobody asked for."""
    with pool(32, 8, 128, "bf16") as p:
        b = Batch(p, [130, 64], [6, 30], seed=14)
        b.run()
        T = sum(b.n)
        m = torch.cat([b.q[0].reshape(T, -1), b.k[0].reshape(T, -1), b.v[0].reshape(T, -1)], dim=1).contiguous()
        q, k, v = m[:, :4096].view(T, 32, 128), m[:, 4096:5120].view(T, 8, 128), m[:, 5120:].view(T, 8, 128)
        out = torch.empty_like(b.out[0])
        sled.sled_tree_begin(p.pool, b.reqs, b.n, b.trees, b.ws)
        sled.sled_tree_attention(p.pool, 0, q, k, v, out, None, b.ws)
        torch.cuda.synchronize()
        assert torch.equal(out, b.out[0])


@pytest.mark.parametrize("heads", ["8b", "f32_128"])
@pytest.mark.parametrize("L", [37, 3000])
def test_values_that_are_not_finite_stay_with_those_who_see_them(heads, L):
    """Nodes 2 and 5 of a tree hold infinities and NaN; a slot behind the context does too, from a request closed before."""
    with pool(*HEADS[heads], n_pages=260) as p:
        g = generator(3)
        r, K, V = p.open(4000, g)
        bad = torch.full_like(V, float("nan"))
        sled.sled_kvpool_close(p.pool, r)
        r = sled.sled_kvpool_open(p.pool)
        sled.sled_kv_append(p.pool, [r], [4000], [bad], [bad])
        sled.sled_kvpool_close(p.pool, r)
        b = Batch(p, [L], [9], seed=15)
        b.trees = [[-1, 0, 0, 1, 2, 3, 4, 5, 0]]
        clean = b.k.clone(), b.v.clone()
        b.run()
        want, want_lse = b.out.clone(), b.lse.clone()
        b.k[0, 2, 0], b.v[0, 2, 0, 3] = float("nan"), float("inf")
        b.v[0, 5, 1, 7], b.v[0, 5, 1, 8] = float("-inf"), float("nan")
        b.run()
        G = p.shape.group
        for j in range(9):
            for kv in range(p.shape.n_kv_heads):
                h = slice(kv * G, (kv + 1) * G)
                got = b.out[0, j, h].float()
                if kv == 0 and j in (2, 4, 6):      # see the NaN key
                    assert bool(torch.isnan(got).all()) and bool(torch.isnan(b.lse[0, j, h]).all())
                elif kv == 1 and j in (5, 7):
                    assert bool((got[:, 7] == float("-inf")).all()) and bool(torch.isnan(got[:, 8]).all())
                    rest = [d for d in range(p.shape.head_dim) if d not in (7, 8)]
                    assert torch.equal(b.out[0, j, h][:, rest], want[0, j, h][:, rest])
                else:
                    assert torch.equal(b.out[0, j, h], want[0, j, h]) and torch.equal(b.lse[0, j, h], want_lse[0, j, h])
        b.k, b.v = clean
        b.run()
        assert torch.equal(b.out, want)
        b.check()


def test_batch_invariant_pools_give_the_same_bits_in_any_batch():
    with pool(32, 8, 128, "bf16", n_pages=1200, max_requests=32, invariant=True) as p:
        b = Batch(p, [3100] + [700] * 11, [17] + [64] * 11, seed=16)
        b.run()
        b.check()
        a = Batch(p, [5], [3], seed=17)
        a.ctx, a.n, a.trees, a.reqs, a.q, a.k, a.v = [3100], [17], b.trees[:1], b.reqs[:1], b.q[:, :17].contiguous(), b.k[:, :17].contiguous(), b.v[:, :17].contiguous()
        a.out, a.lse, a.ws = torch.empty_like(a.q), torch.empty(1, 17, 32, device="cuda"), p.workspace(1, 17, 3200)
        a.run()
        assert torch.equal(a.out, b.out[:, :17]) and torch.equal(a.lse, b.lse[:, :17])


# ------------------------------------------------------------------------------------------------ mass
@pytest.mark.parametrize("heads,ctx,nodes", CASES + [("8b", [3000, 700], [64, 20]), ("70b", [1500], [64])],
                         ids=[f"{h}-{'_'.join(map(str, c))}-{'_'.join(map(str, n))}" for h, c, n in CASES + [("8b", [3000, 700], [64, 20]), ("70b", [1500], [64])]])
def test_mass_against_the_formula(heads, ctx, nodes):
    with pool(*HEADS[heads], layers=2) as p:
        b = Batch(p, ctx, nodes, seed=21, layers=2)
        s = p.shape
        cap = max(L + n for L, n in zip(ctx, nodes)) + 3
        mass = torch.rand(16, 2, s.n_kv_heads, cap, generator=generator(1), device="cuda")
        before = mass.clone()
        b.run()
        for l in (1, 0):
            sled.sled_tree_mass(p.pool, l, b.q[l], b.lse[l], mass, b.ws)
        torch.cuda.synchronize()
        same = torch.ones_like(mass, dtype=torch.bool)
        for i, (L, n) in enumerate(zip(ctx, nodes)):
            for l in range(2):
                (_, lse, w, big, _), _ = b.plain(i, l)
                add = w.view(n, s.n_kv_heads, s.group, L + n).sum(dim=(0, 2))
                had = before[b.reqs[i], l, :, :L + n].double().clone()
                had[:, L:] = 0.0
                # a weight is off by what its score and its row's lse are off by, an exponential's last bits, and float32 sums of n G
                # terms; the sum with what was there is rounded once more
                rel = float((2 * (s.head_dim + 8) * 2.0**-24 * big.max() + 2.0**-21 * lse.abs().max() + 2.0**-19)) + n * s.group * 2.0**-24
                err = (mass[b.reqs[i], l, :, :L + n].double() - had - add).abs()
                tol = rel * add + 2.0**-24 * (had + add) + 1e-30
                assert bool((err <= tol * 1.01).all()), f"request {i} layer {l}: {float((err / tol).max())} of what is allowed"
                same[b.reqs[i], l, :, :L + n] = False
        assert torch.equal(mass[same], before[same])    # nothing else was touched
        again = before.clone()
        for l in range(2):
            sled.sled_tree_mass(p.pool, l, b.q[l], b.lse[l], again, b.ws)
        torch.cuda.synchronize()
        assert torch.equal(again, mass)


# ------------------------------------------------------------------------------------------------ graphs, refusals
def test_captured_layers_replay_on_new_inputs():
    """Attention and mass of one step in a graph: replays with other inputs in the same buffers, eager work of the pool between them."""
    with pool(32, 8, 128, "bf16", layers=2) as p:
        b = Batch(p, [700, 33], [12, 40], seed=31, layers=2)
        cap = 800
        mass = torch.zeros(16, 2, 8, cap, device="cuda")

        def step():
            for l in range(2):
                sled.sled_tree_attention(p.pool, l, b.q[l], b.k[l], b.v[l], b.out[l], b.lse[l], b.ws)
                sled.sled_tree_mass(p.pool, l, b.q[l], b.lse[l], mass, b.ws)

        sled.sled_tree_begin(p.pool, b.reqs, b.n, b.trees, b.ws)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for seed in (1, 2, 3):
            g = generator(seed)
            for x in (b.q, b.k, b.v):
                x.copy_(torch.randn(x.shape, generator=g, device="cuda").to(x.dtype))
            mass.zero_()
            step()
            torch.cuda.synchronize()
            want = b.out.clone(), b.lse.clone(), mass.clone()
            b.out.zero_(), b.lse.zero_(), mass.zero_()
            other, _, _ = p.open(50, g)        # eager work of the same pool
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(b.out, want[0]) and torch.equal(b.lse, want[1]) and torch.equal(mass, want[2])
            sled.sled_kvpool_close(p.pool, other)


def test_calls_that_cannot_be_captured_say_so():
    with pool(32, 8, 128, "bf16") as p:
        b = Batch(p, [70], [5], seed=32)
        b.run()
        graph = torch.cuda.CUDAGraph()
        errors = []
        x = torch.zeros(8, device="cuda")
        a, path = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, 64, dtype=torch.int32, device="cuda")
        with torch.cuda.graph(graph):
            x += 1
            for call in (lambda: sled.sled_tree_begin(p.pool, b.reqs, b.n, b.trees, b.ws), lambda: sled.sled_tree_commit(p.pool, b.reqs, a, path)):
                try:
                    call()
                except sled.SledError as e:
                    errors.append(e)
        assert len(errors) == 2 and all(e.code == sled.ESTATE and "captured" in str(e) for e in errors)
        graph.replay()
        torch.cuda.synchronize()


def _refused(code, what, call):
    with pytest.raises(sled.SledError) as e:
        call()
    assert e.value.code == code and what in str(e.value), str(e.value)


def test_refusals():
    with pool(32, 8, 128, "bf16", n_pages=20) as p:
        b = Batch(p, [100, 20], [5, 3], seed=33)
        begin = lambda reqs=b.reqs, n=b.n, trees=b.trees, ws=b.ws: sled.sled_tree_begin(p.pool, reqs, n, trees, ws)
        attend = lambda layer=0, q=b.q[0], ws=b.ws: sled.sled_tree_attention(p.pool, layer, q, b.k[0], b.v[0], b.out[0], b.lse[0], ws)
        mass = torch.zeros(16, 1, 8, 105, device="cuda")
        _refused(sled.ESTATE, "sled_tree_begin", attend)
        _refused(sled.ESTATE, "sled_tree_begin", lambda: sled.sled_tree_mass(p.pool, 0, b.q[0], b.lse[0], mass, b.ws))
        _refused(sled.EINVAL, "not open", lambda: begin(reqs=[b.reqs[0], 9]))
        _refused(sled.EINVAL, "twice", lambda: begin(reqs=[b.reqs[0], b.reqs[0]]))
        _refused(sled.EINVAL, "nodes", lambda: begin(n=[5, 0], trees=[b.trees[0], []]))
        _refused(sled.EINVAL, "nodes", lambda: begin(n=[5, 65], trees=[b.trees[0], random_tree(np.random.default_rng(0), 65)]))
        _refused(sled.EINVAL, "come before", lambda: begin(trees=[[-1, 0, 2, 0, 0], b.trees[1]]))
        _refused(sled.EINVAL, "come before", lambda: begin(trees=[[-1, -1, 0, 0, 0], b.trees[1]]))
        _refused(sled.EINVAL, "workspace", lambda: begin(ws=b.ws[:256]))
        _refused(sled.EINVAL, "aligned", lambda: begin(ws=b.ws[16:]))
        r, _, _ = p.open(160, generator(1))
        _refused(sled.ENOMEM, "exhausted", lambda: begin(reqs=[r], n=[64], trees=[random_tree(np.random.default_rng(0), 64)]))
        _refused(sled.ESTATE, "sled_tree_begin", attend)
        sled.sled_kvpool_close(p.pool, r)
        begin()
        _refused(sled.EINVAL, "layer", lambda: attend(layer=1))
        _refused(sled.EINVAL, "layer", lambda: attend(layer=-1))
        _refused(sled.EINVAL, "workspace", lambda: attend(ws=torch.empty_like(b.ws)))
        big = torch.zeros(8, 32 * 128 + 4, dtype=torch.bfloat16, device="cuda")
        _refused(sled.EINVAL, "aligned", lambda: attend(q=big[:, :4096].view(8, 32, 128)))
        _refused(sled.EINVAL, "mass rows", lambda: sled.sled_tree_mass(p.pool, 0, b.q[0], b.lse[0], mass[..., :104].contiguous(), b.ws))
        attend()
        sled.sled_tree_mass(p.pool, 0, b.q[0], b.lse[0], mass, b.ws)
        a, path = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.full((2, 64), -1, dtype=torch.int32, device="cuda")
        _refused(sled.EINVAL, "mass rows", lambda: sled.sled_tree_commit(p.pool, b.reqs, a, path, mass[..., :104].contiguous()))
        _refused(sled.ESTATE, "staged", lambda: sled.sled_kv_append(p.pool, b.reqs, accept_len=a))     # a chain's commit is not a tree's
        sled.sled_tree_commit(p.pool, b.reqs[:1], a[:1], path[:1])
        _refused(sled.ESTATE, "sled_tree_begin", attend)                                               # lengths have changed
        _refused(sled.ESTATE, "staged", lambda: sled.sled_tree_commit(p.pool, b.reqs, a, path))
        sled.sled_tree_commit(p.pool, b.reqs[1:], a[1:], path[1:])
        assert sled.sled_kvpool_lengths(p.pool, b.reqs) == [101, 21]
        for spoil in (lambda: sled.sled_kv_append(p.pool, [b.reqs[0]], [1], [b.K[0][:, :1].contiguous()], [b.V[0][:, :1].contiguous()]),
                      lambda: sled.sled_kvpool_close(p.pool, b.reqs[0])):
            begin()
            spoil()
            _refused(sled.ESTATE, "sled_tree_begin", attend)
        sled.sled_tree_commit(p.pool, b.reqs[1:], a[1:], path[1:])                                     # the other tree's commit still stands
        assert sled.sled_kvpool_lengths(p.pool, b.reqs[1:]) == [22]


def test_another_stream():
    with pool(32, 8, 128, "bf16") as p:
        b = Batch(p, [500, 31], [20, 7], seed=34)
        b.run()
        want = b.out.clone()
        torch.cuda.synchronize()
        st = torch.cuda.Stream()
        with torch.cuda.stream(st):
            b.out.zero_()
            sled.sled_tree_begin(p.pool, b.reqs, b.n, b.trees, b.ws)
            sled.sled_tree_attention(p.pool, 0, b.q[0], b.k[0], b.v[0], b.out[0], b.lse[0], b.ws)
        st.synchronize()
        assert torch.equal(b.out, want)


def test_half_step_of_bf16_is_what_the_bounds_count():
    assert BF16_HALF_STEP == 2.0**-8
