"""Steps over trees as the model runs them: the mass of every single token against the oracle, low-bit weights, batches of many rows; and mass over
pools so large that a workgroup goes through several runs of pages."""
import math

import numpy as np
import pytest
import torch

from oracle import sled_oracle as O
from paper_2506_09397_amd import sled, synth
from paper_2506_09397_amd.runtime import Verifier
from helpers import oracle_model
from test_gpu_tree_attention import HEADS, Batch
from test_gpu_tree_edges import mass_of
from test_gpu_tree_step import oracle_tree, setup
from tree_common import ancestors, pool, random_tree

pytestmark = pytest.mark.gpu


def oracle_mass(om, K, V, parent, tokens, stored):
    """([layers, kv heads, L + n] mass of a step, largest sum of |q||k| / sqrt(D)): node by node along its ancestors, over the K/V that the step has put
    into its nodes' slots (stored: two [layers, n, kv heads, D])."""
    L, n, D = K.shape[1], len(parent), om.head_dim
    mass, big = np.zeros((om.n_layers, om.n_kv_heads, L + n)), 0.0
    E = om.weights.embed()
    for j in range(n):
        way = ancestors(parent, j)
        h = E[np.asarray([tokens[i] for i in way])].astype(np.float64)
        pos = np.arange(L, L + len(way))
        at = list(range(L)) + [L + i for i in way]
        for l in range(om.n_layers):
            W = om.weights.layer(l)
            q = O.rope((O.rmsnorm(h[-1:], W["g_attn"], om.rms_eps) @ W["wq"].T).reshape(1, om.n_q_heads, D), pos[-1:], om.rope_theta)[0]
            kv = stored[0][l][way], stored[1][l][way]
            keys = np.concatenate([K[l], kv[0]])
            for hq in range(om.n_q_heads):
                k = keys[:, hq // om.group]
                s = k @ q[hq] / math.sqrt(D)
                big = max(big, float((np.abs(k) @ np.abs(q[hq])).max()) / math.sqrt(D))
                w = np.exp(s - s.max())
                mass[l, hq // om.group, at] += w / w.sum()
            h, _, _ = O.layer_rows(om, W, h, pos, K[l], V[l], stored=kv)
    return mass, big


@pytest.mark.parametrize("kind", ["tiny", "tiny_bf16"])
def test_mass_of_a_step_token_by_token(kind):
    ctx, nodes = [33, 0, 120], [10, 7, 24]
    shape, v, w, reqs, KV, trees, tokens = setup(kind, ctx, nodes, seed=18, mass_cap=200)
    tok = torch.from_numpy(tokens).cuda()
    rng = torch.Generator(device="cuda").manual_seed(1)
    for r, L in zip(reqs, ctx):
        v.mass[r, :, :, :L] = torch.rand(shape.n_layers, shape.n_kv_heads, L, generator=rng, device="cuda")
    before = v.mass.clone()
    v.verify_tree(reqs, trees, tok)
    om = oracle_model(shape, w)
    at = 0
    for i, (r, L, n) in enumerate(zip(reqs, ctx, nodes)):
        stored = [synth.as_f64(x) for x in v.read_kv(r, L, n)]
        want, big = oracle_mass(om, synth.as_f64(KV[i][0]), synth.as_f64(KV[i][1]), trees[i], tokens[at : at + n], stored)
        had = before[r, :, :, : L + n].double().cpu().numpy()
        got = v.mass[r, :, :, : L + n].double().cpu().numpy() - had
        # A query is a sum of 256 products with activations of 16 bits (bf16 models: pairs), magnitudes 16 times the result's, and the layers before have done
        # the same: 2^-17 x 16 x a few, 2^-11 of |q||k|.  A weight is off by twice its score; the sum was rounded onto what was there.
        tol = 2.0 * (2.0**-11 * big + 2.0**-18) * want + 2.0**-22 * (had + want) + 1e-9
        err = np.abs(got - want)
        print(f"{kind} L={L} nodes={n}: worst {float((err / tol).max()):.3f} of what is allowed, largest |q||k| {big:.1f}")
        assert (err <= tol).all()
        assert bool((v.mass[r, :, :, L + n :] == 0).all())
        at += n
    v.destroy()


@pytest.mark.parametrize("cls", [synth.SynthWeightsW8, synth.SynthWeightsW4], ids=["8bit", "4bit"])
@pytest.mark.parametrize("ctx,nodes", [([0, 40, 17, 100], [9, 21, 1, 12]), ([64, 200, 5, 31], [64, 50, 64, 40])], ids=["43_rows", "218_rows"])
def test_trees_with_lowbit_weights(cls, ctx, nodes):
    shape = synth.SHAPES["tiny_bf16"]
    w = cls(shape, seed=2, device="cuda", std=0.02, gain_jitter=0.1)
    B = len(ctx)
    v = Verifier(shape, w, sum(ctx) // 16 + 8 * B, B, B, sum(ctx) + 16 * B)
    v.enable_trees(64, sum(ctx))
    rng = np.random.default_rng(8)
    reqs = [v.open() for _ in ctx]
    KV = [synth.context_kv(shape, L, seed=3, req=i, device="cuda") for i, L in enumerate(ctx)]
    some = [i for i, L in enumerate(ctx) if L]
    v.append_context([reqs[i] for i in some], [KV[i][0] for i in some], [KV[i][1] for i in some])
    trees = [random_tree(rng, n) for n in nodes]
    tokens = rng.integers(0, shape.vocab, size=sum(nodes)).astype(np.int32)
    logits = v.verify_tree(reqs, trees, torch.from_numpy(tokens).cuda()).cpu().numpy()
    om = oracle_model(shape, w)
    at = 0
    for i, n in enumerate(nodes):
        want = oracle_tree(om, synth.as_f64(KV[i][0]), synth.as_f64(KV[i][1]), trees[i], tokens[at : at + n])
        assert np.abs(logits[at : at + n] - want).max() < 5e-3      # as for chains with such weights
        at += n
    v.destroy()


def test_mass_over_a_pool_of_many_pages():
    """More than 8192 runs of 16 pages: a workgroup takes two of them, with rows that stay in LDS between them and rows that do not fit."""
    ctx, nodes = [16500 + 7 * i for i in range(16)], [64, 1, 20, 32, 33] + [2] * 11
    with pool(*HEADS["70b"], n_pages=sum(L // 16 + 6 for L in ctx)) as p:
        b = Batch(p, ctx, nodes, seed=61, q_scale=1.0)
        b.run()
        cap = max(L + n for L, n in zip(ctx, nodes))
        mass = torch.zeros(16, 1, 8, cap, device="cuda")
        sled.sled_tree_mass(p.pool, 0, b.q[0], b.lse[0], mass, b.ws)
        torch.cuda.synchronize()
        for i in (0, 1, 2, 3, 4, 15):
            m, off = mass_of(b, i)
            got = mass[b.reqs[i], 0].double()
            err = (got[:, : ctx[i] + nodes[i]] - m).abs()
            assert bool((err <= off).all()), f"request {i}: {float((err / off).max())} of what is allowed"
            assert bool((got[:, ctx[i] + nodes[i] :] == 0).all())
        again = torch.zeros_like(mass)
        sled.sled_tree_mass(p.pool, 0, b.q[0], b.lse[0], again, b.ws)
        torch.cuda.synchronize()
        assert torch.equal(again, mass)
