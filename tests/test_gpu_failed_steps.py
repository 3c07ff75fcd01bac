"""Steps that fail after some of their work is on its way leave nothing to commit.  A failure is forced from the host: a HIP call with a device number
that does not exist leaves an error behind, which the next launch of the library finds and reports (the launch itself is sound).  Nothing of torch's own may be launched in between."""
import numpy as np
import pytest
import torch

from paper_2506_09397_amd import sled, synth
from gpu_common import build_verifier
from tree_common import random_tree

pytestmark = pytest.mark.gpu

KINDS = ["tiny", "tiny_bf16"]


class Rounds:
    def __init__(self, kind, mass_cap=0):
        shape = synth.SHAPES[kind]
        self.shape = shape
        self.v, _ = build_verifier(shape, 3, n_pages=60, max_requests=3, B_max=3, ctx_tokens_max=400, gain_jitter=0.1, std=0.08)
        self.v.enable_trees(16, 300, mass_cap=mass_cap, max_requests=3)
        rng = np.random.default_rng(4)
        self.ctx, nodes = [20, 33, 7], [5, 16, 9]
        self.reqs = [self.v.open_bounded() if mass_cap else self.v.open() for _ in self.ctx]
        KV = [synth.context_kv(shape, L, seed=2, req=i, device="cuda") for i, L in enumerate(self.ctx)]
        self.v.append_context(self.reqs, [a for a, _ in KV], [b for _, b in KV])
        self.trees = [random_tree(rng, n) for n in nodes]
        self.tokens = torch.from_numpy(rng.integers(0, shape.vocab, size=sum(nodes)).astype(np.int32)).cuda()
        self.none = torch.zeros(3, dtype=torch.int32, device="cuda")
        self.path = torch.full((3, sled.TREE_MAX), -1, dtype=torch.int32, device="cuda")

    def fails(self, call):
        assert self.v.lengths(self.reqs) is not None       # (waits, and looks at everything that has come back)
        torch.cuda.synchronize()
        assert sled.lib().hipSetDevice(9999) != 0
        with pytest.raises(sled.SledError) as e:
            call()
        assert e.value.code == sled.EHIP and "launch failed" in str(e.value)
        torch.cuda.synchronize()

    def no_commit(self, call):
        with pytest.raises(sled.SledError) as e:
            call()
        assert e.value.code == sled.ESTATE


@pytest.mark.parametrize("kind", KINDS)
def test_a_tree_step_that_fails_stages_nothing(kind):
    t = Rounds(kind, mass_cap=80)
    v = t.v
    want = v.verify_tree(t.reqs, t.trees, t.tokens).clone()
    v.commit_tree(t.reqs[:1], t.none[:1], t.path[:1])
    v.mass.zero_()
    rest = t.tokens[5:].clone()
    t.fails(lambda: v.verify_tree(t.reqs[1:], t.trees[1:], rest))
    for r in t.reqs:
        t.no_commit(lambda: v.commit_tree([r], t.none[:1], t.path[:1]))
    again = v.verify_tree(t.reqs[1:], t.trees[1:], rest)
    # (another batch: float32 sums in another order)
    assert float((again - want[5:]).abs().max()) < (1e-4 if kind == "tiny" else 2e-2)
    for r, L, tree in zip(t.reqs[1:], t.ctx[1:], t.trees[1:]):
        n = len(tree)
        total = v.mass[r, :, :, :L + n].double().sum(dim=2)
        assert float((total - n * t.shape.group).abs().max()) < 1e-4 * n * t.shape.group and bool((v.mass[r, :, :, L + n:] == 0).all())
    v.commit_tree(t.reqs[1:], t.none[1:], t.path[1:])
    assert v.lengths(t.reqs) == [L + 1 for L in t.ctx]
    v.destroy()


@pytest.mark.parametrize("kind", KINDS)
def test_a_chain_step_that_fails_drops_what_its_requests_had_staged(kind):
    t = Rounds(kind)
    v = t.v
    v.verify_tree(t.reqs, t.trees, t.tokens)
    four = t.tokens[:4].clone()
    t.fails(lambda: v.verify(t.reqs[:2], [2, 0], four))
    for r in t.reqs[:2]:
        t.no_commit(lambda: v.commit_tree([r], t.none[:1], t.path[:1]))
    v.commit_tree(t.reqs[2:], t.none[:1], t.path[:1])          # the tree of a request that had no part in it
    v.verify(t.reqs, [1, 2, 0], t.tokens[:6].clone())
    t.fails(lambda: v.verify(t.reqs[:1], [3], four))
    t.no_commit(lambda: v.commit(t.reqs[:1], t.none[:1]))
    v.commit(t.reqs[1:], t.none[1:])
    assert v.lengths(t.reqs) == [20, 34, 9]
    v.destroy()


@pytest.mark.parametrize("kind", KINDS)
def test_a_commit_or_an_append_that_fails_drops_what_was_staged(kind):
    t = Rounds(kind)
    v, s = t.v, t.shape
    K, V = (torch.randn(s.n_layers, 2, s.n_kv_heads, s.head_dim, device="cuda").to(s.torch_dtype) for _ in range(2))
    v.verify_tree(t.reqs, t.trees, t.tokens)
    t.fails(lambda: v.append_context(t.reqs[:1], [K], [V]))
    t.no_commit(lambda: v.commit_tree(t.reqs[:1], t.none[:1], t.path[:1]))
    t.fails(lambda: v.commit_tree(t.reqs[1:2], t.none[1:2], t.path[1:2]))
    t.no_commit(lambda: v.commit_tree(t.reqs[1:2], t.none[:1], t.path[:1]))
    v.commit_tree(t.reqs[2:], t.none[:1], t.path[:1])
    assert v.lengths(t.reqs) == [20, 33, 8]
    v.verify_tree(t.reqs, t.trees, t.tokens)
    v.commit_tree(t.reqs, t.none, t.path)
    assert v.lengths(t.reqs) == [21, 34, 9]
    v.destroy()


def test_a_refused_step_leaves_what_is_staged():
    """Nothing is launched by a call whose arguments are refused."""
    t = Rounds("tiny_bf16")
    v = t.v
    v.verify_tree(t.reqs, t.trees, t.tokens)
    small = v.tree_ws[:4096]
    with pytest.raises(sled.SledError):
        sled.sled_verify_tree(v.model, v.pool, t.reqs, [len(x) for x in t.trees], t.trees, t.tokens, v.tree_logits[:30], small)
    with pytest.raises(sled.SledError):
        sled.sled_verify_batch(v.model, v.pool, t.reqs, [1, 1, 1], t.tokens[:6].clone(), v.logits[:6], small)
    v.commit_tree(t.reqs, t.none, t.path)
    assert v.lengths(t.reqs) == [L + 1 for L in t.ctx]
    v.destroy()
