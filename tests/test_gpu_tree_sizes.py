"""Tree operators called with workspaces that were sized for something larger."""
import numpy as np
import pytest
import torch

import test_gpu_accept_tree as accept
from paper_2506_09397_amd import serving, sled, synth
from paper_2506_09397_amd.runtime import Verifier
from tree_common import random_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", [sled.GREEDY, sled.SAMPLE], ids=["greedy", "sample"])
def test_acceptance_with_a_workspace_for_the_largest_batch(mode):
    V, nodes = 20011, 64
    ws = sled.workspace(sled.sled_accept_tree_workspace_bytes(32, 32 * nodes, V))
    for sizes in ([1], [9], [49] * 31, [48] * 32, [49] * 32, [64] * 32):      # 1536 rows are scanned first when sampling, 1568 are not
        trees = [random_tree(np.random.default_rng(i), n) for i, n in enumerate(sizes)]
        logits, tokens, u = accept.case(trees, V, seed=len(sizes))
        ws.random_(0, 255)
        got = [x.cpu().numpy() for x in accept.run(mode, trees, logits, tokens, u, 0.75, ws=ws)]
        want, margin = accept.walk(mode, trees, logits.cpu().numpy(), tokens.cpu().numpy(), u.cpu().numpy(), 0.75)
        assert margin > 1e-12
        assert [(int(a), p.tolist(), int(t)) for a, p, t in zip(*got)] == want


def test_a_verifier_for_many_large_trees_accepts_small_batches():
    """Room for 32 trees of 64 nodes, steps of one tree and of a few."""
    shape = synth.SHAPES["tiny_bf16"]
    v = Verifier(shape, synth.SynthWeights(shape, seed=1, device="cuda"), 400, 32, 32, 4000)
    v.enable_trees(64, 2000)
    rng = np.random.default_rng(2)
    reqs = [v.open() for _ in range(5)]
    for B in (1, 5):
        trees = [random_tree(rng, n) for n in (3, 64, 63, 9, 33)[:B]]
        tokens = torch.from_numpy(rng.integers(0, shape.vocab, size=sum(map(len, trees))).astype(np.int32)).cuda()
        logits = v.verify_tree(reqs[:B], trees, tokens)
        a, path, t = v.accept_tree(sled.GREEDY, trees, logits, tokens)
        v.commit_tree(reqs[:B], a, path)
        want, _ = accept.walk(sled.GREEDY, trees, logits.cpu().numpy(), tokens.cpu().numpy(), None, 1.0)
        assert [(int(x), p, int(y)) for x, p, y in zip(a.tolist(), path.tolist(), t.tolist())] == want
    v.destroy()


def test_a_device_that_drafts_more_than_the_verifier_holds():
    """Its tree is cut; the other devices of the batch get their answers."""
    shape = synth.SHAPES["tiny_bf16"]
    v = Verifier(shape, synth.SynthWeights(shape, seed=1, device="cuda"), 60, 3, 3, 400)
    v.enable_trees(6, 200, mass_cap=60, max_requests=3)
    server = serving.Server(v, 3, trees=True, kv_budget=48, kv_recent=8)
    for d in range(3):
        server.open(d, prompt=list(range(10 + d)))
    server.submit(0, 0, 7, [1, 2, 3])
    server.submit(1, 0, 7, list(range(63)), parents=[0] * 63)
    server.submit(2, 0, 7, [5])
    answers = server.run_batch()
    assert [r.device for r in answers] == [0, 1, 2]
    assert v.lengths([server.req_of[d] for d in range(3)]) == [10 + d + r.accept_len + 1 for d, r in enumerate(answers)]
    v.destroy()


def test_mass_for_all_requests_of_the_pool_unless_said_otherwise():
    shape = synth.SHAPES["tiny_bf16"]
    v = Verifier(shape, synth.SynthWeights(shape, seed=1, device="cuda"), 40, 5, 2, 200)
    with pytest.raises(AssertionError, match="every request"):
        v.enable_trees(6, 100, mass_cap=50, max_requests=4)
    v.enable_trees(6, 100, mass_cap=50)
    assert v.mass.shape[0] == 5
    r = v.open_bounded()
    v.verify_tree([r], [[-1, 0, 0]], torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert abs(float(v.mass[r].sum()) - shape.n_layers * 3 * shape.n_q_heads) < 1e-2     # a weight of one a row, head and layer
    v.destroy()
