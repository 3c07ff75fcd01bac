"""sled_accept_tree on logits whose banned tokens hold large negative numbers in place of minus infinity: they weigh exactly nothing, also for a
uniform of zero, which names the lowest id that weighs anything."""
import numpy as np
import pytest
import torch

import test_gpu_accept_tree as accept
from paper_2506_09397_amd import sled
from tree_common import random_tree

pytestmark = pytest.mark.gpu

LOWEST = torch.finfo(torch.float32).min


@pytest.mark.parametrize("temperature", [0.25, 0.5, 1.0, 4.0])
@pytest.mark.parametrize("mask", [LOWEST, -1e37, -1e30, -1e20, -1e4], ids=lambda x: f"{x:.0e}")
@pytest.mark.parametrize("requests", [1, 24, 64])      # rows scanned first, and (beyond 1536) gone through by their walk alone
def test_banned_tokens_weigh_nothing(requests, mask, temperature):
    V = 13000
    rng = np.random.default_rng(3)
    trees = [random_tree(rng, 33) for _ in range(requests)]
    logits, tokens, u = accept.case(trees, V, seed=9)
    logits[:, :4500] = mask           # more than a whole piece of a row, and parts of others
    logits[:, 6000:6100] = mask
    logits[:, 11000:] = mask
    tokens.clamp_(4500, 10999)
    u[0::3] = 0.0
    u[1::3] = 1.0 - 2.0**-24
    want = accept.check(sled.SAMPLE, trees, logits, tokens, u, temperature)
    assert all(4500 <= w[2] < 11000 for w in want)
    accept.check(sled.GREEDY, trees, logits, tokens, None)


@pytest.mark.parametrize("requests", [1, 64])
def test_weights_that_float64_can_and_cannot_hold(requests):
    """A token 700 below the row's best weighs 1e-304 and may be named by a uniform of zero; one 760 below weighs nothing."""
    V = 9000
    trees = [[-1]] * (33 * requests)
    logits = torch.full((33 * requests, V), -float("inf"), device="cuda")
    logits[:, 5000] = 10.0
    logits[0::2, 40], logits[1::2, 40] = 10.0 - 700.0, 10.0 - 760.0
    u = torch.zeros(33 * requests, device="cuda")
    tokens = torch.zeros(33 * requests, dtype=torch.int32, device="cuda")
    for a in range(0, len(trees), 1000):
        _, _, o = accept.run(sled.SAMPLE, trees[a:a + 1000], logits[a:a + 1000], tokens[a:a + 1000], u[a:a + 1000])
        assert o.tolist() == [40 if (a + i) % 2 == 0 else 5000 for i in range(len(o))]
