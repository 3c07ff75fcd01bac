"""Workspaces of the tree operators without a GPU: what is enough for a batch is enough for every smaller one."""
import itertools

import pytest

from paper_2506_09397_amd import sled


@pytest.mark.parametrize("vocab", [2, 3, 4, 4096, 4097, 50257, 128256, 2000000])
def test_acceptance_over_a_smaller_batch_never_needs_more(vocab):
    need = sled.sled_accept_tree_workspace_bytes
    # rows around the sizes at which a call stops scanning first (1024 and 1536) and at which a shape no longer travels with the launch (2048)
    rows = [1, 2, 9, 64, 256, 257, 1023, 1024, 1025, 1535, 1536, 1537, 2047, 2048, 2049, 4096, 65536]
    batches = [1, 2, 63, 64, 65, 1024]
    for (b0, b1), (t0, t1) in itertools.product(zip(batches, batches[1:]), zip(rows, rows[1:])):
        assert need(b0, t0, vocab) <= need(b0, t1, vocab) <= need(b1, t1, vocab), (b0, b1, t0, t1)
