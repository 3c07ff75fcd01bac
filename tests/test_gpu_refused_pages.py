"""Tree plans and evictions that are refused for want of pages (or of workspace) keep none of those they had taken for the first requests of the call."""
import numpy as np
import pytest
import torch

from paper_2506_09397_amd import sled
from tree_common import generator, pool, random_tree

pytestmark = pytest.mark.gpu


def test_plans():
    with pool(32, 8, 128, "bf16", n_pages=20) as p:
        g, rng = generator(1), np.random.default_rng(1)
        (a, _, _), (b, _, _) = p.open(100, g), p.open(90, g)          # 7 and 6 pages: 7 are free
        trees = [random_tree(rng, 64) for _ in range(2)]
        ws = p.workspace(2, 128, 318)
        for code, reqs, w in ((sled.ENOMEM, [a, b], ws), (sled.EINVAL, [a], ws[:256])):
            with pytest.raises(sled.SledError) as e:
                sled.sled_tree_begin(p.pool, reqs, [64] * len(reqs), trees[:len(reqs)], w)
            assert e.value.code == code
            c, _, _ = p.open(112, g)                                    # all seven
            sled.sled_kvpool_close(p.pool, c)
        # what is staged keeps its pages through a refusal
        sled.sled_tree_begin(p.pool, [a], [40], [random_tree(rng, 40)], ws)
        with pytest.raises(sled.SledError):
            sled.sled_tree_begin(p.pool, [a, b], [64, 64], trees, ws)
        none = torch.zeros(1, dtype=torch.int32, device="cuda")
        path = torch.full((1, sled.TREE_MAX), -1, dtype=torch.int32, device="cuda")
        sled.sled_kv_read(p.pool, a, 100, 40, *(torch.empty(1, 40, 8, 128, dtype=p.dt, device="cuda") for _ in range(2)))
        sled.sled_tree_commit(p.pool, [a], none, path)
        assert sled.sled_kvpool_lengths(p.pool, [a, b]) == [101, 90]


def test_evictions_into_other_requests():
    with pool(32, 8, 128, "bf16", n_pages=20) as p:
        g = generator(2)
        (a, _, _), (b, _, _) = p.open(100, g), p.open(90, g)
        mass, ws = torch.zeros(16, 1, 8, 100, device="cuda"), sled.workspace(sled.sled_kv_evict_workspace_bytes(p.model, 2, 80))
        dst = [sled.sled_kvpool_open(p.pool) for _ in range(2)]
        with pytest.raises(sled.SledError) as e:
            sled.sled_kv_evict(p.pool, [a, b], [80, 80], 0, 0, mass, ws, dst_ids=dst)      # five pages each
        assert e.value.code == sled.ENOMEM
        c, _, _ = p.open(112, g)
        assert sled.sled_kvpool_lengths(p.pool, [a, b, *dst, c]) == [100, 90, 0, 0, 112]
