"""Trees and eviction without a GPU: what is refused is refused before anything is launched, and the helpers of the GPU tests."""
import ctypes as C

import numpy as np
import pytest

from paper_2506_09397_amd import sled
from tree_common import ancestors, depths, random_tree, seen_matrix


def _accept(mode=sled.GREEDY, B=2, n=(2, 3), parent=(-1, 0, -1, 0, 1), vocab=100, temperature=1.0, ws=4096, ws_bytes=1 << 20, u=None, ptr=256):
    return sled.lib().sled_accept_tree(mode, B, (C.c_int * len(n))(*n), (C.c_int * len(parent))(*parent), vocab, temperature, ptr, ptr, u, ptr, ptr, ptr, ws,
                                       ws_bytes, None)


@pytest.mark.parametrize("kw,what", [
    (dict(mode=7), "mode"), (dict(mode=sled.SAMPLE), "needs u"), (dict(B=0), "batch size"), (dict(B=1025, n=(1,) * 1025, parent=(-1,) * 1025), "batch size"),
    (dict(vocab=1), "vocab"), (dict(vocab=2000001), "vocab"), (dict(temperature=0.0), "temperature"), (dict(temperature=float("nan")), "temperature"),
    (dict(n=(2, 0)), "nodes"), (dict(n=(65, 1), parent=(-1,) + tuple(range(64)) + (-1,)), "nodes"), (dict(parent=(-1, 1, -1, 0, 1)), "come before"),
    (dict(parent=(-1, 0, -1, -1, 1)), "come before"), (dict(ws=4096 + 64), "aligned"), (dict(ws_bytes=255), "workspace"), (dict(ptr=None), "null"),
])
def test_accept_tree_refuses(kw, what):
    assert _accept(**kw) == sled.EINVAL
    assert what in sled.lib().sled_last_error().decode()


def test_null_handles_are_refused():
    L = sled.lib()
    one = (C.c_int * 1)(1)
    assert L.sled_tree_begin(None, 1, one, one, one, 256, 1 << 20, None) == sled.EINVAL
    assert L.sled_tree_attention(None, 0, 256, 128, 256, 128, 256, 128, 256, None, 256, None) == sled.EINVAL
    assert L.sled_tree_mass(None, 0, 256, 128, 256, 256, 16, 256, None) == sled.EINVAL
    assert L.sled_tree_commit(None, 1, one, 256, 256, None, 0, None) == sled.EINVAL
    assert L.sled_verify_tree(None, None, 1, one, one, one, 256, 256, None, 0, 256, 1 << 20, None) == sled.EINVAL
    assert L.sled_kv_evict(None, 1, one, None, one, 0, 0, 256, 16, 256, 1 << 20, None) == sled.EINVAL
    assert L.sled_kvpool_positions(None, 1, one, one, None) == sled.EINVAL
    assert L.sled_tree_workspace_bytes(None, 1, 1, 1) == 0 and L.sled_verify_tree_workspace_bytes(None, 1, 1, 1) == 0
    assert L.sled_kv_evict_workspace_bytes(None, 1, 1) == 0
    assert L.sled_accept_tree_workspace_bytes(0, 1, 100) == 0 and L.sled_accept_tree_workspace_bytes(1, 1, 100) > 0


def test_binding_wants_a_parent_for_every_node():
    with pytest.raises(AssertionError):
        sled._parents([2, 3], [[-1, 0], [-1, 0]])
    assert list(sled._parents([2, 3], [[5, 0], [-1, 0, 1]])) == [-1, 0, -1, 0, 1]


@pytest.mark.parametrize("kind", ["mixed", "chain", "star"])
def test_helpers(kind):
    rng = np.random.default_rng(1)
    for n in (1, 2, 17, 64):
        p = random_tree(rng, n, kind)
        assert len(p) == n and all(0 <= p[j] < j for j in range(1, n))
        see = seen_matrix(p)
        for j in range(n):
            way = ancestors(p, j)
            assert way[0] == 0 and way[-1] == j and len(way) == depths(p)[j] + 1
            assert sorted(np.nonzero(see[j].numpy())[0].tolist()) == way
