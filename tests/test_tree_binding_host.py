"""The binding's checks of tensors that go with a plan or a pool: the C entry points get pointers and cannot see sizes."""
import pytest
import torch

from paper_2506_09397_amd import sled, synth

POOL, MODEL = 0x5EAF00D, 0x5EAF00E     # (handles of nothing: every call below is refused before the library is asked)


class Called(Exception):
    pass


class NoLibrary:
    def __getattr__(self, name):
        def call(*a):
            raise Called(name)
        return call


@pytest.fixture
def known(monkeypatch):
    shape = synth.ModelShape(2, 256, 32, 8, 128, 256, 1024, "bf16", 10000.0)
    info = sled._PoolInfo(shape, 4)
    monkeypatch.setitem(sled._models, MODEL, shape)
    monkeypatch.setitem(sled._pools, POOL, info)
    monkeypatch.setattr(sled, "lib", NoLibrary)
    monkeypatch.setattr(sled, "_ptr", lambda t: 256)               # (tensors of the CPU stand in for device memory)
    monkeypatch.setattr(sled, "_rows", lambda t, shape: (256, 1))
    monkeypatch.setattr(sled, "_stream", lambda: 0)
    return info


def rows(n, h, D=128, dtype=torch.bfloat16):
    return torch.zeros(n, h, D, dtype=dtype)


WS = torch.zeros(256, dtype=torch.uint8)


@pytest.mark.parametrize("q,k", [((11, 32), (11, 8)), ((13, 32), (13, 8)), ((12, 31), (12, 8)), ((12, 32), (12, 7)), ((12, 64), (12, 8)), ((0, 32), (0, 8))])
def test_attention_takes_the_planned_rows_and_the_models_heads(known, q, k):
    known.plan(12)
    with pytest.raises(AssertionError, match="trees at hand"):
        sled.sled_tree_attention(POOL, 0, rows(*q), rows(*k), rows(*k), rows(*q), torch.zeros(q), WS)


@pytest.mark.parametrize("dtype,D", [(torch.float32, 128), (torch.float16, 128), (torch.bfloat16, 64)])
def test_attention_takes_the_models_type_and_width(known, dtype, D):
    known.plan(12)
    with pytest.raises(AssertionError, match="trees at hand"):
        sled.sled_tree_attention(POOL, 0, rows(12, 32, D, dtype), rows(12, 8, D, dtype), rows(12, 8, D, dtype), rows(12, 32, D, dtype), None, WS)


@pytest.mark.parametrize("q,dtype", [((11, 32), torch.bfloat16), ((12, 16), torch.bfloat16), ((12, 32), torch.float32)])
def test_mass_takes_the_planned_rows(known, q, dtype):
    known.plan(12)
    with pytest.raises(AssertionError, match="trees at hand"):
        sled.sled_tree_mass(POOL, 0, rows(*q, dtype=dtype), torch.zeros(q), torch.zeros(4, 2, 8, 50), WS)


@pytest.mark.parametrize("shape", [(3, 2, 8, 50), (0, 2, 8, 50), (4, 1, 8, 50), (4, 2, 7, 50), (4, 8, 2, 50), (4, 2, 400)])
def test_mass_covers_the_pool(known, shape):
    known.plan(12)
    mass, i32 = torch.zeros(shape), torch.zeros(1, dtype=torch.int32)
    calls = [lambda: sled.sled_tree_mass(POOL, 0, rows(12, 32), torch.zeros(12, 32), mass, WS),
             lambda: sled.sled_tree_commit(POOL, [0], i32, torch.zeros(1, 64, dtype=torch.int32), mass),
             lambda: sled.sled_kv_evict(POOL, [0], [5], 0, 0, mass, WS),
             lambda: sled.sled_verify_tree(MODEL, POOL, [0], [1], [[-1]], i32, torch.zeros(1, 1024), WS, mass)]
    for call in calls:
        with pytest.raises(AssertionError, match="mass"):
            call()


@pytest.mark.parametrize("shape", [(3, 1023), (3, 1025), (2, 1024), (3,), (3, 1024, 1)])
def test_logits_of_a_tree_step_have_the_models_vocabulary(known, shape):
    with pytest.raises(AssertionError):
        sled.sled_verify_tree(MODEL, POOL, [0], [3], [[-1, 0, 0]], torch.zeros(3, dtype=torch.int32), torch.zeros(shape), WS)


def test_what_fits_goes_to_the_library(known):
    assert sled._mass(POOL, torch.zeros(9, 2, 8, 50)) == (256, 50) and sled._mass(POOL, None) == (None, 0)     # (more rows than requests are fine)
    q, k, mass = rows(12, 32), rows(12, 8), torch.zeros(4, 2, 8, 50)
    for rows_planned in (0, 12):      # before any plan the library itself refuses
        known.plan(rows_planned)
        with pytest.raises(Called, match="sled_tree_attention"):
            sled.sled_tree_attention(POOL, 0, q, k, k, q, None, WS)
        with pytest.raises(Called, match="sled_tree_mass"):
            sled.sled_tree_mass(POOL, 0, q, torch.zeros(12, 32), mass, WS)
    with pytest.raises(Called, match="sled_verify_tree"):
        sled.sled_verify_tree(MODEL, POOL, [0], [3], [[-1, 0, 0]], torch.zeros(3, dtype=torch.int32), torch.zeros(3, 1024), WS, mass)
