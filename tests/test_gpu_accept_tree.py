"""sled_accept_tree against a walk written out in 64 bits on the host: whole numbers, equal wherever the choice is not a tie of rounding."""
import numpy as np
import pytest
import torch

from paper_2506_09397_amd import sled, synth
from tree_common import depths, generator, random_tree

pytestmark = pytest.mark.gpu


def walk(mode, trees, logits, tokens, u, temperature):
    """(accept_len, path, out_token, smallest distance of a draw from a border of the cumulative sums, in probability)."""
    out, at, margin = [], 0, 1.0
    tau = float(np.float32(temperature))
    for p in trees:
        cur, way = 0, []
        while True:
            z = logits[at + cur].astype(np.float64)
            if mode == sled.GREEDY:
                t = int(np.argmax(z))
            else:
                w = np.exp((z - z.max()) / tau)
                c = np.cumsum(w)
                target = float(u[at + cur]) * c[-1]
                over = np.nonzero(c > target)[0]
                t = int(over[0]) if len(over) else int(np.nonzero(w > 0)[0][-1])
                margin = min(margin, float(np.abs(c - target).min() / c[-1]) if target > 0 else 1.0)
            kids = [j for j in range(1, len(p)) if p[j] == cur and tokens[at + j] == t]
            if not kids:
                break
            cur = kids[0]
            way.append(cur)
        out.append((len(way), way + [-1] * (sled.TREE_MAX - len(way)), t))
        at += len(p)
    return out, margin


def case(trees, vocab, seed, follow=0.75, sigma=2.0):
    """Trees whose tokens follow the target: with probability `follow` a node's first child drafts the token of the highest logit."""
    g, rng = generator(seed), np.random.default_rng(seed)
    T = sum(len(t) for t in trees)
    logits = sigma * torch.randn(T, vocab, generator=g, device="cuda")
    tokens = torch.randint(0, vocab, (T,), generator=g, device="cuda", dtype=torch.int32)
    top = logits.argmax(dim=1).cpu().numpy()
    tk = tokens.cpu().numpy()
    at = 0
    for p in trees:
        seen = set()
        for j in range(1, len(p)):
            if rng.random() < (follow if p[j] not in seen else 0.1):
                tk[at + j] = top[at + p[j]]
            seen.add(p[j])
        at += len(p)
    return logits, torch.from_numpy(tk).cuda(), torch.rand(T, generator=g, device="cuda")


def run(mode, trees, logits, tokens, u, temperature=1.0, ws=None):
    B, (T, V) = len(trees), logits.shape
    n = [len(t) for t in trees]
    ws = sled.workspace(sled.sled_accept_tree_workspace_bytes(B, T, V)) if ws is None else ws
    a, o = (torch.full((B,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    path = torch.full((B, sled.TREE_MAX), -7, dtype=torch.int32, device="cuda")
    sled.sled_accept_tree(mode, n, trees, V, temperature, logits, tokens, u, a, path, o, ws)
    torch.cuda.synchronize()
    return a, path, o


def check(mode, trees, logits, tokens, u, temperature=1.0):
    got = [x.cpu().numpy() for x in run(mode, trees, logits, tokens, u, temperature)]
    want, margin = walk(mode, trees, logits.cpu().numpy(), tokens.cpu().numpy(), None if u is None else u.cpu().numpy(), temperature)
    assert margin > 1e-12, "the inputs hold a draw on a border"
    for i, (ln, path, t) in enumerate(want):
        assert (int(got[0][i]), int(got[2][i])) == (ln, t), f"tree {i} of {len(trees[i])} nodes"
        assert got[1][i].tolist() == path
    return want


SIZES = [
    # (trees' sizes, vocabulary): few rows (all scanned first), many rows (a workgroup goes through those of its walk), odd and small vocabularies, one piece and several
    ([1], 2), ([1], 128256), ([9], 128256), ([64], 50257), ([5, 1, 64, 17], 4099), ([32] * 16, 128256), ([3, 64, 40, 1] * 10, 32001), ([64] * 8, 128256),
    ([2, 7] * 60, 1000), ([1] * 1024, 37), ([64, 64, 64, 64, 64, 64, 64, 64] * 10, 257),
]


@pytest.mark.parametrize("mode", [sled.GREEDY, sled.SAMPLE], ids=["greedy", "sample"])
@pytest.mark.parametrize("sizes,vocab", SIZES, ids=[f"{len(s)}x{max(s)}-{v}" for s, v in SIZES])
def test_walk(mode, sizes, vocab):
    rng = np.random.default_rng(len(sizes) + vocab)
    trees = [random_tree(rng, n) for n in sizes]
    logits, tokens, u = case(trees, vocab, seed=len(sizes), sigma=6.0 if mode == sled.SAMPLE else 2.0)
    want = check(mode, trees, logits, tokens, u if mode == sled.SAMPLE else None, 0.75 if mode == sled.SAMPLE else 1.0)
    if mode == sled.GREEDY and len(sizes) > 3 and max(sizes) > 8 and vocab > 300:
        assert max(w[0] for w in want) >= 2    # the case is about walks (draws seldom fall on a drafted token here: chains of 64 do that)


@pytest.mark.parametrize("mode", [sled.GREEDY, sled.SAMPLE], ids=["greedy", "sample"])
@pytest.mark.parametrize("requests", [1, 40])
def test_a_chain_of_64_accepted_whole(mode, requests):
    trees = [random_tree(None, 64, "chain")] * requests
    logits, tokens, u = case(trees, 20011, seed=3, follow=1.0)
    rows = torch.arange(64 * requests, device="cuda")[:-1]
    logits[rows, tokens[1:].long()] = 60.0
    want = check(mode, trees, logits, tokens, u if mode == sled.SAMPLE else None)
    assert [w[0] for w in want] == [63] * requests


def test_ties_go_to_the_lowest_id_and_the_lowest_child():
    V = 9000
    trees = [[-1, 0, 0, 0, 2, 2], [-1, 0, 0]]
    logits = torch.zeros(9, V, device="cuda")
    logits[0, [8999, 5000, 4100]] = 3.0        # a tie across pieces
    logits[2, [77, 76]] = 1.0
    tokens = torch.tensor([1, 5000, 4100, 4100, 76, 76, 1, 0, 0], dtype=torch.int32, device="cuda")
    want = check(sled.GREEDY, trees, logits, tokens, None)
    assert want[0][:2] == (2, [2, 4] + [-1] * 62) and want[1][0] == 1 and want[1][2] == 0


@pytest.mark.parametrize("mode", [sled.GREEDY, sled.SAMPLE], ids=["greedy", "sample"])
@pytest.mark.parametrize("requests", [1, 24])
def test_banned_tokens_are_never_named(mode, requests):
    """Logits of minus infinity, whole pieces of the vocabulary of them, and draws at both ends."""
    V = 40000
    rng = np.random.default_rng(2)
    trees = [random_tree(rng, 33) for _ in range(requests)]
    logits, tokens, u = case(trees, V, seed=8)
    logits[:, :12345] = -float("inf")
    logits[:, 20000:] = -float("inf")
    tokens.clamp_(12345, 19999)
    u[0::3] = 0.0
    u[1::3] = 1.0 - 2.0**-24
    want = check(mode, trees, logits, tokens, u if mode == sled.SAMPLE else None)
    assert all(12345 <= w[2] < 20000 for w in want)


def test_out_of_vocabulary_drafts_are_not_accepted():
    trees = [[-1, 0, 0, 1]]
    logits, tokens, _ = case(trees, 500, seed=4)
    tokens[1], tokens[2] = -1, 500
    want = check(sled.GREEDY, trees, logits, tokens, None)
    assert want[0][0] == 0


@pytest.mark.parametrize("mode", [sled.GREEDY, sled.SAMPLE], ids=["greedy", "sample"])
def test_a_chain_walks_like_sled_accept(mode):
    """Greedy: the chain rule of sled_accept.  Sampling: the same with a drafter that is certain of its draft, whose accept test and
    residual leave the target's distribution; here only that both end at the first node whose draw is another token."""
    k, V = [8, 3, 0, 15, 6], 8192
    trees = [random_tree(None, n + 1, "chain") for n in k]
    logits, tokens, u = case(trees, V, seed=6)
    a, path, o = run(mode, trees, logits, tokens, u)
    if mode == sled.GREEDY:
        T = sum(k) + len(k)
        ws = sled.workspace(sled.sled_accept_workspace_bytes(len(k), T, V))
        a2, o2 = torch.empty_like(a), torch.empty_like(o)
        sled.sled_accept(sled.GREEDY, k, V, 1.0, logits, tokens, None, None, None, a2, o2, ws)
        torch.cuda.synchronize()
        assert torch.equal(a, a2) and torch.equal(o, o2)
    for i in range(len(k)):
        assert path[i, : int(a[i])].tolist() == list(range(1, int(a[i]) + 1))


def test_draws_follow_the_targets_distribution():
    """Chi-square of the first token over 4096 trees with the same root row: 15 degrees of freedom, 60 is far beyond chance (2e-7)."""
    V, N = 16, 1024
    g = generator(9)
    row = torch.randn(V, generator=g, device="cuda")
    counts = np.zeros(V)
    trees = [[-1, 0, 0]] * N
    for _ in range(4):
        logits = row.expand(3 * N, V).contiguous()
        tokens = torch.randint(0, V, (3 * N,), generator=g, device="cuda", dtype=torch.int32)
        u = torch.rand(3 * N, generator=g, device="cuda")
        a, path, o = run(sled.SAMPLE, trees, logits, tokens, u, 1.0)
        tk = tokens.view(N, 3)
        first = torch.where(a > 0, tk[torch.arange(N, device="cuda"), path[:, 0].clamp_min(0).long()], o)
        counts += np.bincount(first.cpu().numpy(), minlength=V)
    e = torch.softmax(row.double(), dim=0).cpu().numpy() * 4 * N
    assert ((counts - e) ** 2 / e).sum() < 60.0


@pytest.mark.parametrize("mode", [sled.GREEDY, sled.SAMPLE], ids=["greedy", "sample"])
@pytest.mark.parametrize("sizes,vocab", [([9, 3], 30000), ([64] * 40, 32000)], ids=["few_rows", "many_rows"])
def test_captured_and_replayed(mode, sizes, vocab):
    trees = [random_tree(np.random.default_rng(1), n) for n in sizes]
    logits, tokens, u = case(trees, vocab, seed=1)
    B, T = len(trees), sum(sizes)
    ws = sled.workspace(sled.sled_accept_tree_workspace_bytes(B, T, vocab))
    a, o = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    path = torch.zeros(B, sled.TREE_MAX, dtype=torch.int32, device="cuda")
    call = lambda: sled.sled_accept_tree(mode, sizes, trees, vocab, 1.0, logits, tokens, u, a, path, o, ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (2, 3, 4):
        l2, t2, u2 = case(trees, vocab, seed=seed)
        logits.copy_(l2), tokens.copy_(t2), u.copy_(u2)
        want = run(mode, trees, logits, tokens, u)
        a.zero_(), path.zero_(), o.zero_(), ws.random_(0, 255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((a, path, o), want))


def test_workspace_is_asked_for_what_is_used():
    trees = [[-1, 0, 0]] * 3
    logits, tokens, u = case(trees, 1000, seed=1)
    need = sled.sled_accept_tree_workspace_bytes(3, 9, 1000)
    ws = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    run(sled.SAMPLE, trees, logits, tokens, u, ws=ws[:need])
    assert bool((ws[need:] == 0x5A).all())
    with pytest.raises(sled.SledError):
        run(sled.SAMPLE, trees, logits, tokens, u, ws=ws[: need - 256])


def test_helpers_depth():
    assert depths([-1, 0, 0, 1, 3]) == [0, 1, 1, 2, 3] and synth.SHAPES
