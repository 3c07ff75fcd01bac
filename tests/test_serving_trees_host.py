"""Host logic of serving trees and of the cache budget against a stand-in verifier on the CPU."""
import pytest
import torch

from paper_2506_09397_amd import serving, sled
from test_serving_host import ToyShape, ToyVerifier, toy_truth


class ToyTrees(ToyVerifier):
    mass = True

    def __init__(self):
        super().__init__()
        self.cut = []
        self.size = {}

    def open_bounded(self):
        return self.open()

    def verify_tree(self, reqs, parents, tokens):
        self.calls += 1
        toks, rows, off = tokens.tolist(), [], 0
        for r, p in zip(reqs, parents):
            mine = toks[off: off + len(p)]
            self.staged[r] = mine
            for j in range(len(p)):
                way = [j]
                while way[-1]:
                    way.append(p[way[-1]])
                row = torch.zeros(ToyShape.vocab)
                row[self.f(self.ctx[r] + [mine[i] for i in reversed(way)])] = 1.0
                rows.append(row)
            off += len(p)
        return torch.stack(rows)

    def accept_tree(self, mode, parents, logits, tokens, u=None, temperature=1.0):
        assert mode == sled.GREEDY and u is None
        toks, off = tokens.tolist(), 0
        a, paths, t = [], torch.full((len(parents), sled.TREE_MAX), -1, dtype=torch.int32), []
        for i, p in enumerate(parents):
            cur, n = 0, 0
            while True:
                best = int(logits[off + cur].argmax())
                kids = [j for j in range(1, len(p)) if p[j] == cur and toks[off + j] == best]
                if not kids:
                    break
                cur = kids[0]
                paths[i, n] = cur
                n += 1
            a.append(n)
            t.append(best)
            off += len(p)
        return torch.tensor(a, dtype=torch.int32), paths, torch.tensor(t, dtype=torch.int32)

    def commit_tree(self, reqs, a, path):
        for i, r in enumerate(reqs):
            mine = self.staged.pop(r)
            self.ctx[r] += [mine[0]] + [mine[j] for j in path[i, : int(a[i])].tolist()]

    def evict(self, reqs, keep, first, recent):
        self.cut.append((list(reqs), list(keep), first, recent))


@pytest.mark.parametrize("beta,lose_every,batch,width", [(1.0, 0, 4, 1), (0.6, 3, 3, 3), (0.0, 0, 1, 2), (0.5, 2, 8, 6)])
def test_trees_end_with_the_targets_own_text(beta, lose_every, batch, width):
    v = ToyTrees()
    s = serving.Server(v, batch, device="cpu", trees=True)
    n_dev, n_new = 5, 30
    truth = {d: toy_truth([3, 1, 4][: d % 3] + [10 + d], n_new) for d in range(n_dev)}
    for d in range(n_dev):
        s.open(d, prompt=[3, 1, 4][: d % 3])
    drafters = {d: serving.TreeDrafter(truth[d], ToyShape.vocab, beta, d, width) for d in range(n_dev)}
    res = serving.simulate(s, drafters, {d: 10 + d for d in range(n_dev)}, n_new, 4, draft_ms_per_token=1.0, seed=1, lose_every=lose_every)
    assert res["devices_off_replayed_path"] == 0 and all(res["texts"][d] == truth[d] for d in range(n_dev))


def test_wider_trees_take_fewer_steps():
    def steps(width):
        v = ToyTrees()
        s = serving.Server(v, 1, device="cpu", trees=True)
        s.open(0)
        truth = toy_truth([10], 200)
        return serving.simulate(s, {0: serving.TreeDrafter(truth, ToyShape.vocab, 0.5, 0, width)}, {0: 10}, 200, 4, 1.0)["steps"]
    assert steps(4) < steps(1)


def test_tree_drafter_stays_within_a_tree():
    d = serving.TreeDrafter(list(range(100)), 500, 0.7, 0, 9)
    drafts, parents = d.draft_tree(0, 15)
    assert len(drafts) == len(parents) == 63 and all(0 <= p <= j for j, p in enumerate(parents))


def test_rounds_carry_their_paths_and_replay():
    v = ToyTrees()
    s = serving.Server(v, 2, device="cpu", trees=True)
    for d in range(2):
        s.open(d)
    t = toy_truth([5], 3)
    s.submit(0, 0, 5, [(t[0] + 1) % 97, t[0], t[1], t[1]], parents=[0, 0, 1, 2])
    s.submit(1, 0, 5, [t[0], t[1], 96 - t[2]])             # a chain is a tree too
    r = s.run_batch()
    assert r[0].path == [2, 4] and r[0].accept_len == 2 and r[0].out_token == t[2] and r[0].accepted([(t[0] + 1) % 97, t[0], t[1], t[1]]) == t[:2]
    assert r[1].path == [1, 2] and r[1].out_token == t[2]
    again = s.submit(0, 0, 5, [1])
    assert again.replayed and again.path == [2, 4]
    assert v.ctx[s.req_of[0]] == v.ctx[s.req_of[1]] == [5] + t[:2]
    s.submit(0, 1, t[2], list(range(200)))
    assert len(s.queue[-1].drafts) == sled.TREE_MAX - 1
    for bad in ([0, 2], [-1, 0], [0]):
        with pytest.raises(ValueError):
            s.submit(1, 1, 5, [1, 2], parents=bad)
    with pytest.raises(ValueError):
        serving.Server(ToyVerifier(), 1, device="cpu").submit(0, 0, 5, [1], parents=[0])


def test_budget_cuts_sessions_that_outgrow_it():
    v = ToyTrees()
    s = serving.Server(v, 2, device="cpu", trees=True, kv_budget=20, kv_first=2, kv_recent=5)
    s.open(0, prompt=list(range(19)))
    s.open(1, prompt=[1, 2, 3])
    with pytest.raises(AssertionError):
        s.open(2, prompt=list(range(21)))
    for rnd in range(2):
        s.submit(0, rnd, 5, [])
        s.submit(1, rnd, 5, [])
        s.run_batch()
    assert v.cut == [([s.req_of[0]], [15], 2, 5)] and s.length == {0: 15, 1: 5} and s.evictions == 1
    s.close(0)
    assert s.length == {1: 5}
    with pytest.raises(AssertionError):
        serving.Server(v, 2, device="cpu", kv_budget=20)
    with pytest.raises(AssertionError):
        serving.Server(v, 2, device="cpu", trees=True, kv_budget=20, kv_recent=64)
