"""One device's tree against the room that the verifier was given, on the CPU."""
import pytest

from paper_2506_09397_amd import serving
from test_serving_host import ToyVerifier, toy_truth
from test_serving_trees_host import ToyTrees


class Tight(ToyTrees):
    """Buffers for trees of so many nodes."""

    def __init__(self, nodes_max):
        super().__init__()
        self.nodes_max = nodes_max

    def verify_tree(self, reqs, parents, tokens):
        assert all(len(p) <= self.nodes_max for p in parents), "more rows than the buffers have"
        return super().verify_tree(reqs, parents, tokens)


@pytest.mark.parametrize("nodes_max", [1, 2, 5, 63])
def test_a_large_tree_is_cut_and_the_others_of_its_batch_are_answered(nodes_max):
    v = Tight(nodes_max)
    s = serving.Server(v, 3, device="cpu", trees=True)
    for d in range(3):
        s.open(d)
    t = toy_truth([5], 80)
    s.submit(0, 0, 5, t[:1])
    s.submit(1, 0, 5, t[:70])                                     # a chain longer than any tree
    s.submit(2, 0, 5, [(t[0] + 1) % 97, t[0]] + t[1:40], parents=[0, 0] + list(range(2, 41)))
    answers = s.run_batch()
    assert [r.device for r in answers] == [0, 1, 2]
    assert answers[0].accept_len == min(1, nodes_max - 1) and answers[1].accept_len == nodes_max - 1
    assert answers[2].accept_len == max(0, min(40, nodes_max - 2)) and answers[2].path == list(range(2, 2 + answers[2].accept_len))
    for r in answers:
        assert v.ctx[s.req_of[r.device]] == [5] + t[: r.accept_len] and r.out_token == t[r.accept_len]


def test_a_verifier_without_a_limit_takes_the_largest_trees():
    s = serving.Server(ToyTrees(), 1, device="cpu", trees=True)
    s.open(0)
    t = toy_truth([5], 80)
    s.submit(0, 0, 5, t[:70])
    assert s.run_batch()[0].accept_len == 63


@pytest.mark.parametrize("trees", [False, True])
def test_token_ids_that_no_step_can_take_are_refused_where_they_come_in(trees):
    """... and not when the batch they are in has left the queue."""
    s = serving.Server(ToyTrees() if trees else ToyVerifier(), 2, device="cpu", trees=trees)
    for d in range(2):
        s.open(d)
    t = toy_truth([5], 3)
    s.submit(0, 0, 5, t[:2])
    for pending, drafts in ((5, [1, 2**31]), (5, [-(2**31) - 1]), (2**40, [])):
        with pytest.raises(ValueError, match="32 bits"):
            s.submit(1, 0, pending, drafts)
    s.submit(1, 0, 5, [t[0]])
    assert [r.accept_len for r in s.run_batch()] == [2, 1]
