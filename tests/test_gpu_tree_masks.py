"""stem_tree_masks against its definition: trees of every depth, words of every number, parents that are none, rows of nobody."""
import random

import pytest
import torch

from paper_2603_06274_amd import tree_binding as tb

import tree_util as tu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def whole(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def check(parents, new, past, max_new, offset, padding=0, cu=None):
    T = sum(new) + padding
    cu = cu or [sum(new[:r]) for r in range(len(new) + 1)]
    masks = torch.full((T, tb.mask_words(max_new)), 77, dtype=torch.int64, device=DEV)
    positions, status = torch.full((T,), 77, dtype=torch.int32, device=DEV), whole([5])
    flat = [p for ps in parents for p in ps] + [3] * padding
    lens = [p + n for p, n in zip(past, new)]
    args = tb.TreeShape(len(new), T, max_new, offset), whole(flat), whole(lens), whole(cu)
    tb.stem_tree_masks(*args, positions, masks, status)
    again = torch.full_like(masks, 77)
    tb.stem_tree_masks(*args, None, again, whole([0]))
    assert torch.equal(again, masks)
    masks, positions, strange, t = masks.tolist(), positions.tolist(), 5, 0
    for r, n in enumerate(new):
        sees, depth = tu.ancestors(parents[r], n)
        for i in range(n):
            if i < max_new:
                strange += not -1 <= parents[r][i] < i
                assert masks[t] == tu.words(sees[i], tb.mask_words(max_new)), (r, i)
                assert positions[t] == offset + past[r] + depth[i], (r, i)
            else:
                strange += 1
                assert set(masks[t]) == {77} and positions[t] == 77
            t += 1
    for x in range(t, T):
        assert set(masks[x]) == {77} and positions[x] == 77
    assert status.item() == strange


@pytest.mark.parametrize("max_new", [1, 2, 63, 64, 65, 128, 129, 256, 300, 512, 700, 1024])
@pytest.mark.parametrize("branch", [1, 3, 10000])
def test_trees(max_new, branch):
    rng = random.Random(max_new * 7 + branch)
    new = [max_new, 0, 1, rng.randint(1, max_new), max(max_new - 1, 0)]
    parents = [tu.random_parents(rng, n, branch) for n in new]
    check(parents, new, [rng.randint(0, 5000) for _ in new], max_new, 131072, padding=3)


def test_forests_and_parents_that_are_none():
    check([[-1, -1, 0, 1, -1, 4], [5, 1, 7, -2, 2, 1 << 30], [-(1 << 31)]], [6, 6, 1], [0, 9, 100], 6, 0)


def test_more_new_tokens_than_max_new():
    rng = random.Random(1)
    check([tu.random_parents(rng, 9, 2), tu.random_parents(rng, 70, 3)], [9, 70], [4, 4], 8, 10)


def test_no_requests_new_tokens_and_many_requests():
    rng = random.Random(2)
    new = [rng.randint(0, 3) for _ in range(3000)]
    check([tu.random_parents(rng, n, 2) for n in new], new, [rng.randint(0, 99) for _ in new], 3, 7, padding=1)
    tb.stem_tree_masks(tb.TreeShape(2, 0, 4), whole([]), whole([0, 0]), whole([0, 0, 0]), None,
                       torch.empty(0, 1, dtype=torch.int64, device=DEV), whole([0]))
