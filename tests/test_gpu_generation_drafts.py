"""Drafted trees in the example of generation: right guesses are kept, in as few passes
as there can be, and the rows of a path that does not lie in front move up in the cache."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import generate
    finally:
        sys.path.pop(0)
    return generate


# (the words of a tree as places of the answer, None a wrong one; parents; the path that is right; passes for 9
# words: the prompts', then 9 - 1 by as many at a time as the path is long)
TREES = [
    ([0, 1, 2, 3, 4], [-1, 0, 1, 2, 3], [0, 1, 2, 3, 4, 5], 3),
    ([None, 0, None, 1], [-1, -1, 1, 1], [0, 2, 4], 4),
    ([None, None, 0, None, None, 1, 2], [-1, 0, -1, 2, 2, 2, 5], [0, 3, 6, 7], 3),
]


@pytest.mark.parametrize("words,parents,path,passes", TREES)
def test_right_guesses_are_kept(example, monkeypatch, words, parents, path, passes):
    model = example.Decoder(dtype=torch.float32, seed=3)  # (fp32: no two words are near enough for the sums' order to matter)
    prompts = example.batch(64, 12, 7)
    count = 9
    want = example.greedy(model, prompts, count + 5).tolist()
    kept, keep = [], example.keep

    def guesses(i, answer):
        ahead = want[i][len(answer):]
        # (a wrong word differs from all that follow, so that no other path is right)
        wrong = next(w for w in range(64) if w not in ahead)
        return [wrong if at is None else ahead[at] for at in words], parents

    def keeping(caches, old, paths):
        kept.append(paths)
        keep(caches, old, paths)

    monkeypatch.setattr(example, "keep", keeping)
    got, took = example.drafted(model, prompts, count, guesses)
    assert got.tolist() == [w[:count] for w in want]
    assert took == passes
    assert all(p == path for p in kept[0])
