"""What callers of the 8-bit layer, the choice of tokens and the reordering of states may rely on, as far as no GPU is needed."""
import random

import pytest

from paper_2002_02645_amd import binding


def test_a_choice_s_workspace_serves_smaller_calls():
    f = binding.freeze_beam_workspace_bytes
    for beams, vocab, k in ((4, 32000, 4), (1, 131072, 16), (8, 50257, 8), (64, 1000, 64), (3, 1, 1), (5, 1025, 7)):
        sizes = [f(g, beams, vocab, k) for g in list(range(1, 1200)) + [2000, 4000, 5000, (1 << 20) // beams]]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), (beams, vocab, k)
    rng = random.Random(3)
    for _ in range(3000):
        g, beams, vocab, k = rng.randint(1, 2000), rng.randint(1, 64), int(2 ** rng.uniform(0, 18)), rng.randint(1, 64)
        most = f(g, beams, vocab, k)
        assert most >= f(rng.randint(1, g), rng.randint(1, beams), rng.randint(1, vocab), rng.randint(1, k)) > 0
