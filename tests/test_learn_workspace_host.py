"""The workspace of cross entropy stays within what the header says of it, over the whole range of sizes."""
import random

import pytest

from paper_2607_07388_amd import tfe


def up(x, to):
    return -(-x // to) * to


def stated(rows, vocab, dim):
    pitch, piece = up(dim, 64), min(up(vocab, 256), max(4096, (1 << 27) // rows))
    tiles = up(rows, 256 if rows > 128 else 128 if rows > 64 else 64)
    lists = 16 * rows + 4 * vocab + (1 << 15)  # numbers a row and a token, and what parts begin at
    return (7 * tiles * piece + 2 * piece * pitch + 4 * rows * pitch + max(1 << 26, 4 * rows * pitch)
            + 8 * min(rows, 16384) * (vocab // 128 + 33) + lists)


@pytest.mark.parametrize("size", [(1, 1, 1), (1, 151936, 1024), (64, 151936, 1024), (4096, 151936, 1024),
                                  (65536, 151936, 64), (1 << 20, 1 << 18, 16384), (1 << 20, 1, 1)])
def test_named_sizes(size):
    assert 0 < tfe.tfe_cross_entropy_workspace(*size) <= stated(*size)


def test_drawn_sizes():
    rng = random.Random(1)
    for _ in range(20000):
        size = tuple(int(most ** rng.random()) for most in (1 << 20, 1 << 18, 16384))
        assert 0 < tfe.tfe_cross_entropy_workspace(*size) <= stated(*size), size
