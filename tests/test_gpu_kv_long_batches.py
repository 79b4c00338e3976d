"""Attention of batches of thousands of sequences: a workgroup finds its run among all their lengths."""
import pytest
import torch

from test_gpu_kv import attention_case, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [64, 65, 128, 4096, 5001])
def test_single_tokens_of_many_sequences(lib, margin, n):
    """Uneven contexts, sequences without rows among them and at both ends."""
    new = [int(i % 5 != 0 and i + 1 < n) for i in range(n)]
    b, k, v, gen = make(n, 1, 32, 16, [(37 * i) % 90 for i in range(n)], new)
    attention_case(lib, margin, b, k, v, gen, 4)


def test_pieces_of_many_sequences(lib, margin):
    """Tiles of many query rows, a chain's row tiles counted by the formula."""
    n = 700
    new = [(0, 1, 3, 0, 20)[i % 5] if i != 333 else 150 for i in range(n)]
    b, k, v, gen = make(7, 1, 32, 16, [(29 * i) % 150 for i in range(n)], new)
    attention_case(lib, margin, b, k, v, gen, 4)


def test_trees_of_many_sequences(lib, margin):
    n = 600
    b, k, v, gen = make(9, 2, 32, 16, [(31 * i) % 70 for i in range(n)], [(i * 7) % 12 for i in range(n)], "tree")
    attention_case(lib, margin, b, k, v, gen, 8)
