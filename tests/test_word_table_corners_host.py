"""Workspaces and refusals of the word-table operators at the borders of what they take: everything is found on the host."""
import ctypes

import pytest
import torch

from paper_1409_5402_amd import binding
from test_word_tables_host import B, F, H, rows


def workspace(n, v, w, type=F):
    got = ctypes.c_size_t()
    assert binding.load().same_lda_embed_grad_workspace(ctypes.byref(rows(rows=n, width=w, type=type)), ctypes.byref(rows(rows=v, width=w, type=type)), ctypes.byref(got)) == 0
    return got.value


def test_a_gradient_of_no_tokens_needs_no_workspace():
    """Whatever the table's size: it is a table of zeros, and takes no sort."""
    for v, w in [(1, 1), ((1 << 30) - 1, 1), (1 << 30, 1), ((1 << 31) - 1, 1), (1 << 25, 4096), ((1 << 31) - 1, 1 << 20)]:
        for type in (F, B, H):
            assert workspace(0, v, w, type) == 0


def test_a_gradient_in_one_launch_stays_below_the_largest_grid():
    """Up to 8192 tokens need no workspace where they are taken in one launch, with 1024 threads for every 256 words and 64 chunks of a
    row at least; a launch has fewer than 2^32."""
    for v in [(1 << 30) - 1024, (1 << 30) - 257, (1 << 30) - 256, (1 << 30) - 255, (1 << 30) - 1, 1 << 30, (1 << 29) - 1, (1 << 29) - 128, (1 << 28) - 1, (1 << 28) - 257, (1 << 22) - 1]:
        for w in (1, 64, 65, 128, 129, 256, 1 << 14, 1 << 20):
            if workspace(5, v, w) == 0:
                assert -(-v // 256) * -(-w // 64) * 1024 < 1 << 32, (v, w)
    assert workspace(8192, 4_000_000, 64) == 0 and workspace(5, (1 << 30) - 1024, 1) == 0          # and is not left without need


def test_tensors_and_microscaled_matrices_are_told_apart():
    """Where one is given for the other, the call says so."""
    x, t = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    q = binding.MicroMatrix(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8), 8)
    for call in (lambda: binding.micro_product(x, x), lambda: binding.micro_product(q, x), lambda: binding.micro_product(torch.zeros(100, 8), x), lambda: binding.micro_dequantize(x),
                 lambda: binding.embed_grad(q, t, 5), lambda: binding.micro_quantize(q)):
        with pytest.raises(TypeError, match="MicroMatrix"):
            call()


def test_gradients_without_a_row_are_refused():
    with pytest.raises(ValueError, match="grad has shape"):
        binding.embed_grad(torch.tensor(1.0), torch.tensor(1), 5)
    with pytest.raises(ValueError, match="grad has shape"):
        binding.embed_grad(torch.zeros(4), torch.zeros(4, dtype=torch.int64), 5)


def test_many_words_are_not_scanned_by_a_workgroup_each_beyond_8192_tokens():
    """A workgroup of the one launch reads the whole list for 256 words: 16,384 tokens into a million words took 143 us, 61 by the sort."""
    for v, n, w, one_launch in [(1 << 18, 16_384, 16, True), ((1 << 18) + 1, 16_384, 16, False), ((1 << 18) + 1, 8193, 128, False), ((1 << 18) + 1, 8193, 129, True), (1_000_000, 8192, 16, True),
                                (1_000_000, 16_000, 16, False), (2000, 16_385, 16, False)]:
        assert (workspace(n, v, w) == 0) == one_launch, (v, n, w)
