"""Workspaces and refusals of the word-table operators at the borders of what they take: everything is found on the host."""
import ctypes


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
