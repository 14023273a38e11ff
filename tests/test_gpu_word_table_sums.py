"""Sums of the word-table operators: the order they are taken in."""
import numpy as np
import pytest
import torch

from paper_1409_5402_amd import binding
from test_gpu_word_tables import DEV, guarded, numbers_of, words

pytestmark = pytest.mark.gpu


def one_launch(n, width, dtype):
    """Whether the gradient is taken without a sort (of few words): its workspace is empty."""
    return n <= (16384 if width * torch.finfo(dtype).bits // 8 <= 2048 else 8192)


# the cut of a run has to be the same for rows in chunks of eight, four, two and one elements, a row per 64 lanes to a row per lane
@pytest.mark.parametrize("n, V, width", [(16_385, 3, 64), (60_000, 5, 16),
                                         (60_000, 5, 8), (200_000, 3, 4), (40_000, 3, 2), (20_000, 2, 520)])
def test_gradient_has_the_same_bits_in_every_layout(n, V, width):
    """Values that bfloat16 holds, so that all types can be given: where the path to the sums is the same, so are the bits."""
    rng = np.random.default_rng(n + width)
    G = numbers_of(rng, n, width, torch.bfloat16).to(DEV)
    t = torch.from_numpy(words(rng, n, V, "skewed")).to(DEV)
    want = binding.embed_grad(G.float(), t, V, 1.5)
    for dtype in (torch.float32, torch.bfloat16):
        if one_launch(n, width, dtype) != one_launch(n, width, torch.float32):
            continue
        for stride, offset in ((width, 0), (width, 1), (width + 1, 0), (width + 2, 2), (width + 8, 8)):
            g, _ = guarded(n, width, dtype, stride, offset)
            g.copy_(G)
            for out_stride, out_offset in ((width, 0), (width + 1, 0), (width, 1), (width + 2, 0)):
                out, check = guarded(V, width, torch.float32, out_stride, out_offset)
                binding.embed_grad(g, t, scale=1.5, out=out)
                assert torch.equal(out, want), (dtype, stride, offset, out_stride, out_offset)
                check()
        short = binding.embed_grad(G.to(dtype), t.int(), V, 1.5, dtype=torch.bfloat16)
        assert torch.equal(short, want.to(torch.bfloat16))


def test_the_widest_rows():
    """Runs that are joined by one group of lanes and by a workgroup, in more groups of columns than stand side by side in a grid."""
    n, width = 8400, (1 << 20) - 1                                            # 17.6 GB
    t = torch.zeros(n, dtype=torch.int32, device=DEV)
    t[::42] = 1
    g = torch.ones((n, width), dtype=torch.bfloat16, device=DEV)
    g[:, width - 1] = 2.0
    g[5, 524_300] = 3.0
    got = binding.embed_grad(g, t, 3, dtype=torch.float32)
    want = torch.zeros(3, width, device=DEV)
    want[0], want[1] = 8200.0, 200.0
    want[:, width - 1] *= 2.0
    want[0, 524_300] += 2.0
    assert torch.equal(got, want)
