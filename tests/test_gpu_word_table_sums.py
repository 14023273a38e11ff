"""Sums of the gradient by word: the order they are taken in and how far that lets them be off.

How far a gradient may be off follows from how its sum is cut.  A binary32 sum in which every term passes at most d additions is
off by at most d u times the sum of the terms' magnitudes, u = 2^-24 (to first order; 1.01 covers the rest).  Of a word's t tokens:

  up to 64                    one chain:                                               d = t
  more, in one launch         pieces of p = max(16, 8 ceil(t / 2048)) tokens, 16 sums
                              of every 16th of them, those in pairs:                   d = p + ceil(ceil(t / p) / 16) + 4
  more, by sorted tokens      r <= t / 64 + 2 sums of at most 64 tokens, in order:     d = 64 + r
                              or, more than 32 of them, 128 parts of those, in pairs:  d = 64 + ceil(r / 128) + 7

Then comes one product with the scale and one rounding to the output's type, u + eps/2 of the value."""
import numpy as np
import pytest
import torch

from oracle import word_tables as wt
from paper_1409_5402_amd import binding
from test_gpu_word_tables import DEV, TYPES, U, close, guarded, numbers_of, words

pytestmark = pytest.mark.gpu


def one_launch(n, width, dtype):
    """Whether the gradient is taken without a sort (of few words): its workspace is empty."""
    return n <= (16384 if width * torch.finfo(dtype).bits // 8 <= 2048 else 8192)


def depth(t, few):
    t = np.asarray(t, np.int64)
    if few:
        p = np.maximum(16, 8 * -(-t // 2048))
        cut = p + -(-(-(-t // p)) // 16) + 4
    else:
        r = t // 64 + 2
        cut = 64 + np.where(r <= 32, r, -(-r // 128) + 7)
    return np.where(t <= 64, t, np.minimum(t, cut))


@pytest.mark.parametrize("n, width", [(16_384, 512), (16_384, 66), (16_384, 8), (8192, 520), (9001, 520), (16_385, 24), (70_000, 16)])
@pytest.mark.parametrize("every", [16, 64, 250, 1024])
def test_long_runs_are_summed_in_short_chains(n, width, every):
    """A one, then 2^-25 until the next one: a chain of m additions that begins with the one loses (m - 1) 2^-25."""
    g = torch.full((n, width), 2.0 ** -25, device=DEV)
    g[::every] = 1.0
    ones = -(-n // every)
    want = ones + (n - ones) * 2.0 ** -25                                     # exact in binary64
    got = binding.embed_grad(g, torch.ones(n, dtype=torch.int64, device=DEV), 3)
    bound = 1.01 * U * float(depth(n, one_launch(n, width, torch.float32))) * want + U * want
    assert torch.all(got[[0, 2]] == 0)
    far = (got[1].double() - want).abs().max().item()
    assert far <= bound, (far / (U * want), bound / (U * want))


@pytest.mark.parametrize("n, V, width", [(65, 1, 8), (1000, 3, 300), (5000, 40, 1000), (8000, 3, 300), (12_000, 5, 66), (16_000, 5, 66), (16_384, 700, 6), (16_385, 700, 6), (20_000, 3, 130),
                                         (30_000, 40, 257), (200_000, 5, 16)])
@pytest.mark.parametrize("grad", TYPES)
def test_gradient_within_what_its_cuts_allow(n, V, width, grad):
    rng = np.random.default_rng(n + width)
    G = numbers_of(rng, n, width, TYPES[grad])
    t = words(rng, n, V, "skewed")
    got = binding.embed_grad(G.to(DEV), torch.from_numpy(t).to(DEV), V, -0.75, dtype=torch.float32)
    want, size, terms = wt.embed_grad(G.double().numpy(), t, V, -0.75)
    close(got, want, torch.float32, 1.01 * U * depth(terms, one_launch(n, width, TYPES[grad]))[:, None] * size)


# the cut of a run has to be the same for rows in chunks of eight, four, two and one elements, a row per 64 lanes to a row per lane
@pytest.mark.parametrize("n, V, width", [(300, 2, 64), (5000, 3, 64), (16_384, 2, 256), (8192, 3, 520), (8000, 9, 48), (16_000, 5, 16), (3000, 2, 8), (3000, 2, 4), (16_385, 3, 64), (60_000, 5, 16),
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
