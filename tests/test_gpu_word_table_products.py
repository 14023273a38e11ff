"""The product of four-bit matrices in every form of its kernel and every output type, on numbers whose sums are exact."""
import numpy as np
import pytest
import torch

from oracle import word_tables as wt
from test_gpu_word_tables import DEV, TYPES, guarded, micro, random_micro
from paper_1409_5402_amd import binding

pytestmark = pytest.mark.gpu


def numbers_on_device(codes, scales, width):
    """What codes and scales stand for, in binary64, by the list of sizes."""
    codes, scales = torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV)
    size = torch.tensor(np.concatenate((wt.SIZES, -wt.SIZES)), dtype=torch.float64, device=DEV)
    half = torch.stack((codes & 15, codes >> 4), dim=2).flatten(1).long()
    return (size[half] * torch.exp2(scales.double() - 127).repeat_interleave(wt.BLOCK, dim=1))[:, :width].contiguous()


# tiles of 256 x 256 (8, 9, 33 and 64 groups of 128 elements), of 128 x 128 in two stages and in one, of 64 x 64; remainders of rows,
# of columns and of groups
FORMS = [(4096, 4096, 1024), (4100, 4152, 1100), (3900, 4300, 4224), (4096, 4096, 8192), (4352, 3841, 1152), (1500, 3000, 640), (1536, 2048, 900), (2050, 33_000, 200), (2100, 33_000, 100), (520, 712, 1500),
         (512, 512, 384), (17, 70_000, 1100), (64, 40_000, 2048), (40, 300_000, 100), (64, 140_000, 256), (300, 30_000, 1024), (20, 8192, 1152), (31, 8300, 1300), (25, 16_385, 512),
         (16, 4100, 1024), (9, 4096, 1152), (3, 40_000, 1280), (32, 180_000, 384)]


@pytest.mark.parametrize("M, N, K", FORMS)
def test_every_form_and_output_type_is_exact(M, N, K):
    """Scales of one: every sum is a multiple of 1/4 below 2^22, exact in binary32 in any order, and rounded once to the output's type."""
    rng = np.random.default_rng(M + 3 * N + K)
    a, b = random_micro(rng, M, K, 127, 128), random_micro(rng, N, K, 127, 128)
    a[1][::3, 0], b[1][::5, (K - 1) // 32] = 126, 128                # (and a few of a half and of two: multiples of 1/8 below 2^21)
    want = numbers_on_device(*a, K) @ numbers_on_device(*b, K).t()
    assert float(want.abs().max()) < 2 ** 21 and torch.equal(want.float().double(), want)
    qa, qb = micro(*a, K), micro(*b, K)
    for dtype in TYPES.values():
        rounded = want.float().to(dtype)
        for stride, offset in ((-(-N // 8) * 8, 8), (N + 5, 3)):          # stores of 16 bytes, and of an element each
            got, check = guarded(M, N, dtype, stride, offset)
            binding.micro_product(qa, qb, out=got)
            assert torch.equal(got, rounded), (dtype, stride, torch.nonzero(got != rounded)[:5])
            check()
            del got


@pytest.mark.parametrize("M, N, K", [(16, 4096, 1024), (16, 5000, 1024), (9, 40_000, 1152), (1, 33_000, 1025), (12, 4200, 1280), (3, 33_000, 5000), (16, 70_000, 500)])
def test_rounding_in_the_call_gives_the_same_bits(M, N, K):
    """Whole rows per wave, quarters, 16 and 64 rows of the table: the form does not depend on where `a` is rounded."""
    rng = np.random.default_rng(M + N + K)
    b = micro(*random_micro(rng, N, K, 120, 130), K)
    for dtype in TYPES.values():
        x = torch.from_numpy(rng.normal(size=(M, K))).to(dtype).to(DEV)
        assert torch.equal(binding.micro_product(x, b, 0.5, dtype=dtype), binding.micro_product(binding.micro_quantize(x), b, 0.5, dtype=dtype))
