"""The product with grouped four-bit integers in every form of its kernels, for every pair of a type of rows and a size of groups, and of
positive numbers: every element of every result is compared, with inputs and bounds that are finite.

Tolerance, u = 2^-24: products of 16-bit numbers are exact, rows in binary32 are three of them; each of a group's N = G (3 G) additions is taken
to be off by a whole step, 2 u, and two fused additions per group by u: (2 N + 2 groups) u times the sum over groups of (15 |s| + |b|) sum |a|.
Then come the scale, u, and the output's type, eps / 2 with half of its least subnormal number as the floor."""
import numpy as np
import pytest
import torch

from oracle import word_rows as wr
from paper_1409_5402_amd import binding

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
PAIRS = [(t, g) for t in TYPES for g in (32, 64, 128)]


def numbers(rows, cols, positive, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(rows, cols, device=DEV, generator=g)
    return torch.exp(1.5 * x) / cols ** 0.5 if positive else x * torch.exp(0.5 * torch.randn(cols, device=DEV, generator=g))


def sizes(x, q):
    """The sum over groups of (15 |s| + |b|) sum |a| for every element of the product."""
    groups = q.scales.shape[1]
    A = torch.nn.functional.pad(x.double().abs(), (0, groups * q.group - x.shape[1])).view(len(x), groups, q.group).sum(2)
    return A @ (15.0 * q.scales[:, :, 0].double().abs() + q.scales[:, :, 1].double().abs()).t().contiguous()


def compare(x, q, want, size, scale):
    """Into every output type, strided rows in a larger buffer that stays as it was otherwise."""
    M, N = want.shape
    n = q.group * (3 if x.dtype == torch.float32 else 1)
    extra = abs(scale) * (2 * n + 2 * q.scales.shape[1]) * U * size
    assert torch.isfinite(x).all() and torch.isfinite(q.scales).all() and torch.isfinite(size).all()
    for out in TYPES.values():
        f = torch.finfo(out)
        bound = 1.01 * extra + (f.eps / 2 + 1.01 * U) * (want.abs() + extra) + f.smallest_normal * f.eps / 2
        assert ((want.abs() + bound) < f.max).all()
        buffer = torch.full((M * (N + 3) + 300,), 7.0, dtype=out, device=DEV)
        got = torch.as_strided(buffer, (M, N), (N + 3, 1), 1)
        binding.group_product(x, q, scale, out=got)
        bad = ~((got.double() - want).abs() <= bound)
        assert not bad.any(), (out, int(bad.sum()), torch.argwhere(bad)[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist())
        got.fill_(7.0)
        assert torch.all(buffer == 7.0)


# Rows of a x rows of b x width, and what they go in.  Few rows: the blocks of 128 elements in a wave and the waves that share a row; tiles: rows of
# a x of b of a workgroup, in binary32 and in 16 bits, with one trip, two or many.
FORMS = [(1, 40, 100), (3, 130_000, 128), (5, 40, 100),                                   # 1 block, 1 wave
         (4, 33, 250), (2, 50_000, 200), (13, 50, 300), (9, 300, 1000), (33, 31, 513),    # 2 blocks, 1, 2, 4 and 8 waves
         (3, 70, 1300), (16, 300, 2048), (100, 90, 300),
         (2, 130, 4000), (9, 257, 3000), (16, 1500, 4096),                                # 4 blocks, 8 waves
         (520, 49_200, 130), (513, 49_201, 1030),                                         # 64 x 256, 64 x 256
         (130, 99_000, 70), (65, 40_001, 200), (70, 17_000, 3000),                        # 32 x 128, 64 x 256 and 64 x 128
         (50, 12_001, 1100), (40, 9001, 4200),                                            # 32 x 128, 64 x 64
         (20, 131_100, 70), (20, 33_000, 700), (31, 17_000, 2050),                        # 32 x 128, 32 x 128
         (35, 5003, 4300), (40, 6400, 2000), (17, 9000, 4097),                            # 32 x 64, 32 x 64
         (33, 700, 4200),                                                                 # 16 x 64, 32 x 64
         (7, 300, 4300), (1, 4099, 8200), (16, 33_000, 4500)]                             # 16 x 64, 16 x 128


@pytest.mark.parametrize("positive", [False, True])
@pytest.mark.parametrize("dtype, group", PAIRS)
@pytest.mark.parametrize("M, N, K", FORMS)
def test_every_form_for_every_type_and_size_of_groups(M, N, K, dtype, group, positive):
    """Against the product in double, on the device, with what the table stands for in double."""
    x = numbers(M, K, positive, M + K).to(TYPES[dtype])
    q = binding.group_quantize(numbers(N, K, positive, N + group), group)
    e = torch.arange(K, device=DEV)
    at = e % 128                                             # word 4 (at % 32 // 8) + at // 32, half byte at % 8 // 2, the odd ones four on
    half = at % 8 // 2 + 4 * (at % 2)
    codes = q.codes[:, e // 128 * 64 + 4 * (4 * (at % 32 // 8) + at // 32) + half // 2]
    code = torch.where(half % 2 == 1, codes >> 4, codes & 15)
    w = code.double() * q.scales[:, :, 0].double().repeat_interleave(group, 1)[:, :K] + q.scales[:, :, 1].double().repeat_interleave(group, 1)[:, :K]
    compare(x, q, -0.25 * (x.double() @ w.t().contiguous()), sizes(x, q), -0.25)


@pytest.mark.parametrize("dtype, group", PAIRS)
@pytest.mark.parametrize("M, N, K", [(1, 1, 1), (1, 16, 128), (1, 17, 129), (3, 5, 31), (5, 33, 250), (6, 40, 96), (13, 100, 300), (16, 64, 256), (17, 31, 130), (31, 65, 512), (33, 20, 200), (64, 48, 384), (65, 130, 64),
                                     (130, 70, 160), (1, 17, 4101), (17, 31, 4130), (33, 20, 4200), (65, 130, 4097), (130, 70, 4224)])
def test_positive_numbers_against_the_oracle(M, N, K, dtype, group):
    """Rounded by the oracle too, and summed by it in double: nothing cancels, and no element is left out."""
    x, w = numbers(M, K, True, M).to(TYPES[dtype]), numbers(N, K, True, N)
    q = binding.group_quantize(w, group)
    want, size = wr.group_product(x.double().cpu().numpy(), *wr.group_quantize(w.double().cpu().numpy(), group), 1.5)
    compare(x, q, torch.from_numpy(want).to(DEV), torch.from_numpy(size).to(DEV) / 1.5, 1.5)
