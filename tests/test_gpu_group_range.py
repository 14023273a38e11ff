"""Grouped four-bit integers at the ends of what numbers can be: rounding and reading back, and the product, against the oracle in
double (oracle/word_rows.py)."""
import numpy as np
import pytest
import torch

from oracle import word_rows as wr
from paper_1409_5402_amd import binding

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
U = 2.0 ** -24
TOP = float(torch.finfo(torch.float32).max)
GROUPS = [32, 64, 128]


# ---- rounding and reading back

def read_back(x, group):
    """The form is the oracle's, and what it stands for is finite and q s + b rounded once (2^-24); within a step of the number, or, of a
    number below the least finite bfloat16, at that."""
    width = x.shape[1]
    q = binding.group_quantize(x.to(DEV), group)
    oq, s, b = wr.group_quantize(x.double().numpy(), group)
    scales = q.scales.double().cpu().numpy()
    assert np.array_equal(scales[:, :, 0], s) and np.array_equal(scales[:, :, 1], b) and np.array_equal(q.codes.cpu().numpy(), wr.group_layout(oq))
    got, want = binding.group_dequantize(q).double().cpu().numpy(), wr.group_numbers(oq, s, b, width)
    assert np.isfinite(got).all() and (np.abs(got - want) <= U * np.abs(want)).all()
    assert (np.abs(want - x.double().numpy()) <= np.maximum(np.repeat(np.abs(s), group, axis=1)[:, :width], TOP - wr.BF16_MAX)).all()
    t = torch.arange(len(x) - 1, -1, -1, device=DEV)
    assert torch.equal(binding.embed(q, t).flip(0), binding.group_dequantize(q))
    kept = binding.embed(q, t, 0.5, drop=binding.Dropout(0.5, 3)).flip(0)
    assert torch.all((kept == 0) | (kept == binding.group_dequantize(q)))


@pytest.mark.parametrize("group", GROUPS)
def test_a_group_whose_span_is_beyond_binary32_is_read_back(group):
    """q s alone may be beyond binary32 where q s + b is not."""
    rng = np.random.default_rng(group)
    x = rng.uniform(-TOP, TOP, (9, 300))
    x[0, ::2], x[0, 1::2] = -TOP, TOP
    x[1, ::2], x[1, 1::2] = -3e38, 2e38
    x[2] = np.linspace(-TOP, TOP, 300)
    x[3:6] *= 0.99
    x[6] = np.where(rng.uniform(size=300) < 0.1, 3.2e38, -3.2e38)
    read_back(torch.from_numpy(x).float(), group)


@pytest.mark.parametrize("group", GROUPS)
def test_groups_beyond_the_last_finite_bfloat16_numbers_are_read_back(group):
    """Groups that lie wholly below the least one have a step below 0, and b + 15 s stays within binary32 there too."""
    rng = np.random.default_rng(group)
    low = -wr.BF16_MAX
    x = np.zeros((10, 300))
    x[0], x[1], x[2] = -TOP, TOP, (low - TOP) / 2
    x[3] = np.linspace(-TOP, low, 300)
    x[4] = np.linspace(-low, TOP, 300)
    x[5, ::2] = -TOP
    x[6, ::2] = TOP
    x[7] = low
    x[8] = -low
    x[9] = rng.uniform(-TOP, low, 300)
    read_back(torch.from_numpy(x).float(), group)
