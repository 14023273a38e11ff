"""Calls at the borders of what the word-table operators take."""
import numpy as np
import pytest
import torch

from helpers import csc_from_dense
from paper_1409_5402_amd import binding
from test_gpu_word_tables import DEV, TYPES, guarded

pytestmark = pytest.mark.gpu


def test_gradient_of_no_tokens_into_large_tables():
    """Zeros, also where rows and their width are beyond what one launch of a workgroup per 256 words takes."""
    none = torch.zeros(0, dtype=torch.int64, device=DEV)
    for rows, width in ((1 << 30, 1), ((1 << 31) - 1, 1), (1 << 24, 100)):
        out = torch.ones((rows, width), dtype=torch.bfloat16, device=DEV)
        binding.embed_grad(out[:0], none, out=out, accumulate=True)
        assert bool(torch.all(out[-1] == 1.0)) and bool(torch.all(out[0] == 1.0))
        binding.embed_grad(out[:0], none, out=out, scale=-2.0)
        assert out.count_nonzero().item() == 0
        del out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width, stride, offset", [(8, 8, 0), (50, 50, 0), (50, 53, 1), (1, 3, 2), (1032, 1040, 8)])
def test_gradient_of_no_tokens_fills_rows_only(width, stride, offset, dtype):
    out, check = guarded(37, width, TYPES[dtype], stride, offset)
    for grad in TYPES.values():
        out.fill_(3.0)
        binding.embed_grad(torch.zeros(0, width, dtype=grad, device=DEV), torch.zeros(0, dtype=torch.int32, device=DEV), out=out)
        assert torch.all(out == 0.0)
    check()


def test_gradient_of_few_tokens_into_the_longest_tables():
    """The last table that a launch of a workgroup per 256 words takes, and the first ones that go by way of the sort."""
    for rows in ((1 << 30) - 257, (1 << 30) - 1, 1 << 30):
        t = torch.tensor([rows - 1, 0, rows, rows - 1, -1, 77], device=DEV)
        g = torch.tensor([[1.0], [2.0], [50.0], [4.0], [60.0], [8.0]], device=DEV)
        out = torch.ones((rows, 1), dtype=torch.bfloat16, device=DEV)
        binding.embed_grad(g, t, out=out)
        assert out[rows - 1].item() == 5.0 and out[0].item() == 2.0 and out[77].item() == 8.0 and out.count_nonzero().item() == 3
        del out


def test_microscaled_outputs_are_refused():
    x, t = torch.zeros(4, 8, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV)
    q = binding.micro_quantize(x)
    for call in (lambda: binding.embed(x, t, out=q), lambda: binding.embed_grad(x, t, out=q), lambda: binding.micro_dequantize(q, out=q),
                 lambda: binding.micro_product(x, q, out=binding.micro_quantize(torch.zeros(4, 4, device=DEV)))):
        with pytest.raises(TypeError, match="MicroMatrix"):
            call()


def test_gradient_of_rows_that_share_memory_or_are_not_contiguous():
    """What torch's backward passes hand on: of a sum the expanded gradient, of a transposed result a transposed one."""
    t = torch.tensor([[1, 2, 3], [3, -1, 0]], device=DEV)
    row = torch.arange(1.0, 6.0, device=DEV)
    for shape, ids in (((6, 5), t.view(6)), ((2, 3, 5), t)):
        for g in (row.expand(shape), torch.tensor(1.0, device=DEV).expand(shape), torch.zeros(2, 1, 1, device=DEV).add(row[:2].view(2, 1, 1)).expand(2, 3, 5).reshape(shape),
                  torch.randn(5, 6, device=DEV).t().reshape(shape) if len(shape) == 3 else torch.randn(5, 6, device=DEV).t(), torch.randn(6, 10, device=DEV)[:, ::2].view(shape)):
            assert torch.equal(binding.embed_grad(g, ids, 4), binding.embed_grad(g.contiguous(), ids, 4))
    one = torch.randn(1, 10, device=DEV)[:, ::2]
    assert torch.equal(binding.embed_grad(one, torch.tensor([2], device=DEV), 3)[2], one[0])
    x = torch.randn(4, 5, device=DEV, requires_grad=True)
    (x[t.view(6).clamp(min=0)] * (t.view(6, 1) >= 0)).sum().backward()
    assert torch.equal(binding.embed_grad(torch.ones((), device=DEV).expand(6, 5), t.view(6), 4), x.grad)


def test_autograd_sees_constants_and_rewritten_outputs():
    """Results have no gradient function, as the docstrings say; what a call writes into an `out` that a backward pass has kept ends that
    pass with torch's error, not with a wrong gradient."""
    T = torch.randn(6, 8, device=DEV, requires_grad=True)
    t = torch.tensor([1, 5, 0], device=DEV)
    q = binding.micro_quantize(T)
    for y in (binding.embed(T, t), binding.embed_grad(T, torch.arange(6, device=DEV), 6), binding.micro_product(T, q), binding.micro_dequantize(q)):
        assert y.grad_fn is None and not y.requires_grad
    for call in (lambda out: binding.embed(T, t, out=out), lambda out: binding.embed_grad(T, torch.arange(6, device=DEV), out=out[:6]), lambda out: binding.embed_grad(T, torch.arange(6, device=DEV), out=out, accumulate=True),
                 lambda out: binding.micro_dequantize(q[:3], out=out), lambda out: binding.micro_product(T[:3], binding.micro_quantize(torch.ones(8, 8, device=DEV)), out=out)):
        out = torch.randn(3, 8, device=DEV)
        x = torch.ones(3, 8, device=DEV, requires_grad=True)
        y = (x * out).sum()                                                    # keeps out for x's gradient
        call(out)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    with torch.inference_mode():
        out = torch.empty(3, 8, device=DEV)
    binding.embed(T, t, out=out)
    assert torch.equal(out, T.detach()[t])
    X = csc_from_dense(np.array([[1, 2, 0], [0, 3, 1]]))
    model = binding.SameLDA(X.D, X.V, X.colptr, X.rowidx, X.val, 4, 0.1, 0.01, seed=1, m0=5)
    phi = torch.ones(3, 4, device=DEV)
    y = (torch.ones(3, 4, device=DEV, requires_grad=True) * phi).sum()
    model.get(binding.PHI, out=phi)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    model.close()
