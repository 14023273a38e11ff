"""Refusals of the word-table operators: everything here is found on the host, before any device call."""
import ctypes

import pytest
import torch

from paper_1409_5402_amd import binding

EINVAL = -1
F, B, H, M = 0, 1, 2, 3
P = 1 << 20        # an address that is only looked at


class Rows(ctypes.Structure):
    """same_lda_rows, field by field."""
    _fields_ = [("data", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64), ("stride", ctypes.c_int64), ("width", ctypes.c_int32), ("type", ctypes.c_int32)]


def rows(rows=4, width=8, type=F, stride=None, data=P, scales=None):
    return Rows(data, scales if scales is not None else (P if type == M else None), rows, width if stride is None else stride, width, type)


def refused(rc, *words):
    assert rc == EINVAL
    text = binding.load().same_lda_last_error(None).decode()
    for w in words:
        assert w in text, text


BAD_MATRICES = [
    (dict(type=4), "unknown type"), (dict(type=-1), "unknown type"), (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(width=0), "elements"),
    (dict(width=(1 << 20) + 1), "elements"), (dict(stride=7), "stride"), (dict(stride=1 << 61), "stride"), (dict(data=None), "no data"), (dict(data=P + 2), "aligned"),
    (dict(type=M, data=P + 8), "aligned"), (dict(type=M, scales=P + 2), "aligned"), (dict(type=M, scales=0), "no data"),
]


@pytest.mark.parametrize("bad, word", BAD_MATRICES)
def test_bad_matrices_are_refused_by_every_operator(bad, word):
    L = binding.load()
    m = rows(**bad)
    ok, okm = rows(), rows(type=M)
    ref = ctypes.byref
    n = ctypes.c_size_t()
    refused(L.same_lda_embed(ref(m), P, 4, 1.0, ref(ok), None), word)
    refused(L.same_lda_micro_product(ref(m), ref(okm), 1.0, ref(ok), None), word)
    if bad.get("type") != M:
        refused(L.same_lda_embed(ref(ok), P, 4, 1.0, ref(m), None), word)
        refused(L.same_lda_embed_grad(ref(m), P, 4, 1.0, 0, ref(ok), P, 1 << 30, None), word)
        refused(L.same_lda_embed_grad(ref(ok), P, 4, 1.0, 0, ref(m), P, 1 << 30, None), word)
        refused(L.same_lda_embed_grad_workspace(ref(m), ref(ok), ref(n)), word)
        refused(L.same_lda_micro_quantize(ref(m), ref(okm), None), word)
    else:
        refused(L.same_lda_micro_quantize(ref(ok), ref(m), None), word)
        refused(L.same_lda_micro_product(ref(okm), ref(m), 1.0, ref(ok), None), word)


def test_shapes_types_tokens_and_scales_are_refused():
    L, ref = binding.load(), ctypes.byref
    a, m = rows(), rows(type=M)
    n = ctypes.c_size_t()
    for call in (lambda s, tb, t: L.same_lda_embed(ref(a), t, tb, s, ref(a), None), lambda s, tb, t: L.same_lda_embed_grad(ref(a), t, tb, s, 0, ref(a), P, 1 << 30, None)):
        refused(call(float("nan"), 4, P), "finite")
        refused(call(float("inf"), 8, P), "finite")
        refused(call(1.0, 2, P), "bytes")
        refused(call(1.0, 8, P + 4), "aligned")
    refused(L.same_lda_embed(None, P, 4, 1.0, ref(a), None), "null")
    refused(L.same_lda_embed(ref(a), P, 4, 1.0, None, None), "null")
    refused(L.same_lda_embed(ref(a), P, 4, 1.0, ref(m), None), "must not be microscaled")
    refused(L.same_lda_embed(ref(a), P, 4, 1.0, ref(rows(width=7)), None), "elements")
    refused(L.same_lda_embed(ref(a), None, 4, 1.0, ref(rows(rows=3)), None), "without tokens")
    refused(L.same_lda_embed_grad(ref(a), None, 4, 1.0, 0, ref(a), P, 1 << 30, None), "null")
    refused(L.same_lda_embed_grad(ref(a), P, 4, 1.0, 0, ref(rows(width=7)), P, 1 << 30, None), "elements")
    refused(L.same_lda_embed_grad(ref(m), P, 4, 1.0, 0, ref(a), P, 1 << 30, None), "must not be microscaled")
    refused(L.same_lda_embed_grad_workspace(ref(a), ref(a), None), "null")
    many = rows(rows=50_000)
    assert L.same_lda_embed_grad_workspace(ref(many), ref(a), ref(n)) == 0 and n.value > 0
    refused(L.same_lda_embed_grad(ref(many), P, 4, 1.0, 0, ref(a), P, n.value - 1, None), "workspace")
    refused(L.same_lda_embed_grad(ref(many), P, 4, 1.0, 0, ref(a), None, n.value, None), "workspace")
    refused(L.same_lda_embed_grad(ref(many), P, 4, 1.0, 0, ref(a), P + 8, n.value, None), "workspace")
    refused(L.same_lda_micro_quantize(ref(m), ref(m), None), "must not be microscaled")
    refused(L.same_lda_micro_quantize(ref(a), ref(a), None), "must be microscaled")
    refused(L.same_lda_micro_quantize(ref(a), ref(rows(type=M, rows=5)), None), "into")
    refused(L.same_lda_micro_quantize(ref(a), ref(rows(type=M, width=9)), None), "into")
    refused(L.same_lda_micro_product(ref(m), ref(a), 1.0, ref(rows(width=4)), None), "must be microscaled")
    refused(L.same_lda_micro_product(ref(rows(rows=65)), ref(m), 1.0, ref(rows(rows=65, width=4)), None), "must be microscaled")
    refused(L.same_lda_micro_product(ref(rows(rows=2, width=8193)), ref(rows(type=M, width=8193)), 1.0, ref(rows(rows=2, width=4)), None), "must be microscaled")
    refused(L.same_lda_micro_product(ref(m), ref(rows(type=M, width=9)), 1.0, ref(rows(width=4)), None), "elements")
    refused(L.same_lda_micro_product(ref(m), ref(m), 1.0, ref(rows(width=5)), None), "do not give")
    refused(L.same_lda_micro_product(ref(m), ref(m), 1.0, ref(rows(rows=5, width=4)), None), "do not give")
    refused(L.same_lda_micro_product(ref(m), ref(m), float("nan"), ref(rows(width=4)), None), "finite")
    refused(L.same_lda_micro_product(ref(m), ref(m), 1.0, ref(m), None), "must not be microscaled")
    refused(L.same_lda_micro_size(-1, 8, ref(n), ref(n)), "shape")
    refused(L.same_lda_micro_size(1, 0, ref(n), ref(n)), "shape")
    refused(L.same_lda_micro_size(1, 8, None, ref(n)), "null")


def test_empty_calls_do_nothing():
    L, ref = binding.load(), ctypes.byref
    e, a = rows(rows=0, data=None), rows()
    em, m = rows(rows=0, type=M, data=None, scales=0), rows(type=M)
    assert L.same_lda_embed(ref(e), None, 4, 1.0, ref(e), None) == 0
    assert L.same_lda_embed(ref(a), P, 8, 1.0, ref(e), None) == 0
    assert L.same_lda_embed_grad(ref(e), None, 4, 1.0, 1, ref(a), None, 0, None) == 0       # nothing to add
    assert L.same_lda_embed_grad(ref(a), P, 4, 1.0, 0, ref(e), None, 0, None) == 0
    assert L.same_lda_micro_quantize(ref(e), ref(em), None) == 0
    assert L.same_lda_micro_product(ref(em), ref(m), 1.0, ref(rows(rows=0, width=4, data=None)), None) == 0
    assert L.same_lda_micro_product(ref(m), ref(em), 1.0, None, None) == 0


def test_sizes_of_microscaled_matrices():
    L, ref = binding.load(), ctypes.byref
    c, s = ctypes.c_size_t(), ctypes.c_size_t()
    for r, w, code, scale in [(0, 1, 0, 0), (3, 1, 192, 12), (3, 128, 192, 12), (3, 129, 384, 24), ((1 << 31) - 1, 1 << 20, ((1 << 31) - 1) << 19, ((1 << 31) - 1) << 15)]:
        assert L.same_lda_micro_size(r, w, ref(c), ref(s)) == 0 and (c.value, s.value) == (code, scale)


def test_workspace_grows_with_the_call_and_not_by_much():
    L, ref = binding.load(), ctypes.byref
    last = 0
    for n, v, w in [(1, 1, 1), (300, 10, 64), (300, 100_000, 64), (1_000_000, 100_000, 64), (1_000_000, 100_000, 256), ((1 << 31) - 1, (1 << 31) - 1, 256)]:
        got = ctypes.c_size_t()
        assert L.same_lda_embed_grad_workspace(ref(rows(rows=n, width=w)), ref(rows(rows=v, width=w)), ref(got)) == 0
        assert last <= got.value <= 64 * (n + v) + n * w // 8 + (1 << 20)
        last = got.value


def test_binding_refuses_what_it_cannot_pass_on():
    x = torch.zeros(4, 8)
    t = torch.zeros(4, dtype=torch.int64)
    codes, scales = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8)
    q = binding.MicroMatrix(codes, scales, 8)
    assert q.shape == (4, 8) and q[1:3].shape == (2, 8) and q[1:3].codes.data_ptr() == codes.data_ptr() + 64
    for bad in [(codes[:, :32], scales, 8), (codes, scales[:, :2], 8), (codes, scales, 129), (codes, scales, 0), (codes.to(torch.int8), scales, 8), (codes[::2], scales[:2], 8), (codes, scales[:3], 8)]:
        with pytest.raises(ValueError):
            binding.MicroMatrix(*bad)
    with pytest.raises(TypeError):
        q[0]
    with pytest.raises(TypeError):
        q[::2]
    for call in (lambda: binding.embed(x, t), lambda: binding.embed_grad(x, t, 5), lambda: binding.micro_quantize(x), lambda: binding.micro_dequantize(q), lambda: binding.micro_product(q, q)):
        with pytest.raises(ValueError, match="GPU"):            # no CPU form
            call()
    with pytest.raises(TypeError):
        binding.embed(x, t.float())
    with pytest.raises(ValueError):
        binding.embed_grad(x, t[:3], 5)
    with pytest.raises(ValueError):
        binding.embed_grad(x, t)
    with pytest.raises(ValueError):
        binding.embed_grad(x, t, 5, accumulate=True)
    with pytest.raises(TypeError):
        binding._rows(x.double())
    with pytest.raises(ValueError):
        binding._rows(x.t())
    with pytest.raises(ValueError):
        binding._rows(x[0])
    for view, stride in ((x[:, 2:7], 8), (x[1:2, 2:7], 5)):
        r = Rows.from_buffer_copy(binding._rows(view))
        assert (r.data, r.scales, r.rows, r.stride, r.width, r.type) == (view.data_ptr(), None, view.shape[0], stride, 5, F)
    r = Rows.from_buffer_copy(binding._rows(q))
    assert (r.data, r.scales, r.rows, r.width, r.type) == (codes.data_ptr(), scales.data_ptr(), 4, 8, M)
