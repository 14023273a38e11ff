"""Refusals of dropout and of the operators on grouped integers: everything here is found on the host, before any device call."""
import copy
import ctypes
import pickle

import pytest
import torch

from paper_1409_5402_amd import binding

EINVAL = -1
F, B, H, M = 0, 1, 2, 3
GROUPS = (32, 64, 128)
P = 1 << 20        # an address that is only looked at
ref = ctypes.byref


class Rows(ctypes.Structure):
    """same_lda_rows, field by field."""
    _fields_ = [("data", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64), ("stride", ctypes.c_int64), ("width", ctypes.c_int32), ("type", ctypes.c_int32)]


class Drop(ctypes.Structure):
    """same_lda_drop, field by field."""
    _fields_ = [("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("step", ctypes.c_uint64), ("step_at", ctypes.c_void_p)]


def rows(rows=4, width=8, type=F, stride=None, data=P, scales=None):
    return Rows(data, scales if scales is not None else (P if type >= M else None), rows, width if stride is None else stride, width, type)


def refused(rc, *words):
    assert rc == EINVAL
    text = binding.load().same_lda_last_error(None).decode()
    for w in words:
        assert w in text, text


BAD_NUMBERS = [(dict(type=5), "unknown type"), (dict(type=16), "unknown type"), (dict(type=256), "unknown type"), (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(width=0), "elements"),
               (dict(width=(1 << 20) + 1), "elements"), (dict(stride=7), "stride"), (dict(stride=1 << 61), "stride"), (dict(data=None), "no data"), (dict(data=P + 2), "aligned")]


@pytest.mark.parametrize("bad, word", BAD_NUMBERS)
def test_bad_matrices_are_refused(bad, word):
    L, m, ok, g, d = binding.load(), rows(**bad), rows(), rows(type=64), Drop(0.5, 1, 2, None)
    refused(L.same_lda_dropout(ref(m), ref(d), ref(ok), None), word)
    refused(L.same_lda_dropout(ref(ok), ref(d), ref(m), None), word)
    refused(L.same_lda_embed_dropout(ref(m), P, 4, 1.0, ref(d), ref(ok), None), word)
    refused(L.same_lda_embed_dropout(ref(ok), P, 4, 1.0, ref(d), ref(m), None), word)
    refused(L.same_lda_embed_dropout_grad(ref(m), P, 4, 1.0, ref(d), 0, ref(ok), P, 1 << 30, None), word)
    refused(L.same_lda_embed_dropout_grad(ref(ok), P, 4, 1.0, ref(d), 0, ref(m), P, 1 << 30, None), word)
    refused(L.same_lda_group_quantize(ref(m), ref(g), None), word)
    refused(L.same_lda_group_product(ref(m), ref(g), 1.0, ref(ok), P, 1 << 40, None), word)


@pytest.mark.parametrize("group", GROUPS)
def test_bad_grouped_matrices_are_refused(group):
    L, ok, d = binding.load(), rows(), Drop(0.5, 1, 2, None)
    for bad, word in [(dict(data=P + 8), "aligned"), (dict(scales=P + 2), "aligned"), (dict(scales=0), "no data"), (dict(data=None), "no data"), (dict(rows=-1), "rows"), (dict(width=0), "elements")]:
        m = rows(type=group, **bad)
        refused(L.same_lda_embed(ref(m), P, 4, 1.0, ref(ok), None), word)
        refused(L.same_lda_embed_dropout(ref(m), P, 4, 1.0, ref(d), ref(ok), None), word)
        refused(L.same_lda_group_quantize(ref(ok), ref(m), None), word)
        refused(L.same_lda_group_product(ref(ok), ref(m), 1.0, ref(ok), P, 1 << 40, None), word)


@pytest.mark.parametrize("p, word", [(-0.1, "[0, 1]"), (1.1, "[0, 1]"), (float("nan"), "[0, 1]"), (float("inf"), "[0, 1]")])
def test_probabilities_and_steps_are_refused(p, word):
    L, ok = binding.load(), rows()
    for d, w in [(Drop(p, 1, 2, None), word), (Drop(0.5, 1, 1 << 56, None), "step"), (Drop(0.5, 1, 0, P + 4), "aligned"), (None, "null")]:
        d = None if d is None else ref(d)
        refused(L.same_lda_dropout(ref(ok), d, ref(ok), None), w)
        refused(L.same_lda_embed_dropout(ref(ok), P, 4, 1.0, d, ref(ok), None), w)
        refused(L.same_lda_embed_dropout_grad(ref(ok), P, 4, 1.0, d, 0, ref(ok), P, 1 << 30, None), w)


def test_shapes_types_tokens_and_scales_are_refused():
    L, a, m, g, d = binding.load(), rows(), rows(type=M), rows(type=32), Drop(0.5, 1, 2, None)
    n = ctypes.c_size_t()
    for call in (lambda s, tb, t, d=d: L.same_lda_embed_dropout(ref(a), t, tb, s, ref(d), ref(a), None), lambda s, tb, t, d=d: L.same_lda_embed_dropout_grad(ref(a), t, tb, s, ref(d), 0, ref(a), P, 1 << 30, None)):
        refused(call(float("nan"), 4, P), "finite")
        refused(call(float("inf"), 8, P), "finite")
        refused(call(3e38, 8, P, Drop(0.9, 1, 2, None)), "beyond")           # the scale of what is kept
        refused(call(1.0, 2, P), "bytes")
        refused(call(1.0, 8, P + 4), "aligned")
    for x, o, word in [(None, a, "null"), (a, None, "null"), (m, a, "must not be microscaled"), (g, a, "must not be grouped"), (a, m, "must not be microscaled"), (a, g, "must not be grouped"),
                       (a, rows(rows=5), "into"), (a, rows(width=9), "into")]:
        refused(L.same_lda_dropout(x and ref(x), ref(d), o and ref(o), None), word)
    refused(L.same_lda_embed_dropout(ref(a), P, 4, 1.0, ref(d), ref(g), None), "must not be grouped")
    refused(L.same_lda_embed_dropout(ref(a), P, 4, 1.0, ref(d), ref(rows(width=7)), None), "elements")
    refused(L.same_lda_embed_dropout(ref(a), None, 4, 1.0, ref(d), ref(rows(rows=3)), None), "without tokens")
    refused(L.same_lda_embed(ref(a), P, 4, 1.0, ref(g), None), "must not be grouped")
    refused(L.same_lda_embed_grad(ref(g), P, 4, 1.0, 0, ref(a), P, 1 << 30, None), "must not be grouped")
    refused(L.same_lda_embed_dropout_grad(ref(a), None, 4, 1.0, ref(d), 0, ref(a), P, 1 << 30, None), "null")
    refused(L.same_lda_embed_dropout_grad(ref(a), P, 4, 1.0, ref(d), 0, ref(g), P, 1 << 30, None), "must not be grouped")
    many = rows(rows=50_000)
    assert L.same_lda_embed_dropout_grad_workspace(ref(many), ref(a), ref(n)) == 0 and n.value > 0
    refused(L.same_lda_embed_dropout_grad_workspace(ref(many), ref(a), None), "null")
    refused(L.same_lda_embed_dropout_grad_workspace(ref(many), ref(rows(width=7)), ref(n)), "elements")
    refused(L.same_lda_embed_dropout_grad(ref(many), P, 4, 1.0, ref(d), 0, ref(a), P, n.value - 1, None), "workspace")
    refused(L.same_lda_micro_quantize(ref(g), ref(m), None), "must not be grouped")
    refused(L.same_lda_micro_quantize(ref(a), ref(g), None), "must be microscaled")
    refused(L.same_lda_micro_product(ref(g), ref(m), 1.0, ref(rows(width=4)), None), "must not be grouped")
    refused(L.same_lda_micro_product(ref(a), ref(g), 1.0, ref(rows(width=4)), None), "must be microscaled")
    refused(L.same_lda_group_quantize(ref(g), ref(g), None), "must not be grouped")
    refused(L.same_lda_group_quantize(ref(m), ref(g), None), "must not be microscaled")
    refused(L.same_lda_group_quantize(ref(a), ref(a), None), "must be grouped")
    refused(L.same_lda_group_quantize(ref(a), ref(m), None), "must be grouped")
    refused(L.same_lda_group_quantize(ref(a), ref(rows(type=64, rows=5)), None), "into")
    refused(L.same_lda_group_quantize(ref(a), ref(rows(type=64, width=9)), None), "into")
    refused(L.same_lda_group_product(ref(g), ref(g), 1.0, ref(rows(width=4)), P, 1 << 40, None), "must not be grouped")
    refused(L.same_lda_group_product(ref(m), ref(g), 1.0, ref(rows(width=4)), P, 1 << 40, None), "must not be microscaled")
    refused(L.same_lda_group_product(ref(a), ref(m), 1.0, ref(rows(width=4)), P, 1 << 40, None), "must be grouped")
    refused(L.same_lda_group_product(ref(a), ref(a), 1.0, ref(rows(width=4)), P, 1 << 40, None), "must be grouped")
    refused(L.same_lda_group_product(ref(a), ref(rows(type=32, width=9)), 1.0, ref(rows(width=4)), P, 1 << 40, None), "elements")
    refused(L.same_lda_group_product(ref(a), ref(g), 1.0, ref(rows(width=5)), P, 1 << 40, None), "do not give")
    refused(L.same_lda_group_product(ref(a), ref(g), 1.0, ref(rows(rows=5, width=4)), P, 1 << 40, None), "do not give")
    refused(L.same_lda_group_product(ref(a), ref(g), float("nan"), ref(rows(width=4)), P, 1 << 40, None), "finite")
    refused(L.same_lda_group_product(ref(a), ref(g), 1.0, ref(g), P, 1 << 40, None), "must not be grouped")
    for bad in [(-1, 8, 32), (1 << 31, 8, 32), (1, 0, 32), (1, (1 << 20) + 1, 32), (1, 8, 16), (1, 8, 0), (1, 8, 256), (1, 8, 3)]:
        refused(L.same_lda_group_size(*bad, ref(n), ref(n)), "shape")
    refused(L.same_lda_group_size(1, 8, 32, None, ref(n)), "null")


def test_empty_calls_do_nothing():
    L, e, a, d = binding.load(), rows(rows=0, data=None), rows(), Drop(0.5, 1, 2, None)
    eg, g = rows(rows=0, type=64, data=None, scales=0), rows(type=64)
    assert L.same_lda_dropout(ref(e), ref(d), ref(e), None) == 0
    assert L.same_lda_embed_dropout(ref(a), P, 8, 1.0, ref(d), ref(e), None) == 0
    assert L.same_lda_embed_dropout(ref(e), None, 8, 1.0, ref(d), ref(e), None) == 0
    assert L.same_lda_embed_dropout_grad(ref(e), None, 4, 1.0, ref(d), 1, ref(a), None, 0, None) == 0
    assert L.same_lda_embed_dropout_grad(ref(a), P, 4, 1.0, ref(d), 0, ref(e), None, 0, None) == 0
    assert L.same_lda_embed(ref(g), P, 8, 1.0, ref(e), None) == 0
    assert L.same_lda_group_quantize(ref(e), ref(eg), None) == 0
    assert L.same_lda_group_product(ref(e), ref(g), 1.0, ref(rows(rows=0, width=4, data=None)), P, 1 << 40, None) == 0
    assert L.same_lda_group_product(ref(a), ref(eg), 1.0, None, P, 1 << 40, None) == 0


def test_sizes_of_grouped_matrices():
    L, c, s = binding.load(), ctypes.c_size_t(), ctypes.c_size_t()
    for r, w, group, code, scale in [(0, 1, 32, 0, 0), (3, 1, 32, 192, 48), (3, 128, 64, 192, 24), (3, 129, 128, 384, 24), ((1 << 31) - 1, 1 << 20, 32, ((1 << 31) - 1) << 19, ((1 << 31) - 1) << 17)]:
        assert L.same_lda_group_size(r, w, group, ref(c), ref(s)) == 0 and (c.value, s.value) == (code, scale)


def test_workspaces_of_products_and_of_gradients():
    L, n, m = binding.load(), ctypes.c_size_t(), ctypes.c_size_t()
    for r, w, t, words, some in [(1, 4096, F, 1 << 30, False), (16, 4096, B, 4, False), (16, 4097, B, 4, True), (17, 8, H, 131_072, False), (17, 8, H, 131_073, True), (0, 8, F, 4, False),
                                 (512, 4096, B, 256, False), (512, 4096, B, 257, True), (5000, 1 << 20, F, 4, True), ((1 << 31) - 1, 128, B, (1 << 31) - 1, True)]:
        assert L.same_lda_group_product_workspace(ref(rows(rows=r, width=w, type=t)), ref(rows(type=64, rows=words, width=w)), ref(n)) == 0 and (n.value > 0) == some
        # rows laid down are 256 MB or 4096 rows, in three pieces of two bytes, and 128 more; sums are 3 KB for 16 rows and 32 groups, whose operands are 16 KB or more
        assert n.value <= (1 + 3 / 16) * max((1 << 28) + (1 << 20), 4096 * (w + 1024) * 6)
    refused(L.same_lda_group_product_workspace(ref(rows()), ref(rows(type=64)), None), "null")
    refused(L.same_lda_group_product_workspace(ref(rows()), ref(rows(type=64, width=9)), ref(n)), "elements")
    a, g, out = rows(rows=20, width=4200), rows(type=64, width=4200), rows(rows=20, width=4)
    assert L.same_lda_group_product_workspace(ref(a), ref(g), ref(n)) == 0
    for space, size in [(P, n.value - 1), (None, n.value), (P + 8, n.value)]:
        refused(L.same_lda_group_product(ref(a), ref(g), 1.0, ref(out), space, size, None), "workspace")
    # wide rows of a few thousand tokens are sorted where the lookup had dropout
    assert L.same_lda_embed_grad_workspace(ref(rows(rows=8000, width=1024)), ref(rows(width=1024)), ref(n)) == 0 and n.value == 0
    assert L.same_lda_embed_dropout_grad_workspace(ref(rows(rows=8000, width=1024)), ref(rows(width=1024)), ref(m)) == 0 and m.value > 0


def test_binding_refuses_what_it_cannot_pass_on():
    x, t = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    codes, scales = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 2, 2, dtype=torch.bfloat16)
    q = binding.GroupMatrix(codes, scales, 8, 64)
    assert q.shape == (4, 8) and q[1:3].shape == (2, 8) and q[1:3].codes.data_ptr() == codes.data_ptr() + 64 and q[1:3].scales.data_ptr() == scales.data_ptr() + 8
    for bad in [(codes[:, :32], scales, 8, 64), (codes, scales[:, :1], 8, 64), (codes, scales, 129, 64), (codes, scales, 0, 64), (codes.to(torch.int8), scales, 8, 64), (codes[::2], scales[:2], 8, 64),
                (codes, scales[:3], 8, 64), (codes, scales, 8, 32), (codes, scales, 8, 48), (codes, scales.half(), 8, 64)]:
        with pytest.raises(ValueError):
            binding.GroupMatrix(*bad)
    for bad in (0, slice(None, None, 2)):
        with pytest.raises(TypeError):
            q[bad]
    d = binding.Dropout(0.5, 1, 2)
    for call in (lambda: binding.embed(x, t, drop=d), lambda: binding.embed_grad(x, t, 5, drop=d), lambda: binding.dropout(x, d), lambda: binding.group_quantize(x), lambda: binding.group_dequantize(q),
                 lambda: binding.group_product(x, q), lambda: binding.embed(q, t)):
        with pytest.raises(ValueError, match="GPU"):            # no CPU form
            call()
    m = binding.MicroMatrix(codes, torch.zeros(4, 4, dtype=torch.uint8), 8)
    for call in (lambda: binding.dropout(x, 0.5), lambda: binding.dropout(q, d), lambda: binding.dropout(m, d), lambda: binding.group_quantize(q), lambda: binding.group_dequantize(x), lambda: binding.group_dequantize(m),
                 lambda: binding.group_product(x, x), lambda: binding.group_product(x, m), lambda: binding.group_product(q, q), lambda: binding.micro_product(q, m), lambda: binding.micro_product(x, q),
                 lambda: binding.embed_grad(q, t, 5), lambda: binding.micro_quantize(q), lambda: binding.Dropout(0.5, 1, torch.zeros(2, dtype=torch.int64)), lambda: binding.Dropout(0.5, 1, torch.zeros(1)),
                 lambda: binding.Dropout(0.5, 1, 2.0), lambda: binding.Dropout(0.5, 1.0)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: binding.Dropout(-0.1, 1), lambda: binding.Dropout(1.5, 1), lambda: binding.Dropout(float("nan"), 1), lambda: binding.Dropout(0.5, -1), lambda: binding.Dropout(0.5, 1 << 64),
                 lambda: binding.Dropout(0.5, 1, -1), lambda: binding.Dropout(0.5, 1, 1 << 56), lambda: binding.dropout(torch.tensor(1.0), d), lambda: binding.dropout(torch.zeros(3, 0), d)):
        with pytest.raises(ValueError):
            call()
    r = Rows.from_buffer_copy(binding._rows(q))
    assert (r.data, r.scales, r.rows, r.width, r.type) == (codes.data_ptr(), scales.data_ptr(), 4, 8, 64)
    s = torch.tensor([5])
    v = Drop.from_buffer_copy(binding._drop(binding.Dropout(0.25, (1 << 64) - 1, s)))
    assert (v.p, v.seed, v.step, v.step_at) == (0.25, (1 << 64) - 1, 0, s.data_ptr())
    v = Drop.from_buffer_copy(binding._drop(binding.Dropout(0.25, 7, (1 << 56) - 1)))
    assert (v.p, v.seed, v.step, v.step_at) == (0.25, 7, (1 << 56) - 1, None)


def test_a_dropout_passes_on_what_it_holds_when_it_is_used():
    """What is passed to the library is what the object says: its numbers cannot be changed under it, and the address of a step in
    a tensor is that of the call, also after the tensor has other memory or the object was copied."""
    d = binding.Dropout(0.5, 7, 2)
    for name, value in (("p", 0.9), ("seed", 8), ("step", 3)):
        with pytest.raises(AttributeError):
            setattr(d, name, value)
    with pytest.raises(AttributeError):
        d.step += 1
    assert (d.p, d.seed, d.step) == (0.5, 7, 2)

    def at(d):
        v = Drop.from_buffer_copy(binding._drop(d))
        return v.p, v.seed, v.step, v.step_at

    assert at(d) == (0.5, 7, 2, None) and at(copy.deepcopy(d)) == at(pickle.loads(pickle.dumps(d))) == at(d)
    s = torch.tensor([5])
    d = binding.Dropout(0.25, 9, s)
    assert d.step is s and at(d) == (0.25, 9, 0, s.data_ptr())
    first, other = s.data_ptr(), torch.tensor([6, 7])
    s.set_(other.untyped_storage(), 1, (1,))
    assert first != s.data_ptr() == other.data_ptr() + 8 and at(d) == (0.25, 9, 0, s.data_ptr())
    s.data = torch.tensor([8])
    assert at(d) == (0.25, 9, 0, s.data_ptr())
    e = copy.deepcopy(d)
    assert e.step is not s and at(e) == (0.25, 9, 0, e.step.data_ptr()) and at(d)[3] == s.data_ptr()
    s.resize_(2)
    with pytest.raises(TypeError):            # no step any more
        binding._drop(d)
    s.resize_(0)
    with pytest.raises(TypeError):
        binding._drop(d)


def test_refusals_name_the_call_that_was_made():
    L, a, n = binding.load(), rows(), ctypes.c_size_t()
    many = rows(rows=50_000)
    for drop, name in ((Drop(0.5, 1, 2, None), "embed_dropout_grad: "), (None, "embed_grad: ")):
        def call(g, tokens, size, scale, t, space, bytes):
            if drop is None:
                return L.same_lda_embed_grad(g, tokens, size, scale, 0, t, space, bytes, None)
            return L.same_lda_embed_dropout_grad(g, tokens, size, scale, ref(drop), 0, t, space, bytes, None)
        space = L.same_lda_embed_grad_workspace if drop is None else L.same_lda_embed_dropout_grad_workspace
        ok = (ref(a), P, 4, 1.0, ref(a), P, 1 << 30)
        for at, value in [(0, None), (4, None), (0, ref(rows(type=5))), (4, ref(rows(type=64))), (4, ref(rows(width=7))), (2, 2), (1, P + 2), (1, None), (3, float("nan"))]:
            refused(call(*ok[:at], value, *ok[at + 1:]), name)
        for at, bytes in ((P, 0), (None, 1 << 30), (P + 8, 1 << 30)):
            refused(call(ref(many), P, 4, 1.0, ref(a), at, bytes), name, "workspace")
        for bad in [(None, ref(a), ref(n)), (ref(a), ref(rows(width=7)), ref(n)), (ref(a), ref(a), None)]:
            refused(space(*bad), name)
