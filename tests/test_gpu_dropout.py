"""Dropout of matrices, of lookups and of their gradient, against the oracle in double (oracle/word_rows.py), element by element.

Tolerances.  u = 2^-24 is half a step of binary32, eps/2 half a step of the output's type (with its smallest subnormal over 2 as the
absolute floor).  A kept element is one product in binary32 with a factor that was rounded to binary32, and one rounding: 2 u + eps/2; a
dropped one is 0.  A gradient's sum of m terms in binary32 in any order is off by at most m u times the sum of their magnitudes (1.01
covers higher orders), then comes the same factor."""
import numpy as np
import pytest
import torch

from oracle import word_rows as wr
from paper_1409_5402_amd import binding

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def close(got, want, dtype, extra=0.0):
    f = torch.finfo(dtype)
    got = got.double().cpu().numpy()
    bound = 1.01 * extra + (f.eps / 2 + 2.01 * U) * (np.abs(want) + extra) + f.smallest_normal * f.eps / 2
    bad = ~(np.abs(got - want) <= bound) & ~(np.isnan(got) & np.isnan(want)) & ~(got == want)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


def numbers_of(rng, rows, cols, dtype):
    return torch.from_numpy(rng.normal(size=(rows, cols)) * np.exp(rng.normal(size=cols))).to(dtype)


def words(rng, n, V):
    t = np.minimum((V * rng.uniform(size=n) ** 3).astype(np.int64), V - 1)
    t[rng.uniform(size=n) < 0.1] = -1
    return t


def guarded(rows, cols, dtype, stride=None, offset=0):
    """A matrix inside a larger buffer of sevens, and a check that nothing around it was written."""
    stride = cols if stride is None else stride
    buf = torch.full((offset + rows * stride + 300,), 7.0, dtype=dtype, device=DEV)
    view = torch.as_strided(buf, (rows, cols), (stride, 1), offset)

    def check():
        b = buf.clone()
        torch.as_strided(b, (rows, cols), (stride, 1), offset).fill_(7.0)
        assert torch.all(b == 7.0)
    return view, check


# ---- of a matrix

@pytest.mark.parametrize("width", [1, 2, 7, 8, 9, 50, 256, 1000])
@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("x", TYPES)
def test_dropout_matches_the_oracle(x, out, width):
    rng = np.random.default_rng(width)
    X = numbers_of(rng, 61, width, TYPES[x])
    got, check = guarded(61, width, TYPES[out], offset=16)
    binding.dropout(X.to(DEV), binding.Dropout(0.3, 0xFEDCBA9876543210, 11), out=got)
    close(got, wr.dropout(X.double().numpy(), 0.3, 0xFEDCBA9876543210, 11), TYPES[out])
    check()


@pytest.mark.parametrize("stride, offset", [(64, 0), (65, 0), (66, 1), (64, 3), (72, 8), (200, 5)])
@pytest.mark.parametrize("dtype", TYPES)
def test_dropout_strides_and_alignment(dtype, stride, offset):
    rng = np.random.default_rng(stride + offset)
    X = numbers_of(rng, 23, 64, TYPES[dtype])
    x, _ = guarded(23, 64, TYPES[dtype], stride, offset)
    x.copy_(X)
    got, check = guarded(23, 64, TYPES[dtype], stride + 3, 1)
    d = binding.Dropout(0.5, 3, 4)
    binding.dropout(x, d, out=got)
    close(got, wr.dropout(X.double().numpy(), 0.5, 3, 4), TYPES[dtype])
    check()
    assert torch.equal(binding.dropout(x, d, out=x), got)          # in place

def test_the_border_is_decided_by_all_32_bits():
    """A probability whose border is one element's own number drops it, the next border keeps it; 65,536 elements meet a tie of 16 bits."""
    rows, width, seed, step = 300, 1024, 123, (5 << 32) + 6
    r = wr.bits(rows, width, seed, step)
    x = torch.ones(rows, width, device=DEV)
    for i, j in [(0, 0), (17, 5), (299, 1023), (100, 514)]:
        for over in (0, 1):
            p = 1.0 - (int(r[i, j]) + over) / 2.0 ** 32
            got = binding.dropout(x, binding.Dropout(p, seed, step)).cpu().numpy() != 0
            assert got[i, j] == bool(over) and np.array_equal(got, r < int(r[i, j]) + over)


@pytest.mark.parametrize("p", [0.0, 1e-9, 0.1, 1.0 - 1e-7, 1.0])
def test_probabilities_at_the_ends_and_what_is_dropped_does_not_count(p):
    X = torch.full((40, 130), 1.0, device=DEV)
    X[::3] = float("nan")
    X[1::3] = float("-inf")
    got = binding.dropout(X, binding.Dropout(p, 5, 6)).cpu()
    k = torch.from_numpy(wr.kept(40, 130, p, 5, 6))
    assert torch.all(got[~k] == 0)
    assert torch.all(torch.isnan(got[::3]) == k[::3]) and torch.all(torch.isinf(got[1::3]) == k[1::3])
    if p == 0.0:
        assert k.all() and torch.equal(got[2::3], X[2::3].cpu())


def test_shapes_of_tensors_and_gradients():
    d = binding.Dropout(0.4, 8, 9)
    x = torch.randn(5, 3, 6, 33, device=DEV)
    got = binding.dropout(x, d)
    assert got.shape == x.shape and torch.equal(got.view(-1, 33), binding.dropout(x.view(-1, 33), d))
    assert torch.equal(binding.dropout(x[0, 0, 0], d), binding.dropout(x[0, 0, :1], d)[0])
    t = x.transpose(0, 1)
    assert torch.equal(binding.dropout(t, d), binding.dropout(t.contiguous(), d))
    e = torch.ones(1, 33, device=DEV).expand(7, 33)                       # the gradient of a sum
    assert torch.equal(binding.dropout(e, d), binding.dropout(e.contiguous(), d))
    assert binding.dropout(x[:0], d).shape == (0, 3, 6, 33)
    assert binding.dropout(x, d, dtype=torch.bfloat16).dtype == torch.bfloat16
    # <dy, f(x)> = <f'(dy), x> for a linear f: the call is its own gradient; and by differences, which are exact here
    dy = torch.randint(-4, 5, x.shape, device=DEV).float()
    xi = torch.randint(-4, 5, x.shape, device=DEV).float()
    half = binding.Dropout(0.5, 8, 9)
    assert torch.equal((dy * binding.dropout(xi, half)).sum(), (binding.dropout(dy, half) * xi).sum())
    one = xi.clone()
    one[2, 1, 3] += 1.0
    assert torch.equal((binding.dropout(one, half) - binding.dropout(xi, half))[2, 1, 3], binding.dropout(torch.ones_like(xi), half)[2, 1, 3])


def test_another_seed_or_step_is_another_choice_and_the_same_the_same():
    x = torch.ones(64, 1000, device=DEV)
    a = binding.dropout(x, binding.Dropout(0.5, 1, 0))
    assert torch.equal(a, binding.dropout(x, binding.Dropout(0.5, 1, 0)))
    for seed, step in [(2, 0), (1, 1), (1 + (1 << 32), 0), (1, 1 << 32), (1, 1 << 55)]:
        assert 0.4 < (binding.dropout(x, binding.Dropout(0.5, seed, step)) == a).float().mean().item() < 0.6


def test_wide_rows_and_many_rows():
    """The widest rows, and more elements than one launch has threads for chunks of them."""
    x = torch.ones(3, 1 << 20, dtype=torch.bfloat16, device=DEV)
    got = binding.dropout(x, binding.Dropout(0.25, 4, 4))
    assert np.array_equal((got != 0).cpu().numpy(), wr.kept(3, 1 << 20, 0.25, 4, 4))
    x = torch.ones(2_200_003, 5, dtype=torch.float16, device=DEV)
    got = binding.dropout(x, binding.Dropout(0.25, 4, 5))
    assert np.array_equal((got != 0).cpu().numpy(), wr.kept(2_200_003, 5, 0.25, 4, 5))


def test_offsets_beyond_32_bits():
    rows, width = 70_000, 65_536                                          # 4.6e9 elements, 9.2 GB
    x = torch.ones(rows, width, dtype=torch.bfloat16, device=DEV)
    binding.dropout(x, binding.Dropout(0.5, 4, 4), out=x)
    for row in (0, 65_535, 65_536, rows - 1):
        assert np.array_equal((x[row:row + 1] != 0).cpu().numpy(), wr.kept(1, width, 0.5, 4, 4, first=row))


# ---- of a lookup

@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("table", list(TYPES) + ["micro", "groups"])
@pytest.mark.parametrize("width", [1, 3, 8, 50, 65, 256, 1000])
def test_lookup_with_dropout_matches_the_oracle(width, table, out):
    rng = np.random.default_rng(width)
    T = numbers_of(rng, 37, width, TYPES.get(table, torch.float32))
    t = words(rng, 53, 37)
    t[:4] = [37, -5, 1 << 33, 36]
    on = T.to(DEV)
    if table == "micro":
        on = binding.micro_quantize(on)
        T = binding.micro_dequantize(on).cpu()
    elif table == "groups":
        on = binding.group_quantize(on, 32)
        T = binding.group_dequantize(on).cpu()
    got, check = guarded(53, width, TYPES[out], offset=16)
    d = binding.Dropout(0.2, 99, 7)
    binding.embed(on, torch.from_numpy(t).to(DEV), 1.75, out=got, drop=d)
    rows = np.where(((t >= 0) & (t < 37))[:, None], T.double().numpy()[np.where((t >= 0) & (t < 37), t, 0)], 0.0)
    # (a number of four bits that a table's read-back rounded to binary32 once more: u)
    close(got, wr.dropout(rows, 0.2, 99, 7, 1.75), TYPES[out], U * np.abs(rows) * 1.75 / 0.8)
    check()
    ids = torch.from_numpy(t.reshape(1, 53).astype(np.int32) if abs(t).max() < 1 << 31 else np.where(t > 1 << 31, -1, t).reshape(1, 53).astype(np.int32)).to(DEV)
    assert torch.equal(binding.embed(on, ids, 1.75, dtype=TYPES[out], drop=d)[0], got)


def test_lookup_without_probability_is_the_lookup_and_padding_is_zeros():
    T = torch.full((5, 64), float("nan"), device=DEV)
    T[2] = 1.0
    t = torch.tensor([2, -1, 5, 2], device=DEV)
    got = binding.embed(T, t, drop=binding.Dropout(0.0, 1))
    assert torch.equal(got, binding.embed(T, t)) and got.sum().item() == 128.0
    got = binding.embed(T, t, drop=binding.Dropout(0.5, 1))
    assert torch.all(got[1:3] == 0) and torch.all((got == 0) | (got == 2.0))
    assert torch.all(binding.embed(T[:0], t, drop=binding.Dropout(0.5, 1)) == 0)
    assert torch.equal(got, binding.dropout(binding.embed(T, t), binding.Dropout(0.5, 1)))      # the same places


# ---- the gradient of a lookup

def both(grad, t, V, scale, p, seed, step, dtype, extra_terms=0, **more):
    got = binding.embed_grad(grad, t, V, scale, dtype=dtype, drop=binding.Dropout(p, seed, step), **more)
    want, size, terms = wr.embed_dropout_grad(grad.double().cpu().numpy(), t.cpu().numpy(), V, p, seed, step, scale)
    close(got, want, dtype, (terms[:, None] + extra_terms) * U * size)
    return got


@pytest.mark.parametrize("out", ["f32", "same"])
@pytest.mark.parametrize("grad", TYPES)
@pytest.mark.parametrize("width", [1, 2, 3, 4, 8, 12, 50, 65, 66, 256, 1000])
def test_gradient_matches_the_oracle(width, grad, out):
    rng = np.random.default_rng(width)
    D = numbers_of(rng, 700, width, TYPES[grad]).to(DEV)
    t = torch.from_numpy(words(rng, 700, 23)).to(DEV)
    both(D, t, 23, 1.25, 0.3, 17, 18, TYPES[grad if out == "same" else "f32"])


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("n, V, width", [(20_000, 40, 16), (20_000, 30_000, 10), (17_000, 300, 66), (20_001, 500, 9), (18_000, 100, 128), (9_000, 50, 600), (16_384, 3, 24),
                                         (8_000, 60, 100), (8_192, 3, 128), (8_100, 40_000, 330), (16_000, 70_000, 50), (16_384, 66_000, 9), (16_383, 70_000, 64)])
def test_gradient_of_sorted_tokens_and_long_runs(n, V, width, grad):
    rng = np.random.default_rng(n + width)
    D = numbers_of(rng, n, width, TYPES[grad]).to(DEV)
    t = torch.from_numpy(words(rng, n, V)).to(DEV)
    both(D, t, V, 1.0, 0.1, 1, 2, torch.float32)


def test_gradient_bits_do_not_depend_on_strides_nor_on_what_was_dropped():
    rng = np.random.default_rng(0)
    for n, width in [(300, 65), (300, 64), (20_000, 36), (20_000, 33)]:
        D = numbers_of(rng, n, width, torch.float32).to(DEV)
        t = torch.from_numpy(words(rng, n, 31)).to(DEV)
        d = binding.Dropout(0.4, 6, 1 << 40)
        want = binding.embed_grad(D, t, 31, drop=d)
        for stride, offset in [(width + 1, 0), (width + 3, 1), (width + 4, 2)]:
            g, _ = guarded(n, width, torch.float32, stride, offset)
            g.copy_(D)
            g[~torch.from_numpy(wr.kept(n, width, 0.4, 6, 1 << 40)).to(DEV)] = float("nan")
            assert torch.equal(binding.embed_grad(g, t.int(), 31, drop=d), want)
        # dropping with p = 0 is the plain gradient; masked numbers by hand are the same sum
        assert torch.equal(binding.embed_grad(D, t, 31, drop=binding.Dropout(0.0, 1)), binding.embed_grad(D, t, 31))
        masked = torch.where(torch.from_numpy(wr.kept(n, width, 0.4, 6, 1 << 40)).to(DEV), D, 0.0)
        assert torch.equal(binding.embed_grad(masked, t, 31, float(np.float32(1 / 0.6))), want)


def test_gradient_accumulates_and_empty_lists():
    rng = np.random.default_rng(1)
    D = torch.randint(-8, 9, (500, 40), device=DEV).float()
    t = torch.from_numpy(words(rng, 500, 70)).to(DEV)
    t[t == 5] = 6
    d = binding.Dropout(0.5, 2, 2)
    out = torch.full((70, 40), 3.0, device=DEV)
    out[5] = float("nan")                                            # a word without a token is not touched
    fresh = binding.embed_grad(D, t, 70, drop=d)
    binding.embed_grad(D, t, out=out, accumulate=True, drop=d)
    assert torch.isnan(out[5]).all() and torch.equal(out[6:], fresh[6:] + 3.0) and torch.equal(out[:5], fresh[:5] + 3.0)
    assert torch.all(binding.embed_grad(D[:0], t[:0], 70, drop=d) == 0)
    assert torch.all(binding.embed_grad(D, torch.full_like(t, -1), 70, drop=d) == 0)
    assert torch.all(binding.embed_grad(D, t, 70, drop=binding.Dropout(1.0, 2, 2)) == 0)


def test_gradient_is_that_of_the_lookup_by_differences():
    """The lookup is linear and everything here is a small integer times a power of two: differences are exact."""
    rng = np.random.default_rng(2)
    V, E, n = 19, 21, 150
    T, D = (torch.from_numpy(rng.integers(-4, 5, s)).float().to(DEV) for s in ((V, E), (n, E)))
    t = torch.from_numpy(words(rng, n, V)).to(DEV)
    d = binding.Dropout(0.5, 31, 32)
    G = binding.embed_grad(D, t, V, 2.0, drop=d)
    at = (D * binding.embed(T, t, 2.0, drop=d)).sum()
    for w, j in [(0, 0), (3, 20), (18, 7), (1, 8)]:
        moved = T.clone()
        moved[w, j] += 1.0
        assert (D * binding.embed(moved, t, 2.0, drop=d)).sum() - at == G[w, j]


# ---- steps in device memory, graphs, streams

def test_a_captured_step_draws_anew_in_every_replay():
    V, E, n = 50, 72, 200
    T, D = torch.randn(V, E, device=DEV), torch.randn(n, E, device=DEV)
    t = torch.randint(-1, V, (n,), device=DEV)
    step = torch.tensor([10], device=DEV)
    d = binding.Dropout(0.3, 77, step)
    rows, G, y = torch.empty(n, E, device=DEV), torch.empty(V, E, device=DEV), torch.empty(n, E, device=DEV)

    def work():
        binding.embed(T, t, out=rows, drop=d)
        binding.dropout(rows, d, out=y)
        binding.embed_grad(D, t, out=G, drop=d)
        step.add_(1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    step.fill_(10)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    step.fill_(10)
    seen = []
    for k in range(10, 14):
        graph.replay()
        fixed = binding.Dropout(0.3, 77, k)
        want = binding.embed(T, t, drop=fixed)
        torch.cuda.synchronize()
        assert torch.equal(rows, want) and torch.equal(y, binding.dropout(want, fixed)) and torch.equal(G, binding.embed_grad(D, t, V, drop=fixed))
        seen.append(rows.clone())
    assert step.item() == 14 and not torch.equal(seen[0], seen[1])


def test_on_another_stream():
    x = torch.randn(3000, 500, device=DEV)
    d = binding.Dropout(0.3, 1, 2)
    want = binding.dropout(x, d)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = x * 2.0
        got = binding.dropout(y, d)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want * 2.0)


def test_refusals_on_the_device():
    x, t, d = torch.zeros(4, 8, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV), binding.Dropout(0.5, 1)
    far = binding.Dropout(0.5, 1, torch.zeros(1, dtype=torch.int64))           # a step in host memory
    for error, call in [(TypeError, lambda: binding.dropout(x.double(), d)), (TypeError, lambda: binding.dropout(x, d, dtype=torch.int32)), (ValueError, lambda: binding.dropout(x, d, out=x[:3])),
                        (ValueError, lambda: binding.dropout(x, d, out=torch.zeros(4, 8))), (ValueError, lambda: binding.dropout(x, far)), (ValueError, lambda: binding.embed(x, t, drop=far)),
                        (ValueError, lambda: binding.embed_grad(x, t, 5, drop=far)), (TypeError, lambda: binding.embed(x, t, drop=0.5)), (TypeError, lambda: binding.embed_grad(x, t, 5, drop=0.5)),
                        (ValueError, lambda: binding.dropout(x, d, out=x.t())), (binding.SameLdaError, lambda: binding.embed(x, t, 3e38, drop=binding.Dropout(0.9, 1)))]:
        with pytest.raises(error):
            call()
