"""The word-table operators against their oracle in double (oracle/word_tables.py), element by element.

Tolerances.  u = 2^-24 is half a step of binary32, eps/2 half a step of the output's type (with its smallest subnormal over 2
as the absolute floor).  A lookup is one product in binary32 and one rounding: u + eps/2.  A sum of m terms in binary32 in any order is
off by at most m u times the sum of their magnitudes (to first order; 1.01 covers the rest); a run of more than 256 tokens may be
summed in pieces, so m counts the terms of a piece and the pieces.  Then one product and one rounding: u + eps/2.
Products of four-bit numbers are exact in binary32, and every addition of the matrix instruction is taken to be off by a whole
step: 2 u per term.  Rounding to four bits and reading back are exact."""
import threading

import numpy as np
import pytest
import torch

from helpers import csc_from_dense
from oracle import word_tables as wt
from paper_1409_5402_amd import binding

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def half_step(dtype):
    f = torch.finfo(dtype)
    return f.eps / 2, f.smallest_normal * f.eps / 2


def close(got, want, dtype, extra=0.0):
    """|got - want| <= extra + what rounding once to binary32 and once to dtype may cost"""
    rel, floor = half_step(dtype)
    got = got.double().cpu().numpy()
    bound = extra + (rel + U) * (np.abs(want) + extra) + floor
    bad = ~(np.abs(got - want) <= bound) & ~(np.isnan(got) & np.isnan(want))
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


def numbers_of(rng, rows, cols, dtype):
    """Normal numbers with columns of different size, rounded to dtype."""
    x = rng.normal(size=(rows, cols)) * np.exp(rng.normal(size=cols))
    return torch.from_numpy(x).to(dtype)


def words(rng, n, V, kind):
    t = rng.integers(0, V, n) if kind == "even" else np.minimum((V * rng.uniform(size=n) ** 4).astype(np.int64), V - 1)
    t = t.astype(np.int64)
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


# ---- lookup

@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("table", TYPES)
@pytest.mark.parametrize("width", [1, 2, 3, 8, 50, 64, 65, 256, 1000])
def test_embed_matches_the_oracle(width, table, out):
    rng = np.random.default_rng(width)
    T = numbers_of(rng, 37, width, TYPES[table])
    t = words(rng, 53, 37, "even")
    t[:4] = [37, -5, 1 << 33, 36]
    got, check = guarded(53, width, TYPES[out], offset=16)
    binding.embed(T.to(DEV), torch.from_numpy(t).to(DEV), 1.75, out=got)
    close(got, wt.embed(T.double().numpy(), t, 1.75), TYPES[out])
    check()
    # one rounding to binary32 and one to the output's type: the same bits as on the host
    same = torch.where(torch.from_numpy((t >= 0) & (t < 37)).unsqueeze(1), (T.float()[np.where((t >= 0) & (t < 37), t, 0)] * 1.75), torch.zeros(()))
    assert torch.equal(got.cpu(), same.to(TYPES[out]))


@pytest.mark.parametrize("stride, offset", [(64, 0), (65, 0), (66, 0), (64, 1), (64, 2), (72, 8), (200, 3)])
@pytest.mark.parametrize("dtype", TYPES)
def test_embed_strides_and_alignment(dtype, stride, offset):
    rng = np.random.default_rng(stride + offset)
    T = numbers_of(rng, 20, 64, TYPES[dtype])
    table, _ = guarded(20, 64, TYPES[dtype], stride, offset)
    table.copy_(T)
    t = words(rng, 31, 20, "even").astype(np.int32)
    got, check = guarded(31, 64, TYPES[dtype], stride + 3, 1)
    binding.embed(table, torch.from_numpy(t).to(DEV), -0.5, out=got)
    close(got, wt.embed(T.double().numpy(), t, -0.5), TYPES[dtype])
    check()


def test_embed_shapes_of_tokens_and_the_longest_and_shortest_lists():
    T = torch.arange(35, dtype=torch.float32, device=DEV).view(7, 5)
    t = torch.tensor([[1, 2, 3], [6, -1, 0]], device=DEV)
    out = binding.embed(T, t, 2.0, dtype=torch.bfloat16)
    assert out.shape == (2, 3, 5) and out.dtype == torch.bfloat16 and out[1, 0, 4] == 68 and torch.all(out[1, 1] == 0)
    assert binding.embed(T, t[:0]).shape == (0, 3, 5)
    assert torch.equal(binding.embed(T, torch.tensor(4, device=DEV)), T[4])
    g = torch.arange(30, dtype=torch.float32, device=DEV).view(2, 3, 5)
    assert torch.equal(binding.embed_grad(g, t, 7), binding.embed_grad(g.view(6, 5), t.view(6), 7))
    assert torch.equal(binding.embed_grad(g.transpose(0, 1), t.t(), 7), binding.embed_grad(g, t, 7))     # not contiguous: copied
    big = torch.randint(0, 7, (3_000_001,), device=DEV)
    assert torch.equal(binding.embed(T, big), T[big])
    assert torch.all(binding.embed(T[:0], t) == 0)                # a table without rows: no id names one


def test_refusals_on_the_device():
    """What the binding refuses with tensors on a GPU: types, shapes, places."""
    T, t = torch.zeros(4, 8, device=DEV), torch.zeros(3, dtype=torch.int64, device=DEV)
    q = binding.micro_quantize(T)
    for error, call in [(TypeError, lambda: binding.embed(T, t, dtype=torch.float64)), (TypeError, lambda: binding.embed(T.double(), t)),
                        (ValueError, lambda: binding.embed(T, t.cpu())), (ValueError, lambda: binding.embed(T.cpu(), t)), (ValueError, lambda: binding.embed(T, t, out=T)),
                        (ValueError, lambda: binding.embed(T, t, dtype=torch.float16, out=T[:3])), (ValueError, lambda: binding.embed(T.t(), t)),
                        (binding.SameLdaError, lambda: binding.embed(T, t, float("nan"))), (ValueError, lambda: binding.embed_grad(T[:3], t, 5, out=T)),
                        (ValueError, lambda: binding.embed_grad(T, t, 5)), (binding.SameLdaError, lambda: binding.embed_grad(T[:3], t, 5, float("inf"))),
                        (TypeError, lambda: binding.micro_dequantize(q, dtype=torch.int32)), (TypeError, lambda: binding.micro_quantize(T, out=T)),
                        (binding.SameLdaError, lambda: binding.micro_quantize(T[:, :4], out=q)), (binding.SameLdaError, lambda: binding.micro_product(q, binding.micro_quantize(T[:, :7].contiguous()))),
                        (ValueError, lambda: binding.micro_product(q, q, out=T)), (ValueError, lambda: binding.micro_product(T.cpu(), q))]:
        with pytest.raises(error):
            call()


def test_padding_never_reads_the_table_nor_the_gradient():
    T = torch.full((5, 64), float("nan"), device=DEV)
    T[2] = 1.0
    t = torch.tensor([2, -1, 5, 2], device=DEV)
    assert torch.equal(binding.embed(T, t).sum(1).cpu(), torch.tensor([64.0, 0.0, 0.0, 64.0]))
    g = torch.ones(4, 64, device=DEV)
    g[1], g[2] = float("nan"), float("inf")
    got = binding.embed_grad(g, t, 5)
    assert torch.all(got[2] == 2.0) and got.sum().item() == 128.0
    x = torch.tensor([[float("inf"), 1.0], [float("nan"), 2.0], [3.0, float("-inf")]], device=DEV)   # what is read goes on
    assert torch.equal(torch.isfinite(binding.embed(x, torch.tensor([2, 1, 0], device=DEV))).cpu(), torch.tensor([[True, False], [False, True], [False, True]]))
    s = binding.embed_grad(x, torch.tensor([0, 0, 1], device=DEV), 2)
    assert torch.isnan(s[0, 0]) and s[0, 1] == 3.0 and s[1, 1] == float("-inf")
    for n in (3000, 12_000, 40_000):                              # every way to the sums: most rows stand for no word
        t = torch.randint(0, 300, (n,), device=DEV)
        t[::3], t[1::3] = -1, 300 + 300 * torch.randint(0, 1 << 40, (len(t[1::3]),), device=DEV)
        t[1], t[4] = 1 << 33, -(1 << 40)
        g = torch.full((n, 24), float("nan"), device=DEV)
        known = (t >= 0) & (t < 300)
        g[known] = torch.randint(-8, 9, (int(known.sum()), 24), device=DEV).float()
        want = torch.zeros(300, 24, dtype=torch.float64).index_add_(0, t[known].cpu(), g[known].double().cpu())
        assert torch.equal(binding.embed_grad(g, t, 300).double().cpu(), want)
        none = torch.full((n,), -1, device=DEV)
        assert torch.all(binding.embed_grad(g, none, 300) == 0.0)
        assert torch.all(binding.embed_grad(g, none, out=torch.full((300, 24), 2.0, device=DEV), accumulate=True) == 2.0)


# ---- gradient

def check_grad(G, t, V, scale, got, out, before=None):
    want, size, terms = wt.embed_grad(G.double().numpy(), t, V, scale)
    deep = np.minimum(terms, 256 + terms // 256 + 2).astype(np.float64)[:, None]
    extra = 1.01 * U * deep * size + U * size
    if before is not None:
        want = want + before
        extra = extra + 2 * U * (np.abs(before) + size)
    close(got, want, out, extra)
    if before is not None:
        untouched = torch.from_numpy(terms == 0)
        assert torch.equal(got.cpu()[untouched].double(), torch.from_numpy(before)[untouched])


# one token, tiles of the sort and their borders, runs of every length up to several pieces, words in one, two and three digits
@pytest.mark.parametrize("n, V, width", [(1, 1, 1), (1, 5000, 64), (2, 3, 65), (77, 2000, 50), (255, 1, 16), (256, 1, 16), (257, 1, 16), (513, 2, 24), (4095, 10, 3),
                                         (4096, 300, 8), (4097, 511, 8), (4100, 512, 12), (2048, 5000, 20), (2049, 700, 7), (8192, 900, 12), (8193, 900, 12), (16_384, 700, 6), (16_385, 700, 6), (16_000, 5, 66), (12_000, 40_000, 2), (8000, 3, 300), (7001, 20_000, 1), (6000, 1300, 2), (5000, 40, 1000), (63, 1, 8), (64, 2, 8),
                                         (65, 1, 8), (9001, 70_000, 33), (20_000, 3, 130), (22_345, 300_000, 4), (30_000, 40, 257), (19_001, 70_000, 33), (20_480, 511, 8), (20_481, 512, 12)])
@pytest.mark.parametrize("kind", ["even", "skewed"])
def test_embed_grad_matches_the_oracle(n, V, width, kind):
    rng = np.random.default_rng(n + V)
    G = numbers_of(rng, n, width, torch.float32)
    t = words(rng, n, V, kind)
    if n > 3:
        t[3] = V + 1
    got, check = guarded(V, width, torch.float32, offset=4)
    binding.embed_grad(G.to(DEV), torch.from_numpy(t).to(DEV), scale=1.5, out=got)
    check_grad(G, t, V, 1.5, got, torch.float32)
    check()
    again = binding.embed_grad(G.to(DEV), torch.from_numpy(t.astype(np.int32)).to(DEV), V, 1.5)
    assert torch.equal(again, got)                                   # the other type of tokens, the same bits


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("grad", TYPES)
@pytest.mark.parametrize("n, width", [(1500, 5), (1500, 16), (1500, 66), (1500, 512), (17_000, 5), (17_000, 16), (17_000, 66), (9000, 1032)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_grad_types_strides_and_accumulation(grad, out, n, width, accumulate):
    rng = np.random.default_rng(width)
    V = 23
    G = numbers_of(rng, n, width, TYPES[grad]) * 0.25
    t = words(rng, n, V, "skewed")
    t[t == 20] = 19
    stride = width + (8 if width % 8 == 0 else 3)
    g, _ = guarded(n, width, TYPES[grad], stride, 8)
    g.copy_(G)
    got, check = guarded(V, width, TYPES[out], stride, 16)
    before = None
    if accumulate:
        old = numbers_of(rng, V, width, TYPES[out])
        got.copy_(old)
        before = old.double().numpy()
    binding.embed_grad(g, torch.from_numpy(t).to(DEV), scale=-0.75, out=got, accumulate=accumulate)
    check_grad(G, t, V, -0.75, got, TYPES[out], before)
    check()


def test_embed_grad_is_exact_on_integers_and_on_one_word():
    for n in (1, 256, 300, 5000, 70_001):
        g = torch.randint(-8, 9, (n, 40), device=DEV, dtype=torch.float32)
        t = torch.full((n,), 2, device=DEV, dtype=torch.int32)
        got = binding.embed_grad(g, t, 4)                            # sums below 2^24: every order gives the integer
        assert torch.equal(got[2].double(), g.double().sum(0)) and torch.all(got[[0, 1, 3]] == 0)
    # many tokens: words of two digits and of three, tiles of either size, words that are few and many for the tokens
    for n, V, width in [(200_003, 5000, 20), (70_001, 300_000, 3), (70_001, 270_000, 2), (4_300_001, 600, 2)]:
        g = torch.randint(-8, 9, (n, width), device=DEV, dtype=torch.float32)
        t = (torch.rand(n, device=DEV, dtype=torch.float64) ** 6 * V).long()
        want = torch.zeros(V, width, dtype=torch.float64).index_add_(0, t.cpu(), g.double().cpu())
        assert torch.equal(binding.embed_grad(g, t, V).double().cpu(), want)


def test_embed_grad_without_tokens_or_words():
    g = torch.ones(3, 8, device=DEV)
    out = torch.full((6, 8), 5.0, device=DEV)
    binding.embed_grad(g[:0], torch.zeros(0, dtype=torch.int64, device=DEV), out=out, accumulate=True)
    assert torch.all(out == 5.0)
    binding.embed_grad(g[:0], torch.zeros(0, dtype=torch.int64, device=DEV), out=out)
    assert torch.all(out == 0.0)
    out.fill_(5.0)
    binding.embed_grad(g, torch.full((3,), -1, device=DEV), out=out, accumulate=True)
    assert torch.all(out == 5.0)
    binding.embed_grad(g, torch.full((3,), -1, device=DEV), out=out)
    assert torch.all(out == 0.0)
    assert binding.embed_grad(g, torch.zeros(3, dtype=torch.int64, device=DEV), 0).shape == (0, 8)


def test_gradient_against_differences_of_the_lookup():
    """Small integers: the lookup, a weighted sum of its rows and the difference quotient are exact in binary32."""
    rng = np.random.default_rng(5)
    t = torch.from_numpy(words(rng, 40, 6, "even")).to(DEV)
    T = torch.from_numpy(rng.integers(-9, 10, (6, 3)).astype(np.float32)).to(DEV)
    w = torch.from_numpy(rng.integers(-9, 10, (40, 3)).astype(np.float32)).to(DEV)
    g = binding.embed_grad(w, t, 6, 2.0)
    base = (binding.embed(T, t, 2.0) * w).sum()
    for r in range(6):
        for c in range(3):
            up = T.clone()
            up[r, c] += 1.0
            assert ((binding.embed(up, t, 2.0) * w).sum() - base).item() == g[r, c].item()


# ---- four bits

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, width", [(1, 1), (3, 31), (5, 32), (4, 33), (7, 50), (2, 127), (9, 128), (6, 129), (3, 250), (2, 1000)])
def test_quantize_and_back_are_exact(rows, width, dtype):
    rng = np.random.default_rng(width)
    x = numbers_of(rng, rows, width, TYPES[dtype])
    x.view(-1)[::7] = 0.0
    x[0, width // 2] = -0.0
    codes, scales = wt.quantize(x.double().numpy())
    src, _ = guarded(rows, width, TYPES[dtype], width + 5, 3)
    src.copy_(x)
    for y in (x.to(DEV), src):
        q = binding.micro_quantize(y)
        assert q.shape == (rows, width)
        assert np.array_equal(q.scales.cpu().numpy(), scales) and np.array_equal(q.codes.cpu().numpy(), codes)
    want = wt.numbers(codes, scales, width)
    for name in TYPES:
        got, check = guarded(rows, width, TYPES[name], width + 1, 2)
        binding.micro_dequantize(q, out=got)
        close(got, want, TYPES[name])
        check()
    assert np.array_equal(binding.micro_dequantize(q).cpu().double().numpy(), want)


def test_quantize_every_tie_every_exponent_and_bad_blocks():
    steps = np.array([0, .2, .25, .26, .5, .74, .75, .76, 1, 1.25, 1.3, 1.5, 1.75, 1.8, 2, 2.4, 2.5, 2.6, 3, 3.4, 3.5, 3.6, 4, 4.9, 5, 5.1, 6, 6.9, 7, 7.5, 7.99, 4.0])
    x = np.stack([np.concatenate((steps, -steps)) * 2.0 ** (e - 2) for e in range(-149, 126)]).astype(np.float32)
    just = np.nextafter(x, np.float32(np.inf))                       # one step above every border, and one below
    x = np.concatenate((x, just, np.nextafter(x, np.float32(-np.inf))))
    bad = np.zeros((5, 64), np.float32)
    bad[0, 3], bad[1, 40], bad[2, 0], bad[3, :], bad[4, 63] = np.nan, np.inf, -np.inf, 1e38, 3.4e38
    x = np.concatenate((x, bad))
    codes, scales = wt.quantize(x)
    q = binding.micro_quantize(torch.from_numpy(x).to(DEV))
    assert np.array_equal(q.scales.cpu().numpy(), scales) and np.array_equal(q.codes.cpu().numpy(), codes)
    got = binding.micro_dequantize(q).cpu().numpy()
    np.testing.assert_array_equal(got, wt.numbers(codes, scales, 64).astype(np.float32))
    assert np.isnan(got[-5, :32]).all() and np.isfinite(got[-5, 32:]).all()


@pytest.mark.parametrize("width", [1, 2, 50, 64, 200, 256])
@pytest.mark.parametrize("out", TYPES)
def test_embed_from_four_bits(width, out):
    rng = np.random.default_rng(width)
    x = numbers_of(rng, 29, width, torch.float32)
    codes, scales = wt.quantize(x.double().numpy())
    q = binding.MicroMatrix(torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), width)
    t = words(rng, 45, 29, "even")
    got, check = guarded(45, width, TYPES[out], width + (width & 1), 8)
    binding.embed(q, torch.from_numpy(t).to(DEV), 1.7, out=got)
    close(got, wt.embed(wt.numbers(codes, scales, width), t, np.float32(1.7)), TYPES[out])
    check()
    assert torch.equal(binding.embed(q[3:9], torch.tensor([0, 5], device=DEV)), binding.micro_dequantize(q)[[3, 8]])


def random_micro(rng, rows, width, low=117, high=135):
    """Codes and scales at random, zero in the filling."""
    groups = -(-width // 128)
    half = rng.integers(0, 16, (rows, groups * 128)).astype(np.uint8)
    half[:, width:] = 0
    scales = rng.integers(low, high, (rows, groups * 4)).astype(np.uint8)
    scales[:, -(-width // 32):] = 0
    return half[:, 0::2] | (half[:, 1::2] << 4), scales


def micro(codes, scales, width):
    return binding.MicroMatrix(torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), width)


PRODUCTS = [(1, 1, 1), (1, 100, 33), (1, 1000, 256), (2, 17, 129), (5, 300, 1000), (13, 501, 640), (16, 16, 128), (16, 4096, 512), (17, 65, 129), (33, 1, 4096), (64, 64, 256),
            (100, 1030, 200), (128, 128, 384), (130, 257, 384), (255, 300, 1024), (300, 513, 2048), (512, 520, 640), (1025, 300, 256), (20, 33_000, 1030), (31, 4500, 1024), (40, 36_000, 700), (25, 300, 500), (70, 700, 384), (1300, 1500, 640), (2100, 5000, 100)]


@pytest.mark.parametrize("M, N, K", PRODUCTS)
@pytest.mark.parametrize("out", TYPES)
def test_product_matches_the_oracle(M, N, K, out):
    rng = np.random.default_rng(M + N + K)
    a, b = random_micro(rng, M, K, 120, 130), random_micro(rng, N, K, 120, 130)
    want, size = wt.product(wt.numbers(*a, K), wt.numbers(*b, K), 2.0 ** -7)
    got, check = guarded(M, N, TYPES[out], N + 5, 3)
    binding.micro_product(micro(*a, K), micro(*b, K), 2.0 ** -7, out=got)
    close(got, want, TYPES[out], 2 * U * K * size)
    check()
    aligned, check = guarded(M, N, TYPES[out], -(-N // 8) * 8, 8)
    binding.micro_product(micro(*a, K), micro(*b, K), 2.0 ** -7, out=aligned)
    assert torch.equal(aligned, got)
    check()


@pytest.mark.parametrize("M, N, K", PRODUCTS + [(3, 2000, 8192), (700, 900, 1100), (2048, 64, 320), (4100, 4150, 1100), (3900, 4300, 1200)])
def test_product_of_small_numbers_is_exact(M, N, K):
    """Scales of one: every sum is a multiple of 1/4 below 2^22, exact in binary32 in any order; a wrong pairing of elements or
    blocks shows."""
    rng = np.random.default_rng(M * 7 + N + K)
    a, b = random_micro(rng, M, K, 127, 128), random_micro(rng, N, K, 127, 128)
    want = wt.numbers(*a, K) @ wt.numbers(*b, K).T
    got = binding.micro_product(micro(*a, K), micro(*b, K))
    assert np.array_equal(got.cpu().double().numpy(), want)
    # and blocks that differ by powers of two: one block of a row counts, the others are zero
    a[0][:, :], a[1][:, :] = 0, 0
    for i in range(M):
        block = rng.integers(0, -(-K // 32))
        n = min(32, K - block * 32)
        a[0][i, block * 16:block * 16 + n // 2] = rng.integers(0, 256, n // 2)
        a[1][i, block] = rng.integers(100, 150)
    b[1][:, :-(-K // 32)] = rng.integers(100, 150, (N, -(-K // 32)))
    want = wt.numbers(*a, K) @ wt.numbers(*b, K).T
    got = binding.micro_product(micro(*a, K), micro(*b, K))
    assert np.array_equal(got.cpu().double().numpy(), want)


@pytest.mark.parametrize("M, N", [(1, 70), (40, 70), (300, 270)])
def test_product_bad_blocks_spoil_their_rows_only(M, N):
    rng = np.random.default_rng(M)
    a, b = random_micro(rng, M, 200), random_micro(rng, N, 200)
    a[1][M - 1, 2] = 255
    b[1][3, 6] = 255
    got = binding.micro_product(micro(*a, 200), micro(*b, 200)).cpu().numpy()
    want = np.zeros((M, N), bool)
    want[M - 1, :], want[:, 3] = True, True
    assert np.array_equal(np.isnan(got), want)


@pytest.mark.parametrize("M, N, K", [(1, 130, 1), (1, 130, 300), (5, 33, 300), (16, 1000, 1024), (3, 70, 1025), (1, 500, 16384), (1, 40_000, 1500), (2, 300, 8192), (2, 300, 8193), (17, 64, 8), (17, 3000, 963), (32, 2000, 512), (33, 100, 496), (50, 900, 70), (64, 5000, 256), (64, 30, 1), (65, 200, 100),
                                     (300, 130, 300)])
def test_product_rounds_a_matrix_first(M, N, K):
    """In the same call where it is small (64 rows, 16384 elements, above 16 rows by a small table), in a call before otherwise: up
    to 16 rows the same kernel, so the same bits.  Above, the two are sums of the same terms in two orders: each is off by
    at most 2 u K times the sum of the magnitudes (as above), so they differ by twice that and the rounding of either."""
    rng = np.random.default_rng(M + K)
    numbers = random_micro(rng, N, K)
    b = micro(*numbers, K)
    for dtype in TYPES.values():
        x = numbers_of(rng, M, K, dtype).to(DEV)
        x.view(-1)[::5] = 0.0
        q = binding.micro_quantize(x)
        want = binding.micro_product(q, b, 0.5, dtype=dtype)
        view, _ = guarded(M, K, dtype, K + 3, 1)
        view.copy_(x)
        for y in (x, view):
            got = binding.micro_product(y, b, 0.5, dtype=dtype)
            if M <= 16:
                assert torch.equal(got, want)
            else:
                _, size = wt.product(wt.numbers(q.codes.cpu().numpy(), q.scales.cpu().numpy(), K), wt.numbers(*numbers, K), 0.5)
                rel, floor = half_step(dtype)
                far = (got.double() - want.double()).abs().cpu().numpy()
                assert np.all(far <= 4 * U * K * size + 2 * (rel + U) * (np.abs(want.double().cpu().numpy()) + 4 * U * K * size) + 2 * floor)
        x[M - 1, K // 2] = float("nan")
        assert torch.isnan(binding.micro_product(x, b)[M - 1]).all()


def test_product_without_rows():
    rng = np.random.default_rng(0)
    a, b = micro(*random_micro(rng, 3, 40), 40), micro(*random_micro(rng, 4, 40), 40)
    assert binding.micro_product(a[:0], b).shape == (0, 4)
    assert binding.micro_product(a, b[:0]).shape == (3, 0)


# ---- streams, graphs, sizes

def everything(T, t, g, x):
    """All operators in a row, as a training step and the serving of its table use them."""
    e = binding.embed(T, t, 2.0)
    dT = binding.embed_grad(g, t, T.shape[0], 2.0)
    q = binding.micro_quantize(T - 0.01 * dT)
    return e, dT, q.codes, q.scales, binding.embed(q, t, dtype=torch.bfloat16), binding.micro_product(x, q), binding.micro_dequantize(q)


def inputs(seed, n, rows, V=700, E=416):
    rng = np.random.default_rng(seed)
    return (numbers_of(rng, V, E, torch.float32).to(DEV), torch.from_numpy(words(rng, n, V, "skewed")).to(DEV), numbers_of(rng, n, E, torch.float32).to(DEV),
            numbers_of(rng, rows, E, torch.bfloat16).to(DEV))


# the gradient in one launch and by a sort, the product that rounds by itself, in small tiles and in large ones
CALLS = [(3000, 7), (40_000, 70), (12_000, 5000)]


@pytest.mark.parametrize("n, rows", CALLS)
def test_other_streams_at_once_give_the_same(n, rows):
    sets = [inputs(s, n, rows) for s in range(3)]
    want = [everything(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = []
    for s, st in zip(sets, streams):
        with torch.cuda.stream(st):
            got.append([everything(*s) for _ in range(4)][-1])
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(a, b) for a, b in zip(w, g))


def test_threads_at_once_give_the_same():
    sets = [inputs(s, 20_000, 40) for s in range(4)]
    want = [everything(*s) for s in sets]
    torch.cuda.synchronize()
    got = [None] * len(sets)

    def work(k):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(5):
                got[k] = everything(*sets[k])
                try:
                    binding.micro_product(sets[k][3], binding.micro_quantize(sets[k][0][:, :100 + k]))
                except binding.SameLdaError as e:                     # the text is the calling thread's
                    assert f"and of {100 + k} elements" in str(e)
                else:
                    raise AssertionError
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(sets))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for w, g in zip(want, got):
        assert all(torch.equal(a, b) for a, b in zip(w, g))


@pytest.mark.parametrize("n, rows", CALLS)
def test_captured_calls_replay_on_new_inputs(n, rows):
    a, b = inputs(1, n, rows), inputs(2, n, rows)
    held = [x.clone() for x in a]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        everything(*held)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):                                                # two graphs of the same calls, replayed in turn
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = everything(*held)
        graphs.append((g, out))
    for s in (a, b, a, b):
        want = everything(*s)
        for h, x in zip(held, s):
            h.copy_(x)
        for g, out in graphs:
            g.replay()
        torch.cuda.synchronize()
        for g, out in graphs:
            assert all(torch.equal(x, y) for x, y in zip(want, out))


def test_offsets_beyond_32_bits():
    rows, width = 2_200_000, 1024                                     # 4.5 GB, 2.25 G elements
    T = torch.zeros(rows, width, dtype=torch.bfloat16, device=DEV)
    T[rows - 1], T[rows - 2, 5] = 3.0, 4.0
    t = torch.tensor([rows - 1, rows - 2, 0], device=DEV)
    e = binding.embed(T, t)
    assert torch.all(e[0] == 3.0) and e[1, 5] == 4.0 and e[1].sum() == 4.0 and e[2].sum() == 0.0
    g = binding.embed_grad(e, t, out=T)
    assert torch.all(T[rows - 1] == 3.0) and T[rows - 2, 5] == 4.0 and T[:rows - 2].count_nonzero() == 0 and g is T
    del T, g
    n = 2_200_000                                                     # the gradient's rows pass 2^31 elements
    G = torch.zeros(n, width, dtype=torch.bfloat16, device=DEV)
    G[n - 3:] = 1.0
    out = binding.embed_grad(G, (torch.arange(n, device=DEV) >= n - 3).long(), 2, dtype=torch.float32)
    assert torch.all(out[0] == 0) and torch.all(out[1] == 3.0)
    q = binding.micro_quantize(G)
    del G
    y = binding.micro_product(q[n - 4:], q)
    assert torch.all(y[0] == 0) and torch.all(y[1:, n - 3:] == 1024.0) and y.count_nonzero() == 9
    y = binding.micro_product(q, q[n - 4:], dtype=torch.bfloat16)
    assert torch.all(y[n - 3:, 1:] == 1024.0) and y.count_nonzero() == 9


def test_product_of_many_short_rows():
    n = (1 << 28) + 70                                                # codes beyond 2^32 bytes, more rows than one launch takes
    codes = torch.zeros(n, 64, dtype=torch.uint8, device=DEV)
    codes[n - 1, 0] = 0x22
    q = binding.MicroMatrix(codes, torch.full((n, 4), 127, dtype=torch.uint8, device=DEV), 128)
    for rows in (1, 20):
        a = binding.micro_quantize(torch.ones(rows, 128, device=DEV))
        y = binding.micro_product(a, q, dtype=torch.bfloat16)
        assert torch.all(y[:, n - 1] == 2.0) and y.count_nonzero() == rows


def test_with_a_fitted_model():
    """phi of a small model: copied out on the device, its rows looked up, kept in four bits, and the predictive weights of all
    documents over the vocabulary; theta and phi rounded to four bits against the same product of what they stand for."""
    rng = np.random.default_rng(9)
    counts = rng.integers(1, 9, size=(40, 120)) * (rng.uniform(size=(40, 120)) < 0.3)
    X = csc_from_dense(counts)
    g = binding.SameLDA(X.D, X.V, X.colptr, X.rowidx, X.val, 24, 0.1, 0.01, seed=4, m0=10)
    g.sweep(10)
    phi = g.get(binding.PHI, out=torch.empty(X.V, 24, device=DEV))
    theta = g.get(binding.THETA, out=torch.empty(X.D, 24, device=DEV))
    assert np.array_equal(phi.cpu().numpy(), g.get(binding.PHI)) and np.array_equal(theta.cpu().numpy(), g.get(binding.THETA))
    assert np.array_equal(g.get(binding.NDK, out=torch.empty(X.D, 24, dtype=torch.int32, device=DEV)).cpu().numpy().astype(np.uint32), g.get(binding.NDK))
    with pytest.raises(ValueError):
        g.get(binding.PHI, out=torch.empty(X.V, 25, device=DEV))
    ids = torch.from_numpy(X.rowidx).to(DEV)
    assert torch.equal(binding.embed(phi, ids), phi[ids.long()])
    q = binding.micro_quantize(phi)
    y = binding.micro_product(theta, q)
    a, b = wt.quantize(theta.cpu().numpy()), wt.quantize(phi.cpu().numpy())
    want, size = wt.product(wt.numbers(*a, 24), wt.numbers(*b, 24), 1.0)
    close(y, want, torch.float32, 2 * U * 24 * size)
    # the gradient of sum over the tokens of c log p(w | d), p = theta . phi_w / sum theta, with respect to phi, by words
    doc = np.repeat(np.arange(X.D), np.diff(X.colptr))
    mu = torch.from_numpy(g.sddmm()).to(DEV)
    rows = theta[torch.from_numpy(doc).to(DEV)] * (torch.from_numpy(X.val).to(DEV) / mu).unsqueeze(1)
    got = binding.embed_grad(rows, ids, X.V)
    want, size, terms = wt.embed_grad(rows.cpu().double().numpy(), X.rowidx, X.V, 1.0)
    close(got, want, torch.float32, 1.01 * U * (terms[:, None] + 1) * size)
    g.close()
