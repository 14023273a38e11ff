"""Grouped four-bit integers: rounding, reading back, lookup and product, against the oracle in double (oracle/word_rows.py).

Rounding and the layout are exact.  Reading back is q s + b, rounded once to binary32 (u = 2^-24) and once to the output's type.

Product.  A group adds s D + b S with D = sum a q and S = sum a.  Products of 16-bit numbers are exact, rows in
binary32 are three of them; every addition of a matrix instruction is taken to be off by a whole step, 2 u: with N = G or 3 G terms,
D is off by 2 u N times 15 A and S by 2 u N times A, A = sum |a| over the group.  Two fused additions per group round (u each, of sums
below the whole).  All of it is at most (2 N + 2 groups) u times M = sum over groups of (15 s + |b|) A, which the oracle gives; then
the scale and the output's type: u + eps/2."""
import numpy as np
import pytest
import torch

from oracle import word_rows as wr
from paper_1409_5402_amd import binding

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
GROUPS = [32, 64, 128]


def half_step(dtype):
    f = torch.finfo(dtype)
    return f.eps / 2, f.smallest_normal * f.eps / 2


def close(got, want, dtype, extra=0.0):
    rel, floor = half_step(dtype)
    got = got.double().cpu().numpy()
    bound = 1.01 * extra + (rel + 1.01 * U) * (np.abs(want) + extra) + floor
    bad = ~(np.abs(got - want) <= bound) & ~(np.isnan(got) & np.isnan(want)) & ~(got == want) & ~np.isinf(bound)
    most = torch.finfo(dtype).max * (1 + rel)                             # from here on the nearest number of the type is infinite
    bad &= ~((want + bound >= most) & (got == np.inf)) & ~((want - bound <= -most) & (got == -np.inf))
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


def numbers_of(rng, rows, cols, dtype, positive=False):
    x = rng.normal(size=(rows, cols)) * np.exp(rng.normal(size=cols))
    return torch.from_numpy(np.exp(1.5 * x) / cols if positive else x).to(dtype)


def parts(q):
    """codes (bytes), steps and bases of a GroupMatrix as the oracle has them"""
    s = q.scales.double().cpu().numpy()
    return q.codes.cpu().numpy(), s[:, :, 0], s[:, :, 1]


def guarded(rows, cols, dtype, stride=None, offset=0):
    stride = cols if stride is None else stride
    buf = torch.full((offset + rows * stride + 300,), 7.0, dtype=dtype, device=DEV)
    view = torch.as_strided(buf, (rows, cols), (stride, 1), offset)

    def check():
        b = buf.clone()
        torch.as_strided(b, (rows, cols), (stride, 1), offset).fill_(7.0)
        assert torch.all(b == 7.0)
    return view, check


def same(q, x, group):
    """The grouped form of x is the oracle's, bit for bit."""
    codes, step, base = parts(q)
    oq, os_, ob = wr.group_quantize(x.double().cpu().numpy(), group)
    assert np.array_equal(step, os_, equal_nan=True) and np.array_equal(base, ob, equal_nan=True)
    assert not (codes != wr.group_layout(oq)).any()


# ---- rounding, reading back, lookup

@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [1, 7, 8, 31, 33, 127, 128, 129, 250, 256])
def test_rounding_is_the_oracles_bit_for_bit(width, dtype, group):
    rng = np.random.default_rng(width)
    x = numbers_of(rng, 19, width, TYPES[dtype])
    x[3] = x[3].abs()
    x[4] = -x[4].abs()
    x[5] = 0.0
    x[6] = 1.5
    q = binding.group_quantize(x.to(DEV), group)
    same(q, x, group)
    oq, s, b = wr.group_quantize(x.double().numpy(), group)
    for out in TYPES.values():
        close(binding.group_dequantize(q, dtype=out), wr.group_numbers(oq, s, b, width), out)


def test_rounding_of_ties_borders_and_the_ends_of_the_range():
    top = float(torch.finfo(torch.float32).max)
    rng = np.random.default_rng(1)
    ties = torch.zeros(64, 128)
    ties[:, 0], ties[:, 1] = 0.0, 15.0
    ties[:, 2:] = torch.from_numpy(rng.integers(0, 31, (64, 126))).float() / 2                       # every half of a step
    ties[1::2] = torch.nextafter(ties[1::2], torch.tensor(torch.inf))                                # and just off it
    ties[2::4] = torch.nextafter(ties[2::4], torch.tensor(-torch.inf))
    ties *= 2.0 ** torch.arange(-32, 32).unsqueeze(1)
    ends = torch.zeros(12, 128)
    ends[0, 0] = top
    ends[1, 0], ends[1, 1] = top, -top
    ends[2, 5] = 2.0 ** -149
    ends[3] = 2.0 ** -140 * torch.arange(128)
    ends[4] = -top
    ends[5, 3] = float("nan")
    ends[6, 100] = float("inf")
    ends[7, 31] = float("-inf")
    ends[8] = -0.0
    ends[9] = 1e30 + 1e23 * torch.arange(128)
    ends[10, 1:] = 1e-38 * torch.arange(1, 128)
    ends[11] = -1e30 - 1e23 * torch.arange(128)
    offset = torch.from_numpy(1000 + rng.normal(size=(20, 128))).float()
    small = torch.from_numpy(rng.normal(size=(40, 128)) * 2.0 ** np.arange(-148, -108)[:, None]).float()      # steps that are subnormal, or nearly
    large = torch.from_numpy(rng.normal(size=(8, 128)) * 2.0 ** np.arange(118, 126)[:, None]).float()
    coarse = torch.from_numpy(rng.integers(-60, 61, (200, 128)) / 4).bfloat16().float()                       # many numbers on a border
    for x in (ties, ends, offset, small, large, coarse):
        for group in GROUPS:
            same(binding.group_quantize(x.to(DEV), group), x, group)


@pytest.mark.parametrize("stride, offset", [(70, 0), (71, 0), (70, 1), (72, 3), (80, 8)])
@pytest.mark.parametrize("dtype", TYPES)
def test_rounding_of_strided_rows_and_into_given_places(dtype, stride, offset):
    rng = np.random.default_rng(stride)
    X = numbers_of(rng, 21, 70, TYPES[dtype])
    x, _ = guarded(21, 70, TYPES[dtype], stride, offset)
    x.copy_(X)
    q = binding.group_quantize(x, 32)
    same(q, X, 32)
    out = binding.GroupMatrix(torch.empty_like(q.codes), torch.empty_like(q.scales), 70, 32)
    assert binding.group_quantize(x, out=out) is out and torch.equal(out.codes, q.codes) and torch.equal(out.scales, q.scales)


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("width", [1, 9, 50, 128, 200, 1000])
def test_lookup_of_grouped_rows(width, group, out):
    rng = np.random.default_rng(width)
    q = binding.group_quantize(numbers_of(rng, 37, width, torch.float32).to(DEV), group)
    codes, s, b = parts(q)
    t = rng.integers(-1, 38, 53)
    oq, _, _ = wr.group_quantize(numbers_of(np.random.default_rng(width), 37, width, torch.float32).double().numpy(), group)
    known = (t >= 0) & (t < 37)
    want = np.where(known[:, None], wr.group_numbers(oq, s, b, width)[np.where(known, t, 0)], 0.0) * 1.75
    got, check = guarded(53, width, TYPES[out], width + 5, 3)
    binding.embed(q, torch.from_numpy(t).to(DEV), 1.75, out=got)
    close(got, want, TYPES[out], U * np.abs(want))
    check()
    assert torch.equal(binding.embed(q, torch.from_numpy(t.astype(np.int32)).to(DEV), 1.75, dtype=TYPES[out]), got)
    assert torch.equal(binding.group_dequantize(q[3:20]), binding.group_dequantize(q)[3:20])


# ---- product

def tolerance(a, size, q):
    n = q.group * (3 if a.dtype == torch.float32 else 1)
    # s D and b S are at most M: where that is beyond binary32 they may be infinite, and nothing is said of the result
    most = float(torch.finfo(torch.float32).max)
    # a group's D = sum a q, q up to 15, is infinite where 15 sum |a| is beyond binary32, however small the step that it is multiplied with
    A = np.abs(a.double().cpu().numpy())
    D = 15.0 * np.pad(A, ((0, 0), (0, -A.shape[1] % q.group))).reshape(A.shape[0], -1, q.group).sum(2).max(axis=1)
    return np.where((size < most) & (D < most)[:, None], (2 * n + 2 * q.scales.shape[1]) * U * size, np.inf)


def product_case(rng, M, N, K, dtype, group, out, scale=1.0, positive=False, a=None):
    x = numbers_of(rng, M, K, TYPES[dtype], positive)
    w = numbers_of(rng, N, K, torch.float32, positive)
    q = binding.group_quantize(w.to(DEV), group)
    oq, s, b = wr.group_quantize(w.double().numpy(), group) if N * K <= 60_000 else (None, None, None)
    if oq is None:                                        # large: what the table stands for, read back (tested above)
        _, s, b = parts(q)
        numbers = binding.group_dequantize(q).double().cpu().numpy()
        A = np.abs(x.double().numpy())
        A = np.pad(A, ((0, 0), (0, s.shape[1] * group - K))).reshape(M, -1, group).sum(2)
        want, size = scale * (x.double().numpy() @ numbers.T), abs(scale) * (A @ (15.0 * np.abs(s) + np.abs(b)).T)
        size = size + scale * size / 2                    # the read-back's own rounding is below u |w|
    else:
        want, size = wr.group_product(x.double().numpy(), oq, s, b, scale)
    got, check = guarded(M, N, TYPES[out], N + 3, 1) if a is None else a
    binding.group_product(x.to(DEV), q, scale, out=got)
    close(got, want, TYPES[out], tolerance(x, size, q))
    check()
    return x, q, got


SHAPES = [(1, 1, 1), (1, 16, 128), (1, 17, 129), (3, 5, 31), (5, 33, 250), (6, 40, 96), (13, 100, 300), (16, 64, 256), (17, 31, 130), (31, 65, 512), (33, 20, 200), (64, 48, 384), (65, 130, 64), (130, 70, 160),
          (1, 17, 4101), (17, 31, 4130), (33, 20, 4200), (65, 130, 4097), (130, 70, 4224)]


@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M, N, K", SHAPES)
def test_product_matches_the_oracle(M, N, K, dtype, group):
    rng = np.random.default_rng(M + N + K)
    product_case(rng, M, N, K, dtype, group, "f32", 0.5)
    product_case(rng, M, N, K, dtype, group, dtype, positive=True)


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_product_in_every_pair_of_types(dtype, out):
    product_case(np.random.default_rng(5), 9, 50, 190, dtype, 64, out, -1.5)
    product_case(np.random.default_rng(6), 40, 50, 190, dtype, 64, out, -1.5)
    product_case(np.random.default_rng(7), 40, 50, 4190, dtype, 64, out, -1.5)


@pytest.mark.parametrize("M, N, K", [(1, 500, 50), (1, 700, 256), (6, 300, 100), (30, 200, 512), (100, 90, 300)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", GROUPS)
def test_product_of_topic_weights(group, dtype, M, N, K):
    """Rows and a table of positive numbers, a few of them large: nothing cancels in the result."""
    rng = np.random.default_rng(K)
    x = torch.from_numpy(np.exp(1.5 * rng.normal(size=(M, K))) / K).to(TYPES[dtype])
    q = binding.group_quantize(torch.from_numpy(np.exp(1.5 * rng.normal(size=(N, K))) / K).float().to(DEV), group)
    _, s, b = parts(q)
    numbers = binding.group_dequantize(q).double().cpu().numpy()
    A = np.pad(np.abs(x.double().numpy()), ((0, 0), (0, s.shape[1] * group - K))).reshape(M, -1, group).sum(2)
    size = A @ (15.0 * np.abs(s) + np.abs(b)).T
    close(binding.group_product(x.to(DEV), q, dtype=torch.float32), x.double().numpy() @ numbers.T, torch.float32, tolerance(x, size, q) + U * size)


LONG = [(1, 3000, 4096), (2, 300, 16_384), (4, 700, 8_200), (5, 1000, 1000), (13, 2000, 2048), (16, 5000, 520), (20, 900, 4100), (48, 1500, 1024), (100, 1200, 768), (300, 600, 2050), (513, 257, 640)]


@pytest.mark.parametrize("dtype, group", [("f32", 32), ("bf16", 64), ("f16", 128), ("f32", 128), ("bf16", 32)])
@pytest.mark.parametrize("M, N, K", LONG)
def test_product_of_long_rows_and_many(M, N, K, dtype, group):
    product_case(np.random.default_rng(M + N), M, N, K, dtype, group, "f32")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M", [1, 8, 9, 16])
@pytest.mark.parametrize("K", [257, 384, 511, 513, 1030, 1537, 2049, 3000, 3968, 4095, 4097])
def test_product_of_few_rows_of_every_length(K, M, dtype):
    """Every way in which few rows are shared out between waves, the last of them with a part or none of a row."""
    for N, group in ((1, 32), (40, 64), (131, 128)):
        product_case(np.random.default_rng(K + M), M, N, K, dtype, group, "f32")


@pytest.mark.parametrize("dtype, group", [("f32", 64), ("bf16", 32), ("f16", 128), ("bf16", 64)])
@pytest.mark.parametrize("M, N, K", [(520, 49_200, 130), (65, 40_000, 200), (50, 12_000, 1100), (40, 6400, 2000), (33, 700, 4200), (20, 33_000, 700), (20, 600, 520), (7, 300, 4300), (130, 99_000, 70), (500, 600, 400)])
def test_product_in_every_form(M, N, K, dtype, group):
    """Tiles of every size, which the numbers of rows choose: against the product in double on the device, at its bound."""
    rng = np.random.default_rng(M)
    x = numbers_of(rng, M, K, TYPES[dtype]).to(DEV)
    q = binding.group_quantize(torch.randn(N, K, device=DEV, generator=torch.Generator(device=DEV).manual_seed(K)), group)
    want = x.double() @ binding.group_dequantize(q).double().t().contiguous()
    A = torch.nn.functional.pad(x.abs().double(), (0, q.scales.shape[1] * group - K)).view(M, -1, group).sum(2)
    size = A @ (15.0 * q.scales[:, :, 0].abs().double() + q.scales[:, :, 1].abs().double()).t().contiguous()
    n = group * (3 if dtype == "f32" else 1)
    bound = 1.01 * (2 * n + 3 + 2 * q.scales.shape[1]) * U * size + 2.01 * U * want.abs()
    got, check = guarded(M, N, torch.float32, N + 1, 1)
    binding.group_product(x, q, out=got)
    assert ((got.double() - want).abs() <= bound).all()
    check()


@pytest.mark.parametrize("M, N, K", [(1, 100, 700), (4, 90, 384), (7, 130, 1100), (16, 257, 4224), (33, 200, 900), (200, 300, 640), (33, 200, 4224), (200, 300, 4160)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", GROUPS)
def test_product_is_exact_where_binary32_is(group, dtype, M, N, K):
    """Small integers, steps and bases powers of two: every number on the way fits binary32, so the result is the integer."""
    rng = np.random.default_rng(K)
    a = torch.from_numpy(rng.integers(-3, 4, (M, K))).to(TYPES[dtype])
    codes = torch.from_numpy(rng.integers(0, 256, (N, -(-K // 128) * 64))).to(torch.uint8)
    n = -(-K // 128) * (128 // group)
    scales = torch.from_numpy(np.stack((2.0 ** rng.integers(-1, 2, (N, n)), rng.integers(-4, 5, (N, n))), axis=2)).to(torch.bfloat16)
    q = binding.GroupMatrix(codes.to(DEV), scales.to(DEV), K, group)
    w = binding.group_dequantize(q).double().cpu()
    got = binding.group_product(a.to(DEV), q, dtype=torch.float32)
    assert torch.equal(got.double().cpu(), a.double() @ w.t())


@pytest.mark.parametrize("K", [700, 4300])
@pytest.mark.parametrize("M", [1, 4, 5, 13, 40, 150])
def test_rows_in_binary32_count_with_all_their_bits(M, K):
    """One odd integer of 18 bits in each row, which no two 8-bit pieces hold: with codes as they are every sum fits binary32."""
    N, blocks = 40, -(-K // 128)
    rng = np.random.default_rng(M)
    a = torch.zeros(M, K)
    a[torch.arange(M), torch.from_numpy(rng.integers(0, K, M))] = torch.from_numpy((2 * rng.integers(1 << 16, 1 << 17, M) + 1) * rng.choice([-1, 1], M)).float()
    codes = torch.from_numpy(rng.integers(0, 256, (N, 64 * blocks))).to(torch.uint8)
    scales = torch.zeros(N, 2 * blocks, 2, dtype=torch.bfloat16)
    scales[:, :, 0] = 0.25
    q = binding.GroupMatrix(codes.to(DEV), scales.to(DEV), K, 64)
    w = binding.group_dequantize(q).double().cpu()
    assert torch.equal(binding.group_product(a.to(DEV), q).double().cpu(), a.double() @ w.t())


@pytest.mark.parametrize("K", [200, 4200])
@pytest.mark.parametrize("stride, offset", [(0, 0), (1, 0), (0, 1), (3, 5), (8, 8)])
@pytest.mark.parametrize("dtype", TYPES)
def test_product_of_strided_rows(dtype, stride, offset, K):
    rng = np.random.default_rng(200 + stride)
    q = binding.group_quantize(numbers_of(rng, 77, K, torch.float32).to(DEV), 32)
    for M in (1, 7, 30, 90):
        X = numbers_of(rng, M, K, TYPES[dtype])
        x, _ = guarded(M, K, TYPES[dtype], K + stride, offset)
        x.copy_(X)
        want = binding.group_product(X.to(DEV), q)
        assert torch.equal(binding.group_product(x, q), want)
        for o, s in ((0, 77), (1, 78), (4, 80)):
            out, check = guarded(M, 77, TYPES[dtype], s, o)
            assert torch.equal(binding.group_product(x, q, out=out), want)
            check()


@pytest.mark.parametrize("K", [300, 4300])
@pytest.mark.parametrize("dtype", TYPES)
def test_a_rows_result_does_not_depend_on_other_rows_being_finite(dtype, K):
    rng = np.random.default_rng(8)
    for M in (3, 12, 40, 130):
        x = numbers_of(rng, M, K, TYPES[dtype])
        w = numbers_of(rng, 50, K, torch.float32)
        good = binding.group_product(x.to(DEV), binding.group_quantize(w.to(DEV), 64))
        w[20, 100] = float("nan")
        q = binding.group_quantize(w.to(DEV), 64)
        y = x.clone()
        y[1, K - 1] = float("inf")
        y[2, 0] = float("nan")
        got = binding.group_product(y.to(DEV), q)
        rest = torch.ones(M, dtype=torch.bool)
        rest[1:3] = False
        cols = torch.ones(50, dtype=torch.bool)
        cols[20] = False
        assert torch.equal(got[rest][:, cols].cpu(), good[rest][:, cols].cpu())
        assert not torch.isfinite(got[1:3]).any() and torch.isnan(got[:, 20]).all()


def test_what_stands_behind_a_rows_end_does_not_count():
    """Codes behind the last element are zeros by the form, a table made elsewhere may hold others; and rows of a go on in memory."""
    rng = np.random.default_rng(9)
    for K in (1, 100, 130, 250, 4110):
        for M in (1, 6, 20, 70):
            q = binding.group_quantize(numbers_of(rng, 30, K, torch.float32).to(DEV), 32)
            x, _ = guarded(M, K, torch.bfloat16, K + 140, 1)
            x.copy_(numbers_of(rng, M, K, torch.bfloat16))
            wide = torch.as_strided(x, (M, K + 130), (K + 140, 1), 1)
            want = binding.group_product(x, q, dtype=torch.float32)
            wide[:, K:] = float("nan")
            assert torch.equal(binding.group_product(x, q, dtype=torch.float32), want)
            behind = torch.arange(q.codes.shape[1] * 2) >= K                   # element e of a block: word 4 (e // 8 % 4) + e // 32, half byte 4 (e % 2) + e % 8 // 2
            e = torch.arange(len(behind))[behind]
            half = e // 128 * 128 + (4 * (e // 8 % 4) + e % 128 // 32) * 8 + 4 * (e % 2) + e % 8 // 2
            mask = torch.zeros(len(behind), dtype=torch.uint8)
            mask[half] = 15
            q.codes |= (mask[::2] | mask[1::2] << 4).to(DEV)
            assert torch.equal(binding.group_product(x, q, dtype=torch.float32), want)


def test_streams_and_graphs_and_repeats():
    rng = np.random.default_rng(10)
    for M, N, K in [(1, 3000, 1024), (13, 2000, 2048), (200, 700, 512), (200, 700, 4200)]:
        x = numbers_of(rng, M, K, torch.bfloat16).to(DEV)
        q = binding.group_quantize(numbers_of(rng, N, K, torch.float32).to(DEV), 64)
        want = binding.group_product(x, q)
        for _ in range(3):
            assert torch.equal(binding.group_product(x, q), want)
        s = [torch.cuda.Stream() for _ in range(2)]
        outs = []
        for st in s:
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                outs.append(binding.group_product(x * 2.0, q))
        for st in s:
            torch.cuda.current_stream().wait_stream(st)
        assert all(torch.equal(o, want * 2.0) for o in outs)
        out, src = torch.empty_like(want), x.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            binding.group_product(src, q, out=out)
        for k in range(3):
            src.copy_(x * 2.0 ** k)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want * 2.0 ** k)


def test_many_rows_of_both():
    x = torch.ones(70_001, 16, dtype=torch.bfloat16, device=DEV)
    w = torch.arange(40, device=DEV).float().unsqueeze(1).expand(40, 16).contiguous()
    got = binding.group_product(x, binding.group_quantize(w, 32))
    assert torch.equal(got, (w[:, 0] * 16).bfloat16().expand(70_001, 40))
    w = torch.ones(300_001, 16, device=DEV)
    w[::2] = 3.0
    got = binding.group_product(x[:2], binding.group_quantize(w, 32))
    assert torch.equal(got, (w[:, 0] * 16).bfloat16().expand(2, 300_001))


def test_offsets_beyond_32_bits():
    """A table of more than 4 GiB of codes, and a product of more than 2^32 elements."""
    N, K = 140_000, 65_536
    codes = torch.zeros(N, K // 2, dtype=torch.uint8, device=DEV)
    scales = torch.zeros(N, K // 128, 2, dtype=torch.bfloat16, device=DEV)
    scales[:, :, 0] = 1.0
    codes[-1] = 0x11
    q = binding.GroupMatrix(codes, scales, K, 128)
    x = torch.ones(2, K, dtype=torch.bfloat16, device=DEV)
    got = binding.group_product(x, q, dtype=torch.float32)
    assert torch.all(got[:, :-1] == 0) and torch.all(got[:, -1] == K)
    assert torch.all(binding.embed(q, torch.tensor([N - 1], device=DEV)) == 1.0)
    del codes, scales, q
    x = torch.ones(70_000, 16, dtype=torch.bfloat16, device=DEV)
    w = torch.ones(65_537, 16, device=DEV)
    w[-1] = 2.0
    got = binding.group_product(x, binding.group_quantize(w, 32))
    assert got[-1, -1].item() == 32.0 and got[-1, -2].item() == 16.0 and got[40_000, 7].item() == 16.0


def test_refusals_on_the_device():
    x, q = torch.zeros(4, 8, device=DEV), binding.group_quantize(torch.ones(5, 8, device=DEV))
    for error, call in [(TypeError, lambda: binding.group_product(x.double(), q)), (ValueError, lambda: binding.group_product(x.cpu(), q)), (ValueError, lambda: binding.group_product(x, q, out=x)),
                        (ValueError, lambda: binding.group_product(x.t(), q)), (binding.SameLdaError, lambda: binding.group_product(x[:, :4], q)), (binding.SameLdaError, lambda: binding.group_product(x, q, float("inf"))),
                        (ValueError, lambda: binding.group_quantize(x, 48)), (ValueError, lambda: binding.group_quantize(x[0])), (TypeError, lambda: binding.group_quantize(x, out=x)), (TypeError, lambda: binding.group_dequantize(q, dtype=torch.float64)),
                        (binding.SameLdaError, lambda: binding.group_quantize(x, out=q)), (TypeError, lambda: binding.group_quantize(x.double())), (TypeError, lambda: binding.group_product(x, q, out=q))]:
        with pytest.raises(error):
            call()


# ---- as they are used together

def test_a_table_is_trained_with_dropout_and_served_from_four_bits():
    """Two steps of gradient descent on a table whose looked-up rows are dropped out, next to the same in torch with the oracle's
    choice; then the table in grouped integers, looked up and multiplied."""
    rng = np.random.default_rng(11)
    V, E, n = 60, 96, 90
    T = numbers_of(rng, V, E, torch.float32).to(DEV)
    ref = T.double().clone()
    t = torch.from_numpy(rng.integers(-1, V, n)).to(DEV)
    target = torch.randn(n, E, device=DEV)
    for step in range(2):
        d = binding.Dropout(0.25, 5, step)
        rows = binding.embed(T, t, drop=d)
        T -= 0.1 * binding.embed_grad(rows - target, t, V, drop=d)
        leaf = ref.clone().requires_grad_()
        known = (t >= 0).unsqueeze(1)
        keep = torch.from_numpy(wr.kept(n, E, 0.25, 5, step)).to(DEV)
        looked = torch.where(known & keep, leaf[t.clamp(min=0)] / 0.75, 0.0)
        ((looked - target.double()) ** 2 / 2).sum().backward()
        ref = (leaf - 0.1 * leaf.grad).detach()
    # per step: some ten roundings of numbers below the largest on the way
    assert (T.double() - ref).abs().max().item() <= 40 * U * max(T.abs().max().item(), target.abs().max().item() * 4)
    q = binding.group_quantize(T, 32)
    read = binding.group_dequantize(q)
    assert torch.equal(binding.embed(q, t.clamp(min=0)), read[t.clamp(min=0)])
    step = q.scales[:, :, 0].float().repeat_interleave(32, dim=1)[:, :E]
    assert ((read - T).abs() <= 0.54 * step + 2.0 ** -23 * T.abs()).all()
    x = torch.randn(4, E, device=DEV)
    A = x.abs().double().view(4, -1, 32).sum(2).cpu().numpy()
    _, s, b = parts(q)
    size = A @ (15.0 * np.abs(s)[:, :3] + np.abs(b[:, :3])).T
    close(binding.group_product(x, q), (x.double() @ read.double().t()).cpu().numpy(), torch.float32, tolerance(x, size, q) + U * size)
