"""The word-table operators as cases that can be prepared, run and checked one by one.

Four kinds of pass over a table with one row per word (phi of a topic model, or any embedding table):

  embed     rows of the table for a list of tokens, times a scale
  grad      the table's gradient from the gradient of those rows: sums over the tokens of each word
  quantize  a matrix to microscaled four-bit floating point (blocks of 32 with a power of two) and back to numbers
  product   rows of numbers, quantised in the call, times every row of a table that is kept in four bits

Where `own` is false the operators are computed in elementary torch operations, otherwise by the library's kernels.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 32          # elements that share a scale
GROUP = 128         # rows of the four-bit form are filled up with zero blocks to a multiple of this


def _case(name, op, **more):
    c = {"op": op, **more}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one token on its way into a model whose table is the news collection's phi (100,000 words, 256 topics): latency
        _case("embed_one_token", "embed", n=1, V=100_000, E=256, table="float32", out="float32", tokens="int64", scale=1.0, pad=0.0),
        # a training batch of 64 documents of 4096 tokens, table rows of 1024, the usual scale sqrt(1024), some padding
        _case("embed_batch", "embed", n=262_144, V=100_000, E=1024, table="bfloat16", out="bfloat16", tokens="int64", scale=32.0, pad=0.02),
        # a prompt of odd length out of the table that serving keeps in four bits
        _case("embed_prompt_four_bits", "embed", n=4_099, V=100_000, E=1024, table="four bits", out="bfloat16", tokens="int32", scale=32.0, pad=0.0),
        # a step on one short document, a toy table with the usual fifty topics
        _case("grad_short", "grad", n=77, V=2_000, E=50, grad="float32", out="float32", tokens="int64", scale=1.0, pad=0.0),
        # a step on a million tokens of the news collection: a few words hold a tenth of all tokens each
        _case("grad_news", "grad", n=1_000_003, V=100_000, E=256, grad="float32", out="float32", tokens="int32", scale=1.0, pad=0.0),
        # a bf16 training step with padded documents, the scale of the lookup
        _case("grad_batch", "grad", n=65_537, V=32_003, E=1024, grad="bfloat16", out="bfloat16", tokens="int64", scale=32.0, pad=0.05),
        # a small odd matrix of activations
        _case("quantize_small", "quantize", R=333, C=250, x="float16", out="float32"),
        # phi of the news collection, as it is laid down for serving
        _case("quantize_phi", "quantize", R=100_000, C=256, x="float32", out="float32"),
        # one document's topic weights against every word
        _case("product_one_document", "product", M=1, N=100_000, K=256, x="float32", out="float32"),
        # the words of a few requests that are served together, wider rows, an odd vocabulary
        _case("product_few_rows", "product", M=13, N=50_021, K=4096, x="bfloat16", out="bfloat16"),
        # predictive weights of a block of documents over the whole vocabulary: the output is what counts
        _case("product_documents", "product", M=2_048, N=100_000, K=256, x="float32", out="float32"),
        # a large square product
        _case("product_large", "product", M=8_192, N=8_192, K=8_192, x="bfloat16", out="bfloat16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(lo * (hi / lo) ** rng.random())


def draw(rng):
    """One more case: all four operators, sizes over their logarithm, odd ones and round ones."""
    def size(lo, hi):
        n = _log_uniform(rng, lo, hi)
        return max(lo, n // 64 * 64) if rng.random() < 0.5 else n

    op = rng.choice(["embed", "embed", "grad", "grad", "quantize", "product", "product", "product"])
    floats = ["float32", "bfloat16", "float16"]
    if op in ("embed", "grad"):
        E = size(16, 4_096)
        V = size(1_000, min(140_000, 140_000_000 // E))
        n = size(1, min(1_000_000, 268_000_000 // E))
        more = dict(n=n, V=V, E=E, tokens=rng.choice(["int32", "int64"]), scale=rng.choice([1.0, round(math.sqrt(E), 3)]), pad=rng.choice([0.0, 0.05]))
        if op == "embed":
            table = rng.choice(floats + ["four bits"])
            return _case(None, op, table=table, out=rng.choice(floats) if table == "four bits" else table, **more)
        grad = rng.choice(floats)
        return _case(None, op, grad=grad, out=rng.choice(["float32", grad]), **more)
    if op == "quantize":
        C = size(16, 8_192)
        return _case(None, op, R=size(1, min(140_000, 67_000_000 // C)), C=C, x=rng.choice(floats), out=rng.choice(floats))
    K = size(16, 8_192)
    M = size(1, 16) if rng.random() < 0.4 else size(17, 4_096)
    N = size(100, min(140_000, 200_000_000 // M, 500_000_000 // K, 540_000_000_000 // (M * K)))
    return _case(None, op, M=M, N=N, K=K, x=rng.choice(floats), out=rng.choice(floats))


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _tokens(case, g):
    """Word ids with the skew of natural text (the r-th word has weight 1 / r^1.1); padding is -1."""
    up_to = torch.arange(1, case["V"] + 1, dtype=torch.float64).pow(-1.1).cumsum(dim=0)
    u = torch.rand(case["n"], device="cuda", generator=g, dtype=torch.float64) * float(up_to[-1])
    t = torch.searchsorted(up_to.cuda(), u).clamp(max=case["V"] - 1)
    if case["pad"]:
        t = torch.where(torch.rand(case["n"], device="cuda", generator=g) < case["pad"], torch.full_like(t, -1), t)
    return t.to(getattr(torch, case["tokens"]))


def _normal(g, rows, cols, dtype):
    """Activations: normal numbers, a few columns much larger than the rest."""
    x = torch.randn(rows, cols, device="cuda", generator=g)
    x *= torch.exp(0.5 * torch.randn(cols, device="cuda", generator=g))
    return x.to(getattr(torch, dtype))


def _weights(g, rows, cols, dtype):
    """Topic weights: positive, a few large entries in each row."""
    x = torch.exp(1.5 * torch.randn(rows, cols, device="cuda", generator=g))
    return (x / cols).to(getattr(torch, dtype))


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    if case["op"] == "embed":
        if case["table"] == "four bits":
            s["table"] = _four_bits(_normal(g, case["V"], case["E"], "float32"))
        else:
            s["table"] = _normal(g, case["V"], case["E"], case["table"])
        s["tokens"] = _tokens(case, g)
    elif case["op"] == "grad":
        s["grad"] = (1e-3 * _normal(g, case["n"], case["E"], "float32")).to(getattr(torch, case["grad"]))
        s["tokens"] = _tokens(case, g)
    elif case["op"] == "quantize":
        s["x"] = _normal(g, case["R"], case["C"], case["x"]) if case["x"] != "float32" else _weights(g, case["R"], case["C"], case["x"])
    else:
        make = _weights if case["K"] <= 1_024 else _normal
        s["x"] = make(g, case["M"], case["K"], case["x"])
        s["table"] = _four_bits(make(g, case["N"], case["K"], "float32"))
    return s


def _steps(x):
    """Blocks of x in binary32 [rows, blocks, 32] (the last one filled up with zeros) and the exponent of each block's
    scale: the largest power of two in the block over the 4 of the largest four-bit number 6 = 1.5 * 4; 128 where a block
    holds an infinity or a NaN."""
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    b = torch.zeros(rows, blocks * BLOCK, device=x.device, dtype=torch.float32)
    b[:, :cols] = x.float()
    b = b.view(rows, blocks, BLOCK)
    top = b.abs().amax(dim=2)
    e = torch.frexp(top).exponent - 3                   # top = m * 2^exponent with m in [1/2, 1)
    e = torch.where(top == 0, torch.full_like(e, -127), e).clamp(-127, 127)
    return b, torch.where(torch.isfinite(top), e, torch.full_like(e, 128))


def _power(e):
    """2^e in binary32 for e in -127 .. 127 (the lowest one is subnormal), NaN for 128."""
    bits = torch.where(e == -127, torch.full_like(e, 0x00400000), (e + 127) << 23)
    return torch.where(e == 128, torch.full_like(e, 0x7FC00000), bits).to(torch.int32).view(torch.float32)


def _codes(b, e):
    """Sign and nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 (ties to the even code) of every number over its block's scale."""
    t = b.abs() * _power(torch.where(e == 128, torch.zeros_like(e), -e)).unsqueeze(2)
    near = torch.where(t < 2, torch.round(2 * t), torch.where(t < 4, torch.round(t) + 2, (torch.round(t / 2) + 4).clamp(max=7)))
    code = torch.where(torch.isfinite(t), near, torch.zeros_like(t)).to(torch.uint8) | (torch.signbit(b).to(torch.uint8) << 3)
    return torch.where((e == 128).unsqueeze(2), torch.zeros_like(code), code)


def _four_bits(x):
    """x in the form that serving keeps: codes, two to a byte with the even element in the low half, and a byte 127 + e per
    block; rows filled up with zero blocks to a multiple of 128 elements."""
    b, e = _steps(x)
    rows, blocks = e.shape
    code = _codes(b, e)
    room = -(-blocks * BLOCK // GROUP) * GROUP
    codes = torch.zeros(rows, room // 2, device=x.device, dtype=torch.uint8)
    codes[:, :blocks * BLOCK // 2] = (code[:, :, 0::2] | (code[:, :, 1::2] << 4)).view(rows, -1)
    scales = torch.zeros(rows, room // BLOCK, device=x.device, dtype=torch.uint8)
    scales[:, :blocks] = (e + 127).to(torch.uint8)
    return codes, scales, x.shape[1]


def _numbers(codes, scales, width):
    """The numbers that the four-bit form stands for, in binary32."""
    code = torch.stack((codes & 15, codes >> 4), dim=2).view(codes.shape[0], -1).to(torch.int32)
    m = code & 7
    size = torch.where(m < 4, m * 0.5, torch.where(m < 6, m - 2.0, 2.0 * m - 8.0))
    value = torch.where(code > 7, -size, size).view(codes.shape[0], -1, BLOCK)
    return (value * _power(scales.to(torch.int32) - 127).unsqueeze(2)).view(codes.shape[0], -1)[:, :width]


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        from paper_1409_5402_amd import binding
        out = getattr(torch, case["out"])
        if op == "embed":
            table = state["table"] if case["table"] != "four bits" else binding.MicroMatrix(*state["table"])
            return binding.embed(table, state["tokens"], case["scale"], dtype=out)
        if op == "grad":
            return binding.embed_grad(state["grad"], state["tokens"], case["V"], case["scale"], dtype=out)
        if op == "quantize":
            return binding.micro_dequantize(binding.micro_quantize(state["x"]), dtype=out)
        return binding.micro_product(state["x"], binding.MicroMatrix(*state["table"]), dtype=out)
    out = getattr(torch, case["out"])
    if op == "embed":
        t = state["tokens"].long()
        known = (t >= 0) & (t < case["V"])
        at = torch.where(known, t, torch.zeros_like(t))
        if case["table"] == "four bits":
            codes, scales, width = state["table"]
            rows = _numbers(codes[at], scales[at], width)
        else:
            rows = state["table"][at].float()
        return torch.where(known.unsqueeze(1), rows * case["scale"], torch.zeros_like(rows)).to(out)
    if op == "grad":
        word, order = torch.sort(state["tokens"].long(), stable=True)
        d = state["grad"][order].t().double().contiguous()
        before = torch.cat((torch.zeros_like(d[:, :1]), d.cumsum(dim=1)), dim=1)    # running sums, taken at the words' borders
        ends = torch.searchsorted(word, torch.arange(case["V"] + 1, device="cuda"))
        return ((before[:, ends[1:]] - before[:, ends[:-1]]).t() * case["scale"]).to(out).contiguous()
    if op == "quantize":
        b, e = _steps(state["x"])
        code = _codes(b, e).to(torch.int32)
        m = code & 7
        size = torch.where(m < 4, m * 0.5, torch.where(m < 6, m - 2.0, 2.0 * m - 8.0))
        value = torch.where(code > 7, -size, size) * _power(e).unsqueeze(2)
        return value.view(case["R"], -1)[:, :case["C"]].to(out)
    x = _numbers(*_four_bits(state["x"]))
    return (x @ _numbers(*state["table"]).t()).to(out)


_BYTES = {"float32": 4, "bfloat16": 2, "float16": 2, "int32": 4, "int64": 8}


def _row_bytes(case, kind, width):
    return width * 17 / 32 if kind == "four bits" else width * _BYTES[kind]


def _distinct(V, n):
    """How many different words n tokens with weights 1 / r^1.1 hold on average."""
    r = torch.arange(1, V + 1, dtype=torch.float64).pow(-1.1)
    return float((1 - (1 - r / r.sum()).pow(n)).sum())


def work(case):
    op = case["op"]
    if op == "embed":
        n, E = case["n"], case["E"]
        rows = _distinct(case["V"], n * (1 - case["pad"]))
        return {"bytes": rows * _row_bytes(case, case["table"], E) + n * (_BYTES[case["tokens"]] + E * _BYTES[case["out"]]), "flops": n * E}
    if op == "grad":
        n, E = case["n"], case["E"]
        used = n * (1 - case["pad"])
        return {"bytes": used * E * _BYTES[case["grad"]] + n * _BYTES[case["tokens"]] + case["V"] * E * _BYTES[case["out"]], "flops": used * E}
    if op == "quantize":
        return {"bytes": case["R"] * case["C"] * (_BYTES[case["x"]] + 2 * 17 / 32 + _BYTES[case["out"]]), "flops": 3 * case["R"] * case["C"]}
    M, N, K = case["M"], case["N"], case["K"]
    return {"bytes": M * K * _BYTES[case["x"]] + N * K * 17 / 32 + M * N * _BYTES[case["out"]], "flops": 2 * M * N * K}


_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _exact_rounding(x):
    """Microscaled values of x from the definition, in 64 bits: per block the largest power of two that is not above its
    largest magnitude, over 4; per number the nearest of the sizes by the middles between them, the even code on a middle."""
    rows, cols = x.shape
    whole = torch.nn.functional.pad(x.double(), (0, -cols % BLOCK)).unflatten(1, (-1, BLOCK))
    powers = torch.tensor([2.0 ** k for k in range(-160, 129)], dtype=torch.float64, device=x.device)
    top = whole.abs().amax(dim=2, keepdim=True)
    e = (torch.bucketize(top, powers, right=True) - 1 - 160).clamp(min=-125) - 2
    scale = powers[e + 160]
    size = torch.tensor(_E2M1, dtype=torch.float64, device=x.device)
    middle = (size[1:] + size[:-1]) / 2
    t = whole.abs() / scale
    low = torch.bucketize(t, middle)
    code = torch.where(low % 2 == 0, low, torch.bucketize(t, middle, right=True))
    return torch.copysign(size[code] * scale, whole).flatten(1)[:, :cols]


def _exact_table(codes, scales, width):
    signed = torch.tensor(_E2M1 + [-v for v in _E2M1], dtype=torch.float64, device=codes.device)
    powers = torch.tensor([2.0 ** (s - 127) for s in range(255)] + [math.nan], dtype=torch.float64, device=codes.device)
    value = torch.empty(codes.shape[0], 2 * codes.shape[1], dtype=torch.float64, device=codes.device)
    value[:, 0::2] = signed[(codes % 16).long()]
    value[:, 1::2] = signed[(codes // 16).long()]
    return (value * powers[scales.long()].repeat_interleave(BLOCK, dim=1))[:, :width]


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "embed":
        codes = case["table"] == "four bits"
        out = torch.zeros(case["n"], case["E"], dtype=torch.float64, device="cuda")
        used = torch.nonzero((state["tokens"] >= 0) & (state["tokens"] < case["V"])).squeeze(1)
        words = state["tokens"][used].long()
        if codes:
            c, s, width = state["table"]
            out[used] = _exact_table(c[words], s[words], width) * case["scale"]
        else:
            out[used] = state["table"][words].double() * case["scale"]
        return out
    if case["op"] == "grad":
        out = torch.zeros(case["V"] + 1, case["E"], dtype=torch.float64, device="cuda")
        t = state["tokens"].long()
        t = torch.where((t >= 0) & (t < case["V"]), t, torch.full_like(t, case["V"]))   # a row behind the table for padding
        return out.index_add_(0, t, state["grad"].double())[:-1] * case["scale"]
    if case["op"] == "quantize":
        return _exact_rounding(state["x"])
    return _exact_rounding(state["x"]) @ _exact_table(*state["table"]).t()
