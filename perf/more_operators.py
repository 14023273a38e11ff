"""More word-table operators as cases that can be prepared, run and checked one by one.

Five kinds of pass over a table with one row per word (phi of a topic model, or any embedding table) and the rows made of it:

  dropout   a step's dropout of a matrix and of its gradient, from the seed alone: no mask is kept between the two
  lookup    rows of the table for a list of tokens, with dropout in training, out of grouped four-bit integers in serving
  grad      the table's gradient from the gradient of those rows, the lookup's dropout repeated
  group     a matrix to four-bit integers with a step and a base per group, and back to numbers
  product   rows of numbers, as they are, times every row of a table that is kept in that form

Where `own` is false the operators are computed in elementary torch operations, otherwise by the library's kernels.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128         # rows of the four-bit form are filled up to a multiple of this


def _case(name, op, **more):
    c = {"op": op, **more}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the topic weights of one document on their way into a model (256 topics), and back: latency
        _case("dropout_one_row", "dropout", n=1, E=256, x="float32", p=0.1),
        # the rows of 16 documents of 4096 tokens, a training step in bf16
        _case("dropout_batch", "dropout", n=65_536, E=1024, x="bfloat16", p=0.1),
        # a training batch of 32 documents of 4096 tokens, some padding, the usual scale sqrt(1024)
        _case("lookup_batch", "lookup", n=131_072, V=100_000, E=1024, table="bfloat16", out="bfloat16", tokens="int64", scale=32.0, pad=0.02, p=0.1),
        # a prompt of odd length out of the table that serving keeps in grouped integers, no dropout
        _case("lookup_prompt_grouped", "lookup", n=4_099, V=100_000, E=1024, table="groups of 64", out="bfloat16", tokens="int32", scale=32.0, pad=0.0, p=0.0),
        # a step on one short document, a toy table with the usual fifty topics
        _case("grad_short", "grad", n=77, V=2_000, E=50, grad="float32", out="float32", tokens="int64", scale=1.0, pad=0.0, p=0.5),
        # a step on a million tokens of the news collection: a few words hold a tenth of all tokens each
        _case("grad_news", "grad", n=1_000_003, V=100_000, E=256, grad="float32", out="float32", tokens="int32", scale=1.0, pad=0.0, p=0.1),
        # a small odd matrix of activations
        _case("group_small", "group", R=333, C=250, x="float16", out="float32", group=32),
        # phi of the news collection, as it is laid down for serving
        _case("group_phi", "group", R=100_000, C=256, x="float32", out="float32", group=64),
        # one document's topic weights against every word
        _case("product_one_document", "product", M=1, N=100_000, K=256, x="float32", out="float32", group=64),
        # the next word of one request, wide rows, an odd vocabulary
        _case("product_one_row", "product", M=1, N=50_021, K=4096, x="bfloat16", out="bfloat16", group=128),
        # the words of a few requests that are served together, in binary32
        _case("product_few_rows", "product", M=13, N=50_021, K=4096, x="float32", out="float32", group=64),
        # the scores of all words for a block of a prompt
        _case("product_prompt", "product", M=512, N=50_021, K=1024, x="float16", out="float16", group=128),
    ]


def _log_uniform(rng, lo, hi):
    return int(lo * (hi / lo) ** rng.random())


def draw(rng):
    """One more case: all five operators, sizes over their logarithm, odd ones and round ones."""
    def size(lo, hi):
        n = _log_uniform(rng, lo, hi)
        return max(lo, n // 64 * 64) if rng.random() < 0.5 else n

    op = rng.choice(["dropout", "lookup", "lookup", "grad", "group", "product", "product", "product"])
    floats = ["float32", "bfloat16", "float16"]
    groups = [32, 64, 128]
    p = rng.choice([0.1, 0.15, 0.3, 0.5])
    if op == "dropout":
        E = size(16, 8_192)
        return _case(None, op, n=size(1, 67_000_000 // E), E=E, x=rng.choice(floats), p=p)
    if op in ("lookup", "grad"):
        E = size(16, 4_096)
        V = size(1_000, min(140_000, 140_000_000 // E))
        n = size(1, min(1_000_000, 134_000_000 // E))
        more = dict(n=n, V=V, E=E, tokens=rng.choice(["int32", "int64"]), scale=rng.choice([1.0, round(math.sqrt(E), 3)]), pad=rng.choice([0.0, 0.05]))
        if op == "lookup":
            table = rng.choice(floats + ["groups of %d" % rng.choice(groups)])
            grouped = table not in floats
            return _case(None, op, table=table, out=rng.choice(floats) if grouped else table, p=0.0 if grouped else p, **more)
        grad = rng.choice(floats)
        return _case(None, op, grad=grad, out=rng.choice(["float32", grad]), p=p, **more)
    if op == "group":
        C = size(16, 8_192)
        return _case(None, op, R=size(1, min(140_000, 67_000_000 // C)), C=C, x=rng.choice(floats), out=rng.choice(floats), group=rng.choice(groups))
    K = size(16, 8_192)
    M = size(1, 16) if rng.random() < 0.6 else size(17, 512)
    N = size(100, min(140_000, 50_000_000 // M, 400_000_000 // K, 26_000_000_000 // (M * K)))
    x = rng.choice(floats)
    return _case(None, op, M=M, N=N, K=K, x=x, out=rng.choice(["float32", x]), group=rng.choice(groups))


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


def _group_of(table):
    return int(table.split()[-1])


def prepare(case, seed):
    g = _generator(seed)
    # the program's seed of its random numbers and the number of the step that it is at
    s = {"case": case, "seed": (seed * 0x9E3779B97F4A7C15 + 12345) % 2 ** 63, "step": 1000 + seed}
    if case["op"] == "dropout":
        s["x"] = _normal(g, case["n"], case["E"], case["x"])
        s["dy"] = (1e-3 * _normal(g, case["n"], case["E"], "float32")).to(getattr(torch, case["x"]))
    elif case["op"] == "lookup":
        if case["table"].startswith("groups"):
            s["table"] = _grouped(_normal(g, case["V"], case["E"], "float32"), _group_of(case["table"]))
        else:
            s["table"] = _normal(g, case["V"], case["E"], case["table"])
        s["tokens"] = _tokens(case, g)
    elif case["op"] == "grad":
        s["grad"] = (1e-3 * _normal(g, case["n"], case["E"], "float32")).to(getattr(torch, case["grad"]))
        s["tokens"] = _tokens(case, g)
    elif case["op"] == "group":
        s["x"] = _normal(g, case["R"], case["C"], case["x"]) if case["x"] != "float32" else _weights(g, case["R"], case["C"], case["x"])
    else:
        make = _weights if case["K"] <= 1_024 else _normal
        s["x"] = make(g, case["M"], case["K"], case["x"])
        s["table"] = _grouped(make(g, case["N"], case["K"], "float32"), case["group"])
    return s


# ---- dropout: element (i, j) is kept where its 32 random bits are below (1 - p) 2^32.  The bits of columns 8 c .. 8 c + 7 come from
# two blocks of Philox4x32-10 under the seed, at the counters (c, i, step, 4 2^28) and (c, i, step, 4 2^28 + 2^27): column 8 c + e has
# half e % 2 (the low one first) of word e / 2 of either block, the first block's on top.

def _philox(c0, c1, c2, c3, seed):
    """Ten rounds on tensors of 32-bit counters (int64): a product of two such numbers is right modulo 2^64."""
    low = 0xFFFFFFFF
    k0, k1 = seed & low, seed >> 32 & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _kept(rows, width, p, seed, step):
    c = torch.arange(-(-width // 8), device="cuda").unsqueeze(0)
    i = torch.arange(rows, device="cuda").unsqueeze(1)

    def halves(second):
        c3 = torch.full_like(c, 4 << 28 | second << 27 | step >> 32)
        words = _philox(c.expand(rows, -1), i, torch.full_like(c, step & 0xFFFFFFFF), c3, seed)
        return torch.stack([half for w in words for half in (w & 0xFFFF, w >> 16)], dim=2).view(rows, -1)[:, :width]

    return (halves(0) << 16 | halves(1)) < int(round((1.0 - p) * 2 ** 32))


def _dropped(x, factor, p, seed, step, dtype):
    return torch.where(_kept(*x.shape, p, seed, step), x.float() * torch.tensor(factor, dtype=torch.float32, device="cuda"), 0.0).to(dtype)


# ---- grouped four-bit integers: an element is q s + b with q in 0 .. 15; s and b, in bfloat16, belong to a group of 32, 64 or 128
# elements of a row.  Of a group's least and largest number b is the least rounded down, s = (largest - b) / 15 rounded to binary32
# and on to bfloat16, q the nearest integer to (x - b) / s, ties to even.

def _low(x):
    """x in binary32 rounded down to bfloat16, not below the least finite one."""
    bits = x.view(torch.int32)
    cut = bits & -65536
    cut = torch.where((bits < 0) & (cut != bits), cut + 65536, cut)             # towards minus infinity: away from zero below it
    return cut.view(torch.float32).clamp(min=torch.finfo(torch.bfloat16).min) + 0.0


def _integers(x, group):
    """Codes [rows, groups, group] of x, and its steps and bases [rows, groups] in binary32."""
    rows, cols = x.shape
    n = -(-cols // group)
    d = torch.zeros(rows, n * group, dtype=torch.float32, device=x.device)
    d[:, :cols] = x.float()
    last = torch.arange(n * group, device=x.device).view(n, group) < cols
    d = d.view(rows, n, group)
    least, most = torch.where(last, d, math.inf).amin(dim=2), torch.where(last, d, -math.inf).amax(dim=2)
    base = _low(least)
    fifteen = torch.full((1, 1), 15.0, dtype=torch.float64, device=x.device)            # a tensor: division by a number is a product with its inverse
    step = ((most.double() - base.double()) / fifteen).float().to(torch.bfloat16)
    over = base.double() + 15 * step.double() > torch.finfo(torch.float32).max
    step = torch.where(over, (step.view(torch.int16) - 1).view(torch.bfloat16), step).float()
    q = ((d.double() - base.double().unsqueeze(2)) / step.double().unsqueeze(2)).round().clamp(0, 15)
    q = torch.where(last & (step != 0).unsqueeze(2), q, 0.0).to(torch.int32)
    bad = ~torch.isfinite(least) | ~torch.isfinite(most)
    return torch.where(bad.unsqueeze(2), 0, q), torch.where(bad, math.nan, step), torch.where(bad, math.nan, base)


def _grouped(x, group):
    """x in the form that serving keeps: codes, 64 bytes per 128 elements, and per group its step and base in bfloat16.  Of 128
    elements the word 4 h + j of 32 bits has the eight from 32 j + 8 h on, the even ones in its low half, the odd ones in the high."""
    q, step, base = _integers(x, group)
    rows, blocks = x.shape[0], -(-x.shape[1] // BLOCK)
    codes = torch.zeros(rows, blocks * BLOCK, dtype=torch.int64, device=x.device)
    codes[:, :q.shape[1] * group] = q.view(rows, -1)
    v = codes.view(rows, blocks, 4, 4, 4, 2).permute(0, 1, 3, 2, 4, 5)          # (j, h, t, odd) to (h, j, t, odd)
    place = (torch.arange(4, device=x.device).unsqueeze(1) * 4) + torch.tensor([0, 16], device=x.device)
    words = (v << place).sum(dim=(4, 5))
    words = torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32).contiguous()
    scales = torch.zeros(rows, blocks * BLOCK // group, 2, dtype=torch.bfloat16, device=x.device)
    scales[:, :step.shape[1], 0], scales[:, :step.shape[1], 1] = step.to(torch.bfloat16), base.to(torch.bfloat16)
    return words.view(torch.uint8).view(rows, -1), scales, x.shape[1], group


def _numbers(codes, scales, width, group):
    """The numbers that the grouped form stands for, in binary32."""
    rows = codes.shape[0]
    words = codes.view(torch.int32).view(rows, -1, 4, 4, 1, 1)
    place = (torch.arange(4, device=codes.device, dtype=torch.int32).unsqueeze(1) * 4) + torch.tensor([0, 16], device=codes.device, dtype=torch.int32)
    q = (words >> place & 15).permute(0, 1, 3, 2, 4, 5).reshape(rows, -1, group).float()
    s = scales.float()
    return (q * s[:, :, 0:1] + s[:, :, 1:2]).view(rows, -1)[:, :width]


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        from paper_1409_5402_amd import binding
        drop = binding.Dropout(case["p"], state["seed"], state["step"]) if case.get("p") else None
        if op == "dropout":
            return {"y": binding.dropout(state["x"], drop), "dx": binding.dropout(state["dy"], drop)}
        out = getattr(torch, case["out"])
        if op == "lookup":
            table = binding.GroupMatrix(*state["table"]) if case["table"].startswith("groups") else state["table"]
            return binding.embed(table, state["tokens"], case["scale"], dtype=out, drop=drop)
        if op == "grad":
            return binding.embed_grad(state["grad"], state["tokens"], case["V"], case["scale"], dtype=out, drop=drop)
        if op == "group":
            return binding.group_dequantize(binding.group_quantize(state["x"], case["group"]), dtype=out)
        return binding.group_product(state["x"], binding.GroupMatrix(*state["table"]), dtype=out)
    if op == "dropout":
        at = (1.0 / (1.0 - case["p"]), case["p"], state["seed"], state["step"], state["x"].dtype)
        return {"y": _dropped(state["x"], *at), "dx": _dropped(state["dy"], *at)}
    out = getattr(torch, case["out"])
    if op == "lookup":
        t = state["tokens"].long()
        known = (t >= 0) & (t < case["V"])
        at = torch.where(known, t, torch.zeros_like(t))
        if case["table"].startswith("groups"):
            codes, scales, width, group = state["table"]
            rows = _numbers(codes[at], scales[at], width, group)
        else:
            rows = state["table"][at].float()
        rows = torch.where(known.unsqueeze(1), rows, 0.0)
        if not case["p"]:
            return (rows * case["scale"]).to(out)
        return _dropped(rows, case["scale"] / (1.0 - case["p"]), case["p"], state["seed"], state["step"], out)
    if op == "grad":
        d = torch.where(_kept(case["n"], case["E"], case["p"], state["seed"], state["step"]), state["grad"], 0.0)
        word, order = torch.sort(state["tokens"].long(), stable=True)
        d = d[order].t().double().contiguous()
        before = torch.cat((torch.zeros_like(d[:, :1]), d.cumsum(dim=1)), dim=1)    # running sums, taken at the words' borders
        ends = torch.searchsorted(word, torch.arange(case["V"] + 1, device="cuda"))
        return ((before[:, ends[1:]] - before[:, ends[:-1]]).t() * (case["scale"] / (1.0 - case["p"]))).to(out).contiguous()
    if op == "group":
        q, step, base = _integers(state["x"], case["group"])
        return (q * step.unsqueeze(2) + base.unsqueeze(2)).view(case["R"], -1)[:, :case["C"]].to(out).contiguous()
    return (state["x"].float() @ _numbers(*state["table"]).t()).to(out)


_BYTES = {"float32": 4, "bfloat16": 2, "float16": 2, "int32": 4, "int64": 8}


def _row_bytes(kind, width):
    return width * (0.5 + 4 / _group_of(kind)) if kind.startswith("groups") else width * _BYTES[kind]


def _distinct(V, n):
    """How many different words n tokens with weights 1 / r^1.1 hold on average."""
    r = torch.arange(1, V + 1, dtype=torch.float64).pow(-1.1)
    return float((1 - (1 - r / r.sum()).pow(n)).sum())


def work(case):
    op = case["op"]
    if op == "dropout":
        return {"bytes": 4 * case["n"] * case["E"] * _BYTES[case["x"]], "flops": 2 * case["n"] * case["E"]}
    if op == "lookup":
        n, E = case["n"], case["E"]
        rows = _distinct(case["V"], n * (1 - case["pad"]))
        return {"bytes": rows * _row_bytes(case["table"], E) + n * (_BYTES[case["tokens"]] + E * _BYTES[case["out"]]), "flops": n * E}
    if op == "grad":
        n, E = case["n"], case["E"]
        used = n * (1 - case["pad"])
        return {"bytes": used * E * _BYTES[case["grad"]] + n * _BYTES[case["tokens"]] + case["V"] * E * _BYTES[case["out"]], "flops": used * E}
    if op == "group":
        kind = "groups of %d" % case["group"]
        return {"bytes": case["R"] * (case["C"] * (_BYTES[case["x"]] + _BYTES[case["out"]]) + 2 * _row_bytes(kind, case["C"])), "flops": 4 * case["R"] * case["C"]}
    M, N, K = case["M"], case["N"], case["K"]
    return {"bytes": M * K * _BYTES[case["x"]] + N * _row_bytes("groups of %d" % case["group"], K) + M * N * _BYTES[case["out"]], "flops": 2 * M * N * K}


# ---- the definitions in 64 bits, apart from the plain forms above

def _exact_words(counter, key):
    """Philox4x32-10 with the products' halves made of 16-bit pieces."""
    def product(x, m):
        low = (x & 0xFFFF) * m                                              # below 2^48
        high = (x >> 16) * m + (low >> 16)
        return high >> 16, ((high & 0xFFFF) << 16) | (low & 0xFFFF)

    x = list(counter)
    for r in range(10):
        k = [(key % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32, (key // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32]
        h0, l0 = product(x[0], 0xD2511F53)
        h1, l1 = product(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ k[0], l1, h0 ^ x[3] ^ k[1], l0]
    return x


def _exact_mask(rows, width, p, seed, step):
    """1.0 where an element is kept, by its place alone."""
    mask = torch.zeros(rows, -(-width // 8) * 8, dtype=torch.float64, device="cuda")
    for lo in range(0, rows, 1 << 17):
        n = min(rows - lo, 1 << 17)
        i = torch.arange(lo, lo + n, device="cuda")[:, None].expand(n, mask.shape[1] // 8)
        c = torch.arange(mask.shape[1] // 8, device="cuda")[None, :].expand_as(i)
        same = torch.zeros_like(i)
        top = _exact_words((c, i, same + step % 2 ** 32, same + 0x40000000 + step // 2 ** 32), seed)
        low = _exact_words((c, i, same + step % 2 ** 32, same + 0x48000000 + step // 2 ** 32), seed)
        for e in range(8):
            bits = (top[e // 2] // 65536 ** (e % 2) % 65536) * 65536 + low[e // 2] // 65536 ** (e % 2) % 65536
            mask[lo:lo + n, e::8] = (bits.double() / 2.0 ** 32 < round((1.0 - p) * 2 ** 32) / 2.0 ** 32).double()
    return mask[:, :width]


def _exact_table(codes, scales, width, group):
    """Element by element: of 128 the one at 32 j + 8 h + e is in byte 16 h + 4 j + e / 4 of 0 .. 1 (its low half and its
    high half hold the pairs in turn), the odd ones two bytes on."""
    k = torch.arange(width, device=codes.device)
    at = k % BLOCK
    j, h, e = at // 32, at % 32 // 8, at % 8
    byte = k // BLOCK * 64 + 16 * h + 4 * j + 2 * (e % 2) + e // 4
    q = torch.where(e // 2 % 2 == 1, codes[:, byte] // 16, codes[:, byte] % 16).double()
    return q * scales[:, k // group, 0].double() + scales[:, k // group, 1].double()


def _exact_rounding(x, group):
    """Group by group: the border between q and q + 1 is at base + (q + 1/2) step, and belongs to the even one."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    powers = torch.tensor([2.0 ** k for k in range(-133, 120)], dtype=torch.float64, device=x.device)
    fifteen = torch.tensor([[15.0]], dtype=torch.float64, device=x.device)              # a division by a tensor is rounded once
    for lo in range(0, x.shape[1], group):
        d = x[:, lo:lo + group].double()
        least, most = d.min(dim=1, keepdim=True).values, d.max(dim=1, keepdim=True).values
        unit = powers[(torch.frexp(least.abs()).exponent.long() - 8 + 133).clamp(min=0)]        # of bfloat16's eight digits
        base = torch.floor(least / unit) * unit
        s = ((most - base) / fifteen).to(torch.float32).double()
        unit = powers[(torch.frexp(s).exponent.long() - 8 + 133).clamp(min=0)]
        step = torch.round(s / unit) * unit
        q = torch.zeros_like(d)
        for k in range(15):
            border = base + (k + 0.5) * step
            q += ((d > border) | ((d == border) & (k % 2 == 1))).double()
        out[:, lo:lo + group] = base + q * step
    return out


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "dropout":
        mask = _exact_mask(case["n"], case["E"], case["p"], state["seed"], state["step"]) / (1.0 - case["p"])
        return {"y": state["x"].double() * mask, "dx": state["dy"].double() * mask}
    if op == "lookup":
        out = torch.zeros(case["n"], case["E"], dtype=torch.float64, device="cuda")
        used = torch.nonzero((state["tokens"] >= 0) & (state["tokens"] < case["V"])).squeeze(1)
        words = state["tokens"][used].long()
        if case["table"].startswith("groups"):
            codes, scales, width, group = state["table"]
            out[used] = _exact_table(codes[words], scales[words], width, group) * case["scale"]
        else:
            out[used] = state["table"][words].double() * case["scale"]
        return out if not case["p"] else out * _exact_mask(*out.shape, case["p"], state["seed"], state["step"]) / (1.0 - case["p"])
    if op == "grad":
        out = torch.zeros(case["V"] + 1, case["E"], dtype=torch.float64, device="cuda")
        t = state["tokens"].long()
        t = torch.where((t >= 0) & (t < case["V"]), t, torch.full_like(t, case["V"]))   # a row behind the table for padding
        d = state["grad"].double() * _exact_mask(case["n"], case["E"], case["p"], state["seed"], state["step"])
        return out.index_add_(0, t, d)[:-1] * (case["scale"] / (1.0 - case["p"]))
    if op == "group":
        return _exact_rounding(state["x"], case["group"])
    return state["x"].double() @ _exact_table(*state["table"]).t()
