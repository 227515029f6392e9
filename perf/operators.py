"""Performance cases of the operators around a token table: the lookup with
scaling, its gradient by sorted tokens, the global gradient norm with
clipping, and the table in microscaled 4-bit floating point (quantisation,
lookup, product).

A case is a dict of plain values.  ``op`` names the operator:

  embed    Store.embed of ``n`` ids over a table of ``keys`` rows of ``dim``;
           ``layout`` is the table's: "fp32", "bf16", or "mx4" (MX4.embed)
  grad     Store.embed_grad ("dense") or Store.embed_grad_rows ("rows") of
           ``n`` ids
  clip     ClipPlan.clip of ``tensors`` tensors with ``total`` elements
  quant    mx4_quantize of a [rows, dim] table, and the values it stands for
  product  mx4_product of ``m`` queries with a table of ``rows`` rows

``pad`` is the share of ids that are padding.  A pass is one call (for
``quant`` the quantisation and the restored values); its outputs are what the
call returns.  Where ``own`` is false the same results come from elementary
torch operations.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
PAD = -1
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
BLOCK = 32   # values that share a scale


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # one new token of one sequence: latency alone
        dict(name="embed_1_d512", op="embed", layout="fp32", keys=50_021, dim=512, n=1, out="bf16", pad=0.0),
        # a training batch of 32 padded sequences of 2,048 tokens over a wide table
        dict(name="embed_64k_d2048", op="embed", layout="fp32", keys=65_536, dim=2048, n=65_536, out="bf16", pad=0.05),
        # a serving batch of word vectors out of a 4-bit table, at a width that ends inside a block
        dict(name="embed_213k_d300_mx4", op="embed", layout="mx4", keys=1_000_000, dim=300, n=212_992, out="bf16",
             pad=0.0),
        # the smallest gradient: an odd number of tokens of a large vocabulary, as merged rows
        dict(name="grad_1k_d300_rows", op="grad", form="rows", keys=1_000_000, dim=300, n=1021, gin="fp32", out="fp32",
             pad=0.0),
        # a training batch of 16 padded sequences, the dense gradient of a tied table
        dict(name="grad_32k_d1024_dense", op="grad", form="dense", keys=65_536, dim=1024, n=32_768, gin="bf16",
             out="fp32", pad=0.1),
        # 1M occurrences over 10M rows of 100: most rows met once, the hottest 50,000 times
        dict(name="grad_1m_d100_rows", op="grad", form="rows", keys=10_000_000, dim=100, n=1_048_576, gin="fp32",
             out="fp32", pad=0.0),
        # the dense layers of a small model
        dict(name="clip_14_250k", op="clip", tensors=14, total=250_000, gin="fp32", clips=True),
        # all gradients of a model of half a billion parameters
        dict(name="clip_291_500m", op="clip", tensors=291, total=500_000_000, gin="bf16", clips=True),
        # a batch of queries
        dict(name="quant_1k_d256", op="quant", rows=1024, dim=256, gin="bf16", out="bf16"),
        # a table of 4.6M entities with 128 complex components
        dict(name="quant_4m6_d256", op="quant", rows=4_600_822, dim=256, gin="fp32", out="bf16"),
        # one query against that table: every entity's score
        dict(name="product_1_4m6_d256", op="product", m=1, rows=4_600_822, dim=256, out="fp32"),
        # logits of 2,048 positions over a tied vocabulary
        dict(name="product_2k_131k_d512", op="product", m=2048, rows=131_072, dim=512, out="bf16"),
    ]


def _logu(rng, lo, hi):
    """An integer in [lo, hi], uniform over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _dim(rng, hi):
    """A row width: any up to 512 floats, wider ones a multiple of four."""
    d = _logu(rng, 16, hi)
    return d if d <= 512 else d // 4 * 4


def draw(rng):
    op = rng.choice(["embed", "grad", "clip", "quant", "product"])
    kind = rng.choice(sorted(TYPES))
    out = rng.choice(sorted(TYPES))
    pad = rng.choice([0.0, 0.0, 0.1, 0.5])
    if op == "embed":
        layout = rng.choice(["fp32", "bf16", "mx4"])
        dim = _dim(rng, 512 if layout == "bf16" else 2048)
        return dict(op=op, layout=layout, keys=_logu(rng, 500, min(2_000_000, 200_000_000 // dim)), dim=dim,
                    n=_logu(rng, 1, min(400_000, 100_000_000 // dim)), out=out, pad=pad)
    if op == "grad":
        dim = _dim(rng, 2048)
        return dict(op=op, form=rng.choice(["dense", "rows"]), keys=_logu(rng, 500, min(1_000_000, 67_000_000 // dim)),
                    dim=dim, n=_logu(rng, 1, min(500_000, 67_000_000 // dim)), gin=kind, out=out, pad=pad)
    if op == "clip":
        k = _logu(rng, 1, 400)
        return dict(op=op, tensors=k, total=_logu(rng, 10 * k, 200_000_000), gin=rng.choice(sorted(TYPES) + ["mixed"]),
                    clips=rng.random() < 0.7)
    if op == "quant":
        dim = _logu(rng, 16, 4096)
        return dict(op=op, rows=_logu(rng, 1, 400_000_000 // dim), dim=dim, gin=kind, out=out)
    dim = _logu(rng, 16, 2048)
    m = _logu(rng, 1, 2048)
    rows = _logu(rng, 500, min(4_000_000, 1_000_000_000 // dim, 200_000_000 // m, 130_000_000_000 // (m * dim)))
    return dict(op=op, m=m, rows=rows, dim=dim, out=out)


# ---------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _ids(g, n, keys, pad):
    """Token ids: Zipf ranks (exponent 1) scattered over the table; `pad` of them, at the end of each stretch
    of 2,048, are padding.  The seed says which ids and in which order; how often each of them comes is the
    case's, so that the number of distinct ids is too."""
    at = torch.arange(n, device=DEV)
    real = torch.ones_like(at, dtype=torch.bool)
    if pad > 0.0:
        real = at % 2048 < max(1, int(min(n, 2048) * (1.0 - pad)))
    count = int(real.sum())
    u = torch.rand(count, generator=_gen(n + keys), device=DEV, dtype=torch.float64)
    rank = torch.floor(torch.pow(float(keys), u)).long().clamp_(1, keys) - 1
    first = int(torch.randint(keys, (1,), generator=g, device=DEV))
    ids = torch.full_like(at, PAD)
    ids[real] = (rank[torch.randperm(count, generator=g, device=DEV)] * 2_654_435_761 + first) % keys
    return ids


def _normal(g, shape, std, kind):
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(std)
    return x if kind == torch.float32 else x.to(kind)


def _table(g, rows, dim, kind):
    """Rows of unlike lengths, as trained ones are."""
    x = torch.randn((rows, dim), generator=g, device=DEV, dtype=torch.float32)
    x.mul_(torch.exp(torch.randn((rows, 1), generator=g, device=DEV)).mul_(0.1))
    return x if kind == torch.float32 else x.to(kind)


def _sizes(tensors, total):
    """Sizes of a model's tensors: mostly matrices, with short vectors between them."""
    r = random.Random(tensors * 1_000_003 + total)
    w = [math.exp(r.uniform(-7.0, 0.0)) if i % 3 else 1.0 for i in range(tensors)]
    return [max(1, int(total * x / sum(w))) for x in w]


def _packed(x):
    """(codes, scales) of the microscaled 4-bit form of x [rows, dim], two codes a byte, the first in the low
    half, rows padded to whole blocks of 32."""
    rows, dim = x.shape
    nb = -(-dim // BLOCK)
    x = torch.nn.functional.pad(x.float(), (0, nb * BLOCK - dim)).view(rows, nb, BLOCK)
    e = torch.frexp(x.abs().amax(-1))[1].sub_(3).clamp_(-127, 127)   # floor(log2 max) - 2
    e = torch.where(x.abs().amax(-1) == 0.0, torch.full_like(e, -127), e)
    inv = ((127 - e).clamp_(0, 254) << 23)
    inv = torch.where(e == 127, torch.full_like(inv, 1 << 22), inv).view(torch.float32)   # 2^-e
    v = x * inv[..., None]
    a = v.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = (code + 8 * torch.signbit(v)).to(torch.uint8).view(rows, nb * BLOCK)
    return code[:, 0::2] | (code[:, 1::2] << 4), (e + 127).to(torch.uint8)


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    st = dict(case=case)
    if op == "embed":
        st["scale"] = math.sqrt(case["dim"])
        st["ids"] = _ids(g, case["n"], case["keys"], case["pad"])
        if case["layout"] == "mx4":
            st["codes"], st["scales"] = _packed(_table(g, case["keys"], case["dim"], torch.float32))
        else:
            st["W"] = _table(g, case["keys"], case["dim"], TYPES[case["layout"]])
            st["G"] = torch.ones((case["keys"], case["dim"]), device=DEV)
    elif op == "grad":
        st["scale"] = math.sqrt(case["dim"])
        st["ids"] = _ids(g, case["n"], case["keys"], case["pad"])
        st["dout"] = _normal(g, (case["n"], case["dim"]), 1e-2, TYPES[case["gin"]])
        st["W"] = torch.zeros((case["keys"], case["dim"]), device=DEV)
        st["G"] = torch.ones((case["keys"], case["dim"]), device=DEV)
        if case["form"] == "dense":
            st["grad"] = torch.zeros((case["keys"], case["dim"]), dtype=TYPES[case["out"]], device=DEV)
    elif op == "clip":
        sizes = _sizes(case["tensors"], case["total"])
        mixed = ["fp32", "bf16", "fp16"]
        kinds = [mixed[i % 3] if case["gin"] == "mixed" else case["gin"] for i in range(len(sizes))]
        # one buffer a type for all tensors' gradients, as a training program keeps them, each on 64 elements
        ends = {k: 0 for k in kinds}
        spans = []
        for k, n in zip(kinds, sizes):
            spans.append((k, ends[k], n))
            ends[k] += -(-n // 64) * 64
        flat = {k: _normal(g, (n,), 1e-3, TYPES[k]) for k, n in ends.items()}
        st["flat"] = {k: torch.zeros_like(x) for k, x in flat.items()}
        st["grads"] = [flat[k][at:at + n] for k, at, n in spans]
        st["outs"] = [st["flat"][k][at:at + n] for k, at, n in spans]
        st["max_norm"] = 1e-3 * math.sqrt(sum(sizes)) * (0.37 if case["clips"] else 2.0)
    elif op == "quant":
        st["x"] = _table(g, case["rows"], case["dim"], TYPES[case["gin"]])
    else:
        st["scale"] = 1.0 / math.sqrt(case["dim"])
        st["a"] = _packed(_table(g, case["m"], case["dim"], torch.float32))
        st["b"] = _packed(_table(g, case["rows"], case["dim"], torch.float32))
    if own:
        from paper_2206_00470_amd import MX4, ClipPlan, Store
        if op == "clip":
            st["plan"] = ClipPlan(st["grads"], st["outs"])
        elif op in ("embed", "grad"):
            st["table"] = (MX4(st["codes"], st["scales"], case["dim"]) if "codes" in st else
                           Store(st["W"], st["G"]))
        elif op == "product":
            st["qa"], st["qb"] = MX4(*st["a"], case["dim"]), MX4(*st["b"], case["dim"])
    return st


# ---------------------------------------------------------------- the plain forms
def _values(codes, scales, dim):
    """The values of packed rows, fp32 [rows, dim]."""
    rows, nb = scales.shape
    c = torch.stack((codes & 15, codes >> 4), dim=-1).view(rows, nb, BLOCK)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0],
                        device=codes.device)
    s = scales.int()
    s = torch.where(s == 0, torch.full_like(s, 1 << 22), s << 23).view(torch.float32)
    return (grid[c.int()] * s[..., None]).view(rows, nb * BLOCK)[:, :dim]


def _embed(st):
    case, ids = st["case"], st["ids"]
    at = ids.clamp(min=0)
    rows = (_values(st["codes"][at], st["scales"][at], case["dim"]) if case["layout"] == "mx4" else
            st["W"][at].float())
    rows = torch.where((ids == PAD)[:, None], torch.zeros_like(rows), rows * st["scale"])
    return rows.to(TYPES[case["out"]])


def _grad(st):
    case = st["case"]
    keep = st["ids"] != PAD
    # sums of many terms: in 64 bits
    terms = st["dout"].double() * keep[:, None]
    if case["form"] == "dense":
        dw = torch.zeros((case["keys"], case["dim"]), dtype=torch.float64, device=DEV)
        dw.index_add_(0, st["ids"].clamp(min=0), terms)
        return (dw * st["scale"]).to(TYPES[case["out"]])
    uniq, inv = torch.unique(st["ids"][keep], return_inverse=True)
    dw = torch.zeros((uniq.numel(), case["dim"]), dtype=torch.float64, device=DEV)
    dw.index_add_(0, inv, terms[keep])
    return uniq, (dw * st["scale"]).to(TYPES[case["out"]])


def _clip(st):
    # a long sum: in 64 bits
    norm = torch.stack([x.double().square().sum() for x in st["grads"]]).sum().sqrt()
    coef = torch.where(norm > st["max_norm"], st["max_norm"] / norm, torch.ones_like(norm)).float()
    _ = [o.copy_(x.float() * coef) for x, o in zip(st["grads"], st["outs"])]
    return norm.reshape(1), st["flat"]


def run(st):
    case = st["case"]
    op = case["op"]
    if own:
        from paper_2206_00470_amd import mx4_product, mx4_quantize
        if op == "embed":
            return st["table"].embed(st["ids"], scale=st["scale"], dtype=TYPES[case["out"]], pad=PAD)
        if op == "grad" and case["form"] == "dense":
            return st["table"].embed_grad(st["ids"], st["dout"], scale=st["scale"], pad=PAD, out=st["grad"])
        if op == "grad":
            return st["table"].embed_grad_rows(st["ids"], st["dout"], scale=st["scale"], pad=PAD,
                                               dtype=TYPES[case["out"]])
        if op == "clip":
            return st["plan"].clip(st["max_norm"]), st["flat"]
        if op == "quant":
            return mx4_quantize(st["x"]).dequantize(TYPES[case["out"]])
        return mx4_product(st["qa"], st["qb"], scale=st["scale"], dtype=TYPES[case["out"]])
    if op == "embed":
        return _embed(st)
    if op == "grad":
        return _grad(st)
    if op == "clip":
        return _clip(st)
    if op == "quant":
        codes, scales = _packed(st["x"])
        return _values(codes, scales, case["dim"]).to(TYPES[case["out"]])
    a, b = _values(*st["a"], case["dim"]), _values(*st["b"], case["dim"])
    return (torch.matmul(a, b.t()) * st["scale"]).to(TYPES[case["out"]])


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    op, d = case["op"], case.get("dim", 0)
    mx4 = 17 * -(-d // BLOCK)   # bytes of a packed row
    if op == "embed":
        row = mx4 if case["layout"] == "mx4" else BYTES[case["layout"]] * d
        return dict(bytes=8 * case["n"] + min(case["n"], case["keys"]) * row + case["n"] * d * BYTES[case["out"]],
                    flops=case["n"] * d)
    if op == "grad":
        rows = case["keys"] if case["form"] == "dense" else min(case["n"], case["keys"])
        return dict(bytes=case["n"] * (8 + d * BYTES[case["gin"]]) + rows * d * BYTES[case["out"]],
                    flops=case["n"] * d)
    if op == "clip":
        b = 8 / 3 if case["gin"] == "mixed" else BYTES[case["gin"]]
        return dict(bytes=2 * b * case["total"], flops=3 * case["total"])
    if op == "quant":
        return dict(bytes=case["rows"] * (d * (BYTES[case["gin"]] + BYTES[case["out"]]) + mx4), flops=3 * case["rows"] * d)
    return dict(bytes=(case["m"] + case["rows"]) * mx4 + case["m"] * case["rows"] * BYTES[case["out"]],
                flops=2 * case["m"] * case["rows"] * d)


# ---------------------------------------------------------------- 64 bits
_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _pow2(e):
    """2^e in 64 bits, from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_values(codes, scales, dim):
    """Packed rows by the format's definition: (-1)^s m 2^(scale - 127), in 64 bits."""
    rows = codes.shape[0]
    mag = torch.tensor(_E2M1, dtype=torch.float64, device=codes.device)
    x = torch.empty((rows, 2 * codes.shape[1]), dtype=torch.float64, device=codes.device)
    for half in (0, 1):
        c = (codes >> (4 * half)).long() & 15
        x[:, half::2] = mag[c & 7] * (1 - 2 * (c >> 3))
    x *= _pow2(scales.long() - 127).repeat_interleave(BLOCK, dim=1)
    return x[:, :dim]


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        out = torch.zeros((case["n"], case["dim"]), dtype=torch.float64, device=DEV)
        real = (st["ids"] != PAD).nonzero()[:, 0]
        at = st["ids"][real]
        rows = (_exact_values(st["codes"][at], st["scales"][at], case["dim"]) if case["layout"] == "mx4" else
                st["W"][at].double())
        out[real] = rows * st["scale"]
        return out
    if op == "grad":
        # sorted tokens, each token's sum a difference of running sums over its stretch
        real = (st["ids"] != PAD).nonzero()[:, 0]
        ids, order = torch.sort(st["ids"][real], stable=True)
        uniq, count = torch.unique_consecutive(ids, return_counts=True)
        last = torch.cumsum(count, 0)
        dw = torch.zeros((uniq.numel(), case["dim"]), dtype=torch.float64, device=DEV)
        wide = max(1, 200_000_000 // max(1, ids.numel()))
        for c in range(0, case["dim"], wide):
            run_sum = torch.cumsum(st["dout"][real[order], c:c + wide].double(), 0)
            run_sum = torch.nn.functional.pad(run_sum, (0, 0, 1, 0))
            dw[:, c:c + wide] = (run_sum[last] - run_sum[last - count]) * st["scale"]
        if case["form"] == "rows":
            return uniq, dw
        full = torch.zeros((case["keys"], case["dim"]), dtype=torch.float64, device=DEV)
        full[uniq] = dw
        return full
    if op == "clip":
        total = math.fsum(float(torch.dot(x.double(), x.double())) for x in st["grads"])
        norm = math.sqrt(total)
        coef = min(1.0, st["max_norm"] / norm)
        flat = {k: torch.zeros(x.numel(), dtype=torch.float64, device=DEV) for k, x in st["flat"].items()}
        size = {torch.float32: ("fp32", 4), torch.bfloat16: ("bf16", 2), torch.float16: ("fp16", 2)}
        for x, o in zip(st["grads"], st["outs"]):
            k, b = size[o.dtype]
            at = (o.data_ptr() - st["flat"][k].data_ptr()) // b
            flat[k][at:at + o.numel()] = x.double() * coef
        return np.array([norm]), flat
    if op == "quant":
        out = torch.empty((case["rows"], case["dim"]), dtype=torch.float64, device=DEV)
        for r in range(0, case["rows"], 1 << 20):
            x = st["x"][r:r + (1 << 20)].double()
            for c in range(0, case["dim"], BLOCK):
                v = x[:, c:c + BLOCK]
                top = v.abs().amax(1, keepdim=True)
                e = torch.floor(torch.log2(top)).clamp(-1000.0, 1000.0)
                e = e + (_pow2(e + 1) <= top).double() - (_pow2(e) > top).double()   # the logarithm is rounded
                unit = _pow2((e - 2.0).clamp(-127.0, 127.0))
                a = v / unit
                step = torch.where(a.abs() < 2.0, 0.5, torch.where(a.abs() < 4.0, 1.0, 2.0))
                out[r:r + (1 << 20), c:c + BLOCK] = (torch.round(a / step) * step).clamp(-6.0, 6.0) * unit
        return out
    a, b = _exact_values(*st["a"], case["dim"]), _exact_values(*st["b"], case["dim"])
    return torch.matmul(a, b.t()) * st["scale"]
