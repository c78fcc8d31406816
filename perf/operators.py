"""The performance cases of the operators for language models: what a trainer or a server has them do, one pass each.

A case's "op" says what one pass runs:

  quantize   a matrix to 8-bit floating point with a scale for each block of 128, its transpose too where "both" is set
  product    the product of two such matrices, as a forward pass or a decoding step makes it
  step       the training step of one linear layer in 8 bits: its weight, input and output gradient are quantized, and
             three products give the output, the gradient of the input and that of the weight
  count      tokens of prompts, or one of each running sequence, entered into the sequences' sets and counts
  adjust     penalties for repeated tokens, biases and a grammar's masks on a batch's logits

Matrices hold normal values, some rows and columns of which are larger; tokens are Zipf distributed.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
BLOCK = 128
TOP = 448.0  # the largest e4m3 value
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # activations of a decoding batch before a layer's product: latency
        dict(name="quantize_32x2048", op="quantize", rows=32, dim=2048, stride=2048, type="bf16", kind="row", scale="e8m0", both=False),
        # activations of a training batch, in both directions for the forward and the weight's gradient
        dict(name="quantize_8192x4096_both", op="quantize", rows=8192, dim=4096, stride=4096, type="bf16", kind="row", scale="e8m0", both=True),
        # a whole embedding table (1 M rows of 128) in tiles with ordinary scales, from its fp32 rows
        dict(name="quantize_table_1m", op="quantize", rows=1_000_000, dim=128, stride=128, type="f32", kind="tile", scale="f32", both=False),
        # the logits of one sequence: the output matrix is read once
        dict(name="product_1x32000x4096", op="product", m=1, n=32000, k=4096, a="row", b="tile", scale="e8m0", out="f32", add=False),
        # the logits of a decoding batch, odd vocabulary, ordinary scales
        dict(name="product_48x50257x2048", op="product", m=48, n=50257, k=2048, a="row", b="tile", scale="f32", out="bf16", add=False),
        # odd sizes that end inside tiles and blocks, onto a residual
        dict(name="product_1000x1111x1100", op="product", m=1000, n=1111, k=1100, a="row", b="row", scale="e8m0", out="f16", add=True),
        # a large layer's forward pass
        dict(name="product_16384x8192x8192", op="product", m=16384, n=8192, k=8192, a="row", b="tile", scale="e8m0", out="bf16", add=False),
        # a layer's training step, gradients of the weight added up in fp32
        dict(name="step_8192x4096x4096", op="step", m=8192, n=4096, k=4096, type="bf16", scale="e8m0"),
        # prompts of a batch enter emptied slots, ragged lengths
        dict(name="count_prompts_64x8192", op="count", n=64, slots=64, vocab=131072, longest=8192, index="i64", restart=True),
        # one new token of each running sequence
        dict(name="count_step_256", op="count", n=256, slots=300, vocab=131072, longest=1, index="i64", restart=False),
        # the logits of a few sequences, odd vocabulary
        dict(name="adjust_8x50257", op="adjust", n=8, slots=16, vocab=50257, type="f32", seen=600, penalties=True, bias=40, masks=4),
        # the logits of a large batch with every adjustment
        dict(name="adjust_512x131072", op="adjust", n=512, slots=512, vocab=131072, type="bf16", seen=3000, penalties=True, bias=100, masks=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size of the range: as it comes (odd as often as not), or the multiple of 128 next to it."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.6 else min(hi, max(lo, (n + 64) // BLOCK * BLOCK or BLOCK))


def draw(rng):
    op = rng.choice(["quantize", "product", "product", "step", "count", "adjust"])
    if op == "quantize":
        dim = _size(rng, 32, 16384)
        rows = _size(rng, 1, max(1, min(1_000_000, (1 << 26) // dim)))
        return dict(op=op, rows=rows, dim=dim, stride=dim + rng.choice([0, 0, 8, 13]), type=rng.choice(["f32", "bf16", "f16"]),
                    kind=rng.choice(["row", "tile"]), scale=rng.choice(["e8m0", "f32"]), both=rng.random() < 0.5)
    if op == "product":
        k = _size(rng, 64, 16384)
        n = _size(rng, 16, 65536)
        m = _size(rng, 1, max(1, min(16384, (1 << 39) // (n * k))))
        return dict(op=op, m=m, n=n, k=k, a=rng.choice(["row", "row", "tile"]), b=rng.choice(["row", "tile", "tile"]),
                    scale=rng.choice(["e8m0", "e8m0", "f32"]), out=rng.choice(["bf16", "bf16", "f16", "f32"]), add=rng.random() < 0.3)
    if op == "step":
        return dict(op=op, m=_size(rng, 64, 8192), n=_size(rng, 128, 4096), k=_size(rng, 128, 4096), type=rng.choice(["bf16", "f16", "f32"]),
                    scale=rng.choice(["e8m0", "f32"]))
    vocab = _size(rng, 300, 262144)
    index = rng.choice(["i32", "i64"])
    if op == "count":
        n = _log_int(rng, 1, min(512, (1 << 25) // vocab))
        restart = rng.random() < 0.5
        return dict(op=op, n=n, slots=n + rng.randrange(0, 40), vocab=vocab, longest=_log_int(rng, 2, 16384) if restart else 1, index=index,
                    restart=restart)
    n = _log_int(rng, 1, min(512, (1 << 26) // vocab))
    return dict(op=op, n=n, slots=n + rng.randrange(0, 40), vocab=vocab, type=rng.choice(["f32", "bf16", "f16"]), seen=_log_int(rng, 1, 8000),
                penalties=rng.random() < 0.8, bias=rng.choice([0, 0, 7, 300]), masks=rng.choice([0, 1, n]))


# ---- inputs -------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _matrix(g, rows, dim, stride, dtype, sigma=1.0):
    """Normal values; one row in sixteen and one column in fifty is ten times larger, a hundredth of the rows is zero."""
    x = torch.zeros(rows, stride, dtype=torch.float32, device=DEV)
    x.normal_(0.0, sigma, generator=g)
    r = torch.rand(rows, generator=g, device=DEV)
    x *= torch.where(r < 1 / 16, 10.0, torch.where(r > 0.99, 0.0, 1.0)).unsqueeze(1)
    x *= torch.where(torch.rand(stride, generator=g, device=DEV) < 0.02, 10.0, 1.0)
    return x.to(dtype)[:, :dim]


def _tokens(g, n, vocab):
    """Zipf(1) distributed tokens in a scattered order of the vocabulary."""
    u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
    rank = torch.exp(u * math.log(vocab + 1)).to(torch.int64) - 1
    return (rank.clamp(0, vocab - 1) * 7919 + 12345) % vocab


def _words(vocab):
    return (vocab + 31) // 32


def _operand(g, rows, k, kind, scale):
    """A quantized matrix as the program holds it: random codes of a normal distribution and scales around 2^-6."""
    blocks, rounded = -(-k // BLOCK), -(-rows // BLOCK) * BLOCK
    codes = torch.zeros(rows, blocks * BLOCK, dtype=torch.uint8, device=DEV)
    for at in range(0, rows, 8192):
        part = codes[at:at + 8192, :k]
        v = torch.empty(part.shape, dtype=torch.float32, device=DEV).normal_(0.0, 120.0, generator=g).clamp_(-TOP, TOP)
        part.copy_(v.to(torch.float8_e4m3fn).view(torch.uint8))
    shape = (blocks, rounded if kind == "row" else rounded // BLOCK)
    s = torch.empty(shape, dtype=torch.float32, device=DEV).uniform_(-8.0, -4.0, generator=g)
    s = s.round().to(torch.int32).add_(127).to(torch.uint8) if scale == "e8m0" else torch.exp2(s)
    return codes, s


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    s = {"case": c}
    if c["op"] == "quantize":
        s["x"] = _matrix(g, c["rows"], c["dim"], c["stride"], TYPES[c["type"]])
        s["out"] = _room(c["rows"], c["dim"], c["kind"], c["scale"])
        s["out_t"] = _room(c["dim"], c["rows"], c["kind"], c["scale"]) if c["both"] else None
    elif c["op"] == "product":
        s["a"] = _operand(g, c["m"], c["k"], c["a"], c["scale"])
        s["b"] = _operand(g, c["n"], c["k"], c["b"], c["scale"])
        s["out"] = torch.empty(c["m"], c["n"], dtype=TYPES[c["out"]], device=DEV)
        # as large as the sums, so that neither hides the other's rounding
        s["residual"] = s["out"].normal_(0.0, math.sqrt(c["k"]), generator=g).clone() if c["add"] else None
    elif c["op"] == "step":
        t = TYPES[c["type"]]
        s["w"] = _matrix(g, c["n"], c["k"], c["k"], torch.float32, 0.02)
        s["x"] = _matrix(g, c["m"], c["k"], c["k"], t)
        s["dy"] = _matrix(g, c["m"], c["n"], c["n"], t, 0.01)
        s["dw"] = torch.empty(c["n"], c["k"], dtype=torch.float32, device=DEV)
        s["y"] = torch.empty(c["m"], c["n"], dtype=t, device=DEV)
        s["dx"] = torch.empty(c["m"], c["k"], dtype=t, device=DEV)
    elif c["op"] == "count":
        n, vocab = c["n"], c["vocab"]
        s["slots"] = torch.randperm(c["slots"], generator=g, device=DEV)[:n].to(torch.int32)
        s["offsets"] = None
        total = n
        if c["longest"] > 1:
            lengths = torch.exp(torch.rand(n, generator=g, device=DEV) * math.log(c["longest"] + 1)).to(torch.int64) - 1
            lengths[0] = c["longest"]
            s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), lengths.cumsum(0)])
            total = int(s["offsets"][-1])
        s["tokens"] = _tokens(g, total, vocab).to(torch.int32 if c["index"] == "i32" else torch.int64)
        s["seen"] = torch.zeros(c["slots"], _words(vocab), dtype=torch.int32, device=DEV)
        s["counts"] = torch.zeros(c["slots"], vocab, dtype=torch.int32, device=DEV)
    else:
        n, vocab = c["n"], c["vocab"]
        s["logits"] = torch.empty(n, vocab, dtype=torch.float32, device=DEV).normal_(0.0, 4.0, generator=g).to(TYPES[c["type"]])
        s["out"] = torch.empty_like(s["logits"])
        s["slots"] = torch.randperm(c["slots"], generator=g, device=DEV)[:n].to(torch.int32)
        s["seen"] = s["counts"] = s["repetition"] = s["frequency"] = s["presence"] = None
        if c["penalties"]:
            tokens = _tokens(g, c["slots"] * c["seen"], vocab).reshape(c["slots"], c["seen"])
            said = tokens[:, : max(1, c["seen"] // 2)]  # the rest was in the prompt
            s["counts"] = torch.zeros(c["slots"], vocab, dtype=torch.int32, device=DEV).scatter_add_(1, said, torch.ones_like(said, dtype=torch.int32))
            marked = torch.zeros(c["slots"], _words(vocab) * 32, dtype=torch.bool, device=DEV).scatter_(1, tokens, True)
            s["seen"] = _packed(marked)
            s["repetition"] = 1.0 + torch.rand(n, generator=g, device=DEV) * 0.5
            s["frequency"] = torch.rand(n, generator=g, device=DEV)
            s["presence"] = torch.rand(n, generator=g, device=DEV) * 2 - 0.5
        s["bias"] = None
        if c["bias"]:
            per = min(c["bias"], vocab)
            lengths = torch.randint(0, per + 1, (n,), generator=g, device=DEV)
            offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), lengths.cumsum(0)])
            first = torch.randint(0, vocab // per, (n, per), generator=g, device=DEV) + torch.arange(per, device=DEV) * (vocab // per)
            keep = torch.arange(per, device=DEV) < lengths.unsqueeze(1)
            tokens = first[keep].to(torch.int32)
            s["bias"] = (offsets, tokens, torch.empty(tokens.numel(), dtype=torch.float32, device=DEV).normal_(0.0, 5.0, generator=g))
        s["masks"] = s["mask_of"] = None
        if c["masks"]:
            dense = torch.rand(c["masks"], 1, generator=g, device=DEV)  # grammars that allow little and such that allow most
            s["masks"] = _packed(torch.rand(c["masks"], _words(vocab) * 32, generator=g, device=DEV) < dense)
            s["mask_of"] = torch.randint(-1, c["masks"], (n,), generator=g, device=DEV).to(torch.int32)
    return s


def _packed(bits):
    w = bits.reshape(bits.shape[0], -1, 32).to(torch.int64) << torch.arange(32, device=DEV)
    return w.sum(dim=2).to(torch.int32)  # the same 32 bits


def _room(rows, dim, kind, scale):
    """Buffers of a quantized matrix: codes with rows of whole blocks, scales by block and row (or tile)."""
    blocks, rounded = -(-dim // BLOCK), -(-rows // BLOCK) * BLOCK
    return (torch.empty(rows, blocks * BLOCK, dtype=torch.uint8, device=DEV),
            torch.empty(blocks, rounded if kind == "row" else rounded // BLOCK, dtype=torch.uint8 if scale == "e8m0" else torch.float32, device=DEV))


# ---- the framework's operators ------------------------------------------------------------------------------

_handle = []


def _ctx():
    import paper_2010_08679_amd as P
    if not _handle:
        _handle.append(P.cnr_create(0))
    return P, _handle[0]


def _run_own(s):
    c = s["case"]
    P, ctx = _ctx()
    kinds = {"row": P.CNR_BLOCK_ROW, "tile": P.CNR_BLOCK_TILE}
    if c["op"] == "quantize":
        out = P.BlockMatrix(*s["out"], c["rows"], c["dim"], kinds[c["kind"]])
        out_t = P.BlockMatrix(*s["out_t"], c["dim"], c["rows"], kinds[c["kind"]]) if c["both"] else None
        P.quantize_blocks(ctx, s["x"], out, out_t)
        return _quantized(c, s["out"], s["out_t"])
    if c["op"] == "product":
        a = P.BlockMatrix(*s["a"], c["m"], c["k"], kinds[c["a"]])
        b = P.BlockMatrix(*s["b"], c["n"], c["k"], kinds[c["b"]])
        if c["add"]:
            s["out"].copy_(s["residual"])
        return P.block_product(ctx, a, b, s["out"], accumulate=c["add"], workspace=_kept(s, lambda: P.block_workspace(ctx, c["m"], c["n"], c["k"])))
    if c["op"] == "step":
        layer = _kept(s, lambda: P.BlockLinear(ctx, c["n"], c["k"], c["m"], P.CNR_SCALE_E8M0 if c["scale"] == "e8m0" else P.CNR_SCALE_F32))
        layer.load(s["w"])
        y = layer.forward(s["x"], s["y"])
        dx, dw = layer.backward(s["dy"], s["dx"], s["dw"])
        return {"y": y, "dx": dx, "dw": dw}
    ledger = _kept(s, lambda: P.TokenLedger(ctx, c["slots"], c["vocab"], seen=s["seen"], counts=s["counts"]))
    if c["op"] == "count":
        ledger.count(s["tokens"], s["offsets"], s["slots"], restart=c["restart"])
        return {"seen": s["seen"], "counts": s["counts"]}
    return ledger.adjust(s["logits"], s["out"], slots=s["slots"], repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"],
                         bias=s["bias"], masks=s["masks"], mask_of=s["mask_of"])


def _kept(s, make):
    """The workspace or layer that a program makes once and keeps."""
    if "kept" not in s:
        s["kept"] = make()
    return s["kept"]


def _quantized(c, out, out_t):
    """Codes as the e4m3 values that they are, and the scales that blocks have (rows beyond the last block's have none)."""
    got = {"codes": out[0].view(torch.float8_e4m3fn), "scale": out[1][:, : _scales(c["rows"], c["kind"])]}
    if out_t is not None:
        got |= {"codes_t": out_t[0].view(torch.float8_e4m3fn), "scale_t": out_t[1][:, : _scales(c["dim"], c["kind"])]}
    return got


def _scales(rows, kind):
    return rows if kind == "row" else -(-rows // BLOCK)


# ---- plain forms ------------------------------------------------------------------------------------------------

def _power(e, dtype):
    """2^e from its bits: the device's exponentials are not exact."""
    if dtype == torch.float64:
        return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _plain_quantize(x, kind, scale):
    """(e4m3 codes with rows of whole blocks, scales [block][row or tile]) of x.  With scales of any value a code is decided in 64
    bits, as a quotient next to the border of two codes needs; powers of two divide exactly in 32."""
    rows, dim = x.shape
    wide = torch.float64 if scale == "f32" else torch.float32
    high = BLOCK if kind == "tile" else 1
    v = torch.nn.functional.pad(x.to(wide), (0, -dim % BLOCK, 0, -rows % high))
    v = v.reshape(v.shape[0] // high, high, -1, BLOCK)
    amax = v.abs().amax(dim=(1, 3))
    if scale == "e8m0":
        fraction, exponent = torch.frexp(amax)  # amax = fraction 2^exponent, 448 = 0.875 2^9
        e = (exponent - 9 + (fraction > 0.875)).clamp(min=-126)
        e = torch.where(amax > 0, e, torch.zeros_like(e))
        s = _power(e, torch.float32)
        kept = (e + 127).to(torch.uint8)
    else:
        s = torch.where(amax > 0, (amax / TOP).float().clamp(min=2.0 ** -126), 1.0)
        kept = s
    q = v / s.to(wide)[:, None, :, None]
    step = _power(torch.frexp(q)[1].clamp(min=-5) - 4, wide)  # between two neighbouring codes
    q = (torch.round(q / step) * step).reshape(-1, v.shape[2] * BLOCK)[:rows]
    return q.float().to(torch.float8_e4m3fn), kept.t().contiguous()


def _plain_values(codes, scale, rows, kind):
    """The float32 values that a quantized matrix stands for."""
    s = _power(scale.to(torch.int32) - 127, torch.float32) if scale.dtype == torch.uint8 else scale
    s = s.repeat_interleave(BLOCK, dim=1) if kind == "tile" else s
    v = codes.view(torch.float8_e4m3fn).float().reshape(rows, -1, BLOCK)
    return (v * s.t()[:rows].unsqueeze(2)).reshape(rows, -1)


def _plain_linear(c, w, x, dy):
    t = TYPES[c["type"]]

    def values(m, kind):
        q, s = _plain_quantize(m, kind, c["scale"])
        return _plain_values(q, s, m.shape[0], kind)[:, : m.shape[1]]

    wide = values(w, "tile")
    return {"y": (values(x, "row") @ wide.t()).to(t), "dx": (values(dy, "row") @ wide).to(t), "dw": values(dy.t(), "row") @ values(x.t(), "row").t()}


def _plain_count(s):
    c = s["case"]
    vocab, words = c["vocab"], _words(c["vocab"])
    seen, counts, tokens = s["seen"], s["counts"], s["tokens"].to(torch.int64)
    slots = s["slots"].to(torch.int64)
    if c["restart"]:
        seen[slots] = 0
        counts[slots] = 0
    which = torch.arange(tokens.numel(), device=tokens.device)
    if s["offsets"] is not None:
        which = torch.searchsorted(s["offsets"], which, right=True) - 1
    place = torch.sort(slots[which] * vocab + tokens).values
    counts.view(-1).index_add_(0, place, torch.ones_like(place, dtype=torch.int32))
    first = torch.ones_like(place, dtype=torch.bool)
    first[1:] = place[1:] != place[:-1]
    token = place % vocab
    word = place // vocab * words + token // 32
    new = first & ((seen.view(-1)[word] >> (token % 32)) & 1 == 0)
    seen.view(-1).index_add_(0, word, (new.to(torch.int64) << (token % 32)).to(torch.int32))
    return {"seen": seen, "counts": counts}


def _bits(words, vocab):
    t = torch.arange(vocab, device=words.device)
    return (words[:, t // 32] >> (t % 32).to(torch.int32)) & 1 != 0


def _plain_adjust(s):
    vocab = s["case"]["vocab"]
    v = s["logits"].float()
    slots = s["slots"].to(torch.int64)
    if s["seen"] is not None:
        count = s["counts"][slots].float()
        again = torch.where(v > 0, v / s["repetition"][:, None], v * s["repetition"][:, None])
        v = torch.where(_bits(s["seen"], vocab)[slots], again, v)
        v = v - s["frequency"][:, None] * count
        v = v - s["presence"][:, None] * (count > 0)
    if s["bias"] is not None:
        offsets, tokens, values = s["bias"]
        row = torch.searchsorted(offsets, torch.arange(tokens.numel(), device=tokens.device), right=True) - 1
        v = v.index_put((row, tokens.to(torch.int64)), values, accumulate=True)
    if s["masks"] is not None:
        of = s["mask_of"].to(torch.int64)
        allowed = _bits(s["masks"], vocab)[of.clamp(min=0)] | (of < 0)[:, None]
        v = torch.where(allowed, v, -math.inf)
    return v.to(s["logits"].dtype)


def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    if c["op"] == "quantize":
        out, out_t = _plain_quantize(s["x"], c["kind"], c["scale"]), None
        if c["both"]:
            out_t = _plain_quantize(s["x"].t(), c["kind"], c["scale"])
        return _quantized(c, out, out_t)
    if c["op"] == "product":
        v = _plain_values(*s["a"], c["m"], c["a"]) @ _plain_values(*s["b"], c["n"], c["b"]).t()
        return (v + s["residual"].float() if c["add"] else v).to(TYPES[c["out"]])
    if c["op"] == "step":
        return _plain_linear(c, s["w"], s["x"], s["dy"])
    return _plain_count(s) if c["op"] == "count" else _plain_adjust(s)


# ---- what a pass has to read, write and compute -------------------------------------------------------------

def _held(rows, dim, kind, scale):
    """Bytes of a quantized matrix."""
    return rows * dim + -(-dim // BLOCK) * _scales(rows, kind) * (1 if scale == "e8m0" else 4)


def work(c):
    if c["op"] == "quantize":
        there = _held(c["rows"], c["dim"], c["kind"], c["scale"]) + (_held(c["dim"], c["rows"], c["kind"], c["scale"]) if c["both"] else 0)
        return {"bytes": c["rows"] * c["dim"] * SIZE[c["type"]] + there, "flops": 2 * c["rows"] * c["dim"]}
    if c["op"] == "product":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": _held(m, k, c["a"], c["scale"]) + _held(n, k, c["b"], c["scale"]) + m * n * SIZE[c["out"]] * (2 if c["add"] else 1),
                "flops": 2 * m * n * k}
    if c["op"] == "step":
        m, n, k, t = c["m"], c["n"], c["k"], SIZE[c["type"]]
        return {"bytes": n * k * (4 + 4) + 2 * t * (m * k + m * n), "flops": 6 * m * n * k}
    words = _words(c["vocab"])
    if c["op"] == "count":
        total = c["n"] * (c["longest"] / math.log(c["longest"] + 1) if c["longest"] > 1 else 1)
        return {"bytes": total * (8 if c["index"] == "i64" else 4) + total * 16 + (c["n"] * (c["vocab"] + words) * 4 if c["restart"] else 0), "flops": 0}
    elements = c["n"] * c["vocab"]
    state = c["n"] * (words * 4 + min(c["vocab"], c["seen"]) * 4) if c["penalties"] else 0
    return {"bytes": 2 * elements * SIZE[c["type"]] + state + c["n"] * c["bias"] * 4 + min(c["masks"], c["n"]) * words * 4, "flops": 8 * elements}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def _e4m3():
    """Every e4m3 value from 0 up, by code."""
    code = np.arange(127)
    e, m = code >> 3, code & 7
    return torch.tensor(np.where(e > 0, np.ldexp(1 + m / 8, e - 7), np.ldexp(m / 8, -6)), device=DEV)


def _two_to(e):
    """2^e in 64 bits, e a tensor of whole numbers above -1000."""
    table = torch.tensor(np.ldexp(1.0, np.arange(-1000, 1000)), device=DEV)
    return table[e.to(torch.int64) + 1000]


def _exact_quantize(x, kind, scale):
    """(values of the codes [rows][whole blocks], scales [block][row or tile], in 64 bits what each code is multiplied with)."""
    rows, dim = x.shape
    x = x.double()
    blocks, tiles = -(-dim // BLOCK), -(-rows // BLOCK)
    whole = torch.zeros(tiles * BLOCK, blocks * BLOCK, dtype=torch.float64, device=DEV)
    whole[:rows, :dim] = x
    largest = whole.abs().reshape(tiles * BLOCK, blocks, BLOCK).max(dim=2).values
    if kind == "tile":
        largest = largest.reshape(tiles, BLOCK, blocks).max(dim=1).values
    if scale == "e8m0":
        e = torch.ceil(torch.log2(largest / TOP)).clamp(min=-126)
        e = e - (largest <= TOP * _two_to(e - 1)).double()  # the logarithm may be a bit off next to a power of two
        e = e + (largest > TOP * _two_to(e)).double()
        e = torch.where(largest > 0, e.clamp(min=-126), torch.zeros_like(e))
        s, kept = _two_to(e), (e + 127).to(torch.uint8)
    else:
        s = torch.where(largest > 0, (largest / TOP).float().double().clamp(min=2.0 ** -126), torch.ones_like(largest))
        kept = s
    each = s.repeat_interleave(BLOCK, dim=0) if kind == "tile" else s
    each = each[:rows]
    grid = _e4m3()
    middle = (grid[1:] + grid[:-1]) / 2
    q = (whole[:rows].reshape(rows, blocks, BLOCK) / each.unsqueeze(2)).reshape(rows, -1)
    below = torch.bucketize(q.abs(), middle, right=False)
    above = torch.bucketize(q.abs(), middle, right=True)  # one more where q is half-way between two codes
    value = torch.copysign(grid[torch.where(below % 2 == 0, below, above)], q)
    return value, kept[: _scales(rows, kind)].t().contiguous(), each


def _exact_values(x, kind, scale):
    value, _, each = _exact_quantize(x, kind, scale)
    rows, dim = x.shape
    return (value.reshape(rows, -1, BLOCK) * each.unsqueeze(2)).reshape(rows, -1)[:, :dim]


def _exact_operand(codes, scale, rows, kind):
    value = torch.cat([_e4m3(), torch.full((1,), math.nan, device=DEV, dtype=torch.float64)])
    value = torch.cat([value, -value])[codes.to(torch.int64)]
    s = _two_to(scale.to(torch.int64) - 127) if scale.dtype == torch.uint8 else scale.double()
    row = torch.arange(rows, device=DEV)
    s = s[:, row // BLOCK if kind == "tile" else row]  # [block][row]
    return value * s.t().repeat_interleave(BLOCK, dim=1)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "quantize":
        value, kept, _ = _exact_quantize(s["x"], c["kind"], c["scale"])
        got = {"codes": value, "scale": kept}
        if c["both"]:
            got["codes_t"], got["scale_t"], _ = _exact_quantize(s["x"].t().contiguous(), c["kind"], c["scale"])
        return got
    if c["op"] == "product":
        v = _exact_operand(*s["a"], c["m"], c["a"]) @ _exact_operand(*s["b"], c["n"], c["b"]).t()
        return v + s["residual"].double() if c["add"] else v
    if c["op"] == "step":
        w, x, dy = (_exact_values(s["w"], "tile", c["scale"]), _exact_values(s["x"], "row", c["scale"]), _exact_values(s["dy"], "row", c["scale"]))
        x_t, dy_t = (_exact_values(v.t().contiguous(), "row", c["scale"]) for v in (s["x"], s["dy"]))
        return {"y": x @ w.t(), "dx": dy @ w, "dw": dy_t @ x_t.t()}
    if c["op"] == "count":
        slots, tokens = s["slots"].cpu().numpy(), s["tokens"].cpu().numpy()
        offsets = np.arange(c["n"] + 1) if s["offsets"] is None else s["offsets"].cpu().numpy()
        counts = np.zeros((c["slots"], c["vocab"]), dtype=np.int32)
        for i in range(c["n"]):
            counts[slots[i]] += np.bincount(tokens[offsets[i]:offsets[i + 1]], minlength=c["vocab"]).astype(np.int32)
        bits = np.zeros((c["slots"], _words(c["vocab"]) * 32), dtype=np.uint8)
        bits[:, : c["vocab"]] = counts > 0
        return {"seen": np.packbits(bits, axis=1, bitorder="little").view(np.int32), "counts": counts}
    v = s["logits"].double()
    for i in range(c["n"]):
        row, slot = v[i], int(s["slots"][i])
        if c["penalties"]:
            marks = np.unpackbits(s["seen"][slot].cpu().numpy().view(np.uint8), bitorder="little")[: c["vocab"]]
            at = torch.from_numpy(np.flatnonzero(marks)).to(DEV)
            rep, f, p = (float(s[name][i]) for name in ("repetition", "frequency", "presence"))
            row[at] = torch.where(row[at] > 0, row[at] / rep, row[at] * rep)
            count = s["counts"][slot].double()
            row -= f * count
            row[count > 0] -= p
        if s["bias"] is not None:
            lo, hi = int(s["bias"][0][i]), int(s["bias"][0][i + 1])
            row[s["bias"][1][lo:hi].to(torch.int64)] += s["bias"][2][lo:hi].double()
        if s["masks"] is not None and int(s["mask_of"][i]) >= 0:
            marks = np.unpackbits(s["masks"][int(s["mask_of"][i])].cpu().numpy().view(np.uint8), bitorder="little")[: c["vocab"]]
            row[torch.from_numpy(np.flatnonzero(marks == 0)).to(DEV)] = -math.inf
    return v
