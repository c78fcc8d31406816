"""More performance cases of the operators for language models: losses of the matrix that gives the logits, and top logits.

A case's "op" says what one pass runs:

  score    the losses of tokens alone, forward: softmax cross entropy over the vocabulary, whose logits are not kept
  step     the same in training: losses, then the gradients of the hidden states and of the matrix
  distill  a training step of a student whose targets are a teacher's top logits, at a temperature
  top      the largest logits of each row with their tokens, and the logarithm of the sum of all exponentials

Hidden states hold normal values and some of their target's row, so that some tokens are certain and some are not; tokens are Zipf
distributed; a tenth of the targets are padding (-100), some rows of the teacher's end early (-1).
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # the log probability of one token of a sequence that is served: the matrix is read once
        dict(name="score_1x32000x4096", op="score", n=1, vocab=32000, dim=4096, stride=4096, type="bf16", index="i64"),
        # the losses of an evaluation's tokens
        dict(name="score_4096x131072x4096", op="score", n=4096, vocab=131072, dim=4096, stride=4096, type="bf16", index="i64"),
        # odd sizes that end inside tiles, rows that start at any element
        dict(name="step_1000x1111x1100", op="step", n=1000, vocab=1111, dim=1100, stride=1113, type="f16", index="i32", grad="f16", add=False),
        # a training batch of a model with an odd vocabulary
        dict(name="step_8192x50257x2048", op="step", n=8192, vocab=50257, dim=2048, stride=2048, type="bf16", index="i64", grad="bf16", add=False),
        # an fp32 table that is trained as the matrix of the logits too: its gradient is added to that of the look-ups
        dict(name="step_2048x32000x1024_f32", op="step", n=2048, vocab=32000, dim=1024, stride=1024, type="f32", index="i64", grad="f32", add=True),
        # a large batch of a large model
        dict(name="step_16384x131072x4096", op="step", n=16384, vocab=131072, dim=4096, stride=4096, type="bf16", index="i64", grad="bf16", add=False),
        # a short batch of a student in half precision, few top logits
        dict(name="distill_333x50257x1024_top20", op="distill", n=333, vocab=50257, dim=1024, stride=1024, type="f16", index="i32", grad="f16", add=False,
             top=20, teacher="f16", temperature=1.0),
        # a student's micro-batch: the gradient of the matrix is added up in fp32 over several
        dict(name="distill_8192x32000x4096_top64", op="distill", n=8192, vocab=32000, dim=4096, stride=4096, type="bf16", index="i64", grad="f32", add=True,
             top=64, teacher="bf16", temperature=2.0),
        # the most likely tokens of one sequence
        dict(name="top50_1x50257", op="top", n=1, vocab=50257, stride=50257, type="f32", top=50),
        # those of a large decoding batch
        dict(name="top64_512x131072", op="top", n=512, vocab=131072, stride=131072, type="bf16", top=64),
        # a teacher's logits of a training batch, kept for its students
        dict(name="top64_8192x32000", op="top", n=8192, vocab=32000, stride=32000, type="bf16", top=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size of the range: as it comes (odd as often as not), or the multiple of 64 next to it."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.6 else min(hi, max(lo, (n + 32) // 64 * 64 or 64))


def draw(rng):
    op = rng.choice(["score", "step", "step", "distill", "distill", "top"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "top":
        vocab = _size(rng, 100, 262144)
        return dict(op=op, n=_log_int(rng, 1, min(8192, (1 << 28) // vocab)), vocab=vocab, stride=vocab + rng.choice([0, 0, 8, 13]), type=kind,
                    top=min(vocab, _log_int(rng, 1, 256)))
    dim = _size(rng, 32, 8192)
    vocab = _size(rng, 128, 262144)
    most = (1 << 41) // (vocab * dim) if kind != "f32" else (1 << 37) // (vocab * dim)
    n = _size(rng, 1, max(1, min(16384, most)))
    c = dict(op=op, n=n, vocab=vocab, dim=dim, stride=dim + rng.choice([0, 0, 8, 13]), type=kind, index=rng.choice(["i32", "i64"]))
    if op == "score":
        return c
    c |= dict(grad=rng.choice([kind, kind, "f32"]), add=rng.random() < 0.4)
    if op == "distill":
        c |= dict(top=min(vocab, _log_int(rng, 1, 256)), teacher=rng.choice(["f32", "bf16", "f16"]), temperature=rng.choice([0.5, 1.0, 2.0, 4.0]))
    return c


# ---- inputs -------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, rows, columns, stride, dtype, sigma):
    """Rows `stride` apart."""
    x = torch.empty(rows, stride, dtype=dtype, device=DEV)
    for at in range(0, rows, 16384):
        part = x[at:at + 16384]
        part.copy_(torch.empty(part.shape, dtype=torch.float32, device=DEV).normal_(0.0, sigma, generator=g))
    return x[:, :columns]


def _tokens(g, n, vocab):
    """Zipf(1) distributed tokens in a scattered order of the vocabulary."""
    u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
    rank = torch.exp(u * math.log(vocab + 1)).to(torch.int64) - 1
    return (rank.clamp(0, vocab - 1) * 7919 + 12345) % vocab


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    n, vocab, t = c["n"], c["vocab"], TYPES[c["type"]]
    s = {"case": c}
    if c["op"] == "top":
        z = _normal(g, n, vocab, c["stride"], t, 4.0)
        # a grammar's mask in every fourth row: some leave most, some a few tokens
        for i in range(0, n, 4 * max(1, n // 64)):
            z[i, torch.rand(vocab, generator=g, device=DEV) < torch.rand(1, generator=g, device=DEV)] = -math.inf
        s["logits"] = z
        return s
    dim = c["dim"]
    w = _normal(g, vocab, dim, c["stride"], t, 1.0 / math.sqrt(dim))
    token = _tokens(g, n, vocab)
    h = torch.empty(n, c["stride"], dtype=torch.float32, device=DEV).normal_(0.0, 2.5, generator=g)
    h[:, :dim] += w[token].float() * torch.empty(n, 1, device=DEV).uniform_(0.0, 16.0, generator=g)
    s["weight"], s["hidden"] = w, h.to(t)[:, :dim]
    kind = torch.int32 if c["index"] == "i32" else torch.int64
    if c["op"] == "distill":
        k = c["top"]
        each = torch.randint(0, vocab // k, (n, k), generator=g, device=DEV) + torch.arange(k, device=DEV) * (vocab // k)
        each = each.gather(1, torch.rand(n, k, generator=g, device=DEV).argsort(dim=1))  # in no order
        ends = torch.where(torch.rand(n, generator=g, device=DEV) < 0.1, torch.randint(0, k + 1, (n,), generator=g, device=DEV), k)
        s["tokens"] = torch.where(torch.arange(k, device=DEV) < ends[:, None], each, -1).to(kind)
        largest_first = torch.empty(n, k, device=DEV).normal_(8.0, 4.0, generator=g).sort(dim=1, descending=True).values
        s["teacher"] = largest_first.to(TYPES[c["teacher"]])
    else:
        s["tokens"] = torch.where(torch.rand(n, generator=g, device=DEV) < 0.1 if n > 1 else torch.zeros(n, dtype=torch.bool, device=DEV), -100, token).to(kind)
    if c["op"] != "score":
        # what the mean over the batch gives each loss, or weights of its own to each
        s["dloss"] = torch.full((n,), 1.0 / n, device=DEV) * torch.empty(n, device=DEV).uniform_(0.5, 1.5, generator=g)
        s["dhidden"] = torch.empty(n, dim, dtype=t, device=DEV)
        s["dweight"] = torch.empty(vocab, dim, dtype=TYPES[c["grad"]], device=DEV)
        # as large as a token's part of the gradient
        s["there"] = _normal(g, vocab, dim, dim, TYPES[c["grad"]], 1.0 / n) if c["add"] else None
    return s


# ---- the framework's operators ------------------------------------------------------------------------------

_handle = []


def _ctx():
    import paper_2010_08679_amd as P
    if not _handle:
        _handle.append(P.cnr_create(0))
    return P, _handle[0]


def _kept(s, make):
    """The workspace that a program makes once and keeps."""
    if "kept" not in s:
        s["kept"] = make()
    return s["kept"]


def _run_own(s):
    c = s["case"]
    P, ctx = _ctx()
    if c["op"] == "top":
        tokens, values, lse = P.top_logits(ctx, s["logits"], c["top"])
        return {"tokens": tokens, "values": values, "lse": lse}
    training = c["op"] != "score"
    loss = _kept(s, lambda: P.VocabularyLoss(ctx, c["vocab"], c["dim"], c["n"], TYPES[c["type"]], top=c.get("top", 1), training=training,
                                             gradient_dtype=TYPES[c["grad"]] if training else None))
    if c["op"] == "distill":
        losses = loss.distill(s["hidden"], s["weight"], s["tokens"], s["teacher"], c["temperature"])
    else:
        losses = loss.cross_entropy(s["hidden"], s["weight"], s["tokens"], training=training)
    if not training:
        return losses
    if c["add"]:
        s["dweight"].copy_(s["there"])
    dhidden, dweight = loss.backward(s["dloss"], s["dhidden"], s["dweight"], accumulate=c["add"])
    return {"losses": losses, "dhidden": dhidden, "dweight": dweight}


# ---- plain forms ------------------------------------------------------------------------------------------------

def _plain_lse(z):
    """log sum exp of each row; of a row of -infinity that."""
    top = z.amax(dim=1, keepdim=True).clamp(min=-3e38)
    return top.squeeze(1) + torch.log(torch.exp(z - top).sum(dim=1))


def _plain_teacher(c, tokens, teacher):
    """(tokens with 0 for none, the teacher's probabilities, their logarithms with 0 for none)."""
    there = (tokens >= 0) & (tokens < c["vocab"])
    v = torch.where(there, teacher / c["temperature"], -math.inf)
    log_q = v - _plain_lse(v)[:, None]
    there = there & (log_q > -math.inf)  # a row without entries has NaN there
    return torch.where(there, tokens, 0), torch.where(there, torch.exp(log_q), 0.0), torch.where(there, log_q, 0.0)


def _plain_loss(s):
    c = s["case"]
    h, w, tokens = s["hidden"].float(), s["weight"].float(), s["tokens"].to(torch.int64)
    z = h @ w.t()
    heat = c.get("temperature", 1.0)
    if c["op"] == "distill":
        z.mul_(1.0 / heat)
        at, q, log_q = _plain_teacher(c, tokens, s["teacher"].float())
    else:
        counts = ((tokens >= 0) & (tokens < c["vocab"]))[:, None]
        at, q = torch.where(counts, tokens[:, None], 0), counts.float()
        log_q = torch.zeros_like(q)
    lse = _plain_lse(z)
    losses = (q * (log_q - z.gather(1, at) + lse[:, None])).sum(dim=1)
    if c["op"] == "score":
        return losses
    g = s["dloss"] / heat
    some = q.sum(dim=1) > 0
    dz = z.sub_(lse[:, None]).exp_().mul_(torch.where(some, g, 0.0)[:, None])
    dz.scatter_add_(1, at, -q * g[:, None])
    dw = dz.t() @ h
    if c["add"]:
        dw += s["there"].float()
    return {"losses": losses, "dhidden": (dz @ w).to(TYPES[c["type"]]), "dweight": dw.to(TYPES[c["grad"]])}


def _plain_top(s):
    k = s["case"]["top"]
    z = s["logits"]
    values, tokens = torch.sort(z, dim=1, descending=True, stable=True)
    return {"tokens": tokens[:, :k].to(torch.int32), "values": values[:, :k], "lse": _plain_lse(z.float())}


def run(s):
    if own:
        return _run_own(s)
    return _plain_top(s) if s["case"]["op"] == "top" else _plain_loss(s)


# ---- what a pass has to read, write and compute -------------------------------------------------------------

def work(c):
    n, vocab, e = c["n"], c["vocab"], SIZE[c["type"]]
    if c["op"] == "top":
        return {"bytes": n * vocab * e + n * c["top"] * (4 + e) + 4 * n, "flops": 2 * n * vocab}
    dim = c["dim"]
    given = (n + vocab) * dim * e + n * (4 if c["index"] == "i32" else 8) * c.get("top", 1) + 4 * n
    if c["op"] == "score":
        return {"bytes": given, "flops": 2 * n * vocab * dim}
    if c["op"] == "distill":
        given += n * c["top"] * SIZE[c["teacher"]]
    # the logits and two products; computing the logits twice is a choice
    return {"bytes": given + 4 * n + n * dim * e + vocab * dim * SIZE[c["grad"]] * (2 if c["add"] else 1), "flops": 6 * n * vocab * dim}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def _exact_top(c, z):
    """Each row's keys are unique whole numbers: the value's place among all values of its type, then the lower token."""
    n, vocab, k = c["n"], c["vocab"], c["top"]
    tokens = torch.empty(n, k, dtype=torch.int32, device=DEV)
    lse = torch.empty(n, dtype=torch.float64, device=DEV)
    for at in range(0, n, 256):
        part = z[at:at + 256]
        bits = part.float().view(torch.int32).to(torch.int64)  # exact, in order but for the sign
        place = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
        key = place * (1 << 31) - torch.arange(vocab, device=DEV)
        best = torch.topk(key, k, dim=1, sorted=True).values
        tokens[at:at + 256] = ((-best) % (1 << 31)).to(torch.int32)
        lse[at:at + 256] = torch.logsumexp(part.double(), dim=1)
    return {"tokens": tokens, "values": z.gather(1, tokens.to(torch.int64)).double(), "lse": lse}


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "top":
        return _exact_top(c, s["logits"])
    n, vocab, dim = c["n"], c["vocab"], c["dim"]
    heat = c.get("temperature", 1.0)
    w = s["weight"].double()
    losses = torch.zeros(n, dtype=torch.float64, device=DEV)
    training = c["op"] != "score"
    if training:
        dh = torch.empty(n, dim, dtype=torch.float64, device=DEV)
        dw = s["there"].double() if c["add"] else torch.zeros(vocab, dim, dtype=torch.float64, device=DEV)
    step = max(1, (1 << 28) // vocab)
    for lo in range(0, n, step):
        hi = min(n, lo + step)
        h = s["hidden"][lo:hi].double()
        log_p = torch.log_softmax(h @ w.t() / heat, dim=1)
        wanted = torch.zeros_like(log_p)  # the targets' probabilities over the whole vocabulary
        ids = s["tokens"][lo:hi].to(torch.int64)
        if c["op"] == "distill":
            valid = (ids >= 0) & (ids < vocab)
            given = s["teacher"][lo:hi].double() / heat
            weights = torch.where(valid, torch.exp(given - given.max(dim=1, keepdim=True).values), 0.0)
            share = weights / weights.sum(dim=1, keepdim=True).clamp(min=1e-320)
            wanted.scatter_add_(1, ids.clamp(0, vocab - 1), share)
        else:
            valid = (ids >= 0) & (ids < vocab)
            share = valid.double()[:, None]
            wanted.scatter_add_(1, ids.clamp(0, vocab - 1)[:, None], share)
        # tokens are distinct within a row here, so the entropy is that of the shares
        negative_entropy = torch.where(share > 0, share * torch.log(share.clamp(min=1e-320)), 0.0).sum(dim=1)
        losses[lo:hi] = negative_entropy - torch.where(wanted > 0, wanted * log_p, 0.0).sum(dim=1)
        if training:
            mass = wanted.sum(dim=1, keepdim=True)  # 1, or 0 in a row that is left out
            dz = (mass * torch.exp(log_p) - wanted) * (s["dloss"][lo:hi].double() / heat)[:, None]
            dh[lo:hi] = dz @ w
            dw += dz.t() @ h
    return {"losses": losses, "dhidden": dh, "dweight": dw} if training else losses
