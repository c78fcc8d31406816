"""Losses over a vocabulary, their gradients and top logits in 64 bits, with bounds on what fp32 sums and roundings to the operands' type may be off by.

Test infrastructure only: torch tensors on any device, no code shared with the library.
"""
import math

import torch

# half a step, relative to the value
ROUNDING = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# and of the smallest values, for which that is nothing: halves below 2^-14 are 2^-24 apart, so a result is off by up to 2^-25; those of the other types are below 2^-133
SMALLEST = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def shares(tokens, vocab, logits=None, temperature=1.0):
    """float64 [n, top]: the probability of each entry; 0 for those that do not count."""
    there = (tokens >= 0) & (tokens < vocab)
    if logits is None:
        return there.double()
    v = torch.where(there, logits.double() / temperature, -math.inf)
    most = v.max(dim=1, keepdim=True).values if tokens.shape[1] else v.sum(dim=1, keepdim=True) - math.inf
    left = most > -math.inf
    e = torch.where(left & there, torch.exp(v - torch.where(left, most, 0.0)), 0.0)
    return torch.where(left, e / torch.where(left, e.sum(dim=1, keepdim=True), 1.0), 0.0)


def loss(hidden, weight, tokens, logits=None, temperature=1.0, dloss=None, there=None, parts=1):
    """A dict of (value, bound) for losses and, with dloss, dhidden and dweight; `there`: what the weight's gradient is added to; `parts`: numbers of the operands'
    type that dz is held in for the weight's gradient.  Rows that are left out may hold anything."""
    kind = hidden.dtype
    u, e = 2.0 ** -24, ROUNDING[kind]
    n, dim = hidden.shape
    vocab = weight.shape[0]
    tokens = tokens.to(torch.int64)
    tokens = tokens[:, None] if tokens.dim() == 1 else tokens
    q = shares(tokens, vocab, logits, temperature)
    counts = (q.sum(dim=1) != 0) if tokens.shape[1] else torch.zeros(n, dtype=torch.bool, device=hidden.device)  # NaN counts
    adds = counts if dloss is None else counts & (dloss != 0)
    x, w = torch.where(counts[:, None], hidden.double(), 0.0), weight.double()
    z = x @ w.t() / temperature
    # a sum of dim products, each added with one rounding: at most dim + 1 of them; the scaling to base 2 and its undoing are a few more of |z|
    z_off = ((dim + 8) * u * (x.abs() @ w.abs().t()) / temperature) + 4 * u
    # a float as three bfloat16: zero parts and what is below bfloat16's smallest number, 2^-133, are held as that number: three parts, each off by 2^-133 at most
    part = 2.0 ** -131 if kind == torch.float32 else 0.0
    z_off = z_off + part * (x.abs().sum(dim=1)[:, None] + w.abs().sum(dim=1)[None, :]) / temperature
    lse = torch.logsumexp(z, dim=1) if vocab else torch.full((n,), -math.inf, dtype=torch.float64, device=hidden.device)
    most_off = z_off.max(dim=1).values if vocab else torch.zeros_like(lse)
    at = tokens.clamp(0, max(vocab - 1, 0))
    picked = z.gather(1, at) if vocab else torch.zeros_like(q)
    terms = torch.where(q != 0, q * (torch.log(torch.where(q != 0, q, 1.0)) - picked), 0.0)
    value = torch.where(counts, terms.sum(dim=1) + lse, 0.0)
    # the entries' logarithms and shares come from a softmax in fp32 of their own: some roundings of the largest magnitude in it, and of the sum's
    # vocab + top terms; the parts of the sum are joined pairwise, a rounding or two for each level and a multiplication by a power each
    entropy = torch.where(q != 0, q * torch.log(torch.where(q != 0, q, 1.0)), 0.0).abs().sum(dim=1)
    given = 0.0 if logits is None else torch.where(q != 0, logits.double() / temperature, 0.0).abs().max(dim=1).values
    picked_size = torch.where(q != 0, picked.abs(), 0.0).sum(dim=1)
    off = 2 * most_off + (math.log2(vocab + 2) * 4 + 300) * u + (tokens.shape[1] + 8) * u * (entropy + picked_size + 1) + 16 * u * (lse.abs() + given)
    got = {"losses": (value, torch.where(counts, off, 0.0))}
    if dloss is None:
        return got
    g = torch.where(adds, dloss.double() / temperature, 0.0)
    p = torch.where(adds[:, None], torch.exp(z - lse[:, None]), 0.0)
    want = torch.zeros_like(z)
    if vocab:
        want.scatter_add_(1, at, torch.where(adds[:, None], q, 0.0))
    dz = g[:, None] * (p - want)
    # the exponent's error, that of the logarithm of the sum, and the shares'
    p_off = p * (torch.expm1(z_off + 2 * most_off[:, None] + (math.log2(vocab + 2) * 4 + 300) * u) + 32 * u * (z.abs() + lse.abs()[:, None]))
    dz_off = g.abs()[:, None] * (p_off + want * (tokens.shape[1] + 32) * u * (1 + (given[:, None] if logits is not None else 0.0))) + 4 * u * dz.abs()
    if kind == torch.float16 and n:
        dz_off += 2.0 ** -38 * g.abs().max()  # half a step of the smallest halves, which the largest gradient is 2^13 above at least
    kept = torch.where(adds[:, None], x, 0.0)

    def sums(a, a_off, b, terms):
        """a b with a off by a_off, added up in fp32 (two sums where a is in two parts; parts of sums joined: 20 more)."""
        # below 2^-126 numbers of fp32 are 2^-149 apart: each of up to six additions a term, of the joins and of what follows is off by half of that besides
        smallest = part * (a.abs().sum(dim=1)[:, None] + b.abs().sum(dim=0)[None, :]) + (6 * terms + 64) * 2.0 ** -150
        return a @ b, a_off @ b.abs() + (terms + 32) * u * ((a.abs() + a_off) @ b.abs()) + smallest

    dh, dh_off = sums(dz, dz_off + e * dz.abs(), w, vocab)
    dw, dw_off = sums(dz.t(), (dz_off + e ** parts * dz.abs()).t(), kept, n)
    # the gradients' sums are of numbers scaled, and rounded once more at the end
    got["dhidden"] = dh, dh_off + e * (dh.abs() + dh_off) + SMALLEST[kind]
    if there is not None:
        dw = dw + there.double()
    out = u if parts == 2 or kind == torch.float32 else e
    got["dweight"] = dw, dw_off + parts * out * (dw.abs() + dw_off) + (0.0 if out == u else SMALLEST[kind]) + (0.0 if there is None else 2 * u * there.double().abs())
    return got


def place(v):
    """Whole numbers in the order of the values, NaN last, -0 as 0."""
    bits = v.float().view(torch.int32).to(torch.int64)
    order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    return torch.where(torch.isnan(v), 1 << 31, order)


def top(logits, k):
    """(tokens int32 [n, k], values [n, k], lse float64 [n]) by sorting unique keys."""
    n, vocab = logits.shape
    key = place(logits) * (1 << 31) - torch.arange(vocab, device=logits.device)
    order = key.argsort(dim=1, descending=True)[:, :k]
    tokens = torch.full((n, k), -1, dtype=torch.int32, device=logits.device)
    values = torch.full((n, k), -math.inf, dtype=logits.dtype, device=logits.device)
    tokens[:, : order.shape[1]] = order.to(torch.int32)
    values[:, : order.shape[1]] = logits.gather(1, order)
    lse = torch.logsumexp(logits.double(), dim=1) if vocab else torch.full((n,), -math.inf, dtype=torch.float64, device=logits.device)
    return tokens, values, lse
