"""Losses over the vocabulary and top logits at the edges of their values, sizes and places: certain tokens, small floats, infinite weights, rows and vocabularies that go by pieces,
results next to operands."""
import math

import pytest
import torch

import paper_2010_08679_amd as P
from oracle import losses as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def ctx():
    c = P.cnr_create(0)
    yield c
    torch.cuda.synchronize()
    P.cnr_destroy(c)


def _near(got, want, name):
    value, off = want
    wrong = ~((got.double() - value).abs() <= off)
    assert not bool(wrong.any()), "%s: %d of %d, e.g. %r for %r +- %r" % (
        name, int(wrong.sum()), wrong.numel(), got[wrong][0].item(), value[wrong][0].item(), off[wrong][0].item())


def _normal(g, n, dim, sigma=1.0):
    return torch.empty(n, dim, device=DEV).normal_(0.0, sigma, generator=g)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,vocab,dim,pad", [(1, 500, 512, 0), (8, 2000, 512, 0), (16, 20000, 520, 3), (40, 20000, 1000, 0), (64, 700, 512, 1), (70, 700, 600, 1), (300, 2000, 512, 0),
                                             (1500, 9000, 512, 0)])
def test_certain_tokens_lose_nothing(ctx, n, vocab, dim, pad, kind):
    """Logits of thousands whose largest is the target's by hundreds: the loss is what the other tokens leave, nothing, however large |z| is.  The exponential of the
    largest is that of a rounding's size, off by a step of 2^-23 with it; the logarithm of one next to 1 is as near; the sum of both is added and multiplied
    with a rounding each: below 2^-20 all together.  With one token the teacher is the target."""
    g, t = torch.Generator(device=DEV).manual_seed(n), TYPES[kind]
    w = _normal(g, vocab, dim + pad).to(t)[:, :dim]
    targets = torch.randint(0, vocab, (n,), generator=g, device=DEV)
    x = (4.0 * w[targets].float() + _normal(g, n, dim)).to(t)
    z = x.double() @ w.double().t()
    assert float((z.topk(2, dim=1).values @ torch.tensor([1.0, -1.0], dtype=torch.float64, device=DEV)).min()) > 100 and bool((z.argmax(dim=1) == targets).all())
    targets[::7] = -100
    loss = P.VocabularyLoss(ctx, vocab, dim, n, t)
    hard = loss.cross_entropy(x, w, targets)
    assert 0.0 <= float(hard.min()) and float(hard.max()) <= 2.0 ** -20
    soft = loss.distill(x, w, targets[:, None].contiguous(), torch.zeros(n, 1, device=DEV))
    assert float(soft.abs().max()) <= 2.0 ** -20


@pytest.mark.parametrize("kind,n,vocab,top", [("f32", 5, 300, 1024), ("bf16", 16, 70001, 64), ("f16", 3, 4096, 7), ("f32", 60, 33000, 40), ("bf16", 1, 1_000_000, 3)])
def test_entries_of_few_rows_are_found_in_the_product(ctx, kind, n, vocab, top):
    """Entries that are crowded into a few tokens, at both ends of the vocabulary, or nowhere, where few rows go without tiles."""
    g, t = torch.Generator(device=DEV).manual_seed(top), TYPES[kind]
    x, w = _normal(g, n, 40, 2.0).to(t), _normal(g, vocab, 40, 0.2).to(t)
    tokens = torch.randint(0, vocab, (n, top), generator=g, device=DEV)
    tokens[1::4] = vocab - 1 - torch.randint(0, 5, tokens[1::4].shape, generator=g, device=DEV)
    tokens[2::4] = torch.randint(0, 20, tokens[2::4].shape, generator=g, device=DEV)
    tokens[3::4, 1:] = -1
    logits, dloss = _normal(g, n, top, 3.0), torch.rand(n, generator=g, device=DEV)
    want = R.loss(x, w, tokens, logits, 2.0, dloss)
    loss = P.VocabularyLoss(ctx, vocab, 40, n, t, top=top)
    _near(loss.distill(x, w, tokens, logits, 2.0), want["losses"], "losses")
    dx, dw = loss.backward(dloss)
    _near(dx, want["dhidden"], "dhidden")
    _near(dw, want["dweight"], "dweight")


@pytest.mark.parametrize("exponent", [-90, -114, -122])
@pytest.mark.parametrize("n,vocab,dim", [(100, 300, 64), (300, 2000, 200), (10, 300, 64)])
def test_small_floats_are_as_exact_as_others(ctx, n, vocab, dim, exponent):
    """Hidden states of few bits around 2^exponent, whose further parts are zeros, and a weight that makes ordinary logits of them."""
    g = torch.Generator(device=DEV).manual_seed(n)
    x = (1.0 + torch.rand(n, dim, generator=g, device=DEV)).bfloat16().float() * 2.0 ** exponent
    w = _normal(g, vocab, dim) * 2.0 ** (-exponent - 2)
    targets, dloss = torch.randint(0, vocab, (n,), generator=g, device=DEV), torch.rand(n, generator=g, device=DEV)
    want = R.loss(x, w, targets, dloss=dloss)
    loss = P.VocabularyLoss(ctx, vocab, dim, n, torch.float32)
    _near(loss.cross_entropy(x, w, targets), want["losses"], "losses")
    dx, dw = loss.backward(dloss)
    _near(dx, want["dhidden"], "dhidden")
    _near(dw, want["dweight"], "dweight")


@pytest.mark.parametrize("small", [1.0, 2.0 ** -110 * (1 + 2.0 ** -23), 2.0 ** -130, 2.0 ** -140, 2.0 ** -149])
@pytest.mark.parametrize("n", [5, 100])
def test_minus_infinity_times_a_small_float(ctx, n, small):
    """A float of which a part is below bfloat16's smallest number, or all of it: -infinity times it is -infinity, a token without probability."""
    vocab, dim = 300, 40
    g = torch.Generator(device=DEV).manual_seed(6)
    x, w = _normal(g, n, dim, 2.0), _normal(g, vocab, dim, 0.2)
    x[:, -1] = small
    w[:, -1] = 0.0
    gone = torch.arange(vocab, device=DEV) % 3 == 1
    w[gone, -1] = -math.inf
    targets = torch.randint(0, vocab // 3, (n,), generator=g, device=DEV) * 3
    kept = (~gone).nonzero()[:, 0]
    got = P.VocabularyLoss(ctx, vocab, dim, n, torch.float32).cross_entropy(x, w, targets)
    _near(got, R.loss(x, w[kept], torch.searchsorted(kept, targets))["losses"], "losses")


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,vocab,dim", [(8, 500, 64), (40, 500, 72), (100, 500, 64), (500, 9000, 40), (2100, 40000, 64)])
def test_rows_that_are_left_out_have_no_gradient_whatever_the_weight_holds(ctx, kind, n, vocab, dim):
    """Infinities and NaN in the weight make every other row's loss and gradient NaN, and not those of padding, of a teacher without entries or with a dloss of 0."""
    g, t = torch.Generator(device=DEV).manual_seed(n), TYPES[kind]
    x, w = _normal(g, n, dim).to(t), _normal(g, vocab, dim, 0.2).to(t)
    w[7], w[9, 3] = math.inf, math.nan
    targets = torch.randint(10, vocab, (n,), generator=g, device=DEV)
    dloss = torch.ones(n, device=DEV)
    targets[::4], dloss[1::4] = -100, 0.0
    none = (targets < 0) | (dloss == 0)
    loss = P.VocabularyLoss(ctx, vocab, dim, n, t, top=2)
    tokens = torch.stack([targets, torch.where(targets < 0, -1, 11)], dim=1)
    for losses in (lambda: loss.cross_entropy(x, w, targets), lambda: loss.distill(x, w, tokens, torch.zeros(n, 2, device=DEV))):
        got = losses()
        assert bool((got[targets < 0] == 0).all()) and bool(got[targets >= 0].isnan().all())
        dx, _ = loss.backward(dloss)
        assert bool((dx[none] == 0).all()) and bool(dx[~none].isnan().any(dim=1).all())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,vocab,top", [(3, 900, 50), (1300, 5003, 100), (2, 131_075, 300)])
def test_top_values_are_the_rows_own_bits(ctx, kind, n, vocab, top):
    """Zeros keep their signs and NaN their bits, in rows of few and of many such."""
    t = TYPES[kind]
    whole = torch.int32 if kind == "f32" else torch.int16
    g = torch.Generator(device=DEV).manual_seed(vocab)
    x = -_normal(g, n, vocab).abs().to(t)
    x[:, torch.randint(0, vocab, (30,), generator=g, device=DEV)] = 0.0
    x[:, torch.randint(0, vocab, (30,), generator=g, device=DEV)] = -0.0
    x[1] = -0.0
    x[1, 5::7] = 0.0
    exponent = {"f32": 0x7F800000, "bf16": 0x7F80, "f16": 0x7C00}[kind]
    payload = torch.randint(1, 0x70, (vocab // 9 + 1,), generator=g, device=DEV).to(whole)
    bits = x.view(whole)
    bits[0, ::9] = (payload | exponent)[: len(bits[0, ::9])]
    bits[0, 4::9] = (payload | (exponent - (1 << (31 if kind == "f32" else 15))))[: len(bits[0, 4::9])]  # the same, negative
    tokens, values, _ = P.top_logits(ctx, x, top)
    assert torch.equal(tokens, R.top(x, top)[0])
    assert torch.equal(values.view(whole), bits.gather(1, tokens.long()))


def test_rows_that_are_laid_out_by_several_launches(ctx):
    """More than 2^28 pieces of 16 bytes, of rows at an odd distance; the rows around the border and behind it are those with a gradient."""
    n, vocab, dim = 131_200, 100, 16392
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.empty(n, dim + 1, dtype=torch.bfloat16, device=DEV)[:, :dim]
    for at in range(0, n, 8200):
        x[at:at + 8200] = _normal(g, 8200, dim)
    w = (_normal(g, vocab, dim) / 128.0).bfloat16()
    targets, dloss = torch.randint(0, vocab, (n,), generator=g, device=DEV), torch.rand(n, generator=g, device=DEV)
    border = (1 << 28) * 8 // (dim + 56)  # (whole blocks of 64 elements)
    assert n - 1000 < border < n - 500
    dloss[: border - 1000] = 0.0
    loss = P.VocabularyLoss(ctx, vocab, dim, n)
    losses = loss.cross_entropy(x, w, targets)
    dx, dw = loss.backward(dloss)
    for at in range(0, n, 8200):
        part = slice(at, at + 8200)
        _near(losses[part], R.loss(x[part], w, targets[part])["losses"], "losses")
    assert not bool(dx[: border - 1000].any())
    want = R.loss(x[border - 1000:], w, targets[border - 1000:], dloss=dloss[border - 1000:])
    _near(dx[border - 1000:], want["dhidden"], "dhidden")
    _near(dw, want["dweight"], "dweight")


@pytest.mark.parametrize("kind,n,vocab,dim,grad", [("bf16", 3, (1 << 23) + 300, 7, "bf16"), ("f16", 2, (1 << 23) + 17, 5, "f32"), ("f32", 40, (1 << 21) + 100, 8, "f32")])
def test_few_rows_of_a_vocabulary_of_several_pieces(ctx, kind, n, vocab, dim, grad):
    """Targets and entries on both sides of the border between the pieces of dz, onto a gradient that is there."""
    piece = (1 << 23) if n <= 16 else 1 << 21
    g, t = torch.Generator(device=DEV).manual_seed(n), TYPES[kind]
    x, w = _normal(g, n, dim, 2.0).to(t), _normal(g, vocab, dim).to(t)
    targets, dloss = torch.randint(0, vocab, (n,), generator=g, device=DEV), torch.rand(n, generator=g, device=DEV)
    targets[0], targets[1] = piece, piece - 1
    there = _normal(g, vocab, dim, 1e-3).to(TYPES[grad])
    tokens = torch.stack([targets, targets.flip(0), torch.full_like(targets, vocab - 1), torch.full_like(targets, -1)], dim=1)
    logits = _normal(g, n, 4)
    loss = P.VocabularyLoss(ctx, vocab, dim, n, t, top=4, gradient_dtype=TYPES[grad])
    assert loss._space.numel() < 3 << 29
    for teacher in ((targets,), (tokens, logits, 2.0)):
        want = R.loss(x, w, *teacher, dloss=dloss, there=there, parts=2 if grad != kind else 1)
        _near(loss.cross_entropy(x, w, *teacher) if len(teacher) == 1 else loss.distill(x, w, *teacher), want["losses"], "losses")
        dx, dw = loss.backward(dloss, dweight=there.clone(), accumulate=True)
        _near(dx, want["dhidden"], "dhidden")
        _near(dw, want["dweight"], "dweight")


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n", [10, 200])
def test_results_that_lie_between_the_operands_rows(ctx, kind, n):
    """Column ranges of one matrix share nothing, whatever rows they have; one column more and they do."""
    t, vocab, dim = TYPES[kind], 300, 64
    g = torch.Generator(device=DEV).manual_seed(n)
    states, table = _normal(g, n, 3 * dim).to(t), _normal(g, vocab, 2 * dim, 0.2).to(t)
    x, w, dx, dw = states[:, :dim], table[:, dim:], states[:, dim:2 * dim], table[:, :dim]
    before = states[:, 2 * dim:].clone()
    targets, dloss = torch.randint(0, vocab, (n,), generator=g, device=DEV), torch.rand(n, generator=g, device=DEV)
    want = R.loss(x.clone(), w.clone(), targets, dloss=dloss)
    loss = P.VocabularyLoss(ctx, vocab, dim, n, t)
    _near(loss.cross_entropy(x, w, targets), want["losses"], "losses")
    for kw in (dict(dhidden=states[:, dim - 1:2 * dim - 1]), dict(dweight=table[:, 1:dim + 1]), dict(dhidden=table[:n, dim - 8:2 * dim - 8])):
        with pytest.raises(ValueError, match="overlaps"):
            loss.backward(dloss, **kw)
    loss.backward(dloss, dx, dw)
    _near(dx, want["dhidden"], "dhidden")
    _near(dw, want["dweight"], "dweight")
    assert torch.equal(states[:, 2 * dim:], before)


def test_results_that_overlap_what_is_read_are_refused(ctx):
    n, vocab, dim = 20, 300, 64
    g = torch.Generator(device=DEV).manual_seed(1)
    x, w, targets = _normal(g, n, dim), _normal(g, vocab, dim, 0.2), torch.randint(0, vocab, (n,), generator=g, device=DEV)
    tokens, logits, dloss = torch.randint(0, vocab, (n, 4), generator=g, device=DEV), _normal(g, n, 4), torch.ones(n, device=DEV)
    loss = P.VocabularyLoss(ctx, vocab, dim, n, torch.float32, top=4)
    for call in (lambda: loss.cross_entropy(x, w, targets, out=x.view(-1)[100:120]), lambda: loss.cross_entropy(x, w, targets, out=w.view(-1)[-20:]),
                 lambda: loss.distill(x, w, tokens, logits, out=logits.view(-1)[3:23]), lambda: loss.cross_entropy(x, w, targets, out=loss._state[:20])):
        with pytest.raises(ValueError, match="overlaps"):
            call()
    loss.cross_entropy(x, w, targets)
    with pytest.raises(ValueError, match="overlaps"):
        loss.backward(dloss, loss._space.view(torch.float32)[: n * dim].view(n, dim))
    many = torch.zeros(n * dim, device=DEV)
    with pytest.raises(ValueError, match="overlaps"):
        loss.backward(many[50:50 + n], many.view(n, dim))
    z = _normal(g, n, vocab)
    room = torch.zeros(n * 8, device=DEV)
    for kw in (dict(values=z.view(-1)[:n * 4].view(n, 4)), dict(lse=z[3, 5:5 + n]), dict(tokens=z.view(torch.int32).view(-1)[-n * 4:].view(n, 4)),
               dict(values=room[: n * 4].view(n, 4), lse=room[n * 4 - 1: n * 5 - 1])):
        with pytest.raises(ValueError, match="overlaps"):
            P.top_logits(ctx, z, 4, **kw)
    # side by side, between the rows, and operands that share memory
    held = _normal(g, n, vocab + 8)
    want = R.top(held[:, :vocab], 4)
    got = P.top_logits(ctx, held[:, :vocab], 4, values=room[: n * 4].view(n, 4), lse=room[n * 4: n * 5])
    assert torch.equal(got[0], want[0]) and torch.equal(room[: n * 4].view(n, 4), want[1])
    got = P.top_logits(ctx, held[:1, :vocab], 8, values=held.view(-1)[vocab: vocab + 8].view(1, 8))
    assert torch.equal(got[1], R.top(held[:1, :vocab], 8)[1])
    _near(loss.cross_entropy(w[5:5 + n], w, targets), R.loss(w[5:5 + n], w, targets)["losses"], "losses")


# floats of 17 to 64 rows by two fragments of a large vocabulary, few rows and a large weight; weights that are laid out a piece at a time in the forward pass, floats and rows at an odd distance
PIECES = [("f32", 24, 20000, 136, 0, None), ("f32", 50, 20001, 72, 0, None), ("f32", 17, 16400, 33, 1, None), ("f32", 70, 720_000, 40, 0, 699_136), ("f32", 130, 720_000, 8, 0, 699_136),
          ("bf16", 20, 2_098_000, 8, 1, 1 << 21), ("f16", 90, 2_098_000, 9, 0, 1 << 21), ("bf16", 16, 99_000, 512, 0, None), ("f16", 1, 99_000, 512, 0, None)]


@pytest.mark.parametrize("kind,n,vocab,dim,pad,border", PIECES)
def test_steps_of_few_rows_of_floats_and_of_weights_in_pieces(ctx, kind, n, vocab, dim, pad, border):
    """Targets and entries on both sides of the border between two pieces."""
    g, t = torch.Generator(device=DEV).manual_seed(n), TYPES[kind]
    x, w = _normal(g, n, dim + pad, 2.0).to(t)[:, :dim], _normal(g, vocab, dim + pad, 1.0 / math.sqrt(dim)).to(t)[:, :dim]
    targets, dloss = torch.randint(0, vocab, (n,), generator=g, device=DEV), torch.rand(n, generator=g, device=DEV)
    tokens = torch.randint(0, vocab, (n, 20), generator=g, device=DEV)
    if border is not None:
        targets[::3], targets[1::3] = border - 1, border
        tokens[1::2] = border - 10 + torch.arange(20, device=DEV)
        tokens[::5] = border - 1
    tokens[-1, 3:] = -1
    logits = _normal(g, n, 20, 3.0)
    loss = P.VocabularyLoss(ctx, vocab, dim, n, t, top=20)
    for teacher in ((targets,), (tokens, logits, 2.0)):
        losses = loss.cross_entropy(x, w, *teacher) if len(teacher) == 1 else loss.distill(x, w, *teacher)
        dx, dw = loss.backward(dloss)
        want = R.loss(x, w, *teacher, dloss=dloss)
        _near(losses, want["losses"], "losses")
        _near(dx, want["dhidden"], "dhidden")
        _near(dw, want["dweight"], "dweight")


@pytest.mark.parametrize("n", [5, 17, 64, 100, 128])
def test_gradients_in_fp32_of_few_rows_are_those_of_fp32(ctx, n):
    """One row with a gradient, one product in each logit, so dweight is p times dloss times a number.  Roundings on the way, of a logarithm of 30 terms below 8: its own
    2^-21, its sum 2^-22, the exponent 2^-22, times log(2); the exponential's and the terms' 2^-23 each, the product's 2^-24, four of sums 2^-24: below 1.3e-6 together.
    A dz of two bfloat16 is off by up to 2^-17 = 7.6e-6."""
    vocab = 30
    for seed in range(8):
        g = torch.Generator(device=DEV).manual_seed(seed)
        x, w = _normal(g, n, 1).bfloat16(), _normal(g, vocab, 1).bfloat16()
        targets, dloss = torch.zeros(n, dtype=torch.int64, device=DEV), torch.zeros(n, device=DEV)
        dloss[n // 2] = 1.0 + seed / 7
        loss = P.VocabularyLoss(ctx, vocab, 1, n, gradient_dtype=torch.float32)
        loss.cross_entropy(x, w, targets)
        _, dw = loss.backward(dloss)
        a = x[n // 2, 0].double()
        want = torch.softmax(a * w[:, 0].double(), dim=0) * a * dloss[n // 2].double()
        assert float(((dw[1:, 0].double() - want[1:]) / want[1:]).abs().max()) < 1.3e-6
