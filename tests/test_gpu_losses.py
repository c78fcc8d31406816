"""Losses over the vocabulary, their gradients and top logits on the GPU against 64 bits; bounds are those of oracle/losses.py."""
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


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _rows(g, n, dim, dtype, sigma, pad=0, offset=0):
    """n rows of dim normal values, dim + pad elements apart, the first `offset` elements into its memory."""
    x = torch.empty(offset + n * (dim + pad), device=DEV).normal_(0.0, sigma, generator=g).to(dtype)
    return x[offset:].view(n, dim + pad)[:, :dim]


def _near(got, want, name):
    value, off = want
    wrong = ~((got.double() - value).abs() <= off)
    assert not bool(wrong.any()), "%s: %d of %d, e.g. %r for %r +- %r" % (
        name, int(wrong.sum()), wrong.numel(), got[wrong][0].item(), value[wrong][0].item(), off[wrong][0].item())


def _targets(g, n, vocab, kind=torch.int64):
    t = torch.randint(0, vocab, (n,), generator=g, device=DEV)
    return torch.where(torch.rand(n, generator=g, device=DEV) < 0.2, -100, t).to(kind)


def _teacher(g, n, vocab, top, dtype, kind=torch.int64):
    """Tokens with repetitions and padding, one row in ten without any."""
    tokens = torch.randint(0, vocab, (n, top), generator=g, device=DEV)
    tokens = torch.where(torch.rand(n, top, generator=g, device=DEV) < 0.1, -1, tokens)
    tokens = torch.where(torch.rand(n, 1, generator=g, device=DEV) < 0.1, -5, tokens)
    return tokens.to(kind), torch.empty(n, top, device=DEV).normal_(0.0, 3.0, generator=g).to(dtype)


SIZES = [(1, 1, 1), (1, 1000, 64), (2, 63, 3), (16, 2049, 200), (17, 64, 128), (64, 65, 65), (65, 257, 31), (130, 1000, 128), (257, 2, 40), (300, 2049, 320),
         (129, 4097, 1)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,vocab,dim", SIZES)
def test_cross_entropy_and_its_gradients(ctx, n, vocab, dim, kind):
    g, t = _gen(n + vocab), TYPES[kind]
    x, w = _rows(g, n, dim, t, 2.0), _rows(g, vocab, dim, t, 1.0 / math.sqrt(dim))
    targets = _targets(g, n, vocab, torch.int32 if n % 2 else torch.int64)
    dloss = torch.empty(n, device=DEV).uniform_(-1.0, 1.0, generator=g)
    want = R.loss(x, w, targets, dloss=dloss)
    loss = P.VocabularyLoss(ctx, vocab, dim, n, t)
    _near(loss.cross_entropy(x, w, targets), want["losses"], "losses")
    dx, dw = loss.backward(dloss)
    _near(dx, want["dhidden"], "dhidden")
    _near(dw, want["dweight"], "dweight")
    assert P.cnr_poll_errors(ctx) == (P.CNR_OK, 0, 0)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,vocab,dim,top", [(1, 5, 4, 1), (3, 300, 64, 7), (33, 1000, 100, 64), (70, 1025, 128, 300), (200, 129, 48, 1024), (257, 3000, 256, 20)])
def test_distillation_and_its_gradients(ctx, n, vocab, dim, top, kind):
    g, t = _gen(n + top), TYPES[kind]
    x, w = _rows(g, n, dim, t, 2.0), _rows(g, vocab, dim, t, 1.0 / math.sqrt(dim))
    tokens, logits = _teacher(g, n, vocab, top, TYPES[["f32", "bf16", "f16"][n % 3]])
    dloss = torch.empty(n, device=DEV).uniform_(0.0, 1.0, generator=g)
    for temperature in (1.0, 3.0):
        want = R.loss(x, w, tokens, logits, temperature, dloss)
        loss = P.VocabularyLoss(ctx, vocab, dim, n, t, top=top)
        _near(loss.distill(x, w, tokens, logits, temperature), want["losses"], "losses")
        dx, dw = loss.backward(dloss)
        _near(dx, want["dhidden"], "dhidden")
        _near(dw, want["dweight"], "dweight")
    assert P.cnr_poll_errors(ctx) == (P.CNR_OK, 0, 0)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("grad", ["same", "f32"])
@pytest.mark.parametrize("n,vocab,dim", [(50, 500, 100), (300, 1000, 256)])
def test_gradients_onto_what_is_there(ctx, n, vocab, dim, kind, grad):
    """Strided operands that start anywhere, strided results, the weight's gradient added up in its own type or in fp32."""
    g, t = _gen(n), TYPES[kind]
    to = t if grad == "same" else torch.float32
    x, w = _rows(g, n, dim, t, 2.0, pad=3, offset=1), _rows(g, vocab, dim, t, 0.1, pad=5, offset=3)
    targets = _targets(g, n, vocab)
    dloss = torch.empty(n, device=DEV).uniform_(0.0, 1.0, generator=g)
    there = _rows(g, vocab, dim, to, 1.0, pad=7, offset=1)
    want = R.loss(x, w, targets, dloss=dloss, there=there.clone(), parts=2 if to != t else 1)
    around = there.as_strided((vocab, dim + 7), (dim + 7, 1))[:, dim:][:-1].clone()
    dx = torch.full((n, dim + 4), 7.0, dtype=t, device=DEV)
    loss = P.VocabularyLoss(ctx, vocab, dim, n + 100, t, gradient_dtype=to)
    _near(loss.cross_entropy(x, w, targets), want["losses"], "losses")
    got, dw = loss.backward(dloss, dx[:, :dim], there, accumulate=True)
    _near(got, want["dhidden"], "dhidden")
    _near(dw, want["dweight"], "dweight")
    assert dw.data_ptr() == there.data_ptr() and bool((dx[:, dim:] == 7.0).all())
    assert torch.equal(there.as_strided((vocab, dim + 7), (dim + 7, 1))[:, dim:][:-1], around)
    # one of the two alone is the same
    again = loss.backward(dloss, weight=False)
    assert again[1] is None and torch.equal(again[0], got)


@pytest.mark.parametrize("kind", list(TYPES))
def test_rows_that_are_left_out_reach_nothing(ctx, kind):
    """Padding, tokens outside the vocabulary and a dloss of 0, on rows that hold NaN and infinities; a whole batch of such rows."""
    t, n, vocab, dim = TYPES[kind], 96, 777, 64
    g = _gen(5)
    x, w = _rows(g, n, dim, t, 2.0), _rows(g, vocab, dim, t, 0.2)
    targets = torch.randint(0, vocab, (n,), generator=g, device=DEV)
    targets[::3] = -100
    targets[1::9] = vocab
    targets[4::9] = 1 << 40
    dloss = torch.empty(n, device=DEV).uniform_(0.5, 1.0, generator=g)
    dloss[2::6] = 0.0
    outside = int((targets >= vocab).sum())
    left_out = (targets < 0) | (targets >= vocab)
    clean = x.clone()
    x[left_out | (dloss == 0)] = math.nan
    x[::3] = math.inf
    clean[dloss == 0] = 0.0
    want = R.loss(clean, w, targets, dloss=dloss)
    dloss[left_out] = math.nan
    loss = P.VocabularyLoss(ctx, vocab, dim, n, t)
    losses = loss.cross_entropy(x, w, targets)
    counts = ~left_out & (dloss != 0)
    assert bool((losses[left_out] == 0).all()) and bool(losses[~left_out & (dloss == 0)].isnan().all())
    _near(losses[counts], tuple(v[counts] for v in want["losses"]), "losses")
    dx, dw = loss.backward(dloss)
    _near(dx, want["dhidden"], "dhidden")
    _near(dw, want["dweight"], "dweight")
    assert P.cnr_poll_errors(ctx) == (P.CNR_E_INDEX_RANGE, outside, 0)
    none = torch.full_like(targets, -1)
    assert bool((loss.cross_entropy(x, w, none) == 0).all())
    dx, dw = loss.backward(dloss)
    assert bool((dx == 0).all()) and bool((dw == 0).all())
    assert P.cnr_poll_errors(ctx) == (P.CNR_OK, 0, 0)


def test_a_teacher_without_logits_and_with_odd_ones(ctx):
    """-infinity everywhere leaves a row out, in places it is no probability; tokens outside the vocabulary are counted; NaN and infinity give NaN."""
    n, vocab, dim, top = 40, 300, 64, 6
    g = _gen(9)
    x, w = _rows(g, n, dim, torch.float32, 2.0), _rows(g, vocab, dim, torch.float32, 0.2)
    tokens = torch.randint(0, vocab, (n, top), generator=g, device=DEV)
    logits = torch.empty(n, top, device=DEV).normal_(generator=g)
    logits[0] = -math.inf
    logits[1, 2:] = -math.inf
    tokens[2, 1:4] = vocab + 3
    tokens[3] = 7  # one token, six times
    logits[2, 2] = math.nan  # where no token is
    logits[4, 5], logits[5, 0] = math.nan, math.inf
    loss = P.VocabularyLoss(ctx, vocab, dim, n, torch.float32, top=top)
    losses = loss.distill(x, w, tokens, logits, 2.0)
    assert float(losses[0]) == 0.0 and bool(losses[4:6].isnan().all())
    assert P.cnr_poll_errors(ctx) == (P.CNR_E_INDEX_RANGE, 3, 0)
    dloss = torch.ones(n, device=DEV)
    dloss[4:6] = 0.0  # what is NaN stays out of the sums
    tokens[4:6] = -1
    want = R.loss(x, w, tokens, logits, 2.0, dloss)
    rest = torch.arange(n, device=DEV) >= 6
    rest[:4] = True
    _near(losses[rest], tuple(v[rest] for v in want["losses"]), "losses")
    dx, dw = loss.backward(dloss)
    _near(dx, want["dhidden"], "dhidden")
    _near(dw, want["dweight"], "dweight")


def test_gradients_are_the_losses_differences(ctx):
    """Central differences of the losses along random directions, by the 64-bit definition and by the library's own losses."""
    n, vocab, dim, top = 24, 200, 32, 5
    g = _gen(3)
    x, w = _rows(g, n, dim, torch.float32, 1.0), _rows(g, vocab, dim, torch.float32, 0.3)
    tokens, logits = _teacher(g, n, vocab, top, torch.float32)
    dloss = torch.empty(n, device=DEV).uniform_(0.5, 1.0, generator=g)
    loss = P.VocabularyLoss(ctx, vocab, dim, n, torch.float32, top=top)
    loss.distill(x, w, tokens, logits, 1.5)
    dx, dw = loss.backward(dloss)
    along_x, along_w = _rows(g, n, dim, torch.float32, 1.0), _rows(g, vocab, dim, torch.float32, 1.0)
    slope = float((dx.double() * along_x).sum() + (dw.double() * along_w).sum())
    step = 2.0 ** -6

    def total(by, losses):
        return float((losses((x + by * along_x).float(), (w + by * along_w).float()).double() * dloss).sum())

    own = [total(by, lambda a, b: loss.distill(a, b, tokens, logits, 1.5, training=False)) for by in (step, -step, step / 2, -step / 2)]
    # Richardson's combination of two steps leaves an error of the fourth order, found from a third step by the definition
    exact = [total(by, lambda a, b: R.loss(a, b, tokens, logits, 1.5)["losses"][0]) for by in (step, -step, step / 2, -step / 2, step / 4, -step / 4)]

    def slopes(v):
        return [(v[2 * i] - v[2 * i + 1]) / (2 * step / 2 ** i) for i in range(len(v) // 2)]

    d = slopes(exact)
    coarse, fine = (4 * d[1] - d[0]) / 3, (4 * d[2] - d[1]) / 3
    assert abs(slope - fine) <= 2 * abs(fine - coarse) + 1e-5 * abs(fine)
    # each own loss is off by its bound at most
    off = float((R.loss(x, w, tokens, logits, 1.5)["losses"][1] * dloss).sum()) * 2 / step * 3
    d = slopes(own)
    assert abs((4 * d[1] - d[0]) / 3 - slope) <= 2 * abs(fine - coarse) + off + 1e-5 * abs(fine)


# ---- top logits -----------------------------------------------------------------------------------------------------

def _same(got, want, off=None):
    for a, b in zip(got[:2], want[:2]):
        assert torch.equal(torch.nan_to_num(a, nan=1e30) if a.is_floating_point() else a, torch.nan_to_num(b, nan=1e30) if b.is_floating_point() else b)
    if off is not None:
        finite = want[2].isfinite()
        assert torch.equal(got[2][~finite].double().nan_to_num(nan=5.0), want[2][~finite].nan_to_num(nan=5.0))
        assert bool(((got[2].double() - want[2]).abs() <= off * (1 + want[2].abs()))[finite].all())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,vocab,top,pad", [(1, 1, 1, 0), (1, 50257, 50, 0), (3, 7, 20, 1), (2, 4096, 1024, 0), (5, 5000, 1000, 3), (70, 32000, 64, 0), (9, 131073, 256, 5),
                                             (4, 300001, 7, 0), (3, 1023, 0, 0)])
def test_top_logits(ctx, n, vocab, top, pad, kind):
    x = _rows(_gen(n), n, vocab, TYPES[kind], 4.0, pad=pad, offset=pad)
    # a sum of vocab exponentials: a few roundings for each of at most vocab / 1024 steps of a thread and of the joins, each exponential off by
    # 2^-22 and the rounding of its argument, of up to 40
    _same(P.top_logits(ctx, x, top), R.top(x, top), (vocab / 1024 * 8 + 300) * 2.0 ** -24)


@pytest.mark.parametrize("kind", list(TYPES))
def test_top_logits_of_rows_with_ties_masks_and_odd_values(ctx, kind):
    t, vocab, top = TYPES[kind], 20000, 100
    g = _gen(1)
    x = _rows(g, 16, vocab, t, 1.0)
    x[0] = -math.inf
    x[1] = -math.inf
    x[1, 7777] = 1.0
    x[2] = 3.0
    x[3] = torch.randint(0, 3, (vocab,), generator=g, device=DEV).to(t)
    x[4, ::1000] = math.nan
    x[5, 5::1000] = math.inf
    x[6] = torch.arange(vocab, device=DEV).float().div(vocab).to(t)  # ascending
    x[7] = -x[6]
    x[8] = -0.0
    x[8, ::2] = 0.0
    x[9] = torch.finfo(t).min
    x[10, 1024 * 4: 1024 * 4 + 4] = 50.0
    x[11] = -math.inf
    x[11, -50:] = 1.0
    x[12] = -100.0
    share = torch.arange(vocab, device=DEV) // (16 // x.element_size()) % 1024 == 3  # all in one thread's share
    x[12, share] = torch.arange(int(share.sum()), device=DEV).to(t)
    x[13, : vocab // 2] = math.nan
    x[14] = torch.finfo(t).max
    x[15] = -math.nan
    _same(P.top_logits(ctx, x, top), R.top(x, top), (vocab / 1024 * 8 + 300) * 2.0 ** -24)


def test_top_logits_written_to_given_rooms(ctx):
    x = _rows(_gen(2), 5, 900, torch.bfloat16, 1.0)
    tokens, values, lse = torch.full((6, 8), 9, dtype=torch.int32, device=DEV), torch.full((6, 8), 9.0, dtype=torch.bfloat16, device=DEV), torch.full((6,), 9.0, device=DEV)
    P.top_logits(ctx, x, 8, tokens, values, lse)
    want = R.top(x, 8)
    _same((tokens[:5], values[:5]), want)
    assert bool((tokens[5] == 9).all()) and bool((values[5] == 9).all()) and float(lse[5]) == 9.0
    P.cnr_top_logits(ctx, x, 8, tokens=None, values=None, lse=lse)
    P.cnr_top_logits(ctx, x, 8, tokens=tokens)
    _same((tokens[:5], values[:5]), want)
    empty = P.top_logits(ctx, x[:, :0], 2)
    assert bool((empty[0] == -1).all()) and bool((empty[1] == -math.inf).all()) and bool((empty[2] == -math.inf).all())
    assert P.top_logits(ctx, x[:0], 3)[0].shape == (0, 3)


# ---- together -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_a_student_learns_from_a_teachers_top_logits(ctx, kind):
    """The teacher's logits by the block product, its top logits, the student's distillation and cross entropy onto one gradient."""
    t, n, vocab, dim, top = TYPES[kind], 200, 1500, 128, 16
    g = _gen(8)
    hidden, matrix = _rows(g, n, dim, torch.float32, 1.0), P.BlockMatrix.empty(vocab, dim, P.CNR_BLOCK_TILE)
    P.quantize_blocks(ctx, _rows(g, vocab, dim, torch.float32, 0.2), matrix)
    teacher = P.block_product(ctx, P.quantize_blocks(ctx, hidden), matrix, torch.empty(n, vocab, device=DEV))
    tokens, logits, lse = P.top_logits(ctx, teacher, top)
    _same((tokens, logits), R.top(teacher, top))
    assert bool((torch.exp(logits - lse[:, None]).sum(dim=1) <= 1.0 + 1e-5).all())
    x, w = _rows(g, n, dim, t, 1.0), _rows(g, vocab, dim, t, 0.2)
    targets, dloss = _targets(g, n, vocab), torch.full((n,), 1.0 / n, device=DEV)
    loss = P.VocabularyLoss(ctx, vocab, dim, n, t, top=top, gradient_dtype=torch.float32)
    soft = R.loss(x, w, tokens, logits, 2.0, 4.0 * dloss, parts=2 if kind != "f32" else 1)
    _near(loss.distill(x, w, tokens, logits, 2.0), soft["losses"], "losses")
    dx, dw = loss.backward(4.0 * dloss)
    _near(dx, soft["dhidden"], "dhidden")
    _near(dw, soft["dweight"], "dweight")
    hard = R.loss(x, w, targets, dloss=dloss, there=dw.clone(), parts=2 if kind != "f32" else 1)
    _near(loss.cross_entropy(x, w, targets), hard["losses"], "losses")
    dx, dw = loss.backward(dloss, dweight=dw, accumulate=True)
    _near(dx, hard["dhidden"], "dhidden")
    _near(dw, hard["dweight"], "dweight")
