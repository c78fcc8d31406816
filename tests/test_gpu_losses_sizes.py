"""Losses over the vocabulary and top logits at the sizes where they take other kernels, split their work or pass 32 bits, on other streams and in graphs."""
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


def _rows(g, n, dim, dtype, sigma, pad=0):
    return torch.empty(n, dim + pad, device=DEV).normal_(0.0, sigma, generator=g).to(dtype)[:, :dim]


def _near(got, want, name):
    value, off = want
    wrong = ~((got.double() - value).abs() <= off)
    assert not bool(wrong.any()), "%s: %d of %d, e.g. %r for %r +- %r" % (
        name, int(wrong.sum()), wrong.numel(), got[wrong][0].item(), value[wrong][0].item(), off[wrong][0].item())


def _case(n, vocab, dim, t, seed=1, pad=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x, w = _rows(g, n, dim, t, 2.0, pad), _rows(g, vocab, dim, t, 1.0 / math.sqrt(dim), pad)
    targets = torch.randint(0, vocab, (n,), generator=g, device=DEV)
    targets[::7] = -100
    return x, w, targets, torch.empty(n, device=DEV).uniform_(0.5, 1.0, generator=g) / n


# each tile size, sums in parts, whole rounds of tiles and a rest, a vocabulary in pieces; few rows with a small and a large weight
SIZES = [("bf16", 16, 33000, 512, 0), ("bf16", 16, 33000, 512, 1), ("bf16", 3, 40000, 72, 0), ("f32", 9, 20000, 300, 0), ("f16", 40, 30000, 136, 0), ("bf16", 64, 20000, 264, 3),
         ("f16", 200, 9000, 1032, 0), ("bf16", 700, 3000, 640, 0), ("bf16", 2100, 40000, 64, 0), ("f16", 4096, 8300, 264, 0), ("f32", 600, 2000, 520, 0), ("f32", 4000, 30000, 40, 0),
         ("bf16", 5000, 60000, 40, 0), ("f32", 40, 3000, 1000, 2)]


@pytest.mark.parametrize("kind,n,vocab,dim,pad", SIZES)
def test_steps_of_every_plan(ctx, kind, n, vocab, dim, pad):
    t = TYPES[kind]
    x, w, targets, dloss = _case(n, vocab, dim, t, pad=pad)
    for to in {t, torch.float32}:
        want = R.loss(x, w, targets, dloss=dloss, parts=2 if to != t else 1)
        loss = P.VocabularyLoss(ctx, vocab, dim, n, t, gradient_dtype=to)
        _near(loss.cross_entropy(x, w, targets), want["losses"], "losses")
        dx, dw = loss.backward(dloss)
        _near(dx, want["dhidden"], "dhidden")
        _near(dw, want["dweight"], "dweight")


@pytest.mark.parametrize("kind,n,vocab,dim", [("bf16", 5, 40000, 512), ("bf16", 33, 20000, 200), ("f16", 300, 9000, 136), ("bf16", 2100, 33000, 64), ("f32", 500, 4000, 128), ("bf16", 700, 600, 64)])
def test_distillation_of_every_plan(ctx, kind, n, vocab, dim):
    """Entries all over the vocabulary, and crowded into a few tokens at either end of it."""
    t, top = TYPES[kind], 40
    x, w, _, dloss = _case(n, vocab, dim, t)
    g = torch.Generator(device=DEV).manual_seed(2)
    tokens = torch.randint(0, vocab, (n, top), generator=g, device=DEV)
    tokens[1::3] = vocab - 1 - torch.randint(0, 60, (len(tokens[1::3]), top), generator=g, device=DEV)
    tokens[2::3] = torch.randint(0, 300, (len(tokens[2::3]), top), generator=g, device=DEV)
    logits = torch.empty(n, top, device=DEV).normal_(0.0, 3.0, generator=g).to(t)
    want = R.loss(x, w, tokens, logits, 2.0, dloss)
    loss = P.VocabularyLoss(ctx, vocab, dim, n, t, top=top)
    _near(loss.distill(x, w, tokens, logits, 2.0), want["losses"], "losses")
    tokens.zero_()  # the backward pass has them in its state
    dx, dw = loss.backward(dloss)
    _near(dx, want["dhidden"], "dhidden")
    _near(dw, want["dweight"], "dweight")


def test_more_rows_than_go_at_a_time(ctx):
    """Rows whose stats do not fit the room for them go in groups; looked at are the first, the last and those at a border."""
    n, vocab, dim = 200_000, 90_000, 8
    x, w, targets, _ = _case(n, vocab, dim, torch.bfloat16)
    got = P.VocabularyLoss(ctx, vocab, dim, n, training=False).cross_entropy(x, w, targets, training=False)
    tokens = targets[:, None].contiguous()
    soft = P.VocabularyLoss(ctx, vocab, dim, n, training=False).distill(x, w, tokens, torch.zeros(n, 1, device=DEV), training=False)
    for at in range(0, n, n // 50):
        _near(got[at:at + 20], R.loss(x[at:at + 20], w, targets[at:at + 20])["losses"], "losses")
        _near(soft[at:at + 20], R.loss(x[at:at + 20], w, tokens[at:at + 20], torch.zeros(20, 1, device=DEV))["losses"], "losses")
    _near(got[-300:], R.loss(x[-300:], w, targets[-300:])["losses"], "losses")


def test_matrices_of_more_than_2_32_bytes(ctx):
    """Offsets that pass 32 bits: a weight and its gradient of 5 GB, logits of 5 GB."""
    n, vocab, dim = 20, 310_000, 8192
    x, w, targets, dloss = _case(n, vocab, dim, torch.bfloat16)
    targets[1:4] = vocab - 1 - torch.arange(3, device=DEV)
    loss = P.VocabularyLoss(ctx, vocab, dim, n)
    losses = loss.cross_entropy(x, w, targets)
    z = torch.cat([x.double() @ w[at:at + 20000].double().t() for at in range(0, vocab, 20000)], dim=1)
    lse, counts = torch.logsumexp(z, dim=1), targets >= 0
    want = torch.where(counts, lse - z.gather(1, targets.clamp(min=0)[:, None])[:, 0], 0.0)
    assert bool(((losses.double() - want).abs() <= 1e-3).all())  # sums of 8192 products of up to 2^-24 of |z| of up to 1000 each
    dx, dw = loss.backward(dloss)
    dz = torch.where(counts, dloss.double(), 0.0)[:, None] * torch.exp(z - lse[:, None])
    dz.scatter_add_(1, targets.clamp(min=0)[:, None], -torch.where(counts, dloss.double(), 0.0)[:, None])
    for at in (0, 100_000, 262_000, vocab - 1000):
        part = dz[:, at:at + 1000].t()
        # dz and the result are rounded to bfloat16 (2^-8 each), and the losses' differences reach 1e-3 of p
        off = 2.0 ** -8 * (part @ x.double()).abs() + (2.0 ** -8 + 2e-3) * (part.abs() @ x.double().abs()) + 1e-12
        assert bool(((dw[at:at + 1000].double() - part @ x.double()).abs() <= off).all())
    got, off = torch.zeros_like(dx, dtype=torch.float64), torch.zeros_like(dx, dtype=torch.float64)
    for at in range(0, vocab, 20000):
        got += dz[:, at:at + 20000] @ w[at:at + 20000].double()
        off += dz[:, at:at + 20000].abs() @ w[at:at + 20000].double().abs()
    assert bool(((dx.double() - got).abs() <= 2.0 ** -8 * got.abs() + (2.0 ** -8 + 2e-3) * off + 1e-12).all())
    del z, dz, dw, w, loss
    rows = torch.randn(20_000, 131_080, device=DEV, dtype=torch.bfloat16)
    tokens, values, lse = P.top_logits(ctx, rows, 5)
    want = R.top(rows[-50:], 5)
    assert torch.equal(tokens[-50:], want[0]) and torch.equal(values[-50:], want[1]) and bool(((lse[-50:].double() - want[2]).abs() < 1e-4).all())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,vocab,top", [(1, 400_000, 100), (600, 4097, 30), (600, 70_001, 150), (900, 33_000, 300), (1300, 5003, 8), (1300, 40_000, 192), (2000, 300, 192), (1100, 130, 130),
                                         (520, 131_072, 64), (1200, 17, 3)])
def test_top_logits_by_few_and_many_threads(ctx, n, vocab, top, kind):
    g = torch.Generator(device=DEV).manual_seed(n + top)
    x = _rows(g, n, vocab, TYPES[kind], 3.0, pad=vocab % 3)
    x[::5, torch.rand(vocab, generator=g, device=DEV) < 0.9] = -math.inf
    tokens, values, lse = P.top_logits(ctx, x, top)
    want = R.top(x, top)
    assert torch.equal(tokens, want[0]) and torch.equal(values, want[1])
    finite = want[2].isfinite()
    assert bool(((lse.double() - want[2]).abs() <= (vocab / 256 * 8 + 300) * 2.0 ** -24 * (1 + want[2].abs()))[finite].all()) and torch.equal(lse.isfinite(), finite)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,dim,pad", [(7, 72, 8), (7, 71, 9), (100, 72, 8), (100, 200, 56), (100, 71, 9), (100, 8, 8)])
def test_what_lies_between_rows_is_not_read_for_a_result(ctx, kind, n, dim, pad):
    """Rows that end within a block of the products, with NaN behind them; before and behind the matrices too."""
    t, vocab = TYPES[kind], 1500
    g = torch.Generator(device=DEV).manual_seed(4)

    def held(rows, sigma):
        whole = torch.full((rows + 2, dim + pad), math.nan, dtype=t, device=DEV)
        whole[1:-1, :dim] = torch.empty(rows, dim, device=DEV).normal_(0.0, sigma, generator=g).to(t)
        return whole, whole[1:-1, :dim]

    (_, x), (_, w) = held(n, 2.0), held(vocab, 0.2)
    targets = torch.randint(0, vocab, (n,), generator=g, device=DEV)
    dloss = torch.empty(n, device=DEV).uniform_(0.5, 1.0, generator=g)
    want = R.loss(x, w, targets, dloss=dloss)
    loss = P.VocabularyLoss(ctx, vocab, dim, n, t)
    _near(loss.cross_entropy(x, w, targets), want["losses"], "losses")
    (all_x, dx), (all_w, dw) = held(n, 1.0), held(vocab, 1.0)
    loss.backward(dloss, dx, dw)
    _near(dx, want["dhidden"], "dhidden")
    _near(dw, want["dweight"], "dweight")
    for whole in (all_x, all_w):
        assert bool(whole[0].isnan().all()) and bool(whole[-1].isnan().all()) and bool(whole[:, dim:].isnan().all())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n", [5, 40])
def test_tokens_whose_logits_are_minus_infinity(ctx, kind, n):
    """A bias of -infinity as a column of the weight takes tokens out: no probability, a loss of infinity where one is the target."""
    t, vocab, dim = TYPES[kind], 700, 40
    g = torch.Generator(device=DEV).manual_seed(6)
    x, w = _rows(g, n, dim, t, 2.0), _rows(g, vocab, dim, t, 0.2)
    x[:, -1] = 1.0
    w[:, -1] = 0.0
    gone = torch.arange(vocab, device=DEV) % 3 == 1
    w[gone, -1] = -math.inf
    targets = torch.randint(0, vocab // 3, (n,), generator=g, device=DEV) * 3
    targets[3] = 4
    got = P.VocabularyLoss(ctx, vocab, dim, n, t).cross_entropy(x, w, targets)
    assert float(got[3]) == math.inf
    kept = (~gone).nonzero()[:, 0]
    where = torch.searchsorted(kept, targets)
    rest = targets != 4
    want = R.loss(x[rest], w[kept], where[rest])["losses"]
    _near(got[rest], want, "losses")


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,threads", [(2, 1024), (1300, 256)])
def test_top_logits_that_are_in_a_few_threads_shares(ctx, n, threads, kind):
    """The largest 50 shares hold more than there is room for, their values all different or many the same; ties at the end of the row."""
    t, vocab, top = TYPES[kind], 200_003 if n == 2 else 30_003, 100
    x = torch.full((n, vocab), -100.0, dtype=t, device=DEV)
    share = torch.arange(vocab, device=DEV) // (16 // x.element_size()) % threads < 50
    count = int(share.sum())
    x[0, share] = torch.rand(count, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(t)
    x[1, share] = torch.arange(count, device=DEV).remainder(7).to(t)
    if n > 2:
        x[2, -60:] = 1.0
        x[3] = -math.inf
        x[3, -130:] = 2.0
        x[4, ::2] = math.nan
        x[5, 1::2] = 7.0
        x[6:] = torch.randint(0, 3, (n - 6, vocab), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).to(t)
    tokens, values, lse = P.top_logits(ctx, x, top)
    want = R.top(x, top)
    assert torch.equal(tokens, want[0]) and torch.equal(values.nan_to_num(nan=1e4), want[1].nan_to_num(nan=1e4))
    finite = want[2].isfinite()
    assert bool(((lse.double() - want[2]).abs() <= (vocab / 256 * 8 + 300) * 2.0 ** -24 * (1 + want[2].abs()))[finite].all()) and bool(lse[~finite].isnan().all())


# ---- fewer rows than it was made for, streams, graphs ------------------------------------------------------------------

def test_one_object_serves_all_numbers_of_rows(ctx):
    vocab, dim, most = 3000, 128, 700
    x, w, targets, dloss = _case(most, vocab, dim, torch.bfloat16)
    loss = P.VocabularyLoss(ctx, vocab, dim, most, gradient_dtype=torch.float32)
    for n in (most, 1, 16, 17, 64, 300, 0, most):
        want = R.loss(x[:n], w, targets[:n], dloss=dloss[:n], parts=2)
        _near(loss.cross_entropy(x[:n], w, targets[:n]), want["losses"], "losses")
        kept = loss.cross_entropy(x[:5], w, targets[:5], training=False)  # in between, without a backward pass
        assert torch.equal(kept, P.VocabularyLoss(ctx, vocab, dim, 5).cross_entropy(x[:5], w, targets[:5]))
        dx, dw = loss.backward(dloss[:n])
        _near(dx, want["dhidden"], "dhidden")
        _near(dw, want["dweight"], "dweight")


def test_sizes_of_zero(ctx):
    for n, vocab, dim in ((0, 10, 8), (5, 0, 8), (40, 0, 8), (5, 10, 0), (40, 10, 0), (0, 0, 0)):
        x, w = torch.zeros(n, dim, device=DEV), torch.zeros(vocab, dim, device=DEV)
        loss = P.VocabularyLoss(ctx, vocab, dim, n, torch.float32, top=2)
        targets = torch.zeros(n, dtype=torch.int64, device=DEV)
        losses = loss.cross_entropy(x, w, targets)
        want = math.log(vocab) if vocab else 0.0  # without a vocabulary every target is outside of it
        assert losses.shape == (n,) and bool(((losses - want).abs() <= 1e-6).all())
        dx, dw = loss.backward(torch.ones(n, device=DEV), torch.full_like(x, 7), torch.full_like(w, 7))
        assert bool((dx == 0).all()) and bool((dw == 0).all())
        _, dw = loss.backward(torch.ones(n, device=DEV), dweight=torch.full_like(w, 7), accumulate=True)
        assert bool((dw == 7).all()) or n
        soft = loss.distill(x, w, torch.zeros(n, 0, dtype=torch.int64, device=DEV), torch.zeros(n, 0, device=DEV))
        assert bool((soft == 0).all())
        dx, dw = loss.backward(torch.ones(n, device=DEV))
        assert bool((dx == 0).all()) and bool((dw == 0).all())
        P.cnr_poll_errors(ctx)


def test_another_stream_while_the_current_one_is_busy(ctx):
    n, vocab, dim, top = 300, 4000, 256, 8
    x, w, targets, dloss = _case(n, vocab, dim, torch.bfloat16)
    z = (x.float() @ w.float().t()).contiguous()
    want = P.VocabularyLoss(ctx, vocab, dim, n, top=top)
    losses = want.cross_entropy(x, w, targets)
    dx, dw = want.backward(dloss)
    tokens, values, lse = P.top_logits(ctx, z, top)
    soft = want.distill(x, w, tokens, values, 2.0)
    busy, side = torch.randn(4096, 4096, device=DEV), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        old = [torch.empty(t.numel(), dtype=t.dtype, device=DEV) for t in (dx, dw, losses, want._space, want._state, tokens, values, lse)]
        for _ in range(20):
            busy = (busy @ busy).clamp_(-1, 1)
        for t in old:
            t.fill_(7)
        del old, t
        loss = P.VocabularyLoss(ctx, vocab, dim, n, top=top)
        got = [loss.cross_entropy(x, w, targets, stream=side), *loss.backward(dloss, stream=side), *P.top_logits(ctx, z, top, stream=side)]
        got.append(loss.distill(x, w, got[3], got[4], 2.0, stream=side))
        torch.cuda.synchronize()
        for a, b in zip(got, (losses, dx, dw, tokens, values, lse, soft)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("kind,n,dim", [("bf16", 300, 256), ("f16", 9, 100), ("f32", 70, 64)])
def test_a_graph_replayed_gives_what_eager_calls_give(ctx, kind, n, dim):
    """Two graphs of one object, other inputs in the same memory before each replay, eager work in between."""
    vocab, top, t = 4000, 8, TYPES[kind]
    x, w, targets, dloss = _case(n, vocab, dim, t)
    z = torch.empty(n, vocab, device=DEV)
    loss, graphs, got = P.VocabularyLoss(ctx, vocab, dim, n, t, top=top), [], []

    def hard():
        return [loss.cross_entropy(x, w, targets), *loss.backward(dloss)]

    def soft():
        tokens, values, lse = P.top_logits(ctx, z, top)
        return [tokens, values, lse, loss.distill(x, w, tokens, values, 2.0), *loss.backward(dloss)]

    for call in (hard, soft):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got.append(call())
        graphs.append(graph)
    for seed in range(4):
        a, b, c, d = _case(n, vocab, dim, t, seed=seed)
        for to, new in ((x, a), (w, b), (targets, c), (dloss, d)):
            to.copy_(new)
        z.normal_(generator=torch.Generator(device=DEV).manual_seed(seed))
        wanted = [hard(), soft()]
        for i in (0, 1) if seed % 2 else (1, 0):
            for r in got[i]:
                r.zero_()
            graphs[i].replay()
            torch.cuda.synchronize()
            for r, v in zip(got[i], wanted[i]):
                assert torch.equal(r, v)


def test_results_that_overlap_are_refused(ctx):
    x, w, targets, dloss = _case(20, 300, 64, torch.float32)
    loss = P.VocabularyLoss(ctx, 300, 64, 20, torch.float32)
    loss.cross_entropy(x, w, targets)
    both = torch.zeros(320, 64, device=DEV)
    for kw in (dict(dhidden=x), dict(dweight=w), dict(dhidden=w[5:25]), dict(dhidden=both[290:310], dweight=both[:300])):
        with pytest.raises(ValueError, match="overlaps"):
            loss.backward(dloss, **kw)
    dx, dw = loss.backward(dloss, both[300:], both[:300])  # side by side is in order
    want = R.loss(x, w, targets, dloss=dloss)
    _near(dx, want["dhidden"], "dhidden")
    _near(dw, want["dweight"], "dweight")


def test_a_vocabulary_of_more_tokens_than_a_piece(ctx):
    n, vocab, dim = 20, (1 << 20) + 700, 8
    x, w, targets, dloss = _case(n, vocab, dim, torch.bfloat16)
    targets[0], targets[1] = vocab - 1, 1 << 20
    want = R.loss(x, w, targets, dloss=dloss, parts=2)
    loss = P.VocabularyLoss(ctx, vocab, dim, n, gradient_dtype=torch.float32)
    _near(loss.cross_entropy(x, w, targets), want["losses"], "losses")
    dx, dw = loss.backward(dloss)
    _near(dx, want["dhidden"], "dhidden")
    _near(dw, want["dweight"], "dweight")


def test_what_is_written_has_a_new_version(ctx):
    x, w, targets, dloss = _case(20, 300, 64, torch.float32)
    loss = P.VocabularyLoss(ctx, 300, 64, 20, torch.float32)
    out, dx, dw = torch.zeros(20, device=DEV), torch.zeros_like(x), torch.zeros_like(w)
    tokens, values, lse = torch.zeros(20, 4, dtype=torch.int32, device=DEV), torch.zeros(20, 4, device=DEV), torch.zeros(20, device=DEV)
    scale = torch.ones(20, device=DEV, requires_grad=True)
    saved = (scale * out).sum()
    written, read = (out, dx, dw, tokens, values, lse), (x, w, targets, dloss)
    before = [t._version for t in (*written, *read)]
    loss.cross_entropy(x, w, targets, out)
    loss.backward(dloss, dx, dw)
    P.top_logits(ctx, w[:20], 4, tokens, values, lse)
    after = [t._version for t in (*written, *read)]
    assert all(a > b for a, b in zip(after[:6], before)) and after[6:] == before[6:]
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        saved.backward()
