"""The operators for language models against their definitions in 64 bits (oracle/blocks.py)."""
import numpy as np
import pytest
import torch

import paper_2010_08679_amd as P
from oracle import blocks as R
from paper_2010_08679_amd import lm_binding as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
KIND = {"row": P.CNR_BLOCK_ROW, "tile": P.CNR_BLOCK_TILE}
SCALE = {"e8m0": P.CNR_SCALE_E8M0, "f32": P.CNR_SCALE_F32}


@pytest.fixture(scope="module")
def ctx():
    c = P.cnr_create(0)
    yield c
    torch.cuda.synchronize()
    P.cnr_destroy(c)


def _wide(t):
    return t.detach().cpu().double().numpy()


def _scale64(scale):
    s = scale.cpu().numpy()
    return np.ldexp(1.0, s.astype(np.int64) - 127) if s.dtype == np.uint8 else s.astype(np.float64)


def _blocked(codes, s, kind, scale):
    """A BlockMatrix of these codes and 64-bit scales [block][row or tile]; what belongs to no row is filled with rubbish."""
    m = P.BlockMatrix.empty(codes.shape[0], codes.shape[1], KIND[kind], SCALE[scale])
    m.codes.copy_(torch.from_numpy(codes))
    held = np.full(tuple(m.scale.shape), 250 if scale == "e8m0" else np.nan)
    held[:, : s.shape[1]] = np.log2(s) + 127 if scale == "e8m0" else s
    m.scale.copy_(torch.from_numpy(held).to(m.scale.dtype))
    return m


def _same_codes(got, want):
    """A NaN may be either of its two codes."""
    nan = (want & 127) == 127
    assert np.array_equal((got & 127) == 127, nan)
    assert np.array_equal(got[~nan], want[~nan])


# ---- quantization ---------------------------------------------------------------------------------------------------

def _input(rows, dim, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, dim, generator=g)
    x *= torch.exp2(torch.randint(-12, 12, (rows, 1), generator=g).float())
    x *= torch.exp2(torch.randint(-6, 6, (1, dim), generator=g).float())
    return x.to(dtype)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind", ["row", "tile"])
@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("rows,dim,pad", [(1, 1, 0), (1, 128, 0), (5, 127, 1), (16, 256, 0), (128, 128, 8), (129, 257, 0), (300, 1000, 13), (700, 136, 0)])
def test_quantize_equals_the_definition(ctx, type, kind, scale, rows, dim, pad):
    whole = torch.full((rows, dim + pad), 3e4, dtype=TYPES[type])  # what lies between rows must not count
    whole[:, :dim] = _input(rows, dim, TYPES[type], 7 * rows + dim)
    x = whole.to(DEV)[:, :dim]
    out = P.BlockMatrix.empty(rows, dim, KIND[kind], SCALE[scale])
    out_t = P.BlockMatrix.empty(dim, rows, KIND[kind], SCALE[scale])
    alone = P.BlockMatrix.empty(rows, dim, KIND[kind], SCALE[scale])
    alone_t = P.BlockMatrix.empty(dim, rows, KIND[kind], SCALE[scale])
    for m in (out, out_t, alone, alone_t):
        m.codes.fill_(0x55)
    P.quantize_blocks(ctx, x, out, out_t)
    P.quantize_blocks(ctx, x, alone)
    P.quantize_blocks(ctx, x, None, alone_t)
    for m, y in ((out, _wide(x)), (alone, _wide(x)), (out_t, _wide(x).T), (alone_t, _wide(x).T)):
        codes, s = R.quantize(y, kind, scale)
        assert np.array_equal(_scale64(m.scale)[:, : s.shape[1]], s)
        _same_codes(m.codes.cpu().numpy(), codes)


def _special(dtype):
    """Rows that a scale or a rounding could get wrong."""
    big, small = torch.finfo(dtype).max, torch.finfo(dtype).tiny
    rows = [torch.zeros(128), torch.full((128,), big), torch.full((128,), small / 4), torch.linspace(-448, 448, 128),
            torch.tensor(R.E4M3[:127].tolist() + [0.0]), torch.tensor([448.0] + ((R.E4M3[1:127] + R.E4M3[:126]) / 2).tolist() + [0.0]),
            torch.tensor([1.75] + [0.25] * 127), torch.tensor([float(np.nextafter(np.float32(1.75), np.float32(2)))] + [0.25] * 127),
            torch.full((128,), -0.0), torch.randn(128, generator=torch.Generator().manual_seed(3)) * small]
    with_odd = torch.randn(128, generator=torch.Generator().manual_seed(4))
    for i, v in enumerate((float("inf"), float("-inf"), float("nan"), -float("nan"))):
        with_odd[20 * i + 3] = v
    rows += [with_odd, torch.full((128,), float("nan")), torch.full((128,), float("inf"))]
    return torch.stack([r.double() for r in rows]).to(dtype)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("scale", ["e8m0", "f32"])
def test_quantize_special_values(ctx, type, scale):
    x = _special(TYPES[type])
    # every row as a block of its own, as a column of the transpose's blocks, and as a tile
    out = P.quantize_blocks(ctx, x.to(DEV), P.BlockMatrix.empty(len(x), 128, P.CNR_BLOCK_ROW, SCALE[scale]))
    codes, s = R.quantize(_wide(x), "row", scale)
    assert np.array_equal(_scale64(out.scale)[:, : len(x)], s)
    _same_codes(out.codes.cpu().numpy(), codes)
    turned = P.BlockMatrix.empty(len(x), 128, P.CNR_BLOCK_ROW, SCALE[scale])
    P.quantize_blocks(ctx, x.t().contiguous().to(DEV), None, turned)
    assert np.array_equal(_scale64(turned.scale)[:, : len(x)], s)
    _same_codes(turned.codes.cpu().numpy(), codes)
    for i in range(len(x)):
        tile = x[i:i + 1].to(DEV)
        m = P.quantize_blocks(ctx, tile, P.BlockMatrix.empty(1, 128, P.CNR_BLOCK_TILE, SCALE[scale]))
        _same_codes(m.codes.cpu().numpy(), codes[i:i + 1])
        assert _scale64(m.scale)[0, 0] == s[0, i]


def test_quantize_next_to_the_middle_of_two_codes(ctx):
    # fp32 values within a few steps of every middle between two codes, at scales whose quotients are not exact
    g = torch.Generator().manual_seed(11)
    rows = []
    for _ in range(64):
        top = float(torch.rand(1, generator=g)) * 3 + 0.01
        s = np.float64(np.float32(np.float64(np.float32(top)) / 448.0))
        mid = ((R.E4M3[1:127] + R.E4M3[:126]) / 2) * s
        v = np.float32(mid)
        for _ in range(int(torch.randint(0, 3, (1,), generator=g))):
            v = np.nextafter(v, np.float32(0 if torch.rand(1, generator=g) < 0.5 else 10))
        rows.append(np.concatenate([[np.float32(top)], v, [np.float32(0)]]).astype(np.float32))
    x = torch.from_numpy(np.stack(rows))
    out = P.quantize_blocks(ctx, x.to(DEV), P.BlockMatrix.empty(64, 128, P.CNR_BLOCK_ROW, P.CNR_SCALE_F32))
    codes, _ = R.quantize(_wide(x), "row", "f32")
    assert np.array_equal(out.codes.cpu().numpy(), codes)


def test_quantize_nothing(ctx):
    for rows, dim in ((0, 128), (5, 0), (0, 0)):
        out = P.BlockMatrix.empty(rows, dim)
        P.quantize_blocks(ctx, torch.zeros(rows, dim, device=DEV), out)
    torch.cuda.synchronize()


# ---- products -------------------------------------------------------------------------------------------------------

def _operand(rows, k, kind, scale, seed, exact=False):
    """Codes with rows of whole blocks and scales [block][row or tile]; `exact`: small whole numbers and scales that leave sums exact."""
    g = np.random.default_rng(seed)
    blocks = -(-k // 128)
    codes = np.zeros((rows, blocks * 128), dtype=np.uint8)
    if exact:
        codes[:, :k] = R.encode(g.integers(-4, 5, (rows, k)).astype(np.float64))
        e = g.integers(-1, 2, (blocks, rows if kind == "row" else -(-rows // 128)))
        return codes, 2.0 ** e
    codes[:, :k] = R.encode(np.clip(g.normal(0, 100, (rows, k)), -448, 448))
    e = g.uniform(-10, 3, (blocks, rows if kind == "row" else -(-rows // 128)))
    return codes, 2.0 ** np.round(e) if scale == "e8m0" else (2.0 ** e).astype(np.float32).astype(np.float64)


def _check(got, want, sums, out, k):
    """`sums`: of the products' magnitudes.  A result is rounded by at most half a step; the fp32 sum of k products is off by at most
    k + 128 roundings of 2^-23 of those sums (the scales' roundings among them); the 8-bit instructions drop less than 2^-13 of the largest of eight
    products for each of the other seven."""
    bound = torch.finfo(TYPES[out]).eps / 2 * np.abs(want) + (k + 128) * 2.0 ** -23 * sums + (0 if out == "f32" else 7 * 2.0 ** -13 * sums)
    if out == "f16":
        bound += 2.0 ** -25  # half a step of the smallest values
    assert got.shape == want.shape
    top = float(torch.finfo(TYPES[out]).max)
    over = np.abs(want) + bound > top  # beyond the type, or so near that it may round to infinity
    assert np.all((np.abs(got) >= np.minimum(np.abs(want) - bound, top))[over] & (np.sign(got[over]) == np.sign(want[over])))
    assert np.all(np.abs(got - want)[~over] <= bound[~over]), float(np.max((np.abs(got - want) - bound)[~over]))


SIZES = [(1, 1, 1), (1, 16, 128), (3, 50, 127), (16, 16, 129), (1, 1000, 2048), (7, 257, 640), (33, 130, 384), (64, 640, 1100),
         (65, 96, 300), (100, 200, 4096), (128, 128, 128), (129, 300, 257), (256, 256, 512), (300, 513, 900), (515, 770, 130)]


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_product_equals_the_definition(ctx, out, scale, m, n, k):
    for a_kind, b_kind in (("row", "tile"), ("row", "row"), ("tile", "row"), ("tile", "tile")):
        (ca, sa), (cb, sb) = _operand(m, k, a_kind, scale, m + n), _operand(n, k, b_kind, scale, n + k)
        a, b = R.values(ca, sa, a_kind), R.values(cb, sb, b_kind)
        if out == "f16":  # keep results in range
            sa = sa / 256
            a = a / 256
        want, sums = a @ b.T, np.abs(a) @ np.abs(b).T
        x, y = _blocked(ca, sa, a_kind, scale), _blocked(cb, sb, b_kind, scale)
        got = torch.full((m, n), 7.0, dtype=TYPES[out], device=DEV)
        P.block_product(ctx, x, y, got, workspace=P.block_workspace(ctx, m, n, k))
        _check(_wide(got), want, sums, out, k)
        again = torch.full((m, n + 3), 7.0, dtype=TYPES[out], device=DEV)  # rows further apart, what lies between them kept; no workspace
        P.block_product(ctx, x, y, again[:, :n])
        _check(_wide(again[:, :n]), want, sums, out, k)
        assert bool((again[:, n:] == 7.0).all())


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("m,n,k", [(1, 33, 700), (20, 300, 384), (64, 64, 64), (150, 260, 140), (260, 520, 256), (64, 64, 2100)])
def test_product_of_whole_numbers_is_exact_and_added(ctx, out, scale, m, n, k):
    # sums of small whole numbers need no rounding before the last one; accumulated onto whole numbers as well
    (ca, sa), (cb, sb) = _operand(m, k, "row", scale, 5, True), _operand(n, k, "tile", scale, 6, True)
    want = R.values(ca, sa, "row") @ R.values(cb, sb, "tile").T
    x, y = _blocked(ca, sa, "row", scale), _blocked(cb, sb, "tile", scale)
    start = np.random.default_rng(2).integers(-9, 10, (m, n)).astype(np.float64)
    to = torch.from_numpy(start).to(TYPES[out]).to(DEV)
    space = P.block_workspace(ctx, m, n, k)
    P.block_product(ctx, x, y, to, accumulate=True, workspace=space)
    rounded = torch.from_numpy(want + start).to(torch.float32).to(TYPES[out])
    assert torch.equal(to.cpu(), rounded)
    P.block_product(ctx, x, y, to, workspace=space)
    assert torch.equal(to.cpu(), torch.from_numpy(want).to(torch.float32).to(TYPES[out]))


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(20, 40), (200, 300)])
def test_product_nan_stays_in_its_row_and_column(ctx, out, m, n):
    k = 300
    (ca, sa), (cb, sb) = _operand(m, k, "row", "e8m0", 1), _operand(n, k, "row", "e8m0", 2)
    ca[m - 1, 5] = 0x7f
    cb[3, 290] = 0xff
    want = R.values(ca, sa, "row") @ R.values(cb, sb, "row").T
    got = _wide(P.block_product(ctx, _blocked(ca, sa, "row", "e8m0"), _blocked(cb, sb, "row", "e8m0"), torch.empty(m, n, dtype=TYPES[out], device=DEV)))
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(want).sum() == m + n - 1


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m", [3, 200])
def test_product_of_extreme_scales(ctx, out, m):
    # the smallest and the largest scales against each other, and a large scale of a block that is zero
    n, k = 140, 256
    for scale, low, high in (("e8m0", 2.0 ** -120, 2.0 ** 118), ("f32", 2.0 ** -100, 1.5 * 2.0 ** 110)):
        (ca, _), (cb, _) = _operand(m, k, "row", scale, 1, True), _operand(n, k, "row", scale, 2, True)
        ca[:, 128:] = 0
        sa, sb = np.full((2, m), low), np.full((2, n), high)
        sa[1] = high
        want = R.values(ca, sa, "row") @ R.values(cb, sb, "row").T
        got = _wide(P.block_product(ctx, _blocked(ca, sa, "row", scale), _blocked(cb, sb, "row", scale), torch.empty(m, n, dtype=TYPES[out], device=DEV)))
        assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want))


def test_product_of_nothing(ctx):
    for m, n, k in ((0, 5, 128), (5, 0, 128), (0, 0, 0)):
        P.block_product(ctx, P.BlockMatrix.empty(m, k), P.BlockMatrix.empty(n, k), torch.empty(m, n, device=DEV))
    out = torch.full((5, 6), 3.0, device=DEV)
    P.block_product(ctx, P.BlockMatrix.empty(5, 0), P.BlockMatrix.empty(6, 0), out, accumulate=True)
    assert bool((out == 3.0).all())
    P.block_product(ctx, P.BlockMatrix.empty(5, 0), P.BlockMatrix.empty(6, 0), out)
    assert bool((out == 0.0).all())


# ---- the layer ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("tokens,n_in,n_out", [(1, 64, 48), (130, 200, 257), (300, 128, 384), (70, 513, 100)])
@pytest.mark.parametrize("type", ["f32", "bf16"])
@pytest.mark.parametrize("scale", ["e8m0", "f32"])
def test_linear_layer_and_its_gradients(ctx, tokens, n_in, n_out, type, scale):
    layer = P.BlockLinear(ctx, n_out, n_in, 300, SCALE[scale])
    w, x, dy = _input(n_out, n_in, torch.float32, 1), _input(tokens, n_in, TYPES[type], 2), _input(tokens, n_out, TYPES[type], 3)
    layer.load(w.to(DEV))
    y = layer.forward(x.to(DEV))
    dx, dw = layer.backward(dy.to(DEV))
    start = dw.clone()
    layer.backward(dy.to(DEV), dx, dw, accumulate=True)

    def q(m, kind):
        return R.values(*R.quantize(_wide(m), kind, scale), kind)[:, : m.shape[1]]

    wq = q(w, "tile")
    for got, a, b, t, k in ((y, q(x, "row"), wq, type, n_in), (dx, q(dy, "row"), wq.T, type, n_out),
                            (dw, None, None, "f32", tokens), (start, q(dy.t(), "row"), q(x.t(), "row"), "f32", tokens)):
        if a is None:  # added to itself
            assert torch.equal(got, start + start)
        else:
            _check(_wide(got), a @ b.T, np.abs(a) @ np.abs(b).T, t, k)


def test_linear_gradients_against_differences(ctx):
    # values that 8 bits hold exactly, before and after a step of each input: the loss <y, dy> is then linear in each and the
    # difference is the derivative
    g = np.random.default_rng(3)
    tokens, n_in, n_out = 40, 72, 56
    w, x, dy = (torch.from_numpy(g.integers(-3, 4, s).astype(np.float32)) for s in ((n_out, n_in), (tokens, n_in), (tokens, n_out)))
    layer = P.BlockLinear(ctx, n_out, n_in, tokens)

    def loss(w, x):
        layer.load(w.to(DEV))
        return float((_wide(layer.forward(x.to(DEV))) * _wide(dy)).sum())

    base = loss(w, x)
    dx, dw = layer.backward(dy.to(DEV))
    for i, j in ((0, 0), (7, 71), (39, 30)):
        up = x.clone()
        up[i, j] += 1
        assert loss(w, up) - base == float(dx[i, j])
    for i, j in ((0, 0), (55, 71), (20, 33)):
        up = w.clone()
        up[i, j] += 1
        assert loss(up, x) - base == float(dw[i, j])


# ---- tokens -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("vocab", [1, 31, 32, 300, 5003])
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_count_equals_the_definition(ctx, vocab, index):
    g = np.random.default_rng(vocab)
    n_slots, n = 9, 7
    ledger = P.TokenLedger(ctx, n_slots, vocab)
    seen, counts = np.zeros((n_slots, vocab), bool), np.zeros((n_slots, vocab), np.int64)
    bad = 0
    for step, (lengths, prompt, restart) in enumerate([((0, 900, 1, 0, 257, 2, 64), True, True), ((1,) * n, False, False), ((3, 0, 5, 1000, 0, 1, 0), False, False),
                                                       ((2, 0, 0, 1, 300, 0, 9), False, True), ((1,) * n, False, False)]):
        slots = g.permutation(n_slots)[:n].astype(np.int32)
        if step == 2:
            slots[1] = slots[0]  # two sequences share a slot
        offsets = np.concatenate([[0], np.cumsum(lengths)])
        tokens = np.minimum(g.zipf(1.3, offsets[-1]) - 1, vocab + 1) - (g.random(offsets[-1]) < 0.05) * 100_000  # some are padding or beyond
        each = all(v == 1 for v in lengths)
        ledger.count(torch.from_numpy(tokens).to(index).to(DEV), None if each else torch.from_numpy(offsets.astype(np.int64)).to(DEV),
                     torch.from_numpy(slots).to(DEV), prompt=prompt, restart=restart)
        R.count(seen, counts, vocab, tokens, offsets, slots, prompt, restart)
        bad += int(((tokens < 0) | (tokens >= vocab)).sum())
        assert np.array_equal(ledger.counts.cpu().numpy(), counts)
        assert np.array_equal(ledger.seen.cpu().numpy(), R.pack_bits(seen))
    st, n_bad, flags = P.cnr_poll_errors(ctx)
    assert (n_bad, flags) == (bad, 0)


def test_count_skips_slots_that_there_are_not(ctx):
    ledger = P.TokenLedger(ctx, 2, 50)
    before = ledger.counts.clone()
    ledger.count(torch.tensor([3, 4, 5], device=DEV), None, torch.tensor([2, -1, 1], dtype=torch.int32, device=DEV), restart=True)
    st, n_bad, flags = P.cnr_poll_errors(ctx)
    assert st == P.CNR_E_ROW_ID and flags == P.CNR_FLAG_ROW_ID
    before[1, 5] = 1
    assert torch.equal(ledger.counts, before)
    # offsets that reach beyond the tokens; no sequences; no tokens
    ledger.count(torch.tensor([7, 8], device=DEV), torch.tensor([0, 1, 90], device=DEV))
    ledger.count(torch.empty(0, dtype=torch.int64, device=DEV))
    ledger.count(torch.empty(0, dtype=torch.int64, device=DEV), torch.tensor([0, 0], device=DEV))
    before[0, 7] = before[1, 8] = 1
    assert torch.equal(ledger.counts, before)
    assert P.cnr_poll_errors(ctx) == (P.CNR_OK, 0, 0)


def _adjust_case(n, vocab, dtype, seed):
    g = np.random.default_rng(seed)
    logits = torch.from_numpy(g.normal(0, 5, (n, vocab))).to(dtype)
    logits[:, :: 7] = 0.0
    logits[0, : min(vocab, 6)] = torch.tensor([float("inf"), float("-inf"), float("nan"), torch.finfo(dtype).min, torch.finfo(dtype).max, -0.0])[: min(vocab, 6)].to(dtype)
    slots = n + 2
    counts = g.integers(0, 4, (slots, vocab)) * (g.random((slots, vocab)) < 0.3)
    seen = (counts > 0) | (g.random((slots, vocab)) < 0.2)
    per = [np.sort(g.permutation(vocab)[: g.integers(0, min(vocab, k) + 1)]) for k in ([1, 40, vocab] * n)[:n]]
    values = [g.normal(0, 3, len(p)).astype(np.float32) for p in per]
    for v in values:
        v[: 1] = -np.inf
    masks = g.random((n + 1, vocab)) < g.random((n + 1, 1))
    masks[1] = False  # a grammar that allows nothing
    return dict(logits=logits, counts=counts, seen=seen, which=g.permutation(slots)[:n].astype(np.int32), per=per, values=values, masks=masks,
                mask_of=g.integers(-1, n + 1, n).astype(np.int32), rep=(1 + g.random(n)).astype(np.float32), freq=g.normal(0, 1, n).astype(np.float32),
                pres=g.normal(0, 1, n).astype(np.float32))


def _close(got, want, dtype, size):
    """Six fp32 operations, each off by half a step of a value no larger than `size`, and one rounding to the type."""
    got = _wide(got)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    top = float(torch.finfo(dtype).max)
    fine = np.isfinite(want) & (np.abs(want) <= top)
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    over = np.isfinite(want) & ~fine  # beyond the type: the largest value or infinity, by how it rounds
    assert np.all((np.abs(got[over]) >= top) & (np.sign(got[over]) == np.sign(want[over])))
    bound = torch.finfo(dtype).eps / 2 * np.abs(want[fine]) + 6 * 2.0 ** -24 * size[fine] + float(torch.finfo(dtype).tiny) * torch.finfo(dtype).eps / 2
    assert np.all(np.abs(got[fine] - want[fine]) <= bound)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,vocab,pad", [(1, 1, 0), (2, 7, 0), (1, 32, 0), (3, 33, 5), (5, 2047, 1), (4, 2048, 0), (2, 2049, 0), (3, 9001, 0)])
@pytest.mark.parametrize("what", ["all", "penalties", "bias", "masks", "nothing"])
def test_adjust_equals_the_definition(ctx, type, n, vocab, pad, what):
    dtype = TYPES[type]
    c = _adjust_case(n, vocab, dtype, 31 * n + vocab)
    ledger = P.TokenLedger(ctx, n + 2, vocab, seen=torch.from_numpy(R.pack_bits(c["seen"])).to(DEV), counts=torch.from_numpy(c["counts"].astype(np.int32)).to(DEV))
    held = torch.full((n, vocab + pad), 9.0, dtype=dtype, device=DEV)
    held[:, :vocab] = c["logits"].to(DEV)
    given, want = {}, {}
    if what in ("all", "penalties"):
        given |= {k: torch.from_numpy(c[s]).to(DEV) for k, s in (("repetition", "rep"), ("frequency", "freq"), ("presence", "pres"), ("slots", "which"))}
        want |= dict(seen=c["seen"][c["which"]], counts=c["counts"][c["which"]], repetition=c["rep"], frequency=c["freq"], presence=c["pres"])
    if what in ("all", "bias"):
        offsets = np.concatenate([[0], np.cumsum([len(p) for p in c["per"]])])
        given["bias"] = tuple(torch.from_numpy(v).to(DEV) for v in (offsets.astype(np.int64), np.concatenate(c["per"]).astype(np.int32),
                                                                      np.concatenate(c["values"]).astype(np.float32)))
        want["biases"] = [list(zip(p, v)) for p, v in zip(c["per"], c["values"])]
    if what in ("all", "masks"):
        words = torch.from_numpy(R.pack_bits(c["masks"])).to(DEV)
        if vocab % 32:
            words[:, -1] |= -1 << (vocab % 32)  # bits beyond the vocabulary mean nothing
        given |= dict(masks=words, mask_of=torch.from_numpy(c["mask_of"]).to(DEV))
        want["allowed"] = np.where(c["mask_of"][:, None] < 0, True, c["masks"][c["mask_of"]])
    ref = R.adjust(_wide(c["logits"]), **want)
    size = np.abs(np.nan_to_num(_wide(c["logits"]), posinf=0, neginf=0)) * 2 + 40
    out = torch.empty(n, vocab, dtype=dtype, device=DEV)
    assert ledger.adjust(held[:, :vocab], out, **given) is out
    _close(out, ref, dtype, size)
    ledger.adjust(held[:, :vocab], **given)  # in place
    assert torch.equal(held[:, :vocab].isnan(), out.isnan()) and torch.equal(held[:, :vocab].nan_to_num(), out.nan_to_num())
    assert bool((held[:, vocab:] == 9.0).all())
    assert P.cnr_poll_errors(ctx) == (P.CNR_OK, 0, 0)


def test_adjust_parts_of_the_penalties_and_ids_that_there_are_not(ctx):
    c = _adjust_case(4, 500, torch.float32, 3)
    c["logits"] = c["logits"].nan_to_num(0.0, 1.0, -1.0).clamp(-100, 100)
    seen, counts = torch.from_numpy(R.pack_bits(c["seen"])).to(DEV), torch.from_numpy(c["counts"].astype(np.int32)).to(DEV)
    x = c["logits"].to(DEV)
    for name, key in (("repetition", "rep"), ("frequency", "freq"), ("presence", "pres")):
        out = P.TokenLedger(ctx, 6, 500, seen, counts).adjust(x, torch.empty_like(x), **{name: torch.from_numpy(c[key]).to(DEV)})
        _close(out, R.adjust(_wide(x), c["seen"][:4], c["counts"][:4], **{name: c[key]}), torch.float32, np.abs(_wide(x)) * 2 + 40)
    # no counts: the repetition penalty alone
    out = P.TokenLedger(ctx, 6, 500, seen).adjust(x, torch.empty_like(x), repetition=torch.from_numpy(c["rep"]).to(DEV), frequency=torch.from_numpy(c["freq"]).to(DEV))
    _close(out, R.adjust(_wide(x), c["seen"][:4], None, c["rep"]), torch.float32, np.abs(_wide(x)) * 2 + 40)
    # negative slots and masks: rows without; ones that there are not: the same, and reported
    rep = torch.from_numpy(c["rep"]).to(DEV)
    masks = torch.zeros(2, 16, dtype=torch.int32, device=DEV)
    ledger = P.TokenLedger(ctx, 6, 500, seen, counts)
    out = ledger.adjust(x, torch.empty_like(x), slots=torch.full((4,), -1, dtype=torch.int32, device=DEV), repetition=rep, masks=masks,
                        mask_of=torch.full((4,), -2, dtype=torch.int32, device=DEV))
    assert torch.equal(out, x) and P.cnr_poll_errors(ctx) == (P.CNR_OK, 0, 0)
    out = ledger.adjust(x, torch.empty_like(x), slots=torch.full((4,), 6, dtype=torch.int32, device=DEV), repetition=rep, masks=masks,
                        mask_of=torch.full((4,), 2, dtype=torch.int32, device=DEV))
    st, _, flags = P.cnr_poll_errors(ctx)
    assert torch.equal(out, x) and st == P.CNR_E_ROW_ID and flags == P.CNR_FLAG_ROW_ID


# ---- streams and graphs -----------------------------------------------------------------------------------------------

def test_another_stream_and_a_graph_replayed(ctx):
    g = torch.Generator(device=DEV).manual_seed(1)
    n, dim, vocab = 40, 300, 1000
    table = torch.randn(vocab, dim, generator=g, device=DEV)
    layer = P.BlockLinear(ctx, vocab, dim, n)
    x, dy = torch.randn(n, dim, generator=g, device=DEV).bfloat16(), torch.randn(n, vocab, generator=g, device=DEV).bfloat16()
    ledger = P.TokenLedger(ctx, n, vocab)
    tokens = torch.randint(0, vocab, (n,), generator=g, device=DEV)
    rep = torch.full((n,), 1.3, device=DEV)
    y, dx, dw = torch.empty(n, vocab, device=DEV, dtype=torch.bfloat16), torch.empty_like(x), torch.empty_like(table)

    def step():
        layer.load(table)
        layer.forward(x, y)
        layer.backward(dy, dx, dw)
        ledger.count(tokens, restart=True)
        ledger.adjust(y, repetition=rep)

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (y, dx, dw, ledger.counts, ledger.seen)]

    step()
    first = results()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    assert all(torch.equal(a, b) for a, b in zip(results(), first))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        x.copy_(torch.randn(n, dim, generator=g, device=DEV))
        tokens.copy_(torch.randint(0, vocab, (n,), generator=g, device=DEV))
        step()
        want = results()
        for t in (y, dx, dw):
            t.zero_()
        ledger.counts.fill_(9)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(results(), want)), k
    assert P.cnr_poll_errors(ctx) == (P.CNR_OK, 0, 0)


def test_a_layers_graph_outlives_calls_of_other_sizes(ctx):
    # the workspace that a graph was captured with stays while the layer lives
    g = torch.Generator(device=DEV).manual_seed(2)
    n_in, n_out = 16384, 1024
    layer = P.BlockLinear(ctx, n_out, n_in, 300)
    layer.load(torch.randn(n_out, n_in, generator=g, device=DEV))
    x = torch.randn(64, n_in, generator=g, device=DEV).bfloat16()
    y = torch.empty(64, n_out, dtype=torch.bfloat16, device=DEV)
    assert P.block_workspace(ctx, 64, n_out, n_in) is not None
    want = layer.forward(x, training=False)
    space = layer._for(64)[4]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(x, y, training=False)
    for tokens in (300, 1, 130, 300):
        layer.forward(torch.randn(tokens, n_in, generator=g, device=DEV).bfloat16(), training=False)
        assert any(s is space for s in layer._spaces)
        other = torch.zeros(space.numel(), dtype=torch.uint8, device=DEV)  # takes the memory if it is free
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and not bool(other.any())


# ---- the two ways of the binding ----------------------------------------------------------------------------------------

WAYS = ["extension", "general"]


@pytest.fixture(params=WAYS)
def way(request, monkeypatch):
    """The calls through the extension, and without it."""
    L.load()
    if request.param == "general":
        for name in ("_quantize", "_product", "_count", "_adjust"):
            monkeypatch.setattr(L, name, L._no_call)
    else:
        assert L._quantize is not L._no_call
    return request.param


def test_both_ways_take_the_same(ctx, way):
    g = np.random.default_rng(1)
    m, n, k = 5, 40, 200
    held = torch.from_numpy(g.normal(0, 1, (m, k + 3))).float().to(DEV)
    w = torch.from_numpy(g.normal(0, 1, (n, k))).to(torch.float16).to(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, side):
        x, x_t, y = P.BlockMatrix.empty(m, k), P.BlockMatrix.empty(k, m), P.BlockMatrix.empty(n, k, P.CNR_BLOCK_TILE)
        torch.cuda.synchronize()
        P.quantize_blocks(ctx, held[:, :k], x, x_t, stream)
        P.quantize_blocks(ctx, w, y, stream=stream)
        out = torch.zeros(m, n + 1, device=DEV)[:, :n]
        space = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        P.block_product(ctx, x, y, out, workspace=space, stream=stream)
        P.block_product(ctx, x, y, out, accumulate=True, stream=stream)
        torch.cuda.synchronize()
        a, b = (R.values(*R.quantize(_wide(v), kind, "e8m0"), kind) for v, kind in ((held[:, :k], "row"), (w, "tile")))
        _check(_wide(out), 2 * a @ b.T, 2 * np.abs(a) @ np.abs(b).T, "f32", 2 * k)
        assert np.array_equal(x_t.codes.cpu().numpy(), R.quantize(_wide(held[:, :k]).T, "row", "e8m0")[0])
    for index in (torch.int32, torch.int64):
        ledger, bits = P.TokenLedger(ctx, 4, n), P.TokenLedger(ctx, 4, n, torch.zeros(4, 2, dtype=torch.int32, device=DEV))
        seen, counts = np.zeros((4, n), bool), np.zeros((4, n), np.int64)
        tokens, offsets, slots = g.integers(0, n, 9), np.array([0, 3, 3, 9]), np.array([2, 0, 1], np.int32)
        given = torch.from_numpy(tokens).to(index).to(DEV), torch.from_numpy(offsets).to(DEV), torch.from_numpy(slots).to(DEV)
        for one in (ledger, bits):
            one.count(*given, prompt=True, restart=True)
            one.count(given[0][:4])
        R.count(seen, counts, n, tokens, offsets, slots, True, True)
        R.count(seen, counts, n, tokens[:4], np.arange(5), np.arange(4))
        assert np.array_equal(ledger.counts.cpu().numpy(), counts) and np.array_equal(ledger.seen.cpu().numpy(), R.pack_bits(seen))
        assert torch.equal(bits.seen, ledger.seen) and bits.counts is None
    logits = torch.from_numpy(g.normal(0, 3, (3, n))).float().to(DEV)
    p = [torch.from_numpy(g.random(3).astype(np.float32) + 0.5).to(DEV) for _ in range(3)]
    allowed = g.random((2, n)) < 0.5
    biases = [[(1, 2.0)], [], [(0, -1.0), (39, 3.0)]]
    got = ledger.adjust(logits, torch.empty_like(logits), slots=given[2], repetition=p[0], frequency=p[1], presence=p[2],
                        bias=(torch.tensor([0, 1, 1, 3], device=DEV), torch.tensor([1, 0, 39], dtype=torch.int32, device=DEV), torch.tensor([2.0, -1.0, 3.0], device=DEV)),
                        masks=torch.from_numpy(R.pack_bits(allowed)).to(DEV), mask_of=torch.tensor([1, -1, 0], dtype=torch.int32, device=DEV))
    want = R.adjust(_wide(logits), seen[slots], counts[slots], *(v.cpu().numpy() for v in p), biases, np.where(np.array([1, -1, 0])[:, None] < 0, True, allowed[[1, 0, 0]]))
    _close(got, want, torch.float32, np.abs(_wide(logits)) * 2 + 40)
    assert torch.equal(ledger.adjust(logits, torch.empty_like(logits)), logits)
    assert P.cnr_poll_errors(ctx) == (P.CNR_OK, 0, 0)


def test_both_ways_refuse_the_same(ctx, way):
    x, out = torch.zeros(8, 200, device=DEV), P.BlockMatrix.empty(8, 200)
    w, y = P.BlockMatrix.empty(6, 200, P.CNR_BLOCK_TILE, P.CNR_SCALE_F32), torch.zeros(8, 6, device=DEV)
    for error, call in [
            (TypeError, lambda: L.cnr_quantize_blocks(ctx, x.double(), 0, 0, out.codes, out.scale)),
            (TypeError, lambda: L.cnr_quantize_blocks(ctx, x.cpu(), 0, 0, out.codes, out.scale)),
            (ValueError, lambda: L.cnr_quantize_blocks(ctx, x[0], 0, 0, out.codes, out.scale)),
            (ValueError, lambda: L.cnr_quantize_blocks(ctx, x.t(), 0, 0, out.codes, out.scale)),
            (ValueError, lambda: L.cnr_quantize_blocks(ctx, x[:, :1].expand(8, 200), 0, 0, out.codes, out.scale)),
            (ValueError, lambda: L.cnr_quantize_blocks(ctx, x[:1].expand(8, 200), 0, 0, out.codes, out.scale)),
            (ValueError, lambda: L.cnr_quantize_blocks(ctx, x, 0, 0, out.codes[:7], out.scale)),
            (ValueError, lambda: L.cnr_quantize_blocks(ctx, x, 0, 0, out.codes, None)),
            (ValueError, lambda: L.cnr_quantize_blocks(ctx, x, 2, 0, out.codes, out.scale)),
            (TypeError, lambda: L.cnr_quantize_blocks(ctx, x, 0, 1, out.codes, out.scale)),
            (ValueError, lambda: L.cnr_quantize_blocks(ctx, x, 0, 0, None, None, out.codes, out.scale)),
            (P.CnrError, lambda: L.cnr_quantize_blocks(ctx, x, 0, 0, None, None)),
            (P.CnrError, lambda: L.cnr_quantize_blocks(None, x, 0, 0, out.codes, out.scale)),
            (P.CnrError, lambda: L.cnr_quantize_blocks(ctx, x, 0, 0, torch.zeros(2049, dtype=torch.uint8, device=DEV)[1:], out.scale)),
            (TypeError, lambda: P.block_product(ctx, out, w, y)),  # scales of two types
            (ValueError, lambda: P.block_product(ctx, out, out, y)),
            (ValueError, lambda: L.cnr_block_product(ctx, out.codes, out.scale, 0, 9, out.codes, out.scale, 0, 6, 200, y)),
            (ValueError, lambda: L.cnr_block_product(ctx, out.codes, out.scale, 0, 8, out.codes, out.scale, 0, 7, 200, y)),
            (ValueError, lambda: L.cnr_block_product(ctx, out.codes, out.scale, 0, 8, out.codes, out.scale, 0, 6, 257, y)),
            (TypeError, lambda: L.cnr_block_product(ctx, out.codes, out.scale, 0, 8, out.codes, out.scale, 0, 6, 200, y.int())),
            (TypeError, lambda: L.cnr_count_tokens(ctx, out.scale[:1], None, 1, 8, torch.zeros(1, dtype=torch.int64, device=DEV))),
            (TypeError, lambda: P.TokenLedger(ctx, 2, 40).count(torch.zeros(2, dtype=torch.int16, device=DEV))),
            (TypeError, lambda: P.TokenLedger(ctx, 2, 40).count(torch.zeros(2, dtype=torch.int64, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV))),
            (ValueError, lambda: P.TokenLedger(ctx, 2, 40).count(torch.zeros(2, dtype=torch.int64, device=DEV), torch.zeros(0, dtype=torch.int64, device=DEV))),
            (ValueError, lambda: P.TokenLedger(ctx, 2, 40).count(torch.zeros(2, dtype=torch.int64, device=DEV), slots=torch.zeros(1, dtype=torch.int32, device=DEV))),
            (ValueError, lambda: P.TokenLedger(ctx, 2, 40, counts=torch.zeros(79, dtype=torch.int32, device=DEV)).count(torch.zeros(2, dtype=torch.int64, device=DEV))),
            (ValueError, lambda: L.cnr_adjust_logits(ctx, x, x[:, 1:])),
            (ValueError, lambda: L.cnr_adjust_logits(ctx, x[:4], x[3:7])),
            (ValueError, lambda: L.cnr_adjust_logits(ctx, x, x.half())),
            (ValueError, lambda: L.cnr_adjust_logits(ctx, x, x, repetition=torch.ones(7, device=DEV))),
            (TypeError, lambda: L.cnr_adjust_logits(ctx, x, x, repetition=torch.ones(8, device=DEV, dtype=torch.float64))),
            (ValueError, lambda: L.cnr_adjust_logits(ctx, x, x, bias_offsets=torch.zeros(9, dtype=torch.int64, device=DEV))),
            (ValueError, lambda: L.cnr_adjust_logits(ctx, x, x, bias_offsets=torch.zeros(8, dtype=torch.int64, device=DEV), bias_tokens=torch.zeros(1, dtype=torch.int32, device=DEV),
                                                     bias_values=torch.zeros(1, device=DEV))),
            (ValueError, lambda: L.cnr_adjust_logits(ctx, x, x, masks=torch.zeros(8, 6, dtype=torch.int32, device=DEV), n_masks=8)),
            (P.CnrError, lambda: L.cnr_adjust_logits(None, x, x))]:
        with pytest.raises(error):
            call()
    torch.cuda.synchronize()
    assert P.cnr_poll_errors(ctx) == (P.CNR_OK, 0, 0)


def test_the_example_trains_checkpoints_and_decodes():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_and_decode.py")
    spec = importlib.util.spec_from_file_location("train_and_decode", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main()
    assert r["losses"][0] > 5.0 and r["losses"][-1] < 0.5  # ln 500 = 6.2 to begin with
    assert r["errors"] == (P.CNR_OK, 0, 0)
    for way in ("written", "resumed"):
        for prompt, tokens in zip(r["prompts"], r[way]):
            assert len(set(prompt + tokens)) == len(prompt) + 12 and 38 not in tokens
            if prompt != [5]:  # 5 is followed by 38, which the grammar forbids
                assert tokens[0] == (7 * prompt[-1] + 3) % example.VOCAB
