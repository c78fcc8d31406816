"""The operators for language models at the sizes where they take another kernel, split their work or pass 32 bits.  Inputs are drawn as in
test_gpu_language.py, references are 64-bit."""
import numpy as np
import pytest
import torch

import paper_2010_08679_amd as P
from oracle import blocks as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def ctx():
    c = P.cnr_create(0)
    yield c
    torch.cuda.synchronize()
    P.cnr_destroy(c)


# ---- products -------------------------------------------------------------------------------------------------------

def _whole(rows, k, kind, scale, seed):
    """A BlockMatrix of whole numbers up to 4 with scales of 1/2, 1 and 2, and its values: sums of up to 2^24 / 256 products are exact in fp32."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    m = P.BlockMatrix.empty(rows, k, kind, scale)
    v = torch.randint(-4, 5, (rows, k), generator=g, device=DEV).float()
    m.codes.zero_()
    m.codes[:, :k] = v.to(torch.float8_e4m3fn).view(torch.uint8)
    e = torch.randint(-1, 2, tuple(m.scale.shape), generator=g, device=DEV)
    m.scale.copy_((127 + e).to(torch.uint8) if scale == P.CNR_SCALE_E8M0 else torch.tensor([0.5, 1.0, 2.0], device=DEV)[e + 1])
    each = torch.tensor([0.5, 1.0, 2.0], device=DEV, dtype=torch.float64)[e + 1].repeat_interleave(128, 0)[:k]
    each = (each.repeat_interleave(128, 1) if kind == P.CNR_BLOCK_TILE else each)[:, :rows].t()
    return m, v.double() * each


# few and many tiles of each size, without a remainder and with one; sums in 1, 2, 4 and 8 parts; the kernel for few rows at both ends
SIZES = [(1, 40, 9000), (17, 513, 128), (2049, 4097, 128), (4100, 2050, 300), (4096, 4096, 512), (500, 4097, 128), (2049, 1000, 300), (500, 2050, 4100),
         (257, 4097, 9000), (100, 4097, 4100), (1000, 513, 9000), (500, 513, 4100), (257, 1000, 9000), (4100, 4097, 300), (2049, 9000, 300),
         (1000, 4097, 9000), (1000, 4097, 128), (500, 9000, 300), (2049, 513, 9000), (64, 4097, 9000), (17, 9000, 9000), (1000, 1000, 300),
         (100, 9000, 300), (4100, 130, 9000), (500, 513, 4100), (4100, 40, 9000), (100, 1000, 9000), (64, 2050, 9000)]


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("scale", [P.CNR_SCALE_E8M0, P.CNR_SCALE_F32])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_product_of_whole_numbers_is_exact_in_every_kernel(ctx, out, scale, m, n, k):
    for a_kind, b_kind in ((P.CNR_BLOCK_ROW, P.CNR_BLOCK_TILE), (P.CNR_BLOCK_ROW, P.CNR_BLOCK_ROW)):
        (a, av), (b, bv) = _whole(m, k, a_kind, scale, m), _whole(n, k, b_kind, scale, n + 1)
        want = av @ bv.t()
        space = P.block_workspace(ctx, m, n, k)
        if space is not None:
            space.fill_(255)  # its contents do not matter
        held = torch.full((m, n + 5), 3.0, dtype=TYPES[out], device=DEV)
        got = held[:, 1 : n + 1]  # aligned to an element only
        P.block_product(ctx, a, b, got, workspace=space)
        assert torch.equal(got, want.float().to(TYPES[out]))
        start = torch.randint(-9, 10, (m, n), device=DEV, generator=torch.Generator(device=DEV).manual_seed(5)).double()
        got.copy_(start)
        P.block_product(ctx, a, b, got, accumulate=True, workspace=space)
        assert torch.equal(got, (want + start).float().to(TYPES[out]))
        P.block_product(ctx, a, b, got)  # no workspace: never in parts
        assert torch.equal(got, want.float().to(TYPES[out]))
        assert bool((held[:, :1] == 3.0).all()) and bool((held[:, n + 1 :] == 3.0).all())


@pytest.mark.parametrize("scale", [P.CNR_SCALE_E8M0, P.CNR_SCALE_F32])
@pytest.mark.parametrize("m", [2, 300])
def test_product_with_more_than_4_gib_of_codes(ctx, m, scale):
    n, k = 600_000, 8192  # B: 4.9e9 codes
    a, av = _whole(m, k, P.CNR_BLOCK_ROW, scale, 1)
    b = P.BlockMatrix.empty(n, k, P.CNR_BLOCK_TILE, scale)
    part, values = _whole(12_800, k, P.CNR_BLOCK_TILE, scale, 2)
    for i in range(0, n, 12_800):  # 46.875 times the same
        rows, tiles = min(12_800, n - i), (min(12_800, n - i) + 127) // 128
        b.codes[i : i + rows] = part.codes[:rows]
        b.scale[:, i // 128 : i // 128 + tiles] = part.scale[:, :tiles]
    out = P.block_product(ctx, a, b, torch.empty(m, n, dtype=torch.bfloat16, device=DEV), workspace=P.block_workspace(ctx, m, n, k))
    want = (av @ values.t()).float().bfloat16()
    for i in range(0, n, 12_800):
        rows = min(12_800, n - i)
        assert torch.equal(out[:, i : i + rows], want[:, :rows]), i


@pytest.mark.parametrize("scale", [P.CNR_SCALE_E8M0, P.CNR_SCALE_F32])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(1_200_000, 10), (2_100_037, 1), (3, 1_500_011)])
def test_product_of_a_table_with_a_few_rows_either_way(ctx, out, scale, m, n):
    # more than 2^16 workgroups of 16 rows; in parts that end inside a tile
    (a, av), (b, bv) = _whole(m, 100, P.CNR_BLOCK_TILE, scale, 1), _whole(n, 100, P.CNR_BLOCK_ROW, scale, 2)
    got = torch.full((m, n + 1), 3.0, dtype=TYPES[out], device=DEV)
    P.block_product(ctx, a, b, got[:, :n])
    assert torch.equal(got[:, :n], (av @ bv.t()).float().to(TYPES[out])) and bool((got[:, n] == 3.0).all())


def test_product_with_more_columns_than_a_grid_has_threads(ctx):
    n = (1 << 28) + 77  # 34 GB of codes, of which one in 128 is in the matrix
    a, av = _whole(1, 1, P.CNR_BLOCK_ROW, P.CNR_SCALE_E8M0, 1)
    a.codes[0, 0], a.scale[0, 0] = 0x40, 128  # 2 * 2
    b = P.BlockMatrix.empty(n, 1, P.CNR_BLOCK_TILE)
    b.codes.zero_()
    b.codes[:, 0] = (torch.arange(n, device=DEV) % 9 + 0x38).to(torch.uint8)  # 1, 1.125, ... 2
    b.scale.copy_((torch.arange(b.scale.shape[1], device=DEV) % 3 + 126).to(torch.uint8))
    out = P.block_product(ctx, a, b)
    i = torch.arange(n, device=DEV)
    assert torch.equal(out[0], (4 * (1 + (i % 9) / 8) * 2.0 ** (i // 128 % 3 - 1)).bfloat16())


def test_product_with_more_than_4_gi_outputs(ctx):
    m, n, k = 66_000, 66_000, 130
    a, av = _whole(m, k, P.CNR_BLOCK_ROW, P.CNR_SCALE_E8M0, 1)
    b, bv = _whole(n, k, P.CNR_BLOCK_ROW, P.CNR_SCALE_E8M0, 2)
    out = P.block_product(ctx, a, b, torch.empty(m, n, dtype=torch.bfloat16, device=DEV))
    for i in range(0, m, 6000):
        assert torch.equal(out[i : i + 6000], (av[i : i + 6000] @ bv.t()).float().bfloat16()), i


def test_quantize_more_than_4_gi_elements(ctx):
    rows, dim = 70_000, 66_000
    x = torch.randn(rows, dim, dtype=torch.bfloat16, device=DEV)
    out, out_t = P.BlockMatrix.empty(rows, dim, P.CNR_BLOCK_ROW), P.BlockMatrix.empty(dim, rows, P.CNR_BLOCK_ROW)
    P.quantize_blocks(ctx, x, out, out_t)
    for where, got, m in ((slice(69_950, 70_000), out, x[69_950:]), (slice(65_990, 66_000), out_t, x[:, 65_990:].t())):
        codes, scale = R.quantize(m.double().cpu().numpy(), "row", "e8m0")
        assert np.array_equal(got.codes[where].cpu().numpy(), codes)
        assert np.array_equal(got.scale[:, where].cpu().numpy().astype(np.int64) - 127, np.log2(scale).astype(np.int64))


# ---- tokens -----------------------------------------------------------------------------------------------------------

def _tokens(g, total, vocab):
    tokens = np.minimum(g.zipf(1.1, total) - 1, vocab + 1)  # some beyond the vocabulary
    return np.where(g.random(total) < 0.01, -1 - tokens, tokens)


@pytest.mark.parametrize("index", [torch.int32, torch.int64])
@pytest.mark.parametrize("vocab", [33, 16384, 40_001])
# sequences that begin: many, few, shorter and longer than a workgroup's share; that go on: token by token, and slice by slice
@pytest.mark.parametrize("lengths", [(0, 1, 700, 4096, 513, 5000, 0), (0, 40_000, 3, 60_000, 9000, 0, 1), (140_000, 3), (1, 0, 0), (0,)])
@pytest.mark.parametrize("prompt,restart", [(False, True), (True, True), (False, False), (True, False)])
def test_count_at_every_length(ctx, index, vocab, lengths, prompt, restart):
    g = np.random.default_rng(len(lengths) + vocab)
    n, n_slots = len(lengths), 6
    offsets = np.concatenate([[0], np.cumsum(lengths)])
    tokens = _tokens(g, offsets[-1], vocab)
    bad = int(((tokens < 0) | (tokens >= vocab)).sum())
    for shared in (False, True):
        slots = g.integers(0, 3, n) if shared else (g.permutation(max(n, n_slots))[:n] % n_slots)
        if not shared and n > n_slots:
            slots[-1] = n_slots  # a slot that there is not, of a single token
        start = g.integers(0, 3, (n_slots, vocab))
        seen, counts = start > 0, start.astype(np.int64).copy()
        keeps = np.ones(n, bool) if slots.max() < n_slots else slots < n_slots
        ledger = P.TokenLedger(ctx, n_slots, vocab, torch.from_numpy(R.pack_bits(seen)).to(DEV), torch.from_numpy(counts.astype(np.int32)).to(DEV))
        bits = P.TokenLedger(ctx, n_slots, vocab, ledger.seen.clone())  # without counts
        given = (torch.from_numpy(tokens).to(index).to(DEV), torch.from_numpy(offsets).to(DEV), torch.from_numpy(slots.astype(np.int32)).to(DEV))
        ledger.count(*given, prompt=prompt, restart=restart)
        bits.count(*given, prompt=prompt, restart=restart)
        kept = offsets.copy()
        if not keeps.all():  # the definition without the sequence that has no slot, the last one
            kept = kept[:-1]
        R.count(seen, counts, vocab, tokens[: kept[-1]], kept, slots[keeps].astype(np.int32), prompt, restart)
        assert np.array_equal(ledger.counts.cpu().numpy(), counts)
        assert np.array_equal(ledger.seen.cpu().numpy(), R.pack_bits(seen)) and torch.equal(bits.seen, ledger.seen)
        st, n_bad, flags = P.cnr_poll_errors(ctx)
        missing = tokens[kept[-1] :]
        here = bad - int(((missing < 0) | (missing >= vocab)).sum())
        assert (n_bad, flags) == (2 * here, 0 if keeps.all() or lengths[-1] == 0 else P.CNR_FLAG_ROW_ID)  # a sequence without tokens needs no slot


@pytest.mark.parametrize("n", [4096, 4097, 40_000])
@pytest.mark.parametrize("prompt", [False, True])
def test_count_of_many_sequences_that_begin(ctx, n, prompt):
    g = np.random.default_rng(n)
    n_slots, vocab = n // 2, 70
    lengths = g.integers(0, 9, n)
    offsets = np.concatenate([[0], np.cumsum(lengths)])
    tokens, slots = g.integers(0, vocab, offsets[-1]), g.integers(0, n_slots, n).astype(np.int32)
    start = g.integers(0, 3, (n_slots, vocab))
    seen, counts = start > 0, start.astype(np.int64).copy()
    ledger = P.TokenLedger(ctx, n_slots, vocab, torch.from_numpy(R.pack_bits(seen)).to(DEV), torch.from_numpy(counts.astype(np.int32)).to(DEV))
    ledger.count(torch.from_numpy(tokens).to(DEV), torch.from_numpy(offsets).to(DEV), torch.from_numpy(slots).to(DEV), prompt=prompt, restart=True)
    R.count(seen, counts, vocab, tokens, offsets, slots, prompt, True)
    assert np.array_equal(ledger.counts.cpu().numpy(), counts) and np.array_equal(ledger.seen.cpu().numpy(), R.pack_bits(seen))
    assert P.cnr_poll_errors(ctx) == (P.CNR_OK, 0, 0)


@pytest.mark.parametrize("restart", [True, False])
def test_count_of_slots_beyond_4_gib(ctx, restart):
    vocab, n_slots, n = 131_072, 9000, 40  # 4.7 GB of counts
    ledger = P.TokenLedger(ctx, n_slots, vocab)
    g = np.random.default_rng(1)
    slots = np.arange(n_slots - n, n_slots).astype(np.int32)
    lengths = g.integers(0, 20_000 if not restart else 500, n)
    offsets = np.concatenate([[0], np.cumsum(lengths)])
    tokens = g.integers(0, vocab, offsets[-1])
    ledger.count(torch.from_numpy(tokens).to(DEV), torch.from_numpy(offsets).to(DEV), torch.from_numpy(slots).to(DEV), restart=restart)
    seen, counts = np.zeros((n, vocab), bool), np.zeros((n, vocab), np.int64)
    R.count(seen, counts, vocab, tokens, offsets, np.arange(n).astype(np.int32))
    assert np.array_equal(ledger.counts[-n:].cpu().numpy(), counts) and np.array_equal(ledger.seen[-n:].cpu().numpy(), R.pack_bits(seen))
    assert not bool(ledger.counts[:-n].any()) and not bool(ledger.seen[:-n].any())


# ---- logits -----------------------------------------------------------------------------------------------------------

def _expected(x, seen, counts, rep, freq, pres, allowed, bias):
    """The definition in 64 bits on the GPU, for finite logits."""
    v = x.double()
    r = rep.double()[:, None]
    v = torch.where(seen, torch.where(v > 0, v / r, v * r), v)
    v = v - freq.double()[:, None] * counts - pres.double()[:, None] * (counts > 0)
    return torch.where(allowed, v + bias, torch.full_like(v, -torch.inf))


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,vocab,pad", [(600, 33_001, 3), (520, 32_768, 0), (130, 131_072, 0), (3, 50_257, 0)])
@pytest.mark.parametrize("biased", [0, 300, 5000])
def test_adjust_many_long_rows(ctx, type, n, vocab, pad, biased):
    dtype = TYPES[type]
    g = torch.Generator(device=DEV).manual_seed(n + biased)
    held = torch.full((n, vocab + pad), 9.0, dtype=dtype, device=DEV)
    x = (torch.randn(n, vocab, generator=g, device=DEV) * 5).to(dtype)
    held[:, :vocab] = x
    counts = torch.randint(1, 4, (n, vocab), generator=g, device=DEV) * (torch.rand(n, vocab, generator=g, device=DEV) < 0.03)
    seen = (counts > 0) | (torch.rand(n, vocab, generator=g, device=DEV) < 0.02)
    allowed = torch.rand(n, vocab, generator=g, device=DEV) < 0.5
    rep, freq, pres = 1 + torch.rand(n, generator=g, device=DEV), torch.rand(n, generator=g, device=DEV), torch.rand(n, generator=g, device=DEV) - 0.5
    added = torch.zeros(n, vocab, dtype=torch.float64, device=DEV)
    bias = None
    if biased:  # every third row has none, the others a window of the list's tokens, all of one stretch or spread out
        tokens, values, offsets = [], [], [0]
        for i in range(n):
            number = 0 if i % 3 == 0 else biased
            first = (i * 977) % (vocab - biased) if i % 2 else 0
            step = 1 if i % 2 else vocab // biased
            at = first + step * torch.arange(number, device=DEV)
            v = torch.randn(number, generator=g, device=DEV)
            added[i, at] = v.double()
            tokens.append(at), values.append(v), offsets.append(offsets[-1] + number)
        bias = (torch.tensor(offsets, device=DEV), torch.cat(tokens).int(), torch.cat(values))

    def packed(bits):
        full = torch.zeros(n, (vocab + 31) // 32 * 32, dtype=torch.bool, device=DEV)
        full[:, :vocab] = bits
        return (full.view(n, -1, 32).long() << torch.arange(32, device=DEV)).sum(2).to(torch.int32)

    ledger = P.TokenLedger(ctx, n, vocab, packed(seen), counts.int())
    ledger.adjust(held[:, :vocab], repetition=rep, frequency=freq, presence=pres, bias=bias, masks=packed(allowed))
    got, want = held[:, :vocab].double(), _expected(x, seen, counts, rep, freq, pres, allowed, added)
    assert torch.equal(got.isinf(), ~allowed)
    # six fp32 operations of values up to twice the logit and what is added, and one rounding to the type
    size = x.double().abs() * 2 + 8
    bound = torch.finfo(dtype).eps / 2 * want.abs() + 6 * 2.0 ** -24 * size + float(torch.finfo(dtype).tiny) * torch.finfo(dtype).eps / 2
    assert bool(((got - want).abs() <= bound)[allowed].all())
    assert bool((held[:, vocab:] == 9.0).all())
    assert P.cnr_poll_errors(ctx) == (P.CNR_OK, 0, 0)


def test_adjust_more_than_4_gi_logits(ctx):
    n, vocab = 33_000, 131_072
    x = torch.zeros(n, vocab, dtype=torch.bfloat16, device=DEV)
    seen = torch.zeros(n, vocab // 32, dtype=torch.int32, device=DEV)
    counts = torch.zeros(n, vocab, dtype=torch.int32, device=DEV)
    seen[-1, -1] = 1 << 30
    counts[-1, -2] = 3
    masks = torch.full((1, vocab // 32), -1, dtype=torch.int32, device=DEV)
    masks[0, 7] = ~(1 << 5)
    ones = torch.ones(n, device=DEV)
    P.TokenLedger(ctx, n, vocab, seen, counts).adjust(x, frequency=ones, presence=ones, masks=masks, mask_of=torch.zeros(n, dtype=torch.int32, device=DEV))
    assert float(x[-1, -2]) == -4.0 and bool((x[:, 7 * 32 + 5] == -torch.inf).all())
    x[-1, -2] = 0
    x[:, 7 * 32 + 5] = 0
    assert not any(bool(part.any()) for part in x.split(1000))


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind", ["row", "tile"])
def test_quantize_many_quotients_with_scales_of_any_value(ctx, type, kind):
    # blocks of all magnitudes, the smallest ones among them, with values next to the middles of codes
    g = torch.Generator().manual_seed(9)
    rows, dim = 640, 512
    x = torch.randn(rows, dim, generator=g, dtype=torch.float64)
    high = 128 if kind == "tile" else 1
    x *= 2.0 ** torch.randint(-150, 127, (rows // high, dim // 128), generator=g).double().repeat_interleave(high, 0).repeat_interleave(128, 1)
    x = x.clamp(-3e38, 3e38)
    whole = x.to(TYPES[type])
    whole = torch.where(whole.isfinite(), whole, torch.zeros_like(whole))
    s = R.quantize(whole.double().numpy(), kind, "f32")[1]  # [block][row or tile]
    each = torch.from_numpy(s if kind == "row" else s.repeat(128, axis=1)).t().repeat_interleave(128, 1)
    code = torch.randint(0, 126, (rows, dim), generator=g)
    middle = torch.from_numpy((R.E4M3[1:127] + R.E4M3[:126]) / 2)[code] * each
    near = torch.nextafter(middle.float(), torch.where(torch.rand(rows, dim, generator=g) < 0.5, 0.0, 3e38)) if type == "f32" else middle
    take = torch.rand(rows, dim, generator=g) < 0.02
    limit = whole.abs().reshape(-1, high, dim // 128, 128).amax(dim=(1, 3)).repeat_interleave(high, 0).repeat_interleave(128, 1)
    whole = torch.where(take & (near.to(TYPES[type]) <= limit), near.to(TYPES[type]), whole)
    out = P.BlockMatrix.empty(rows, dim, P.CNR_BLOCK_TILE if kind == "tile" else P.CNR_BLOCK_ROW, P.CNR_SCALE_F32)
    P.quantize_blocks(ctx, whole.to(DEV), out)
    codes, s = R.quantize(whole.double().numpy(), kind, "f32")
    assert np.array_equal(out.scale.cpu().numpy().astype(np.float64)[:, : s.shape[1]], s)
    assert np.array_equal(out.codes.cpu().numpy(), codes)
