"""What the operators for language models write is known to autograd as changed, through the extension and without it."""
import pytest
import torch

import paper_2010_08679_amd as P
from paper_2010_08679_amd import lm_binding as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = P.cnr_create(0)
    yield c
    torch.cuda.synchronize()
    P.cnr_destroy(c)


@pytest.fixture(params=["extension", "general"], autouse=True)
def way(request, monkeypatch):
    L.load()
    if request.param == "general":
        for name in ("_quantize", "_product", "_count", "_adjust"):
            monkeypatch.setattr(L, name, L._no_call)


def test_a_saved_logit_that_is_adjusted_in_place_is_no_silent_error(ctx):
    logits = torch.randn(3, 40, device=DEV)
    scale = torch.ones(3, 40, device=DEV, requires_grad=True)
    loss = (scale * logits).sum()  # saves the logits
    P.TokenLedger(ctx, 3, 40).adjust(logits, masks=torch.zeros(3, 2, dtype=torch.int32, device=DEV))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    loss = (scale * logits.clamp(-9, 9)).sum()
    P.TokenLedger(ctx, 3, 40).adjust(logits, torch.empty_like(logits))  # read only
    loss.backward()


def test_everything_written_has_a_new_version(ctx):
    x = torch.randn(5, 200, device=DEV)
    out, out_t, w = P.BlockMatrix.empty(5, 200), P.BlockMatrix.empty(200, 5), P.BlockMatrix.empty(7, 200)
    P.quantize_blocks(ctx, torch.randn(7, 200, device=DEV), w)
    held = torch.zeros(5, 9, device=DEV)
    ledger = P.TokenLedger(ctx, 2, 40)
    tokens = torch.zeros(2, dtype=torch.int64, device=DEV)
    for call, written in ((lambda: P.quantize_blocks(ctx, x, out, out_t), (out.codes, out.scale, out_t.codes, out_t.scale)),
                          (lambda: P.quantize_blocks(ctx, x, None, out_t), (out_t.codes, out_t.scale)),
                          (lambda: P.block_product(ctx, out, w, held[:, :7]), (held,)),
                          (lambda: ledger.count(tokens), (ledger.seen, ledger.counts))):
        read = [t for t in (x, out.codes, out.scale, out_t.codes, w.codes, w.scale, tokens) if not any(t is u for u in written)]
        before, kept = [t._version for t in written], [t._version for t in read]
        call()
        assert all(t._version > v for t, v in zip(written, before))
        assert [t._version for t in read] == kept


def test_refused_calls_change_no_version(ctx):
    x, out = torch.randn(5, 200, device=DEV), P.BlockMatrix.empty(5, 200)
    before = out.codes._version
    with pytest.raises(P.CnrError):
        L.cnr_quantize_blocks(None, x, P.CNR_BLOCK_ROW, P.CNR_SCALE_E8M0, out.codes, out.scale)
    assert out.codes._version == before


def test_inference_tensors_are_written_too(ctx):
    with torch.inference_mode():
        logits, x, out = torch.zeros(2, 40, device=DEV), torch.ones(5, 200, device=DEV), P.BlockMatrix.empty(5, 200)
    masks = torch.zeros(2, 2, dtype=torch.int32, device=DEV)
    ledger = P.TokenLedger(ctx, 2, 40)
    for mode in (torch.inference_mode(), torch.no_grad()):
        with mode:
            logits.zero_() if torch.is_inference_mode_enabled() else None
            ledger.adjust(logits, masks=masks)
            P.quantize_blocks(ctx, x, out)
        assert bool((logits == -torch.inf).all()) and int(out.codes[0, 0]) != 0
