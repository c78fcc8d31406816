"""Arguments of the operators for language models that would have reached the device: sizes that no buffer has, rows of another length.  No kernel is launched."""
import ctypes

import pytest
import torch

import paper_2010_08679_amd as P
from paper_2010_08679_amd import lm_binding as L

A = 1 << 20  # an address that is aligned to anything; never read


def _adjust(**given):
    ctx = ctypes.create_string_buffer(4096)  # no call gets as far as using it
    return L.load().cnr_adjust_logits(ctypes.addressof(ctx), A, 64, 2 * A, 64, P.CNR_FLOAT_F32, 2, 64, P.cnr_adjustments(**given), None)


@pytest.mark.parametrize("number", [1 << 31, 1 << 40, (1 << 64) - 1])
def test_more_slots_or_masks_than_there_can_be(number):
    # as ctypes passes a negative number
    assert _adjust(seen=A, n_slots=number) == P.CNR_E_TOO_LARGE
    assert _adjust(masks=A, n_masks=number) == P.CNR_E_TOO_LARGE


def test_masks_of_another_vocabulary():
    # rows of words that are longer than the vocabulary's hold enough of them, but not where they are looked for
    ledger = P.TokenLedger(None, 2, 40, device="cpu")
    for shape in ((3, 3), (3, 1), (6,), (1, 3, 2)):
        with pytest.raises(ValueError):
            ledger.adjust(torch.zeros(2, 40), masks=torch.zeros(shape, dtype=torch.int32), mask_of=torch.zeros(2, dtype=torch.int32))


def test_states_of_another_vocabulary():
    words = torch.zeros(2, 2, dtype=torch.int32)
    P.TokenLedger(None, 2, 40, words.view(-1), torch.zeros(80, dtype=torch.int32))
    P.TokenLedger(None, 2, 40, words, torch.zeros(3, 40, dtype=torch.int32))
    for seen, counts in ((torch.zeros(2, 3, dtype=torch.int32), None), (words, torch.zeros(2, 41, dtype=torch.int32)), (None, torch.zeros(2, 64, dtype=torch.int32))):
        with pytest.raises(ValueError):
            P.TokenLedger(None, 2, 40, seen, counts, device="cpu")
