"""A small student of a language model's teacher: the teacher is trained as in train_and_decode.py, its top logits are kept, and a smaller student learns from them
and from the data, by losses over the vocabulary that never hold all logits.  The student's table, which gives its logits too, is tracked, and its touched
rows are saved and restored.

Run on an MI355X:  python examples/distill_student.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2010_08679_amd as P  # noqa: E402
from examples.train_and_decode import DIM, VOCAB, train  # noqa: E402

STUDENT, TOKENS, TOP, HEAT = 64, 512, 16, 2.0


def teachers_top(ctx, table, head, tokens):
    """The teacher's top logits after each token: (tokens, logits), by its 8-bit product."""
    weight = P.BlockMatrix.empty(VOCAB, DIM, P.CNR_BLOCK_TILE, device=table.device)
    P.quantize_blocks(ctx, head, weight)
    logits = P.block_product(ctx, P.quantize_blocks(ctx, table[tokens]), weight, torch.empty(len(tokens), VOCAB, device=table.device))
    return P.top_logits(ctx, logits, TOP)[:2]


def distill(ctx, teacher, table, turn, steps, checkpointer, seed=0):
    """`steps` steps of the student, whose hidden state is a token's row of `table` times `turn` and whose logits are its products with all rows of `table`; the
    losses, half the teacher's and half the data's."""
    g = torch.Generator(device=table.device).manual_seed(seed)
    loss = P.VocabularyLoss(ctx, VOCAB, STUDENT, TOKENS, torch.float32, top=TOP)
    half = torch.full((TOKENS,), 0.5 / TOKENS, device=table.device)
    losses, every_row = [], torch.arange(VOCAB, device=table.device)
    for _ in range(steps):
        now = torch.randint(0, VOCAB, (TOKENS,), generator=g, device=table.device)
        rows = table[now]
        hidden = rows @ turn
        tokens, logits = teachers_top(ctx, *teacher, now)
        soft = loss.distill(hidden, table, tokens, logits, HEAT)
        dhidden, dtable = loss.backward(half * HEAT * HEAT)  # what the temperature takes from the gradient
        hard = loss.cross_entropy(hidden, table, (7 * now + 3) % VOCAB)
        dhidden = dhidden + loss.backward(half, dweight=dtable, accumulate=True)[0]
        losses.append(float((soft + hard).mean()) / 2)
        dtable.index_add_(0, now, dhidden @ turn.t())
        turn -= 4.0 * (rows.t() @ dhidden)
        table -= 4.0 * dtable
        checkpointer.mark(every_row)
    return losses


def main(device="cuda:0", steps=60):
    ctx = P.cnr_create(0)
    g = torch.Generator(device=device).manual_seed(1)
    teacher = [torch.randn(VOCAB, DIM, generator=g, device=device) * 0.1 for _ in range(2)]
    tracked = [P.TableCheckpointer(ctx, VOCAB, DIM, device=device) for _ in teacher]
    for ck in tracked:
        ck.clear()
    train(ctx, *teacher, 100, *tracked)
    table, turn = torch.randn(VOCAB, STUDENT, generator=g, device=device) * 0.3, torch.randn(STUDENT, STUDENT, generator=g, device=device) * 0.1
    before, checkpointer = table.clone(), P.TableCheckpointer(ctx, VOCAB, STUDENT, device=device)
    checkpointer.clear()
    losses = distill(ctx, teacher, table, turn, steps, checkpointer)
    checkpointer.compact()
    checkpointer.restore(before, checkpointer.encode(table, checkpointer.alloc_output(bits=8)))
    results = {"losses": losses, "table": table, "resumed": before, "errors": P.cnr_poll_errors(ctx)}
    P.cnr_destroy(ctx)
    return results


if __name__ == "__main__":
    r = main()
    print("loss %.3f -> %.3f" % (r["losses"][0], r["losses"][-1]))
