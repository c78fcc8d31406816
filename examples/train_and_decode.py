"""A small language model trained, checkpointed and served: an embedding table and the matrix that gives the logits, whose touched rows are
tracked and saved, an output layer in 8-bit blocks, and decoding with penalties and a grammar's masks, by the model in memory and by one that
is resumed from nothing but the checkpoints.

The data are chains token -> (7 token + 3) mod vocabulary.  Run on an MI355X:  python examples/train_and_decode.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2010_08679_amd as P  # noqa: E402

VOCAB, DIM, TOKENS = 500, 128, 1024


def train(ctx, table, head, steps, table_checkpointer, head_checkpointer, seed=0):
    """`steps` steps on the cross-entropy of the next token; the losses.  The table's updates are sparse, the head's dense; both are tracked."""
    g = torch.Generator(device=table.device).manual_seed(seed)
    layer = P.BlockLinear(ctx, VOCAB, DIM, TOKENS)
    logits = torch.empty(TOKENS, VOCAB, dtype=torch.bfloat16, device=table.device)
    dx, dw = torch.empty(TOKENS, DIM, dtype=torch.bfloat16, device=table.device), torch.empty_like(head)
    losses, every_row = [], torch.arange(VOCAB, device=table.device)
    for _ in range(steps):
        now = torch.randint(0, VOCAB, (TOKENS,), generator=g, device=table.device)
        after = (7 * now + 3) % VOCAB
        layer.load(head)
        layer.forward(table[now].bfloat16(), logits)
        p = torch.softmax(logits.float(), dim=1)
        losses.append(float(-torch.log(p.gather(1, after[:, None])).mean()))
        p.scatter_add_(1, after[:, None], torch.full_like(p[:, :1], -1.0))  # d loss / d logits, times the number of tokens
        layer.backward(p.bfloat16(), dx, dw)
        head -= 0.02 * dw
        table.index_add_(0, now, dx.float(), alpha=-0.02)
        table_checkpointer.mark(now)
        head_checkpointer.mark(every_row)
    return losses


def decode(ctx, table, head, prompts, steps, forbidden):
    """`steps` tokens for each prompt (a list of lists): greedy, no token twice (nor of the prompt), none of `forbidden`."""
    device, n = table.device, len(prompts)
    ledger = P.TokenLedger(ctx, n, VOCAB, device=device)
    lengths = torch.tensor([0] + [len(p) for p in prompts], device=device)
    ledger.count(torch.tensor([t for p in prompts for t in p], device=device), lengths.cumsum(0), prompt=True, restart=True)
    allowed = torch.ones(1, (VOCAB + 31) // 32 * 32, dtype=torch.bool, device=device)
    allowed[0, list(forbidden)] = False
    masks = (allowed.view(1, -1, 32).long() << torch.arange(32, device=device)).sum(2).to(torch.int32)
    mask_of = torch.zeros(n, dtype=torch.int32, device=device)
    # a positive logit divided by it, a negative one multiplied: what was seen falls far behind
    repetition = torch.full((n,), 1000.0, device=device)
    presence = torch.full((n,), 1000.0, device=device)
    weight = P.BlockMatrix.empty(VOCAB, DIM, P.CNR_BLOCK_TILE, device=device)
    P.quantize_blocks(ctx, head, weight)
    x = P.BlockMatrix.empty(n, DIM, device=device)
    logits, space = torch.empty(n, VOCAB, device=device), P.block_workspace(ctx, n, VOCAB, DIM, device)
    last, written = torch.tensor([p[-1] for p in prompts], device=device), []
    for _ in range(steps):
        P.quantize_blocks(ctx, table[last], x)
        P.block_product(ctx, x, weight, logits, workspace=space)
        ledger.adjust(logits, repetition=repetition, presence=presence, masks=masks, mask_of=mask_of)
        last = logits.argmax(dim=1)
        ledger.count(last)
        written.append(last)
    return torch.stack(written, dim=1).tolist()


def main(device="cuda:0", steps=150):
    ctx = P.cnr_create(0)
    g = torch.Generator(device=device).manual_seed(1)
    table = torch.randn(VOCAB, DIM, generator=g, device=device) * 0.1
    head = torch.randn(VOCAB, DIM, generator=g, device=device) * 0.1
    resumed = [table.clone(), head.clone()]  # as they were before training, when the last full checkpoint was taken
    checkpointers = [P.TableCheckpointer(ctx, VOCAB, DIM, device=device) for _ in resumed]
    for ck in checkpointers:
        ck.clear()
    losses = train(ctx, table, head, steps, *checkpointers)
    for ck, trained, stale in zip(checkpointers, (table, head), resumed):
        ck.compact()
        ck.restore(stale, ck.encode(trained, ck.alloc_output(bits=8)))
    prompts = [[5], [9, 66], [100, 203, 424]]
    results = {"losses": losses, "written": decode(ctx, table, head, prompts, 12, forbidden=[38]),
               "resumed": decode(ctx, *resumed, prompts, 12, forbidden=[38]), "prompts": prompts, "errors": P.cnr_poll_errors(ctx),
               "trained_matrices": (table, head), "resumed_matrices": tuple(resumed)}
    P.cnr_destroy(ctx)
    return results


if __name__ == "__main__":
    r = main()
    print("loss %.3f -> %.3f" % (r["losses"][0], r["losses"][-1]))
    for prompt, a, b in zip(r["prompts"], r["written"], r["resumed"]):
        print(prompt, "->", a, "" if a == b else "from the checkpoint: %s" % b)
