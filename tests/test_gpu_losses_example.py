"""The example of a student runs, its gradients are those of the definition, and what its checkpoint holds is its table."""
import math

import pytest
import torch

import paper_2010_08679_amd as P
from examples import distill_student as E
from oracle import losses as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_a_student_is_distilled_and_checkpointed():
    r = E.main(steps=5)
    assert len(r["losses"]) == 5 and all(math.isfinite(v) for v in r["losses"]) and r["errors"] == (P.CNR_OK, 0, 0)
    # 8 bits: 255 steps from a row's smallest value to its largest, each value off by half a step at most
    spread = r["table"].max(dim=1).values - r["table"].min(dim=1).values
    assert bool(((r["table"] - r["resumed"]).abs() <= spread[:, None] * (0.5 / 255 + 1e-5) + 1e-6).all())


def test_its_gradients_are_the_definitions():
    """One step from given tables: the change of the table is the gradient's."""
    ctx = P.cnr_create(0)
    g = torch.Generator(device=DEV).manual_seed(3)
    teacher = [torch.randn(E.VOCAB, E.DIM, generator=g, device=DEV) * 0.1 for _ in range(2)]
    table, turn = torch.randn(E.VOCAB, E.STUDENT, generator=g, device=DEV) * 0.3, torch.randn(E.STUDENT, E.STUDENT, generator=g, device=DEV) * 0.1
    checkpointer = P.TableCheckpointer(ctx, E.VOCAB, E.STUDENT, device=DEV)
    checkpointer.clear()
    before, turned = table.clone(), turn.clone()
    now = torch.randint(0, E.VOCAB, (E.TOKENS,), generator=torch.Generator(device=DEV).manual_seed(7), device=DEV)
    losses = E.distill(ctx, teacher, table, turn, 1, checkpointer, seed=7)
    w, t = before.double().requires_grad_(), turned.double().requires_grad_()
    tokens, logits = E.teachers_top(ctx, *teacher, now)
    z = (w[now] @ t) @ w.t()
    q = R.shares(tokens.long(), E.VOCAB, logits, E.HEAT)
    soft = (q * (q.log() - torch.log_softmax(z / E.HEAT, dim=1).gather(1, tokens.long()))).sum(dim=1)
    hard = torch.nn.functional.cross_entropy(z, (7 * now + 3) % E.VOCAB, reduction="none")
    assert abs(losses[0] - float((soft + hard).detach().mean()) / 2) < 1e-5
    dw, dt = torch.autograd.grad((0.5 * E.HEAT ** 2 * soft + 0.5 * hard).mean(), (w, t))
    # sums of up to 512 products in fp32, and the step's rounding of values of up to 2
    assert float((table - before + 4.0 * dw).abs().max()) < 1e-5 and float((turn - turned + 4.0 * dt).abs().max()) < 1e-5
    P.cnr_destroy(ctx)
