"""Losses over the vocabulary and top logits without a GPU: the header, the binding, every refusal, the workspace's sizes, the oracle's pins."""
import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

import paper_2010_08679_amd as P
from oracle import losses as R
from paper_2010_08679_amd import loss_binding as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, ALIGN, TOO_LARGE = P.CNR_OK, P.CNR_E_INVALID, P.CNR_E_ALIGN, P.CNR_E_TOO_LARGE
F32, BF16, F16 = P.CNR_FLOAT_F32, P.CNR_FLOAT_BF16, P.CNR_FLOAT_F16


def test_header_is_plain_c_and_every_export_links(tmp_path):
    S.load()
    exe, pkg = str(tmp_path / "abi_check"), os.path.join(ROOT, "paper_2010_08679_amd")
    subprocess.check_call(["gcc", "-std=c99", "-pedantic", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "c", "loss_abi_check.c"),
                           "-o", exe, "-L", pkg, "-lcnr", "-Wl,-rpath," + pkg, "-Wl,-rpath,/opt/rocm/lib", "-L/opt/rocm/lib"])
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0, (out.returncode, out.stdout, out.stderr)
    assert int(out.stdout.split(":")[1].split()[0]) == len(S.LOSS_EXPORTS)


def test_binding_names_everything_that_the_header_declares():
    with open(os.path.join(ROOT, "include", "cnr_loss.h")) as f:
        header = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    assert set(re.findall(r"\b(cnr_[a-z_]+)\(", header)) == set(S.LOSS_EXPORTS)
    limits = dict(re.findall(r"#define (CNR_LOSS_MAX_[A-Z]+) (\d+)u", header))
    assert len(limits) == 4 and all(getattr(P, name) == int(value) for name, value in limits.items())


@pytest.mark.parametrize("struct", [P.cnr_vocabulary, P.cnr_targets])
def test_structs_are_laid_out_as_in_c(tmp_path, struct):
    src, exe, name = tmp_path / "s.c", str(tmp_path / "s"), struct.__name__
    names = [f for f, _ in struct._fields_]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "cnr_loss.h"\nint main(void){printf("%%zu", sizeof(%s));' % name +
                   "".join('printf(" %%zu", offsetof(%s, %s));' % (name, n) for n in names) + "return 0;}\n")
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe])
    got = [int(v) for v in subprocess.run([exe], capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(struct)] + [getattr(struct, n).offset for n in names]


# ---- refusals: all of them come before a context's device is looked at ---------------------------------------------------

A = 1 << 20  # an address that is aligned to anything; never read
CTX = ctypes.create_string_buffer(4096)  # a context that no call gets as far as using


def _call(name, **changed):
    """The call's status with good arguments but for `changed`."""
    v = dict(hidden=A, hidden_stride=64, weight=A, weight_stride=64, type=BF16, n=8, vocab=100, dim=64)
    t = dict(tokens=A, token_type=0, token_stride=1, top=1, logits=None, logit_type=0, logit_stride=0, temperature=0.0)
    rest = {
        "cnr_vocabulary_loss": dict(ctx=ctypes.addressof(CTX), v=None, t=None, loss=A, state=A, workspace=A, workspace_bytes=1 << 40, stream=None),
        "cnr_vocabulary_loss_backward": dict(ctx=ctypes.addressof(CTX), v=None, t=None, state=A, dloss=A, dhidden=A, dhidden_stride=64, dweight=A, dweight_type=BF16,
                                             dweight_stride=64, accumulate=0, workspace=A, workspace_bytes=1 << 40, stream=None),
        "cnr_top_logits": dict(ctx=ctypes.addressof(CTX), logits=A, stride=64, type=0, n=8, vocab=64, top=5, tokens=A, values=A, lse=A, stream=None),
    }[name]
    if name != "cnr_top_logits":
        v, t = ({k: changed.pop(k, x) for k, x in d.items()} for d in (v, t))
        rest["v"], rest["t"] = ctypes.byref(P.cnr_vocabulary(**v)), ctypes.byref(P.cnr_targets(**t))
    assert not set(changed) - set(rest), changed
    return getattr(S.load(), name)(*(rest | changed).values())


TEACHER = dict(logits=A, logit_type=F32, logit_stride=4, top=4, token_stride=4, temperature=1.0)
BOTH = [
    (INVALID, dict(ctx=None)), (INVALID, dict(v=None)), (INVALID, dict(t=None)), (INVALID, dict(type=3)), (INVALID, dict(type=-1)), (INVALID, dict(token_type=2)),
    (INVALID, dict(hidden_stride=63)), (INVALID, dict(weight_stride=63)), (INVALID, dict(token_stride=0)), (INVALID, dict(top=2, token_stride=2)), (INVALID, dict(top=0)),
    (INVALID, TEACHER | dict(logit_stride=3)), (INVALID, TEACHER | dict(token_stride=3)), (INVALID, TEACHER | dict(logit_type=3)),
    (INVALID, TEACHER | dict(temperature=0.0)), (INVALID, TEACHER | dict(temperature=-1.0)), (INVALID, TEACHER | dict(temperature=math.nan)),
    (INVALID, TEACHER | dict(temperature=math.inf)), (INVALID, dict(hidden=None)), (INVALID, dict(weight=None)), (INVALID, dict(tokens=None)),
    (INVALID, dict(workspace_bytes=0)), (INVALID, dict(workspace=None)),
    (TOO_LARGE, dict(n=(1 << 20) + 1)), (TOO_LARGE, dict(vocab=(1 << 27) + 1)), (TOO_LARGE, dict(dim=(1 << 20) + 1, hidden_stride=1 << 21, weight_stride=1 << 21)),
    (TOO_LARGE, TEACHER | dict(top=1025, token_stride=1025, logit_stride=1025)),
    (ALIGN, dict(hidden=A + 1)), (ALIGN, dict(weight=A + 1)), (ALIGN, dict(hidden=A + 2, type=F32)), (ALIGN, dict(tokens=A + 2)), (ALIGN, dict(tokens=A + 4, token_type=1)),
    (ALIGN, TEACHER | dict(logits=A + 2)), (ALIGN, dict(workspace=A + 128)), (ALIGN, dict(state=A + 2)),
]


@pytest.mark.parametrize("name,status,changed", [(name, *b) for name in ("cnr_vocabulary_loss", "cnr_vocabulary_loss_backward") for b in BOTH] + [
    ("cnr_vocabulary_loss", INVALID, TEACHER | dict(state=None)), ("cnr_vocabulary_loss", INVALID, dict(loss=None)), ("cnr_vocabulary_loss", ALIGN, dict(loss=A + 1)), ("cnr_vocabulary_loss", OK, dict(n=0, hidden=None, tokens=None)),
    ("cnr_vocabulary_loss_backward", INVALID, dict(state=None)), ("cnr_vocabulary_loss_backward", INVALID, dict(dloss=None)),
    ("cnr_vocabulary_loss_backward", INVALID, dict(dhidden_stride=63)), ("cnr_vocabulary_loss_backward", INVALID, dict(dweight_stride=63)),
    ("cnr_vocabulary_loss_backward", INVALID, dict(dweight_type=F16)), ("cnr_vocabulary_loss_backward", INVALID, dict(dweight_type=BF16, type=F32, dhidden_stride=64)),
    ("cnr_vocabulary_loss_backward", ALIGN, dict(dhidden=A + 1)), ("cnr_vocabulary_loss_backward", ALIGN, dict(dweight=A + 2, dweight_type=F32)),
    ("cnr_vocabulary_loss_backward", ALIGN, dict(dloss=A + 2)), ("cnr_vocabulary_loss_backward", OK, dict(dhidden=None, dweight=None)),
    ("cnr_top_logits", INVALID, dict(ctx=None)), ("cnr_top_logits", INVALID, dict(type=3)), ("cnr_top_logits", INVALID, dict(stride=63)),
    ("cnr_top_logits", INVALID, dict(logits=None)), ("cnr_top_logits", ALIGN, dict(logits=A + 2)), ("cnr_top_logits", ALIGN, dict(tokens=A + 2)),
    ("cnr_top_logits", ALIGN, dict(values=A + 2)), ("cnr_top_logits", ALIGN, dict(lse=A + 1)), ("cnr_top_logits", TOO_LARGE, dict(top=1025)),
    ("cnr_top_logits", TOO_LARGE, dict(vocab=1 << 31, stride=1 << 31)), ("cnr_top_logits", TOO_LARGE, dict(n=1 << 31)), ("cnr_top_logits", OK, dict(n=0)),
    ("cnr_top_logits", OK, dict(top=0, lse=None)), ("cnr_top_logits", OK, dict(tokens=None, values=None, lse=None)),
])
def test_calls_refuse_what_they_cannot_take(name, status, changed):
    assert _call(name, **changed) == status


@pytest.mark.parametrize("type", [F32, BF16, F16])
@pytest.mark.parametrize("training", [False, True])
def test_a_workspace_serves_fewer_rows_as_well(type, training):
    """Sizes grow with the number of rows, and what each call takes of them is checked by the call: these are the borders of its rules."""
    for vocab, dim in ((1, 1), (300, 64), (50257, 1000), (131072, 4096), (1 << 20, 64)):
        sizes = [P.cnr_loss_workspace_bytes(n, vocab, dim, type, training, F32) for n in (1, 2, 15, 16, 17, 31, 64, 65, 255, 256, 257, 1000, 2047, 4096, 16384, 40000, 1 << 20)]
        assert sizes == sorted(sizes) and sizes[0] > 0
    assert P.cnr_loss_workspace_bytes(0, 5, 5, type, training, type) == P.cnr_loss_workspace_bytes(5, 0, 5, type, training, type) == 0
    # far from all logits in memory
    assert P.cnr_loss_workspace_bytes(65536, 262144, 1024, BF16, training, BF16) < 65536 * 262144 * 2 / 8


def test_binding_refuses_host_tensors_wrong_types_and_sizes():
    x, w, t = torch.zeros(4, 8), torch.zeros(10, 8), torch.zeros(4, dtype=torch.int64)
    loss = P.VocabularyLoss(None, 10, 8, 4, torch.float32, top=3, device="cpu")
    with pytest.raises(TypeError):
        loss.cross_entropy(x, w, t)  # not on the GPU
    for bad in ((torch.zeros(4, 7), w), (x, torch.zeros(11, 8)), (torch.zeros(5, 8), w), (torch.zeros(4), w)):
        with pytest.raises(ValueError):
            loss.cross_entropy(*bad, t)
    with pytest.raises(TypeError):
        loss.cross_entropy(x.bfloat16(), w, t)
    with pytest.raises(ValueError):
        loss.distill(x, w, torch.zeros(4, 4, dtype=torch.int64), torch.zeros(4, 4))
    with pytest.raises(ValueError):
        loss.distill(x, w, t, torch.zeros(4))
    with pytest.raises(ValueError):
        loss.backward(torch.zeros(4))
    with pytest.raises(ValueError):
        P.VocabularyLoss(None, 10, 8, 4, torch.float32, training=False, device="cpu").cross_entropy(x, w, t)
    with pytest.raises(TypeError):
        P.VocabularyLoss(None, 10, 8, 4, torch.float64, device="cpu")
    with pytest.raises(TypeError):
        P.VocabularyLoss(None, 10, 8, 4, torch.bfloat16, gradient_dtype=torch.float16, device="cpu")
    for top in (0, 1025):
        with pytest.raises(ValueError):
            P.VocabularyLoss(None, 10, 8, 4, top=top, device="cpu")
    for sizes in ((11, 8, (1 << 20) + 1), ((1 << 27) + 1, 8, 4), (10, (1 << 20) + 1, 4), (-1, 8, 4)):
        with pytest.raises(ValueError):
            P.VocabularyLoss(None, *sizes, device="cpu")
    with pytest.raises(TypeError):
        P.top_logits(None, x, 2)
    loss._last = (x, w, t, None, 1.0)
    with pytest.raises(ValueError):
        loss.backward(torch.zeros(4), accumulate=True)
    with pytest.raises(TypeError):
        loss.backward(torch.zeros(4), dweight=torch.zeros(10, 8, dtype=torch.bfloat16))


# ---- the oracle's pins --------------------------------------------------------------------------------------------------

def test_oracle_losses_are_torchs():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(9, 12, generator=g, dtype=torch.float64).float().requires_grad_()
    w = torch.randn(30, 12, generator=g, dtype=torch.float64).float().requires_grad_()
    targets = torch.randint(0, 30, (9,), generator=g)
    targets[2], targets[5] = -100, 30
    each = torch.rand(9, generator=g)
    z = x.double() @ w.double().t()
    want = torch.nn.functional.cross_entropy(z, torch.where(targets == 30, -100, targets), reduction="none")
    grads = torch.autograd.grad((want * each).sum(), (x, w), retain_graph=True)
    got = R.loss(x.detach(), w.detach(), targets, dloss=each)
    assert torch.allclose(got["losses"][0], want, atol=1e-12)
    for name, v in zip(("dhidden", "dweight"), grads):
        assert torch.allclose(got[name][0].float(), v, atol=1e-6)
    tokens, logits = torch.randint(-1, 30, (9, 5), generator=g), torch.randn(9, 5, generator=g)
    tokens[4] = -1
    tokens[3, 1] = tokens[3, 0] = 7
    q = torch.softmax(torch.where(tokens >= 0, logits.double() / 2, -math.inf), dim=1).nan_to_num()
    full = torch.zeros(9, 30, dtype=torch.float64).scatter_add_(1, tokens.clamp(min=0), q)
    log_p = torch.log_softmax(z / 2, dim=1)
    want = (torch.where(q > 0, q * q.log(), 0.0)).sum(1) - (full * log_p).sum(1)
    grads = torch.autograd.grad((want * each).sum(), (x, w))
    got = R.loss(x.detach(), w.detach(), tokens, logits, 2.0, each)
    assert torch.allclose(got["losses"][0], want, atol=1e-12)
    for name, v in zip(("dhidden", "dweight"), grads):
        assert torch.allclose(got[name][0].float(), v, atol=1e-6)


def test_oracle_top_by_hand():
    v = torch.tensor([[1.0, math.nan, -0.0, 0.0, math.inf, -math.inf, 1.0]])
    tokens, values, lse = R.top(v, 9)
    assert tokens.tolist() == [[1, 4, 0, 6, 2, 3, 5, -1, -1]] and math.isnan(float(lse)) and values[0, -1] == -math.inf


@pytest.mark.parametrize("name", ["cnr_vocabulary_loss", "cnr_vocabulary_loss_backward"])
@pytest.mark.parametrize("temperature", [2.0 ** -127, 1e-39, 2.0 ** -149, -0.0, 3.2e38])
def test_temperatures_that_1_cannot_be_divided_by_are_refused(name, temperature):
    """Below 2^-126 log2(e) / T is infinite, and a logit of 0 would be NaN."""
    assert _call(name, **(TEACHER | dict(temperature=temperature))) == INVALID
    # (what comes after the temperature's check)
    assert _call(name, **(TEACHER | dict(temperature=2.0 ** -126, tokens=A + 2))) == ALIGN


def test_plans_at_the_limits_of_the_sizes(tmp_path):
    """What the calls ask for of grids and workspaces, computed on the CPU from their own header."""
    exe = str(tmp_path / "loss_plan")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-D__HIP_PLATFORM_AMD__", "-isystem", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"),
                           "-I", os.path.join(ROOT, "paper_2010_08679_amd", "csrc"), os.path.join(ROOT, "tests", "c", "loss_plan.cpp"), "-o", exe])
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout + out.stderr


def test_places_that_share_bytes():
    """Matrices in one memory, against the sets of their bytes."""
    g = torch.Generator().manual_seed(1)

    def place():
        n, width, gap, at = (int(torch.randint(lo, hi, (), generator=g)) for lo, hi in ((1, 6), (1, 8), (0, 9), (0, 40)))
        return at, n, width, width + gap if n > 1 else int(torch.randint(0, 9, (), generator=g))

    def held(p):
        at, n, width, step = p
        return {at + i * step + j for i in range(n) for j in range(width)}

    same = together = 0
    for _ in range(4000):
        a, b = place(), place()
        if torch.randint(0, 2, (), generator=g) and a[1] > 1 and b[1] > 1 and a[3] >= b[2]:
            b = (*b[:3], a[3])  # rows of one matrix
            same += 1
        share = bool(held(a) & held(b))
        together += share
        assert S._share(a, b) == S._share(b, a) == share, (a, b)
    assert same > 300 and 500 < together < 3500
    assert not S._share((0, 0, 1, 1), (0, 1, 1, 1)) and not S._share((0, 1, 1, 1), (0, 4, 0, 1))
    # large ones in no more time
    assert not S._share((0, 1 << 20, 64, 128), (64, 1 << 20, 64, 128)) and S._share((0, 1 << 20, 64, 128), (63, 1 << 20, 64, 128))


def test_a_refused_loss_leaves_the_one_before_to_its_backward_pass():
    x, w, t = torch.zeros(4, 8), torch.zeros(10, 8), torch.zeros(4, dtype=torch.int64)
    loss = P.VocabularyLoss(None, 10, 8, 4, torch.float32, top=3, device="cpu")
    loss._last = before = (x, w, t, None, 1.0)
    for call in (lambda: loss.cross_entropy(x, w, t), lambda: loss.distill(x, w, t[:, None], torch.zeros(4, 1)), lambda: loss.cross_entropy(x, w, t, training=False),
                 lambda: loss.cross_entropy(x.half(), w, t), lambda: loss.cross_entropy(x, w[:9], t)):
        with pytest.raises((TypeError, ValueError)):
            call()
        assert loss._last is before
