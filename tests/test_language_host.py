"""CPU-side checks of the operators for language models: exports and constants of the header, refusals of the C calls and of
the binding, sizes, and the oracle's own pins.  No kernel is launched here."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import paper_2010_08679_amd as P
from oracle import blocks as R
from paper_2010_08679_amd import build, lm_binding as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, ALIGN, TOO_LARGE = P.CNR_OK, P.CNR_E_INVALID, P.CNR_E_ALIGN, P.CNR_E_TOO_LARGE


def _header():
    text = open(os.path.join(ROOT, "include", "cnr_lm.h")).read()
    return re.sub(r"/\*.*?\*/", "", text, flags=re.S)


def test_library_exports_every_declared_symbol():
    declared = sorted(set(re.findall(r"\b(cnr_[a-z0-9_]+)\s*\(", _header())))
    assert sorted(L.LM_EXPORTS) == declared
    for name in declared:
        assert hasattr(L.load(), name) and callable(getattr(P, name)), name


def test_binding_constants_equal_the_header():
    header = {k: int(v) for k, v in re.findall(r"(CNR_[A-Z0-9_]+)\s*=\s*(\d+)", _header())}
    header |= {k: int(v) for k, v in re.findall(r"#define\s+(CNR_[A-Z0-9_]+)\s+(\d+)u?\s*$", _header(), flags=re.M)}
    assert len(header) >= 9
    for name, value in header.items():
        assert getattr(P, name) == value, name


def test_header_is_plain_c_and_every_export_links(tmp_path):
    L.load()
    exe, pkg = str(tmp_path / "abi_check"), os.path.join(ROOT, "paper_2010_08679_amd")
    subprocess.check_call(["gcc", "-std=c99", "-pedantic", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"),
                           os.path.join(ROOT, "tests", "c", "lm_abi_check.c"), "-o", exe, "-L", pkg, "-lcnr",
                           "-Wl,-rpath," + pkg, "-Wl,-rpath,/opt/rocm/lib", "-L/opt/rocm/lib"])
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0, (out.returncode, out.stdout, out.stderr)
    assert int(out.stdout.split(":")[1].split()[0]) == len(L.LM_EXPORTS)


def test_adjustments_are_laid_out_as_in_c(tmp_path):
    src, exe = tmp_path / "s.c", str(tmp_path / "s")
    names = [f for f, _ in P.cnr_adjustments._fields_]
    src.write_text('#include <stdio.h>\n#include "cnr_lm.h"\nint main(void){printf("%zu", sizeof(cnr_adjustments));' +
                   "".join('printf(" %%zu", offsetof(cnr_adjustments, %s));' % n for n in names) + "return 0;}\n")
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe])
    got = [int(v) for v in subprocess.run([exe], capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(P.cnr_adjustments)] + [getattr(P.cnr_adjustments, n).offset for n in names]


def test_nans_count_where_they_are_ordinary_inputs():
    for s in build.sources():
        flags = build.flags_of(s)
        assert ("-fno-honor-nans" in flags) == (not os.path.basename(s).startswith("lm_")), s
        assert "-packed-fp32-ops" in flags and "-ffp-contract=off" in flags


# ---- refusals: all of them come before a context's device is looked at ---------------------------------------------------

A = 1 << 20  # an address that is aligned to anything; never read


def _call(name, **changed):
    """The call's status with good arguments but for `changed`, on a context that no call gets as far as using."""
    ctx = ctypes.addressof(_call.ctx)
    good = {
        "cnr_quantize_blocks": dict(ctx=ctx, x=A, type=0, n_rows=8, dim=64, stride=64, kind=0, scale_type=0, codes=A, scale=A, codes_t=A, scale_t=A, stream=None),
        "cnr_block_product": dict(ctx=ctx, a_codes=A, a_scale=A, a_kind=0, m=8, b_codes=A, b_scale=A, b_kind=1, n=8, k=64, scale_type=0, out=A, out_type=0,
                                  out_stride=8, accumulate=0, workspace=A, stream=None),
        "cnr_count_tokens": dict(ctx=ctx, seen=A, counts=A, n_slots=4, vocab=99, tokens=A, n_tokens=4, type=0, offsets=A, slots=A, n=4, prompt=0, restart=0,
                                 stream=None),
        "cnr_adjust_logits": dict(ctx=ctx, logits=A, stride=64, out=2 * A, out_stride=64, type=0, n=2, vocab=64, adjustments=P.cnr_adjustments(), stream=None),
    }[name]
    assert not set(changed) - set(good), changed
    return getattr(L.load(), name)(*(good | changed).values())


_call.ctx = ctypes.create_string_buffer(4096)


@pytest.mark.parametrize("name,status,changed", [
    ("cnr_quantize_blocks", INVALID, dict(ctx=None)), ("cnr_quantize_blocks", INVALID, dict(type=3)), ("cnr_quantize_blocks", INVALID, dict(kind=2)),
    ("cnr_quantize_blocks", INVALID, dict(kind=-1)), ("cnr_quantize_blocks", INVALID, dict(scale_type=2)), ("cnr_quantize_blocks", INVALID, dict(stride=63)),
    ("cnr_quantize_blocks", INVALID, dict(x=None)), ("cnr_quantize_blocks", INVALID, dict(scale=None)), ("cnr_quantize_blocks", INVALID, dict(codes_t=None)),
    ("cnr_quantize_blocks", INVALID, dict(codes=None, scale=None, codes_t=None, scale_t=None)),
    ("cnr_quantize_blocks", ALIGN, dict(x=A + 2)), ("cnr_quantize_blocks", ALIGN, dict(x=A + 1, type=1)), ("cnr_quantize_blocks", ALIGN, dict(codes=A + 8)),
    ("cnr_quantize_blocks", ALIGN, dict(scale=A + 4)), ("cnr_quantize_blocks", ALIGN, dict(codes_t=A + 1)), ("cnr_quantize_blocks", ALIGN, dict(scale_t=A + 1)),
    ("cnr_quantize_blocks", TOO_LARGE, dict(n_rows=1 << 31)), ("cnr_quantize_blocks", TOO_LARGE, dict(dim=1 << 31, stride=1 << 31)),
    ("cnr_quantize_blocks", TOO_LARGE, dict(n_rows=1 << 30, dim=1 << 12, stride=1 << 12)),
    ("cnr_quantize_blocks", OK, dict(n_rows=0, x=None)), ("cnr_quantize_blocks", OK, dict(dim=0)),
    ("cnr_block_product", INVALID, dict(ctx=None)), ("cnr_block_product", INVALID, dict(out_type=7)), ("cnr_block_product", INVALID, dict(a_kind=5)),
    ("cnr_block_product", INVALID, dict(b_kind=-1)), ("cnr_block_product", INVALID, dict(scale_type=-1)), ("cnr_block_product", INVALID, dict(out_stride=7)),
    ("cnr_block_product", INVALID, dict(out=None)), ("cnr_block_product", INVALID, dict(a_codes=None)), ("cnr_block_product", INVALID, dict(b_scale=None)),
    ("cnr_block_product", ALIGN, dict(a_codes=A + 8)), ("cnr_block_product", ALIGN, dict(b_codes=A + 1)), ("cnr_block_product", ALIGN, dict(a_scale=A + 2)),
    ("cnr_block_product", ALIGN, dict(b_scale=A + 8)), ("cnr_block_product", ALIGN, dict(out=A + 2)), ("cnr_block_product", ALIGN, dict(workspace=A + 8)),
    ("cnr_block_product", TOO_LARGE, dict(m=1 << 31)), ("cnr_block_product", TOO_LARGE, dict(n=1 << 31, out_stride=1 << 31)),
    ("cnr_block_product", TOO_LARGE, dict(k=1 << 31)), ("cnr_block_product", TOO_LARGE, dict(m=1 << 20, n=1 << 20, out_stride=1 << 20)),
    ("cnr_block_product", TOO_LARGE, dict(m=1 << 20, k=1 << 24)),
    ("cnr_block_product", OK, dict(m=0)), ("cnr_block_product", OK, dict(n=0)), ("cnr_block_product", OK, dict(k=0, accumulate=1)),
    ("cnr_count_tokens", INVALID, dict(ctx=None)), ("cnr_count_tokens", INVALID, dict(type=2)), ("cnr_count_tokens", INVALID, dict(seen=None)),
    ("cnr_count_tokens", INVALID, dict(tokens=None)), ("cnr_count_tokens", INVALID, dict(offsets=None, n=3)),
    ("cnr_count_tokens", ALIGN, dict(seen=A + 2)), ("cnr_count_tokens", ALIGN, dict(counts=A + 1)), ("cnr_count_tokens", ALIGN, dict(tokens=A + 4, type=1)),
    ("cnr_count_tokens", ALIGN, dict(offsets=A + 4)), ("cnr_count_tokens", ALIGN, dict(slots=A + 2)),
    ("cnr_count_tokens", TOO_LARGE, dict(vocab=1 << 31)), ("cnr_count_tokens", TOO_LARGE, dict(n=1 << 31)), ("cnr_count_tokens", TOO_LARGE, dict(n_tokens=1 << 31)),
    ("cnr_count_tokens", TOO_LARGE, dict(n_slots=1 << 31)), ("cnr_count_tokens", OK, dict(n=0)),
    ("cnr_adjust_logits", INVALID, dict(ctx=None)), ("cnr_adjust_logits", INVALID, dict(adjustments=None)), ("cnr_adjust_logits", INVALID, dict(type=3)),
    ("cnr_adjust_logits", INVALID, dict(stride=63)), ("cnr_adjust_logits", INVALID, dict(out_stride=63)), ("cnr_adjust_logits", INVALID, dict(logits=None)),
    ("cnr_adjust_logits", INVALID, dict(out=None)), ("cnr_adjust_logits", INVALID, dict(out=A, out_stride=65)),
    ("cnr_adjust_logits", INVALID, dict(adjustments=P.cnr_adjustments(bias_offsets=A, n_bias=3, bias_tokens=A))),
    ("cnr_adjust_logits", ALIGN, dict(logits=A + 1)), ("cnr_adjust_logits", ALIGN, dict(out=A + 2)),
    ("cnr_adjust_logits", ALIGN, dict(adjustments=P.cnr_adjustments(masks=A + 2, n_masks=2))),
    ("cnr_adjust_logits", ALIGN, dict(adjustments=P.cnr_adjustments(bias_offsets=A + 4))),
    ("cnr_adjust_logits", TOO_LARGE, dict(vocab=1 << 31, stride=1 << 31, out_stride=1 << 31)), ("cnr_adjust_logits", TOO_LARGE, dict(n=1 << 31)),
    ("cnr_adjust_logits", OK, dict(n=0)), ("cnr_adjust_logits", OK, dict(vocab=0)),
])
def test_calls_refuse_what_they_cannot_take(name, status, changed):
    assert _call(name, **changed) == status


def test_binding_refuses_host_tensors_wrong_types_and_sizes():
    x = torch.zeros(8, 200)
    with pytest.raises(TypeError):
        P.quantize_blocks(None, x, P.BlockMatrix.empty(8, 200, device="cpu"))
    with pytest.raises(ValueError):
        P.quantize_blocks(None, x, P.BlockMatrix.empty(8, 201, device="cpu"))
    with pytest.raises(ValueError):
        P.quantize_blocks(None, x, P.BlockMatrix.empty(8, 200, device="cpu"), P.BlockMatrix.empty(200, 8, P.CNR_BLOCK_TILE, device="cpu"))
    with pytest.raises(ValueError):
        P.quantize_blocks(None, x, P.BlockMatrix.empty(8, 200, device="cpu"), P.BlockMatrix.empty(200, 8, scale_type=P.CNR_SCALE_F32, device="cpu"))
    a, b = P.BlockMatrix.empty(4, 100, device="cpu"), P.BlockMatrix.empty(6, 101, device="cpu")
    with pytest.raises(ValueError):
        P.block_product(None, a, b)
    b = P.BlockMatrix.empty(6, 100, device="cpu")
    with pytest.raises(ValueError):
        P.block_product(None, a, b, torch.empty(4, 7))
    with pytest.raises(ValueError):
        P.block_product(None, a, b, accumulate=True)
    with pytest.raises(TypeError):
        P.block_product(None, a, b, torch.empty(4, 6))
    with pytest.raises(ValueError):
        L._blocked(a.codes[:3], a.scale, 4, 100, 0, 0, "A")
    with pytest.raises(ValueError):
        L._blocked(a.codes, a.scale, 4, 100, 3, 0, "A")
    with pytest.raises(ValueError):
        L._listed(torch.zeros(3), 4, torch.float32, "presence")
    ledger = P.TokenLedger(None, 2, 40, device="cpu")
    with pytest.raises(TypeError):
        ledger.count(torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        ledger.adjust(torch.zeros(2, 41))
    with pytest.raises(TypeError):
        ledger.adjust(torch.zeros(2, 40))
    layer = P.BlockLinear(None, 6, 4, 3, device="cpu")
    with pytest.raises(ValueError):
        layer.forward(torch.zeros(4, 4))
    with pytest.raises(ValueError):
        layer.backward(torch.zeros(3, 6))


def test_sizes_of_blocked_matrices():
    for rows in (0, 1, 127, 128, 129, 1000):
        for dim in (0, 1, 128, 300):
            for kind in (P.CNR_BLOCK_ROW, P.CNR_BLOCK_TILE):
                for scale, dtype in ((P.CNR_SCALE_E8M0, torch.uint8), (P.CNR_SCALE_F32, torch.float32)):
                    m = P.BlockMatrix.empty(rows, dim, kind, scale, "cpu")
                    assert m.codes.shape == (rows, P.cnr_block_row_bytes(dim)) and m.scale_type == scale and m.scale.dtype == dtype
                    assert m.scale.shape[1] == P.cnr_block_scale_stride(rows, kind) and m.scale.numel() == P.cnr_block_scale_count(rows, dim, kind)


# ---- the oracle's pins --------------------------------------------------------------------------------------------------

def test_oracle_codes_equal_torch_casts():
    x = torch.cat([torch.tensor(R.E4M3[:127]).float(), torch.linspace(-448, 448, 9001), torch.randn(5000)])
    assert np.array_equal(R.encode(x.double().numpy()), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert np.array_equal(R.encode(R.E4M3[:127]), np.arange(127)) and list(R.encode(np.array([np.nan, np.inf, -0.0]))) == [127, 127, 128]


def test_oracle_scales_by_hand():
    amax = np.array([0.0, 448.0, 448.0000001, 1.75, 1.7500001, 1.0, 2.0 ** -140, 3.4e38])
    assert list(np.log2(R.scales(amax, "e8m0"))) == [0, 0, 1, -8, -7, -8, -126, 120]
    assert list(R.scales(amax[[0, 1, 6]], "f32")) == [1.0, 1.0, 2.0 ** -126]


def test_oracle_values_come_back():
    x = np.random.default_rng(1).normal(0, 3, (150, 200))
    for kind in ("row", "tile"):
        for scale in ("e8m0", "f32"):
            codes, s = R.quantize(x, kind, scale)
            back = R.values(codes, s, kind)[:, :200]
            each = (s.T if kind == "row" else s.T.repeat(128, axis=0)[:150]).repeat(128, axis=1)[:, :200]
            assert np.all(np.abs(back - x) <= np.maximum(np.abs(x) * 2.0 ** -4, each * 2.0 ** -10) * (1 + 1e-12))
