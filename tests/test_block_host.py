"""The calls of the gated block, dropout and the verification of drafted tokens refuse what they must before any CUDA call is
made, and lm.py packs their descriptors as the header lays them out.  No kernel is launched here."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

import block_reference as R
from paper_2005_06728_b200 import binding, build, lm
from test_lm_host import err, offsets

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GATED = ("x w_gate w_up h gate up dx dw_gate dw_up type weight_type dw_type activation accumulate n_outer n_inner dim width "
         "x_stride_outer x_stride_inner h_stride_outer h_stride_inner gate_stride_outer gate_stride_inner up_stride_outer up_stride_inner "
         "dx_stride_outer dx_stride_inner w_gate_stride w_up_stride dw_gate_stride dw_up_stride").split()
DROPOUT = ("x residual out counter type out_type n_outer n_inner dim x_stride_outer x_stride_inner residual_stride_outer "
           "residual_stride_inner out_stride_outer out_stride_inner seed offset p").split()
VERIFY = ("target draft tokens uniforms out_tokens accepted logp type token_type batch drafts vocab target_stride_batch "
          "target_stride_row draft_stride_batch draft_stride_row token_stride_batch token_stride_row uniform_stride_batch "
          "uniform_stride_row inv_temp draft_inv_temp").split()


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def native(fmt):
    """The native format as offsets() reads it."""
    return fmt.replace("Q", "q").replace("d", "q")


@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not available")
def test_descriptors_are_packed_as_the_header_lays_them_out(tmp_path):
    src = tmp_path / "layout.c"
    body = ""
    for name, fields in (("odsgd_gated_desc", GATED), ("odsgd_dropout_desc", DROPOUT), ("odsgd_verify_desc", VERIFY)):
        body += "".join(f'printf("%zu ", offsetof({name}, {f}));\n' for f in fields)
        body += f'printf("%zu\\n", sizeof({name}));\n'
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "odsgd.h"\nint main(void) {\n' + body + "return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", f"-I{os.path.join(ROOT, 'include')}", str(src), "-o", str(exe)], check=True)
    lines = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines()
    for line, packed, fields in zip(lines, (lm._GATED, lm._DROPOUT, lm._VERIFY), (GATED, DROPOUT, VERIFY)):
        *want, size = map(int, line.split())
        got, end = offsets(native(packed.format))
        assert got == want and end == size == packed.size and len(got) == len(fields)


def test_constants_match_the_header():
    text = open(os.path.join(ROOT, "include", "odsgd.h")).read()
    assert "#define ODSGD_SILU 0" in text and "#define ODSGD_GELU 1" in text and lm._ACTIVATIONS == {"silu": 0, "gelu": 1}
    assert "#define ODSGD_MAX_DRAFTS 255" in text


def test_no_load_of_the_read_only_path():
    for name in os.listdir(build.CSRC):
        if name.startswith(("odsgd_lm", "odsgd_gated", "odsgd_dropout", "odsgd_verify")):
            text = open(os.path.join(build.CSRC, name)).read()
            assert "__ldg" not in text and "global.nc" not in text, name
            if "__global__" in text:
                assert text.count("__global__") <= text.count("dependent_launch_prologue();"), name


# addresses that are never dereferenced: the checks only look at their values
GOOD_GATED = dict(x=0x1000000, w_gate=0x2000000, w_up=0x2100000, h=0x3000000, gate=0x3100000, up=0x3200000, dx=0x4000000, dw_gate=0x5000000,
                  dw_up=0x5100000, type=lm.BF16, weight_type=lm.BF16, dw_type=lm.F32, activation=0, accumulate=0, n_outer=4, n_inner=8, dim=64,
                  width=96, x_stride_outer=512, x_stride_inner=64, h_stride_outer=768, h_stride_inner=96, gate_stride_outer=768,
                  gate_stride_inner=96, up_stride_outer=768, up_stride_inner=96, dx_stride_outer=512, dx_stride_inner=64, w_gate_stride=64,
                  w_up_stride=64, dw_gate_stride=64, dw_up_stride=64)


def gated(**over):
    d = dict(GOOD_GATED, **over)
    return lm._GATED.pack(*[d[f] for f in GATED])


WS = ctypes.c_void_p(0x6000000)
BOTH = [
    (dict(type=lm.F32), binding.ERR_ARG, "type"),
    (dict(type=9), binding.ERR_ARG, "type"),
    (dict(weight_type=lm.F16), binding.ERR_ARG, "weight_type"),
    (dict(activation=2), binding.ERR_ARG, "activation"),
    (dict(n_outer=-1), binding.ERR_ARG, "negative"),
    (dict(n_outer=1 << 62, n_inner=1 << 62), binding.ERR_UNSUPPORTED, "tokens"),
    (dict(n_outer=1 << 13, n_inner=1 << 12), binding.ERR_UNSUPPORTED, "tokens"),
    (dict(dim=0), binding.ERR_ARG, "dim"),
    (dict(width=0), binding.ERR_ARG, "width"),
    (dict(width=(1 << 20) + 1), binding.ERR_UNSUPPORTED, "limits"),
    (dict(w_gate_stride=63), binding.ERR_ARG, "stride"),
    (dict(w_up_stride=63), binding.ERR_ARG, "stride"),
    (dict(gate=0), binding.ERR_ARG, "gate"),
    (dict(x=0), binding.ERR_ARG, "x is NULL"),
    (dict(w_up=0), binding.ERR_ARG, "w_up"),
    (dict(x=0x1000001), binding.ERR_ALIGN, "x"),
    (dict(w_gate=0x2000001), binding.ERR_ALIGN, "w_gate"),
    (dict(x_stride_outer=-1), binding.ERR_ARG, "stride"),
    (dict(x_stride_outer=1 << 62), binding.ERR_UNSUPPORTED, "address range"),
]


@pytest.mark.parametrize("over,code,word", BOTH)
def test_gated_calls_refuse(lib, over, code, word):
    need = ctypes.c_size_t()
    for backward, call in ((0, lib.odsgd_gated_forward), (1, lib.odsgd_gated_backward)):
        assert lib.odsgd_gated_workspace(gated(**over), backward, ctypes.byref(need)) == code and word in err(lib)
        assert call(gated(**over), WS, 1 << 30, None) == code and word in err(lib)


@pytest.mark.parametrize("over,code,word", [
    (dict(dx=0, dw_gate=0, dw_up=0), binding.ERR_ARG, "wanted"),
    (dict(dw_gate=0), binding.ERR_ARG, "together"),
    (dict(dw_type=lm.F16), binding.ERR_ARG, "dw_type"),
    (dict(dw_type=lm.BF16, accumulate=1), binding.ERR_ARG, "added"),
    (dict(dw_up_stride=63), binding.ERR_ARG, "stride"),
    (dict(gate=0, up=0), binding.ERR_ARG, "gate"),
    (dict(dx=0x1000000), binding.ERR_OVERLAP, "dx overlaps x"),
    (dict(dx=0x3100000), binding.ERR_OVERLAP, "dx"),
    (dict(dw_gate=0x2000000), binding.ERR_OVERLAP, "dw_gate"),
    (dict(dw_gate=0x5100000), binding.ERR_OVERLAP, "dw_gate"),
    (dict(dw_gate=0x1000000), binding.ERR_OVERLAP, "dw_gate overlaps x"),
    (dict(dx=0x2000000), binding.ERR_OVERLAP, "w_gate overlaps dx"),
    (dict(dx_stride_inner=32), binding.ERR_OVERLAP, "rows"),
    (dict(dw_gate=0x5000002), binding.ERR_ALIGN, "dw_gate"),
])
def test_gated_backward_refuses(lib, over, code, word):
    assert lib.odsgd_gated_backward(gated(**over), WS, 1 << 30, None) == code and word in err(lib)


def test_gated_forward_overlaps_and_workspace(lib):
    for over in (dict(h=0x1000000), dict(h=0x2000000), dict(gate=0x3000000), dict(up=0x3100000), dict(h_stride_inner=95), dict(h_stride_outer=0)):
        assert lib.odsgd_gated_forward(gated(**over), WS, 1 << 30, None) == binding.ERR_OVERLAP
    need = ctypes.c_size_t(7)
    assert lib.odsgd_gated_workspace(gated(), 0, ctypes.byref(need)) == binding.OK and need.value == 0
    assert lib.odsgd_gated_workspace(gated(), 0, None) == binding.ERR_ARG
    assert lib.odsgd_gated_workspace(None, 0, ctypes.byref(need)) == binding.ERR_ARG
    # weights of 32 bits, unaligned weights, rows of x that do not fold: laid out
    for over, size in ((dict(weight_type=lm.F32), 2 * 96 * 64 * 2), (dict(w_gate_stride=65), 96 * 64 * 2), (dict(x=0x1000002), 32 * 64 * 2),
                       (dict(x_stride_outer=1024), 32 * 64 * 2), (dict(x_stride_inner=0, x_stride_outer=0), 32 * 64 * 2)):
        assert lib.odsgd_gated_workspace(gated(**over), 0, ctypes.byref(need)) == binding.OK and need.value == size
        assert lib.odsgd_gated_forward(gated(**over), WS, size - 1, None) == binding.ERR_ARG and "workspace" in err(lib)
        assert lib.odsgd_gated_forward(gated(**over), None, 0, None) == binding.ERR_ARG and "workspace" in err(lib)
        assert lib.odsgd_gated_forward(gated(**over), ctypes.c_void_p(0x6000008), 1 << 30, None) == binding.ERR_ALIGN
        assert lib.odsgd_gated_forward(gated(**over), ctypes.c_void_p(0x3000000), 1 << 30, None) == binding.ERR_OVERLAP
    assert lib.odsgd_gated_workspace(gated(), 1, ctypes.byref(need)) == binding.OK and need.value == 2 * 32 * 128 * 2
    assert lib.odsgd_gated_backward(gated(), ctypes.c_void_p(0x4000000), 1 << 30, None) == binding.ERR_OVERLAP
    # without tokens nothing is launched, nor with gradients that are only added to
    assert lib.odsgd_gated_forward(gated(n_outer=0, x=0, h=0, gate=0, up=0), None, 0, None) == binding.OK
    assert lib.odsgd_gated_backward(gated(n_inner=0, accumulate=1), None, 0, None) == binding.OK


GOOD_DROPOUT = dict(x=0x1000000, residual=0x2000000, out=0x3000000, counter=0, type=lm.BF16, out_type=lm.F32, n_outer=4, n_inner=8, dim=40,
                    x_stride_outer=320, x_stride_inner=40, residual_stride_outer=320, residual_stride_inner=40, out_stride_outer=320,
                    out_stride_inner=40, seed=1, offset=2, p=0.25)


def dropout(**over):
    d = dict(GOOD_DROPOUT, **over)
    return lm._DROPOUT.pack(*[d[f] for f in DROPOUT])


@pytest.mark.parametrize("over,code,word", [
    (dict(type=lm.I32), binding.ERR_ARG, "type"),
    (dict(out_type=7), binding.ERR_ARG, "out_type"),
    (dict(n_inner=-1), binding.ERR_ARG, "negative"),
    (dict(n_outer=1 << 62, n_inner=1 << 62), binding.ERR_UNSUPPORTED, "rows"),
    (dict(dim=0), binding.ERR_ARG, "dim"),
    (dict(dim=(1 << 20) + 1), binding.ERR_UNSUPPORTED, "dim"),
    (dict(p=-1e-9), binding.ERR_ARG, "p must"),
    (dict(p=1.0), binding.ERR_ARG, "p must"),
    (dict(p=65535.6 / 65536), binding.ERR_ARG, "p must"),
    (dict(p=float("nan")), binding.ERR_ARG, "p must"),
    (dict(counter=0x5000004), binding.ERR_ALIGN, "counter"),
    (dict(counter=0x3000008), binding.ERR_OVERLAP, "counter"),
    (dict(x=0), binding.ERR_ARG, "x is NULL"),
    (dict(out=0), binding.ERR_ARG, "out is NULL"),
    (dict(x=0x1000001), binding.ERR_ALIGN, "x"),
    (dict(residual=0x2000002), binding.ERR_ALIGN, "residual"),
    (dict(out=0x1000000), binding.ERR_OVERLAP, "out overlaps x"),
    (dict(out=0x2000004), binding.ERR_OVERLAP, "out overlaps residual"),
    (dict(out=0x2000000, out_stride_inner=44, out_stride_outer=400), binding.ERR_OVERLAP, "out overlaps residual"),
    (dict(out=0x1000004, type=lm.F32), binding.ERR_OVERLAP, "out overlaps x"),
    (dict(out_stride_inner=39), binding.ERR_OVERLAP, "rows"),
    (dict(x_stride_inner=-40), binding.ERR_ARG, "stride"),
])
def test_dropout_refuses(lib, over, code, word):
    assert lib.odsgd_dropout(dropout(**over), None) == code and word in err(lib)


def test_dropout_without_rows(lib):
    assert lib.odsgd_dropout(dropout(n_outer=0, x=0, residual=0, out=0), None) == binding.OK
    assert lib.odsgd_dropout(None, None) == binding.ERR_ARG


def test_philox_known_answers():
    """The published test vectors of Philox4x32-10."""
    assert R.philox(0, 0, 0) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = (1 << 64) - 1
    assert R.philox(ones, ones, ones) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert R.philox(0x85A308D3243F6A88, 0x0370734413198A2E, 0x299F31D0A4093822) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


GOOD_VERIFY = dict(target=0x1000000, draft=0x2000000, tokens=0x3000000, uniforms=0x3100000, out_tokens=0x4000000, accepted=0x4100000, logp=0x4200000,
                   type=lm.BF16, token_type=lm.I64, batch=4, drafts=3, vocab=1000, target_stride_batch=4000, target_stride_row=1000,
                   draft_stride_batch=3000, draft_stride_row=1000, token_stride_batch=3, token_stride_row=1, uniform_stride_batch=4,
                   uniform_stride_row=1, inv_temp=1.0, draft_inv_temp=1.0)


def verify(**over):
    d = dict(GOOD_VERIFY, **over)
    return lm._VERIFY.pack(*[d[f] for f in VERIFY])


@pytest.mark.parametrize("over,code,word", [
    (dict(type=lm.I64), binding.ERR_ARG, "type"),
    (dict(token_type=lm.F32), binding.ERR_ARG, "token_type"),
    (dict(batch=-1), binding.ERR_ARG, "negative"),
    (dict(drafts=-1), binding.ERR_ARG, "negative"),
    (dict(vocab=0), binding.ERR_ARG, "vocab"),
    (dict(drafts=256), binding.ERR_UNSUPPORTED, "limits"),
    (dict(batch=(1 << 16) + 1), binding.ERR_UNSUPPORTED, "limits"),
    (dict(vocab=(1 << 30) + 1), binding.ERR_UNSUPPORTED, "limits"),
    (dict(inv_temp=0.0), binding.ERR_ARG, "inv_temp"),
    (dict(inv_temp=float("inf")), binding.ERR_ARG, "inv_temp"),
    (dict(draft_inv_temp=float("nan")), binding.ERR_ARG, "inv_temp"),
    (dict(target=0), binding.ERR_ARG, "target"),
    (dict(tokens=0), binding.ERR_ARG, "tokens"),
    (dict(uniforms=0), binding.ERR_ARG, "uniforms"),
    (dict(accepted=0), binding.ERR_ARG, "accepted"),
    (dict(logp=0), binding.ERR_ARG, "logp"),
    (dict(out_tokens=0x4000004), binding.ERR_ALIGN, "out_tokens"),
    (dict(draft=0x2000001), binding.ERR_ALIGN, "draft"),
    (dict(target_stride_row=-1), binding.ERR_ARG, "stride"),
    (dict(target_stride_batch=1 << 62), binding.ERR_UNSUPPORTED, "address range"),
    (dict(out_tokens=0x3000000), binding.ERR_OVERLAP, "out_tokens overlaps tokens"),
    (dict(logp=0x1000000), binding.ERR_OVERLAP, "logp overlaps target"),
    (dict(accepted=0x2000000), binding.ERR_OVERLAP, "accepted overlaps draft"),
    (dict(accepted=0x3100000), binding.ERR_OVERLAP, "accepted overlaps uniforms"),
    (dict(logp=0x4000010), binding.ERR_OVERLAP, "out_tokens overlaps logp"),
])
def test_verify_refuses(lib, over, code, word):
    assert lib.odsgd_verify_draft(verify(**over), WS, 1 << 30, None) == code and word in err(lib)


def test_verify_workspace(lib):
    need = ctypes.c_size_t()
    assert lib.odsgd_verify_workspace(verify(), ctypes.byref(need)) == binding.OK and need.value > 0
    assert lib.odsgd_verify_draft(verify(), WS, need.value - 1, None) == binding.ERR_ARG and "workspace" in err(lib)
    assert lib.odsgd_verify_draft(verify(), None, 1 << 30, None) == binding.ERR_ARG and "workspace" in err(lib)
    assert lib.odsgd_verify_draft(verify(), ctypes.c_void_p(0x6000008), 1 << 30, None) == binding.ERR_ALIGN
    assert lib.odsgd_verify_draft(verify(), ctypes.c_void_p(0x2000000), 1 << 30, None) == binding.ERR_OVERLAP
    assert lib.odsgd_verify_workspace(None, ctypes.byref(need)) == binding.ERR_ARG
    assert lib.odsgd_verify_workspace(verify(vocab=0), ctypes.byref(need)) == binding.ERR_ARG
    assert lib.odsgd_verify_workspace(verify(type=7), ctypes.byref(need)) == binding.ERR_ARG
    assert lib.odsgd_verify_workspace(verify(drafts=300), ctypes.byref(need)) == binding.ERR_UNSUPPORTED
    # a workspace as large as all shapes allow does not overflow
    assert lib.odsgd_verify_workspace(verify(batch=1 << 16, drafts=255, vocab=1 << 30), ctypes.byref(need)) == binding.OK
    # nothing to verify: nothing is launched
    assert lib.odsgd_verify_draft(verify(batch=0, target=0, draft=0, tokens=0, uniforms=0, out_tokens=0, accepted=0, logp=0), WS, 1 << 30, None) == binding.OK


def test_stalled_waits_refuses_no_place(lib):
    assert lib.odsgd_stalled_waits(None) == binding.ERR_ARG
