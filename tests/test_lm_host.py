"""The language-model calls of the C ABI refuse what they must before any CUDA call is made, and lm.py
packs their descriptors as the header lays them out.  No kernel is launched here."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2005_06728_b200 import binding, build, lm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EMBED = ("tokens act table token_type act_type table_type accumulate n_outer n_inner token_stride_outer token_stride_inner "
         "act_stride_outer act_stride_inner vocab dim table_stride padding_token scale").split()
POLICY = ("logits labels old_logp ref_logp advantages weights dlogits logp lse stats type label_type n_outer n_inner vocab "
          "logits_stride_outer logits_stride_inner label_stride_outer label_stride_inner old_stride_outer old_stride_inner "
          "ref_stride_outer ref_stride_inner adv_stride_outer adv_stride_inner weight_stride_outer weight_stride_inner "
          "dlogits_stride_outer dlogits_stride_inner inv_temp clip_low clip_high kl_coef grad_scale").split()
TENSOR = "data numel offset type group".split()


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def err(lib):
    return lib.odsgd_last_error(None).decode()


def offsets(fmt):
    """Offset of each field of a native struct format, and its size."""
    out, at = [], 0
    for count, code in re.findall(r"(\d*)([PNiqfx])", fmt):
        for _ in range(int(count or 1)):
            size = {"P": 8, "N": 8, "q": 8, "i": 4, "f": 4, "x": 1}[code]
            if code != "x":
                at = -(-at // size) * size
                out.append(at)
            at += size
    return out, at


@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not available")
def test_descriptors_are_packed_as_the_header_lays_them_out(tmp_path):
    src = tmp_path / "layout.c"
    body = ""
    for struct, fields in (("odsgd_embed_desc", EMBED), ("odsgd_policy_desc", POLICY), ("odsgd_grad_tensor", TENSOR)):
        body += "".join(f'printf("%zu ", offsetof({struct}, {f}));\n' for f in fields)
        body += f'printf("%zu\\n", sizeof({struct}));\n'
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "odsgd.h"\nint main(void) {\n' + body + "return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", f"-I{os.path.join(ROOT, 'include')}", str(src), "-o", str(exe)], check=True)
    lines = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines()
    for line, packed, fields in zip(lines, (lm._EMBED, lm._POLICY, lm._GRAD_TENSOR), (EMBED, POLICY, TENSOR)):
        *want, size = map(int, line.split())
        got, end = offsets(packed.format)
        assert got == want and end == size == packed.size and len(got) == len(fields)


def test_constants_match_the_header():
    text = open(os.path.join(ROOT, "include", "odsgd.h")).read()
    for name, value in (("F32", lm.F32), ("BF16", lm.BF16), ("F16", lm.F16), ("I32", lm.I32), ("I64", lm.I64)):
        assert re.search(rf"#define ODSGD_{name} {value}\b", text)
    assert "#define ODSGD_MAX_TOKENS (1 << 24)" in text and lm.MAX_TOKENS == 1 << 24


# addresses that are never dereferenced: the checks only look at their values
GOOD_EMBED = dict(tokens=0x1000000, act=0x2000000, table=0x3000000, token_type=lm.I64, act_type=lm.BF16, table_type=lm.F32,
                  accumulate=0, n_outer=4, n_inner=8, token_stride_outer=8, token_stride_inner=1, act_stride_outer=128,
                  act_stride_inner=16, vocab=100, dim=16, table_stride=16, padding_token=-1, scale=1.0)


def embed(**over):
    d = dict(GOOD_EMBED, **over)
    return lm._EMBED.pack(*[d[f] for f in EMBED])


@pytest.mark.parametrize("over,code,word", [
    (dict(token_type=lm.F32), binding.ERR_ARG, "token_type"),
    (dict(act_type=lm.I32), binding.ERR_ARG, "act_type"),
    (dict(table_type=9), binding.ERR_ARG, "table_type"),
    (dict(n_outer=-1), binding.ERR_ARG, "negative"),
    (dict(n_outer=1 << 13, n_inner=1 << 12), binding.ERR_UNSUPPORTED, "tokens"),
    (dict(n_outer=1 << 62, n_inner=1 << 62), binding.ERR_UNSUPPORTED, "tokens"),
    (dict(vocab=0), binding.ERR_ARG, "vocab"),
    (dict(dim=0), binding.ERR_ARG, "dim"),
    (dict(vocab=1 << 31), binding.ERR_UNSUPPORTED, "limits"),
    (dict(dim=(1 << 20) + 1, table_stride=1 << 21), binding.ERR_UNSUPPORTED, "limits"),
    (dict(table_stride=15), binding.ERR_ARG, "table_stride"),
    (dict(scale=float("inf")), binding.ERR_ARG, "scale"),
    (dict(table=0), binding.ERR_ARG, "table"),
    (dict(tokens=0), binding.ERR_ARG, "tokens"),
    (dict(act=0), binding.ERR_ARG, "act"),
    (dict(table=0x3000002), binding.ERR_ALIGN, "table"),
    (dict(tokens=0x1000004), binding.ERR_ALIGN, "tokens"),
    (dict(act=0x2000001), binding.ERR_ALIGN, "act"),
    (dict(token_stride_outer=-8), binding.ERR_ARG, "stride"),
    (dict(act_stride_outer=1 << 62), binding.ERR_UNSUPPORTED, "address range"),
])
def test_embed_calls_refuse(lib, over, code, word):
    ws = ctypes.c_void_p(0x4000000)
    assert lib.odsgd_embed_lookup(embed(**over), None) == code and word in err(lib)
    assert lib.odsgd_embed_grad(embed(**over), ws, 1 << 30, None) == code and word in err(lib)


def test_embed_overlaps_and_workspace(lib):
    ws = ctypes.c_void_p(0x4000000)
    # what is written may not overlap anything; two inputs may
    assert lib.odsgd_embed_lookup(embed(act=0x3000000 + 4 * 1599), None) == binding.ERR_OVERLAP
    assert lib.odsgd_embed_lookup(embed(act=0x1000000), None) == binding.ERR_OVERLAP
    assert lib.odsgd_embed_lookup(embed(act_stride_inner=8), None) == binding.ERR_OVERLAP and "rows" in err(lib)
    assert lib.odsgd_embed_lookup(embed(act_stride_outer=0), None) == binding.ERR_OVERLAP
    assert lib.odsgd_embed_grad(embed(act=0x3000000 + 4 * 1599), ws, 1 << 30, None) == binding.ERR_OVERLAP
    assert lib.odsgd_embed_grad(embed(tokens=0x3000000 + 8 * 100), ws, 1 << 30, None) == binding.ERR_OVERLAP
    assert lib.odsgd_embed_grad(embed(table_type=lm.BF16), ws, 1 << 30, None) == binding.ERR_ARG
    need = ctypes.c_size_t(7)
    assert lib.odsgd_embed_grad_workspace(embed(act=0, tokens=0, table=0), ctypes.byref(need)) == binding.OK and need.value > 0
    assert lib.odsgd_embed_grad(embed(), None, 1 << 30, None) == binding.ERR_ARG and "workspace" in err(lib)
    assert lib.odsgd_embed_grad(embed(), ctypes.c_void_p(0x4000008), 1 << 30, None) == binding.ERR_ALIGN
    assert lib.odsgd_embed_grad(embed(), ws, need.value - 1, None) == binding.ERR_ARG and str(need.value) in err(lib)
    for at in (0x2000000 - 16, 0x3000000 + 4 * 1596, 0x1000000):
        assert lib.odsgd_embed_grad(embed(), ctypes.c_void_p(at), need.value, None) == binding.ERR_OVERLAP and "workspace" in err(lib)
    big = ctypes.c_size_t()
    assert lib.odsgd_embed_grad_workspace(embed(n_outer=1 << 12, n_inner=1 << 12, dim=4096), ctypes.byref(big)) == binding.OK
    assert big.value > 4 * 4 * (1 << 24), "sizes beyond 32 bits"
    assert lib.odsgd_embed_grad_workspace(embed(n_outer=1 << 13, n_inner=1 << 12), ctypes.byref(big)) == binding.ERR_UNSUPPORTED
    assert lib.odsgd_embed_grad_workspace(None, ctypes.byref(big)) == binding.ERR_ARG
    assert lib.odsgd_embed_lookup(None, None) == binding.ERR_ARG and lib.odsgd_embed_grad(None, ws, 0, None) == binding.ERR_ARG
    assert lib.odsgd_embed_lookup(embed(n_outer=0, tokens=0, act=0), None) == binding.OK, "no tokens, nothing to do"


GOOD_POLICY = dict(logits=0x1000000, labels=0x2000000, old_logp=0x2100000, ref_logp=0x2200000, advantages=0x2300000,
                   weights=0x2400000, dlogits=0x3000000, logp=0x4000000, lse=0x4100000, stats=0x4200000, type=lm.BF16,
                   label_type=lm.I64, n_outer=4, n_inner=8, vocab=100, logits_stride_outer=800, logits_stride_inner=100,
                   label_stride_outer=8, label_stride_inner=1, old_stride_outer=8, old_stride_inner=1, ref_stride_outer=8,
                   ref_stride_inner=1, adv_stride_outer=1, adv_stride_inner=0, weight_stride_outer=0, weight_stride_inner=0,
                   dlogits_stride_outer=800, dlogits_stride_inner=100, inv_temp=1.0, clip_low=0.2, clip_high=0.2, kl_coef=0.1,
                   grad_scale=1.0)


def policy(**over):
    d = dict(GOOD_POLICY, **over)
    return lm._POLICY.pack(*[d[f] for f in POLICY])


@pytest.mark.parametrize("over,code,word", [
    (dict(type=lm.I64), binding.ERR_ARG, "type"),
    (dict(label_type=lm.F32), binding.ERR_ARG, "label_type"),
    (dict(n_inner=-1), binding.ERR_ARG, "negative"),
    (dict(n_outer=1 << 14, n_inner=1 << 13), binding.ERR_UNSUPPORTED, "rows"),
    (dict(vocab=0), binding.ERR_ARG, "vocab"),
    (dict(vocab=(1 << 30) + 1), binding.ERR_UNSUPPORTED, "vocab"),
    (dict(inv_temp=0.0), binding.ERR_ARG, "inv_temp"),
    (dict(inv_temp=-1.0), binding.ERR_ARG, "inv_temp"),
    (dict(inv_temp=float("nan")), binding.ERR_ARG, "inv_temp"),
    (dict(logits=0), binding.ERR_ARG, "logits"),
    (dict(labels=0), binding.ERR_ARG, "labels"),
    (dict(logp=0), binding.ERR_ARG, "logp"),
    (dict(logits=0x1000001), binding.ERR_ALIGN, "logits"),
    (dict(labels=0x2000004), binding.ERR_ALIGN, "labels"),
    (dict(logp=0x4000002), binding.ERR_ALIGN, "logp"),
    (dict(logits_stride_inner=-100), binding.ERR_ARG, "stride"),
    (dict(logits_stride_outer=1 << 62), binding.ERR_UNSUPPORTED, "address range"),
    (dict(logp=0x1000000 + 64), binding.ERR_OVERLAP, "logp"),
])
def test_score_and_loss_refuse(lib, over, code, word):
    assert lib.odsgd_token_logprob(policy(**over), None) == code and word in err(lib)
    assert lib.odsgd_policy_loss(policy(**over), ctypes.c_void_p(0x5000000), 1 << 20, None) == code and word in err(lib)


@pytest.mark.parametrize("over,code,word", [
    (dict(clip_low=-0.1), binding.ERR_ARG, "clip"),
    (dict(clip_high=float("nan")), binding.ERR_ARG, "clip"),
    (dict(kl_coef=float("inf")), binding.ERR_ARG, "kl_coef"),
    (dict(grad_scale=float("nan")), binding.ERR_ARG, "grad_scale"),
    (dict(ref_logp=0), binding.ERR_ARG, "ref_logp"),
    (dict(stats=0), binding.ERR_ARG, "stats"),
    (dict(stats=0x4200002), binding.ERR_ALIGN, "stats"),
    (dict(old_logp=0), binding.ERR_ARG, "old_logp"),
    (dict(advantages=0), binding.ERR_ARG, "advantages"),
    (dict(weights=0), binding.ERR_ARG, "weights"),
    (dict(dlogits=0), binding.ERR_ARG, "dlogits"),
    (dict(dlogits=0x3000001), binding.ERR_ALIGN, "dlogits"),
    (dict(dlogits=0x1000000 + 200), binding.ERR_OVERLAP, "dlogits"),
    (dict(dlogits=0x1000000, dlogits_stride_outer=900), binding.ERR_OVERLAP, "dlogits"),
    (dict(dlogits_stride_inner=99), binding.ERR_OVERLAP, "rows"),
    (dict(dlogits_stride_outer=0), binding.ERR_OVERLAP, "rows"),
    (dict(stats=0x4000000), binding.ERR_OVERLAP, "stats"),
    (dict(stats=0x3000000 + 8), binding.ERR_OVERLAP, "stats"),
    (dict(logp=0x2100000), binding.ERR_OVERLAP, "logp"),
])
def test_loss_refuses(lib, over, code, word):
    assert lib.odsgd_policy_loss(policy(**over), ctypes.c_void_p(0x5000000), 1 << 20, None) == code and word in err(lib)


def test_loss_workspace_and_empty_calls(lib):
    need = ctypes.c_size_t()
    assert lib.odsgd_policy_loss_workspace(policy(), ctypes.byref(need)) == binding.OK and need.value == 12 * 32
    assert lib.odsgd_policy_loss(policy(), None, 1 << 20, None) == binding.ERR_ARG
    assert lib.odsgd_policy_loss(policy(), ctypes.c_void_p(0x5000004), 1 << 20, None) == binding.ERR_ALIGN
    assert lib.odsgd_policy_loss(policy(), ctypes.c_void_p(0x5000000), need.value - 1, None) == binding.ERR_ARG
    for at in (0x1000000, 0x3000000 + 32, 0x4000000, 0x4200000, 0x2000000):
        assert lib.odsgd_policy_loss(policy(), ctypes.c_void_p(at), need.value, None) == binding.ERR_OVERLAP and "workspace" in err(lib)
    assert lib.odsgd_token_logprob(None, None) == binding.ERR_ARG and lib.odsgd_policy_loss(None, None, 0, None) == binding.ERR_ARG
    assert lib.odsgd_token_logprob(policy(n_inner=0, logits=0, labels=0, logp=0), None) == binding.OK
    # the transposed batch: rows interleave, and do not overlap
    over = dict(dlogits_stride_outer=100, dlogits_stride_inner=400)
    rc = lib.odsgd_policy_loss(policy(dlogits=0x1000000, logits_stride_outer=100, logits_stride_inner=400, kl_coef=float("nan"), **over),
                               ctypes.c_void_p(0x5000000), 1 << 20, None)
    assert rc == binding.ERR_ARG and "kl_coef" in err(lib)


def grad_set(lib, tensors, n_groups=2, arenas=None, arena_len=0):
    h = ctypes.c_void_p(1)
    packed = b"".join(lm._GRAD_TENSOR.pack(*t) for t in tensors)
    tab = None
    if arenas is not None:
        tab = (ctypes.c_void_p * len(arenas))(*arenas)
    rc = lib.odsgd_grad_set_create(ctypes.byref(h), packed if tensors else None, len(tensors), n_groups, tab, arena_len, None)
    assert rc == binding.OK or h.value is None, "*out is NULL on failure"
    return rc


def test_gradient_sets_refuse(lib):
    t = (0x1000000, 100, 0, lm.F32, 0)
    arenas = [0x2000000, 0x3000000]
    assert grad_set(lib, [t], n_groups=0) == binding.ERR_ARG
    assert grad_set(lib, [t], n_groups=binding.MAX_WORKERS + 1) == binding.ERR_ARG
    assert grad_set(lib, [t[:3] + (lm.I32, 0)]) == binding.ERR_ARG and "type" in err(lib)
    assert grad_set(lib, [t[:4] + (2,)]) == binding.ERR_ARG and "group" in err(lib)
    assert grad_set(lib, [(0,) + t[1:]]) == binding.ERR_ARG and "NULL" in err(lib)
    assert grad_set(lib, [(0x1000002,) + t[1:]]) == binding.ERR_ALIGN
    assert grad_set(lib, [(0x1000000, 1 << 60, 0, lm.F32, 0)]) == binding.ERR_ARG
    assert grad_set(lib, [t, (0x1000000 + 396, 10, 0, lm.F32, 1)]) == binding.ERR_OVERLAP, "scaled in place"
    assert grad_set(lib, [t], arenas=[0x2000000, 0], arena_len=100) == binding.ERR_ARG and "arenas[1]" in err(lib)
    assert grad_set(lib, [t], arenas=[0x2000000, 0x3000002], arena_len=100) == binding.ERR_ALIGN
    assert grad_set(lib, [t], arenas=arenas, arena_len=99) == binding.ERR_ARG and "beyond" in err(lib)
    assert grad_set(lib, [(0x1000000, 100, 1, lm.F32, 0)], arenas=arenas, arena_len=100) == binding.ERR_ARG
    assert grad_set(lib, [(0x1000000, 1, (1 << 64) - 1, lm.F32, 0)], arenas=arenas, arena_len=100) == binding.ERR_ARG
    assert grad_set(lib, [t, (0x1100000, 10, 99, lm.F32, 0)], arenas=arenas, arena_len=200) == binding.ERR_OVERLAP
    assert grad_set(lib, [(0x2000000, 100, 0, lm.F32, 0)], arenas=arenas, arena_len=100) == binding.ERR_OVERLAP
    assert grad_set(lib, [t, t[:4] + (1,)], arenas=[0x2000000, 0x2000000], arena_len=100) == binding.ERR_OVERLAP
    assert lib.odsgd_grad_set_create(None, None, 0, 1, None, 0, None) == binding.ERR_ARG
    null = ctypes.c_void_p()
    assert lib.odsgd_grad_set_norm(null, None, None) == binding.ERR_ARG
    assert lib.odsgd_grad_set_clip(null, 1.0, None, None) == binding.ERR_ARG
    assert lib.odsgd_grad_set_destroy(null) == binding.ERR_ARG


def test_leading_axes_fold_into_two_levels():
    t = torch.zeros(2, 3, 4, 5)
    assert lm._levels(t, 3, "t") == (20, 5) and lm._sizes(t.shape[:3]) == (6, 4)
    assert lm._levels(t[:, :, 1:], 3, "t") == (20, 5) and lm._sizes((2, 3, 3)) == (6, 3)
    assert lm._levels(t[:1], 3, "t") == (20, 5)
    assert lm._levels(torch.zeros(3).expand(2, 3), 2, "t") == (0, 1)
    assert lm._levels(t, 0, "t") == (0, 0) and lm._sizes(()) == (1, 1) and lm._sizes((7,)) == (1, 7)
    with pytest.raises(ValueError, match="two strided levels"):
        lm._levels(t[:, 1:], 3, "t")
    with pytest.raises(ValueError, match="last axis"):
        lm._rows(t.transpose(2, 3), 3, "t")
    with pytest.raises(TypeError, match="CUDA"):
        lm._need(t, "t", lm._FLOATS, 0)
