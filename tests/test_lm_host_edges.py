"""Host side of the language-model calls: shapes and buffers beside those of test_lm_host.  No kernel is
launched here."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2005_06728_b200 import binding, build, lm
from test_lm_host import policy


@pytest.mark.parametrize("shape", [(3, 0, 4), (0, 3, 4), (3, 4, 0), (5, 0, 3, 8), (5, 3, 0, 8), (2, 0, 0, 8), (0, 2, 3, 4, 5)])
def test_empty_tensors_fold(shape):
    """A tensor without elements folds whatever its axes: none of its strides is used."""
    lead = len(shape)
    for t in (torch.zeros(shape), torch.zeros(shape).transpose(0, 1), torch.zeros((*shape, 2))[..., 1]):
        a, b = lm._levels(t, lead, "t")
        assert a >= 0 and b >= 0
        outer, inner = lm._sizes(t.shape)
        assert outer * inner == 0
    assert lm._rows(torch.zeros((*shape, 6)), lead, "t") is not None


def test_axes_that_do_not_fold_are_still_refused():
    with pytest.raises(ValueError, match="two strided levels"):
        lm._levels(torch.zeros(2, 3, 4, 5)[:, 1:], 3, "t")


def test_a_loss_without_rows_needs_no_reference():
    """An empty tensor has no address: the KL term of no rows is taken from none."""
    lib = binding.load_library()
    for over in (dict(n_outer=0), dict(n_inner=0)):
        # refused for its workspace, which is looked at after the rows' buffers
        d = policy(logits=0, labels=0, old_logp=0, ref_logp=0, advantages=0, weights=0, dlogits=0, logp=0, **over)
        assert lib.odsgd_policy_loss(d, None, 16, None) == binding.ERR_ARG and "workspace" in lib.odsgd_last_error(None).decode()


def test_no_load_of_the_read_only_path():
    """A grid that may begin while the one ahead of it writes must not read through the path for memory that
    nothing writes while the grid exists."""
    with open(os.path.join(build.CSRC, "odsgd_lm_kernels.cuh")) as f:
        text = f.read()
    assert "griddepcontrol.wait" in text and "__ldg" not in text and "global.nc" not in text


@pytest.mark.parametrize("over", [
    dict(n_outer=1, dlogits_stride_outer=0),
    dict(n_outer=1, logits_stride_outer=0, dlogits_stride_outer=12345),
    dict(n_inner=1, dlogits_stride_inner=7),
    dict(n_outer=1, n_inner=1, dlogits_stride_outer=3, dlogits_stride_inner=0),
])
def test_a_gradient_in_place_of_one_row_has_any_stride(over):
    """The stride of a level with one place says nothing about where its rows lie."""
    lib = binding.load_library()
    # refused for its workspace, which is looked at after the buffers
    d = policy(dlogits=0x1000000, **over)
    assert lib.odsgd_policy_loss(d, None, 1 << 20, None) == binding.ERR_ARG and "workspace" in lib.odsgd_last_error(None).decode()


@pytest.mark.parametrize("over", [dict(n_outer=2, dlogits_stride_outer=900), dict(n_inner=2, dlogits_stride_inner=200),
                                  dict(n_outer=1, n_inner=2, dlogits_stride_inner=150)])
def test_a_gradient_over_the_logits_of_other_strides_is_still_refused(over):
    lib = binding.load_library()
    assert lib.odsgd_policy_loss(policy(dlogits=0x1000000, **over), None, 1 << 20, None) == binding.ERR_OVERLAP


LIMITED = """
import ctypes, resource, sys
sys.path.insert(0, {root!r})
from paper_2005_06728_b200 import binding, lm
lib = binding.load_library()
assert lib.odsgd_token_logprob(None, None) == binding.ERR_ARG  # leaves its text
with open("/proc/self/status") as f:
    held = next(int(line.split()[1]) for line in f if line.startswith("VmSize")) * 1024
resource.setrlimit(resource.RLIMIT_AS, (held + (1 << 30), held + (1 << 30)))
h = ctypes.c_void_p(1)
t = lm._GRAD_TENSOR.pack(0x1000000, 1 << 42, 0, lm.F32, 0)  # a table of 6 GB
rc = lib.odsgd_grad_set_create(ctypes.byref(h), t, 1, 1, None, 0, None)
print(rc, h.value, lib.odsgd_last_error(None).decode())
"""


def test_running_out_of_host_memory_says_so():
    """Nothing is thrown across the boundary, and the text is not that of an earlier failure."""
    code = LIMITED.format(root=build.ROOT)
    out = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=600)
    assert out.returncode == 0, out.stderr[-2000:]
    assert out.stdout.split(maxsplit=2) == [str(binding.ERR_ARG), "None", "out of host memory\n"]
