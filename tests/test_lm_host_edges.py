"""Host side of the language-model calls: shapes and buffers beside those of test_lm_host.  No kernel is
launched here."""
import pytest
import torch

from paper_2005_06728_b200 import lm


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
