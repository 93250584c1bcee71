"""C-ABI checks, without a GPU, of scalars at the ends of fp32's range (target-side calls)."""
import pytest

from paper_2609_21858_gb300 import pps
from test_abi_target import _attention


@pytest.mark.parametrize("scale", [2.4e38, -2.4e38, 3.4e38])
def test_attention_refuses_a_scale_whose_logarithms_are_infinite(scale):
    """The softmax is formed in powers of two: scale * log2(e) has to be finite, too."""
    assert _attention(scale=scale) == pps.ERR_INVALID_ARG


@pytest.mark.parametrize("scale", [2.3e38, -2.3e38, 1e-45, -0.0])
def test_attention_takes_every_other_scale(scale):
    assert _attention(scale=scale) == pps.OK
