"""pps_adjust_logits refuses what says something about an argument that is missing."""
import pytest
import torch

from paper_2609_21858_gb300 import pps
from test_abi_more import P, _adjust
from test_gpu_adjust import BF, Case


@pytest.mark.parametrize("bad", [dict(prompt=P), dict(prompt=P, node_tok=P), dict(bias_tok=P), dict(bias_val=P), dict(n_bias=1),
                                 dict(bias_tok=P, bias_val=P, n_bias=3)])
def test_the_abi_refuses(bad):
    assert _adjust(**bad) == pps.ERR_INVALID_ARG
    assert _adjust(n=2, n_seq=1, **bad) == pps.ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("slow", [False, True])  # by the extension, or by a named stream
def test_the_binding_refuses(slow):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    c = Case([3, 2], 300, BF, [20, 30], [1, 2], bias=10, seed=15)
    more = dict(stream=torch.cuda.current_stream()) if slow else {}
    c.call(**more)
    for bad in (dict(bias_off=None), dict(bias_off=None, bias_tok=None), dict(bias_off=None, bias_val=None), dict(text=None),
                dict(text=None, prompt_len=None)):
        with pytest.raises(TypeError):
            c.call(**bad, **more)
    with pytest.raises(pps.PPSError) as e:
        c.call(text=None, text_len=None, **more)  # a prompt of no text
    assert e.value.code == pps.ERR_INVALID_ARG
