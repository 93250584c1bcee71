"""pps_adjust_logits where an argument is there but empty."""
import pytest
import torch

from paper_2609_21858_gb300 import pps
from test_abi_more import P, _adjust
from test_gpu_adjust import BF, F32, Case, i32


def test_texts_of_no_columns_in_the_abi():
    assert _adjust(rep=P, lens=P) == pps.OK and _adjust(rep=P, lens=P, prompt=P) == pps.OK
    assert _adjust(n_seq=2, lens=P, cap=4, text_stride=4) == pps.ERR_INVALID_ARG  # four columns of no text


@pytest.fixture
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    pps.lib()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("slow", [False, True])  # by the extension, or by a named stream
@pytest.mark.parametrize("rows", [[1], [3, 2]])
def test_a_text_without_columns(cuda, rows, slow, dt):
    n = len(rows)
    more = dict(stream=torch.cuda.current_stream()) if slow else {}
    text = dict(text=torch.zeros(n, 0, dtype=torch.int32, device="cuda"), text_len=i32([0] * n), prompt_len=i32([0] * n))
    laws = dict(repetition=torch.full((n,), 1.5, device="cuda"), frequency=torch.ones(n, device="cuda"))
    c = Case(rows, 5000, dt, nodes=None, seed=1)
    status = i32([0])
    assert torch.equal(c.call(status=status, **text, **laws, **more), c.x) and int(status) == 0
    c = Case(rows, 5000, dt, bias=9, grammar=True, seed=2)  # beside the rows' paths
    assert torch.equal(c.call(status=status, **text, **more), c.check()) and int(status) == 0
    c.call(status=status, **{**text, "text_len": i32([0] * (n - 1) + [1])}, **more)  # a token that no column holds
    assert int(status) == pps.FLAG_INDEX


@pytest.mark.gpu
@pytest.mark.parametrize("slow", [False, True])
def test_no_rows_and_no_sequences(cuda, slow):
    more = dict(stream=torch.cuda.current_stream()) if slow else {}
    x, one = torch.zeros(0, 300, dtype=BF, device="cuda"), torch.ones(2, device="cuda")
    none = i32([])
    for laws in (dict(repetition=one), dict(frequency=one, presence=one), {}):
        for path in (dict(node_tok=none), dict(node_tok=none, node_mask=torch.zeros(0, 1, dtype=torch.int32, device="cuda"))):
            assert pps.adjust_logits(x, i32([0, 0, 0]), **laws, **path, **more).shape == (0, 300)
    x = torch.randn(4, 300, device="cuda")
    out = torch.full_like(x, 9.0)
    empty = dict(text=i32([]).view(0, 0), text_len=none, prompt_len=none, repetition=torch.ones(0, device="cuda"))
    assert pps.adjust_logits(x, i32([0]), **empty, out=out, **more) is out and bool((out == 9).all())
