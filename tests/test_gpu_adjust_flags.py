"""pps_adjust_logits: what is cut or left out is flagged, and the rest is what it is without it."""
import pytest
import torch

from paper_2609_21858_gb300 import pps
from test_gpu_adjust import BF, F32, Case, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    pps.lib()


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("lens,prompt,cut", [([20, 30], [21, 5], [20, 5]), ([20, 30], [0, 2 ** 31 - 1], [0, 30]),
                                             ([0, 30], [1, 30], [0, 30]), ([20, 30], [3, -1], [3, 0])])
def test_prompts_longer_than_their_text(lens, prompt, cut, dt):
    c = Case([3, 2], 3000, dt, lens, cut, near=40, seed=1)
    want, status = c.check(), i32([0])
    got = c.call(prompt_len=i32(prompt), status=status)
    assert int(status) == pps.FLAG_INDEX and torch.equal(got, want)
    status.zero_()
    c.call(prompt_len=i32(lens), status=status)  # all of it is prompt
    assert int(status) == 0
