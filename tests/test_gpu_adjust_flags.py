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


@pytest.mark.parametrize("rows,words", [([33, 2], 1), ([1, 65], 2), ([40, 40, 3], 1)])
def test_masks_without_a_bit_for_every_row(rows, words):
    c = Case(rows, 3000, BF, near=20, seed=2)
    have = c.args["node_mask"].shape[1]
    assert have == words + 1
    for s in range(len(rows)):
        c.sees[s][:, 32 * words:] = False  # what a mask of `words` words can say
    want, size = c.exact()
    status = i32([0])
    got = c.call(node_mask=c.args["node_mask"][:, :words].contiguous(), status=status)
    assert int(status) == pps.FLAG_INDEX
    # five operations in fp32, 2^-24 of the terms each, and the result's rounding (2^-8, half a step of bf16)
    assert bool(((got.double() - want).abs() <= 6 * 2.0 ** -24 * size + 2.0 ** -8 * want.abs()).all())
    status.zero_()
    c.call(status=status)
    assert int(status) == 0


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("wrong", [-1, 3000, -2 ** 31, 2 ** 31 - 1])
@pytest.mark.parametrize("key,at", [("text", (1, 2)), ("text", (0, 0)), ("node_tok", (1,)), ("node_tok", (4,)), ("bias_tok", (0,)), ("bias_tok", (7,))])
def test_a_wrong_token_counts_as_left_out(key, at, wrong, dt):
    c = Case([3, 2], 3000, dt, [20, 30], near=25, bias=30, seed=12)
    off = c.args["bias_off"].tolist()
    assert off[-1] > 7
    c.args[key] = c.args[key].clone()
    c.args[key][at] = wrong
    seen = True
    if key == "text":
        c.text[at[0]] = torch.cat([c.text[at[0]][:at[1]], c.text[at[0]][at[1] + 1:]])
    elif key == "node_tok":
        s = 0 if at[0] < 3 else 1
        seen = bool(c.sees[s][:, at[0] - c.off[s]].any())
        c.sees[s][:, at[0] - c.off[s]] = False
    else:
        entries = list(zip(c.args["bias_tok"].tolist(), c.args["bias_val"].tolist()))
        c.bias = [{t: v for t, v in entries[a:b] if t != wrong} for a, b in zip(off, off[1:])]
    status = i32([0])
    got = c.call(status=status)
    assert int(status) == (pps.FLAG_INDEX if seen else 0)
    if key == "node_tok":
        c.args["node_tok"][at] = 0  # (of no path: any token will do)
    want, size = c.exact()
    assert bool(((got.double() - want).abs() <= 6 * 2.0 ** -24 * size + (2.0 ** -8 if dt is BF else 0) * want.abs()).all())
