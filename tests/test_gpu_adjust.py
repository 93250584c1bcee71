"""pps_adjust_logits against the formulas in 64 bits."""
import math
import random

import pytest
import torch

from paper_2609_21858_gb300 import pps

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    pps.lib()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def words(bits):
    x = (torch.nn.functional.pad(bits, (0, -bits.shape[-1] % 32)).unflatten(-1, (-1, 32)).long()
         << torch.arange(32, device=bits.device)).sum(-1)
    return torch.where(x >= 1 << 31, x - (1 << 32), x).to(torch.int32)


class Case:
    def __init__(self, rows, V, dt=BF, text=(), prompt=None, nodes="tree", laws=("rep", "freq", "pres"), bias=0, grammar=False,
                 seed=0, near=None):
        """rows: how many rows each sequence has; text: lengths of the texts ((): none); near: tokens come from [0, near)."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        rng = random.Random(seed)
        self.rows, self.V, self.dt = rows, V, dt
        n, n_seq = sum(rows), len(rows)
        tok = lambda *s: torch.randint(0, near or V, s, generator=g, device="cuda", dtype=torch.int32)
        self.x = (3 * torch.randn(n, V, generator=g, device="cuda")).to(dt)
        self.off = [sum(rows[:i]) for i in range(n_seq + 1)]
        a = self.args = dict(seq_off=i32(self.off))
        self.text, self.prompt = [], prompt or [0] * n_seq
        if text:
            a["text"] = tok(n_seq, max(text) + 3)
            a["text_len"] = i32(list(text))
            if prompt:
                a["prompt_len"] = i32(prompt)
            self.text = [a["text"][s, :m] for s, m in enumerate(text)]
        self.sees = [torch.ones(m, m, dtype=torch.bool).tril() for m in rows]
        if nodes:
            a["node_tok"] = tok(n)
        if nodes == "tree":
            most = -(-max(rows) // 32) * 32
            cpu = torch.Generator().manual_seed(seed)
            self.sees = [torch.rand(m, m, generator=cpu) < min(0.5, 20 / max(m, 1)) for m in rows]
            bits = torch.zeros(n, most)
            for s, m in enumerate(rows):
                bits[self.off[s]:self.off[s] + m, :m] = self.sees[s]
            a["node_mask"] = words(bits.bool()).cuda()
        for name, key, lo, hi in (("rep", "repetition", 1.0, 1.5), ("freq", "frequency", -0.2, 0.8), ("pres", "presence", -0.3, 0.6)):
            if name in laws and (text or nodes):
                a[key] = lo + (hi - lo) * torch.rand(n_seq, generator=g, device="cuda")
        self.bias = [{} for _ in rows]
        if bias:
            m = [rng.randint(0, bias) for _ in rows]
            t, v = tok(sum(m) + 1), 4 * torch.randn(sum(m) + 1, generator=g, device="cuda")
            a.update(bias_off=i32([sum(m[:i]) for i in range(n_seq + 1)]), bias_tok=t, bias_val=v)
            at = 0
            for s in range(n_seq):
                for t1, v1 in zip(t[at:at + m[s]].tolist(), v[at:at + m[s]].tolist()):
                    self.bias[s][t1] = v1  # the last of a token's
                at += m[s]
        self.bits = None
        if grammar:
            share = torch.tensor([0.97, 0.5, 0.01, 0.0], device="cuda")[torch.randint(0, 4, (n,), generator=g, device="cuda")]
            self.bits = torch.rand(n, V, generator=g, device="cuda") < share[:, None]
            a["allowed"] = words(self.bits).contiguous()

    def call(self, **kw):
        return pps.adjust_logits(**{**dict(logits=self.x, **self.args), **kw})

    def exact(self):
        """The definition in 64 bits, and the size of the terms."""
        y, a = self.x.double(), self.args
        size = y.abs()
        one = lambda key, s, default: float(a[key][s]) if key in a else default
        for s, m in enumerate(self.rows):
            text = self.text[s].long() if self.text else torch.zeros(0, dtype=torch.long, device="cuda")
            p = min(self.prompt[s], text.numel())
            before, after = torch.bincount(text[:p], minlength=self.V), torch.bincount(text[p:], minlength=self.V)
            for i in range(m):
                r = self.off[s] + i
                c = after.clone()
                if "node_tok" in a:
                    path = a["node_tok"][self.off[s]:self.off[s] + m][self.sees[s][i].cuda()]
                    c += torch.bincount(path.long(), minlength=self.V)
                if "text" in a or "node_tok" in a:
                    rep = torch.where(before + c > 0, one("repetition", s, 1.0), 1.0)
                    x = y[r]
                    x = torch.where(x > 0, x / rep, x * rep)
                    f, q = one("frequency", s, 0.0), one("presence", s, 0.0)
                    y[r] = x - f * c - q * (c > 0)
                    size[r] = torch.maximum(size[r], x.abs()) + abs(f) * c + abs(q)
                for t, v in self.bias[s].items():
                    y[r, t] += v
                    size[r, t] += abs(v)
        if self.bits is not None:
            y[~self.bits] = -math.inf
        return y, size

    def check(self, **kw):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        want, size = self.exact()
        got = self.call(status=status, **kw)
        assert int(status) == 0
        # five operations in fp32, 2^-24 of the terms each, and the result's rounding
        tol = 6 * 2.0 ** -24 * size + (2.0 ** -8 if self.dt is BF else 0) * want.abs().clamp(max=1e30)
        fine = torch.isfinite(want)
        assert torch.equal(torch.isneginf(got), torch.isneginf(want))
        err = (got.double() - want).abs()
        assert bool((err <= tol)[fine].all()), f"worst excess {(err - tol)[fine].max().item():.3g}"
        return got


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [1, 7, 31, 1000, 4095, 4096, 4097, 8200, 32000, 50001])
@pytest.mark.parametrize("rows", [[1], [3, 1, 9], [17]])
def test_vocabularies_and_rows(dt, V, rows):
    n = len(rows)
    Case(rows, V, dt, [5, 300, 40][:n], [2, 0, 40][:n], seed=V).check()
    Case(rows, V, dt, [5, 300, 40][:n], bias=30, grammar=True, nodes="chain", seed=V + 1).check()
    Case(rows, V, dt, nodes=None, bias=30, seed=V + 2).check()
    Case(rows, V, dt, nodes=None, grammar=True, seed=V + 3).check()


@pytest.mark.parametrize("dt", [BF, F32])
def test_tokens_that_repeat(dt):
    # counts of many, on paths, in prompts and outputs at once, and biases that name a token again
    Case([41, 5], 9000, dt, [700, 90], [300, 90], near=25, bias=60, grammar=True, seed=1).check()
    Case([60], 5000, dt, nodes="chain", near=3, seed=2).check()
    Case([70], 5000, dt, [100], near=3, seed=3).check()
    Case([12] * 9, 40, dt, [50] * 9, near=2, seed=4).check()


@pytest.mark.parametrize("laws", [(), ("rep",), ("freq",), ("pres",), ("freq", "pres")])
def test_each_law_alone(laws):
    Case([6, 2], 3000, F32, [60, 0], [10, 0], laws=laws, seed=5).check()


def test_longest_texts_and_large_vocabularies():
    Case([4], 152063, F32, [60000], [20000], seed=6, bias=500, grammar=True).check()
    Case([41] * 3, 128256, BF, [3000, 0, 17], seed=7).check()


def test_strides_alignments_and_in_place():
    for dt in (BF, F32):
        for V, pad, shift in ((9001, 0, 0), (9001, 3, 1), (4096, 8, 0), (5000, 5, 3)):
            c = Case([3, 9, 1], V, dt, [40, 400, 4], bias=10, grammar=True, near=3000, seed=V + pad)
            want = c.check()
            flat = torch.zeros(c.x.shape[0] * (V + pad) + shift, dtype=dt, device="cuda")[shift:].view(-1, V + pad)
            x = flat[:, :V]
            x.copy_(c.x)
            assert torch.equal(c.call(logits=x), want)
            out = torch.full((c.x.shape[0], V + 11), 7.0, dtype=dt, device="cuda")
            assert torch.equal(c.call(logits=x, out=out[:, 2:V + 2]), want)
            assert bool((out[:, :2] == 7).all()) and bool((out[:, V + 2:] == 7).all())
            assert torch.equal(c.call(logits=x, out=x), want) and torch.equal(x, want)
            assert not bool(flat[:, V:].any())
    # wider rows of masks, text columns past the longest
    c = Case([3, 2], 2000, BF, [10, 20], grammar=True, seed=9)
    want = c.check()
    one = c.args["allowed"][3:4].expand(5, -1)  # the same mask for all rows
    assert torch.equal(c.call(allowed=one), c.call(allowed=one.contiguous()))
    wide = torch.full((5, 70), -1, dtype=torch.int32, device="cuda")
    wide[:, :63] = c.args["allowed"]
    text = torch.full((2, 90), -3, dtype=torch.int32, device="cuda")
    text[:, :23] = c.args["text"]
    assert torch.equal(c.call(allowed=wide[:, :63], text=text[:, :23]), want) and torch.equal(c.call(text=text), want)


def test_rows_of_no_sequence_and_sequences_without_rows():
    c = Case([2, 0, 3], 500, BF, [5, 6, 7], seed=10)
    want = c.check()
    x = torch.cat([c.x, c.x[:4]])
    out = torch.full_like(x, 9.0)
    more = {k: torch.cat([c.args[k], c.args[k][:4]]) for k in ("node_tok", "node_mask")}
    got = c.call(logits=x, out=out, **more)
    assert torch.equal(got[:5], want) and bool((got[5:] == 9).all())
    assert c.call(logits=c.x[:0], seq_off=i32([0, 0, 0, 0]), node_tok=c.args["node_tok"][:0], node_mask=c.args["node_mask"][:0]).shape == (0, 500)


def test_numbers_that_are_not_finite():
    c = Case([2], 200, F32, [50], laws=("rep", "freq", "pres"), grammar=True, seed=11)
    c.bits[:] = True
    c.bits[:, ::7] = False
    c.args["allowed"] = words(c.bits)
    c.x[0, :60] = float("nan")
    c.x[0, 60:80], c.x[1, :30] = float("-inf"), float("inf")
    got, (want, _) = c.call(), c.exact()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    for inf in (math.inf, -math.inf):
        assert torch.equal(got == inf, want == inf)


def test_tokens_offsets_and_lengths_out_of_range_are_flagged_and_harmless():
    c = Case([3, 2], 3000, BF, [20, 30], bias=10, seed=12)
    want = c.check()
    for key, at, wrong in (("text", (0, 25), None), ("text", (1, 2), -1), ("text", (1, 2), 3000), ("node_tok", (1,), 3000),
                           ("node_tok", (1,), -2 ** 31), ("bias_tok", (0,), 2 ** 31 - 1)):
        t = c.args[key].clone()
        if wrong is None:
            t[:, 30:] = -1  # past the length: never read
        else:
            t[at] = wrong
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = c.call(status=status, **{key: t})
        if wrong is None:
            assert int(status) == 0 and torch.equal(got, want)
        elif key != "bias_tok" or int(c.args["bias_off"][-1]) > 0:
            assert int(status) == (pps.FLAG_INDEX if key != "node_tok" or any(bool(x[:, 1].any()) for x in c.sees[:1]) else 0)
    status.zero_()
    got = c.call(status=status, text_len=i32([20, 99]))  # more than the text has: cut there
    assert int(status) == pps.FLAG_INDEX and torch.equal(got[:3], want[:3])
    status.zero_()
    out = torch.full_like(want, 9.0)
    got = c.call(status=status, seq_off=i32([0, 3, 9]), out=out)
    assert int(status) == pps.FLAG_INDEX and torch.equal(got[:3], want[:3]) and bool((got[3:] == 9).all())
    status.zero_()
    c = Case([100], 3000, BF, nodes="chain", seed=13)  # a path of more than 64
    c.call(status=status)
    assert int(status) == pps.FLAG_INDEX


def test_another_stream_a_graph_and_the_same_bits():
    c = Case([5, 41], 60001, BF, [500, 80], near=400, bias=90, grammar=True, seed=14)
    want = c.check()
    assert torch.equal(c.call(), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.call(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call(out=out)
    graph.replay()
    assert torch.equal(out, want)


def test_more_than_2_31_logits():
    n, V = 17000, 128256
    if torch.cuda.mem_get_info()[0] < 12e9:
        pytest.skip("needs 9 GB")
    x = torch.zeros(n, V, dtype=BF, device="cuda")
    x[-1, -5:] = 1
    tok = torch.zeros(n, dtype=torch.int32, device="cuda")
    tok[-1] = V - 2
    pps.adjust_logits(x, torch.arange(n + 1, dtype=torch.int32, device="cuda"), node_tok=tok,
                      presence=torch.full((n,), 0.5, device="cuda"), out=x)
    assert x[-1, -5:].tolist() == [1, 1, 1, 0.5, 1] and float(x[-2, 0]) == -0.5 and float(x[-1, 0]) == 0


def test_refusals():
    c = Case([3, 2], 300, BF, [20, 30], [1, 2], bias=10, grammar=True, seed=15)
    a = c.args
    for bad in (dict(logits=c.x.half()), dict(logits=c.x.cpu()), dict(logits=None), dict(seq_off=a["seq_off"].long()), dict(seq_off=None),
                dict(text=a["text"].long()), dict(text_len=None), dict(node_tok=[1]), dict(node_mask=a["node_mask"].float()),
                dict(repetition=a["repetition"].double()), dict(bias_tok=None), dict(bias_val=a["bias_val"].half()),
                dict(allowed=a["allowed"].long()), dict(out=c.x.float()), dict(status=3), dict(logits=c.x.T)):
        with pytest.raises(TypeError):
            c.call(**bad)
    for bad in (dict(text=a["text"][:1]), dict(text_len=a["text_len"][:1]), dict(prompt_len=a["prompt_len"][:1]),
                dict(node_tok=a["node_tok"][:4]), dict(node_mask=a["node_mask"][:4]), dict(presence=a["presence"][:1]),
                dict(bias_off=a["bias_off"][:2]), dict(bias_val=a["bias_val"][:1]), dict(allowed=a["allowed"][:, :9]),
                dict(out=c.x[:4]), dict(out=c.x[:, :299])):
        with pytest.raises(ValueError):
            c.call(**bad)

    def code(**kw):
        with pytest.raises(pps.PPSError) as e:
            c.call(**kw)
        return e.value.code

    assert code(text=None, text_len=None, node_tok=None, node_mask=None) == pps.ERR_INVALID_ARG  # laws without tokens
    assert code(node_tok=None) == pps.ERR_INVALID_ARG
    assert code(logits=c.x[:1].expand(5, -1)) == pps.ERR_INVALID_ARG  # rows that overlap
    assert code(out=torch.empty(1, 300, dtype=BF, device="cuda").expand(5, -1)) == pps.ERR_INVALID_ARG
