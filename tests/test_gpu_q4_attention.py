"""pps_paged_attention_q4 against the formula in 64 bits: lengths, masks, head layouts, pages, strides, refusals."""
import random

import pytest
import torch

import test_gpu_attention as sixteen
from paper_2609_21858_gb300 import pps
from q4_format import values
from test_gpu_attention import BF, F16, U, _cuda  # noqa: F401

pytestmark = pytest.mark.gpu


class Case(sixteen.Case):
    """As the 16-bit cache's cases, of codes and scales; slots past a sequence's end hold scales that are NaN."""

    def __init__(self, q_len, kv_len, heads, kv_heads, d, page, dt=BF, tree=False, layout="head", seed=0, spare=1,
                 q_scale=2.0, unit=False):
        super().__init__(q_len, kv_len, heads, kv_heads, 8, page, dt, tree, "token", seed, spare, q_scale)
        g = torch.Generator(device="cuda").manual_seed(seed + 1000)
        n_pages = self.k_cache.shape[0]
        self.d = d
        self.q = (torch.randn(sum(q_len), heads, d, generator=g, device="cuda") * q_scale).to(dt)

        def pool(n, fill):
            shape = (n_pages, kv_heads, page, n) if layout == "head" else (n_pages, page, kv_heads, n)
            x = torch.full(shape, fill, dtype=torch.uint8, device="cuda")
            return x.transpose(1, 2) if layout == "head" else x

        units = [0.5 + torch.rand(kv_heads, generator=g, device="cuda") for _ in range(2)] if unit else [None, None]
        self.cache = pps.CacheQ4(pool(d // 2, 0x55), pool(d // 2, 0x55), pool(pps.q4_scale_bytes(d), 0x7f),
                                 pool(pps.q4_scale_bytes(d), 0x7f), *units)
        self.keys, self.values = [], []
        for s, length in enumerate(kv_len):
            j = torch.arange(length, device="cuda")
            at = (self.pages[s].long()[j // page] if length else j), j % page
            for codes, scales, u, into in ((self.cache.k, self.cache.k_scale, units[0], self.keys),
                                           (self.cache.v, self.cache.v_scale, units[1], self.values)):
                codes[at] = torch.randint(0, 256, (length, kv_heads, d // 2), generator=g, device="cuda", dtype=torch.uint8)
                # scales from 1/8 to 1/2: values of a size of one; bytes past the heads' last block stay NaN
                x = scales[at]
                x[..., :d // 16] = torch.randint(0x20, 0x31, (length, kv_heads, d // 16), generator=g, device="cuda", dtype=torch.uint8)
                scales[at] = x
                into.append(values(codes[at], scales[at], u))

    def call(self, **kw):
        args = dict(q=self.q, cache=self.cache, pages=self.pages, kv_len=self.kv, q_off=self.q_off, mask=self.mask)
        return pps.paged_attention_q4(**{**args, **kw})

    def nan_rows(self):
        """The tokens' heads that are NaN by the formula, and so in the call's result; the others are right."""
        (out, size, _), got = self.exact(), self.call()
        bad = torch.isnan(out).any(-1)
        assert bool(bad.any()) and bool((~bad).any()) and torch.equal(torch.isnan(got).any(-1), bad)
        err, tol = (got.double() - out).abs(), 1.01 * U[self.dt] * out.abs() + (1.01 * U[F16] + 2e-4) * size + 2.0 ** -24
        assert bool((err <= tol)[~bad].all())
        return bad

    def compare(self, got, lse, scale=None):
        out, size, want = self.exact(scale)
        # the weights are rounded once to fp16, the result to its type; scores carry fp32 errors (products of 128 channels summed in
        # fp32: below 2^-21 of sum |q k| scale, here under 100)
        err, tol = (got.double() - out).abs(), 1.01 * U[self.dt] * out.abs() + (1.01 * U[F16] + 2e-4) * size + 2.0 ** -24
        assert bool((err <= tol).all()), f"worst excess {(err - tol).max().item():.3g}"
        seen = torch.isfinite(want)
        assert bool((torch.isneginf(lse) == ~seen).all())
        assert bool(((lse.double() - want)[seen].abs() <= 2e-4 + 1e-6 * want[seen].abs()).all())
        assert bool((got[~seen] == 0).all())


@pytest.mark.parametrize("heads,kv_heads,d", [(32, 8, 128), (28, 4, 128), (14, 2, 64), (6, 6, 64), (16, 1, 128),
                                              (20, 4, 80), (3, 1, 16), (9, 3, 112), (5, 5, 48), (130, 1, 64), (40, 2, 32)])
@pytest.mark.parametrize("dt", [BF, F16])
def test_one_token_each(heads, kv_heads, d, dt):
    kv = [1, 2, 127, 128, 129, 255, 256, 257, 700, 1, 1111]
    Case([1] * len(kv), kv, heads, kv_heads, d, 16, dt, seed=heads + d, unit=heads % 4 == 0).check()


@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256, 512])
@pytest.mark.parametrize("layout", ["token", "head"])
def test_page_sizes_and_layouts(page, layout):
    Case([1, 5, 40], [300, 513, 1030], 8, 2, 128, page, BF, layout=layout, seed=page).check()
    Case([3, 1, 70], [129, 5, 400], 4, 4, 64, page, F16, layout=layout, seed=page + 1, tree=True, unit=True).check()
    Case([1, 1, 1], [129, 5, 400], 4, 4, 80, page, BF, layout=layout, seed=page + 2).check()


# chunks whose packed rows (tokens x group) end inside, at and past a tile of rows
@pytest.mark.parametrize("heads,kv_heads,d", [(4, 4, 128), (8, 2, 128), (7, 1, 64), (12, 4, 80)])
@pytest.mark.parametrize("n", [2, 3, 4, 5, 9, 31, 32, 33, 63, 64, 65, 85, 86, 127, 128, 129, 256, 257, 385, 600])
def test_chunks(heads, kv_heads, d, n):
    Case([n, 1, n], [n, 77, n + 200], heads, kv_heads, d, 16, BF, seed=n + d).check()


@pytest.mark.parametrize("dt", [BF, F16])
def test_ragged_batches(dt):
    rng = random.Random(3)
    for seed in range(6):
        q_len = [rng.choice([0, 1, 2, 17, 130, rng.randint(1, 400)]) for _ in range(rng.randint(1, 40))]
        kv_len = [max(n, rng.choice([n, n + 1, rng.randint(0, 900)])) for n in q_len]
        heads, kv_heads = rng.choice([(8, 2), (4, 4), (7, 1)])
        if sum(q_len):
            Case(q_len, kv_len, heads, kv_heads, rng.choice([64, 128]), rng.choice([8, 16, 64]), dt, seed=seed).check()
    # single tokens and nothing between them
    Case([0, 1, 0, 0, 1, 0], [50, 300, 0, 2, 1, 900], 8, 2, 128, 16, dt, seed=9).check()


def test_sequences_without_keys_and_tokens_that_see_nothing():
    Case([4, 3, 2, 1], [0, 1, 2, 0], 8, 2, 64, 16, seed=1).check()
    Case([300, 200], [100, 0], 4, 4, 128, 16, seed=2).check()
    Case([1, 1], [0, 3], 4, 4, 128, 16, seed=2).check()
    Case([5, 40, 33], [5, 40, 33], 8, 2, 128, 16, F16, tree=True, seed=3).check()


@pytest.mark.parametrize("dt", [BF, F16])
@pytest.mark.parametrize("n,prefix", [(1, 50), (2, 127), (3, 1000), (31, 97), (32, 96), (33, 95), (41, 128), (41, 1000), (64, 1),
                                      (65, 300), (200, 77), (300, 513)])
def test_trees(n, prefix, dt):
    Case([n, n, 1], [n + prefix, n, 1 + prefix], 8, 2, 128, 16, dt, tree=True, seed=n + prefix).check()


def test_long_sequences_split_over_the_whole_gpu():
    Case([1], [40001], 8, 1, 128, 64, BF, seed=1).check()
    Case([1, 1], [20011, 3], 4, 4, 64, 16, F16, seed=2).check()
    Case([41], [30000], 8, 2, 128, 16, BF, tree=True, seed=3).check()
    Case([130], [9000], 4, 2, 128, 256, F16, seed=4).check()
    Case([3], [30000], 8, 2, 128, 16, BF, tree=True, seed=5).check()


@pytest.mark.parametrize("dt", [BF, F16])
def test_large_scores_equal_scores_and_queries_of_any_size(dt):
    Case([1, 65], [600, 777], 8, 2, 128, 16, dt, seed=5, q_scale=20.0).compare_loosely()
    Case([1, 65], [600, 777], 8, 2, 128, 16, dt, seed=6, q_scale=0.0).check()
    # a rising ramp of scores: every tile raises the maximum
    for n in (1, 70):
        c = Case([n], [3000], 4, 1, 64, 16, dt, seed=7)
        c.q.fill_(1.0)
        at = c.pages[0].long()[torch.arange(3000, device="cuda") // 16], torch.arange(3000, device="cuda") % 16
        c.cache.k[at] = 0x22  # code 1
        x = c.cache.k_scale[at]
        x[..., :4] = (torch.arange(3000, device="cuda") // 25).to(torch.uint8)[:, None, None]  # scales from 0 to 2^8.5
        c.cache.k_scale[at] = x
        c.keys[0] = values(c.cache.k[at], c.cache.k_scale[at])
        c.compare_loosely()
    # queries whose products with the scale are of a size of one, far from fp16's range
    if dt is BF:
        for power in (-100, -20, 20, 100):
            for n in (1, 70):
                c = Case([n], [300], 8, 2, 128, 16, dt, seed=8)
                c.q = (c.q.double() * 2.0 ** power).to(dt)
                c.check(scale=128 ** -0.5 * 2.0 ** -power)


def _loosely(self):
    """Scores of hundreds: their fp32 error, 2^-21 of sum |q k| scale, is what the weights are off by."""
    out, size, _ = self.exact()
    most = max(float(k.abs().sum(-1).max()) for k in self.keys) * float(self.q.abs().max()) * self.d ** -0.5
    got = self.call()
    tol = 1.01 * U[self.dt] * out.abs() + (1.01 * U[F16] + 2 * most * 2.0 ** -21) * size + 2.0 ** -24
    err = (got.double() - out).abs()
    assert bool((err <= tol).all()), f"worst excess {(err - tol).max().item():.3g}"


Case.compare_loosely = _loosely


def test_scale_and_other_tensors_strides():
    for q_len in ([3, 50], [1, 1], [1, 2]):
        c = Case(q_len, [100, 300], 8, 2, 64, 16, BF, seed=8)
        n = sum(q_len)
        c.check(scale=0.3)
        c.check(scale=0.0)
        c.check(scale=-0.1)
        wide = torch.zeros(n, 8 + 4, 64 + 8, dtype=BF, device="cuda")
        wide[:, 2:10, :64] = c.q
        c.q = wide[:, 2:10, :64]
        out = torch.full((8, n, 64), 5.0, dtype=BF, device="cuda").transpose(0, 1)  # head-major output
        c.check(out=out)
        pages = torch.full((2, c.pages.shape[1] + 9), -1, dtype=torch.int32, device="cuda")
        pages[:, :c.pages.shape[1]] = c.pages
        c.pages = pages[:, :c.pages.shape[1]]
        c.check()
        # codes and scales of other strides: rows 8 and 4 bytes apart from what would be 16
        def moved(t, more):
            x = torch.zeros(t.shape[:3] + (t.shape[3] + more,), dtype=torch.uint8, device="cuda")[..., :t.shape[3]]
            x.copy_(t)
            return x
        c.cache = c.cache._replace(k=moved(c.cache.k, 8), v=moved(c.cache.v, 8), k_scale=moved(c.cache.k_scale, 4),
                                   v_scale=moved(c.cache.v_scale, 4))
        c.check()


def test_same_answers_again_and_on_another_stream():
    for q_len in ([1, 41, 300], [1, 1, 1]):
        c = Case(q_len, [5000, 700, 900], 8, 2, 128, 16, BF, seed=9)
        ws = pps.attention_q4_workspace(sum(q_len), 8, 2, 128)
        first = c.call(ws=ws)
        ws.fill_(255)  # what a workspace holds does not matter
        assert torch.equal(c.call(ws=ws), first)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = c.call(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, first)


def test_in_a_cuda_graph_with_lengths_that_change():
    for q_len in ([1, 1, 1], [41, 41, 41]):
        c = Case(q_len, [500, 900, 130], 8, 2, 128, 16, BF, seed=10)
        ws, out = pps.attention_q4_workspace(sum(q_len), 8, 2, 128), torch.empty_like(c.q)
        c.call(ws=ws, out=out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.call(ws=ws, out=out)
        for lens in ([500, 900, 130], [47, 900, 41], [42, 43, 129]):
            c.kv.copy_(torch.tensor(lens, dtype=torch.int32))
            graph.replay()
            c.kv_len, keys, vals = lens, c.keys, c.values
            c.keys, c.values = [k[:n] for k, n in zip(keys, lens)], [v[:n] for v, n in zip(vals, lens)]
            want, size, _ = c.exact()
            c.keys, c.values = keys, vals
            err = (out.double() - want).abs()
            assert bool((err <= 1.01 * U[BF] * want.abs() + (1.01 * U[F16] + 2e-4) * size + 2.0 ** -24).all())


@pytest.mark.parametrize("q_len", [[1, 1, 1, 1], [1, 2, 1, 1], [40, 50, 1, 60]])
def test_bad_tables_lengths_and_offsets_are_flagged_and_harmless(q_len):
    c = Case(q_len, [100, 60, 40, 70], 8, 2, 128, 16, BF, seed=11)
    good = c.call()
    n_pages = c.cache.k.shape[0]
    of = [slice(a, b) for a, b in zip(c.off, c.off[1:])]
    others = lambda got, s: all(torch.equal(got[of[i]], good[of[i]]) for i in range(4) if i != s)

    def flagged(**kw):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = c.call(status=status, **kw)
        assert int(status.item()) == pps.FLAG_INDEX
        return got

    for wrong in (-1, n_pages, 2 ** 31 - 1):
        pages = c.pages.clone()
        pages[1, 1] = wrong
        got = flagged(pages=pages)
        assert others(got, 1) and bool(torch.isfinite(got).all())  # the page reads as zeros
    kv = c.kv.clone()
    kv[2] = -4
    got = flagged(kv_len=kv)
    assert others(got, 2) and not bool(got[of[2]].any())
    columns = c.pages.shape[1]
    full = c.pages.clamp(min=0).contiguous()
    kv[2] = columns * 16 + 1  # one more than the table holds: cut there
    for t in (c.cache.k_scale, c.cache.v_scale):
        t[t == 0x7f] = 0x30
    got = flagged(kv_len=kv, pages=full)
    kv[2] = columns * 16
    assert torch.equal(got, c.call(kv_len=kv, pages=full))
    good = c.call()
    out = torch.full_like(good, 9.0)
    off = c.off[:3] + [c.off[2] - 1, c.off[4]]
    got = flagged(q_off=torch.tensor(off, dtype=torch.int32, device="cuda"), out=out)
    assert all(torch.equal(got[of[i]], good[of[i]]) for i in (0,))
    out.fill_(9.0)
    got = flagged(q_off=torch.tensor(c.off[:4] + [2 ** 30], dtype=torch.int32, device="cuda"), out=out)
    assert others(got, 3) and bool((got[of[3]] == 9).all())


def test_tokens_of_no_sequence_are_left_as_they_were():
    for q_len in ([1, 1], [30, 60]):
        c = Case(q_len, [100, 300], 8, 2, 128, 16, BF, seed=12)
        n = sum(q_len)
        q = torch.cat([c.q, c.q[:7]])
        out, lse = torch.full_like(q, 9.0), torch.full((n + 7, 8), 9.0, device="cuda")
        got = c.call(q=q, out=out, lse=lse)
        c.compare(got[:n], lse[:n])
        assert bool((got[n:] == 9).all()) and bool((lse[n:] == 9).all())


def test_nothing_to_do():
    c = Case([1, 1], [5, 6], 4, 2, 64, 16, seed=12)
    assert c.call(q=c.q[:0], q_off=torch.zeros(3, dtype=torch.int32, device="cuda")).shape == (0, 4, 64)
    none = pps.CacheQ4(*(t[:0] for t in c.cache[:4]))
    assert not bool(c.call(cache=none, pages=c.pages[:, :0], kv_len=c.kv * 0).any())


@pytest.mark.parametrize("q_len", [[1, 1, 1], [3, 1, 2], [50, 41, 60]])
@pytest.mark.parametrize("x", [float("nan"), float("inf"), float("-inf")])
def test_queries_that_are_not_finite(q_len, x):
    c = Case(q_len, [70, 300, 5000], 8, 2, 128, 16, BF, seed=1)
    c.q[1, 1, 5] = x
    assert bool(c.nan_rows()[1, 1])


@pytest.mark.parametrize("q_len", [[1, 1], [3, 2], [50, 60]])
def test_keys_that_are_nan_reach_the_tokens_that_see_them(q_len):
    c = Case(q_len, [300, 900], 8, 2, 128, 16, F16, seed=5)
    for j in (100, 299):  # before the new tokens; the last token's own
        at = int(c.pages[0, j // 16]), j % 16
        keep = c.cache.k_scale[at].clone()
        c.cache.k_scale[at][1, 3] = 0x7f  # a block of key head 1
        c.keys[0][j, 1, 48:64] = float("nan")
        c.nan_rows()
        c.cache.k_scale[at] = keep
        c.keys[0][j, 1] = values(c.cache.k[at], c.cache.k_scale[at])[1]


def test_refusals():
    c = Case([1, 2], [20, 30], 4, 2, 64, 16, seed=13)
    k = c.cache
    for bad in (dict(q=c.q.float()), dict(cache=k.k), dict(cache=None), dict(pages=c.pages.long()), dict(q=7), dict(kv_len=None),
                dict(kv_len=c.kv.long()), dict(q_off=c.q_off.cpu()), dict(mask=torch.zeros(3, 1, device="cuda")),
                dict(lse=torch.zeros(12, dtype=torch.float64, device="cuda")), dict(out=c.q.half()),
                dict(cache=k._replace(k=k.k.to(torch.int8))), dict(cache=k._replace(k_scale=None))):
        with pytest.raises(TypeError):
            c.call(**bad)
    for bad in (dict(cache=k._replace(v=k.v[:, :8])), dict(q=c.q[..., :32]), dict(q_off=c.q_off[:2]),
                dict(mask=torch.zeros(2, 1, dtype=torch.int32, device="cuda")), dict(out=c.q[:2]),
                dict(mask=torch.zeros(3, 0, dtype=torch.int32, device="cuda")),
                dict(lse=torch.zeros(5, device="cuda")), dict(cache=k._replace(v=k.v.contiguous()))):
        with pytest.raises(ValueError):
            c.call(**bad)

    def code(**kw):
        with pytest.raises(pps.PPSError) as e:
            c.call(**kw)
        return e.value.code

    assert code(q=c.q[:, :3]) == pps.ERR_INVALID_ARG  # heads that the key heads do not divide
    assert code(scale=float("nan")) == pps.ERR_INVALID_ARG
    assert code(ws=torch.empty(16, dtype=torch.uint8, device="cuda")) == pps.ERR_WORKSPACE
    assert code(pages=c.pages[:1].expand(2, -1)) == pps.ERR_INVALID_ARG  # rows of the table that overlap
    for d, page in ((144, 16), (64, 12), (64, 4)):
        assert code(q=torch.zeros(3, 4, d, dtype=BF, device="cuda"), cache=pps.cache_q4(3, page, 2, d)) == pps.ERR_UNSUPPORTED
    odd = torch.zeros(3 * 2 * 16 * 36, dtype=torch.uint8, device="cuda").view(3, 16, 2, 36)[..., :32]
    assert code(cache=pps.CacheQ4(odd, odd, k.k_scale[:3], k.v_scale[:3])) == pps.ERR_INVALID_ARG  # rows that are not 8-byte aligned
