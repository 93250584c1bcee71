"""pps_paged_attention against the formula in 64 bits: lengths, masks, head layouts, pages, strides, refusals."""
import math
import random

import pytest
import torch

from paper_2609_21858_gb300 import pps

pytestmark = pytest.mark.gpu

BF, F16 = torch.bfloat16, torch.float16
U = {BF: 2.0 ** -8, F16: 2.0 ** -11}  # unit roundoff


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    pps.lib()


class Case:
    """q_len and kv_len of every sequence; what slots past a sequence's end hold is NaN."""

    def __init__(self, q_len, kv_len, heads, kv_heads, d, page, dt=BF, tree=False, layout="token", seed=0, spare=1,
                 q_scale=2.0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.q_len, self.kv_len, self.heads, self.kv_heads, self.d, self.page, self.dt = (q_len, kv_len, heads, kv_heads, d,
                                                                                         page, dt)
        n_seq, n = len(q_len), sum(q_len)
        held = [-(-x // page) for x in kv_len]
        n_pages = sum(held) + 2
        order = torch.randperm(n_pages, generator=g, device="cuda").tolist()
        width = max(held) + spare
        table = [[-7] * width for _ in range(n_seq)]
        self.keys, self.values = [], []
        pools = []
        for _ in range(2):
            shape = (n_pages, kv_heads, page, d) if layout == "head" else (n_pages, page, kv_heads, d)
            x = torch.full(shape, float("nan"), dtype=dt, device="cuda")
            pools.append(x.transpose(1, 2) if layout == "head" else x)
        at = 0
        for s in range(n_seq):
            mine = order[at:at + held[s]]
            at += held[s]
            table[s][:held[s]] = mine
            j = torch.arange(kv_len[s], device="cuda")
            page_of = torch.tensor(mine, device="cuda", dtype=torch.long)[j // page] if kv_len[s] else j
            for pool, into in zip(pools, (self.keys, self.values)):
                x = torch.randn(kv_len[s], kv_heads, d, generator=g, device="cuda").to(dt)
                pool[page_of, j % page] = x
                into.append(x)
        self.k_cache, self.v_cache = pools
        self.pages = torch.tensor(table, dtype=torch.int32, device="cuda").view(n_seq, width)
        self.q = (torch.randn(n, heads, d, generator=g, device="cuda") * q_scale).to(dt)
        off = [0]
        for x in q_len:
            off.append(off[-1] + x)
        self.off = off
        self.q_off = torch.tensor(off, dtype=torch.int32, device="cuda")
        self.kv = torch.tensor(kv_len, dtype=torch.int32, device="cuda")
        self.mask = self.bits = None
        if tree:
            words = max(1, -(-max(q_len) // 32))
            self.mask = torch.randint(-2 ** 31, 2 ** 31, (n, words), generator=g, device="cuda").to(torch.int32)
            if n > 2:
                self.mask[n // 2] = 0  # sees nothing of its own tree
            self.bits = ((self.mask[:, :, None].long() >> torch.arange(32, device="cuda")) & 1).flatten(1).bool()

    def call(self, **kw):
        args = dict(q=self.q, k_cache=self.k_cache, v_cache=self.v_cache, pages=self.pages, kv_len=self.kv,
                    q_off=self.q_off, mask=self.mask)
        return pps.paged_attention(**{**args, **kw})

    def exact(self, scale=None):
        """(out, sum_j w_j |v_j| / sum_j w_j, lse) in 64 bits."""
        scale = 1 / math.sqrt(self.d) if scale is None else scale
        out = torch.zeros(self.q.shape, dtype=torch.float64, device="cuda")
        size, lse = torch.zeros_like(out), torch.full(self.q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
        group = self.heads // self.kv_heads
        for s, (n, L) in enumerate(zip(self.q_len, self.kv_len)):
            if n == 0 or L == 0:
                continue
            a, b = self.off[s], self.off[s] + n
            rel = torch.arange(L, device="cuda") - (L - n)
            i = torch.arange(n, device="cuda")[:, None]
            if self.mask is None:
                sees = rel[None, :] <= i
            else:
                own = self.bits[a:b][:, rel.clamp(min=0)] if n else None
                sees = (rel[None, :] < 0) | own
            k, v = (x[s].double().repeat_interleave(group, dim=1) for x in (self.keys, self.values))
            w = torch.einsum("ihd,jhd->hij", self.q[a:b].double(), k) * scale
            w = w.masked_fill(~sees[None], -math.inf)
            l = torch.logsumexp(w, dim=-1)
            p = torch.where(torch.isinf(l)[..., None], 0.0, torch.exp(w - l.clamp(min=-1e300)[..., None]))
            out[a:b] = torch.einsum("hij,jhd->ihd", p, v)
            size[a:b] = torch.einsum("hij,jhd->ihd", p, v.abs())
            lse[a:b] = l.T
        return out, size, lse

    def check(self, **kw):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        lse = torch.full(self.q.shape[:2], 7.0, dtype=torch.float32, device="cuda")
        got = self.call(status=status, lse=lse, **kw)
        assert int(status.item()) == 0
        self.compare(got, lse, kw.get("scale"))
        return got

    def compare(self, got, lse, scale=None):
        out, size, want = self.exact(scale)
        # the weights and the result are each rounded once to 16 bits; scores carry fp32 errors (products of 128
        # channels summed in fp32: below 2^-21 of sum |q k| scale, here under 40), weights of fp16 below 2^-24 are
        # subnormal
        err, tol = (got.double() - out).abs(), 1.01 * U[self.dt] * (out.abs() + size) + 1e-4 * size + 2.0 ** -24
        assert bool((err <= tol).all()), f"worst excess {(err - tol).max().item():.3g}"
        seen = torch.isfinite(want)
        assert bool((torch.isneginf(lse) == ~seen).all())
        assert bool(((lse.double() - want)[seen].abs() <= 1e-4 + 1e-6 * want[seen].abs()).all())
        assert bool((got[~seen] == 0).all())


@pytest.mark.parametrize("heads,kv_heads,d", [(32, 8, 128), (28, 4, 128), (14, 2, 64), (6, 6, 64), (16, 1, 128),
                                              (20, 4, 80), (3, 1, 8), (9, 3, 104), (5, 5, 40), (130, 1, 64)])
@pytest.mark.parametrize("dt", [BF, F16])
def test_one_token_each(heads, kv_heads, d, dt):
    kv = [1, 2, 127, 128, 129, 255, 256, 257, 700, 1, 1111]
    Case([1] * len(kv), kv, heads, kv_heads, d, 16, dt, seed=heads + d).check()


@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256, 512])
@pytest.mark.parametrize("layout", ["token", "head"])
def test_page_sizes_and_layouts(page, layout):
    Case([1, 5, 40], [300, 513, 1030], 8, 2, 128, page, BF, layout=layout, seed=page).check()
    Case([3, 1, 70], [129, 5, 400], 4, 4, 64, page, F16, layout=layout, seed=page + 1, tree=True).check()


# chunks whose packed rows (tokens x group) end inside, at and past a tile of 128 and of 256 rows
@pytest.mark.parametrize("heads,kv_heads,d", [(4, 4, 128), (8, 2, 128), (7, 1, 64), (12, 4, 80)])
@pytest.mark.parametrize("n", [2, 31, 32, 33, 63, 64, 65, 85, 86, 127, 128, 129, 256, 257, 385, 600])
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


def test_sequences_without_keys_and_tokens_that_see_nothing():
    # more tokens than keys: the first tokens' positions lie before the first key
    Case([4, 3, 2, 1], [0, 1, 2, 0], 8, 2, 64, 16, seed=1).check()
    Case([300, 200], [100, 0], 4, 4, 128, 16, seed=2).check()
    # trees without a prefix, some masks empty
    Case([5, 40, 33], [5, 40, 33], 8, 2, 128, 16, F16, tree=True, seed=3).check()


@pytest.mark.parametrize("dt", [BF, F16])
@pytest.mark.parametrize("n,prefix", [(1, 50), (2, 127), (31, 97), (32, 96), (33, 95), (41, 128), (41, 1000), (64, 1),
                                      (65, 300), (200, 77), (300, 513)])
def test_trees(n, prefix, dt):
    Case([n, n, 1], [n + prefix, n, 1 + prefix], 8, 2, 128, 16, dt, tree=True, seed=n + prefix).check()


def test_long_sequences_split_over_the_whole_gpu():
    Case([1], [40001], 8, 1, 128, 64, BF, seed=1).check()
    Case([1, 1], [20011, 3], 4, 4, 64, 16, F16, seed=2).check()
    Case([41], [30000], 8, 2, 128, 16, BF, tree=True, seed=3).check()
    Case([130], [9000], 4, 2, 128, 256, F16, seed=4).check()


def test_large_scores_and_equal_scores():
    # a few keys carry all the weight, at any place; the running maximum rises late
    c = Case([1, 65], [600, 777], 8, 2, 128, 16, BF, seed=5, q_scale=30.0)
    c.check()
    # all scores zero: the mean of the values
    c = Case([1, 65], [600, 777], 8, 2, 128, 16, BF, seed=6, q_scale=0.0)
    c.check()
    # a rising ramp of scores: every tile raises the maximum
    c = Case([1], [3000], 4, 1, 64, 16, BF, seed=7)
    c.q.fill_(1.0)
    for j in range(3000):
        c.keys[0][j] = 0.02 * j
    page_of = c.pages[0].long()[torch.arange(3000, device="cuda") // 16]
    c.k_cache[page_of, torch.arange(3000, device="cuda") % 16] = c.keys[0]
    c.check()


def test_scale_and_other_tensors_strides():
    c = Case([3, 50], [100, 300], 8, 2, 64, 16, BF, seed=8)
    c.check(scale=0.3)
    c.check(scale=0.0)
    c.check(scale=-0.1)
    wide = torch.zeros(53, 8 + 4, 64 + 8, dtype=BF, device="cuda")
    wide[:, 2:10, :64] = c.q
    c.q = wide[:, 2:10, :64]
    assert not c.q.is_contiguous()
    out = torch.full((8, 53, 64), 5.0, dtype=BF, device="cuda").transpose(0, 1)  # head-major output
    c.check(out=out)
    pages = torch.full((2, c.pages.shape[1] + 9), -1, dtype=torch.int32, device="cuda")
    pages[:, :c.pages.shape[1]] = c.pages
    c.pages = pages[:, :c.pages.shape[1]]
    c.check()


def test_same_answers_again_and_on_another_stream():
    c = Case([1, 41, 300], [5000, 700, 900], 8, 2, 128, 16, BF, seed=9)
    ws = pps.attention_workspace(342, 8, 2, 128)
    first = c.call(ws=ws)
    ws.fill_(255)  # what a workspace holds does not matter
    assert torch.equal(c.call(ws=ws), first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.call(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, first)


def test_in_a_cuda_graph_with_lengths_that_change():
    c = Case([1, 1, 1], [500, 900, 130], 8, 2, 128, 16, BF, seed=10)
    ws, out = pps.attention_workspace(3, 8, 2, 128), torch.empty_like(c.q)
    c.call(ws=ws, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call(ws=ws, out=out)
    for lens in ([500, 900, 130], [17, 900, 0], [1, 2, 129]):
        c.kv.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        c.kv_len, keys, values = lens, c.keys, c.values
        c.keys, c.values = [k[:n] for k, n in zip(keys, lens)], [v[:n] for v, n in zip(values, lens)]
        want, size, _ = c.exact()
        c.keys, c.values = keys, values
        err = (out.double() - want).abs()
        assert bool((err <= 1.01 * U[BF] * (want.abs() + size) + 1e-4 * size + 2.0 ** -24).all())


def test_bad_tables_lengths_and_offsets_are_flagged_and_harmless():
    c = Case([1, 2, 1, 1], [100, 60, 40, 30], 8, 2, 128, 16, BF, seed=11)
    good = c.call()
    n_pages = c.k_cache.shape[0]

    def flagged(**kw):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = c.call(status=status, **kw)
        assert int(status.item()) == pps.FLAG_INDEX
        return got

    for wrong in (-1, n_pages, 2 ** 31 - 1):
        pages = c.pages.clone()
        pages[1, 1] = wrong
        got = flagged(pages=pages)
        assert torch.equal(got[[0, 3, 4]], good[[0, 3, 4]])
        assert bool(torch.isfinite(got).all())  # the page reads as zeros
    kv = c.kv.clone()
    kv[2] = -4
    got = flagged(kv_len=kv)
    assert torch.equal(got[[0, 1, 2, 4]], good[[0, 1, 2, 4]]) and not bool(got[3].any())
    columns = c.pages.shape[1]
    full = c.pages.clamp(min=0).contiguous()
    kv[2] = columns * 16 + 1  # one more than the table holds: cut there
    k0, v0 = torch.nan_to_num(c.k_cache), torch.nan_to_num(c.v_cache)
    got = flagged(kv_len=kv, pages=full, k_cache=k0, v_cache=v0)
    kv[2] = columns * 16
    assert torch.equal(got, c.call(kv_len=kv, pages=full, k_cache=k0, v_cache=v0))
    out = torch.full_like(good, 9.0)
    got = flagged(q_off=torch.tensor([0, 1, 3, 2, 5], dtype=torch.int32, device="cuda"), out=out)
    assert torch.equal(got[:2], good[:2])  # token 2 is claimed by the second and the last sequence
    out.fill_(9.0)
    got = flagged(q_off=torch.tensor([0, 1, 3, 4, 2 ** 30], dtype=torch.int32, device="cuda"), out=out)
    assert torch.equal(got[:4], good[:4]) and bool((got[4] == 9).all())


def test_nothing_to_do():
    c = Case([1, 1], [5, 6], 4, 2, 64, 16, seed=12)
    assert c.call(q=c.q[:0], q_off=torch.zeros(3, dtype=torch.int32, device="cuda")).shape == (0, 4, 64)
    got = c.call(k_cache=c.k_cache[:0], v_cache=c.v_cache[:0], pages=c.pages[:, :0], kv_len=c.kv * 0)
    assert not bool(got.any())


def test_refusals():
    c = Case([1, 2], [20, 30], 4, 2, 64, 16, seed=13)
    for bad in (dict(q=c.q.float()), dict(q=c.q.half()), dict(k_cache=c.k_cache[0]), dict(pages=c.pages.long()),
                dict(kv_len=c.kv.long()), dict(q_off=c.q_off.cpu()), dict(mask=torch.zeros(3, 1, device="cuda")),
                dict(lse=torch.zeros(12, dtype=torch.float64, device="cuda")), dict(out=c.q.half())):
        with pytest.raises(TypeError):
            c.call(**bad)
    for bad in (dict(v_cache=c.v_cache[:, :8]), dict(q=c.q[..., :32]), dict(q_off=c.q_off[:2]),
                dict(mask=torch.zeros(2, 1, dtype=torch.int32, device="cuda")), dict(out=c.q[:2]),
                dict(mask=torch.zeros(3, 0, dtype=torch.int32, device="cuda")),
                dict(lse=torch.zeros(5, device="cuda"))):
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
    for d, page in ((136, 16), (64, 12), (64, 4)):
        k, v = (torch.zeros(3, page, 2, d, dtype=BF, device="cuda") for _ in range(2))
        assert code(q=torch.zeros(3, 4, d, dtype=BF, device="cuda"), k_cache=k, v_cache=v) == pps.ERR_UNSUPPORTED
    k, v = (torch.zeros(3 * 16 * 2 * 68, dtype=BF, device="cuda").view(3, 16, 2, 68)[..., :64] for _ in range(2))
    assert code(k_cache=k, v_cache=v) == pps.ERR_INVALID_ARG  # rows that are not 16-byte aligned
