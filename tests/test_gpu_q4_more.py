"""The 4-bit cache's calls where offsets pass 32 bits, where one kernel hands over to the other, from several threads and from two graphs."""
import threading

import pytest
import torch

import test_gpu_q4_append as appends
from paper_2609_21858_gb300 import pps
from test_gpu_q4_attention import BF, F16, Case, _cuda  # noqa: F401

pytestmark = pytest.mark.gpu


# rows of a sequence and key head around 32, on average and by sequence
@pytest.mark.parametrize("heads,kv_heads", [(32, 1), (33, 1), (31, 1), (8, 2), (6, 6)])
@pytest.mark.parametrize("q_len", [[1, 1], [8, 8], [8, 9], [9, 9], [1, 15], [2, 130, 0, 0, 0, 0, 0, 0], [32, 32], [33, 33]])
def test_where_the_kernels_meet(heads, kv_heads, q_len):
    Case(q_len, [n + 3 * i + 200 for i, n in enumerate(q_len)], heads, kv_heads, 64, 16, BF, seed=heads + len(q_len)).check()
    Case(q_len, [n + 3 * i + 70 for i, n in enumerate(q_len)], heads, kv_heads, 128, 8, F16, tree=True, seed=heads + len(q_len)).check()


@pytest.mark.parametrize("heads,kv_heads,d", [(8, 2, 128), (4, 4, 64), (6, 1, 128), (3, 1, 64)])
@pytest.mark.parametrize("page", [16, 32, 128])
@pytest.mark.parametrize("more", [(0, 0), (16, 8), (48, 4), (8, 8)])
def test_rows_that_lie_apart(heads, kv_heads, d, page, more):
    """Pages token by token, rows of codes and of scales with something between them, a page that is missing."""
    c = Case([1, 2, 1], [700, 131, 2 * page + 1], heads, kv_heads, d, page, BF, layout="token", seed=page + d, unit=True)

    def apart(t, n):
        x = torch.full(t.shape[:3] + (t.shape[3] + n,), 0x7f, dtype=torch.uint8, device="cuda")
        x[..., :t.shape[3]] = t
        return x[..., :t.shape[3]]

    k = c.cache
    c.cache = k._replace(k=apart(k.k, more[0]), v=apart(k.v, more[0]), k_scale=apart(k.k_scale, more[1]), v_scale=apart(k.v_scale, more[1]))
    good = c.check()
    pages, status = c.pages.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    pages[1, 0] = c.cache.k.shape[0]
    got = c.call(pages=pages, status=status)
    assert int(status.item()) == pps.FLAG_INDEX and torch.equal(got[:1], good[:1]) and torch.equal(got[3:], good[3:])
    assert bool(torch.isfinite(got).all())


def test_a_cache_of_one_page():
    for layout in ("token", "head"):
        for d in (64, 128):
            c = Case([1], [61], 8, 2, d, 64, F16, layout=layout, seed=d)
            at = int(c.pages[0, 0])
            c.cache = pps.CacheQ4(*(t[at:at + 1] for t in c.cache[:4]))
            c.pages.fill_(0)
            c.check()


@pytest.mark.parametrize("q_len", [[1, 1], [2, 3], [50, 60]])
@pytest.mark.parametrize("dt", [BF, F16])
def test_factors_on_scores_that_vanish(q_len, dt):
    """Units and queries whose product with the scale has no number in 32 bits: equal weights."""
    c = Case(q_len, [300, 90], 8, 2, 64, 16, dt, seed=14)
    c.cache = c.cache._replace(k_unit=torch.full((2,), 1e-30, device="cuda"))
    c.keys = [k.double() * 1e-30 for k in c.keys]
    if dt is BF:
        c.q = (c.q.double() * 2.0 ** -110).to(dt)
    c.check()
    c.check(scale=1e-38)


def test_a_tree_whose_first_nodes_are_not_seen():
    """Seven rows of a key head, whose first keys no row sees, at scales down to the smallest."""
    c = Case([200, 1, 1, 1, 1, 1, 1, 1], [200, 3, 3, 3, 3, 3, 3, 3], 1, 1, 64, 16, BF, tree=True, seed=15)
    c.mask[:200, :5] = 0
    c.bits[:200, :160] = False
    for scale in (None, 1e-20, 1e-38, 0.0):
        c.check(**({} if scale is None else dict(scale=scale)))
    c.q = (c.q.double() * 2.0 ** -120).to(BF)
    c.check()


def _i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def far(cache, pages, layout):
    """The cache's pages behind so many others that their bytes lie past 2^32, and the table that says so."""
    n, page, heads, d2 = cache.k.shape
    first = 2 ** 32 // (page * heads * d2) + 5

    def moved(t):
        shape = (first + n, heads, page, t.shape[3]) if layout == "head" else (first + n, page, heads, t.shape[3])
        x = torch.zeros(shape, dtype=torch.uint8, device="cuda")
        x = x.transpose(1, 2) if layout == "head" else x
        x[first:] = t
        return x

    return cache._replace(**{k: moved(getattr(cache, k)) for k in ("k", "v", "k_scale", "v_scale")}), torch.where(pages >= 0, pages + first, pages)


@pytest.mark.parametrize("layout", ["token", "head"])
def test_caches_past_32_bits(layout):
    for q_len in ([1, 1, 1], [40, 33, 70]):
        c = Case(q_len, [500, 333, 70], 8, 8, 128, 64, BF, layout=layout, seed=3)
        c.cache, c.pages = far(c.cache, c.pages, layout)
        c.check()
    # what is appended there is what is appended near, it reads back, and the pages before it are left as they were
    n, rows = 9, torch.randn(3, 9, 8, 128, device="cuda").to(BF)
    near, near_at = pps.cache_q4(2, 64, 8, 128), torch.arange(3, 3 + n, device="cuda")
    first = c.cache.k.shape[0] - 2
    slot = first * 64 + near_at
    for cache, at in ((near, near_at), (c.cache, slot)):
        pps.kv_append_q4(rows[0], rows[1], rows[2], None, at, cache, None)
    for a, b in zip(near[:4], c.cache[:4]):
        assert torch.equal(a[0, 3:3 + n], b[first, 3:3 + n])
    for a, b in zip(pps.kv_read_q4(near, near_at), pps.kv_read_q4(c.cache, slot)):
        assert torch.equal(a, b) and bool(a.any())
    assert not any(bool(t[:20].any()) for t in c.cache[:4])


@pytest.mark.parametrize("named", [False, True])
def test_threads(named):
    """Several threads, each on a stream of its own and without a workspace."""
    jobs = []
    for i in range(6):
        attend = Case([1, 1, 1] if i % 2 else [1, 30 + i, 40], [3000 + 500 * i, 200, 900], 8, 2, 128 if i % 3 else 64, 16, BF if i % 2 else F16, seed=i)
        x = torch.randn(9 + i, 30001 + 16 * i, device="cuda").to(BF)
        text = torch.randint(0, x.shape[1], (3, 50), device="cuda", dtype=torch.int32)
        off, lens, laws = _i32(0, 2, 3, 9 + i), _i32(50, 7, 33), torch.tensor([1.3, 1.0, 2.0], device="cuda")
        shape = lambda x=x, off=off, text=text, lens=lens, laws=laws, **kw: pps.adjust_logits(
            x, off, text=text, text_len=lens, repetition=laws, presence=laws, **kw)
        jobs.append((attend, shape, attend.call(), shape()))
    torch.cuda.synchronize()
    wrong = []

    def work(attend, shape, out, shaped):
        try:
            stream = torch.cuda.Stream()
            kw = dict(stream=stream) if named else {}
            with torch.cuda.stream(stream):
                for _ in range(30):
                    a, b = attend.call(**kw), shape(**kw)
                    if not torch.equal(a, out) or not torch.equal(b, shaped):
                        wrong.append("differs")
                stream.synchronize()
        except Exception as e:  # a thread's exception would be lost
            wrong.append(repr(e))

    threads = [threading.Thread(target=work, args=job) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong


def test_two_graphs_at_the_same_time_with_a_workspace_each():
    cases = [Case([1] * 5, [4000, 900, 20, 7000, 3], 8, 2, 128, 16, BF, seed=1), Case([41, 9], [5000, 600], 8, 2, 128, 16, BF, seed=2)]
    graphs, outs, wants, streams = [], [], [], []
    for c in cases:
        ws, out = pps.attention_q4_workspace(sum(c.q_len), 8, 2, 128), torch.empty_like(c.q)
        wants.append(c.call(ws=ws, out=out).clone())
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _ in range(20):
                c.call(ws=ws, out=out)
        graphs.append((graph, ws))
        outs.append(out.fill_(3.0))
        streams.append(torch.cuda.Stream())
    torch.cuda.synchronize()
    for _ in range(5):
        for (graph, _ws), stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, wants))


@pytest.mark.parametrize("n,hq,hk,d,rot,page,dt", [(9001, 28, 4, 128, 128, 16, F16), (7777, 6, 2, 64, 48, 32, BF), (20011, 1, 1, 32, 32, 64, BF)])
@pytest.mark.parametrize("norm,offset", [(False, 0), (True, 0), (True, 4)])
def test_appends_whose_warps_take_many_tokens(n, hq, hk, d, rot, page, dt, norm, offset):
    appends.test_against_the_formulas(n, hq, hk, d, rot, page, dt, norm, False, "head", offset, True)


class Server:
    """Three sequences, pages from a pool, five tokens a step of which two are kept."""

    def __init__(self):
        g = torch.Generator(device="cuda").manual_seed(5)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF)
        self.q, self.k, self.v, self.logits = rnd(17, 8, 64), rnd(17, 2, 64), rnd(17, 2, 64), rnd(17, 5003)
        self.cache, self.rope = pps.cache_q4(64, 16, 2, 64), pps.rope_table(512, 64)
        self.pages, self.held = torch.full((3, 20), -1, dtype=torch.int32, device="cuda"), _i32(0, 0, 0)
        self.free_list, self.free_count = torch.randperm(64, generator=g, device="cuda").int(), _i32(64)
        self.kv_len, self.new, self.laws = _i32(30, 0, 100), _i32(5, 5, 5), torch.tensor([1.3, 2.0, 0.5], device="cuda")
        self.text = torch.randint(0, 5003, (3, 200), generator=g, device="cuda", dtype=torch.int32)
        self.status = _i32(0)
        # what the sequences hold already
        pool = (self.pages, self.held, self.free_list, self.free_count)
        at = pps.kv_reserve(*pool, _i32(0, 0, 0), self.kv_len, 16, 130)
        pps.kv_append_q4(rnd(130, 8, 64), rnd(130, 2, 64), rnd(130, 2, 64), at["pos"], at["slot"], self.cache, self.rope)

    def step(self):
        pool = (self.pages, self.held, self.free_list, self.free_count)
        at = pps.kv_reserve(*pool, self.kv_len, self.new, 16, 17, status=self.status)  # a batch padded by two
        q = pps.kv_append_q4(self.q, self.k, self.v, at["pos"], at["slot"], self.cache, self.rope, status=self.status)
        a = pps.paged_attention_q4(q, self.cache, self.pages, at["kv_len"], at["q_off"], out=torch.zeros_like(q), status=self.status)
        x = pps.adjust_logits(self.logits, at["q_off"], text=self.text, text_len=self.kv_len, repetition=self.laws, frequency=self.laws,
                              out=torch.zeros_like(self.logits), status=self.status)
        self.kv_len.add_(2)
        pps.kv_trim(*pool, self.kv_len, 16, status=self.status)
        k, v = pps.kv_read_q4(self.cache, at["slot"])
        return a, x, k, v, at["slot"], at["pos"], at["seq"]


def test_a_step_of_all_calls_captured_and_replayed():
    eager, server = Server(), Server()
    want = [[t.clone() for t in eager.step()] for _ in range(12)]
    assert int(eager.status) == 0 and bool((want[0][4][15:] == -1).all()) and not bool(want[0][0][15:].any())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = server.step()
    for w in want:
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, w))
    assert int(server.status) == 0 and torch.equal(server.held, eager.held) and torch.equal(server.free_count, eager.free_count)
    assert torch.equal(server.kv_len, _i32(54, 24, 124)) and torch.equal(server.held, _i32(4, 2, 8))
    # the two tokens that each step kept are in the cache, in the pages that the table says
    k, _ = pps.kv_read_q4(server.cache, server.pages[1, 0].long() * 16 + torch.arange(16, device="cuda"))
    last = pps.cache_q4(1, 16, 2, 64)
    at = torch.tensor([14, 15], device="cuda")
    pps.kv_append_q4(server.q[5:7], server.k[5:7], server.v[5:7], at.int(), at, last, server.rope)
    assert torch.equal(k[14:], pps.kv_read_q4(last, at)[0])
