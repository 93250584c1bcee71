"""pps_kv_reserve and pps_kv_trim against a plain restatement, sequence by sequence."""
import random

import pytest
import torch

from paper_2609_21858_gb300 import pps

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    pps.lib()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Pool:
    """Tables, pool and lengths, on the device and as lists."""

    def __init__(self, lens, columns, page, spare, rng, extra_columns=0, lose=0):
        self.page, self.columns, self.lens = page, columns, list(lens)
        held = [-(-n // page) for n in lens]
        assert max(held, default=0) <= columns
        order = list(range(sum(held) + spare))
        rng.shuffle(order)
        self.table, at = [], 0
        for h in held:
            self.table.append(order[at:at + h])
            at += h
        self.free = order[at:]
        self.cap = len(order) - lose
        self.n_seq = len(lens)
        wide = torch.full((self.n_seq, columns + extra_columns), -9, dtype=torch.int32, device="cuda")
        self.pages = wide[:, :columns]
        self.wide = wide
        for s, row in enumerate(self.table):
            self.pages[s] = i32(row + [-1] * (columns - len(row)))
        self.held = i32(held)
        self.free_list = i32((self.free + [-5] * self.cap)[:self.cap])
        self.free_count = i32([len(self.free)])

    def reserve(self, n_new, n_tok, pos_off=None, status=0, **kw):
        flags = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = pps.kv_reserve(self.pages, self.held, self.free_list, self.free_count, i32(self.lens), i32(n_new), self.page,
                             n_tok, pos_off=None if pos_off is None else i32(pos_off), status=flags, **kw)
        want = dict(q_off=[0], kv_len=[], slot=[], pos=[], seq=[])
        room, over = len(self.free), False
        asked = 0
        for s, n in enumerate(n_new):
            total = self.lens[s] + n
            upto = -(-total // self.page)
            need = max(0, upto - len(self.table[s])) if n else 0
            served = upto <= self.columns
            if served:
                asked += need
                if need and asked > room:
                    served, over = False, True
            if served:
                for _ in range(need):
                    self.table[s].append(self.free.pop())
            for i in range(n):
                place = self.lens[s] + i
                t = len(want["slot"])
                want["slot"].append(self.table[s][place // self.page] * self.page + place % self.page if served else -1)
                want["pos"].append(self.lens[s] + (i if pos_off is None or t >= n_tok else pos_off[t]))
                want["seq"].append(s)
            want["q_off"].append(want["q_off"][-1] + n)
            want["kv_len"].append(total if served else 0)
        for name, fill in (("slot", -1), ("pos", 0), ("seq", -1)):
            want[name] = (want[name] + [fill] * n_tok)[:n_tok]
        for name, x in want.items():
            if name in got:
                assert got[name].tolist() == x, name
        assert bool(int(flags) & pps.FLAG_POOL) == over
        assert int(flags) & ~pps.FLAG_POOL == status
        self.check()
        return want

    def trim(self, keep, status=0):
        flags = torch.zeros(1, dtype=torch.int32, device="cuda")
        pps.kv_trim(self.pages, self.held, self.free_list, self.free_count, i32(keep), self.page, status=flags)
        back = []
        for s, n in enumerate(keep):
            k = min(-(-max(n, 0) // self.page), len(self.table[s]))
            back += self.table[s][k:]
            self.table[s] = self.table[s][:k]
        self.free += back[::-1]
        self.free = self.free[:self.cap]
        assert int(flags) == status
        self.check()

    def check(self):
        for s, row in enumerate(self.table):
            assert self.pages[s].tolist() == row + [-1] * (self.columns - len(row))
        assert self.held.tolist() == [len(r) for r in self.table]
        assert self.free_count.tolist() == [len(self.free)]
        assert self.free_list[:len(self.free)].tolist() == self.free
        assert bool((self.wide[:, self.columns:] == -9).all())


@pytest.mark.parametrize("n_seq,q,most,page", [(1, 1, 0, 16), (1, 1, 50, 16), (8, 1, 400, 16), (3, 41, 300, 8), (64, 41, 900, 16),
                                               (5, 7, 100, 3), (600, 3, 40, 1), (513, 5, 200, 64), (2, 3000, 100, 16),
                                               (1, 20000, 5, 8), (2000, 1, 60, 16)])
@pytest.mark.parametrize("short", [False, True])
def test_steps(n_seq, q, most, page, short):
    rng = random.Random(n_seq * 7 + q)
    lens = [rng.randint(0, most) for _ in range(n_seq)]
    columns = -(-(most + 3 * q) // page) + 1
    spare = sum(-(-(n + q) // page) + (-n // page) for n in lens) // (2 if short else 1) + (0 if short else 3 * n_seq * (q // page + 2))
    p = Pool(lens, columns, page, spare, rng, extra_columns=n_seq % 3)
    for step in range(3):
        n_new = [rng.choice([q, q, rng.randint(0, q), 0]) for _ in range(n_seq)]
        n_tok = sum(n_new) + (9 if step == 1 else 0)
        pos_off = [rng.randint(0, 9) for _ in range(n_tok)] if step == 2 else None
        want = p.reserve(n_new, n_tok, pos_off)
        keep = [max(n, min(rng.randint(n, n + m), w)) for n, m, w in zip(p.lens, n_new, want["kv_len"])]
        if step == 1 and n_seq > 1:
            keep[0] = 0  # one sequence ends
        p.trim(keep)
        p.lens = keep


def test_trim_is_the_inverse_of_reserve():
    rng = random.Random(5)
    p = Pool([30, 0, 17, 64], 20, 16, 40, rng)
    before, table = list(p.free), [list(r) for r in p.table]
    want = p.reserve([41, 3, 100, 0], 144)
    p.trim(p.lens)
    assert p.free == before and p.table == table
    assert p.reserve([41, 3, 100, 0], 144) == want  # the same pages again


def test_a_pool_that_is_empty_and_rows_that_are_full():
    rng = random.Random(6)
    p = Pool([16, 15, 32], 3, 16, 0, rng)
    want = p.reserve([0, 1, 0], 1)  # has room in its last page
    assert want["kv_len"] == [16, 16, 32]
    p = Pool([16, 15, 32], 3, 16, 2, rng)
    p.reserve([1, 1, 40], 42, status=pps.FLAG_INDEX)  # the last passes its columns, and demands nothing
    p = Pool([0, 0, 0, 0], 9, 16, 4, rng)
    want = p.reserve([40, 40, 1, 0], 81)  # 3 of 4; 3 more do not fit; nor does one after them
    assert want["kv_len"] == [40, 0, 0, 0]


def test_more_tokens_than_the_outputs_hold():
    p = Pool([5, 6], 4, 16, 9, random.Random(7))
    p.reserve([10, 20], 17, status=pps.FLAG_INDEX)


def test_lengths_that_are_negative_and_tables_that_are_wrong():
    rng = random.Random(8)
    p = Pool([5, 20, 6], 4, 16, 9, rng)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = pps.kv_reserve(p.pages, p.held, p.free_list, p.free_count, i32([5, -3, 6]), i32([1, 2, -4]), 16, 3, status=flags)
    assert int(flags) == pps.FLAG_INDEX and got["q_off"].tolist() == [0, 1, 3, 3] and got["kv_len"].tolist() == [6, 2, 6]
    flags.zero_()
    p.held[1] = 77  # more than there are columns
    pps.kv_reserve(p.pages, p.held, p.free_list, p.free_count, i32([5, 20, 6]), i32([1, 2, 1]), 16, 4, status=flags)
    assert int(flags) == pps.FLAG_INDEX
    flags.zero_()
    p = Pool([5, 20, 6], 4, 16, 9, rng)
    p.pages[0, 0] = -1  # a held column without a page
    got = pps.kv_reserve(p.pages, p.held, p.free_list, p.free_count, i32([5, 20, 6]), i32([1, 1, 1]), 16, 3, status=flags)
    assert int(flags) == pps.FLAG_INDEX and got["slot"].tolist()[0] == -1
    p = Pool([5, 20, 6], 4, 16, 9, rng)
    p.trim([5, 90, 0], status=pps.FLAG_INDEX)  # more than is held: kept as it is
    p = Pool([5, 20, 6], 4, 16, 9, rng, lose=2)
    flags.zero_()
    pps.kv_trim(p.pages, p.held, p.free_list, p.free_count, i32([0, 0, 0]), 16, status=flags)  # four pages for a list with room for two
    assert int(flags) == pps.FLAG_INDEX and int(p.free_count) == p.cap


def test_outputs_given_in_place_lengths_streams_and_graphs():
    p = Pool([5, 30], 8, 16, 9, random.Random(9))
    lens, new = i32([5, 30]), i32([3, 4])
    out = dict(q_off=i32([0] * 3), kv_len=lens, slot=torch.zeros(9, dtype=torch.int64, device="cuda"), pos=i32([0] * 9))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pps.kv_reserve(p.pages, p.held, p.free_list, p.free_count, lens, new, 16, 9, out=out, stream=side)
    side.synchronize()
    assert got is out and lens.tolist() == [8, 34] and out["pos"].tolist() == [5, 6, 7, 30, 31, 32, 33, 0, 0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pps.kv_reserve(p.pages, p.held, p.free_list, p.free_count, lens, new, 16, 9, out=out)
    for want in ([11, 38], [14, 42], [17, 46]):  # the lengths move on by themselves
        graph.replay()
        assert lens.tolist() == want
    slots = out["slot"].tolist()[:7]
    rows = [p.pages[s].tolist() for s in range(2)]
    assert slots == [rows[0][x // 16] * 16 + x % 16 for x in (14, 15, 16)] + [rows[1][x // 16] * 16 + x % 16 for x in range(42, 46)]
    none = pps.kv_reserve(p.pages[:0], p.held, p.free_list, p.free_count, lens[:0], new[:0], 16, 3)
    assert none["q_off"].tolist() == [0] and none["slot"].tolist() == [-1] * 3
    pps.kv_trim(p.pages[:0], p.held, p.free_list, p.free_count, lens[:0], 16)


def test_refusals():
    p = Pool([5, 30], 8, 16, 9, random.Random(9))
    ok = dict(pages=p.pages, held=p.held, free_list=p.free_list, free_count=p.free_count, kv_len=i32([5, 30]), n_new=i32([3, 4]),
              page_size=16, n_tok=7)
    pps.kv_reserve(**ok)
    trim = {k: v for k, v in ok.items() if k not in ("kv_len", "n_new", "n_tok")}
    for bad in (dict(pages=p.pages.long()), dict(held=p.held.cpu()), dict(free_list=None), dict(free_count=[1]), dict(pages=None)):
        with pytest.raises(TypeError):
            pps.kv_reserve(**{**ok, **bad})
        with pytest.raises(TypeError):
            pps.kv_trim(**{**trim, **bad}, keep=i32([1, 2]))
    for bad in (dict(kv_len=None), dict(n_new=i32([1, 2]).float()), dict(pos_off=[1]), dict(status=3), dict(out=dict(q_off=i32([0, 0, 0])))):
        with pytest.raises(TypeError):
            pps.kv_reserve(**{**ok, **bad})
    for bad in (dict(held=p.held[:1]), dict(kv_len=i32([1])), dict(n_new=i32([1])), dict(pos_off=i32([1] * 6))):
        with pytest.raises(ValueError):
            pps.kv_reserve(**{**ok, **bad})
    with pytest.raises(ValueError):
        pps.kv_trim(**trim, keep=i32([1]))

    def code(fn, **kw):
        with pytest.raises(pps.PPSError) as e:
            fn(**kw)
        return e.value.code

    assert code(pps.kv_reserve, **{**ok, "page_size": 0}) == pps.ERR_INVALID_ARG
    assert code(pps.kv_trim, **{**trim, "page_size": 0}, keep=i32([1, 2])) == pps.ERR_INVALID_ARG
    n = 8193
    many = dict(pages=torch.zeros(n, 1, dtype=torch.int32, device="cuda"), held=i32([0] * n))
    assert code(pps.kv_reserve, **{**ok, **many, "kv_len": i32([0] * n), "n_new": i32([0] * n)}) == pps.ERR_UNSUPPORTED
    assert code(pps.kv_trim, **{**trim, **many}, keep=i32([0] * n)) == pps.ERR_UNSUPPORTED
