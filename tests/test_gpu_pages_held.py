"""pps_kv_reserve where a sequence holds fewer pages than the tokens that it is said to have."""
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


@pytest.mark.parametrize("n_new", [0, 1, 3, 100])
@pytest.mark.parametrize("held,length", [(0, 1), (1, 17), (2, 40), (0, 40)])
def test_it_gets_nothing_and_the_others_what_they_need(held, length, n_new):
    page, columns = 16, 12
    pages = torch.full((3, columns), -1, dtype=torch.int32, device="cuda")
    pages[0, :1], pages[2, :2] = 20, i32([21, 22])
    if held:
        pages[1, :held] = i32(list(range(30, 30 + held)))
    before, holds = pages.clone(), i32([1, held, 2])
    free, count, status = i32(list(range(9))), i32([9]), i32([0])
    got = pps.kv_reserve(pages, holds, free, count, i32([16, length, 20]), i32([2, n_new, 13]), page, 15 + n_new, status=status)
    assert int(status) == pps.FLAG_INDEX
    assert got["kv_len"].tolist() == [18, 0, 33] and got["q_off"].tolist() == [0, 2, 2 + n_new, 15 + n_new]
    # the pool's top two pages go to the first and the last
    assert int(count) == 7 and holds.tolist() == [2, held, 3]
    before[0, 1], before[2, 2] = 8, 7
    assert torch.equal(pages, before)
    slot = got["slot"].tolist()
    assert slot[:2] == [8 * 16, 8 * 16 + 1] and slot[2:2 + n_new] == [-1] * n_new
    assert slot[2 + n_new:] == [22 * 16 + i for i in range(4, 16)] + [7 * 16]


def test_of_many_sequences_every_other_one():
    n, page = 700, 4
    held = [(s % 5) for s in range(n)]
    length = [h * page + (1 + s % 7 if s % 2 else -min(s % 3, h * page)) for s, h in enumerate(held)]
    n_new = [1 + s % 6 for s in range(n)]
    pages = torch.full((n, 9), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, h in enumerate(held):
        if h:
            pages[s, :h] = i32(list(range(at, at + h)))
        at += h
    status, count = i32([0]), i32([3000])
    holds = i32(held)
    got = pps.kv_reserve(pages, holds, i32(list(range(at, at + 3000))), count, i32(length), i32(n_new), page, sum(n_new), status=status)
    assert int(status) == pps.FLAG_INDEX
    served = [s % 2 == 0 for s in range(n)]
    assert got["kv_len"].tolist() == [m + k if y else 0 for m, k, y in zip(length, n_new, served)]
    want = [-(-(m + k) // page) if y else h for m, k, h, y in zip(length, n_new, held, served)]
    want = [max(w, h) for w, h in zip(want, held)]
    assert holds.tolist() == want and int(count) == 3000 - sum(want) + sum(held)
    slot, k = got["slot"].tolist(), 0
    rows = pages.tolist()
    for s in range(n):
        for i in range(n_new[s]):
            place = length[s] + i
            assert slot[k] == (rows[s][place // page] * page + place % page if served[s] else -1)
            k += 1
