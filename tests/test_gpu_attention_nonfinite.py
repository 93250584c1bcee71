"""pps_paged_attention with queries and keys that are not finite: NaN for the tokens whose scores they reach, nothing else."""
import pytest
import torch

from test_gpu_attention import BF, F16, U, Case, _cuda  # noqa: F401

pytestmark = pytest.mark.gpu


def check(c, scale=None):
    """Against the formula, NaN where it is."""
    want, size, _ = c.exact(scale)
    lse = torch.full(c.q.shape[:2], 7.0, dtype=torch.float32, device="cuda")
    got = c.call(lse=lse, **({} if scale is None else dict(scale=scale)))
    bad = torch.isnan(want).any(-1)
    assert bool(bad.any()) and bool((~bad).any())
    assert bool(torch.isnan(got[bad]).all()) and bool(torch.isnan(lse[bad]).all())
    # the tolerance of test_gpu_attention for the others
    err, tol = (got.double() - want).abs(), 1.01 * U[c.dt] * (want.abs() + size) + 1e-4 * size + 2.0 ** -24
    assert bool((err <= tol)[~bad].all())


def put_key(c, s, j, x):
    """Key j of sequence s, in the pages and in the list."""
    c.keys[s][j] = x
    c.k_cache[int(c.pages[s, j // c.page]), j % c.page] = c.keys[s][j]


def cases(tree):
    """One part, both streams, cut items, several row blocks."""
    yield Case([1, 1, 1], [70, 300, 5000], 8, 2, 128, 16, BF, tree=tree, seed=1)
    yield Case([41, 60, 3], [500, 700, 40], 8, 2, 64, 16, F16, tree=tree, seed=2)
    yield Case([64], [20000], 4, 4, 128, 64, BF, tree=tree, seed=3)
    if not tree:
        yield Case([600, 2], [900, 300], 8, 2, 128, 16, BF, seed=4)


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("x", [float("nan"), float("inf")])
def test_queries(tree, x):
    for c in cases(tree):
        c.q[c.q.shape[0] // 2, 1] = x  # inf: some keys' scores are +inf or inf - inf
        c.q[0, 3, 5] = float("nan")
        check(c)


@pytest.mark.parametrize("tree", [False, True])
def test_keys_before_the_new_tokens(tree):
    for c in cases(tree):
        n, length = c.q_len[0], c.kv_len[0]
        at = (length - n) // 2
        put_key(c, 0, at, torch.cat([c.keys[0][at][:1] * float("nan"), c.keys[0][at][1:]]))  # of one key head
        check(c)


@pytest.mark.parametrize("x", [float("nan"), float("inf"), float("-inf")])
def test_keys_that_are_not_seen(x):
    """A later token's key, or another branch's, does not matter."""
    c = Case([50, 300], [400, 900], 8, 2, 128, 16, BF, seed=5)
    good = c.call()
    for s in range(2):
        put_key(c, s, c.kv_len[s] - 1, x)
    got, last = c.call(), torch.tensor([49, 349], device="cuda")
    others = torch.ones(350, dtype=torch.bool, device="cuda")
    others[last] = False
    assert torch.equal(got[others], good[others])
    c = Case([40], [333], 8, 2, 64, 16, F16, tree=True, seed=6)
    c.mask[:] = c.mask & ~(1 << 7)  # no token sees node 7
    c.bits[:, 7] = False
    good = c.call()
    put_key(c, 0, 333 - 40 + 7, x)
    assert torch.equal(c.call(), good)


def test_a_scale_of_zero_and_tokens_that_see_nothing():
    c = Case([40], [40], 8, 2, 64, 16, F16, tree=True, seed=7)
    c.mask[5] = 0
    c.bits[5] = False
    c.check(scale=0.0)
    c.check()
