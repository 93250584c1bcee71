"""pps_paged_attention where the cut of the work into shares can go wrong: many sequences, few long ones among many short,
cuts within a few key tiles of an item's ends, items without keys."""
import random

import pytest
import torch

from test_gpu_attention import BF, F16, Case, _cuda  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_seq", [33, 152, 153, 383, 384, 385, 769, 1500])
def test_many_sequences(n_seq):
    rng = random.Random(n_seq)
    kv = [rng.choice([0, 1, 3, 16, 127, 129, 200, 500]) for _ in range(n_seq)]
    c = Case([min(1, x) if rng.random() < 0.9 else 0 for x in kv], kv, 4, 2, 64, 16, seed=n_seq)
    c.check()


@pytest.mark.parametrize("at", [0, 7, 399])
def test_one_long_sequence_among_many_short(at):
    kv = [40] * 400
    kv[at] = 60000
    Case([1] * 400, kv, 8, 2, 64, 32, F16, seed=at).check()


@pytest.mark.parametrize("seed", range(12))
def test_random_mixtures(seed):
    """Steps of every kind in one call; the shares' cuts fall anywhere."""
    rng = random.Random(100 + seed)
    log = lambda lo, hi: int(lo * (hi / lo) ** rng.random())
    n_seq = log(2, 60)
    heads, kv_heads, d = rng.choice([(8, 2, 128), (4, 4, 64), (7, 1, 64), (5, 1, 80), (12, 3, 128)])
    kv = [log(1, rng.choice([300, 3000, 9000])) for _ in range(n_seq)]
    q = [min(x, rng.choice([1, 1, 2, 5, 40, 150, 700])) for x in kv]
    tree = rng.random() < 0.4
    if tree:
        q = [min(x, 64) for x in q]
    Case(q, kv, heads, kv_heads, d, rng.choice([8, 16, 64, 256]), rng.choice([BF, F16]), tree=tree,
         layout=rng.choice(["token", "head"]), seed=seed).check()


@pytest.mark.parametrize("tiles", [1, 2, 3, 7, 12, 13, 25])
@pytest.mark.parametrize("n_seq", [151, 152, 153, 160])
def test_cuts_near_the_ends_of_items(tiles, n_seq):
    """Equal items, about one per share: every cut lies a little further into its item than the one before."""
    Case([1] * n_seq, [128 * tiles - 5] * n_seq, 1, 1, 64, 128, seed=tiles).check()
