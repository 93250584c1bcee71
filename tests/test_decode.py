"""The decoding loop's own bookkeeping (no GPU): ancestor masks, cache slots, where accepted nodes go."""
import numpy as np
import pytest
import torch

from paper_2609_21858_gb300.decode import Cache, Decoder, Session


def session(branching, n_seq=3, capacity=96):
    model = Decoder(50, 16, 1, 2, 1, 8, max_pos=128, device="cpu")
    return Session(model, branching, n_seq, capacity)


def parents(t):
    p = [-1] * t.nodes_per_seq
    for row in range(t.draft_per_seq):
        for c in t.child_node[row]:
            if c >= 0:
                p[c] = int(t.draft_node[row])
    return p


@pytest.mark.parametrize("branching", [(1, 1, 1), (2, 3), (4, 1, 1), (3, 3, 3, 1)])
def test_mask_is_ancestors(branching):
    s = session(branching)
    up, n = parents(s.tree), s.nodes
    want = np.zeros((n, n), bool)
    for b in range(n):
        c = b
        while c >= 0:
            want[b, c] = True
            c = up[c]
    words = s.mask.numpy().view(np.uint32)
    assert words.shape == (3 * n, -(-n // 32))
    got = (words[:, np.arange(n) // 32] >> (np.arange(n) % 32).astype(np.uint32)) & 1
    assert np.array_equal(got.astype(bool), np.tile(want, (3, 1)))


def test_levels_cover_the_tree():
    s = session((3, 2, 1))
    depth = s.depth.view(3, -1)[0].tolist()
    for d, (lo, hi) in enumerate(s.levels):
        assert depth[lo:hi] == [d] * (hi - lo) and depth.count(d) == hi - lo
        assert s.row_k.view(3, -1)[0, lo:hi].tolist() == [s.tree.branching[d]] * (hi - lo)


def test_slots_are_distinct():
    c = Cache(4, 50, 1, 1, 8, page_size=8, device="cpu")
    assert c.capacity == 56 and sorted(c.pages.view(-1).tolist()) == list(range(28))
    seq = torch.arange(4).repeat_interleave(56)
    pos = torch.arange(56).repeat(4)
    assert sorted(c.slots(seq, pos).tolist()) == list(range(4 * 56))


@pytest.mark.parametrize("branching", [(2, 3), (4, 1, 1), (3, 2, 2)])
def test_kept_slots_follow_the_walk(branching):
    """Random walks: the nodes of the path of accepted tokens go behind the prefix, in order; the rest nowhere."""
    rng = np.random.default_rng(1)
    s = session(branching, n_seq=40, capacity=96)
    t = s.tree
    s.length = torch.tensor(rng.integers(0, 60, 40))
    lists = np.full((t.n_draft, t.K), -1, np.int32)
    for r in range(t.n_draft):
        lists[r, :t.row_k[r]] = rng.permutation(50)[:t.row_k[r]]
    accept, emitted = np.zeros(40, np.int32), np.full((40, t.gamma + 1), -1, np.int32)
    want = np.full(t.n_nodes, -1, np.int64)
    for q in range(40):
        node = int(t.seq_off[q])
        accept[q] = rng.integers(0, t.gamma + 1)
        for d in range(accept[q]):
            row = t.node_draft_row[node]
            k = rng.integers(0, t.row_k[row])
            emitted[q, d] = lists[row, k]
            node = int(t.child_node[row, k])
            want[node] = int(s.cache.slots(torch.tensor([q]), s.length[q:q + 1] + 1 + d))
        emitted[q, accept[q]] = 49 if accept[q] == t.gamma else next(
            x for x in range(50) if x not in lists[t.node_draft_row[node]])
    v = dict(emitted=torch.tensor(emitted), accept_len=torch.tensor(accept))
    assert np.array_equal(s._kept_slots(torch.tensor(lists), v).numpy(), want)


def test_refusals():
    s = session((2, 1), n_seq=2, capacity=20)
    with pytest.raises(ValueError):
        s.prefill([[1]])
    with pytest.raises(ValueError):
        s.prefill([[1], []])
    with pytest.raises(ValueError):
        s.prefill([[1], [0] * 40])
    with pytest.raises(ValueError):
        s.step(coupling=True)
    s.most = s.cache.capacity
    with pytest.raises(ValueError):
        s.step()
