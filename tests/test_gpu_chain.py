"""pps_verify_chain against Alg. 1 in 64 bits: acceptance, residuals, chain shapes, odd rows, refusals."""
import math

import numpy as np
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


def _law(row, T):
    x = row.double().cpu().numpy() / T
    x = np.where(np.isnan(x), -np.inf, x)
    m = x.max()
    if m == -np.inf:
        return np.zeros_like(x)
    e = np.where(x == m, 1.0, np.exp(np.subtract(x, m, where=x != m, out=np.zeros_like(x))))
    return e / e.sum()


def _last(left, fallback, noise):
    """The emitted token, and whether another one's score is within 1e-5 of it."""
    w = left if (left > 0).any() else fallback
    if not (w > 0).any():
        return -1, False
    score = np.where(w > 0, w / noise, -1.0)
    i = int(score.argmax())
    second = np.delete(score, i).max() if score.size > 1 else -1.0
    return i, second > score[i] * (1 - 1e-5)


def _check(p, q, gamma, seq_off, draft_row, tok, u, noise, T=1.0, got=None, exempt=0):
    got = got or pps.verify_chain(p, q, gamma, seq_off, draft_row, tok, u, noise, temperature=T)
    off, rows, toks, us = seq_off.tolist(), draft_row.tolist(), tok.tolist(), u.double().tolist()
    V = p.shape[1]
    acc, ne, em = got["accept_len"].tolist(), got["n_emitted"].tolist(), got["emitted"].tolist()
    prob = got["accept_prob"].double().tolist()
    skipped = 0
    for s in range(len(off) - 1):
        said, near = [], False
        open_, n = True, min(off[s + 1] - off[s] - 1, gamma)
        for j in range(n + 1):
            c = off[s] + j
            r = rows[c] if j < n and 0 <= rows[c] < q.shape[0] else -1
            P = _law(p[c], T)
            if r >= 0:
                Q = _law(q[r], T)
                x = toks[r]
                px, qx = (P[x], Q[x]) if 0 <= x < V else (0.0, 0.0)
                want = 0.0 if px == 0 else 1.0 if qx == 0 else min(1.0, px / qx)
                # fp32 softmax: logits scaled by log2(e) / T (|x| / T up to 200 here, 2^-24 of it each way), sums to 1e-6
                assert abs(prob[r] - want) <= 5e-5 * want + 1e-38, (s, j)
            if not open_:
                continue
            if r >= 0:
                near = near or abs(us[r] * qx - px) < 1e-5 * px
                if us[r] * qx < px:
                    said.append(x)
                    continue
            left = np.maximum(P - Q, 0) if r >= 0 and Q.any() else P
            left = np.where(left > 1e-6 * P, left, 0.0)  # differences within the fp32 error of their terms
            i, tie = _last(left, P, noise[s, :V].double().cpu().numpy())
            near, open_ = near or tie, False
            said += [i] if i >= 0 else []
            length = j
        if near:
            skipped += 1
            continue
        assert acc[s] == length and ne[s] == len(said), (s, acc[s], length)
        assert em[s] == said + [-1] * (gamma + 1 - len(said)), s
    assert skipped <= exempt, f"{skipped} sequences decided by less than 1e-5"
    return got


def _chains(lengths, V, dt, seed, spread=0.7, permute=True, T=1.0):
    """Chains of the given lengths whose drafted tokens are samples of the drafter's law."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    off = [0]
    for n in lengths:
        off.append(off[-1] + n + 1)
    n_draft = sum(lengths)
    order = torch.randperm(n_draft, generator=g, device="cuda").tolist() if permute else list(range(n_draft))
    rows, nodes, at = [], [0] * n_draft, 0
    for s, n in enumerate(lengths):
        for j in range(n):
            rows.append(order[at])
            nodes[order[at]] = off[s] + j
            at += 1
        rows.append(-1)
    p = 2.0 * torch.randn(off[-1], V, generator=g, device="cuda")
    q = p[nodes] + spread * torch.randn(n_draft, V, generator=g, device="cuda")
    p, q = p.to(dt), q.to(dt)
    e = torch.rand(n_draft, V, generator=g, device="cuda").clamp(min=1e-12).log().neg()
    tok = (q.float() / T - e.log()).argmax(-1).to(torch.int32) if n_draft else torch.zeros(0, dtype=torch.int32, device="cuda")
    u = torch.rand(n_draft, generator=g, device="cuda")
    noise = torch.rand(len(lengths), V, generator=g, device="cuda").clamp(min=1e-9).log().neg().clamp(min=1e-9)
    i32 = dict(dtype=torch.int32, device="cuda")
    return p, q, max(lengths), torch.tensor(off, **i32), torch.tensor(rows, **i32), tok, u, noise


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 64, 1000, 4099, 16383, 32000])
def test_against_the_definition(V, dt):
    _check(*_chains([5, 0, 1, 3, 8, 2, 5, 5], V, dt, V), exempt=1)


@pytest.mark.parametrize("dt,V,T", [(BF, 128256, 1.0), (F32, 152063, 0.7), (BF, 65537, 1.6)])
def test_large_vocabularies(dt, V, T):
    _check(*_chains([5, 4, 0, 2], V, dt, V, T=T), T=T)


def test_many_sequences_of_every_outcome():
    args = _chains([6] * 400, 500, BF, 3, spread=1.0)
    got = _check(*args, exempt=2)
    lengths = np.bincount(got["accept_len"].cpu().numpy(), minlength=7)
    assert (lengths > 0).all(), lengths  # chains cut at each depth, and whole ones


def test_the_emitted_tokens_follow_the_target():
    # one node and its draft, 60000 times: the first emitted token is a sample of P whatever Q is (Alg. 1)
    n, V = 60000, 6
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    pr, qr = torch.tensor([0.5, 1.5, -1.0, 0.0, 2.0, -3.0]), torch.tensor([1.0, 0.0, 0.0, 1.0, 0.5, -9.0])
    p, q = (x.to("cuda").repeat(k * n, 1) for x, k in ((pr, 2), (qr, 1)))
    e = torch.rand(2 * n, V, generator=g, device="cuda").clamp(min=1e-9).log().neg()
    tok = (qr.cuda() - e[n:].log()).argmax(-1).to(torch.int32)
    i32 = dict(dtype=torch.int32, device="cuda")
    rows = torch.stack([torch.arange(n, **i32), torch.full((n,), -1, **i32)], 1).flatten().contiguous()
    got = pps.verify_chain(p, q, 1, torch.arange(n + 1, **i32) * 2, rows, tok, torch.rand(n, generator=g, device="cuda"),
                           e[:n].contiguous())
    count = np.bincount(got["emitted"][:, 0].cpu().numpy(), minlength=V)
    law = _law(pr, 1.0)
    chi2 = float(((count - n * law) ** 2 / (n * law)).sum())
    assert chi2 < 25.7, chi2  # 1e-4 of chi-square with 5 degrees of freedom
    alpha = float(np.minimum(law, _law(qr, 1.0)).sum())  # acceptance rate = 1 - TV(P, Q)
    rate = float((got["accept_len"] == 1).double().mean())
    assert abs(rate - alpha) < 4 * math.sqrt(alpha * (1 - alpha) / n)


@pytest.mark.parametrize("dt", [BF, F32])
def test_odd_logits(dt):
    V = 300
    p, q, gamma, off, rows, tok, u, noise = _chains([2] * 8, V, dt, 17, permute=False)
    nan, inf = float("nan"), float("inf")
    p[0, ::2] = -inf                  # half the target's tokens are impossible
    p[3, 1::3], q[2, 5] = nan, nan    # NaN counts as -inf
    p[6] = -inf                       # no usable logit: nothing is emitted
    p[9, 17], p[9, 40] = inf, inf     # the row's whole mass, shared
    q[8] = -inf                       # a drafter without mass: accepted where the target has some
    p[15:17] = -65504.0               # the lowest value of a masked type everywhere: a uniform law
    q[12] = q[12] * 0 + 3.0e38        # huge equal logits
    p[21] = q[14]                     # equal rows: accepted
    _check(p, q, gamma, off, rows, tok, u, noise, exempt=1)


def test_a_residual_that_is_zero_is_replaced_by_the_target():
    p, q, gamma, off, rows, tok, u, noise = _chains([1, 1], 1000, F32, 5, permute=False)
    q[:] = p[[0, 2]]
    tok[0] = 5000  # no token of the vocabulary: rejected, with nothing left of P - Q
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = pps.verify_chain(p, q, gamma, off, rows, tok, u, noise, status=status)
    assert int(status.item()) == pps.FLAG_INDEX
    _check(p, q, gamma, off, rows, tok, u, noise, got=got)
    assert got["accept_len"].tolist() == [0, 1] and got["emitted"][0, 0].item() >= 0


def test_chain_ends_and_rows_out_of_range():
    args = list(_chains([4, 4, 4, 4], 700, BF, 23, spread=0.05))
    args[4][6] = -1  # the second chain ends after its first token
    _check(*args)
    args[4][11] = 16  # a draft row past the last one ends the chain, and is flagged
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = pps.verify_chain(*args, status=status)
    assert int(status.item()) == pps.FLAG_INDEX
    _check(*args, got=got)
    args[2] = 2  # gamma below the chains' lengths: cut there
    _check(*args)
    args[2] = 9
    _check(*args)


def test_sequences_outside_the_rows_are_flagged():
    p, q, gamma, off, rows, tok, u, noise = _chains([2, 2, 2], 100, BF, 29, permute=False)
    for bad in ([0, 3, 3, 9], [0, 3, 6, 10], [-1, 3, 6, 9], [0, 6, 3, 9]):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = pps.verify_chain(p, q, gamma, torch.tensor(bad, dtype=torch.int32, device="cuda"), rows, tok, u, noise,
                               status=status)
        assert int(status.item()) == pps.FLAG_INDEX
        wrong = [s for s in range(3) if not 0 <= bad[s] < bad[s + 1] <= 9]
        assert all(got["n_emitted"][s].item() == 0 and (got["emitted"][s] == -1).all() for s in wrong)


def test_strided_rows_another_stream_and_a_used_workspace():
    p, q, gamma, off, rows, tok, u, noise = _chains([5, 3, 0], 4099, BF, 31)
    want = _check(p, q, gamma, off, rows, tok, u, noise)
    wide = [torch.full((x.shape[0], x.shape[1] + k), float("inf"), dtype=x.dtype, device="cuda")
            for x, k in ((p, 3), (q, 13), (noise, 5))]
    for w, x in zip(wide, (p, q, noise)):
        w[:, 1:x.shape[1] + 1] = x  # rows that start on odd offsets, between other values
    p2, q2, noise2 = (w[:, 1:4100] for w in wide)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = torch.full((pps.chain_workspace(11, 8, 3).numel(),), 255, dtype=torch.uint8, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    for kw in (dict(), dict(ws=ws), dict(ws=ws), dict(stream=side)):
        got = pps.verify_chain(p2, q2, gamma, off, rows, tok, u, noise2, **kw)
        torch.cuda.synchronize()
        for k in want:
            if k != "accept_prob":
                assert torch.equal(got[k], want[k]), k
        assert torch.allclose(got["accept_prob"], want["accept_prob"], rtol=1e-5, atol=0)


def test_no_drafts_at_all():
    p, _, _, off, rows, tok, u, noise = _chains([0, 0], 50, F32, 37)
    got = _check(p, p[:0], 0, off, rows, tok, u, noise)
    assert got["accept_len"].tolist() == [0, 0]


def test_refusals():
    p, q, gamma, off, rows, tok, u, noise = _chains([2, 1], 64, BF, 41)
    ok = [p, q, gamma, off, rows, tok, u, noise]

    def swapped(i, x):
        return [x if j == i else y for j, y in enumerate(ok)]

    for i, x in ((0, p.half()), (0, p[0]), (3, off.long()), (5, tok.long()), (6, u.double()), (7, noise.double())):
        with pytest.raises((TypeError, ValueError)):
            pps.verify_chain(*swapped(i, x))
    for i, x in ((1, q[:, :63]), (1, q.float()), (4, rows[:4]), (5, tok[:2]), (6, u[:2]), (7, noise[:1]), (7, noise[:, :63])):
        with pytest.raises(ValueError):
            pps.verify_chain(*swapped(i, x))

    def code(*args, **kw):
        with pytest.raises(pps.PPSError) as e:
            pps.verify_chain(*args, **kw)
        return e.value.code

    assert code(*ok, temperature=0.0) == pps.ERR_INVALID_ARG
    assert code(*swapped(2, 65)) == pps.ERR_INVALID_ARG
    assert code(*swapped(2, -1), out=dict(accept_len=rows, n_emitted=rows, emitted=rows)) == pps.ERR_INVALID_ARG
    assert code(*ok, ws=torch.empty(8, dtype=torch.uint8, device="cuda")) == pps.ERR_WORKSPACE
    with pytest.raises(TypeError):
        pps.verify_chain(*ok, out=dict(accept_len=rows))
