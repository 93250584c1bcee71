"""The target model's side of a decoding step, operator by operator, as cases to be timed and compared.

Between a draft block and its verification stand the target model's layers.  Three operators of that side:

* ``append``  queries and keys of new tokens are normed per head (optionally) and rotated to their positions; keys and
              values go to their slots of a paged cache;
* ``attend``  attention of the new tokens (one a sequence, the nodes of a draft tree, or a chunk of a prompt) over the
              paged cache;
* ``chain``   the token-level maximal coupling: a drafted chain is accepted or corrected from given random numbers.

``run`` computes a pass in plain torch, in 32 bits, or through the package where ``own`` is set; ``exact`` restates it
in 64 bits from the definitions.
"""
import math
import random

import torch

own = False

DEV = "cuda"
_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "fp32": 4}


def _append(name, n_tok, heads, kv_heads, d, page, dtype="bf16", norm=False, rot=None, interleaved=False,
            layout="token", max_pos=131072):
    case = {"kind": "append", "n_tok": n_tok, "heads": heads, "kv_heads": kv_heads, "d": d, "page": page,
            "dtype": dtype, "norm": norm, "rot": rot or d, "interleaved": interleaved, "layout": layout,
            "max_pos": max_pos}
    return dict(case, name=name) if name else case


def _attend(name, n_seq, q_max, kv_max, heads, kv_heads, d, page, dtype="bf16", K=0, gamma=0, layout="token"):
    """K > 0: the tokens are the 1 + K * gamma nodes of K draft chains of gamma tokens; else causal chunks of up to
    q_max tokens.  Sequences hold kv_max / 4 to kv_max keys, the new tokens' own among them."""
    case = {"kind": "attend", "n_seq": n_seq, "q_max": 1 + K * gamma if K else q_max, "kv_max": kv_max, "heads": heads,
            "kv_heads": kv_heads, "d": d, "page": page, "dtype": dtype, "K": K, "gamma": gamma, "layout": layout}
    return dict(case, name=name) if name else case


def _chain(name, n_seq, gamma, vocab, dtype="bf16", temperature=1.0, ragged=False):
    case = {"kind": "chain", "n_seq": n_seq, "gamma": gamma, "vocab": vocab, "dtype": dtype,
            "temperature": temperature, "ragged": ragged}
    return dict(case, name=name) if name else case


def listed():
    return [
        # plain decoding of eight sequences: one token each; a launch
        _append("append_tokens", 8, 32, 8, 128, 16),
        # the 64 x 41 draft-tree nodes of the benchmark's step, in the half precision of the paper's runs, heads normed
        _append("append_tree", 2624, 28, 4, 128, 16, dtype="f16", norm=True),
        # a prompt's chunk, 64 channels a head
        _append("append_chunk", 16384, 32, 8, 64, 64),
        # one interactive sequence, a short context: the smallest call
        _attend("token_short", 1, 1, 900, 32, 8, 128, 16),
        # 64 sequences decoding a token each over contexts of mixed lengths
        _attend("token_batch", 64, 1, 8000, 32, 8, 128, 16),
        # one sequence with a long document behind it
        _attend("token_long", 1, 1, 130001, 28, 4, 128, 32, dtype="f16"),
        # the target's pass over the benchmark's draft trees: 8 chains of 5 and the root, 64 sequences
        _attend("tree_batch", 64, 0, 4100, 32, 8, 128, 16, K=8, gamma=5),
        # ragged prompt chunks of a small draft model, pages laid out head by head
        _attend("chunk_ragged", 7, 777, 2900, 14, 2, 64, 64, dtype="f16", layout="head"),
        # a long prompt's second half
        _attend("chunk_long", 1, 8192, 16384, 32, 8, 128, 128),
        # one interactive sequence of a small vocabulary
        _chain("chain_one", 1, 5, 32000),
        # the benchmark's batch: 64 sequences, five drafted tokens each
        _chain("chain_batch", 64, 5, 128256),
        # fp32 logits over the largest vocabulary, chains of differing lengths, a vocabulary of odd size
        _chain("chain_fp32", 16, 8, 152063, dtype="fp32", temperature=0.7, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "chain"])
    heads, kv_heads, d = rng.choice([(32, 8, 128), (28, 4, 128), (32, 32, 128), (32, 8, 64), (14, 2, 64), (12, 12, 64),
                                     (16, 1, 128), (20, 4, 80)])
    page, layout = rng.choice([8, 16, 16, 32, 64, 128, 256]), rng.choice(["token", "token", "head"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if kind == "append":
        rot = rng.choice([d, d, d // 2])
        return _append("", _log_int(rng, 1, 16384), heads, kv_heads, d, page, dtype, rng.random() < 0.5, rot,
                       rng.random() < 0.3, layout, _log_int(rng, 20000, 131072))
    if kind == "attend":
        form = rng.choice(["token", "tree", "chunk"])
        while True:
            if form == "token":
                case = _attend("", _log_int(rng, 1, 128), 1, _log_int(rng, 30, 130000), heads, kv_heads, d, page, dtype,
                               layout=layout)
            elif form == "tree":
                case = _attend("", _log_int(rng, 1, 64), 0, _log_int(rng, 60, 30000), heads, kv_heads, d, page, dtype,
                               rng.randint(2, 10), rng.randint(1, 6), layout)
            else:
                q = _log_int(rng, 2, 8192)
                case = _attend("", _log_int(rng, 1, 16), q, q + rng.randint(0, 8192), heads, kv_heads, d, page, dtype,
                               layout=layout)
            rows = case["n_seq"] * case["kv_max"]
            if case["kv_max"] >= 4 * case["q_max"] or form == "chunk":
                if rows * case["kv_heads"] * case["d"] < 1.2e9 and rows * case["q_max"] * case["heads"] <= 4.3e9:
                    return case
    case = _chain("", _log_int(rng, 1, 96), rng.randint(1, 10), _log_int(rng, 1000, 152064),
                  rng.choice(["bf16", "bf16", "fp32"]), rng.choice([0.6, 1.0, 1.0, 1.4]), rng.random() < 0.5)
    while case["n_seq"] > 1 and work(case)["bytes"] > 1.0e9:
        case["n_seq"] = case["n_seq"] * 2 // 3
    return case


# ---------------------------------------------------------------- inputs

class _State:
    pass


def _gen(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _pool(gen, n_pages, case):
    """A cache half [pages, slots, heads, channels]; "head": each page laid out head by head in memory."""
    shape = [n_pages, case["page"], case["kv_heads"], case["d"]]
    if case["layout"] == "head":
        shape[1], shape[2] = shape[2], shape[1]
    x = torch.randn(shape, generator=gen, device=DEV, dtype=_DTYPES[case["dtype"]])
    return x.transpose(1, 2) if case["layout"] == "head" else x


def _prepare_append(case, seed):
    s, gen, dt = _State(), _gen(seed), _DTYPES[case["dtype"]]
    n, hq, hk, d, rot = case["n_tok"], case["heads"], case["kv_heads"], case["d"], case["rot"]
    # one projection's output, of which queries, keys and values are views
    qkv = torch.randn(n, (hq + 2 * hk) * d, generator=gen, device=DEV, dtype=torch.float32).mul_(1.5).to(dt)
    s.q, s.k, s.v = (x.view(n, -1, d) for x in qkv.split([hq * d, hk * d, hk * d], dim=1))
    s.pos = torch.randint(0, case["max_pos"], (n,), generator=gen, device=DEV, dtype=torch.int32)
    n_pages = -(-n // case["page"]) + 3
    s.k_cache, s.v_cache = _pool(gen, n_pages, case), _pool(gen, n_pages, case)
    s.slot = torch.randperm(n_pages * case["page"], generator=gen, device=DEV)[:n].contiguous()
    s.q_norm = s.k_norm = None
    if case["norm"]:
        s.q_norm, s.k_norm = ((1 + 0.2 * torch.randn(d, generator=gen, device=DEV)).to(dt) for _ in range(2))
    # cosines and sines of every position, rounded to 32 bits
    t = (torch.arange(case["max_pos"], device=DEV, dtype=torch.float64)[:, None]
         * 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot))
    s.rope = torch.cat([t.cos(), t.sin()], dim=1).float()
    s.out = torch.empty(n, hq, d, device=DEV, dtype=dt)
    return s


def _prepare_attend(case, seed):
    # lengths belong to the case; what fills them comes from the seed
    s, gen, rng, dt = _State(), _gen(seed), random.Random(case["kv_max"]), _DTYPES[case["dtype"]]
    n_seq, page, d = case["n_seq"], case["page"], case["d"]
    if case["K"] or case["q_max"] == 1:
        q_len = [case["q_max"]] * n_seq
    else:
        q_len = [case["q_max"]] + [rng.randint(1, case["q_max"]) for _ in range(n_seq - 1)]
    kv_len = [max(n, case["kv_max"] if i == 0 else rng.randint(case["kv_max"] // 4, case["kv_max"]))
              for i, n in enumerate(q_len)]
    s.max_q, s.max_kv, s.n_tok = max(q_len), max(kv_len), sum(q_len)
    held = [-(-n // page) for n in kv_len]
    n_pages = sum(held) + 5
    s.k_cache, s.v_cache = _pool(gen, n_pages, case), _pool(gen, n_pages, case)
    perm = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    width = max(held) + 1
    at = torch.arange(width, device=DEV)[None, :]
    first = _i32([sum(held[:i]) for i in range(n_seq)])[:, None]
    s.pages = torch.where(at < _i32(held)[:, None], perm[(first + at).clamp(max=n_pages - 1)], -1).contiguous()
    s.kv_len, s.q_off = _i32(kv_len), _i32([sum(q_len[:i]) for i in range(n_seq + 1)])
    s.q = torch.randn(s.n_tok, case["heads"], d, generator=gen, device=DEV, dtype=torch.float32).mul_(2).to(dt)
    s.mask = None
    if case["K"]:  # node 1 + k * gamma + j is the j-th of chain k: it sees the root, its own chain up to itself
        node = torch.arange(1, case["q_max"])
        chain, depth = (node - 1) // case["gamma"], (node - 1) % case["gamma"]
        sees = torch.zeros(case["q_max"], -(-case["q_max"] // 32) * 32, dtype=torch.int64)
        sees[:, 0] = 1
        sees[1:, 1:case["q_max"]] = (chain[:, None] == chain[None, :]) & (depth[:, None] >= depth[None, :])
        words = (sees.view(case["q_max"], -1, 32) << torch.arange(32)).sum(-1)
        words = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)
        s.mask = words.to(DEV).repeat(n_seq, 1).contiguous()
    s.out = torch.empty(s.n_tok, case["heads"], d, device=DEV, dtype=dt)
    return s


def _prepare_chain(case, seed):
    s, gen, rng, dt = _State(), _gen(seed), random.Random(case["vocab"]), _DTYPES[case["dtype"]]
    n_seq, gamma, V = case["n_seq"], case["gamma"], case["vocab"]
    length = [rng.randint(0, gamma) if case["ragged"] and i else gamma for i in range(n_seq)]
    n_draft = sum(length)
    off = [sum(length[:i]) + i for i in range(n_seq + 1)]
    # draft rows depth by depth, as the drafter made them
    at = sorted((j, i) for i in range(n_seq) for j in range(length[i]))
    row = {p: r for r, p in enumerate(at)}
    s.node_draft_row = _i32([row.get((j, i), -1) for i in range(n_seq) for j in range(length[i] + 1)])
    s.seq_off = _i32(off)
    # target logits: those of a 1 / rank law and noise; the drafter's: the target's and noise of its own
    base = -torch.log(torch.arange(1, V + 1, device=DEV, dtype=torch.float32))
    p = base[torch.randperm(V, generator=gen, device=DEV)] + 1.5 * torch.randn(off[-1], V, generator=gen, device=DEV)
    s.p = p.to(dt)
    node = torch.tensor([off[i] + j for j, i in at], device=DEV, dtype=torch.int64)
    q = p[node] + 0.7 * torch.randn(n_draft, V, generator=gen, device=DEV)
    s.q = q.to(dt)
    # the drafted tokens are samples of the drafter's law
    race = torch.rand(n_draft, V, generator=gen, device=DEV).clamp_(min=1e-12).log_().neg_().log_()
    s.tok = (s.q.float() / case["temperature"] - race).argmax(-1).to(torch.int32)
    s.u = torch.rand(n_draft, generator=gen, device=DEV)
    s.noise = torch.rand(n_seq, V, generator=gen, device=DEV).clamp_(min=1e-9).log_().neg_().clamp_(min=1e-9)
    return s


_PREPARE = {"append": _prepare_append, "attend": _prepare_attend, "chain": _prepare_chain}


def prepare(case, seed):
    s = _PREPARE[case["kind"]](case, seed)
    s.case = case
    return s


# ---------------------------------------------------------------- one pass, plain

def _norm_rotate(x, weight, s, case):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight.float()
    rot = case["rot"]
    table = s.rope[s.pos.long()][:, None, :]
    cos, sin = table[..., :rot // 2], table[..., rot // 2:]
    if case["interleaved"]:
        a, b = x[..., :rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _plain_append(s, case):
    page, at = s.slot // case["page"], s.slot % case["page"]
    dt = s.q.dtype
    s.out.copy_(_norm_rotate(s.q, s.q_norm, s, case).to(dt))
    s.k_cache[page, at] = _norm_rotate(s.k, s.k_norm, s, case).to(dt)
    s.v_cache[page, at] = s.v
    return {"q": s.out, "k_cache": s.k_cache, "v_cache": s.v_cache}


def _plain_attend(s, case):
    n_seq, m, L, hq, hk, d = case["n_seq"], s.max_q, s.max_kv, case["heads"], case["kv_heads"], case["d"]
    j = torch.arange(L, device=DEV)
    page, at = s.pages.long().clamp(min=0)[:, j // case["page"]], j % case["page"]
    k, v = s.k_cache[page, at].float(), s.v_cache[page, at].float()  # [n_seq, L, hk, d]
    q_len, i = s.q_off[1:] - s.q_off[:-1], torch.arange(m, device=DEV)
    token = (s.q_off[:-1, None] + i).clamp(max=s.n_tok - 1).long()
    q = s.q[token].float().view(n_seq, m, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(n_seq, hk, -1, d)
    score = (q @ k.permute(0, 2, 3, 1)).mul_(d ** -0.5).view(n_seq, hk, hq // hk, m, L)
    rel = (j - (s.kv_len - q_len)[:, None])[:, None, :]  # the key's place among the new tokens; < 0: before them
    if s.mask is None:
        sees = rel <= i[:, None]
    else:
        word = (rel.clamp(0, 32 * s.mask.shape[1] - 1) // 32).expand(-1, m, -1)
        sees = (rel < 0) | ((rel < q_len[:, None, None]) & ((s.mask[token].gather(2, word) >> (rel % 32)) & 1 > 0))
    score.masked_fill_(~sees[:, None, None], -math.inf)
    score.sub_(score.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = score.sum(-1, keepdim=True)
    o = (score.view(n_seq, hk, -1, L) @ v.permute(0, 2, 1, 3)).view(n_seq, hk, hq // hk, m, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(n_seq, m, hq, d)
    seq = torch.repeat_interleave(torch.arange(n_seq, device=DEV), q_len, output_size=s.n_tok)
    s.out.copy_(o[seq, torch.arange(s.n_tok, device=DEV) - s.q_off[seq]])
    return s.out


def _softmax_rows(x, temperature):
    x = x.float() / temperature
    e = (x - x.amax(-1, keepdim=True)).exp_()
    return e.div_(e.sum(-1, keepdim=True))


def _plain_chain(s, case):
    n_seq, gamma, n_draft = case["n_seq"], case["gamma"], s.tok.numel()
    p, q = _softmax_rows(s.p, case["temperature"]), _softmax_rows(s.q, case["temperature"])
    depth, length = torch.arange(gamma, device=DEV), s.seq_off[1:] - s.seq_off[:-1] - 1
    has = depth < length[:, None]
    node = torch.where(has, s.seq_off[:-1, None] + depth, 0).long()
    row = torch.where(has, s.node_draft_row[node], 0).long()
    tok = s.tok[row].long()
    px, qx = p[node, tok], q[row, tok]
    accepted = (has & (s.u[row] * qx < px)).int().cumprod(1)
    n = accepted.sum(1).int()
    prob = torch.zeros(n_draft + 1, device=DEV).index_put_((torch.where(has, row, n_draft),), (px / qx).clamp(max=1))
    # the last token: of the residual after a rejection, of the target's own law past the chain's end
    last = (s.seq_off[:-1] + n).long()
    cut = n < length
    left = p[last] - torch.where(cut[:, None], q[torch.where(cut, s.node_draft_row[last], 0).long()], 0.0)
    left = torch.where((left > 0).any(1, keepdim=True), left, p[last]).clamp_(min=0)
    final = (left / s.noise).argmax(1).int()
    at = torch.arange(gamma + 1, device=DEV)
    drafted = torch.cat([tok.int(), torch.zeros(n_seq, 1, dtype=torch.int32, device=DEV)], dim=1)
    emitted = torch.where(at < n[:, None], drafted, torch.where(at == n[:, None], final[:, None], -1))
    return {"accept_len": n, "n_emitted": n + 1, "emitted": emitted, "accept_prob": prob[:n_draft]}


_PLAIN = {"append": _plain_append, "attend": _plain_attend, "chain": _plain_chain}


# ---------------------------------------------------------------- one pass, by the package

def _own_append(s, case):
    from paper_2609_21858_gb300 import pps
    q = pps.kv_append(s.q, s.k, s.v, s.pos, s.slot, s.k_cache, s.v_cache, s.rope, q_norm=s.q_norm, k_norm=s.k_norm,
                      eps=1e-6, interleaved=case["interleaved"], out=s.out)
    return {"q": q, "k_cache": s.k_cache, "v_cache": s.v_cache}


def _own_attend(s, case):
    from paper_2609_21858_gb300 import pps
    return pps.paged_attention(s.q, s.k_cache, s.v_cache, s.pages, s.kv_len, s.q_off, mask=s.mask, out=s.out)


def _own_chain(s, case):
    from paper_2609_21858_gb300 import pps
    return pps.verify_chain(s.p, s.q, case["gamma"], s.seq_off, s.node_draft_row, s.tok, s.u, s.noise,
                            temperature=case["temperature"])


_OWN = {"append": _own_append, "attend": _own_attend, "chain": _own_chain}


def run(state):
    return (_OWN if own else _PLAIN)[state.case["kind"]](state, state.case)


# ---------------------------------------------------------------- what a pass cannot do without

def _lengths(case):
    """The mean lengths of a case's sequences, for its work: (new tokens, keys)."""
    if case["K"] or case["q_max"] == 1 or case["n_seq"] == 1:
        q = case["q_max"]
    else:
        q = (case["q_max"] + (case["n_seq"] - 1) * (1 + case["q_max"]) / 2) / case["n_seq"]
    kv = (case["kv_max"] + (case["n_seq"] - 1) * 0.625 * case["kv_max"]) / case["n_seq"]
    return q, max(q, kv)


def work(case):
    if case["kind"] == "append":
        n, hq, hk, d, e = case["n_tok"], case["heads"], case["kv_heads"], case["d"], _BYTES[case["dtype"]]
        return {"bytes": n * (2 * (hq + 2 * hk) * d * e + 4 * case["rot"] + 12), "flops": n * (hq + hk) * d * 10}
    if case["kind"] == "attend":
        (q, kv), n_seq, hq, hk, d = _lengths(case), case["n_seq"], case["heads"], case["kv_heads"], case["d"]
        pairs = kv - q + (1 + case["gamma"] / 2 if case["K"] else (q + 1) / 2)  # visible keys of a token, on average
        return {"bytes": n_seq * 2 * d * _BYTES[case["dtype"]] * (q * hq + kv * hk),
                "flops": 4 * d * hq * n_seq * q * pairs}
    drafts = case["n_seq"] * case["gamma"]
    if case["ragged"]:
        drafts = case["gamma"] + (case["n_seq"] - 1) * case["gamma"] / 2
    rows = 2 * drafts + case["n_seq"]
    return {"bytes": case["vocab"] * (rows * _BYTES[case["dtype"]] + 4 * case["n_seq"]) + 12 * rows,
            "flops": 5 * rows * case["vocab"]}


# ---------------------------------------------------------------- the same in 64 bits, from the definitions

def _exact_append(s, case):
    def heads(x, weight):
        x = x.double().clone()
        if weight is not None:
            x = weight.double() * x / ((x ** 2).sum(-1, keepdim=True) / case["d"] + 1e-6) ** 0.5
        half = case["rot"] // 2
        c = torch.arange(half, device=DEV)
        first, second = (2 * c, 2 * c + 1) if case["interleaved"] else (c, c + half)
        # the pair as a complex number, turned by the table's
        turn = torch.complex(s.rope[s.pos.long(), :half].double(), s.rope[s.pos.long(), half:].double())[:, None]
        z = torch.complex(x[..., first], x[..., second]) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    k_cache, v_cache = s.k_cache.double(), s.v_cache.double()
    k_cache[s.slot // case["page"], s.slot % case["page"]] = heads(s.k, s.k_norm)
    v_cache[s.slot // case["page"], s.slot % case["page"]] = s.v.double()
    return {"q": heads(s.q, s.q_norm), "k_cache": k_cache, "v_cache": v_cache}


def _exact_attend(s, case):
    out = torch.zeros(s.out.shape, dtype=torch.float64, device=DEV)
    group, off, lens = case["heads"] // case["kv_heads"], s.q_off.tolist(), s.kv_len.tolist()
    for i, n_kv in enumerate(lens):
        a, b = off[i], off[i + 1]
        n = b - a
        sees = torch.ones(n, n_kv, dtype=torch.bool, device=DEV)
        if s.mask is None:
            sees = sees.tril(n_kv - n)
        else:
            bits = (s.mask[a:b, :, None].long() >> torch.arange(32, device=DEV)) & 1
            sees[:, n_kv - n:] = bits.flatten(1)[:, :n] > 0
        held = s.pages[i, :-(-n_kv // case["page"])].long()
        for h in range(case["kv_heads"]):
            k, v = (x[held, :, h].flatten(0, 1)[:n_kv].double() for x in (s.k_cache, s.v_cache))
            for g in range(h * group, (h + 1) * group):
                w = (s.q[a:b, g].double() @ k.T) / math.sqrt(case["d"])
                w = torch.softmax(w.masked_fill_(~sees, -math.inf), dim=-1)
                out[a:b, g] = w @ v
    return out


def _exact_chain(s, case):
    gamma, T = case["gamma"], case["temperature"]
    off, draft_row, toks, us = s.seq_off.tolist(), s.node_draft_row.tolist(), s.tok.tolist(), s.u.tolist()
    prob, n, emitted = [0.0] * len(toks), [], []
    for i in range(case["n_seq"]):
        said, over = [], False
        for c in range(off[i], off[i + 1]):
            law = torch.softmax(s.p[c].double() / T, dim=0)
            r = draft_row[c]
            if r >= 0:
                drafter = torch.softmax(s.q[r].double() / T, dim=0)
                ratio = float(law[toks[r]] / drafter[toks[r]])
                prob[r] = min(1.0, ratio)
            if over:
                continue
            if r >= 0 and us[r] < ratio:
                said.append(toks[r])
                continue
            left = law if r < 0 else (law - drafter).clamp(min=0)
            said.append(int((left / s.noise[i].double()).argmax()))
            over = True
        n.append(len(said) - 1)
        emitted.append(said + [-1] * (gamma + 1 - len(said)))
    return {"accept_len": _i32(n), "n_emitted": _i32(n) + 1, "emitted": _i32(emitted),
            "accept_prob": torch.tensor(prob, dtype=torch.float64, device=DEV)}


_EXACT = {"append": _exact_append, "attend": _exact_attend, "chain": _exact_chain}


def exact(case, seed):
    return _EXACT[case["kind"]](prepare(case, seed), case)
