"""What a server needs beside the target side's calls, operator by operator, as cases to be timed and compared.

* ``append4``  queries and keys of new tokens are normed (optionally) and rotated, keys and values are written to a paged
               cache held in 4 bits, and the cache is read back as the values it stands for;
* ``attend4``  attention of the new tokens (one a sequence, the nodes of a draft tree, or a chunk of a prompt) over a
               cache held in 4 bits;
* ``pages``    page tables, slots and positions of a step's tokens from the requests' lengths, pages taken from a pool
               and, after the step, given back;
* ``adjust``   penalties for repeated tokens (those on a draft tree's path among them), biases and grammar masks on logits.

The cache in 4 bits: blocks of 16 channels of a head are held as e2m1 codes (two a byte, the even channel low) and an e4m3
scale, beside a unit per head: value = unit * scale * code.

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
_CODES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _append(name, n_tok, heads, kv_heads, d, page, dtype="bf16", norm=False, rot=None, interleaved=False, layout="head",
            unit=False, max_pos=131072):
    case = {"kind": "append4", "n_tok": n_tok, "heads": heads, "kv_heads": kv_heads, "d": d, "page": page, "dtype": dtype,
            "norm": norm, "rot": rot or d, "interleaved": interleaved, "layout": layout, "unit": unit, "max_pos": max_pos}
    return dict(case, name=name) if name else case


def _attend(name, n_seq, q_max, kv_max, heads, kv_heads, d, page, dtype="bf16", K=0, gamma=0, layout="head", unit=False):
    """K > 0: the tokens are the 1 + K * gamma nodes of K draft chains of gamma tokens; else causal chunks of up to
    q_max tokens.  Sequences hold kv_max / 4 to kv_max keys, the new tokens' own among them."""
    case = {"kind": "attend4", "n_seq": n_seq, "q_max": 1 + K * gamma if K else q_max, "kv_max": kv_max, "heads": heads,
            "kv_heads": kv_heads, "d": d, "page": page, "dtype": dtype, "K": K, "gamma": gamma, "layout": layout,
            "unit": unit}
    return dict(case, name=name) if name else case


def _pages(name, n_seq, q_max, kv_max, page, ragged=False, tree=0, short=False):
    """tree > 0: every sequence brings the nodes of chains of `tree` tokens, whose positions repeat; short: the pool
    does not hold what the last sequences want."""
    case = {"kind": "pages", "n_seq": n_seq, "q_max": q_max, "kv_max": kv_max, "page": page, "ragged": ragged,
            "tree": tree, "short": short}
    return dict(case, name=name) if name else case


def _adjust(name, n_seq, K, gamma, vocab, text_max, dtype="bf16", penalties=True, bias=0, grammar=False):
    """K draft chains of gamma tokens and their root a sequence (K = 1: a chain; gamma = 0: a row)."""
    case = {"kind": "adjust", "n_seq": n_seq, "K": K, "gamma": gamma, "vocab": vocab, "text_max": text_max,
            "dtype": dtype, "penalties": penalties, "bias": bias, "grammar": grammar}
    return dict(case, name=name) if name else case


def listed():
    return [
        # plain decoding of eight sequences, heads normed
        _append("append4_tokens", 8, 32, 8, 128, 16, norm=True),
        # a prompt's chunk, in the half precision of the paper's runs
        _append("append4_chunk", 16384, 28, 4, 128, 16, dtype="f16", unit=True),
        # one interactive sequence, a short context
        _attend("token4_short", 1, 1, 900, 32, 8, 128, 16),
        # 64 sequences decoding a token each over contexts of mixed lengths
        _attend("token4_batch", 64, 1, 8000, 32, 8, 128, 16),
        # one sequence with a long document behind it, pages laid out token by token
        _attend("token4_long", 1, 1, 130001, 28, 4, 128, 32, dtype="f16", layout="token", unit=True),
        # the target's pass over the benchmark's draft trees: 8 chains of 5 and the root, 64 sequences
        _attend("tree4_batch", 64, 0, 4100, 32, 8, 128, 16, K=8, gamma=5),
        # ragged prompt chunks of a small draft model
        _attend("chunk4_ragged", 7, 777, 2900, 14, 2, 64, 64, dtype="f16"),
        # eight interactive sequences, a token each: the smallest call
        _pages("pages_tokens", 8, 1, 4000, 16),
        # a large server's step: 512 draft trees of 41 nodes
        _pages("pages_trees", 512, 41, 16000, 16, tree=5),
        # one interactive sequence of a small vocabulary
        _adjust("adjust_one", 1, 1, 0, 32000, 600),
        # the benchmark's trees, 64 x 41 rows, over conversations of up to 3000 tokens
        _adjust("adjust_trees", 64, 8, 5, 128256, 3000),
        # constrained decoding along chains: fp32 logits, the largest vocabulary, of odd size, biases and grammar masks
        _adjust("adjust_grammar", 16, 1, 8, 152063, 9000, dtype="fp32", bias=200, grammar=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append4", "attend4", "attend4", "attend4", "pages", "adjust"])
    heads, kv_heads, d = rng.choice([(32, 8, 128), (28, 4, 128), (32, 32, 128), (32, 8, 64), (14, 2, 64), (12, 12, 64),
                                     (16, 1, 128), (20, 4, 80)])
    page, layout = rng.choice([8, 16, 16, 32, 64, 128, 256]), rng.choice(["head", "head", "token"])
    dtype, unit = rng.choice(["bf16", "bf16", "f16"]), rng.random() < 0.5
    if kind == "append4":
        n = _log_int(rng, 1, 16384)
        # (a norm's last bit decides between two codes where a channel lies next to the border of both)
        return _append("", n, heads, kv_heads, d, page, dtype, n * kv_heads * d < 40000 and rng.random() < 0.7,
                       rng.choice([d, d, d // 2]), rng.random() < 0.3, layout, unit, _log_int(rng, 20000, 131072))
    if kind == "attend4":
        form = rng.choice(["token", "token", "tree", "chunk"])
        while True:
            if form == "token":
                case = _attend("", _log_int(rng, 1, 128), 1, _log_int(rng, 30, 130000), heads, kv_heads, d, page, dtype,
                               layout=layout, unit=unit)
            elif form == "tree":
                case = _attend("", _log_int(rng, 1, 64), 0, _log_int(rng, 60, 30000), heads, kv_heads, d, page, dtype,
                               rng.randint(2, 10), rng.randint(1, 6), layout, unit)
            else:
                q = _log_int(rng, 2, 2048)
                case = _attend("", _log_int(rng, 1, 16), q, q + rng.randint(0, 8192), heads, kv_heads, d, page, dtype,
                               layout=layout, unit=unit)
            rows = case["n_seq"] * case["kv_max"]
            if case["kv_max"] >= 4 * case["q_max"] or form == "chunk":
                if rows * case["kv_heads"] * case["d"] < 0.55e9 and rows * case["q_max"] * case["heads"] <= 3.4e8:
                    return case
    if kind == "pages":
        q = _log_int(rng, 1, 512)
        return _pages("", _log_int(rng, 1, min(2000, 21000 // q)), q, _log_int(rng, 1, 16000), page, rng.random() < 0.5,
                      rng.choice([0, 0, 4]), rng.random() < 0.2)
    while True:
        case = _adjust("", _log_int(rng, 1, 96), *rng.choice([(1, 0), (1, rng.randint(1, 10)), (rng.randint(2, 8), rng.randint(1, 6))]),
                       _log_int(rng, 1000, 152064), _log_int(rng, 1, 20000), rng.choice(["bf16", "bf16", "fp32"]),
                       rng.random() < 0.8, rng.choice([0, 0, 50, 300]), rng.random() < 0.4)
        if work(case)["bytes"] <= 1.3e9:
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


def _scale_bytes(d):
    """Bytes that the scales of a head's d channels take: one for 16 channels, filled up to four."""
    return 4 * -(-d // 64)


def _quantise(x, unit):
    """[..., heads, d] in fp32 -> codes [..., heads, d / 2] and scales [..., heads, bytes], both uint8."""
    z = (x * (1.0 / unit)[:, None]).unflatten(-1, (-1, 16))
    top = z.abs().amax(-1)
    scale = (top / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
    s = scale.float()[..., None]
    m = torch.where(s > 0, z.abs() / s, 0.0)
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0))
    code = (code + 8 * (z < 0)).flatten(-2)
    packed = code[..., 0::2] + 16 * code[..., 1::2]
    scale = scale.view(torch.uint8)
    return packed.to(torch.uint8), torch.nn.functional.pad(scale, (0, _scale_bytes(x.shape[-1]) - scale.shape[-1]))


def _value(codes, scales, unit):
    """The values in fp32 that codes [..., heads, d / 2] and scales stand for."""
    table = torch.tensor(_CODES + tuple(-c for c in _CODES), device=DEV)
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).int()
    s = scales[..., :c.shape[-1] // 16].contiguous().view(torch.float8_e4m3fn).float() * unit[:, None]
    return (table[c].unflatten(-1, (-1, 16)) * s[..., None]).flatten(-2)


def _units(gen, case):
    if not case["unit"]:
        return torch.ones(case["kv_heads"], device=DEV)
    return 0.25 + torch.rand(case["kv_heads"], generator=gen, device=DEV)


def _paged(x, case):
    """[pages, slots, heads, ...] as it is, or ("head") laid out head by head in each page."""
    return x.transpose(1, 2).contiguous().transpose(1, 2) if case["layout"] == "head" else x.contiguous()


def _prepare_append(case, seed):
    s, gen, dt = _State(), _gen(seed), _DTYPES[case["dtype"]]
    n, hq, hk, d, rot = case["n_tok"], case["heads"], case["kv_heads"], case["d"], case["rot"]
    # one projection's output, of which queries, keys and values are views
    qkv = torch.randn(n, (hq + 2 * hk) * d, generator=gen, device=DEV, dtype=torch.float32).mul_(1.5).to(dt)
    s.q, s.k, s.v = (x.view(n, -1, d) for x in qkv.split([hq * d, hk * d, hk * d], dim=1))
    s.pos = torch.randint(0, case["max_pos"], (n,), generator=gen, device=DEV, dtype=torch.int32)
    n_pages = -(-n // case["page"]) + 3
    shape = (n_pages, case["page"], hk)
    s.codes = [_paged(torch.randint(0, 256, shape + (d // 2,), generator=gen, device=DEV, dtype=torch.uint8), case)
               for _ in range(2)]
    s.scales = [_paged(torch.randint(24, 72, shape + (_scale_bytes(d),), generator=gen, device=DEV, dtype=torch.uint8), case)
                for _ in range(2)]
    s.unit = [_units(gen, case), _units(gen, case)]
    s.slot = torch.randperm(n_pages * case["page"], generator=gen, device=DEV)[:n].contiguous()
    s.every = torch.arange(n_pages * case["page"], device=DEV)
    s.q_norm = s.k_norm = None
    if case["norm"]:
        s.q_norm, s.k_norm = ((1 + 0.2 * torch.randn(d, generator=gen, device=DEV)).to(dt) for _ in range(2))
    # cosines and sines of every position, rounded to 32 bits
    t = (torch.arange(case["max_pos"], device=DEV, dtype=torch.float64)[:, None]
         * 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot))
    s.rope = torch.cat([t.cos(), t.sin()], dim=1).float()
    s.out = torch.empty(n, hq, d, device=DEV, dtype=dt)
    return s


def _lengths(case):
    """New tokens and keys of every sequence: they belong to the case; what fills them comes from the seed."""
    rng, n_seq = random.Random(case["kv_max"]), case["n_seq"]
    if case["K"] or case["q_max"] == 1:
        q_len = [case["q_max"]] * n_seq
    else:
        q_len = [case["q_max"]] + [rng.randint(1, case["q_max"]) for _ in range(n_seq - 1)]
    kv_len = [max(n, case["kv_max"] if i == 0 else rng.randint(case["kv_max"] // 4, case["kv_max"]))
              for i, n in enumerate(q_len)]
    return q_len, kv_len


def _tree_sees(K, gamma):
    """Node 1 + k * gamma + j is the j-th of chain k: it sees the root and its own chain up to itself."""
    n = 1 + K * gamma
    node = torch.arange(1, n)
    chain, depth = (node - 1) // max(gamma, 1), (node - 1) % max(gamma, 1)
    sees = torch.zeros(n, -(-n // 32) * 32, dtype=torch.int64)
    sees[:, 0] = 1
    sees[1:, 1:n] = (chain[:, None] == chain[None, :]) & (depth[:, None] >= depth[None, :])
    return sees


def _words(bits):
    """int32 words of [..., 32 * words] bits, the first bit lowest."""
    x = (bits.unflatten(-1, (-1, 32)).long() << torch.arange(32, device=bits.device)).sum(-1)
    return torch.where(x >= 1 << 31, x - (1 << 32), x).to(torch.int32)


def _prepare_attend(case, seed):
    s, gen, dt = _State(), _gen(seed), _DTYPES[case["dtype"]]
    n_seq, page, d, hk = case["n_seq"], case["page"], case["d"], case["kv_heads"]
    q_len, kv_len = _lengths(case)
    s.max_q, s.max_kv, s.n_tok = max(q_len), max(kv_len), sum(q_len)
    held = [-(-n // page) for n in kv_len]
    n_pages = sum(held) + 5
    s.codes, s.scales, s.unit = [], [], [_units(gen, case), _units(gen, case)]
    for unit in s.unit:
        x = torch.randn(n_pages, page, hk, d, generator=gen, device=DEV)
        codes, scales = _quantise(x, unit)
        s.codes.append(_paged(codes, case))
        s.scales.append(_paged(scales, case))
    perm = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    width = max(held) + 1
    at = torch.arange(width, device=DEV)[None, :]
    first = _i32([sum(held[:i]) for i in range(n_seq)])[:, None]
    s.pages = torch.where(at < _i32(held)[:, None], perm[(first + at).clamp(max=n_pages - 1)], -1).contiguous()
    s.kv_len, s.q_off = _i32(kv_len), _i32([sum(q_len[:i]) for i in range(n_seq + 1)])
    s.q = torch.randn(s.n_tok, case["heads"], d, generator=gen, device=DEV, dtype=torch.float32).mul_(2).to(dt)
    s.mask = None
    if case["K"]:
        s.mask = _words(_tree_sees(case["K"], case["gamma"])).to(DEV).repeat(n_seq, 1).contiguous()
    s.out = torch.empty(s.n_tok, case["heads"], d, device=DEV, dtype=dt)
    return s


def _prepare_pages(case, seed):
    s, gen, rng = _State(), _gen(seed), random.Random(case["kv_max"])
    n_seq, page, q = case["n_seq"], case["page"], case["q_max"]
    n_new = [rng.randint(0, q) if case["ragged"] and i else q for i in range(n_seq)]
    lens = [case["kv_max"] if i == 0 else rng.randint(0, case["kv_max"]) for i in range(n_seq)]
    held = [-(-n // page) for n in lens]
    want = sum(max(0, -(-(n + m) // page) - h) for n, m, h in zip(lens, n_new, held))
    spare = want * 3 // 4 if case["short"] else want + 7
    n_pages = sum(held) + spare
    s.n_tok = sum(n_new) + 5  # a batch padded to its captured size
    s.kv_len, s.n_new, s.held = _i32(lens), _i32(n_new), _i32(held)
    s.keep = _i32([n + (rng.randint(1, m) if m else 0) for n, m in zip(lens, n_new)])
    perm = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    width = -(-(case["kv_max"] + q) // page) + 1
    at = torch.arange(width, device=DEV)[None, :]
    first = _i32([0] + held).cumsum(0)[:-1, None]
    s.pages = torch.where(at < s.held[:, None], perm[(first + at).clamp(max=n_pages - 1)], -1).int().contiguous()
    s.free_list = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
    s.free_list[:spare] = perm[n_pages - spare:]
    s.free_count = _i32([spare])
    s.pos_off = None
    if case["tree"]:  # the depth of a node: the root, then chains of `tree` tokens
        i = torch.arange(s.n_tok, device=DEV)
        off = _i32([0] + n_new).cumsum(0)
        i = i - off[torch.searchsorted(off[1:], i, right=True).clamp(max=n_seq - 1)]
        s.pos_off = torch.where(i == 0, 0, 1 + (i - 1) % case["tree"]).int()
    return s


def _prepare_adjust(case, seed):
    s, gen, rng, dt = _State(), _gen(seed), random.Random(case["text_max"]), _DTYPES[case["dtype"]]
    n_seq, V = case["n_seq"], case["vocab"]
    nodes = 1 + case["K"] * case["gamma"]
    n = n_seq * nodes
    s.seq_off = _i32([i * nodes for i in range(n_seq + 1)])
    # tokens and logits of one 1 / rank law
    rank = torch.randperm(V, generator=gen, device=DEV)
    by_rank = rank.argsort().to(torch.int32)
    base = -torch.log(rank + 1.0)

    def tokens(*shape):
        return by_rank[(V ** torch.rand(shape, generator=gen, device=DEV, dtype=torch.float64)).long().clamp(max=V) - 1]

    s.logits = (base + 1.5 * torch.randn(n, V, generator=gen, device=DEV)).to(dt)
    s.text = s.length = s.prompt = s.node_tok = s.node_mask = s.rep = s.freq = s.pres = None
    if case["penalties"]:
        length = [case["text_max"] if i == 0 else rng.randint(0, case["text_max"]) for i in range(n_seq)]
        s.length, s.prompt = _i32(length), _i32([rng.randint(0, m) for m in length])
        s.text = tokens(n_seq, case["text_max"] + 8)
        s.node_tok = tokens(n)
        if case["K"] > 1:
            s.node_mask = _words(_tree_sees(case["K"], case["gamma"])).to(DEV).repeat(n_seq, 1).contiguous()
        u = torch.rand(3, n_seq, generator=gen, device=DEV)
        s.rep, s.freq, s.pres = 1 + 0.3 * u[0], 0.7 * u[1], 0.5 * u[2]
    s.bias_off = s.bias_tok = s.bias_val = s.allowed = None
    if case["bias"]:
        m = [rng.randint(0, case["bias"]) for _ in range(n_seq)]
        s.bias_off = _i32([sum(m[:i]) for i in range(n_seq + 1)])
        m = [min(x, V) for x in m]
        s.bias_tok = torch.cat([torch.randperm(V, generator=gen, device=DEV)[:x] for x in m] + [rank[:1]]).int()
        s.bias_off = _i32([sum(m[:i]) for i in range(n_seq + 1)])
        s.bias_val = 5 * torch.randn(s.bias_tok.numel(), generator=gen, device=DEV)
    if case["grammar"]:  # within a text nearly everything is allowed, at a structure's border a few tokens
        share = _pick(gen, (0.95, 0.5, 0.003), n)
        bits = torch.rand(n, -(-V // 32) * 32, generator=gen, device=DEV) < share[:, None]
        s.allowed = _words(bits).contiguous()
    s.out = torch.empty_like(s.logits)
    return s


def _pick(gen, values, n):
    return torch.tensor(values, device=DEV)[torch.randint(0, len(values), (n,), generator=gen, device=DEV)]


_PREPARE = {"append4": _prepare_append, "attend4": _prepare_attend, "pages": _prepare_pages, "adjust": _prepare_adjust}


def prepare(case, seed):
    s = _PREPARE[case["kind"]](case, seed)
    s.case = case
    return s


# ---------------------------------------------------------------- one pass, plain

def _norm_rotate(x, weight, s, case):
    x = x.float()
    if weight is not None:
        x = x * (torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight.float())
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
    new = [_norm_rotate(s.k, s.k_norm, s, case), s.v.float()]
    read = []
    page_all, at_all = s.every // case["page"], s.every % case["page"]
    for codes, scales, unit, x in zip(s.codes, s.scales, s.unit, new):
        codes[page, at], scales[page, at] = _quantise(x, unit)
        read.append(_value(codes[page_all, at_all], scales[page_all, at_all], unit).to(dt))
    return {"q": s.out, "k": read[0], "v": read[1]}


def _plain_attend(s, case):
    n_seq, m, L, hq, hk, d = case["n_seq"], s.max_q, s.max_kv, case["heads"], case["kv_heads"], case["d"]
    j = torch.arange(L, device=DEV)
    page, at = s.pages.long().clamp(min=0)[:, j // case["page"]], j % case["page"]
    k, v = (_value(c[page, at], x[page, at], u) for c, x, u in zip(s.codes, s.scales, s.unit))  # [n_seq, L, hk, d]
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


def _plain_pages(s, case):
    page, (n_seq, width) = case["page"], s.pages.shape
    at = torch.arange(width, device=DEV)
    # the step: each sequence's pages up to its new length, the pool's last ones first, sequences in order
    total = s.kv_len + s.n_new
    upto = (total + page - 1) // page
    fits = upto <= width
    need = torch.where(fits & (s.n_new > 0), (upto - s.held).clamp(min=0), 0)
    cum = need.cumsum(0)
    served = fits & ((need == 0) | (cum <= s.free_count))
    given = torch.where(served, need, 0)
    k = (cum - need)[:, None] + at - s.held[:, None]
    new = (at >= s.held[:, None]) & (at < (s.held + given)[:, None])
    taken = s.free_list[(s.free_count - 1 - k).clamp(0, s.free_list.numel() - 1).long()]
    s.pages.copy_(torch.where(new, taken, s.pages))
    s.held += given
    s.free_count -= given.sum().int()
    q_off = torch.cat([s.n_new.new_zeros(1), s.n_new.cumsum(0).int()])
    i = torch.arange(s.n_tok, device=DEV)
    seq = torch.searchsorted(q_off[1:], i, right=True).clamp(max=n_seq - 1)
    there = (i < q_off[-1]) & served[seq]
    place = s.kv_len[seq] + i - q_off[seq]
    got = s.pages[seq, (place // page).clamp(max=width - 1).long()].long()
    slot = torch.where(there, got * page + place % page, -1)
    pos = torch.where(i < q_off[-1], s.kv_len[seq] + (i - q_off[seq] if s.pos_off is None else s.pos_off), 0).int()
    out = {"q_off": q_off, "kv_len": torch.where(served, total, 0).int(), "slot": slot, "pos": pos,
           "seq": torch.where(i < q_off[-1], seq, -1).int()}
    # after the step: pages behind what is kept go back, so that the next ones to be taken are the same again
    keep = torch.minimum((s.keep + page - 1) // page, s.held)
    back = s.held - keep
    cum = back.cumsum(0)
    k = (cum - back)[:, None] + at - keep[:, None]
    gone = (at >= keep[:, None]) & (at < s.held[:, None])
    to = torch.where(gone, s.free_count + cum[-1] - 1 - k, s.free_list.numel()).long()
    s.free_list.copy_(torch.cat([s.free_list, s.free_list[:1]]).scatter_(0, to.flatten(), s.pages.flatten())[:-1])
    s.pages.masked_fill_(gone, -1)
    s.held.copy_(keep)
    s.free_count += cum[-1].int()
    return dict(out, pages=s.pages, held=s.held, free_list=s.free_list, free_count=s.free_count)


def _plain_adjust(s, case):
    V, n = case["vocab"], s.logits.shape[0]
    row = torch.arange(n, device=DEV)
    seq = torch.searchsorted(s.seq_off[1:], row.int(), right=True)
    x = s.logits.float()
    if s.text is not None:
        at = torch.arange(s.text.shape[1], device=DEV)
        one = torch.ones((), dtype=torch.int32, device=DEV)
        prompt, output = (torch.zeros(case["n_seq"], V + 1, dtype=torch.int32, device=DEV).scatter_add_(
            1, torch.where(which, s.text, V).long(), one.expand(s.text.shape)) for which in (
                at < s.prompt[:, None], (at >= s.prompt[:, None]) & (at < s.length[:, None])))
        count = output[seq, :V]
        nodes = 1 + case["K"] * case["gamma"]
        i = torch.arange(nodes, device=DEV)
        if s.node_mask is None:
            sees = i <= (row - s.seq_off[seq])[:, None]
        else:
            sees = (s.node_mask[:, i // 32] >> (i % 32)) & 1 > 0
        count.scatter_add_(1, s.node_tok[s.seq_off[seq][:, None] + i].long(), sees.int())
        said = (count > 0) | (prompt[seq, :V] > 0)
        rep = s.rep[seq][:, None]
        x = torch.where(said, torch.where(x > 0, x / rep, x * rep), x)
        x = x - s.freq[seq][:, None] * count
        x = x - s.pres[seq][:, None] * (count > 0)
        del count, said
    if s.bias_tok is not None:
        m = int(s.bias_tok.numel()) - 1
        owner = torch.searchsorted(s.bias_off[1:], torch.arange(m, device=DEV, dtype=torch.int32), right=True)
        bias = torch.zeros(case["n_seq"], V, device=DEV)
        bias[owner, s.bias_tok[:m].long()] = s.bias_val[:m]
        x = x + bias[seq]
    if s.allowed is not None:
        t = torch.arange(V, device=DEV)
        x = torch.where((s.allowed[:, t // 32] >> (t % 32)) & 1 > 0, x, -math.inf)
    s.out.copy_(x)
    return s.out


_PLAIN = {"append4": _plain_append, "attend4": _plain_attend, "pages": _plain_pages, "adjust": _plain_adjust}


# ---------------------------------------------------------------- one pass, by the package

def _cache(s, case):
    from paper_2609_21858_gb300 import pps
    k_unit, v_unit = s.unit if case["unit"] else (None, None)
    return pps.CacheQ4(s.codes[0], s.codes[1], s.scales[0], s.scales[1], k_unit, v_unit)


def _own_append(s, case):
    from paper_2609_21858_gb300 import pps
    cache = _cache(s, case)
    q = pps.kv_append_q4(s.q, s.k, s.v, s.pos, s.slot, cache, s.rope, q_norm=s.q_norm, k_norm=s.k_norm, eps=1e-6,
                         interleaved=case["interleaved"], out=s.out)
    k, v = pps.kv_read_q4(cache, s.every, dtype=s.q.dtype)
    return {"q": q, "k": k, "v": v}


def _own_attend(s, case):
    from paper_2609_21858_gb300 import pps
    return pps.paged_attention_q4(s.q, _cache(s, case), s.pages, s.kv_len, s.q_off, mask=s.mask, out=s.out)


def _own_pages(s, case):
    from paper_2609_21858_gb300 import pps
    out = pps.kv_reserve(s.pages, s.held, s.free_list, s.free_count, s.kv_len, s.n_new, case["page"], s.n_tok,
                         pos_off=s.pos_off)
    pps.kv_trim(s.pages, s.held, s.free_list, s.free_count, s.keep, case["page"])
    return dict(out, pages=s.pages, held=s.held, free_list=s.free_list, free_count=s.free_count)


def _own_adjust(s, case):
    from paper_2609_21858_gb300 import pps
    return pps.adjust_logits(s.logits, s.seq_off, text=s.text, text_len=s.length, prompt_len=s.prompt, node_tok=s.node_tok,
                             node_mask=s.node_mask, repetition=s.rep, frequency=s.freq, presence=s.pres,
                             bias_off=s.bias_off, bias_tok=s.bias_tok, bias_val=s.bias_val, allowed=s.allowed, out=s.out)


_OWN = {"append4": _own_append, "attend4": _own_attend, "pages": _own_pages, "adjust": _own_adjust}


def run(state):
    return (_OWN if own else _PLAIN)[state.case["kind"]](state, state.case)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["kind"] == "append4":
        n, hq, hk, d, e = case["n_tok"], case["heads"], case["kv_heads"], case["d"], _BYTES[case["dtype"]]
        held, slots = 2 * hk * (d // 2 + d // 16), (-(-n // case["page"]) + 3) * case["page"]
        # projections in, queries and the cache's new rows out; then the whole cache in, its values out
        return {"bytes": n * ((2 * hq + 2 * hk) * d * e + held + 4 * case["rot"] + 12) + slots * (held + 2 * hk * d * e + 8),
                "flops": n * (hq + 2 * hk) * d * 10 + slots * 2 * hk * d}
    if case["kind"] == "attend4":
        q_len, kv_len = _lengths(case)
        hq, hk, d = case["heads"], case["kv_heads"], case["d"]
        own_keys = [m * (1 + case["gamma"] / 2 if case["K"] else (m + 1) / 2) for m in q_len]  # of a token's new ones, in all
        pairs = sum(m * (n - m) + o for m, n, o in zip(q_len, kv_len, own_keys))
        return {"bytes": 2 * _BYTES[case["dtype"]] * d * hq * sum(q_len) + 2 * hk * (d // 2 + d // 16) * sum(kv_len),
                "flops": 4 * d * hq * pairs}
    if case["kind"] == "pages":
        n = case["n_seq"]
        tok = n * (case["q_max"] / 2 if case["ragged"] else case["q_max"])
        new = tok / case["page"] + n / 2
        return {"bytes": tok * 20 + n * 4 * 9 + new * 4 * 5, "flops": 10 * (tok + n)}
    nodes = 1 + case["K"] * case["gamma"]
    n, V = case["n_seq"] * nodes, case["vocab"]
    return {"bytes": n * V * (2 * _BYTES[case["dtype"]] + case["grammar"] / 8)
            + case["penalties"] * 4 * (case["n_seq"] * case["text_max"] / 2 + n) + 4 * case["bias"] * case["n_seq"],
            "flops": n * V * 4}


# ---------------------------------------------------------------- the same in 64 bits, from the definitions

def _exact_block(z):
    """The values that [..., blocks, 16] numbers in 64 bits are held as, in units."""
    want = (z.abs().amax(-1, keepdim=True) / 6).clamp(max=448.0)
    step = 2.0 ** (torch.frexp(want).exponent - 1).clamp(min=-6).double() / 8  # of e4m3 numbers there
    scale = torch.round(want / step) * step
    m = torch.where(scale > 0, z / scale, 0.0).clamp(-6, 6)
    step = torch.where(m.abs() < 2, 0.5, torch.where(m.abs() < 4, 1.0, 2.0))  # of e2m1 numbers
    return torch.round(m / step) * step * scale


def _exact_held(codes, scales, unit, d):
    """Codes and scales [..., heads, bytes], byte by byte from the formats' definitions."""
    nib = torch.stack([codes % 16, codes // 16], dim=-1).flatten(-2).long()
    e, m = (nib % 8) // 2, (nib % 2).double()
    x = torch.where(e == 0, m / 2, 2.0 ** (e - 1).double() * (1 + m / 2)) * (1 - 2 * (nib // 8))
    b = scales[..., :d // 16].long()
    e, m = (b % 128) // 8, (b % 8).double()
    s = torch.where(e == 0, m / 512, 2.0 ** (e - 7).double() * (1 + m / 8))
    return (x.unflatten(-1, (-1, 16)) * s[..., None]).flatten(-2) * unit.double()[:, None]


def _exact_append(s, case):
    d, page = case["d"], case["page"]

    def heads(x, weight):
        x = x.double().clone()
        if weight is not None:
            x = weight.double() * x / ((x ** 2).sum(-1, keepdim=True) / d + 1e-6) ** 0.5
        half = case["rot"] // 2
        c = torch.arange(half, device=DEV)
        first, second = (2 * c, 2 * c + 1) if case["interleaved"] else (c, c + half)
        # the pair as a complex number, turned by the table's
        turn = torch.complex(s.rope[s.pos.long(), :half].double(), s.rope[s.pos.long(), half:].double())[:, None]
        z = torch.complex(x[..., first], x[..., second]) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    out = {"q": heads(s.q, s.q_norm)}
    for name, codes, scales, unit, x in zip("kv", s.codes, s.scales, s.unit, (heads(s.k, s.k_norm), s.v.double())):
        held = _exact_held(codes, scales, unit, d)
        x = x / unit.double()[:, None]
        held[s.slot // page, s.slot % page] = _exact_block(x.unflatten(-1, (-1, 16))).flatten(-2) * unit.double()[:, None]
        out[name] = held.flatten(0, 1)
    return out


def _exact_attend(s, case):
    out = torch.zeros(s.out.shape, dtype=torch.float64, device=DEV)
    group, off, lens, d = case["heads"] // case["kv_heads"], s.q_off.tolist(), s.kv_len.tolist(), case["d"]
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
            k, v = (_exact_held(c[held, :, h:h + 1], x[held, :, h:h + 1], u[h:h + 1], d).flatten(0, 1)[:n_kv, 0]
                    for c, x, u in zip(s.codes, s.scales, s.unit))
            for g in range(h * group, (h + 1) * group):
                w = (s.q[a:b, g].double() @ k.T) / math.sqrt(d)
                w = torch.softmax(w.masked_fill_(~sees, -math.inf), dim=-1)
                out[a:b, g] = w @ v
    return out


def _exact_adjust(s, case):
    V, nodes = case["vocab"], 1 + case["K"] * case["gamma"]
    out = s.logits.double()
    sees = _tree_sees(case["K"], case["gamma"])[:, :nodes].bool().to(DEV) if case["K"] > 1 else torch.ones(
        nodes, nodes, dtype=torch.bool, device=DEV).tril()
    for i in range(case["n_seq"]):
        rows = slice(i * nodes, (i + 1) * nodes)
        if s.text is not None:
            text, p, n = s.text[i].long(), int(s.prompt[i]), int(s.length[i])
            before, after = torch.bincount(text[:p], minlength=V), torch.bincount(text[p:n], minlength=V)
            for j in range(nodes):
                count = after + torch.bincount(s.node_tok[rows][sees[j]].long(), minlength=V)
                x = out[i * nodes + j]
                rep = torch.where(before + count > 0, s.rep[i].double(), 1.0)
                x.copy_(torch.where(x > 0, x / rep, x * rep) - s.freq[i].double() * count - s.pres[i].double() * (count > 0))
        if s.bias_tok is not None:
            a, b = int(s.bias_off[i]), int(s.bias_off[i + 1])
            out[rows, s.bias_tok[a:b].long()] += s.bias_val[a:b].double()
        if s.allowed is not None:
            bits = (s.allowed[rows, :, None] >> torch.arange(32, device=DEV)) & 1
            out[rows].masked_fill_(bits.flatten(1)[:, :V] == 0, -math.inf)
    return out


def exact(case, seed):
    if case["kind"] == "pages":
        return None  # whole numbers only
    s = prepare(case, seed)
    return {"append4": _exact_append, "attend4": _exact_attend, "adjust": _exact_adjust}[case["kind"]](s, case)
