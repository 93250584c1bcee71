"""A speculative decoding loop over a paged cache: the library's calls in the order of a serving step.

One step of `Session`, for all its sequences at once and without waiting for the device:

  draft      per depth, pps_lmhead_draft_list on the drafter's hidden rows (here: the token's embedding)
  target     per layer, pps_kv_append (norm, rotation, keys and values into the cache's pages) and
             pps_paged_attention (the step's nodes over the cache, ancestors by mask)
  verify     pps_lmhead_verify_tree (the keyed race of every node and the walk), or, for chains,
             pps_verify_chain (the token-level maximal coupling) on pps_lmhead_logits
  keep       the accepted nodes' keys and values move up behind the prefix: pps_kv_append once more, with
             slot -1 for the others (a chain's nodes already lie there)

`Decoder` is a small stand-in for a model: attention layers with random weights, whose projections are torch
matmuls.  `python -m paper_2609_21858_gb300.decode` runs it.
"""
from __future__ import annotations

import argparse

import torch
import torch.nn.functional as F

from . import pps, synth


class Cache:
    """Paged keys and values of every layer, and each sequence's page table (its pages in no order)."""

    def __init__(self, n_seq: int, capacity: int, layers: int, kv_heads: int, head_dim: int, page_size: int = 16,
                 dtype=torch.bfloat16, device="cuda"):
        columns = -(-capacity // page_size)
        self.page_size, self.capacity = page_size, columns * page_size
        shape = (layers, n_seq * columns, page_size, kv_heads, head_dim)
        self.k = torch.zeros(shape, dtype=dtype, device=device)
        self.v = torch.zeros(shape, dtype=dtype, device=device)
        gen = torch.Generator().manual_seed(n_seq * columns)
        self.pages = torch.randperm(n_seq * columns, generator=gen).to(torch.int32).view(n_seq, columns).to(device)

    def slots(self, seq: torch.Tensor, pos: torch.Tensor) -> torch.Tensor:
        """The cache slots of positions `pos` of sequences `seq` (int64)."""
        return self.pages[seq, pos // self.page_size].long() * self.page_size + pos % self.page_size


class Decoder:
    """Attention layers with random weights, tied to nothing: x += Wo attention(norm x), then the LM head."""

    def __init__(self, vocab: int, width: int, layers: int, heads: int, kv_heads: int, head_dim: int,
                 max_pos: int = 4096, qk_norm: bool = True, dtype=torch.bfloat16, seed: int = 0, device="cuda"):
        self.vocab, self.width, self.heads, self.kv_heads, self.head_dim = vocab, width, heads, kv_heads, head_dim
        gen = torch.Generator().manual_seed(seed)

        def normal(*shape, std=1.0):
            return (torch.randn(shape, generator=gen) * std).to(dtype).to(device)

        self.embed = normal(vocab, width)
        self.head = normal(vocab, width, std=2.0 * width ** -0.5)
        self.wqkv = [normal((heads + 2 * kv_heads) * head_dim, width, std=width ** -0.5) for _ in range(layers)]
        self.wo = [normal(width, heads * head_dim, std=(heads * head_dim) ** -0.5) for _ in range(layers)]
        self.qk = [normal(2, head_dim, std=0.1) + 1 if qk_norm else (None, None) for _ in range(layers)]
        self.rope = pps.rope_table(max_pos, head_dim, device=device)

    def norm(self, x):
        return F.rms_norm(x, (self.width,), eps=1e-6)

    def forward(self, tok, pos, slot, cache: Cache, kv_len, q_off, mask=None, status=None):
        """The hidden rows of new tokens (one per token, for the LM head) and each layer's keys and values as
        projected.  Sequence s's tokens are q_off[s] .. q_off[s+1]-1; kv_len counts them in."""
        n, hd = tok.numel(), self.head_dim
        x = self.embed[tok.long()]
        kept = []
        for l, (wqkv, wo, (qn, kn)) in enumerate(zip(self.wqkv, self.wo, self.qk)):
            y = (self.norm(x) @ wqkv.T).view(n, -1, hd)
            q, k, v = y.split([self.heads, self.kv_heads, self.kv_heads], dim=1)
            q = pps.kv_append(q, k, v, pos, slot, cache.k[l], cache.v[l], self.rope, qn, kn, status=status)
            a = pps.paged_attention(q, cache.k[l], cache.v[l], cache.pages, kv_len, q_off, mask=mask, status=status)
            x = x + a.view(n, -1) @ wo.T
            kept.append((k, v))
        return self.norm(x), kept

    def keep(self, kept, pos, slot, cache: Cache, status=None):
        """Write tokens' keys and values, as `forward` returned them, to other slots (< 0: not written)."""
        for l, (k, v) in enumerate(kept):
            kn = self.qk[l][1]
            pps.kv_append(k, k, v, pos, slot, cache.k[l], cache.v[l], self.rope, None, kn, status=status)


class Session:
    """Sequences that decode together.  `branching[d]`: children of a node of depth d; all ones: chains.
    `text` [n_seq, ...] holds the tokens, `length` [n_seq] how many of them the cache holds (the next one,
    text[s, length[s]], is known and not cached yet)."""

    def __init__(self, model: Decoder, branching, n_seq: int, capacity: int, key: int = 1, temperature: float = 1.0,
                 page_size: int = 16):
        dev, i32 = model.embed.device, torch.int32
        self.model, self.temperature, self.device = model, temperature, dev
        self.tree = t = synth.make_tree(branching, n_seq)
        self.nodes, self.width = t.nodes_per_seq, t.gamma + 1
        self.cache = Cache(n_seq, capacity, len(model.wo), model.kv_heads, model.head_dim, page_size,
                           model.embed.dtype, dev)
        put = lambda x: torch.as_tensor(x).to(dev)
        self.seq_off, self.node_draft_row, self.child_node = put(t.seq_off), put(t.node_draft_row), put(t.child_node)
        self.depth, self.row_k = put(t.node_depth).long(), put(t.row_k)
        self.seq = torch.arange(n_seq, device=dev)
        self.node_seq = self.seq.repeat_interleave(self.nodes)
        self.node_index = torch.arange(self.nodes, device=dev).repeat(n_seq)
        # node b of a sequence sees itself and its ancestors
        parent = [-1] * self.nodes
        for row, children in zip(t.draft_node[:t.draft_per_seq], t.child_node):
            for c in children:
                if c >= 0:
                    parent[c] = int(row)
        words = -(-self.nodes // 32)
        bits = [0] * self.nodes
        for b in range(self.nodes):
            bits[b] = 1 << b | (bits[parent[b]] if b else 0)
        mask = torch.tensor([[(x >> 32 * w) & 0xffffffff for w in range(words)] for x in bits], dtype=torch.int64)
        self.mask = mask.to(i32).repeat(n_seq, 1).to(dev)  # modulo 2^32: the same bits
        # nodes of a depth are neighbours, and so are the draft lists of those with children
        count, self.levels, first = 1, [], 0
        for b in t.branching:
            self.levels.append((first, first + count))
            first, count = first + count, count * b
        self.key = (torch.arange(n_seq, device=dev, dtype=torch.int64) + 1) * key
        self.zero = torch.zeros(t.n_nodes, dtype=torch.int64, device=dev)
        self.node_key = self.key[self.node_seq]
        self.status = torch.zeros(1, dtype=i32, device=dev)
        self.length = torch.zeros(n_seq, dtype=torch.int64, device=dev)
        self.text = torch.full((n_seq, self.cache.capacity + self.width), -1, dtype=i32, device=dev)
        self.most = 0  # what no length passes
        self.gen = torch.Generator(device=dev).manual_seed(key)

    def prefill(self, prompts):
        """Take in the prompts (lists of tokens, one or more each): all but the last token into the cache."""
        if len(prompts) != self.tree.n_seq or any(len(p) < 1 for p in prompts):
            raise ValueError(f"{self.tree.n_seq} prompts of one token or more")
        n = [len(p) - 1 for p in prompts]
        self.most = max(n)
        self._room(0)
        put = lambda x, dt: torch.tensor(x, dtype=dt, device=self.device)
        for s, p in enumerate(prompts):
            self.text[s, :len(p)] = put(p, torch.int32)
        self.length = put(n, torch.int64)
        if sum(n) == 0:
            return
        tok = put([x for p in prompts for x in p[:-1]], torch.int64)
        pos = put([i for m in n for i in range(m)], torch.int64)
        seq = self.seq.repeat_interleave(self.length)
        off = [0]
        for m in n:
            off.append(off[-1] + m)
        self.model.forward(tok, pos.int(), self.cache.slots(seq, pos), self.cache, self.length.int(),
                           put(off, torch.int32), status=self.status)

    def _room(self, more: int):
        if self.most + more > self.cache.capacity:
            raise ValueError(f"sequences of up to {self.most} + {more} tokens; the cache holds {self.cache.capacity}")

    def _draft(self):
        """The nodes' tokens and the draft lists, depth by depth."""
        t, n = self.tree, self.tree.n_seq
        tok = torch.zeros(n, self.nodes, dtype=torch.int64, device=self.device)
        tok[:, 0] = self.text[self.seq, self.length]
        lists = torch.full((n, t.draft_per_seq, t.K), -1, dtype=torch.int32, device=self.device)
        counts = torch.zeros(n, t.draft_per_seq, dtype=torch.int32, device=self.device)
        for d, (lo, hi) in enumerate(self.levels):
            rows = n * (hi - lo)
            pos = (self.length + d + 1).int().repeat_interleave(hi - lo)
            row_k = self.row_k.view(n, -1)[:, lo:hi].flatten().contiguous()
            x = self.model.norm(self.model.embed[tok[:, lo:hi].reshape(-1)])
            y = pps.lmhead_draft_list(x, self.model.head, self.key.repeat_interleave(hi - lo), self.zero[:rows], pos,
                                      t.K, row_k=row_k, temperature=self.temperature, status=self.status)
            lists[:, lo:hi] = y["tok"].view(n, hi - lo, t.K)
            counts[:, lo:hi] = y["ndist"].view(n, hi - lo)
            b = t.branching[d]
            # a list that ran short has -1 entries; their nodes are never reached, and any token will do
            tok[:, hi:hi + b * (hi - lo)] = lists[:, lo:hi, :b].reshape(n, -1).clamp_min(0)
        return tok.view(-1), lists.view(-1, t.K), counts.view(-1)

    def step(self, coupling: bool = False):
        """Draft, score and verify once; returns the verification's outputs (on the device).  coupling: chains
        only, pps_verify_chain in place of the keyed race."""
        t, model = self.tree, self.model
        if coupling and t.K != 1:
            raise ValueError("the token-level coupling verifies chains (branching of ones)")
        self._room(self.nodes)
        tok, lists, counts = self._draft()
        start = self.length[self.node_seq]
        pos = (start + self.depth).int()
        slot = self.cache.slots(self.node_seq, start + self.node_index)
        mask = self.mask if t.K > 1 else None  # a chain's nodes lie in their order: causal
        hidden, kept = model.forward(tok, pos, slot, self.cache, (self.length + self.nodes).int(), self.seq_off, mask,
                                     self.status)
        if coupling:
            drafter = model.norm(model.embed[tok.view(-1, self.nodes)[:, :-1].reshape(-1)])
            u = torch.rand(t.n_draft, generator=self.gen, device=self.device)
            noise = torch.empty(t.n_seq, model.vocab, device=self.device).exponential_(generator=self.gen)
            v = pps.verify_chain(pps.lmhead_logits(hidden, model.head), pps.lmhead_logits(drafter, model.head), t.gamma,
                                 self.seq_off, self.node_draft_row, lists.view(-1), u, noise, self.temperature,
                                 status=self.status)
        else:
            v = pps.lmhead_verify_tree(hidden, model.head, self.node_key, self.zero, pos + 1, t.gamma, self.seq_off,
                                       self.node_draft_row, lists, counts, self.child_node, self.temperature,
                                       status=self.status)
        if t.K > 1:
            model.keep(kept, pos, self._kept_slots(lists, v), self.cache, self.status)
        at = self.length[:, None] + 1 + torch.arange(self.width, device=self.device)
        self.text.scatter_(1, at, v["emitted"])
        self.length = self.length + v["n_emitted"]
        self.most += self.width
        return v

    def _kept_slots(self, lists, v):
        """Where the accepted nodes go: the node of depth d to the d-th slot after the root's; -1 for the others."""
        slot = torch.full((self.tree.n_nodes + 1,), -1, dtype=torch.int64, device=self.device)
        node = self.seq_off[:-1].long()
        child = self.child_node.view(lists.shape)
        for d in range(self.tree.gamma):
            row = self.node_draft_row[node].long()
            hit = (lists[row] == v["emitted"][:, d:d + 1]) & (d < v["accept_len"])[:, None]
            taken, nxt = hit.any(1), child[row, hit.int().argmax(1)].long()
            slot[torch.where(taken, nxt, self.tree.n_nodes)] = self.cache.slots(self.seq, self.length + 1 + d)
            node = torch.where(taken, nxt, node)
        return slot[:-1].contiguous()

    def tokens(self):
        """The tokens so far, a list per sequence (waits for the device)."""
        flags = int(self.status)
        if flags:
            raise pps.PPSError(f"status flags {flags:#x}")
        return [row[:n + 1] for row, n in zip(self.text.tolist(), self.length.tolist())]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--branching", default="4,1,1,1", help="children per depth; all ones: chains")
    ap.add_argument("--coupling", action="store_true", help="chains: the token-level coupling, not the keyed race")
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--steps", type=int, default=16)
    a = ap.parse_args(argv)
    branching = [int(x) for x in a.branching.split(",")]
    model = Decoder(vocab=8000, width=1024, layers=4, heads=16, kv_heads=4, head_dim=64)
    s = Session(model, branching, a.sequences, 64 + a.steps * (len(branching) + 1) + 256)
    s.prefill([[(7 * i + j) % 8000 for j in range(1 + 5 * i % 60)] for i in range(a.sequences)])
    accepted = torch.zeros((), dtype=torch.float64, device=s.device)
    for _ in range(a.steps):
        accepted += s.step(a.coupling)["accept_len"].double().mean()
    text = s.tokens()
    print(f"{a.sequences} sequences, {a.steps} steps: {accepted.item() / a.steps:.2f} accepted per step, "
          f"lengths {[len(x) for x in text]}")


if __name__ == "__main__":
    main()
