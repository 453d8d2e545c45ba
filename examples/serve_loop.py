"""A serving loop of a multi-block diffusion language model around this package, with a one-layer random model.

Every forward runs the committed blocks that are not in the cache yet and the window of block slots behind them
(kv_tables, kv_write, kv_attention with the engine's block-causal mask), reads the LM head at the window's masked
positions (commit_step), and moves the window on (commit_sweep). The window's own keys and values are written for the
forward and given back after it; committed blocks are computed once more with their final tokens and stay ("one-step cache writes").
A request whose table has no room for the next forward stands still from then on, with all that it has committed.
Nothing waits for the GPU inside the loop.

    python examples/serve_loop.py [steps]
"""

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2609_33887_gb300 as bdc  # noqa: E402


class Model:
    """Embedding, one attention layer with grouped heads, residual, LM head: enough to run every operator."""

    def __init__(self, vocab=4096, d=512, n_q=8, n_kv=2, dim=64, max_len=4096, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def w(*shape, std):
            return (torch.randn(*shape, generator=g, device="cuda") * std).to(torch.bfloat16)

        self.vocab, self.n_q, self.n_kv, self.dim = vocab, n_q, n_kv, dim
        self.embed, self.place = w(vocab + 1, d, std=1.0), w(max_len, d, std=0.5)  # the last row: the mask token
        self.qkv, self.out = w((n_q + 2 * n_kv) * dim, d, std=d ** -0.5), w(d, n_q * dim, std=(n_q * dim) ** -0.5)
        self.head = w(vocab, d, std=3 * d ** -0.5)


class Server:
    def __init__(self, model, n_seq=6, n_slots=3, block_len=16, page=32, max_len=768, tau=0.3):
        self.m, self.n_seq, self.B, self.L, self.page, self.tau = model, n_seq, n_slots, block_len, page, [tau]
        self.W, self.max_len = n_slots * block_len, -(-max_len // page) * page  # as many tokens as its table's pages hold
        n_pages = n_seq * (self.max_len // page)
        self.cache = bdc.kv_cache(n_pages, page, model.n_kv, model.dim)

        def ints(*shape, fill=0, dtype=torch.int32):
            return torch.full(shape, fill, dtype=dtype, device="cuda")

        self.table = ints(n_seq, self.max_len // page, fill=-1)
        self.free = torch.randperm(n_pages, device="cuda").to(torch.int32)
        self.pool = torch.tensor([0, n_pages], dtype=torch.int64, device="cuda")
        self.lens = ints(n_seq)        # tokens that stay in the cache
        self.pending = ints(n_seq)     # committed blocks that the next forward computes once more
        self.blocks = ints(n_seq, self.W)  # their tokens
        self.tokens = ints(n_seq * self.W, fill=model.vocab)
        self.masked = ints(n_seq * self.W, fill=1, dtype=torch.uint8)
        self.flags = ints(n_seq * n_slots, fill=bdc.BD_BLOCK_ACTIVE, dtype=torch.uint8)
        self.flags[::n_slots] |= bdc.BD_BLOCK_FALLBACK_ELIGIBLE

    def tables(self, lens, new, max_tokens):
        r = bdc.kv_tables(lens, new, self.table, self.free, self.pool, page_size=self.page, max_tokens=max_tokens)
        self.pool = r.pool
        return r

    def forward(self):
        """Hidden states [n_seq * W, d] of the window; the forward's tables and attention are kept to be looked at."""
        m, W, most = self.m, self.W, 2 * self.n_seq * self.W
        kept = self.pending * self.L
        t = self.t = self.tables(self.lens, kept + W, most)
        i = torch.arange(most, device="cuda")
        s = torch.searchsorted(t.query_start[1:], i, right=True).clamp(max=self.n_seq - 1)
        o = i - t.query_start[s]  # of the request's new tokens: first the committed blocks, then the window
        inside = o >= kept[s]
        token = torch.where(inside, self.tokens.view(self.n_seq, W)[s, (o - kept[s]).clamp(0, W - 1)],
                            self.blocks[s, o.clamp(0, W - 1)])
        x = m.embed[token] + m.place[t.positions.clamp(0, len(m.place) - 1)]
        qkv = (x @ m.qkv.T).view(most, -1, m.dim)
        q, k, v = qkv.split([m.n_q, m.n_kv, m.n_kv], 1)
        bdc.kv_write(k, v, t.slot_map, self.cache)
        self.q, self.a = q, bdc.kv_attention(q, self.cache, self.table, t.kv_lens, t.query_start, max_q_len=2 * W,
                                             max_kv_len=self.max_len, mask_block=self.L)
        rows = (t.query_start[:-1] + kept)[:, None] + torch.arange(W, device="cuda")
        rows = rows.reshape(-1)
        return x[rows] + self.a[rows].reshape(len(rows), -1) @ m.out.T

    def step(self):
        """One forward, commit and sweep; returns (blocks committed [n_seq], positions resolved [n_seq])."""
        hidden = self.forward()
        tokens, _, commit, _ = bdc.commit_step(hidden, self.m.head, self.masked, self.flags, self.n_seq, self.B, self.L,
                                               self.tau)
        # a request that got no pages was computed over the wrong tokens: its commits are dropped, its window stays
        served = self.t.status == 0
        commit = torch.where(served[:, None], commit.view(self.n_seq, self.W), 0).view(-1)
        blocks, done, resolved = bdc.commit_sweep(
            self.tokens, self.masked, self.flags, self.n_seq, self.B, self.L, tokens, commit, 0,
            mask_token_id=self.m.vocab, options=bdc.BD_SWEEP_ADMIT | bdc.BD_SWEEP_ELIGIBLE_OLDEST)
        # the window's pages go back; the blocks that this forward computed with their final tokens stay
        self.lens = self.tables(self.t.kv_lens, torch.where(served, -self.W, 0).int(), 0).kv_lens
        self.blocks = torch.where(served[:, None], blocks.view(self.n_seq, self.W), self.blocks)
        self.pending = torch.where(served, done, self.pending)
        return done, resolved


def main(steps=40):
    server = Server(Model())
    total = torch.zeros(2, dtype=torch.int64, device="cuda")
    for _ in range(steps):
        done, resolved = server.step()
        total += torch.stack([done.sum(), resolved.sum()])
    blocks, positions = total.tolist()
    print(f"{steps} forwards of {server.n_seq} requests: {positions} positions resolved, {blocks} blocks committed, "
          f"{int(server.lens.sum())} tokens in the cache, {positions / steps / server.n_seq:.2f} tokens per forward")


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 40)
