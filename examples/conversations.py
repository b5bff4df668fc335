"""Conversations on one stored document, through a small decoder.

A document is read once: its rows become a block in the cache's page pool.
Each conversation is given that block (no bytes are copied), reads its own
question on top of it, and answers token by token:

  document   per layer: kvg_cache_append_qkv + kvg_prompt_attention;
             then kvg_deposit into a pool-resident store
  question   kvg_graft into every conversation; per layer the packed questions
             of all of them: kvg_cache_append_qkv + kvg_prompt_attention
  answer     per step and layer one token of each conversation:
             kvg_cache_append_qkv + kvg_decode_attention_shared

The decoder has random weights: what it shows is the order of the calls.

    python examples/conversations.py [--fp8] [--document N] [--conversations N] [--steps N]
"""
import argparse
import math
import os
import sys
from dataclasses import dataclass

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_14431_gb300 import kvg  # noqa: E402

EPS = 1e-6


@dataclass
class Shape:
    layers: int = 4
    q_heads: int = 32
    kv_heads: int = 16
    head_dim: int = 128
    width: int = 2048
    hidden: int = 4096
    tokens: int = 8000  # of the vocabulary
    theta: float = 1e6
    page: int = 64


class Decoder:
    """Random weights, bf16; attention is handed in."""

    def __init__(self, shape: Shape, seed: int = 0, device: str = "cuda"):
        g = torch.Generator().manual_seed(seed)

        def weight(*size):
            return (torch.randn(*size, generator=g) * size[-1] ** -0.5).to(torch.bfloat16).to(device)

        s, d = shape, shape.head_dim
        self.shape = s
        self.embed = (torch.randn(s.tokens, s.width, generator=g)).to(torch.bfloat16).to(device)
        self.layers = [{"qkv": weight((s.q_heads + 2 * s.kv_heads) * d, s.width), "o": weight(s.width, s.q_heads * d),
                        "up": weight(2 * s.hidden, s.width), "down": weight(s.width, s.hidden),
                        "q_norm": (1 + 0.1 * torch.randn(d, generator=g)).to(torch.bfloat16).to(device),
                        "k_norm": (1 + 0.1 * torch.randn(d, generator=g)).to(torch.bfloat16).to(device)}
                       for _ in range(s.layers)]

    def __call__(self, tokens, attention):
        """Hidden states of the packed tokens; attention(layer, weights, q, k, v) -> [T][q heads x head_dim]."""
        s, x = self.shape, self.embed[tokens]
        for i, w in enumerate(self.layers):
            heads = F.linear(F.rms_norm(x, (s.width,), eps=EPS), w["qkv"]).view(len(x), -1, s.head_dim)
            x = x + F.linear(attention(i, w, *heads.split([s.q_heads, s.kv_heads, s.kv_heads], dim=1)), w["o"])
            gate, up = F.linear(F.rms_norm(x, (s.width,), eps=EPS), w["up"]).chunk(2, dim=-1)
            x = x + F.linear(F.silu(gate) * up, w["down"])
        return x

    def logits(self, x):
        return F.linear(F.rms_norm(x, (self.shape.width,), eps=EPS), self.embed)


class Conversations:
    """A batch of conversations on one document."""

    def __init__(self, model: Decoder, document, batch: int, most_rows: int, fp8: bool = False):
        """most_rows: of a conversation, behind the document."""
        s = model.shape
        self.model, self.batch = model, batch
        kind = kvg.KVG_KV_E4M3 if fp8 else kvg.KVG_KV_BF16
        scale = 0.0625 if fp8 else 1.0  # of the E4M3 codes: keys and values of a few units
        dims = kvg.make_dims(s.layers, s.kv_heads, s.head_dim, s.page, s.theta, kvg.KVG_ROPE_HALF, kind, scale, scale)
        block_pages, own_pages = -(-len(document) // s.page), -(-most_rows // s.page) + 1
        # the document's pages twice: while it is read, and as the stored block
        self.cache = kvg.Cache(dims, 2 * block_pages + batch * own_pages, batch + 1,
                               (block_pages + own_pages) * s.page)
        self.store = kvg.PoolStore(self.cache, block_pages * self.cache.view.page_bytes * 2 * s.layers + (1 << 20))
        self.rotary = kvg.Rotary(s.head_dim, s.head_dim, s.theta, kvg.KVG_ROPE_HALF)
        self.rows = [0] * batch

        reader = batch
        self._forward(document, [reader], [len(document)], [0])
        self.block = kvg.kvg_deposit(self.store.h, self.cache.h, reader, 0, len(document))
        kvg.kvg_cache_release(self.cache.h, reader)
        for b in range(batch):
            kvg.kvg_graft(self.store.h, self.block, self.cache.h, b)
            self.rows[b] = len(document)

    def _forward(self, tokens, seqs, n_rows, past, step=False):
        """Hidden states of n_rows new tokens per sequence, behind `past` rows each."""
        s, device = self.model.shape, tokens.device
        if step:
            positions = torch.tensor(past, dtype=torch.int32).to(device)
        else:
            positions = torch.cat([torch.arange(p, p + n, dtype=torch.int32) for p, n in zip(past, n_rows)]).to(device)
        out = torch.empty(len(tokens), s.q_heads, s.head_dim, dtype=torch.bfloat16, device=device)
        queries, scale = torch.empty_like(out), 1 / math.sqrt(s.head_dim)

        def attention(layer, w, q, k, v):
            qkv = kvg.make_qkv(q, k, v, w["q_norm"], w["k_norm"], EPS)
            kvg.kvg_cache_append_qkv(self.cache.h, layer, seqs, n_rows, qkv, self.rotary.h, positions.data_ptr(),
                                     queries.data_ptr())
            if step:
                kvg.kvg_decode_attention_shared(self.cache.h, layer, seqs, queries.data_ptr(), s.q_heads,
                                                out.data_ptr(), scale)
            else:
                kvg.kvg_prompt_attention(self.cache.h, layer, seqs, n_rows, queries.data_ptr(), s.q_heads,
                                         out.data_ptr(), scale)
            return out.view(len(tokens), -1)

        return self.model(tokens, attention)

    def ask(self, questions):
        """Reads each conversation's tokens (a list of tensors, some may be empty); hidden states, packed."""
        n_rows = [len(q) for q in questions]
        x = self._forward(torch.cat(questions), list(range(self.batch)), n_rows, self.rows)
        self.rows = [r + n for r, n in zip(self.rows, n_rows)]
        return x

    def step(self, tokens):
        """One token of each conversation; hidden states [batch][width]."""
        x = self._forward(tokens, list(range(self.batch)), [1] * self.batch, self.rows, step=True)
        self.rows = [r + 1 for r in self.rows]
        return x

    def check(self):
        """Raises what a kernel reported."""
        kvg.kvg_sync(self.cache.h)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--document", type=int, default=8192, help="tokens")
    ap.add_argument("--conversations", type=int, default=32)
    ap.add_argument("--steps", type=int, default=32, help="answered tokens")
    ap.add_argument("--fp8", action="store_true", help="E4M3 cache")
    a = ap.parse_args()
    shape = Shape()
    model = Decoder(shape)
    g = torch.Generator().manual_seed(1)

    def draw(n):
        return torch.randint(shape.tokens, (n,), generator=g).cuda()

    events = [torch.cuda.Event(enable_timing=True) for _ in range(4)]
    questions = [draw(17 + 13 * b % 101) for b in range(a.conversations)]
    document = draw(a.document)
    for timed in (False, True):  # the first pass warms up
        launches = kvg.kvg_launch_count()
        events[0].record()
        talk = Conversations(model, document, a.conversations, 128 + a.steps, a.fp8)
        events[1].record()
        x = talk.ask(questions)
        ends = torch.tensor([len(q) for q in questions]).cumsum(0) - 1
        token = model.logits(x[ends.cuda()]).argmax(-1)
        events[2].record()
        for _ in range(a.steps):
            token = model.logits(talk.step(token)).argmax(-1)
        events[3].record()
        talk.check()
    ms = [events[i].elapsed_time(events[i + 1]) for i in range(3)]
    print(f"document of {a.document} tokens read and stored: {ms[0]:.2f} ms")
    print(f"{sum(len(q) for q in questions)} tokens of {a.conversations} questions on it: {ms[1]:.2f} ms")
    print(f"{a.steps} steps of {a.conversations} tokens: {ms[2] / a.steps:.3f} ms each")
    print(f"{kvg.kvg_launch_count() - launches} launches of the library's kernels")


if __name__ == "__main__":
    main()
