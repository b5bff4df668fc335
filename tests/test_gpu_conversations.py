"""The example of conversations on one stored document against the same decoder
in 64 bits, each conversation read from its first token on.

Bounds, on a token's hidden state relative to its norm: some 13 roundings to
bf16 a layer (both norms, projections, rotated heads, softmax weights,
attention, activations, residual), each 2^-9 / sqrt(3) = 0.0011 rms of a branch
that is no longer than the state; three layers in quadrature 0.007, at most
doubled by the scores' errors and tripled for the worst of some hundred tokens:
0.04.  E4M3 rows add half a step of 2^-4 at most (rms 0.026 of a key or value)
to the attention's branch: 0.1."""
import math
import os

import pytest
import torch
import torch.nn.functional as F

os.environ.setdefault("KVG_SHARED_MIN_KB", "1")  # small batches read their common pages together too

from examples import conversations as ex
from kvg_testlib import need_gpu

SHAPE = ex.Shape(layers=3, q_heads=4, kv_heads=2, head_dim=64, width=128, hidden=192, tokens=500, theta=1e4, page=16)
FP8 = ex.Shape(**{**vars(SHAPE), "head_dim": 128})  # (E4M3 decode needs heads of 128 or 256)
LENGTHS = [3, 0, 17, 1, 40]


def plain(model, tokens, shift=0):
    """The decoder over one conversation's tokens in 64 bits; the mistake of positions from `shift` on starting
    over is planted by shift > 0."""
    s, n, d = model.shape, len(tokens), model.shape.head_dim
    x = model.embed.double()[tokens]
    pos = torch.arange(n, device=tokens.device)
    if shift:
        pos = torch.where(pos < shift, pos, pos - shift)
    angle = pos[:, None, None] * s.theta ** (-torch.arange(0, d, 2, device=tokens.device).double() / d)

    def norm(x, w=None):
        y = x / (x.square().mean(-1, keepdim=True) + ex.EPS).sqrt()
        return y if w is None else y * w.double()

    def rotate(x):
        a, b = x.chunk(2, dim=-1)
        return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)

    for w in model.layers:
        heads = F.linear(norm(x), w["qkv"].double()).view(n, -1, d)
        q, k, v = heads.split([s.q_heads, s.kv_heads, s.kv_heads], dim=1)
        q, k = rotate(norm(q, w["q_norm"])), rotate(norm(k, w["k_norm"]))
        k, v = (t.repeat_interleave(s.q_heads // s.kv_heads, dim=1) for t in (k, v))
        scores = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(d)
        later = torch.ones(n, n, dtype=torch.bool, device=tokens.device).triu(1)
        o = torch.einsum("hij,jhd->ihd", scores.masked_fill(later, -math.inf).softmax(-1), v)
        x = x + F.linear(o.reshape(n, -1), w["o"].double())
        gate, up = F.linear(norm(x), w["up"].double()).chunk(2, dim=-1)
        x = x + F.linear(F.silu(gate) * up, w["down"].double())
    return x


def worst(x, ref):
    return ((x.double() - ref).norm(dim=-1) / ref.norm(dim=-1)).max().item()


def test_the_bound_tells_a_mistake():
    """The same decoder in bf16 keeps the bound; positions that start over behind the document do not."""
    model = ex.Decoder(SHAPE, device="cpu")
    tokens = torch.randint(SHAPE.tokens, (120,), generator=torch.Generator().manual_seed(2))
    ref = plain(model, tokens)

    def attention(i, w, q, k, v):
        n, d = len(q), SHAPE.head_dim
        angle = torch.arange(n)[:, None, None] * SHAPE.theta ** (-torch.arange(0, d, 2) / d)

        def rotate(x, w):
            a, b = F.rms_norm(x.float(), (d,), w.float(), ex.EPS).chunk(2, dim=-1)
            return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1).to(x.dtype)

        q, k = rotate(q, w["q_norm"]), rotate(k, w["k_norm"])
        q, k, v = (t.transpose(0, 1) for t in (q, k, v))
        o = F.scaled_dot_product_attention(q, k, v, is_causal=True, enable_gqa=True)
        return o.transpose(0, 1).reshape(n, -1)

    assert worst(model(tokens, attention), ref) < 0.04
    assert worst(plain(model, tokens, 100)[100:], ref[100:]) > 0.1


@pytest.mark.gpu
@pytest.mark.parametrize("document", [1, 96, 203])
@pytest.mark.parametrize("fp8", [False, True])
def test_conversations_match_the_plain_decoder(document, fp8):
    need_gpu()
    model = ex.Decoder(FP8 if fp8 else SHAPE)
    g = torch.Generator().manual_seed(document)

    def draw(n):
        return torch.randint(SHAPE.tokens, (n,), generator=g).cuda()

    text, questions = draw(document), [draw(n) for n in LENGTHS]
    talk = ex.Conversations(model, text, len(LENGTHS), 64, fp8)
    answers = [draw(len(LENGTHS)) for _ in range(3)]
    got = list(talk.ask(questions).split(LENGTHS))
    for a in answers:
        got = [torch.cat([x, y[None]]) for x, y in zip(got, talk.step(a))]
    talk.check()
    for b, x in enumerate(got):
        tokens = torch.cat([text, questions[b]] + [a[b:b + 1] for a in answers])
        assert worst(x, plain(model, tokens)[document:]) < (0.1 if fp8 else 0.04), b
