"""Operators of contexts that hold more than text, as measured work: a plain form
of each in elementary torch operations, and the calls a user makes of the library.

  axes     new tokens' projections become cache rows, as with the library's
           rotary positions, but a token has a position on each of several axes
           (time, height, width): the pairs of a head are shared out among the
           axes, in sections or in turn, on one ladder of frequencies or with a
           ladder to each axis.  The measured call writes one layer of rows
           that are already open, as each layer of a model but the first does.
  cross    attention of packed decoder rows to the states of an encoder, whose
           keys and values lie in the paged cache: each row attends to every row
           of its sequence's states, whatever their number.
  weights  attention of the last rows of each sequence (one token, or a prompt)
           that also returns what weight each cached row received, summed over
           heads, layers and query rows.
  evict    a sequence's rows thinned to a number of them: the first few, the
           last ones and the heaviest in between, in their old order, with their
           positions and weights.  The thinned copy goes to another sequence;
           the full one stays for other conversations.

Geometries are those of the repository's workloads (kvg_synth.py).  Rows and
queries are N(0, 1) draws rounded to bf16; fp8 caches use its per-tensor scale.

The library keeps rows behind a cache handle and the plain forms keep them in
torch tensors, so prepare() fills one or the other from the same draws.
"""
from __future__ import annotations

import math
import random

import torch

own = False

# query heads, kv heads, head_dim, page size, RoPE base
MODELS = {
    "tiny": (4, 2, 64, 16, 1e4),
    "12b": (16, 8, 256, 64, 1e4),
    "31b": (32, 16, 128, 64, 1e6),
}
FP8_SCALE = 0.0625  # per-tensor K and V scale of the fp8 caches
EPS = 1e-6          # of the root mean square norm


def listed():
    return [
        # one token of one conversation about an image: latency and launches count
        {"name": "axes_step_1", "kind": "axes", "model": "31b", "batch": 1, "rows_lo": 1, "rows_hi": 1,
         "past_lo": 2110, "past_hi": 2110, "norm": True, "rotary": 128, "style": "half", "axes": 3,
         "layout": "sections"},
        # packed prompts of text and images, into an fp8 cache, pairs given to the axes in turn
        {"name": "axes_images_fp8", "kind": "axes", "model": "12b", "fp8": True, "batch": 5, "rows_lo": 3,
         "rows_hi": 901, "past_lo": 0, "past_hi": 700, "norm": True, "rotary": 256, "style": "half", "axes": 3,
         "layout": "turns", "fused": True},
        # a video's frames (an odd number of rows) in one prompt
        {"name": "axes_video_12b", "kind": "axes", "model": "12b", "batch": 1, "rows_lo": 8191, "rows_hi": 8191,
         "past_lo": 64, "past_hi": 64, "norm": True, "rotary": 256, "style": "half", "axes": 3,
         "layout": "sections", "fused": True},
        # a short prompt on a few states
        {"name": "cross_tiny", "kind": "cross", "model": "tiny", "layers": 1, "batch": 1, "rows_lo": 37,
         "rows_hi": 37, "states_lo": 250, "states_hi": 250},
        # a few candidate tokens of each of 24 conversations, on states of different lengths
        {"name": "cross_candidates_12b", "kind": "cross", "model": "12b", "layers": 1, "batch": 24, "rows_lo": 2,
         "rows_hi": 5, "states_lo": 257, "states_hi": 4099},
        # packed prompts on states of different lengths in an fp8 cache
        {"name": "cross_packed_fp8", "kind": "cross", "model": "31b", "fp8": True, "layers": 1, "batch": 11,
         "rows_lo": 1, "rows_hi": 803, "states_lo": 1, "states_hi": 2501},
        # a long text on a long recording's states
        {"name": "cross_long_31b", "kind": "cross", "model": "31b", "layers": 1, "batch": 1, "rows_lo": 8191,
         "rows_hi": 8191, "states_lo": 12001, "states_hi": 12001},
        # a token of one conversation
        {"name": "weights_step_1", "kind": "weights", "model": "31b", "layers": 1, "batch": 1, "rows_lo": 1,
         "rows_hi": 1, "past_lo": 2110, "past_hi": 2110},
        # a decode step of a batch, two layers in a call
        {"name": "weights_step_b16", "kind": "weights", "model": "12b", "layers": 2, "batch": 16, "rows_lo": 1,
         "rows_hi": 1, "past_lo": 1201, "past_hi": 8192},
        # a question, or a document's next part, on a context whose rows it weighs
        {"name": "weights_prompt_12b", "kind": "weights", "model": "12b", "layers": 1, "batch": 1, "rows_lo": 2047,
         "rows_hi": 2047, "past_lo": 6145, "past_hi": 6145},
        # the smallest fixture's block and what was said on it
        {"name": "evict_tiny", "kind": "evict", "model": "tiny", "layers": 2, "batch": 1, "rows_lo": 293,
         "rows_hi": 293, "keep": 131, "first": 4, "last": 32},
        # long conversations, four layers of them, down to a budget
        {"name": "evict_12b", "kind": "evict", "model": "12b", "layers": 4, "batch": 3, "rows_lo": 5003,
         "rows_hi": 16384, "keep": 4097, "first": 4, "last": 512},
    ]


def _size(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]; odd ones as often as even."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["axes", "cross", "weights", "evict"])
    model = rng.choice(["tiny", "12b", "31b", "12b", "31b"])
    hq, hkv, d, page, _ = MODELS[model]
    case = {"kind": kind, "model": model}
    if rng.random() < 0.25:
        case["page"] = page = rng.choice([16, 24, 32, 48, 80, 128])
    if model != "tiny" and rng.random() < 0.35:
        case["fp8"] = True
    if kind == "axes":
        case["batch"] = batch = _size(rng, 1, 64)
        hi = _size(rng, 1, 8191 // batch) if rng.random() < 0.7 else 1
        case["rows_lo"], case["rows_hi"] = max(1, int(hi * rng.random())), hi
        case["past_hi"] = _size(rng, 1, 2900) - 1
        case["past_lo"] = int(case["past_hi"] * rng.random())
        case["norm"] = rng.random() < 0.6
        case["rotary"] = rng.choice([d, d, d // 2])
        case["style"] = rng.choice(["half", "half", "interleaved"])
        case["axes"] = rng.choice([2, 3, 3, 4])
        case["layout"] = rng.choice(["sections", "turns", "own"])
        case["fused"] = rng.random() < 0.5
        return case
    if kind == "evict":
        case["layers"] = rng.choice([1, 2, 3, 4])
        case["batch"] = batch = _size(rng, 1, 8)
        case["rows_hi"] = hi = _size(rng, 30, 32768 // batch)
        case["rows_lo"] = max(1, int(hi * rng.random()))
        case["keep"] = keep = _size(rng, 12, max(13, min(hi, 12000 // batch)))
        case["first"], case["last"] = rng.randrange(5), int((keep - 5) * rng.random())
        return case
    case["layers"] = rng.choice([1, 1, 2])
    case["batch"] = batch = _size(rng, 1, 40)
    if kind == "cross":
        states = _size(rng, 1, 12001)
        hi = _size(rng, 1, 4096) if rng.random() < 0.6 else rng.randrange(1, 9)
        while (case["layers"] * batch * hi * states * hq > 1.5e9
               or case["layers"] * batch * d * (hkv * states + hq * hi) > 2.5e8):
            hi, batch, states = max(1, hi * 2 // 3), max(1, batch - batch // 3), max(1, states * 3 // 4)
        case["batch"] = batch
        case["rows_lo"], case["rows_hi"] = max(1, int(hi * rng.random())), hi
        case["states_lo"], case["states_hi"] = max(1, int(states * rng.random())), states
        return case
    total = _size(rng, 40, 16000)  # rows of a sequence, restored ones included
    hi = 1 if rng.random() < 0.5 else _size(rng, 1, min(total, 3000))
    while (case["layers"] * batch * hi * total * hq > 4e8
           or case["layers"] * batch * d * (hkv * total + hq * hi) > 2.5e8):
        hi, batch, total = max(1, hi // 2), max(1, batch - batch // 3), max(hi, total * 3 // 4)
    case["batch"] = batch
    case["rows_lo"], case["rows_hi"] = max(1, int(hi * rng.random())), hi
    case["past_hi"] = total - hi
    case["past_lo"] = int(case["past_hi"] * rng.random())
    if rng.random() < 0.25:
        case["window"] = _size(rng, 64, 4096)
    return case


# ------------------------------------------------------------- geometry --

def _geo(case):
    hq, hkv, d, page, theta = MODELS[case["model"]]
    return hq, hkv, d, int(case.get("page", page)), theta


def _spread(lo, hi, n, step):
    """n lengths spread evenly over [lo, hi], in an order mixed by `step`."""
    return [hi] if n == 1 else [lo + (hi - lo) * ((i * step) % n) // (n - 1) for i in range(n)]


def _rows(case):
    return _spread(case["rows_lo"], case["rows_hi"], case["batch"], 7919)


def _past(case):
    if case["kind"] == "cross":
        return _spread(case["states_lo"], case["states_hi"], case["batch"], 104729)
    return _spread(case["past_lo"], case["past_hi"], case["batch"], 104729)


def _context(case):
    """Rows that each sequence has in the cache when its query rows attend."""
    return _past(case) if case["kind"] == "cross" else [p + n for p, n in zip(_past(case), _rows(case))]


def _draws(seed, device="cuda"):
    """Generator of N(0, 1) draws rounded to bf16, the same for the same seed."""
    g = torch.Generator(device=device)
    g.manual_seed(int(seed))
    return lambda *shape: torch.randn(shape, generator=g, device=device).to(torch.bfloat16)


def _sections(case):
    """Pairs of each axis: less for the first (time) of three or four; in turn, an
    axis but the first has no more than its turns."""
    pairs, n = case["rotary"] // 2, case["axes"]
    other = pairs // 2 if n == 2 else pairs * 5 // 16 if n == 3 else pairs // 4
    if case["layout"] == "turns":
        other = min(other, (pairs - n + 1) // n)
    return [pairs - other * (n - 1)] + [other] * (n - 1)


def _axis_of_pairs(case):
    """The axis of each pair, and its place on the ladder of frequencies with the ladder's length."""
    sections, n = _sections(case), case["axes"]
    pairs = sum(sections)
    if case["layout"] == "turns":
        axis = [i % n if i // n < sections[i % n] else 0 for i in range(pairs)]
    else:
        axis = [a for a, s in enumerate(sections) for _ in range(s)]
    if case["layout"] == "own":
        return axis, [j for s in sections for j in range(s)], [s for s in sections for _ in range(s)]
    return axis, list(range(pairs)), [pairs] * pairs


def _places(case, seed):
    """Positions [axes][T] of packed rows: runs of text, whose positions are the same on
    every axis, and images or frames, grids on the axes but the first."""
    rng, n = random.Random(seed), case["axes"]
    columns = []
    for past, rows in zip(_past(case), _rows(case)):
        at, left = past, rows
        while left > 0:
            run = min(left, rng.randrange(1, 60))
            columns += [[t] * n for t in range(at, at + run)]
            at, left = at + run, left - run
            high, wide = rng.randrange(8, 40), rng.randrange(8, 40)
            grid = [[at, at + h, at + w, at + (h ^ w)][:n] for h in range(high) for w in range(wide)][:left]
            columns += grid
            at, left = at + max(high, wide), left - len(grid)
    return torch.tensor(columns, dtype=torch.int32).T.contiguous().cuda()


def _axes_inputs(case, seed):
    hq, hkv, d, _, _ = _geo(case)
    t = sum(_rows(case))
    draws = _draws(seed)
    if case.get("fused"):  # one projection's output, queries, keys and values side by side
        q, k, v = draws(t, hq + 2 * hkv, d).split([hq, hkv, hkv], dim=1)
    else:
        q, k, v = draws(t, hq, d), draws(t, hkv, d), draws(t, hkv, d)
    wq = wk = None
    if case["norm"]:
        wq, wk = ((1 + 0.1 * draws(d).float()).to(torch.bfloat16) for _ in range(2))
    return q, k, v, wq, wk, _places(case, seed)


def _attention_inputs(case, seed):
    """Queries of the packed rows, and keys and values of every row, sequence after sequence."""
    hq, hkv, d, _, _ = _geo(case)
    draws = _draws(seed)
    n_l, n = case["layers"], sum(_context(case))
    return draws(n_l, sum(_rows(case)), hq, d), draws(n_l, n, hkv, d), draws(n_l, n, hkv, d)


def _evict_inputs(case, seed):
    """Keys and values of every row, and its weight: many light rows, few heavy ones, some of none at all."""
    hq, hkv, d, _, _ = _geo(case)
    draws = _draws(seed)
    n_l, n = case["layers"], sum(_rows(case))
    weight = torch.exp(2 * draws(n).float()) * (draws(n) > -1.5)
    return draws(n_l, n, hkv, d), draws(n_l, n, hkv, d), weight


def _stored(case, x):
    """Rows as the cache holds them: E4M3 codes of x / scale in an fp8 cache."""
    return (x.float() / FP8_SCALE).to(torch.float8_e4m3fn) if case.get("fp8") else x


def _bits(x):
    """E4M3 codes as bytes, which every kind of indexing takes."""
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _pages(total, page):
    """First page of each sequence, and the pages in all, when sequences take pages in turn."""
    need = [-(-n // page) for n in total]
    return [sum(need[:i]) for i in range(len(need))], sum(need)


# -------------------------------------------------------------- prepare --

def _kind(case):
    return torch.float8_e4m3fn if case.get("fp8") else torch.bfloat16


class _Memory:
    """Device memory of the library as a torch tensor, which keeps its owner alive."""

    def __init__(self, owner, ptr, n):
        self.owner = owner
        self.__cuda_array_interface__ = {"shape": (n,), "typestr": "|u1", "data": (int(ptr), False), "version": 3}


def _cache(case, layers, seqs, slots, n_pages):
    """A cache, its pool zeroed and as a tensor."""
    from paper_2607_14431_gb300 import kvg
    hq, hkv, d, page, theta = _geo(case)
    dims = kvg.make_dims(layers, hkv, d, page, theta,
                         kvg.KVG_ROPE_INTERLEAVED if case.get("style") == "interleaved" else kvg.KVG_ROPE_HALF,
                         kvg.KVG_KV_E4M3 if case.get("fp8") else kvg.KVG_KV_BF16, FP8_SCALE, FP8_SCALE)
    cache = kvg.Cache(dims, n_pages, seqs, slots)
    pool = torch.as_tensor(_Memory(cache, cache.view.pool, cache.view.pool_bytes), device="cuda")
    pool.zero_()
    return kvg, cache, pool.view(_kind(case)).view(layers, 2, -1, hkv, page, d)


def _fill(kvg, cache, seq, k, v):
    """Appends rows k, v [L][n][Hkv][D] of an empty sequence, at positions from 0."""
    n = k.shape[1]
    if n:
        k, v = k.contiguous(), v.contiguous()
        pos = torch.arange(n, dtype=torch.int32, device="cuda")
        kvg.kvg_cache_append(cache.h, seq, k.data_ptr(), v.data_ptr(), pos.data_ptr(), n)
        torch.cuda.synchronize()


def _prepare_axes(case, seed):
    hq, hkv, d, page, theta = _geo(case)
    rows, past = _rows(case), _past(case)
    q, k, v, wq, wk, places = _axes_inputs(case, seed)
    total = [p + n for p, n in zip(past, rows)]
    first, n_pages = _pages(total, page)
    s = {"q": q, "k": k, "v": v, "wq": wq, "wk": wk, "places": places, "q_out": torch.empty_like(q.contiguous())}
    if own:
        kvg, cache, pool = _cache(case, 2, len(total), max(total), n_pages)
        # pages in the order in which the rows below ask for them, so that each lands where the plain form's does
        had = [-(-p // page) for p in past]
        kvg.kvg_cache_set_free_order(
            cache.h, [f + j for f, h in zip(first, had) for j in range(h)]
            + [f + j for f, h, n in zip(first, had, total) for j in range(h, -(-n // page))])
        for b, p in enumerate(past):
            zero = torch.zeros(2, p, hkv, d, dtype=torch.bfloat16, device="cuda")
            _fill(kvg, cache, b, zero, zero)
        layout = {"sections": kvg.KVG_ROPE_AXES_SECTIONS, "turns": kvg.KVG_ROPE_AXES_TURNS,
                  "own": kvg.KVG_ROPE_AXES_OWN}[case["layout"]]
        rotary = kvg.Rotary(d, case["rotary"], theta, cache.dims.rope_style, sections=_sections(case), layout=layout)
        qkv = kvg.make_qkv(q, k, v, q_norm=wq, k_norm=wk, eps=EPS)
        s |= {"kvg": kvg, "cache": cache, "pool": pool[1], "rotary": rotary, "qkv": qkv, "rows": rows,
              "seqs": list(range(len(rows)))}
        # layer 0 opens the rows; run() writes layer 1 of them
        kvg.kvg_cache_append_qkv(cache.h, 0, s["seqs"], rows, qkv, rotary.h, places.data_ptr(), s["q_out"].data_ptr())
        torch.cuda.synchronize()
        return s
    s["pool"] = torch.zeros(2, n_pages, hkv, page, d, dtype=torch.bfloat16, device="cuda").to(_kind(case))
    slots = torch.cat([torch.arange(p, p + n) + f * page for f, p, n in zip(first, past, rows)]).cuda()
    s |= {"page": slots // page, "row": slots % page}
    axis, place, ladder = (torch.tensor(x, dtype=torch.float64) for x in _axis_of_pairs(case))
    s |= {"axis": axis.long().cuda(), "freq": (theta ** (-place / ladder)).cuda()}
    return s


def _prepare_attention(case, seed):
    """Queries, and a cache that holds the sequences' rows."""
    hq, hkv, d, page, _ = _geo(case)
    rows, total = _rows(case), _context(case)
    q, k, v = _attention_inputs(case, seed)
    n_l = case["layers"]
    s = {"q": q, "out": torch.empty_like(q), "scale": 1 / math.sqrt(d), "layer": -1 if n_l > 1 else 0,
         "weights": torch.zeros(len(total), max(total), device="cuda")}
    if own:
        kvg, cache, _ = _cache(case, n_l, len(total), max(total), _pages(total, page)[1])
        if case.get("window"):
            kvg.kvg_cache_set_layer_windows(cache.h, [case["window"]] * n_l)
        at = 0
        for b, n in enumerate(total):
            _fill(kvg, cache, b, k[:, at:at + n], v[:, at:at + n])
            at += n
        s |= {"kvg": kvg, "cache": cache, "rows": rows, "seqs": list(range(len(rows)))}
        return s
    first, n_pages = _pages(total, page)
    pool = torch.zeros(n_l, 2, n_pages * page, hkv, d, dtype=torch.bfloat16, device="cuda")
    slots = torch.cat([torch.arange(n) + f * page for f, n in zip(first, total)]).cuda()
    pool[:, 0, slots], pool[:, 1, slots] = k, v
    pool = _stored(case, pool).view(n_l, 2, n_pages, page, hkv, d).transpose(3, 4).contiguous()
    most = -(-max(total) // page)
    table = torch.tensor([[f + min(j, -(-n // page) - 1) for j in range(most)] for f, n in zip(first, total)])
    # where a packed query row sits in the padded batch
    b_of = torch.cat([torch.full((n,), b) for b, n in enumerate(rows)]).cuda()
    t_of = torch.cat([torch.arange(n) for n in rows]).cuda()
    s |= {"pool": pool, "table": table.cuda(), "b_of": b_of, "t_of": t_of, "most_rows": max(rows),
          "total": torch.tensor(total, device="cuda"), "n_rows": torch.tensor(rows, device="cuda")}
    return s


def _prepare_evict(case, seed):
    """Sequences 0 .. B - 1 hold the rows, B .. 2B - 1 get the thinned copies, in pages behind theirs."""
    hq, hkv, d, page, _ = _geo(case)
    rows = _rows(case)
    keep = [min(n, case["keep"]) for n in rows]
    k, v, weight = _evict_inputs(case, seed)
    batch, n_l, slots = len(rows), case["layers"], max(rows)
    weights = torch.zeros(2 * batch, slots, device="cuda")
    at = 0
    for b, n in enumerate(rows):
        weights[b, :n] = weight[at:at + n]
        at += n
    first, n_pages = _pages(rows + keep, page)
    s = {"weights": weights, "keep": keep, "first": first}
    if own:
        kvg, cache, pool = _cache(case, n_l, 2 * batch, slots, n_pages)
        at = 0
        for b, n in enumerate(rows):
            _fill(kvg, cache, b, k[:, at:at + n], v[:, at:at + n])
            at += n
        positions = torch.as_tensor(_Memory(cache, cache.view.positions, 8 * batch * slots), device="cuda")
        s |= {"kvg": kvg, "cache": cache, "pool": pool, "positions": positions.view(torch.int32).view(2 * batch, slots),
              "from": list(range(batch)), "to": list(range(batch, 2 * batch)), "rows": [case["keep"]] * batch}
        return s
    pool = torch.zeros(n_l, 2, n_pages * page, hkv, d, dtype=torch.bfloat16, device="cuda")
    at = torch.cat([torch.arange(n) + f * page for f, n in zip(first, rows)]).cuda()
    pool[:, 0, at], pool[:, 1, at] = k, v
    s["pool"] = _stored(case, pool).view(n_l, 2, n_pages, page, hkv, d).transpose(3, 4).contiguous()
    s["positions"] = torch.full((2 * batch, slots), -1, dtype=torch.int32, device="cuda")
    for b, n in enumerate(rows):
        s["positions"][b, :n] = torch.arange(n)
    return s


def prepare(case, seed):
    s = {"axes": _prepare_axes, "cross": _prepare_attention, "weights": _prepare_attention,
         "evict": _prepare_evict}[case["kind"]](case, seed)
    s["case"] = case
    return s


# ------------------------------------------------------------------ run --

def _normed(x, w):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()


def _rotated(x, cos, sin, interleaved):
    r = 2 * cos.shape[-1]
    cos, sin, turn, rest = cos[:, None], sin[:, None], x[..., :r], x[..., r:]
    if interleaved:
        a, b = turn[..., 0::2], turn[..., 1::2]
        turn = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = turn[..., : r // 2], turn[..., r // 2:]
        turn = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turn, rest], -1)


def _plain_axes(s):
    case = s["case"]
    q, k = s["q"].float(), s["k"].float()
    if case["norm"]:
        q, k = _normed(q, s["wq"]), _normed(k, s["wk"])
    angle = s["places"].T[:, s["axis"]].double() * s["freq"]
    cos, sin = angle.cos().float(), angle.sin().float()
    q, k = (_rotated(x, cos, sin, case["style"] == "interleaved") for x in (q, k))
    k = _stored(case, k) if case.get("fp8") else k.to(torch.bfloat16)
    pool, at = _bits(s["pool"]), (s["page"], slice(None), s["row"])
    pool[(0, *at)], pool[(1, *at)] = _bits(k), _bits(_stored(case, s["v"]))
    return q.to(torch.bfloat16), s["pool"]


def _plain_attention(s):
    """One layer after the other, the batch padded to its longest rows and context."""
    case = s["case"]
    hq, hkv, d, page, _ = _geo(case)
    g, scale = hq // hkv, FP8_SCALE if case.get("fp8") else 1.0
    batch, pages = s["table"].shape
    n, columns = s["most_rows"], pages * page
    column = torch.arange(columns, device="cuda")
    last = s["total"][:, None] - 1
    if case["kind"] == "weights":  # own row of each query: the sequence's last ones
        last = last - s["n_rows"][:, None] + 1 + torch.arange(n, device="cuda")
    mask = column <= last[..., None]
    if case.get("window"):
        mask &= column > last[..., None] - case["window"]
    outs, weights = [], torch.zeros(batch, columns, device="cuda")
    for l in range(case["layers"]):
        kv = _bits(s["pool"])[l][:, s["table"]].view(s["pool"].dtype).float() * scale  # [2][B][pages][Hkv][P][D]
        k, v = kv.transpose(3, 4).reshape(2, batch, columns, hkv, d).transpose(2, 3)
        q = torch.zeros(batch, n, hq, d, device="cuda")
        q[s["b_of"], s["t_of"]] = s["q"][l].float()
        q = q.view(batch, n, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(batch, hkv, g * n, d)
        x = torch.matmul(q * s["scale"], k.transpose(-1, -2)).view(batch, hkv, g, n, columns)
        x.masked_fill_(~mask[:, None, None], -math.inf)
        x = x.sub_(x.amax(-1, keepdim=True)).exp_()
        x /= x.sum(-1, keepdim=True)
        out = torch.matmul(x, v[:, :, None]).permute(0, 3, 1, 2, 4).reshape(batch, n, hq, d)
        outs.append(out[s["b_of"], s["t_of"]].to(torch.bfloat16))
        if case["kind"] == "weights":
            seen = torch.arange(n, device="cuda") < s["n_rows"][:, None]  # not the padding's rows
            weights += x.sum((1, 2)).masked_fill_(~seen[..., None], 0).sum(1)
    out = torch.stack(outs)
    return out if case["kind"] == "cross" else (out, weights[:, :s["weights"].shape[1]])


def _plain_evict(s):
    case = s["case"]
    page = s["pool"].shape[4]
    pool, rows, batch = _bits(s["pool"]), _rows(case), case["batch"]
    for b, (n, keep) in enumerate(zip(rows, s["keep"])):
        weight = s["weights"][b, :n].clone()
        if n > keep:
            weight[:case["first"]] = math.inf
            weight[n - case["last"]:] = math.inf
        kept = torch.argsort(weight, descending=True, stable=True)[:keep].sort().values
        to = torch.arange(keep, device="cuda")
        src, dst = kept + s["first"][b] * page, to + s["first"][batch + b] * page
        pool[:, :, dst // page, :, dst % page] = pool[:, :, src // page, :, src % page]
        s["positions"][batch + b, :keep] = s["positions"][b, kept]
        s["weights"][batch + b, :keep] = s["weights"][b, kept]
    return s["pool"][:, :, s["first"][batch]:], s["positions"][batch:], s["weights"][batch:]


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        return {"axes": _plain_axes, "cross": _plain_attention, "weights": _plain_attention,
                "evict": _plain_evict}[kind](s)
    kvg, cache = s["kvg"], s["cache"]
    if kind == "axes":
        kvg.kvg_cache_append_qkv(cache.h, 1, s["seqs"], s["rows"], s["qkv"], s["rotary"].h, s["places"].data_ptr(),
                                 s["q_out"].data_ptr())
        return s["q_out"], s["pool"]
    if kind == "evict":
        kvg.kvg_cache_evict(cache.h, s["from"], s["rows"], case["first"], case["last"], s["weights"].data_ptr(),
                            dst_ids=s["to"])
        batch = case["batch"]
        return s["pool"][:, :, s["first"][batch]:], s["positions"][batch:], s["weights"][batch:]
    hq = s["q"].shape[-2]
    if kind == "cross":
        kvg.kvg_cross_attention(cache.h, s["layer"], s["seqs"], s["rows"], s["q"].data_ptr(), hq, s["out"].data_ptr(),
                                s["scale"])
        return s["out"]
    # (decay 0: the weights of this call alone)
    kvg.kvg_attention_weights(cache.h, s["layer"], s["seqs"], s["rows"], s["q"].data_ptr(), hq, s["out"].data_ptr(),
                              s["scale"], s["weights"].data_ptr(), 0.0)
    return s["out"], s["weights"]


# ----------------------------------------------------------------- work --

def _visible(case):
    """(query row, cached row) pairs that attend, and cached rows that any query reads."""
    pairs = read = 0
    w = case.get("window") or 1 << 60
    for n, p in zip(_rows(case), _past(case)):
        if case["kind"] == "cross":
            pairs, read = pairs + n * p, read + p
            continue
        short = max(0, min(n, w - p - 1))  # queries that see fewer rows than the window
        pairs += short * p + short * (short + 1) // 2 + (n - short) * min(w, p + n)
        read += min(p + n, w + n - 1)
    return pairs, read


def work(case):
    hq, hkv, d, page, _ = _geo(case)
    e = 1 if case.get("fp8") else 2
    if case["kind"] == "axes":
        t = sum(_rows(case))
        return {"bytes": t * (d * (2 * (hq + 2 * hkv) + 2 * hq + 2 * hkv * e) + 4 * case["axes"]),
                "flops": t * d * 8 * (hq + hkv)}
    n_l = case["layers"]
    if case["kind"] == "evict":
        n, kept = sum(_rows(case)), sum(min(x, case["keep"]) for x in _rows(case))
        # each weight once, and of the kept rows keys, values, positions and weights read and written
        return {"bytes": 4 * n + kept * (2 * n_l * 2 * hkv * d * e + 12), "flops": n}
    pairs, read = _visible(case)
    extra = 4 * sum(_context(case)) if case["kind"] == "weights" else 0
    return {"bytes": n_l * (read * hkv * d * 2 * e + sum(_rows(case)) * hq * d * 4) + extra,
            "flops": n_l * 4 * hq * d * pairs}


# ---------------------------------------------------------------- exact --

def _exact_axes(case, seed):
    hq, hkv, d, page, theta = _geo(case)
    q, k, v, wq, wk, places = _axes_inputs(case, seed)
    r, n, sections = case["rotary"], case["axes"], _sections(case)
    # pair by pair: its axis, and its frequency
    axis, f = [], []
    if case["layout"] == "own":
        for a in range(n):
            axis += [a] * sections[a]
            f += [math.exp(-j / sections[a] * math.log(theta)) for j in range(sections[a])]
    else:
        f = [math.exp(-2 * i / r * math.log(theta)) for i in range(r // 2)]
        for i in range(r // 2):
            if case["layout"] == "sections":
                axis.append(next(a for a in range(n) if i < sum(sections[:a + 1])))
            else:
                axis.append(next((a for a in range(1, n) if i in range(a, n * sections[a], n)), 0))
    angle = places.double()[axis].T * torch.tensor(f, dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones_like(angle), angle)

    def heads(x, w):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / d + EPS) * w.double()
        first = torch.arange(0, r, 2) if case["style"] == "interleaved" else torch.arange(r // 2)
        second = first + (1 if case["style"] == "interleaved" else r // 2)
        z = torch.complex(x[..., first], x[..., second]) * turn[:, None]
        y = x.clone()
        y[..., first], y[..., second] = z.real, z.imag
        return y

    rows, past = _rows(case), _past(case)
    first, n_pages = _pages([p + n for p, n in zip(past, rows)], page)
    flat = torch.zeros(2, n_pages * page, hkv, d, dtype=torch.float64, device="cuda")
    at = 0
    keys, values = heads(k, wk), v.double()
    if case.get("fp8"):
        keys, values = keys / FP8_SCALE, values / FP8_SCALE
    for fp, p, n in zip(first, past, rows):
        flat[0, fp * page + p:fp * page + p + n] = keys[at:at + n]
        flat[1, fp * page + p:fp * page + p + n] = values[at:at + n]
        at += n
    return heads(q, wq), flat.view(2, n_pages, page, hkv, d).transpose(2, 3)


def _as_read(case, x):
    return _stored(case, x).double() * FP8_SCALE if case.get("fp8") else x


def _exact_attention(case, seed, step=1024):
    """Sequence by sequence and head by head, some rows at a time."""
    hq, hkv, d, page, _ = _geo(case)
    q, k, v = _attention_inputs(case, seed)
    k, v = _as_read(case, k), _as_read(case, v)
    total, window = _context(case), case.get("window") or 1 << 60
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    weights = torch.zeros(len(total), max(total), dtype=torch.float64, device="cuda")
    for l in range(case["layers"]):
        row = at = 0
        for b, (n, m) in enumerate(zip(_rows(case), total)):
            column = torch.arange(m, device="cuda")
            for h in range(hq):
                kh, vh = (x[l, at:at + m, h // (hq // hkv)].double() for x in (k, v))
                for i in range(0, n, step):
                    j = min(n, i + step)
                    x = (q[l, row + i:row + j, h].double() @ kh.T) * d ** -0.5
                    if case["kind"] == "weights":
                        mine = m - n + torch.arange(i, j, device="cuda")[:, None]
                        x = torch.where((column <= mine) & (column > mine - window), x, -math.inf)
                    x = torch.softmax(x, -1)
                    out[l, row + i:row + j, h] = x @ vh
                    weights[b, :m] += x.sum(0)
            row, at = row + n, at + m
    return out if case["kind"] == "cross" else (out, weights)


def _exact_evict(case, seed):
    hq, hkv, d, page, _ = _geo(case)
    k, v, weight = _evict_inputs(case, seed)
    k, v = (_stored(case, x).double() for x in (k, v))
    rows, slots = _rows(case), max(_rows(case))
    keep = [min(n, case["keep"]) for n in rows]
    first, n_pages = _pages(keep, page)
    flat = torch.zeros(case["layers"], 2, n_pages * page, hkv, d, dtype=torch.float64, device="cuda")
    positions = torch.full((len(rows), slots), -1, dtype=torch.int32, device="cuda")
    weights = torch.zeros(len(rows), slots, dtype=torch.float64, device="cuda")
    at = 0
    for b, (n, m) in enumerate(zip(rows, keep)):
        w = weight[at:at + n].tolist()
        kept = list(range(n))
        if n > m:
            middle = sorted(range(case["first"], n - case["last"]), key=lambda i: (-w[i], i))
            kept = sorted(list(range(case["first"])) + middle[:m - case["first"] - case["last"]]
                          + list(range(n - case["last"], n)))
        i = torch.tensor(kept, device="cuda")
        flat[:, 0, first[b] * page:first[b] * page + m] = k[:, at + i]
        flat[:, 1, first[b] * page:first[b] * page + m] = v[:, at + i]
        positions[b, :m] = i.int()
        weights[b, :m] = weight[at + i].double()
        at += n
    return flat.view(case["layers"], 2, n_pages, page, hkv, d).transpose(3, 4), positions, weights


def exact(case, seed):
    return {"axes": _exact_axes, "cross": _exact_attention, "weights": _exact_attention,
            "evict": _exact_evict}[case["kind"]](case, seed)
