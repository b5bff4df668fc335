"""The operators of a forward pass over a grafted context, as measured work: a
plain form of each in elementary torch operations, and the calls a user makes
of the library.

  append   the projections of new tokens become rows of the paged cache: root
           mean square norm of each query and key head, rotary positions (half
           or interleaved pairs, part of the head, scaled for long contexts),
           keys and values written to their pages (quantized for an fp8
           cache), rotated queries returned.  Prompts of different lengths are
           packed; a decode step is a batch of prompts of one token.  The
           measured call writes one layer of rows that are already open, as
           each layer of a model but the first does.
  prompt   causal attention of packed prompts over a paged cache: each new
           row attends to its sequence's restored rows and to the new rows up
           to itself, over the last `window` of them on a windowed layer.
  shared   decode attention of a batch whose sequences were given the same
           stored block (the pages are shared), each with a tail of its own:
           the common pages are read once for the whole batch.

Geometries are those of the repository's workloads (kvg_synth.py).  Rows and
queries are N(0, 1) draws rounded to bf16; fp8 caches use its per-tensor scale.

The library keeps rows behind a cache handle and the plain forms keep them in
torch tensors, so prepare() fills one or the other from the same draws.
"""
from __future__ import annotations

import math

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
ORIGINAL, FACTOR, BETA_FAST, BETA_SLOW = 4096, 8.0, 32.0, 1.0  # context scaling


def listed():
    return [
        # one token of one conversation: latency and launches count
        {"name": "append_step_1", "kind": "append", "model": "31b", "batch": 1, "rows_lo": 1, "rows_hi": 1,
         "past_lo": 2110, "past_hi": 2110, "norm": True, "rotary": 128, "style": "half", "scaling": "none"},
        # a decode step of continuous batching on an fp8 cache
        {"name": "append_step_fp8_b48", "kind": "append", "model": "12b", "fp8": True, "batch": 48, "rows_lo": 1,
         "rows_hi": 1, "past_lo": 97, "past_hi": 1533, "norm": True, "rotary": 256, "style": "half",
         "scaling": "linear", "fused": True},
        # one long prompt (an odd length), projections in one buffer
        {"name": "append_prompt_12b", "kind": "append", "model": "12b", "batch": 1, "rows_lo": 8191, "rows_hi": 8191,
         "past_lo": 64, "past_hi": 64, "norm": True, "rotary": 256, "style": "half", "scaling": "none",
         "fused": True},
        # packed prompts, half of each head rotated in interleaved pairs with blended frequencies
        {"name": "append_packed_31b", "kind": "append", "model": "31b", "batch": 23, "rows_lo": 1, "rows_hi": 1417,
         "past_lo": 0, "past_hi": 700, "norm": False, "rotary": 64, "style": "interleaved", "scaling": "yarn"},
        # a short question on the smallest fixture's block
        {"name": "prompt_tiny", "kind": "prompt", "model": "tiny", "batch": 1, "rows_lo": 37, "rows_hi": 37,
         "past_lo": 256, "past_hi": 256},
        # a chat turn on a restored 8,192-token block
        {"name": "prompt_turn_12b", "kind": "prompt", "model": "12b", "batch": 1, "rows_lo": 499, "rows_hi": 499,
         "past_lo": 8192, "past_hi": 8192},
        # packed prompts of different lengths, some on a context, some fresh; windowed layer of an fp8 cache
        {"name": "prompt_packed_fp8", "kind": "prompt", "model": "31b", "fp8": True, "batch": 13, "rows_lo": 1,
         "rows_hi": 1501, "past_lo": 0, "past_hi": 903, "window": 1024},
        # a long prompt from nothing, head_dim 256
        {"name": "prompt_long_12b", "kind": "prompt", "model": "12b", "batch": 1, "rows_lo": 8191, "rows_hi": 8191,
         "past_lo": 0, "past_hi": 0},
        # a long document on top of a 16,384-token block
        {"name": "prompt_long_31b", "kind": "prompt", "model": "31b", "batch": 1, "rows_lo": 8192, "rows_hi": 8192,
         "past_lo": 16384, "past_hi": 16384},
        # a handful of conversations on the smallest fixture's block
        {"name": "shared_tiny", "kind": "shared", "model": "tiny", "layers": 1, "batch": 4, "prefix": 256,
         "tail_lo": 1, "tail_hi": 40},
        # a system prompt's block under 32 conversations, two layers in a call
        {"name": "shared_12b_b32", "kind": "shared", "model": "12b", "layers": 2, "batch": 32, "prefix": 8192,
         "tail_lo": 5, "tail_hi": 611},
        # a long document under many short questions, fp8
        {"name": "shared_31b_fp8_b96", "kind": "shared", "model": "31b", "fp8": True, "layers": 1, "batch": 96,
         "prefix": 32768, "tail_lo": 1, "tail_hi": 257},
    ]


def _size(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]; odd ones as often as even."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "prompt", "prompt", "shared"])
    model = rng.choice(["tiny", "12b", "31b", "12b", "31b"])
    hq, hkv, d, page, _ = MODELS[model]
    case = {"kind": kind, "model": model}
    if rng.random() < 0.25:
        case["page"] = page = rng.choice([16, 24, 32, 48, 80, 128])
    if model != "tiny" and rng.random() < 0.35:
        case["fp8"] = True
    if kind == "append":
        case["batch"] = batch = _size(rng, 1, 64)
        hi = _size(rng, 1, 8191 // batch) if rng.random() < 0.7 else 1
        case["rows_lo"], case["rows_hi"] = max(1, int(hi * rng.random())), hi
        case["past_hi"] = _size(rng, 1, 3000) - 1
        case["past_lo"] = int(case["past_hi"] * rng.random())
        case["norm"] = rng.random() < 0.6
        case["rotary"] = rng.choice([d, d, d // 2, d // 4])
        case["style"] = rng.choice(["half", "half", "interleaved"])
        case["scaling"] = rng.choice(["none", "linear", "yarn"])
        case["fused"] = rng.random() < 0.5
    elif kind == "prompt":
        case["batch"] = batch = _size(rng, 1, 40)
        total = _size(rng, 40, 24000)  # rows of a sequence, restored ones included
        hi = _size(rng, 2, min(total, 8192))
        while batch * hi * total * hq > 2e9:
            hi, batch = max(2, hi // 2), max(1, batch - batch // 3)
        case["batch"] = batch
        case["rows_lo"], case["rows_hi"] = max(1, int(hi * rng.random())), hi
        case["past_hi"] = total - hi
        case["past_lo"] = int(case["past_hi"] * rng.random())
        if rng.random() < 0.3:
            case["window"] = _size(rng, 64, 4096)
    else:
        case["layers"] = rng.choice([1, 1, 2, 3])
        case["batch"] = _size(rng, 2, 96)
        case["prefix"] = _size(rng, page, min(24000, 1024 * page))
        case["tail_hi"] = _size(rng, 1, 600)
        case["tail_lo"] = max(1, int(case["tail_hi"] * rng.random()))
        if rng.random() < 0.2:
            case["window"] = _size(rng, 64, 8192)
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
    return _spread(case["past_lo"], case["past_hi"], case["batch"], 104729)


def _tails(case):
    return _spread(case["tail_lo"], case["tail_hi"], case["batch"], 7919)


def _draws(seed, device="cuda"):
    """Generator of N(0, 1) draws rounded to bf16, the same for the same seed."""
    g = torch.Generator(device=device)
    g.manual_seed(int(seed))
    return lambda *shape: torch.randn(shape, generator=g, device=device).to(torch.bfloat16)


def _inverse_frequencies(case, theta):
    """Rotation per position of each pair, in 64 bits, and the factor on cos and sin.
    Blended scaling: a pair that turns r times over the original context keeps its
    frequency for r >= BETA_FAST, has it divided by FACTOR for r <= BETA_SLOW, and a
    blend of the two, linear in r, in between."""
    r = case["rotary"]
    f = theta ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)
    if case["scaling"] == "linear":
        return f / FACTOR, 1.0
    if case["scaling"] == "yarn":
        turns = ORIGINAL * f / (2 * math.pi)
        keep = ((turns - BETA_SLOW) / (BETA_FAST - BETA_SLOW)).clamp(0, 1)
        return f / FACTOR * (1 - keep) + f * keep, 0.1 * math.log(FACTOR) + 1
    return f, 1.0


def _append_inputs(case, seed):
    hq, hkv, d, _, _ = _geo(case)
    rows, past = _rows(case), _past(case)
    t = sum(rows)
    draws = _draws(seed)
    if case.get("fused"):  # one projection's output, queries, keys and values side by side
        x = draws(t, hq + 2 * hkv, d)
        q, k, v = x.split([hq, hkv, hkv], dim=1)
    else:
        q, k, v = draws(t, hq, d), draws(t, hkv, d), draws(t, hkv, d)
    wq = wk = None
    if case["norm"]:
        wq, wk = ((1 + 0.1 * draws(d).float()).to(torch.bfloat16) for _ in range(2))
    positions = torch.cat([torch.arange(p, p + n) for p, n in zip(past, rows)]).to(torch.int32).cuda()
    return q, k, v, wq, wk, positions


def _prompt_inputs(case, seed):
    """Queries of the packed rows, and keys and values of every row, sequence after sequence."""
    hq, hkv, d, _, _ = _geo(case)
    draws = _draws(seed)
    n = sum(_rows(case)) + sum(_past(case))
    return draws(sum(_rows(case)), hq, d), draws(n, hkv, d), draws(n, hkv, d)


def _shared_inputs(case, seed):
    """Queries, the shared rows and the tails' rows, sequence after sequence."""
    hq, hkv, d, _, _ = _geo(case)
    draws = _draws(seed)
    n_l, n_t = case["layers"], sum(_tails(case))
    return (draws(n_l, case["batch"], hq, d), draws(n_l, case["prefix"], hkv, d), draws(n_l, case["prefix"], hkv, d),
            draws(n_l, n_t, hkv, d), draws(n_l, n_t, hkv, d))


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

def _dims(kvg, case, layers):
    hq, hkv, d, page, theta = _geo(case)
    return kvg.make_dims(layers, hkv, d, page, theta,
                         kvg.KVG_ROPE_INTERLEAVED if case.get("style") == "interleaved" else kvg.KVG_ROPE_HALF,
                         kvg.KVG_KV_E4M3 if case.get("fp8") else kvg.KVG_KV_BF16, FP8_SCALE, FP8_SCALE)


class _Memory:
    """Device memory of the library as a torch tensor, which keeps its owner alive."""

    def __init__(self, owner, ptr, n):
        self.owner = owner
        self.__cuda_array_interface__ = {"shape": (n,), "typestr": "|u1", "data": (int(ptr), False), "version": 3}


def _append_cache(case, layers, total):
    """A cache that holds `total` rows per sequence, its pool zeroed and as a tensor."""
    from paper_2607_14431_gb300 import kvg
    hq, hkv, d, page, _ = _geo(case)
    cache = kvg.Cache(_dims(kvg, case, layers), _pages(total, page)[1], len(total), max(total))
    pool = torch.as_tensor(_Memory(cache, cache.view.pool, cache.view.pool_bytes), device="cuda")
    pool.zero_()
    kind = torch.float8_e4m3fn if case.get("fp8") else torch.bfloat16
    return kvg, cache, pool.view(kind).view(layers, 2, -1, hkv, page, d)


def _fill(kvg, cache, seq, k, v, first=0):
    """Appends rows k, v [L][n][Hkv][D] of a sequence, at positions from `first`."""
    n = k.shape[1]
    if n:
        k, v = k.contiguous(), v.contiguous()
        pos = torch.arange(first, first + n, dtype=torch.int32, device="cuda")
        kvg.kvg_cache_append(cache.h, seq, k.data_ptr(), v.data_ptr(), pos.data_ptr(), n)
        torch.cuda.synchronize()


def _prepare_append(case, seed):
    hq, hkv, d, page, theta = _geo(case)
    rows, past = _rows(case), _past(case)
    q, k, v, wq, wk, positions = _append_inputs(case, seed)
    total = [p + n for p, n in zip(past, rows)]
    first, n_pages = _pages(total, page)
    s = {"q": q, "k": k, "v": v, "wq": wq, "wk": wk, "positions": positions, "q_out": torch.empty_like(q.contiguous())}
    if own:
        kvg, cache, pool = _append_cache(case, 2, total)
        # pages in the order in which the rows below ask for them, so that each lands where the plain form's does
        had = [-(-p // page) for p in past]
        kvg.kvg_cache_set_free_order(
            cache.h, [f + j for f, h in zip(first, had) for j in range(h)]
            + [f + j for f, h, n in zip(first, had, total) for j in range(h, -(-n // page))])
        for b, p in enumerate(past):
            zero = torch.zeros(2, p, hkv, d, dtype=torch.bfloat16, device="cuda")
            _fill(kvg, cache, b, zero, zero)
        scaling = {"none": kvg.KVG_ROPE_SCALING_NONE, "linear": kvg.KVG_ROPE_SCALING_LINEAR,
                   "yarn": kvg.KVG_ROPE_SCALING_YARN}[case["scaling"]]
        rotary = kvg.Rotary(d, case["rotary"], theta, cache.dims.rope_style, scaling, FACTOR, ORIGINAL, BETA_FAST,
                            BETA_SLOW, 0.1 * math.log(FACTOR) + 1 if case["scaling"] == "yarn" else 1.0)
        qkv = kvg.make_qkv(q, k, v, q_norm=wq, k_norm=wk, eps=EPS)
        s |= {"kvg": kvg, "cache": cache, "pool": pool[1], "rotary": rotary, "qkv": qkv, "rows": rows,
              "seqs": list(range(len(rows)))}
        # layer 0 opens the rows; run() writes layer 1 of them
        kvg.kvg_cache_append_qkv(cache.h, 0, s["seqs"], rows, qkv, rotary.h, positions.data_ptr(),
                                 s["q_out"].data_ptr())
        torch.cuda.synchronize()
    else:
        kind = torch.float8_e4m3fn if case.get("fp8") else torch.bfloat16
        s["pool"] = torch.zeros(2, n_pages, hkv, page, d, dtype=torch.bfloat16, device="cuda").to(kind)
        slots = torch.cat([torch.arange(p, p + n) + f * page for f, p, n in zip(first, past, rows)]).cuda()
        s |= {"page": slots // page, "row": slots % page}
        f, m = _inverse_frequencies(case, theta)
        s |= {"freq": f.float().cuda(), "factor": m}
    return s


def _prepare_prompt(case, seed):
    hq, hkv, d, page, _ = _geo(case)
    rows, past = _rows(case), _past(case)
    q, k, v = _prompt_inputs(case, seed)
    total = [p + n for p, n in zip(past, rows)]
    s = {"q": q, "out": torch.empty_like(q), "scale": 1 / math.sqrt(d)}
    if own:
        kvg, cache, _ = _append_cache(case, 1, total)
        if case.get("window"):
            kvg.kvg_cache_set_layer_windows(cache.h, [case["window"]])
        at = 0
        for b, n in enumerate(total):
            _fill(kvg, cache, b, k[None, at:at + n], v[None, at:at + n])
            at += n
        s |= {"kvg": kvg, "cache": cache, "rows": rows, "seqs": list(range(len(rows)))}
        return s
    first, n_pages = _pages(total, page)
    kind = torch.float8_e4m3fn if case.get("fp8") else torch.bfloat16
    pool = torch.zeros(2, n_pages * page, hkv, d, dtype=torch.bfloat16, device="cuda")
    slots = torch.cat([torch.arange(n) + f * page for f, n in zip(first, total)]).cuda()
    pool[0, slots], pool[1, slots] = k, v
    pool = _stored(case, pool).view(2, n_pages, page, hkv, d).transpose(2, 3).contiguous()
    most = -(-max(total) // page)
    table = torch.tensor([[f + min(j, -(-n // page) - 1) for j in range(most)] for f, n in zip(first, total)])
    # where a packed query row sits in the padded batch
    b_of = torch.cat([torch.full((n,), b) for b, n in enumerate(rows)]).cuda()
    t_of = torch.cat([torch.arange(n) for n in rows]).cuda()
    s |= {"pool": pool, "table": table.cuda(), "b_of": b_of, "t_of": t_of,
          "past": torch.tensor(past, device="cuda"), "most_rows": max(rows)}
    return s


def _prepare_shared(case, seed):
    hq, hkv, d, page, _ = _geo(case)
    tails, n_l, batch, prefix = _tails(case), case["layers"], case["batch"], case["prefix"]
    q, kp, vp, kt, vt = _shared_inputs(case, seed)
    s = {"q": q, "out": torch.empty_like(q), "scale": 1 / math.sqrt(d)}
    if own:
        from paper_2607_14431_gb300 import kvg
        most = prefix + page + max(tails)
        # the block's pages, the source sequence's, and each sequence's own
        n_pages = 2 * (-(-prefix // page)) + sum(-(-n // page) + 1 for n in tails)
        cache = kvg.Cache(_dims(kvg, case, n_l), n_pages, batch + 1, most)
        store = kvg.PoolStore(cache, 1 << 30)
        _fill(kvg, cache, batch, kp, vp)
        block = kvg.kvg_deposit(store.h, cache.h, batch, 0, prefix)
        kvg.kvg_cache_release(cache.h, batch)
        at = 0
        for b, n in enumerate(tails):
            kvg.kvg_graft(store.h, block, cache.h, b)
            _fill(kvg, cache, b, kt[:, at:at + n], vt[:, at:at + n], prefix)
            at += n
        if case.get("window"):
            kvg.kvg_cache_set_layer_windows(cache.h, [case["window"]] * n_l)
        torch.cuda.synchronize()
        s |= {"kvg": kvg, "cache": cache, "store": store, "seqs": list(range(batch)),
              "layer": -1 if n_l > 1 else 0}
        return s
    k = torch.zeros(n_l, batch, max(tails), hkv, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    at = 0
    for b, n in enumerate(tails):
        k[:, b, :n], v[:, b, :n] = kt[:, at:at + n], vt[:, at:at + n]
        at += n
    s |= {"kp": _stored(case, kp), "vp": _stored(case, vp), "kt": _stored(case, k), "vt": _stored(case, v),
          "tails": torch.tensor(tails, device="cuda")}
    return s


def prepare(case, seed):
    s = {"append": _prepare_append, "prompt": _prepare_prompt, "shared": _prepare_shared}[case["kind"]](case, seed)
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


def _plain_append(s):
    case = s["case"]
    q, k = s["q"].float(), s["k"].float()
    if case["norm"]:
        q, k = _normed(q, s["wq"]), _normed(k, s["wk"])
    angle = s["positions"].float()[:, None] * s["freq"]
    cos, sin = angle.cos() * s["factor"], angle.sin() * s["factor"]
    q, k = (_rotated(x, cos, sin, case["style"] == "interleaved") for x in (q, k))
    k = _stored(case, k) if case.get("fp8") else k.to(torch.bfloat16)
    pool, at = _bits(s["pool"]), (s["page"], slice(None), s["row"])
    pool[(0, *at)], pool[(1, *at)] = _bits(k), _bits(_stored(case, s["v"]))
    return q.to(torch.bfloat16), s["pool"]


def _softmax_product(score, mask, v):
    """Weights exp(score - max) over the columns the mask leaves, divided by their sum, times v."""
    score = score.masked_fill_(~mask, -math.inf)
    score = score.sub_(score.amax(-1, keepdim=True)).exp_()
    return torch.matmul(score, v) / score.sum(-1, keepdim=True)


def _plain_prompt(s):
    case = s["case"]
    hq, hkv, d, page, _ = _geo(case)
    scale = FP8_SCALE if case.get("fp8") else 1.0
    kv = _bits(s["pool"])[:, s["table"]].view(s["pool"].dtype).float() * scale  # [2][B][pages][Hkv][P][D]
    batch, pages = s["table"].shape
    k, v = kv.transpose(3, 4).reshape(2, batch, pages * page, hkv, d).transpose(2, 3)
    n = s["most_rows"]
    q = torch.zeros(batch, n, hq, d, device="cuda")
    q[s["b_of"], s["t_of"]] = s["q"].float()
    q = q.view(batch, n, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(batch, hkv, hq // hkv * n, d)
    score = torch.matmul(q * s["scale"], k.transpose(-1, -2)).view(batch, hkv, hq // hkv, n, pages * page)
    column = torch.arange(pages * page, device="cuda")
    at = s["past"][:, None] + torch.arange(n, device="cuda")  # own row of each query
    mask = column <= at[..., None]
    if case.get("window"):
        mask &= column > at[..., None] - case["window"]
    out = _softmax_product(score, mask[:, None, None], v[:, :, None])
    return out.permute(0, 3, 1, 2, 4).reshape(batch, n, hq, d)[s["b_of"], s["t_of"]].to(torch.bfloat16)


def _plain_shared(s):
    case = s["case"]
    hq, hkv, d, page, _ = _geo(case)
    n_l, batch, prefix = case["layers"], case["batch"], case["prefix"]
    g = hq // hkv
    scale = FP8_SCALE if case.get("fp8") else 1.0
    q = s["q"].float().view(n_l, batch, hkv, g, d) * s["scale"]
    kp, vp = (x.float().transpose(1, 2) * scale for x in (s["kp"], s["vp"]))            # [L][Hkv][N][D]
    kt, vt = (x.float().transpose(2, 3) * scale for x in (s["kt"], s["vt"]))            # [L][B][Hkv][n][D]
    # the shared rows' scores for the whole batch at once, then each sequence's own
    sp = torch.matmul(q.transpose(1, 2).reshape(n_l, hkv, batch * g, d), kp.transpose(-1, -2))
    sp = sp.view(n_l, hkv, batch, g, prefix)
    st = torch.matmul(q, kt.transpose(-1, -2)).transpose(1, 2)                           # [L][Hkv][B][g][n]
    column = torch.arange(prefix + kt.shape[3], device="cuda")
    end = prefix + s["tails"]
    mask = column < end[:, None]
    if case.get("window"):
        mask &= column >= end[:, None] - case["window"]
    score = torch.cat([sp, st], -1).masked_fill_(~mask[:, None], -math.inf)
    w = score.sub_(score.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(w[..., :prefix].reshape(n_l, hkv, batch * g, prefix), vp).view(n_l, hkv, batch, g, d)
    o += torch.matmul(w[..., prefix:].transpose(1, 2), vt).transpose(1, 2)
    o /= w.sum(-1, keepdim=True)
    return o.transpose(1, 2).reshape(n_l, batch, hq, d).to(torch.bfloat16)


def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"append": _plain_append, "prompt": _plain_prompt, "shared": _plain_shared}[kind](s)
    kvg, cache = s["kvg"], s["cache"]
    hq = s["q"].shape[-2]
    if kind == "append":
        kvg.kvg_cache_append_qkv(cache.h, 1, s["seqs"], s["rows"], s["qkv"], s["rotary"].h,
                                 s["positions"].data_ptr(), s["q_out"].data_ptr())
        return s["q_out"], s["pool"]
    if kind == "prompt":
        kvg.kvg_prompt_attention(cache.h, 0, s["seqs"], s["rows"], s["q"].data_ptr(), hq, s["out"].data_ptr(),
                                 s["scale"])
    else:
        kvg.kvg_decode_attention_shared(cache.h, s["layer"], s["seqs"], s["q"].data_ptr(), hq, s["out"].data_ptr(),
                                        s["scale"])
    return s["out"]


# ----------------------------------------------------------------- work --

def _visible(case):
    """(query row, cached row) pairs that attend, and cached rows that any query reads."""
    pairs = read = 0
    w = case.get("window") or 1 << 60
    for n, p in zip(_rows(case), _past(case)):
        short = max(0, min(n, w - p - 1))  # queries that see fewer rows than the window
        pairs += short * p + short * (short + 1) // 2 + (n - short) * min(w, p + n)
        read += min(p + n, w + n - 1)
    return pairs, read


def work(case):
    hq, hkv, d, page, _ = _geo(case)
    e = 1 if case.get("fp8") else 2
    if case["kind"] == "append":
        t = sum(_rows(case))
        return {"bytes": t * d * (2 * (hq + 2 * hkv) + 2 * hq + 2 * hkv * e), "flops": t * d * 8 * (hq + hkv)}
    if case["kind"] == "prompt":
        pairs, read = _visible(case)
        return {"bytes": read * hkv * d * 2 * e + sum(_rows(case)) * hq * d * 4, "flops": 4 * hq * d * pairs}
    n_l, batch, prefix, w = case["layers"], case["batch"], case["prefix"], case.get("window") or 1 << 60
    tails = [min(n, w) for n in _tails(case)]
    heads = [max(0, min(prefix, w - n)) for n in _tails(case)]
    return {"bytes": n_l * (2 * hkv * d * e * (max(heads) + sum(tails)) + batch * hq * d * 4),
            "flops": n_l * 4 * hq * d * (sum(heads) + sum(tails))}


# ---------------------------------------------------------------- exact --

def _exact_append(case, seed):
    hq, hkv, d, page, theta = _geo(case)
    q, k, v, wq, wk, positions = _append_inputs(case, seed)
    r = case["rotary"]
    pair = torch.arange(r // 2, dtype=torch.float64, device="cuda")
    f = torch.exp(-2 * pair / r * math.log(theta))
    m = 1.0
    if case["scaling"] == "linear":
        f = f / FACTOR
    elif case["scaling"] == "yarn":
        ramp = torch.clamp((ORIGINAL * f / (2 * math.pi) - BETA_SLOW) / (BETA_FAST - BETA_SLOW), 0, 1)
        f, m = f * (ramp + (1 - ramp) / FACTOR), 1 + 0.1 * math.log(FACTOR)
    turn = torch.polar(torch.full((), m, dtype=torch.float64, device="cuda"), positions.double()[:, None] * f)

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


def _exact_attention(q, k, v, scale, last, window, step=1024):
    """Attention of rows q [n][H][D] over k, v [N][Hkv][D], row i over the columns
    last[i] - window < j <= last[i], in 64 bits, some rows at a time."""
    n, h, d = q.shape
    g = h // k.shape[1]
    out = torch.empty(n, h, d, dtype=torch.float64, device="cuda")
    column = torch.arange(k.shape[0], device="cuda")
    for head in range(h):
        kh, vh = k[:, head // g].double(), v[:, head // g].double()
        for i in range(0, n, step):
            end = int(last[i:i + step].max()) + 1
            at = last[i:i + step, None]
            x = (q[i:i + step, head].double() @ kh[:end].T) * scale
            x = torch.where((column[:end] <= at) & (column[:end] > at - window), x, -math.inf)
            out[i:i + step, head] = torch.softmax(x, -1) @ vh[:end]
    return out


def _as_read(case, x):
    return _stored(case, x).double() * FP8_SCALE if case.get("fp8") else x


def _exact_prompt(case, seed):
    hq, hkv, d, page, _ = _geo(case)
    q, k, v = _prompt_inputs(case, seed)
    k, v = _as_read(case, k), _as_read(case, v)
    outs, at, row = [], 0, 0
    for n, p in zip(_rows(case), _past(case)):
        last = torch.arange(p, p + n, device="cuda")
        outs.append(_exact_attention(q[row:row + n], k[at:at + p + n], v[at:at + p + n], d ** -0.5, last,
                                     case.get("window") or 1 << 60))
        at, row = at + p + n, row + n
    return torch.cat(outs)


def _exact_shared(case, seed):
    hq, hkv, d, page, _ = _geo(case)
    q, kp, vp, kt, vt = _shared_inputs(case, seed)
    kp, vp, kt, vt = (_as_read(case, x) for x in (kp, vp, kt, vt))
    out, at = torch.empty(q.shape, dtype=torch.float64, device="cuda"), 0
    for b, n in enumerate(_tails(case)):
        for l in range(case["layers"]):
            k, v = (torch.cat([x[l], y[l, at:at + n]]) for x, y in ((kp, kt), (vp, vt)))
            last = torch.tensor([case["prefix"] + n - 1], device="cuda")
            first = max(0, case["prefix"] + n - (case.get("window") or 1 << 60))
            # all heads of the row at once: one query against the rows of its kv head
            kk, vv = k[first:].double().transpose(0, 1), v[first:].double().transpose(0, 1)
            x = torch.matmul(q[l, b].double().view(hkv, hq // hkv, d), kk.transpose(1, 2)) * d ** -0.5
            out[l, b] = torch.matmul(torch.softmax(x, -1), vv).reshape(hq, d)
        at += n
    return out


def exact(case, seed):
    return {"append": _exact_append, "prompt": _exact_prompt, "shared": _exact_shared}[case["kind"]](case, seed)
