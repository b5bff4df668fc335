"""kvg_cache_append_qkv against its formula in 64 bits: norm of each head,
rotary positions, rows in their pages, page tables, fills and position tags.

Bounds, from the roundings of one value z = m (a cos - b sin), a and b normed:
the fp32 norm is off by at most 16 x 2^-24 of a value (sum of squares 13
roundings at most, halved by the root; reciprocal root 2 ulp; two products),
the angle by pi 2^-25 (fraction rounded to fp32), cos and sin by another 2 ulp
of 2^-24, the factor and the two products by 2^-23: less than 2^-19 of
m (|a| + |b|) in all.  On top comes one rounding: half a step of bf16, or of
the E4M3 grid."""
import numpy as np
import pytest
import torch

from kvg_testlib import dev_view, need_gpu

pytestmark = pytest.mark.gpu
FP32 = 2.0 ** -19


@pytest.fixture(scope="module")
def kvg():
    return need_gpu()


def draws(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape).astype(np.float32)


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).cuda()


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def frequencies(rot, theta, scaling="none", factor=1.0, original=0, fast=32.0, slow=1.0):
    f = np.array([theta ** (-2.0 * i / rot) for i in range(rot // 2)])
    if scaling == "linear":
        f = f / factor
    elif scaling == "yarn":
        keep = np.clip((original * f / (2 * np.pi) - slow) / (fast - slow), 0, 1)
        f = f / factor * (1 - keep) + f * keep
    return f


def reference(x, w, eps, offset, pos, f, interleaved, m):
    """(value, |a| + |b| of its pair) of heads x [T][H][D] in 64 bits."""
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (w + offset) if w is not None else x.copy()
    n, size = len(f), np.abs(y)
    if n:
        a = np.arange(n) * 2 if interleaved else np.arange(n)
        b = a + 1 if interleaved else a + n
        ang = pos.astype(np.float64)[:, None, None] * f
        c, s = np.cos(ang) * m, np.sin(ang) * m
        ya, yb = y[..., a].copy(), y[..., b].copy()
        both = (np.abs(ya) + np.abs(yb)) * abs(m)
        y[..., a], y[..., b] = ya * c - yb * s, yb * c + ya * s
        size[..., a] = size[..., b] = both
    return y, size


def half_step(x, bits):
    """Half the distance between neighbours of |x| with `bits` bits after the leading one."""
    return np.ldexp(0.5, np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -126))).astype(int) - bits)


def check_bf16(got, ref, size):
    err = np.abs(got - ref) - half_step(ref, 7) - FP32 * size
    assert err.max() <= 0, (err.max(), np.abs(got - ref).max())


def check_e4m3(got, ref, size, scale):
    """got: code values; ref, size in units of the cached value."""
    x = np.clip(ref / scale, -448, 448)
    step = np.maximum(half_step(x, 3), 2.0 ** -10)  # subnormal codes are 2^-9 apart
    err = np.abs(got - x) - step - (FP32 + 2.0 ** -23) * size / scale
    assert err.max() <= 0, err.max()


def pool_values(cache, dims):
    v = cache.view
    raw = dev_view(v.pool, v.pool_bytes, torch.uint8)
    kind = torch.float8_e4m3fn if dims.kv_dtype else torch.bfloat16
    return raw.view(kind).view(dims.n_layers, 2, v.n_pages, dims.n_kv_heads, dims.page_size, dims.head_dim)


def tables(cache):
    v = cache.view
    return [dev_view(ptr, 4 * v.max_seqs * n, torch.int32).view(v.max_seqs, n).cpu().numpy()
            for ptr, n in ((v.page_table, v.max_pages), (v.page_fill, v.max_pages), (v.positions, v.max_slots))]


def make_cache(kvg, n_layers, hkv, d, page, rows, fp8=False, style=0, seqs=None, scale=0.0625, extra=0):
    dims = kvg.make_dims(n_layers, hkv, d, page, 1e4, style, 1 if fp8 else 0, scale, scale)
    n_pages = sum(-(-(n + extra) // page) for n in rows) + 1
    cache = kvg.Cache(dims, n_pages, seqs or len(rows), max(rows) + extra + page)
    kvg.kvg_cache_set_free_order(cache.h, np.random.default_rng(1).permutation(n_pages))
    return cache, dims


def rows_of(cache, dims, seq, n, layer, kv, first=0):
    """The cached rows [n][Hkv][D] of a sequence's slots, through its page table."""
    table = tables(cache)[0][seq]
    s = np.arange(first, first + n)
    pages, at = torch.from_numpy(table[s // dims.page_size]).long().cuda(), torch.from_numpy(s % dims.page_size).cuda()
    pool = pool_values(cache, dims)
    if pool.dtype == torch.float8_e4m3fn:
        pool = pool.float()
    return f64(pool[layer, kv][pages, :, at])


# layers, Hq, Hkv, D, page, rows per sequence, fp8, rotary_dim, style, scaling, norm, fused, first position
CASES = [
    (2, 4, 2, 64, 16, [5, 0, 37, 1], False, 64, 0, "none", True, False, 0),
    (1, 4, 4, 64, 7, [130], True, 32, 1, "none", True, True, 100),
    (2, 32, 16, 128, 64, [1, 1, 1], False, 128, 0, "yarn", True, True, 30000),
    (1, 8, 2, 128, 24, [65, 64, 63], True, 48, 0, "linear", False, False, 7),
    (1, 8, 8, 128, 1, [9, 3], False, 16, 1, "yarn", True, True, 0),
    (2, 16, 8, 256, 64, [70], False, 256, 0, "none", True, True, 2 ** 31 - 71),
    (1, 2, 1, 256, 80, [161, 2], True, 256, 1, "none", True, False, 131072),
    (1, 40, 40, 128, 33, [40], False, 0, 0, "none", False, False, 0),
    (1, 0, 2, 64, 16, [20], False, 64, 0, "none", True, True, 5),
    (1, 96, 4, 256, 16, [3], False, 112, 0, "none", True, True, 1),
]


def build(kvg, case, seed=3):
    n_l, hq, hkv, d, page, rows, fp8, rot, style, scaling, norm, fused, pos0 = case
    t = sum(rows)
    x = bf16(draws(seed, n_l, t, hq + 2 * hkv, d))
    q, k, v = x.split([hq, hkv, hkv], dim=2)
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    wq, wk = (bf16(1 + 0.2 * draws(seed + 1 + i, n_l, d)) for i in range(2))
    pos = np.concatenate([pos0 + np.arange(n) for n in rows]).astype(np.int32)
    m = 0.1 * np.log(8.0) + 1 if scaling == "yarn" else 1.0
    rotary = kvg.Rotary(d, rot, 1e4, style, {"none": 0, "linear": 1, "yarn": 2}[scaling], 8.0, 4096, 32.0, 1.0, m)
    f = frequencies(rot, 1e4, scaling, 8.0, 4096)
    qkv = kvg.make_qkv(q if hq else None, k, v, wq if norm and hq else None, wk if norm else None, 1e-5, 0.0)
    qo = torch.zeros(n_l, t, hq, d, dtype=torch.bfloat16, device="cuda")
    return q, k, v, (wq, wk) if norm else (None, None), pos, np.float32(m).item(), rotary, f, qkv, qo


def check(cache, dims, rows, case, q, k, v, w, pos, m, f, qo, offset=0.0, eps=1e-5, first=0):
    n_l, hq, hkv, d, page, _, fp8, rot, style = case[:9]
    eps = float(np.float32(eps))
    for l in range(n_l):
        wq, wk = (None if x is None else f64(x[l]) for x in w)
        if hq:
            check_bf16(f64(qo[l]), *reference(f64(q[l]), wq, eps, offset, pos, f, style, m))
        ref, size = reference(f64(k[l]), wk, eps, offset, pos, f, style, m)
        val, at = f64(v[l]), 0
        for b, n in enumerate(rows):
            if n:
                gk, gv = (rows_of(cache, dims, b, n, l, kv, first) for kv in (0, 1))
                if fp8:
                    check_e4m3(gk, ref[at:at + n], size[at:at + n], 0.0625)
                    check_e4m3(gv, val[at:at + n], np.zeros_like(gv), 0.0625)
                else:
                    check_bf16(gk, ref[at:at + n], size[at:at + n])
                    assert np.array_equal(gv, val[at:at + n])
            at += n


@pytest.mark.parametrize("case", CASES, ids=[f"{c[1]}x{c[2]}x{c[3]}p{c[4]}{'fp8' if c[6] else ''}r{c[7]}" for c in CASES])
def test_rows_queries_and_tables(kvg, case):
    n_l, hq, hkv, d, page, rows, fp8, rot, style = case[:9]
    q, k, v, w, pos, m, rotary, f, qkv, qo = build(kvg, case)
    cache, dims = make_cache(kvg, n_l, hkv, d, page, rows, fp8, style)
    pd = torch.from_numpy(pos).cuda()
    kvg.kvg_cache_append_qkv(cache.h, -1, list(range(len(rows))), rows, qkv, rotary.h, pd.data_ptr(),
                             qo.data_ptr() if hq else None)
    torch.cuda.synchronize()
    kvg.kvg_sync(cache.h)
    check(cache, dims, rows, case, q, k, v, w, pos, m, f, qo)
    _, fill, tags = tables(cache)
    at = 0
    for b, n in enumerate(rows):
        assert kvg.kvg_cache_seq_info(cache.h, b) == (n, -(-n // page))
        want = [min(page, n - j * page) for j in range(-(-n // page))]
        assert fill[b, :len(want)].tolist() == want and not fill[b, len(want):].any()
        assert np.array_equal(tags[b, :n], pos[at:at + n]) and (tags[b, n:] == -1).all()
        at += n


def test_layer_by_layer_and_in_place_equal_all_layers_at_once(kvg):
    case = CASES[0]
    rows = case[5]
    outs = []
    for how in range(2):
        q, k, v, w, pos, m, rotary, f, qkv, qo = build(kvg, case)
        cache, dims = make_cache(kvg, 2, 2, 64, 16, rows)
        pool_values(cache, dims).zero_()
        pd = torch.from_numpy(pos).cuda()
        if how == 0:
            kvg.kvg_cache_append_qkv(cache.h, -1, [0, 1, 2, 3], rows, qkv, rotary.h, pd.data_ptr(), qo.data_ptr())
        else:
            for l in (0, 1, 1):
                one = kvg.make_qkv(q[l].clone(), k[l], v[l], w[0][l], w[1][l], 1e-5)
                x = q[l].clone()
                one = kvg.make_qkv(x, k[l], v[l], w[0][l], w[1][l], 1e-5)
                kvg.kvg_cache_append_qkv(cache.h, l, [0, 1, 2, 3], rows, one, rotary.h, pd.data_ptr(), x.data_ptr())
                qo[l] = x
        torch.cuda.synchronize()
        outs.append((qo.view(torch.int16).cpu(), pool_values(cache, dims).view(torch.int16).cpu(), tables(cache)))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    assert all(np.array_equal(a, b) for a, b in zip(outs[0][2], outs[1][2]))


@pytest.mark.parametrize("fp8", [False, True])
def test_without_norm_and_rotation_it_is_the_append(kvg, fp8):
    n_l, hkv, d, page, n = 2, 4, 128, 24, 133
    k, v = bf16(30 * draws(5, n_l, n, hkv, d)), bf16(30 * draws(6, n_l, n, hkv, d))
    pos = torch.arange(n, dtype=torch.int32).cuda()
    pools = []
    for how in range(2):
        cache, dims = make_cache(kvg, n_l, hkv, d, page, [n], fp8)
        pool_values(cache, dims).view(torch.uint8).zero_()
        if how:
            kvg.kvg_cache_append_qkv(cache.h, -1, [0], [n], kvg.make_qkv(None, k, v), None, pos.data_ptr(), None)
        else:
            kvg.kvg_cache_append(cache.h, 0, k.data_ptr(), v.data_ptr(), pos.data_ptr(), n)
        torch.cuda.synchronize()
        pools.append((pool_values(cache, dims).view(torch.uint8).cpu(), tables(cache)))
    assert torch.equal(pools[0][0], pools[1][0])
    assert all(np.array_equal(a, b) for a, b in zip(pools[0][1], pools[1][1]))


def test_many_sequences_and_more_pages_than_a_launch_takes(kvg):
    """300 sequences (a launch takes 256) and 4,500 pages of one row (a launch takes 1,024)."""
    rows = [1 + 4200 * (b == 7) for b in range(300)]
    case = (1, 2, 1, 64, 1, rows, False, 64, 0, "none", True, True, 11)
    q, k, v, w, pos, m, rotary, f, qkv, qo = build(kvg, case)
    cache, dims = make_cache(kvg, 1, 1, 64, 1, rows)
    pd = torch.from_numpy(pos).cuda()
    kvg.kvg_cache_append_qkv(cache.h, 0, list(range(300)), rows, qkv, rotary.h, pd.data_ptr(), qo.data_ptr())
    torch.cuda.synchronize()
    check(cache, dims, rows, case, q, k, v, w, pos, m, f, qo)
    assert tables(cache)[1][7, :4201].tolist() == [1] * 4201


def test_rows_follow_others_and_norm_offset(kvg):
    """Rows behind 21 earlier ones, weights as w + 1, position tags of any value, an infinity and a NaN kept to their rows."""
    case = (1, 4, 2, 128, 16, [19], False, 128, 0, "none", True, True, 0)
    q, k, v, w, pos, m, rotary, f, _, qo = build(kvg, case)
    pos = np.array([-5, -1, 0, 2 ** 31 - 1] + list(range(1000, 1015)), np.int32)
    k[0, 3, 1, 5], q[0, 2, 0, 0] = float("inf"), float("nan")
    cache, dims = make_cache(kvg, 1, 2, 128, 16, [19], extra=21)
    old = bf16(draws(9, 1, 21, 2, 128))
    pd, po = torch.from_numpy(pos).cuda(), torch.arange(21, dtype=torch.int32).cuda()
    kvg.kvg_cache_append(cache.h, 0, old.data_ptr(), old.data_ptr(), po.data_ptr(), 21)
    qkv = kvg.make_qkv(q, k, v, *w, 1e-5, 1.0)
    kvg.kvg_cache_append_qkv(cache.h, 0, [0], [19], qkv, rotary.h, pd.data_ptr(), qo.data_ptr())
    torch.cuda.synchronize()
    assert np.array_equal(rows_of(cache, dims, 0, 21, 0, 0), f64(old[0]))
    assert np.isnan(f64(qo[0, 2, 0])).all() and np.isnan(rows_of(cache, dims, 0, 19, 0, 0, 21)[3, 1]).any()
    eps = float(np.float32(1e-5))
    ref, size = reference(f64(q[0]), f64(w[0][0]), eps, 1.0, pos, f, 0, m)
    fine = np.isfinite(ref)
    fine[2, 0] = False
    check_bf16(np.where(fine, f64(qo[0]), 0), np.where(fine, ref, 0), np.where(fine, size, 0))
    with np.errstate(invalid="ignore"):
        ref, size = reference(f64(k[0]), f64(w[1][0]), eps, 1.0, pos, f, 0, m)
    fine = np.ones_like(ref, bool)
    fine[3, 1] = False
    got = rows_of(cache, dims, 0, 19, 0, 0, 21)
    check_bf16(np.where(fine, got, 0), np.where(fine, ref, 0), np.where(fine, size, 0))
    assert np.array_equal(tables(cache)[2][0, 21:40], pos)


def test_refusals_change_nothing(kvg):
    case = (2, 4, 2, 64, 16, [10, 4], False, 64, 0, "none", True, True, 0)
    q, k, v, w, pos, m, rotary, f, qkv, qo = build(kvg, case)
    dims = kvg.make_dims(2, 2, 64, 16)
    cache = kvg.Cache(dims, 3, 3, 40)
    pd = torch.from_numpy(pos).cuda()

    def refused(status, layer=0, seqs=(0, 1), rows=(10, 4), x=qkv, rot=rotary.h, out=qo.data_ptr()):
        with pytest.raises(kvg.KvgError) as e:
            kvg.kvg_cache_append_qkv(cache.h, layer, list(seqs), list(rows), x, rot, pd.data_ptr(), out)
        assert e.value.status == status, e.value

    arg, cap = kvg.KVG_ERR_ARG, kvg.KVG_ERR_CAPACITY
    refused(arg, layer=2)
    refused(arg, layer=-2)
    refused(arg, seqs=(0, 0))
    refused(arg, seqs=(0, 3))
    refused(arg, rows=(10, -1))
    refused(arg, layer=1)                      # nothing was opened
    refused(cap, rows=(41, 1))                 # max_slots
    refused(cap, rows=(33, 17))                # pages
    refused(arg, out=None)
    refused(arg, out=qo.data_ptr() + 2)
    refused(arg, x=kvg.make_qkv(None, k, v))   # no queries, but a place for them
    wide = kvg.Rotary(128, 64)
    refused(arg, rot=wide.h)
    odd = kvg.make_qkv(q, k, v)
    odd.k_token += 4
    refused(arg, x=odd)
    assert [kvg.kvg_cache_seq_info(cache.h, b) for b in range(2)] == [(0, 0), (0, 0)]
    kvg.kvg_cache_append_qkv(cache.h, 0, [0, 1], [10, 4], qkv, rotary.h, pd.data_ptr(), qo.data_ptr())
    refused(arg, layer=1, rows=(9, 4))
    kvg.kvg_cache_append_qkv(cache.h, 1, [1, 0], [4, 10], qkv, rotary.h, pd.data_ptr(), qo.data_ptr())
    kvg.kvg_cache_append(cache.h, 1, k.data_ptr(), v.data_ptr(), pd.data_ptr(), 1)
    refused(arg, layer=1, seqs=(1,), rows=(4,))  # no longer the last rows
    kvg.kvg_cache_release(cache.h, 0)
    refused(arg, layer=1, seqs=(0,), rows=(10,))
    torch.cuda.synchronize()
    kvg.kvg_sync(cache.h)


def test_rotary_refusals():
    kvg = need_gpu()
    for bad in (dict(head_dim=96, rotary_dim=64), dict(head_dim=64, rotary_dim=80), dict(head_dim=64, rotary_dim=24),
                dict(head_dim=64, rotary_dim=-16), dict(head_dim=64, rotary_dim=64, theta=0.5),
                dict(head_dim=64, rotary_dim=64, style=2), dict(head_dim=64, rotary_dim=64, scaling=3),
                dict(head_dim=64, rotary_dim=64, scaling=1, factor=0.5),
                dict(head_dim=64, rotary_dim=64, scaling=2, factor=4.0, original_positions=0),
                dict(head_dim=64, rotary_dim=64, scaling=2, factor=4.0, original_positions=4096, beta_fast=1.0),
                dict(head_dim=64, rotary_dim=64, attention_factor=float("nan"))):
        with pytest.raises(kvg.KvgError) as e:
            kvg.Rotary(**bad)
        assert e.value.status == kvg.KVG_ERR_ARG
