"""kvg_cache_append_qkv with positions on several axes against the formula in 64
bits, written out pair by pair.  The bounds are those of one axis
(test_gpu_append_qkv): only the position that a pair's frequency is multiplied
with differs."""
import numpy as np
import pytest
import torch

from kvg_testlib import need_gpu
from test_gpu_append_qkv import bf16, check_bf16, check_e4m3, draws, f64, make_cache, rows_of, tables

pytestmark = pytest.mark.gpu
SECTIONS, TURNS, OWN = 0, 1, 2


@pytest.fixture(scope="module")
def kvg():
    return need_gpu()


def pairs_of(sections, layout, theta):
    """(axis, frequency) of each pair."""
    n, total = len(sections), sum(sections)
    if layout == TURNS:
        left = list(sections)
        axis = []
        for i in range(total):
            a = i % n
            if a and left[a] == 0:
                a = 0
            left[a] -= 1
            axis.append(a)
        return axis, [theta ** (-i / total) for i in range(total)]
    axis = [a for a, s in enumerate(sections) for _ in range(s)]
    if layout == SECTIONS:
        return axis, [theta ** (-i / total) for i in range(total)]
    return axis, [theta ** (-j / s) for s in sections for j in range(s)]


def turned(x, w, eps, angle, interleaved):
    """(value, |a| + |b| of its pair) of heads x [T][H][D], angles [T][pairs]."""
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w if w is not None else x.copy()
    size, n = np.abs(y), angle.shape[1]
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        c, s = np.cos(angle[:, i])[:, None], np.sin(angle[:, i])[:, None]
        ya, yb = y[..., a].copy(), y[..., b].copy()
        y[..., a], y[..., b] = ya * c - yb * s, yb * c + ya * s
        size[..., a] = size[..., b] = np.abs(ya) + np.abs(yb)
    return y, size


# layers, Hq, Hkv, D, page, rows per sequence, fp8, sections, layout, style, norm, places from
CASES = [
    (2, 4, 2, 64, 16, [5, 0, 37, 1], False, [8, 12, 12], SECTIONS, 0, True, 0),
    (1, 4, 4, 64, 7, [130], True, [12, 10, 10], TURNS, 1, True, 100),
    (2, 32, 16, 128, 64, [1, 1, 1], False, [16, 24, 24], SECTIONS, 0, True, 30000),
    (1, 8, 2, 128, 24, [65, 64, 63], True, [32, 32], OWN, 0, False, 7),
    (1, 8, 8, 128, 1, [9, 3], False, [2, 2, 2, 2], TURNS, 1, True, -5),
    (2, 16, 8, 256, 64, [70], False, [48, 40, 40], TURNS, 0, True, 2 ** 31 - 200),
    (1, 2, 1, 256, 80, [161, 2], True, [10, 0, 54, 64], OWN, 1, True, 131072),
    (1, 0, 2, 64, 16, [20], False, [0, 32], SECTIONS, 0, True, -2 ** 31),
    (1, 96, 4, 256, 16, [3], False, [56], SECTIONS, 0, True, 1),
    (1, 4, 2, 64, 16, [2000, 7, 513], False, [24, 8], SECTIONS, 0, True, 0),
]


@pytest.mark.parametrize("case", CASES, ids=[f"{c[3]}p{c[4]}{'fp8' if c[6] else ''}x{len(c[7])}l{c[8]}" for c in CASES])
def test_rows_and_queries(kvg, case):
    n_l, hq, hkv, d, page, rows, fp8, sections, layout, style, norm, at = case
    t, eps = sum(rows), float(np.float32(1e-5))
    x = bf16(draws(3, n_l, t, hq + 2 * hkv, d))
    q, k, v = x.split([hq, hkv, hkv], dim=2)
    wq, wk = (bf16(1 + 0.2 * draws(4 + i, n_l, d)) for i in range(2))
    places = (at + np.random.default_rng(5).integers(0, 200, (len(sections), t))).astype(np.int32)
    rotary = kvg.Rotary(d, 2 * sum(sections), 1e4, style, sections=sections, layout=layout)
    qkv = kvg.make_qkv(q if hq else None, k, v, wq if norm and hq else None, wk if norm else None, 1e-5, 0.0)
    qo = torch.zeros(n_l, t, hq, d, dtype=torch.bfloat16, device="cuda")
    cache, dims = make_cache(kvg, n_l, hkv, d, page, rows, fp8, style)
    pd = torch.from_numpy(places).cuda()
    kvg.kvg_cache_append_qkv(cache.h, -1, list(range(len(rows))), rows, qkv, rotary.h, pd.data_ptr(),
                             qo.data_ptr() if hq else None)
    torch.cuda.synchronize()
    axis, f = pairs_of(sections, layout, 1e4)
    angle = places[axis].T.astype(np.float64) * np.array(f)
    for l in range(n_l):
        if hq:
            check_bf16(f64(qo[l]), *turned(f64(q[l]), f64(wq[l]) if norm else None, eps, angle, style))
        ref, size = turned(f64(k[l]), f64(wk[l]) if norm else None, eps, angle, style)
        val, first = f64(v[l]), 0
        for b, n in enumerate(rows):
            if n:
                gk, gv = (rows_of(cache, dims, b, n, l, kv) for kv in (0, 1))
                if fp8:
                    check_e4m3(gk, ref[first:first + n], size[first:first + n], 0.0625)
                    check_e4m3(gv, val[first:first + n], np.zeros_like(gv), 0.0625)
                else:
                    check_bf16(gk, ref[first:first + n], size[first:first + n])
                    assert np.array_equal(gv, val[first:first + n])
                assert np.array_equal(tables(cache)[2][b][:n], places[0, first:first + n])  # the tags: axis 0
            first += n


@pytest.mark.parametrize("layout", [SECTIONS, TURNS, OWN])
@pytest.mark.parametrize("style", [0, 1])
def test_equal_places_and_one_axis_are_the_plain_rotary(kvg, layout, style):
    """Text: the same position on every axis gives the bits that one axis gives."""
    d, t = 128, 75
    q, k, v = bf16(draws(1, t, 8, d)).split([4, 2, 2], dim=1)
    qkv = kvg.make_qkv(q, k, v)
    pos = torch.arange(t, dtype=torch.int32, device="cuda") * 1000
    got = []
    for sections in (None, [64], [24, 20, 20]):
        if layout == OWN and sections and len(sections) > 1:
            continue  # (other frequencies)
        rotary = kvg.Rotary(d, d, 1e6, style, sections=sections, layout=layout)
        cache, dims = make_cache(kvg, 1, 2, d, 16, [t], style=style)
        out = torch.zeros(t, 4, d, dtype=torch.bfloat16, device="cuda")
        places = pos.repeat(len(sections) if sections else 1, 1).contiguous()
        kvg.kvg_cache_append_qkv(cache.h, 0, [0], [t], qkv, rotary.h, places.data_ptr(), out.data_ptr())
        torch.cuda.synchronize()
        got.append((f64(out), rows_of(cache, dims, 0, t, 0, 0)))
    for q_out, keys in got[1:]:
        assert np.array_equal(q_out, got[0][0]) and np.array_equal(keys, got[0][1])


def test_scaled_frequencies(kvg):
    """Scaling applies to each pair's own frequency."""
    d, t, sections = 64, 9, [16, 16]
    q, k, v = bf16(draws(2, t, 4, d)).split([2, 1, 1], dim=1)
    places = np.array([np.arange(t) * 37, np.arange(t)[::-1] * 911], np.int32)
    pd = torch.from_numpy(places).cuda()
    for scaling in (1, 2):
        rotary = kvg.Rotary(d, d, 1e4, 0, scaling, 8.0, 4096, 32.0, 1.0, sections=sections, layout=OWN)
        cache, dims = make_cache(kvg, 1, 1, d, 16, [t])
        out = torch.zeros(t, 2, d, dtype=torch.bfloat16, device="cuda")
        kvg.kvg_cache_append_qkv(cache.h, 0, [0], [t], kvg.make_qkv(q, k, v), rotary.h, pd.data_ptr(), out.data_ptr())
        torch.cuda.synchronize()
        axis, f = pairs_of(sections, OWN, 1e4)
        f = np.array(f)
        keep = np.clip((4096 * f / (2 * np.pi) - 1) / 31, 0, 1) if scaling == 2 else 0.0
        angle = places[axis].T * (f / 8 * (1 - keep) + f * keep)
        check_bf16(f64(out), *turned(f64(q), None, 0, angle, False))
        check_bf16(rows_of(cache, dims, 0, t, 0, 0), *turned(f64(k), None, 0, angle, False))


def test_more_segments_than_a_launch_takes(kvg):
    """Positions are found by axis over all the call's tokens, in its second launch too."""
    d, n = 64, 300
    rows = [1 + b % 3 for b in range(n)]
    t = sum(rows)
    q, k, v = bf16(draws(6, t, 4, d)).split([2, 1, 1], dim=1)
    places = np.random.default_rng(7).integers(0, 5000, (3, t)).astype(np.int32)
    pd = torch.from_numpy(places).cuda()
    cache, dims = make_cache(kvg, 1, 1, d, 16, rows)
    out = torch.zeros(t, 2, d, dtype=torch.bfloat16, device="cuda")
    rotary = kvg.Rotary(d, d, 1e4, sections=[12, 10, 10], layout=TURNS)
    kvg.kvg_cache_append_qkv(cache.h, 0, list(range(n)), rows, kvg.make_qkv(q, k, v), rotary.h, pd.data_ptr(),
                             out.data_ptr())
    torch.cuda.synchronize()
    axis, f = pairs_of([12, 10, 10], TURNS, 1e4)
    check_bf16(f64(out), *turned(f64(q), None, 0, places[axis].T * np.array(f), False))


def test_layers_one_by_one(kvg):
    """Layer 0 opens the rows with tags of axis 0, the others fill them."""
    d, t, n_l = 128, 33, 3
    x = bf16(draws(8, n_l, t, 8, d))
    places = torch.from_numpy(np.random.default_rng(9).integers(0, 500, (2, t)).astype(np.int32)).cuda()
    rotary = kvg.Rotary(d, 64, 1e4, sections=[20, 12])
    pools = []
    for one_by_one in (False, True):
        cache, dims = make_cache(kvg, n_l, 2, d, 16, [t])
        out = torch.zeros(n_l, t, 4, d, dtype=torch.bfloat16, device="cuda")
        if one_by_one:
            for l in (0, 2, 1):
                q, k, v = x[l].split([4, 2, 2], dim=1)
                kvg.kvg_cache_append_qkv(cache.h, l, [0], [t], kvg.make_qkv(q, k, v), rotary.h, places.data_ptr(),
                                         out[l].data_ptr())
        else:
            q, k, v = x.split([4, 2, 2], dim=2)
            kvg.kvg_cache_append_qkv(cache.h, -1, [0], [t], kvg.make_qkv(q, k, v), rotary.h, places.data_ptr(),
                                     out.data_ptr())
        torch.cuda.synchronize()
        pools.append([f64(out)] + [rows_of(cache, dims, 0, t, l, 0) for l in range(n_l)])
    assert all(np.array_equal(a, b) for a, b in zip(*pools))
