"""Relocated grafts (delta != 0) of rows that were appended with positions on several
axes: the graft turns a whole head by one position, which is what moving every
axis by delta does where each pair has the frequency that one axis would give it."""
import numpy as np
import pytest
import torch

from kvg_testlib import need_gpu
from test_gpu_append_qkv import FP32, bf16, draws, f64, half_step, make_cache, rows_of, tables
from test_gpu_rotary_axes import OWN, SECTIONS, TURNS, pairs_of, turned

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvg():
    return need_gpu()


def relocated(kvg, layout, sections, style, delta, scaling=0):
    """(tags, keys of the relocated graft, keys in 64 bits with every axis moved by delta, |a| + |b| of each pair)."""
    d, t, page = 2 * sum(sections), 100, 16
    k, v = bf16(draws(11, t, 2, d)), bf16(draws(12, t, 2, d))
    places = np.random.default_rng(13).integers(0, 300, (len(sections), t)).astype(np.int32)
    cache, dims = make_cache(kvg, 1, 2, d, page, [t, t], style=style)
    rotary = kvg.Rotary(d, d, 1e4, style, scaling, 4.0 if scaling else 1.0, sections=sections, layout=layout)
    pd = torch.from_numpy(places).cuda()
    kvg.kvg_cache_append_qkv(cache.h, 0, [0], [t], kvg.make_qkv(None, k, v), rotary.h, pd.data_ptr(), None)
    store = kvg.Store(dims, kvg.KVG_RESIDENCY_HBM, 1 << 24)
    block = kvg.kvg_deposit(store.h, cache.h, 0, 0, t)
    kvg.kvg_graft(store.h, block, cache.h, 1, -1, delta, kvg.KVG_GRAFT_SYNC)
    torch.cuda.synchronize()
    axis, f = pairs_of(sections, layout, 1e4)
    angle = (places[axis].T.astype(np.float64) + delta) * np.array(f) / (4.0 if scaling else 1.0)
    tags = tables(cache)[2][1][:t]
    assert np.array_equal(tags, places[0] + delta)
    assert np.array_equal(rows_of(cache, dims, 1, t, 0, 1), f64(v))
    return rows_of(cache, dims, 1, t, 0, 0), *turned(f64(k), None, 0, angle, style)


def excess(got, ref, size):
    """How far the keys are beyond their two roundings to bf16: the stored key's two components, each at most half a
    step of |a| + |b|, turned (|cos| + |sin| <= sqrt 2), then half a step of the value, which may lie beside a
    power of two; each rotation 2^-19 of |a| + |b|."""
    first = np.sqrt(2) * half_step(size, 7)
    return np.abs(got - ref) - first - half_step(np.abs(ref) + first, 7) - 2 * FP32 * size


@pytest.mark.parametrize("delta", [1, 4096, 100000])
@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("layout,sections", [(SECTIONS, [16, 24, 24]), (TURNS, [24, 20, 20]), (SECTIONS, [12, 20]),
                                             (OWN, [64])])
def test_every_axis_moves_by_delta(kvg, layout, sections, style, delta):
    assert excess(*relocated(kvg, layout, sections, style, delta)).max() <= 0


@pytest.mark.parametrize("layout,sections,scaling", [(OWN, [32, 32], 0), (SECTIONS, [16, 24, 24], 1)])
def test_other_frequencies_do_not_fit(kvg, layout, sections, scaling):
    """Ladders of their own and scaled frequencies are not the ones that the graft turns by: no refusal, other keys."""
    assert excess(*relocated(kvg, layout, sections, 0, 4096, scaling)).max() > 0.5
