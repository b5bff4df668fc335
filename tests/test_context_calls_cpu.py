"""Host-side refusals of the calls for contexts that hold more than text (axes of
rotary positions, cross attention), answered without a GPU."""
import ctypes

import pytest

from paper_2607_14431_gb300 import build, kvg


@pytest.fixture(scope="module")
def lib():
    build.build()
    return kvg.lib()


@pytest.mark.parametrize("sections,layout", [
    ([], 0), ([13, 13, 13, 13, 12], 0), ([64, -1, 1], 0), ([32, 31], 0), ([32, 33], 1), ([64], 3), ([64], -1),
    ([21, 22, 21], 1),  # pairs 1, 4, ..., 64 of 64
    ([0, 64], 1), ([2 ** 31 - 1, 2 ** 31 - 1, 66], 0),
])
def test_axes_that_are_refused(lib, sections, layout):
    for good, how in (([22, 21, 21], 1), ([24, 20, 20], 1), ([0, 64], 2), ([64, 0, 0, 0], 0), ([32, 32], 1)):
        kvg.Rotary(128, 128, 1e4, sections=good, layout=how).close()
    with pytest.raises(kvg.KvgError) as e:
        kvg.Rotary(128, 128, 1e4, sections=sections, layout=layout)
    assert e.value.status == kvg.KVG_ERR_ARG


def test_descriptions_are_checked_with_axes_too(lib):
    for fields in ({"head_dim": 96}, {"rotary_dim": 24}, {"style": 2}, {"theta": 0.5}, {"scaling": 1, "factor": 0.5}):
        with pytest.raises(kvg.KvgError):
            kvg.Rotary(**({"head_dim": 128, "rotary_dim": 128, "sections": [32, 32]} | fields))


def test_null_arguments(lib):
    h, scale, d = ctypes.c_void_p(), ctypes.c_float(1.0), kvg.kvg_rotary_desc(128, 128, 0, 0, 1e4)
    pairs = (ctypes.c_int32 * 1)(64)
    assert lib.kvg_rotary_create_axes(None, pairs, 1, 0, ctypes.byref(h)) == kvg.KVG_ERR_ARG
    assert lib.kvg_rotary_create_axes(ctypes.byref(d), None, 1, 0, ctypes.byref(h)) == kvg.KVG_ERR_ARG
    assert lib.kvg_rotary_create_axes(ctypes.byref(d), pairs, 1, 0, None) == kvg.KVG_ERR_ARG
    assert lib.kvg_cross_attention(None, 0, None, None, 1, None, 4, None, scale, None) == kvg.KVG_ERR_ARG


def test_the_binding_asks_for_a_count_per_sequence():
    with pytest.raises(ValueError):
        kvg.kvg_cross_attention(None, 0, [0], [1, 2], 0, 4, 0, 1.0)


def test_eviction_refusals(lib):
    ids = (ctypes.c_int32 * 1)(0)
    w = ctypes.c_void_p(16)
    assert lib.kvg_cache_evict(None, ids, None, ids, 1, 0, 0, w, None) == kvg.KVG_ERR_ARG
    with pytest.raises(ValueError):
        kvg.kvg_cache_evict(None, [0], [1, 2], 0, 0, 16)
    with pytest.raises(ValueError):
        kvg.kvg_cache_evict(None, [0], [1], 0, 0, 16, dst_ids=[1, 2])


def test_weights_refusals(lib):
    f = ctypes.c_float(1.0)
    assert lib.kvg_attention_weights(None, 0, None, None, 1, None, 4, None, f, None, f, None) == kvg.KVG_ERR_ARG
    with pytest.raises(ValueError):
        kvg.kvg_attention_weights(None, 0, [0], [1, 2], 0, 4, 0, 1.0, 16, 0.0)
