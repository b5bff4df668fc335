"""Host-side refusals of the forward pass's calls (rotary descriptions, null
arguments, row counts), answered without a GPU."""
import ctypes

import pytest

from paper_2607_14431_gb300 import build, kvg


@pytest.fixture(scope="module")
def lib():
    build.build()
    return kvg.lib()


@pytest.mark.parametrize("fields", [
    {"head_dim": 96}, {"rotary_dim": 136}, {"rotary_dim": 24}, {"rotary_dim": -16}, {"style": 2}, {"scaling": 3},
    {"theta": 0.5}, {"theta": float("nan")}, {"theta": float("inf")},
    {"scaling": kvg.KVG_ROPE_SCALING_LINEAR, "factor": 0.5},
    {"scaling": kvg.KVG_ROPE_SCALING_LINEAR, "factor": float("nan")},
    {"scaling": kvg.KVG_ROPE_SCALING_YARN, "factor": 4.0, "original_positions": 0},
])
def test_rotary_descriptions_that_are_refused(lib, fields):
    kvg.Rotary(128, 128, 1e4).close()
    with pytest.raises(kvg.KvgError) as e:
        kvg.Rotary(**({"head_dim": 128, "rotary_dim": 128} | fields))
    assert e.value.status == kvg.KVG_ERR_ARG


def test_null_arguments(lib):
    h, scale = ctypes.c_void_p(), ctypes.c_float(1.0)
    assert lib.kvg_rotary_create(None, ctypes.byref(h)) == kvg.KVG_ERR_ARG
    lib.kvg_rotary_destroy(None)
    qkv = kvg.kvg_qkv()
    assert lib.kvg_cache_append_qkv(None, 0, None, None, 1, ctypes.byref(qkv), None, None, None,
                                    None) == kvg.KVG_ERR_ARG
    assert lib.kvg_prompt_attention(None, 0, None, None, 1, None, 4, None, scale, None) == kvg.KVG_ERR_ARG
    assert lib.kvg_decode_attention_shared(None, 0, None, 1, None, 4, None, scale, None) == kvg.KVG_ERR_ARG


def test_the_binding_asks_for_a_count_per_sequence():
    with pytest.raises(ValueError):
        kvg.kvg_cache_append_qkv(None, 0, [0, 1], [1], kvg.kvg_qkv(), None, 0, None)
    with pytest.raises(ValueError):
        kvg.kvg_prompt_attention(None, 0, [0], [1, 2], 0, 4, 0, 1.0)
