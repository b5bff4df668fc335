"""Which launches a decode on a shared block takes: the common pages get their
own where the rows' windows leave enough of them to be read again, counted per
window, by default from 120 MB on."""
import os
import subprocess
import sys

import pytest
import torch

from kvg_testlib import need_gpu
from test_gpu_prompt_attention import normal
from test_gpu_shared_decode import Shared

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvg():
    return need_gpu()


def launches(bed, call, hq, seqs, layer, q):
    """Output and launches of a call that has run before."""
    bed.decode(call, hq, seqs, layer, 0.1, q)
    n = bed.kvg.kvg_launch_count()
    return bed.decode(call, hq, seqs, layer, 0.1, q), bed.kvg.kvg_launch_count() - n


def both(bed, hq, seqs, layer, seed=4):
    q = normal(seed, bed.dims.n_layers if layer < 0 else 1, len(seqs), hq, bed.d)
    return [launches(bed, c, hq, seqs, layer, q) for c in ("kvg_decode_attention", "kvg_decode_attention_shared")]


@pytest.mark.parametrize("tails", [[100, 250, 130], [100, 60, 130]])
def test_windows_that_leave_nothing_to_share_are_the_decode(kvg, tails):
    """No row's window reaches the block, or one row's does."""
    bed = Shared(kvg, 2, 2, 128, 64, 3, [1000], 300)
    for b, n in enumerate(tails):
        bed.give(b, 0, n, 10 * b)
    kvg.kvg_cache_set_layer_windows(bed.cache.h, [100, 100])
    (want, n), (got, m) = both(bed, 4, [0, 1, 2], -1)
    assert m == n and torch.equal(want.view(torch.int16), got.view(torch.int16))
    bed.verify(4, [0, 1, 2], [100, 100])


@pytest.mark.parametrize("windows,prompts", [([0, 100, 0, 100], 1), ([100, 0, 500, 600], 3), ([100, 90, 40, 30], 0)])
def test_each_window_is_counted_by_itself(kvg, windows, prompts):
    """Only layers whose windows reach the block read it with all rows at once."""
    bed = Shared(kvg, 4, 2, 128, 64, 4, [1500], 300)
    for b, n in enumerate([100, 140, 250, 300]):
        bed.give(b, 0, n, 10 * b)
    kvg.kvg_cache_set_layer_windows(bed.cache.h, windows)
    (_, n), (_, m) = both(bed, 4, [0, 1, 2, 3], -1)
    assert m == n + prompts
    bed.verify(4, [0, 1, 2, 3], windows)


def test_groups_of_which_a_window_reaches_one(kvg):
    bed = Shared(kvg, 2, 1, 256, 64, 6, [900, 1300], 400, True)
    for b in range(6):
        bed.give(b, b % 2, [30, 380, 20, 390, 10, 400][b], 10 * b)
    windows = [350, 0]
    kvg.kvg_cache_set_layer_windows(bed.cache.h, windows)
    bed.verify(2, [0, 1, 2, 3, 4, 5], windows)
    bed.verify(2, [5, 0, 3, 2], windows)


DEFAULT = """
import os, sys
sys.path.insert(0, {tests!r})
sys.path.insert(0, {root!r})
from kvg_testlib import need_gpu
kvg = need_gpu()
import test_gpu_shared_windows as t
from kvg_testlib import compare_decode
os.environ.pop("KVG_SHARED_MIN_KB", None)
bed = t.Shared(kvg, 1, 8, 256, 64, 32, [8192, 4096], 600)
for b in range(32):
    bed.give(b, 0, 600, 10 * b)
seqs = list(range(32))
for window, more in ((0, 1), (1024, 0), (1100, 1), (600, 0)):
    # 31 rows x (window - 600) slots x 8 KB: 2,032 MB, 108, 127 and nothing
    kvg.kvg_cache_set_layer_windows(bed.cache.h, [window])
    (want, n), (got, m) = t.both(bed, 16, seqs, 0)
    assert m == n + more, (window, n, m)
    assert (want.float() - got.float()).abs().max() < 1e-2
    assert more or t.torch.equal(want.view(t.torch.int16), got.view(t.torch.int16))
kvg.kvg_cache_set_layer_windows(bed.cache.h, [0])
for b in range(5):
    kvg.kvg_cache_release(bed.cache.h, b)
    bed.give(b, 1, 7 * b + 1, 10 * b)
for rows, more in ((4, 0), (5, 1)):  # 101 MB, 134
    (want, n), (got, m) = t.both(bed, 16, list(range(rows)), 0)
    assert m == n + more, (rows, n, m)
    assert (want.float() - got.float()).abs().max() < 1e-2
print("as it should be")
"""


def test_the_default_rule(kvg):
    """In a process without KVG_SHARED_MIN_KB, which is read once."""
    tests = os.path.dirname(os.path.abspath(__file__))
    code = DEFAULT.format(tests=tests, root=os.path.dirname(tests))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "as it should be" in r.stdout, r.stdout + r.stderr
