"""Windowed prompts behind pages that end early (a grafted block whose rows do
not fill its last page): the rows against the definition, and key tiles that no
window reaches are left out as they are without such pages."""
import math
import statistics

import pytest
import torch

from kvg_testlib import need_gpu
from test_gpu_prompt_attention import Bed, normal, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvg():
    return need_gpu()


def behind_blocks(kvg, lens, rows, window, d=128, hkv=2, page=64, fp8=False):
    """Sequence 0: stored blocks of these lengths, then `rows` rows."""
    slots = sum(-(-n // page) * page for n in lens) + rows
    bed = Bed(kvg, 1, hkv, d, page, -(-slots // page) + -(-max(lens) // page) + 1, 2, slots + page, fp8)
    store = kvg.Store(bed.dims, kvg.KVG_RESIDENCY_HBM, 1 << 28)
    for i, n in enumerate(lens):
        bed.append(1, n, 50 + i)
        block = kvg.kvg_deposit(store.h, bed.cache.h, 1, 0, n)
        kvg.kvg_graft(store.h, block, bed.cache.h, 0)
        torch.cuda.synchronize()
        kvg.kvg_cache_release(bed.cache.h, 1)
    bed.append(0, rows, 3)
    bed.store = store
    kvg.kvg_cache_set_layer_windows(bed.cache.h, [window])
    return bed


@pytest.mark.parametrize("d,page,fp8", [(64, 16, False), (128, 64, False), (256, 48, False), (128, 64, True)])
@pytest.mark.parametrize("lens", [[75, 700], [700, 75], [75, 75, 5, 300], [1, 1, 640], [641, 1, 1]])
@pytest.mark.parametrize("window,rows", [(100, 650), (300, 420), (5000, 150)])
def test_rows_against_the_definition(kvg, d, page, fp8, lens, window, rows):
    bed = behind_blocks(kvg, lens, rows, window, d, 1, page, fp8)
    run(bed, 2, [0], [rows], window)
    run(bed, 2, [0], [rows - 33], window)


def time_of(kvg, lens, rows, window):
    bed = behind_blocks(kvg, lens, rows, window)
    q = normal(1, 1, rows, 4, 128)
    out = torch.empty_like(q)
    times = []
    for _ in range(9):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        kvg.kvg_prompt_attention(bed.cache.h, 0, [0], [rows], q.data_ptr(), 4, out.data_ptr(), 1 / math.sqrt(128))
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b))
    return statistics.median(times)


@pytest.mark.parametrize("lens", [[5000, 2048], [5000, 640]])
def test_a_page_that_ends_early_costs_no_more_key_tiles(kvg, lens):
    """Behind the window of every row, and in the first rows' windows: 16,384 rows with windows of 1,024 see some
    10 key tiles an item; from the first row's window on it would be up to 137."""
    full = time_of(kvg, [5056, lens[1]], 16384, 1024)  # 79 whole pages
    assert time_of(kvg, lens, 16384, 1024) < 2 * full
