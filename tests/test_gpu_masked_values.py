"""Values that are not finite reach the rows that attend to them, no others,
whatever the context's length and however many there are (bounds: the decode
gate's).  A row that attends to +inf only is +inf there, to -inf only -inf, to
both or to a NaN it is NaN."""
import math

import pytest
import torch

from kvg_testlib import dev_view, need_gpu
from test_gpu_prompt_attention import Bed, check, normal, reference

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def kvg():
    return need_gpu()


def call(bed, hq, seq, rows, q):
    out = torch.full_like(q, -7.0)
    bed.kvg.kvg_prompt_attention(bed.cache.h, 0, [seq], [rows], q.data_ptr(), hq, out.data_ptr(), 1 / math.sqrt(bed.d))
    torch.cuda.synchronize()
    bed.kvg.kvg_sync(bed.cache.h)
    return out[0]


def compare(got, ref, what):
    """The finite elements by the gate, the others by kind."""
    check(got, ref, what)
    for kind in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(kind(got.float()), kind(ref)), what


def test_a_masked_value_behind_400_000_rows(kvg):
    """More work items than SMs, so that items follow the one whose rows the value must not reach."""
    n, total, seen = 40000, 400000, 150
    bed = Bed(kvg, 1, 1, 64, 64, total // 64 + 1, 1, total)
    bed.append(0, total, 1)
    for back, value in ((seen, NAN), (seen + 700, INF), (seen + 20000, -INF)):
        bed.put(0, 0, 1, total - back, value)
    q = normal(3, 1, n, 1, 64)
    out = call(bed, 1, 0, n, q)
    for first, rows in ((n - 300, 300), (n - 900, 120), (n - 20100, 150), (0, 60)):
        at = total - n + first  # slots before the rows
        slots, k, v = bed.rows(0, 0)
        bed.rows = lambda *_, end=at + rows: (slots[:end], k[:end], v[:end])
        compare(out[first:first + rows], reference(bed, 0, 0, q[0, first:first + rows], rows, 0, 1 / 8), f"rows from {first}")
        del bed.rows


@pytest.mark.parametrize("d,g,fp8", [(64, 2, False), (128, 4, False), (256, 2, False), (128, 2, True), (256, 1, True)])
@pytest.mark.parametrize("rows,window", [(20, 0), (300, 0), (300, 130), (130, 1000)])
def test_values_of_every_kind(kvg, d, g, fp8, rows, window):
    """Few rows on 9,000 (keys are split) and several tiles of rows; the values near a mask's edge and far from it."""
    total = 9000 + rows
    bed = Bed(kvg, 1, 2, d, 64, 150, 1, 9400, fp8)
    bed.append(0, total, 1)
    if window:
        kvg.kvg_cache_set_layer_windows(bed.cache.h, [window])
    values = [NAN] if fp8 else [INF, -INF, NAN]
    for i, back in enumerate((rows // 2, rows // 3, 2, rows + 5)):
        bed.put(0, 0, 1, total - back, values[i % len(values)])
    if window:
        bed.put(0, 0, 1, total - rows - window + 12, values[0])
        bed.put(0, 0, 1, total - rows // 2 - window, values[-2 if len(values) > 1 else 0])
    q = normal(4, 1, rows, 2 * g, d)
    compare(call(bed, 2 * g, 0, rows, q), reference(bed, 0, 0, q[0], rows, window, 1 / math.sqrt(d)), "rows")


@pytest.mark.parametrize("d,fp8", [(64, False), (256, False), (128, True)])
def test_every_value_of_many_rows(kvg, d, fp8):
    """The last 200 rows' values are all NaN: the rows before them are as without."""
    bed = Bed(kvg, 1, 1, d, 48, 22, 1, 1000, fp8)
    bed.append(0, 900, 1)
    q = normal(4, 1, 500, 2, d)
    v = bed.cache.view
    table = dev_view(v.page_table, 4 * v.max_seqs * v.max_pages, torch.int32).view(v.max_seqs, -1)[0].tolist()
    for s in range(700, 900):
        bed.pool.view(torch.uint8 if fp8 else torch.int16)[0, 1, table[s // 48], :, s % 48] = 0x7f if fp8 else 0x7fc0
    out = call(bed, 2, 0, 500, q)
    assert torch.isnan(out[300:].float()).all()
    compare(out, reference(bed, 0, 0, q[0], 500, 0, 1 / math.sqrt(d)), "rows")
