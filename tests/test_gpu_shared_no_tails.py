"""Decode on a shared block whose rows have no pages of their own, or some of
them none: what the merge gets is the block's partial results alone."""
import pytest
import torch

from kvg_testlib import need_gpu
from test_gpu_shared_decode import Shared

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvg():
    return need_gpu()


@pytest.mark.parametrize("d,g,page,fp8", [(64, 8, 16, False), (128, 2, 64, False), (128, 4, 64, True), (256, 2, 48, False)])
@pytest.mark.parametrize("tails", [[0, 0, 0], [0, 5, 0, 90]])
@pytest.mark.parametrize("windows", [[0, 0], [0, 70]])
def test_rows_that_end_with_the_block(kvg, d, g, page, fp8, tails, windows):
    bed = Shared(kvg, 2, 2, d, page, len(tails), [30 * page], 100, fp8)
    for b, n in enumerate(tails):
        bed.give(b, 0, n, 10 * b)
        assert kvg.kvg_cache_seq_info(bed.cache.h, b)[0] == 30 * page + n
    kvg.kvg_cache_set_layer_windows(bed.cache.h, windows)
    seqs = list(range(len(tails)))
    first = bed.verify(2 * g, seqs, windows)
    assert torch.equal(first.view(torch.int16), bed.verify(2 * g, seqs, windows).view(torch.int16))
    bed.verify(2 * g, seqs[::-1], windows, layer=1)
