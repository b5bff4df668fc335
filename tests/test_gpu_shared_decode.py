"""kvg_decode_attention_shared against its definition in 64 bits over each
sequence's rows (bounds: the decode gate's), for batches whose sequences were
given the same pool-resident block."""
import math
import os

import pytest
import torch

from kvg_testlib import need_gpu
from test_gpu_prompt_attention import Bed, check, normal, reference

pytestmark = pytest.mark.gpu
os.environ.setdefault("KVG_SHARED_MIN_KB", "1")  # the launches for common pages also where they do not pay


@pytest.fixture(scope="module")
def kvg():
    return need_gpu()


class Shared(Bed):
    """Sequences 0 .. n-1 on pool-resident blocks; the last sequence makes the blocks."""

    def __init__(self, kvg, n_layers, hkv, d, page, n, prefixes, tail, fp8=False):
        pages = sum(2 * (-(-x // page)) for x in prefixes) + n * (-(-tail // page) + 2) + 1
        super().__init__(kvg, n_layers, hkv, d, page, pages, n + 1, sum(prefixes) + tail + page * (len(prefixes) + 1), fp8)
        self.store = kvg.PoolStore(self.cache, 1 << 26)
        self.blocks = []
        for i, x in enumerate(prefixes):
            self.append(n, x, 1000 + 7 * i)
            self.blocks.append(kvg.kvg_deposit(self.store.h, self.cache.h, n, 0, x))
            kvg.kvg_cache_release(self.cache.h, n)

    def give(self, seq, block, tail, seed):
        if block is not None:
            self.kvg.kvg_graft(self.store.h, self.blocks[block], self.cache.h, seq)
        self.append(seq, tail, seed)

    def decode(self, call, hq, seqs, layer, scale, q, stream=None):
        out = torch.full_like(q, float("nan"))
        getattr(self.kvg, call)(self.cache.h, layer, seqs, q.data_ptr(), hq, out.data_ptr(), scale, stream=stream)
        torch.cuda.synchronize()
        self.kvg.kvg_sync(self.cache.h)
        return out

    def verify(self, hq, seqs, windows=None, layer=-1, scale=None, seed=5, q=None):
        n_l = self.dims.n_layers if layer < 0 else 1
        scale = 1 / math.sqrt(self.d) if scale is None else scale
        q = normal(seed, n_l, len(seqs), hq, self.d) if q is None else q
        out = self.decode("kvg_decode_attention_shared", hq, seqs, layer, scale, q)
        for i in range(n_l):
            l = i if layer < 0 else layer
            for b, s in enumerate(seqs):
                if self.kvg.kvg_cache_seq_info(self.cache.h, s)[0] == 0:
                    assert not out[i, b].any()
                    continue
                check(out[i, b:b + 1], reference(self, s, l, q[i, b:b + 1], 1, (windows or [0] * 99)[l], scale),
                      f"row {b} layer {l}")
        return out


# layers, Hkv, G, D, page, prefix, tails, window, fp8
CASES = [
    (1, 2, 2, 64, 16, 256, [1, 7, 40, 16], 0, False),
    (2, 2, 1, 64, 16, 1000, [1, 90], 0, False),
    (1, 1, 8, 64, 64, 700, list(range(1, 40)), 0, False),
    (2, 2, 2, 128, 64, 4096, [3, 64, 65, 200, 1], 0, False),
    (1, 2, 4, 128, 64, 3000, [5 * i + 1 for i in range(33)], 0, False),
    (1, 1, 2, 128, 64, 2048, [i % 70 + 1 for i in range(130)], 0, False),
    (2, 2, 2, 256, 64, 2048, [9, 130, 1], 0, False),
    (1, 1, 1, 256, 48, 1500, [i + 1 for i in range(140)], 0, False),
    (1, 2, 2, 128, 64, 3000, [17, 1, 300], 0, True),
    (2, 1, 2, 256, 16, 1999, [1, 2, 3, 4, 5], 0, True),
    (1, 2, 4, 128, 64, 1111, [i + 1 for i in range(70)], 0, True),
    (1, 2, 2, 128, 64, 1000, [3, 70, 300, 600], 500, False),
    (1, 1, 2, 256, 64, 1000, [1, 90, 130], 100, True),
    (1, 2, 2, 64, 16, 512, [1, 40], 16, False),
    (1, 2, 2, 128, 7, 400, [1, 20, 9], 0, False),
    (1, 1, 2, 128, 100, 950, [1, 20, 150], 300, False),
    (1, 1, 2, 256, 200, 1300, [1, 20, 250], 0, False),
    (1, 2, 2, 64, 1, 90, [1, 20], 0, False),
]


@pytest.mark.parametrize("case", CASES, ids=[f"L{c[0]}x{c[1]}x{c[2]}x{c[3]}p{c[4]}b{len(c[6])}w{c[7]}{'fp8' if c[8] else ''}" for c in CASES])
def test_rows_against_the_definition(kvg, case):
    n_l, hkv, g, d, page, prefix, tails, window, fp8 = case
    bed = Shared(kvg, n_l, hkv, d, page, len(tails), [prefix], max(tails), fp8)
    for b, n in enumerate(tails):
        bed.give(b, 0, n, 10 * b)
    windows = [window] * n_l
    if window:
        kvg.kvg_cache_set_layer_windows(bed.cache.h, windows)
    first = bed.verify(hkv * g, list(range(len(tails))), windows)
    again = bed.verify(hkv * g, list(range(len(tails))), windows)
    assert torch.equal(first.view(torch.int16), again.view(torch.int16))


def test_groups_loners_repeats_and_an_empty_sequence(kvg):
    bed = Shared(kvg, 2, 2, 128, 64, 12, [1500, 2000], 200)
    for b in range(11):  # 11 stays empty
        bed.give(b, [0, 1, None][b % 3], 30 + 9 * b, 10 * b)
    bed.verify(4, [3, 1, 2, 0, 4, 11, 8, 7, 9, 0, 3, 5])
    bed.verify(4, [2, 11, 5])


def test_layers_of_different_windows(kvg):
    bed = Shared(kvg, 4, 2, 128, 64, 5, [1500], 300)
    windows = [0, 1000, 64, 1000]
    kvg.kvg_cache_set_layer_windows(bed.cache.h, windows)
    for b in range(5):
        bed.give(b, 0, [1, 63, 64, 200, 300][b], 10 * b)
    every = bed.verify(4, [0, 1, 2, 3, 4], windows)
    q = normal(5, 4, 5, 4, 128)
    for l in range(4):
        bed.verify(4, [0, 1, 2, 3, 4], windows, layer=l, q=q[l:l + 1].contiguous())
    assert torch.isfinite(every.float()).all()


def test_more_rows_than_a_launch_takes(kvg):
    bed = Shared(kvg, 1, 1, 64, 16, 300, [600], 20)
    for b in range(300):
        bed.give(b, 0, b % 19 + 1, 10 * b)
    bed.verify(2, list(range(300)))


def test_blocks_one_after_the_other(kvg):
    """Two blocks in a row, the first not filling its last page, then a block that only some have."""
    bed = Shared(kvg, 1, 2, 128, 64, 6, [1000, 700], 100)
    for b in range(6):
        bed.give(b, 0, 0, 0)
        if b < 4:
            bed.give(b, 1, 0, 0)
        bed.append(b, 7 * b + 1, 10 * b)
    bed.verify(4, [0, 1, 2, 3, 4, 5])
    bed.verify(4, [1, 2])


def test_without_common_pages_it_is_the_decode(kvg):
    bed = Shared(kvg, 2, 2, 128, 64, 3, [100], 500)
    for b in range(3):
        bed.give(b, None, 100 + 200 * b, b)
    q = normal(3, 2, 3, 4, 128)
    outs = [bed.decode(call, 4, [2, 0, 1], -1, 0.1, q) for call in ("kvg_decode_attention_shared", "kvg_decode_attention")]
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))


@pytest.mark.parametrize("d,fp8", [(128, False), (256, True)])
def test_rows_that_are_not_finite(kvg, d, fp8):
    """A value that is not finite in the block reaches the rows whose window sees it, no others."""
    bed = Shared(kvg, 1, 1, d, 64, 4, [2000], 400, fp8)
    for b in range(4):
        bed.give(b, 0, [1, 100, 250, 400][b], 10 * b)
    kvg.kvg_cache_set_layer_windows(bed.cache.h, [600])
    bed.put(0, 0, 1, 1600, float("nan"))  # seen by the rows of lengths 2001 and 2100
    out = bed.verify(2, [0, 1, 2, 3], [600])
    assert [bool(torch.isfinite(out[0, b].float()).all()) for b in range(4)] == [False, False, True, True]
    q = normal(8, 1, 4, 2, d)
    q[0, 2, 1, 3] = float("nan")
    bed.put(0, 0, 1, 1600, 0.5)
    out = bed.decode("kvg_decode_attention_shared", 2, [0, 1, 2, 3], 0, 0.1, q)
    assert torch.isnan(out[0, 2, 1].float()).all() and int(torch.isnan(out.float()).sum()) == d


def test_scales(kvg):
    bed = Shared(kvg, 1, 2, 128, 64, 3, [1200], 100)
    for b in range(3):
        bed.give(b, 0, 30 * b + 1, 10 * b)
    for scale in (-0.1, 0.0, 3.0):
        bed.verify(4, [0, 1, 2], scale=scale)


def test_calls_on_two_streams(kvg):
    bed = Shared(kvg, 1, 2, 128, 64, 8, [5000], 300)
    for b in range(8):
        bed.give(b, 0, 30 * b + 1, 10 * b)
    q = normal(6, 2, 1, 4, 4, 128)
    seqs = [[0, 2, 4, 6], [1, 3, 5, 7]]
    want = [bed.decode("kvg_decode_attention_shared", 4, seqs[i], 0, 0.1, q[i]) for i in range(2)]
    got = torch.empty_like(q)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for i, s in enumerate(streams):
            kvg.kvg_decode_attention_shared(bed.cache.h, 0, seqs[i], q[i].data_ptr(), 4, got[i].data_ptr(), 0.1, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(want[i].view(torch.int16), got[i].view(torch.int16)) for i in range(2))


def test_refusals(kvg):
    bed = Shared(kvg, 2, 2, 64, 16, 2, [100], 20)
    for b in range(2):
        bed.give(b, 0, 5, b)
    q = normal(1, 2, 2, 4, 64)
    out = torch.zeros_like(q)

    def refused(layer=0, seqs=(0, 1), qp=q.data_ptr(), hq=4, op=out.data_ptr()):
        with pytest.raises(kvg.KvgError) as e:
            kvg.kvg_decode_attention_shared(bed.cache.h, layer, list(seqs), qp, hq, op, 0.1)
        assert e.value.status == kvg.KVG_ERR_ARG

    refused(layer=2)
    refused(seqs=(0, 3))
    refused(seqs=())
    refused(hq=5)
    refused(hq=12)
    refused(qp=None)
    refused(op=None)
    refused(qp=q.data_ptr() + 2)
    torch.cuda.synchronize()
    assert not out.any()
