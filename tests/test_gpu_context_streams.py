"""Cross attention of a few rows and eviction in place where streams and graphs share
a cache's scratch."""
import numpy as np
import pytest
import torch

from kvg_testlib import need_gpu
from test_gpu_cross_attention import States
from test_gpu_evict import Bed, heavy_tailed
from test_gpu_prompt_attention import normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvg():
    return need_gpu()


def few(kvg, bed, seqs, rows, q, out, **kw):
    kvg.kvg_cross_attention(bed.cache.h, 0, seqs, rows, q.data_ptr(), q.shape[-2], out.data_ptr(), 0.1, **kw)


@pytest.mark.parametrize("fp8", [False, True])
def test_a_few_rows_on_two_streams(kvg, fp8):
    """Two streams that share the cache's scratch, each as on one stream."""
    bed = States(kvg, 1, 2, 128, 64, [13000, 12000], fp8)
    q = normal(6, 2, 4, 4, 128)
    want, got = torch.empty_like(q), torch.empty_like(q)
    for i in range(2):
        few(kvg, bed, [i], [4], q[i], want[i])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for i, s in enumerate(streams):
            few(kvg, bed, [i], [4], q[i], got[i], stream=s)
    torch.cuda.synchronize()
    assert torch.equal(want.view(torch.int16), got.view(torch.int16))


@pytest.mark.parametrize("fp8", [False, True])
def test_a_few_rows_in_a_graph(kvg, fp8):
    """Replays on new queries, eager calls that grow the scratch between them."""
    bed = States(kvg, 1, 2, 128, 64, [0, 9000, 333], fp8)
    q, out = normal(1, 1, 9, 4, 128), torch.zeros(1, 9, 4, 128, dtype=torch.bfloat16, device="cuda")

    def call():
        few(kvg, bed, [1, 0, 2], [4, 2, 3], q, out)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    many = normal(5, 1, 1400, 4, 128)
    for i in (2, 3):
        q.copy_(normal(i, 1, 9, 4, 128))
        call()
        want = out.clone()
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))
        assert not out[:, 4:6].any() and out[:, :4].any()
        few(kvg, bed, [2, 1, 2], [400, 700, 300], many, torch.empty_like(many))


def kept_rows(bed, seq):
    """What a sequence holds: its rows of every plane by slot, tags, weights."""
    pool, (table, _, pos), weights = bed.snapshot()
    n = bed.slots(seq)[0]
    s = np.arange(n)
    pages, at = torch.from_numpy(table[seq][s // bed.page].astype(np.int64)).cuda(), torch.from_numpy(s % bed.page).cuda()
    return pool[:, :, pages, :, at], pos[seq][:n], weights[seq][:n]


@pytest.mark.parametrize("n", [3000, 40000])
def test_eviction_in_place_on_two_streams(kvg, n):
    """Each stream thins its sequence again and again; the scratch is shared.  As on one stream."""
    held = []
    for streams in ([None] * 2, [torch.cuda.Stream() for _ in range(2)]):
        bed = Bed(kvg, 2, 2, 64, 16, 2 * (n // 16 + 1), 2, n + 16, seed=4)
        torch.manual_seed(5)
        bed.rng = np.random.default_rng(6)
        for b in range(2):
            bed.append(b, n - 7 * b)
            bed.set_weights(b, heavy_tailed(bed.rng, n - 7 * b))
        torch.cuda.synchronize()
        for keep in range(n - 100, n // 3, -(n // 11)):
            for b, s in enumerate(streams):
                kvg.kvg_cache_evict(bed.cache.h, [b], [keep - 5 * b], 4, 20, bed.weights.data_ptr(), stream=s)
        torch.cuda.synchronize()
        kvg.kvg_sync(bed.cache.h)
        held.append([kept_rows(bed, b) for b in range(2)])
    for one, two in zip(*held):
        assert torch.equal(one[0], two[0])
        assert np.array_equal(one[1], two[1]) and np.array_equal(one[2].view(np.int32), two[2].view(np.int32))


def test_eviction_waits_for_attention_on_another_stream(kvg):
    """Rows that a call on another stream still reads are thinned after it."""
    bed = States(kvg, 1, 4, 128, 64, [30000])
    weights = torch.rand(1, bed.cache.view.max_slots, device="cuda")
    q = normal(7, 1, 3000, 8, 128)
    want, got = torch.empty_like(q), torch.empty_like(q)
    few(kvg, bed, [0], [3000], q, want)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    few(kvg, bed, [0], [3000], q, got, stream=streams[0])
    kvg.kvg_cache_evict(bed.cache.h, [0], [1000], 4, 20, weights.data_ptr(), stream=streams[1])
    torch.cuda.synchronize()
    kvg.kvg_sync(bed.cache.h)
    assert torch.equal(want.view(torch.int16), got.view(torch.int16))
    assert kvg.kvg_cache_seq_info(bed.cache.h, 0)[0] == 1000
