"""kvg_cross_attention against its definition in 64 bits over the cache's own
rows.  The bounds are those of the decode gate (kvg_testlib.compare_decode), as
for prompts: the kernel and its roundings are the same."""
import math

import numpy as np
import pytest
import torch

from kvg_testlib import need_gpu
from test_gpu_prompt_attention import Bed, check, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvg():
    return need_gpu()


def reference(bed, seq, layer, q, window, scale):
    """[n][Hq][D]: every row over the sequence's last `window` valid rows."""
    if not bed.total[seq]:
        return torch.zeros(q.shape, dtype=torch.float64)
    slots, k, v = bed.rows(seq, layer)
    if window:
        k, v = k[-window:], v[-window:]
    g = q.shape[1] // bed.hkv
    x = torch.einsum("nhd,khd->hnk", q.double(), k.repeat_interleave(g, 1)) * scale
    return torch.einsum("hnk,khd->nhd", torch.softmax(x, -1), v.repeat_interleave(g, 1))


class States(Bed):
    def __init__(self, kvg, n_layers, hkv, d, page, total, fp8=False, extra=2):
        super().__init__(kvg, n_layers, hkv, d, page, sum(-(-n // page) for n in total) + extra, len(total),
                         max(max(total), 1) + page, fp8)
        self.total = list(total)
        for b, n in enumerate(total):
            self.append(b, n, 10 * b)


def run(bed, hq, seqs, rows, window=0, layer=0, scale=None, seed=77, q=None, **kw):
    kvg, n_l = bed.kvg, bed.dims.n_layers if layer < 0 else 1
    scale = 1 / math.sqrt(bed.d) if scale is None else scale
    q = normal(seed, n_l, sum(rows), hq, bed.d) if q is None else q
    out = torch.full_like(q, float("nan"))
    kvg.kvg_cross_attention(bed.cache.h, layer, seqs, rows, q.data_ptr(), hq, out.data_ptr(), scale, **kw)
    torch.cuda.synchronize()
    kvg.kvg_sync(bed.cache.h)
    windows = window if isinstance(window, list) else [window] * bed.dims.n_layers
    for i in range(n_l):
        at, l = 0, i if layer < 0 else layer
        for s, n in zip(seqs, rows):
            if n:
                check(out[i, at:at + n], reference(bed, s, l, q[i, at:at + n], windows[l], scale), f"seq {s} layer {l}")
            at += n
    return out


# Hkv, G, D, page, window, fp8, (states, rows) of each sequence
CASES = [
    (2, 2, 64, 16, 0, False, [(256, 37), (7, 5)]),
    (1, 8, 64, 64, 0, False, [(1000, 150), (1, 1), (3, 200)]),
    (2, 1, 64, 16, 50, False, [(300, 129), (20, 64)]),
    (2, 2, 128, 64, 0, False, [(700, 257), (128, 128), (1, 127)]),
    (2, 4, 128, 64, 100, False, [(500, 200), (99, 65), (100, 3)]),
    (1, 1, 128, 128, 0, False, [(130, 513)]),
    (2, 2, 256, 64, 0, False, [(300, 199), (65, 130)]),
    (1, 1, 256, 16, 64, False, [(100, 260)]),
    (2, 2, 128, 64, 0, True, [(500, 200), (33, 33)]),
    (1, 4, 128, 16, 70, True, [(200, 150)]),
    (2, 1, 256, 64, 0, True, [(290, 200), (64, 64)]),
    (1, 2, 256, 48, 33, True, [(150, 90)]),
    # pages that are no multiple of 8 rows, of one row, and past a tile
    (2, 2, 128, 7, 0, False, [(40, 90), (14, 14)]),
    (2, 2, 64, 1, 0, False, [(30, 40)]),
    (1, 2, 256, 129, 0, False, [(400, 200)]),
    (1, 1, 128, 300, 64, True, [(299, 150)]),
]


@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}x{c[1]}x{c[2]}p{c[3]}w{c[4]}{'fp8' if c[5] else ''}" for c in CASES])
def test_rows_against_the_definition(kvg, case):
    hkv, g, d, page, window, fp8, lens = case
    bed = States(kvg, 1, hkv, d, page, [s for s, _ in lens], fp8)
    if window:
        kvg.kvg_cache_set_layer_windows(bed.cache.h, [window])
    args = bed, hkv * g, list(range(len(lens))), [n for _, n in lens], window
    assert torch.equal(run(*args).view(torch.int16), run(*args).view(torch.int16))


@pytest.mark.parametrize("d,g,fp8", [(64, 2, False), (128, 2, False), (256, 1, False), (128, 4, True), (256, 2, True)])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 127, 128, 129, 257])
def test_lengths_around_the_tiles(kvg, d, g, fp8, n):
    """States and rows of n; rows on one state; one row's worth beside many."""
    bed = States(kvg, 1, 1, d, 64, [n, 1, 700], fp8)
    run(bed, g, [0, 1, 2], [n, n, 1])
    run(bed, g, [2, 0], [n, 3])


@pytest.mark.parametrize("hkv,g,d,page,fp8", [
    (2, 1, 64, 16, False), (2, 2, 64, 64, False), (1, 8, 64, 24, False), (2, 4, 64, 7, False),
    (3, 2, 128, 64, False), (2, 4, 128, 16, False), (1, 1, 128, 48, False), (2, 1, 256, 64, False), (2, 2, 256, 16, False),
    (2, 2, 128, 64, True), (1, 4, 128, 16, True), (2, 1, 128, 32, True), (2, 2, 256, 64, True), (1, 1, 256, 48, True)])
def test_a_few_rows_each(kvg, hkv, g, d, page, fp8):
    """Rows that the decode kernel takes, all of a sequence's at once or (fp8, long states) in two turns."""
    total = [1, 900, 33, 0, 2100, 64, 1500]
    bed = States(kvg, 2, hkv, d, page, total, fp8)
    most = 8 // g
    rng = np.random.default_rng(d + g)
    for rows in ([most] * 7, list(rng.integers(0, most + 1, 7)), [0, most, 0, 1, 0, 0, most]):
        rows = [int(x) for x in rows]
        args = bed, hkv * g, [0, 1, 2, 3, 4, 5, 6], rows
        assert torch.equal(run(*args, layer=-1).view(torch.int16), run(*args, layer=-1).view(torch.int16))
        kvg.kvg_cache_set_layer_windows(bed.cache.h, [100, 0])
        run(*args, [100, 0], layer=-1)
        run(*args, 100, layer=0)
        kvg.kvg_cache_set_layer_windows(bed.cache.h, [])
    run(bed, hkv * g, [4, 6, 1], [2 * most, most + 1, 1])
    run(bed, hkv * g, [4, 4, 0, 4], [most, 1, most, most])


def test_a_few_rows_of_many_sequences(kvg):
    n = 300
    bed = States(kvg, 1, 1, 128, 16, [(b * 37) % 90 for b in range(n)])
    run(bed, 2, list(range(n)), [(b * 13) % 5 for b in range(n)])


def test_a_few_rows_on_grafted_blocks(kvg):
    bed = Bed(kvg, 1, 2, 128, 64, 40, 3, 1024)
    store = kvg.Store(bed.dims, kvg.KVG_RESIDENCY_HBM, 1 << 28)
    bed.append(2, 150, 1)
    block = kvg.kvg_deposit(store.h, bed.cache.h, 2, 0, 75)
    for _ in range(3):
        kvg.kvg_graft(store.h, block, bed.cache.h, 0)
    bed.total = [225, 0, 150]
    for window in (0, 70):
        kvg.kvg_cache_set_layer_windows(bed.cache.h, [window])
        run(bed, 4, [0, 1, 2], [4, 3, 2], window)


def test_states_of_no_rows(kvg):
    """Rows of an empty sequence get zeros, among others and alone, in every layer."""
    bed = States(kvg, 2, 2, 128, 64, [0, 100, 0], extra=4)
    out = run(bed, 4, [0, 1, 2], [3, 4, 2], layer=-1)  # (few)
    assert not out[:, :3].any() and not out[:, 7:].any() and out[:, 3:7].all(-1).all()
    out = run(bed, 4, [0, 1, 2, 0], [3, 5, 70, 0], layer=-1)
    assert not out[:, :3].any() and not out[:, 8:].any() and out[:, 3:8].all(-1).all()
    assert not run(bed, 4, [0, 2], [2, 2]).any()
    assert not run(bed, 4, [0], [1]).any()


def test_rows_past_2_gib_of_a_layer_without_states(kvg):
    bed = States(kvg, 2, 8, 256, 64, [0, 70])
    n, hq = [262_150, 3], 16  # a layer's outputs: 2^31 bytes and more
    q = torch.zeros(2, sum(n), hq, 256, dtype=torch.bfloat16, device="cuda")
    q[:, -3:] = normal(3, 2, 3, hq, 256)
    out = torch.full_like(q, float("nan"))
    kvg.kvg_cross_attention(bed.cache.h, -1, [0, 1], n, q.data_ptr(), hq, out.data_ptr(), 1 / 16)
    torch.cuda.synchronize()
    kvg.kvg_sync(bed.cache.h)
    assert not out[:, :-3].any()
    for l in range(2):
        check(out[l, -3:], reference(bed, 1, l, q[l, -3:], 0, 1 / 16), f"layer {l}")


def test_a_sequence_named_more_than_once(kvg):
    bed = States(kvg, 1, 2, 128, 64, [333, 90])
    q = normal(4, 1, 60, 4, 128)
    run(bed, 4, [0, 1, 0, 0], [17, 3, 1, 39], q=q)


@pytest.mark.parametrize("d,g,fp8", [(128, 2, False), (256, 2, False), (128, 2, True), (64, 4, False)])
def test_few_rows_on_long_states(kvg, d, g, fp8):
    """Key ranges of the one sequence's few rows on many SMs."""
    bed = States(kvg, 1, 2, d, 64, [20001, 40], fp8)
    run(bed, 2 * g, [0, 1], [5, 2])
    run(bed, 2 * g, [1, 0], [300, 2])


@pytest.mark.parametrize("fp8", [False, True])
def test_many_rows_of_empty_and_short_states_beside_long_ones(kvg, fp8):
    bed = States(kvg, 2, 2, 128, 64, [0, 5000, 3], fp8)
    run(bed, 4, [0, 1, 2], [2000, 4, 2], layer=-1)
    run(bed, 4, [0, 1, 2], [5, 4, 900], layer=-1)


def test_layers_of_different_windows_in_one_call(kvg):
    bed = States(kvg, 4, 2, 128, 64, [570, 333])
    windows = [0, 100, 0, 30]
    kvg.kvg_cache_set_layer_windows(bed.cache.h, windows)
    every = run(bed, 4, [0, 1], [70, 33], windows, layer=-1)
    q = normal(77, 4, 103, 4, 128)
    for l in range(4):
        one = run(bed, 4, [0, 1], [70, 33], windows, layer=l, q=q[l:l + 1].contiguous())
        assert torch.equal(one[0].view(torch.int16), every[l].view(torch.int16))


def test_many_sequences(kvg):
    """More than a launch takes, rows and states of zero and one among them."""
    n = 300
    bed = States(kvg, 1, 1, 64, 16, [(b * 37) % 90 for b in range(n)])
    run(bed, 2, list(range(n)), [(b * 13) % 5 for b in range(n)])


@pytest.mark.parametrize("window", [0, 70])
def test_unfilled_page_tails_between_grafted_blocks(kvg, window):
    """States of several stored blocks, each at a page's start."""
    bed = Bed(kvg, 1, 2, 128, 64, 40, 3, 1024)
    store = kvg.Store(bed.dims, kvg.KVG_RESIDENCY_HBM, 1 << 28)
    if window:
        kvg.kvg_cache_set_layer_windows(bed.cache.h, [window])
    bed.append(2, 150, 1)
    block = kvg.kvg_deposit(store.h, bed.cache.h, 2, 0, 75)
    for _ in range(3):
        kvg.kvg_graft(store.h, block, bed.cache.h, 0)
    bed.total = [225, 0, 150]
    run(bed, 4, [0, 2], [100, 5], window)
    run(bed, 4, [0, 0], [1, 2], window)


@pytest.mark.parametrize("d,fp8", [(64, False), (128, False), (256, False), (128, True), (256, True)])
def test_values_behind_the_states_do_not_matter(kvg, d, fp8):
    """The last page's rows past the fill, and rows before a window, hold NaN."""
    bed = States(kvg, 1, 1, d, 64, [100], fp8)
    bed.put(0, 0, 1, 20, float("nan"))
    kvg.kvg_cache_set_layer_windows(bed.cache.h, [60])
    out = run(bed, 2, [0], [70], 60)
    assert torch.isfinite(out.float()).all()
    # without the window every row attends to it
    kvg.kvg_cache_set_layer_windows(bed.cache.h, [])
    q = normal(3, 1, 70, 2, d)
    out = torch.zeros_like(q)
    kvg.kvg_cross_attention(bed.cache.h, 0, [0], [70], q.data_ptr(), 2, out.data_ptr(), 0.1)
    torch.cuda.synchronize()
    assert torch.isnan(out[..., :2].float()).all() and torch.isfinite(out[..., 2:].float()).all()


def test_scales_large_negative_and_zero(kvg):
    bed = States(kvg, 1, 2, 128, 64, [400])
    for scale in (-0.1, 0.0, 3.0, -3.0):
        run(bed, 4, [0], [200], scale=scale)


def test_a_batch_of_one_row_each_is_the_decode(kvg):
    bed = States(kvg, 2, 2, 128, 64, [1, 64, 333])
    q = normal(9, 2, 4, 4, 128)
    outs = [torch.empty_like(q) for _ in range(2)]
    kvg.kvg_cross_attention(bed.cache.h, -1, [2, 0, 1, 2], [1] * 4, q.data_ptr(), 4, outs[0].data_ptr(), 0.1)
    kvg.kvg_decode_attention(bed.cache.h, -1, [2, 0, 1, 2], q.data_ptr(), 4, outs[1].data_ptr(), 0.1)
    torch.cuda.synchronize()
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))


def test_calls_on_two_streams(kvg):
    """Two streams that share the cache's scratch, each row as on one stream."""
    bed = States(kvg, 1, 2, 128, 64, [13000, 12000])
    q = normal(6, 2, 40, 4, 128)
    want, got = torch.empty_like(q), torch.empty_like(q)
    for i in range(2):
        kvg.kvg_cross_attention(bed.cache.h, 0, [i], [40], q[i].data_ptr(), 4, want[i].data_ptr(), 0.1)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for i, s in enumerate(streams):
            kvg.kvg_cross_attention(bed.cache.h, 0, [i], [40], q[i].data_ptr(), 4, got[i].data_ptr(), 0.1, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(want.view(torch.int16), got.view(torch.int16))


def test_a_captured_call_replays_on_new_queries(kvg):
    """Capture on another stream than the eager calls; the scratch grows between two replays."""
    bed = States(kvg, 1, 2, 128, 64, [0, 9000, 333])
    q, out = normal(1, 1, 50, 4, 128), torch.zeros(1, 50, 4, 128, dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()

    def call(rows=(30, 5, 15)):
        kvg.kvg_cross_attention(bed.cache.h, 0, [1, 0, 2], list(rows), q.data_ptr(), 4, out.data_ptr(), 0.1)

    with pytest.raises(kvg.KvgError):  # nothing has grown the scratch: refused, and the capture goes on
        with torch.cuda.graph(graph):
            call()
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in (2, 3):
        q.copy_(normal(i, 1, 50, 4, 128))
        call()
        want = out.clone()
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))
        many = normal(5, 1, 1400, 4, 128)
        run(bed, 4, [2, 1, 2], [400, 700, 300], q=many)
    # decode steps
    q1, o1 = normal(7, 1, 2, 4, 128), torch.zeros(1, 2, 4, 128, dtype=torch.bfloat16, device="cuda")
    kvg.kvg_decode_attention(bed.cache.h, 0, [1, 2], q1.data_ptr(), 4, o1.data_ptr(), 0.1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvg.kvg_decode_attention(bed.cache.h, 0, [1, 2], q1.data_ptr(), 4, o1.data_ptr(), 0.1)
    want = o1.clone()
    o1.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o1.view(torch.int16), want.view(torch.int16))


def test_refusals(kvg):
    bed = States(kvg, 2, 2, 64, 16, [50, 0])
    q = normal(1, 2, 60, 4, 64)
    out = torch.zeros_like(q)

    def refused(layer=0, seqs=(0,), rows=(50,), qp=q.data_ptr(), hq=4, op=out.data_ptr()):
        with pytest.raises(kvg.KvgError) as e:
            kvg.kvg_cross_attention(bed.cache.h, layer, list(seqs), list(rows), qp, hq, op, 0.1)
        assert e.value.status == kvg.KVG_ERR_ARG

    refused(layer=2)
    refused(layer=-2)
    refused(seqs=(2,))
    refused(seqs=(-1,))
    refused(rows=(-1,))
    refused(rows=(2 ** 31 - 1,))  # x 4 heads
    refused(hq=5)
    refused(hq=0)
    refused(qp=None)
    refused(op=None)
    refused(qp=q.data_ptr() + 2)
    refused(op=out.data_ptr() + 8)
    refused(seqs=(), rows=())
    kvg.kvg_cross_attention(bed.cache.h, 0, [0, 1], [0, 0], q.data_ptr(), 4, out.data_ptr(), 0.1)
    torch.cuda.synchronize()
    assert not out.any()
