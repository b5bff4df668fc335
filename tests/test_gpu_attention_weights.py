"""kvg_attention_weights against its definition in 64 bits over the cache's own
rows.  Outputs have the bounds of the decode gate (kvg_testlib.compare_decode).

A weight is w = 2^(c s - lse) in fp32, c s the scaled score and lse = log2 of the
sum, or a maximum and a quotient.  What it is off by, relative to itself: ln 2
times the error of its exponent, and the exponential and the sums.  The score: D
products of 16-bit values, exact, summed in fp32; a tensor core may drop, not
round, what is below the last bit of the largest term, so each of D additions is
off by at most 2^-22 of the largest partial sum, which |q| |k| bounds: 2^-22 D |q|
|k| at worst, and 2^-22 sqrt(D) |q| |k| for errors of no common sign; with c |q|
|k| <= S (computed from the case's queries and keys) that is S sqrt(D) 2^-22.  The
product with c and the difference round exponents of up to S + 20 by 2^-24 each;
lse itself carries the same errors, averaged.  exp2 and log2 are off by 2 units of
2^-23, the n additions of a sum of n positive terms by n 2^-24 at worst; sums here
are formed from many short ones, at most 2,048 terms one after the other, 2^-13 at
worst and sqrt(2,048) 2^-24 = 2^-18.5 for errors of no common sign.  So weights are
within 4 (S sqrt(D) 2^-22 + 2^-18.5 + 2^-20) of themselves, the 4 for the maximum
over many."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from kvg_testlib import dev_view, need_gpu
from test_gpu_prompt_attention import Bed, check, normal
from test_gpu_prompt_attention import reference as attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvg():
    return need_gpu()


def received(bed, seq, layer, q, n, window, scale):
    """([slots] weights in 64 bits, bound on c |q| |k|) of the sequence's last n rows."""
    slots, k, _ = bed.rows(seq, layer)
    total, g = k.shape[0], q.shape[1] // bed.hkv
    last, column = torch.arange(total - n, total, device="cuda"), torch.arange(total, device="cuda")
    mask = column <= last[:, None]
    if window:
        mask &= column > last[:, None] - window
    k = k.repeat_interleave(g, 1)
    x = torch.einsum("nhd,khd->hnk", q.double(), k) * scale
    w = torch.softmax(torch.where(mask, x, -math.inf), -1).sum((0, 1))
    out = torch.zeros(bed.cache.view.max_slots, dtype=torch.float64, device="cuda")
    out[torch.from_numpy(slots).cuda()] = w
    top = abs(scale) * 1.4427 * float(q.double().norm(dim=-1).max() * k.norm(dim=-1).max())
    return out, top


def run(bed, hq, seqs, rows, window=0, layer=0, scale=None, seed=77, q=None, decay=0.0, before=None, **kw):
    """Runs the call, checks outputs and weights; returns both."""
    kvg, n_l, v = bed.kvg, bed.dims.n_layers if layer < 0 else 1, bed.cache.view
    scale = 1 / math.sqrt(bed.d) if scale is None else scale
    q = normal(seed, n_l, sum(rows), hq, bed.d) if q is None else q
    out = torch.full_like(q, float("nan"))
    # (what is not read may be anything)
    weights = torch.full((v.max_seqs, v.max_slots), float("nan"), device="cuda") if before is None else before.clone()
    start = weights.clone()
    kvg.kvg_attention_weights(bed.cache.h, layer, seqs, rows, q.data_ptr(), hq, out.data_ptr(), scale,
                              weights.data_ptr(), decay, **kw)
    torch.cuda.synchronize()
    kvg.kvg_sync(bed.cache.h)
    windows = window if isinstance(window, list) else [window] * bed.dims.n_layers
    want, top = {}, 0.0
    for i in range(n_l):
        at, l = 0, i if layer < 0 else layer
        for s, n in zip(seqs, rows):
            if n:
                rows_q = q[i, at:at + n]
                check(out[i, at:at + n], attention(bed, s, l, rows_q, n, windows[l], scale), f"seq {s} layer {l}")
                w, t = received(bed, s, l, rows_q, n, windows[l], scale)
                want[s], top = want.get(s, 0) + w, max(top, t)
            at += n
    rel = 4 * (top * math.sqrt(bed.d) * 2.0 ** -22 + 2.0 ** -18.5 + 2.0 ** -20)
    for s in range(v.max_seqs):
        n = kvg.kvg_cache_seq_info(bed.cache.h, s)[0]
        if s not in want:  # left as it is
            assert torch.equal(weights[s].view(torch.int32), start[s].view(torch.int32))
            continue
        assert torch.equal(weights[s, n:].view(torch.int32), start[s, n:].view(torch.int32))
        ref = want[s][:n] + (decay * start[s, :n].double() if decay else 0)
        size = want[s][:n] + (abs(decay) * start[s, :n].double().abs() if decay else 0)
        err = (weights[s, :n].double() - ref).abs()
        # (below 2^-126 a weight may be flushed to zero, as many times as there are rows)
        over = err - rel * size - 2.0 ** -126 * hq * n_l * max(rows)
        assert float(over.max()) <= 0, (s, float((err / size.clamp_min(1e-30)).max()), rel)
        if not decay:
            assert not weights[s, :n][want[s][:n] == 0].any()
    return out, weights


# Hkv, G, D, page, window, fp8, (rows before, query rows) of each sequence
CASES = [
    (2, 2, 64, 16, 0, False, [(256, 37), (0, 5)]),
    (2, 1, 64, 16, 50, False, [(0, 300), (77, 129)]),
    (1, 8, 64, 64, 0, False, [(1000, 150), (0, 1), (3, 2)]),
    (2, 2, 128, 64, 0, False, [(700, 257), (0, 128), (1, 127)]),
    (2, 4, 128, 64, 100, False, [(500, 200), (0, 65)]),
    (1, 1, 128, 128, 0, False, [(130, 513)]),
    (2, 2, 256, 64, 0, False, [(300, 199), (0, 130)]),
    (1, 1, 256, 16, 64, False, [(100, 260)]),
    (2, 2, 128, 64, 0, True, [(500, 200), (0, 33)]),
    (1, 4, 128, 16, 70, True, [(200, 150)]),
    (2, 1, 256, 64, 0, True, [(90, 200), (64, 64)]),
    (1, 2, 256, 48, 33, True, [(150, 90)]),
    # pages that are no multiple of 8 rows, of one row, and past a tile
    (2, 2, 128, 7, 0, False, [(40, 90), (0, 14)]),
    (2, 2, 64, 1, 0, False, [(30, 40)]),
    (2, 1, 128, 24, 0, False, [(100, 200)]),
    (1, 2, 128, 33, 45, False, [(66, 100)]),
    (1, 2, 128, 100, 0, False, [(250, 160)]),
    (1, 2, 256, 129, 0, False, [(200, 200)]),
    (1, 1, 64, 200, 0, False, [(399, 210)]),
    (2, 2, 128, 20, 0, True, [(50, 75)]),
    (1, 1, 128, 300, 64, True, [(299, 150)]),
]


def bed_of(kvg, case, n_layers=1, extra=0):
    hkv, g, d, page, window, fp8, lens = case
    total = [a + n for a, n in lens]
    bed = Bed(kvg, n_layers, hkv, d, page, sum(-(-n // page) for n in total) + 2, len(lens) + extra, max(total) + 3, fp8)
    if window:
        kvg.kvg_cache_set_layer_windows(bed.cache.h, [window] * n_layers)
    for b, n in enumerate(total):
        bed.append(b, n, 10 * b)
    return bed


@pytest.mark.parametrize("step", [True, False], ids=["step", "prompt"])
@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}x{c[1]}x{c[2]}p{c[3]}w{c[4]}{'fp8' if c[5] else ''}" for c in CASES])
def test_rows_against_the_definition(kvg, case, step):
    hkv, g, d, page, window, fp8, lens = case
    bed = bed_of(kvg, case)
    args = bed, hkv * g, list(range(len(lens))), [1 if step else n for _, n in lens], window
    first, again = run(*args), run(*args)
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(first, again))


@pytest.mark.parametrize("d,g,fp8", [(64, 2, False), (128, 2, False), (256, 1, False), (128, 4, True), (256, 2, True)])
@pytest.mark.parametrize("n", [2, 31, 64, 65, 128, 129, 255, 256, 257, 511])
def test_lengths_around_the_tiles(kvg, d, g, fp8, n):
    bed = Bed(kvg, 1, 1, d, 64, 24, 2, 900, fp8)
    bed.append(0, 300 + n, 1)
    bed.append(1, n, 5)
    run(bed, g, [0, 1], [n, n])
    run(bed, g, [1, 0], [1, 1])
    run(bed, g, [1, 0], [n, 0])


@pytest.mark.parametrize("d,g,fp8", [(64, 4, False), (128, 2, False), (256, 2, False), (128, 2, True)])
def test_few_rows_on_a_long_context(kvg, d, g, fp8):
    bed = Bed(kvg, 1, 2, d, 64, 330, 3, 20000, fp8)
    bed.append(0, 20000, 1)
    bed.append(1, 40, 5)
    run(bed, 2 * g, [0, 1], [17, 3])
    run(bed, 2 * g, [1, 0], [40, 1])
    run(bed, 2 * g, [1, 0], [1, 1])
    run(bed, 2 * g, [0], [1])


def test_many_rows(kvg):
    """Query ranges of one key tile in several work items."""
    for d in (128, 256):
        bed = Bed(kvg, 1, 1, d, 64, 60, 1, 3600)
        bed.append(0, 3600, 1)
        run(bed, 2, [0], [2900])
        kvg.kvg_cache_set_layer_windows(bed.cache.h, [700])
        run(bed, 2, [0], [2900], 700)


@pytest.mark.parametrize("rows", [[1, 1], [70, 333], [70, 1]])
def test_layers_of_different_windows_in_one_call(kvg, rows):
    bed = Bed(kvg, 4, 2, 128, 64, 30, 2, 800)
    windows = [0, 100, 0, 30]
    kvg.kvg_cache_set_layer_windows(bed.cache.h, windows)
    bed.append(0, 570, 1)
    bed.append(1, 333, 3)
    before = torch.rand(2, 800, device="cuda")
    for decay in (0.0, 1.0, 0.5, -2.0):
        run(bed, 4, [0, 1], rows, windows, layer=-1, decay=decay, before=before)
    run(bed, 4, [1, 0], rows, windows, layer=2, decay=0.75, before=before)
    run(bed, 4, [1], rows[:1], windows, layer=1, decay=0.0)
    kvg.kvg_cache_set_layer_windows(bed.cache.h, [5, 0, 9, 13])  # more windows than a launch has
    run(bed, 4, [0, 1], rows, [5, 0, 9, 13], layer=-1, decay=0.5, before=before)


@pytest.mark.parametrize("most", [1, 5])
def test_many_sequences(kvg, most):
    """More than a launch takes, lengths zero and one among them; sequences without rows keep their weights."""
    n = 300
    lens = [(b * 37) % 90 for b in range(n)]
    rows = [min(x, (b * 13) % 5, most) for b, x in enumerate(lens)]
    bed = Bed(kvg, 1, 1, 64, 16, sum(-(-x // 16) for x in lens) + 1, n, 96)
    for b, x in enumerate(lens):
        bed.append(b, x, 2 * b)
    run(bed, 2, list(range(n)), rows, decay=0.5, before=torch.rand(n, 96, device="cuda"))


@pytest.mark.parametrize("d,page,window", [(64, 1, 0), (64, 1, 70), (256, 1, 0)])
def test_more_work_than_an_sm_looks_ahead(kvg, d, page, window):
    """Some 20,000 pairs of key tiles, of 16 slots each, for few rows each."""
    n_l, hkv, per = 4, 8, 32
    lens = [(500 + 17 * i, 2 + i % 3) for i in range(28 if d == 64 else 16)]
    if window:
        lens = [(a, n) for a, n in lens] * 4
    assert window or sum(-(-(a + n) // per) for a, n in lens) * hkv * n_l > 96 * (152 if d == 64 else 76)
    bed = bed_of(kvg, (hkv, 1, d, page, window, False, lens), n_layers=n_l)
    run(bed, hkv, list(range(len(lens))), [n for _, n in lens], window, layer=-1)


@pytest.mark.parametrize("window", [0, 70])
@pytest.mark.parametrize("rows", [100, 1])
def test_unfilled_page_tails_between_grafted_blocks(kvg, window, rows):
    bed = Bed(kvg, 1, 2, 128, 64, 40, 3, 1024)
    store = kvg.Store(bed.dims, kvg.KVG_RESIDENCY_HBM, 1 << 28)
    if window:
        kvg.kvg_cache_set_layer_windows(bed.cache.h, [window])
    bed.append(2, 150, 1)
    block = kvg.kvg_deposit(store.h, bed.cache.h, 2, 0, 75)
    for _ in range(3):
        kvg.kvg_graft(store.h, block, bed.cache.h, 0)
    bed.append(0, 100, 3)
    run(bed, 4, [0, 2], [rows, rows], window)
    if rows == 100:
        run(bed, 4, [0], [20], window)
        with pytest.raises(kvg.KvgError):  # the last slots include a block's unfilled tail
            run(bed, 4, [0], [200], window)


@pytest.mark.parametrize("d,fp8", [(64, False), (128, False), (256, False), (128, True), (256, True)])
@pytest.mark.parametrize("rows", [350, 1])
def test_values_that_are_not_finite_leave_the_weights(kvg, d, fp8, rows):
    bed = Bed(kvg, 1, 1, d, 64, 12, 1, 700, fp8)
    bed.append(0, 600, 1)
    for i, slot in enumerate([333, 450]):
        bed.put(0, 0, 1, slot, float("nan"))
    if rows > 1:
        run(bed, 2, [0], [rows])
    q = normal(5, 1, rows, 2, d)
    out, weights = torch.empty_like(q), torch.zeros(1, 700, device="cuda")

    def call():
        kvg.kvg_attention_weights(bed.cache.h, 0, [0], [rows], q.data_ptr(), 2, out.data_ptr(), 0.1, weights.data_ptr(), 0.0)
        torch.cuda.synchronize()
        return weights[0, :600]

    want, _ = received(bed, 0, 0, q[0], rows, 0, 0.1)
    assert torch.allclose(call().double(), want[:600], rtol=1e-3)
    # a key that is NaN: the weights of every row that attends to it are
    bed.put(0, 0, 0, 420, float("nan"))
    got = torch.isnan(call()).cpu().numpy()
    assert got.all()
    # a query that is NaN: the slots that it attends to
    bed.put(0, 0, 0, 420, 1.0)
    if rows > 1:
        q[0, 100] = float("nan")  # of slot 350
        assert np.array_equal(torch.isnan(call()).cpu().numpy(), np.arange(600) <= 350)


def test_scales_large_negative_and_zero(kvg):
    bed = Bed(kvg, 1, 2, 128, 64, 12, 1, 700)
    bed.append(0, 400, 1)
    for scale in (-0.1, 0.0, 1.0, -1.0):
        for rows in (200, 1):
            run(bed, 4, [0], [rows], scale=scale)


def test_growing_scores_move_the_maximum(kvg):
    bed = Bed(kvg, 1, 1, 128, 64, 20, 1, 1100)
    for i in range(10):
        bed.append(0, 100, 10 * i, scale=2.0 ** (i - 6))
    for rows in (400, 1):
        run(bed, 2, [0], [rows])


def test_outputs_are_those_of_the_plain_calls(kvg):
    """Bit for bit: accumulating weights changes no output."""
    bed = Bed(kvg, 2, 2, 128, 64, 40, 3, 700)
    for b, n in enumerate((1, 64, 633)):
        bed.append(b, n, b)
    weights = torch.zeros(3, 700, device="cuda")
    for rows in ([1, 1, 1], [1, 30, 500]):
        q = normal(9, 2, sum(rows), 4, 128)
        outs = [torch.empty_like(q) for _ in range(2)]
        kvg.kvg_attention_weights(bed.cache.h, -1, [0, 1, 2], rows, q.data_ptr(), 4, outs[0].data_ptr(), 0.1,
                                  weights.data_ptr(), 1.0)
        kvg.kvg_prompt_attention(bed.cache.h, -1, [0, 1, 2], rows, q.data_ptr(), 4, outs[1].data_ptr(), 0.1)
        torch.cuda.synchronize()
        assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))
        total = weights.sum(1).cpu().numpy()
        assert np.allclose(total, 8 * np.array([1, rows[1], rows[2]]) + (8 if rows[1] > 1 else 0), rtol=1e-4)


def test_pages_past_4_gib(kvg):
    """Pages at the far end of a pool of 5.2 GB."""
    n = 10000
    bed = Bed(kvg, 1, 8, 256, 64, n, 1, 1000, order=np.arange(n)[::-1])
    bed.append(0, 700, 1)
    run(bed, 16, [0], [200])
    run(bed, 16, [0], [1])


@pytest.mark.parametrize("rows", [1, 40])
def test_calls_on_two_streams(kvg, rows):
    """Two streams that share the cache's scratch, each as on one stream."""
    bed = Bed(kvg, 1, 2, 128, 64, 420, 2, 13000)
    bed.append(0, 13000, 1)
    bed.append(1, 12000, 3)
    q = normal(6, 2, rows, 4, 128)
    out, want, got = torch.empty_like(q), torch.zeros(2, 13000, device="cuda"), torch.zeros(2, 13000, device="cuda")

    def call(i, to, **kw):
        kvg.kvg_attention_weights(bed.cache.h, 0, [i], [rows], q[i].data_ptr(), 4, out[i].data_ptr(), 0.1, to.data_ptr(),
                                  0.0, **kw)

    for i in range(2):
        call(i, want)
    first = out.clone()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for i, s in enumerate(streams):
            call(i, got, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(want, got) and torch.equal(first.view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("rows", [(30, 5), (1, 1)])
def test_a_captured_call_accumulates_at_every_replay(kvg, rows, fp8):
    bed = Bed(kvg, 1, 2, 128, 64, 160, 2, 9000, fp8)
    bed.append(0, 9000, 1)
    bed.append(1, 333, 3)
    q = normal(1, 1, sum(rows), 4, 128)
    out, weights = torch.zeros_like(q), torch.zeros(2, 9000, device="cuda")

    def call():
        kvg.kvg_attention_weights(bed.cache.h, 0, [0, 1], list(rows), q.data_ptr(), 4, out.data_ptr(), 0.1,
                                  weights.data_ptr(), 0.5)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    got = []
    for replay in (True, False):
        weights.zero_()
        for i in (2, 3, 4):
            q.copy_(normal(i, 1, sum(rows), 4, 128))
            graph.replay() if replay else call()
        torch.cuda.synchronize()
        got += [weights.clone(), out.clone().float()]
    assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[3])


def test_refusals(kvg):
    bed = Bed(kvg, 2, 2, 64, 16, 20, 2, 100)
    bed.append(0, 50, 1)
    q = normal(1, 2, 60, 4, 64)
    out, weights = torch.zeros_like(q), torch.zeros(2, 100, device="cuda")

    def refused(layer=0, seqs=(0,), rows=(50,), qp=q.data_ptr(), hq=4, op=out.data_ptr(), wp=weights.data_ptr(), decay=1.0):
        with pytest.raises(kvg.KvgError) as e:
            kvg.kvg_attention_weights(bed.cache.h, layer, list(seqs), list(rows), qp, hq, op, 0.1, wp, decay)
        assert e.value.status == kvg.KVG_ERR_ARG

    refused(layer=2)
    refused(seqs=(2,))
    refused(rows=(51,))
    refused(rows=(-1,))
    refused(seqs=(1,), rows=(1,))
    refused(seqs=(0, 0), rows=(1, 1))
    refused(hq=5)
    refused(hq=12)
    refused(qp=None)
    refused(op=None)
    refused(wp=None)
    refused(wp=weights.data_ptr() + 2)
    refused(op=out.data_ptr() + 8)
    refused(seqs=(), rows=())
    for decay in (float("nan"), float("inf")):
        refused(decay=decay)
    kvg.kvg_attention_weights(bed.cache.h, 0, [0, 1, 0], [0, 0, 0], q.data_ptr(), 4, out.data_ptr(), 0.1,
                              weights.data_ptr(), 1.0)
    torch.cuda.synchronize()
    assert not out.any() and not weights.any()
    v = bed.cache.view
    assert dev_view(v.page_fill, 4, torch.int32).item() == 16


def test_little_scratch(kvg):
    """What does not fit the scratch at once is done layer by layer, rows by rows: the same tests with 8 KB of it."""
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", __file__, "-k",
                        "many_sequences or layers_of_different or unfilled or plain_calls"],
                       env=os.environ | {"KVG_WEIGHTS_SCRATCH_KB": "8"}, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:]
