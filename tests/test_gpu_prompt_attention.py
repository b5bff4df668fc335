"""kvg_prompt_attention against its definition in 64 bits over the cache's own
rows.  The bounds are those of the decode gate (kvg_testlib.compare_decode):
the kernel's roundings are the same, softmax weights to 16 bits before the
product with the values and the output to bf16."""
import math

import numpy as np
import pytest
import torch

import oracle
from kvg_testlib import compare_decode, dev_view, need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvg():
    return need_gpu()


def normal(seed, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


class Bed:
    """A cache whose pool starts as NaNs, and its contents row by row."""

    def __init__(self, kvg, n_layers, hkv, d, page, n_pages, seqs, slots, fp8=False, order=None):
        self.kvg, self.hkv, self.d, self.page = kvg, hkv, d, page
        self.dims = kvg.make_dims(n_layers, hkv, d, page, 1e4, 0, int(fp8), 0.0625, 0.03125)
        self.cache = kvg.Cache(self.dims, n_pages, seqs, slots)
        kvg.kvg_cache_set_free_order(self.cache.h, np.random.default_rng(2).permutation(n_pages)
                                     if order is None else order)
        v = self.cache.view
        dev_view(v.pool, v.pool_bytes, torch.uint8).fill_(0x7f)  # a NaN in E4M3 (bf16: 3.4e38, replaced next)
        if not fp8:
            dev_view(v.pool, v.pool_bytes, torch.int16).fill_(0x7fbf)
        raw = dev_view(v.pool, v.pool_bytes, torch.uint8)
        self.pool = raw.view(torch.float8_e4m3fn if fp8 else torch.bfloat16)
        self.pool = self.pool.view(n_layers, 2, n_pages, hkv, page, d)
        self.scales = (0.0625, 0.03125) if fp8 else (1.0, 1.0)

    def append(self, seq, n, seed, scale=1.0):
        if n:
            k, v = (normal(seed + i, self.dims.n_layers, n, self.hkv, self.d) for i in (0, 1))
            k = k * scale  # the gate's absolute bound is one for N(0, 1) values
            pos = torch.arange(n, dtype=torch.int32, device="cuda")
            self.kvg.kvg_cache_append(self.cache.h, seq, k.data_ptr(), v.data_ptr(), pos.data_ptr(), n)
            torch.cuda.synchronize()

    def rows(self, seq, layer):
        """Slots of the valid rows, and their keys and values [N][Hkv][D] in 64 bits."""
        v = self.cache.view
        table, fill = (dev_view(x, 4 * v.max_seqs * v.max_pages, torch.int32).view(v.max_seqs, -1)[seq].cpu().numpy()
                       for x in (v.page_table, v.page_fill))
        slots = np.concatenate([np.arange(j * self.page, j * self.page + f) for j, f in enumerate(fill) if f])
        pages = torch.from_numpy(table[slots // self.page].astype(np.int64)).cuda()
        at = torch.from_numpy(slots % self.page).cuda()
        kv = [self.pool[layer, i].float()[pages, :, at].double() * self.scales[i] for i in (0, 1)]
        return slots, kv[0], kv[1]

    def put(self, seq, layer, kv, slot, value):
        """Overwrites a cached row's first two elements of every head."""
        v = self.cache.view
        table = dev_view(v.page_table, 4 * v.max_seqs * v.max_pages, torch.int32).view(v.max_seqs, -1)
        pg = int(table[seq, slot // self.page])
        self.pool[layer, kv, pg, :, slot % self.page, :2] = torch.tensor(value, device="cuda").to(self.pool.dtype)


def reference(bed, seq, layer, q, n, window, scale):
    """[n][Hq][D]: the sequence's last n rows, a masked row left out of the sums."""
    slots, k, v = bed.rows(seq, layer)
    total, hq = k.shape[0], q.shape[1]
    g = hq // bed.hkv
    last = torch.arange(total - n, total, device="cuda")
    column = torch.arange(total, device="cuda")
    mask = column <= last[:, None]
    if window:
        mask &= column > last[:, None] - window
    x = torch.einsum("nhd,khd->hnk", q.double(), k.repeat_interleave(g, 1)) * scale
    w = torch.softmax(torch.where(mask, x, -math.inf), -1)
    v = v.repeat_interleave(g, 1)
    out = torch.einsum("hnk,khd->nhd", w, torch.nan_to_num(v, nan=0.0, posinf=0.0, neginf=0.0))
    bad = ~torch.isfinite(v).all(-1).all(-1)
    for j in torch.nonzero(bad)[:, 0].tolist():  # the few rows that are not finite: only where they are seen
        seen = mask[:, j]
        term = w[:, seen, j].T[:, :, None] * v[j]
        out[seen] += term - torch.where(torch.isfinite(v[j]), term, 0.0)
    return out


def run(bed, hq, seqs, rows, window=0, layer=0, scale=None, seed=77, q=None):
    """Runs the call for the packed rows and checks every row; returns the output."""
    kvg, n_l = bed.kvg, bed.dims.n_layers if layer < 0 else 1
    t = sum(rows)
    scale = 1 / math.sqrt(bed.d) if scale is None else scale
    q = normal(seed, n_l, t, hq, bed.d) if q is None else q
    out = torch.full_like(q, float("nan"))
    kvg.kvg_prompt_attention(bed.cache.h, layer, seqs, rows, q.data_ptr(), hq, out.data_ptr(), scale)
    torch.cuda.synchronize()
    kvg.kvg_sync(bed.cache.h)
    windows = window if isinstance(window, list) else [window] * bed.dims.n_layers
    for i in range(n_l):
        at = 0
        for s, n in zip(seqs, rows):
            if n:
                l = i if layer < 0 else layer
                check(out[i, at:at + n], reference(bed, s, l, q[i, at:at + n], n, windows[l], scale), f"seq {s} layer {l}")
            at += n
    return out


def check(got, ref, what):
    """Row by row; where the reference is not finite the output is not either."""
    bits, ref = got.contiguous().view(torch.int16).cpu().numpy().view(np.uint16), ref.cpu().numpy()
    for i in range(len(ref)):
        fine = np.isfinite(ref[i])
        assert np.array_equal(fine, np.isfinite(oracle.bf16_to_f64(bits[i]))), f"{what} row {i}"
        compare_decode(oracle, bits[i][fine], ref[i][fine], what=f"{what} row {i}")


# Hkv, G, D, page, window, fp8, (restored, new) rows of each sequence
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


@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}x{c[1]}x{c[2]}p{c[3]}w{c[4]}{'fp8' if c[5] else ''}" for c in CASES])
def test_rows_against_the_definition(kvg, case):
    hkv, g, d, page, window, fp8, lens = case
    total = [a + n for a, n in lens]
    bed = Bed(kvg, 1, hkv, d, page, sum(-(-n // page) for n in total) + 2, len(lens), max(total), fp8)
    if window:
        kvg.kvg_cache_set_layer_windows(bed.cache.h, [window])
    for b, (a, n) in enumerate(lens):
        bed.append(b, a, 10 * b)
        bed.append(b, n, 10 * b + 5)
    first = run(bed, hkv * g, list(range(len(lens))), [n for _, n in lens], window)
    again = run(bed, hkv * g, list(range(len(lens))), [n for _, n in lens], window)
    assert torch.equal(first.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("d,g,fp8", [(64, 2, False), (128, 2, False), (256, 1, False), (128, 4, True), (256, 2, True)])
@pytest.mark.parametrize("n", [2, 31, 64, 65, 128, 129, 255, 256, 257])
def test_lengths_around_the_tiles(kvg, d, g, fp8, n):
    bed = Bed(kvg, 1, 1, d, 64, 16, 2, 900, fp8)
    bed.append(0, 300, 1)
    bed.append(0, n, 3)
    bed.append(1, n, 5)
    run(bed, g, [0, 1], [n, n])


@pytest.mark.parametrize("d,g,fp8", [(128, 2, False), (256, 2, False), (128, 2, True)])
def test_few_rows_on_a_long_context(kvg, d, g, fp8):
    bed = Bed(kvg, 1, 2, d, 64, 330, 3, 20000, fp8)
    bed.append(0, 20000 - 17, 1)
    bed.append(0, 17, 3)
    bed.append(1, 40, 5)
    run(bed, 2 * g, [0, 1], [17, 3])
    run(bed, 2 * g, [1, 0], [40, 1])


def test_layers_of_different_windows_in_one_call(kvg):
    bed = Bed(kvg, 4, 2, 128, 64, 30, 2, 800)
    windows = [0, 100, 0, 30]
    kvg.kvg_cache_set_layer_windows(bed.cache.h, windows)
    bed.append(0, 500, 1)
    bed.append(1, 333, 3)
    every = run(bed, 4, [0, 1], [70, 333], windows, layer=-1)
    q = normal(77, 4, 403, 4, 128)
    for l in range(4):
        one = run(bed, 4, [0, 1], [70, 333], windows, layer=l, q=q[l:l + 1].contiguous())
        assert torch.equal(one[0].view(torch.int16), every[l].view(torch.int16))


def test_many_sequences(kvg):
    """More than a launch takes, lengths zero and one among them."""
    n = 300
    lens = [(b * 37) % 90 for b in range(n)]
    rows = [min(x, (b * 13) % 5) for b, x in enumerate(lens)]
    rows[270], lens[270] = 60, 80
    bed = Bed(kvg, 1, 1, 64, 16, sum(-(-x // 16) for x in lens) + 1, n, 96)
    for b, x in enumerate(lens):
        bed.append(b, x, 2 * b)
    run(bed, 2, list(range(n)), rows)


@pytest.mark.parametrize("d,fp8", [(64, False), (128, False), (256, False), (128, True), (256, True)])
@pytest.mark.parametrize("most", [4, 200])
def test_an_sm_takes_many_items_of_few_tiles(kvg, d, fp8, most):
    """Six work items and more for each SM, of one to three key tiles (rows above 128 / G: two streams)."""
    rng = np.random.default_rng(d + most)
    batch = 120 if most == 4 else 40
    rows, past = rng.integers(1, most, batch), rng.integers(0, 190, batch)
    rows[0] = 2  # (not all of one row)
    need = int(sum(-(-(r + p) // 32) for r, p in zip(rows, past)))
    bed = Bed(kvg, 1, 8 if most == 4 else 16, d, 32, need, batch, 400, fp8=fp8)
    for b in range(batch):
        bed.append(b, int(rows[b] + past[b]), 10 * b)
    run(bed, 2 * bed.hkv, list(range(batch)), [int(x) for x in rows])


@pytest.mark.parametrize("window", [0, 70])
def test_unfilled_page_tails_between_grafted_blocks(kvg, window):
    bed = Bed(kvg, 1, 2, 128, 64, 40, 3, 1024)
    store = kvg.Store(bed.dims, kvg.KVG_RESIDENCY_HBM, 1 << 28)
    if window:
        kvg.kvg_cache_set_layer_windows(bed.cache.h, [window])
    bed.append(2, 150, 1)
    block = kvg.kvg_deposit(store.h, bed.cache.h, 2, 0, 75)
    for _ in range(3):
        kvg.kvg_graft(store.h, block, bed.cache.h, 0)
    bed.append(0, 100, 3)
    run(bed, 4, [0, 2], [100, 150], window)
    with pytest.raises(kvg.KvgError) as e:  # the last slots include a block's unfilled tail
        run(bed, 4, [0], [200], window)
    assert e.value.status == kvg.KVG_ERR_ARG


@pytest.mark.parametrize("d,fp8", [(64, False), (128, False), (256, False), (128, True), (256, True)])
@pytest.mark.parametrize("window", [0, 90])
def test_rows_that_are_not_finite_reach_only_those_that_see_them(kvg, d, fp8, window):
    bed = Bed(kvg, 1, 1, d, 64, 12, 1, 700, fp8)
    if window:
        kvg.kvg_cache_set_layer_windows(bed.cache.h, [window])
    bed.append(0, 600, 1)
    values = [float("nan")] if fp8 else [float("inf"), float("-inf"), float("nan")]
    for i, slot in enumerate([333, 450, 599][:len(values)]):
        bed.put(0, 0, 1, slot, values[i])
    run(bed, 2, [0], [350], window)
    bed.put(0, 0, 0, 520, float("nan"))  # a key: every row that sees it is NaN
    q = normal(5, 1, 350, 2, d)
    out = torch.empty_like(q)
    kvg.kvg_prompt_attention(bed.cache.h, 0, [0], [350], q.data_ptr(), 2, out.data_ptr(), 0.1)
    torch.cuda.synchronize()
    nan = torch.isnan(out[0].float()).all(-1).all(-1).cpu().numpy()
    sees = (np.arange(250, 600) >= 520) & (np.arange(250, 600) < 520 + (window or 1000))
    assert np.array_equal(nan, sees)


def test_scales_large_negative_and_zero(kvg):
    bed = Bed(kvg, 1, 2, 128, 64, 12, 1, 700)
    bed.append(0, 400, 1)
    for scale in (-0.1, 0.0, 3.0, -3.0):
        run(bed, 4, [0], [200], scale=scale)


def test_growing_scores_move_the_maximum(kvg):
    """Keys whose size grows along the sequence: the running maximum grows in every tile."""
    bed = Bed(kvg, 1, 1, 128, 64, 20, 1, 1100)
    for i in range(10):
        bed.append(0, 100, 10 * i, scale=2.0 ** (i - 4))
    run(bed, 2, [0], [400])


def test_pages_past_4_gib(kvg):
    """Pages at the far end of a pool of 5.2 GB."""
    n = 10000
    bed = Bed(kvg, 1, 8, 256, 64, n, 1, 1000, order=np.arange(n)[::-1])
    bed.append(0, 700, 1)
    run(bed, 16, [0], [200])


def test_one_row_each_is_the_decode(kvg):
    bed = Bed(kvg, 2, 2, 128, 64, 20, 3, 400)
    for b, n in enumerate((1, 64, 333)):
        bed.append(b, n, b)
    q = normal(9, 2, 3, 4, 128)
    outs = [torch.empty_like(q) for _ in range(2)]
    kvg.kvg_prompt_attention(bed.cache.h, -1, [2, 0, 1], [1, 1, 1], q.data_ptr(), 4, outs[0].data_ptr(), 0.1)
    kvg.kvg_decode_attention(bed.cache.h, -1, [2, 0, 1], q.data_ptr(), 4, outs[1].data_ptr(), 0.1)
    torch.cuda.synchronize()
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))


def test_calls_on_two_streams(kvg):
    """Two streams that share the cache's scratch, each row as on one stream."""
    bed = Bed(kvg, 1, 2, 128, 64, 420, 2, 13000)
    bed.append(0, 13000, 1)
    bed.append(1, 12000, 3)
    q = normal(6, 2, 40, 4, 128)
    want, got = torch.empty_like(q), torch.empty_like(q)
    for i in range(2):
        kvg.kvg_prompt_attention(bed.cache.h, 0, [i], [40], q[i].data_ptr(), 4, want[i].data_ptr(), 0.1)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for i, s in enumerate(streams):
            kvg.kvg_prompt_attention(bed.cache.h, 0, [i], [40], q[i].data_ptr(), 4, got[i].data_ptr(), 0.1, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(want.view(torch.int16), got.view(torch.int16))


def test_refusals(kvg):
    bed = Bed(kvg, 2, 2, 64, 16, 20, 2, 100)
    bed.append(0, 50, 1)
    q = normal(1, 2, 60, 4, 64)
    out = torch.zeros_like(q)

    def refused(layer=0, seqs=(0,), rows=(50,), qp=q.data_ptr(), hq=4, op=out.data_ptr()):
        with pytest.raises(kvg.KvgError) as e:
            kvg.kvg_prompt_attention(bed.cache.h, layer, list(seqs), list(rows), qp, hq, op, 0.1)
        assert e.value.status == kvg.KVG_ERR_ARG

    refused(layer=2)
    refused(layer=-2)
    refused(seqs=(2,))
    refused(rows=(51,))
    refused(rows=(-1,))
    refused(seqs=(1,), rows=(1,))
    refused(hq=5)
    refused(hq=12)
    refused(qp=None)
    refused(op=None)
    refused(qp=q.data_ptr() + 2)
    refused(op=out.data_ptr() + 8)
    refused(seqs=(), rows=())
    kvg.kvg_prompt_attention(bed.cache.h, 0, [0, 1], [0, 0], q.data_ptr(), 4, out.data_ptr(), 0.1)
    torch.cuda.synchronize()
    assert not out.any()
    kvg.kvg_sync(bed.cache.h)
