"""kvg_cache_evict against its definition, bit for bit: which rows are kept, where
they go, and that nothing else of the pool changes."""
import numpy as np
import pytest
import torch

from kvg_testlib import dev_view, need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvg():
    return need_gpu()


class Bed:
    """A cache of random bytes, its tables, and the weights."""

    def __init__(self, kvg, n_layers, hkv, d, page, n_pages, seqs, slots, fp8=False, seed=1):
        self.kvg, self.page, self.rng = kvg, page, np.random.default_rng(seed)
        self.dims = kvg.make_dims(n_layers, hkv, d, page, 1e4, 0, int(fp8), 0.0625, 0.0625)
        self.cache = kvg.Cache(self.dims, n_pages, seqs, slots)
        kvg.kvg_cache_set_free_order(self.cache.h, self.rng.permutation(n_pages))
        v = self.cache.view
        raw = dev_view(v.pool, v.pool_bytes, torch.uint8)
        raw.copy_(torch.randint(256, raw.shape, dtype=torch.uint8, device="cuda"))
        self.pool = raw.view(n_layers, 2, n_pages, hkv, page, d * (1 if fp8 else 2))
        self.weights = torch.zeros(seqs, slots, device="cuda")

    def append(self, seq, n, first=0):
        if n:
            shape = self.dims.n_layers, n, self.dims.n_kv_heads, self.dims.head_dim
            k, v = (torch.randn(shape, device="cuda").to(torch.bfloat16) for _ in range(2))
            pos = torch.from_numpy(self.rng.integers(0, 2 ** 31 - 1, n).astype(np.int32)).cuda()
            self.kvg.kvg_cache_append(self.cache.h, seq, k.data_ptr(), v.data_ptr(), pos.data_ptr(), n)
            torch.cuda.synchronize()

    def set_weights(self, seq, w):
        self.weights[seq, :len(w)] = torch.as_tensor(np.asarray(w, np.float32)).cuda()

    def tables(self):
        v = self.cache.view
        return [dev_view(p, 4 * v.max_seqs * n, torch.int32).view(v.max_seqs, n).cpu().numpy().copy()
                for p, n in ((v.page_table, v.max_pages), (v.page_fill, v.max_pages), (v.positions, v.max_slots))]

    def snapshot(self):
        torch.cuda.synchronize()
        return self.pool.clone(), self.tables(), self.weights.cpu().numpy().copy()

    def slots(self, seq):
        return self.kvg.kvg_cache_seq_info(self.cache.h, seq)


def kept_slots(fill, page, weights, rows, first, last):
    """Slots of the rows that stay, from the definition."""
    valid = [j * page + r for j, f in enumerate(fill) for r in range(f)]
    if len(valid) <= rows:
        return valid
    end = len(valid) - last
    order = sorted(range(first, end), key=lambda i: (0 if weights[valid[i]] != weights[valid[i]] else 1,
                                                     weights[valid[i]] if weights[valid[i]] == weights[valid[i]] else 0.0),
                   reverse=True)  # (sort is stable and keeps the earlier of equals first, reversed too)
    middle = sorted(order[:rows - first - last])
    return valid[:first] + [valid[i] for i in middle] + valid[end:]


def evict(bed, seqs, rows, first, last, dst=None, **kw):
    """Runs the call and checks everything that it may and may not change."""
    pool, (table, fill, pos), weights = bed.snapshot()
    old = {s: bed.slots(s) for s in set(seqs) | set(dst or [])}
    bed.kvg.kvg_cache_evict(bed.cache.h, list(seqs), list(rows), first, last, bed.weights.data_ptr(), dst_ids=dst, **kw)
    torch.cuda.synchronize()
    bed.kvg.kvg_sync(bed.cache.h)
    got_pool, (got_table, got_fill, got_pos), got_weights = bed.snapshot()
    page = bed.page
    want_table, want_fill, want_pos, want_weights = table.copy(), fill.copy(), pos.copy(), weights.copy()
    want = pool.clone()
    for src, to, n in zip(seqs, dst or seqs, rows):
        n_slots = old[src][0]
        kept = kept_slots(fill[src][:-(-n_slots // page)], page, weights[src], n, first, last)
        m, pages = len(kept), -(-len(kept) // page)
        assert bed.slots(to) == (m, pages)
        new = got_table[to][:pages]
        assert len(set(new)) == pages and (new >= 0).all()
        want_table[to] = -1
        want_table[to][:pages] = new
        want_fill[to] = 0
        want_fill[to][:pages] = [min(page, m - j * page) for j in range(pages)]
        if m:
            k = np.array(kept)
            sp, sr = torch.from_numpy(table[src][k // page].astype(np.int64)).cuda(), torch.from_numpy(k % page).cuda()
            j = np.arange(m)
            dp, dr = torch.from_numpy(new[j // page].astype(np.int64)).cuda(), torch.from_numpy(j % page).cuda()
            want[:, :, dp, :, dr] = pool[:, :, sp, :, sr]
            want_pos[to][:m], want_weights[to][:m] = pos[src][k], weights[src][k]
        if not (to == src and m == n_slots):
            want_pos[to][m:max(m, old[to][0])] = -1
            want_weights[to][m:max(m, old[to][0])] = 0
    # a page belongs to one sequence, or is a block's
    assert torch.equal(got_pool, want)
    assert np.array_equal(got_table, want_table) and np.array_equal(got_fill, want_fill)
    assert np.array_equal(got_pos, want_pos)
    assert np.array_equal(got_weights.view(np.int32), want_weights.view(np.int32))
    return got_table


def heavy_tailed(rng, n):
    return np.exp(2 * rng.standard_normal(n)) * (rng.random(n) > 0.1)


# layers, Hkv, D, page, fp8, rows per sequence, kept, first, last
CASES = [
    (2, 2, 64, 16, False, [293], 131, 4, 32),
    (1, 3, 128, 64, False, [1000, 64, 1, 700], 200, 1, 50),
    (2, 2, 256, 64, False, [513, 129], 128, 0, 0),
    (1, 2, 128, 24, True, [333, 95], 77, 5, 0),
    (1, 1, 256, 7, True, [100, 50], 49, 0, 49),
    (1, 2, 64, 16, True, [90], 13, 13, 0),
    (1, 1, 64, 1, False, [60, 9], 17, 2, 3),
    (1, 4, 64, 33, False, [5000, 2047, 3999], 2048, 4, 100),
    (1, 1, 128, 128, False, [1024, 1025, 1023, 2048, 33], 32, 1, 1),
]


@pytest.mark.parametrize("how", ["in place", "to others"])
@pytest.mark.parametrize("case", CASES, ids=[f"{c[1]}x{c[2]}p{c[3]}{'fp8' if c[4] else ''}k{c[6]}" for c in CASES])
def test_kept_rows(kvg, case, how):
    n_l, hkv, d, page, fp8, lens, keep, first, last = case
    batch = len(lens)
    bed = Bed(kvg, n_l, hkv, d, page, 2 * sum(-(-n // page) for n in lens) + 3, 2 * batch, max(lens) + page, fp8)
    for b, n in enumerate(lens):
        bed.append(b, n)
        bed.set_weights(b, heavy_tailed(bed.rng, n))
    dst = None if how == "in place" else list(range(batch, 2 * batch))
    evict(bed, range(batch), [keep] * batch, first, last, dst)
    evict(bed, range(batch), [keep // 2 + first // 2 + last // 2 + 1] * batch, first // 2, last // 2, dst)
    for b in range(batch):  # and rows behind them
        bed.append(dst[b] if dst else b, 5)
    assert bed.slots(dst[0] if dst else 0)[0] >= 5


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 1023, 1024, 1025, 2049, 4097])
def test_lengths_around_the_chunks(kvg, n):
    bed = Bed(kvg, 1, 1, 64, 16, 2 * (n // 16 + 1), 2, n + 16)
    bed.append(0, n)
    bed.set_weights(0, heavy_tailed(bed.rng, n))
    for keep in sorted({n, n - 1, n // 2, 1, 0}, reverse=True):
        evict(bed, [0], [keep], 0, 0, [1])
    for keep in sorted({n - 1, n // 2, 1, 0}, reverse=True):
        evict(bed, [0], [keep], 0, 0)


@pytest.mark.parametrize("how", ["in place", "to another"])
@pytest.mark.parametrize("ties", [False, True])
def test_more_rows_than_a_cluster_holds_at_once(kvg, how, ties):
    n = 70001
    bed = Bed(kvg, 1, 1, 64, 64, 2200, 2, 70100)
    bed.append(0, n)
    w = heavy_tailed(bed.rng, n)
    bed.set_weights(0, np.round(w) if ties else w)
    for keep, first, last in [(66000, 4, 1000), (40000, 4, 33000), (5000, 0, 0), (33, 3, 0)]:
        evict(bed, [0], [keep], first, last, None if how == "in place" else [1])


WEIGHTS = {
    "all equal": lambda rng, n: np.full(n, 0.25),
    "zeros of both signs": lambda rng, n: np.where(rng.random(n) < 0.5, 0.0, -0.0),
    "few values": lambda rng, n: rng.integers(0, 3, n),
    "negative ones": lambda rng, n: rng.standard_normal(n),
    "not finite": lambda rng, n: rng.choice([np.nan, np.inf, -np.inf, 0.0, -0.0, 1.0, -np.nan], n),
    "only NaN": lambda rng, n: np.full(n, np.nan),
    "one digit apart": lambda rng, n: (0x3f800000 + rng.integers(0, 300, n)).astype(np.int32).view(np.float32),
    "subnormal": lambda rng, n: rng.integers(0, 500, n).astype(np.int32).view(np.float32),
    "falling": lambda rng, n: np.arange(n, 0, -1),
    "rising": lambda rng, n: np.arange(n),
}


@pytest.mark.parametrize("kind", WEIGHTS)
def test_orders_of_weights(kvg, kind):
    bed = Bed(kvg, 1, 1, 64, 16, 400, 2, 3000)
    for n, keep, first, last in [(2500, 700, 4, 64), (2500, 2499, 0, 0), (1500, 33, 0, 1), (40, 1, 0, 0)]:
        bed.kvg.kvg_cache_release(bed.cache.h, 0)
        bed.append(0, n)
        bed.set_weights(0, WEIGHTS[kind](bed.rng, n))
        evict(bed, [0], [keep], first, last, [1])
        evict(bed, [0], [keep], first, last)


@pytest.mark.parametrize("how", ["in place", "to another"])
def test_unfilled_page_tails_between_grafted_blocks(kvg, how):
    """Slots without a row are not kept, whatever their weight, and the gaps close."""
    bed = Bed(kvg, 2, 2, 64, 16, 80, 3, 500)
    store = kvg.Store(bed.dims, kvg.KVG_RESIDENCY_HBM, 1 << 28)
    bed.append(2, 75)
    block = kvg.kvg_deposit(store.h, bed.cache.h, 2, 0, 75)
    for keep, first, last in [(100, 3, 20), (150, 80, 0), (150, 0, 76), (165, 5, 5), (400, 0, 0)]:
        kvg.kvg_cache_release(bed.cache.h, 0)
        for _ in range(2):
            kvg.kvg_graft(store.h, block, bed.cache.h, 0)
        bed.append(0, 20)
        bed.set_weights(0, 1 + bed.rng.random(bed.slots(0)[0]))
        evict(bed, [0], [keep], first, last, None if how == "in place" else [1])


@pytest.mark.parametrize("how", ["in place", "to others"])
def test_pages_of_stored_blocks_are_not_written(kvg, how):
    """Sequences that point at a pool-resident block: its pages keep their bytes (the whole pool is compared), the
    first ones stay shared, and everything can be released."""
    bed = Bed(kvg, 1, 2, 128, 16, 150, 6, 400)
    store = kvg.PoolStore(bed.cache, 1 << 24)
    bed.append(5, 200)
    block = kvg.kvg_deposit(store.h, bed.cache.h, 5, 0, 200)
    kvg.kvg_cache_release(bed.cache.h, 5)
    for b in range(3):
        kvg.kvg_graft(store.h, block, bed.cache.h, b)
        bed.append(b, 10 * b)
        bed.set_weights(b, heavy_tailed(bed.rng, 200 + 10 * b))
    before = bed.tables()[0]
    dst = None if how == "in place" else [3, 4, 5]
    table = evict(bed, [0, 1, 2], [100, 90, 205], 40, 20, dst)
    for i, b in enumerate(dst or [0, 1, 2]):
        assert np.array_equal(table[b][:2], before[i][:2]) and not set(table[b][2:]) & set(before[0][:13]) - {-1}
    # the thinned sequences' common pages are still read together, and give what the decode gives
    q = torch.randn(1, 3, 4, 128, device="cuda").to(torch.bfloat16)
    outs = [torch.empty_like(q) for _ in range(2)]
    kvg.kvg_decode_attention(bed.cache.h, 0, dst or [0, 1, 2], q.data_ptr(), 4, outs[0].data_ptr(), 0.1)
    kvg.kvg_decode_attention_shared(bed.cache.h, 0, dst or [0, 1, 2], q.data_ptr(), 4, outs[1].data_ptr(), 0.1)
    torch.cuda.synchronize()
    assert torch.allclose(outs[0].float(), outs[1].float(), atol=2e-2, equal_nan=True)
    evict(bed, dst or [0, 1, 2], [50, 90, 3], 2, 1)
    evict(bed, [0, 1, 2], [0, 0, 0], 0, 0, dst)
    for b in range(6):
        kvg.kvg_cache_release(bed.cache.h, b)
    # every page but the block's is free again
    for b in range(5):
        bed.append(b, 400)
    bed.append(5, (150 - 13 - 5 * 25) * 16)
    kvg.kvg_cache_release(bed.cache.h, 3)
    kvg.kvg_graft(store.h, block, bed.cache.h, 3)
    evict(bed, [3], [150], 0, 0)


def test_a_block_behind_rows_of_its_own(kvg):
    """A sequence whose own pages come before a block's: those that stay, stay the block's."""
    bed = Bed(kvg, 1, 1, 64, 16, 60, 3, 400)
    store = kvg.PoolStore(bed.cache, 1 << 24)
    bed.append(2, 100)
    block = kvg.kvg_deposit(store.h, bed.cache.h, 2, 0, 100)
    for rows, first in [(120, 100), (110, 64), (130, 32), (120, 0)]:
        kvg.kvg_cache_release(bed.cache.h, 0)
        bed.append(0, 48)
        kvg.kvg_graft(store.h, block, bed.cache.h, 0)
        bed.set_weights(0, heavy_tailed(bed.rng, 148))
        evict(bed, [0], [rows], first, 3, [1])
        evict(bed, [0], [rows], first, 3)
    out = torch.zeros(1, 2, 2, 64, dtype=torch.bfloat16, device="cuda")
    kvg.kvg_decode_attention_shared(bed.cache.h, 0, [0, 1], torch.randn_like(out).data_ptr(), 2, out.data_ptr(), 0.1)
    kvg.kvg_sync(bed.cache.h)


def test_one_source_for_several_and_other_orders(kvg):
    bed = Bed(kvg, 1, 2, 64, 16, 120, 6, 300)
    bed.append(0, 200)
    bed.append(1, 77)
    bed.append(3, 150)  # (a destination that holds rows already, more than it will)
    bed.set_weights(0, heavy_tailed(bed.rng, 200))
    bed.set_weights(1, heavy_tailed(bed.rng, 77))
    bed.set_weights(3, heavy_tailed(bed.rng, 150))
    evict(bed, [0, 0, 0, 1], [50, 100, 200, 76], 2, 2, [3, 5, 4, 1])
    evict(bed, [2], [10], 2, 2, [4])  # an empty source
    evict(bed, [0], [60], 2, 2, [2])  # a destination that was empty


def test_more_sequences_than_a_launch_takes(kvg):
    n = 150
    bed = Bed(kvg, 1, 1, 64, 16, 20 * n, n, 160)
    for b in range(n):
        bed.append(b, (b * 37) % 150)
        bed.set_weights(b, heavy_tailed(bed.rng, (b * 37) % 150))
    evict(bed, range(n), [(b * 13) % 100 + 2 for b in range(n)], 1, 1)


@pytest.mark.parametrize("how", ["in place", "to another"])
def test_more_pages_than_a_launch_takes(kvg, how):
    bed = Bed(kvg, 1, 2, 64, 1, 9000, 4, 4000)
    for b, n in enumerate((3500, 40, 2000)):
        bed.append(b, n)
        bed.set_weights(b, heavy_tailed(bed.rng, n))
    if how == "in place":
        evict(bed, [1, 0, 2], [30, 2500, 1024], 3, 3)
    else:
        evict(bed, [0], [2500], 3, 3, [3])


def test_attention_over_what_is_left_is_that_of_the_same_rows(kvg):
    """Decode over a thinned sequence against a cache that was only ever given its rows, bit for bit."""
    bed = Bed(kvg, 2, 2, 128, 64, 40, 2, 1000)
    shape = 2, 900, 2, 128
    k, v = (torch.randn(shape, device="cuda").to(torch.bfloat16) for _ in range(2))
    pos = torch.arange(900, dtype=torch.int32, device="cuda")
    kvg.kvg_cache_append(bed.cache.h, 0, k.data_ptr(), v.data_ptr(), pos.data_ptr(), 900)
    w = heavy_tailed(bed.rng, 900)
    bed.set_weights(0, w)
    evict(bed, [0], [333], 4, 100)
    kept = torch.tensor(kept_slots([64] * 14 + [4], 64, np.asarray(w, np.float32), 333, 4, 100), device="cuda")
    fresh = Bed(kvg, 2, 2, 128, 64, 40, 2, 1000, seed=5)
    kk, vv, pp = k[:, kept].contiguous(), v[:, kept].contiguous(), pos[kept].contiguous()
    kvg.kvg_cache_append(fresh.cache.h, 0, kk.data_ptr(), vv.data_ptr(), pp.data_ptr(), 333)
    q = torch.randn(2, 1, 4, 128, device="cuda").to(torch.bfloat16)
    outs = []
    for b in (bed, fresh):
        b.append(0, 0)
        out = torch.empty_like(q)
        kvg.kvg_decode_attention(b.cache.h, -1, [0], q.data_ptr(), 4, out.data_ptr(), 0.1)
        torch.cuda.synchronize()
        outs.append(out.view(torch.int16))
    assert torch.equal(*outs)


def test_calls_on_two_streams(kvg):
    """Two streams that share the cache's scratch."""
    bed = Bed(kvg, 2, 2, 64, 16, 900, 4, 4000)
    for b in (0, 1):
        bed.append(b, 3000 + b)
        bed.set_weights(b, heavy_tailed(bed.rng, 3000 + b))
    streams = [torch.cuda.Stream() for _ in range(2)]
    evict(bed, [0], [1000], 4, 50, [2])
    evict(bed, [1], [1100], 4, 50, [3])
    want = bed.snapshot()
    torch.cuda.synchronize()
    for _ in range(20):
        for b, s in enumerate(streams):
            kvg.kvg_cache_evict(bed.cache.h, [b], [1000 + 100 * b], 4, 50, bed.weights.data_ptr(), dst_ids=[2 + b], stream=s)
    got = bed.snapshot()
    assert torch.equal(got[0], want[0]) and all(np.array_equal(a, b) for a, b in zip(got[1], want[1]))


def test_pages_far_into_a_pool(kvg):
    """Pages at the far end of a pool of 5.2 GB."""
    bed = Bed(kvg, 1, 8, 256, 64, 10000, 2, 1000)
    bed.kvg.kvg_cache_set_free_order(bed.cache.h, np.arange(10000)[::-1])
    bed.append(0, 700)
    bed.set_weights(0, heavy_tailed(bed.rng, 700))
    v = bed.cache.view
    pool = bed.pool[:, :, 9900:].clone()
    bed.kvg.kvg_cache_evict(bed.cache.h, [0], [100], 4, 10, bed.weights.data_ptr(), dst_ids=[1])
    torch.cuda.synchronize()
    table = bed.tables()[0]
    k = np.array(kept_slots([64] * 10 + [60], 64, bed.weights[0].cpu().numpy(), 100, 4, 10))
    got = bed.pool[0, :, torch.from_numpy(table[1][np.arange(100) // 64].astype(np.int64)).cuda(), :,
                   torch.arange(100, device="cuda") % 64]
    want = pool[0, :, torch.from_numpy(table[0][k // 64].astype(np.int64) - 9900).cuda(), :,
                torch.from_numpy(k % 64).cuda()]
    assert v.pool_bytes > 5 * 10 ** 9 and torch.equal(got, want)


def test_refusals_change_nothing(kvg):
    bed = Bed(kvg, 2, 2, 64, 16, 22, 4, 200)
    bed.append(0, 150)
    bed.append(1, 100)
    bed.set_weights(0, heavy_tailed(bed.rng, 150))
    before = bed.snapshot()

    def refused(seqs=(0,), rows=(50,), first=1, last=1, weights=bed.weights.data_ptr(), dst=None,
                status=kvg.KVG_ERR_ARG):
        with pytest.raises(kvg.KvgError) as e:
            kvg.kvg_cache_evict(bed.cache.h, list(seqs), list(rows), first, last, weights, dst_ids=dst)
        assert e.value.status == status

    refused(seqs=(4,))
    refused(seqs=(-1,))
    refused(dst=[4])
    refused(rows=(-1,), first=0, last=0)
    refused(rows=(1,))
    refused(first=-1)
    refused(last=-1)
    refused(first=2 ** 31 - 1, last=2 ** 31 - 1)
    refused(weights=None)
    refused(weights=bed.weights.data_ptr() + 2)
    refused(seqs=(), rows=())
    refused(seqs=(0, 0), rows=(50, 40))
    refused(seqs=(0, 1), rows=(50, 40), dst=[2, 2])
    refused(seqs=(0, 1), rows=(50, 40), dst=[1, 2])  # 1 would be read and written
    refused(seqs=(0, 0), rows=(50, 40), dst=[0, 2])
    refused(rows=(150,), dst=[2], status=kvg.KVG_ERR_CAPACITY)  # 10 pages, 5 are free
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        refused()
        bed.weights.add_(0)  # (a graph of something)
    after = bed.snapshot()
    assert torch.equal(before[0], after[0]) and all(np.array_equal(a, b) for a, b in zip(before[1], after[1]))
    assert bed.slots(0) == (150, 10)
    evict(bed, [0], [50], 1, 1)
