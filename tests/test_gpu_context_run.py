"""The calls for contexts that hold more than text, one after the other as a
decoder with an encoder would make them: rows with positions on three axes enter
the cache, the prompt's attention weighs them, the context is thinned, decode
steps weigh and thin it further, and every step also attends to the encoder's
states.  Each step is checked against its definition in 64 bits over the rows that
the cache holds, and the choice of rows against the weights of that definition."""
import math

import numpy as np
import pytest
import torch

from kvg_testlib import dev_view, need_gpu
from test_gpu_prompt_attention import Bed, check, normal

pytestmark = pytest.mark.gpu
LAYERS, HQ, HKV = 2, 4, 2


@pytest.fixture(scope="module")
def kvg():
    return need_gpu()


def attend(q, k, v, scale, past=None):
    """(out [n][Hq][D], weights [N]); row i sees the first past + i + 1 rows, or (past None) all."""
    k, v = (x.repeat_interleave(HQ // HKV, 1) for x in (k, v))
    x = torch.einsum("nhd,khd->hnk", q.double(), k) * scale
    if past is not None:
        x = x.masked_fill(torch.arange(k.shape[0], device="cuda") > past + torch.arange(len(q), device="cuda")[:, None], -math.inf)
    w = torch.softmax(x, -1)
    return torch.einsum("hnk,khd->nhd", w, v), w.sum((0, 1))


@pytest.mark.parametrize("d,page,fp8", [(128, 64, False), (256, 16, False), (128, 16, True), (64, 24, False)])
def test_prompt_thin_steps_and_cross_attention(kvg, d, page, fp8):
    lens, budget, first, last, steps = [300, 77, 130], 100, 4, 16, 5
    bed = Bed(kvg, LAYERS, HKV, d, page, 120 if page < 64 else 40, 3, 400, fp8)
    states = Bed(kvg, LAYERS, HKV, d, page, 60 if page < 64 else 20, 2, 400, fp8)
    for b, n in enumerate((211, 64)):
        states.append(b, n, 100 + b)
    rotary = kvg.Rotary(d, d, 1e4, sections=[d // 4, d // 8, d // 8], layout=kvg.KVG_ROPE_AXES_SECTIONS)
    weights = torch.zeros(3, 400, device="cuda")
    sums = [torch.zeros(0, dtype=torch.float64, device="cuda") for _ in lens]  # of the rows that are left, in 64 bits
    tags = [np.zeros(0, np.int32) for _ in lens]
    scale, rng = 1 / math.sqrt(d), np.random.default_rng(5)

    def forward(rows, seed, decay):
        t = sum(rows)
        places = torch.from_numpy(rng.integers(0, 1000, (3, t)).astype(np.int32)).cuda()
        x = normal(seed, LAYERS, t, HQ + 2 * HKV, d)
        q_out, out = (torch.zeros(LAYERS, t, HQ, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        crossed = torch.zeros_like(out)
        for l in range(LAYERS):
            qkv = kvg.make_qkv(*x[l].split([HQ, HKV, HKV], dim=1))
            kvg.kvg_cache_append_qkv(bed.cache.h, l, [0, 1, 2], rows, qkv, rotary.h, places.data_ptr(), q_out[l].data_ptr())
            kvg.kvg_attention_weights(bed.cache.h, l, [0, 1, 2], rows, q_out[l].data_ptr(), HQ, out[l].data_ptr(), scale,
                                      weights.data_ptr(), decay if l == 0 else 1.0)
            kvg.kvg_cross_attention(states.cache.h, l, [0, 1, 0], rows, out[l].data_ptr(), HQ, crossed[l].data_ptr(), scale)
        torch.cuda.synchronize()
        at = 0
        for b, n in enumerate(rows):
            if n == 0:
                continue  # (left as it is, not decayed either)
            total = torch.zeros(len(tags[b]) + n, dtype=torch.float64, device="cuda")
            total[:len(tags[b])] = decay * sums[b]
            for l in range(LAYERS):
                _, k, v = bed.rows(b, l)
                assert len(k) == len(total)
                want, w = attend(q_out[l, at:at + n], k, v, scale, len(k) - n)
                check(out[l, at:at + n], want, f"seq {b} layer {l}")
                total += w
                _, k, v = states.rows([0, 1, 0][b], l)
                check(crossed[l, at:at + n], attend(out[l, at:at + n], k, v, scale)[0], f"states of {b} layer {l}")
            sums[b] = total
            tags[b] = np.concatenate([tags[b], places[0, at:at + n].cpu().numpy()])
            got = weights[b, :len(total)].double()
            assert float(((got - total).abs() / total).max()) < 1e-3  # (test_gpu_attention_weights has the bound)
            at += n

    def thin():
        before = weights.double()
        kvg.kvg_cache_evict(bed.cache.h, [0, 1, 2], [budget] * 3, first, last, weights.data_ptr())
        torch.cuda.synchronize()
        v = bed.cache.view
        pos = dev_view(v.positions, 4 * v.max_seqs * v.max_slots, torch.int32).view(v.max_seqs, -1).cpu().numpy()
        for b in range(3):
            n = len(tags[b])
            kept = np.arange(n)
            if n > budget:
                middle = before[b, first:n - last].cpu().numpy()
                best = np.argsort(-middle, kind="stable")[:budget - first - last] + first
                kept = np.concatenate([np.arange(first), np.sort(best), np.arange(n - last, n)])
            assert kvg.kvg_cache_seq_info(bed.cache.h, b)[0] == len(kept)
            assert np.array_equal(pos[b, :len(kept)], tags[b][kept])
            tags[b], sums[b] = tags[b][kept], sums[b][torch.from_numpy(kept).cuda()]

    forward(lens, 1, 1.0)
    thin()
    for i in range(steps):
        forward([1, 1, 1], 10 + i, 0.9)
        if i % 2:
            thin()
    forward([40, 0, 3], 30, 0.5)
    kvg.kvg_sync(bed.cache.h)
    kvg.kvg_sync(states.cache.h)
