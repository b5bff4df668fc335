"""The scratch of kvg_attention_weights: how it grows with a sequence, and what
KVG_WEIGHTS_SCRATCH_KB bounds."""
import json
import os
import subprocess
import sys

import pytest
import torch

from kvg_testlib import need_gpu
from test_gpu_prompt_attention import Bed, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvg():
    return need_gpu()


def growing(kvg, n, steps, capture):
    """Decodes `steps` tokens onto a sequence of n rows, each step captured (after an eager call, or one only where the
    capture was refused); returns how many captures were refused and the device memory taken meanwhile."""
    hq, n_l, d = 16, 16, 64
    bed = Bed(kvg, n_l, 4, d, 64, n // 64 + 4, 1, n + 128)
    bed.append(0, n, 1)
    q = normal(3, n_l, 1, hq, d)
    out, weights = torch.zeros_like(q), torch.zeros(1, n + 128, device="cuda")

    def call():
        kvg.kvg_attention_weights(bed.cache.h, -1, [0], [1], q.data_ptr(), hq, out.data_ptr(), 0.125, weights.data_ptr(), 0.0)

    def captured():
        graph = torch.cuda.CUDAGraph()
        try:
            with torch.cuda.graph(graph):
                call()
        except kvg.KvgError:
            return None
        return graph

    call()
    captured()  # (what the first capture takes)
    torch.cuda.synchronize()
    before, refused = torch.cuda.mem_get_info()[0], 0
    for i in range(steps):
        bed.append(0, 1, 10 + i)
        if not capture:
            call()
        graph = captured()
        if graph is None:
            refused += 1
            call()
            graph = captured()
        call()
        want, seen = out.clone(), weights.clone()
        out.zero_()
        weights.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        m = n + 1 + i
        assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and torch.equal(weights[:, :m], seen[:, :m])
        assert abs(float(weights[0, :m].sum()) - hq * n_l) < 1e-3 * hq * n_l
    return refused, before - torch.cuda.mem_get_info()[0]


def test_steps_of_a_growing_sequence_are_captured_without_an_eager_call(kvg):
    """The scores take 1 KB a slot.  A buffer grows by a half at a time, so that of 40 steps one is refused at most."""
    refused, _ = growing(kvg, 3000, 40, True)
    assert refused <= 1


def test_captured_steps_of_a_growing_sequence_keep_little(kvg):
    """What graphs may still replay is kept: of 12 MB of scores each time they grow, which is not with every step (then
    it would be 480 MB).  The first buffer, the next one of half as much again, and what graphs take beside them."""
    _, taken = growing(kvg, 12000, 40, False)
    assert taken <= 100 << 20


PROBE = r"""
import json, sys
sys.path[:0] = [sys.argv[1], sys.argv[2]]
import torch
from kvg_testlib import need_gpu
from test_gpu_attention_weights import run
from test_gpu_prompt_attention import Bed, normal
kvg = need_gpu()

def launches(bed, hq, *args, **kw):
    n = kvg.kvg_launch_count()
    run(bed, hq, *args, **kw)  # (checks outputs and weights)
    return kvg.kvg_launch_count() - n

res = {}
bed = Bed(kvg, 4, 2, 64, 64, 40, 3, 800)
for b, n in enumerate((300, 640, 700)):
    bed.append(b, n, 1 + b)
res["steps of four layers"] = launches(bed, 4, [0, 1, 2], [1, 1, 1], layer=-1)
res["steps of a layer"] = launches(bed, 4, [0, 1, 2], [1, 1, 1], layer=1)
res["prompts of four layers"] = launches(bed, 4, [0, 1, 2], [30, 200, 5], layer=-1)
res["prompts of a layer"] = launches(bed, 4, [0, 1, 2], [30, 200, 5], layer=1, decay=0.5,
                                     before=torch.rand(3, 800, device="cuda"))
kvg.kvg_cache_set_layer_windows(bed.cache.h, [400, 0, 400, 90])
res["windows"] = launches(bed, 4, [2, 1, 0], [100, 2, 77], [400, 0, 400, 90], layer=-1, decay=-1.0,
                          before=torch.rand(3, 800, device="cuda"))

# 48 sequences of 8,000 rows, 8 KV heads of one layer: 12.6 MB of sums
bed = Bed(kvg, 1, 8, 64, 64, 48 * 125, 48, 8000)
for b in range(48):
    bed.append(b, 8000, b)
q = normal(5, 1, 144, 8, 64)
out, weights = torch.zeros_like(q), torch.zeros(48, 8000, device="cuda")

def call(n):
    kvg.kvg_attention_weights(bed.cache.h, 0, list(range(n)), [3] * n, q.data_ptr(), 8, out.data_ptr(), 0.125,
                              weights.data_ptr(), 0.0)
    torch.cuda.synchronize()

kvg.kvg_prompt_attention(bed.cache.h, 0, list(range(48)), [3] * 48, q.data_ptr(), 8, out.data_ptr(), 0.125)
call(1)
before = torch.cuda.mem_get_info()[0]
call(48)
res["bytes"] = before - torch.cuda.mem_get_info()[0]
print(json.dumps(res))
"""


def probed(kb):
    need_gpu()
    here = os.path.dirname(os.path.abspath(__file__))
    env = {k: v for k, v in os.environ.items() if k != "KVG_WEIGHTS_SCRATCH_KB"}
    r = subprocess.run([sys.executable, "-c", PROBE, os.path.dirname(here), here],
                       env=env | ({"KVG_WEIGHTS_SCRATCH_KB": str(kb)} if kb else {}), capture_output=True, text=True,
                       timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    return json.loads(r.stdout.strip().splitlines()[-1])


def test_little_scratch_takes_more_launches_and_little_memory(kvg):
    """8 KB: a layer's scores of one row, and the sums of one sequence and layer, at a time.  The sums of a batch are
    divided among passes (the buffer has 1 MB at least; logarithms take 5 KB here)."""
    plain, little = probed(0), probed(8)
    for what, n in plain.items():
        if what != "bytes":
            assert little[what] > n, what
    # Two launches a pass.  The sums of 700 and of 640 rows, 3 pairs of 128-key tiles, take 3 x 256 x 2 heads x 4 B = 6 KB:
    # a layer at a time; those of 300 rows, 2 pairs, 4 KB: two layers at a time.  No two sequences go together.
    assert little["prompts of four layers"] - plain["prompts of four layers"] == 2 * (4 + 4 + 2 - 1)
    assert little["prompts of a layer"] - plain["prompts of a layer"] == 2 * (3 - 1)
    assert plain["bytes"] >= 12 << 20 and little["bytes"] <= 4 << 20
