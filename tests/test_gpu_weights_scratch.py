"""The scratch of kvg_attention_weights: how it grows with a sequence, and what
KVG_WEIGHTS_SCRATCH_KB bounds."""
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
