"""make_qkv: tensors that are not what kvg_qkv describes are refused before
their memory is read as if they were; a stride that nothing uses does not
matter."""
import pytest
import torch

from paper_2607_14431_gb300 import kvg

BF16 = torch.bfloat16


def qkv(q=(5, 4, 64), k=(5, 2, 64), v=(5, 2, 64), dtype=BF16, **kw):
    return kvg.make_qkv(*(None if s is None else torch.zeros(s, dtype=dtype) for s in (q, k, v)), **kw)


def test_other_types_are_refused():
    for dtype in (torch.float16, torch.float32, torch.float8_e4m3fn):
        with pytest.raises(ValueError):
            qkv(dtype=dtype)
    with pytest.raises(ValueError):
        qkv(q_norm=torch.ones(64, dtype=torch.float16))
    assert qkv().n_q_heads == 4 and qkv(dtype=torch.int16).k_token == 128  # bf16, or its bits


@pytest.mark.parametrize("shapes", [
    {"q": (4, 4, 64)}, {"v": (4, 2, 64)}, {"q": (5, 4, 128)}, {"v": (5, 4, 64)}, {"v": (5, 2, 128)},
    {"q": (3, 5, 4, 64), "k": (2, 5, 2, 64), "v": (2, 5, 2, 64)}])
def test_shapes_that_do_not_agree_are_refused(shapes):
    with pytest.raises(ValueError):
        qkv(**shapes)


def test_weights_of_another_head_dim_are_refused():
    with pytest.raises(ValueError):
        qkv(k_norm=torch.ones(128, dtype=BF16))
    qkv(k_norm=torch.ones(64, dtype=BF16))
    qkv((2, 5, 4, 64), (2, 5, 2, 64), (2, 5, 2, 64), q_norm=torch.ones(2, 64, dtype=BF16))
    qkv((1, 5, 4, 64))  # one layer, named or not


def test_one_token_of_a_wide_buffer():
    """Rows of 8 x 64 + 3 elements: a token's stride is no multiple of 8, but there is one token."""
    x = torch.zeros(1, 8 * 64 + 3, dtype=BF16)[:, :512].view(1, 8, 64)
    c = kvg.make_qkv(*x.split([4, 2, 2], dim=1))
    assert (c.q_token, c.k_token, c.v_token) == (0, 0, 0) and (c.k - c.q, c.v - c.k) == (512, 256)
