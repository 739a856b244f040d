"""Sizes and strides that the calls hold in 32 bits: refused in the library's manner where they are wider, and not looked at where no
index is multiplied with them."""
import pytest
import torch

import paper_2402_06262_b200 as R

pytestmark = pytest.mark.gpu
UNSUPPORTED = 2


def rotate(S, start):
    x = torch.randn(S, 1, 3, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    Q, K, V = torch.zeros(S, 1, 1, 1, 64, device="cuda"), torch.zeros(S, 1, 1, 64, device="cuda"), torch.zeros(S, 1, 1, 64, device="cuda")
    rotary = R.Rotary(64, [0.1] * 32)
    R.roco_norm_rotate(rotary, x[:, :, :1], x[:, :, 1:2], x[:, :, 2:], Q, K, V, start=start)
    return Q, K, V


def test_stride_of_the_only_start():
    """A column of a table of one row may have any stride."""
    one = torch.tensor([9], dtype=torch.int32, device="cuda")
    for wide in (2 ** 31, 2 ** 40):
        start = one.as_strided((1,), (wide,))
        assert start.stride(0) == wide
        assert all(torch.equal(a, b) for a, b in zip(rotate(1, start), rotate(1, one)))


def test_starts_too_far_apart_are_refused():
    table = torch.empty(2 ** 31 + 1, dtype=torch.int32, device="cuda")
    with pytest.raises(R.RocoError) as e:
        rotate(2, table.as_strided((2,), (2 ** 31,)))
    assert e.value.code == UNSUPPORTED


def test_vocabularies_beyond_32_bits_are_refused():
    target = torch.empty(1, 1, 2 ** 31, dtype=torch.bfloat16, device="cuda")
    i, u = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, 1, device="cuda")
    with pytest.raises(R.RocoError) as e:
        R.roco_tree_verify(target, i, i, u, u[0], i, i[0], i[0], i[0])
    assert e.value.code == UNSUPPORTED
