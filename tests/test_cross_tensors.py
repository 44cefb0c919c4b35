"""What cross attention is told of torch tensors: address and stride of their rows."""
import pytest
import torch

from paper_2408_04275_amd import binding as mm


def strides(*tensors):
    t = mm.make_cross_attn_tensors(*tensors)
    return t.ld_q, t.ld_k, t.ld_v, t.ld_o


def test_strides_of_rows_and_of_columns_of_wider_ones():
    q, kv, o = torch.zeros(3, 32), torch.zeros(5, 80), torch.zeros(3, 48)[:, :32]
    assert strides(q, kv[:, :32], kv[:, 32:64], o) == (32, 80, 80, 48)
    g = mm.make_cross_attn_grads(o, None, kv[:, :32], kv[:, 32:64])
    assert (g.d_q, g.ld_dq, g.ld_do, g.ld_dk, g.ld_dv) == (None, 0, 48, 80, 80) and g.d_v - g.d_k == 128


def test_one_row_has_no_stride_of_its_own():
    # torch keeps any number there: a transposed column is a contiguous row with a stride of 1
    one = torch.zeros(32, 1).t()
    assert one.is_contiguous() and one.stride(0) == 1
    assert strides(one, one, one, one) == (32,) * 4
    assert strides(torch.zeros(4, 32)[:1], torch.zeros(0, 32), torch.zeros(1, 64)[:, 32:], one)[1:] == (32, 32, 32)


def test_columns_that_are_not_neighbours_are_refused():
    bad = torch.zeros(32, 4).t()
    for args in ((bad, bad, bad, bad), (torch.zeros(4, 64)[:, ::2],) * 4, (torch.zeros(2, 2, 16),) * 4):
        with pytest.raises(ValueError):
            mm.make_cross_attn_tensors(*args)
