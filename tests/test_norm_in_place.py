"""CPU-side check of layer norm in place: the rows of both tensors are the same ones, or the call is refused.  (Accepted calls get an unaligned pointer,
which is looked at after the shape: nothing is launched.)"""
import pytest

from paper_2505_03803_amd import binding as B
from test_heads_abi import FAKE, norm, norm_backward


@pytest.mark.parametrize("M,xs,ys,status", [(4, 128, 0, B.ERR_SHAPE), (4, 0, 72, B.ERR_SHAPE), (2, 72, 80, B.ERR_SHAPE),
                                            (4, 128, 128, B.ERR_ALIGN), (4, 64, 0, B.ERR_ALIGN),
                                            (1, 128, 0, B.ERR_ALIGN)])
def test_strides_in_place(M, xs, ys, status):
    assert norm(M=M, xs=xs, ys=ys, w=FAKE + 2) == status
    assert norm(M=M, xs=xs, ys=ys, y=FAKE + 16, w=FAKE + 2) == B.ERR_ALIGN
    assert norm_backward(M=M, dys=xs, dxs=ys, w=FAKE + 2) == status
    assert norm_backward(M=M, dys=xs, dxs=ys, dx=FAKE + 16, w=FAKE + 2) == B.ERR_ALIGN
