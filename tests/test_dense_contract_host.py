"""What the argument blocks and the binding of the operators around the MoE layer promise, where no GPU is needed to see it."""
import ctypes as C

import pytest
import torch

import paper_2604_19503_amd as R
from paper_2604_19503_amd import binding as B

P = 0x100000                                             # an address whose alignment suits everything; nobody reads it


def _ffn_io(**kw):
    io = B.FfnIO()
    for k, v in {**dict(T=4, H=256, I=128, x_q=P, ld_x=256, x_s=P, ld_xs=4, w13_q=P, w13_s=P, w2_q=P, w2_s=P, out=P, ld_out=256, workspace=P, workspace_bytes=1 << 20), **kw}.items():
        setattr(io, k, v)
    return io


@pytest.mark.parametrize("sums", [-1, 2])
def test_feed_forward_refuses_unknown_sums(sums):
    lib = R.load_library()
    assert lib.realb_gated_ffn_fp8(C.byref(_ffn_io(T=100, ld_xs=100, sums=sums)), None) == -1 and b"sums" in lib.realb_last_error()


def test_sums_lie_where_older_blocks_had_padding():
    """A caller that fills the block field by field and clears it first needs no change."""
    assert B.FfnIO.sums.offset == 12 and B.FfnIO.x_q.offset == 16
