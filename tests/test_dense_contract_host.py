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


@pytest.mark.parametrize("I", [128, 1408, 4096])
def test_a_workspace_for_the_largest_batch_holds_smaller_ones(I):
    """h of few rows is FP32, of more rows codes: what the size function returns never falls where T grows."""
    size = R.load_library().realb_gated_ffn_workspace_bytes
    sizes = [size(T, I) for T in range(0, 700)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))
    for T, need in ((1, 4 * I), (64, 64 * 4 * I), (65, 65 * I + 68 * (I // 128) * 4), (600, 600 * I + 600 * (I // 128) * 4)):
        assert sizes[T] >= need


def test_a_call_refuses_only_what_it_cannot_use():
    """One byte less than h takes is refused; a workspace of the largest of several batches is not (those calls go on to the next check)."""
    lib = R.load_library()
    for T, need in ((17, 17 * 128 * 4), (64, 64 * 128 * 4), (65, 65 * 128 + 68 * 4)):
        for room, why in ((need - 1, b"workspace"), (need, b"rows of out"), (lib.realb_gated_ffn_workspace_bytes(65, 128), b"rows of out")):
            assert lib.realb_gated_ffn_fp8(C.byref(_ffn_io(T=T, ld_xs=T, workspace_bytes=room, ld_out=1)), None) == -1
            assert why in lib.realb_last_error(), (T, room, lib.realb_last_error())
