"""The example's decoder block over several ranks: the sum of their partial outputs goes into the stream, on each of them.  Two ranks one after the
other on one GPU, the second's output handed to the first; bounds as in test_gpu_decoder_block.py."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import bf16 as obf, dense, layer as olayer
from gpu_helpers import BF16_TOL, FP4_E2E_TOL, rel_fro
from test_gpu_decoder_block import _np, _value, _weight

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("T,force", [(40, 0), (300, 1)])
def test_the_block_adds_all_ranks_outputs(T, force):
    import paper_2604_19503_amd as R
    from decoder_block import DecoderBlockHalf
    H, I, E, k, D = 256, 128, 16, 2, 2
    parts = []
    ranks = [DecoderBlockHalf(T, E=E, k=k, D=D, H=H, I=I, I_shared=384, rank=r, force=force, scale=0.5, seed=T,
                              sum_ranks=(lambda t: parts.append(t.clone())) if r else (lambda t: t.add_(parts[0]))) for r in (0, 1)]
    stream = _np(ranks[0].stream)
    assert not torch.equal(ranks[0].w13, ranks[1].w13) and torch.equal(ranks[0].w_shared13, ranks[1].w_shared13)
    for half in reversed(ranks):
        assert half.run() == force
    torch.cuda.synchronize()
    bits = lambda t: R.bits_from_bf16(t)  # noqa: E731
    want = 0.0
    for r, half in enumerate(ranks):
        assert torch.equal(half.x, ranks[0].x) and torch.equal(half.logits, ranks[0].logits)
        inp = dict(logits=half.logits.cpu().numpy(), is_vision=half.is_vision.cpu().numpy(), x=bits(half.x), w13=bits(half.w13), w2=bits(half.w2))
        want = want + olayer.rank_layer(inp, E, k, D, r, 0.9, force=force)["out"]
    half = ranks[0]
    got = obf.bits_to_f64(bits(half.buf.out))
    assert np.linalg.norm(got - want) <= (FP4_E2E_TOL if force else BF16_TOL) * np.linalg.norm(want)
    y = dense.gated_ffn(_value(half.x_q), _weight(half.w_shared13), _weight(half.w_shared2), got)[2]
    assert rel_fro(_np(half.y), y) <= FP4_E2E_TOL
    stream1 = dense.residual_norm(stream, _np(half.projected), pre_w=_np(half.norm_w))[0]
    stream2 = dense.residual_norm(stream1, _np(half.y), scale=0.5, pre_w=_np(half.next_norm_w))[0]
    assert np.abs(_np(half.stream) - stream2).max() <= 1e-5 * (1 + np.abs(stream2).max())
