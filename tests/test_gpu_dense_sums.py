"""How the E4M3 products sum: FP32 where the contract says so, the 8-bit instruction's cut where it says that.

Bounds: FP32 sums (one multiply-add per block of K onto a partial sum, some 16 roundings inside a block) are within (blocks + 16) 2^-24 S of
the formula, S = sum |x||w|; a BF16 output adds half a unit, 2^-8 relative.  Such sums of h change a code of it (a step of at most an eighth) in at most 1e-4 of the
cases, which adds less than 9e-4 in quadrature to the 1.66e-3 of the output's rounding: 2e-3 in the norm."""
import numpy as np
import pytest
import torch

from oracle import dense
from gpu_helpers import rel_fro, say
from test_gpu_dense import _acts, _bf16, _np, _rows_of, _weight_of

pytestmark = pytest.mark.gpu

F32_NORM_TOL = 2e-3


@pytest.fixture(scope="module")
def R():
    import paper_2604_19503_amd as R
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    R.load_library()
    return R


def _f32_bound(S, K):
    return 2.0 ** -24 * (-(-K // 128) + 16) * S


def _feed_forward(R, T, H, I, add, f32_sums):
    rng = np.random.default_rng(T + H + I)
    x, xv = _rows_of(R, _acts(rng, T, H))
    w13, v13 = _weight_of(R, rng.standard_normal((2 * I, H)) * 0.02)
    w2, v2 = _weight_of(R, rng.standard_normal((H, I)) * 0.02)
    a = _bf16(rng.standard_normal((T, H))) if add else None
    need = R.load_library().realb_gated_ffn_workspace_bytes(T, I)
    work = torch.zeros(need + 16, dtype=torch.uint8, device="cuda")
    work[need:] = 0x5A
    out = torch.full((T + 1, H), 9.0, dtype=torch.bfloat16, device="cuda")
    R.gated_ffn_fp8(R.make_ffn_io(x, w13, w2, out[:T], add=a, workspace=work[:need], f32_sums=f32_sums))
    torch.cuda.synchronize()
    assert bool((work[need:] == 0x5A).all()) and bool((out[T] == 9.0).all())
    return xv, v13, v2, None if a is None else _np(a), work, _np(out[:T])


@pytest.mark.parametrize("T,H,I,add", [(65, 256, 384, True), (130, 640, 1408, False), (300, 128, 1408, True), (700, 2048, 768, False), (1922, 128, 384, False), (6500, 256, 640, True)])
def test_feed_forward_with_fp32_sums(R, T, H, I, add):
    say("gpu-sums", f"ffn {T} x {H} x {I}, FP32 sums")
    xv, v13, v2, a, work, got = _feed_forward(R, T, H, I, add, True)
    q = work[: T * I].view(T, I).cpu().numpy()
    s = work[T * I: T * I + (I // 128) * (-(-T // 4) * 4) * 4].view(torch.float32).view(I // 128, -1)[:, :T].cpu().numpy()
    gu, S = xv @ v13.T, np.abs(xv) @ np.abs(v13).T
    h, g = dense.swiglu(gu), gu[:, :I]
    moved = _f32_bound(S[:, I:] * np.abs(g / (1 + np.exp(-g))) + S[:, :I] * 1.1 * np.abs(gu[:, I:]), H)
    hv = dense.decode_rows(q, s)
    step = np.maximum(2.0 ** -4 * np.abs(h), 2.0 ** -10 * np.repeat(s.T, 128, 1))
    # (a code's value is at most 1.07 of what it stands for; SwiGLU in FP32: 1e-5 of the element)
    assert (np.abs(hv - h) <= 1.07 * moved + 1.001 * step + 1e-5 * np.abs(h) + 1e-30).all()
    staged = dense.linear(hv, v2, None, a)
    S2 = np.abs(hv) @ np.abs(v2).T + (0.0 if a is None else np.abs(a))
    assert (np.abs(got - staged) <= _f32_bound(S2, I) + 1.001 * 2.0 ** -8 * np.abs(staged) + 1e-30).all()
    end_to_end = rel_fro(got, dense.gated_ffn(xv, v13, v2, a)[2])
    say("gpu-sums", f"off the formula by {end_to_end:.2e}")
    assert end_to_end <= F32_NORM_TOL


def test_fp32_sums_are_what_few_rows_have_anyway(R):
    for T in (1, 24, 64):
        outs = [_feed_forward(R, T, 256, 384, True, f32)[-1] for f32 in (False, True)]
        assert np.array_equal(*outs)
