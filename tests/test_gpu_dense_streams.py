"""What the binding allocates by itself and the streams that use it: another stream's pending work on memory of its own pool is left
alone, and nobody gets a workspace back while a call uses it.  The streams are ordered by nothing but that; a device-side sleep keeps one behind the other."""
import numpy as np
import pytest
import torch

from test_gpu_dense import _bf16, _rows_of, _weight_of

pytestmark = pytest.mark.gpu

SLEEP = 100_000_000                                      # cycles, some 50 ms


@pytest.fixture(scope="module")
def R():
    import paper_2604_19503_amd as R
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    R.load_library()
    return R


def _block(R, T, H=256, I=384):
    rng = np.random.default_rng(T)
    x, _ = _rows_of(R, rng.standard_normal((T, H)))
    w13, _ = _weight_of(R, rng.standard_normal((2 * I, H)) * 0.05)
    w2, _ = _weight_of(R, rng.standard_normal((H, I)) * 0.05)
    want, out = (torch.zeros((T, H), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    R.gated_ffn_fp8(R.make_ffn_io(x, w13, w2, want))
    torch.cuda.synchronize()
    return (x, w13, w2, out), want, R.load_library().realb_gated_ffn_workspace_bytes(T, I)


@pytest.mark.parametrize("T", [24, 300])
def test_a_call_on_another_stream_leaves_pending_work_alone(R, T):
    args, want, need = _block(R, T)
    side = torch.cuda.Stream()
    copy = torch.empty(need, dtype=torch.uint8, device="cuda")
    victim = torch.full((need,), 1, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    torch.cuda._sleep(SLEEP)
    copy.copy_(victim)                                   # pending while the call runs
    del victim
    io = R.make_ffn_io(*args)
    R.gated_ffn_fp8(io, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert bool((copy == 1).all()) and torch.equal(args[3], want)


@pytest.mark.parametrize("T", [24, 300])
def test_arguments_may_go_while_the_call_runs(R, T):
    args, want, need = _block(R, T)
    side = torch.cuda.Stream()
    io = R.make_ffn_io(*args)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(SLEEP)
    R.gated_ffn_fp8(io, stream=side)
    del io
    others = [torch.full((need,), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(4)]      # on the current stream, at once
    torch.cuda.synchronize()
    assert torch.equal(args[3], want) and all(bool((t == 0x7F).all()) for t in others)


def test_encoders_leave_pending_work_alone(R):
    rng = np.random.default_rng(1)
    x = _bf16(rng.standard_normal((256, 512)))
    want_r, want_w = R.quantize_rows_fp8(x), R.quantize_blocks_fp8(x)
    copy = torch.empty((256, 512), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    for encode, want in ((R.quantize_rows_fp8, want_r), (R.quantize_blocks_fp8, want_w)):
        victim = torch.full((256, 512), 1, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        torch.cuda._sleep(SLEEP)
        copy.copy_(victim)
        del victim
        got = encode(x, stream=side)
        side.synchronize()
        torch.cuda.synchronize()
        assert bool((copy == 1).all()) and torch.equal(got.q, want.q)
        assert torch.equal(got.s[:, :256] if got.s.shape[1] >= 256 else got.s, want.s[:, :256] if want.s.shape[1] >= 256 else want.s)
