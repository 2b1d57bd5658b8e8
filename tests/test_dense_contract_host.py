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


# ---- streams: the binding on CPU tensors, with stand-ins for streams, their memory pools and the library
class _Stream:
    def __init__(self, number):
        self.cuda_stream, self.device_index = number, 0


@pytest.fixture
def pools(monkeypatch):
    """current: the stream whose pool serves an allocation; pool_of: address -> stream; calls: (operator, stream, workspace)."""
    class World:
        current, pool_of, calls, kept = 1, {}, [], []
        needs = R.load_library().realb_gated_ffn_workspace_bytes

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            self.before = World.current
            World.current = World.current if self.stream is None else self.stream.cuda_stream

        def __exit__(self, *_):
            World.current = self.before

    def recorded(make):
        def alloc(*a, **k):
            t = make(*a, **k)
            World.pool_of[t.data_ptr()] = World.current
            World.kept.append(t)
            return t
        return alloc

    class Library:
        realb_gated_ffn_workspace_bytes = staticmethod(World.needs)

        def __getattr__(self, name):
            def call(*a):
                at = a[0]._obj.workspace if name == "realb_gated_ffn_fp8" else None
                stream = a[-1].value if isinstance(a[-1], C.c_void_p) else a[-1]
                World.calls.append((name, stream, at, a))
                return 0
            return call

    monkeypatch.setattr(B, "_LIB", Library())
    monkeypatch.setattr(B, "_same_device", lambda first, *others: 0)
    monkeypatch.setattr(torch.cuda, "stream", On)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: _Stream(World.current))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch, "empty", recorded(torch.empty))
    monkeypatch.setattr(torch, "zeros", recorded(torch.zeros))
    return World


def _u8(*s):
    return torch.ones(s, dtype=torch.uint8)


def _f32(*s):
    return torch.ones(s, dtype=torch.float32)


def _ffn_args(T=100, H=128, I=128):
    return (R.Fp8Rows(_u8(T, H), _f32(1, T)), R.Fp8Weight(_u8(2 * I, H), _f32(2, 1)), R.Fp8Weight(_u8(H, I), _f32(1, 1)),
            torch.ones((T, H), dtype=torch.bfloat16))


def test_a_workspace_comes_from_the_pool_of_the_stream_that_uses_it(pools):
    """Memory of another stream's pool may be in use there, and goes back there while the call still runs."""
    io = R.make_ffn_io(*_ffn_args())
    for stream in (None, _Stream(7), _Stream(8), _Stream(7), None):
        R.gated_ffn_fp8(io, stream=stream)
    used = [(stream, at) for _, stream, at, _ in pools.calls]
    assert [s for s, _ in used] == [1, 7, 8, 7, 1]
    assert all(pools.pool_of[at] == s for s, at in used)
    assert used[1] == used[3] and used[0] == used[4]     # one workspace a stream, kept with the argument block
    with torch.cuda.stream(_Stream(9)):                  # made under a stream
        io = R.make_ffn_io(*_ffn_args())
        R.gated_ffn_fp8(io)
    R.gated_ffn_fp8(io)
    assert [(s, pools.pool_of[at]) for _, s, at, _ in pools.calls[-2:]] == [(9, 9), (1, 1)]


def test_a_workspace_of_the_callers_stays_in_use_on_every_stream(pools):
    work = _u8(100 * 128 + 400 + 64 * 128 * 4)
    io = R.make_ffn_io(*_ffn_args(), workspace=work)
    for stream in (None, _Stream(7)):
        R.gated_ffn_fp8(io, stream=stream)
    assert [at for _, _, at, _ in pools.calls] == [work.data_ptr()] * 2


@pytest.mark.parametrize("stream,pool", [(None, 1), (_Stream(7), 7)])
def test_encoders_allocate_where_they_run(pools, stream, pool):
    x = torch.ones((32, 128), dtype=torch.bfloat16)
    rows, w = R.quantize_rows_fp8(x, stream=stream), R.quantize_blocks_fp8(x, stream=stream)
    fp4, nv = R.quantize_rows_fp4(x, stream=stream), R.quantize_rows_nvfp4(x, 1.0, stream=stream)
    for t in (rows.q, rows.s, w.q, w.s, *fp4, *nv, R.amax_bf16(x, stream=stream)):
        assert pools.pool_of[t.data_ptr()] == pool
    assert [s for _, s, _, _ in pools.calls] == [pool] * 5


def _calls_on(stream):
    """Every call of the operators around the layer on `stream`, as functions."""
    bf = lambda *s: torch.ones(s, dtype=torch.bfloat16)  # noqa: E731
    x, w13, w2, out = _ffn_args()
    norm = R.make_norm_io(bf(4, 128), res_out=bf(4, 128))
    linear, ffn = R.make_linear_io(x, w2, bf(100, 128)), R.make_ffn_io(x, w13, w2, out, workspace=_u8(1 << 17))
    return [lambda: R.residual_norm(norm, stream=stream), lambda: R.linear_fp8(linear, stream=stream), lambda: R.gated_ffn_fp8(ffn, stream=stream),
            lambda: R.quantize_rows_fp8(bf(100, 128), out=x, stream=stream), lambda: R.quantize_blocks_fp8(bf(128, 128), out=w2, stream=stream)]


@pytest.mark.parametrize("tensors,current,stream", [(1, 0, None), (1, 1, 0), (1, 0, 1), (0, 1, None), (0, 0, 1)])
def test_tensors_of_another_gpu_than_the_calls_are_refused(pools, monkeypatch, tensors, current, stream):
    """The kernels are launched on the current GPU: another GPU's stream or tensors would be a launch error, or addresses it cannot reach."""
    monkeypatch.setattr(B, "_same_device", lambda first, *others: tensors)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current)

    def on(gpu):
        s = _Stream(5)
        s.device_index = gpu
        return s
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: on(current))
    for call in _calls_on(None if stream is None else on(stream)):
        with pytest.raises(R.RealbError, match="GPU"):
            call()
    assert not pools.calls


def test_calls_on_the_tensors_gpu_go_through(pools):
    for stream in (None, _Stream(7)):
        for call in _calls_on(stream):
            call()
    assert len(pools.calls) == 10
