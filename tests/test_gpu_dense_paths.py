"""Every kernel of the E4M3 products, in the forms that large calls take (dense_paths.py; test_dense_paths_host.py checks that they are launched): every
element of every output against the formula in 64 bits, worked out on the GPU from the operands' codes and scales.

Bounds: (blocks + 16) 2^-24 S for FP32 sums (F32 outputs, up to 64 rows, feed-forward blocks that ask for them) with S = sum |x||w|.  The 8-bit
instruction cuts off of any 8 products what lies 13 bits below the largest: at the worst 7 * 2^-13 S, which among hundreds of millions of elements some
come near (1.2 * 2^-13 S, all products of a short row cut the same way); in the norm it disappears, so products are 2e-3 off there.  Plus half a unit of the
output; h of the feed-forward block within half a code step and what such sums move it.
Up to 64 rows the feed-forward's output is compared end to end: element-wise as there, and 2e-3 in the norm where there are 8192 codes of h or more (one of
them on the other side of a rounding boundary, in at most 1e-4 of the cases, then moves the norm by some 0.06 / sqrt(8192) = 7e-4, in quadrature to 1.66e-3)."""
import numpy as np
import pytest
import torch

import dense_paths as D
from oracle import dense
from gpu_helpers import rel_fro, row_report, say
from test_gpu_dense import _np

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    import paper_2604_19503_amd as R
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    R.load_library()
    return R


class _Maker:
    """Operands from the framework's encoders (bit-exact in their own tests) and their values in 64 bits."""

    def __init__(self, R, seed):
        self.R, self.gen = R, torch.Generator(device="cuda")
        self.gen.manual_seed(seed)

    def randn(self, *shape, std=1.0):
        return torch.randn(shape, generator=self.gen, device="cuda").mul_(std)

    def rows(self, M, K):
        """One channel in 64 twenty times as large, a row and a block of zeros; odd M: rows in the middle of wider ones that hold NaN."""
        x = self.randn(M, K)
        x[:, ::64] *= 20.0
        if M > 2:
            x[1] = 0.0
            x[2, :128] = 0.0
        q = torch.full((M, K + 16 * (M % 2)), 0x7F, dtype=torch.uint8, device="cuda")[:, :K]
        s = torch.full((-(-K // 128), M + 3), float("nan"), device="cuda")
        got = self.R.quantize_rows_fp8(x.to(torch.bfloat16), out=self.R.Fp8Rows(q, s))
        return got, row_values(got.q, got.s)

    def weights(self, N, K, std=0.02):
        w = self.R.quantize_blocks_fp8(self.randn(N, K, std=std).to(torch.bfloat16))
        v = w.q.view(torch.float8_e4m3fn).double()
        return w, v * w.s.double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]

    def out(self, M, N, pitch, dtype):
        """[M, N] in the middle of nines: the rows' ends, a row behind the last one."""
        room = torch.full((M + 1, N + pitch), 9.0, dtype=dtype, device="cuda")
        return room, room[:M, :N]


def row_values(q, s):
    rows, K = q.shape
    return q.contiguous().view(torch.float8_e4m3fn).double() * s[:, :rows].double().t().repeat_interleave(128, 1)[:, :K]


def _sums(x, w):
    return x @ w.t().contiguous(), x.abs() @ w.abs().t().contiguous()


def _unit(K, fp32):
    return 2.0 ** -24 * (-(-K // 128) + 16) if fp32 else 7 * 2.0 ** -13


def _check(got, want, S, K, fp32, f32_out, extra=None):
    """Every element within its bound."""
    bound = _unit(K, fp32) * S + (2.0 ** -23 if f32_out else 1.001 * 2.0 ** -8) * want.abs() + 1e-30
    if extra is not None:
        bound += (_unit(K, True) if fp32 else 2.0 ** -20) * extra
    bad = ~((got.double() - want).abs() <= bound)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[0].tolist())
    assert got.numel() < 1000 or float((got.double() - want).norm() / want.norm()) <= 2e-3


def _untouched(room, y, pitch):
    assert bool((room[y.shape[0]] == 9.0).all()) and (pitch == 0 or bool((room[:, y.shape[1]:] == 9.0).all()))


@pytest.mark.parametrize("c", [c for c in D.ALL if c["op"] == "linear"], ids=D.name)
def test_product(R, c):
    M, N, K, f32 = c["M"], c["N"], c["K"], c["out"] == "f32"
    say("gpu-paths", f"linear {D.name(c)}: {', '.join(c['kernels'])}")
    make = _Maker(R, M + N + K)
    (x, xv), (w, wv) = make.rows(M, K), make.weights(N, K)
    dt = torch.float32 if f32 else torch.bfloat16
    room, y = make.out(M, N, c["pitch"], dt)
    b = make.randn(N).to(torch.bfloat16) if c["bias"] else None
    a = make.randn(M, N).to(dt) if c["add"] else None
    if c["in_place"]:
        y.copy_(a)
    R.linear_fp8(R.make_linear_io(x, w, y, bias=b, add=y if c["in_place"] else a))
    torch.cuda.synchronize()
    _untouched(room, y, c["pitch"])
    want, S = _sums(xv, wv)
    extra = torch.zeros_like(S)
    for t in (b, a):
        if t is not None:
            want += t.double()
            extra += t.double().abs()
    _check(y, want, S, K, f32 or M <= 64, f32, extra)


@pytest.mark.parametrize("c", D.FFN, ids=D.name)
def test_feed_forward(R, c):
    T, H, I = c["T"], c["H"], c["I"]
    say("gpu-paths", f"ffn {D.name(c)}: {', '.join(c['kernels'])}")
    make = _Maker(R, T + H + I)
    (x, xv), (w13, v13), (w2, v2) = make.rows(T, H), make.weights(2 * I, H), make.weights(H, I)
    room, y = make.out(T, H, c["pitch"], torch.bfloat16)
    a = make.randn(T, H).to(torch.bfloat16) if c["add"] else None
    need = R.load_library().realb_gated_ffn_workspace_bytes(T, I)
    work = torch.zeros(need + 16, dtype=torch.uint8, device="cuda")
    work[need:] = 0x5A
    R.gated_ffn_fp8(R.make_ffn_io(x, w13, w2, y, add=a, workspace=work[:need], f32_sums=c["f32_sums"]))
    torch.cuda.synchronize()
    assert bool((work[need:] == 0x5A).all())
    _untouched(room, y, c["pitch"])
    if T <= 64:
        want = dense.gated_ffn(xv.cpu().numpy(), v13.cpu().numpy(), v2.cpu().numpy(), None if a is None else _np(a))[2]
        got = _np(y)
        assert row_report(got, want)[1] == 0
        assert T * I < 8192 or rel_fro(got, want) <= 2e-3
        return
    fp32 = c["f32_sums"]
    q = work[: T * I].view(T, I)
    s = work[T * I: T * I + (I // 128) * (-(-T // 4) * 4) * 4].view(torch.float32).view(I // 128, -1)
    hv = row_values(q, s)
    gu, S = _sums(xv, v13)
    g, u, Sg, Su = gu[:, :I], gu[:, I:], S[:, :I], S[:, I:]
    sig = torch.sigmoid(g)
    h = g * sig * u
    moved = _unit(H, fp32) * (Su * (g * sig).abs() + Sg * 1.1 * u.abs())
    step = torch.maximum(2.0 ** -4 * h.abs(), 2.0 ** -10 * s[:, :T].double().t().repeat_interleave(128, 1))
    bad = ~((hv - h).abs() <= 1.07 * moved + 1.001 * step + 1e-5 * h.abs() + 1e-30)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[0].tolist())
    top, scales = h.abs().unflatten(1, (-1, 128)).amax(2), s[:, :T].double().t() * 448.0
    spread = moved.unflatten(1, (-1, 128)).amax(2)
    assert bool(((scales - top).abs() <= spread + 1e-5 * top + 2.0 ** -99).all())
    staged, S2 = _sums(hv, v2)
    extra = None
    if a is not None:
        staged += a.double()
        extra = a.double().abs()
    _check(y, staged, S2, I, fp32, False, extra)


# ---------------------------------------------------------------------------------------------- what a row may and may not depend on
def _same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("M,N,K,out", [(19000, 4000, 256, "bf16"), (32700, 4095, 144, "bf16"), (4000, 2047, 256, "f32")])
def test_a_row_of_nan_leaves_other_rows_of_a_large_product_alone(R, M, N, K, out):
    make = _Maker(R, M)
    (x, _), (w, _) = make.rows(M, K), make.weights(N, K)
    outs = []
    for bad in (False, True):
        if bad:
            x.q[M // 2, 100] = 0x7F
            x.s[1, 3] = float("inf")
        y = torch.empty((M, N), dtype=torch.bfloat16 if out == "bf16" else torch.float32, device="cuda")
        R.linear_fp8(R.make_linear_io(x, w, y))
        torch.cuda.synchronize()
        outs.append(y)
    rest = torch.ones(M, dtype=torch.bool, device="cuda")
    rest[[M // 2, 3]] = False
    assert _same_bits(outs[0][rest], outs[1][rest])
    assert bool(torch.isnan(outs[1][M // 2].float()).all()) and not bool(torch.isfinite(outs[1][3].float()).any())


@pytest.mark.parametrize("T,H,I,f32_sums", [(40, 256, 384, False), (300, 256, 384, False), (300, 256, 384, True), (3001, 256, 768, False), (16300, 128, 1024, False)])
def test_a_row_of_nan_leaves_other_rows_of_the_feed_forward_alone(R, T, H, I, f32_sums):
    """The maximum of a block of h passes NaN by, so that it rests on the codes to carry it."""
    make = _Maker(R, T)
    (x, _), (w13, _), (w2, _) = make.rows(T, H), make.weights(2 * I, H), make.weights(H, I)
    outs = []
    for bad in (False, True):
        if bad:
            x.q[T // 2, 100] = 0x7F
            x.s[0, 3] = float("inf")
        y = torch.empty((T, H), dtype=torch.bfloat16, device="cuda")
        R.gated_ffn_fp8(R.make_ffn_io(x, w13, w2, y, f32_sums=f32_sums))
        torch.cuda.synchronize()
        outs.append(y)
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[[T // 2, 3]] = False
    assert _same_bits(outs[0][rest], outs[1][rest])
    assert bool(torch.isnan(outs[1][T // 2].float()).all()) and not bool(torch.isfinite(outs[1][3].float()).any())


@pytest.mark.parametrize("M,N,K", [(32700, 4096, 640), (19000, 4001, 272), (33001, 4090, 400)])
def test_a_rows_bits_do_not_depend_on_the_tiles_it_is_in(R, M, N, K):
    """Rows of a large product, and the same rows in products of 65 to 2000 rows."""
    make = _Maker(R, M)
    (x, _), (w, _) = make.rows(M, K), make.weights(N, K)
    y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    R.linear_fp8(R.make_linear_io(x, w, y))
    for first, rows in ((0, 65), (255, 300), (M - 2000, 2000), (M // 2, 1000)):
        part = torch.empty((rows, N), dtype=torch.bfloat16, device="cuda")
        R.linear_fp8(R.make_linear_io(R.Fp8Rows(x.q[first: first + rows].contiguous(), x.s[:, first: first + rows].contiguous()), w, part))
        torch.cuda.synchronize()
        assert _same_bits(part, y[first: first + rows]), (first, rows)


# ---------------------------------------------------------------------------------------------- the instruction's cut
def test_what_the_8_bit_instruction_cuts_off(R):
    """Two products of +-L cancel, the one among 8 consecutive products with a small one s of either sign, the other 64 columns further on: what is left of
    s.  FP32 sums leave s, whatever its size (L + s is exact up to 2^-23 L).  The instruction leaves s within 2^-13 L, and nothing of it from 2^-15 L down:
    the cut of the contract is there, and no larger than it says."""
    M, N, K = 70, 64, 128
    L = 2.0 ** 14
    for out in ("bf16", "f32"):
        for j in range(0, 21):
            for sign in (1.0, -1.0):
                xc, wc = torch.zeros((M, K), device="cuda"), torch.zeros((N, K), device="cuda")
                xc[:, 1], wc[:, 1] = 2.0 ** 7, 2.0 ** 7                     # L
                xc[:, 65], wc[:, 65] = 2.0 ** 7, -(2.0 ** 7)                # -L
                e = 14 - j                                                  # s = 2^e, out of codes between 2^-9 and 2^8
                hi = max(min(e, 7), -6)
                xc[:, 3], wc[:, 3] = 2.0 ** hi, sign * 2.0 ** (e - hi)
                x = R.Fp8Rows(xc.to(torch.float8_e4m3fn).view(torch.uint8), torch.ones((1, M), device="cuda"))
                w = R.Fp8Weight(wc.to(torch.float8_e4m3fn).view(torch.uint8), torch.ones((1, 1), device="cuda"))
                y = torch.empty((M, N), dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
                R.linear_fp8(R.make_linear_io(x, w, y))
                torch.cuda.synchronize()
                s = sign * 2.0 ** e
                if out == "f32":
                    assert bool((y == s).all()), (j, sign, float(y[0, 0]))
                else:
                    assert bool(((y.float() - s).abs() <= 2.0 ** -13 * L).all()), (j, sign, float(y[0, 0]))
                    assert j < 15 or sign < 0 or bool((y == 0.0).all()), (j, float(y[0, 0]))
