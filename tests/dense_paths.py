"""Calls that between them launch every kernel of the operators around the MoE layer, on a GPU of 256 compute units, in the forms that large calls
take: several tiles per block, one K block and many, odd pitches, streamed outputs, a second launch for the last rows.

Each: the call's arguments, the kernels that it launches in order (the host test replays the choice and checks them), and notes on the form:
tiles: tiles of 256 rows of the first kernel, in each of which more than 256 means that a block takes several."""


def linear(M, N, K, *kernels, out="bf16", bias=False, add=False, pitch=0, in_place=False):
    return dict(op="linear", M=M, N=N, K=K, out=out, bias=bias, add=add or in_place, pitch=pitch, in_place=in_place, kernels=kernels)


def ffn(T, H, I, *kernels, add=False, f32_sums=False, pitch=0):
    return dict(op="ffn", T=T, H=H, I=I, add=add, f32_sums=f32_sums, pitch=pitch, kernels=kernels)


def name(c):
    return "-".join(str(c[k]) for k in (("M", "N", "K", "out") if c["op"] == "linear" else ("T", "H", "I", "f32_sums"))) + ("-in-place" if c.get("in_place") else "")


def _big(gate_up, ragged, streamed):
    return "fp8_big_kernel<%s, %s, %s>" % tuple(str(b).lower() for b in (gate_up, ragged, streamed))


def _tile(gate_up, wide, f32, shape):
    shapes = {"64x64": "1, 4, 2, 4, 2", "128x64": "2, 4, 2, 4, 2", "128x128": "4, 2, 2, 2, 4" if wide else "2, 4, 2, 2, 4", "128x128 once": "2, 4, 4, 4, 2",
              "64x256": "2, 2, 4, 3, 4", "128x256": "4, 2, 4, 3, 4" if wide else "2, 4, 4, 3, 4"}
    return "fp8_tile_kernel<%s, %s, %s, %s>" % (*(str(b).lower() for b in (gate_up, wide, f32)), shapes[shape])


def _few(rows, kind):
    return "fp8_few_kernel<%d, (realb::FewKind)%d, 8>" % (rows, ("linear", "linear f32", "gate/up", "down").index(kind))


LINEAR_BIG = [
    linear(32700, 4090, 128, _big(False, False, True), bias=True, add=True, pitch=3),      # one K block: transfers two tiles ahead
    linear(32700, 4096, 640, _big(False, False, True)),
    linear(32700, 4095, 144, _big(False, True, True), bias=True, add=True, pitch=2),
    linear(32700, 4096, 16, _big(False, True, True), pitch=8),
    linear(19000, 4000, 384, _big(False, False, False), add=True),
    linear(19000, 4001, 272, _big(False, True, False), bias=True, pitch=7),
    linear(23700, 2700, 256, _big(False, False, False), bias=True),                        # a panel of 8 columns and 3 behind it
    linear(16300, 4096, 8192, _big(False, False, False)),                                  # 64 K blocks, the most that a tile's scales have room for
    linear(33001, 4096, 128, _big(False, False, True), _tile(False, False, False, "64x64"), in_place=True),
    linear(33001, 4090, 400, _big(False, True, True), _tile(False, False, False, "64x64"), bias=True, add=True, pitch=5),
]
LINEAR_SMALL = [linear(M, N, K, _tile(False, out == "f32", out == "f32", shape), out=out, bias=N % 2 == 0, add=K % 3 == 0, pitch=N % 4)
                for shape, M, N in (("64x64", 65, 200), ("64x64", 300, 1999), ("128x64", 1000, 2001), ("128x128 once", 2000, 1410), ("128x128", 4000, 2047))
                for K in (16, 384, 1168) for out in ("bf16", "f32")]
LINEAR_DEEP = [                                          # more than 64 K blocks: the weights' scales are fetched again
    linear(100, 300, 8208, _tile(False, False, False, "64x64"), bias=True),
    linear(1000, 2001, 16400, _tile(False, False, False, "128x64")),
    linear(2000, 1410, 8192 + 128, _tile(False, False, False, "128x128 once"), add=True),
    linear(16300, 2048, 8208, _tile(False, False, False, "128x128")),
    linear(300, 1999, 16400, _tile(False, True, True, "64x64"), out="f32"),
    linear(24, 200, 16400, _few(2, "linear"), bias=True),
]
LINEAR_FEW = [linear(M, N, K, _few(-(-M // 16), "linear f32" if out == "f32" else "linear"), out=out, bias=M % 2 == 0, add=M % 3 == 0, pitch=M % 2)
              for M in (1, 9, 16, 17, 40, 48, 64) for N, K in ((57, 16), (320, 1168), (64, 8208)) for out in ("bf16", "f32")]

FFN = [
    ffn(16300, 128, 1024, _big(True, False, False), _tile(False, False, False, "128x64"), add=True),
    ffn(16300, 1024, 1024, _big(True, False, False), _big(False, False, False), pitch=3),
    ffn(19400, 256, 1280, _big(True, False, False), _tile(False, False, False, "128x128")),                                    # a panel of 8 columns and 2 behind it
    ffn(17000, 128, 1024, _big(True, False, False), _tile(True, False, False, "64x256"), _tile(False, False, False, "128x128 once"), add=True),
    ffn(6000, 256, 1408, _big(True, False, False), _tile(True, False, False, "64x256"), _tile(False, False, False, "128x64")),
    ffn(8488, 384, 1408, _big(True, False, False), _tile(True, False, False, "128x256"), _tile(False, False, False, "128x128 once")),
    ffn(3001, 256, 768, _tile(True, False, False, "128x256"), _tile(False, False, False, "64x64"), add=True),
    ffn(3001, 1152, 768, _tile(True, False, False, "128x256"), _tile(False, False, False, "128x128 once"), pitch=1),
    ffn(100, 8320, 256, _tile(True, False, False, "64x256"), _tile(False, False, False, "128x64"), add=True),                   # 65 K blocks
    ffn(3001, 8320, 768, _tile(True, False, False, "128x256"), _big(False, False, False)),
    ffn(100, 8320, 256, _tile(True, True, False, "64x256"), _tile(False, True, False, "128x64"), f32_sums=True),
    ffn(130, 640, 1152, _tile(True, True, False, "64x256"), _tile(False, True, False, "64x64"), f32_sums=True),
    ffn(3001, 8320, 768, _tile(True, True, False, "128x256"), _tile(False, True, False, "128x128"), f32_sums=True, add=True),
    ffn(1000, 2048, 384, _tile(True, True, False, "64x256"), _tile(False, True, False, "128x64"), f32_sums=True, pitch=3),
    ffn(2000, 1408, 384, _tile(True, True, False, "64x256"), _tile(False, True, False, "128x128 once"), f32_sums=True),
    *(ffn(T, H, I, _few(-(-T // 16), "gate/up"), _few(-(-T // 16), "down"), add=T % 2 == 0, pitch=T % 3)
      for T in (5, 31, 40, 64) for H, I in ((256, 384), (8320, 128), (128, 2048))),
]
ALL = LINEAR_BIG + LINEAR_SMALL + LINEAR_DEEP + LINEAR_FEW + FFN
