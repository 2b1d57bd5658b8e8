"""Which kernels the calls of dense_paths.py launch, from the library itself (in a child process, against stand-ins for the HIP runtime, hip_calls.c:
nothing runs): the GPU tests of those calls then reach every kernel of the operators around the MoE layer, and go on doing so when the
choice of tiles changes."""
import ctypes as C
import json
import os
import re
import subprocess
import sys

import pytest

import dense_paths as D

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2604_19503_amd", "librealb.so")
P = 0x10000000                                           # every tensor: an address that nobody reads
SLOTS = 256                                              # blocks of 256-row tiles at once, a compute unit each


def replay(stub_path):
    """[(return value, [(kernel, blocks)])] of the calls, in their order."""
    stub = C.CDLL(stub_path, mode=C.RTLD_GLOBAL)
    stub.calls_log.restype = C.c_char_p
    lib = C.CDLL(LIB)
    sys.path.insert(0, ROOT)
    from paper_2604_19503_amd import binding as B
    out = []
    for c in D.ALL:
        if c["op"] == "linear":
            io, call = B.LinearIO(), lib.realb_linear_fp8
            io.M, io.N, io.K, io.x_q, io.ld_x, io.x_s, io.ld_xs, io.w_q, io.w_s = c["M"], c["N"], c["K"], P, c["K"], P, c["M"], P, P
            io.out, io.ld_out, io.out_type = P, c["N"] + c["pitch"], int(c["out"] == "f32")
            io.bias = P if c["bias"] else None
            io.add, io.ld_add = (P, io.ld_out) if c["add"] else (None, 0)
        else:
            io, call = B.FfnIO(), lib.realb_gated_ffn_fp8
            io.T, io.H, io.I, io.sums = c["T"], c["H"], c["I"], int(c["f32_sums"])
            io.x_q, io.ld_x, io.x_s, io.ld_xs = P, c["H"], P, c["T"]
            io.w13_q = io.w13_s = io.w2_q = io.w2_s = io.out = io.workspace = P
            io.ld_out, io.workspace_bytes = c["H"] + c["pitch"], 1 << 40
        stub.calls_clear()
        rc = call(C.byref(io), None)
        lines = stub.calls_log().decode().splitlines()
        out.append([rc, [re.match(r"launch (\S+) grid (\d+)", l).groups() for l in lines]])
    return out


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("hip_calls") / "libhip_calls.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", path, os.path.join(ROOT, "tests", "hip_calls.c")], check=True)
    done = subprocess.run([sys.executable, os.path.abspath(__file__), path], capture_output=True, text=True, timeout=120)
    assert done.returncode == 0, done.stderr
    got = json.loads(done.stdout.splitlines()[-1])
    plain = _demangled([k for _, calls in got for k, _ in calls])
    return [(rc, [(plain[k], int(blocks)) for k, blocks in calls]) for rc, calls in got]


def _demangled(names):
    names = sorted(set(names))
    text = subprocess.run(["c++filt"], input="\n".join(names), capture_output=True, text=True, check=True).stdout
    return dict(zip(names, (re.match(r"(?:void )?realb::(?:__device_stub__)?(.*?)\(realb::Fp8Gemm\)", l)[1] for l in text.splitlines())))


def test_every_call_launches_what_its_entry_says(launches):
    for c, (rc, calls) in zip(D.ALL, launches):
        assert rc == 0 and tuple(k for k, _ in calls) == c["kernels"], (D.name(c), rc, calls)


def test_every_kernel_is_launched(launches):
    """All kernels of the products that the library holds."""
    text = subprocess.run(["nm", LIB], capture_output=True, text=True, check=True).stdout
    held = {l.split()[-1] for l in text.splitlines() if "__device_stub__fp8_" in l and "Fp8Gemm" in l}
    assert len(held) > 20
    assert set(_demangled(held).values()) == {k for _, calls in launches for k, _ in calls}


def test_large_tiles_run_several_to_a_block(launches):
    """Every kernel of 256-row tiles, with one K block too where it can have one."""
    several, one_block = set(), set()
    for c, (_, calls) in zip(D.ALL, launches):
        for i, (kernel, blocks) in enumerate(calls):
            if not kernel.startswith("fp8_big"):
                continue
            down = c["op"] == "ffn" and not kernel.startswith("fp8_big_kernel<true")
            rows, cols, K = (c["M"], -(-c["N"] // 256), c["K"]) if c["op"] == "linear" else (c["T"], -(-c["H"] // 256) if down else c["I"] // 128, c["I"] if down else c["H"])
            if -(-rows // 256) * cols > SLOTS and blocks == SLOTS:
                several.add(kernel)
                if K <= 128:
                    one_block.add(kernel)
    kernels = {k for _, calls in launches for k, _ in calls if k.startswith("fp8_big")}
    assert len(kernels) == 5 and several == kernels
    assert {D._big(False, False, True), D._big(False, True, True), D._big(True, False, False)} <= one_block


if __name__ == "__main__":
    print(json.dumps(replay(sys.argv[1])))
