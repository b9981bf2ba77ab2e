"""Launches of a training step's operators at the ends of their documented ranges, without a GPU: a library that stands in for the
runtime's launch calls records them (tests/launch_probe.cpp).  A launch counts fewer than 2^32 threads along each axis."""
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
P = 4096           # an address that is never read: nothing is launched

RECORD = """
import ctypes, json, sys
probe = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
sys.path.insert(0, sys.argv[2])
from paper_2312_08538_amd import binding as B
L = B.lib()
assert probe.probe_kernels() > 100          # the library's kernels are known to the probe, so its launches go there too
probe.probe_launch.restype = ctypes.c_char_p
out = []
for name, args in json.loads(sys.stdin.read()):
    probe.probe_clear()
    d = B.conef_drop(p=0.25, site=0, seed=1, step=0)
    code = getattr(L, name)(*[ctypes.byref(d) if a == "drop" else a for a in args])
    v = (ctypes.c_uint32 * 6)()
    launches = [(probe.probe_launch(i, v).decode(), *v) for i in range(probe.probe_launches())]
    out.append([code, launches])
probe.probe_names.restype = ctypes.c_char_p
print(json.dumps([out, probe.probe_names().decode().split()]))
"""


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    """record([(call, arguments), ...]): [(code, [(kernel, grid x, y, z, block x, y, z), ...]), ...]; record.names(): all kernels"""
    so = tmp_path_factory.mktemp("probe") / "launch_probe.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", str(so), os.path.join(HERE, "launch_probe.cpp")], check=True)

    def go(calls):
        run = subprocess.run([sys.executable, "-c", RECORD, str(so), os.path.dirname(HERE)], input=json.dumps(calls), check=True,
                             capture_output=True, text=True)
        return json.loads(run.stdout)

    def calls_only(calls):
        return go(calls)[0]

    calls_only.names = lambda: go([])[1]
    return calls_only


def groups(launch):
    _, gx, gy, gz, bx, by, bz = launch
    for g, b in ((gx, bx), (gy, by), (gz, bz)):
        assert 0 < g * b < 1 << 32, launch
    return gx * gy * gz


def launches_of(record, call, kernel):
    (code, seen), = record([call])
    assert code == 0
    sizes = [groups(launch) for launch in seen]
    found = [n for n, launch in zip(sizes, seen) if kernel in launch[0]]
    assert found, seen
    return found


@pytest.mark.parametrize("cols", [1, 64, 1 << 20, (1 << 27) - 32, 1 << 27, (1 << 27) + 5, (1 << 31) - 1])
def test_sums_over_rows_of_any_width(record, cols):
    n, = launches_of(record, ("conef_norm_backward", [None, 1, cols, 0, P, cols, P, cols, P, P, P, 0, 0, P, cols, 0, 0, P, P, P, 0]),
                     "k_norm_columns")
    assert n * 64 >= 2 * cols


@pytest.mark.parametrize("m", [1, 16, 17, 33, 64])
@pytest.mark.parametrize("n", [50304, (1 << 26) + 8, (1 << 28) - 16, 1 << 28, (1 << 28) + 24, (1 << 30) - 1])
@pytest.mark.parametrize("k", [24, 96])
def test_products_of_few_rows_and_any_width(record, m, n, k):
    call = ("conef_mx_product", [P, P, P, P, m, n, k, 1.0, 0.0, P, n, 1, 0, 0])
    if max(m * -(-n // 8), n * -(-k // 8)) >= 1 << 32:                              # beyond the documented range
        assert record([call]) == [[-1, []]]
        return
    launches_of(record, call, "k_mx_")


@pytest.mark.parametrize("rows,cols", [(1, 8), (1021, 1001), ((1 << 26) - 1, 512), ((1 << 31) - 1, 9), ((1 << 31) - 2, 16), (1 << 17, (1 << 18) - 8),
                                       (2, (1 << 31) - 1)])
def test_dropout_of_every_size(record, rows, cols):
    octets = rows * -(-cols // 8)
    for call in (("conef_dropout_forward", ["drop", rows, cols, 1, P, cols, P, cols, P, cols, 0]),
                 ("conef_dropout_backward", ["drop", rows, cols, 1, P, cols, P, cols, 0])):
        n, = launches_of(record, call, "k_dropout")
        assert n * 256 >= octets


MX_SIDES = [(16, 768), (8192, 8192), ((1 << 30) - 1, 1), ((1 << 30) - 64, 32), ((1 << 30) - 128, 8), (1, (1 << 30) - 1), (8, (1 << 30) - 127),
            ((1 << 27) + 3, 200)]


@pytest.mark.parametrize("rows,cols", MX_SIDES)
def test_quantisation_of_every_size(record, rows, cols):
    """A workgroup takes 64 rows of 128 columns, or 128 of 64 if it quantises by columns too."""
    for by_rows, by_cols in ((P, 0), (0, P), (P, P)):
        for rounding in (0, 1):
            n, = launches_of(record, ("conef_mx_quantise", [P, cols, rows, cols, 1, rounding, 1, 0, 0, by_rows, by_rows, by_cols, by_cols, 0]),
                             "k_mx_quantise")
            padded = (-(-rows // 128) * 2 * -(-cols // 128)) if by_cols else -(-rows // 64) * -(-cols // 128)
            assert n >= padded


@pytest.mark.parametrize("rows,cols", MX_SIDES)
def test_values_of_every_size(record, rows, cols):
    """A wave takes 16 rows of 128 columns."""
    for dtype in (0, 1):
        n, = launches_of(record, ("conef_mx_dequantise", [P, P, rows, cols, P, cols, dtype, 0]), "k_mx_dequantise")
        assert n * 4 >= -(-rows // 16) * -(-cols // 128)


def test_every_kernel_is_reached(record, tmp_path):
    """Calls of every kind on sizes on both sides of every rule; what they launch are all the kernels that there are."""
    calls = []
    for dtype in (0, 1):
        calls.append(("conef_dropout_backward", ["drop", 4, 8, dtype, P, 8, P, 8, 0]))
        for cols in (8, 100, 200, 400, 800, 1500, 2500, 3500, 4500, 5500, 6500, 7500, 10000, 15000, 20000):
            norm = [1e-5, 2000, cols, dtype, P, cols]
            calls += [("conef_norm_forward", [None, *norm, 0, 0, P, P, 0, 0, 2 * P, cols, 0, 0, 0]),
                      ("conef_norm_forward", ["drop", *norm, P, cols, P, P, P, cols, 2 * P, cols, 0, 0, 0]),
                      ("conef_norm_backward", [None, 2000, cols, dtype, P, cols, P, cols, P, P, P, 0, 0, 2 * P, cols, 0, 0, P, P, P, 0])]
        for rounding in (0, 1):
            for rows in (100, 16384):
                for q, qt in ((P, 0), (0, P), (P, P)):
                    calls.append(("conef_mx_quantise", [P, 8192, rows, 8192, dtype, rounding, 1, 0, 0, q, q, qt, qt, 0]))
        for rows in (100, 16384):
            calls.append(("conef_mx_dequantise", [P, P, rows, 8192, P, 8192, dtype, 0]))
        for beta in (0.0, 1.0):
            # rows of few, of 32, of 64, on four and eight waves; tiny whole and in parts; small, wide, large, streamed
            for m, n, k in ((1, 8192, 128), (1, 50304, 2048), (1, 8192, 2048), (1, 2048, 8192), (32, 8192, 128), (32, 8192, 2048), (32, 2048, 8192),
                            (64, 8192, 128), (64, 2048, 2048), (64, 2048, 8192), (512, 512, 512), (256, 256, 8192), (4096, 4096, 512), (8192, 8192, 512),
                            (4096, 4096, 2048), (4096, 8192, 2048), (4096, 4096, 8192), (8192, 2048, 8192), (8160, 8192, 8192), (8192, 8192, 2048),
                            (8192, 16392, 2048), (16384, 16384, 2048)):
                for c in (P, P + 4):
                    calls.append(("conef_mx_product", [P, P, P, P, m, n, k, 1.0, beta, c, n, dtype, P, 0]))
    reached = set()
    for code, seen in record(calls):
        assert code == 0
        for launch in seen:
            groups(launch)
            reached.add(launch[0])
    there = {n for n in record.names() if any(k in n for k in ("k_dropout", "k_norm_", "k_mx_"))}
    assert reached == there, sorted(there - reached)
