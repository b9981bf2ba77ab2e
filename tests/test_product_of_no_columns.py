"""Products of packed operands with sides of zero, without a GPU: what they need is nothing, and asking for it or calling them does not end the process.  Each case runs in a
process of its own, so that one that ends is named."""
import subprocess
import sys

import pytest

SIZES = """
import sys
from paper_2312_08538_amd import binding as B
name, m, n, k = sys.argv[1], *map(int, sys.argv[2:5])
assert getattr(B, f"conef_{name}_product_workspace")(m, n, k) == 0
form = (0,) if name == "q8" else ()
a, s, b, t, c = (4096 * i for i in range(1, 6))          # never read
if 0 in (m, n):
    for room in (0, 4096):
        assert getattr(B.lib(), f"conef_{name}_product")(a, s, *form, b, t, m, n, k, 1.0, 0.0, c, max(n, 1), 0, room, 0) == B.OK
print("done")
"""

# the binding asks for the size wherever a workspace is passed: tensors without memory, and the library's own size call behind a product that does nothing
BINDING = """
import ctypes, sys
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
from paper_2312_08538_amd import binding as B
name, m, n, k = sys.argv[1], *map(int, sys.argv[2:5])
calls = []
nothing = ctypes.CFUNCTYPE(ctypes.c_int)(lambda: calls.append(1) or B.OK)

@ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_size_t, ctypes.POINTER(ctypes.c_int))
def device_of(stream, device):
    device[0] = 0
    return 0

at = lambda f: ctypes.cast(f, ctypes.c_void_p).value
size = at(getattr(B.lib(), f"conef_{name}_product_workspace"))
face = B.face()
face.connect(B.conef_drop, B.ConefError, (*(size if name == "mx" and i == 7 else at(nothing) for i in range(9)), at(device_of)))
face.connect_8bit(tuple(size if name == "q8" and i == 2 else at(nothing) for i in range(10)))
sizes = getattr(B, f"conef_{name}_sizes")
with FakeTensorMode():
    pack = lambda r, c: tuple(torch.empty(sizes(r, c)[key], dtype=torch.uint8, device="cuda:0") for key in ("code_bytes", "scale_bytes"))
    form = (0,) if name == "q8" else ()
    getattr(B, f"conef_{name}_product")(pack(m, k), *form, pack(n, k), k, 1.0, 0.0, torch.empty(m, n, device="cuda:0"),
                                        torch.empty(256, dtype=torch.uint8, device="cuda:0"), 0)
assert calls == [1]
print("done")
"""

SHAPES = [(17, 0, 4096), (65, 0, 8192), (100, 0, 8192), (100, 0, 1 << 27), (1 << 20, 0, 8192), (0, 100, 8192), (0, 0, 8192), (100, 100, 0)]


def run(code, *args):
    done = subprocess.run([sys.executable, "-c", code, *map(str, args)], capture_output=True, text=True)
    assert done.returncode == 0 and done.stdout.strip() == "done", (done.returncode, done.stderr[-500:])


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("name", ["q8", "mx"])
def test_a_product_of_nothing_needs_nothing(name, m, n, k):
    run(SIZES, name, m, n, k)


@pytest.mark.parametrize("name", ["q8", "mx"])
def test_the_binding_takes_a_product_of_no_columns(name):
    run(BINDING, name, 100, 0, 8192)
