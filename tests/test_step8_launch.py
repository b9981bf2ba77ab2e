"""Launches of a step in 8 bits at the ends of their documented ranges, without a GPU (as tests/test_layers_launch.py), and what the compiler notes about its kernels."""
import re

import pytest

from test_kernel_metadata import kernels  # noqa: F401  (the fixture)
from test_layers_launch import MX_SIDES, P, groups, launches_of, record  # noqa: F401  (record: the fixture)


@pytest.mark.parametrize("rows,cols", MX_SIDES)
def test_quantisation_of_every_size(record, rows, cols):  # noqa: F811
    """A workgroup takes 64 rows of 128 columns, or 128 of 128 if it quantises by columns too."""
    for by_rows, by_cols in ((P, 0), (0, P), (P, P)):
        n, = launches_of(record, ("conef_q8_quantise", [P, cols, rows, cols, 1, 0, by_rows, by_rows, by_cols, by_cols, 0]), "k_q8_quantise")
        assert n >= -(-rows // (128 if by_cols else 64)) * -(-cols // 128)


@pytest.mark.parametrize("rows,cols", MX_SIDES)
def test_values_of_every_size(record, rows, cols):  # noqa: F811
    for dtype in (0, 1):
        n, = launches_of(record, ("conef_q8_dequantise", [P, P, rows, cols, 0, P, cols, dtype, 0]), "k_q8_dequantise")
        assert n * 4 >= -(-rows // 16) * -(-cols // 128)


@pytest.mark.parametrize("m,n,k", [(1, (1 << 30) - 1, 24), (16, (1 << 28) + 24, 96), (64, (1 << 28) - 16, 24), (65, (1 << 28) - 16, 24), ((1 << 28) - 16, 65, 24), (128, 16, 1 << 27),
                                   ((1 << 17) - 1, 1 << 17, 128), (8, 16, (1 << 30) - 127)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_products_of_every_size(record, m, n, k, dtype):  # noqa: F811
    seen = launches_of(record, ("conef_q8_product", [P, P, 0, P, P, m, n, k, 1.0, 0.0, P, n, dtype, P, 0]), "k_q8_")
    assert max(seen) >= 1


@pytest.mark.parametrize("rows,cols", [(1, 8), (1021, 1001), ((1 << 26) - 1, 512), ((1 << 31) - 1, 9), (1, (1 << 31) - 1), (3, 1 << 27), (1 << 17, (1 << 18) - 8)])
def test_norms_of_every_size(record, rows, cols):  # noqa: F811
    launches_of(record, ("conef_rms_forward", [1e-5, rows, cols, 1, P, cols, P, cols, P, P, cols, 2 * P, cols, 0, 0, 0, 0]), "k_rms_forward")
    launches_of(record, ("conef_rms_backward", [rows, cols, 1, P, cols, P, cols, P, P, 0, 0, P, cols, P, P, 0]), "k_rms_backward")
    if rows < 1 << 30 and cols < 1 << 30 and cols * -(-rows // 8) < 1 << 32:
        launches_of(record, ("conef_rms_forward", [1e-5, rows, cols, 1, P, cols, P, cols, P, P, cols, 0, 0, P, P, 0, 0]), "k_rms_forward")


LOSSES = [(1, 1, 1), (1, (1 << 30) - 1, 24), ((1 << 30) - 1, 1, 8), (1 << 18, (1 << 17) - 8, 40), (64, (1 << 28) - 8, 64), (1, 8, (1 << 30) - 8), (1 << 20, 5000, 4096)]


@pytest.mark.parametrize("tokens,vocab,width", LOSSES)
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("skew", [0, 4])                 # what lies as the kernels take it, and what is packed first
def test_losses_of_every_size(record, tokens, vocab, width, dtype, skew):  # noqa: F811
    calls = [("conef_loss_forward", [tokens, vocab, width, dtype, P, width, P + skew, width, P, P, 2 * P, P, 0]),
             ("conef_loss_backward", [tokens, vocab, width, dtype, P, width, P + skew, width, P, P, P, 1.0, 0.0, 2 * P, width, 3 * P, width, P, 0])]
    for code, seen in record(calls):
        assert code == 0 and seen
        for launch in seen:
            groups(launch)


def test_every_kernel_is_reached(record):  # noqa: F811
    """Calls of every kind on sizes on both sides of every rule; what they launch are all the kernels that there are."""
    calls = []
    for dtype in (0, 1):
        for cols in (8, 100, 200, 400, 800, 1500, 3500, 5500, 7500, 10000, 20000):
            for rows in (200, 2000, 20000):
                for packed in (0, P):
                    norm = [1e-5, rows, cols, dtype, P, cols]
                    calls += [("conef_rms_forward", [*norm, 0, 0, P, 0, 0, 2 * P, cols, packed, packed, 0, 0]),
                              ("conef_rms_forward", [*norm, P, cols, P, P, cols, 2 * P, cols, packed, packed, 0, 0])]
                calls.append(("conef_rms_backward", [rows, cols, dtype, P, cols, P, cols, P, P, 0, 0, 2 * P, cols, P, P, 0]))
        for form in (0, 1):
            for q, qt in ((P, 0), (0, P), (P, P)):
                calls.append(("conef_q8_quantise", [P, 8192, 100, 8192, dtype, form, q, q, qt, qt, 0]))
            for rows in (100, 16384):
                calls.append(("conef_q8_dequantise", [P, P, rows, 8192, form, P, 8192, dtype, 0]))
            for beta in (0.0, 1.0):
                for m, n, k in ((1, 8192, 128), (1, 50304, 2048), (1, 8192, 2048), (1, 2048, 8192), (32, 8192, 128), (32, 8192, 2048), (32, 2048, 8192), (64, 8192, 128),
                                (64, 2048, 2048), (64, 2048, 8192), (512, 512, 512), (256, 256, 8192), (2048, 2048, 512), (4096, 4096, 512), (8192, 8192, 512), (4096, 4096, 2048),
                                (4096, 8192, 2048), (4096, 4096, 8192), (8192, 2048, 8192), (8160, 8192, 8192), (8192, 8192, 2048), (8192, 16392, 2048), (16384, 16384, 2048), (4096, 2304, 512), (4096, 2048, 512), (200000, 128, 512), (4096, 2048, 2048), (4096, 2048, 8192), (4096, 2304, 8192), (32, 4096, 2048)):
                    for c in (P, P + 4):
                        calls.append(("conef_q8_product", [P, P, form, P, P, m, n, k, 1.0, beta, c, n, dtype, P, 0]))
        for tokens, vocab, width in ((16, 50304, 768), (64, 300, 64), (200, 3000, 300), (1000, 5000, 500), (2048, 2048, 2048), (4096, 50304, 2048), (16, 50304, 2048), (4096, 4096, 512), (9000, 9000, 24), (16384, 10000, 4096), (4096, 2304, 512), (30000, 10000, 128)):
            for skew in (0, 4):
                calls += [("conef_loss_forward", [tokens, vocab, width, dtype, P, width, P + skew, width, P, P, 2 * P, P, 0]),
                          ("conef_loss_backward", [tokens, vocab, width, dtype, P, width, P + skew, width, P, P, P, 1.0, 0.5, 2 * P, width, 3 * P, width, P, 0])]
    reached = set()
    for code, seen in record(calls):
        assert code == 0
        for launch in seen:
            groups(launch)
            reached.add(launch[0])
    there = {n for n in record.names() if any(k in n for k in ("k_q8_", "k_rms_", "k_loss_"))}
    assert reached == there, sorted(there - reached)


def test_no_kernel_spills(kernels):  # noqa: F811
    found = {k: v for k, v in kernels.items() if re.match(r"k_(q8|rms|loss)_", k)}
    assert len(found) > 100
    for k, v in found.items():
        assert v["spills"] == 0, (k, v)
