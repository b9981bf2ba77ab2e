"""What the compiler notes about the kernels of a training step's operators: registers that the tiles were sized for, and no spills."""
import re

from test_kernel_metadata import kernels  # noqa: F401  (the fixture)


def of(kernels, name):  # noqa: F811
    found = {k: v for k, v in kernels.items() if re.match(name + r"[<(]|" + name + r"$", k)}
    assert found, f"no kernel {name}"
    return found


def test_no_kernel_spills(kernels):  # noqa: F811
    for name in ("k_dropout", "k_norm_forward", "k_norm_backward", "k_norm_forward_long", "k_norm_backward_long", "k_norm_column_parts",
                 "k_norm_columns", "k_mx_quantise", "k_mx_dequantise", "k_mx_product", "k_mx_stream", "k_mx_rows", "k_mx_join"):
        for k, v in of(kernels, name).items():
            assert v["spills"] == 0, (k, v)


def test_tiles_of_the_product_leave_room_for_the_workgroups_that_a_cu_is_to_hold(kernels):  # noqa: F811
    """512 registers a SIMD: the last template argument is how many waves are to share them."""
    for k, v in of(kernels, "k_mx_product").items():
        waves = int(k.rstrip(">").split(",")[-1])
        assert v["vgprs"] <= 512 // waves, (k, v)


def test_backward_pass_of_the_norm_fits_its_workgroups(kernels):  # noqa: F811
    """Launched as many workgroups to a CU as its registers allow in bf16: four of 256 threads with a wave and an octet a lane to a row, one of 512
    threads and more, else two; fp32 may take a wave less to a SIMD."""
    for k, v in of(kernels, "k_norm_backward").items():
        bf16, lanes, octets = re.findall(r"[\w]+", k.split("<")[1])
        lanes, octets = int(lanes), int(octets)
        groups = 1 if lanes >= 512 else 4 if (lanes, octets) == (64, 1) else 2
        waves = -(-groups * max(lanes, 256) // 256)
        assert v["vgprs"] <= 512 // (waves if bf16 == "true" else max(2, waves - 1)) // 8 * 8, (k, v)
