"""How many rows of a packed norm a workgroup takes goes by how far they fill the card's turns; a row's results do not: on both sides of that rule, bit for bit those of calls on few
rows."""
import pytest

from test_gpu_step8 import env, test_norm_of_many_rows_is_that_of_few as rows_alone  # noqa: F401  (env: the fixture)

pytestmark = pytest.mark.gpu


# one whole turn, a little more, the side of one and a half that takes few rows a workgroup and the one that takes many, two turns
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("rows,cols", [(16384, 1100), (19000, 1100), (20000, 1100), (32000, 1100), (8192, 2100), (12000, 2100), (13000, 2100), (16384, 2100), (4096, 4200), (5000, 4200),
                                       (7000, 4200), (4096, 6200), (6200, 6200), (8192, 300), (13000, 60), (9000, 700)])
def test_rows_in_turns_of_any_filling(env, rows, cols, bf16, fused):  # noqa: F811
    rows_alone(env, rows, cols, bf16, fused)
