"""Products of 8-bit operands at the ends of the scales for which they are documented to be exact in fp32: what an element stands for is a multiple of 2^-133 below 2^128."""
import pytest

import step8_ref as R
from test_gpu_layers import env  # noqa: F401  (the fixture)
from test_gpu_step8 import cut_error, room_of, wide_error

pytestmark = pytest.mark.gpu


def operand(torch, rows, cols, form, byte, low, high, key):
    """(packed pair, values in 64 bits): codes whose exponents' field is from low to high - 1, one in sixteen zero, and one scale byte"""
    g = torch.Generator(device="cuda:0").manual_seed(key)
    r, c, bits = -(-rows // 64) * 64, -(-cols // 128) * 128, R.BITS[form]
    draw = lambda lo, hi: torch.randint(lo, hi, (rows, cols), dtype=torch.uint8, device="cuda:0", generator=g)          # noqa: E731
    some = (draw(low, high) << bits) + draw(0, 1 << bits) + 128 * draw(0, 2)
    some[draw(0, 16) == 0] = 0
    if form == R.E4M3:
        some[(some & 127) == 127] -= 1                   # (no NaN)
    codes = torch.zeros(r, c, dtype=torch.uint8, device="cuda:0")
    codes[:rows, :cols] = some
    scales = torch.zeros(c // 128, r, dtype=torch.uint8, device="cuda:0")
    scales[:, :rows] = byte
    values = torch.tensor(R.table(form), device="cuda:0")[some.long()] * 2.0 ** (byte - 127)
    return (codes.view(r // 16, 16, c // 128, 8, 16).permute(0, 2, 3, 1, 4).reshape(-1).contiguous(), scales.view(-1)), values


# few rows, every size of tile, the long axis in parts
@pytest.mark.parametrize("m,n,k", [(5, 40, 300), (40, 64, 1000), (100, 90, 300), (128, 64, 9000), (2000, 1700, 300), (4096, 2048, 4224), (3500, 3600, 4224)])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("form", [R.E4M3, R.E5M2])
@pytest.mark.parametrize("small", ["a", "b"])
@pytest.mark.parametrize("any_code", [False, True])
def test_scales_at_the_ends_of_their_range(env, m, n, k, bf16, form, small, any_code):  # noqa: F811
    torch, B = env
    if any_code:                 # the bytes of which every finite code fits: last places of 2^-9 and 2^-16, largest codes of 1.75 2^8 and 1.75 2^15
        low = {R.E4M3: (3, 0, 16), R.E5M2: (10, 0, 31)}
        high = {R.E4M3: (246, 0, 16), R.E5M2: (239, 0, 31)}
    else:                        # the smallest: 2^-127 (byte 0), codes whose last place is 2^-6 at least; the largest: codes below 2^8 over a scale of 2^120, 2^15 over 2^113
        low = {R.E4M3: (0, 4, 15), R.E5M2: (0, 11, 30)}
        high = {R.E4M3: (247, 1, 15), R.E5M2: (240, 1, 30)}
    a, A = operand(torch, m, k, form, *(low if small == "a" else high)[form], 1)
    b, W = operand(torch, n, k, R.E4M3, *(high if small == "a" else low)[R.E4M3], 2)
    least, most = (A, W) if small == "a" else (W, A)
    assert float(most.abs().max()) < 2.0 ** 128 and bool((least * 2.0 ** 133 == (least * 2.0 ** 133).round()).all())
    c = torch.full((m, n), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda:0")
    alpha = 2.0 ** -10
    B.conef_q8_product(a, form, b, k, alpha, 0.0, c, room_of(torch, B.conef_q8_product_workspace(m, n, k)), B.Model.stream_handle())
    want = alpha * torch.mm(A, W.t())
    far = alpha * wide_error(torch.mm(A.abs(), W.abs().t()), k) + want.abs() * 2 * R.U32
    if bf16:
        far += alpha * cut_error(A, W, k, torch)
        far += (want.abs() + far) * R.U16
    assert bool(((c.double() - want).abs() <= far).all())
