"""Room that the loss of a vocabulary's logits asks for: of a wide weight it holds a piece, for few tokens as for many.  No kernel is launched."""
import pytest

from paper_2312_08538_amd import binding as B


@pytest.mark.parametrize("dtype,size", [(B.BF16, 2), (B.F32, 4)])
@pytest.mark.parametrize("tokens", [0, 1, 16, 128])
def test_few_tokens_of_a_wide_weight(tokens, dtype, size):
    for vocab, width in ((256000, 8192), (128000, 16000), (1000003, 4099)):
        assert B.conef_loss_workspace(tokens, vocab, width, dtype) < vocab * width * size // 3
    # a weight that is one piece: once, not twice; the gradient of its logits twice, in tokens rounded up to 64; x twice; dx in as many parts as there are workgroups for
    w, d, x = 50304 * 2048 * size, -(-tokens // 64) * 64 * 50304 * size, -(-tokens // 64) * 64 * 2048 * size
    assert B.conef_loss_workspace(tokens, 50304, 2048, dtype) <= w + 2 * d + 2 * x + 3 * 256 * 64 * 64 * 4 + 16 * 256


def test_room_of_few_tokens_is_that_of_a_batch():
    assert max(B.conef_loss_workspace(t, 256000, 8192, B.BF16) for t in (1, 16, 128, 1024, 8192)) < 1 << 30


def test_rooms_that_the_header_states():
    assert B.conef_loss_workspace(65536, 50304, 2048, B.BF16) < 2.25e9
