"""Tokens without a target, whatever their rows of x hold: they add nothing to either gradient, bit for bit what rows of zeros add."""
import pytest

from test_gpu_layers import env  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


# rows on 16 bytes and not, every size of tile, several pieces of the vocabulary, tokens beyond a turned tile's 128
@pytest.mark.parametrize("tokens,vocab,width", [(1, 40, 8), (40, 300, 64), (129, 700, 65), (300, 9000, 24), (1001, 1300, 515), (3000, 3100, 520), (8500, 9000, 64)])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("weighted", [False, True])
def test_rows_without_a_target_reach_no_gradient(env, tokens, vocab, width, bf16, weighted):  # noqa: F811
    torch, B = env
    dt, st = torch.bfloat16 if bf16 else torch.float32, B.Model.stream_handle()
    g = torch.Generator(device="cuda:0").manual_seed(tokens + width)
    x = torch.randn(tokens, width, device="cuda:0", generator=g).to(dt)
    w = (torch.randn(vocab, width, device="cuda:0", generator=g) * (2 / width ** 0.5)).to(dt)
    t = torch.randint(0, vocab, (tokens,), device="cuda:0", generator=g)
    none = torch.rand(tokens, device="cuda:0", generator=g) < 0.3
    none[-1] = True
    t[none] = torch.tensor([-100, -1, vocab, 2 ** 62], device="cuda:0")[torch.randint(0, 4, (int(none.sum()),), device="cuda:0", generator=g)]
    dloss = torch.rand(tokens, device="cuda:0", generator=g) if weighted else None
    lse = torch.empty(tokens, device="cuda:0")
    ws = torch.full((B.conef_loss_workspace(tokens, vocab, width, dt),), 0xFF, dtype=torch.uint8, device="cuda:0")

    def gradients(x):
        B.conef_loss_forward(x, w, t, None, lse, ws, st)
        dx, dw, alone = torch.full_like(x, 7.0), torch.full_like(w, 7.0), torch.full_like(w, 7.0)
        B.conef_loss_backward(x, w, t, lse, dloss, 0.5, 0.0, dx, dw, ws, st)
        B.conef_loss_backward(x, w, t, lse, dloss, 0.5, 0.0, None, alone, ws, st)
        assert torch.equal(alone.isnan(), dw.isnan()) and torch.equal(alone.nan_to_num(), dw.nan_to_num())
        return dx, dw

    want_x, want_w = gradients(torch.where(none[:, None], torch.zeros_like(x), x))
    assert bool(want_w.isfinite().all()) and (bool(want_w.any()) or tokens == 1)
    for value in (1.0, float("nan"), float("inf"), -float("inf")):
        dx, dw = gradients(torch.where(none[:, None], torch.full_like(x, value), x))
        assert torch.equal(dx, want_x) and torch.equal(dw, want_w), value
