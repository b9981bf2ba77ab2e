"""Few tokens under a weight so wide that it is worked on in pieces: against 64 bits, and nothing behind the workspace is written."""
import pytest

import step8_ref as R
from test_gpu_layers import env  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu
U, U16 = R.U32, R.U16


@pytest.mark.parametrize("tokens,vocab,width,bf16", [(3, 40000, 16504, True), (70, 40000, 16501, True), (1, 21000, 16504, False), (33, 21001, 16501, False)])
def test_pieces_of_a_wide_weight(env, tokens, vocab, width, bf16):  # noqa: F811
    torch, B = env
    dt, st = torch.bfloat16 if bf16 else torch.float32, B.Model.stream_handle()
    g = torch.Generator(device="cuda:0").manual_seed(tokens)
    x = torch.randn(tokens, width, device="cuda:0", generator=g).to(dt)
    w = (torch.randn(vocab, width, device="cuda:0", generator=g) * (2 / width ** 0.5)).to(dt)
    t = torch.randint(0, vocab, (tokens,), device="cuda:0", generator=g)
    t[0], rows = vocab - 1, torch.arange(tokens, device="cuda:0")
    dloss = torch.rand(tokens, device="cuda:0", generator=g) + 0.5
    n = B.conef_loss_workspace(tokens, vocab, width, dt)
    assert n < w.nbytes
    room = torch.full((n + 4096,), 0xFF, dtype=torch.uint8, device="cuda:0")
    ws = room[:n]
    lse = torch.empty(tokens, device="cuda:0")
    loss, dx, dw = torch.empty_like(lse), torch.empty_like(x), torch.full_like(w, float("nan"))
    B.conef_loss_forward(x, w, t, loss, lse, ws, st)
    ws.fill_(0xFF)
    B.conef_loss_backward(x, w, t, lse, dloss, 0.25, 0.0, dx, dw, ws, st)
    W = w.double()
    logits = torch.mm(x.double(), W.t())
    want = torch.logsumexp(logits, 1)
    # a logit is off by 2^-23 sqrt(width) times the root of its terms' squares (2), and no more than four times that
    e = 4 * 2.0 ** -23 * width ** 0.5 * 2 + 80 * U + 3 * U * want.abs()
    assert bool(((lse.double() - want).abs() <= e).all()) and bool(((loss.double() - (want - logits[rows, t])).abs() <= 2 * e).all())
    d = torch.exp(logits - want[:, None])
    d[rows, t] -= 1
    d *= dloss.double()[:, None]
    for got, exp in ((dx, torch.mm(d, W)), (dw, 0.25 * torch.mm(d.t(), x.double()))):
        far = float((got.double() - exp).norm() / exp.norm())
        # bf16: d's rounding and the result's, 2^-8 each at the most; fp32: a logit's error above, and the sums'
        assert far <= (1.5 * U16 if bf16 else 4 * 2.0 ** -23 * (width ** 0.5 + 8)), far
    assert bool((room[n:] == 0xFF).all())
