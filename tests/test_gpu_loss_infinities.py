"""lse and loss of rows with infinite logits are the limits that the definition has: log(sum exp l) of a row with plus infinity is that, minus infinity counts for nothing, and only
NaN, or infinity less infinity, is NaN."""
import pytest

from test_gpu_layers import env  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


# rows on 16 bytes and not, every size of tile, several tiles to a row
@pytest.mark.parametrize("tokens,vocab,width", [(3, 5, 8), (5, 3000, 40), (70, 300, 65), (600, 1300, 96), (600, 1301, 33), (3000, 3100, 72), (8500, 9000, 24)])
@pytest.mark.parametrize("bf16", [False, True])
def test_limits(env, tokens, vocab, width, bf16):  # noqa: F811
    torch, B = env
    dt, st, inf = torch.bfloat16 if bf16 else torch.float32, B.Model.stream_handle(), float("inf")
    g = torch.Generator(device="cuda:0").manual_seed(tokens + vocab)
    x = torch.randn(tokens, width, device="cuda:0", generator=g).to(dt)
    w = (torch.randn(vocab, width, device="cuda:0", generator=g) / width ** 0.5).to(dt)
    word, rows = vocab // 2, torch.arange(tokens, device="cuda:0")
    t = torch.randint(0, vocab, (tokens,), device="cuda:0", generator=g)
    t[0], t[1] = word, 0
    ws = torch.full((B.conef_loss_workspace(tokens, vocab, width, dt),), 0xFF, dtype=torch.uint8, device="cuda:0")
    loss, lse = torch.empty(tokens, device="cuda:0"), torch.empty(tokens, device="cuda:0")

    def check(sign, every):
        """One word, or every word, of infinite logits: of a token's row the sign"""
        X, W = x.clone(), w.clone()
        X[:, 0] = sign.to(dt)
        W[:, 0] = inf if every else 0.0
        W[word, 0] = inf
        B.conef_loss_forward(X, W, t, loss, lse, ws, st)
        logits = torch.mm(x.double()[:, 1:], w.double()[:, 1:].t())
        endless = sign.double() * inf                                    # (0 times infinity: NaN)
        logits[:, :] = endless[:, None] if every else logits
        logits[:, word] = endless
        want = torch.logsumexp(logits, 1)
        wanted = want - logits[rows, t]
        for got, exp in ((lse, want), (loss, wanted)):
            assert torch.equal(got.isnan(), exp.isnan()) and torch.equal(got.isposinf(), exp.isposinf()) and torch.equal(got.isneginf(), exp.isneginf())
            there = exp.isfinite()
            # logits of order 1, whose sums' errors are far below this
            assert bool(((got.double() - exp).abs()[there] <= 1e-4 * (1 + exp.abs()[there])).all())

    mixed = torch.randint(-1, 2, (tokens,), device="cuda:0", generator=g)
    mixed[:3] = torch.tensor([1, 1, -1], device="cuda:0")
    for every in (False, True):
        check(mixed, every)
        check(torch.ones_like(mixed), every)
        check(-torch.ones_like(mixed), every)
