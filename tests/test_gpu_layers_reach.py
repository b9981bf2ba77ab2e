"""What the sizes of test_gpu_layers do not reach: products and values that are written past the caches, rows of the widest norms
beyond the first of a workgroup, outputs in the place of every input that they may replace, scales of NaN in every size of tile.

Operands of products are random codes and scales, packed and decoded here, on the device and in 64 bits."""
import numpy as np
import pytest

import layers_ref as R
import test_gpu_layers as T
from test_gpu_layers import SEED, STEP, U, Strided, column_vector, env, norm_inputs  # noqa: F401  (env: the fixture)

pytestmark = pytest.mark.gpu


def operand(torch, rows, cols, key):
    """(packed pair, its values in 64 bits [rows, cols], a scale byte's place (row, block) -> index): codes of all kinds, scales of 2^-4 to 2^4."""
    g = torch.Generator(device="cuda:0").manual_seed(key)
    r, c = -(-rows // 64) * 64, -(-cols // 128) * 128
    codes = torch.zeros(r, c, dtype=torch.uint8, device="cuda:0")
    codes[:rows, :cols] = torch.randint(0, 16, (rows, cols), dtype=torch.uint8, device="cuda:0", generator=g)
    scales = torch.zeros(r, c // 32, dtype=torch.uint8, device="cuda:0")
    scales[:rows, :-(-cols // 32)] = torch.randint(123, 132, (rows, -(-cols // 32)), dtype=torch.uint8, device="cuda:0", generator=g)
    grid = torch.tensor(np.concatenate([R.GRID, -R.GRID]), device="cuda:0")
    values = grid[codes[:rows, :cols].long()] * torch.exp2(scales[:rows].double() - 127).repeat_interleave(32, 1)[:, :cols]
    # code byte ((i / 16) P + j / 128) 1024 + (j / 32 % 4) 256 + (i % 16) 16 + (j % 32) / 2
    pairs = codes[:, 0::2] | (codes[:, 1::2] << 4)
    pc = pairs.view(r // 16, 16, c // 128, 4, 16).permute(0, 2, 3, 1, 4).reshape(-1).contiguous()
    # scale byte ((i / 64) P + j / 128) 256 + (j / 32 % 4) 64 + (i % 16) 4 + (i % 64) / 16
    ps = scales.view(r // 64, 4, 16, c // 128, 4).permute(0, 3, 4, 2, 1).reshape(-1).contiguous()
    return (pc, ps), values, lambda i, b: ((i // 64) * (c // 128) + b // 4) * 256 + (b % 4) * 64 + (i % 16) * 4 + (i % 64) // 16


def product_error(torch, A, W, k, want, alpha, old, bf16):
    """as test_gpu_layers.product_tolerance, and a rounding of the factors' products and of the result"""
    far = alpha * torch.mm(A.abs(), W.abs().t()) * ((5 * (-(-k // 128)) + 24) * 2.0 ** -23)
    if old is not None:
        far += 2 * U * old.abs()
    return far + want.abs() * (2 * U + (R.U16 * 1.01 if bf16 else 0))


# small tiles, wide tiles, streams; C above the size from which it is written past the caches, its rows on 64 bytes (the last: on 16)
@pytest.mark.parametrize("m,n,pitch,k,bf16", [(4100, 4221, 4224, 600, True), (4100, 4224, 4224, 600, False), (4100, 4224, 4224, 1600, True),
                                              (4100, 4221, 4224, 1600, False), (8448, 16381, 16384, 1600, True), (8448, 8448, 8448, 1537, False),
                                              (8448, 16392, 16392, 1600, True)])
@pytest.mark.parametrize("beta", [0.0, 1.0])
def test_product_past_the_caches(env, m, n, pitch, k, bf16, beta):  # noqa: F811
    torch, B = env
    (a, A, _), (b, W, _) = operand(torch, m, k, 1), operand(torch, n, k, 2)
    size = 2 if bf16 else 4
    c = torch.full((m, pitch), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda:0")
    assert c.data_ptr() % 64 == 0 and pitch * size % 16 == 0 and m * n * size > 32 << 20
    if beta:
        c.normal_(generator=torch.Generator(device="cuda:0").manual_seed(3))
    gap, old = c[:, n:].clone(), c[:, :n].double() if beta else None
    assert B.conef_mx_product_workspace(m, n, k) == 0
    B.conef_mx_product(a, b, k, 0.125, beta, c[:, :n], None, B.Model.stream_handle())
    want = 0.125 * torch.mm(A, W.t())
    if beta:
        want += old
    assert bool(((c[:, :n].double() - want).abs() <= product_error(torch, A, W, k, want, 0.125, old, bf16)).all())
    assert torch.equal(c[:, n:].isnan(), gap.isnan()) and torch.equal(c[:, n:].nan_to_num(), gap.nan_to_num())


@pytest.mark.parametrize("m,n,k", [(8, 300, 50257), (300, 200, 50257), (1030, 600, 50257)])
def test_product_over_a_vocabulary(env, m, n, k):  # noqa: F811
    torch, B = env
    (a, A, _), (b, W, _) = operand(torch, m, k, 4), operand(torch, n, k, 5)
    c = torch.empty(m, n, device="cuda:0")
    ws = torch.full((B.conef_mx_product_workspace(m, n, k),), 0xFF, dtype=torch.uint8, device="cuda:0")
    B.conef_mx_product(a, b, k, 1.0, 0.0, c, ws, B.Model.stream_handle())
    want = torch.mm(A, W.t())
    assert bool(((c.double() - want).abs() <= product_error(torch, A, W, k, want, 1.0, None, False)).all())


def test_product_of_one_row_and_more_than_2_28_columns(env):  # noqa: F811
    """B is zero but for its last rows and some at a distance: 17 GB of codes."""
    torch, B = env
    n, k = (1 << 28) + 24, 96
    (a, A, _), (tail, W, _) = operand(torch, 1, k, 10), operand(torch, 64, k, 11)
    sizes = B.conef_mx_sizes(n, k)
    b = tuple(torch.zeros(sizes[s], dtype=torch.uint8, device="cuda:0") for s in ("code_bytes", "scale_bytes"))
    places = [0, 1 << 25, (1 << 28) - 64, -(-n // 64) * 64 - 64]
    for at in places:
        for whole, part in zip(b, tail):
            whole[at // 64 * part.numel():at // 64 * part.numel() + part.numel()] = part
    c = torch.full((1, n), 7.0, dtype=torch.bfloat16, device="cuda:0")
    B.conef_mx_product(a, b, k, 1.0, 0.0, c, None, B.Model.stream_handle())
    want = torch.mm(A, W.t())
    far = product_error(torch, A, W, k, want, 1.0, None, True)
    for at in places:
        got = c[:, at:at + 64]
        assert bool(((got.double() - want[:, :got.shape[1]]).abs() <= far[:, :got.shape[1]]).all()), at
        got.zero_()
    assert not bool(c.any())


@pytest.mark.parametrize("m,n,k", [(2000, 1700, 300), (3500, 3600, 1537), (3500, 3600, 4200), (8200, 8190, 1537)])
def test_scales_of_nan_in_every_size_of_tile(env, m, n, k):  # noqa: F811
    """A row of A and one of B with a block that is NaN: that row and that column of C are, and nothing else is."""
    torch, B = env
    (a, A, at_a), (b, W, at_b) = operand(torch, m, k, 6), operand(torch, n, k, 7)
    i, j = m - 5, n // 2 + 1
    a[1][at_a(i, (k - 1) // 32)] = 255
    b[1][at_b(j, 2)] = 255
    c = torch.empty(m, n, device="cuda:0")
    B.conef_mx_product(a, b, k, 1.0, 0.0, c, None, B.Model.stream_handle())
    nan = torch.zeros(m, n, dtype=torch.bool, device="cuda:0")
    nan[i], nan[:, j] = True, True
    assert torch.equal(c.isnan(), nan)
    want = torch.mm(A, W.t())
    assert bool(((c.double() - want).abs() <= product_error(torch, A, W, k, want, 1.0, None, False))[~nan].all())


@pytest.mark.parametrize("bf16", [False, True])
def test_values_past_the_caches(env, bf16):  # noqa: F811
    torch, B = env
    rows, cols, pitch = 4100, 4221, 4224
    q, want, _ = operand(torch, rows, cols, 8)
    out = torch.full((rows, pitch), 77.0, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda:0")
    assert out.data_ptr() % 64 == 0 and rows * cols * out.element_size() > 32 << 20
    B.conef_mx_dequantise(q, out[:, :cols], B.Model.stream_handle())
    assert torch.equal(out[:, :cols].double(), want)
    assert bool((out[:, cols:] == 77.0).all())


@pytest.mark.parametrize("by_cols", [False, True])
def test_quantisation_of_the_longest_side(env, by_cols):  # noqa: F811
    """2^30 - 1 elements, one a row or all of them one row: 64 or 32 GiB of codes and back."""
    torch, B = env
    st, n = B.Model.stream_handle(), (1 << 30) - 1
    x = torch.zeros(n, 1, dtype=torch.bfloat16, device="cuda:0")
    x.normal_(generator=torch.Generator(device="cuda:0").manual_seed(12))
    q = B.mx_alloc(*((1, n) if by_cols else (n, 1)))
    B.conef_mx_quantise(x, B.MX_NEAREST, 0, 0, 0, None if by_cols else q, q if by_cols else None, st)
    out = torch.full((1, n) if by_cols else (n, 1), 7.0, device="cuda:0")
    B.conef_mx_dequantise(q, out, st)
    for first in (0, 1 << 27, (1 << 29) - 64, (1 << 30) - 192):
        part = x[first:first + 192].float().cpu().numpy()
        want = R.mx_decode(*R.mx_encode(part.T if by_cols else part))
        T.same_bits(out.view(-1)[first:first + 192].cpu().numpy(), want.reshape(-1))


# ---------------------------------------------------------------------------------------------- dropout
def test_dropout_of_all_the_octets_that_a_counter_counts(env):  # noqa: F811
    """2^32 - 2 of them, in place: 39 GB."""
    torch, B = env
    rows, cols, p, tail = (1 << 31) - 1, 9, 0.25, 40
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda:0")
    B.conef_dropout_backward(B.conef_drop(p=p, site=0, seed=SEED, step=STEP), x, x, B.Model.stream_handle())
    t = int(np.floor(p * 65536 + 0.5))
    for first in (0, (1 << 28) - tail // 2, rows - tail):
        u = np.array([[R.philox((2 * i + o, R.DROP, STEP & 0xFFFFFFFF, STEP >> 32), (SEED & 0xFFFFFFFF, SEED >> 32)) for o in (0, 1)]
                      for i in range(first, first + tail)], dtype=np.uint64)
        halves = np.stack([u & np.uint64(0xFFFF), u >> np.uint64(16)], -1).reshape(tail, 16)[:, :cols].astype(np.int64)
        T.same_bits(x[first:first + tail].float().cpu().numpy(), R.bf16(np.where(halves >= t, np.float32(65536.0 / (65536 - t)), np.float32(0))))


# ---------------------------------------------------------------------------------------------- norms
WIDE = [(1100, 9001), (1100, 12288), (1100, 12289), (1100, 16384), (1100, 16385)]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,cols", WIDE)
@pytest.mark.parametrize("skip,gap,p,residual", [(0, 0, None, False), (1, 3, 0.2, True)])
def test_wide_norms_of_many_rows(env, rows, cols, bf16, skip, gap, p, residual):  # noqa: F811
    """More rows than workgroups."""
    T.test_norm_forward(env, rows, cols, bf16, skip, gap, p, residual)
    T.test_norm_backward(env, rows, cols, bf16, skip, gap, p, residual)


PLACES = [(5, 7), (33, 1001), (700, 2049), (30, 5003), (300, 9001), (4, 20001)]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,cols", PLACES)
def test_forward_outputs_in_the_place_of_their_inputs(env, rows, cols, bf16):  # noqa: F811
    torch, B = env
    st = B.Model.stream_handle()
    g, x, gamma, beta = norm_inputs(rows, cols, bf16, 3)
    r = R.rounded(g.standard_normal((rows, cols)), bf16)
    d = B.conef_drop(p=0.2, site=4, seed=SEED, step=STEP)
    G, Bt = column_vector(torch, gamma), column_vector(torch, beta)

    def new(v=None):
        return Strided(torch, rows, cols, bf16, 1, 3, v)

    def norm(X, Rr, Z, Y):
        mean, rstd = torch.empty(rows, device="cuda:0"), torch.empty(rows, device="cuda:0")
        B.conef_norm_forward(d, 1e-5, X.t, Rr.t, G, Bt, Z.t, Y.t, mean, rstd, st)
        for m in (X, Rr, Z, Y):
            m.check_canary()
        return Z.t.clone(), Y.t.clone(), mean, rstd

    want = norm(new(x), new(r), new(), new())
    for z, y in (("r", None), ("x", None), ("r", "x"), ("x", "r"), (None, "x"), (None, "r")):
        X, Rr = new(x), new(r)
        place = {"x": X, "r": Rr}
        for got, exp in zip(norm(X, Rr, place.get(z) or new(), place.get(y) or new()), want):
            assert torch.equal(got, exp), (z, y)
    sums = R.dropped_sum(x, r, 0.2, SEED, 4, STEP, bf16)
    for over in ("x", "r"):
        X, Rr = new(x), new(r)
        out = X if over == "x" else Rr
        B.conef_dropout_forward(d, X.t, Rr.t, out.t, st)
        T.same_bits(out.numpy(), sums)
        out.check_canary()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,cols", PLACES)
def test_backward_outputs_in_the_place_of_their_inputs_and_alone(env, rows, cols, bf16):  # noqa: F811
    torch, B = env
    st = B.Model.stream_handle()
    g, z, gamma, beta = norm_inputs(rows, cols, bf16, 4)
    dy, dz_in = (R.rounded(g.standard_normal((rows, cols)), bf16) for _ in range(2))
    _, m64, s64, _ = R.norm(z, gamma, beta, 1e-5)
    d = B.conef_drop(p=0.2, site=4, seed=SEED, step=STEP)
    G, mean, rstd = (column_vector(torch, v) for v in (gamma, m64, s64))
    ws = torch.full((B.conef_norm_workspace(rows, cols),), 0xFF, dtype=torch.uint8, device="cuda:0")

    def run(dz=None, dx=None, columns=("dgamma", "dbeta")):
        """dz, dx: an input's name, whose buffer they take; the outputs"""
        M = {k: Strided(torch, rows, cols, bf16, 1, 3, v) for k, v in (("dy", dy), ("z", z), ("dz_in", dz_in), ("dz", None), ("dx", None))}
        c = {k: torch.full((cols,), 7.0, device="cuda:0") if k in columns else None for k in ("dgamma", "dbeta")}
        to = M[dz or "dz"], M[dx or "dx"]
        B.conef_norm_backward(d, M["dy"].t, M["z"].t, G, mean, rstd, M["dz_in"].t, to[0].t, to[1].t, c["dgamma"], c["dbeta"],
                              ws if columns else None, st)
        for m in M.values():
            m.check_canary()
        return {"dz": to[0].t, "dx": to[1].t, **c}

    want = run()
    for dz, dx in (("dz_in", None), ("z", None), (None, "dy"), (None, "z"), (None, "dz_in"), ("dz_in", "dy"), ("dy", "dz_in"), ("z", "dy")):
        got = run(dz, dx)
        for k in want:
            assert torch.equal(got[k], want[k]), (dz, dx, k)
    for columns in (("dgamma",), ("dbeta",), ()):
        got = run(columns=columns)
        for k in ("dz", "dx", *columns):
            assert torch.equal(got[k], want[k]), (columns, k)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("cols", [7, 33, 100, 250, 300, 700, 1001, 2001, 2049, 5003, 6145, 9001, 12290])
def test_gradients_of_constant_rows_far_from_zero(env, cols, bf16):  # noqa: F811
    """Rows of 2^110 at eps = 1e-12: (z - mean) rstd is 0 everywhere, and (0 - mean) rstd would be beyond fp32."""
    torch, B = env
    rows = 3
    g, _, gamma, _ = norm_inputs(rows, cols, bf16, 6)
    dy, z = R.rounded(g.standard_normal((rows, cols)), bf16), np.full((rows, cols), 2.0 ** 110, np.float32)
    mean, rstd = z[:, 0].copy(), np.full(rows, 1e6, np.float32)
    D = {k: Strided(torch, rows, cols, bf16, 1, 3, v) for k, v in (("dy", dy), ("z", z), ("dz", None))}
    dgamma, dbeta = torch.full((cols,), 7.0, device="cuda:0"), torch.full((cols,), 7.0, device="cuda:0")
    room = B.conef_norm_workspace(rows, cols)
    ws = torch.full((room,), 0xFF, dtype=torch.uint8, device="cuda:0")
    B.conef_norm_backward(None, D["dy"].t, D["z"].t, column_vector(torch, gamma), column_vector(torch, mean), column_vector(torch, rstd), None, D["dz"].t,
                          None, dgamma, dbeta, ws, B.Model.stream_handle())
    want, wg, wb, hat, a = R.norm_back(dy, z, gamma, mean, rstd)
    tz, tg, tb = T.back_tolerance(dy, hat, a, gamma, rstd, want, rows, cols, room // (8 * cols), bf16)
    assert (np.abs(D["dz"].numpy() - want) <= tz).all()
    assert (np.abs(dgamma.cpu().numpy() - wg) <= tg).all() and (np.abs(dbeta.cpu().numpy() - wb) <= tb).all()
    D["dz"].check_canary()


def test_sums_over_rows_of_more_than_2_27_columns(env):  # noqa: F811
    """Two rows, of which every column's sums are two products and one addition."""
    torch, B = env
    cols = (1 << 27) + 40
    g = torch.Generator(device="cuda:0").manual_seed(9)
    dy, z = (torch.randn(2, cols, device="cuda:0", generator=g).bfloat16() for _ in range(2))
    mean, rstd = torch.tensor([0.25, -0.5], device="cuda:0"), torch.tensor([2.0, 0.75], device="cuda:0")
    dgamma, dbeta = torch.full((cols,), 7.0, device="cuda:0"), torch.full((cols,), 7.0, device="cuda:0")
    ws = torch.empty(B.conef_norm_workspace(2, cols), dtype=torch.uint8, device="cuda:0")
    B.conef_norm_backward(None, dy, z, torch.ones(cols, device="cuda:0"), mean, rstd, None, None, None, dgamma, dbeta, ws, B.Model.stream_handle())
    term = dy.double() * ((z.double() - mean.double()[:, None]) * rstd.double()[:, None])
    assert bool(((dgamma - term.sum(0)).abs() <= 4 * U * term.abs().sum(0)).all())
    assert bool(((dbeta - dy.double().sum(0)).abs() <= U * dy.double().abs().sum(0)).all())


# ---------------------------------------------------------------------------------------------- refusals
def test_each_refusal_says_what_does_not_fit(env):  # noqa: F811
    """None of these reaches a kernel."""
    torch, B = env
    st = B.Model.stream_handle()
    z = lambda *s, **k: torch.zeros(*s, device="cuda:0", **k)                      # noqa: E731
    d, x, v, m = B.conef_drop(p=0.25, site=0, seed=1, step=0), z(4, 8), z(8), z(4)
    q, room = B.mx_alloc(4, 8), B.conef_norm_workspace(4, 8)
    first, like, floats = "a matrix of fp32 or bf16", "a matrix (4, 8) of fp32", "8 contiguous floats"
    for call, why in [
            (lambda: B.conef_dropout_backward(d, z(8, 4).t(), x, st), first), (lambda: B.conef_dropout_backward(d, z(4, 8).double(), x, st), first),
            (lambda: B.conef_dropout_backward(d, z(32), x, st), first), (lambda: B.conef_dropout_backward(d, z(4, 16)[:, ::2], x, st), first),
            (lambda: B.conef_dropout_forward(d, x, z(4, 9), x, st), like), (lambda: B.conef_dropout_forward(d, x, x.bfloat16(), x, st), like),
            (lambda: B.conef_dropout_forward(d, x, z(8, 4).t(), x, st), like), (lambda: B.conef_dropout_forward(d, x, [1], x, st), "a tensor"),
            (lambda: B.conef_dropout_forward(0.1, x, None, x, st), "a conef_drop"),
            *[(lambda g=g: B.conef_norm_forward(None, 1e-5, x, None, g, v, None, x, None, None, st), floats)
              for g in (z(7), z(16)[::2], v.bfloat16(), z(1, 8))],
            (lambda: B.conef_norm_backward(None, x, x, v, m, z(5), None, x, None, None, None, None, st), "4 contiguous floats"),
            (lambda: B.conef_norm_backward(None, x, x, v, m, m, None, x, None, None, v, z(1), st), f"buffer of {room} bytes"),
            (lambda: B.conef_mx_quantise(z(4, 129), B.MX_NEAREST, 0, 0, 0, q, None, st), "buffer of 8192 bytes"),
            (lambda: B.conef_mx_quantise(z(4, 129), B.MX_NEAREST, 0, 0, 0, (B.mx_alloc(4, 129)[0], q[1]), None, st), "buffer of 512 bytes"),
            (lambda: B.conef_mx_quantise(x, B.MX_NEAREST, 0, 0, 0, q[0], None, st), "a pair"),
            (lambda: B.conef_mx_quantise(x, B.MX_NEAREST, 0, 1 << 32, 0, q, None, st), "a site"),
            (lambda: B.conef_mx_dequantise(q, z(65, 8), st), "buffer of 8192 bytes"),
            (lambda: B.conef_mx_product(q, q, 129, 1.0, 0.0, z(4, 4), None, st), "buffer of 8192 bytes"),
            (lambda: B.conef_mx_product(q, q, 8, 1.0, 0.0, z(4, 65), None, st), "buffer of 8192 bytes")]:
        with pytest.raises(B.ConefError) as e:
            call()
        assert e.value.code == B.EINVAL and why in str(e.value), (why, str(e.value))


@pytest.mark.parametrize("rounding", [2, -1, 1 << 32, (1 << 32) + 1, -(1 << 32)])
def test_a_rounding_that_is_none_is_refused(env, rounding):  # noqa: F811
    torch, B = env
    q = B.mx_alloc(4, 8)
    with pytest.raises(B.ConefError) as e:
        B.conef_mx_quantise(torch.zeros(4, 8, device="cuda:0"), rounding, 0, 0, 0, q, None, B.Model.stream_handle())
    assert e.value.code == B.EINVAL


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("cols", [5, 7, 15, 49, 63, 126, 255, 510, 784, 1020, 2041, 4095, 8190, 12286, 16381, 25088, 25998])
def test_constant_rows_have_their_value_as_their_mean(env, cols, bf16):  # noqa: F811
    """Sums of these values are exact in fp32 in any order (cols 125 < 2^24), so the mean is too, and the norm is beta."""
    torch, B = env
    v = torch.tensor([1000.0, -2000.0, 16000.0, 1.0], device="cuda:0")
    x = v[:, None].expand(4, cols).contiguous().to(torch.bfloat16 if bf16 else torch.float32)
    v = x[:, 0].float()
    gamma, beta = (column_vector(torch, t) for t in norm_inputs(1, cols, False, 7)[2:])
    y, z, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty_like(v), torch.empty_like(v)
    for fused in (False, True):
        B.conef_norm_forward(None, 1e-5, x, torch.zeros_like(x) if fused else None, gamma, beta, z if fused else None, y, mean, rstd, B.Model.stream_handle())
        assert torch.equal(mean, v)
        assert torch.equal(y, beta.to(x.dtype)[None, :].expand(4, cols))
        assert bool(((rstd.double() - 1e-5 ** -0.5).abs() <= 4 * U * rstd).all())
